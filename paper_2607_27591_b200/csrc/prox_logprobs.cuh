// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits (prox_token_logprobs).
//
//   z = x / temperature,  lse = log sum_v exp(z_v),  log p(v) = z_v - lse,  H = -sum_v p_v log p_v = log s - w / s
//   with m = max z,  s = sum exp(z - m),  w = sum (z - m) exp(z - m)
//
// One pass over the logits: a thread keeps its own m, s and w and rescales the two when its maximum rises.  2048 rows of 131072
// bf16 logits take 97 us in a graph (5.5 TB/s; 110 us as calls of their own, 4.9 TB/s); one row 4.5 us, with 20 top alternatives
// 10 us, all of it latency (two barriers of the cluster and three of lists).  Bound by HBM; next
// comes the special-function unit (one exponential a logit: 16 a cycle and SM, three quarters of its rate while HBM delivers
// 16-bit logits).  A row goes to one block, or to a cluster of up to 8 where there are fewer rows than the GPU has
// room for; its blocks' sums and lists meet in shared memory of the first block, in their order.
//
// Top alternatives.  Order: by value, then the lower index; as one 64-bit key, value bits made monotonic above, inverted
// index below.  A block takes rounds of 4 vectors a thread.  The vectors' maxima are known from the softmax; in the first round
// the k-th largest of the maxima of 64 groups of threads is a floor that k logits reach, so only vectors that reach it are noted,
// by their number.  Noted vectors are looked at all together (process): their logits above the floor go to a list, and behind the
// first round, and whenever the list fills up, the k-th largest in it is the new floor (settle).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace prox {
namespace lp {

enum { kBf16 = 0, kFp32 = 1, kFp16 = 2 };

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxTop = 32;
constexpr int kVectors = 4;              // 16-byte vectors of a thread and round
constexpr int kList = 2 * kThreads;      // candidates of a block
constexpr int kItems = 2 * kVectors * kThreads;   // vectors noted
constexpr int kMaxCluster = 8;

struct Args {
  const uint8_t* x;
  long long row_bytes;     // from one row to the next
  int V;
  float inv_temperature;
  const int* given;        // [T][n_given]
  int n_given;
  float* logprob;          // [T][n_given]
  float* entropy;          // [T] or null
  int k;
  float* top_logprob;      // [T][k]
  int* top_index;          // [T][k]
  int S;                   // blocks of a row
};

template <int DT> struct Type { using T = uint16_t; static constexpr int kSize = 2, kPer = 8; };
template <> struct Type<kFp32> { using T = float; static constexpr int kSize = 4, kPer = 4; };

template <int DT>
__device__ __forceinline__ float widen(typename Type<DT>::T v) {
  if constexpr (DT == kFp32) return v;
  else if constexpr (DT == kBf16) return __uint_as_float((uint32_t)v << 16);
  else return __half2float(__ushort_as_half(v));
}

template <int DT>
__device__ __forceinline__ void widen(float (&f)[Type<DT>::kPer], const uint4& v) {
  const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (DT == kFp32) {
      f[j] = __uint_as_float(e[j]);
    } else if constexpr (DT == kBf16) {
      f[2 * j] = __uint_as_float(e[j] << 16);
      f[2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
    } else {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&e[j]));
      f[2 * j] = p.x;
      f[2 * j + 1] = p.y;
    }
  }
}

// Larger key: larger value, then lower index.  What is no number comes first, -0 and 0 are one value.
__device__ __forceinline__ unsigned long long key_of(float v, int index) {
  uint32_t u = __float_as_uint(v + 0.0f);
  u = (u & 0x7fffffffu) > 0x7f800000u ? 0xffffffffu : u & 0x80000000u ? ~u : u | 0x80000000u;
  return (unsigned long long)u << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(unsigned long long key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)~(uint32_t)key; }
// The largest key below all of value v (which is a number).
__device__ __forceinline__ unsigned long long key_below(float v) { return (key_of(v, 0) & ~0xffffffffull) - 1; }

// Running softmax sums: m in logits, d = (x - m) log2 e / temperature, s = sum 2^d, w = sum d 2^d.
struct Sums { float m, s, w; };

__device__ __forceinline__ float exp2_fast(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// 2^-256 is 0: what lies that far below, or is -inf, counts as nothing (and is kept from making 0 * infinity in w).
// fmaxf drops what is no number; the maximum keeps it, in a round and from round to round (max_nan), and a maximum that is no
// number or infinite makes results that are no numbers.
__device__ __forceinline__ float clamp_low(float d) { return fmaxf(d, -256.f); }
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void raise(Sums& a, float m, float c) {
  const float d = clamp_low((a.m - m) * c), f = exp2_fast(d);
  a.w = fmaf(d, a.s, a.w) * f;
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  const float m = max_nan(a.m, b.m);
  raise(a, m, c);
  raise(b, m, c);
  return {m, a.s + b.s, a.w + b.w};
}

// Two fp32 numbers at a time: half the issue slots
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(float& a, float& b, uint64_t v) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

__device__ __forceinline__ uint32_t cluster_address(const void* p, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_barrier() { asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory"); }

// What a block keeps for the top alternatives.
template <bool TOP>
struct Top {
  unsigned long long list[TOP ? kList : 1], tops[TOP ? kThreads : 1], best[TOP ? kMaxTop : 1];
  unsigned long long floor_key;          // only keys above it count
  int items[TOP ? kItems : 1], n_items, count;
};

// The k largest of the list's first n keys, in order, to its front; raises the floor.  All threads; n <= kList.  (Not inlined, as
// process: what is rare is kept from the registers of the loop around it.)
__device__ __noinline__ void settle(Top<true>& s, int n, int k) {
  const int tid = threadIdx.x, parts = n <= kThreads / 4 ? 4 : n <= kThreads / 2 ? 2 : 1;
  for (int i0 = 0; i0 < n; i0 += kThreads / parts) {
    const int i = i0 + tid / parts;
    const unsigned long long mine = i < n ? s.list[i] : ~0ull;
    int above = 0;
#pragma unroll 8
    for (int j = tid % parts; j < n; j += parts) above += s.list[j] > mine;
    if (parts > 1) above += __shfl_xor_sync(0xffffffffu, above, 1);
    if (parts > 2) above += __shfl_xor_sync(0xffffffffu, above, 2);
    if (i < n && tid % parts == 0 && above < k) s.best[above] = mine;
  }
  __syncthreads();
  if (tid < min(n, k)) s.list[tid] = s.best[tid];
  if (tid == 0) {
    s.count = min(n, k);
    if (n >= k) s.floor_key = max(s.floor_key, s.best[k - 1]);
  }
  __syncthreads();
}

// Looks at the n noted vectors of a row.  All threads, behind a barrier; leaves none.
template <int DT>
__device__ __noinline__ void process(Top<true>& s, int n, int k, const uint8_t* start, int head, int V) {
  using T = typename Type<DT>::T;
  constexpr int kPer = Type<DT>::kPer;
  const int tid = threadIdx.x;
  auto key_at = [&](int item, int e) -> unsigned long long {   // of a noted vector's logit e; 0 if it is none
    const int index = s.items[item] * kPer + e - head;
    if (index < 0 || index >= V) return 0;
    return key_of(widen<DT>(reinterpret_cast<const T*>(start)[index]), index);
  };
  if (n > kThreads / 2) {
    // so many (rising or equal logits): the k-th largest of the threads' largest keys is a floor too
    unsigned long long most = 0;
#pragma unroll 1
    for (int i = tid; i < n; i += kThreads)
      for (int e = 0; e < kPer; ++e) most = max(most, key_at(i, e));
    s.tops[tid] = most;
    if (tid == 0) s.best[0] = 0;
    __syncthreads();
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < kThreads; ++j) above += s.tops[j] > most;
    if (above == k - 1 && most) s.best[0] = most;              // (keys differ; threads without a logit have 0)
    __syncthreads();
    if (tid == 0 && s.best[0]) s.floor_key = max(s.floor_key, s.best[0] - 1);
    __syncthreads();
  }
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += kThreads / kPer) {
    const int i = i0 + tid / kPer;
    int end = 0;
    if (i < n) {
      const unsigned long long key = key_at(i, tid % kPer);
      if (key > s.floor_key) {
        end = atomicAdd(&s.count, 1) + 1;
        s.list[end - 1] = key;
      }
    }
    if (__syncthreads_or(end > kList / 2)) settle(s, s.count, k);   // (at most kThreads more)
  }
  if (tid == 0) s.n_items = 0;
  __syncthreads();
}

template <int DT, bool TOP>
__global__ void __launch_bounds__(kThreads, 2) logprobs_kernel(const Args a) {
  using T = typename Type<DT>::T;
  constexpr int kPer = Type<DT>::kPer, kSize = Type<DT>::kSize;
  __shared__ Sums warp_sums[kWarps];
  __shared__ Sums block_sums;
  __shared__ Top<TOP> top;
  __shared__ float group_max[64];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int S = a.S, rank = blockIdx.x % S;
  const long long row = blockIdx.x / S;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // the row as 16-byte vectors: the first and last may lie partly outside; element e of vector q is logit q kPer + e - head
  const uint8_t* start = a.x + row * a.row_bytes;
  const int head = (int)(reinterpret_cast<uintptr_t>(start) & 15) / kSize;
  const uint8_t* base = start - head * kSize;
  const int nv = (head + a.V + kPer - 1) / kPer;
  const int q0 = (int)((long long)nv * rank / S), q1 = (int)((long long)nv * (rank + 1) / S);
  const float c = 1.4426950408889634f * a.inv_temperature;

  auto load = [&](int q) -> uint4 {
    if (q >= q1) q = -1;
    const int first = q * kPer - head;
    if (q >= 0 && first >= 0 && first + kPer <= a.V) {
      uint4 v;
      asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(base + (size_t)q * 16));
      return v;
    }
    // an end of the row, or behind the block's share: -inf where there is no logit
    alignas(16) T e[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const bool in = q >= 0 && first + j >= 0 && first + j < a.V;
      if constexpr (DT == kFp32) e[j] = in ? reinterpret_cast<const float*>(start)[first + j] : __uint_as_float(0xff800000u);
      else e[j] = in ? reinterpret_cast<const uint16_t*>(start)[first + j] : (uint16_t)(DT == kBf16 ? 0xff80 : 0xfc00);
    }
    return *reinterpret_cast<const uint4*>(e);
  };

  if (TOP) {
    if (tid == 0) { top.count = 0; top.n_items = 0; top.floor_key = 0; }
  }
  Sums sum = {-3.402823466e38f, 0.f, 0.f};
  uint4 now[kVectors], next[kVectors];
#pragma unroll
  for (int j = 0; j < kVectors; ++j) now[j] = load(q0 + tid + j * kThreads);

  const int whole0 = max(q0, head ? 1 : 0), whole1 = min(q1, (head + a.V) / kPer);   // vectors that lie inside the row
  const uint8_t* ahead = base + ((size_t)q0 + tid + kVectors * kThreads) * 16;       // the next round's

  // the given tokens' logits, on their way behind the first round's (the first kThreads of them)
  float given_logit = 0.f;
  int given = -1;
  if (rank == 0 && tid < a.n_given) {
    given = a.given[row * a.n_given + tid];
    if (given >= 0 && given < a.V) given_logit = widen<DT>(reinterpret_cast<const T*>(start)[given]);
  }

  bool first_round = true;
  for (int qr = q0; qr < q1; qr += kVectors * kThreads) {
    const int q = qr + tid;
    const bool more = qr + kVectors * kThreads < q1;
    if (qr + kVectors * kThreads >= whole0 && qr + 2 * kVectors * kThreads <= whole1) {
#pragma unroll
      for (int j = 0; j < kVectors; ++j)
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(next[j].x), "=r"(next[j].y), "=r"(next[j].z), "=r"(next[j].w) : "l"(ahead + j * (kThreads * 16)));
    } else if (more) {
#pragma unroll
      for (int j = 0; j < kVectors; ++j) next[j] = load(q + (kVectors + j) * kThreads);
    }
    ahead += kVectors * kThreads * 16;
    float vector_max[kVectors];
#pragma unroll
    for (int j = 0; j < kVectors; ++j) {
      float x[kPer];
      widen<DT>(x, now[j]);
      vector_max[j] = x[0];
#pragma unroll
      for (int e = 1; e < kPer; ++e) vector_max[j] = max_nan(vector_max[j], x[e]);
    }
    float most = vector_max[0];
#pragma unroll
    for (int j = 1; j < kVectors; ++j) most = max_nan(most, vector_max[j]);
    if (!(most <= sum.m)) raise(sum, max_nan(sum.m, most), c);   // (a maximum that is no number stays one)
    {
      uint64_t s2 = pair(0.f, 0.f), w2 = s2;
      const uint64_t minus_m = pair(-sum.m, -sum.m), c2 = pair(c, c);
#pragma unroll
      for (int j = 0; j < kVectors; ++j) {
        float x[kPer];
        widen<DT>(x, now[j]);
#pragma unroll
        for (int e = 0; e < kPer; e += 2) {
          float d0, d1;
          unpair(d0, d1, mul2(add2(pair(x[e], x[e + 1]), minus_m), c2));
          d0 = clamp_low(d0);
          d1 = clamp_low(d1);
          const uint64_t p = pair(exp2_fast(d0), exp2_fast(d1));
          s2 = add2(s2, p);
          w2 = fma2(pair(d0, d1), p, w2);
        }
      }
      float s0, s1, w0, w1;
      unpair(s0, s1, s2);
      unpair(w0, w1, w2);
      sum.s += s0 + s1;
      sum.w += w0 + w1;
    }
    if constexpr (TOP) {
      const bool start_floor = first_round;
      if (first_round) {
        // a floor that at least k logits reach: the k-th largest of the maxima of 64 groups of eight threads
        first_round = false;
        float gm = most;
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, o));
        if ((tid & 7) == 0) group_max[tid >> 3] = gm;
        __syncthreads();
        const float mine = group_max[tid >> 3];
        int above = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int o = (tid & 7) * 8 + j;
          const float v = group_max[o];
          above += v > mine || (v == mine && o < tid >> 3);
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
        if ((tid & 7) == 0 && above == a.k - 1 && mine == mine) top.floor_key = key_below(mine);
        __syncthreads();
      }
      const float floor_v = value_of(top.floor_key + 1);           // (of a key below all of a value: that value; 0: the lowest)
      int end = 0;
      if (!(most < floor_v)) {
#pragma unroll
        for (int j = 0; j < kVectors; ++j)
          if (!(vector_max[j] < floor_v) && q + j * kThreads < q1) {
            end = atomicAdd(&top.n_items, 1) + 1;
            top.items[end - 1] = q + j * kThreads;
          }
      }
      if (__syncthreads_or(end > kItems / 2) || (start_floor && more)) {
        process<DT>(top, top.n_items, a.k, start, head, a.V);
        if (start_floor) settle(top, top.count, a.k);                        // the k-th largest of the first round: later ones bring few above it
      }
    }
#pragma unroll
    for (int j = 0; j < kVectors; ++j) now[j] = next[j];
  }

  // the block's sums: lanes, warps
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Sums other = {__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.s, o), __shfl_xor_sync(0xffffffffu, sum.w, o)};
    sum = lane & o ? join(other, sum, c) : join(sum, other, c);
  }
  if (lane == 0) warp_sums[warp] = sum;
  __syncthreads();
  if constexpr (TOP) {
    process<DT>(top, top.n_items, a.k, start, head, a.V);
    settle(top, top.count, a.k);
  }
  // of as many sums as there are (a power of two), one a lane of the first warp: joined in pairs
  auto join_lanes = [&](Sums v, int n) {
    for (int o = 1; o < n; o <<= 1) {
      const Sums other = {__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o), __shfl_xor_sync(0xffffffffu, v.w, o)};
      v = lane & o ? join(other, v, c) : join(v, other, c);
    }
    return v;
  };
  if (warp == 0) {
    const Sums v = join_lanes(warp_sums[lane % kWarps], kWarps);
    if (lane == 0) block_sums = v;
  }
  if (S > 1) {
    cluster_barrier();
    if (rank == 0) {
      if (warp == 0) {
        const uint32_t at = cluster_address(&block_sums, lane % S);
        Sums v;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v.m) : "r"(at) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v.s) : "r"(at + 4) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v.w) : "r"(at + 8) : "memory");
        v = join_lanes(v, S);
        if (lane == 0) warp_sums[0] = v;
      }
      if constexpr (TOP) {
        for (int i = tid; i < (S - 1) * a.k; i += kThreads) {  // (a block may have had fewer logits than k)
          const int r = i / a.k + 1, j = i - (r - 1) * a.k;
          int n;
          unsigned long long key;
          asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(n) : "r"(cluster_address(&top.count, r)) : "memory");
          asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(key) : "r"(cluster_address(&top.list[j], r)) : "memory");
          top.list[kMaxTop + i] = j < n ? key : 0;
        }
      }
    }
    cluster_barrier();                                         // nobody leaves while its memory is read
    if (rank != 0) return;
    if constexpr (TOP) {
      if (tid >= top.count && tid < kMaxTop) top.list[tid] = 0;   // (it has k at most)
      __syncthreads();
      settle(top, kMaxTop + (S - 1) * a.k, a.k);
    }
    if (tid == 0) block_sums = warp_sums[0];
  }
  __syncthreads();
  const Sums all = block_sums;
  const float log_s = logf(all.s);                             // (s >= 1 unless there is no logit above -inf: then -inf)
  auto log_p = [&](float x) {
    if (all.s == 0.f && all.m == -3.402823466e38f) return __uint_as_float(0xff800000u);
    return (x - all.m) * a.inv_temperature - log_s;
  };
  if (tid == 0 && a.entropy)
    a.entropy[row] = all.s == 0.f && all.m == -3.402823466e38f ? 0.f : log_s - 0.6931471805599453f * (all.w / all.s);
  for (int i = tid; i < a.n_given; i += kThreads) {
    if (i >= kThreads) {
      given = a.given[row * a.n_given + i];
      if (given >= 0 && given < a.V) given_logit = widen<DT>(reinterpret_cast<const T*>(start)[given]);
    }
    a.logprob[row * a.n_given + i] = given < 0 ? 0.f : given >= a.V ? __uint_as_float(0x7fffffffu) : log_p(given_logit);
  }
  if (TOP && tid < a.k) {
    a.top_logprob[row * a.k + tid] = log_p(value_of(top.list[tid]));
    a.top_index[row * a.k + tid] = index_of(top.list[tid]);
  }
}

}  // namespace lp
}  // namespace prox
