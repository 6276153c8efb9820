// Weights held in 4 bits: projections of a few tokens (prox_w4_linear) and Stage 2 of the sparse FFN over such
// weights (prox_w4_stage2_ffn; Sec. 4.1 Stage 2, with the low-bit weights that the paper leaves to future work).
//
//   w[n, k] = s[n, k / G] (q[n, k] - z[n, k / G])          q 4 bits, s fp16, z an integer (8 where there are none)
//   y[b, n] = sum_groups s[n, G] ( sum_{k in group} (q[n, k] - z) x[b, k] )
//
// The inner sum runs on warp-level tensor-core tiles (mma.sync m16n8k16, fp32 accumulation): q - z is a small integer
// and exact in bf16 and fp16, so is every product, and the scale enters in fp32 once per group.  All kernels are bound by
// the weight stream; codes are read where the caller has them, once, and never written back in a wider form: unpacked in
// registers, 64 codes of a lane cost about 100 issue slots against the 177 that the SM has while HBM delivers them.  For
// tcgen05 the 16-bit form would have to go through shared memory, four times the bytes that come in, at the rate of
// HBM more than its bandwidth leaves.
//
// Fragment layout of mma.sync.m16n8k16 (g = lane / 4, t = lane % 4):
//   A: a0 = (row g, k 2t..2t+1)  a1 = (row g + 8, same k)  a2 = (row g, k 2t+8..+9)  a3 = (row g + 8, k 2t+8..+9)
//   B: b0 = (k 2t..2t+1, col g)  b1 = (k 2t+8..+9, col g)    C: c0c1 = (row g, col 2t..2t+1)  c2c3 = (row g + 8, same)
// A sum over k does not care which k sits at which place as long as A and B agree.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace prox {
namespace w4 {

enum { kBf16 = 0, kFp32 = 1, kFp16 = 2 };

struct Mat {
  const uint8_t* codes;   // [rows][cols / 2]
  const __half* scales;   // [rows][groups]
  const uint8_t* zeros;   // [rows][groups] or null
};

__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
  uint2 v;
  asm volatile("ld.global.nc.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// XT: type of the tokens (kBf16 or kFp16)
template <int XT>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (XT == kBf16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A code in the low mantissa bits of 2^7 (bf16) or 2^10 (fp16) is that power plus the code; the same with the zero point
// is subtracted, which is exact.
template <int XT> __device__ __forceinline__ constexpr uint32_t magic() { return XT == kBf16 ? 0x43004300u : 0x64006400u; }

template <int XT>
__device__ __forceinline__ uint32_t minus_zero(uint32_t code_pair, uint32_t zero_pair) {
  uint32_t r;
  if (XT == kBf16) asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(code_pair), "r"(zero_pair));
  else asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(code_pair), "r"(zero_pair));
  return r;
}

// Word w: codes of eight columns.  v[e] = columns (e, e + 4).
template <int XT>
__device__ __forceinline__ void unpack(uint32_t (&v)[4], uint32_t w, uint32_t zero_pair) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = minus_zero<XT>(((w >> (4 * e)) & 0x000f000fu) | magic<XT>(), zero_pair);
}

__device__ __forceinline__ void store(void* y, size_t i, float v, int type) {
  if (type == kFp32) static_cast<float*>(y)[i] = v;
  else if (type == kBf16) static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(y)[i] = __float2half_rn(v);
}

__device__ __forceinline__ float cluster_read(const float* p, int rank) {   // a float of another block of the cluster, at the address that it has here
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(r) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// ----------------------------------------------------------------------------
// Rows times tokens: y = x W^T for all rows of a matrix, or gate and up of listed channels with SwiGLU behind them.
//
// A warp owns tiles of 16 rows (linear) or of 8 channels (rows 0-7 of the tile are gate rows, rows 8-15 the up rows of
// the same channels, so that both pre-activations of a channel end in one place) and a run of 128-column chunks; a
// lane reads 16 bytes of its two rows per chunk.  A block has WM tiles side by side and WK warps along the columns of
// each; a cluster of S blocks splits the columns further where the rows alone do not fill the GPU or the tokens do not fit
// in shared memory.  Partial sums meet in shared memory, of the cluster where it has more than one block, in a fixed
// order: results do not depend on timing.
// ----------------------------------------------------------------------------
constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kRing = 4;                 // chunks of a warp in flight: 512 threads x 4 x 32 bytes = 64 KB per SM

struct RowsArgs {
  Mat w, w2;               // linear: w.  gate and up: w and w2
  int rows, K, groups, gstep;   // gstep 0: one scale per row
  const uint16_t* x;
  long long x_stride;
  int B;
  void* y;                 // linear
  long long y_stride;
  int y_type;
  const int* list;         // gate and up: the channels ...
  const int* count;        // ... how many (null: n)
  int n;
  const uint8_t* members;  // bit b: token b keeps the channel (null: one token)
  float* h;                // [B][h_stride]
  int h_stride;
  int S, WM, WK, R;        // R: units whose partial sums a block keeps before the cluster adds them up
  int x_vec;               // x rows start on 16-byte boundaries
};

template <int W, bool ZP>
struct Chunk {             // what a lane holds of one chunk: two rows, 32 codes each, 4 / W groups
  uint32_t q[2][4];
  __half s[2][4 / W];
  uint8_t z[2][ZP ? 4 / W : 1];
};

template <int XT, int W, int NT, bool ZP, bool GATEUP>
__global__ void __launch_bounds__(kRowThreads, 1) rows_kernel(const RowsArgs a) {
  extern __shared__ __align__(16) uint8_t rows_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int S = a.S, WM = a.WM, WK = a.WK;
  const int rank = blockIdx.x % S, cid = blockIdx.x / S, ncl = gridDim.x / S;
  const int C = (a.K + 127) / 128, Cs = (C + S - 1) / S;
  const int cb0 = min(C, rank * Cs), cb1 = min(C, cb0 + Cs);
  constexpr int kTile = NT * 128;                              // floats of a warp's partial tile: [NT][16 rows][8 tokens]
  uint4* xs = reinterpret_cast<uint4*>(rows_smem);             // [chunk][word of a lane][token][t]
  float* red = reinterpret_cast<float*>(rows_smem + (size_t)Cs * 256 * a.B);   // [2][warps][kTile]
  float* part = red + 2 * kRowWarps * kTile;                   // [R][WM * 16][B] (S > 1)
  dep_wait();
  dep_launch();
  int n = a.rows;
  if (GATEUP) {
    n = a.n;
    if (a.count) n = max(0, min(n, *a.count));
  }
  constexpr int kPer = GATEUP ? 8 : 16;                        // list entries of a tile
  const int U = (n + kPer * WM - 1) / (kPer * WM);
  if (cid >= U) return;                                        // the whole cluster
  const int nu = (U - cid - 1) / ncl + 1;

  // the tokens, in the order in which lanes take them: the 8 inputs of a code word as (k, k + 4) pairs
  const int octets = (cb1 - cb0) * 16;
  for (int i = tid; i < octets * a.B; i += kRowThreads) {
    const int b = i / octets, o = i - b * octets;
    const int k = cb0 * 128 + o * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k < a.K) {
      const uint16_t* p = a.x + (size_t)b * a.x_stride + k;
      if (a.x_vec) v = __ldg(reinterpret_cast<const uint4*>(p));
      else {
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = __ldg(p + j);
        v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
      }
    }
    const int c = o >> 4, oc = o & 15;
    const int ot = W == 4 ? oc >> 2 : W == 2 ? (oc & 7) >> 1 : oc & 3;
    const int oi = W == 4 ? oc & 3 : W == 2 ? (oc >> 3) * 2 + (oc & 1) : oc >> 2;
    xs[((c * 4 + oi) * a.B + b) * 4 + ot] = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632),
                                                       __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
  }
  __syncthreads();

  const int wm = warp / WK, wk = warp - wm * WK;
  const int cw = (Cs + WK - 1) / WK;                           // chunks of a warp and unit (the last warps may have fewer)
  const int c0 = cb0 + wk * cw, c1 = wm < WM ? min(cb1, c0 + cw) : c0;
  const int total = nu * cw;

  // loading side: unit lu (of this cluster's units), chunk lc of it
  int lu = 0, lc = 0;
  const uint8_t *q0 = nullptr, *q1 = nullptr;
  size_t r0 = 0, r1 = 0;
  int id_next = 0;
  auto entry = [&](int u) { return ((cid + u * ncl) * WM + wm) * kPer + g; };   // list entry of this lane's first row
  auto fetch_id = [&](int u) {                                 // a channel id is read one unit ahead of its rows
    if (GATEUP && wm < WM) {
      const int id = a.list[min(entry(u), n - 1)];
      id_next = (unsigned)id < (unsigned)a.rows ? id : 0;
    }
  };
  auto open_unit = [&]() {
    if (GATEUP) {
      r0 = r1 = (size_t)id_next;
      q0 = a.w.codes + r0 * (a.K / 2);
      q1 = a.w2.codes + r0 * (a.K / 2);
      if (lu + 1 < nu) fetch_id(lu + 1);
    } else {
      r0 = (size_t)min(entry(lu), a.rows - 1);
      r1 = (size_t)min(entry(lu) + 8, a.rows - 1);
      q0 = a.w.codes + r0 * (a.K / 2);
      q1 = a.w.codes + r1 * (a.K / 2);
    }
  };
  auto load = [&](Chunk<W, ZP>& b) {
    const int c = c0 + lc;
    if (c < c1) {
      const Mat& m1 = GATEUP ? a.w2 : a.w;
#pragma unroll
      for (int j = 0; j < 4 / W; ++j) {
        const int k = c * 128 + j * (32 * W) + t * (8 * W);
        const bool in = k < a.K;
        if (W == 4) {
          const uint4 v0 = in ? ld16(q0 + k / 2) : make_uint4(0, 0, 0, 0), v1 = in ? ld16(q1 + k / 2) : make_uint4(0, 0, 0, 0);
          b.q[0][0] = v0.x; b.q[0][1] = v0.y; b.q[0][2] = v0.z; b.q[0][3] = v0.w;
          b.q[1][0] = v1.x; b.q[1][1] = v1.y; b.q[1][2] = v1.z; b.q[1][3] = v1.w;
        } else if (W == 2) {
          const uint2 v0 = in ? ld8(q0 + k / 2) : make_uint2(0, 0), v1 = in ? ld8(q1 + k / 2) : make_uint2(0, 0);
          b.q[0][2 * j] = v0.x; b.q[0][2 * j + 1] = v0.y;
          b.q[1][2 * j] = v1.x; b.q[1][2 * j + 1] = v1.y;
        } else {
          b.q[0][j] = in ? __ldg(reinterpret_cast<const uint32_t*>(q0 + k / 2)) : 0u;
          b.q[1][j] = in ? __ldg(reinterpret_cast<const uint32_t*>(q1 + k / 2)) : 0u;
        }
        const int gi = min((c * (4 / W) + j) * a.gstep, a.groups - 1);
        b.s[0][j] = a.w.scales[r0 * a.groups + gi];
        b.s[1][j] = m1.scales[r1 * a.groups + gi];
        if (ZP) {
          b.z[0][j] = a.w.zeros[r0 * a.groups + gi];
          b.z[1][j] = m1.zeros[r1 * a.groups + gi];
        }
      }
    }
    if (++lc == cw) {
      lc = 0;
      if (++lu < nu) open_unit();
    }
  };

  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  auto compute = [&](const Chunk<W, ZP>& b, int cc) {
    const int c = c0 + cc;
    if (c >= c1) return;
    const uint4* xc = xs + (size_t)(c - cb0) * 16 * a.B + t;
#pragma unroll
    for (int j = 0; j < 4 / W; ++j) {
      float d[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i) d[i][0] = d[i][1] = d[i][2] = d[i][3] = 0.f;
      uint32_t z0 = magic<XT>() | 0x00080008u, z1 = z0;
      if (ZP) {
        z0 = magic<XT>() | b.z[0][j] * 0x00010001u;
        z1 = magic<XT>() | b.z[1][j] * 0x00010001u;
      }
#pragma unroll
      for (int i = j * W; i < (j + 1) * W; ++i) {
        uint32_t v0[4], v1[4];
        unpack<XT>(v0, b.q[0][i], z0);
        unpack<XT>(v1, b.q[1][i], z1);
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          const uint4 xv = xc[(i * a.B + min(m * 8 + g, a.B - 1)) * 4];   // columns behind the last token: computed, never used
          mma<XT>(d[m], v0[0], v1[0], v0[1], v1[1], xv.x, xv.y);
          mma<XT>(d[m], v0[2], v1[2], v0[3], v1[3], xv.z, xv.w);
        }
      }
      const float s0 = __half2float(b.s[0][j]), s1 = __half2float(b.s[1][j]);
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        acc[m][0] = fmaf(s0, d[m][0], acc[m][0]);
        acc[m][1] = fmaf(s0, d[m][1], acc[m][1]);
        acc[m][2] = fmaf(s1, d[m][2], acc[m][2]);
        acc[m][3] = fmaf(s1, d[m][3], acc[m][3]);
      }
    }
  };
  // one output of unit u: row r of its WM * 16 tile rows (linear), or channel r of its WM * 8 (gate and up)
  auto emit = [&](int u, int r, int b, float v, float up) {
    const int pos = (cid + u * ncl) * WM * kPer + r;
    if (pos >= n) return;
    if (!GATEUP) {
      store(a.y, (size_t)b * a.y_stride + pos, v, a.y_type);
    } else {
      const int id = a.list[pos];
      const bool kept = (unsigned)id < (unsigned)a.rows && (!a.members || (a.members[pos] >> b & 1));
      a.h[(size_t)b * a.h_stride + pos] = kept ? up * (v / (1.0f + expf(-v))) : 0.f;
    }
  };
  const int outs = WM * kPer * a.B;
  auto finish_unit = [&](int u) {
    float* rd = red + (u & 1) * (kRowWarps * kTile);
    if (wm < WM) {
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        float* mine = rd + warp * kTile + m * 128 + g * 8 + 2 * t;
        *reinterpret_cast<float2*>(mine) = make_float2(acc[m][0], acc[m][1]);
        *reinterpret_cast<float2*>(mine + 64) = make_float2(acc[m][2], acc[m][3]);
        acc[m][0] = acc[m][1] = acc[m][2] = acc[m][3] = 0.f;
      }
    }
    __syncthreads();                                           // (two buffers: the next unit's sums do not meet the reads below)
    if (S == 1) {
      for (int i = tid; i < outs; i += kRowThreads) {
        const int b = i / (WM * kPer), r = i - b * (WM * kPer);
        const float* p = rd + (r / kPer) * WK * kTile + (b >> 3) * 128 + (r % kPer) * 8 + (b & 7);
        float v = 0.f, up = 0.f;
        for (int w = 0; w < WK; ++w) {
          v += p[w * kTile];
          if (GATEUP) up += p[w * kTile + 64];
        }
        emit(u, r, b, v, up);
      }
    } else {
      float* mine = part + (u % a.R) * (WM * 16 * a.B);
      for (int i = tid; i < WM * 16 * a.B; i += kRowThreads) {
        const int b = i / (WM * 16), r = i - b * (WM * 16);
        const float* p = rd + (r >> 4) * WK * kTile + (b >> 3) * 128 + (r & 15) * 8 + (b & 7);
        float v = 0.f;
        for (int w = 0; w < WK; ++w) v += p[w * kTile];
        mine[i] = v;
      }
      if ((u + 1) % a.R == 0 || u + 1 == nu) {
        const int first = u - u % a.R, units = u + 1 - first;
        cluster_barrier();
        for (int i = rank * kRowThreads + tid; i < units * outs; i += S * kRowThreads) {
          const int du = i / outs, j = i - du * outs, b = j / (WM * kPer), r = j - b * (WM * kPer);
          const float* p = part + du * (WM * 16 * a.B) + b * (WM * 16) + (GATEUP ? (r >> 3) * 16 + (r & 7) : r);
          float v = 0.f, up = 0.f;
          for (int w = 0; w < S; ++w) {
            v += cluster_read(p, w);
            if (GATEUP) up += cluster_read(p + 8, w);
          }
          emit(first + du, r, b, v, up);
        }
        cluster_barrier();                                     // nobody overwrites or leaves while another block reads
      }
    }
  };

  if (total > 0) { fetch_id(0); open_unit(); }
  Chunk<W, ZP> ring[kRing];
#pragma unroll
  for (int d = 0; d < kRing; ++d)
    if (d < total) load(ring[d]);
  int cc = 0, u = 0;
  for (int it = 0; it < total; it += kRing) {
#pragma unroll
    for (int d = 0; d < kRing; ++d) {
      if (it + d < total) {
        compute(ring[d], cc);
        if (it + d + kRing < total) load(ring[d]);
        if (++cc == cw) { finish_unit(u); cc = 0; ++u; }
      }
    }
  }
}

// ----------------------------------------------------------------------------
// Union of the tokens' channel lists: ascending channels that some token keeps, and a byte with those tokens' bits.
// ----------------------------------------------------------------------------
constexpr int kUnionThreads = 1024;

__global__ void __launch_bounds__(kUnionThreads, 1)
union_kernel(const int* __restrict__ sel, int stride, const int* __restrict__ count, int k2, int B, int F, int* __restrict__ list,
             uint8_t* __restrict__ members, int* __restrict__ n_out) {
  extern __shared__ __align__(16) unsigned un_bits[];          // [F / 4] a byte per channel
  __shared__ int ws[33];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int words = (F + 3) / 4;
  for (int i = tid; i < words; i += kUnionThreads) un_bits[i] = 0;
  dep_wait();
  dep_launch();
  __syncthreads();
  for (int b = 0; b < B; ++b) {
    const int k = count ? max(0, min(k2, count[b])) : k2;
    for (int i = tid; i < k; i += kUnionThreads) {
      const int id = sel[(size_t)b * stride + i];
      if ((unsigned)id < (unsigned)F) atomicOr(un_bits + (id >> 2), (1u << b) << (8 * (id & 3)));
    }
  }
  __syncthreads();
  const int per = (words + kUnionThreads - 1) / kUnionThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
  int mine = 0;
  for (int w = w0; w < w1; ++w) {
    const unsigned v = un_bits[w];
    mine += ((v & 0xffu) != 0) + ((v & 0xff00u) != 0) + ((v & 0xff0000u) != 0) + ((v & 0xff000000u) != 0);
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int p = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += p;
  }
  if (lane == 31) ws[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    int v = ws[lane], s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int p = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += p;
    }
    ws[lane] = s - v;
    if (lane == 31) *n_out = s;
  }
  __syncthreads();
  int at = ws[warp] + inc - mine;
  for (int w = w0; w < w1; ++w) {
    const unsigned v = un_bits[w];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned m = v >> (8 * j) & 0xffu;
      if (m) { list[at] = w * 4 + j; members[at] = (uint8_t)m; ++at; }
    }
  }
}

// ----------------------------------------------------------------------------
// Down projection over listed channels: y[b, d] = sum_r h[b, r] s[r, d / G] (q[r, d] - z).
//
// A cluster of S blocks owns 128 columns (one scale group); its warps take tiles of 16 list entries in turn.  M = columns,
// K = list entries, N = tokens: a lane reads 16 codes of each of its four rows; the codes of two rows side by side are
// an A register.  h s goes in as three bf16 parts (hi + mid + lo, 24 bits), one column of B each, so that nothing is lost
// against fp32.  Sums over warps, parts and blocks in a fixed order.
// ----------------------------------------------------------------------------
constexpr int kDownThreads = 256;
constexpr int kDownWarps = kDownThreads / 32;

struct DownArgs {
  Mat w;                   // [F][D / 2] channel-major
  int D, F, groups, gstep;
  const int* list;
  const int* count;
  int n;
  const float* h;
  int h_stride, B;
  void* y;
  int y_type, S;
};

template <bool ZP>
struct DownTile {          // a lane's share of 16 list entries: four rows, 16 codes each
  uint2 q[4];
  __half s[4];
  uint8_t z[ZP ? 4 : 1];
};

template <int NT, bool ZP>
__global__ void __launch_bounds__(kDownThreads, NT == 1 ? 2 : 1) down_kernel(const DownArgs a) {
  extern __shared__ __align__(16) uint8_t down_smem[];
  float* red = reinterpret_cast<float*>(down_smem);            // [warps][128 columns][NT * 8]
  constexpr int kCols = NT * 8;
  float* part = red + kDownWarps * 128 * kCols;                // [128][B]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int S = a.S, rank = blockIdx.x % S, cg = blockIdx.x / S;
  dep_wait();
  dep_launch();
  int n = a.n;
  if (a.count) n = max(0, min(n, *a.count));
  const int tiles = (n + 15) / 16, step = S * kDownWarps;
  const uint8_t* base = a.w.codes + cg * 64 + g * 8;
  const int gi = cg * a.gstep;

  float acc[8][NT][4];
#pragma unroll
  for (int m = 0; m < 8; ++m)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[m][i][0] = acc[m][i][1] = acc[m][i][2] = acc[m][i][3] = 0.f;

  auto load = [&](DownTile<ZP>& b, int tile) {
    if (tile >= tiles) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int pos = tile * 16 + t * 4 + r;
      int id = a.list[min(pos, n - 1)];
      if ((unsigned)id >= (unsigned)a.F) id = 0;
      b.q[r] = ld8(base + (size_t)id * (a.D / 2));
      b.s[r] = a.w.scales[(size_t)id * a.groups + gi];
      if (ZP) b.z[r] = a.w.zeros[(size_t)id * a.groups + gi];
    }
  };
  auto compute = [&](const DownTile<ZP>& b, int tile) {
    uint32_t bf[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int token = (i * 8 + g) / 3, piece = (i * 8 + g) % 3;
      uint32_t v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int pos = tile * 16 + t * 4 + r;
        float f = 0.f;
        if (pos < n && token < a.B) f = a.h[(size_t)token * a.h_stride + pos] * __half2float(b.s[r]);
        __nv_bfloat16 p = __float2bfloat16_rn(f);
        if (piece > 0) { f -= __bfloat162float(p); p = __float2bfloat16_rn(f); }
        if (piece > 1) { f -= __bfloat162float(p); p = __float2bfloat16_rn(f); }
        v[r] = __bfloat16_as_ushort(p);
      }
      bf[i][0] = v[0] | v[1] << 16;
      bf[i][1] = v[2] | v[3] << 16;
    }
    uint32_t z01 = magic<kBf16>() | 0x00080008u, z23 = z01;
    if (ZP) {
      z01 = magic<kBf16>() | b.z[0] | (uint32_t)b.z[1] << 16;
      z23 = magic<kBf16>() | b.z[2] | (uint32_t)b.z[3] << 16;
    }
#pragma unroll
    for (int hw = 0; hw < 4; ++hw) {                           // four columns of every row at a time
      const uint32_t sel = hw & 1 ? 0x7632u : 0x5410u;
      const uint32_t p01 = hw < 2 ? __byte_perm(b.q[0].x, b.q[1].x, sel) : __byte_perm(b.q[0].y, b.q[1].y, sel);
      const uint32_t p23 = hw < 2 ? __byte_perm(b.q[2].x, b.q[3].x, sel) : __byte_perm(b.q[2].y, b.q[3].y, sel);
      uint32_t v01[4], v23[4];
      unpack<kBf16>(v01, p01, z01);
      unpack<kBf16>(v23, p23, z23);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < NT; ++i)
          mma<kBf16>(acc[hw * 2 + m][i], v01[2 * m], v01[2 * m + 1], v23[2 * m], v23[2 * m + 1], bf[i][0], bf[i][1]);
    }
  };
  constexpr int kDepth = 2;
  DownTile<ZP> ring[kDepth];
  const int first = rank * kDownWarps + warp;
#pragma unroll
  for (int d = 0; d < kDepth; ++d) load(ring[d], first + d * step);
  for (int tile = first; tile < tiles; tile += kDepth * step) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (tile + d * step < tiles) {
        compute(ring[d], tile + d * step);
        load(ring[d], tile + (d + kDepth) * step);
      }
    }
  }
  // column of acc[m], tile row g (c0, c1) or g + 8 (c2, c3): g * 16 + 2 m, or + 1
#pragma unroll
  for (int m = 0; m < 8; ++m)
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float* p = red + (size_t)(warp * 128 + g * 16 + 2 * m) * kCols + i * 8 + 2 * t;
      *reinterpret_cast<float2*>(p) = make_float2(acc[m][i][0], acc[m][i][1]);
      *reinterpret_cast<float2*>(p + kCols) = make_float2(acc[m][i][2], acc[m][i][3]);
    }
  __syncthreads();
  for (int i = tid; i < 128 * a.B; i += kDownThreads) {
    const int b = i >> 7, d = i & 127;
    float v = 0.f;
    for (int w = 0; w < kDownWarps; ++w) {
      const float* p = red + (size_t)(w * 128 + d) * kCols + b * 3;
      v += p[0] + (p[1] + p[2]);
    }
    part[i] = v;
  }
  if (S > 1) cluster_barrier();
  else __syncthreads();
  for (int i = rank * kDownThreads + tid; i < 128 * a.B; i += S * kDownThreads) {
    float v = 0.f;
    for (int w = 0; w < S; ++w) v += S > 1 ? cluster_read(part + i, w) : part[i];
    store(a.y, (size_t)(i >> 7) * a.D + cg * 128 + (i & 127), v, a.y_type);
  }
  if (S > 1) cluster_barrier();
}

// ----------------------------------------------------------------------------
// Packer: symmetric codes of bf16 weights, the rule of the proxies (scale = fp16(max|w| / 7), round to nearest even).  A
// warp per group; bound by HBM, offline.
// ----------------------------------------------------------------------------
__global__ void __launch_bounds__(256)
quantize_kernel(const uint32_t* __restrict__ w, int rows, int cols, int width, int groups, uint8_t* __restrict__ codes,
                __half* __restrict__ scales) {
  const long long job = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (job >= (long long)rows * groups) return;
  const long long row = job / groups;
  const int gi = (int)(job - row * groups);
  const int p0 = gi * (width / 2), p1 = min(cols / 2, p0 + width / 2);   // pairs of columns
  const uint32_t* src = w + row * (cols / 2);
  float m = 0.f;
  for (int p = p0 + lane; p < p1; p += 32) {
    const uint32_t v = src[p];
    m = fmaxf(m, fmaxf(fabsf(__uint_as_float(v << 16)), fabsf(__uint_as_float(v & 0xffff0000u))));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const __half sh = __float2half_rn(__fdiv_rn(m, 7.0f));
  const float s = __half2float(sh);
  for (int p = p0 + lane; p < p1; p += 32) {
    const uint32_t v = src[p];
    int c[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float f = __uint_as_float(j ? v & 0xffff0000u : v << 16);
      const float q = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(f, s)), -7.f), 7.f) : 0.f;
      c[j] = (int)q + 8;
    }
    codes[row * (cols / 2) + p] = (uint8_t)(c[0] | c[1] << 4);
  }
  if (lane == 0) scales[row * groups + gi] = sh;
}

}  // namespace w4
}  // namespace prox
