// Weights held in 4 bits: projections of a few tokens (prox_w4_linear) and Stage 2 of the sparse FFN over such
// weights (prox_w4_stage2_ffn; Sec. 4.1 Stage 2, with the low-bit weights that the paper leaves to future work).
//
//   w[n, k] = s[n, k / G] (q[n, k] - z[n, k / G])          q 4 bits, s fp16, z an integer (8 where there are none)
//   y[b, n] = sum_groups s[n, G] ( sum_{k in group} (q[n, k] - z) x[b, k] )
//
// The inner sum is a sum of whole numbers: a token's inputs are written as fixed-point numbers of 30 bits below the
// token's largest, x = X 2^-e, and X as four signed base-256 digits, each a column of the B operand of the warp-level tensor-core
// tile mma.sync m16n8k32 (s8 x s8 -> s32).  A code becomes an s8 operand by one shift and two logic operations for eight of
// them, 16 (q - 8): three issue slots against nine in a 16-bit form (shift, four masks, four operations that take the
// zero point off), and a tile step covers twice the columns.  Sums are exact; scales enter in fp32 once per group.  All
// kernels are to be bound by the weight stream: codes are read where the caller has them, once, and never written back in a
// wider form.  What limits them next is the issue rate: while HBM delivers 1 KB to an SM it issues 177 instructions.  tcgen05
// would want the codes unpacked in shared memory (it takes its operand from there): once in, once out and once in again
// for the tile, more than the shared memory's bandwidth leaves at that rate, and a scale per group would have its sums read
// back from tensor memory at two bytes for one of codes.
//
// Fragment layout of mma.sync.m16n8k32 (g = lane / 4, t = lane % 4; four k a register):
//   A: a0 = (row g, k 4t..4t+3)  a1 = (row g + 8, same k)  a2 = (row g, k 4t+16..+19)  a3 = (row g + 8, same as a2)
//   B: b0 = (k 4t..4t+3, col g)  b1 = (k 4t+16..+19, col g)    C: c0c1 = (row g, col 2t..2t+1)  c2c3 = (row g + 8, same)
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
__device__ __forceinline__ uint32_t ld4(const void* p) {
  uint32_t v;
  asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint16_t ld2(const void* p) {
  uint16_t v;
  asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint16_t ld1(const void* p) {
  uint16_t v;
  asm volatile("ld.global.nc.u8 %0, [%1];" : "=h"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
  uint2 v;
  asm volatile("ld.global.nc.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

__device__ __forceinline__ void mma(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A byte holds two codes: 16 (code - 8) of the low and of the high ones of four bytes.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return ((w << 4) & 0xf0f0f0f0u) ^ 0x80808080u; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return (w & 0xf0f0f0f0u) ^ 0x80808080u; }

// The four signed base-256 digits of a number, |v| <= 2^30, lowest in the lowest byte.
__device__ __forceinline__ uint32_t digits(int v) { return ((uint32_t)v + 0x80808080u) ^ 0x80808080u; }

// Byte j of four words, word i at byte i of r[j].
__device__ __forceinline__ void transpose(uint32_t (&r)[4], uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab0 = __byte_perm(a, b, 0x5140), ab1 = __byte_perm(a, b, 0x7362), cd0 = __byte_perm(c, d, 0x5140), cd1 = __byte_perm(c, d, 0x7362);
  r[0] = __byte_perm(ab0, cd0, 0x5410);
  r[1] = __byte_perm(ab0, cd0, 0x7632);
  r[2] = __byte_perm(ab1, cd1, 0x5410);
  r[3] = __byte_perm(ab1, cd1, 0x7632);
}

// Fixed point of numbers up to the fp32 magnitude whose bits are `most`: times 2^e they are below 2^30.  What is not finite
// has no fixed point: its results are made NaN (scale_back).
__device__ __forceinline__ int fixed_exponent(uint32_t most) { return 156 - max((int)(most >> 23), 1); }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float times_pow2(float v, int e) {           // e in -250 .. 250
  const int a = max(-126, min(126, e));
  return v * pow2(a) * pow2(max(-126, min(126, e - a)));
}
__device__ __forceinline__ float scale_back(float v, uint32_t most) {   // codes are 16 (q - 8): another 2^-4
  return most >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : times_pow2(v, -fixed_exponent(most) - 4);
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
// in shared memory.  With one warp along the columns nothing is shared and warps run on their own; else partial sums meet
// in shared memory, of the cluster where it has more than one block, in a fixed order: results do not depend on timing.
// ----------------------------------------------------------------------------
constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kRing = 4;                 // chunks of a warp in flight (a batch): 512 threads x 4 x 32 bytes = 64 KB per SM
constexpr int kMaxPass = 8;              // tokens of a pass over the weights: 32 columns of digits
constexpr int kMaxSlices = 128;          // column slices of the down projection: 16384 / 128

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
  float* h;                // see emit
  unsigned* hmax;          // [blocks][B] bits of the largest |h| that a block has written
  unsigned* tickets;       // of the down projection behind it: set to 0
  int S, WM, WK, R;        // R: units whose partial sums a block keeps before the cluster adds them up
  int x_half;              // x is fp16 (else bf16)
  int x_vec;               // x rows start on 16-byte boundaries
};

// Chunks of a block of a cluster, of a warp along the columns: whole batches
__host__ __device__ constexpr int rows_share(int C, int S) { return S == 1 ? C : ((C + S - 1) / S + kRing - 1) / kRing * kRing; }
__host__ __device__ constexpr int rows_run(int Cs, int WK) { return ((Cs + WK - 1) / WK + kRing - 1) / kRing * kRing; }

// Shared memory behind the tokens' digits: sums of the digits of a group (zero points only), warps' partial tiles, block's sums
__host__ __device__ constexpr size_t rows_digit_bytes(int chunks, int B) { return (size_t)chunks * 512 * B; }
__host__ __device__ constexpr size_t rows_fixed_bytes(int chunks, int B, int words, bool zp) {
  return rows_digit_bytes(chunks, B) + (zp ? (size_t)chunks * (4 / words) * B * 16 : 0);
}
__host__ __device__ constexpr size_t rows_red_bytes(int nt) { return (size_t)2 * kRowWarps * nt * 512; }   // only where WK > 1

// What a lane holds of its two rows: a chunk's codes, and the scales and zero points of a batch of kRing chunks.
struct Codes { uint32_t q[2][4]; };
template <int W, bool ZP>
struct Scales {
  static constexpr int kGroups = kRing * 4 / W;
  uint32_t s[2][kGroups / 2];            // two a word
  uint32_t z[2][ZP ? kGroups / 4 : 1];   // four a word
};

__device__ __forceinline__ void inputs_of(float (&f)[8], const uint4& v, bool half) {
  const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (half) {
      f[2 * j] = __half2float(__ushort_as_half((unsigned short)e[j]));
      f[2 * j + 1] = __half2float(__ushort_as_half((unsigned short)(e[j] >> 16)));
    } else {
      f[2 * j] = __uint_as_float(e[j] << 16);
      f[2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
    }
  }
}

template <int W, int NT, bool ZP, bool GATEUP>
__global__ void __launch_bounds__(kRowThreads, 1) rows_kernel(const RowsArgs a) {
  extern __shared__ __align__(16) uint8_t rows_smem[];
  __shared__ unsigned xmax[kMaxPass], hm[kMaxPass];            // bits of the largest magnitude of a token's inputs, of its h
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int S = a.S, WM = a.WM, WK = a.WK, B = a.B, cols = 4 * B;
  const int rank = blockIdx.x % S, cid = blockIdx.x / S, ncl = gridDim.x / S;
  const int C = (a.K + 127) / 128, Cs = rows_share(C, S);
  const int cb0 = min(C, rank * Cs), cb1 = min(C, cb0 + Cs);
  constexpr int kTile = NT * 128;                              // a warp's partial tile: [NT][16 rows][8 columns]
  uint4* xs = reinterpret_cast<uint4*>(rows_smem);             // [chunk][two words of a lane][column][t]
  int* sx = reinterpret_cast<int*>(rows_smem + rows_digit_bytes(Cs, B));   // [group][column]
  float* red = reinterpret_cast<float*>(rows_smem + rows_fixed_bytes(Cs, B, W, ZP));   // [2][warps][kTile] (WK > 1)
  float* part = red + (WK > 1 ? 2 * kRowWarps * kTile : 0);    // [R][B][WM * 16] (S > 1)
  if (tid < kMaxPass) xmax[tid] = hm[tid] = 0;
  __syncthreads();
  dep_wait();
  dep_launch();
  int n = a.rows;
  if (GATEUP) {
    n = a.n;
    if (a.count) n = max(0, min(n, *a.count));
    if (blockIdx.x == 0 && tid < kMaxSlices) a.tickets[tid] = 0;
  }
  constexpr int kPer = GATEUP ? 8 : 16;                        // list entries of a tile
  const int U = (n + kPer * WM - 1) / (kPer * WM);
  if (cid >= U) {                                              // the whole cluster
    if (GATEUP && tid < B) a.hmax[blockIdx.x * B + tid] = 0;
    return;
  }
  const int nu = (U - cid - 1) / ncl + 1;

  // The tokens' digits, in the order in which lanes take them.  Of a code word, columns 0, 2, 4, 6 are the low codes
  // (b0) and 1, 3, 5, 7 the high ones (b1).  Two passes over x: the largest magnitude, then the digits; the first few
  // inputs of a thread stay in registers in between.
  {
    const int octets = (cb1 - cb0) * 16, items = octets * B;
    constexpr int kKeep = 4;
    uint4 keep[kKeep];
    auto read = [&](int i) {
      const int b = i / octets, k = cb0 * 128 + (i - b * octets) * 8;
      if (k >= a.K) return make_uint4(0, 0, 0, 0);
      const uint16_t* p = a.x + (size_t)b * a.x_stride + k;
      if (a.x_vec) return __ldg(reinterpret_cast<const uint4*>(p));
      uint32_t e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = __ldg(p + j);
      return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    };
    auto raise = [&](int i, const uint4& v) {
      float f[8];
      inputs_of(f, v, a.x_half);
      unsigned m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(f[j]) & 0x7fffffffu);
      if (m > xmax[i / octets]) atomicMax(xmax + i / octets, m);
    };
    auto write = [&](int i, const uint4& v) {
      const int b = i / octets, o = i - b * octets, e = fixed_exponent(xmax[b]);
      float f[8];
      inputs_of(f, v, a.x_half);
      uint32_t d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = digits(__float2int_rn(times_pow2(f[j], e)));
      uint32_t lo[4], hi[4];
      transpose(lo, d[0], d[2], d[4], d[6]);
      transpose(hi, d[1], d[3], d[5], d[7]);
      const int c = o >> 4, oc = o & 15;
      const int ot = W == 4 ? oc >> 2 : W == 2 ? (oc & 7) >> 1 : oc & 3;
      const int oi = W == 4 ? oc & 3 : W == 2 ? (oc >> 3) * 2 + (oc & 1) : oc >> 2;
      uint2* at = reinterpret_cast<uint2*>(xs + ((c * 2 + (oi >> 1)) * cols + b * 4) * 4 + ot) + (oi & 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j * 8] = make_uint2(lo[j], hi[j]);
    };
#pragma unroll
    for (int j = 0; j < kKeep; ++j)
      if (tid + j * kRowThreads < items) keep[j] = read(tid + j * kRowThreads);
#pragma unroll
    for (int j = 0; j < kKeep; ++j)
      if (tid + j * kRowThreads < items) raise(tid + j * kRowThreads, keep[j]);
    for (int i = tid + kKeep * kRowThreads; i < items; i += kRowThreads) raise(i, read(i));
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeep; ++j)
      if (tid + j * kRowThreads < items) write(tid + j * kRowThreads, keep[j]);
    for (int i = tid + kKeep * kRowThreads; i < items; i += kRowThreads) write(i, read(i));
  }
  __syncthreads();
  if (ZP) {
    for (int i = tid; i < (cb1 - cb0) * (4 / W) * cols; i += kRowThreads) {
      const int grp = i / cols, col = i - grp * cols, c = grp / (4 / W), j = grp % (4 / W);
      int sum = 0;
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int oi = j * W + w;
          const uint2 v = *(reinterpret_cast<const uint2*>(xs + ((c * 2 + (oi >> 1)) * cols + col) * 4 + q) + (oi & 1));
          sum = __dp4a((int)v.x, 0x01010101, __dp4a((int)v.y, 0x01010101, sum));
        }
      sx[i] = sum;
    }
    __syncthreads();
  }

  const int wm = warp / WK, wk = warp - wm * WK;
  const int cw = rows_run(Cs, WK), nb = cw / kRing;            // chunks and batches of a warp and unit (the last warps may have fewer)
  const int c0 = cb0 + wk * cw, c1 = wm < WM ? min(cb1, c0 + cw) : c0;

  // loading side: unit lu (of this cluster's units), batch lb of it
  int lu = 0, lb = 0;
  const uint8_t *q0 = nullptr, *q1 = nullptr;                  // the lane's two rows, at the batch
  const __half *s0 = nullptr, *s1 = nullptr;                   // ... at their starts
  const uint8_t *z0 = nullptr, *z1 = nullptr;
  int id_next = 0;
  auto entry = [&](int u) { return ((cid + u * ncl) * WM + wm) * kPer + g; };   // list entry of this lane's first row
  auto fetch_id = [&](int u) {                                 // a channel id is read one unit ahead of its rows
    if (GATEUP) {
      const int id = a.list[min(entry(u), n - 1)];
      id_next = (unsigned)id < (unsigned)a.rows ? id : 0;
    }
  };
  auto open_unit = [&]() {
    size_t r0, r1;
    if (GATEUP) {
      r0 = r1 = (size_t)id_next;
      if (lu + 1 < nu) fetch_id(lu + 1);
    } else {
      r0 = (size_t)min(entry(lu), a.rows - 1);
      r1 = (size_t)min(entry(lu) + 8, a.rows - 1);
    }
    const Mat& m1 = GATEUP ? a.w2 : a.w;
    q0 = a.w.codes + r0 * (a.K / 2) + (size_t)c0 * 64 + t * (4 * W);
    q1 = m1.codes + r1 * (a.K / 2) + (size_t)c0 * 64 + t * (4 * W);
    s0 = a.w.scales + r0 * a.groups;
    s1 = m1.scales + r1 * a.groups;
    if (ZP) {
      z0 = a.w.zeros + r0 * a.groups;
      z1 = m1.zeros + r1 * a.groups;
    }
  };
  // Codes of chunk d of batch lb.  A batch inside the row is read without any check; in the last one of a ragged row, what lies
  // behind the row or the warp's chunks is read again from the row's start and meets digits that are 0, or is not used.
  const int whole = min(c1, a.K / 128);                        // chunks before this one lie inside the row
  auto load = [&](Codes& b, int d) {
    const bool inside = c0 + lb * kRing + d < whole;
#pragma unroll
    for (int j = 0; j < 4 / W; ++j) {
      int at = d * 64 + j * (16 * W);
      if (!inside) {
        const int k = (c0 + lb * kRing + d) * 128 + j * (32 * W) + t * (8 * W);
        if (k >= a.K || c0 + lb * kRing + d >= c1) at = -((c0 + lb * kRing) * 64 + t * (4 * W));
      }
      if (W == 4) {
        const uint4 v0 = ld16(q0 + at), v1 = ld16(q1 + at);
        b.q[0][0] = v0.x; b.q[0][1] = v0.y; b.q[0][2] = v0.z; b.q[0][3] = v0.w;
        b.q[1][0] = v1.x; b.q[1][1] = v1.y; b.q[1][2] = v1.z; b.q[1][3] = v1.w;
      } else if (W == 2) {
        const uint2 v0 = ld8(q0 + at), v1 = ld8(q1 + at);
        b.q[0][2 * j] = v0.x; b.q[0][2 * j + 1] = v0.y;
        b.q[1][2 * j] = v1.x; b.q[1][2 * j + 1] = v1.y;
      } else {
        b.q[0][j] = ld4(q0 + at);
        b.q[1][j] = ld4(q1 + at);
      }
    }
  };
  // scales and zero points of batch lb: in wide loads where every row's start is aligned for them
  using S_ = Scales<W, ZP>;
  constexpr int kG = S_::kGroups;
  const bool wide = a.groups % kG == 0;
  auto load_scales = [&](S_& b) {
    const int gi = (c0 + lb * kRing) * (4 / W);
    if (wide && gi + kG <= a.groups) {
      if (kG == 4) {
        const uint2 v0 = ld8(s0 + gi), v1 = ld8(s1 + gi);
        b.s[0][0] = v0.x; b.s[0][1] = v0.y; b.s[1][0] = v1.x; b.s[1][1] = v1.y;
      } else {
#pragma unroll
        for (int i = 0; i < kG / 8; ++i) {
          const uint4 v0 = ld16(s0 + gi + i * 8), v1 = ld16(s1 + gi + i * 8);
          b.s[0][4 * i] = v0.x; b.s[0][4 * i + 1] = v0.y; b.s[0][4 * i + 2] = v0.z; b.s[0][4 * i + 3] = v0.w;
          b.s[1][4 * i] = v1.x; b.s[1][4 * i + 1] = v1.y; b.s[1][4 * i + 2] = v1.z; b.s[1][4 * i + 3] = v1.w;
        }
      }
      if (ZP) {
#pragma unroll
        for (int i = 0; i < kG / 4; ++i) {
          b.z[0][i] = ld4(z0 + gi + i * 4);
          b.z[1][i] = ld4(z1 + gi + i * 4);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        const int at = a.gstep ? min(gi + i, a.groups - 1) : 0;
        const uint32_t v0 = ld2(s0 + at), v1 = ld2(s1 + at);
        b.s[0][i / 2] = i & 1 ? b.s[0][i / 2] | v0 << 16 : v0;
        b.s[1][i / 2] = i & 1 ? b.s[1][i / 2] | v1 << 16 : v1;
        if (ZP) {
          const uint32_t x0 = ld1(z0 + at), x1 = ld1(z1 + at);
          b.z[0][i / 4] = i & 3 ? b.z[0][i / 4] | x0 << (8 * (i & 3)) : x0;
          b.z[1][i / 4] = i & 3 ? b.z[1][i / 4] | x1 << (8 * (i & 3)) : x1;
        }
      }
    }
  };
  auto advance = [&]() {                                       // to the next batch (behind the last one: that again)
    if (lb + 1 < nb) {
      ++lb;
      q0 += kRing * 64;
      q1 += kRing * 64;
    } else if (lu + 1 < nu) {
      ++lu;
      lb = 0;
      open_unit();
    }
  };

  int at_col[NT], at_sx[NT];                                   // columns behind the last token: computed, never used
#pragma unroll
  for (int m = 0; m < NT; ++m) {
    at_col[m] = min(m * 8 + g, cols - 1) * 4 + t;
    at_sx[m] = min(m * 8 + 2 * t, cols - 2);
  }
  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  // sums start at 1.5 2^23 as an fp32 number has it: with it the sum is the number's mantissa (|sum| <= 2^22)
  constexpr int kBias = 0x4b400000;
  auto compute = [&](const Codes& b, const S_& sc, int batch, int i4) {   // chunk i4 of the batch
    const int c = c0 + batch * kRing + i4;
    if (c >= c1) return;
    const uint4* xc = xs + (c - cb0) * 8 * cols;
    uint4 xv[NT];
#pragma unroll
    for (int j = 0; j < 4 / W; ++j) {
      const int gi = i4 * (4 / W) + j;
      int d[NT][4];
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        if (ZP) {                                              // 16 (q - z) = 16 (q - 8) + 16 (8 - z)
          const int2 v = *reinterpret_cast<const int2*>(sx + ((c - cb0) * (4 / W) + j) * cols + at_sx[m]);
          const int e0 = 128 - 16 * (int)(sc.z[0][gi / 4] >> (8 * (gi & 3)) & 0xff), e1 = 128 - 16 * (int)(sc.z[1][gi / 4] >> (8 * (gi & 3)) & 0xff);
          d[m][0] = kBias + e0 * v.x; d[m][1] = kBias + e0 * v.y;
          d[m][2] = kBias + e1 * v.x; d[m][3] = kBias + e1 * v.y;
        } else {
          d[m][0] = d[m][1] = d[m][2] = d[m][3] = kBias;
        }
      }
#pragma unroll
      for (int i = j * W; i < (j + 1) * W; ++i) {
        const uint32_t a0 = low_codes(b.q[0][i]), a1 = low_codes(b.q[1][i]), a2 = high_codes(b.q[0][i]), a3 = high_codes(b.q[1][i]);
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          if (!(i & 1)) xv[m] = xc[(i >> 1) * cols * 4 + at_col[m]];
          mma(d[m], a0, a1, a2, a3, i & 1 ? xv[m].z : xv[m].x, i & 1 ? xv[m].w : xv[m].y);
        }
      }
      const float f0 = __half2float(__ushort_as_half((unsigned short)(sc.s[0][gi / 2] >> (16 * (gi & 1))))),
                  f1 = __half2float(__ushort_as_half((unsigned short)(sc.s[1][gi / 2] >> (16 * (gi & 1)))));
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][e] = fmaf(e < 2 ? f0 : f1, __int_as_float(d[m][e]) - 12582912.f, acc[m][e]);
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
      const float h = kept ? up * (v / (1.0f + expf(-v))) : 0.f;
      // [tile of 32 entries][token][8 t + r]: entry r * 4 + t of the tile, as lanes t of the down projection take them
      a.h[((size_t)(pos >> 5) * B + b) * 32 + (pos & 3) * 8 + (pos >> 2 & 7)] = h;
      const unsigned m = __float_as_uint(h) & 0x7fffffffu;
      if (m > hm[b]) atomicMax(hm + b, m);
    }
  };
  const int outs = WM * kPer * B;
  auto cluster_sum = [&](int u) {                              // sums of units u - u % R .. u over the blocks
    const int first = u - u % a.R, units = u + 1 - first;
    cluster_barrier();
    for (int i = rank * kRowThreads + tid; i < units * outs; i += S * kRowThreads) {
      const int du = i / outs, j = i - du * outs, b = j / (WM * kPer), r = j - b * (WM * kPer);
      const float* p = part + du * (WM * 16 * B) + b * (WM * 16) + (GATEUP ? (r >> 3) * 16 + (r & 7) : r);
      float v = 0.f, up = 0.f;
      for (int w = 0; w < S; ++w) {
        v += cluster_read(p, w);
        if (GATEUP) up += cluster_read(p + 8, w);
      }
      emit(first + du, r, b, v, up);
    }
    cluster_barrier();                                         // nobody overwrites or leaves while another block reads
  };
  auto finish_unit = [&](int u) {
    float* mine = part + (S > 1 ? (u % a.R) * (WM * 16 * B) : 0);
    if (WK == 1) {
      // lane t has digits 0, 1 (t even) or 2, 3 (t odd) of token 2 m + t / 2; even lanes go on with row g, odd ones with row g + 8
      if (wm < WM) {
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          float v[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p = fmaf(acc[m][2 * e + 1], 256.f, acc[m][2 * e]), o = __shfl_xor_sync(0xffffffffu, p, 1);
            v[e] = fmaf(t & 1 ? p : o, 65536.f, t & 1 ? o : p);
            acc[m][2 * e] = acc[m][2 * e + 1] = 0.f;
          }
          const int b = m * 2 + (t >> 1);
          if (b < B) {
            if (S > 1) mine[b * (WM * 16) + wm * 16 + g + (t & 1) * 8] = scale_back(t & 1 ? v[1] : v[0], xmax[b]);
            else if (!GATEUP) emit(u, wm * 16 + g + (t & 1) * 8, b, scale_back(t & 1 ? v[1] : v[0], xmax[b]), 0.f);
            else if (!(t & 1)) emit(u, wm * 8 + g, b, scale_back(v[0], xmax[b]), scale_back(v[1], xmax[b]));
          }
        }
      }
    } else {
      float* rd = red + (u & 1) * (kRowWarps * kTile);
      if (wm < WM) {
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          float* at = rd + warp * kTile + m * 128 + g * 8 + 2 * t;
          *reinterpret_cast<float2*>(at) = make_float2(acc[m][0], acc[m][1]);
          *reinterpret_cast<float2*>(at + 64) = make_float2(acc[m][2], acc[m][3]);
          acc[m][0] = acc[m][1] = acc[m][2] = acc[m][3] = 0.f;
        }
      }
      __syncthreads();                                         // (two buffers: the next unit's sums do not meet the reads below)
      for (int i = tid; i < (S > 1 ? WM * 16 * B : outs); i += kRowThreads) {
        const int rows = S > 1 ? WM * 16 : WM * kPer, b = i / rows, r = i - b * rows;
        const int row = S == 1 && GATEUP ? (r >> 3) * 16 + (r & 7) : r;
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < (GATEUP ? 2 : 1); ++e) {           // (gate and up where the unit ends here)
          if (e == 1 && S > 1) break;
          const float* p = rd + (row >> 4) * WK * kTile + (b >> 1) * 128 + ((row & 15) + 8 * e) * 8 + (b & 1) * 4;
          float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int w = 0; w < WK; ++w) {
            const float4 o = *reinterpret_cast<const float4*>(p + w * kTile);
            q.x += o.x; q.y += o.y; q.z += o.z; q.w += o.w;
          }
          v[e] = scale_back(((q.w * 256.f + q.z) * 256.f + q.y) * 256.f + q.x, xmax[b]);
        }
        if (S > 1) mine[i] = v[0];
        else emit(u, r, b, v[0], v[1]);
      }
    }
    if (S > 1 && ((u + 1) % a.R == 0 || u + 1 == nu)) cluster_sum(u);
  };

  Codes ring[kRing];
  S_ now, next;
  if (wm < WM) {
    fetch_id(0);
    open_unit();
#pragma unroll
    for (int d = 0; d < kRing; ++d) load(ring[d], d);
    load_scales(now);
  }
  for (int u = 0; u < nu; ++u) {
    if (wm < WM) {                                             // (others have no tile of their own)
      for (int batch = 0; batch < nb; ++batch) {
        advance();
        load_scales(next);
#pragma unroll
        for (int d = 0; d < kRing; ++d) {
          compute(ring[d], now, batch, d);
          load(ring[d], d);
        }
        now = next;
      }
    }
    finish_unit(u);
  }
  if (GATEUP) {
    __syncthreads();
    if (tid < B) a.hmax[blockIdx.x * B + tid] = hm[tid];
  }
}

// ----------------------------------------------------------------------------
// Union of the tokens' channel lists: ascending channels that some token keeps, and a byte with those tokens' bits.
// A cluster of eight blocks, each with an eighth of the channels: every block looks through all lists for its own.  (A
// token names a channel at most once, so its bit needs no atomic; tokens follow one another.)
// ----------------------------------------------------------------------------
constexpr int kUnionThreads = 512;
constexpr int kUnionBlocks = 8;

__global__ void __launch_bounds__(kUnionThreads, 1)
union_kernel(const int* __restrict__ sel, int stride, const int* __restrict__ count, int k2, int B, int F, int* __restrict__ list,
             uint8_t* __restrict__ members, int* __restrict__ n_out) {
  extern __shared__ __align__(16) uint8_t un_bytes[];          // a byte per channel of this block
  __shared__ int ws[33], total;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x;
  const int share = (F + 4 * kUnionBlocks - 1) / (4 * kUnionBlocks) * 4, f0 = min(F, rank * share), nf = min(F, f0 + share) - f0;
  const int words = (nf + 3) / 4;
  unsigned* un_words = reinterpret_cast<unsigned*>(un_bytes);
  for (int i = tid; i < words; i += kUnionThreads) un_words[i] = 0;
  dep_wait();
  dep_launch();
  constexpr int kAhead = 16;
  for (int b = 0; b < B; ++b) {
    __syncthreads();
    const int k = count ? max(0, min(k2, count[b])) : k2;
    const int* from = sel + (size_t)b * stride;
    for (int i = tid; i < k; i += kAhead * kUnionThreads) {
      int id[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) id[j] = i + j * kUnionThreads < k ? from[i + j * kUnionThreads] : -1;
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (id[j] >= 0 && (unsigned)(id[j] - f0) < (unsigned)nf) un_bytes[id[j] - f0] |= (uint8_t)(1u << b);
    }
  }
  __syncthreads();
  const int per = (words + kUnionThreads - 1) / kUnionThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
  int mine = 0;
  for (int w = w0; w < w1; ++w) {
    const unsigned v = un_words[w];
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
    int v = lane < kUnionThreads / 32 ? ws[lane] : 0, s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int p = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += p;
    }
    ws[lane] = s - v;
    if (lane == 31) total = s;
  }
  cluster_barrier();
  int before = 0, all = 0;
  for (int r = 0; r < kUnionBlocks; ++r) {
    const int c = __float_as_int(cluster_read(reinterpret_cast<const float*>(&total), r));
    if (r < rank) before += c;
    all += c;
  }
  if (rank == 0 && tid == 0) *n_out = all;
  int at = before + ws[warp] + inc - mine;
  for (int w = w0; w < w1; ++w) {
    const unsigned v = un_words[w];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned m = v >> (8 * j) & 0xffu;
      if (m) { list[at] = f0 + w * 4 + j; members[at] = (uint8_t)m; ++at; }
    }
  }
  cluster_barrier();                                           // `total` is read by the others
}

// ----------------------------------------------------------------------------
// Down projection over listed channels: y[b, d] = sum_r h[b, r] s[r, d / G] (q[r, d] - z).
//
// M = columns, K = list entries, N = digits of the tokens' h s.  A warp owns 128 columns (one scale group) and takes
// tiles of 32 entries: 64 bytes of each of 32 rows, copied to its own stages in shared memory with what else the tile needs
// (scales, zero points, h); four rows' bytes are transposed into A registers.  h s is a fixed-point number of 30 bits below
// the largest that the warp can meet (the token's largest |h|, which the kernel before it has left, times the largest
// scale of the warp's rows), so one whole-number sum runs over all tiles: |digit| <= 128, |16 (q - 8)| <= 128, at most 65536
// entries, below 2^31.
// WC warps of a block are side by side in the columns (what they read of h and of the scales' sectors they share
// through L1), the other warps and the blocks of a slice split the entries.  Partial sums of the blocks go to the workspace;
// the block that finishes a slice adds them up, in the order of the blocks: results do not depend on timing.
// ----------------------------------------------------------------------------
constexpr int kDownBlocks = 160;         // blocks at most (the workspace is sized for them)
constexpr int kRowBlocks = 256;          // of the gate and up kernel, at most (their largest |h|)
__host__ __device__ constexpr int down_threads(int nt) { return nt >= 3 ? 256 : 512; }   // 32 sums a thread and 8 columns of digits
__host__ __device__ constexpr int down_stages(int nt) { return nt >= 3 ? 6 : 4; }        // 12 KB of codes a warp in flight, or 8

struct DownArgs {
  Mat w;                   // [F][D / 2] channel-major
  int D, F, groups, gstep;
  const int* list;
  const int* count;
  int n;
  const float* h;          // [tile][token][32], see rows_kernel
  const unsigned* hmax;    // [hblocks][B]
  int hblocks, B;
  void* y;
  int y_type;
  int WC, slices, splits;
  float* part;             // [slice][split][B][WC * 128]
  unsigned* tickets;       // [slice]
};

// bytes of a stage: 32 rows of codes, a word each of scales, zero points and where to look in them, h
__host__ __device__ constexpr int down_stage(int B) { return 2048 + 128 + 128 + 128 + 128 * B; }

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_l1(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// The aligned word that holds element i of an array of n elements of SIZE bytes, without what lies behind the array.
template <int SIZE>
__device__ __forceinline__ void copy_word(uint32_t dst, const void* base, long long i, long long n) {
  const long long w = i * SIZE & ~3LL, left = n * SIZE - w;
  const int bytes = left < 4 ? (int)left : 4;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(static_cast<const uint8_t*>(base) + w), "r"(bytes) : "memory");
}

template <int NT, bool ZP>
__global__ void __launch_bounds__(down_threads(NT), 1) down_kernel(const DownArgs a) {
  extern __shared__ __align__(16) uint8_t down_smem[];
  constexpr int kThreads = down_threads(NT), kWarps = kThreads / 32, kStages = down_stages(NT);
  __shared__ unsigned last, hm[kMaxPass];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, B = a.B;
  const int slice = blockIdx.x % a.slices, split = blockIdx.x / a.slices;
  const int WC = a.WC, WR = kWarps / WC, wc = warp % WC, wr = warp / WC;
  const int cg = slice * WC + wc;                              // the warp's group of 128 columns
  const bool active = cg * 128 < a.D;
  const int stage = down_stage(B);
  uint8_t* mine = down_smem + warp * (kStages * stage);
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  if (tid < kMaxPass) hm[tid] = 0;
  __syncthreads();
  dep_wait();
  dep_launch();
  int n = a.n;
  if (a.count) n = max(0, min(n, *a.count));
  const int tiles = (n + 31) / 32;
  const int b0 = (int)((long long)tiles * split / a.splits), b1 = active ? (int)((long long)tiles * (split + 1) / a.splits) : b0;
  const int gi = cg * a.gstep;
  const long long all = (long long)a.F * a.groups;

  // id of entry `lane` of a tile; entries behind the list repeat its last one (their h is not used)
  auto fetch = [&](int tile) {
    int id = 0;
    if (tile < b1) {
      id = a.list[min(tile * 32 + lane, n - 1)];
      if ((unsigned)id >= (unsigned)a.F) id = 0;
    }
    return id;
  };
  auto issue = [&](int tile, int slot, int id) {
    if (tile < b1) {
      const uint32_t at = mine_at + slot * stage;
#pragma unroll
      for (int p = 0; p < 4; ++p) {                            // row r at r * 64; its 16-byte pieces swapped so that lanes t do not meet
        const int r = p * 8 + (lane >> 2), piece = lane & 3;
        const int rid = __shfl_sync(0xffffffffu, id, r);
        copy16(at + r * 64 + ((piece ^ (r & 2)) << 4), a.w.codes + (size_t)rid * (a.D / 2) + cg * 64 + piece * 16);
      }
      const uint32_t word = at + 2048 + (lane & 3) * 32 + (lane >> 2) * 4;   // [t][r] of entry r * 4 + t
      const long long i = (long long)id * a.groups + gi;
      *reinterpret_cast<uint32_t*>(mine + slot * stage + 2304 + lane * 4) = (uint32_t)i;
      copy_word<2>(word, a.w.scales, i, all);
      if (ZP) copy_word<1>(word + 128, a.w.zeros, i, all);
#pragma unroll
      for (int p = 0; p < (NT + 1) / 2; ++p)
        if (p * 32 + lane < 8 * B) copy16_l1(at + 2432 + (p * 32 + lane) * 16, a.h + (size_t)tile * 32 * B + (p * 32 + lane) * 4);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const int first = b0 + wr;
  int id_next = fetch(first);
#pragma unroll 1
  for (int d = 0; d < kStages; ++d) {
    const int id = id_next;
    id_next = fetch(first + (d + 1) * WR);
    issue(first + d * WR, d, id);
  }

  // the fixed point of every token: 30 bits below max |h| max s
  for (int i = tid; i < a.hblocks * B; i += kThreads) {
    const unsigned m = a.hmax[i];
    if (m > hm[i % B]) atomicMax(hm + i % B, m);
  }
  unsigned smax = 0;
  for (int tile = first; tile < b1; tile += WR) smax = max(smax, (unsigned)ld2(a.w.scales + (long long)fetch(tile) * a.groups + gi) & 0x7fffu);
  smax = __reduce_max_sync(0xffffffffu, smax);
  const float top = __half2float(__ushort_as_half((unsigned short)smax));
  __syncthreads();
  auto most_of = [&](int b) { return __float_as_uint(__uint_as_float(hm[b]) * top) & 0x7fffffffu; };
  int token[NT];
  float factor[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    token[i] = min(i * 2 + (g >> 2), B - 1);                   // columns behind the last token: computed, never used
    factor[i] = pow2(min(fixed_exponent(most_of(token[i])) - 1, 126));   // (the product is rounded: one bit of room)
  }
  int acc[8][NT][4], zacc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    zacc[i][0] = zacc[i][1] = zacc[i][2] = zacc[i][3] = 0;
#pragma unroll
    for (int m = 0; m < 8; ++m) acc[m][i][0] = acc[m][i][1] = acc[m][i][2] = acc[m][i][3] = 0;
  }
  auto compute = [&](int tile, int slot) {
    const uint8_t* st = mine + slot * stage;
    const unsigned i_low = *reinterpret_cast<const uint32_t*>(st + 2304 + lane * 4);   // of entry `lane`: where in the word its scale is
    const unsigned odd = __ballot_sync(0xffffffffu, i_low & 1) >> t;
    // A lane's column is digit g & 3 of a token.  The four lanes of a token make two of the eight numbers each that a lane t
    // needs, and exchange them byte by byte: a 4 x 4 transpose over lanes g ^ 1 and g ^ 2
    const int r0 = (g & 3) * 2;                                // rows r0, r0 + 1 (entries 4 r + t)
    const uint2 sw = *reinterpret_cast<const uint2*>(st + 2048 + t * 32 + r0 * 4);
    const float s0 = __half2float(__ushort_as_half((unsigned short)(sw.x >> ((odd >> (r0 * 4) & 1) << 4))));
    const float s1 = __half2float(__ushort_as_half((unsigned short)(sw.y >> ((odd >> (r0 * 4 + 4) & 1) << 4))));
    const bool in0 = tile * 32 + r0 * 4 + t < n, in1 = tile * 32 + r0 * 4 + 4 + t < n;
    uint32_t bf[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float2 h = *reinterpret_cast<const float2*>(st + 2432 + token[i] * 128 + t * 32 + r0 * 4);
      const uint32_t d0 = digits(in0 ? __float2int_rn(h.x * factor[i] * s0) : 0), d1 = digits(in1 ? __float2int_rn(h.y * factor[i] * s1) : 0);
      // bytes 0, 1 of both numbers, and bytes 2, 3: lanes of digits 0, 1 keep the former and get those of the lane two further on
      const uint32_t low = __byte_perm(d0, d1, 0x5140), high = __byte_perm(d0, d1, 0x7362);   // (d0.0 d1.0 d0.1 d1.1), (.2 .2 .3 .3)
      const uint32_t keep = g & 2 ? high : low, got = __shfl_xor_sync(0xffffffffu, g & 2 ? low : high, 8);
      // numbers 2 (g & 1) .. +1 in one, 4 + 2 (g & 1) .. +1 in the other; byte pairs: digit 0 or 1 (of this half)
      const uint32_t first4 = g & 2 ? got : keep, last4 = g & 2 ? keep : got;
      const uint32_t stay = __byte_perm(first4, last4, g & 1 ? 0x7632 : 0x5410), give = __byte_perm(first4, last4, g & 1 ? 0x5410 : 0x7632);
      const uint32_t other = __shfl_xor_sync(0xffffffffu, give, 4);
      bf[i][0] = __byte_perm(g & 1 ? other : stay, g & 1 ? stay : other, 0x5410);
      bf[i][1] = __byte_perm(g & 1 ? other : stay, g & 1 ? stay : other, 0x7632);
    }
    if (ZP) {                                                  // 16 (q - z) = 16 (q - 8) + 2 * 8 (8 - z), the same for all columns
      const unsigned two = __ballot_sync(0xffffffffu, i_low & 2) >> t;
      uint32_t zr[2];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint4 w = *reinterpret_cast<const uint4*>(st + 2176 + t * 32 + p * 16);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
        zr[p] = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int b = p * 16 + r * 4;
          zr[p] |= (uint32_t)((8 - (int)(v[r] >> ((odd >> b & 1) * 8 + (two >> b & 1) * 16) & 0xff)) * 8 & 0xff) << (8 * r);
        }
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) mma(zacc[i], zr[0], zr[0], zr[1], zr[1], bf[i][0], bf[i][1]);
    }
    uint2 q[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) q[r] = *reinterpret_cast<const uint2*>(st + (r * 4 + t) * 64 + (((g >> 1) ^ (t & 2)) << 4) + (g & 1) * 8);
#pragma unroll
    for (int hw = 0; hw < 2; ++hw) {                           // eight columns of every row at a time
      uint32_t lo[4], hi[4];
      if (hw == 0) {
        transpose(lo, q[0].x, q[1].x, q[2].x, q[3].x);
        transpose(hi, q[4].x, q[5].x, q[6].x, q[7].x);
      } else {
        transpose(lo, q[0].y, q[1].y, q[2].y, q[3].y);
        transpose(hi, q[4].y, q[5].y, q[6].y, q[7].y);
      }
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const uint32_t a0 = low_codes(lo[m]), a1 = high_codes(lo[m]), a2 = low_codes(hi[m]), a3 = high_codes(hi[m]);
#pragma unroll
        for (int i = 0; i < NT; ++i) mma(acc[hw * 4 + m][i], a0, a1, a2, a3, bf[i][0], bf[i][1]);
      }
    }
  };
  int slot = 0;
#pragma unroll 1
  for (int tile = first; tile < b1; tile += WR) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    __syncwarp();
    compute(tile, slot);
    __syncwarp();
    const int id = id_next;
    id_next = fetch(tile + (kStages + 1) * WR);
    issue(tile + kStages * WR, slot, id);
    if (++slot == kStages) slot = 0;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  // the warps' sums, one row of warps after the other: red[b][WC * 128]
  float* red = reinterpret_cast<float*>(down_smem);
  const int width = WC * 128;
  for (int r = 0; r < WR; ++r) {
    if (wr == r) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int b = i * 2 + (t >> 1);                        // lane t has digits 0, 1 (t even) or 2, 3 (t odd)
        const unsigned most = b < B ? most_of(b) : 0u;
#pragma unroll
        for (int m = 0; m < 8; ++m) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {                        // column g * 16 + 2 m + e of the warp's
            const int c0 = acc[m][i][2 * e] + (ZP ? 2 * zacc[i][2 * e] : 0), c1 = acc[m][i][2 * e + 1] + (ZP ? 2 * zacc[i][2 * e + 1] : 0);
            const float p = fmaf((float)c1, 256.f, (float)c0), o = __shfl_xor_sync(0xffffffffu, p, 1);
            float v = fmaf(t & 1 ? p : o, 65536.f, t & 1 ? o : p);
            if (b < B && (t & 1) == e) {
              v = most >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : times_pow2(v, -min(fixed_exponent(most) - 1, 126) - 4);
              float* at = red + b * width + wc * 128 + g * 16 + 2 * m + e;
              *at = r ? *at + v : v;
            }
          }
        }
      }
    }
    __syncthreads();
  }
  const bool direct = a.splits == 1;
  const int outs = width * B;
  float* out = a.part + ((size_t)slice * a.splits + split) * outs;
  for (int i = tid; i < outs; i += kThreads) {
    const int b = i / width, d = slice * width + i - b * width;
    if (!direct) __stcg(out + i, red[i]);
    else if (d < a.D) store(a.y, (size_t)b * a.D + d, red[i], a.y_type);
  }
  if (direct) return;
  __threadfence();
  __syncthreads();
  if (tid == 0) last = atomicAdd(a.tickets + slice, 1u) + 1 == (unsigned)a.splits;
  __syncthreads();
  if (!last) return;
  __threadfence();
  const float* in = a.part + (size_t)slice * a.splits * outs;
  for (int i = tid; i < outs; i += kThreads) {
    const int b = i / width, d = slice * width + i - b * width;
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < a.splits; ++k) v += __ldcg(in + (size_t)k * outs + i);
    if (d < a.D) store(a.y, (size_t)b * a.D + d, v, a.y_type);
  }
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
