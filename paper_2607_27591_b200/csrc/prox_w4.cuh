// Weights held in 4 bits: projections of a few tokens (prox_w4_linear) and Stage 2 of the sparse FFN over such
// weights (prox_w4_stage2_ffn; Sec. 4.1 Stage 2, with the low-bit weights that the paper leaves to future work).
//
//   w[n, k] = s[n, k / G] (q[n, k] - z[n, k / G])          q 4 bits, s fp16, z an integer (8 where there are none)
//   y[b, n] = sum_groups s[n, G] ( sum_{k in group} (q[n, k] - z) x[b, k] )
//
// The inner sum is a sum of whole numbers: a token's inputs are written as fixed-point numbers of 30 bits below the
// token's largest, x = X 2^-e, and X as four signed base-256 digits, each a column of the B operand of the warp-level tensor-core
// tile mma.sync m16n8k32 (u8 x s8 -> s32).  Eight codes become two u8 operands by a mask each, the low codes and 16 times the
// high ones: two issue slots against nine in a 16-bit form (shift, four masks, four operations that take the
// zero point off), and a tile step covers twice the columns.  Low and high codes have sums of their own, which start at what the
// zero point takes off.  Sums are exact; scales enter in fp32 once per group.  All
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
  asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t ld4(const void* p) {
  uint32_t v;
  asm volatile("ld.global.nc.L2::256B.u32 %0, [%1];" : "=r"(v) : "l"(p));
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
  asm volatile("ld.global.nc.L2::256B.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

__device__ __forceinline__ void mma(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A byte holds two codes: the low ones of four bytes, and 16 times the high ones.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x0f0f0f0fu; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0xf0f0f0f0u; }

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
__device__ __forceinline__ float scale_back(float v, uint32_t most) {
  return most >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : times_pow2(v, -fixed_exponent(most));
}

__device__ __forceinline__ void store(void* y, size_t i, float v, int type) {
  if (type == kFp32) static_cast<float*>(y)[i] = v;
  else if (type == kBf16) static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(y)[i] = __float2half_rn(v);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_l1(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int bytes = 4) {   // bytes in 0..4: the rest is 0
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// The aligned word that holds element i of an array of n elements of SIZE bytes, without what lies behind the array.
template <int SIZE>
__device__ __forceinline__ void copy_word(uint32_t dst, const void* base, long long i, long long n) {
  const long long w = i * SIZE & ~3LL, left = n * SIZE - w;
  const int bytes = left < 4 ? (int)left : 4;
  copy4(dst, static_cast<const uint8_t*>(base) + w, bytes);
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
  int S, WM, WK, R;        // R: units whose partial sums a block keeps before the cluster adds them up
  int x_half;              // x is fp16 (else bf16)
  int x_vec;               // x rows start on 16-byte boundaries
};

struct Codes { uint32_t q[2][4]; };      // what a lane holds of its two rows and a chunk

// A warp's scales and zero points of a batch, 16 rows: bytes of a row (with room for where an element lies in its word)
template <int W>
struct Side {
  static constexpr int kGroups = kRing * 4 / W;
  static constexpr int kScales = W == 4 ? 16 : W == 2 ? 32 : 48;
  static constexpr int kZeros = W == 4 ? 8 : W == 2 ? 16 : 32;
};
__host__ __device__ constexpr int rows_side_bytes(int words, bool zp) {   // of a warp, two batches
  return 2 * 16 * ((words == 4 ? 16 : words == 2 ? 32 : 48) + (zp ? words == 4 ? 8 : words == 2 ? 16 : 32 : 0));
}

// Chunks of a block of a cluster, of a warp along the columns: whole batches
__host__ __device__ constexpr int rows_share(int C, int S) { return S == 1 ? C : ((C + S - 1) / S + kRing - 1) / kRing * kRing; }
__host__ __device__ constexpr int rows_run(int Cs, int WK) { return ((Cs + WK - 1) / WK + kRing - 1) / kRing * kRing; }

// Shared memory behind the tokens' digits: where a group's sums start, warps' scales, warps' partial tiles, the block's sums.
// Start of a column pair (2 i, 2 i + 1) of a group, low and high codes: with zero points the sums of the digits that a zero
// point multiplies (4 words); else what the zero point 8 takes off, as the four C registers of either sum (8 words)
__host__ __device__ constexpr size_t rows_digit_bytes(int chunks, int nt) { return (size_t)chunks * 1024 * nt; }
__host__ __device__ constexpr size_t rows_fixed_bytes(int chunks, int nt, int words, bool zp) {
  return rows_digit_bytes(chunks, nt) + (size_t)chunks * (4 / words) * 4 * nt * (zp ? 16 : 32) + (size_t)kRowWarps * rows_side_bytes(words, zp);
}
__host__ __device__ constexpr size_t rows_red_bytes(int nt) { return (size_t)2 * kRowWarps * nt * 512; }   // only where WK > 1

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
  __shared__ int sid[3][GATEUP ? kRowWarps * 8 : 1];           // per unit (three alive at a time) and channel: what emit needs of it
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int S = a.S, WM = a.WM, WK = a.WK, B = a.B;
  constexpr int cols = 8 * NT, pairs = 4 * NT;                 // of digits: two tokens a step of 8 (behind the last token: whatever is there, never used)
  const int rank = blockIdx.x % S, cid = blockIdx.x / S, ncl = gridDim.x / S;
  const int C = (a.K + 127) / 128, Cs = rows_share(C, S);
  const int cb0 = min(C, rank * Cs), cb1 = min(C, cb0 + Cs);
  constexpr int kTile = NT * 128;                              // a warp's partial tile: [NT][16 rows][8 columns]
  uint4* xs = reinterpret_cast<uint4*>(rows_smem);             // [chunk][two words of a lane][column][t]
  int4* sx = reinterpret_cast<int4*>(rows_smem + rows_digit_bytes(Cs, NT));   // [group][pair of columns][1 or 2]
  uint8_t* side = rows_smem + rows_fixed_bytes(Cs, NT, W, ZP) - (kRowWarps - warp) * rows_side_bytes(W, ZP);   // this warp's, two batches
  const uint32_t side_at = (uint32_t)__cvta_generic_to_shared(side);
  float* red = reinterpret_cast<float*>(rows_smem + rows_fixed_bytes(Cs, NT, W, ZP));   // [2][warps][kTile] (WK > 1)
  float* part = red + (WK > 1 ? 2 * kRowWarps * kTile : 0);    // [R][B][WM * 16] (S > 1)
  if (tid < kMaxPass) xmax[tid] = hm[tid] = 0;
  __syncthreads();
  dep_wait();
  dep_launch();
  constexpr int kPer = GATEUP ? 8 : 16;                        // list entries of a tile
  const int wm = warp / WK, wk = warp - wm * WK;
  int id_next = 0;                                             // GATEUP: channel, and its tokens' bits from bit 20 on; 0 if it is none
  auto entry = [&](int u) { return ((cid + u * ncl) * WM + wm) * kPer + g; };   // list entry of this lane's first row
  auto fetch_id = [&](int u) {                                 // a channel id is read one unit ahead of its rows
    if (GATEUP) {
      const int pos = min(entry(u), max(a.n - 1, 0)), id = a.n > 0 ? a.list[pos] : -1;   // (an id behind the list's end is not used)
      const int tokens = a.members ? a.members[pos] : 1;
      id_next = (unsigned)id < (unsigned)a.rows ? id | tokens << 20 : 0;
    }
  };
  if (wm < WM) fetch_id(0);
  int n = a.rows;
  if (GATEUP) {
    n = a.n;
    if (a.count) n = max(0, min(n, *a.count));
  }
  const int U = (n + kPer * WM - 1) / (kPer * WM);
  if (cid >= U) {                                              // the whole cluster
    if (GATEUP && tid < B) a.hmax[blockIdx.x * B + tid] = 0;
    return;
  }
  const int nu = (U - cid - 1) / ncl + 1;

  const int cw = rows_run(Cs, WK), nb = cw / kRing;            // chunks and batches of a warp and unit (the last warps may have fewer)
  const int c0 = cb0 + wk * cw, c1 = wm < WM ? min(cb1, c0 + cw) : c0;

  // loading side: unit lu (of this cluster's units), batch lb of it
  int lu = 0, lb = 0;
  const uint8_t *q0 = nullptr, *q1 = nullptr;                  // the lane's two rows, at the batch
  int r0 = 0, r1 = 0;                                          // their numbers
  auto open_unit = [&]() {
    if (GATEUP) {
      r0 = r1 = id_next & 0xfffff;
      if (wk == 0 && t == 0) sid[lu % 3][wm * 8 + g] = id_next;
      if (lu + 1 < nu) fetch_id(lu + 1);
    } else {
      r0 = min(entry(lu), a.rows - 1);
      r1 = min(entry(lu) + 8, a.rows - 1);
    }
    q0 = a.w.codes + (size_t)r0 * (a.K / 2) + (size_t)c0 * 64 + t * (4 * W);
    q1 = (GATEUP ? a.w2.codes : a.w.codes) + (size_t)r1 * (a.K / 2) + (size_t)c0 * 64 + t * (4 * W);
  };
  // Codes of chunk d of batch lb.  A batch inside the row is read without any check; in the last one of a ragged row, what lies
  // behind the row or the warp's chunks is read again from the row's start and meets digits that are 0, or is not used.
  const int whole = min(c1, a.K / 128);                        // chunks before this one lie inside the row
  auto load = [&](Codes& b, int d, bool inside) {
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
  // Scales and zero points of batch lb of the tile's 16 rows, copied to shared memory: whole where every row's start is aligned
  // for it, else the words that hold them (a row's elements then start somewhere in its first word: `shift`)
  using Sd = Side<W>;
  constexpr int kG = Sd::kGroups, kWordsS = (2 * kG + 5) / 4, kWordsZ = (kG + 6) / 4;
  auto load_side = [&](int buffer) {
    const int gi = a.gstep ? (c0 + lb * kRing) * (4 / W) : 0;
    const uint32_t to = side_at + buffer * (rows_side_bytes(W, ZP) / 2), to_z = to + 16 * Sd::kScales;
    const bool whole_rows = a.groups % (ZP ? kG : kG < 8 ? kG : 8) == 0 && gi + kG <= a.groups;
    // lanes 4 i hold the numbers of rows i and i + 8
    auto row_of = [&](int i) {
      const int x0 = __shfl_sync(0xffffffffu, r0, (i & 7) * 4), x1 = __shfl_sync(0xffffffffu, r1, (i & 7) * 4);
      return i < 8 ? x0 : x1;
    };
    auto mat_of = [&](int i) -> const Mat& { return GATEUP && i >= 8 ? a.w2 : a.w; };
    if (whole_rows) {
      const int i = W == 1 ? lane >> 1 : lane & 15;
      const long long at = (long long)row_of(i) * a.groups + gi;
      if (W == 4 && lane < 16) copy8(to + i * Sd::kScales, mat_of(i).scales + at);
      if (W == 2 && lane < 16) copy16_l1(to + i * Sd::kScales, mat_of(i).scales + at);
      if (W == 1) copy16_l1(to + i * Sd::kScales + (lane & 1) * 16, mat_of(i).scales + at + (lane & 1) * 8);
      if (ZP) {
        if (W == 4 && lane < 16) copy4(to_z + i * Sd::kZeros, mat_of(i).zeros + at);
        if (W == 2 && lane < 16) copy8(to_z + i * Sd::kZeros, mat_of(i).zeros + at);
        if (W == 1 && !(lane & 1)) copy16_l1(to_z + i * Sd::kZeros, mat_of(i).zeros + at);
      }
    } else {
      const long long bytes = (long long)a.rows * a.groups * 2;
#pragma unroll
      for (int p = 0; p < (16 * kWordsS + 31) / 32; ++p) {
        const int e = p * 32 + lane, i = e / kWordsS & 15, w = e % kWordsS;
        const long long at = (((long long)row_of(i) * a.groups + gi) * 2 & ~3LL) + w * 4;
        if (e < 16 * kWordsS)
          copy4(to + i * Sd::kScales + w * 4, reinterpret_cast<const uint8_t*>(mat_of(i).scales) + (at < bytes ? at : 0), at < bytes ? (int)min(4LL, bytes - at) : 0);
      }
      if (ZP) {
        const long long zbytes = bytes / 2;
#pragma unroll
        for (int p = 0; p < (16 * kWordsZ + 31) / 32; ++p) {
          const int e = p * 32 + lane, i = e / kWordsZ & 15, w = e % kWordsZ;
          const long long at = (((long long)row_of(i) * a.groups + gi) & ~3LL) + w * 4;
          if (e < 16 * kWordsZ) copy4(to_z + i * Sd::kZeros + w * 4, mat_of(i).zeros + (at < zbytes ? at : 0), at < zbytes ? (int)min(4LL, zbytes - at) : 0);
        }
      }
    }
    copies_end();
    // byte offsets of this lane's rows in their first words: scales of row g and g + 8, zero points of row g and g + 8
    const unsigned e0 = (unsigned)r0 * (unsigned)a.groups + gi, e1 = (unsigned)r1 * (unsigned)a.groups + gi;
    return (e0 & 1) * 2 | (e1 & 1) << 9 | (e0 & 3) << 16 | (e1 & 3) << 24;
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

  // The tokens' digits, in the order in which lanes take them.  Of a code word, columns 0, 2, 4, 6 are the low codes
  // (b0) and 1, 3, 5, 7 the high ones (b1).  Two passes over x: the largest magnitude, then the digits; the first few
  // inputs of a thread stay in registers in between.
  Codes ring[kRing];
  uint32_t shift_now = 0;
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
    if (wm < WM) {                                             // the first weights: on their way meanwhile
      open_unit();
#pragma unroll
      for (int d = 0; d < kRing; ++d) load(ring[d], d, false);
      shift_now = load_side(0);
    }
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
  // sums start at 1.5 2^23 as an fp32 number has it: with it the sum is the number's mantissa (|sum| <= 2^22)
  constexpr int kBias = 0x4b400000;
  for (int i = tid; i < (cb1 - cb0) * (4 / W) * pairs; i += kRowThreads) {
    const int grp = i / pairs, pair = i - grp * pairs, c = grp / (4 / W), j = grp % (4 / W);
    int lo[2] = {0, 0}, hi[2] = {0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int oi = j * W + w;
          const uint2 v = *(reinterpret_cast<const uint2*>(xs + ((c * 2 + (oi >> 1)) * cols + pair * 2 + e) * 4 + q) + (oi & 1));
          lo[e] = __dp4a((int)v.x, 0x01010101, lo[e]);
          hi[e] = __dp4a((int)v.y, 0x01010101, hi[e]);
        }
    if (ZP) {
      sx[i] = make_int4(lo[0], lo[1], 16 * hi[0], 16 * hi[1]);
    } else {
      sx[2 * i] = make_int4(kBias - 8 * lo[0], kBias - 8 * lo[1], kBias - 8 * lo[0], kBias - 8 * lo[1]);
      sx[2 * i + 1] = make_int4(kBias - 128 * hi[0], kBias - 128 * hi[1], kBias - 128 * hi[0], kBias - 128 * hi[1]);
    }
  }
  __syncthreads();

  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  auto compute = [&](const Codes& b, const uint8_t* sc, uint32_t shift, int c, int i4) {   // chunk c, i4 of its batch
    const uint4* xc = xs + (c - cb0) * 8 * cols + g * 4 + t;
#pragma unroll
    for (int j = 0; j < 4 / W; ++j) {
      const int gi = a.gstep ? i4 * (4 / W) + j : 0;
      // two words a step: the low codes of both, the high codes of both (a group of one word: the other half is zeros)
      uint32_t lw[(W + 1) / 2][4], hw[(W + 1) / 2][4];
#pragma unroll
      for (int p = 0; p < (W + 1) / 2; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int word = j * W + 2 * p + (e >> 1);
          const uint32_t q = W > 1 || e < 2 ? b.q[e & 1][word & 3] : 0u;
          lw[p][e] = low_codes(q);
          hw[p][e] = high_codes(q);
        }
      const uint8_t* sr = sc + g * Sd::kScales + gi * 2;
      float f0 = __half2float(*reinterpret_cast<const __half*>(sr + (shift & 0xff))),
            f1 = __half2float(*reinterpret_cast<const __half*>(sr + 8 * Sd::kScales + (shift >> 8 & 0xff)));
      if (W < 4 && c * (4 / W) + j >= a.groups) f0 = f1 = 0.f;  // behind the row (the sums are 0: so that a neighbour's scale does not matter)
      int e0 = 0, e1 = 0;
      if (ZP) {
        const uint8_t* zr = sc + 16 * Sd::kScales + g * Sd::kZeros + gi;
        e0 = zr[shift >> 16 & 0xff];
        e1 = zr[8 * Sd::kZeros + (shift >> 24)];
      }
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        int lo[4], hi[4];
        const int at = ((c - cb0) * (4 / W) + j) * pairs + m * 4 + t;
        if (ZP) {
          const int4 v = sx[at];
          lo[0] = kBias - e0 * v.x; lo[1] = kBias - e0 * v.y; lo[2] = kBias - e1 * v.x; lo[3] = kBias - e1 * v.y;
          hi[0] = kBias - e0 * v.z; hi[1] = kBias - e0 * v.w; hi[2] = kBias - e1 * v.z; hi[3] = kBias - e1 * v.w;
        } else {
          const int4 v = sx[2 * at], u = sx[2 * at + 1];
          lo[0] = v.x; lo[1] = v.y; lo[2] = v.z; lo[3] = v.w;
          hi[0] = u.x; hi[1] = u.y; hi[2] = u.z; hi[3] = u.w;
        }
#pragma unroll
        for (int p = 0; p < (W + 1) / 2; ++p) {
          const uint4 v = xc[((j * W + 2 * p) >> 1) * cols * 4 + m * 32];   // low, high columns of one word, of the other
          if (W > 1) {
            mma(lo, lw[p][0], lw[p][1], lw[p][2], lw[p][3], v.x, v.z);
            mma(hi, hw[p][0], hw[p][1], hw[p][2], hw[p][3], v.y, v.w);
          } else {
            mma(lo, lw[p][0], lw[p][1], 0u, 0u, j & 1 ? v.z : v.x, 0u);
            mma(hi, hw[p][0], hw[p][1], 0u, 0u, j & 1 ? v.w : v.y, 0u);
          }
        }
        // (1.5 2^23 + low) + (1.5 2^23 + 16 high) / 16: whole numbers below 2^24, so exact
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[m][e] = fmaf(e < 2 ? f0 : f1, fmaf(__int_as_float(hi[e]), 0.0625f, __int_as_float(lo[e])) - 13369344.f, acc[m][e]);
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
      int what;                                                // the channel's tokens, from bit 20 on
      if (S == 1) {
        what = sid[u % 3][r];
      } else {                                                 // (a cluster ends several units at a time)
        const int id = a.list[pos];
        what = (unsigned)id < (unsigned)a.rows ? (a.members ? a.members[pos] : 1) << 20 : 0;
      }
      const float h = what >> (20 + b) & 1 ? up * (v / (1.0f + expf(-v))) : 0.f;
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

  int buffer = 0;
  for (int u = 0; u < nu; ++u) {
    if (wm < WM) {                                             // (others have no tile of their own)
      for (int batch = 0; batch < nb; ++batch) {
        copies_wait<0>();
        __syncwarp();
        advance();
        const uint32_t shift_next = load_side(buffer ^ 1);
        const uint8_t* sc = side + buffer * (rows_side_bytes(W, ZP) / 2);
        const int c = c0 + batch * kRing;
        if (c + kRing <= c1 && c0 + (lb + 1) * kRing <= whole) {   // (a batch without an end in it, and the next one to load)
#pragma unroll
          for (int d = 0; d < kRing; ++d) {
            compute(ring[d], sc, shift_now, c + d, d);
            load(ring[d], d, true);
          }
        } else {
#pragma unroll
          for (int d = 0; d < kRing; ++d) {
            if (c + d < c1) compute(ring[d], sc, shift_now, c + d, d);
            load(ring[d], d, false);
          }
        }
        __syncwarp();
        shift_now = shift_next;
        buffer ^= 1;
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
// A cluster of eight blocks, each with an eighth of the channels: every block looks through all lists for its own.
// ----------------------------------------------------------------------------
constexpr int kUnionThreads = 1024;
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
  __syncthreads();
  constexpr int kAhead = 16;                                   // (entries of a thread on their way at a time)
  const long long items = (long long)B * k2;
  for (long long i = tid; i < items; i += kAhead * kUnionThreads) {
    int id[kAhead], tok[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int e = (int)min(i + j * kUnionThreads, items - 1), b = e / k2, r = e - b * k2;
      tok[j] = b;
      id[j] = r < (count ? count[b] : k2) && i + j * kUnionThreads < items ? sel[(size_t)b * stride + r] : -1;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int f = id[j] - f0;
      if (id[j] >= 0 && (unsigned)f < (unsigned)nf) atomicOr(un_words + (f >> 2), 1u << (tok[j] + 8 * (f & 3)));
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
// the largest that the block can meet (the token's largest |h|, which the kernel before it has left, times the largest
// scale of the block's rows), so one whole-number sum runs over all tiles: |digit| <= 128, 16 q <= 240, at most 32768
// entries, below 2^30.
// WC warps of a block are side by side in the columns (what they read of h and of the scales' sectors they share
// through L1), the other warps and the S blocks of a cluster split the entries; their sums meet in the cluster's shared memory,
// in a fixed order: results do not depend on timing.
// ----------------------------------------------------------------------------
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
  int WC, S;
};

// bytes of a stage: 32 rows of codes, a word each of scales, zero points and where to look in them, h
__host__ __device__ constexpr int down_stage(int B) { return 2048 + 128 + 128 + 128 + 128 * B; }

template <int NT, bool ZP>
__global__ void __launch_bounds__(down_threads(NT), 1) down_kernel(const DownArgs a) {
  extern __shared__ __align__(16) uint8_t down_smem[];
  constexpr int kThreads = down_threads(NT), kWarps = kThreads / 32, kStages = down_stages(NT);
  __shared__ unsigned hm[kMaxPass], smax;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, B = a.B;
  const int S = a.S, rank = blockIdx.x % S, slice = blockIdx.x / S;
  const int WC = a.WC, WR = kWarps / WC, wc = warp % WC, wr = warp / WC;
  const int cg = slice * WC + wc;                              // the warp's group of 128 columns
  const bool active = cg * 128 < a.D;
  const int stage = down_stage(B);
  uint8_t* mine = down_smem + warp * (kStages * stage);
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  if (tid < kMaxPass) hm[tid] = 0;
  if (tid == kMaxPass) smax = 0;
  __syncthreads();
  // Up to dep_wait nothing is read that the gate and up kernel writes.  (What came before that kernel is complete: it has waited
  // for it before it let this one start.)
  int n = a.n;
  if (a.count) n = max(0, min(n, *a.count));
  const int tiles = (n + 31) / 32;
  const int b0 = (int)((long long)tiles * rank / S), b1 = (int)((long long)tiles * (rank + 1) / S), end = active ? b1 : b0;
  const int gi = cg * a.gstep;
  const long long all = (long long)a.F * a.groups;

  // id of entry `lane` of a tile; entries behind the list repeat its last one (their h is not used)
  auto fetch = [&](int tile) {
    int id = 0;
    if (tile < end) {
      id = a.list[min(tile * 32 + lane, n - 1)];
      if ((unsigned)id >= (unsigned)a.F) id = 0;
    }
    return id;
  };
  auto issue = [&](int tile, int slot, int id) {
    if (tile < end) {
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
    }
  };
  auto issue_h = [&](int tile, int slot) {
    if (tile < end) {
#pragma unroll
      for (int p = 0; p < (NT + 1) / 2; ++p)
        if (p * 32 + lane < 8 * B)
          copy16_l1(mine_at + slot * stage + 2432 + (p * 32 + lane) * 16, a.h + (size_t)tile * 32 * B + (p * 32 + lane) * 4);
    }
  };
  const int first = b0 + wr;
  int id_next;
  {
    int ids[kStages];
#pragma unroll
    for (int d = 0; d < kStages; ++d) ids[d] = fetch(first + d * WR);
    id_next = fetch(first + kStages * WR);
#pragma unroll
    for (int d = 0; d < kStages; ++d) issue(first + d * WR, d, ids[d]);
  }
  // the largest scale of the block's rows and columns: WC scales of a row in one load where they are aligned for it
  {
    const int g0 = slice * WC * a.gstep, width = a.gstep ? min(WC, a.groups - g0) : 1;
    const bool wide = width == WC && a.groups % WC == 0;
    uint32_t most = 0;
    constexpr int kAhead = 4;
    for (int e = b0 * 32 + tid; e < min(n, b1 * 32); e += kAhead * kThreads) {
      long long at[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        int id = a.list[min(e + j * kThreads, n - 1)];
        if ((unsigned)id >= (unsigned)a.F) id = 0;
        at[j] = (long long)id * a.groups + g0;
      }
      if (wide && WC == 8) {
        uint4 v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = __ldg(reinterpret_cast<const uint4*>(a.w.scales + at[j]));
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          most = __vmaxu2(most, __vmaxu2(__vmaxu2(v[j].x & 0x7fff7fffu, v[j].y & 0x7fff7fffu), __vmaxu2(v[j].z & 0x7fff7fffu, v[j].w & 0x7fff7fffu)));
      } else if (wide && WC == 4) {
        uint2 v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = __ldg(reinterpret_cast<const uint2*>(a.w.scales + at[j]));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) most = __vmaxu2(most, __vmaxu2(v[j].x & 0x7fff7fffu, v[j].y & 0x7fff7fffu));
      } else {
        for (int k = 0; k < width; ++k) {
          unsigned v[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) v[j] = __half_as_ushort(__ldg(a.w.scales + at[j] + k));
#pragma unroll
          for (int j = 0; j < kAhead; ++j) most = __vmaxu2(most, v[j] & 0x7fffu);
        }
      }
    }
    most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
    if (lane == 0 && most) atomicMax(&smax, most);
  }
  dep_wait();
  dep_launch();
#pragma unroll
  for (int d = 0; d < kStages; ++d) issue_h(first + d * WR, d);
  copies_end();
  for (int i = tid; i < a.hblocks * B; i += kThreads) {
    const unsigned m = a.hmax[i];
    if (m > hm[i % B]) atomicMax(hm + i % B, m);
  }
  __syncthreads();

  // the fixed point of every token: 30 bits below max |h| max s
  const float top = __half2float(__ushort_as_half((unsigned short)smax));
  auto most_of = [&](int b) { return __float_as_uint(__uint_as_float(hm[b]) * top) & 0x7fffffffu; };
  auto exponent_of = [&](unsigned most) { return min(fixed_exponent(most) - 1, 126); };   // (the product is rounded: one bit of room)
  int token[NT];
  float factor[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    token[i] = min(i * 2 + (g >> 2), B - 1);                   // columns behind the last token: computed, never used
    factor[i] = pow2(exponent_of(most_of(token[i])));
  }

  int acc[8][NT][4], zacc[NT][4];                              // even columns (rows g): sums of q, odd ones (g + 8): of 16 q
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
    uint32_t zr[2] = {0x08080808u, 0x08080808u};               // zero points: a sum of their own, the same for all columns
    if (ZP) {
      const unsigned two = __ballot_sync(0xffffffffu, i_low & 2) >> t;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint4 w = *reinterpret_cast<const uint4*>(st + 2176 + t * 32 + p * 16);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
        zr[p] = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int b = p * 16 + r * 4;
          zr[p] |= (v[r] >> ((odd >> b & 1) * 8 + (two >> b & 1) * 16) & 0xff) << (8 * r);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) mma(zacc[i], zr[0], zr[0], zr[1], zr[1], bf[i][0], bf[i][1]);
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
  copies_wait<0>();
  __syncwarp();
  int slot = 0;
#pragma unroll 1
  for (int tile = first; tile < end; tile += WR) {
    compute(tile, slot);
    __syncwarp();
    const int id = id_next;
    id_next = fetch(tile + (kStages + 1) * WR);
    issue(tile + kStages * WR, slot, id);
    issue_h(tile + kStages * WR, slot);
    copies_end();
    if (++slot == kStages) slot = 0;
    copies_wait<kStages - 1>();                                // the next tile's (the first kStages have come already)
    __syncwarp();
  }
  copies_wait<0>();
  __syncthreads();
  // the warps' sums: red[wr][b][WC * 128]
  float* red = reinterpret_cast<float*>(down_smem);
  const int width = WC * 128, outs = width * B;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int b = i * 2 + (t >> 1);                            // lane t has digits 0, 1 (t even) or 2, 3 (t odd) of the token
    const unsigned most = b < B ? most_of(b) : 0u;
    const int e = -exponent_of(most), e0 = max(-126, min(126, e));
    const float f0 = most >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : pow2(e0), f1 = pow2(max(-126, min(126, e - e0)));
    float* at = red + (size_t)wr * outs + b * width + wc * 128 + g * 16 + (t & 1);
#pragma unroll
    for (int m = 0; m < 8; ++m) {                              // columns g * 16 + 2 m (even lanes), + 1 (odd lanes) of the warp's
      float p[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int d0 = acc[m][i][2 * k] - (k ? 16 : 1) * zacc[i][0], d1 = acc[m][i][2 * k + 1] - (k ? 16 : 1) * zacc[i][1];
        p[k] = fmaf((float)d1, 256.f, (float)d0) * (k ? 0.0625f : 1.f);
      }
      const float o = __shfl_xor_sync(0xffffffffu, t & 1 ? p[0] : p[1], 1);   // the other half of the column that this lane goes on with
      const float v = t & 1 ? fmaf(p[1], 65536.f, o) : fmaf(o, 65536.f, p[0]);
      if (b < B) at[2 * m] = v * f0 * f1;
    }
  }
  __syncthreads();
  for (int i = tid; i < outs; i += kThreads) {
    float v = red[i];
    for (int w = 1; w < WR; ++w) v += red[(size_t)w * outs + i];
    red[i] = v;
  }
  cluster_barrier();
  for (int i = rank * kThreads + tid; i < outs; i += S * kThreads) {
    const int b = i / width, d = slice * width + i - b * width;
    float v = 0.f;
    for (int w = 0; w < S; ++w) v += cluster_read(red + i, w);
    if (d < a.D) store(a.y, (size_t)b * a.D + d, v, a.y_type);
  }
  cluster_barrier();                                           // nobody leaves while another block reads
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
