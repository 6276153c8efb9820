// Weights held in 4 bits: projections of a few tokens (prox_w4_linear) and Stage 2 of the sparse FFN over such
// weights (prox_w4_stage2_ffn; Sec. 4.1 Stage 2, with the low-bit weights that the paper leaves to future work).
//
//   w[n, k] = s[n, k / G] (q[n, k] - z[n, k / G])          q 4 bits, s fp16, z an integer (8 where there are none)
//   y[b, n] = sum_groups s[n, G] ( sum_{k in group} (q[n, k] - z) x[b, k] )
//
// The inner sum is a sum of whole numbers: a token's inputs are written as fixed-point numbers of 26 bits below the
// token's largest, x = X 2^-e, and X as four signed base-256 digits, each a column of the B operand of the warp-level tensor-core
// tile mma.sync m16n8k32 (u8 x s8 -> s32).  (26 bits, so that 16 X has four digits too.  An input is off by 2^-26 of the token's
// largest at most: bf16 inputs are exact down to 2^-18 of it, fp16 ones down to 2^-15.)  Eight codes become two u8 operands by a mask each, the low codes and 16 times the
// high ones: two issue slots against nine in a 16-bit form (shift, four masks, four operations that take the
// zero point off), and a tile step covers twice the columns.  The low codes meet the digits of 16 X and the high ones, 16-fold
// themselves, those of X, so that one sum takes both; it starts at what the zero point takes off.  Sums are exact; scales
// enter in fp32 once per group.  All
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

#include "prox_w4_plan.h"

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

__device__ __forceinline__ void mma(int (&d)[4], const int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
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

// Fixed point of numbers up to the fp32 magnitude whose bits are `most`: times 2^e they are below 2^26.  What is not finite
// has no fixed point: its results are made NaN (scale_back).
__device__ __forceinline__ int fixed_exponent(uint32_t most) { return 152 - max((int)(most >> 23), 1); }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float times_pow2(float v, int e) {           // e in -250 .. 250
  const int a = max(-126, min(126, e));
  return v * pow2(a) * pow2(max(-126, min(126, e - a)));
}
__device__ __forceinline__ float scale_back(float v, uint32_t most) {   // of 16 times a sum
  return most >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : times_pow2(v, -fixed_exponent(most) - 4);
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
// Sum of that float over the S blocks of the cluster (at most 8), in their order; all reads under way at once.
__device__ __forceinline__ float cluster_total(const float* p, int S) {
  float v[8];
#pragma unroll
  for (int w = 0; w < 8; ++w) v[w] = w < S ? cluster_read(p, w) : 0.f;
  float sum = v[0];
#pragma unroll
  for (int w = 1; w < 8; ++w) sum += v[w];
  return sum;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// ----------------------------------------------------------------------------
// Rows times tokens: y = x W^T for all rows of a matrix, or gate and up of listed channels with SwiGLU behind them.
//
// A warp owns tiles of 16 rows (linear) or of 8 channels (rows 0-7 of the tile are gate rows, rows 8-15 the up rows of
// the same channels, so that both pre-activations of a channel end in one place) and a run of 128-column chunks; it copies two
// chunks of its 16 rows at a time, a 128-byte line each, to a ring of its own in shared memory (plain loads of a lane's share, 64
// bytes of a row at a time, were waited for: 70 us against 57 for 131072 x 4096 and one token).  A block has WM tiles side by
// side and WK warps along the columns of each; a cluster of S blocks splits the columns further where the rows alone do not
// fill the GPU or the tokens do not fit in shared memory.  With one warp along the columns nothing is shared and warps run on
// their own; else partial sums meet in shared memory, of the cluster where it has more than one block, in a fixed order: results
// do not depend on timing.
//
// Measured in a chain of calls, weights from HBM (6.57 TB/s copied): one token, 131072 x 4096 with groups of 128: 52 us, 5.3 TB/s;
// 4096 x 4096: 6.3 us, of which the tokens' digits, the first weights and the end of the only unit are latency; eight
// tokens, 4096 x 14336: 23 us.  With eight tokens the issue rate bounds it (about 215 instructions a KB of codes, 1.8 a cycle).
// ----------------------------------------------------------------------------
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
  int S, WM, WK, stages, R;   // R: units whose partial sums a block keeps before the cluster adds them up
  int x_half;              // x is fp16 (else bf16)
  int x_vec;               // x rows start on 16-byte boundaries
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
  __shared__ int sid[8][GATEUP ? kRowWarps * 8 : 1];           // per unit (those on their way, and the last) and channel: the tokens that keep it
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int S = a.S, WM = a.WM, WK = a.WK, B = a.B;
  constexpr int cols = 8 * NT;                                 // of digits: two tokens a step of 8 (behind the last token: whatever is there, never used)
  const int rank = blockIdx.x % S, cid = blockIdx.x / S, ncl = gridDim.x / S;
  const int C = (a.K + 127) / 128, Cs = rows_share(C, S);
  const int cb0 = min(C, rank * Cs), cb1 = min(C, cb0 + Cs);
  constexpr int kTile = NT * 128;                              // a warp's partial tile: [NT][16 rows][8 columns]
  uint4* xs = reinterpret_cast<uint4*>(rows_smem);             // [chunk][two words of a lane][column][t]
  float* sx = reinterpret_cast<float*>(rows_smem + rows_digit_bytes(Cs, NT));   // [group][column], or C registers [group][pair of columns][4]
  using St = Stage<W>;
  uint8_t* stages = rows_smem + rows_fixed_bytes(Cs, NT, W) + warp * a.stages * St::kBytes;   // this warp's
  const uint32_t stages_at = (uint32_t)__cvta_generic_to_shared(stages);
  float* red = reinterpret_cast<float*>(rows_smem + rows_fixed_bytes(Cs, NT, W) + kRowWarps * a.stages * St::kBytes);   // [2][warps][kTile] (WK > 1)
  float* part = red + (WK > 1 ? 2 * kRowWarps * kTile : 0);    // [R][B][WM * 16] (S > 1)
  if (tid < kMaxPass) xmax[tid] = hm[tid] = 0;
  __syncthreads();
  dep_wait();
  dep_launch();
  constexpr int kPer = GATEUP ? 8 : 16;                        // list entries of a tile
  const int wm = warp / WK, wk = warp - wm * WK;
  int id_next = -1, bits_next = 1;                             // GATEUP: a channel and its tokens' bits, as they are in the lists
  // tile of a unit's warps i: the clusters take turns, so that what is left in the last unit is spread over all of them
  auto tile_of = [&](int u, int i) { return (u * WM + i) * ncl + cid; };
  auto entry = [&](int u) { return tile_of(u, wm) * kPer + g; };   // list entry of this lane's first row
  auto fetch_id = [&](int u) {                                 // asked for one unit ahead of its rows, and not looked at before
    if (GATEUP && a.n > 0) {
      const int pos = min(entry(u), a.n - 1);                  // (an entry behind the list's end is not used)
      id_next = a.list[pos];
      if (a.members) bits_next = a.members[pos];
    }
  };
  if (wm < WM) fetch_id(0);
  int n = a.rows;
  if (GATEUP) {
    n = a.n;
    if (a.count) n = max(0, min(n, *a.count));
  }
  const int tiles = (n + kPer - 1) / kPer;
  if (cid >= tiles) {                                          // the whole cluster
    if (GATEUP && tid < B) a.hmax[blockIdx.x * B + tid] = 0;
    return;
  }
  const int nu = (tiles + ncl * WM - 1) / (ncl * WM);          // units of the cluster
  const int mine = wm < WM && tile_of(0, wm) < tiles ? (tiles - 1 - tile_of(0, wm)) / (ncl * WM) + 1 : 0;   // those in which this warp has a tile

  const int cw = rows_run(Cs, WK), nb = cw / kBatch;           // chunks and batches of a warp and unit (the last warps may have fewer)
  const int c0 = cb0 + wk * cw, c1 = wm < WM ? min(cb1, c0 + cw) : c0;

  // loading side: unit lu (of this cluster's units), batch lb of it, into stage lslot
  int lu = 0, lb = 0, lslot = 0;
  constexpr int kG = St::kGroups, kWordsS = (2 * kG + 5) / 4, kWordsZ = (kG + 6) / 4;
  const bool aligned = a.groups % kG == 0;                     // scales of a batch of any row can be copied in one piece
  int r0 = 0, r1 = 0;                                          // numbers of rows g and g + 8 of the tile
  const uint8_t* rows[4];                                      // rows lane / 8, + 4, + 8, + 12 of the tile, at the lane's 16 bytes of a batch
  const __half* side = nullptr;                                // scales of row lane % 16
  const uint8_t* zside = nullptr;
  const int half = a.K / 2, piece = (lane & 7) * 16;
  const int gi0 = a.gstep ? c0 * (4 / W) : 0;
  __shared__ uint8_t shifts[kRowWarps][8][16];                 // of a warp's units on their way: where in its word a row's first element lies
  auto open_unit = [&]() {
    if (GATEUP) {
      const bool known = (unsigned)id_next < (unsigned)a.rows;
      r0 = r1 = known ? id_next : 0;
      if (wk == 0 && t == 0) sid[lu & 7][wm * 8 + g] = known ? bits_next : 0;
      if (lu + 1 < mine) fetch_id(lu + 1);
    } else {
      r0 = min(entry(lu), a.rows - 1);
      r1 = min(entry(lu) + 8, a.rows - 1);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int i = (p & 1) * 4 + (lane >> 3), r = __shfl_sync(0xffffffffu, p < 2 ? r0 : r1, i * 4);
      rows[p] = (GATEUP && p >= 2 ? a.w2.codes : a.w.codes) + (size_t)r * half + (size_t)c0 * 64 + piece;
    }
    const int x0 = __shfl_sync(0xffffffffu, r0, (lane & 7) * 4), x1 = __shfl_sync(0xffffffffu, r1, (lane & 7) * 4);
    const long long first = (long long)(lane & 8 ? x1 : x0) * a.groups + gi0;
    side = (GATEUP && lane & 8 ? a.w2.scales : a.w.scales) + first;
    if (ZP) zside = (GATEUP && lane & 8 ? a.w2.zeros : a.w.zeros) + first;
    if (lane < 16) shifts[warp][lu & 7][lane] = (uint8_t)(first & 3);
  };
  // What a batch needs that is not whole or not aligned: the row's end, scales in the words that hold them
  auto issue_ragged = [&](uint32_t to, int at) {
    // (what lies behind the row or the warp's columns is left as it is: it meets digits that are 0, or is not used)
    if (c0 * 64 + at + piece < min(half, c1 * 64)) {
#pragma unroll
      for (int p = 0; p < 4; ++p) copy16(to + (p * 4 + (lane >> 3)) * St::kPitch + piece, rows[p] + at);
    }
    const long long bytes = (long long)a.rows * a.groups * 2;
    const int ahead = a.gstep ? lb * kG : 0;
#pragma unroll 1
    for (int e = lane; e < 16 * kWordsS + lane; e += 32) {     // (all lanes take every turn)
      const int i = e / kWordsS & 15, w = e % kWordsS;
      const uint8_t* base = reinterpret_cast<const uint8_t*>(GATEUP && i >= 8 ? a.w2.scales : a.w.scales);
      const int x0 = __shfl_sync(0xffffffffu, r0, (i & 7) * 4), x1 = __shfl_sync(0xffffffffu, r1, (i & 7) * 4);
      const long long from = (((long long)(i < 8 ? x0 : x1) * a.groups + gi0 + ahead) * 2 & ~3LL) + w * 4;
      if (e < 16 * kWordsS) copy4(to + St::kAtScales + i * St::kScales + w * 4, base + (from < bytes ? from : 0), from < bytes ? (int)min(4LL, bytes - from) : 0);
    }
  };
  auto issue_zeros = [&](uint32_t to) {
    const long long bytes = (long long)a.rows * a.groups;
    const int ahead = a.gstep ? lb * kG : 0;
#pragma unroll 1
    for (int e = lane; e < 16 * kWordsZ + lane; e += 32) {
      const int i = e / kWordsZ & 15, w = e % kWordsZ;
      const uint8_t* base = GATEUP && i >= 8 ? a.w2.zeros : a.w.zeros;
      const int x0 = __shfl_sync(0xffffffffu, r0, (i & 7) * 4), x1 = __shfl_sync(0xffffffffu, r1, (i & 7) * 4);
      const long long from = (((long long)(i < 8 ? x0 : x1) * a.groups + gi0 + ahead) & ~3LL) + w * 4;
      if (e < 16 * kWordsZ) copy4(to + St::kAtZeros + i * St::kZeros + w * 4, base + (from < bytes ? from : 0), from < bytes ? (int)min(4LL, bytes - from) : 0);
    }
  };
  const int whole_batches = max(0, min(c1, a.K / 128) - c0) / kBatch;   // batches of a unit that are inside the row
  auto issue = [&]() {                                         // the next batch; nothing behind the last one
    if (lu < mine) {
      const uint32_t to = stages_at + lslot * St::kBytes;
      const int at = lb * (kBatch * 64);
      if (aligned && lb < whole_batches) {
#pragma unroll
        for (int p = 0; p < 4; ++p) copy16(to + (p * 4 + (lane >> 3)) * St::kPitch + piece, rows[p] + at);
        if (lane < 16) {
          const uint32_t dst = to + St::kAtScales + lane * St::kScales;
          if (W == 4) copy4(dst, side + lb * kG);
          else if (W == 2) copy8(dst, side + lb * kG);
          else copy16_l1(dst, side + lb * kG);
          if (ZP && W == 2) copy4(to + St::kAtZeros + lane * St::kZeros, zside + lb * kG);
          if (ZP && W == 1) copy8(to + St::kAtZeros + lane * St::kZeros, zside + lb * kG);
        }
        if (ZP && W == 4) issue_zeros(to);                     // (two zero points a row: half a word)
      } else {
        issue_ragged(to, at);
        if (ZP) issue_zeros(to);
      }
      if (++lslot == a.stages) lslot = 0;
      if (++lb == nb) {
        lb = 0;
        if (++lu < mine) open_unit();
      }
    }
    copies_end();
  };

  // The tokens' digits, in the order in which lanes take them.  Of a code word, columns 0, 2, 4, 6 are the low codes and
  // 1, 3, 5, 7 the high ones; a 16-byte entry is the low ones of two words, then their high ones.  First the raw inputs, to the
  // place of their own digits, and the largest magnitudes; then the digits.
  {
    // item: 16 inputs of the columns of two words of a lane t; its raw inputs first lie where its digits 0 and 1 go
    const int items = (cb1 - cb0) * 8;
    auto place = [&](int o, int b) {
      const int c = o >> 3, r = o & 7, ot = W == 1 ? r & 3 : W == 2 ? r & 3 : r >> 1, p = W == 1 ? r >> 2 : W == 2 ? r >> 2 : r & 1;
      return xs + ((c * 2 + p) * cols + b * 4) * 4 + ot;       // digit d 4 d further on
    };
    auto column = [&](int o, int h) {                          // first input of the item's first or second word
      const int c = cb0 + (o >> 3), r = o & 7;
      return c * 128 + (W == 1 ? (r >> 2) * 64 + h * 32 + (r & 3) * 8 : r * 16 + h * 8);
    };
    unsigned most[2 * NT];
#pragma unroll
    for (int b = 0; b < 2 * NT; ++b) most[b] = 0;
#pragma unroll 1
    for (int e = tid; e < items * 2; e += kRowThreads) {       // an item's first word, its second word
      const int o = e >> 1, h = e & 1, k = column(o, h);
      uint4 v[2 * NT];
#pragma unroll
      for (int b = 0; b < 2 * NT; ++b) {
        v[b] = make_uint4(0, 0, 0, 0);
        if (b < B && k < a.K && a.x_vec) v[b] = __ldg(reinterpret_cast<const uint4*>(a.x + (size_t)b * a.x_stride + k));
      }
      if (!a.x_vec && k < a.K) {
#pragma unroll 1
        for (int b = 0; b < B; ++b) {
          const uint16_t* p = a.x + (size_t)b * a.x_stride + k;
          const uint4 u = make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16, p[6] | (uint32_t)p[7] << 16);
#pragma unroll
          for (int i = 0; i < 2 * NT; ++i)
            if (i == b) v[i] = u;
        }
      }
#pragma unroll
      for (int b = 0; b < 2 * NT; ++b) {
        if (b < B) {
          // (magnitudes of 16 bits order as whole numbers, and so do they once they are fp32 numbers)
          const uint32_t m = __vmaxu2(__vmaxu2(v[b].x & 0x7fff7fffu, v[b].y & 0x7fff7fffu), __vmaxu2(v[b].z & 0x7fff7fffu, v[b].w & 0x7fff7fffu));
          most[b] = max(most[b], max(m & 0xffffu, m >> 16));
          place(o, b)[h * 4] = v[b];
        }
      }
    }
#pragma unroll
    for (int b = 0; b < 2 * NT; ++b) {
      if (b < B) {
        const unsigned m = __reduce_max_sync(0xffffffffu, most[b]);
        const unsigned bits = a.x_half ? __float_as_uint(__half2float(__ushort_as_half((unsigned short)m))) : m << 16;
        if (lane == 0 && m) atomicMax(xmax + b, bits);
      }
    }
    if (mine > 0) {                                            // the first weights: on their way meanwhile
      open_unit();
#pragma unroll 1
      for (int d = 0; d < a.stages; ++d) issue();
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < items * B; i += kRowThreads) {
      const int b = i / items, o = i - b * items;
      uint4* at = place(o, b);
      const int e = fixed_exponent(xmax[b]);
      uint32_t lo[2][4], hi[2][4];
      const uint4 raw[2] = {at[0], at[4]};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float f[8];
        inputs_of(f, raw[h], a.x_half);
        uint32_t d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = digits(__float2int_rn(times_pow2(f[j], e)) << (j & 1 ? 0 : 4));   // the low codes' 16-fold
        transpose(lo[h], d[0], d[2], d[4], d[6]);
        transpose(hi[h], d[1], d[3], d[5], d[7]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j * 4] = make_uint4(lo[0][j], lo[1][j], hi[0][j], hi[1][j]);
    }
  }
  __syncthreads();
  // What comes off 16 times a group's sum: the zero point times the digits' sum of the group's high columns 16-fold and low
  // columns: 8 times that, as the C registers that a lane's sums start with, or (zero points) that itself, in fp32.  (Below 2^24
  // all: exact.)
  for (int i = tid; i < (cb1 - cb0) * (4 / W) * cols; i += kRowThreads) {
    const int grp = i / cols, col = i % cols, c = grp / (4 / W), j = grp % (4 / W);
    int lo = 0, hi = 0;
#pragma unroll 1
    for (int oi = j * W; oi < (j + 1) * W; oi += 2)            // (a group of one word: half an entry)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4 v = xs[((c * 2 + (oi >> 1)) * cols + col) * 4 + q];
        if (W > 1 || !(oi & 1)) {
          lo = __dp4a((int)v.x, 0x01010101, lo);
          hi = __dp4a((int)v.z, 0x01010101, hi);
        }
        if (W > 1 || oi & 1) {
          lo = __dp4a((int)v.y, 0x01010101, lo);
          hi = __dp4a((int)v.w, 0x01010101, hi);
        }
      }
    const int sum = lo + 16 * hi;
    if (ZP) sx[i] = (float)sum;
    else reinterpret_cast<int*>(sx)[(i >> 1) * 4 + (i & 1)] = reinterpret_cast<int*>(sx)[(i >> 1) * 4 + 2 + (i & 1)] = -8 * sum;
  }
  __syncthreads();

  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  auto compute = [&](const uint8_t* st, int e0, int e1, int c, int i2) {   // chunk c, i2 of the batch in st; e0, e1: where its rows' first words start
    const uint4* xc = xs + (c - cb0) * 8 * cols + g * 4 + t;
    uint32_t q[2][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint8_t* from = st + (g + 8 * r) * St::kPitch + i2 * 64;
#pragma unroll
      for (int j = 0; j < 4 / W; ++j) {
        if (W == 4) {
          const uint4 v = *reinterpret_cast<const uint4*>(from + t * 16);
          q[r][0] = v.x; q[r][1] = v.y; q[r][2] = v.z; q[r][3] = v.w;
        } else if (W == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(from + j * 32 + t * 8);
          q[r][2 * j] = v.x; q[r][2 * j + 1] = v.y;
        } else {
          q[r][j] = *reinterpret_cast<const uint32_t*>(from + j * 16 + t * 4);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4 / W; ++j) {
      const int gi = a.gstep ? i2 * (4 / W) + j : 0;
      // two words a step: the low codes of both, the high codes of both (a group of one word: the other half is zeros)
      uint32_t lw[(W + 1) / 2][4], hw[(W + 1) / 2][4];
#pragma unroll
      for (int p = 0; p < (W + 1) / 2; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int word = j * W + 2 * p + (e >> 1);
          const uint32_t v = W > 1 || e < 2 ? q[e & 1][word & 3] : 0u;
          lw[p][e] = low_codes(v);
          hw[p][e] = high_codes(v);
        }
      const __half* sr = reinterpret_cast<const __half*>(st + St::kAtScales + g * St::kScales) + gi;
      float f0 = __half2float(sr[e0 & 1]), f1 = __half2float(sr[4 * St::kScales + (e1 & 1)]);
      if (W < 4 && c * (4 / W) + j >= a.groups) f0 = f1 = 0.f;  // behind the row (the sums are 0: so that a neighbour's scale does not matter)
      float z0 = 0.f, z1 = 0.f;
      if (ZP) {
        const uint8_t* zr = st + St::kAtZeros + g * St::kZeros + gi;
        z0 = zr[e0];
        z1 = zr[8 * St::kZeros + e1];
      }
      int d[NT][4];                                            // 16 times the group's sums
      float2 off[NT];
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        const int at = ((c - cb0) * (4 / W) + j) * cols + m * 8 + 2 * t;
        if (ZP) {
          off[m] = *reinterpret_cast<const float2*>(sx + at);
          d[m][0] = d[m][1] = d[m][2] = d[m][3] = 0;
        } else {
          const int4 v = *reinterpret_cast<const int4*>(sx + at * 2);
          d[m][0] = v.x; d[m][1] = v.y; d[m][2] = v.z; d[m][3] = v.w;
        }
      }
#pragma unroll
      for (int p = 0; p < (W + 1) / 2; ++p) {                  // (steps that follow one another are of different sums)
        uint4 v[NT];                                           // low columns of two words, high columns
#pragma unroll
        for (int m = 0; m < NT; ++m) v[m] = xc[((j * W + 2 * p) >> 1) * cols * 4 + m * 32];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          if (W > 1) mma(d[m], d[m], lw[p][0], lw[p][1], lw[p][2], lw[p][3], v[m].x, v[m].y);
          else mma(d[m], d[m], lw[p][0], lw[p][1], hw[p][0], hw[p][1], j & 1 ? v[m].y : v[m].x, j & 1 ? v[m].w : v[m].z);
        }
        if (W > 1) {
#pragma unroll
          for (int m = 0; m < NT; ++m) mma(d[m], d[m], hw[p][0], hw[p][1], hw[p][2], hw[p][3], v[m].z, v[m].w);
        }
      }
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = ZP ? fmaf(e < 2 ? -z0 : -z1, e & 1 ? off[m].y : off[m].x, (float)d[m][e]) : (float)d[m][e];
          acc[m][e] = fmaf(e < 2 ? f0 : f1, v, acc[m][e]);
        }
    }
  };
  // one output of unit u: row r of its WM * 16 tile rows (linear), or channel r of its WM * 8 (gate and up)
  auto emit = [&](int u, int r, int b, float v, float up) {
    const int pos = tile_of(u, r / kPer) * kPer + r % kPer;
    if (pos >= n) return;
    if (!GATEUP) {
      store(a.y, (size_t)b * a.y_stride + pos, v, a.y_type);
    } else {
      int what;                                                // the channel's tokens
      if (S == 1) {
        what = sid[u & 7][r];
      } else {                                                 // (a cluster ends several units at a time)
        const int id = a.list[pos];
        what = (unsigned)id < (unsigned)a.rows ? a.members ? a.members[pos] : 1 : 0;
      }
      const float h = what >> b & 1 ? up * (v / (1.0f + expf(-v))) : 0.f;
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
      emit(first + du, r, b, cluster_total(p, S), GATEUP ? cluster_total(p + 8, S) : 0.f);
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

  int slot = 0;
#pragma unroll 1
  for (int u = 0; u < nu; ++u) {
    if (u < mine) {                                            // (else the warp has no tile in this unit)
      int e0 = shifts[warp][u & 7][g], e1 = shifts[warp][u & 7][8 + g];
#pragma unroll 1
      for (int batch = 0; batch < nb; ++batch) {
        if (a.stages == kMaxStages) copies_wait<kMaxStages - 1>();
        else if (a.stages == 3) copies_wait<2>();
        else copies_wait<1>();
        __syncwarp();
        const uint8_t* st = stages + slot * St::kBytes;
        const int c = c0 + batch * kBatch;
        if (c + kBatch <= c1) {
#pragma unroll
          for (int d = 0; d < kBatch; ++d) compute(st, e0, e1, c + d, d);
        } else if (c < c1) {                                   // (kBatch is 2)
          compute(st, e0, e1, c, 0);
        }
        __syncwarp();
        issue();
        if (++slot == a.stages) slot = 0;
        if (a.gstep) { e0 = (e0 + kG) & 3; e1 = (e1 + kG) & 3; }
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
// Union of the tokens' channel lists: ascending channels that some token keeps, and a byte with those tokens' bits.  8 us for
// eight lists of 6690 (one block alone took 15), 5 us for four of 3345: latency.
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
  constexpr int kAhead = 4;                                    // entries of every token that a thread asks for at a time
  int lens[kMaxPass];
#pragma unroll
  for (int b = 0; b < kMaxPass; ++b) lens[b] = b < B ? count ? max(0, min(k2, count[b])) : k2 : 0;
#pragma unroll 1
  for (int i = tid; i < k2; i += kAhead * kUnionThreads) {
    int id[kMaxPass][kAhead];
#pragma unroll
    for (int b = 0; b < kMaxPass; ++b)
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        id[b][j] = -1;
        if (i + j * kUnionThreads < lens[b]) id[b][j] = sel[(size_t)b * stride + i + j * kUnionThreads];
      }
#pragma unroll
    for (int b = 0; b < kMaxPass; ++b)
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int f = id[b][j] - f0;
        if (id[b][j] >= 0 && (unsigned)f < (unsigned)nf) atomicOr(un_words + (f >> 2), 1u << (b + 8 * (f & 3)));
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
// (scales, zero points, h); four rows' bytes are transposed into A registers.  h s is a fixed-point number, and one
// whole-number sum runs over all tiles: |digit| <= 128, 16 q <= 240, at most 32768 entries, below 2^30.  (h is taken below 1 by a power
// of two first, so that no exponent is out of reach.)  Its exponent is the warp's and the token's: 30 bits are room for 4 times
// the token's largest |h s| in the warp's first tile, times what the list's largest |h| (which the kernel before this has left) is
// above the tile's, 64 times in all at most.  Where a tile brings a product that there is no room for, the token's exponent falls to make
// such room above it, and the numbers that its sums so far stand for are shifted down.  So a product is off by 2^-24 of the token's
// largest in its warp at most, and by 2^-27 of its largest |h| times its largest scale.  Channels that other tokens keep, or that are
// skipped, do not count.
// WC warps of a block are side by side in the columns (what they read of h and of the scales' sectors they share
// through L1), the other warps and the S blocks of a cluster split the entries; their sums meet in the cluster's shared memory,
// in a fixed order: results do not depend on timing.
//
// Measured: 3 us of the 14 us of Stage 2 of 4096 x 12288 with 2867 channels and one token once the h are there; 50 us for 8192 x
// 28672 and eight tokens (106 MB, 2.1 TB/s): four columns of digits a token make it bound by the issue rate.
// ----------------------------------------------------------------------------
__host__ __device__ constexpr int down_threads(int nt) { return nt >= 3 ? 256 : 512; }   // 32 sums a thread and 8 columns of digits
__host__ __device__ constexpr int down_stages(int nt) { return nt >= 3 ? 6 : 4; }        // 12 KB of codes a warp in flight, or 8

constexpr int kMaxPower = 120;           // of fixed-point numbers: what lies below 2^-90 of the largest |h| loses bits
constexpr int kMaxRoom = 6;              // bits kept free above the largest product so far, at most

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

// Exponent that takes numbers up to the fp32 magnitude whose bits are `most` below 1 (below 4 at fp32's upper end): their
// products with scales neither overflow nor run out of exponents.
__device__ __forceinline__ int unit_exponent(uint32_t most) { return max(126 - max((int)(most >> 23), 1), -126); }

// bytes of a stage: 32 rows of codes, a word each of scales, zero points and where to look in them, h
__host__ __device__ constexpr int down_stage(int B) { return 2048 + 128 + 128 + 128 + 128 * B; }

// The sums of the four digits of a number, two of them in this lane and two in the next (odd: the upper ones), for the number
// shifted down by `by` bits, rounded; c[0], c[1] and c[2], c[3] belong to different numbers.
__device__ __forceinline__ void shift_sums(int (&c)[4], int by, int odd) {
#pragma unroll
  for (int k = 0; k < 4; k += 2) {
    const long long mine = c[k] + 256ll * c[k + 1], other = __shfl_xor_sync(0xffffffffu, mine, 1);
    const long long v = odd ? other + mine * 65536 : mine + other * 65536, w = by ? (v + (1ll << (by - 1))) >> by : v;
    const int low = (int)(w & 0xffff);                         // digits 0 and 1, what is left for 2 and 3
    const long long high = w >> 16;
    c[k] = odd ? (int)(high & 0xff) : low & 0xff;
    c[k + 1] = odd ? (int)(high >> 8) : low >> 8;
  }
}

template <int NT, bool ZP>
__global__ void __launch_bounds__(down_threads(NT), 1) down_kernel(const DownArgs a) {
  extern __shared__ __align__(16) uint8_t down_smem[];
  constexpr int kThreads = down_threads(NT), kWarps = kThreads / 32, kStages = down_stages(NT);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, B = a.B;
  __shared__ unsigned hm[kMaxPass];                            // bits of the tokens' largest |h|
  const int S = a.S, rank = blockIdx.x % S, slice = blockIdx.x / S;
  const int WC = a.WC, WR = kWarps / WC, wc = warp % WC, wr = warp / WC;
  const int cg = slice * WC + wc;                              // the warp's group of 128 columns
  const bool active = cg * 128 < a.D;
  const int stage = down_stage(B);
  uint8_t* mine = down_smem + warp * (kStages * stage);
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  if (tid < kMaxPass) hm[tid] = 0;
  __syncthreads();
  // Up to dep_wait nothing is read that the gate and up kernel writes.  (What came before that kernel is complete: it has waited
  // for it before it let this one start.)
  int n = a.n;
  if (a.count) n = max(0, min(n, *a.count));
  const int tiles = (n + 31) / 32;
  const int b0 = (int)((long long)tiles * rank / S), b1 = (int)((long long)tiles * (rank + 1) / S), end = active ? b1 : b0;
  const int gi = cg * a.gstep;
  const long long all = (long long)a.F * a.groups;

  // id of entry `lane` of a tile, as it is in the list; entries behind the list repeat its last one (their h is not used)
  auto fetch = [&](int tile) { return tile < end ? a.list[min(tile * 32 + lane, n - 1)] : 0; };
  auto issue = [&](int tile, int slot, int id) {
    if (tile < end) {
      if ((unsigned)id >= (unsigned)a.F) id = 0;
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
  int token[NT], power[NT][2];                                 // fixed point of tokens 2 i and 2 i + 1: 2^hexp h s times 2^power
  float hscale[NT];                                            // 2^hexp of the lane's tokens
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    token[i] = min(i * 2 + (g >> 2), B - 1);                   // columns behind the last token: computed, never used
    hscale[i] = pow2(unit_exponent(hm[token[i]]));
    power[i][0] = power[i][1] = kMaxPower;                     // (sums of nothing)
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
    float x0[NT], x1[NT];                                      // h s as fixed-point numbers
    auto factor = [&](int i) { return pow2(g < 4 ? power[i][0] : power[i][1]); };
    auto two_h = [&](int i) { return *reinterpret_cast<const float2*>(st + 2432 + token[i] * 128 + t * 32 + r0 * 4); };
    float sum = 0.f;                                           // of magnitudes: whether there is room for all, and all are numbers
    const float s0_in = in0 ? s0 : 0.f, s1_in = in1 ? s1 : 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float2 h = two_h(i);
      x0[i] = h.x * hscale[i] * s0_in * factor(i);
      x1[i] = h.y * hscale[i] * s1_in * factor(i);
      sum += fabsf(x0[i]);
      sum += fabsf(x1[i]);
    }
    if (__any_sync(0xffffffffu, !(sum < 1073741824.f))) {      // the first tile, seldom another
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const float2 h = two_h(i);                             // (0 where the token does not keep the channel: nothing, whatever the scale)
        x0[i] = in0 && h.x != 0.f ? h.x * hscale[i] * s0 : 0.f;
        x1[i] = in1 && h.y != 0.f ? h.y * hscale[i] * s1 : 0.f;
        // the largest |h s| and |h| of the token's 16 lanes, of the other token's
        uint32_t most = max(__float_as_uint(x0[i]) & 0x7fffffffu, __float_as_uint(x1[i]) & 0x7fffffffu);
        uint32_t top = max(in0 ? __float_as_uint(h.x) & 0x7fffffffu : 0u, in1 ? __float_as_uint(h.y) & 0x7fffffffu : 0u);
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
          most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        }
        const uint32_t most_b = __shfl_xor_sync(0xffffffffu, most, 16), top_b = __shfl_xor_sync(0xffffffffu, top, 16);
        int by[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const bool same = (b == 0) == (g < 4);
          const int need = fixed_exponent(same ? most : most_b) + 4;   // below 2^30 (11 at least; -99 for what is not finite)
          const int room = max(2, min(2 + (int)(hm[min(2 * i + b, B - 1)] >> 23) - (int)((same ? top : top_b) >> 23), kMaxRoom));
          by[b] = need < power[i][b] ? power[i][b] - need + room : 0;
          power[i][b] -= by[b];
        }
        x0[i] *= factor(i);
        x1[i] *= factor(i);
        if (tile != first && (by[0] | by[1])) {                // a lane's sums are columns 2 t, 2 t + 1: of one token
          const int mine = min(t & 2 ? by[1] : by[0], 62);
          shift_sums(zacc[i], mine, t & 1);
#pragma unroll
          for (int m = 0; m < 8; ++m) shift_sums(acc[m][i], mine, t & 1);
        }
      }
    }
    uint32_t bf[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const uint32_t d0 = digits(__float2int_rn(x0[i])), d1 = digits(__float2int_rn(x1[i]));
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
    for (int i = 0; i < NT; ++i) mma(zacc[i], zacc[i], zr[0], zr[0], zr[1], zr[1], bf[i][0], bf[i][1]);
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
        for (int i = 0; i < NT; ++i) mma(acc[hw * 4 + m][i], acc[hw * 4 + m][i], a0, a1, a2, a3, bf[i][0], bf[i][1]);
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
    const unsigned most = hm[min(b, B - 1)];
    const int fixed = t & 2 ? power[i][1] : power[i][0], e = -fixed - unit_exponent(most), e0 = max(-126, min(126, e));
    // (a fixed point below 0: some product was not finite)
    const float f0 = most >= 0x7f800000u || fixed < 0 ? __uint_as_float(0x7fffffffu) : pow2(e0), f1 = pow2(max(-126, min(126, e - e0)));
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
    const float v = cluster_total(red + i, S);
    if (d < a.D) store(a.y, (size_t)b * a.D + d, v, a.y_type);
  }
  cluster_barrier();                                           // nobody leaves while another block reads
}

// ----------------------------------------------------------------------------
// Packer: symmetric codes of bf16 weights, the rule of the proxies (scale = fp16(max|w| / 7), round to nearest even).  A
// warp per group, offline: 28672 x 8192 with groups of 128 takes 480 us, 1.2 TB/s (two dependent passes over so few weights and
// one division each bound it); groups of 32, 1.5 ms.
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
