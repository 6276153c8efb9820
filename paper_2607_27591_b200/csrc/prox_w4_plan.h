// Shapes of the kernel that multiplies rows in 4 bits by tokens (rows_kernel): sizes of what a block keeps in shared memory, and the
// choice of a launch.  No CUDA in here: it compiles as plain C++ too.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#ifdef __CUDACC__
#define PROX_HD __host__ __device__
#else
#define PROX_HD
#endif

namespace prox {
namespace w4 {

constexpr int kMaxSmem = 227 * 1024 - 8192;   // dynamic; the kernels have up to 8 KB of their own

constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kBatch = 2;                // chunks that a warp asks for at a time: a 128-byte line of each of 16 rows
constexpr int kMaxStages = 5;            // batches of a warp in shared memory, at most (sid has room for them)
constexpr int kMaxPass = 8;              // tokens of a pass over the weights: 32 columns of digits

// A warp's stage: a batch of its 16 rows (codes with a gap behind every row, so that lanes of one load do not meet), their scales
// and zero points (with room for where an element lies in its word).
template <int W>
struct Stage {
  static constexpr int kGroups = kBatch * 4 / W;
  static constexpr int kPitch = kBatch * 64 + 16 * W;
  static constexpr int kScales = W == 4 ? 8 : W == 2 ? 16 : 32;         // bytes of a row
  static constexpr int kZeros = W == 1 ? 16 : 8;
  static constexpr int kAtScales = 16 * kPitch, kAtZeros = kAtScales + 16 * kScales, kBytes = kAtZeros + 16 * kZeros;
};
PROX_HD constexpr int rows_stage_bytes(int words) { return words == 4 ? Stage<4>::kBytes : words == 2 ? Stage<2>::kBytes : Stage<1>::kBytes; }

// Chunks of a block of a cluster, of a warp along the columns: whole batches
PROX_HD constexpr int rows_share(int C, int S) { return S == 1 ? C : ((C + S - 1) / S + kBatch - 1) / kBatch * kBatch; }
PROX_HD constexpr int rows_run(int Cs, int WK) { return ((Cs + WK - 1) / WK + kBatch - 1) / kBatch * kBatch; }

// Shared memory behind the tokens' digits: what comes off a group's sums, the warps' stages, their partial tiles, the block's sums
PROX_HD constexpr size_t rows_digit_bytes(int chunks, int nt) { return (size_t)chunks * 1024 * nt; }
PROX_HD constexpr size_t rows_fixed_bytes(int chunks, int nt, int words) {
  return rows_digit_bytes(chunks, nt) + (size_t)chunks * (4 / words) * 64 * nt;
}
PROX_HD constexpr size_t rows_red_bytes(int nt) { return (size_t)2 * kRowWarps * nt * 512; }   // only where WK > 1

// Shape of a launch of rows_kernel for `tiles` tiles of 16 rows.  grid 0: there is none.
struct RowsPlan { int S, WM, WK, stages, R, grid; size_t smem; };

// The shape that is done first, in cycles: an SM takes about 48 for 128 columns of a tile when all its warps are busy (18
// more for every 8 further columns of digits), a warp alone 400 (150 more); the end of a unit costs 1500, much less where no warp waits for
// another, the cluster's sum 5000; a token's digits are made at 4 inputs a cycle.
// clusters(S): how many clusters of S blocks the GPU holds at once.
template <typename Clusters>
RowsPlan plan_rows(int tiles, int K, int B, int words, int nt, int sms, Clusters clusters) {
  const int C = (K + 127) / 128;
  RowsPlan best = {};
  double least = 1e30;
  for (int S = 1; S <= 8; S *= 2) {
    const int Cs = rows_share(C, S);
    const int at_once = S == 1 ? sms : std::min(sms / S, clusters(S));
    if (S > 1 && Cs * (S - 1) >= C) break;                   // a block without columns
    for (int WK = 1; WK <= kRowWarps && WK <= 2 * Cs - 1; WK *= 2)
      for (int WM = kRowWarps / WK; WM >= 1; WM /= 2)
        for (int stages : {kMaxStages, 3, 2}) {
          const size_t sum = S > 1 ? (size_t)WM * 64 * B : 0;  // a unit's sums, kept for the cluster
          const size_t fixed = rows_fixed_bytes(Cs, nt, words) + (WK > 1 ? rows_red_bytes(nt) : 0) +
                               (size_t)kRowWarps * stages * rows_stage_bytes(words);
          if (fixed + sum > (size_t)kMaxSmem) continue;
          const int held = std::max(1, std::min(tiles, at_once)), most = (tiles + held - 1) / held, mine = (most + WM - 1) / WM;
          const int R = S > 1 ? (int)std::min<size_t>(std::min(mine, 16), (kMaxSmem - fixed) / sum) : 0;
          const double cost = std::max((double)most * Cs * (30 + 18 * nt), (double)mine * rows_run(Cs, WK) * (250 + 150 * nt)) * (1.0 + 0.3 / stages) +
                              mine * (WK == 1 ? 300.0 : 1500.0) + (S > 1 ? 5000.0 * ((mine + R - 1) / R) : 0.0) + Cs * 32.0 * B;
          if (cost < least - 1e-9) {
            least = cost;
            best = {S, WM, WK, stages, R, held * S, fixed + R * sum};
          }
          break;                                               // (the most stages that fit)
        }
  }
  return best;
}

// Tokens of a pass over the weights of a projection of B tokens: as many as leave a block of a cluster of eight room for two stages
// of 16 tiles and their sums, and as there is a shape for.  (Rows of groups of 32 inputs, too long for four blocks and leaving
// the last of eight without columns, have none for 7 or 8 tokens.)  Fewer tokens need less of everything, so the last pass
// has a shape too.  plan(tokens): their shape.
template <typename Plan>
int linear_pass(int B, int K, int words, Plan plan) {
  const int Cs = rows_share((K + 127) / 128, 8);
  int per = kMaxPass;
  while (per > 1 && rows_fixed_bytes(Cs, (per + 1) / 2, words) + 32 * rows_stage_bytes(words) + 16 * 64 * per > (size_t)kMaxSmem) --per;
  per = std::min(per, B);
  while (per > 0 && !plan(per).grid) --per;
  return per;
}

}  // namespace w4
}  // namespace prox
