// Host side of the calls over weights held in 4 bits.  See include/prox.h for the contract.
#include "prox_host.h"
#include "prox_w4.cuh"

#include <algorithm>
#include <atomic>

using namespace prox;

namespace {

using w4::kMaxSmem;
static_assert(kMaxSmem == kMaxBlockSmem - 8192, "what host_allow_smem asks for");
constexpr int kMaxRowBlocks = 256;       // of the gate and up kernel
constexpr int kFfnTokens = 8;            // tokens of a call of the sparse FFN, as everywhere in the library

// Clusters of S blocks that the GPU holds at once (a block of these kernels has an SM to itself).
template <auto Kern>
int clusters_at_once(int device, int S, int threads, size_t smem) {
  static std::atomic<int> known[kKnownDevices][9];
  std::atomic<int>* kept = device < kKnownDevices ? &known[device][S] : nullptr;
  int n = kept ? kept->load(std::memory_order_relaxed) : 0;
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(S); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = S; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  if (host_allow_smem<Kern>(device) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, Kern, &cfg) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    n = std::max(1, 128 / S);
  }
  if (kept) kept->store(n, std::memory_order_relaxed);
  return n;
}

w4::RowsPlan plan_rows(int tiles, int K, int B, int words, int sms, int dev) {
  return w4::plan_rows(tiles, K, B, words, (B + 1) / 2, sms, [dev](int S) {
    return clusters_at_once<w4::rows_kernel<4, 1, false, false>>(dev, S, w4::kRowThreads, 120 * 1024);
  });
}

template <int W, bool ZP, bool GATEUP>
cudaError_t launch_rows(const w4::RowsArgs& a, int nt, const w4::RowsPlan& p, int dev, cudaStream_t st) {
  switch (nt) {
    case 1: return host_launch<w4::rows_kernel<W, 1, ZP, GATEUP>>(dev, p.grid, w4::kRowThreads, p.smem, p.S, st, a);
    case 2: return host_launch<w4::rows_kernel<W, 2, ZP, GATEUP>>(dev, p.grid, w4::kRowThreads, p.smem, p.S, st, a);
    case 3: return host_launch<w4::rows_kernel<W, 3, ZP, GATEUP>>(dev, p.grid, w4::kRowThreads, p.smem, p.S, st, a);
    default: return host_launch<w4::rows_kernel<W, 4, ZP, GATEUP>>(dev, p.grid, w4::kRowThreads, p.smem, p.S, st, a);
  }
}

template <int W>
cudaError_t launch_linear(const w4::RowsArgs& a, int nt, const w4::RowsPlan& p, int dev, cudaStream_t st) {
  return a.w.zeros ? launch_rows<W, true, false>(a, nt, p, dev, st) : launch_rows<W, false, false>(a, nt, p, dev, st);
}

bool group_known(int g) { return g == 0 || g == 32 || g == 64 || g == 128; }
int groups_of(int cols, int g) { return g ? (cols + g - 1) / g : 1; }

prox_status_t current_device(int* dev) {
  const cudaError_t e = cudaGetDevice(dev);
  return e == cudaSuccess ? PROX_OK : host_map_cuda(e);
}

bool mat_ok(const prox_w4_t* w, int dev) {
  return w && w->codes && w->scales && host_aligned(w->codes, 16) && host_aligned(w->scales, 16) && host_aligned(w->zeros, 16) && host_on_current_device(w->codes, dev) &&
         host_on_current_device(w->scales, dev) && (!w->zeros || host_on_current_device(w->zeros, dev));
}

w4::Mat mat_of(const prox_w4_t* w) { return {w->codes, static_cast<const __half*>(w->scales), w->zeros}; }

struct FfnWorkspace { size_t list, members, count, hmax, h, bytes; };

// [union list | token bits of its entries | its length | largest |h| | h]; one token has no union
FfnWorkspace ffn_workspace(int F, int B) {
  FfnWorkspace w = {};
  const size_t f = ((size_t)F + 31) / 32 * 32;
  if (B > 1) { w.members = f * 4; w.count = w.members + f; w.hmax = w.count + 16; }
  w.h = w.hmax + (size_t)kMaxRowBlocks * B * 4;
  w.bytes = w.h + f * 4 * B;
  return w;
}

template <int NT, bool ZP>
cudaError_t launch_down(w4::DownArgs& a, int sms, int dev, cudaStream_t st) {
  constexpr int kThreads = w4::down_threads(NT), kWarps = kThreads / 32;
  constexpr auto kern = w4::down_kernel<NT, ZP>;
  const int cgs = a.D / 128, tiles = std::max(1, (a.n + 31) / 32);
  const size_t smem = std::max((size_t)kWarps * w4::down_stages(NT) * w4::down_stage(a.B), (size_t)kWarps * 512 * a.B);
  // the shape with the fewest rounds of a tile for every warp; a cluster's sum counts as one
  double least = 1e30;
  for (int S = 8; S >= 1; S /= 2)
    for (int WC = 8; WC >= 1; WC /= 2) {
      const int slices = (cgs + WC - 1) / WC, at_once = S == 1 ? sms : clusters_at_once<kern>(dev, S, kThreads, smem);
      const int waves = (slices + at_once - 1) / at_once, rounds = ((tiles + S - 1) / S + kWarps / WC - 1) / (kWarps / WC);
      if (tiles > 1024 * S) continue;                          // (32768 entries a block: its sums stay below 2^31)
      const double cost = waves * (rounds + 2.0) + (S > 1 ? 1.0 : 0.0) - 0.01 * WC;
      if (cost < least) { least = cost; a.S = S; a.WC = WC; }
    }
  return host_launch<kern>(dev, (cgs + a.WC - 1) / a.WC * a.S, kThreads, smem, a.S, st, a);
}

template <int NT>
cudaError_t launch_down(w4::DownArgs& a, int sms, int dev, cudaStream_t st) {
  return a.w.zeros ? launch_down<NT, true>(a, sms, dev, st) : launch_down<NT, false>(a, sms, dev, st);
}

template <int W, bool ZP, bool GATEUP>
cudaError_t load_rows() {
  return host_load<w4::rows_kernel<W, 1, ZP, GATEUP>, w4::rows_kernel<W, 2, ZP, GATEUP>, w4::rows_kernel<W, 3, ZP, GATEUP>,
                   w4::rows_kernel<W, 4, ZP, GATEUP>>();
}

template <bool ZP>
cudaError_t load_zero_points() {   // kernels of matrices with zero points, or without
  for (cudaError_t (*load)() : {load_rows<1, ZP, false>, load_rows<2, ZP, false>, load_rows<4, ZP, false>, load_rows<4, ZP, true>})
    if (const cudaError_t e = load()) return e;
  return host_load<w4::down_kernel<1, ZP>, w4::down_kernel<2, ZP>, w4::down_kernel<3, ZP>, w4::down_kernel<4, ZP>>();
}

}  // namespace

cudaError_t prox::host_load_w4() {
  if (const cudaError_t e = load_zero_points<false>()) return e;
  if (const cudaError_t e = load_zero_points<true>()) return e;
  return host_load<w4::union_kernel, w4::quantize_kernel>();
}

#define CKL(...)                                        \
  do {                                                   \
    cudaError_t e_ = (__VA_ARGS__);                        \
    if (e_ != cudaSuccess) return host_map_cuda(e_);     \
  } while (0)

extern "C" {

prox_status_t prox_w4_quantize(const void* w_dev, int rows, int cols, int group_size, uint8_t* codes_dev, void* scales_dev, void* stream) {
  if (!w_dev || !codes_dev || !scales_dev || rows < 1 || cols < 1) return PROX_ERR_INVALID_ARG;
  if (!host_aligned(w_dev, 4) || !host_aligned(scales_dev, 2)) return PROX_ERR_INVALID_ARG;
  if (!group_known(group_size) || cols % 32) return PROX_ERR_UNSUPPORTED;
  int dev;
  if (prox_status_t s = current_device(&dev)) return s;
  if (!host_on_current_device(w_dev, dev) || !host_on_current_device(codes_dev, dev) || !host_on_current_device(scales_dev, dev))
    return PROX_ERR_INVALID_ARG;
  const int groups = groups_of(cols, group_size);
  const long long blocks = ((long long)rows * groups + 7) / 8;
  if (blocks > 0x7fffffffLL) return PROX_ERR_UNSUPPORTED;
  w4::quantize_kernel<<<(unsigned)blocks, 256, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint32_t*>(w_dev), rows, cols, group_size ? group_size : cols, groups, codes_dev, static_cast<__half*>(scales_dev));
  CKL(cudaGetLastError());
  return PROX_OK;
}

prox_status_t prox_w4_linear(const prox_w4_t* w, int N, int K, int group_size, const void* x_dev, int64_t x_stride, int x_dtype, int B,
                             void* y_dev, int64_t y_stride, int y_dtype, void* stream) {
  if (!w || !x_dev || !y_dev || N < 1 || K < 1 || B < 1) return PROX_ERR_INVALID_ARG;
  if ((x_dtype != w4::kBf16 && x_dtype != w4::kFp16) || y_dtype < 0 || y_dtype > 2) return PROX_ERR_INVALID_ARG;
  if (!host_aligned(x_dev, 2) || !host_aligned(y_dev, y_dtype == w4::kFp32 ? 4 : 2)) return PROX_ERR_INVALID_ARG;
  if (B > 1 && (x_stride < K || y_stride < N)) return PROX_ERR_INVALID_ARG;
  if (!group_known(group_size) || K % 32 || K > 65536 || N > 0x7fff0000) return PROX_ERR_UNSUPPORTED;
  int dev;
  if (prox_status_t s = current_device(&dev)) return s;
  if (!mat_ok(w, dev) || !host_on_current_device(x_dev, dev) || !host_on_current_device(y_dev, dev)) return PROX_ERR_INVALID_ARG;
  const int sms = host_sm_count(dev);
  w4::RowsArgs a = {};
  a.w = a.w2 = mat_of(w);
  a.rows = N; a.K = K; a.groups = groups_of(K, group_size); a.gstep = group_size != 0;
  a.x_stride = x_stride; a.y_stride = y_stride; a.y_type = y_dtype;
  a.x_half = x_dtype == w4::kFp16;
  a.x_vec = host_aligned(x_dev, 16) && (B == 1 || x_stride % 8 == 0);
  const size_t ysize = y_dtype == w4::kFp32 ? 4 : 2;
  const int words = group_size == 32 ? 1 : group_size == 64 ? 2 : 4;
  auto plan = [&](int tokens) { return plan_rows((N + 15) / 16, K, tokens, words, sms, dev); };
  const int per = w4::linear_pass(B, K, words, plan);
  if (per < 1) return PROX_ERR_UNSUPPORTED;                // before anything is written
  for (int b = 0; b < B; b += per) {
    a.B = std::min(per, B - b);
    a.x = static_cast<const uint16_t*>(x_dev) + (size_t)b * x_stride;
    a.y = static_cast<uint8_t*>(y_dev) + (size_t)b * y_stride * ysize;
    const int nt = (a.B + 1) / 2;
    const w4::RowsPlan p = plan(a.B);
    a.S = p.S; a.WM = p.WM; a.WK = p.WK; a.stages = p.stages; a.R = p.R;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CKL(words == 4 ? launch_linear<4>(a, nt, p, dev, st) : words == 2 ? launch_linear<2>(a, nt, p, dev, st) : launch_linear<1>(a, nt, p, dev, st));
  }
  return PROX_OK;
}

prox_status_t prox_w4_stage2_workspace(int d_model, int d_ff, int B, int64_t* bytes) {
  if (!bytes || d_model < 1 || d_ff < 1 || B < 1 || B > kFfnTokens) return PROX_ERR_INVALID_ARG;
  if (d_model % 128 || d_model > 16384 || d_ff > 65536) return PROX_ERR_UNSUPPORTED;
  *bytes = (int64_t)ffn_workspace(d_ff, B).bytes;
  return PROX_OK;
}

prox_status_t prox_w4_stage2_ffn(const prox_w4_t* gate, const prox_w4_t* up, const prox_w4_t* down_t, int d_model, int d_ff, int group_size,
                                 const void* x_dev, int B, const int32_t* sel_dev, int sel_stride, const int32_t* count_dev_or_null, int k2,
                                 void* y_dev, int out_dtype, void* workspace_dev, int64_t workspace_bytes, void* stream) {
  const int D = d_model, F = d_ff;
  if (!gate || !up || !down_t || !x_dev || !sel_dev || !y_dev || !workspace_dev) return PROX_ERR_INVALID_ARG;
  if (B < 1 || B > kFfnTokens || D < 1 || F < 1 || k2 < 0 || k2 > F || (B > 1 && sel_stride < k2)) return PROX_ERR_INVALID_ARG;
  if (out_dtype != w4::kBf16 && out_dtype != w4::kFp32) return PROX_ERR_INVALID_ARG;
  if (!host_aligned(x_dev, 16) || !host_aligned(workspace_dev, 16) || !host_aligned(sel_dev, 4) || !host_aligned(y_dev, out_dtype ? 4 : 2) ||
      !host_aligned(count_dev_or_null, 4))
    return PROX_ERR_INVALID_ARG;
  if (D % 128 || D > 16384 || F > 65536 || (group_size != 0 && group_size != 128)) return PROX_ERR_UNSUPPORTED;
  // one kernel for all three matrices: either all have zero points or none
  if (!gate->zeros != !up->zeros || !gate->zeros != !down_t->zeros) return PROX_ERR_INVALID_ARG;
  const FfnWorkspace ws = ffn_workspace(F, B);
  if (workspace_bytes < (int64_t)ws.bytes) return PROX_ERR_INVALID_ARG;
  int dev;
  if (prox_status_t s = current_device(&dev)) return s;
  if (!mat_ok(gate, dev) || !mat_ok(up, dev) || !mat_ok(down_t, dev) || !host_on_current_device(x_dev, dev) ||
      !host_on_current_device(sel_dev, dev) || !host_on_current_device(y_dev, dev) || !host_on_current_device(workspace_dev, dev) ||
      (count_dev_or_null && !host_on_current_device(count_dev_or_null, dev)))
    return PROX_ERR_INVALID_ARG;
  const int sms = host_sm_count(dev);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* wsp = static_cast<uint8_t*>(workspace_dev);
  float* h = reinterpret_cast<float*>(wsp + ws.h);
  const int* list = sel_dev;
  const int* count = count_dev_or_null;
  const uint8_t* members = nullptr;
  const int most = B > 1 ? (int)std::min<long long>(F, (long long)B * k2) : k2;   // channels that some token keeps, at most
  const w4::RowsPlan p = plan_rows(std::max(1, (most + 7) / 8), D, B, 4, std::min(sms, kMaxRowBlocks), dev);
  if (!p.grid) return PROX_ERR_UNSUPPORTED;                // before anything is written
  if (B > 1) {
    int* ulist = reinterpret_cast<int*>(wsp + ws.list);
    int* ucount = reinterpret_cast<int*>(wsp + ws.count);
    CKL(host_launch<w4::union_kernel>(dev, w4::kUnionBlocks, w4::kUnionThreads, ((size_t)F + 31) / 32 * 4, w4::kUnionBlocks, st, sel_dev, sel_stride, count_dev_or_null, k2, B, F, ulist,
               wsp + ws.members, ucount));
    list = ulist; count = ucount; members = wsp + ws.members;
  }
  const int groups = groups_of(D, group_size);
  w4::RowsArgs a = {};
  a.w = mat_of(gate); a.w2 = mat_of(up);
  a.rows = F; a.K = D; a.groups = groups; a.gstep = group_size != 0;
  a.x = static_cast<const uint16_t*>(x_dev); a.x_stride = D; a.B = B; a.x_vec = 1;
  a.list = list; a.count = count; a.n = most; a.members = members; a.h = h;
  a.hmax = reinterpret_cast<unsigned*>(wsp + ws.hmax);
  const int nt = (B + 1) / 2;
  a.S = p.S; a.WM = p.WM; a.WK = p.WK; a.stages = p.stages; a.R = p.R;
  CKL(gate->zeros ? launch_rows<4, true, true>(a, nt, p, dev, st) : launch_rows<4, false, true>(a, nt, p, dev, st));
  w4::DownArgs d = {};
  d.w = mat_of(down_t);
  d.D = D; d.F = F; d.groups = groups; d.gstep = group_size != 0;
  d.list = list; d.count = count; d.n = most; d.h = h; d.B = B; d.y = y_dev; d.y_type = out_dtype;
  d.hmax = a.hmax; d.hblocks = p.grid;
  CKL(nt == 1 ? launch_down<1>(d, sms, dev, st) : nt == 2 ? launch_down<2>(d, sms, dev, st) : nt == 3 ? launch_down<3>(d, sms, dev, st)
                                                                                                     : launch_down<4>(d, sms, dev, st));
  return PROX_OK;
}

}  // extern "C"
