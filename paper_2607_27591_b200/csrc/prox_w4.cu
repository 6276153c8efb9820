// Host side of the calls over weights held in 4 bits.  See include/prox.h for the contract.
#include "prox_host.h"
#include "prox_w4.cuh"

#include <algorithm>

using namespace prox;

namespace {

constexpr int kMaxSmem = 227 * 1024;
constexpr int kMaxTokens = 16;           // tokens of one pass over the weights of prox_w4_linear
constexpr int kFfnTokens = 8;            // tokens of a call of the sparse FFN, as everywhere in the library

template <typename... KArgs>
cudaError_t launch(void (*kern)(KArgs...), int grid, int block, size_t smem, int cluster, cudaStream_t st, KArgs... args) {
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kern), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

// Shape of a launch of rows_kernel for `tiles` tiles of 16 rows.
struct RowsPlan { int S, WM, WK, R, grid; size_t smem; };

int floor_pow2(int v) { int p = 1; while (2 * p <= v) p *= 2; return p; }

RowsPlan plan_rows(int tiles, int K, int B, int nt, int sms) {
  RowsPlan p;
  const int C = (K + 127) / 128;
  auto fixed = [&](int R, int WM) { return (size_t)2 * w4::kRowWarps * nt * 512 + (size_t)R * WM * 64 * B; };
  // the tokens have to fit; then columns are split over a cluster while that brings more SMs in
  int S = 1;
  while (S < 8 && (size_t)((C + S - 1) / S) * 256 * B + fixed(4, 16) > (size_t)kMaxSmem) S *= 2;
  while (S < 8 && tiles * S * 2 <= sms && C >= 2 * S) S *= 2;
  const int Cs = (C + S - 1) / S;
  p.S = S;
  p.WK = std::min(w4::kRowWarps, floor_pow2(Cs));
  p.WM = w4::kRowWarps / p.WK;
  while (p.WM > 1 && ((tiles + p.WM - 1) / p.WM) * S < sms) p.WM /= 2;
  const int units = (tiles + p.WM - 1) / p.WM, clusters = std::max(1, std::min(units, sms / S));
  p.grid = clusters * S;
  const int mine = (units + clusters - 1) / clusters;
  p.R = 1;
  if (S > 1)
    while (p.R < mine && (size_t)Cs * 256 * B + fixed(p.R + 1, p.WM) <= (size_t)kMaxSmem && p.R < 16) ++p.R;
  p.smem = (size_t)Cs * 256 * B + fixed(S > 1 ? p.R : 0, p.WM);
  return p;
}

template <int XT, int W, bool ZP>
cudaError_t launch_linear(const w4::RowsArgs& a, int nt, const RowsPlan& p, cudaStream_t st) {
  return nt == 1 ? launch(w4::rows_kernel<XT, W, 1, ZP, false>, p.grid, w4::kRowThreads, p.smem, p.S, st, a)
                 : launch(w4::rows_kernel<XT, W, 2, ZP, false>, p.grid, w4::kRowThreads, p.smem, p.S, st, a);
}

template <int XT>
cudaError_t launch_linear(const w4::RowsArgs& a, int words, int nt, const RowsPlan& p, cudaStream_t st) {
  if (a.w.zeros)
    return words == 4 ? launch_linear<XT, 4, true>(a, nt, p, st) : words == 2 ? launch_linear<XT, 2, true>(a, nt, p, st)
                                                                              : launch_linear<XT, 1, true>(a, nt, p, st);
  return words == 4 ? launch_linear<XT, 4, false>(a, nt, p, st) : words == 2 ? launch_linear<XT, 2, false>(a, nt, p, st)
                                                                             : launch_linear<XT, 1, false>(a, nt, p, st);
}

bool group_known(int g) { return g == 0 || g == 32 || g == 64 || g == 128; }
int groups_of(int cols, int g) { return g ? (cols + g - 1) / g : 1; }

prox_status_t current_device(int* dev) {
  const cudaError_t e = cudaGetDevice(dev);
  return e == cudaSuccess ? PROX_OK : host_map_cuda(e);
}

bool mat_ok(const prox_w4_t* w, int dev) {
  return w && w->codes && w->scales && host_aligned(w->codes, 16) && host_aligned(w->scales, 2) && host_on_current_device(w->codes, dev) &&
         host_on_current_device(w->scales, dev) && (!w->zeros || host_on_current_device(w->zeros, dev));
}

w4::Mat mat_of(const prox_w4_t* w) { return {w->codes, static_cast<const __half*>(w->scales), w->zeros}; }

struct FfnWorkspace { size_t list, members, count, h, bytes; };

// [union list | token bits of its entries | its length | h]; one token needs h alone
FfnWorkspace ffn_workspace(int F, int B) {
  FfnWorkspace w = {};
  const size_t f = ((size_t)F + 15) / 16 * 16;
  if (B > 1) { w.members = f * 4; w.count = w.members + f; w.h = w.count + 16; }
  w.bytes = w.h + f * 4 * B;
  return w;
}

template <bool ZP>
cudaError_t launch_down(const w4::DownArgs& a, int nt, int grid, cudaStream_t st) {
  const size_t smem = (size_t)w4::kDownWarps * 128 * nt * 8 * 4 + (size_t)128 * a.B * 4;
  return nt == 1 ? launch(w4::down_kernel<1, ZP>, grid, w4::kDownThreads, smem, a.S, st, a)
         : nt == 2 ? launch(w4::down_kernel<2, ZP>, grid, w4::kDownThreads, smem, a.S, st, a)
                   : launch(w4::down_kernel<3, ZP>, grid, w4::kDownThreads, smem, a.S, st, a);
}

}  // namespace

#define CKL(expr)                                        \
  do {                                                   \
    cudaError_t e_ = (expr);                             \
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
  if (!group_known(group_size) || K % 32 || K > 65536) return PROX_ERR_UNSUPPORTED;
  int dev;
  if (prox_status_t s = current_device(&dev)) return s;
  if (!mat_ok(w, dev) || !host_on_current_device(x_dev, dev) || !host_on_current_device(y_dev, dev)) return PROX_ERR_INVALID_ARG;
  const int sms = host_sm_count(dev);
  w4::RowsArgs a = {};
  a.w = a.w2 = mat_of(w);
  a.rows = N; a.K = K; a.groups = groups_of(K, group_size); a.gstep = group_size != 0;
  a.x_stride = x_stride; a.y_stride = y_stride; a.y_type = y_dtype;
  a.x_vec = host_aligned(x_dev, 16) && (B == 1 || x_stride % 8 == 0);
  const size_t ysize = y_dtype == w4::kFp32 ? 4 : 2;
  // as many tokens a pass as fit in the shared memory of a cluster
  const int C = (K + 127) / 128, fit = (int)((size_t)(kMaxSmem - 100 * 1024) / ((size_t)(C + 7) / 8 * 256));
  const int per = std::max(1, std::min(kMaxTokens, fit));
  for (int b = 0; b < B; b += per) {
    a.B = std::min(per, B - b);
    a.x = static_cast<const uint16_t*>(x_dev) + (size_t)b * x_stride;
    a.y = static_cast<uint8_t*>(y_dev) + (size_t)b * y_stride * ysize;
    const int nt = a.B > 8 ? 2 : 1;
    const RowsPlan p = plan_rows((N + 15) / 16, K, a.B, nt, sms);
    a.S = p.S; a.WM = p.WM; a.WK = p.WK; a.R = p.R;
    const int words = group_size == 32 ? 1 : group_size == 64 ? 2 : 4;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CKL(x_dtype == w4::kBf16 ? launch_linear<w4::kBf16>(a, words, nt, p, st) : launch_linear<w4::kFp16>(a, words, nt, p, st));
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
  const int h_stride = (F + 15) / 16 * 16;
  const int* list = sel_dev;
  const int* count = count_dev_or_null;
  const uint8_t* members = nullptr;
  int most = k2;                            // channels that some token keeps, at most
  if (B > 1) {
    int* ulist = reinterpret_cast<int*>(wsp + ws.list);
    int* ucount = reinterpret_cast<int*>(wsp + ws.count);
    CKL(launch(w4::union_kernel, 1, w4::kUnionThreads, (size_t)(F + 3) / 4 * 4, 1, st, sel_dev, sel_stride, count_dev_or_null, k2, B, F, ulist,
               wsp + ws.members, ucount));
    list = ulist; count = ucount; members = wsp + ws.members;
    most = (int)std::min<long long>(F, (long long)B * k2);
  }
  const int groups = groups_of(D, group_size);
  if (most > 0) {
    w4::RowsArgs a = {};
    a.w = mat_of(gate); a.w2 = mat_of(up);
    a.rows = F; a.K = D; a.groups = groups; a.gstep = group_size != 0;
    a.x = static_cast<const uint16_t*>(x_dev); a.x_stride = D; a.B = B; a.x_vec = 1;
    a.list = list; a.count = count; a.n = most; a.members = members; a.h = h; a.h_stride = h_stride;
    const RowsPlan p = plan_rows((most + 7) / 8, D, B, 1, sms);
    a.S = p.S; a.WM = p.WM; a.WK = p.WK; a.R = p.R;
    CKL(gate->zeros ? launch(w4::rows_kernel<w4::kBf16, 4, 1, true, true>, p.grid, w4::kRowThreads, p.smem, p.S, st, a)
                    : launch(w4::rows_kernel<w4::kBf16, 4, 1, false, true>, p.grid, w4::kRowThreads, p.smem, p.S, st, a));
  }
  w4::DownArgs d = {};
  d.w = mat_of(down_t);
  d.D = D; d.F = F; d.groups = groups; d.gstep = group_size != 0;
  d.list = list; d.count = count; d.n = most; d.h = h; d.h_stride = h_stride; d.B = B; d.y = y_dev; d.y_type = out_dtype;
  const int cgs = D / 128;
  d.S = 8;
  while (d.S > 1 && cgs * d.S > 2 * sms) d.S /= 2;
  const int nt = (3 * B + 7) / 8;
  CKL(down_t->zeros ? launch_down<true>(d, nt, cgs * d.S, st) : launch_down<false>(d, nt, cgs * d.S, st));
  return PROX_OK;
}

}  // extern "C"
