// Host side of prox_token_logprobs.  See include/prox.h for the contract.
#include "prox_host.h"
#include "prox_logprobs.cuh"

using namespace prox;

namespace {

template <int DT>
cudaError_t launch_logprobs(const lp::Args& a, unsigned grid, int dev, cudaStream_t st) {
  return a.k ? host_launch<lp::logprobs_kernel<DT, true>>(dev, grid, lp::kThreads, 0, a.S, st, a)
             : host_launch<lp::logprobs_kernel<DT, false>>(dev, grid, lp::kThreads, 0, a.S, st, a);
}

}  // namespace

cudaError_t prox::host_load_logprobs() {
  return host_load<lp::logprobs_kernel<lp::kBf16, false>, lp::logprobs_kernel<lp::kBf16, true>, lp::logprobs_kernel<lp::kFp16, false>,
                   lp::logprobs_kernel<lp::kFp16, true>, lp::logprobs_kernel<lp::kFp32, false>, lp::logprobs_kernel<lp::kFp32, true>>();
}

extern "C" prox_status_t prox_token_logprobs(const void* logits_dev, int dtype, int T, int V, int64_t row_stride, float temperature,
                                             const int32_t* given_dev, int n_given, float* logprob_dev, float* entropy_dev_or_null,
                                             int n_top, float* top_logprob_dev, int32_t* top_index_dev, void* stream) {
  if (!logits_dev || T < 1 || V < 1 || n_given < 0 || n_top < 0 || n_top > V || dtype < 0 || dtype > 2) return PROX_ERR_INVALID_ARG;
  if (T > 1 && row_stride < V) return PROX_ERR_INVALID_ARG;
  if (!(temperature >= 1e-30f) || !(temperature <= 1e30f)) return PROX_ERR_INVALID_ARG;
  if (n_given && (!given_dev || !logprob_dev)) return PROX_ERR_INVALID_ARG;
  if (n_top && (!top_logprob_dev || !top_index_dev)) return PROX_ERR_INVALID_ARG;
  if (!n_given && !n_top && !entropy_dev_or_null) return PROX_ERR_INVALID_ARG;
  const int size = dtype == lp::kFp32 ? 4 : 2;
  if (!host_aligned(logits_dev, size) || !host_aligned(given_dev, 4) || !host_aligned(logprob_dev, 4) || !host_aligned(entropy_dev_or_null, 4) ||
      !host_aligned(top_logprob_dev, 4) || !host_aligned(top_index_dev, 4))
    return PROX_ERR_INVALID_ARG;
  if (n_top > lp::kMaxTop || V > 0x7fff0000) return PROX_ERR_UNSUPPORTED;
  int dev;
  if (const cudaError_t e = cudaGetDevice(&dev)) return host_map_cuda(e);
  if (!host_on_current_device(logits_dev, dev) || (n_given && (!host_on_current_device(given_dev, dev) || !host_on_current_device(logprob_dev, dev))) ||
      (entropy_dev_or_null && !host_on_current_device(entropy_dev_or_null, dev)) ||
      (n_top && (!host_on_current_device(top_logprob_dev, dev) || !host_on_current_device(top_index_dev, dev))))
    return PROX_ERR_INVALID_ARG;
  lp::Args a = {};
  a.x = static_cast<const uint8_t*>(logits_dev);
  a.row_bytes = (long long)row_stride * size;
  a.V = V;
  a.inv_temperature = 1.0f / temperature;
  a.given = given_dev; a.n_given = n_given; a.logprob = logprob_dev; a.entropy = entropy_dev_or_null;
  a.k = n_top; a.top_logprob = top_logprob_dev; a.top_index = top_index_dev;
  // blocks of a row: more while the rows do not fill the GPU and every thread still has a vector
  const int sms = host_sm_count(dev), vectors = V / (16 / size);
  a.S = 1;
  while (a.S < lp::kMaxCluster && (long long)T * a.S < sms && vectors / (2 * a.S) >= lp::kThreads) a.S *= 2;
  if ((long long)T * a.S > 0x7fffffffLL) return PROX_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)(T * a.S);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == lp::kBf16 ? launch_logprobs<lp::kBf16>(a, grid, dev, st)
                        : dtype == lp::kFp16 ? launch_logprobs<lp::kFp16>(a, grid, dev, st)
                                             : launch_logprobs<lp::kFp32>(a, grid, dev, st);
  return e == cudaSuccess ? PROX_OK : host_map_cuda(e);
}
