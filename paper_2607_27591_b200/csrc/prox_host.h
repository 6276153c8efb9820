// What the host sides of the library's translation units share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "prox.h"

cudaError_t prox_noalloc_load(int device);

namespace prox {

// Records a CUDA error for prox_last_cuda_error and gives the status for it (prox_api.cu).
prox_status_t host_map_cuda(cudaError_t e);

inline bool host_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The entry points without a handle have no GPU of their own to check against.  A buffer that lies on another GPU
// than the current one, or in pageable host memory, is refused here: a kernel would fault on it.
inline bool host_on_current_device(const void* p, int device) {
  cudaPointerAttributes at;
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    (void)cudaGetLastError();
    return false;
  }
  if (at.type == cudaMemoryTypeDevice) return at.device == device;
  return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeHost && at.devicePointer == p);
}

// Facts about a device that are asked for once and kept (threads that ask at the same time find the same).
constexpr int kKnownDevices = 64;

inline int host_sm_count(int device) {
  static std::atomic<int> known[kKnownDevices];
  std::atomic<int>* at = device < kKnownDevices ? known + device : nullptr;
  int n = at ? at->load(std::memory_order_relaxed) : 0;
  if (n > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
    (void)cudaGetLastError();
    return 148;
  }
  if (at) at->store(n, std::memory_order_relaxed);
  return n;
}

// Loads the code of kernels on the current device.  (CUDA does so at a kernel's first launch otherwise, and may take device memory
// for it.)
template <auto... Kerns>
cudaError_t host_load() {
  cudaError_t e = cudaSuccess;
  cudaFuncAttributes at;
  ((e = e == cudaSuccess ? cudaFuncGetAttributes(&at, reinterpret_cast<const void*>(Kerns)) : e), ...);
  return e;
}
// ... those of the calls without a handle (prox_w4.cu, prox_logprobs.cu; prox_noalloc.cu: prox_noalloc_load above)
cudaError_t host_load_w4();
cudaError_t host_load_logprobs();

constexpr int kMaxBlockSmem = 227 * 1024;

// Lets a kernel with dynamic shared memory have that of a whole SM (once per device).
template <auto Kern>
cudaError_t host_allow_smem(int device) {
  static std::atomic<bool> allowed[kKnownDevices];
  std::atomic<bool>* at = device < kKnownDevices ? allowed + device : nullptr;
  if (at && at->load(std::memory_order_acquire)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(Kern), cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxBlockSmem - 8192);
  if (e == cudaSuccess && at) at->store(true, std::memory_order_release);
  return e;
}

// A launch that may be set up while its predecessor on the stream still runs (the kernel waits for it before it reads
// anything), of clusters of `cluster` blocks.
template <auto Kern, typename... Args>
cudaError_t host_launch(int device, unsigned grid, int block, size_t smem, int cluster, cudaStream_t st, Args... args) {
  if (smem > 0) {
    if (const cudaError_t e = host_allow_smem<Kern>(device)) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, Kern, args...);
}

}  // namespace prox
