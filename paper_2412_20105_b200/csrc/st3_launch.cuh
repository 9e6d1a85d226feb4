// Host helpers of the context-free entry points; included by the .cu files that launch kernels themselves.
#ifndef ST3_LAUNCH_CUH_
#define ST3_LAUNCH_CUH_
#include "st3.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

namespace {

// A launch that may be set up while the one ahead of it in the stream still runs; the kernel waits for it itself.  Its blocks
// come in clusters of `cluster`, if that is more than one.
template <typename... P, typename... A>
st3_status launch_clusters(int cluster, void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const A&... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? ST3_OK : ST3_ERR_CUDA;
}
template <typename... P, typename... A>
st3_status launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const A&... args) {
  return launch_clusters(1, kernel, grid, block, smem, stream, args...);
}

// Raises a kernel's limit of dynamic shared memory, once on each device (a call costs as much as a fifth of a launch).  Two
// first calls at once set the same value twice.
template <auto kKernel>
bool allow_smem(int bytes) {
  static std::atomic<unsigned long long> devices{0};
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  const bool known = device < 64;
  if (known && (devices.load(std::memory_order_acquire) >> device & 1)) return true;
  if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  if (known) devices.fetch_or(1ull << device, std::memory_order_release);
  return true;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder of tensor maps; null if it does not offer one.  Looked up once (initialisation of a local static is
// thread-safe).
inline EncodeTiledFn tensor_map_encoder() {
  static const EncodeTiledFn encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess)
      fn = nullptr;
    return reinterpret_cast<EncodeTiledFn>(fn);
  }();
  return encode;
}

}  // namespace
#endif  // ST3_LAUNCH_CUH_
