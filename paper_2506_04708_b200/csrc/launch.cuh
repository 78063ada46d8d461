// Launch helpers shared by the library's translation units.
#pragma once
#include "../../include/stand.h"

#include <cuda_runtime.h>
#include <stdint.h>
#include <atomic>

namespace stand {

inline int cuda_ok(cudaError_t e) { return e == cudaSuccess ? STAND_OK : STAND_E_CUDA; }
inline int launch_ok() { return cuda_ok(cudaGetLastError()); }

// Are all of these (null among them) multiples of `bytes`?  An element that lies across that boundary would fault.
template <typename... P> bool aligned(size_t bytes, const P*... p) { return ((... | (uintptr_t)p) & (bytes - 1)) == 0; }

unsigned wait_limit();  // polls of a bounded wait (stand_set_wait_limit)

// Raises a kernel's limit of dynamic shared memory, once per device.
struct SmemLimit {
  static constexpr int DEVICES = 64;
  std::atomic<int> done[DEVICES];
  template <typename K> int raise(K* kernel, size_t bytes) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return STAND_E_CUDA;
    if (dev < 0 || dev >= DEVICES) return STAND_E_ARG;
    if (done[dev].load(std::memory_order_acquire)) return STAND_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return STAND_E_CUDA;
    done[dev].store(1, std::memory_order_release);
    return STAND_OK;
  }
};

// Launch with programmatic stream serialisation: the kernel may be scheduled while its predecessor in the
// stream is still running; it calls pdl_wait() before it touches the predecessor's results.
template <typename... P>
int launch_dependent2(void (*kernel)(P...), dim3 grid, unsigned block, cudaStream_t st, size_t smem, const P&... params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cuda_ok(cudaLaunchKernelEx(&cfg, kernel, params...));
}

template <typename P>
int launch_dependent(void (*kernel)(P), dim3 grid, unsigned block, cudaStream_t st, const P& params, size_t smem = 0) {
  return launch_dependent2(kernel, grid, block, st, smem, params);
}

}  // namespace stand
