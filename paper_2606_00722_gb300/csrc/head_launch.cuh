// How the head's kernels follow one another: the next one is set up while the last one
// still runs, and waits for it before it touches memory.
#pragma once
#include <cuda_runtime.h>

#include <stdint.h>

#include <atomic>

#include "../../include/epic.h"

namespace epic {
namespace {

// First in every kernel that launch_next() starts, after what needs no memory; everything before is done and seen then.
__device__ __forceinline__ void follow() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The next kernel may be set up once all CTAs have come here.
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Once for each kernel and device: the shared memory that it may use.  With kNoCache an SM keeps nearly all of its L1 cache as
// shared memory, as the kernels on the tensor units need it: the split changes only on an empty SM, so those that come
// between them ask for the same.
constexpr int kNoCache = 0, kCache = -1;
inline bool prepare_kernel(const void* kernel, int shared) {
  static std::atomic<uintptr_t> done[256];  // kernel and device, by a hash; a place is taken once and kept
  int device;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  const uintptr_t key = (uintptr_t)kernel * 64 + (uintptr_t)device + 1;  // different for all kernels and up to 63 devices
  unsigned at = (unsigned)(key * 0x9e3779b97f4a7c15ull >> 56);
  for (int i = 0; i < 256; i++, at = (at + 1) % 256) {
    const uintptr_t here = done[at].load(std::memory_order_acquire);
    if (here == key) return true;
    if (here == 0) break;
  }
  if (shared == kNoCache &&
      cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess)
    return false;
  if (shared > 0 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared) != cudaSuccess) return false;
  uintptr_t none = 0;
  done[at].compare_exchange_strong(none, key, std::memory_order_release);  // another's now: prepared again the next time
  return true;
}

// most: the largest shared memory that the kernel is ever started with, or one of the above
template <typename... P, typename... A>
epic_status launch_next(void (*kernel)(P...), dim3 grid, int threads, int shared, int most, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = grid;
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = shared;
  c.stream = st;
  c.attrs = &at;
  c.numAttrs = 1;
  if (!prepare_kernel((const void*)kernel, most) || cudaLaunchKernelEx(&c, kernel, static_cast<P>(args)...) != cudaSuccess) {
    cudaGetLastError();
    return EPIC_ERR_CUDA;
  }
  return EPIC_OK;
}

}  // namespace
}  // namespace epic
