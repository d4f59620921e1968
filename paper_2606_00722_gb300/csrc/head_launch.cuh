// How the head's kernels follow one another: the next one is set up while the last one
// still runs, and waits for it before it touches memory.
#pragma once
#include <cuda_runtime.h>

#include <mutex>
#include <set>
#include <utility>

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
  static std::mutex lock;
  static std::set<std::pair<const void*, int>> done;
  int device;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  std::lock_guard<std::mutex> hold(lock);
  if (done.count({kernel, device})) return true;
  if (shared == kNoCache &&
      cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess)
    return false;
  if (shared > 0 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared) != cudaSuccess) return false;
  done.insert({kernel, device});
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
