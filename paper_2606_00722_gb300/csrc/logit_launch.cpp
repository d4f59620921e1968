#include "logit_launch.h"

#include <algorithm>

namespace epic {

// Bytes of a row that one CTA stages, and the most that it may: slices of this size leave room for three CTAs on an SM,
// so that one row's loads run under another's passes.
constexpr size_t kSlice = 64 << 10;
constexpr size_t kSliceMax = 192 << 10;
constexpr int kClusterMax = 8;
constexpr size_t kSmemDefault = 16 << 10;  // with the kernels' own arrays within the 48 KB that need no asking

RowShape row_shape(long long rows, int V, int size) {
  const long long E = 16 / size;
  const long long chunks = V ? (V + E - 1 + E - 1) / E : 0;  // wherever the row starts in its first chunk
  RowShape p = {};
  p.ctas = 1;
  while (p.ctas < kClusterMax && (chunks + p.ctas - 1) / p.ctas * 16 > (long long)kSlice) p.ctas *= 2;
  p.per = (int)((chunks + p.ctas - 1) / p.ctas);
  p.staged = (size_t)p.per * 16 <= kSliceMax;
  p.smem = p.staged ? (size_t)p.per * 16 : 0;
  p.threads = std::min(256, std::max(64, (p.per + 31) / 32 * 32));
  return p;
}

epic_status check_rows(const void* logits, int dtype, int B, int n, int V, int64_t stride_b, int64_t stride_n,
                       const int32_t* pos, int k) {
  if (dtype != EPIC_F32 && dtype != EPIC_F16 && dtype != EPIC_BF16) return EPIC_ERR_INVALID_ARG;
  if (B < 0 || n < 0 || V < 0 || k < 0 || stride_b < 0 || stride_n < 0) return EPIC_ERR_INVALID_ARG;
  if (!pos && k > n) return EPIC_ERR_INVALID_ARG;
  if ((long long)B * k == 0) return EPIC_OK;
  if (n > 0 && V > 0) {
    if (!logits) return EPIC_ERR_INVALID_ARG;
    if ((uintptr_t)logits % (dtype == EPIC_F32 ? 4 : 2)) return EPIC_ERR_INVALID_ARG;
  }
  return EPIC_OK;
}

epic_status launch_rows(const void* kernel, const RowShape& p, long long rows, void* args, cudaStream_t st) {
  if (rows > 0x7fffffffll / p.ctas) return EPIC_ERR_CAPACITY;
  if (p.smem > kSmemDefault &&
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem) != cudaSuccess) {
    cudaGetLastError();
    return EPIC_ERR_CUDA;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * p.ctas));
  cfg.blockDim = dim3(p.threads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = p.ctas;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  void* argv[] = {args};
  if (cudaLaunchKernelExC(&cfg, kernel, argv) != cudaSuccess) {
    cudaGetLastError();
    return EPIC_ERR_CUDA;
  }
  return EPIC_OK;
}

}  // namespace epic
