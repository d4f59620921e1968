#include "logit_launch.h"

#include <algorithm>

namespace epic {

// One CTA a row where the rows fill the GPU (two CTAs on each of the GB300's 152 SMs), or have at most 4,096 chunks: the best
// of 259 rows of 50,021 halves take 12.7 us on the GPU so and 20.1 in clusters of two, those of 64 rows of 32,768 bf16
// (4,096 chunks) 6.2 and 7.5.  Fewer long rows are cut over clusters of up to eight CTAs: a draw by all rules from one row of
// 126,000 takes 9.5 us in four CTAs and 10.4 in one.  In between each form wins somewhere: 64 rows of 33,000 bf16 (4,126
// chunks, cut in two) have their best in 7.8 us, 6.6 in one CTA, a draw by temperature in 9.6 and 8.3, from the nucleus in
// 28.6 and 29.3; the nucleus of 64 rows of 32,768 fp32 takes 25.3 and 29.5.
// Slices are cut further where they would be longer than a histogram's sums allow, for all operators: 1,024 rows of 126,000
// and 150,016 bf16 take, for each token of the vocabulary, 0.49 and 0.54 ns for the 32 best, 0.80 and 0.97 for draws by
// temperature, 2.47 and 2.67 from the nucleus, and 0.96 for loss and gradient in one call.
RowShape row_shape(long long rows, int V, int size, int least, int most) {
  const long long E = 16 / size;
  const long long chunks = V ? (V + E - 2) / E + 1 : 0;  // wherever the row starts in its first chunk
  const long long full = 2 * 152;
  RowShape p = {};
  p.ctas = 1;
  while (p.ctas < kRowCtasMax &&
         (chunks * E > (long long)p.ctas * kSliceElems || (rows * p.ctas * 2 <= full && V / E > p.ctas * 4096)))
    p.ctas *= 2;
  p.per = (int)((chunks + p.ctas - 1) / p.ctas);
  p.threads = (int)std::min<long long>(most, std::max<long long>(least, (p.per + 127) / 128 * 32));
  return p;
}

epic_status check_rows(const void* logits, int dtype, int B, int n, int V, int64_t stride_b, int64_t stride_n,
                       const int32_t* pos, int k) {
  if (dtype != EPIC_F32 && dtype != EPIC_F16 && dtype != EPIC_BF16) return EPIC_ERR_INVALID_ARG;
  if (B < 0 || n < 0 || V < 0 || k < 0 || stride_b < 0 || stride_n < 0) return EPIC_ERR_INVALID_ARG;
  if (!pos && k > n) return EPIC_ERR_INVALID_ARG;
  if (V > 0x7fffffff - 4096) return EPIC_ERR_CAPACITY;  // element indices and what lies past a row's end fit 32 bits
  if ((long long)B * k == 0) return EPIC_OK;
  if (n > 0 && V > 0) {
    if (!logits) return EPIC_ERR_INVALID_ARG;
    if ((uintptr_t)logits % (dtype == EPIC_F32 ? 4 : 2)) return EPIC_ERR_INVALID_ARG;
  }
  return EPIC_OK;
}

epic_status launch_rows(const void* kernel, const RowShape& p, long long rows, void* args, cudaStream_t st) {
  if (rows > 0x7fffffffll / p.ctas) return EPIC_ERR_CAPACITY;
  void* argv[] = {args};
  cudaError_t e;
  if (p.ctas == 1) {
    e = cudaLaunchKernel(kernel, dim3((unsigned)rows), dim3(p.threads), argv, 0, st);
  } else {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * p.ctas));
    cfg.blockDim = dim3(p.threads);
    cfg.stream = st;
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = p.ctas;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelExC(&cfg, kernel, argv);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    return EPIC_ERR_CUDA;
  }
  return EPIC_OK;
}

}  // namespace epic
