// The head in 8-bit integers: rounding of rows to 8 bits with a scale for each, and
// logits z[r][v] = (sum_k q[r][k] w[v][k]) s[r] S[v].
//
// Sums are whole numbers and exact, so logits do not depend on the order of the
// sum; each is rounded to 32 bits as it is scaled and once to its type.
#include "../../include/epic.h"
#include "head_rows.cuh"

namespace epic {
namespace {

struct QuantArgs {
  const void* x;
  long long stride_b, stride_n;
  const int32_t* pos;
  int n, k, d;
  int8_t* q;
  float* scale;
};

constexpr int kQuantThreads = 256;

// A CTA a row: the largest size in one pass, the quotients in a second one, from the caches.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads) k_quantize_rows(QuantArgs a) {
  __shared__ float s_top[kQuantThreads / 32];
  const long long r = blockIdx.x, b = r / a.k;
  const int at = a.pos ? a.pos[r] : (int)(r % a.k);
  int8_t* q = a.q + r * a.d;
  if (at < 0 || at >= a.n) {
    for (int k = threadIdx.x; k < a.d; k += kQuantThreads) q[k] = 0;
    if (threadIdx.x == 0) a.scale[r] = CUDART_NAN_F;
    return;
  }
  const T* x = (const T*)a.x + b * a.stride_b + at * a.stride_n;
  float top = 0.0f;
  for (int k = threadIdx.x; k < a.d; k += kQuantThreads) {
    const float v = fabsf(as_float(x[k]));
    top = v <= top ? top : v;  // a NaN stays
    if (v != v) break;
  }
  for (int o = 16; o; o >>= 1) {
    const float v = __shfl_xor_sync(~0u, top, o);
    top = v <= top || top != top ? top : v;
  }
  if (threadIdx.x % 32 == 0) s_top[threadIdx.x / 32] = top;
  __syncthreads();
  top = s_top[0];
  for (int w = 1; w < kQuantThreads / 32; w++) top = s_top[w] <= top || top != top ? top : s_top[w];
  const float s = __fdiv_rn(top, 127.0f);
  if (threadIdx.x == 0) a.scale[r] = s;
  for (int k = threadIdx.x; k < a.d; k += kQuantThreads) {
    const float v = rintf(__fdiv_rn(as_float(x[k]), s));
    q[k] = s > 0.0f && v == v ? (int8_t)fminf(fmaxf(v, -127.0f), 127.0f) : 0;
  }
}

struct Int8Args {
  const int8_t* q;
  const float* scale;
  const int8_t* head;
  long long head_stride;
  const float* head_scale;
  void* logits;
  long long stride_b, stride_n;
  long long rows;
  int k, d, V;
};

constexpr int kT = 64, kStep = 16;

template <typename T>
__global__ void __launch_bounds__(256) k_int8_logits(Int8Args a) {
  __shared__ int s_q[kStep][kT + 1], s_w[kStep][kT + 1];
  const long long r0 = (long long)blockIdx.y * kT, v0 = (long long)blockIdx.x * kT;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < a.d; k0 += kStep) {
    for (int i = threadIdx.x; i < kStep * kT; i += 256) {
      const int m = i / kStep, k = i % kStep;
      s_q[k][m] = k0 + k < a.d && r0 + m < a.rows ? a.q[(r0 + m) * a.d + k0 + k] : 0;
      s_w[k][m] = k0 + k < a.d && v0 + m < a.V ? a.head[(v0 + m) * a.head_stride + k0 + k] : 0;
    }
    __syncthreads();
    for (int k = 0; k < kStep; k++)
      for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) acc[i][j] += s_q[k][ty + 16 * i] * s_w[k][tx + 16 * j];
    __syncthreads();
  }
  for (int i = 0; i < 4; i++) {
    const long long r = r0 + ty + 16 * i;
    if (r >= a.rows) continue;
    T* z = (T*)a.logits + r / a.k * a.stride_b + r % a.k * a.stride_n;
    for (int j = 0; j < 4; j++) {
      const long long v = v0 + tx + 16 * j;
      if (v < a.V) z[v] = of_float<T>((float)acc[i][j] * a.scale[r] * a.head_scale[v]);
    }
  }
}

template <typename T>
epic_status launch_int8(const Int8Args& a, cudaStream_t st) {
  const long long by = (a.rows + kT - 1) / kT;
  k_int8_logits<T><<<dim3((unsigned)((a.V + (long long)kT - 1) / kT), (unsigned)by), 256, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA;
}

bool bad_type(int dtype) { return dtype != EPIC_F32 && dtype != EPIC_F16 && dtype != EPIC_BF16; }
size_t size_of(int dtype) { return dtype == EPIC_F32 ? 4 : 2; }

// 128 * 128 * kMostProducts is the largest sum that 32 bits hold
constexpr int kMostProducts = 131071;
constexpr long long kMostRows = 1 << 21;

}  // namespace
}  // namespace epic

extern "C" {

epic_status epic_quantize_rows(const void* d_x, int32_t dtype, int32_t B, int32_t n, int32_t d, int64_t stride_b,
                               int64_t stride_n, const int32_t* d_pos, int32_t k, int8_t* d_q, float* d_scale,
                               void* cuda_stream) {
  using namespace epic;
  if (bad_type(dtype) || B < 0 || n < 0 || d < 1 || k < 0 || stride_b < 0 || stride_n < 0 || (!d_pos && k > n))
    return EPIC_ERR_INVALID_ARG;
  const long long rows = (long long)B * k;
  if (rows > 0x7fffffffll) return EPIC_ERR_CAPACITY;
  if (rows == 0) return EPIC_OK;
  if ((!d_x && n > 0) || (uintptr_t)d_x % size_of(dtype) || !d_q || !d_scale || (uintptr_t)d_scale % 4 ||
      (uintptr_t)d_pos % 4)
    return EPIC_ERR_INVALID_ARG;
  const QuantArgs a = {d_x, stride_b, stride_n, d_pos, n, k, d, d_q, d_scale};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (dtype) {
    case EPIC_F32: k_quantize_rows<float><<<(unsigned)rows, kQuantThreads, 0, st>>>(a); break;
    case EPIC_F16: k_quantize_rows<__half><<<(unsigned)rows, kQuantThreads, 0, st>>>(a); break;
    default: k_quantize_rows<__nv_bfloat16><<<(unsigned)rows, kQuantThreads, 0, st>>>(a);
  }
  return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA;
}

epic_status epic_int8_logits_workspace(int32_t B, int32_t k, int32_t d, int32_t V, const int8_t* d_head,
                                       int64_t head_stride, size_t* bytes) {
  using namespace epic;
  if (!bytes || B < 0 || k < 0 || d < 1 || V < 0 || (V > 1 && head_stride < d)) return EPIC_ERR_INVALID_ARG;
  if (d > kMostProducts || V > 0x7fffffff - 4096 || (long long)B * k > kMostRows) return EPIC_ERR_CAPACITY;
  *bytes = 256;
  return EPIC_OK;
}

epic_status epic_int8_logits(const int8_t* d_q, const float* d_scale, int32_t B, int32_t k, int32_t d,
                             const int8_t* d_head, const float* d_head_scale, int32_t V, int64_t head_stride,
                             void* d_logits, int32_t dtype, int64_t stride_b, int64_t stride_n, void* d_workspace,
                             size_t workspace_bytes, void* cuda_stream) {
  using namespace epic;
  size_t need = 0;
  if (bad_type(dtype) || stride_b < 0 || stride_n < 0) return EPIC_ERR_INVALID_ARG;
  const epic_status s = epic_int8_logits_workspace(B, k, d, V, d_head, head_stride, &need);
  if (s != EPIC_OK) return s;
  const long long rows = (long long)B * k;
  if (rows == 0 || V == 0) return EPIC_OK;
  if (!d_q || !d_scale || !d_head || !d_head_scale || !d_logits || (uintptr_t)d_logits % size_of(dtype) ||
      (uintptr_t)d_scale % 4 || (uintptr_t)d_head_scale % 4)
    return EPIC_ERR_INVALID_ARG;
  if (!d_workspace || (uintptr_t)d_workspace % 256 || workspace_bytes < need) return EPIC_ERR_INVALID_ARG;
  const Int8Args a = {d_q, d_scale, d_head, head_stride, d_head_scale, d_logits, stride_b, stride_n, rows, k, d, V};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (dtype) {
    case EPIC_F32: return launch_int8<float>(a, st);
    case EPIC_F16: return launch_int8<__half>(a, st);
    default: return launch_int8<__nv_bfloat16>(a, st);
  }
}

}  // extern "C"
