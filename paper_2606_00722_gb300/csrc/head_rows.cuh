// Arithmetic of the head's loss on one row, the same wherever it is done.
//
// Exponentials are powers of two relative to a whole number: e = 2^(z log2 e - ref).
// The product and the difference are one fused operation, so only the result is
// rounded, and sums relative to different references meet by exact scaling.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <stdint.h>

namespace epic {
namespace {

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// How far, in powers of two, a row's logits may lie above its reference: 2^60 times any vocabulary is in range of 32 bits,
// and so is the inverse of such a sum times a hidden state in bf16.
constexpr float kWindow = 60.0f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^k of a whole k, exact; 0 below 2^-126, +inf above 2^127, NaN for NaN
__device__ __forceinline__ float pow2_whole(float k) {
  if (!(k >= -126.0f)) return k < -126.0f ? 0.0f : CUDART_NAN_F;
  return k > 127.0f ? CUDART_INF_F : __int_as_float(((int)k + 127) << 23);
}

// The whole reference of a largest logit; -inf and NaN take 0
__device__ __forceinline__ float whole_ref(float z) { return z > -CUDART_INF_F ? rintf(z * kLog2E) : 0.0f; }

// (ref, s) and (ref2, s2) as one sum relative to the larger reference; a sum of 0 has none
__device__ __forceinline__ void meet(float& ref, float& s, float ref2, float s2) {
  if (s2 == 0.0f) return;
  const bool up = ref2 > ref;
  const float k = pow2_whole(up ? ref - ref2 : ref2 - ref);
  s = up ? s2 + s * k : s + s2 * k;
  if (up) ref = ref2;
}
constexpr float kNoRef = -3.0e38f;  // of an empty sum

// a record of logits that 32 bits do not hold (+inf): its sum is NaN
__device__ __forceinline__ float2 record(float ref, float s) {
  return fabsf(ref) <= 3.0e38f ? make_float2(ref, s) : make_float2(0.0f, CUDART_NAN_F);
}

template <typename T>
__device__ __forceinline__ float as_float(T v);
template <>
__device__ __forceinline__ float as_float<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float as_float<float>(float v) { return v; }

template <typename T>
__device__ __forceinline__ T of_float(float v);
template <>
__device__ __forceinline__ __half of_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 of_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ float of_float<float>(float v) { return v; }

// What the rounding of a number to 16 bits takes from it
template <typename T>
__device__ __forceinline__ float lost(float v) {
  const float rest = v - as_float(of_float<T>(v));
  return fabsf(rest) < CUDART_INF_F ? rest : 0.0f;
}

// 16 bytes of a row as numbers of 32 bits
template <typename T>
struct Chunk {
  static constexpr int kCount = 16 / sizeof(T);
  float v[kCount];
  __device__ __forceinline__ Chunk(const T* x, int count, bool whole) {
    if (whole && count >= kCount) {
      const uint4 w = *(const uint4*)x;
      const T* t = (const T*)&w;
#pragma unroll
      for (int i = 0; i < kCount; i++) v[i] = as_float(t[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kCount; i++) v[i] = i < count ? as_float(x[i]) : 0.0f;
    }
  }
};

// 16 bytes from byte m of two times 16 on
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, uint32_t m) {
  uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int c = 0; c < 6; c++) x[c] = m & 8 ? x[c + 2] : x[c];
#pragma unroll
  for (int c = 0; c < 5; c++) x[c] = m & 4 ? x[c + 1] : x[c];
  const int by = (m & 3) * 8;
  return make_uint4(__funnelshift_r(x[0], x[1], by), __funnelshift_r(x[1], x[2], by), __funnelshift_r(x[2], x[3], by),
                    __funnelshift_r(x[3], x[4], by));
}

}  // namespace
}  // namespace epic
