// Rows of logits on chip: what the kernels between a model's output and the
// constraint work share.
//
// A row of V logits belongs to a cluster of CTAs.  It is cut into chunks of 16
// bytes from the aligned address at or below its first element; each CTA of
// the cluster owns a run of chunks, staged once in its shared memory, so every
// further pass over the row costs no memory traffic.  Rows that do not fit the
// cluster's shared memory are read from global memory in every pass instead.
// Within a CTA a warp owns a contiguous run of chunks and reads it 32 chunks at
// a time, so sums by warp are sums in index order, and a thread reads in every
// pass the chunks that it staged itself: staging needs no barrier.
//
// The order of a row: value descending, ties by index ascending, as one 64-bit
// key (larger comes first).  NaN and -inf are not in the order.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <type_traits>

namespace epic {
namespace {

namespace cg = cooperative_groups;

typedef unsigned long long u64;

constexpr int kRowThreads = 256;              // most threads of a row CTA
constexpr int kRowWarps = kRowThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_32(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Where the rows are: row r of the call is logits[b][i], b = r / k, i = pos[b][r % k] (or r % k).
struct RowArgs {
  const void* base;
  long long stride_b, stride_n;  // in elements
  const int32_t* pos;            // [B][k] or NULL
  int n, k, V;
  int per;     // chunks per CTA
  int staged;  // the slices fit in shared memory
};

template <typename T>
struct ElemOf {
  static constexpr int E = 16 / sizeof(T);  // elements of a chunk
};

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T>
__device__ __forceinline__ void unpack(const uint4& c, float (&f)[ElemOf<T>::E]) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
  } else if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ uint4 pack(const float (&f)[ElemOf<T>::E]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = __float_as_uint(f[i]);
    } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    } else {
      const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One CTA's part of a row.
template <typename T>
struct Slice {
  static constexpr int E = ElemOf<T>::E;
  const char* row16;  // the row's address, rounded down to 16 bytes
  uint4* buf;         // staged chunks
  int head;           // elements between row16 and the row
  int c0, n;          // first chunk and number of chunks
  int V;
  int wper;      // chunks of a warp: warp w has those from w * wper on
  int wlo, whi;  // this warp's
  bool staged;

  // index of a chunk's first element (negative in a row's first chunk)
  __device__ __forceinline__ long long first(int c) const { return (long long)(c0 + c) * E - head; }

  __device__ uint4 from_global(int c) const {
    const long long i0 = first(c);
    const char* p = row16 + (size_t)(c0 + c) * 16;
    if (i0 >= 0 && i0 + E <= V) return __ldg(reinterpret_cast<const uint4*>(p));
    float f[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
      f[e] = i0 + e >= 0 && i0 + e < V ? to_float<T>(reinterpret_cast<const T*>(p)[e]) : -CUDART_INF_F;
    return pack<T>(f);
  }

  __device__ __forceinline__ uint4 chunk(int c) const { return staged ? buf[c] : from_global(c); }

  // the row of an element already known to be in the slice
  __device__ float at(int idx) const {
    const int c = (idx + head) / E - c0;
    return staged ? to_float<T>(reinterpret_cast<const T*>(buf + c)[(idx + head) % E])
                  : to_float<T>(reinterpret_cast<const T*>(row16)[idx + head]);
  }

  // first and past-the-end index of the elements in the slice
  __device__ __forceinline__ int lo() const { return (int)max(first(0), 0ll); }
  __device__ __forceinline__ int hi() const { return (int)min(max(first(n), 0ll), (long long)V); }

  // the slice of the row at `addr` (NULL: a row of no elements) for CTA `rank` of the cluster
  __device__ void open(const void* addr, int V_, const RowArgs& a, int rank, uint4* shared) {
    V = addr ? V_ : 0;
    const uintptr_t p = reinterpret_cast<uintptr_t>(addr);
    row16 = reinterpret_cast<const char*>(p & ~(uintptr_t)15);
    head = (int)(p & 15) / (int)sizeof(T);
    const long long total = V ? ((long long)head + V + E - 1) / E : 0;
    c0 = rank * a.per;
    n = (int)min(max(total - c0, 0ll), (long long)a.per);
    buf = shared;
    staged = a.staged;
    const int warps = blockDim.x / 32, w = threadIdx.x / 32;
    wper = (n + warps - 1) / warps;
    wlo = min(w * wper, n);
    whi = min(wlo + wper, n);
  }

  // f(c) for each chunk of this thread as it arrives in shared memory: all loads are issued first, in four groups
  template <typename F>
  __device__ __forceinline__ void stage(F f) const {
    const int lane = threadIdx.x % 32;
    if (!staged) {
      for (int c = wlo + lane; c < whi; c += 32) f(from_global(c));
      return;
    }
    const int quarter = (((whi - wlo + 31) / 32 + 3) / 4) * 32;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int end = min(wlo + (g + 1) * quarter, whi);
      for (int c = wlo + g * quarter + lane; c < end; c += 32) {
        const long long i0 = first(c);
        if (i0 >= 0 && i0 + E <= V) {
          const uint32_t dst = (uint32_t)__cvta_generic_to_shared(buf + c);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(row16 + (size_t)(c0 + c) * 16)
                       : "memory");
        } else {
          buf[c] = from_global(c);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
      if (g == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
      if (g == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
      if (g == 3) asm volatile("cp.async.wait_group 0;" ::: "memory");
      const int end = min(wlo + (g + 1) * quarter, whi);
      for (int c = wlo + g * quarter + lane; c < end; c += 32) f(buf[c]);
    }
  }
};

// Running maximum of a thread's chunks, two 16-bit elements an instruction; kNan: NaN if any element is, else NaN is
// left out.
template <typename T, bool kNan>
struct ChunkMax {
  float f;
  uint32_t h;
  __device__ ChunkMax() {
    f = -CUDART_INF_F;
    h = std::is_same_v<T, __nv_bfloat16> ? 0xff80ff80u : 0xfc00fc00u;  // -inf twice
  }
  __device__ __forceinline__ static uint32_t max2(uint32_t a, uint32_t b) {
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
      if constexpr (kNan) {
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
      } else {
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
      }
    } else {
      if constexpr (kNan) {
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
      } else {
        asm("max.f16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
      }
    }
    return a;
  }
  __device__ __forceinline__ static float max1(float a, float b) {
    if constexpr (kNan) {
      asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(a), "f"(b));
      return a;
    }
    return fmaxf(a, b);
  }
  __device__ __forceinline__ void add(const uint4& c) {
    if constexpr (sizeof(T) == 4) {
      f = max1(f, max1(max1(__uint_as_float(c.x), __uint_as_float(c.y)),
                       max1(__uint_as_float(c.z), __uint_as_float(c.w))));
    } else {
      h = max2(h, max2(max2(c.x, c.y), max2(c.z, c.w)));
    }
  }
  __device__ __forceinline__ float value() const {
    if constexpr (sizeof(T) == 4) return f;
    T v[2];
    memcpy(v, &h, 4);
    return max1(to_float<T>(v[0]), to_float<T>(v[1]));
  }
};

template <typename T>
__device__ __forceinline__ const void* row_address(const RowArgs& a, long long r) {
  const long long b = r / a.k;
  const int j = (int)(r - b * a.k);
  const int i = a.pos ? a.pos[r] : j;
  if (i < 0 || i >= a.n || a.V == 0) return nullptr;
  return static_cast<const T*>(a.base) + b * a.stride_b + (long long)i * a.stride_n;
}

// ---------------------------------------------------------------- the order

// floats as unsigned keys in the same order, -0 equal to +0
__device__ __forceinline__ uint32_t value_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ u64 order_key(float z, int idx) { return (u64)value_key(z) << 32 | (uint32_t)~idx; }
__device__ __forceinline__ float order_value(u64 k) { return key_value((uint32_t)(k >> 32)); }
__device__ __forceinline__ int order_index(u64 k) { return (int)~(uint32_t)k; }

}  // namespace
}  // namespace epic
