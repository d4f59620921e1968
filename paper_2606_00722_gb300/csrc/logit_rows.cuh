// Rows of logits: what the kernels between a model's output and the constraint
// work share.
//
// A row of V logits belongs to a cluster of CTAs (one CTA where there are rows
// enough).  It is cut into chunks of 16 bytes from the aligned address at or
// below its first element; a CTA owns a run of chunks (its slice), which its
// warps take in turn by batches of 128, four a lane.  So sums by batch are sums in
// index order, and a lane meets the same chunks in every pass.  Nothing is
// staged: the first pass comes from memory, later ones from the L2 cache, which
// holds the rows in flight (three CTAs of 512 threads an SM are 456 rows, 115 MB
// at 126,000 tokens of 16 bits).  Slices staged in shared memory were slower: an
// SM then holds three of 63 KB, each for the 10 us of two cluster barriers and its
// passes, where 4 us would keep memory busy (the 32 best of 1,024 x 126,000: 111
// us staged in clusters of four, 99 us from L2 with a CTA a row, all else alike).
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

constexpr int kRowThreads = 512;  // most threads of a row CTA
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kRowCluster = 8;  // most CTAs of a row (the portable limit of a cluster)
constexpr float kLog2e = 1.4426950408889634f;

// The warp's number, the same in all lanes also to the compiler: votes and sums in loops over it need no check that the
// lanes have come together (such a check took 300 cycles).
__device__ __forceinline__ int warp_index() { return __shfl_sync(~0u, (int)threadIdx.x / 32, 0); }

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
  int per;  // chunks per CTA
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

constexpr int kBatch = 128;  // chunks that a warp takes at a time, four a lane

template <typename T>
__device__ __forceinline__ uint4 empty_chunk() {  // all -inf
  const uint32_t x = sizeof(T) == 4 ? 0xff800000u : std::is_same_v<T, __nv_bfloat16> ? 0xff80ff80u : 0xfc00fc00u;
  return make_uint4(x, x, x, x);
}

// One CTA's part of a row.
template <typename T>
struct Slice {
  static constexpr int E = ElemOf<T>::E;
  const char* row16;  // the row's address, rounded down to 16 bytes
  int head;           // elements between row16 and the row
  int c0, n;          // first chunk and number of chunks
  int V;
  int flo, fhi;  // the chunks whose 16 bytes are all of this row
  const uint4* ends;  // in shared memory: what the others, the row's first and last, have of it, else -inf

  // index of a chunk's first element (negative in a row's first chunk)
  __device__ __forceinline__ int first(int c) const { return (c0 + c) * E - head; }

  __device__ __forceinline__ const char* address(int c) const { return row16 + (size_t)(c0 + c) * 16; }

  // chunk c of the slice, of -inf past its end
  __device__ __forceinline__ uint4 chunk(int c) const {
    if (c >= flo && c < fhi) return __ldg(reinterpret_cast<const uint4*>(address(c)));
    return c >= n ? empty_chunk<T>() : ends[c < flo ? 0 : 1];
  }

  // the value of an element of the row
  __device__ float at(int idx) const { return to_float<T>(reinterpret_cast<const T*>(row16)[(size_t)head + idx]); }

  // first and past-the-end index of the elements in the slice
  __device__ __forceinline__ int lo() const { return max(first(0), 0); }
  __device__ __forceinline__ int hi() const { return min(max(first(n), 0), V); }

  // the slice of the row at `addr` (NULL: a row of no elements) for CTA `rank` of the cluster
  __device__ void open(const void* addr, const RowArgs& a, int rank, uint4 (&shared)[2]) {
    V = addr ? a.V : 0;
    const uintptr_t p = reinterpret_cast<uintptr_t>(addr);
    row16 = reinterpret_cast<const char*>(p & ~(uintptr_t)15);
    head = (int)(p & 15) / (int)sizeof(T);
    const int total = V ? (head + V - 1) / E + 1 : 0;
    c0 = rank * a.per;
    n = min(max(total - c0, 0), a.per);
    // the row's first and last chunk may have elements of other rows
    flo = c0 == 0 && head > 0 ? 1 : 0;
    fhi = max(c0 + n == total && (head + V) % E != 0 ? n - 1 : n, flo);
    ends = shared;
    if (flo == 0 && fhi == n) return;  // the same in all threads
    if (threadIdx.x < 2) {
      const int c = threadIdx.x == 0 ? 0 : n - 1, i0 = first(c);
      const T* p = reinterpret_cast<const T*>(address(c));
      float f[E];
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = i0 + e >= 0 && i0 + e < V ? to_float<T>(p[e]) : -CUDART_INF_F;
      shared[threadIdx.x] = pack<T>(f);
    }
    __syncthreads();
  }

  // f(v, c) for this warp's batches: v are this lane's chunks c, c + 32, c + 64 and c + 96, of -inf past the slice's end
  template <typename F>
  __device__ __forceinline__ void sweep(F f) const {
    for (int base = warp_index() * kBatch; base < n; base += (int)blockDim.x * 4) {
      uint4 v[4];
      const int c = base + (int)(threadIdx.x % 32);
      if (base >= flo && base + kBatch <= fhi) {
        const uint4* p = reinterpret_cast<const uint4*>(address(c));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __ldg(p + 32 * i);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = chunk(c + 32 * i);
      }
      f(v, c);
    }
  }
};

// The CTAs of a row.  A single one needs no cluster barrier (several times a block's in time).
struct RowGroup {
  unsigned n, rank;
  __device__ RowGroup() : n(cg::this_cluster().num_blocks()), rank(cg::this_cluster().block_rank()) {}
  __device__ __forceinline__ void sync() const {
    if (n == 1)
      __syncthreads();
    else
      cg::this_cluster().sync();
  }
  // CTA r's copy of a shared variable
  template <typename P>
  __device__ __forceinline__ P* at(P* p, unsigned r) const {
    return n == 1 ? p : cg::this_cluster().map_shared_rank(p, r);
  }
};

// Two 32-bit operations in one instruction, each rounded as the single one.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 y;
  asm("{.reg .b64 a, b, y; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; add.rn.f32x2 y, a, b; mov.b64 {%0, %1}, y;}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 y;
  asm("{.reg .b64 a, b, y; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mul.rn.f32x2 y, a, b; mov.b64 {%0, %1}, y;}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 y;
  asm("{.reg .b64 a, b, c, y; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mov.b64 c, {%6, %7}; "
      "fma.rn.f32x2 y, a, b, c; mov.b64 {%0, %1}, y;}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return y;
}

// Running maximum of a thread's chunks, two 16-bit elements an instruction; kNan: NaN if any element is, else NaN is
// left out.
template <typename T, bool kNan>
struct ChunkMax {
  float f;
  uint32_t h;
  __device__ ChunkMax() {
    f = -CUDART_INF_F;
    h = empty_chunk<T>().x;
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
  __device__ __forceinline__ void add(const uint4 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) add(v[i]);
  }
  __device__ __forceinline__ float value() const {
    if constexpr (sizeof(T) == 4) return f;
    T v[2];
    memcpy(v, &h, 4);
    return max1(to_float<T>(v[0]), to_float<T>(v[1]));
  }
};

template <typename T>
__device__ __forceinline__ const T* row_address(const RowArgs& a, int r) {
  const int b = r / a.k, j = r - b * a.k;
  const int i = a.pos ? a.pos[r] : j;
  if (i < 0 || i >= a.n || a.V == 0) return nullptr;
  return static_cast<const T*>(a.base) + b * a.stride_b + i * a.stride_n;
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
