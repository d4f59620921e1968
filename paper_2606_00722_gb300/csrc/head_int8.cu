// The head in 8-bit integers: rounding of rows to 8 bits with a scale for each, and
// logits z[r][v] = (sum_k q[r][k] w[v][k]) s[r] S[v].
//
// Sums are whole numbers and exact, so logits do not depend on the order of the
// sum; each is rounded to 32 bits as it is scaled and once to its type.
#include <cuda.h>

#include <algorithm>

#include "../../include/epic.h"
#include "head_rows.cuh"
#include "tensor_tiles.cuh"

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
  int rows, k, d, V;
  int* failed;
};

// ---- few rows: a warp's lanes along tokens' rows, whole-number products of four bytes an instruction

constexpr int kFewRows = 8, kFewTokens = 4, kFewThreads = 256;
constexpr int kFewBytes = 64 << 10;  // of hidden states that a CTA holds

// Lane l keeps the total over all lanes of v[l % N]; every step halves how many values a lane holds.
template <int N>
__device__ __forceinline__ int totals(int (&v)[N], int lane) {
  int o = 16;
#pragma unroll
  for (int n = N; n > 1; n /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < n / 2; i++) {
      const int give = up ? v[i] : v[i + n / 2], keep = up ? v[i + n / 2] : v[i];
      v[i] = keep + __shfl_xor_sync(~0u, give, o);
    }
  }
  int t = v[0];
  for (; o; o /= 2) t += __shfl_xor_sync(~0u, t, o);
  return t;
}

template <typename T, int R>
__global__ void __launch_bounds__(kFewThreads) k_few_logits(Int8Args a) {
  extern __shared__ int4 s_q[];
  const int lane = threadIdx.x % 32, chunks = (a.d + 15) / 16;
  for (int i = threadIdx.x; i < R * chunks * 16; i += kFewThreads) {
    const int r = i / (chunks * 16), c = i % (chunks * 16);
    ((int8_t*)s_q)[i] = r < a.rows && c < a.d ? a.q[(long long)r * a.d + c] : 0;
  }
  __syncthreads();
  const long long warps = (long long)gridDim.x * (kFewThreads / 32);
  for (long long v0 = (blockIdx.x * (long long)(kFewThreads / 32) + threadIdx.x / 32) * kFewTokens; v0 < a.V;
       v0 += warps * kFewTokens) {
    int sum[R * kFewTokens] = {};
    const int4* w[kFewTokens];
#pragma unroll
    for (int t = 0; t < kFewTokens; t++) w[t] = (const int4*)(a.head + min(v0 + t, (long long)a.V - 1) * a.head_stride);
#pragma unroll 2
    for (int c = lane; c < chunks; c += 32) {
      int4 x[kFewTokens];
#pragma unroll
      for (int t = 0; t < kFewTokens; t++) x[t] = __ldcs(w[t] + c);
#pragma unroll
      for (int r = 0; r < R; r++) {
        const int4 y = s_q[r * chunks + c];
#pragma unroll
        for (int t = 0; t < kFewTokens; t++) {
          int& s = sum[r * kFewTokens + t];
          s = __dp4a(x[t].x, y.x, s);
          s = __dp4a(x[t].y, y.y, s);
          s = __dp4a(x[t].z, y.z, s);
          s = __dp4a(x[t].w, y.w, s);
        }
      }
    }
    // a lane's total is of the value whose number's bits, highest first, are the lane's from bit 4 down
    const int total = totals(sum, lane);
    constexpr int kValues = R * kFewTokens;
    const int at = lane / (32 / kValues), r = at / kFewTokens;
    const long long v = v0 + at % kFewTokens;
    if (lane % (32 / kValues) == 0 && r < a.rows && v < a.V) {
      T* z = (T*)a.logits + r / a.k * a.stride_b + r % a.k * a.stride_n;
      z[v] = of_float<T>((float)total * a.scale[r] * a.head_scale[v]);
    }
  }
}

// ---- many rows: on the tensor units
//
// This GPU's tensor units have no fast products of 8-bit integers, but a product of two of them in fp16 is exact, and so are
// sums in 32-bit floats while they stay below 2^24, which 1,024 products do; they are then taken over into 32-bit
// integers.  A pair of CTAs makes 256 tokens x up to 256 rows.  The head's bytes come through a queue of copies that each
// thread keeps for itself; the thread turns them into fp16 (byte + 128 in the low bits of 1024.0, less 1152) in the
// operand's place.  Hidden states are turned once, in the workspace, and come by boxes.

constexpr int kWorkWarps = 16, kWork = 32 * kWorkWarps, kThreads = kWork + 128;
constexpr int kTileTokens = 256, kHalf = 128, kStepK = 64, kRing = 4, kExactSteps = 1024 / kStepK;
constexpr int kOperandA = kHalf * kStepK * 2, kOperandB = kHalf * kStepK * 2;
constexpr int kQueue = 8, kQueueBytes = kQueue * kWork * 16;  // askew: half as many steps of twice the bytes
constexpr int kShared = kRing * (kOperandA + kOperandB) + kQueueBytes + 1024;
constexpr int kPairs = 76;

struct Int8Bars {
  uint64_t full[kRing], empty[kRing], sums_full[2], sums_empty[2];
  uint32_t sums;
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// four bytes as four numbers of fp16
__device__ __forceinline__ uint2 halves_of(uint32_t w) {
  const uint32_t u = w ^ 0x80808080u;
  const __half2 off = __half2half2(__ushort_as_half(0x6480));  // 1152
  uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 x = __hsub2(*(__half2*)&a, off), y = __hsub2(*(__half2*)&b, off);
  return make_uint2(*(const uint32_t*)&x, *(const uint32_t*)&y);
}

__device__ __forceinline__ uint4 load_shared(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void store_shared(uint32_t at, uint2 a, uint2 b) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a.x), "r"(a.y), "r"(b.x), "r"(b.y) : "memory");
}

// kRows: rows of a tile.  kAskew: rows of the head start anywhere; a thread copies the two aligned chunks of 16 that its 16
// bytes lie in (the first may begin up to 15 bytes ahead of the row, within its aligned 16).
template <typename T, int kRows, bool kAskew>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_int8_tiles(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ Int8Args a) {
  extern __shared__ uint8_t shared_raw[];
  __shared__ Int8Bars bars;
  const uint32_t ring = (smem_address(shared_raw) + 1023) / 1024 * 1024;
  const uint32_t queue = ring + kRing * (kOperandA + kOperandB);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, pair = blockIdx.x / 2;
  const uint32_t rank = cluster_rank();
  const uint32_t full = smem_address(bars.full), empty = smem_address(bars.empty);
  const uint32_t sums_full = smem_address(bars.sums_full), sums_empty = smem_address(bars.sums_empty);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kRing; s++) {
      bar_init(full + 8 * s, 1 + 2 * kWorkWarps);
      bar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < 2; s++) {
      bar_init(sums_full + 8 * s, 1);
      bar_init(sums_empty + 8 * s, 2 * kWorkWarps);
    }
    bar_init_visible();
  }
  if (warp == kWorkWarps) sums_take_pair(smem_address(&bars.sums));
  products_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  const uint32_t sums = bars.sums;
  const int row_tiles = (a.rows + kRows - 1) / kRows, steps = (a.d + kStepK - 1) / kStepK;
  const int tiles = (int)((a.V + (long long)kTileTokens - 1) / kTileTokens) * row_tiles;
  constexpr int kBoxBytes = kRows / 2 * kStepK * 2;
  bool ok = true;

  // Of 96 registers a thread that a block of 256 rows is launched with, 61,440, the four warpgroups that hold sums take 112
  // each and leave the last one 32.
  if (warp >= kWorkWarps) {
    if (kRows == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (warp == kWorkWarps && lane == 0) {  // boxes of hidden states
      const uint32_t full0 = at_rank(full, 0);
      int s = 0;
      uint32_t turn = 0;
      for (int t = pair; ok && t < tiles; t += kPairs) {
        const int r0 = t % row_tiles * kRows + rank * (kRows / 2);
        for (int k = 0; k < steps; k++) {
          if (!(ok = bar_wait(empty + 8 * s, turn ^ 1))) break;
          if (rank == 0) bar_expect(full + 8 * s, 2 * kBoxBytes);
          load_box_pair(&q_map, ring + s * (kOperandA + kOperandB) + kOperandA, full0 + 8 * s, k * kStepK, r0);
          if (++s == kRing) s = 0, turn ^= 1;
        }
      }
    }
    if (warp == kWorkWarps + 1 && lane == 0 && rank == 0) {  // products
      constexpr uint32_t kind = product_kind(false, false, false, kTileTokens, kRows);
      int s = 0, use = 0;
      uint32_t turn = 0;
      for (int t = pair; ok && t < tiles; t += kPairs) {
        for (int k = 0; ok && k < steps; use++) {
          const int half = use & 1, end = min(k + kExactSteps, steps);
          if (!(ok = bar_wait(sums_empty + 8 * half, (use >> 1 & 1) ^ 1))) break;
          products_fence_after();
          for (bool add = false; k < end; k++) {
            if (!(ok = bar_wait(full + 8 * s, turn))) break;
            products_fence_after();
            const uint32_t A = ring + s * (kOperandA + kOperandB);
            const uint64_t da = operand_k(A), db = operand_k(A + kOperandA);
#pragma unroll
            for (int j = 0; j < kStepK / 16; j++, add = true)
              product_pair(sums + half * 256, da + j * kNextK, db + j * kNextK, kind, add);
            products_arrive_pair(empty + 8 * s);
            if (++s == kRing) s = 0, turn ^= 1;
          }
          if (ok) products_arrive_pair(sums_full + 8 * half);
        }
      }
    }
  } else {
    if (kRows == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    constexpr int kCols = kRows / 4;               // a warp's rows of logits
    constexpr int kLoad = kCols < 16 ? kCols : 16;  // at a time
    constexpr int kDepth = kAskew ? kQueue / 2 : kQueue;
    const int tid = threadIdx.x, token = tid / 4, j = tid % 4, quarter = warp % 4, group = warp / 4;
    const uint32_t slot = queue + tid * 16;
    const uint32_t place = token * 128, c0 = ((2 * j) ^ (token & 7)) * 16, c1 = ((2 * j + 1) ^ (token & 7)) * 16;
    const uint32_t full0 = at_rank(full, 0), sums_empty0 = at_rank(sums_empty, 0);
    const uint32_t from = sums + group * kCols + ((uint32_t)quarter * 32 << 16);
    int acc[kCols];
#pragma unroll
    for (int i = 0; i < kCols; i++) acc[i] = 0;

    int ahead_t = pair, ahead_k = 0, ahead_s = 0;  // the next copy
    auto copy = [&] {
      if (ahead_t < tiles) {
        const long long v = (long long)(ahead_t / row_tiles) * kTileTokens + rank * kHalf + token;
        const int k = ahead_k * kStepK + j * 16, left = v < a.V ? a.d - k : 0;
        const int8_t* w = left > 0 ? a.head + v * a.head_stride + k : a.head;
        const uint32_t to = slot + ahead_s * (kAskew ? 2 : 1) * kWork * 16;
        if (!kAskew) {
          copy16(to, w, max(0, min(left, 16)));
        } else {
          const int m = (int)((uintptr_t)w & 15);
          w -= m;
          copy16(to, w, left > 0 ? min(left + m, 16) : 0);
          copy16(to + kWork * 16, left + m > 16 ? w + 16 : w, left > 0 ? max(0, min(left + m - 16, 16)) : 0);
        }
        if (++ahead_s == kDepth) ahead_s = 0;
        if (++ahead_k == steps) ahead_k = 0, ahead_t += kPairs;
      }
      copies_commit();
    };
    int use = 0, waiting = -1, since = 0;  // sums that are taken over next: of tile `waiting`, its last if `whole`
    bool whole = false;
    auto take = [&] {
      const int half = use & 1;
      if (!(ok = bar_wait(sums_full + 8 * half, use >> 1 & 1))) return;
      products_fence_after();
#pragma unroll
      for (int c = 0; c < kCols; c += kLoad) {
        float v[kLoad];
        sums_load(from + half * 256 + c, v);
        sums_loaded(v);
#pragma unroll
        for (int i = 0; i < kLoad; i++) acc[c + i] += __float2int_rn(v[i]);
      }
      products_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(sums_empty0 + 8 * half);
      use++;
      if (whole) {
        const int r0 = waiting % row_tiles * kRows + group * kCols;
        const long long v = (long long)(waiting / row_tiles) * kTileTokens + rank * kHalf + quarter * 32 + lane;
        if (v < a.V) {
          const float S = a.head_scale[v];
          int b = r0 / a.k, i = r0 % a.k;
          T* z = (T*)a.logits + b * a.stride_b + i * a.stride_n + v;
#pragma unroll
          for (int c = 0; c < kCols; c++) {
            if (r0 + c < a.rows) *z = of_float<T>((float)acc[c] * a.scale[r0 + c] * S);
            z += a.stride_n;
            if (++i == a.k) i = 0, b++, z = (T*)a.logits + b * a.stride_b + v;
          }
        }
#pragma unroll
        for (int i = 0; i < kCols; i++) acc[i] = 0;
      }
      waiting = -1;
    };

    int s = 0, qs = 0, t = pair, k = 0;
    uint32_t turn = 0;
    for (int i = 1 - kDepth; t < tiles || waiting >= 0; i++) {
      copy();
      if (i < 0) continue;
      bool end = true;
      if (t < tiles) {
        copies_wait<kDepth - 1>();
        const uint32_t at = slot + qs * (kAskew ? 2 : 1) * kWork * 16;
        if (++qs == kDepth) qs = 0;
        uint4 w = load_shared(at);
        if (kAskew) {
          const long long v = (long long)(t / row_tiles) * kTileTokens + rank * kHalf + token;
          const int m = (int)((uintptr_t)(a.head + min(v, (long long)a.V - 1) * a.head_stride) & 15);
          const uint4 w2 = load_shared(at + kWork * 16);
          uint32_t x[8] = {w.x, w.y, w.z, w.w, w2.x, w2.y, w2.z, w2.w};
#pragma unroll
          for (int i = 0; i < 6; i++) x[i] = m & 8 ? x[i + 2] : x[i];
#pragma unroll
          for (int i = 0; i < 5; i++) x[i] = m & 4 ? x[i + 1] : x[i];
          const int by = (m & 3) * 8;
          w = make_uint4(__funnelshift_r(x[0], x[1], by), __funnelshift_r(x[1], x[2], by), __funnelshift_r(x[2], x[3], by),
                         __funnelshift_r(x[3], x[4], by));
        }
        if (!(ok = bar_wait(empty + 8 * s, turn ^ 1))) break;
        const uint32_t A = ring + s * (kOperandA + kOperandB) + place;
        store_shared(A + c0, halves_of(w.x), halves_of(w.y));
        store_shared(A + c1, halves_of(w.z), halves_of(w.w));
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(full0 + 8 * s);
        if (++s == kRing) s = 0, turn ^= 1;
        end = (k + 1) % kExactSteps == 0 || k + 1 == steps;
      }
      // sums are taken over once the products are past them, or before the next ones are whole
      if (waiting >= 0 && (++since >= kRing || end)) {
        take();
        if (!ok) break;
      }
      if (t < tiles) {
        if (end) waiting = t, whole = k + 1 == steps, since = 0;
        if (++k == steps) k = 0, t += kPairs;
      }
    }
    copies_wait<0>();
  }
  if (!ok) {
    *a.failed = 1;
    let_copies_land();
  }
  products_fence_before();
  __syncwarp();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  if (warp == kWorkWarps) sums_free_pair(sums);
}

// Hidden states of 8 bits as fp16, rows of a multiple of 16 bytes
__global__ void __launch_bounds__(256) k_rows_as_halves(const int8_t* q, __half* to, int d, int ld, long long rows, int* failed) {
  if (blockIdx.x == 0 && threadIdx.x == 0) *failed = 0;
  const int lane = threadIdx.x % 32;
  for (long long r = blockIdx.x * 8ll + threadIdx.x / 32; r < rows; r += gridDim.x * 8ll)
#pragma unroll 4
    for (int k = lane; k < ld; k += 32) to[r * ld + k] = __float2half_rn(k < d ? (float)q[r * d + k] : 0.0f);
}

// ---- on the host

template <typename T, int R>
epic_status launch_few(const Int8Args& a, cudaStream_t st) {
  const int bytes = R * ((a.d + 15) / 16) * 16;
  if (cudaFuncSetAttribute(k_few_logits<T, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
    return cudaGetLastError(), EPIC_ERR_CUDA;
  const long long ctas = (a.V + (long long)kFewThreads / 32 * kFewTokens - 1) / (kFewThreads / 32 * kFewTokens);
  k_few_logits<T, R><<<(unsigned)std::min(ctas, 152ll * 4), kFewThreads, bytes, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA;
}

template <typename T, int kRows>
epic_status launch_tiles(const Int8Args& a, __half* q16, int ld, bool askew, cudaStream_t st) {
  CUtensorMap map;
  if (!make_map(&map, false, q16, ld, a.rows, ld, kRows / 2)) return EPIC_ERR_CUDA;
  const auto kernel = askew ? k_int8_tiles<T, kRows, true> : k_int8_tiles<T, kRows, false>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared) != cudaSuccess)
    return cudaGetLastError(), EPIC_ERR_CUDA;
  kernel<<<2 * kPairs, kThreads, kShared, st>>>(map, a);
  return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA;
}

bool head_lies_askew(const int8_t* head, long long stride, int V) {
  return (uintptr_t)head % 16 != 0 || (V > 1 && stride % 16 != 0);
}

bool few_rows(long long rows, int d, bool askew) {
  return rows <= kFewRows && !askew && (rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8) * (d + 15ll) <= kFewBytes;
}

// Rows of a tile: a step takes the tensor units 2 clocks a row, and about 320 at least for the head's bytes.
int tile_rows(long long rows) {
  int best = 256;
  long long least = -1;
  for (const int n : {256, 128, 64, 32}) {
    const long long cost = (rows + n - 1) / n * std::max(2 * n, 320);
    if (least < 0 || cost < least) best = n, least = cost;
  }
  return best;
}

template <typename T>
epic_status launch_int8(Int8Args a, void* ws, cudaStream_t st) {
  const bool askew = head_lies_askew(a.head, a.head_stride, a.V);
  if (few_rows(a.rows, a.d, askew)) {
    if (a.rows <= 1) return launch_few<T, 1>(a, st);
    if (a.rows <= 2) return launch_few<T, 2>(a, st);
    return a.rows <= 4 ? launch_few<T, 4>(a, st) : launch_few<T, 8>(a, st);
  }
  a.failed = (int*)ws;
  __half* q16 = (__half*)((char*)ws + 256);
  const int ld = (a.d + 7) / 8 * 8;
  k_rows_as_halves<<<(unsigned)std::min(1216, (a.rows + 7) / 8), 256, 0, st>>>(a.q, q16, a.d, ld, a.rows, a.failed);
  if (cudaGetLastError() != cudaSuccess) return EPIC_ERR_CUDA;
  switch (tile_rows(a.rows)) {
    case 32: return launch_tiles<T, 32>(a, q16, ld, askew, st);
    case 64: return launch_tiles<T, 64>(a, q16, ld, askew, st);
    case 128: return launch_tiles<T, 128>(a, q16, ld, askew, st);
    default: return launch_tiles<T, 256>(a, q16, ld, askew, st);
  }
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
  const long long rows = (long long)B * k;
  *bytes = 256;
  if (!few_rows(rows, d, head_lies_askew(d_head, head_stride, V))) *bytes += (size_t)rows * ((d + 7) / 8 * 8) * 2;
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
  const Int8Args a = {d_q, d_scale, d_head, head_stride, d_head_scale, d_logits, stride_b, stride_n, (int)rows, k, d, V, nullptr};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (dtype) {
    case EPIC_F32: return launch_int8<float>(a, d_workspace, st);
    case EPIC_F16: return launch_int8<__half>(a, d_workspace, st);
    default: return launch_int8<__nv_bfloat16>(a, d_workspace, st);
  }
}

}  // extern "C"
