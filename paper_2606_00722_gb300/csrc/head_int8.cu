// The head in 8-bit integers: rounding of rows to 8 bits with a scale for each, and
// logits z[r][v] = (sum_k q[r][k] w[v][k]) s[r] S[v].
//
// Sums are whole numbers and exact, so logits do not depend on the order of the
// sum; each is rounded to 32 bits as it is scaled and once to its type.
#include <cuda.h>

#include <algorithm>

#include "../../include/epic.h"
#include "head_launch.cuh"
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

// |v| as a whole number of the same order, NaN above infinity
__device__ __forceinline__ uint32_t size_order(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A CTA a row: the largest size in one pass, the quotients in a second one, from the caches.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads) k_quantize_rows(QuantArgs a) {
  constexpr int E = Chunk<T>::kCount;
  __shared__ uint32_t s_top[kQuantThreads / 32];
  follow();
  let_next();
  const long long r = blockIdx.x, b = r / a.k;
  const int at = a.pos ? a.pos[r] : (int)(r % a.k);
  int8_t* q = a.q + r * a.d;
  if (at < 0 || at >= a.n) {
    for (int k = threadIdx.x; k < a.d; k += kQuantThreads) q[k] = 0;
    if (threadIdx.x == 0) a.scale[r] = CUDART_NAN_F;
    return;
  }
  const T* x = (const T*)a.x + b * a.stride_b + at * a.stride_n;
  const bool whole = (uintptr_t)x % 16 == 0, words = (uintptr_t)q % 4 == 0;
  uint32_t top = 0;
#pragma unroll 2
  for (int k = threadIdx.x * E; k < a.d; k += kQuantThreads * E) {
    const Chunk<T> c(x + k, a.d - k, whole);
#pragma unroll
    for (int i = 0; i < E; i++) top = max(top, size_order(c.v[i]));
  }
  top = __reduce_max_sync(~0u, top);
  if (threadIdx.x % 32 == 0) s_top[threadIdx.x / 32] = top;
  __syncthreads();
  for (int w = 0; w < kQuantThreads / 32; w++) top = max(top, s_top[w]);
  const float s = __fdiv_rn(__uint_as_float(top), 127.0f);
  if (threadIdx.x == 0) a.scale[r] = s;
#pragma unroll 2
  for (int k = threadIdx.x * E; k < a.d; k += kQuantThreads * E) {
    const Chunk<T> c(x + k, a.d - k, whole);
    uint32_t w[E / 4] = {};
#pragma unroll
    for (int i = 0; i < E; i++) {
      const float v = rintf(__fdiv_rn(c.v[i], s));
      const int n = s > 0.0f && v == v ? (int)fminf(fmaxf(v, -127.0f), 127.0f) : 0;
      w[i / 4] |= (uint32_t)(n & 255) << i % 4 * 8;
    }
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      if (words && k + i + 4 <= a.d) {
        *(uint32_t*)(q + k + i) = w[i / 4];
      } else {
        for (int j = 0; j < 4; j++)
          if (k + i + j < a.d) q[k + i + j] = (int8_t)(w[i / 4] >> j * 8);
      }
    }
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
  long long wait;    // limit of a wait, in clocks
  const int* sizes;  // [rows][ceil(d / 1024)], added up over 1,024 each
};

// ---- few rows: a warp's lanes along tokens' rows, whole-number products of four bytes an instruction
//
// The head is read once: 126,000 x 4,096 bytes for one row in 84 us (6.1 TB/s), for eight, whose products take nearly as long
// as the bytes, in 108.  A warp has four tokens at a time, so that what it reads of the hidden states in shared memory
// serves four.  A row's last 16 bytes may hold bytes behind it: hidden states there are 0.
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
  follow();
  let_next();
  const int lane = threadIdx.x % 32, chunks = (a.d + 15) / 16;
  if (a.d % 16 == 0 && (uintptr_t)a.q % 16 == 0) {
#pragma unroll 4
    for (int i = threadIdx.x; i < R * chunks; i += kFewThreads)
      s_q[i] = i < a.rows * chunks ? ((const int4*)a.q)[i] : make_int4(0, 0, 0, 0);
  } else {
    for (int r = 0; r < R; r++)
#pragma unroll 4
      for (int c = threadIdx.x; c < chunks * 16; c += kFewThreads)
        ((int8_t*)s_q)[r * chunks * 16 + c] = r < a.rows && c < a.d ? a.q[(long long)r * a.d + c] : 0;
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

// 128 * 128 * kMostProducts is the largest sum that 32 bits hold
constexpr int kMostProducts = 131071;

// ---- many rows: on the tensor units
//
// This GPU's tensor units have no fast products of 8-bit integers, but a product of two of them in fp16 is exact, and so are
// sums in 32-bit floats up to 2^24: of 1,024 products, or of twice as many, four times and so on if 128 times the sum of as
// many of a row's sizes stays within it in every row (for normally distributed rows, some 4,000).  Then sums are taken over
// into 32-bit integers.  A pair of CTAs makes 256 tokens x up to 256 rows.  The head's bytes come into a queue in shared
// memory, by boxes or, where rows start anywhere, by copies of the work warps' own, from the aligned 16 bytes that a row's
// part begins in to those that it ends in; the work warps turn them into fp16 (byte + 128 in the low bits of 1024.0, less
// 1152) in tensor memory, where the tensor units take them from.  Hidden states are turned once, in the workspace, and come
// by boxes.  Each of four teams of four warps turns every fourth step, so that four chains of loads, stores and arrivals
// overlap.
//
// What was tried before: an operand in shared memory with copies of the work warps' own, which every fence between what a
// warp writes and the tensor units waits for, 1.5 us a step; a bulk copy for every row, 1.2 us; arrivals released to the
// whole cluster, 1.3 us; one chain, 0.6 us; the operand in shared memory, where it is written and read on top of the queue
// and the hidden states, 80 KB a step, 0.41 us.
constexpr int kWorkWarps = 16, kWork = 32 * kWorkWarps, kThreads = kWork + 128;
constexpr int kTileTokens = 256, kHalf = 128, kStepK = 64, kRing = 8, kTeams = 4, kExactSteps = 1024 / kStepK;
constexpr int kTeam = kWorkWarps / kTeams;  // warps
constexpr int kOperand = kHalf * kStepK * 2;  // bytes of a step of hidden states
// A unit of the queue: 64 bytes of each token by a box; or 80, of a warp's 32 tokens, that the warp copies for itself
template <bool kAskew>
struct Queue {
  static constexpr int kRow = kAskew ? 80 : 64, kUnit = kHalf * kRow, kUnits = kAskew ? 8 : 10;
};
constexpr int kQueue = 10 * kHalf * 64;
static_assert(Queue<true>::kUnits * Queue<true>::kUnit <= kQueue, "the queue of either form has its place");
constexpr int kAhead = Queue<true>::kUnits / kTeams;  // steps of its team that a warp has places for
constexpr int kShared = kRing * kOperand + kQueue + 1024;
constexpr int kPairs = 76;

struct Int8Bars {
  uint64_t full[kRing], empty[kRing], sums_full[2], sums_empty[2], come[10], gone[10];
  uint32_t sums, gave_up;
  int most[8];
};

// 16 bytes at multiples of 16, of which the first `bytes` are read and the rest is 0
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
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
// NaN to the logits of all of a pair's tiles, a thread a token.  (Sizes are hidden from the compiler, which else keeps what it knows
// of them in registers through the whole kernel.)
template <typename T, int kRows>
__device__ __forceinline__ void spoil_tiles(const Int8Args& a) {
  int rows = a.rows, V = a.V, t = blockIdx.x / 2, at = threadIdx.x;
  asm volatile("" : "+r"(rows), "+r"(V), "+r"(t), "+r"(at));
  const int row_tiles = (rows + kRows - 1) / kRows, tiles = (int)((V + (long long)kTileTokens - 1) / kTileTokens) * row_tiles;
  for (; t < tiles; t += kPairs) {
    const long long v = (long long)(t / row_tiles) * kTileTokens + cluster_rank() * kHalf + at % kHalf;
    const int r0 = t % row_tiles * kRows;
    for (int r = r0 + at / kHalf; r < min(r0 + kRows, rows); r += kWork / kHalf)
      if (v < a.V) ((T*)a.logits)[r / a.k * a.stride_b + r % a.k * a.stride_n + v] = of_float<T>(CUDART_NAN_F);
  }
}

// kRows: rows of a tile.  kAskew: rows of the head start anywhere.
template <typename T, int kRows, bool kAskew>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_int8_tiles(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap head_map,
                 const __grid_constant__ Int8Args a) {
  typedef Queue<kAskew> Q;
  extern __shared__ uint8_t shared_raw[];
  __shared__ Int8Bars bars;
  const uint32_t ring = (smem_address(shared_raw) + 1023) / 1024 * 1024;
  const uint32_t queue = ring + kRing * kOperand;
  const int warp = warp_of_thread(), lane = threadIdx.x % 32, pair = blockIdx.x / 2;
  const uint32_t rank = cluster_rank();
  const uint32_t full = smem_address(bars.full), empty = smem_address(bars.empty);
  const uint32_t sums_full = smem_address(bars.sums_full), sums_empty = smem_address(bars.sums_empty);
  const uint32_t come = smem_address(bars.come), gone = smem_address(bars.gone);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kRing; s++) {
      bar_init(full + 8 * s, 1 + 2 * kTeam);
      bar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < Q::kUnits; s++) {
      bar_init(come + 8 * s, 1);
      bar_init(gone + 8 * s, kTeam);
    }
    for (int s = 0; s < 2; s++) {
      bar_init(sums_full + 8 * s, 1);
      bar_init(sums_empty + 8 * s, 2 * kWorkWarps);
    }
    for (int& m : bars.most) m = 0;
    bars.gave_up = 0;
    bar_init_visible();
  }
  if (warp == kWorkWarps) sums_take_pair(smem_address(&bars.sums));
  __syncthreads();
  follow();
  let_next();
  if (a.d > kExactSteps * kStepK) {
    // the largest sums of 2, 4, 8 .. blocks of a row's sizes
    const int blocks = (a.d + kExactSteps * kStepK - 1) / (kExactSteps * kStepK);
    for (int l = 1; 1 << (l - 1) < blocks; l++) {
      int most = 0;
      for (int r = threadIdx.x; r < a.rows; r += kThreads)
        for (int b = 0; b < blocks; b += 1 << l) {
          int sum = 0;
          for (int i = b; i < min(b + (1 << l), blocks); i++) sum += a.sizes[(long long)r * blocks + i];
          most = max(most, sum);
        }
      most = __reduce_max_sync(~0u, most);
      if (lane == 0) atomicMax(&bars.most[l], most);
    }
  }
  products_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  const uint32_t sums = bars.sums;
  const int row_tiles = (a.rows + kRows - 1) / kRows, steps = (a.d + kStepK - 1) / kStepK;
  int exact = kExactSteps;  // steps whose sums are exact
  for (int l = 1; exact < steps && bars.most[l] <= (1 << 24) / 128; l++) exact *= 2;
  const int tiles = (int)((a.V + (long long)kTileTokens - 1) / kTileTokens) * row_tiles;
  constexpr int kBoxBytes = kRows / 2 * kStepK * 2;
  // tensor memory: sums, twice if they leave room for the operand's ring in the last 256 columns
  constexpr int kSums = kRows == 256 ? 1 : 2;
  const uint32_t operands = sums + 256;
  bool ok = a.wait > 0;

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
          if (!(ok = bar_wait(empty + 8 * s, turn ^ 1, a.wait))) break;
          if (rank == 0) bar_expect(full + 8 * s, 2 * kBoxBytes);
          load_box_pair(&q_map, ring + s * kOperand, full0 + 8 * s, k * kStepK, r0);
          if (++s == kRing) s = 0, turn ^= 1;
        }
      }
    }
    if (!kAskew && warp == kWorkWarps + 2 && lane == 0) {  // boxes of the head's bytes
      int s = 0;
      uint32_t turn = 0;
      for (int t = pair; ok && t < tiles; t += kPairs) {
        const int v0 = t / row_tiles * kTileTokens + rank * kHalf;
        for (int k = 0; k < steps; k++) {
          if (!(ok = bar_wait(gone + 8 * s, turn ^ 1, a.wait))) break;
          bar_expect(come + 8 * s, Q::kUnit);
          load_box(&head_map, queue + s * Q::kUnit, come + 8 * s, k * kStepK, v0);
          if (++s == Q::kUnits) s = 0, turn ^= 1;
        }
      }
    }
    if (warp == kWorkWarps + 1 && rank == 0) {  // products
      constexpr uint32_t kind = product_kind(false, false, false, kTileTokens, kRows);
      int s = 0, use = 0;
      uint32_t turn = 0;
      for (int t = pair; ok && t < tiles; t += kPairs) {
        for (int k = 0; ok && k < steps; use++) {
          const int half = use % kSums, end = min(k + exact, steps);
          if (!(ok = bar_wait_warp(sums_empty + 8 * half, (use / kSums & 1) ^ 1, a.wait))) break;
          products_fence_after();
          for (bool add = false; k < end; k++) {
            if (!(ok = bar_wait_warp(full + 8 * s, turn, a.wait))) break;
            products_fence_after();
            if (one_lane()) {
              const uint64_t b = operand_k(ring + s * kOperand);
#pragma unroll
              for (int j = 0; j < kStepK / 16; j++)
                product_pair_in(sums + half * kRows, operands + s * 32 + j * 8, b + j * kNextK, kind, add || j);
              products_arrive_pair(empty + 8 * s);
            }
            __syncwarp();
            add = true;
            if (++s == kRing) s = 0, turn ^= 1;
          }
          if (ok && one_lane()) products_arrive_pair(sums_full + 8 * half);
          __syncwarp();
        }
      }
    }
  } else {
    if (kRows == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    constexpr int kCols = kRows / 4;               // a warp's rows of logits
    constexpr int kLoad = kCols < 32 ? kCols : 32;  // at a time
    constexpr int kPiece = 8, kPieces = kCols / kPiece;
    const int quarter = warp % 4, team = warp / 4, token = quarter * 32 + lane;  // of the CTA's
    const uint32_t full0 = at_rank(full, 0), sums_empty0 = at_rank(sums_empty, 0);
    const uint32_t lanes = (uint32_t)quarter * 32 << 16, from = sums + lanes + team * kCols;
    const int own = (tiles - pair + kPairs - 1) / kPairs, per = (steps + exact - 1) / exact;  // tiles, takes each
    int acc[kCols];
    int use = 0, past = min(exact, steps), out = kPieces;  // the next sums to take over, the step past them, the piece to write

    // The tile before the next sums': its logits are written 8 rows at a time between the steps of the next tile.
    T* z = nullptr;           // the next logit of the lane's token,
    int left = 0, zi = 0;     // how many rows exist; the position of the next one
    float S = 0.0f, scales[(kCols + 31) / 32];  // of the token; of the rows, a lane a row
    bool there = false;
    auto write = [&] {
#pragma unroll
      for (int p = 0; p < kPieces; p++) {
        if (p != out) continue;
#pragma unroll
        for (int c = p * kPiece; c < p * kPiece + kPiece; c++) {
          const float x = (float)acc[c] * __shfl_sync(~0u, scales[c / 32], c % 32) * S;
          if (c < left && there) *z = of_float<T>(x);
          z += a.stride_n;
          if (++zi == a.k) {
            z += a.stride_b - a.k * a.stride_n;
            zi = 0;
          }
        }
      }
      out++;
    };
    auto take = [&] {
      const int half = use % kSums;
      if (!(ok = bar_wait_warp(sums_full + 8 * half, use / kSums & 1, a.wait))) return;
      products_fence_after();
      const bool first = use % per == 0;
#pragma unroll
      for (int c = 0; c < kCols; c += kLoad) {
        float v[kLoad];
        sums_load(from + half * kRows + c, v);
        sums_loaded(v);
#pragma unroll
        for (int i = 0; i < kLoad; i++) acc[c + i] = (first ? 0 : acc[c + i]) + __float2int_rn(v[i]);
      }
      products_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(sums_empty0 + 8 * half);
      const int tile = use / per;
      past = min((tile + 1) * steps, past + exact);
      if (++use % per == 0) {
        past = (tile + 1) * steps + min(exact, steps);
        out = 0;
        const int t = pair + tile * kPairs, r0 = t % row_tiles * kRows + team * kCols;
        const long long v = (long long)(t / row_tiles) * kTileTokens + rank * kHalf + token;
        there = v < a.V;
        left = a.rows - r0;
        S = there ? a.head_scale[v] : 0.0f;
#pragma unroll
        for (int c = 0; c < kCols; c += 32) scales[c / 32] = c + lane < left ? a.scale[r0 + c + lane] : 0.0f;
        zi = r0 % a.k;
        z = (T*)a.logits + r0 / a.k * a.stride_b + zi * a.stride_n + v;
      }
    };

    // n: the team's next step of all, step k of the pair's tile `tile`
    int n = team, tile = n / steps, k = n % steps;

    // A warp's own copies of its 32 tokens' bytes, 5 chunks of 16 each, kAhead - 1 steps of its team ahead: step ahead_k of
    // the pair's tile ahead_tile, into its part of place `ahead`
    int ahead = team, ahead_tile = tile, ahead_k = k;
    auto copy = [&] {
      if (ahead_tile < own) {
        const int v0 = (pair + ahead_tile * kPairs) / row_tiles * kTileTokens + rank * kHalf + quarter * 32;
#pragma unroll
        for (int i = 0; i < 5; i++) {
          const int chunk = i * 32 + lane, row = chunk / 5, v = min(v0 + row, a.V - 1);
          const uintptr_t w = (uintptr_t)(a.head + v * a.head_stride + ahead_k * kStepK), end = w + (a.d - ahead_k * kStepK);
          const uintptr_t first = w & ~(uintptr_t)15, from = first + chunk % 5 * 16;
          copy16(queue + ahead * Q::kUnit + (quarter * 32 * 5 + chunk) * 16, (const void*)(from < end ? from : first),
                 from < end ? (int)min((uintptr_t)16, end - from) : 0);
        }
        if ((ahead += kTeams) >= Q::kUnits) ahead = team;
        for (ahead_k += kTeams; ahead_k >= steps; ahead_k -= steps) ahead_tile++;
      }
      copies_commit();
    };
    if (kAskew)
      for (int i = 1; i < kAhead; i++) copy();
    while (ok) {
      // sums are taken over before the step in whose place this one comes waits for theirs
      const bool due = use < own * per && (tile >= own || past + kRing <= n);
      if (out < kPieces) {
        write();
        if (due || tile >= own) continue;
      } else if (due) {
        take();
        continue;
      }
      if (tile >= own) break;
      const int s = n % kRing, place = n % Q::kUnits;
      const uint32_t at = queue + place * Q::kUnit + token * Q::kRow;
      if (kAskew) {
        copy();
        copies_wait<kAhead - 1>();
        __syncwarp();
      } else {  // (lanes agree behind the step's work, within its memory: here it costs 1.6 % of 4,096 rows through 126,000 x 2,048)
        ok = bar_wait(come + 8 * place, n / Q::kUnits & 1, a.wait);
      }
      ok &= bar_wait(empty + 8 * s, (n / kRing & 1) ^ 1, a.wait);
      products_fence_after();
      uint32_t m = 0;  // bytes ahead of the token's row in its first 16
      if (kAskew) {
        const uint32_t v = (uint32_t)((pair + tile * kPairs) / row_tiles) * kTileTokens + rank * kHalf + token;
        m = ((uint32_t)(uintptr_t)a.head + v * (uint32_t)a.head_stride) & 15;
      }
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        uint32_t x[16];
#pragma unroll
        for (int j = 0; j < 2; j++) {
          uint4 w = load_shared(kAskew ? at + (i + j) * 16 : at + ((i + j) ^ (token >> 1 & 3)) * 16);
          if (kAskew) w = shifted(w, load_shared(at + (i + j + 1) * 16), m);
          const uint32_t y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int c = 0; c < 4; c++) {
            const uint2 h = halves_of(y[c]);
            x[8 * j + 2 * c] = h.x, x[8 * j + 2 * c + 1] = h.y;
          }
        }
        operand_store(operands + lanes + s * 32 + i * 8, x);
      }
      operand_stored();
      products_fence_before();
      if (!(ok = all_came(ok))) break;
      if (lane == 0) {
        bar_arrive_cluster(full0 + 8 * s);
        if (!kAskew) bar_arrive(gone + 8 * place, 1);
      }
      n += kTeams;
      for (k += kTeams; k >= steps; k -= steps) tile++;
    }
  }
  if (!ok) give_up(smem_address(&bars.gave_up));
  products_fence_before();
  __syncwarp();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  if (*(volatile uint32_t*)&bars.gave_up) {  // in both CTAs, or in neither
    let_all_end();
    __syncthreads();
    if (warp < kWorkWarps) spoil_tiles<T, kRows>(a);  // (the other warps lack the registers)
    __syncthreads();
    cluster_arrive();
    cluster_wait();
  }
  if (warp == kWorkWarps) sums_free_pair(sums);
}

// Hidden states of 8 bits as fp16, rows of a multiple of 16 bytes, a CTA a row; and their sizes, added up over 1,024 each
__global__ void __launch_bounds__(256) k_rows_as_halves(const int8_t* q, __half* to, int d, int ld, int* sizes) {
  __shared__ uint32_t s_sum[kMostProducts / 1024 + 1];
  follow();
  let_next();
  const int blocks = (d + 1023) / 1024;
  for (int i = threadIdx.x; i < blocks; i += 256) s_sum[i] = 0;
  __syncthreads();
  const int8_t* x = q + (long long)blockIdx.x * d;
  uint2* y = (uint2*)(to + (long long)blockIdx.x * ld);
  const bool words = (uintptr_t)x % 4 == 0;
#pragma unroll 2
  for (int k = threadIdx.x * 4, i = 0; i < blocks; k += 1024, i++) {
    uint32_t w = 0;
    if (words && k + 4 <= d) {
      w = *(const uint32_t*)(x + k);
    } else {
      for (int j = 0; j < 4; j++)
        if (k + j < d) w |= (uint32_t)(uint8_t)x[k + j] << 8 * j;
    }
    if (k < ld) y[k / 4] = halves_of(w);
    const uint32_t sum = __reduce_add_sync(~0u, __dp4a(__vabs4(w), 0x01010101u, 0u));  // 128 is a byte, too
    if (threadIdx.x % 32 == 0) atomicAdd(&s_sum[i], sum);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < blocks; i += 256) sizes[(long long)blockIdx.x * blocks + i] = (int)s_sum[i];
}

// ---- on the host

template <typename T, int R>
epic_status launch_few(const Int8Args& a, cudaStream_t st) {
  const int bytes = R * ((a.d + 15) / 16) * 16;
  const long long ctas = (a.V + (long long)kFewThreads / 32 * kFewTokens - 1) / (kFewThreads / 32 * kFewTokens);
  return launch_next(k_few_logits<T, R>, (unsigned)std::min(ctas, 152ll * 4), kFewThreads, bytes, kFewBytes, st, a);
}

template <typename T, int kRows>
epic_status launch_tiles(const Int8Args& a, __half* q16, int ld, bool askew, cudaStream_t st) {
  CUtensorMap map;
  if (!make_map(&map, false, q16, ld, a.rows, ld, kRows / 2)) return EPIC_ERR_CUDA;
  CUtensorMap head = map;  // of a head that lies askew: unused
  if (!askew && !make_byte_map(&head, a.head, a.d, a.V, a.V > 1 ? a.head_stride : (a.d + 15) / 16 * 16, kHalf))
    return EPIC_ERR_CUDA;
  const auto kernel = askew ? k_int8_tiles<T, kRows, true> : k_int8_tiles<T, kRows, false>;
  return launch_next(kernel, 2 * kPairs, kThreads, kShared, kShared, st, map, head, a);
}

bool head_lies_askew(const int8_t* head, long long stride, int V) {
  return (uintptr_t)head % 16 != 0 || (V > 1 && (stride % 16 != 0 || stride >= 1ll << 39));
}

// One, four and eight rows through 126,000 x 4,096 take 84, 98 and 108 us so and 114 in tiles, four and eight through 50,000 x
// 1,024 12 and 16, in tiles 19.
bool few_rows(long long rows, int d, bool askew) {
  return rows <= kFewRows && !askew && (rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8) * (d + 15ll) <= kFewBytes;
}

size_t sizes_bytes(long long rows, int d) { return (size_t)(rows * ((d + 1023) / 1024) * 4 + 255) / 256 * 256; }

// Rows of a tile: a step takes the tensor units 2 clocks a row, and about 320 at least for the head's bytes.  Tiles of 64, 128
// and 256 rows (us): 64 rows through 32,768 x 2,048 24, 27, 34; 128 rows 39, 27, 34; through 50,000 x 1,024, 165 rows 41, 37,
// 36; 300 rows 62, 48, 61.
int tile_rows(long long rows) {
  int best = 256;
  long long least = -1;
  for (const int n : {256, 128, 64, 32}) {
    const long long cost = (rows + n - 1) / n * std::max(2 * n, 320);
    if (least < 0 || cost <= least) best = n, least = cost;
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
  a.wait = wait_limit();
  int* sizes = (int*)ws;
  __half* q16 = (__half*)((char*)ws + sizes_bytes(a.rows, a.d));
  const int ld = (a.d + 7) / 8 * 8;
  a.sizes = sizes;
  const epic_status s = launch_next(k_rows_as_halves, a.rows, 256, 0, kNoCache, st, a.q, q16, a.d, ld, sizes);
  if (s != EPIC_OK) return s;
  switch (tile_rows(a.rows)) {
    case 32: return launch_tiles<T, 32>(a, q16, ld, askew, st);
    case 64: return launch_tiles<T, 64>(a, q16, ld, askew, st);
    case 128: return launch_tiles<T, 128>(a, q16, ld, askew, st);
    default: return launch_tiles<T, 256>(a, q16, ld, askew, st);
  }
}

bool bad_type(int dtype) { return dtype != EPIC_F32 && dtype != EPIC_F16 && dtype != EPIC_BF16; }
size_t size_of(int dtype) { return dtype == EPIC_F32 ? 4 : 2; }

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
    case EPIC_F32: return launch_next(k_quantize_rows<float>, (unsigned)rows, kQuantThreads, 0, kCache, st, a);
    case EPIC_F16: return launch_next(k_quantize_rows<__half>, (unsigned)rows, kQuantThreads, 0, kCache, st, a);
    default: return launch_next(k_quantize_rows<__nv_bfloat16>, (unsigned)rows, kQuantThreads, 0, kCache, st, a);
  }
}

epic_status epic_int8_logits_workspace(int32_t B, int32_t k, int32_t d, int32_t V, const int8_t* d_head,
                                       int64_t head_stride, size_t* bytes) {
  using namespace epic;
  if (!bytes || B < 0 || k < 0 || d < 1 || V < 0 || (V > 1 && head_stride < d)) return EPIC_ERR_INVALID_ARG;
  if (d > kMostProducts || V > 0x7fffffff - 4096 || (long long)B * k > kMostRows) return EPIC_ERR_CAPACITY;
  const long long rows = (long long)B * k;
  *bytes = 256;
  if (!few_rows(rows, d, head_lies_askew(d_head, head_stride, V)))
    *bytes = std::max(*bytes, sizes_bytes(rows, d) + (size_t)rows * ((d + 7) / 8 * 8) * 2);
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
  const Int8Args a = {d_q, d_scale, d_head, head_stride, d_head_scale, d_logits, stride_b, stride_n, (int)rows, k, d, V};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (dtype) {
    case EPIC_F32: return launch_int8<float>(a, d_workspace, st);
    case EPIC_F16: return launch_int8<__half>(a, d_workspace, st);
    default: return launch_int8<__nv_bfloat16>(a, d_workspace, st);
  }
}

}  // extern "C"
