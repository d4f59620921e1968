// Softmax cross entropy through a head, without the logits: hidden states [B][n][d], head [V][d].
//
// Per position that counts, with z = W h, y its target, w its weight and g the
// gradient from above:
//   loss = w (lse - z_y),  lse = log sum_v exp z_v
//   dz_v = w g (exp(z_v - lse) - [v = y]),  dh = dz W,  dW = sum over positions of dz h
//
// A call goes through its positions in pieces.  Of each, the positions that
// count are packed (masked training leaves out half and more), then
//   forward:   logits -> records (sums of exponentials by column range) -> loss
//   step:      logits -> records and exponentials e, relative to a reference known before (the target's logit, from a
//              product of two rows) -> loss, and each row's sum S -> dh = (w / S) e W, dW = e^T (h w / S)
//   backward:  logits -> gradients of logits e = g exp(z - lse) from the forward call's lse -> dh = e W, dW = e^T h
// so a step makes the logits once.  e is kept for a piece in 16 bits, like the operands of the products that read it: one
// rounding of at most 2^-8 (bf16) or 2^-11 (fp16), independent ones that a sum over many evens out; so is h w / S, where a
// step multiplies hidden states.  (To round e alone there, the sums would have to be known before e is written: the logits
// made twice, a third more work.)  Rows of a step whose exponentials leave the range, and all of an fp16 step, which has
// not the range at all, get their gradients of logits from the logsumexp in a second pass.  At the target, e - S cancels
// where the model is sure, and is most of a row's gradient: it is minus the sum of the others, summed apart, and comes to the
// sums in 32 bits as they leave the tensor units.
// Sums, references and losses are 32 bits.
#include <stdlib.h>

#include <algorithm>
#include <type_traits>

#include "head_launch.cuh"
#include "head_loss.h"
#include "head_rows.cuh"

namespace epic {
namespace {

constexpr int kPieceRows = 16384;  // most positions of a piece
constexpr int kRowsThreads = 256;
constexpr int kFewRows = 608;   // positions that have a CTA each; see run_head
// More positions are counted by a kernel before, else by every CTA.  Steps with and without (us): 640 positions through 1,000 x 256
// 33 and 31, 1,024 33 and 32, 4,096 45 and 45, 8,192 66 and 68; through 8,000 x 2,048 1,024 120 and 120, 4,096 290 and 292, 8,192 558
// and 564.
constexpr int kCounted = 1024;

struct RowsArgs {
  HeadPlan p;
  const void* hidden;
  long long stride_b, stride_n;
  long long r0;  // first position of the piece
  int n;
  const int32_t* target;
  const float* weight;    // or NULL
  const float* up;        // the backward pass, else NULL
  const float* lse;       // the backward pass, else NULL
  float *loss, *lse_out;  // of positions that do not count: 0; or NULL
  HiddenGrad out;         // grad NULL: none
  int per;                // positions of a CTA, a power of two up to 256
  bool probs;             // rows' references are wanted (a step in bf16)
  bool scaled;            // fp16: gradients of logits relative to the largest factor, times 2^14
  bool again;             // gradients of logits are from a known logsumexp
};

__device__ __forceinline__ float row_factor(const RowsArgs& a, long long r) {
  const int y = a.target[r];
  if (y < 0 || y >= a.p.V) return 0.0f;
  const float w = a.weight ? a.weight[r] : 1.0f;
  return w == 0.0f ? 0.0f : a.up ? w * a.up[r] : w;
}

// Smallest power of two that is not below x > 0, of finite x within 2^-100 .. 2^100; 1 otherwise
__device__ __forceinline__ float pow2_above(float x) {
  if (!(x > 7.9e-31f && x < 1.2e30f)) return 1.0f;
  return pow2_whole((float)(((__float_as_int(x) + 0x7fffff) >> 23) - 127));
}

constexpr float kHalfScale = 14.0f;  // of a row's gradient, 2^-28 of its factor is still a normal number of fp16

// How gradients of logits come from a known logsumexp
__device__ __forceinline__ void know(const HeadPlan& p, int q, float lse, float g, float post) {
  float ref = rintf(lse * kLog2E);
  if (!(fabsf(ref) < 3.0e38f)) ref = 0.0f;
  p.known_ref[q] = ref;
  p.known_mul[q] = g / post * ex2(fmaf(-lse, kLog2E, ref));
}

__device__ __forceinline__ void sum_and_top(int& count, float& top) {
  for (int o = 16; o; o >>= 1) {
    count += __shfl_xor_sync(~0u, count, o);
    top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  }
}

// How many of 256 positions count, and their largest factor
__global__ void __launch_bounds__(kRowsThreads) k_head_count(RowsArgs a) {
  __shared__ int s_count[kRowsThreads / 32];
  __shared__ float s_top[kRowsThreads / 32];
  follow();
  let_next();
  const int i = blockIdx.x * kRowsThreads + threadIdx.x;
  float top = i < a.p.rows ? fabsf(row_factor(a, a.r0 + i)) : 0.0f;
  int count = top != 0.0f;
  sum_and_top(count, top);
  if (threadIdx.x % 32 == 0) s_count[threadIdx.x / 32] = count, s_top[threadIdx.x / 32] = top;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  count = threadIdx.x < kRowsThreads / 32 ? s_count[threadIdx.x] : 0;
  top = threadIdx.x < kRowsThreads / 32 ? s_top[threadIdx.x] : 0.0f;
  sum_and_top(count, top);
  if (threadIdx.x == 0) a.p.counts[blockIdx.x] = count, a.p.tops[blockIdx.x] = top;
}

// Packs the positions that count.  Every CTA counts those before its own, so nothing waits; it also finds the largest
// factor.  A warp copies a row, or with few rows a CTA (kWide), and with `probs` takes its product with the target's row of
// the head.
template <typename T, bool kWide>
__global__ void __launch_bounds__(kRowsThreads) k_head_rows(RowsArgs a) {
  __shared__ int s_before[kRowsThreads / 32], s_all[kRowsThreads / 32];
  __shared__ float s_top[kRowsThreads / 32], s_dot[kRowsThreads / 32];
  follow();
  let_next();
  const HeadPlan& p = a.p;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = kRowsThreads / 32;
  const int first = blockIdx.x * a.per, last = min(first + a.per, p.rows);
  int before = 0, all = 0;
  float top = 0.0f;
  if (p.rows > kCounted) {
    const int own = first / kRowsThreads;
    if (threadIdx.x * kRowsThreads < p.rows) {
      all = p.counts[threadIdx.x];
      top = p.tops[threadIdx.x];
      if (threadIdx.x < own) before = all;
    }
    const int i = own * kRowsThreads + threadIdx.x;
    if (i < first) before += row_factor(a, a.r0 + i) != 0.0f;
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < p.rows; i += kRowsThreads) {
      const float f = row_factor(a, a.r0 + i);
      all += f != 0.0f;
      before += f != 0.0f && i < first;
      top = fmaxf(top, fabsf(f));
    }
  }
  sum_and_top(all, top);
  before = __reduce_add_sync(~0u, before);
  if (lane == 0) s_before[warp] = before, s_all[warp] = all, s_top[warp] = top;
  __syncthreads();
  before = all = 0, top = 0.0f;
  for (int w = 0; w < warps; w++) before += s_before[w], all += s_all[w], top = fmaxf(top, s_top[w]);
  const float post = a.scaled ? pow2_above(top) * pow2_whole(-kHalfScale) : 1.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.count = all, *p.again = a.again, *p.post = post;

  const int at = kWide ? threadIdx.x : lane, step = kWide ? kRowsThreads : 32;  // in a row
  for (int i0 = first; i0 < last; i0 += 32) {
    const long long mine = i0 + lane;
    const float f = mine < last ? row_factor(a, a.r0 + mine) : 0.0f;
    const unsigned there = __ballot_sync(~0u, f != 0.0f);
    for (int j = kWide ? 0 : warp; j < min(32, last - i0); j += kWide ? 1 : warps) {
      const long long i = i0 + j, r = a.r0 + i, b = r / a.n, pos = r % a.n;
      const float g = __shfl_sync(~0u, f, j);
      if (g == 0.0f) {
        if (at == 0 && a.loss) a.loss[r] = 0.0f;
        if (at == 0 && a.lse_out) a.lse_out[r] = 0.0f;
        if (a.out.grad) {
          T* o = (T*)a.out.grad + b * a.out.stride_b + pos * a.out.stride_n;
          const int words = (uintptr_t)o % 16 == 0 ? p.d / 8 : 0;
          for (int k = at; k < words; k += step) ((uint4*)o)[k] = make_uint4(0, 0, 0, 0);
          for (int k = words * 8 + at; k < p.d; k += step) o[k] = of_float<T>(0.0f);
        }
        continue;
      }
      const int q = before + __popc(there & ((1u << j) - 1)), y = a.target[r];
      const T* h = (const T*)a.hidden + b * a.stride_b + pos * a.stride_n;
      const T* w = (const T*)p.head + y * p.ldw;
      uint4* hc = (uint4*)((T*)p.hc + q * p.ldh);
      float dot = 0.0f;
      const bool whole = (uintptr_t)h % 16 == 0;
#pragma unroll 4
      for (int k = at * 8; k < p.ldh; k += step * 8) {
        const Chunk<T> x(h + k, p.d - k, whole);
        uint4 v;
        T* t = (T*)&v;
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = of_float<T>(x.v[i]);
        hc[k / 8] = v;
        if (a.probs) {
          const Chunk<T> y(w + k, p.d - k, true);
#pragma unroll
          for (int i = 0; i < 8; i++) dot = fmaf(x.v[i], y.v[i], dot);
        }
      }
      if (a.probs) {
        for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(~0u, dot, o);
        if (kWide) {
          if (lane == 0) s_dot[warp] = dot;
          __syncthreads();
          dot = 0.0f;
          for (int w = 0; w < warps; w++) dot += s_dot[w];
        }
      }
      if (at == 0) {
        p.src[q] = (int)i;
        p.to[q] = b * a.out.stride_b + pos * a.out.stride_n;
        p.tgt[q] = y;
        p.g[q] = g;
        if (a.probs) p.ref[q] = whole_ref(dot);
        if (a.lse) know(p, q, a.lse[r], g, post);
      }
    }
    before += __popc(there);
  }
  // rows up to the end of the tile
  const int end = (all + kRowTile - 1) / kRowTile * kRowTile;
  for (int q = all + blockIdx.x * warps + warp; q < end; q += gridDim.x * warps)
    for (int k = lane * 8; k < p.ldh; k += 256) {
      *(uint4*)((T*)p.hc + q * p.ldh + k) = make_uint4(0, 0, 0, 0);
      if (p.hs) *(uint4*)((T*)p.hs + q * p.ldh + k) = make_uint4(0, 0, 0, 0);
    }
}

constexpr int kMeetWarps = 8;

struct MeetArgs {
  HeadPlan p;
  long long r0;
  const float* weight;
  float *loss, *lse;  // by position, or NULL
  bool grads;         // factors are wanted, and hs
  bool stored;        // e is there
  bool known;         // as gradients of logits
};

// Each of the CTA's kMeetRows rows counts those before it with the same target, and is listed if they are few.  rank: how many
// they are; complete after the CTA's next barrier.
template <int kMeetRows>
__device__ __forceinline__ void list_targets(const HeadPlan& p, int n, int q0, int (&rank)[kMeetRows]) {
  __shared__ int s_count[kMeetWarps][kMeetRows];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int target[kMeetRows], count[kMeetRows];
#pragma unroll
  for (int i = 0; i < kMeetRows; i++) target[i] = q0 + i < n ? p.tgt[q0 + i] : -1, count[i] = 0;
#pragma unroll 4
  for (int q = threadIdx.x; q < min(n, q0 + kMeetRows); q += kMeetWarps * 32) {
    const int t = p.tgt[q];
#pragma unroll
    for (int i = 0; i < kMeetRows; i++) count[i] += t == target[i] && q < q0 + i;
  }
#pragma unroll
  for (int i = 0; i < kMeetRows; i++) {
    count[i] = __reduce_add_sync(~0u, count[i]);
    if (lane == 0) s_count[warp][i] = count[i];
  }
  __syncthreads();
  const int q = q0 + threadIdx.x;
  if (threadIdx.x >= kMeetRows || q >= n) return;
  int many = 0;
  for (int w = 0; w < kMeetWarps; w++) many += s_count[w][threadIdx.x];
  rank[threadIdx.x] = many;
  if (many < kListed) ((int*)(p.list + p.tgt[q]))[many] = q;
}

// Loss and factors of kMeetRows (8, or with few rows 1) packed rows from their records: as many lanes, the records dealt to
// groups of them and met in a fixed order.
template <typename T, int kMeetRows>
__global__ void __launch_bounds__(kMeetWarps * 32) k_head_meet(MeetArgs a) {
  __shared__ float s_ref[kMeetWarps][kMeetRows], s_sum[kMeetWarps][kMeetRows], s_coef[kMeetRows];
  __shared__ int s_left[kMeetWarps][kMeetRows];
  follow();
  let_next();
  const HeadPlan& p = a.p;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, at = lane % kMeetRows;
  const int n = *p.count, q0 = blockIdx.x * kMeetRows, q = q0 + at;
  if (q0 >= n) return;
  __shared__ int s_rank[kMeetRows];
  if (p.list) list_targets(p, n, q0, s_rank);
  float ref = kNoRef, s = 0.0f;
  int left = 0;
  if (q < n) {
    const float own = a.stored && !a.known ? p.ref[q] : 0.0f;
#pragma unroll 4
    for (int t = threadIdx.x / kMeetRows; t < p.nrec; t += kMeetWarps * 32 / kMeetRows) {
      const float2 x = p.rec[(long long)t * p.cap + q];
      left |= a.stored && x.x != own;
      meet(ref, s, x.x, x.y);
    }
  }
  for (int o = 16; o >= kMeetRows; o >>= 1) {
    const float ref2 = __shfl_down_sync(~0u, ref, o), s2 = __shfl_down_sync(~0u, s, o);
    left |= __shfl_down_sync(~0u, left, o);
    if (lane < o) meet(ref, s, ref2, s2);
  }
  if (lane < kMeetRows) s_ref[warp][at] = ref, s_sum[warp][at] = s, s_left[warp][at] = left;
  __syncthreads();
  if (warp == 0 && lane < kMeetRows) {
    float coef = 0.0f;
    if (q < n) {
      for (int w = 1; w < kMeetWarps; w++) {
        meet(ref, s, s_ref[w][lane], s_sum[w][lane]);
        left |= s_left[w][lane];
      }
      const bool listed = a.grads && s_rank[lane] < kListed;
      if (a.known) {
        p.at_target[q] = (listed ? -s : lost<T>(-s)) * *p.post;
        if (!listed) ((T*)p.e)[q * p.lde + p.tgt[q]] = of_float<T>(-s);
      } else {
        // the others' sum against the target: loss = log(1 + sum / e_y)
        const float zt = p.zt[q], by = s == 0.0f && zt > -CUDART_INF_F ? -CUDART_INF_F : log2f(s) + fmaf(-zt, kLog2E, ref);
        const float x = by * kLn2, small = expf(-fabsf(x)), rest = log1pf(small);
        float nll = x > 0.0f ? x + rest : rest;
        if (!(zt < CUDART_INF_F) || s != s) nll = CUDART_NAN_F;
        const float lse = x > 0.0f ? (ref + log2f(s)) * kLn2 + rest : zt + nll;
        const long long r = a.r0 + p.src[q];
        a.loss[r] = (a.weight ? a.weight[r] : 1.0f) * nll;
        if (a.lse) a.lse[r] = lse;
        if (a.grads) {
          const float g = p.g[q], post = *p.post, most = -g * ((x > 0.0f ? 1.0f : small) / (1.0f + small));
          know(p, q, lse, g, post);
          float at = listed ? most : 0.0f;
          p.e_target[q] = listed ? 0.0f : most / post;
          if (a.stored) {
            const float to = p.ref[q];
            if (left || !(fmaf(zt, kLog2E, -to) <= kWindow)) *p.again = 1;
            const float others = s == 0.0f ? 0.0f : s * pow2_whole(ref - to);
            coef = g / (others + ex2(fmaf(zt, kLog2E, -to)));
            p.coef[q] = coef;
            if (!listed) {
              ((T*)p.e)[q * p.lde + p.tgt[q]] = of_float<T>(-others);
              at = coef * lost<T>(-others);
            }
          }
          p.at_target[q] = at;
        }
      }
    }
    s_coef[lane] = coef;
  }
  if (!p.hs) return;
  __syncthreads();
  const int own = kMeetRows == 1 ? 0 : warp;  // row
  if (q0 + own >= n) return;
  const T* hc = (const T*)p.hc + (long long)(q0 + own) * p.ldh;
  uint4* hs = (uint4*)((T*)p.hs + (long long)(q0 + own) * p.ldh);
  const float coef = s_coef[own];
#pragma unroll 4
  for (int k = (kMeetRows == 1 ? threadIdx.x : lane) * 8; k < p.ldh; k += kMeetRows == 1 ? kMeetWarps * 256 : 256) {
    const Chunk<T> x(hc + k, 8, true);
    uint4 v;
    T* t = (T*)&v;
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = of_float<T>(x.v[i] * coef);
    hs[k / 8] = v;
  }
}

// The head at rows of a multiple of 16 bytes, a warp a row.  8 elements come from the two aligned chunks of 16 bytes that they
// lie in, the lane's own and the next lane's; the first and the last chunk of a row may hold bytes next to it, within the
// same 16.
template <typename T>
__global__ void __launch_bounds__(256) k_head_pack(const T* head, long long stride, T* to, long long ld, int d, int V) {
  follow();
  let_next();
  const int lane = threadIdx.x % 32;
  for (long long v = blockIdx.x * 8ll + threadIdx.x / 32; v < V; v += gridDim.x * 8ll) {
    const uintptr_t w = (uintptr_t)(head + v * stride), end = w + d * sizeof(T);
    const uint32_t m = w % 16;
#pragma unroll 4
    for (int k0 = 0; k0 < ld; k0 += 256) {
      const int k = k0 + lane * 8;
      const uintptr_t from = w - m + k * sizeof(T);
      const uint4 none = make_uint4(0, 0, 0, 0), own = from < end ? *(const uint4*)from : none;
      uint4 next = make_uint4(__shfl_down_sync(~0u, own.x, 1), __shfl_down_sync(~0u, own.y, 1), __shfl_down_sync(~0u, own.z, 1),
                              __shfl_down_sync(~0u, own.w, 1));
      if (lane == 31) next = from + 16 < end ? *(const uint4*)(from + 16) : none;
      if (k >= ld) continue;
      const uint4 x = shifted(own, next, m);
      const uint32_t y[4] = {x.x, x.y, x.z, x.w};
      uint4 out;
      uint32_t* o = (uint32_t*)&out;
#pragma unroll
      for (int i = 0; i < 4; i++) {  // two elements
        const int left = d - k - 2 * i;
        o[i] = left >= 2 ? y[i] : left == 1 ? y[i] & 0xffff : 0u;
      }
      *(uint4*)(to + v * ld + k) = out;
    }
  }
}

template <typename T>
__global__ void k_fill_zero(T* grad, long long stride, int d) {
  follow();
  let_next();
  for (int k = threadIdx.x; k < d; k += blockDim.x) grad[blockIdx.x * stride + k] = of_float<T>(0.0f);
}

// ---------------------------------------------------------------- host

enum HeadForm { kForward = 0, kBackward = 1, kStep = 2 };

size_t round_up(size_t n, size_t m) { return (n + m - 1) / m * m; }

// Where the parts of a workspace lie; base NULL only counts.
struct Carver {
  char* base;
  size_t used;
  template <typename P>
  void take(P*& p, size_t count, size_t size) {
    p = base ? (P*)(base + used) : nullptr;
    used += round_up(count * size, 256);
  }
};

struct HeadCall {
  int form, dtype, B, n, d, V;
  const void* head;
  int64_t head_stride;
};

bool bad_call(const HeadCall& c) {
  return c.form < kForward || c.form > kStep || (c.dtype != EPIC_F16 && c.dtype != EPIC_BF16) || c.B < 0 || c.n < 0 ||
         c.d < 1 || c.V < 0 || (c.V > 1 && c.head_stride < c.d);
}

constexpr int kMostTokens = 0x7fffffff - 4096, kMostWidth = 1 << 20;

// Boxes are copied from rows that start at multiples of 16 bytes; another head is laid out anew, in each call.
bool head_lies_askew(const HeadCall& c, const HeadPlan& p) {
  return (uintptr_t)c.head % 16 != 0 || p.ldw % 8 != 0 || p.ldw >= 1ll << 38;
}

// The plan of the first piece and the bytes that all pieces share
size_t plan_head(const HeadCall& c, void* base, HeadPlan& p) {
  const long long rows = (long long)c.B * c.n;
  p = HeadPlan{};
  p.d = c.d;
  p.V = c.V;
  p.ldw = c.V > 1 ? c.head_stride : (int64_t)round_up(c.d, 8);
  p.head = c.head;
  p.ldh = round_up(c.d, 8);
  p.lde = round_up(std::max(c.V, 1), 64);
  p.ldp = round_up(c.d, 32);
  p.nrec = (c.V + kRecCols - 1) / kRecCols;
  // of what a position keeps: exponentials, or without gradients its records
  const size_t row = c.form != kForward ? p.lde * 2 : std::max(p.nrec, 1) * sizeof(float2);
  size_t bytes = (size_t)2048 << 20;
  if (const char* e = getenv("EPIC_HEAD_PIECE_MB")) bytes = strtoull(e, nullptr, 10) << 20;
  const long long fit = (long long)(bytes / row) / kRowTile * kRowTile;
  p.cap = (int)std::min<long long>(round_up(std::max(rows, 1ll), kRowTile),
                                   std::min<long long>(kPieceRows, std::max<long long>(kRowTile, fit)));
  const size_t cap = p.cap;
  Carver w = {(char*)base, 0};
  w.take(p.count, 1, 4);
  w.take(p.again, 1, 4);
  w.take(p.post, 1, 4);
  w.take(p.counts, kPieceRows / kRowsThreads, 4);
  w.take(p.tops, kPieceRows / kRowsThreads, 4);
  w.take(p.src, cap, 4);
  w.take(p.to, cap, 8);
  w.take(p.tgt, cap, 4);
  for (float** f : {&p.g, &p.zt, &p.ref, &p.coef, &p.known_ref, &p.known_mul, &p.at_target, &p.e_target}) w.take(*f, cap, 4);
  w.take(p.hc, cap * p.ldh, 2);
  if (c.form == kStep && c.dtype == EPIC_BF16) w.take(p.hs, cap * p.ldh, 2);
  w.take(p.rec, cap * p.nrec, sizeof(float2));
  if (c.form != kForward) {
    w.take(p.list, (size_t)c.V, sizeof(int4));
    w.take(p.e, cap * p.lde, 2);
    if (rows > p.cap) w.take(p.acc, (size_t)c.V * p.ldp, 4);
    p.split = split_grads((int)std::min<long long>(rows, p.cap), c.d, c.V);
    if (p.split.hidden_parts > 1) w.take(p.split.hidden, p.split.hidden_parts * cap * p.ldp, 4);
    if (p.split.head_parts > 1) w.take(p.split.head, (size_t)p.split.head_parts * p.split.tokens * p.ldp, 4);
  }
  if (head_lies_askew(c, p)) {
    void* packed;
    w.take(packed, (size_t)c.V * p.ldh, 2);
    p.head = packed;
    p.ldw = p.ldh;
  }
  return w.used;
}

struct HeadTensors {
  const void* hidden;
  int64_t stride_b, stride_n;
  const int32_t* target;
  const float *weight, *lse_in, *up;
  float *loss, *lse;
  void* grad_hidden;
  int64_t gstride_b, gstride_n;
  void* grad_head;
  int64_t ghead_stride;
};

#define EPIC_TRY(call)                     \
  do {                                     \
    const epic_status s_ = (call);         \
    if (s_ != EPIC_OK) return s_;          \
  } while (0)

template <typename T>
epic_status run_head(const HeadCall& c, const HeadTensors& t, HeadPlan p, cudaStream_t st) {
  const long long rows = (long long)c.B * c.n;
  const bool half = c.dtype == EPIC_F16, grads = c.form != kForward;
  if (rows == 0 || c.V == 0) {
    if (rows == 0 && t.grad_head && c.V > 0) {
      EPIC_TRY(launch_next(k_fill_zero<T>, c.V, 256, 0, kNoCache, st, (T*)t.grad_head, t.ghead_stride, c.d));
    }
    if (rows == 0) return EPIC_OK;
  }
  if (c.V > 0 && p.head != c.head) {
    EPIC_TRY(launch_next(k_head_pack<T>, (unsigned)(c.V + 7) / 8, 256, 0, kNoCache, st, (const T*)c.head,
                         c.head_stride, (T*)p.head, p.ldw, c.d, c.V));
  }
  HeadMaps maps;
  if (c.V > 0) EPIC_TRY(make_head_maps(maps, p, c.dtype, grads, t.grad_head, t.ghead_stride));
  for (long long r0 = 0; r0 < rows; r0 += p.cap) {
    p.rows = (int)std::min<long long>(p.cap, rows - r0);
    RowsArgs a = {};
    a.p = p;
    a.hidden = t.hidden;
    a.stride_b = t.stride_b;
    a.stride_n = t.stride_n;
    a.r0 = r0;
    a.n = c.n;
    a.target = t.target;
    a.weight = t.weight;
    a.up = t.up;
    a.lse = t.lse_in;
    a.loss = t.loss;
    a.lse_out = t.lse;
    a.out = {t.grad_hidden, t.gstride_b, t.gstride_n};
    // Few positions have a CTA each, which pays by the row's width.  Steps with a CTA and with a warp a position (us): 300 positions
    // through 1,000 x 256 34 and 33, 608 33 and 31, 1,000 35 and 33, 1,300 39 and 34; through 4,000 x 1,024 300 43 and 45, 608 49 and
    // 51, 1,000 58 and 60, 1,300 74 and 74; through 8,000 x 2,048 300 70 and 77, 608 89 and 100, 1,000 109 and 119, 1,300 125 and 132.
    const bool few = p.rows <= kFewRows;
    a.per = few ? 1 : 8;
    const bool known = c.form == kBackward, stored = known || (grads && !half);
    a.probs = stored && !known;
    a.scaled = half && grads;
    a.again = known || a.scaled;
    if (p.rows > kCounted)
      EPIC_TRY(launch_next(k_head_count, (p.rows + kRowsThreads - 1) / kRowsThreads, kRowsThreads, 0, kNoCache, st, a));
    EPIC_TRY(launch_next(few ? k_head_rows<T, true> : k_head_rows<T, false>, (p.rows + a.per - 1) / a.per, kRowsThreads, 0, kNoCache,
                         st, a));
    if (c.V == 0) continue;
    // A step's exponentials are relative to the target's logit; fp16 has not the range for that and makes them once the
    // logsumexp is known, as do rows that leave the window.
    EPIC_TRY(launch_head_logits(p, maps, c.dtype, {true, stored, known, false}, st));
    const MeetArgs m = {p, r0, t.weight, t.loss, t.lse, grads, stored, known};
    EPIC_TRY(launch_next(few ? k_head_meet<T, 1> : k_head_meet<T, 8>, few ? p.rows : (p.rows + 7) / 8, kMeetWarps * 32, 0, kNoCache,
                         st, m));
    if (grads && !known) EPIC_TRY(launch_head_logits(p, maps, c.dtype, {false, true, true, true}, st));
    if (t.grad_hidden || t.grad_head) {
      const bool first = r0 == 0, last = r0 + p.cap >= rows;
      const HeadSum sum = first ? (last ? kOnly : kFirst) : last ? kLast : kMiddle;
      EPIC_TRY(launch_head_grads(p, maps, c.dtype, a.out, t.grad_head, t.ghead_stride, sum, st));
    }
  }
  return EPIC_OK;
}

bool misaligned(const void* p, size_t to) { return (uintptr_t)p % to != 0; }

epic_status head_call(const HeadCall& c, const HeadTensors& t, void* ws, size_t ws_bytes, void* stream) {
  if (bad_call(c) || t.stride_b < 0 || t.stride_n < 0) return EPIC_ERR_INVALID_ARG;
  if (c.V > kMostTokens || c.d > kMostWidth) return EPIC_ERR_CAPACITY;
  if (t.grad_hidden && (t.gstride_b < 0 || t.gstride_n < 0)) return EPIC_ERR_INVALID_ARG;
  if (t.grad_head && c.V > 1 && t.ghead_stride < c.d) return EPIC_ERR_INVALID_ARG;
  const long long rows = (long long)c.B * c.n;
  for (const void* p : {t.hidden, c.head, (const void*)t.grad_hidden, (const void*)t.grad_head})
    if (misaligned(p, 2)) return EPIC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)t.target, (const void*)t.weight, (const void*)t.lse_in, (const void*)t.up,
                        (const void*)t.loss, (const void*)t.lse})
    if (misaligned(p, 4)) return EPIC_ERR_INVALID_ARG;
  if (c.V > 0 && !c.head && rows > 0) return EPIC_ERR_INVALID_ARG;
  if (rows > 0) {
    if (!t.hidden || !t.target) return EPIC_ERR_INVALID_ARG;
    if (c.form == kBackward ? !t.lse_in || !t.up : !t.loss) return EPIC_ERR_INVALID_ARG;
    if (c.form == kForward && !t.lse) return EPIC_ERR_INVALID_ARG;
  }
  if (rows == 0 && (!t.grad_head || c.V == 0)) return EPIC_OK;
  HeadPlan p;
  if (!ws || misaligned(ws, 256) || ws_bytes < plan_head(c, nullptr, p)) return EPIC_ERR_INVALID_ARG;
  plan_head(c, ws, p);
  cudaStream_t st = (cudaStream_t)stream;
  return c.dtype == EPIC_F16 ? run_head<__half>(c, t, p, st) : run_head<__nv_bfloat16>(c, t, p, st);
}

}  // namespace
}  // namespace epic

extern "C" {

epic_status epic_head_loss_workspace(int32_t form, int32_t dtype, int32_t B, int32_t n, int32_t d, int32_t V,
                                     const void* d_head, int64_t head_stride, size_t* bytes) {
  using namespace epic;
  const HeadCall c = {form, dtype, B, n, d, V, d_head, head_stride};
  if (!bytes || bad_call(c)) return EPIC_ERR_INVALID_ARG;
  if (V > kMostTokens || d > kMostWidth) return EPIC_ERR_CAPACITY;
  HeadPlan p;
  *bytes = plan_head(c, nullptr, p);
  return EPIC_OK;
}

epic_status epic_head_loss_forward(const void* d_hidden, int32_t dtype, int32_t B, int32_t n, int32_t d,
                                   int64_t stride_b, int64_t stride_n, const void* d_head, int32_t V,
                                   int64_t head_stride, const int32_t* d_target, const float* d_weight, float* d_loss,
                                   float* d_lse, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace epic;
  HeadTensors t = {};
  t.hidden = d_hidden;
  t.stride_b = stride_b;
  t.stride_n = stride_n;
  t.target = d_target;
  t.weight = d_weight;
  t.loss = d_loss;
  t.lse = d_lse;
  return head_call({kForward, dtype, B, n, d, V, d_head, head_stride}, t, d_workspace, workspace_bytes, cuda_stream);
}

epic_status epic_head_loss_backward(const void* d_hidden, int32_t dtype, int32_t B, int32_t n, int32_t d,
                                    int64_t stride_b, int64_t stride_n, const void* d_head, int32_t V,
                                    int64_t head_stride, const int32_t* d_target, const float* d_weight,
                                    const float* d_lse, const float* d_grad_loss, void* d_grad_hidden,
                                    int64_t grad_stride_b, int64_t grad_stride_n, void* d_grad_head,
                                    int64_t grad_head_stride, void* d_workspace, size_t workspace_bytes,
                                    void* cuda_stream) {
  using namespace epic;
  HeadTensors t = {};
  t.hidden = d_hidden;
  t.stride_b = stride_b;
  t.stride_n = stride_n;
  t.target = d_target;
  t.weight = d_weight;
  t.lse_in = d_lse;
  t.up = d_grad_loss;
  t.grad_hidden = d_grad_hidden;
  t.gstride_b = grad_stride_b;
  t.gstride_n = grad_stride_n;
  t.grad_head = d_grad_head;
  t.ghead_stride = grad_head_stride;
  return head_call({kBackward, dtype, B, n, d, V, d_head, head_stride}, t, d_workspace, workspace_bytes, cuda_stream);
}

epic_status epic_head_loss_step(const void* d_hidden, int32_t dtype, int32_t B, int32_t n, int32_t d, int64_t stride_b,
                                int64_t stride_n, const void* d_head, int32_t V, int64_t head_stride,
                                const int32_t* d_target, const float* d_weight, float* d_loss, void* d_grad_hidden,
                                int64_t grad_stride_b, int64_t grad_stride_n, void* d_grad_head,
                                int64_t grad_head_stride, void* d_workspace, size_t workspace_bytes,
                                void* cuda_stream) {
  using namespace epic;
  HeadTensors t = {};
  t.hidden = d_hidden;
  t.stride_b = stride_b;
  t.stride_n = stride_n;
  t.target = d_target;
  t.weight = d_weight;
  t.loss = d_loss;
  t.grad_hidden = d_grad_hidden;
  t.gstride_b = grad_stride_b;
  t.gstride_n = grad_stride_n;
  t.grad_head = d_grad_head;
  t.ghead_stride = grad_head_stride;
  return head_call({kStep, dtype, B, n, d, V, d_head, head_stride}, t, d_workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
