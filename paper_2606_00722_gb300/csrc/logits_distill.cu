// Distillation from a teacher's top logits, forward and backward.
//
// Per row, p = softmax(a / tau) over the teacher's entries that count and
// lq = z / tau - logsumexp(z / tau) over the student's whole row:
//   loss   = w tau^2 sum_k p_k (log p_k - lq[t_k])
//   dz_j   = w tau (softmax(z / tau)_j - sum_{k: t_k = j} p_k)
// A row with no entry that counts, or with w = 0, has loss and gradient 0.
// With a' and z' relative to their largest (of the entries, of the row), and
// log A, log Z the logarithms of the sums of exponentials relative to these,
//   loss = w tau sum_k p_k (a'_k - z'[t_k] + tau (log Z - log A)):
// nothing is divided by tau but exponents, so values at the type's lowest and any
// tau stay in range.
// Sums are held in 32 bits; the gradient is rounded once, to the logits' type.
//
// Each row is read from memory once: for the loss in one pass with a running
// maximum, for loss and gradient with a second pass from the caches.  The
// backward pass has the row's logsumexp and reads the row once again.
#include <limits.h>

#include "../../include/epic.h"
#include "logit_launch.h"
#include "logit_rows.cuh"

namespace epic {
namespace {

constexpr int kMaxTargets = 1024;  // most teacher entries of a row
// Largest size of a logsumexp from which the backward pass takes probabilities.  32 bits hold it to 2^-18 there, which is
// the probabilities' relative error; of a row at its type's lowest value they hold the maximum and nothing of the sum.
// Larger ones are taken apart again, from the row.
constexpr float kLseFine = 128.0f;
constexpr int kDistillThreads = 384;
constexpr int kDistillPerSm = 4;

struct DistillArgs {
  RowArgs rows;
  const int32_t* ids;
  const float* vals;
  const uint8_t* valid;  // [rows][K] or NULL
  int K;
  float tau;
  const float* weight;  // [rows] or NULL
  float* loss;          // NULL in the backward pass
  float* lse;           // out, or NULL
  const float* lse_in;  // the backward pass
  const float* up;
  void* grad;  // NULL in the forward pass
  long long gstride_b, gstride_n;
};

struct Targets {
  float p[kMaxTargets];
  float a[kMaxTargets];  // values relative to the largest
  float z[kMaxTargets];  // the student's logits of the tokens
  int id[kMaxTargets];  // -1: does not count
  uint4 ends[2], row_ends[2];
  int any;
  float warp_m[kRowWarps], warp_s[kRowWarps];
  float m, s;  // of the CTA
};

// larger of two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) { return ChunkMax<float, true>::max1(a, b); }

// log2(e) / tau
__device__ __forceinline__ float exponent_scale(float tau) { return fminf(kLog2e / tau, CUDART_MAX_NORMAL_F); }

__device__ __forceinline__ float below_inf(float x) { return x == CUDART_INF_F ? CUDART_MAX_NORMAL_F : x; }

__device__ __forceinline__ float warp_add(float x) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}
__device__ __forceinline__ float warp_max_nan(float x) {
  for (int o = 16; o; o >>= 1) x = max_nan(x, __shfl_xor_sync(~0u, x, o));
  return x;
}

// One warp's work: the row's entries in shared memory, p of them, and whether any counts.  load() asks for what is in
// memory and is called before the pass over the row, finish() after it; entries past the 32nd wait for finish(), which
// returns the logarithm of the sum of exponentials.
template <typename T>
struct Teacher {
  int id;
  float value, z;
  // entry k: its token (-1: does not count), its value, and the student's logit of the token
  __device__ __forceinline__ void entry(const DistillArgs& a, int r, const T* logits, int k) {
    const long long o = (long long)r * a.K + k;
    const int token = a.ids[o];
    const float v = a.vals[o];
    const bool counts = token >= 0 && token < a.rows.V && (!a.valid || a.valid[o] == 1) && v != -CUDART_INF_F;
    id = counts ? token : -1;
    value = v;
    z = counts ? to_float<T>(logits[token]) : 0.0f;
  }
  __device__ __forceinline__ void load(const DistillArgs& a, int r, const T* logits) {
    const int lane = threadIdx.x % 32;
    if (lane < a.K) entry(a, r, logits, lane);
  }
  __device__ __forceinline__ float finish(const DistillArgs& a, int r, const T* logits, Targets& t) {
    const int lane = threadIdx.x % 32;
    float m = -CUDART_INF_F;
#pragma unroll 1
    for (int k = lane; k < a.K; k += 32) {
      if (k >= 32) entry(a, r, logits, k);
      t.id[k] = id;
      t.a[k] = value;
      t.z[k] = z;
      if (id >= 0) m = max_nan(m, value);
    }
    m = warp_max_nan(m);
    if (lane == 0) t.any = m != -CUDART_INF_F;
    float sum = 0.0f;
#pragma unroll 1
    for (int k = lane; k < a.K; k += 32) {
      t.a[k] -= m;
      t.p[k] = t.id[k] >= 0 ? expf(t.a[k] / a.tau) : 0.0f;
      sum += t.p[k];
    }
    sum = warp_add(sum);
#pragma unroll 1
    for (int k = lane; k < a.K; k += 32) t.p[k] /= sum;
    return logf(sum);
  }
};

// A chunk of the row at a distance of `by` bytes (0..15) past the start of `a`, b being the chunk after a.
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int by) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (by & 8)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (by & 4)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  const int bits = 8 * (by & 3);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The slice's elements of a gradient row, g(z) for two of them at a time.  The chunks are the gradient's: where its row
// starts elsewhere in 16 bytes than the logits' row does, two chunks of logits are read for one of gradient.
template <typename T, typename G>
__device__ void write_row(const Slice<T>& s, T* grad, G g) {
  constexpr int E = ElemOf<T>::E;
  const int lo = s.lo(), hi = s.hi();
  const int ghead = (int)(reinterpret_cast<uintptr_t>(grad) & 15) / (int)sizeof(T);
  const auto put = [&](const uint4& v, int i0) {  // elements i0 .. i0 + E - 1
    float f[E];
    unpack<T>(v, f);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 y = g(make_float2(f[e], f[e + 1]));
      f[e] = y.x;
      f[e + 1] = y.y;
    }
    if (i0 >= lo && i0 + E <= hi) {
      *reinterpret_cast<uint4*>(grad + i0) = pack<T>(f);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i0 + e >= lo && i0 + e < hi) grad[i0 + e] = from_float<T>(f[e]);
    }
  };
  if (ghead == s.head) {
    s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + 32 * i < s.n) put(v[i], s.first(c + 32 * i));
    });
    return;
  }
  if (lo >= hi) return;
  // gradient chunk j starts `by` bytes into the chunk of logits at or before its first element
  const int ahead = s.head - ghead, by = ((ahead + E) % E) * (int)sizeof(T), back = ahead < 0 ? 1 : 0;
  for (int j = (lo + ghead) / E + (int)threadIdx.x; j <= (hi - 1 + ghead) / E; j += blockDim.x) {
    const int c = j - back - s.c0;  // of the slice; a neighbour's elements are not put
    uint4 a = empty_chunk<T>(), b = a;
    if (c >= 0 && c < s.n) a = s.chunk(c);
    if (c + 1 >= 0 && c + 1 < s.n) b = s.chunk(c + 1);
    put(shifted(a, b, by), j * E - ghead);
  }
}

template <typename T>
__device__ void write_zeros(const Slice<T>& s, T* grad) {
  constexpr int E = ElemOf<T>::E;
  const int lo = s.lo(), hi = s.hi();
  const int ghead = (int)(reinterpret_cast<uintptr_t>(grad) & 15) / (int)sizeof(T);
  if (lo >= hi) return;
  for (int j = (lo + ghead) / E + (int)threadIdx.x; j <= (hi - 1 + ghead) / E; j += blockDim.x) {
    const int i0 = j * E - ghead;
    if (i0 >= lo && i0 + E <= hi) {
      *reinterpret_cast<uint4*>(grad + i0) = make_uint4(0, 0, 0, 0);
    } else {
      for (int e = 0; e < E; ++e)
        if (i0 + e >= lo && i0 + e < hi) grad[i0 + e] = from_float<T>(0.0f);
    }
  }
}

// coef (q(z) - the target's share) over the slice, coef q(z) being g(z).  The few elements that have a share are written
// again, each by a thread of its own, after a barrier.
template <typename T, typename G>
__device__ __forceinline__ void write_gradient(const Slice<T>& s, T* grad, float coef, const Targets& t, int K, G g) {
  write_row(s, grad, g);
  __syncthreads();
  const int lo = s.lo(), hi = s.hi();
#pragma unroll 1
  for (int k = threadIdx.x; k < K; k += blockDim.x) {
    const int id = t.id[k];
    if (id < lo || id >= hi) continue;
    float p = 0.0f;  // entries of the same token add up, in every thread that has one of them alike
    for (int j = 0; j < K; ++j)
      if (t.id[j] == id) p += t.p[j];
    grad[id] = from_float<T>(g(make_float2(t.z[k], 0.0f)).x - coef * p);
  }
}

template <typename T>
__device__ __forceinline__ T* gradient_row(const DistillArgs& a, int r) {
  const int b = r / a.rows.k;
  return static_cast<T*>(a.grad) + b * a.gstride_b + (r - b * a.rows.k) * a.gstride_n;
}

// This lane's elements of the slice: the maximum (NaN if any is, or +inf) and the sum of 2^((z - maximum) c2).
template <typename T>
__device__ __forceinline__ float lane_sums(const Slice<T>& s, float c2, float* sum) {
  constexpr int E = ElemOf<T>::E;
  float top = -CUDART_INF_F;
  float2 sums = make_float2(0.0f, 0.0f);
  const float2 by = make_float2(c2, c2);
  s.sweep([&](const uint4 (&v)[4], int) {
    ChunkMax<T, true> batch;
    batch.add(v);
    const float x = batch.value();
    if (!(x <= top)) {  // larger, or NaN now or before: maximum and sums stay NaN from then on
      const float now = max_nan(top, x), less = exp2_32((top - now) * c2);
      sums.x *= less;
      sums.y *= less;
      top = now;
    }
    if (top == -CUDART_INF_F) return;
    const float2 off = make_float2(-top, -top);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z[E];
      unpack<T>(v[i], z);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 y = mul2(add2(make_float2(z[e], z[e + 1]), off), by);
        sums = add2(sums, make_float2(exp2_32(y.x), exp2_32(y.y)));
      }
    }
  });
  *sum = sums.x + sums.y;
  return top;
}

// A part's sum relative to a maximum `of`, relative to m instead; a part without elements has maximum -inf and sum 0.
__device__ __forceinline__ float rebase(float sum, float of, float m, float c2) {
  return of == -CUDART_INF_F ? 0.0f : sum * exp2_32((of - m) * c2);
}

// The CTA's, from its lanes'; a barrier included.
__device__ __forceinline__ float cta_sums(Targets& t, float top, float c2, float* sum) {
  const int lane = threadIdx.x % 32, warp = warp_index(), warps = blockDim.x / 32;
  float m = warp_max_nan(top), x = warp_add(rebase(*sum, top, m, c2));
  if (lane == 0) {
    t.warp_m[warp] = m;
    t.warp_s[warp] = x;
  }
  __syncthreads();
  m = warp_max_nan(lane < warps ? t.warp_m[lane] : -CUDART_INF_F);
  *sum = warp_add(lane < warps ? rebase(t.warp_s[lane], t.warp_m[lane], m, c2) : 0.0f);
  return m;
}

// Loss, and with a.grad the gradient: one cluster a row.  Bound by memory, and by the barriers between a row's two passes:
// both for 4,096 rows of 32,768 bf16, half of them of weight 0, take 73 us, 5.5 TB/s where a copy reaches 6.7 (with 384
// threads and four CTAs an SM; 512 and two took 90 when these took 74); the loss of 1,024 rows of 126,000 takes 48, 5.4 TB/s.
// One pass keeps each lane's maximum so far and the sum of
// exponentials relative to it; the gradient's pass reads the row again, from the caches.
template <typename T>
__global__ void __launch_bounds__(kDistillThreads, kDistillPerSm) k_distill(DistillArgs a) {
  __shared__ Targets t;
  auto cluster = cg::this_cluster();
  const unsigned ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const int lane = threadIdx.x % 32, warp = warp_index(), warps = blockDim.x / 32;
  const int r = (int)(blockIdx.x / ctas);
  const float weight = a.weight ? a.weight[r] : 1.0f;
  const T* logits = row_address<T>(a.rows, r);
  T* grad = a.grad ? gradient_row<T>(a, r) : nullptr;
  Slice<T> s;
  s.open(logits, a.rows, rank, t.ends);
  if (weight == 0.0f) {  // the same in all CTAs of the row
    if (rank == 0 && threadIdx.x == 0) {
      a.loss[r] = 0.0f;
      if (a.lse) a.lse[r] = CUDART_INF_F;
    }
    if (grad) write_zeros(s, grad);
    return;
  }
  Teacher<T> teacher;
  if (warp == warps - 1) teacher.load(a, r, logits);
  const float c2 = exponent_scale(a.tau);
  float sum;
  const float top = lane_sums(s, c2, &sum);
  float teacher_log = 0.0f;
  if (warp == warps - 1) teacher_log = teacher.finish(a, r, logits, t);
  float m = cta_sums(t, top, c2, &sum);
  if (ctas > 1) {
    if (threadIdx.x == 0) {
      t.m = m;
      t.s = sum;
    }
    cluster.sync();
    float of = -CUDART_INF_F, x = 0.0f;
    if (lane < (int)ctas) {
      of = *cluster.map_shared_rank(&t.m, lane);
      x = *cluster.map_shared_rank(&t.s, lane);
    }
    m = warp_max_nan(of);
    sum = warp_add(rebase(x, of, m, c2));
  }
  const bool any = t.any;
  const float log_sum = m == -CUDART_INF_F ? -CUDART_INF_F : logf(sum);
  if (rank == 0 && warp == warps - 1) {
    float loss = 0.0f;
    if (any)
      for (int k = lane; k < a.K; k += 32) {
        const float p = t.p[k];
        if (t.id[k] < 0 || p == 0.0f) continue;
        // +inf where the token is at -inf, NaN where the row has NaN or +inf; a row of -inf alone has no sum
        // Quarters of it: p adds up to 1 but for roundings, and so a sum of costs near the largest number stays in range.
        loss += 0.25f * p * (m == -CUDART_INF_F ? CUDART_INF_F : t.a[k] - (t.z[k] - m) + a.tau * (log_sum - teacher_log));
      }
    loss = warp_add(loss);
    if (lane == 0) {
      // the smaller factor first
      a.loss[r] = any ? 4.0f * (a.tau < 1.0f ? weight * (a.tau * loss) : weight * a.tau * loss) : 0.0f;
      // +inf says that nothing flows back
      if (a.lse) a.lse[r] = !any ? CUDART_INF_F : m == -CUDART_INF_F ? m : below_inf(m / a.tau + log_sum);
    }
  }
  if (grad) {
    const float coef = weight * a.tau;
    const float scale = m == -CUDART_INF_F ? 0.0f : coef / sum, at = m == -CUDART_INF_F ? 0.0f : m;
    if (any)
      write_gradient(s, grad, coef, t, a.K, [=](float2 z) {
        const float2 y = mul2(add2(z, make_float2(-at, -at)), make_float2(c2, c2));
        return mul2(make_float2(exp2_32(y.x), exp2_32(y.y)), make_float2(scale, scale));
      });
    else
      write_zeros(s, grad);
  }
  if (ctas > 1) cluster.sync();  // no CTA leaves while its shared memory is read
}

// A whole row's maximum and sum, by one CTA: for a backward pass whose logsumexp is too coarse.
template <typename T>
__device__ __noinline__ float2 row_sums(const DistillArgs& a, int r, Targets& t, float c2) {
  RowArgs rows = a.rows;
  rows.per = INT_MAX;
  Slice<T> s;
  s.open(row_address<T>(rows, r), rows, 0, t.row_ends);
  float sum;
  const float top = lane_sums(s, c2, &sum), m = cta_sums(t, top, c2, &sum);
  return make_float2(m, sum);
}

// The gradient from the row's logsumexp: a CTA per slice, nothing shared between them.  Reads and writes the row once: 1,024
// rows of 126,000 bf16 in 78 us, 6.0 TB/s (a copy's rate: 6.7).
template <typename T>
__global__ void __launch_bounds__(kDistillThreads, kDistillPerSm) k_distill_backward(DistillArgs a, int parts) {
  __shared__ Targets t;
  const int r = (int)(blockIdx.x / (unsigned)parts);
  const float weight = a.weight ? a.weight[r] : 1.0f, lse = a.lse_in[r];
  const float coef = weight == 0.0f || lse == CUDART_INF_F ? 0.0f : weight * a.tau * a.up[r];
  T* grad = gradient_row<T>(a, r);
  Slice<T> s;
  s.open(row_address<T>(a.rows, r), a.rows, (int)(blockIdx.x % parts), t.ends);
  if (coef == 0.0f) {
    write_zeros(s, grad);
    return;
  }
  if (warp_index() == (int)blockDim.x / 32 - 1) {
    Teacher<T> teacher;
    teacher.load(a, r, row_address<T>(a.rows, r));
    teacher.finish(a, r, row_address<T>(a.rows, r), t);
  }
  const float c2 = exponent_scale(a.tau);
  float at = lse * a.tau, scale = coef;
  if (fabsf(lse) > kLseFine) {
    const float2 sums = row_sums<T>(a, r, t, c2);
    at = sums.x == -CUDART_INF_F ? 0.0f : sums.x;
    scale = sums.x == -CUDART_INF_F ? 0.0f : coef / sums.y;  // in a row of -inf alone every probability is 0
  }
  write_gradient(s, grad, coef, t, a.K, [=](float2 z) {
    const float2 y = mul2(add2(z, make_float2(-at, -at)), make_float2(c2, c2));
    return mul2(make_float2(exp2_32(y.x), exp2_32(y.y)), make_float2(scale, scale));
  });
}

template <typename T>
epic_status launch_distill(DistillArgs& a, long long rows, cudaStream_t st) {
  RowShape p = row_shape(rows, a.rows.V, sizeof(T), 64, kDistillThreads);
  a.rows.per = p.per;
  if (!a.lse_in) return launch_rows((const void*)k_distill<T>, p, rows, &a, st);
  if (rows > 0x7fffffffll / p.ctas) return EPIC_ERR_CAPACITY;
  k_distill_backward<T><<<(unsigned)(rows * p.ctas), p.threads, 0, st>>>(a, p.ctas);
  return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA;
}

epic_status distill(DistillArgs& a, const void* logits, int dtype, int B, int n, int V, int64_t sb, int64_t sn,
                    void* stream) {
  if (a.K < 0 || a.gstride_b < 0 || a.gstride_n < 0) return EPIC_ERR_INVALID_ARG;
  if (!(a.tau > 0.0f) || a.tau > 3.0e38f) return EPIC_ERR_INVALID_ARG;
  epic_status s = check_rows(logits, dtype, B, n, V, sb, sn, nullptr, n);
  if (s != EPIC_OK) return s;
  if (a.K > kMaxTargets) return EPIC_ERR_CAPACITY;
  const long long rows = (long long)B * n;
  if (rows == 0) return EPIC_OK;
  if (a.K > 0 && (!a.ids || !a.vals)) return EPIC_ERR_INVALID_ARG;
  if (a.grad && (uintptr_t)a.grad % (dtype == EPIC_F32 ? 4 : 2)) return EPIC_ERR_INVALID_ARG;
  a.rows = {logits, sb, sn, nullptr, n, n, V, 0};
  cudaStream_t st = (cudaStream_t)stream;
  switch (dtype) {
    case EPIC_F32: return launch_distill<float>(a, rows, st);
    case EPIC_F16: return launch_distill<__half>(a, rows, st);
    default: return launch_distill<__nv_bfloat16>(a, rows, st);
  }
}

}  // namespace
}  // namespace epic

extern "C" {

epic_status epic_distill_forward(const void* d_logits, int32_t dtype, int32_t B, int32_t n, int32_t V,
                                 int64_t stride_b, int64_t stride_n, const int32_t* d_ids, const float* d_vals,
                                 const uint8_t* d_valid, int32_t K, float tau, const float* d_weight, float* d_loss,
                                 float* d_lse, void* cuda_stream) {
  using namespace epic;
  if ((long long)B * n > 0 && (!d_loss || !d_lse)) return EPIC_ERR_INVALID_ARG;
  DistillArgs a = {};
  a.ids = d_ids;
  a.vals = d_vals;
  a.valid = d_valid;
  a.K = K;
  a.tau = tau;
  a.weight = d_weight;
  a.loss = d_loss;
  a.lse = d_lse;
  return distill(a, d_logits, dtype, B, n, V, stride_b, stride_n, cuda_stream);
}

epic_status epic_distill_backward(const void* d_logits, int32_t dtype, int32_t B, int32_t n, int32_t V,
                                  int64_t stride_b, int64_t stride_n, const int32_t* d_ids, const float* d_vals,
                                  const uint8_t* d_valid, int32_t K, float tau, const float* d_weight,
                                  const float* d_lse, const float* d_grad_loss, void* d_grad, int64_t grad_stride_b,
                                  int64_t grad_stride_n, void* cuda_stream) {
  using namespace epic;
  if ((long long)B * n > 0 && (!d_lse || !d_grad_loss || (!d_grad && V > 0))) return EPIC_ERR_INVALID_ARG;
  DistillArgs a = {};
  a.ids = d_ids;
  a.vals = d_vals;
  a.valid = d_valid;
  a.K = K;
  a.tau = tau;
  a.weight = d_weight;
  a.lse_in = d_lse;
  a.up = d_grad_loss;
  a.grad = d_grad;
  a.gstride_b = grad_stride_b;
  a.gstride_n = grad_stride_n;
  return distill(a, d_logits, dtype, B, n, V, stride_b, stride_n, cuda_stream);
}

epic_status epic_distill_step(const void* d_logits, int32_t dtype, int32_t B, int32_t n, int32_t V, int64_t stride_b,
                              int64_t stride_n, const int32_t* d_ids, const float* d_vals, const uint8_t* d_valid,
                              int32_t K, float tau, const float* d_weight, float* d_loss, void* d_grad,
                              int64_t grad_stride_b, int64_t grad_stride_n, void* cuda_stream) {
  using namespace epic;
  if ((long long)B * n > 0 && (!d_loss || (!d_grad && V > 0))) return EPIC_ERR_INVALID_ARG;
  DistillArgs a = {};
  a.ids = d_ids;
  a.vals = d_vals;
  a.valid = d_valid;
  a.K = K;
  a.tau = tau;
  a.weight = d_weight;
  a.loss = d_loss;
  a.grad = d_grad;
  a.gstride_b = grad_stride_b;
  a.gstride_n = grad_stride_n;
  return distill(a, d_logits, dtype, B, n, V, stride_b, stride_n, cuda_stream);
}

}  // extern "C"
