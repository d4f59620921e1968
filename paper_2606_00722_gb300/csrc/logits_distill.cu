// Distillation from a teacher's top logits, forward and backward.
//
// Per row, p = softmax(a / tau) over the teacher's entries that count and
// lq = z / tau - logsumexp(z / tau) over the student's whole row:
//   loss   = w tau^2 sum_k p_k (log p_k - lq[t_k])
//   dz_j   = w tau (softmax(z / tau)_j - sum_{k: t_k = j} p_k)
// A row with no entry that counts, or with w = 0, has loss and gradient 0.
// Sums are held in 32 bits; the gradient is rounded once, to the logits' type.
//
// The forward pass and the one that also writes the gradient stage the row in a
// cluster's shared memory (one read of the logits, one write of the gradient);
// the backward pass has the row's logsumexp and streams.
#include "../../include/epic.h"
#include "logit_launch.h"
#include "logit_rows.cuh"

namespace epic {
namespace {

constexpr int kMaxTargets = 1024;  // most teacher entries of a row

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
  float lp[kMaxTargets];
  int id[kMaxTargets];  // -1: does not count
  float red[kRowWarps];
  float value;
};

// larger of two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

struct MaxNan {
  __device__ float operator()(float a, float b) const { return max_nan(a, b); }
};
struct Add {
  __device__ float operator()(float a, float b) const { return a + b; }
};

// one value from all threads, in a fixed order; every thread gets it
template <typename Op>
__device__ float block_reduce(float x, Op op, float* red, float* value) {
  for (int o = 16; o; o >>= 1) x = op(x, __shfl_xor_sync(~0u, x, o));
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = x;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)blockDim.x / 32; ++w) x = op(x, red[w]);
    *value = x;
  }
  __syncthreads();
  x = *value;
  __syncthreads();
  return x;
}

// p and log p of the row's entries; false when none counts
__device__ bool teacher(const DistillArgs& a, long long r, Targets& t) {
  float m = -CUDART_INF_F;
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    const long long o = r * a.K + k;
    const int id = a.ids[o];
    const float v = a.vals[o];
    const bool counts = id >= 0 && id < a.rows.V && (!a.valid || a.valid[o] == 1) && v != -CUDART_INF_F;
    t.id[k] = counts ? id : -1;
    t.lp[k] = v / a.tau;
    if (counts) m = max_nan(m, t.lp[k]);
  }
  m = block_reduce(m, MaxNan(), t.red, &t.value);
  if (m == -CUDART_INF_F) return false;
  float sum = 0.0f;
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    t.lp[k] -= m;
    t.p[k] = t.id[k] >= 0 ? expf(t.lp[k]) : 0.0f;
    sum += t.p[k];
  }
  sum = block_reduce(sum, Add(), t.red, &t.value);
  const float log_sum = logf(sum);
  for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
    t.p[k] /= sum;
    t.lp[k] -= log_sum;
  }
  __syncthreads();
  return true;
}

// The slice's part of a gradient row: q(z) is the student's probability of a logit, the target's share is taken off
// where the slice has it.
template <typename T, typename Q>
__device__ void write_gradient(const Slice<T>& s, T* grad, float coef, const Targets& t, int K, Q q) {
  constexpr int E = ElemOf<T>::E;
  const bool same = (reinterpret_cast<uintptr_t>(grad) & 15) == (uintptr_t)s.head * sizeof(T);
  for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
    float f[E];
    unpack<T>(s.chunk(c), f);
    const long long i0 = s.first(c);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = coef * q(f[e]);
    if (same && i0 >= 0 && i0 + E <= s.V) {
      *reinterpret_cast<uint4*>(grad + i0) = pack<T>(f);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i0 + e >= 0 && i0 + e < s.V) grad[i0 + e] = from_float<T>(f[e]);
    }
  }
  __syncthreads();  // the targets' elements are written again, by whichever thread has them
  const int lo = s.lo(), hi = s.hi();
  for (int k = threadIdx.x; k < K; k += blockDim.x) {
    const int id = t.id[k];
    if (id < lo || id >= hi) continue;
    float p = 0.0f;  // entries of the same token add up, in every thread that has one of them alike
    for (int j = 0; j < K; ++j)
      if (t.id[j] == id) p += t.p[j];
    grad[id] = from_float<T>(coef * (q(s.at(id)) - p));
  }
}

template <typename T>
__device__ void write_zeros(const Slice<T>& s, T* grad) {
  constexpr int E = ElemOf<T>::E;
  const bool same = (reinterpret_cast<uintptr_t>(grad) & 15) == (uintptr_t)s.head * sizeof(T);
  for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
    const long long i0 = s.first(c);
    if (same && i0 >= 0 && i0 + E <= s.V) {
      *reinterpret_cast<uint4*>(grad + i0) = make_uint4(0, 0, 0, 0);
    } else {
      for (int e = 0; e < E; ++e)
        if (i0 + e >= 0 && i0 + e < s.V) grad[i0 + e] = from_float<T>(0.0f);
    }
  }
}

template <typename T>
__device__ __forceinline__ T* gradient_row(const DistillArgs& a, long long r) {
  const long long b = r / a.rows.k;
  return static_cast<T*>(a.grad) + b * a.gstride_b + (r - b * a.rows.k) * a.gstride_n;
}

// loss, and with a.grad the gradient: one cluster a row
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_distill(DistillArgs a) {
  extern __shared__ uint4 staged[];
  __shared__ Targets t;
  __shared__ float cta_m, cta_s;
  auto cluster = cg::this_cluster();
  constexpr int E = ElemOf<T>::E;
  const unsigned ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const long long r = blockIdx.x / ctas;
  const float weight = a.weight ? a.weight[r] : 1.0f;
  T* grad = a.grad ? gradient_row<T>(a, r) : nullptr;
  Slice<T> s;
  const bool skip = weight == 0.0f || !teacher(a, r, t);  // the same in all CTAs of the row
  if (skip) {
    a.rows.staged = 0;
    s.open(row_address<T>(a.rows, r), a.rows.V, a.rows, rank, staged);
    if (rank == 0 && threadIdx.x == 0) {
      a.loss[r] = 0.0f;
      if (a.lse) a.lse[r] = 0.0f;
    }
    if (grad) write_zeros(s, grad);
    return;
  }
  s.open(row_address<T>(a.rows, r), a.rows.V, a.rows, rank, staged);
  const float c2 = kLog2e / a.tau;
  ChunkMax<T, true> top;
  s.stage([&](const uint4& c) { top.add(c); });
  float m = top.value();
  m = block_reduce(m, MaxNan(), t.red, &t.value);
  float sum = 0.0f;
  if (m != -CUDART_INF_F)
    for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
      float f[E];
      unpack<T>(s.chunk(c), f);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += exp2_32((f[e] - m) * c2);
    }
  sum = block_reduce(sum, Add(), t.red, &t.value);
  if (threadIdx.x == 0) {
    cta_m = m;
    cta_s = sum;
  }
  cluster.sync();
  m = -CUDART_INF_F;
  for (unsigned i = 0; i < ctas; ++i) m = max_nan(m, *cluster.map_shared_rank(&cta_m, i));
  sum = 0.0f;
  for (unsigned i = 0; i < ctas; ++i) {
    const float mi = *cluster.map_shared_rank(&cta_m, i);
    if (mi != -CUDART_INF_F) sum += *cluster.map_shared_rank(&cta_s, i) * exp2_32((mi - m) * c2);
  }
  const float log_sum = m == -CUDART_INF_F ? -CUDART_INF_F : logf(sum);
  if (rank == 0) {
    float loss = 0.0f;
    for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
      const float p = t.p[k];
      if (t.id[k] < 0 || p == 0.0f) continue;
      const float z = to_float<T>(static_cast<const T*>(row_address<T>(a.rows, r))[t.id[k]]);
      const float lq = z == -CUDART_INF_F ? z : (z - m) / a.tau - log_sum;
      loss += p * (t.lp[k] - lq);
    }
    loss = block_reduce(loss, Add(), t.red, &t.value);
    if (threadIdx.x == 0) {
      a.loss[r] = weight * a.tau * a.tau * loss;
      if (a.lse) a.lse[r] = m == -CUDART_INF_F ? m : m / a.tau + log_sum;
    }
  }
  if (grad) {
    const float scale = m == -CUDART_INF_F ? 0.0f : 1.0f / sum, at = m == -CUDART_INF_F ? 0.0f : m;
    write_gradient(s, grad, weight * a.tau, t, a.K,
                   [=](float z) { return exp2_32((z - at) * c2) * scale; });
  }
  cluster.sync();  // no CTA leaves while its shared memory is read
}

// the gradient from the row's logsumexp: a CTA per slice, nothing shared between them
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_distill_backward(DistillArgs a, int parts) {
  __shared__ Targets t;
  const long long r = blockIdx.x / parts;
  const float weight = a.weight ? a.weight[r] : 1.0f;
  const float coef = weight == 0.0f ? 0.0f : weight * a.tau * a.up[r];
  T* grad = gradient_row<T>(a, r);
  Slice<T> s;
  s.open(row_address<T>(a.rows, r), a.rows.V, a.rows, (int)(blockIdx.x % parts), nullptr);
  if (coef == 0.0f || !teacher(a, r, t)) {
    write_zeros(s, grad);
    return;
  }
  const float inv = 1.0f / a.tau, lse = a.lse_in[r];
  write_gradient(s, grad, coef, t, a.K, [=](float z) {
    return z == -CUDART_INF_F ? 0.0f : exp2_32(fmaf(z, inv, -lse) * kLog2e);
  });
}

template <typename T>
epic_status launch_distill(DistillArgs& a, long long rows, cudaStream_t st) {
  if (a.lse_in) {
    const RowShape p = row_shape(rows, a.rows.V, sizeof(T));
    a.rows.per = p.per;
    a.rows.staged = 0;
    if (rows > 0x7fffffffll / p.ctas) return EPIC_ERR_CAPACITY;
    k_distill_backward<T><<<(unsigned)(rows * p.ctas), p.threads, 0, st>>>(a, p.ctas);
    return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA;
  }
  const RowShape p = row_shape(rows, a.rows.V, sizeof(T));
  a.rows.per = p.per;
  a.rows.staged = p.staged;
  return launch_rows((const void*)k_distill<T>, p, rows, &a, st);
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
  a.rows = {logits, sb, sn, nullptr, n, n, V, 0, 0};
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
