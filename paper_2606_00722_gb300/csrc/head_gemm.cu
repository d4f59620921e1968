// The three matrix products of the head's loss, in their simplest form: a CTA
// computes a tile of 64 x 64 with operands staged in shared memory in 32 bits.
#include "head_loss.h"
#include "head_rows.cuh"

namespace epic {
namespace {

constexpr int kT = 64, kStep = 16;

struct Tile {
  float a[kStep][kT + 1], b[kStep][kT + 1];
  float out[kT][kT + 1];
};

// out = sum_k fa(k, m) fb(k, n) over the tile at (m0, n0)
template <typename FA, typename FB>
__device__ void tile_product(Tile& t, int K, FA fa, FB fb) {
  float acc[4][4] = {};
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int k0 = 0; k0 < K; k0 += kStep) {
    for (int i = threadIdx.x; i < kStep * kT; i += 256) {
      const int k = i / kT, m = i % kT;
      t.a[k][m] = k0 + k < K ? fa(k0 + k, m) : 0.0f;
      t.b[k][m] = k0 + k < K ? fb(k0 + k, m) : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < kStep; k++)
      for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) acc[i][j] = fmaf(t.a[k][ty * 4 + i], t.b[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; i++)
    for (int j = 0; j < 4; j++) t.out[ty * 4 + i][tx * 4 + j] = acc[i][j];
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(256) k_head_logits(HeadPlan p, LogitsPass pass) {
  __shared__ Tile t;
  if (pass.only_again && *p.again == 0) return;
  const int n = *p.count, m0 = blockIdx.y * kT, v0 = blockIdx.x * kT;
  if (m0 >= (n + kRowTile - 1) / kRowTile * kRowTile) return;
  const T* h = (const T*)p.hc;
  const T* w = (const T*)p.head;
  tile_product(t, p.d, [&](int k, int m) { return as_float(h[(m0 + m) * p.ldh + k]); },
               [&](int k, int v) { return v0 + v < p.V ? as_float(w[(v0 + v) * p.ldw + k]) : 0.0f; });
  if (threadIdx.x >= kT) return;
  const int r = m0 + threadIdx.x, end = min(kT, p.V - v0);
  const float* z = t.out[threadIdx.x];
  const bool real = r < n;
  const int y = real ? p.tgt[r] - v0 : -1;
  const float ref = !real || !pass.probs ? 0.0f : p.ref[r];
  if (pass.sums && real) {
    float m = -CUDART_INF_F;
    for (int j = 0; j < end; j++)
      if (j != y) m = fmaxf(m, z[j]);
    float to = whole_ref(m);
    if (pass.probs && !(m * kLog2E > ref + kWindow)) to = ref;
    float s = 0.0f;
    for (int j = 0; j < end; j++)
      if (j != y) s += ex2(fmaf(z[j], kLog2E, -to));
    p.rec[(long long)blockIdx.x * p.cap + r] = record(to, s);
    if (y >= 0 && y < end) p.zt[r] = z[y];
  }
  if (pass.probs) {
    T* e = (T*)p.e + r * p.lde + v0;
    for (int j = 0; j < kT && v0 + j < p.lde; j++) {
      float v = real && j < end ? ex2(fmaf(z[j], kLog2E, -ref)) : 0.0f;
      if (real && j == y) v = pass.only_again ? p.at[r] : v;
      e[j] = of_float<T>(v);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_hidden_grad(HeadPlan p, HiddenGrad g) {
  __shared__ Tile t;
  const int n = *p.count, m0 = blockIdx.y * kT, c0 = blockIdx.x * kT;
  if (m0 >= n) return;
  const T* e = (const T*)p.e;
  const T* w = (const T*)p.head;
  tile_product(t, p.V, [&](int k, int m) { return as_float(e[(m0 + m) * p.lde + k]); },
               [&](int k, int c) { return c0 + c < p.d ? as_float(w[k * p.ldw + c0 + c]) : 0.0f; });
  for (int i = threadIdx.x; i < kT * kT; i += 256) {
    const int m = i / kT, c = i % kT;
    if (m0 + m >= n || c0 + c >= p.d) continue;
    const long long r = g.r0 + p.src[m0 + m];
    T* out = (T*)g.grad + (r / g.n) * g.stride_b + (r % g.n) * g.stride_n;
    out[c0 + c] = of_float<T>(t.out[m][c] * p.coef[m0 + m]);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_head_grad(HeadPlan p, T* grad, long long stride, HeadSum sum) {
  __shared__ Tile t;
  const int n = *p.count, v0 = blockIdx.x * kT, c0 = blockIdx.y * kT;
  const T* e = (const T*)p.e;
  const T* h = (const T*)p.hs;
  tile_product(t, n, [&](int k, int v) { return v0 + v < p.V ? as_float(e[k * p.lde + v0 + v]) : 0.0f; },
               [&](int k, int c) { return c0 + c < p.d ? as_float(h[k * p.ldh + c0 + c]) : 0.0f; });
  const float post = *p.post;
  for (int i = threadIdx.x; i < kT * kT; i += 256) {
    const int v = i / kT, c = i % kT;
    if (v0 + v >= p.V || c0 + c >= p.d) continue;
    float x = t.out[v][c] * post;
    float* acc = p.acc + (long long)(v0 + v) * p.d + c0 + c;
    if (sum == kMiddle || sum == kLast) x += *acc;
    if (sum == kFirst || sum == kMiddle) *acc = x;
    else grad[(v0 + v) * stride + c0 + c] = of_float<T>(x);
  }
}

epic_status launched() { return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA; }

unsigned tiles(long long n) { return (unsigned)((n + kT - 1) / kT); }

}  // namespace

epic_status launch_head_logits(const HeadPlan& p, int dtype, const LogitsPass& pass, cudaStream_t st) {
  const dim3 grid(tiles(p.V), tiles(p.cap));
  if (dtype == EPIC_F16) k_head_logits<__half><<<grid, 256, 0, st>>>(p, pass);
  else k_head_logits<__nv_bfloat16><<<grid, 256, 0, st>>>(p, pass);
  return launched();
}

epic_status launch_hidden_grad(const HeadPlan& p, int dtype, const HiddenGrad& out, cudaStream_t st) {
  const dim3 grid(tiles(p.d), tiles(p.cap));
  if (dtype == EPIC_F16) k_hidden_grad<__half><<<grid, 256, 0, st>>>(p, out);
  else k_hidden_grad<__nv_bfloat16><<<grid, 256, 0, st>>>(p, out);
  return launched();
}

epic_status launch_head_grad(const HeadPlan& p, int dtype, void* grad, long long stride, HeadSum sum, cudaStream_t st) {
  const dim3 grid(tiles(p.V), tiles(p.d));
  if (dtype == EPIC_F16) k_head_grad<__half><<<grid, 256, 0, st>>>(p, (__half*)grad, stride, sum);
  else k_head_grad<__nv_bfloat16><<<grid, 256, 0, st>>>(p, (__nv_bfloat16*)grad, stride, sum);
  return launched();
}

}  // namespace epic
