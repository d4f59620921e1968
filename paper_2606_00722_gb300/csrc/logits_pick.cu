// Candidates from logits: the K best tokens of a position with their softmax
// confidences (epic_propose_topk), and draws with temperature, top-k, top-p and
// min-p from given uniform numbers (epic_sample_tokens).
//
// With m the row's maximum and c = log2(e) / T a token's weight is
// w = 2^((z - m) c), every operation rounded to 32 bits.  Confidences are w over
// the sum of w in 32 bits.  Sampling adds whole numbers instead,
// q = rint(2^30 w) in 64 bits: such sums are exact, so which token a number
// draws depends on the row and the number alone, not on how the row was split
// (a float CDF over 126,000 tokens has so many boundaries that two orders of
// summation disagree on a draw every few hundred rows).  The grid drops tokens
// less likely than 2^-31 of the likeliest.
//
// The kept tokens of a draw are a prefix of the row's order cut by top-k, then by
// the nucleus, each found as a threshold key by radix selection on counts or on
// masses; the draw is the first kept token in index order whose mass up to and
// with it passes u times the kept mass.
#include "../../include/epic.h"
#include "logit_launch.h"
#include "logit_rows.cuh"

namespace epic {
namespace {

constexpr int kListMax = 1024;   // most keys collected for ranking
constexpr int kMaxK = 256;       // most candidates of a position
constexpr float kGrid = 1073741824.0f;  // 2^30: the weights' grid

struct PickArgs {
  RowArgs rows;
  const float* temperature;  // [B] or NULL
  int K;                     // propose
  int32_t* cand;
  float* conf;
  const int32_t* top_k;  // sample: [B] or NULL
  const float* top_p;
  const float* min_p;
  const float* u;
  int S;
  int32_t* tok;
  float* prob;
};

struct PickShared {
  u64 hist[2][256];
  u64 warp_q[kRowWarps];
  u64 cta_q;
  u64 list[kListMax];
  u64 found, before;
  float warp_f[kRowWarps];
  float cta_f;
  int count;
};

// 2^((z - m) c); a row whose maximum is +inf has weight 1 on its +inf elements and 0 elsewhere
struct Weigher {
  float m, c;
  __device__ __forceinline__ float operator()(float z) const {
    if (m == CUDART_INF_F) return z == m ? 1.0f : 0.0f;
    return exp2_32(__fmul_rn(__fsub_rn(z, m), c));
  }
};

__device__ __forceinline__ uint32_t grid_mass(float w) { return __float2uint_rn(w * kGrid); }

// floor(a q / 2^24) for a <= 2^24, without passing 64 bits
__device__ __forceinline__ u64 share24(u64 a, u64 q) { return a * (q >> 24) + ((a * (q & 0xffffffu)) >> 24); }

template <typename T>
struct Row {
  Slice<T> s;
  cg::cluster_group cluster;
  PickShared& sh;
  int parity;
  static constexpr int E = ElemOf<T>::E;

  __device__ Row(PickShared& shared) : cluster(cg::this_cluster()), sh(shared), parity(0) {}

  // maximum of the row, NaN left out; -inf for a row without elements
  __device__ float maximum() {
    float m = -CUDART_INF_F;
    for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
      float f[E];
      unpack<T>(s.chunk(c), f);
#pragma unroll
      for (int e = 0; e < E; ++e) m = fmaxf(m, f[e]);
    }
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    if (threadIdx.x % 32 == 0) sh.warp_f[threadIdx.x / 32] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < (int)blockDim.x / 32; ++w) m = fmaxf(m, sh.warp_f[w]);
      sh.cta_f = m;
    }
    cluster.sync();
    m = -CUDART_INF_F;
    for (unsigned r = 0; r < cluster.num_blocks(); ++r) m = fmaxf(m, *cluster.map_shared_rank(&sh.cta_f, r));
    return m;
  }

  // The key of the element whose share of the running total covers `target`: with kMass, masses of keys >= floor in
  // order, else counts.  A target past the end gives the last element; a row without elements gives all ones.
  template <bool kMass>
  __device__ u64 select(const Weigher& weigh, u64 floor_key, u64 target) {
    u64 prefix = 0, before = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
      if (shift < 32 && (uint32_t)(s.V - 1) >> shift == 0 && shift > 0 && s.V > 0) {
        prefix |= 0xffull << shift;  // every index has these bits clear
        continue;
      }
      u64* hist = sh.hist[parity];
      for (int i = threadIdx.x; i < 256; i += blockDim.x) hist[i] = 0;
      __syncthreads();
      for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
        float f[E];
        unpack<T>(s.chunk(c), f);
        const long long i0 = s.first(c);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const u64 key = order_key(f[e], (int)(i0 + e));
          if (f[e] > -CUDART_INF_F && key >= floor_key && (shift == 56 || (key ^ prefix) >> (shift + 8) == 0)) {
            const u64 add = kMass ? (u64)grid_mass(weigh(f[e])) : 1ull;
            if (add) atomicAdd(&hist[(key >> shift) & 255], add);
          }
        }
      }
      cluster.sync();
      if (threadIdx.x < 32) {
        // lane l holds bins 255 - 8 l downwards: a scan over lanes is a scan down the order
        u64 b[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          b[i] = 0;
          for (unsigned r = 0; r < cluster.num_blocks(); ++r)
            b[i] += *cluster.map_shared_rank(&hist[255 - 8 * threadIdx.x - i], r);
          sum += b[i];
        }
        u64 upto = sum;
        for (int o = 1; o < 32; o <<= 1) {
          const u64 x = __shfl_up_sync(~0u, upto, o);
          if ((int)threadIdx.x >= o) upto += x;
        }
        const u64 total = __shfl_sync(~0u, upto, 31);
        const u64 t = total && before + total <= target ? before + total - 1 : target;
        const bool mine = total && before + upto - sum <= t && t < before + upto;
        if (mine) {
          u64 at = before + upto - sum;
          int i = 0;
          while (at + b[i] <= t) at += b[i++];
          sh.found = prefix | (u64)(255 - 8 * threadIdx.x - i) << shift;
          sh.before = at;
        }
        if (!total && threadIdx.x == 0) sh.found = ~0ull;
      }
      __syncthreads();
      prefix = sh.found;
      before = sh.before;
      parity ^= 1;
      if (prefix == ~0ull) break;
    }
    return prefix;
  }

  // mass of the row's keys >= floor with w >= min_p; sh.warp_q and sh.cta_q hold the CTA's parts
  __device__ u64 mass(const Weigher& weigh, u64 floor_key, float min_p, u64* mine, u64* ahead) {
    u64 q = 0;
    for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) q += chunk_mass(c, weigh, floor_key, min_p);
    for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if (threadIdx.x % 32 == 0) sh.warp_q[threadIdx.x / 32] = q;
    __syncthreads();
    if (threadIdx.x == 0) {
      q = 0;
      for (int w = 0; w < (int)blockDim.x / 32; ++w) q += sh.warp_q[w];
      sh.cta_q = q;
    }
    cluster.sync();
    u64 all = 0;
    *ahead = 0;
    for (unsigned r = 0; r < cluster.num_blocks(); ++r) {
      const u64 x = *cluster.map_shared_rank(&sh.cta_q, r);
      if (r == cluster.block_rank()) {
        *ahead = all;
        *mine = x;
      }
      all += x;
    }
    cluster.sync();  // cta_q may be written again
    return all;
  }

  __device__ __forceinline__ uint32_t kept_mass(float z, long long idx, const Weigher& weigh, u64 floor_key,
                                                float min_p) const {
    if (!(z > -CUDART_INF_F) || order_key(z, (int)idx) < floor_key) return 0;
    const float w = weigh(z);
    return w >= min_p ? grid_mass(w) : 0;
  }

  __device__ u64 chunk_mass(int c, const Weigher& weigh, u64 floor_key, float min_p) const {
    float f[E];
    unpack<T>(s.chunk(c), f);
    const long long i0 = s.first(c);
    u64 q = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) q += kept_mass(f[e], i0 + e, weigh, floor_key, min_p);
    return q;
  }

  // one warp: the token of the slice whose kept mass covers t (counted from the slice's start)
  __device__ void draw(u64 t, const Weigher& weigh, u64 floor_key, float min_p, u64 all, int32_t* tok, float* prob) {
    const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
    const int wper = (((s.n + warps - 1) / warps) + 31) & ~31;
    int w = 0;
    while (w < warps - 1 && t >= sh.warp_q[w]) t -= sh.warp_q[w++];
    for (int c0 = w * wper; c0 < s.n; c0 += 32) {
      const int c = c0 + lane;
      const u64 q = c < s.n ? chunk_mass(c, weigh, floor_key, min_p) : 0;
      u64 upto = q;
      for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += x;
      }
      const u64 total = __shfl_sync(~0u, upto, 31);
      if (t >= total) {
        t -= total;
        continue;
      }
      if (t >= upto - q && t < upto) {
        t -= upto - q;
        float f[E];
        unpack<T>(s.chunk(c), f);
        for (int e = 0; e < E; ++e) {
          const uint32_t x = kept_mass(f[e], s.first(c) + e, weigh, floor_key, min_p);
          if (t < x) {
            *tok = (int32_t)(s.first(c) + e);
            *prob = weigh(f[e]) * kGrid / (float)all;
            break;
          }
          t -= x;
        }
      }
      break;
    }
  }
};

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_propose(PickArgs a) {
  extern __shared__ uint4 staged[];
  __shared__ PickShared sh;
  Row<T> row(sh);
  constexpr int E = ElemOf<T>::E;
  const unsigned ctas = row.cluster.num_blocks(), rank = row.cluster.block_rank();
  const long long r = blockIdx.x / ctas;
  const float T_ = a.temperature ? a.temperature[r / a.rows.k] : 1.0f;
  const void* addr = T_ >= 0.0f ? row_address<T>(a.rows, r) : nullptr;
  row.s.open(addr, a.rows.V, a.rows, rank, staged);
  if (threadIdx.x == 0) sh.count = 0;
  Weigher weigh;
  weigh.m = row.maximum();
  weigh.c = fminf(__fdiv_rn(kLog2e, T_), CUDART_MAX_NORMAL_F);
  const u64 floor_key = row.template select<false>(weigh, 0, a.K - 1);
  // sum of the weights; keys from the floor on go to the first CTA's list
  int* count = row.cluster.map_shared_rank(&sh.count, 0);
  u64* list = row.cluster.map_shared_rank(sh.list, 0);
  float sum = 0.0f;
  for (int c = row.s.wlo + (int)(threadIdx.x % 32); c < row.s.whi; c += 32) {
    float f[E];
    unpack<T>(row.s.chunk(c), f);
    const long long i0 = row.s.first(c);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float w = weigh(f[e]);
      sum += w > 0.0f ? w : 0.0f;
      if (f[e] > -CUDART_INF_F) {
        const u64 key = order_key(f[e], (int)(i0 + e));
        if (key >= floor_key) list[atomicAdd(count, 1)] = key;
      }
    }
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  if (threadIdx.x % 32 == 0) sh.warp_f[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0f;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) sum += sh.warp_f[w];
    sh.cta_f = sum;
  }
  row.cluster.sync();
  if (rank == 0) {
    sum = 0.0f;
    for (unsigned i = 0; i < ctas; ++i) sum += *row.cluster.map_shared_rank(&sh.cta_f, i);
    const int n = sh.count;
    for (int i = threadIdx.x; i < a.K; i += blockDim.x)
      if (i >= n) {
        a.cand[r * a.K + i] = -1;
        a.conf[r * a.K + i] = 0.0f;
      }
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const u64 key = sh.list[i];
      int at = 0;
      for (int j = 0; j < n; ++j) at += sh.list[j] > key;
      a.cand[r * a.K + at] = order_index(key);
      a.conf[r * a.K + at] = T_ == 0.0f ? (at == 0 ? 1.0f : 0.0f) : weigh(order_value(key)) / sum;
    }
  }
  row.cluster.sync();  // no CTA leaves while its shared memory is read
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_sample(PickArgs a) {
  extern __shared__ uint4 staged[];
  __shared__ PickShared sh;
  Row<T> row(sh);
  const unsigned ctas = row.cluster.num_blocks(), rank = row.cluster.block_rank();
  const long long r = blockIdx.x / ctas, b = r / a.rows.k;
  const float T_ = a.temperature ? a.temperature[b] : 1.0f;
  float top_p = a.top_p ? a.top_p[b] : 1.0f;
  const float min_p = a.min_p ? a.min_p[b] : 0.0f;
  int top_k = a.top_k ? a.top_k[b] : 0;
  const bool good = T_ >= 0.0f && top_p == top_p && min_p == min_p;
  top_p = fminf(fmaxf(top_p, 0.0f), 1.0f);
  const u64 p24 = __float2uint_rn(top_p * 16777216.0f);
  if (T_ == 0.0f || p24 == 0 || min_p > 1.0f) top_k = 1;
  row.s.open(good ? row_address<T>(a.rows, r) : nullptr, a.rows.V, a.rows, rank, staged);
  Weigher weigh;
  weigh.m = row.maximum();
  weigh.c = fminf(__fdiv_rn(kLog2e, T_), CUDART_MAX_NORMAL_F);
  const float floor_w = top_k == 1 ? 0.0f : min_p;
  u64 floor_key = 0, mine = 0, ahead = 0;
  if (top_k > 0 && top_k < a.rows.V) floor_key = row.template select<false>(weigh, 0, top_k - 1);
  if (p24 < (1u << 24) && top_k != 1) {
    const u64 all = row.mass(weigh, floor_key, 0.0f, &mine, &ahead);
    if (all) floor_key = row.template select<true>(weigh, floor_key, share24(p24, all) - 1);
  }
  const u64 all = row.mass(weigh, floor_key, floor_w, &mine, &ahead);
  const int warps = blockDim.x / 32;
  for (int i = threadIdx.x / 32; i < a.S; i += warps) {
    const long long o = r * a.S + i;
    const float u = a.u[o];
    if (all == 0 || !(u >= 0.0f && u <= 1.0f)) {
      if (rank == 0 && threadIdx.x % 32 == 0) {
        a.tok[o] = -1;
        a.prob[o] = 0.0f;
      }
      continue;
    }
    const u64 t = min(share24((u64)(u * 16777216.0f), all), all - 1);
    if (t >= ahead && t < ahead + mine) row.draw(t - ahead, weigh, floor_key, floor_w, all, &a.tok[o], &a.prob[o]);
  }
  row.cluster.sync();
}

template <typename T>
epic_status launch(PickArgs& a, long long rows, bool sample, cudaStream_t st) {
  const RowShape p = row_shape(rows, a.rows.V, sizeof(T));
  a.rows.per = p.per;
  a.rows.staged = p.staged;
  return launch_rows(sample ? (const void*)k_sample<T> : (const void*)k_propose<T>, p, rows, &a, st);
}

epic_status by_type(int dtype, PickArgs& a, long long rows, bool sample, void* stream) {
  cudaStream_t st = (cudaStream_t)stream;
  switch (dtype) {
    case EPIC_F32: return launch<float>(a, rows, sample, st);
    case EPIC_F16: return launch<__half>(a, rows, sample, st);
    default: return launch<__nv_bfloat16>(a, rows, sample, st);
  }
}

}  // namespace
}  // namespace epic

extern "C" {

epic_status epic_propose_topk(const void* d_logits, int32_t dtype, int32_t B, int32_t n, int32_t V, int64_t stride_b,
                              int64_t stride_n, const int32_t* d_pos, int32_t k, const float* d_temperature,
                              int32_t K, int32_t* d_cand, float* d_conf, void* cuda_stream) {
  using namespace epic;
  if (K < 0) return EPIC_ERR_INVALID_ARG;
  epic_status s = check_rows(d_logits, dtype, B, n, V, stride_b, stride_n, d_pos, k);
  if (s != EPIC_OK) return s;
  if (K > kMaxK) return EPIC_ERR_CAPACITY;
  const long long rows = (long long)B * k;
  if (rows == 0 || K == 0) return EPIC_OK;
  if (!d_cand || !d_conf) return EPIC_ERR_INVALID_ARG;
  PickArgs a = {};
  a.rows = {d_logits, stride_b, stride_n, d_pos, n, k, V, 0, 0};
  a.temperature = d_temperature;
  a.K = K;
  a.cand = d_cand;
  a.conf = d_conf;
  return by_type(dtype, a, rows, false, cuda_stream);
}

epic_status epic_sample_tokens(const void* d_logits, int32_t dtype, int32_t B, int32_t n, int32_t V, int64_t stride_b,
                               int64_t stride_n, const int32_t* d_pos, int32_t k, const float* d_temperature,
                               const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, const float* d_u,
                               int32_t S, int32_t* d_tok, float* d_prob, void* cuda_stream) {
  using namespace epic;
  if (S < 0) return EPIC_ERR_INVALID_ARG;
  epic_status s = check_rows(d_logits, dtype, B, n, V, stride_b, stride_n, d_pos, k);
  if (s != EPIC_OK) return s;
  const long long rows = (long long)B * k;
  if (rows == 0 || S == 0) return EPIC_OK;
  if (!d_u || !d_tok || !d_prob) return EPIC_ERR_INVALID_ARG;
  PickArgs a = {};
  a.rows = {d_logits, stride_b, stride_n, d_pos, n, k, V, 0, 0};
  a.temperature = d_temperature;
  a.top_k = d_top_k;
  a.top_p = d_top_p;
  a.min_p = d_min_p;
  a.u = d_u;
  a.S = S;
  a.tok = d_tok;
  a.prob = d_prob;
  return by_type(dtype, a, rows, true, cuda_stream);
}

}  // extern "C"
