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

constexpr int kListMax = 1024;  // most keys collected for ranking
constexpr int kMaxK = 256;      // most candidates of a position, and the longest top-k list
constexpr int kBins = 1024;     // of a threshold's histogram
constexpr float kBinSpan = 32.0f;        // in powers of two below the maximum; lighter tokens weigh nothing
constexpr float kGrid = 1073741824.0f;   // 2^30: the weights' grid

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

// a bin's mass is low + 2^16 high: parts of 16 and 14 bits of each element's, which 65,536 elements of a slice cannot
// make overflow 32 bits (larger slices go by radix selection)
struct Histogram {
  uint32_t low[kBins], high[kBins];
};

struct TopList {  // a sampler's top-k list, in order
  u64 key[kMaxK];
  u64 first[kMaxK];  // kept mass ahead of the entry in index order
  uint32_t q[kMaxK];
  uint32_t kept[kMaxK];
};

struct PickShared {
  union {
    Histogram bins;
    u64 radix[2][256];
    TopList top;
  };
  u64 list[kListMax];
  u64 coarse[kBins / 32];
  u64 warp_q[kRowWarps];
  u64 cta_q;
  u64 found, before;
  float warp_f[kRowWarps], warp_t[kRowWarps];
  float cta_f, cta_t, cta_s;
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

__device__ __forceinline__ u64 warp_sum(u64 x) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}

// sums up to and with each lane
__device__ __forceinline__ u64 warp_scan(u64 x) {
  const int lane = threadIdx.x % 32;
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(~0u, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

template <typename T>
struct Row {
  Slice<T> s;
  cg::cluster_group cluster;
  PickShared& sh;
  int parity;
  static constexpr int E = ElemOf<T>::E;

  __device__ Row(PickShared& shared) : cluster(cg::this_cluster()), sh(shared), parity(0) {}

  // f(value, index) for the elements of this warp's chunks
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
      float z[E];
      unpack<T>(s.chunk(c), z);
      const long long i0 = s.first(c);
#pragma unroll
      for (int e = 0; e < E; ++e) f(z[e], i0 + e);
    }
  }

  // Stages the row.  Returns its maximum, NaN left out (-inf for a row without elements), and a floor that at least K
  // of its elements reach: the lowest over the row's warps of the j-th largest of the lanes' maxima, j times the number
  // of warps being at least K.  (-inf where that says nothing: K or fewer lanes have elements.)
  __device__ float open_top(int K, float* floor) {
    ChunkMax<T, false> top;
    s.stage([&](const uint4& c) { top.add(c); });
    float m = top.value();
    const int warps = blockDim.x / 32, w = threadIdx.x / 32;
    uint32_t key = value_key(m), jth = 0;
    const int j = (K + warps * (int)cluster.num_blocks() - 1) / (warps * (int)cluster.num_blocks());
    if (j <= 32)
      for (int i = 0; i < j; ++i) {
        jth = __reduce_max_sync(~0u, key);
        if (__ffs(__ballot_sync(~0u, key == jth)) - 1 == (int)(threadIdx.x % 32)) key = 0;
      }
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    if (threadIdx.x % 32 == 0) {
      sh.warp_f[w] = m;
      sh.warp_t[w] = jth ? key_value(jth) : -CUDART_INF_F;
    }
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    if (threadIdx.x == 0) {
      float t = sh.warp_t[0];
      for (int i = 1; i < warps; ++i) {
        m = fmaxf(m, sh.warp_f[i]);
        t = fminf(t, sh.warp_t[i]);
      }
      sh.cta_f = m;
      sh.cta_t = t;
    }
    cluster.sync();
    m = -CUDART_INF_F;
    float t = CUDART_INF_F;
    for (unsigned r = 0; r < cluster.num_blocks(); ++r) {
      m = fmaxf(m, *cluster.map_shared_rank(&sh.cta_f, r));
      t = fminf(t, *cluster.map_shared_rank(&sh.cta_t, r));
    }
    *floor = t;
    return m;
  }

  // keys of elements >= floor to the first CTA's list (past its end they are only counted)
  __device__ void collect(float floor) {
    int* count = cluster.map_shared_rank(&sh.count, 0);
    u64* list = cluster.map_shared_rank(sh.list, 0);
    for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) {
      const uint4 v = s.chunk(c);
      ChunkMax<T, false> top;
      top.add(v);
      if (!(top.value() >= floor)) continue;
      float z[E];
      unpack<T>(v, z);
      const long long i0 = s.first(c);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (z[e] >= floor && z[e] > -CUDART_INF_F) {
          const int at = atomicAdd(count, 1);
          if (at < kListMax) list[at] = order_key(z[e], (int)(i0 + e));
        }
    }
  }

  // After a barrier: the K first keys of the row are in the first CTA's list, with others or (where more than a list
  // was collected) alone.
  __device__ void settle(int K) {
    if (*cluster.map_shared_rank(&sh.count, 0) <= kListMax) return;  // the same in all CTAs
    const u64 floor_key = radix_select<false>(Weigher(), 0, K - 1);
    if (cluster.block_rank() == 0 && threadIdx.x == 0) sh.count = 0;
    cluster.sync();
    int* count = cluster.map_shared_rank(&sh.count, 0);
    u64* list = cluster.map_shared_rank(sh.list, 0);
    each([&](float z, long long i) {
      if (z > -CUDART_INF_F && order_key(z, (int)i) >= floor_key) list[atomicAdd(count, 1)] = order_key(z, (int)i);
    });
    cluster.sync();
  }

  // f(rank, key) for the list's keys, by one thread each
  template <typename F>
  __device__ void ranked(F f) const {
    const int n = sh.count;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const u64 key = sh.list[i];
      int at = 0;
      for (int j = 0; j < n; ++j) at += sh.list[j] > key;
      f(at, key);
    }
  }

  // ---- thresholds

  __device__ __forceinline__ bool in_range(float z, long long i, u64 floor_key) const {
    return z > -CUDART_INF_F && order_key(z, (int)i) >= floor_key;
  }

  // The key of the element, among keys >= floor, at which the running total of the order passes the target: with kMass
  // totals are masses and the target floor(arg all / 2^24) - 1, else they are counts and it is arg (or the last).
  // All ones for a row without elements.  One histogram over evenly spaced exponents finds the bin, whose few elements
  // the first CTA ranks; rows of many equal values go by radix selection.
  template <bool kMass>
  __device__ u64 select(const Weigher& weigh, u64 floor_key, u64 arg) {
    if ((long long)s.n * E > 65536) return radix_select<kMass>(weigh, floor_key, arg);
    for (int i = threadIdx.x; i < kBins; i += blockDim.x) sh.bins.low[i] = sh.bins.high[i] = 0;
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    const float scale = weigh.c * (kBins / kBinSpan);
    const auto bin_of = [&](float z) { return min(__float2uint_rz((weigh.m - z) * scale), (uint32_t)kBins - 1); };
    each([&](float z, long long i) {
      if (!in_range(z, i, floor_key)) return;
      const uint32_t b = bin_of(z);
      if (kMass) {
        const uint32_t q = grid_mass(weigh(z));
        if (q & 0xffffu) atomicAdd(&sh.bins.low[b], q & 0xffffu);
        if (q >> 16) atomicAdd(&sh.bins.high[b], q >> 16);
      } else {
        atomicAdd(&sh.bins.low[b], 1u);
      }
    });
    __syncthreads();
    const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
    for (int g = threadIdx.x / 32; g < kBins / 32; g += warps) {
      const u64 x = warp_sum(sh.bins.low[32 * g + lane] + ((u64)sh.bins.high[32 * g + lane] << 16));
      if (lane == 0) sh.coarse[g] = x;
    }
    cluster.sync();
    if (threadIdx.x < 32) {  // every CTA finds the bin for itself
      static_assert(kBins / 32 == 32, "a lane for each group of bins");
      u64 x = 0;
      for (unsigned r = 0; r < cluster.num_blocks(); ++r) x += *cluster.map_shared_rank(&sh.coarse[lane], r);
      u64 upto = warp_scan(x);
      const u64 all = __shfl_sync(~0u, upto, 31);
      const u64 t = kMass ? share24(arg, all) - 1 : min(arg, all - 1);
      const int g = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
      const u64 ahead = __shfl_sync(~0u, upto - x, g);
      x = 0;
      for (unsigned r = 0; r < cluster.num_blocks(); ++r) {
        const Histogram* h = cluster.map_shared_rank(&sh.bins, r);
        x += h->low[32 * g + lane] + ((u64)h->high[32 * g + lane] << 16);
      }
      upto = ahead + warp_scan(x);
      const int l = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
      const u64 before = __shfl_sync(~0u, upto - x, l);
      if (lane == 0) {
        sh.found = all ? (u64)(32 * g + l) : ~0ull;
        sh.before = t - before;  // the target within the bin
      }
    }
    __syncthreads();
    if (sh.found == ~0ull) {
      cluster.sync();
      return ~0ull;
    }
    const uint32_t bin = (uint32_t)sh.found;
    const u64 t = sh.before;
    int* count = cluster.map_shared_rank(&sh.count, 0);
    u64* list = cluster.map_shared_rank(sh.list, 0);
    each([&](float z, long long i) {
      if (bin_of(z) == bin && in_range(z, i, floor_key)) {
        const int at = atomicAdd(count, 1);
        if (at < kListMax) list[at] = order_key(z, (int)i);
      }
    });
    cluster.sync();
    const int n = *count;
    if (n > kListMax) return radix_select<kMass>(weigh, floor_key, arg);
    if (cluster.block_rank() == 0)
      for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const u64 key = sh.list[i];
        u64 ahead = 0;
        for (int j = 0; j < n; ++j)
          if (sh.list[j] > key) ahead += kMass ? grid_mass(weigh(order_value(sh.list[j]))) : 1u;
        const u64 own = kMass ? grid_mass(weigh(order_value(key))) : 1u;
        if (ahead <= t && t < ahead + own) sh.found = key;
      }
    cluster.sync();
    const u64 key = *cluster.map_shared_rank(&sh.found, 0);
    cluster.sync();
    return key;
  }

  // The same by eight bits of the keys at a time.
  template <bool kMass>
  __device__ u64 radix_select(const Weigher& weigh, u64 floor_key, u64 arg) {
    u64 prefix = 0, before = 0, t = 0;
    cluster.sync();
    for (int shift = 56; shift >= 0; shift -= 8) {
      if (shift < 32 && shift > 0 && s.V > 0 && (uint32_t)(s.V - 1) >> shift == 0) {
        prefix |= 0xffull << shift;  // every index has these bits clear
        continue;
      }
      u64* hist = sh.radix[parity];
      for (int i = threadIdx.x; i < 256; i += blockDim.x) hist[i] = 0;
      __syncthreads();
      each([&](float z, long long i) {
        const u64 key = order_key(z, (int)i);
        if (z > -CUDART_INF_F && key >= floor_key && (shift == 56 || (key ^ prefix) >> (shift + 8) == 0)) {
          const u64 add = kMass ? (u64)grid_mass(weigh(z)) : 1ull;
          if (add) atomicAdd(&hist[(key >> shift) & 255], add);
        }
      });
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
        const u64 upto = before + warp_scan(sum);
        const u64 all = __shfl_sync(~0u, upto, 31) - before;
        if (shift == 56) t = kMass ? share24(arg, all) - 1 : min(arg, all - 1);
        if (all && upto - sum <= t && t < upto) {
          u64 at = upto - sum;
          int i = 0;
          while (at + b[i] <= t) at += b[i++];
          sh.found = prefix | (u64)(255 - 8 * threadIdx.x - i) << shift;
          sh.before = at;
        }
        if (!all && threadIdx.x == 0) sh.found = ~0ull;
      }
      __syncthreads();
      prefix = sh.found;
      before = sh.before;
      parity ^= 1;
      if (prefix == ~0ull) break;
    }
    cluster.sync();
    return prefix;
  }

  // ---- masses and draws

  __device__ __forceinline__ uint32_t kept_mass(float z, long long i, const Weigher& weigh, u64 floor_key,
                                                float min_p) const {
    if (!in_range(z, i, floor_key)) return 0;
    const float w = weigh(z);
    return w >= min_p ? grid_mass(w) : 0;
  }

  __device__ __forceinline__ u64 chunk_mass(int c, const Weigher& weigh, u64 floor_key, float min_p) const {
    float z[E];
    unpack<T>(s.chunk(c), z);
    u64 q = 0;
    if (floor_key == 0 && !(min_p > 0.0f) && weigh.m != CUDART_INF_F) {
      // every token is kept; NaN weighs 0 by the conversion
#pragma unroll
      for (int e = 0; e < E; ++e) q += grid_mass(exp2_32(__fmul_rn(__fsub_rn(z[e], weigh.m), weigh.c)));
      return q;
    }
    const long long i0 = s.first(c);
#pragma unroll
    for (int e = 0; e < E; ++e) q += kept_mass(z[e], i0 + e, weigh, floor_key, min_p);
    return q;
  }

  // Mass of the row's kept keys; *mine is the CTA's part, *ahead that of the CTAs before it, sh.warp_q the warps'.
  __device__ u64 mass(const Weigher& weigh, u64 floor_key, float min_p, u64* mine, u64* ahead) {
    u64 q = 0;
    for (int c = s.wlo + (int)(threadIdx.x % 32); c < s.whi; c += 32) q += chunk_mass(c, weigh, floor_key, min_p);
    q = warp_sum(q);
    if (threadIdx.x % 32 == 0) sh.warp_q[threadIdx.x / 32] = q;
    __syncthreads();
    if (threadIdx.x == 0) {
      q = 0;
      for (int w = 0; w < (int)blockDim.x / 32; ++w) q += sh.warp_q[w];
      sh.cta_q = q;
    }
    cluster.sync();
    u64 all = 0;
    *ahead = *mine = 0;
    for (unsigned r = 0; r < cluster.num_blocks(); ++r) {
      const u64 x = *cluster.map_shared_rank(&sh.cta_q, r);
      if (r == cluster.block_rank()) {
        *ahead = all;
        *mine = x;
      }
      all += x;
    }
    return all;
  }

  // one warp: the token of the slice whose kept mass covers t (counted from the slice's start)
  __device__ void draw(u64 t, const Weigher& weigh, u64 floor_key, float min_p, u64 all, int32_t* tok,
                       float* prob) const {
    const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
    int w = 0;
    while (w < warps - 1 && t >= sh.warp_q[w]) t -= sh.warp_q[w++];
    for (int c0 = w * s.wper; c0 < s.n; c0 += 32) {
      // lanes past the warp's last chunk look into the next one's: the answer is never there
      const int c = c0 + lane;
      const u64 q = c < s.n ? chunk_mass(c, weigh, floor_key, min_p) : 0;
      const u64 upto = warp_scan(q);
      const u64 total = __shfl_sync(~0u, upto, 31);
      if (t >= total) {
        t -= total;
        continue;
      }
      if (t >= upto - q && t < upto) {
        t -= upto - q;
        float z[E];
        unpack<T>(s.chunk(c), z);
        for (int e = 0; e < E; ++e) {
          const uint32_t x = kept_mass(z[e], s.first(c) + e, weigh, floor_key, min_p);
          if (t < x) {
            *tok = (int32_t)(s.first(c) + e);
            *prob = weigh(z[e]) * kGrid / (float)all;
            break;
          }
          t -= x;
        }
      }
      break;
    }
  }

  // the first CTA: draws from the top-k list that settle() left
  __device__ void draw_from_list(const Weigher& weigh, int top_k, u64 p24, float min_p, const float* u, int S,
                                 int32_t* tok, float* prob) {
    TopList& l = sh.top;
    const int n = min(top_k, sh.count);
    ranked([&](int at, u64 key) {
      if (at < n) {
        l.key[at] = key;
        l.q[at] = grid_mass(weigh(order_value(key)));
      }
    });
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      u64 before = 0, all = 0;
      for (int j = 0; j < n; ++j) {
        all += l.q[j];
        if (j < i) before += l.q[j];
      }
      l.kept[i] = i == 0 || (before < share24(p24, all) && weigh(order_value(l.key[i])) >= min_p) ? l.q[i] : 0;
    }
    __syncthreads();
    u64 all = 0;
    for (int j = 0; j < n; ++j) all += l.kept[j];
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const int index = order_index(l.key[i]);
      u64 first = 0;
      for (int j = 0; j < n; ++j)
        if (order_index(l.key[j]) < index) first += l.kept[j];
      l.first[i] = first;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < S; d += blockDim.x) {
      const float x = u[d];
      int token = -1;
      float p = 0.0f;
      if (all && x >= 0.0f && x <= 1.0f) {
        const u64 t = min(share24((u64)(x * 16777216.0f), all), all - 1);
        int i = 0;
        while (i < n - 1 && !(t >= l.first[i] && t < l.first[i] + l.kept[i])) ++i;
        token = order_index(l.key[i]);
        p = weigh(order_value(l.key[i])) * kGrid / (float)all;
      }
      tok[d] = token;
      prob[d] = p;
    }
  }
};

// sum of the row's weights over a CTA's warps: `total` is the sum in order of warps, in every thread of the CTA
__device__ __forceinline__ float cta_sum(float x, PickShared& sh) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  if (threadIdx.x % 32 == 0) sh.warp_t[threadIdx.x / 32] = x;
  __syncthreads();
  x = 0.0f;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) x += sh.warp_t[w];
  return x;
}

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
  Weigher weigh;
  float floor;
  weigh.m = row.open_top(a.K, &floor);
  weigh.c = fminf(__fdiv_rn(kLog2e, T_), CUDART_MAX_NORMAL_F);
  row.collect(floor);
  // The sum of the weights, each with its exponent in one fused step: what the rounding of m c adds is common to all
  // and leaves with the division.  NaN and infinities make that sum NaN; it is then taken again with care.
  const float mc = weigh.m * weigh.c;
  float sum = 0.0f;
  for (int c = row.s.wlo + (int)(threadIdx.x % 32); c < row.s.whi; c += 32) {
    float z[E];
    unpack<T>(row.s.chunk(c), z);
#pragma unroll
    for (int e = 0; e < E; ++e) sum += exp2_32(fmaf(z[e], weigh.c, -mc));
  }
  sum = cta_sum(sum, sh);
  if (threadIdx.x == 0) sh.cta_s = sum;
  row.cluster.sync();
  sum = 0.0f;
  for (unsigned i = 0; i < ctas; ++i) sum += *row.cluster.map_shared_rank(&sh.cta_s, i);
  const bool fused = sum == sum;  // the same in all CTAs
  if (!fused) {
    sum = 0.0f;
    row.each([&](float z, long long) {
      const float w = weigh(z);
      sum += w > 0.0f ? w : 0.0f;
    });
    row.cluster.sync();
    sum = cta_sum(sum, sh);
    if (threadIdx.x == 0) sh.cta_s = sum;
    row.cluster.sync();
    sum = 0.0f;
    for (unsigned i = 0; i < ctas; ++i) sum += *row.cluster.map_shared_rank(&sh.cta_s, i);
  }
  row.settle(a.K);
  if (rank == 0) {
    int32_t* cand = a.cand + r * a.K;
    float* conf = a.conf + r * a.K;
    for (int i = sh.count + threadIdx.x; i < a.K; i += blockDim.x) {
      cand[i] = -1;
      conf[i] = 0.0f;
    }
    row.ranked([&](int at, u64 key) {
      if (at >= a.K) return;
      const float z = order_value(key);
      cand[at] = order_index(key);
      conf[at] = T_ == 0.0f ? (at == 0 ? 1.0f : 0.0f) : (fused ? exp2_32(fmaf(z, weigh.c, -mc)) : weigh(z)) / sum;
    });
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
  if (top_k <= 0 || top_k > a.rows.V) top_k = a.rows.V;
  const bool by_list = top_k <= kMaxK;
  row.s.open(good ? row_address<T>(a.rows, r) : nullptr, a.rows.V, a.rows, rank, staged);
  Weigher weigh;
  float floor;
  weigh.m = row.open_top(by_list ? top_k : 0, &floor);
  weigh.c = fminf(__fdiv_rn(kLog2e, T_), CUDART_MAX_NORMAL_F);
  if (by_list) {
    row.collect(floor);
    row.cluster.sync();
    row.settle(top_k);
    if (rank == 0)
      row.draw_from_list(weigh, top_k, p24, min_p, a.u + r * a.S, a.S, a.tok + r * a.S, a.prob + r * a.S);
    row.cluster.sync();
    return;
  }
  u64 floor_key = 0, mine, ahead;
  if (top_k < a.rows.V) floor_key = row.template select<false>(weigh, 0, top_k - 1);
  if (p24 < (1u << 24)) floor_key = row.template select<true>(weigh, floor_key, p24);
  const u64 all = row.mass(weigh, floor_key, min_p, &mine, &ahead);
  for (int i = threadIdx.x / 32; i < a.S; i += blockDim.x / 32) {
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
    if (t >= ahead && t < ahead + mine) row.draw(t - ahead, weigh, floor_key, min_p, all, &a.tok[o], &a.prob[o]);
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
