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

constexpr int kListMax = 512;   // most keys collected for ranking
constexpr int kMaxK = 256;      // most candidates of a position, and the longest top-k list
constexpr int kBins = 2048;     // of a threshold's histogram
constexpr int kGroups = kBins / 32;
constexpr int kParts = 32;      // masses kept of a warp's chunks
constexpr int kTops = 2 * kMaxK + kRowWarps * kRowCluster;
constexpr float kBinsPerUnit = kBins / 32;  // bins to a power of two; past 2^-32 of the maximum weights are 0
constexpr float kGrid = 1073741824.0f;      // 2^30: the weights' grid
constexpr float kMagic = 12582912.0f;       // 1.5 * 2^23: x + kMagic holds rint(x) in its low bits, |x| < 2^22
constexpr uint32_t kMagicBits = 0x4b400000u;

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

// a bin's mass is low + 2^15 high: parts of 15 and 16 bits of each element's mass, whose sums over a slice of at most
// kSliceElems elements fit 32 bits
struct Histogram {
  uint32_t low[kBins], high[kBins];
  u64 group[kGroups];
};

struct TopList {  // a sampler's top-k list, in order
  u64 key[kMaxK];
  u64 first[kMaxK];  // kept mass ahead of the entry in index order
  uint32_t q[kMaxK];
  uint32_t kept[kMaxK];
};

struct Tops {  // largest lane maxima (value keys): of this CTA's warps, and of all of the row's
  uint32_t mine[kTops], all[kTops];
};

struct PickShared {
  union {
    Histogram bins;
    u64 radix[2][256];
    TopList top;
    Tops tops;
  };
  u64 list[kListMax];
  u64 parts[kRowWarps][kParts];  // kept masses by runs of batches
  u64 warp_q[kRowWarps];         // and by warp
  u64 found, before;
  uint32_t row_top, row_floor;  // value keys
  float warp_sum[kRowWarps];
  float sums[kRowCluster];  // in the first CTA
  int count;
};

// 2^((z - m) c); a row whose maximum is +inf has weight 1 on its +inf elements and 0 elsewhere
struct Weigher {
  float m, c;
  __device__ __forceinline__ float operator()(float z) const {
    if (m == CUDART_INF_F) return z == m ? 1.0f : 0.0f;
    return exp2_32(__fmul_rn(__fsub_rn(z, m), c));
  }
  // exponents of two elements
  __device__ __forceinline__ float2 exponents(float a, float b) const {
    return mul2(add2(make_float2(a, b), make_float2(-m, -m)), make_float2(c, c));
  }
  // Whether all elements up to `top` weigh less than 2^-8, so that their masses are below 2^22.  False for NaN.
  __device__ __forceinline__ bool light(float top) const { return __fmul_rn(__fsub_rn(top, m), c) < -8.01f; }
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

// Which tokens are kept: keys from floor_key on, with a weight of at least min_p.
struct Kept {
  u64 floor_key;
  float min_p;
  __device__ __forceinline__ bool all() const { return floor_key == 0 && !(min_p > 0.0f); }
};

template <typename T>
struct Row {
  Slice<T> s;
  cg::cluster_group cluster;
  PickShared& sh;
  int parity;
  static constexpr int E = ElemOf<T>::E;

  __device__ Row(PickShared& shared) : cluster(cg::this_cluster()), sh(shared), parity(0) {}

  // f(value, index) for the elements of this warp's chunks (and -inf past their end)
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(v[i], z);
        const int i0 = s.first(c + 32 * i);
#pragma unroll
        for (int e = 0; e < E; ++e) f(z[e], i0 + e);
      }
    });
  }

  // The row's maximum from the lanes' (NaN left out, -inf for a row without elements).  For K > 0 *floor is a value
  // that at least K elements reach (or -inf): the K-th largest of the largest j lane maxima of every warp, where j gives
  // twice K of them.  About 1.4 K elements of a row in random order reach it; the lowest of the warps' j-th, which needs
  // no ranking, lets ten times K through at one lane maximum a warp.
  __device__ float top_of(float lane_top, int K, float* floor) {
    const int warps = blockDim.x / 32, w = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int all = warps * (int)cluster.num_blocks();
    const int j = K > 0 ? min((2 * K + all - 1) / all, 32) : 1;
    uint32_t key = value_key(lane_top);
    for (int i = 0; i < j; ++i) {
      const uint32_t x = __reduce_max_sync(~0u, key);
      if (lane == 0) sh.tops.mine[w * j + i] = x;
      if (__ffs(__ballot_sync(~0u, key == x)) - 1 == lane) key = 0;
    }
    if (threadIdx.x == 0) {
      sh.count = 0;
      sh.row_floor = 0;
    }
    cluster.sync();
    const int n = all * j, per = warps * j;
    if (K == 0) {  // every warp looks at all warps of the row
      uint32_t m = 0;
      for (int i = lane; i < n; i += 32) m = max(m, *cluster.map_shared_rank(&sh.tops.mine[i % per], i / per));
      m = __reduce_max_sync(~0u, m);
      cluster.sync();  // the tops' memory is free
      return key_value(m);
    }
    for (int i = threadIdx.x; i < n; i += blockDim.x)
      sh.tops.all[i] = *cluster.map_shared_rank(&sh.tops.mine[i % per], i / per);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const uint32_t x = sh.tops.all[i];
      int above = 0;
      for (int o = 0; o < n; ++o) above += sh.tops.all[o] > x || (sh.tops.all[o] == x && o < i);
      if (above == 0) sh.row_top = x;
      if (above == K - 1) sh.row_floor = x;
    }
    __syncthreads();
    *floor = sh.row_floor ? key_value(sh.row_floor) : -CUDART_INF_F;
    return key_value(sh.row_top);
  }

  __device__ float lane_maximum() const {
    ChunkMax<T, false> top;
    s.sweep([&](const uint4 (&v)[4], int) { top.add(v); });
    return top.value();
  }

  // Keys of elements >= floor to the first CTA's list (past its end they are only counted).  A lane whose maximum
  // reaches the floor has such elements; its chunks are looked at by the whole warp.
  __device__ void collect(float floor, float lane_top) {
    int* count = cluster.map_shared_rank(&sh.count, 0);
    u64* list = cluster.map_shared_rank(sh.list, 0);
    const int lane = threadIdx.x % 32;
    for (uint32_t who = __ballot_sync(~0u, lane_top >= floor && lane_top > -CUDART_INF_F); who; who &= who - 1) {
      for (int c = s.wlo + __ffs(who) - 1 + 32 * lane; c < s.whi; c += 32 * 32) {
        float z[E];
        unpack<T>(s.chunk(c), z);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (z[e] >= floor && z[e] > -CUDART_INF_F) {
            const int at = atomicAdd(count, 1);
            if (at < kListMax) list[at] = order_key(z[e], s.first(c) + e);
          }
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
    each([&](float z, int i) {
      if (in_range(z, i, floor_key)) list[atomicAdd(count, 1)] = order_key(z, i);
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

  // ---- masses

  __device__ __forceinline__ bool in_range(float z, int i, u64 floor_key) const {
    return z > -CUDART_INF_F && order_key(z, i) >= floor_key;
  }

  __device__ __forceinline__ uint32_t kept_mass(float z, int i, const Weigher& weigh, const Kept& kept) const {
    if (!in_range(z, i, kept.floor_key)) return 0;
    const float w = weigh(z);
    return w >= kept.min_p ? grid_mass(w) : 0;
  }

  __device__ __forceinline__ u64 chunk_mass(const uint4& v, int c, const Weigher& weigh, const Kept& kept) const {
    float z[E];
    unpack<T>(v, z);
    const int i0 = s.first(c);
    u64 q = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) q += kept_mass(z[e], i0 + e, weigh, kept);
    return q;
  }

  // A lane's kept mass of a batch.  Where all tokens are kept and all weigh below 2^-8 the conversions are additions
  // (the conversion instruction shares its pipe, a quarter of a warp an SM cycle, with the exponential) and 32 masses
  // fit 32 bits.
  __device__ __forceinline__ u64 batch_mass(const uint4 (&v)[4], int c, const Weigher& weigh, const Kept& kept) const {
    if (kept.all()) {
      ChunkMax<T, true> top;
      top.add(v);
      if (weigh.light(top.value())) {
        uint32_t q = 0u - 4u * E * kMagicBits;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float z[E];
          unpack<T>(v[i], z);
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const float2 y = weigh.exponents(z[e], z[e + 1]);
            const float2 x = fma2(make_float2(exp2_32(y.x), exp2_32(y.y)), make_float2(kGrid, kGrid),
                                  make_float2(kMagic, kMagic));
            q += __float_as_uint(x.x) + __float_as_uint(x.y);
          }
        }
        return q;
      }
    }
    u64 q = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) q += chunk_mass(v[i], c + 32 * i, weigh, kept);
    return q;
  }

  // a part is 2^shift batches
  __device__ __forceinline__ int part_shift() const {
    int shift = 0;
    while ((s.wper + kBatch - 1) / kBatch > kParts << shift) ++shift;
    return shift;
  }

  // warp sums of a batch's masses (below 2^35 a lane) into its part
  __device__ __forceinline__ void add_part(u64 q, int c, int shift, u64& total) {
    const uint32_t low = __reduce_add_sync(~0u, (uint32_t)q & 0xffffffu);
    const uint32_t high = __reduce_add_sync(~0u, (uint32_t)(q >> 24));
    if (threadIdx.x % 32 == 0 && (low | high)) {
      const u64 x = low + ((u64)high << 24);
      sh.parts[threadIdx.x / 32][((c - s.wlo) / kBatch) >> shift] += x;
      total += x;
    }
  }

  __device__ void clear_parts() {
    for (int i = threadIdx.x % 32; i < kParts; i += 32) sh.parts[threadIdx.x / 32][i] = 0;
    __syncwarp();
  }

  // masses of the row's kept tokens, by part and by warp
  __device__ void masses(const Weigher& weigh, const Kept& kept) {
    const int shift = part_shift();
    clear_parts();
    u64 total = 0;
    s.sweep([&](const uint4 (&v)[4], int c) { add_part(batch_mass(v, c, weigh, kept), c, shift, total); });
    if (threadIdx.x % 32 == 0) sh.warp_q[threadIdx.x / 32] = total;
  }

  // After a cluster barrier: the row's kept mass, the CTA's own and that of the CTAs ahead of it.  Every warp for itself.
  __device__ u64 all_mass(u64* mine, u64* ahead) const {
    const int warps = blockDim.x / 32, all = warps * (int)cluster.num_blocks();
    const int rank = (int)cluster.block_rank();
    u64 total = 0, own = 0, before = 0;
    for (int i = threadIdx.x % 32; i < all; i += 32) {
      const int r = i / warps;
      const u64 x = *cluster.map_shared_rank(&sh.warp_q[i - r * warps], r);
      total += x;
      if (r < rank) before += x;
      if (r == rank) own += x;
    }
    *mine = warp_sum(own);
    *ahead = warp_sum(before);
    return warp_sum(total);
  }

  // ---- thresholds

  // The key of the element, among keys >= floor, at which the running total of the order passes the target: with kMass
  // totals are masses and the target floor(arg all / 2^24) - 1, else they are counts and it is arg (or the last).
  // All ones for a row without elements.  A histogram over evenly spaced exponents finds the bin; where it has more
  // elements than a list, a second one cuts it again; the first CTA ranks the bin's elements.  Rows of many equal
  // values go by radix selection.
  // With min_p >= 0 the masses of the kept tokens (from the threshold on, of at least min_p) are left by part and by warp
  // as masses() leaves them, a cluster barrier included.
  template <bool kMass>
  __device__ u64 select(const Weigher& weigh, u64 floor_key, u64 arg, float min_p) {
    const int lane = threadIdx.x % 32, warps = blockDim.x / 32, warp = threadIdx.x / 32;
    int* count = cluster.map_shared_rank(&sh.count, 0);
    u64* list = cluster.map_shared_rank(sh.list, 0);
    const bool keep = min_p >= 0.0f;
    const int shift = part_shift();
    u64 t = 0;
    uint32_t outer = 0;  // the bin of the first level
    int n = kListMax + 1;
    const bool fits = (long long)per_cta * E <= kSliceElems && weigh.m < CUDART_INF_F;
    for (int level = 0; level < 2 && fits; ++level) {
      // the cluster's CTAs have left the memory of the bins and the count behind: a barrier is above
      for (int i = threadIdx.x; i < kBins; i += blockDim.x) sh.bins.low[i] = sh.bins.high[i] = 0;
      if (threadIdx.x == 0) sh.count = 0;
      __syncthreads();
      // Bins go down the order, by exponent; in the second level those outside the first's bin are below 0 or kBins.
      const auto bin_of = [&](float y) -> int {
        const float x = fminf(y * -kBinsPerUnit, (float)(kBins - 1));
        const int b = (int)(__float_as_uint(x + kMagic) - kMagicBits);
        if (level == 0) return b;
        if (b != (int)outer) return b < (int)outer ? -1 : kBins;
        return (int)fminf((x - ((float)outer - 0.5f)) * kBins, (float)(kBins - 1));
      };
      const auto exponent = [&](float z) { return __fmul_rn(__fsub_rn(z, weigh.m), weigh.c); };
      each([&](float z, int i) {
        const float y = exponent(z);
        if (kMass) {
          const uint32_t q = grid_mass(exp2_32(y));
          if (q == 0 || (floor_key && order_key(z, i) < floor_key)) return;
          const int b = bin_of(y);
          if (b < 0 || b >= kBins) return;
          atomicAdd(&sh.bins.low[b], q & 0x7fffu);
          if (q >> 15) atomicAdd(&sh.bins.high[b], q >> 15);
        } else {
          if (!in_range(z, i, floor_key)) return;
          const int b = bin_of(y);
          if (b >= 0 && b < kBins) atomicAdd(&sh.bins.low[b], 1u);
        }
      });
      __syncthreads();
      for (int g = warp; g < kGroups; g += warps) {
        const u64 x = warp_sum(sh.bins.low[32 * g + lane] + ((u64)sh.bins.high[32 * g + lane] << 15));
        if (lane == 0) sh.bins.group[g] = x;
      }
      cluster.sync();
      if (warp == 0) {  // every CTA finds the bin for itself
        static_assert(kGroups == 64, "two groups of bins a lane");
        u64 x0 = 0, x1 = 0;
        for (unsigned r = 0; r < cluster.num_blocks(); ++r) {
          const Histogram* h = cluster.map_shared_rank(&sh.bins, r);
          x0 += h->group[2 * lane];
          x1 += h->group[2 * lane + 1];
        }
        u64 upto = warp_scan(x0 + x1);
        const u64 all = __shfl_sync(~0u, upto, 31);
        if (level == 0) t = kMass ? share24(arg, all) - 1 : min(arg, all - 1);
        int g = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
        u64 ahead = __shfl_sync(~0u, upto - x0 - x1, g);
        const u64 half = __shfl_sync(~0u, x0, g);
        g *= 2;
        if (ahead + half <= t) {
          ahead += half;
          ++g;
        }
        u64 x = 0;
        for (unsigned r = 0; r < cluster.num_blocks(); ++r) {
          const Histogram* h = cluster.map_shared_rank(&sh.bins, r);
          x += h->low[32 * g + lane] + ((u64)h->high[32 * g + lane] << 15);
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
        if (lane == 0) sh.warp_q[warp] = 0;
        cluster.sync();
        return ~0ull;
      }
      const int bin = (int)sh.found;
      t = sh.before;
      // the bin's elements to the list; the mass of what is kept for sure to the parts
      u64 total = 0;
      if (keep) clear_parts();
      s.sweep([&](const uint4 (&v)[4], int c) {
        u64 sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float z[E];
          unpack<T>(v[i], z);
          const int i0 = s.first(c + 32 * i);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float y = exponent(z[e]);
            const int b = bin_of(y);
            if (b > bin || !(z[e] > -CUDART_INF_F)) continue;
            if (floor_key && order_key(z[e], i0 + e) < floor_key) continue;
            if (b == bin) {
              const int at = atomicAdd(count, 1);
              if (at < kListMax) list[at] = order_key(z[e], i0 + e);
            } else if (keep) {
              const float w = exp2_32(y);
              if (w >= min_p) sum += grid_mass(w);
            }
          }
        }
        if (keep) add_part(sum, c, shift, total);
      });
      if (keep && lane == 0) sh.warp_q[warp] = total;
      cluster.sync();
      n = *count;
      if (n <= kListMax) break;
      outer = (uint32_t)bin;
      cluster.sync();  // all have seen the count
    }
    if (n > kListMax) {
      const u64 key = radix_select<kMass>(weigh, floor_key, arg);
      if (keep) {
        masses(weigh, Kept{max(key, 1ull), min_p});
        cluster.sync();
      }
      return key;
    }
    if (cluster.block_rank() == 0) {
      for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const u64 key = sh.list[i];
        u64 ahead = 0;
        for (int j = 0; j < n; ++j)
          if (sh.list[j] > key) ahead += kMass ? grid_mass(weigh(order_value(sh.list[j]))) : 1u;
        const u64 own = kMass ? grid_mass(weigh(order_value(key))) : 1u;
        if (ahead <= t && t < ahead + own) sh.found = key;
      }
      __syncthreads();
      if (keep)
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
          const u64 key = sh.list[i];
          const float w = weigh(order_value(key));
          if (key < sh.found || !(w >= min_p)) continue;
          // the element's CTA, warp and part: head is the same in all CTAs, the warps' shares are not
          const int c = (order_index(key) + s.head) / E, r = c / per_cta, at = c - r * per_cta;
          const int there = (slice_chunks(r) + warps - 1) / warps, w_at = at / there;
          int sh_there = 0;
          while ((there + kBatch - 1) / kBatch > kParts << sh_there) ++sh_there;
          const u64 q = grid_mass(w);
          atomicAdd(cluster.map_shared_rank(&sh.parts[w_at][((at - w_at * there) / kBatch) >> sh_there], r), q);
          atomicAdd(cluster.map_shared_rank(&sh.warp_q[w_at], r), q);
        }
    }
    cluster.sync();
    const u64 key = *cluster.map_shared_rank(&sh.found, 0);
    if (!keep) cluster.sync();  // found and the list may be written again
    return key;
  }

  int per_cta;
  // chunks of CTA r's slice
  __device__ int slice_chunks(int r) const {
    const int total = s.V ? (s.head + s.V - 1) / E + 1 : 0;
    return min(max(total - r * per_cta, 0), per_cta);
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
      each([&](float z, int i) {
        const u64 key = order_key(z, i);
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

  // ---- draws

  // one warp: the token of the slice whose kept mass covers t (counted from the slice's start)
  __device__ void draw(u64 t, const Weigher& weigh, const Kept& kept, u64 all, int32_t* tok, float* prob) const {
    const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
    int w = 0;
    while (w < warps - 1 && t >= sh.warp_q[w]) t -= sh.warp_q[w++];
    const u64 part = sh.parts[w][lane];
    const u64 parts = warp_scan(part);
    const int p = min(__popc(__ballot_sync(~0u, parts <= t)), kParts - 1);
    t -= __shfl_sync(~0u, parts - part, p);
    for (int c0 = w * s.wper + ((p << part_shift()) * kBatch); c0 < s.n; c0 += 32) {
      // lanes past the warp's last chunk look into the next one's: the answer is never there
      const int c = c0 + lane;
      uint4 v = empty_chunk<T>();
      if (c < s.n) v = s.chunk(c);
      const u64 q = chunk_mass(v, c, weigh, kept);
      const u64 upto = warp_scan(q);
      const u64 total = __shfl_sync(~0u, upto, 31);
      if (t >= total) {
        t -= total;
        continue;
      }
      if (t >= upto - q && t < upto) {
        t -= upto - q;
        float z[E];
        unpack<T>(v, z);
        float hit = 0.0f;
        int at = -1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t x = kept_mass(z[e], s.first(c) + e, weigh, kept);
          if (at < 0 && t < x) {
            at = e;
            hit = z[e];
          }
          t -= at < 0 ? x : 0;
        }
        *tok = s.first(c) + at;
        *prob = weigh(hit) * kGrid / (float)all;
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

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 2) k_propose(PickArgs a) {
  __shared__ PickShared sh;
  Row<T> row(sh);
  constexpr int E = ElemOf<T>::E;
  const unsigned ctas = row.cluster.num_blocks(), rank = row.cluster.block_rank();
  const long long r = blockIdx.x / ctas;
  const float T_ = a.temperature ? a.temperature[r / a.rows.k] : 1.0f;
  row.s.open(T_ >= 0.0f ? row_address<T>(a.rows, r) : nullptr, a.rows, rank);
  Weigher weigh;
  weigh.c = fminf(__fdiv_rn(kLog2e, T_), CUDART_MAX_NORMAL_F);
  // one pass: each lane's maximum so far and the sum of its weights relative to it
  float top = -CUDART_INF_F;
  float2 sums = make_float2(0.0f, 0.0f);
  row.s.sweep([&](const uint4 (&v)[4], int) {
    ChunkMax<T, false> batch;
    batch.add(v);
    const float x = batch.value();
    if (x > top) {
      const float by = exp2_32((top - x) * weigh.c);
      sums.x *= by;
      sums.y *= by;
      top = x;
    }
    if (top == -CUDART_INF_F) return;
    const Weigher relative{top, weigh.c};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z[E];
      unpack<T>(v[i], z);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 y = relative.exponents(z[e], z[e + 1]);
        sums = add2(sums, make_float2(exp2_32(y.x), exp2_32(y.y)));
      }
    }
  });
  float floor;
  weigh.m = row.top_of(top, a.K, &floor);
  row.collect(floor, top);
  float sum = sums.x + sums.y;
  if (sum != sum || weigh.m == CUDART_INF_F) {  // NaN or +inf among this lane's elements, or +inf in the row
    sum = 0.0f;
    for (int c = row.s.wlo + (int)(threadIdx.x % 32); c < row.s.whi; c += 32) {
      float z[E];
      unpack<T>(row.s.chunk(c), z);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float w = weigh(z[e]);
        sum += w > 0.0f ? w : 0.0f;
      }
    }
  } else {
    sum = top == -CUDART_INF_F ? 0.0f : sum * exp2_32((top - weigh.m) * weigh.c);
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  if (threadIdx.x % 32 == 0) sh.warp_sum[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)blockDim.x / 32; ++w) sum += sh.warp_sum[w];
    *row.cluster.map_shared_rank(&sh.sums[rank], 0) = sum;
  }
  row.cluster.sync();
  row.settle(a.K);
  if (rank != 0) return;
  sum = 0.0f;
  for (unsigned i = 0; i < ctas; ++i) sum += sh.sums[i];
  int32_t* cand = a.cand + r * a.K;
  float* conf = a.conf + r * a.K;
  for (int i = sh.count + threadIdx.x; i < a.K; i += blockDim.x) {
    cand[i] = -1;
    conf[i] = 0.0f;
  }
  row.ranked([&](int at, u64 key) {
    if (at >= a.K) return;
    cand[at] = order_index(key);
    conf[at] = T_ == 0.0f ? (at == 0 ? 1.0f : 0.0f) : weigh(order_value(key)) / sum;
  });
  row.cluster.sync();  // the others have looked at the count
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 2) k_sample(PickArgs a) {
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
  row.per_cta = a.rows.per;
  row.s.open(good ? row_address<T>(a.rows, r) : nullptr, a.rows, rank);
  const float lane_top = row.lane_maximum();
  Weigher weigh;
  float floor;
  weigh.m = row.top_of(lane_top, by_list ? top_k : 0, &floor);
  weigh.c = fminf(__fdiv_rn(kLog2e, T_), CUDART_MAX_NORMAL_F);
  if (by_list) {
    row.collect(floor, lane_top);
    row.cluster.sync();
    row.settle(top_k);
    if (rank != 0) return;
    row.draw_from_list(weigh, top_k, p24, min_p, a.u + r * a.S, a.S, a.tok + r * a.S, a.prob + r * a.S);
    row.cluster.sync();  // the others have looked at the count
    return;
  }
  const bool by_mass = p24 < (1u << 24);
  Kept kept{0, fmaxf(min_p, 0.0f)};
  if (top_k < a.rows.V) kept.floor_key = row.template select<false>(weigh, 0, top_k - 1, by_mass ? -1.0f : kept.min_p);
  if (by_mass) kept.floor_key = row.template select<true>(weigh, kept.floor_key, p24, kept.min_p);
  if (top_k == a.rows.V && !by_mass) {
    row.masses(weigh, kept);
    row.cluster.sync();
  }
  u64 mine, ahead;
  const u64 all = row.all_mass(&mine, &ahead);
  __syncwarp();
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
    if (t >= ahead && t < ahead + mine) row.draw(t - ahead, weigh, kept, all, &a.tok[o], &a.prob[o]);
  }
  row.cluster.sync();  // no CTA leaves while its masses are read
}

template <typename T>
epic_status launch(PickArgs& a, long long rows, bool sample, cudaStream_t st) {
  const RowShape p = row_shape(rows, a.rows.V, sizeof(T));
  a.rows.per = p.per;
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
  a.rows = {d_logits, stride_b, stride_n, d_pos, n, k, V, 0};
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
  a.rows = {d_logits, stride_b, stride_n, d_pos, n, k, V, 0};
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
