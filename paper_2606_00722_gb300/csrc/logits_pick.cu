// Candidates from logits: the K best tokens of a position with their softmax
// confidences (epic_propose_topk), and draws with temperature, top-k, top-p and
// min-p from given uniform numbers (epic_sample_tokens).
//
// With m the row's maximum and c = log2(e) / T a token's weight is
// w = 2^((z - m) c), every operation rounded to 32 bits (the power to 2 units in the
// last place, and to 0 below 2^-126).  Confidences are w over
// the sum of w in 32 bits.  Sampling adds whole numbers instead,
// q = rint(2^30 w) in 64 bits: such sums are exact, so which token a number
// draws depends on the row and the number alone, not on how the row was split
// (a float CDF over 126,000 tokens has so many boundaries that two orders of
// summation disagree on a draw every few hundred rows).  The grid drops tokens
// less likely than 2^-31 of the likeliest.
//
// The kept tokens of a draw are a prefix of the row's order cut by top-k, then by
// the nucleus, each found as a threshold key on a histogram of counts or of masses;
// the draw is the first kept token in index order whose mass up to and with it
// passes u times the kept mass.
#include <limits.h>

#include "../../include/epic.h"
#include "logit_launch.h"
#include "logit_rows.cuh"
#include "mass_parts.h"

namespace epic {
namespace {

constexpr int kListMax = 2048;  // most keys collected for ranking; a power of two, to which sorting fills up
constexpr int kRankMax = 192;  // longest list whose ranks are counted, n^2 / threads steps; longer ones are sorted
constexpr int kMaxK = 256;      // most candidates of a position, and the longest top-k list
constexpr int kMaxV = kRowCtasMax * (kSliceElems - 16);  // 1,047,872: histograms and parts of a row's slices
constexpr int kBins = 2048;     // of a threshold's histogram
constexpr int kGroups = kBins / 32;
constexpr int kLevels = 4;      // of histograms by exponent for one threshold
constexpr int kParts = (kSliceElems + 127) / 128;  // runs of 32 chunks of a slice, whose kept masses are noted
constexpr int kTops = 2 * kMaxK + kRowWarps * kRowCluster;
constexpr float kBinsPerUnit = kBins / 32;  // bins to a power of two; past 2^-32 of the maximum weights are 0
constexpr float kGrid = 1073741824.0f;      // 2^30: the weights' grid
// Rounding to whole numbers by addition: x + kOnes holds rint(x) in its low bits (|x| < 2^22), x + kHigh rint(x / 2^15)
// (|x| < 2^37).
constexpr float kOnes = 12582912.0f;       // 1.5 * 2^23
constexpr float kHigh = 412316860416.0f;   // 1.5 * 2^38
constexpr uint32_t kOnesBits = 0x4b400000u, kHighBits = 0x52c00000u;

// Fewest threads of a CTA: short rows have less to read than to rank, clear and draw.  On the GPU with 64, 128, 256 and 512:
// the 64 best of 80 rows of 1,280 33, 22, 18 and 17 us, draws from them 35, 25, 21 and 20; the nucleus of 2,688 rows of 300
// 86, 72, 78 and 131 (512 leave an SM two rows for four).
constexpr int kPickThreadsMin = 256;

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

// The bins hold the sums of their elements' parts (MassParts, whatever adds to them); counts are sums of low parts of 1.
struct Histogram {
  uint32_t low[kBins], high[kBins];
  u64 group[kGroups];
  __device__ __forceinline__ u64 mass(int i) const { return MassParts{high[i], low[i]}.value(); }
};

struct TopList {  // a sampler's top-k list, in order
  u64 key[kMaxK];
  u64 first[kMaxK];  // kept mass ahead of the entry in index order
  uint32_t q[kMaxK];
  uint32_t kept[kMaxK];
};

struct Tops {  // value keys: largest lane maxima of this CTA's warps, and past kTops of all of the row's; ends of a range
  uint32_t value[2 * kTops];
};

struct PickShared {
  union {
    Histogram bins;
    TopList top;
  };
  Tops tops;
  u64 list[kListMax];
  u64 parts[kParts + kParts / 16];  // kept masses by runs of 32 chunks, at part_at()
  u64 cta_q;  // the CTA's kept mass
  u64 warp_q[kRowWarps];
  uint4 ends[2];
  u64 found, before;
  float bin_low, bin_high;
  int last;
  uint32_t row_top, row_floor;             // value keys
  float sums[kRowWarps * kRowCluster];     // of warps, in the first CTA
  int count;
};

// The temperature of a row; -0 becomes 0.
__device__ __forceinline__ float row_temperature(const PickArgs& a, int r) {
  return a.temperature ? a.temperature[r / a.rows.k] + 0.0f : 1.0f;
}

// log2(e) / T.  A row of a temperature that is none is read like others, and answered with nothing.
__device__ __forceinline__ float exponent_scale(float t) {
  return t >= 0.0f ? fminf(__fdiv_rn(kLog2e, t), CUDART_MAX_NORMAL_F) : 1.0f;
}

// The kernels' shared memory, by name: through a reference kept in an object its loads would be generic ones.
__device__ __forceinline__ PickShared& shared() {
  __shared__ PickShared sh;
  return sh;
}

// 2^((z - m) c); a row whose maximum is +inf has weight 1 on its +inf elements and 0 elsewhere
struct Weigher {
  float m, c;
  __device__ __forceinline__ float operator()(float z) const {
    if (m == CUDART_INF_F) return z == m ? 1.0f : 0.0f;
    return exp2_32(__fmul_rn(__fsub_rn(z, m), c));
  }
  __device__ __forceinline__ float exponent(float z) const { return __fmul_rn(__fsub_rn(z, m), c); }
  __device__ __forceinline__ float2 exponents(float a, float b) const {
    return mul2(add2(make_float2(a, b), make_float2(-m, -m)), make_float2(c, c));
  }
};

// For a row whose largest logit is `most`.  At T = inf every exponent is 0, whatever is taken off: not the largest, from
// which a difference may pass 32 bits.
__device__ __forceinline__ Weigher weigher(float most, float c) {
  return Weigher{c == 0.0f && fabsf(most) < CUDART_INF_F ? 0.0f : most, c};
}

__device__ __forceinline__ uint32_t grid_mass(float w) { return __float2uint_rn(w * kGrid); }

// The masses of two weights in parts, low ones within 2^14 of 0, high and low as bits over kHighBits and kOnesBits.
// Three additions for two elements: the conversion instruction does a quarter of a warp a cycle on the pipe that the
// exponentials need.  Not for NaN.
struct Parts2 {
  uint32_t high[2], low[2];
  __device__ __forceinline__ explicit Parts2(float2 w) {
    const float2 grid = make_float2(kGrid, kGrid);
    const float2 h = fma2(w, grid, make_float2(kHigh, kHigh));
    const float2 rest = add2(make_float2(kHigh + kOnes, kHigh + kOnes), make_float2(-h.x, -h.y));
    const float2 l = fma2(w, grid, rest);
    high[0] = __float_as_uint(h.x);
    high[1] = __float_as_uint(h.y);
    low[0] = __float_as_uint(l.x);
    low[1] = __float_as_uint(l.y);
  }
};

// floor(a q / 2^24) for a <= 2^24, without passing 64 bits
__device__ __forceinline__ u64 share24(u64 a, u64 q) { return a * (q >> 24) + ((a * (q & 0xffffffu)) >> 24); }

// *at += x where x is not 0, without a branch
__device__ __forceinline__ void add_shared(uint32_t* at, uint32_t x) {
  asm volatile("{.reg .pred p; setp.ne.u32 p, %1, 0; @p red.shared.add.u32 [%0], %1;}" ::"r"(
                   (uint32_t)__cvta_generic_to_shared(at)),
               "r"(x)
               : "memory");
}

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

// A place in a row's order; elements at it or ahead of it are `in`.
struct Floor {
  float z;
  int i;
  __device__ __forceinline__ bool in(float value, int index) const { return value > z || (value == z && index <= i); }
};
__device__ __forceinline__ Floor no_floor() { return Floor{-CUDART_INF_F, INT_MIN}; }  // -inf and NaN are not in
__device__ __forceinline__ Floor floor_of(u64 key) {
  if (key == ~0ull) return Floor{CUDART_INF_F, INT_MIN};  // of an empty row: nothing is in
  return Floor{order_value(key), order_index(key)};
}

// Which tokens are kept: from the floor on, with a weight of at least min_p.
struct Kept {
  Floor floor;
  float min_p;
  __device__ __forceinline__ bool all() const { return floor.z == -CUDART_INF_F && !(min_p > 0.0f); }
};

// Of a lane's batches, the largest maximum and that batch's first chunk, and the second largest maximum.
struct LaneTop {
  float first, second;
  int at;
  __device__ LaneTop() {
    first = second = -CUDART_INF_F;
    at = 0;
  }
  __device__ __forceinline__ void add(float x, int c) {
    if (x > first) {
      second = first;
      first = x;
      at = c;
    } else {
      second = fmaxf(second, x);
    }
  }
};

// A gap after every 16 parts: lanes that read runs of them are in different banks.
__device__ __forceinline__ int part_at(int p) { return p + p / 16; }

template <typename T>
struct Row {
  Slice<T> s;
  RowGroup group;
  int per_cta;   // chunks
  bool special;  // this warp's elements have NaN, or the row +inf, or nothing, or T = inf
  static constexpr int E = ElemOf<T>::E;

  // f(value, index) for the elements of this lane's chunks, one at a time: small code for rare ways.  (The whole kernel
  // unrolled was 460 KB, and each phase of a row waited for its instructions.)
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
    for (int base = warp_index() * kBatch; base < s.n; base += (int)blockDim.x * 4)
#pragma unroll 1
      for (int k = 0; k < 4 * E; ++k) {
        const int i = s.first(base + (int)threadIdx.x % 32 + 32 * (k / E)) + k % E;
        if (i >= s.lo() && i < s.hi()) f(s.at(i), i);
      }
  }

  // f(i, how many o < n are ahead(i, o)) for i < n, by one thread each; eight lanes count for one i.  (A vote for every
  // 32 of them took 250 cycles.)
  template <typename A, typename F>
  __device__ __forceinline__ static void each_rank(int n, A ahead, F f) {
    const int part = (int)threadIdx.x % 8;
    for (int i0 = 0; i0 < n; i0 += (int)blockDim.x / 8) {
      const int i = min(i0 + (int)threadIdx.x / 8, n - 1);
      int count = 0;
#pragma unroll 4
      for (int o = part; o < n; o += 8) count += ahead(i, o);
      for (int m = 1; m < 8; m *= 2) count += __shfl_xor_sync(~0u, count, m);
      if (part == 0 && i0 + (int)threadIdx.x / 8 < n) f(i, count);
    }
  }

  // The row's maximum from the lanes' (NaN left out, -inf for a row without elements).  For K > 0 *floor is a value
  // that at least K elements reach (or -inf): the K-th largest of the largest j lane maxima of every warp, where j gives
  // twice K of them.  About 1.4 K elements of a row in random order reach it; the lowest of the warps' j-th, which needs
  // no ranking, lets ten times K through at one lane maximum a warp.
  __device__ float top_of(float lane_top, int K, float* floor) {
    const int w = warp_index(), lane = (int)threadIdx.x % 32;
    // a short row's warps without elements have no say
    const int warps = group.n == 1 ? min((int)blockDim.x / 32, max((s.n + kBatch - 1) / kBatch, 1)) : (int)blockDim.x / 32;
    const int all = warps * (int)group.n;
    const int j = K > 0 ? min((2 * K + all - 1) / all, 32) : 1;
    uint32_t key = value_key(lane_top);
    for (int i = 0; i < j && w < warps; ++i) {
      const uint32_t x = __reduce_max_sync(~0u, key);
      if (lane == 0) shared().tops.value[w * j + i] = x;
      if (__ffs(__ballot_sync(~0u, key == x)) - 1 == lane) key = 0;
    }
    if (threadIdx.x == 0) {
      shared().count = 0;
      shared().row_floor = 0;
    }
    group.sync();
    const int n = all * j, per = warps * j;
    if (K == 0) {  // every warp looks at all warps of the row
      uint32_t m = 0;
      for (int i = lane; i < n; i += 32) m = max(m, *group.at(&shared().tops.value[i % per], i / per));
      return key_value(__reduce_max_sync(~0u, m));
    }
    int from = 0;
    if (group.n > 1) {
      from = kTops;
      for (int i = threadIdx.x; i < n; i += (int)blockDim.x)
        shared().tops.value[from + i] = *group.at(&shared().tops.value[i % per], i / per);
      __syncthreads();
    }
    const uint32_t* tops = &shared().tops.value[from];
    each_rank(n, [&](int i, int o) { return tops[o] > tops[i] || (tops[o] == tops[i] && o < i); },
              [&](int i, int above) {
                if (above == 0) shared().row_top = tops[i];
                if (above == K - 1) shared().row_floor = tops[i];
              });
    __syncthreads();
    *floor = shared().row_floor ? key_value(shared().row_floor) : -CUDART_INF_F;
    return key_value(shared().row_top);
  }

  // the maxima of this lane's batches, NaN left out; `special` tells of NaN
  __device__ __forceinline__ LaneTop lane_top() {
    LaneTop top;
    bool nan = false;
    s.sweep([&](const uint4 (&v)[4], int c) {
      ChunkMax<T, true> batch;
      batch.add(v);
      float x = batch.value();
      if (x != x) {
        nan = true;
        ChunkMax<T, false> numbers;
        numbers.add(v);
        x = numbers.value();
      }
      top.add(x, c);
    });
    special = __any_sync(~0u, nan);
    return top;
  }

  // Keys of elements >= floor to the first CTA's list (past its end they are only counted).  A lane whose maximum
  // reaches the floor has such elements in the batch of its maximum, whose four chunks are looked at by four lanes; where
  // the second of its batches reaches it too (few lanes), the warp looks at all of them.
  __device__ __forceinline__ void collect(float floor, const LaneTop& top) const {
    const int lane = (int)threadIdx.x % 32, w = warp_index();
    int* count = group.at(&shared().count, 0);
    u64* list = group.at(shared().list, 0);
    const auto look = [&](int c) {
      float z[E];
      unpack<T>(s.chunk(c), z);
      uint32_t hits = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) hits |= z[e] >= floor && z[e] > -CUDART_INF_F ? 1u << e : 0u;
      if (!hits) return;
      for (int at = atomicAdd(count, __popc(hits)); hits && at < kListMax; hits &= hits - 1, ++at) {
        const int index = s.first(c) + __ffs(hits) - 1;
        list[at] = order_key(s.at(index), index);
      }
    };
    uint32_t who = __ballot_sync(~0u, top.first >= floor && top.first > -CUDART_INF_F);
    while (who) {
      int of = -1;  // this lane looks at one of the chunks of the lane / 4-th of the next eight
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (lane / 4 == i && who) of = __ffs(who) - 1;
        who &= who - 1;
      }
      const int c = __shfl_sync(~0u, top.at, max(of, 0)) + 32 * (lane % 4);
      if (of >= 0 && c < s.n) look(c);
      __syncwarp();
    }
    for (who = __ballot_sync(~0u, top.second >= floor && top.second > -CUDART_INF_F); who; who &= who - 1) {
      const int of = __ffs(who) - 1, best = __shfl_sync(~0u, top.at, of);
      for (int k = lane;; k += 32) {
        const int base = w * kBatch + of + k / 4 * ((int)blockDim.x * 4);
        if (base >= s.n) break;
        if (base != best && base + 32 * (k % 4) < s.n) look(base + 32 * (k % 4));
      }
      __syncwarp();
    }
  }

  // After a barrier: the K first keys of the row are in the first CTA's list, with others or (where more than a list
  // was collected) alone.
  __device__ void settle(int K, float m) {
    if (*group.at(&shared().count, 0) <= kListMax) return;  // the same in all CTAs
    const Floor floor = floor_of(threshold(*this, Weigher{m, 1.0f}, no_floor(), K - 1, false, -1.0f));
    if (group.rank == 0 && threadIdx.x == 0) shared().count = 0;
    group.sync();
    int* count = group.at(&shared().count, 0);
    u64* list = group.at(shared().list, 0);
    s.sweep([&](const uint4 (&v)[4], int c) {
      ChunkMax<T, false> top;
      top.add(v);
      if (!__any_sync(~0u, top.value() >= floor.z)) return;
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(s.chunk(c + 32 * i), z);
        const int i0 = s.first(c + 32 * i);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (floor.in(z[e], i0 + e)) {
            const int at = atomicAdd(count, 1);
            if (at < kListMax) list[at] = order_key(z[e], i0 + e);
          }
      }
      __syncwarp();
    });
    group.sync();
  }

  // f(rank, key) for the list's keys, by one thread each
  template <typename F>
  __device__ __forceinline__ void ranked(F f) {
    const int n = shared().count;
    if (n > kRankMax) {
      sort_list(n);
      for (int i = (int)threadIdx.x; i < n; i += (int)blockDim.x) f(i, shared().list[i]);
      return;
    }
    each_rank(n, [&](int i, int o) { return shared().list[o] > shared().list[i]; },
              [&](int i, int at) { f(at, shared().list[i]); });
  }

  // ---- masses

  __device__ __forceinline__ uint32_t kept_mass(float z, int i, const Weigher& weigh, const Kept& kept) const {
    if (!kept.floor.in(z, i)) return 0;
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

  // A lane's kept mass of a chunk in parts, whose sums over a warp are below 32 bits.
  template <bool kAll>
  __device__ __forceinline__ MassParts lane_mass(const uint4& v, int c, const Weigher& weigh, const Kept& kept) const {
    MassParts sum = {0, 0};
    if (kAll) sum = {0u - (uint32_t)E * kHighBits, 0u - (uint32_t)E * kOnesBits};
    float z[E];
    unpack<T>(v, z);
    const int i0 = s.first(c);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 y = weigh.exponents(z[e], z[e + 1]);
      const float2 w = make_float2(exp2_32(y.x), exp2_32(y.y));
      const Parts2 q(w);
      if (kAll) {
        sum.high += q.high[0] + q.high[1];
        sum.low += q.low[0] + q.low[1];
      } else {
#pragma unroll
        for (int o = 0; o < 2; ++o)
          if ((o ? w.y : w.x) >= kept.min_p && kept.floor.in(z[e + o], i0 + e + o)) {
            sum.high += q.high[o] - kHighBits;
            sum.low += q.low[o] - kOnesBits;
          }
      }
    }
    return sum;
  }

  // the warp's sum of its lanes' masses of 32 chunks to their part
  __device__ __forceinline__ void add_part(MassParts q, int c) const {
    const MassParts sum = {__reduce_add_sync(~0u, q.high), __reduce_add_sync(~0u, q.low)};
    if (threadIdx.x % 32 == 0 && c < s.n) shared().parts[part_at(c / 32)] = sum.value();
  }
  // before a barrier
  __device__ __forceinline__ void clear_parts() {
    for (int i = (int)threadIdx.x; i < kParts + kParts / 16; i += (int)blockDim.x) shared().parts[i] = 0;
  }

  // masses of the row's kept tokens, by part
  __device__ __noinline__ static void masses(Row row, Weigher weigh, Kept kept) {
    row.clear_parts();
    __syncthreads();
    if (row.special) {
      row.s.sweep([&](const uint4 (&)[4], int c) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          const u64 q = row.chunk_mass(row.s.chunk(c + 32 * i), c + 32 * i, weigh, kept);
          row.add_part(MassParts{(uint32_t)(q >> 15), (uint32_t)q & 0x7fffu}, c + 32 * i);
        }
      });
    } else if (kept.all()) {
      row.s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) row.add_part(row.template lane_mass<true>(v[i], c + 32 * i, weigh, kept), c + 32 * i);
      });
    } else {
      row.s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) row.add_part(row.template lane_mass<false>(v[i], c + 32 * i, weigh, kept), c + 32 * i);
      });
    }
  }

  // After a barrier of the group: the row's kept mass, the CTA's own and that of the CTAs ahead of it, from the parts; every
  // warp for itself.
  __device__ __forceinline__ u64 all_mass(u64* mine, u64* ahead) const {
    const int lane = (int)threadIdx.x % 32, parts = (s.n + 31) / 32;
    u64 own = 0;
#pragma unroll 4
    for (int p = lane; p < parts; p += 32) own += shared().parts[part_at(p)];
    own = warp_sum(own);
    *mine = own;
    *ahead = 0;
    if (group.n == 1) return own;
    if (threadIdx.x == 0) shared().cta_q = own;
    group.sync();
    u64 total = 0;
#pragma unroll 1
    for (unsigned r = 0; r < group.n; ++r) {
      const u64 x = *group.at(&shared().cta_q, r);
      if (r < group.rank) *ahead += x;
      total += x;
    }
    return total;
  }

  // ---- thresholds

  // One level of a threshold's search: kBins bins, evenly spaced in the exponent, that go down the order.  Bin 0 has what
  // is above, the last bin what is below; of the row's values only those from low to below high (NaN: all) count.
  struct Level {
    float from, scale;
    float low, high;
    // kOnes and the bin of an exponent
    __device__ __forceinline__ float place(float y) const {
      return fminf(fmaxf((-y - from) * scale, 0.0f), (float)(kBins - 1)) + kOnes;
    }
    __device__ __forceinline__ int bin(float y) const { return (int)(__float_as_uint(place(y)) - kOnesBits); }
    __device__ __forceinline__ bool has(float z) const { return z >= low && !(z >= high); }
    // the level that resolves bin b, whose values are from `l` to below `h`
    __device__ __forceinline__ void enter(int b, float l, float h) {
      low = l;
      high = h;
      if (b == kBins - 1) {  // what is below, on a coarser scale
        from += (b - 0.5f) / scale;
        scale *= 1.0f / 64;
      } else {
        from += fmaxf(b - 0.5f, 0.0f) / scale;
        scale *= kBins / 2;
      }
    }
  };

  // The elements of a bin of the level, from the floor on, to the first CTA's list; with min_p >= 0 the masses of those of
  // the level's bins ahead and above the level, from the floor on and of at least min_p, to the parts.  kFree: min_p >= 0,
  // there is no floor, and the level is the first.
  template <bool kFree>
  __device__ __forceinline__ void collect_bin(const Weigher& weigh, Floor floor, const Level& level, int bin, float min_p) {
    int* count = group.at(&shared().count, 0);
    u64* list = group.at(shared().list, 0);
    const bool keep = kFree || min_p >= 0.0f;
    bool full = false;  // this lane has seen the list full: how many more there are does not matter
    s.sweep([&](const uint4 (&v)[4], int c) {
      ChunkMax<T, false> top;
      top.add(v);
      const float most = top.value();
      if (!__any_sync(~0u, most > -CUDART_INF_F && level.place(weigh.exponent(most)) <= kOnes + bin)) return;
      uint32_t in_bin = 0;  // a bit for each element
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(v[i], z);
        MassParts sum = {0u - (uint32_t)E * kHighBits, 0u - (uint32_t)E * kOnesBits};
        const int i0 = s.first(c + 32 * i);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 y = weigh.exponents(z[e], z[e + 1]);
          float2 at = fma2(y, make_float2(-kBinsPerUnit, -kBinsPerUnit), make_float2(kOnes, kOnes));
          bool ahead0 = at.x < kOnes + bin, ahead1 = at.y < kOnes + bin;
          bool here0 = at.x == kOnes + bin, here1 = at.y == kOnes + bin;
          if (!kFree) {
            at = make_float2(level.place(y.x), level.place(y.y));
            ahead0 = z[e] >= level.high || (level.has(z[e]) && at.x < kOnes + bin);
            ahead1 = z[e + 1] >= level.high || (level.has(z[e + 1]) && at.y < kOnes + bin);
            here0 = level.has(z[e]) && at.x == kOnes + bin;
            here1 = level.has(z[e + 1]) && at.y == kOnes + bin;
          }
          if (here0) in_bin |= 1u << (E * i + e);
          if (here1) in_bin |= 1u << (E * i + e + 1);
          if (!keep) continue;
          const float2 w = make_float2(exp2_32(y.x), exp2_32(y.y));
          const Parts2 q(w);
          // what is not kept adds a mass of 0
          const bool in0 = ahead0 && w.x >= min_p && (kFree || floor.in(z[e], i0 + e));
          const bool in1 = ahead1 && w.y >= min_p && (kFree || floor.in(z[e + 1], i0 + e + 1));
          sum.high += (in0 ? q.high[0] : kHighBits) + (in1 ? q.high[1] : kHighBits);
          sum.low += (in0 ? q.low[0] : kOnesBits) + (in1 ? q.low[1] : kOnesBits);
        }
        if (keep) add_part(sum, c + 32 * i);
      }
      for (; in_bin; in_bin &= in_bin - 1) {
        const int bit = __ffs(in_bin) - 1, index = s.first(c + 32 * (bit / E)) + bit % E;
        const float z = s.at(index);
        if (full || (!kFree && !floor.in(z, index))) continue;
        const int at = atomicAdd(count, 1);
        full = at >= kListMax;
        if (!full) list[at] = order_key(z, index);
      }
      __syncwarp();
    });
  }

  // After a barrier, before another: the largest and smallest of the level's values from the floor on, by each warp, as
  // value keys to tops[warp] and tops[kRowWarps + warp].
  __device__ __noinline__ static void range_of(Row row, Level level, Floor floor) {
    const int warp = warp_index();
    float most = -CUDART_INF_F, least = CUDART_INF_F;
    row.s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(v[i], z);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (level.has(z[e]) && floor.in(z[e], row.s.first(c + 32 * i) + e)) {
            most = fmaxf(most, z[e]);
            least = fminf(least, z[e]);
          }
      }
    });
    const uint32_t hi = __reduce_max_sync(~0u, value_key(most)), lo = __reduce_min_sync(~0u, value_key(least));
    if (threadIdx.x % 32 == 0) {
      shared().tops.value[warp] = hi;
      shared().tops.value[kRowWarps + warp] = lo;
    }
  }

  // After a barrier of the group: whether the values that range_of() saw are all the same, and that value.
  __device__ __noinline__ static bool one_value(Row row, float* value) {
    const int lane = (int)threadIdx.x % 32, warps = (int)blockDim.x / 32;
    uint32_t most = 0, least = ~0u;
#pragma unroll 1
    for (unsigned r = 0; r < row.group.n; ++r)
      if (lane < warps) {
        most = max(most, *row.group.at(&shared().tops.value[lane], r));
        least = min(least, *row.group.at(&shared().tops.value[kRowWarps + lane], r));
      }
    most = __reduce_max_sync(~0u, most);
    *value = key_value(most);
    return most == __reduce_min_sync(~0u, least);
  }

  // The rest of a threshold's search among elements of one value, which follow each other by index: the key of the one with
  // `ahead` others from the floor on before it.
  __device__ __noinline__ static u64 by_index(Row row, float value, Floor floor, u64 ahead) {
    row.s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(v[i], z);
        uint32_t n = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) n += z[e] == value && floor.in(z[e], row.s.first(c + 32 * i) + e);
        row.add_part(MassParts{0, n}, c + 32 * i);
      }
    });
    row.group.sync();
    u64 mine, before;
    ahead = min(ahead, row.all_mass(&mine, &before) - 1);  // the last one takes what lies past the end
    if (warp_index() == 0 && ahead >= before && ahead < before + mine)
      row.locate(ahead - before, [&](float z, int i) { return z == value && floor.in(z, i) ? 1u : 0u; },
                 [&](float z, int i) { *row.group.at(&shared().found, 0) = order_key(z, i); });
    row.group.sync();
    const u64 key = *row.group.at(&shared().found, 0);
    row.group.sync();
    return key;
  }

  // One warp: the lowest of the level's values whose bin is at most b, to the lower half of the lanes, and the lowest whose
  // bin is less, to the upper half (the level's end where there is none).  The bins do not increase with the value; each
  // half tries sixteen values at a time.
  __device__ __noinline__ static float ends_of_bin(Weigher weigh, Level level, int b) {
    const uint32_t lane = threadIdx.x % 32, part = lane % 16;
    const int shift = lane < 16 ? 0 : 16;
    if (shift) --b;
    const auto in = [&](uint32_t key) { return level.bin(weigh.exponent(key_value(key))) <= b; };
    uint32_t lo = value_key(level.low), hi = level.high <= weigh.m ? value_key(level.high) - 1 : value_key(weigh.m);
    const bool none = !in(hi);
    if (none) lo = hi;
    while (__any_sync(~0u, lo < hi)) {  // the answer is in [lo, hi]
      const uint32_t step = (hi - lo) / 16 + 1;
      const uint32_t hit = __ballot_sync(~0u, in(min(lo + part * step, hi))) >> shift & 0xffffu;
      if (lo < hi) {
        if (!hit) {
          lo = min(lo + 15 * step, hi - 1) + 1;
        } else {
          const int first = __ffs(hit) - 1;
          hi = min(lo + first * step, hi);
          lo = first ? lo + (first - 1) * step + 1 : hi;
        }
      }
    }
    return none ? level.high : key_value(lo);
  }

  // The histogram's sums by groups of 32 bins, four groups of a warp at a time.
  __device__ __forceinline__ static void sum_groups() {
    const int lane = (int)threadIdx.x % 32;
#pragma unroll 1
    for (int g = 4 * warp_index(); g < kGroups; g += (int)blockDim.x / 8) {
      u64 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = shared().bins.mass(32 * (g + i) + lane);
#pragma unroll
      for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += __shfl_xor_sync(~0u, x[i], o);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane == i) shared().bins.group[g + i] = x[i];
    }
  }

  // After a barrier, in one warp: the bin of the cluster's histograms at which the running total passes t, and the rest
  // of t within it, to shared().found and shared().before; all ones for histograms of nothing.  t may be given as a share of
  // all.
  __device__ __forceinline__ void find_bin(u64 t, bool share, bool mass) const {
    static_assert(kGroups == 64, "two groups of bins a lane");
    const int lane = (int)threadIdx.x % 32;
    const unsigned ctas = group.n;
    u64 x0 = 0, x1 = 0;
#pragma unroll
    for (unsigned r = 0; r < kRowCluster; ++r) {  // the loads from all CTAs at once
      if (r >= ctas) break;
      const Histogram* h = group.at(&shared().bins, r);
      x0 += h->group[2 * lane];
      x1 += h->group[2 * lane + 1];
    }
    u64 upto = warp_scan(x0 + x1);
    const u64 all = __shfl_sync(~0u, upto, 31);
    if (share) t = mass ? share24(t, all) - 1 : min(t, all - 1);
    int g = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
    u64 ahead = __shfl_sync(~0u, upto - x0 - x1, g);
    const u64 half = __shfl_sync(~0u, x0, g);
    g *= 2;
    if (ahead + half <= t) {
      ahead += half;
      ++g;
    }
    u64 x = 0;
#pragma unroll 1
    for (unsigned r = 0; r < ctas; ++r) x += group.at(&shared().bins, r)->mass(32 * g + lane);
    upto = ahead + warp_scan(x);
    const int l = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
    const u64 before = __shfl_sync(~0u, upto - x, l);
    if (lane == 0) {
      shared().found = all ? (u64)(32 * g + l) : ~0ull;
      shared().before = t - before;
    }
  }

  // The list's first n keys into descending order.
  __device__ __noinline__ static void sort_list(int n) {
    u64* list = shared().list;
    int size = 32;
    while (size < n) size *= 2;
    if (size <= (int)blockDim.x) {  // a key a thread; exchanges within a warp by shuffles
      const int i = threadIdx.x;
      u64 key = i < n ? list[i] : 0;
      for (int k = 2; k <= size; k *= 2)
        for (int d = k / 2; d; d /= 2) {
          u64 other;
          if (d < 32) {
            other = __shfl_xor_sync(~0u, key, d);
          } else {
            __syncthreads();
            if (i < size) list[i] = key;
            __syncthreads();
            other = list[(i ^ d) % size];
          }
          // the lower place of a descending run takes the larger key
          if (((i & k) == 0) == ((i & d) == 0) ? other > key : other < key) key = other;
        }
      __syncthreads();
      if (i < size) list[i] = key;
      __syncthreads();
      return;
    }
    for (int i = n + threadIdx.x; i < size; i += (int)blockDim.x) list[i] = 0;
    for (int k = 2; k <= size; k *= 2)
      for (int d = k / 2; d; d /= 2) {
        __syncthreads();
        for (int t = threadIdx.x; t < size / 2; t += (int)blockDim.x) {
          const int i = 2 * t - (t & (d - 1));
          const u64 a = list[i], b = list[i + d];
          if ((a < b) == ((i & k) == 0)) {
            list[i] = b;
            list[i + d] = a;
          }
        }
      }
    __syncthreads();
  }

  // The key of the element, among those from the floor on, at which the running total of the order passes the target:
  // with `mass` totals are masses and the target floor(arg all / 2^24) - 1, else they are counts and it is arg (or the
  // last).  All ones for a row without elements.  A histogram over evenly spaced exponents finds the bin; where it has
  // more elements than a list, the next one cuts it again, or where they are equal they are counted off; the first CTA
  // sorts the bin's elements.  What does not fit after kLevels (values whose exponents a high temperature leaves too close),
  // and rows of +inf, is told apart by eight bits of the keys at a time.
  // With min_p >= 0 the masses of the kept tokens (from the threshold on, of at least min_p) are left by part
  // as masses() leaves them, a barrier of the group included.
  __device__ __noinline__ static u64 threshold(Row row, Weigher weigh, Floor floor, u64 arg, bool mass, float min_p) {
    return row.find_threshold(weigh, floor, arg, mass, min_p);
  }
  __device__ __forceinline__ u64 find_threshold(const Weigher& weigh, Floor floor, u64 arg, bool mass, float min_p) {
    const int lane = (int)threadIdx.x % 32, warp = warp_index();
    const bool keep = min_p >= 0.0f, free = floor.z == -CUDART_INF_F;
    Level level{0.0f, kBinsPerUnit, -CUDART_MAX_NORMAL_F, CUDART_NAN_F};
    if (weigh.m == CUDART_INF_F) level.low = -CUDART_INF_F;
    u64 t = arg, prefix = 0;
    int shift = 64;  // digits of the keys from here on are found
    int depth = weigh.m == CUDART_INF_F ? kLevels : 0;
    bool first = true;
    group.sync();
#pragma unroll 1
    for (;; ++depth) {
      // the group's CTAs have left the memory of the bins and the count behind: a barrier is above
      const bool digits = depth >= kLevels;
      if (digits) {
        shift -= 8;
        if (shift < 32 && shift > 0 && s.V > 0 && (uint32_t)(s.V - 1) >> shift == 0) {
          prefix |= 0xffull << shift;  // every index has these bits clear
          continue;
        }
      }
      for (int i = (int)threadIdx.x; i < kBins; i += (int)blockDim.x) shared().bins.low[i] = shared().bins.high[i] = 0;
      if (threadIdx.x == 0) shared().count = 0;
      __syncthreads();
      if (digits) {
        each([&](float z, int i) {
          if (!level.has(z) || !floor.in(z, i)) return;
          const u64 key = order_key(z, i);
          if (shift < 56 && (key ^ prefix) >> (shift + 8)) return;
          const int b = 255 - (int)(key >> shift & 255);
          const MassParts q = mass_parts(mass ? grid_mass(weigh(z)) : 1u);
          add_shared(&shared().bins.low[b], q.low);
          add_shared(&shared().bins.high[b], q.high);
        });
      } else if (mass && first && !special) {
        count_masses(weigh, floor, free);
      } else {
        if (mass)
          count_elements<true>(weigh, floor, level);
        else
          count_elements<false>(weigh, floor, level);
      }
      __syncthreads();
      sum_groups();
      group.sync();
      if (warp == 0) {  // every CTA for itself
        find_bin(t, first, mass);
        __syncwarp();
      }
      first = false;
      __syncthreads();
      if (shared().found == ~0ull) {
        clear_parts();
        group.sync();
        return ~0ull;
      }
      const int bin = (int)shared().found;
      t = shared().before;
      if (digits) {
        prefix |= (u64)(255 - bin) << shift;
        if (shift == 0) break;
        group.sync();  // all have read the bins
        continue;
      }
      if (keep) clear_parts();
      __syncthreads();
      if (free && keep && depth == 0 && bin < kBins - 1)
        collect_bin<true>(weigh, floor, level, bin, min_p);
      else
        collect_bin<false>(weigh, floor, level, bin, min_p);
      group.sync();
      const int n = *group.at(&shared().count, 0);
      if (n <= kListMax) return by_list(n, weigh, t, mass, min_p);
      if (warp == 0) {
        const float end = ends_of_bin(weigh, level, bin);
        if (lane == 0) shared().bin_low = end;
        if (lane == 16) shared().bin_high = end;
      }
      __syncthreads();
      level.enter(bin, shared().bin_low, shared().bin_high);
      range_of(*this, level, floor);
      group.sync();  // all have seen the count
      float value;
      if (one_value(*this, &value)) {
        prefix = by_index(*this, value, floor, mass ? t / max(grid_mass(weigh(value)), 1u) : t);
        break;
      }
    }
    if (keep) masses(*this, weigh, Kept{floor_of(prefix), min_p});
    group.sync();
    return prefix;
  }

  // the first histogram, of masses
  __device__ __forceinline__ void count_masses(const Weigher& weigh, Floor floor, bool free) const {
    s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(v[i], z);
        const int i0 = s.first(c + 32 * i);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 y = weigh.exponents(z[e], z[e + 1]);
          const Parts2 q(make_float2(exp2_32(y.x), exp2_32(y.y)));
          const float2 b = fma2(y, make_float2(-kBinsPerUnit, -kBinsPerUnit), make_float2(kOnes, kOnes));
          // a mass above 0 has an exponent above -32: its bin needs no bound
#pragma unroll
          for (int o = 0; o < 2; ++o) {
            const uint32_t high = q.high[o] - kHighBits, low = q.low[o] - kOnesBits;
            const uint32_t bin = __float_as_uint(o ? b.y : b.x) - kOnesBits;
            const bool in = free || floor.in(z[e + o], i0 + e + o);
            add_shared(&shared().bins.low[bin], in ? low : 0);
            add_shared(&shared().bins.high[bin], in ? high : 0);
          }
        }
      }
    });
  }

  // any level's histogram, of counts or masses
  template <bool kMass>
  __device__ __forceinline__ void count_elements(const Weigher& weigh, Floor floor, const Level& level) const {
    s.sweep([&](const uint4 (&v)[4], int c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[E];
        unpack<T>(v[i], z);
        const int i0 = s.first(c + 32 * i);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float y = weigh.exponent(z[e]);
          const int b = level.bin(y);
          const bool in = level.has(z[e]) && floor.in(z[e], i0 + e);
          if (!kMass) {
            add_shared(&shared().bins.low[b], in ? 1u : 0u);
          } else {
            const MassParts q = mass_parts(in ? grid_mass(exp2_32(y)) : 0u);
            add_shared(&shared().bins.low[b], q.low);
            add_shared(&shared().bins.high[b], q.high);
          }
        }
      }
    });
  }

  // The rest of a threshold's search, in the n elements of the first CTA's list.
  __device__ __forceinline__ u64 by_list(int n, const Weigher& weigh, u64 t, bool mass, float min_p) {
    const int lane = (int)threadIdx.x % 32, warps = (int)blockDim.x / 32, warp = warp_index();
    const bool keep = min_p >= 0.0f;
    if (group.rank == 0) {
      if (threadIdx.x == 0) {  // the answer of an empty list
        shared().found = ~0ull;
        shared().last = -1;
      }
      sort_list(n);
      // the running total down the list
      u64 ahead = 0;
#pragma unroll 1
      for (int i0 = 0; i0 < n; i0 += (int)blockDim.x) {
        const int i = i0 + (int)threadIdx.x;
        const u64 key = i < n ? shared().list[i] : 0;
        const u64 q = i >= n ? 0 : mass ? grid_mass(weigh(order_value(key))) : 1u;
        const u64 upto = warp_scan(q);
        if (lane == 31) shared().warp_q[warp] = upto;
        __syncthreads();
        const u64 w_q = lane < warps ? shared().warp_q[lane] : 0, w_upto = warp_scan(w_q);
        const u64 before = ahead + __shfl_sync(~0u, w_upto - w_q, warp);
        ahead += __shfl_sync(~0u, w_upto, 31);
        if (i < n && passes(before + upto - q, q, t, i == n - 1)) {
          shared().found = key;
          shared().last = i;
        }
        __syncthreads();
      }
      if (keep)
#pragma unroll 1
        for (int i = (int)threadIdx.x; i <= shared().last; i += (int)blockDim.x) {
          const u64 key = shared().list[i];
          const float w = weigh(order_value(key));
          if (!(w >= min_p)) continue;
          // the element's CTA and part
          const int c = (order_index(key) + s.head) / E, r = c / per_cta, at = c - r * per_cta;
          const u64 q = grid_mass(w);
          atomicAdd(group.at(&shared().parts[part_at(at / 32)], r), q);
        }
    }
    group.sync();
    const u64 key = *group.at(&shared().found, 0);
    if (!keep) group.sync();  // found and the list may be written again
    return key;
  }

  // ---- draws

  // one warp: the token of the slice whose kept mass covers t (counted from the slice's start)
  __device__ __noinline__ static void draw(Row row, u64 t, Weigher weigh, Kept kept, u64 all, int32_t* tok, float* prob) {
    row.find_token(t, weigh, kept, all, tok, prob);
  }
  __device__ __forceinline__ void find_token(u64 t, const Weigher& weigh, const Kept& kept, u64 all, int32_t* tok,
                                             float* prob) const {
    locate(t, [&](float z, int i) { return kept_mass(z, i, weigh, kept); },
           [&](float z, int i) {
             *tok = i;
             *prob = weigh(z) * kGrid / (float)all;
           });
  }
  // one warp: found(value, index), by one lane, of the element at which the total of mass(value, index), noted by part,
  // passes t
  template <typename M, typename F>
  __device__ __forceinline__ void locate(u64 t, M mass, F found) const {
    const int lane = (int)threadIdx.x % 32;
    const int parts = (s.n + 31) / 32, per = (parts + 31) / 32;  // parts of a lane
    u64 sum = 0;
#pragma unroll 4
    for (int i = 0; i < per; ++i) sum += lane * per + i < parts ? shared().parts[part_at(lane * per + i)] : 0;
    u64 upto = warp_scan(sum);
    const int l = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
    t -= __shfl_sync(~0u, upto - sum, l);
    sum = lane < per && l * per + lane < parts ? shared().parts[part_at(l * per + lane)] : 0;
    upto = warp_scan(sum);
    const int p = min(__popc(__ballot_sync(~0u, upto <= t)), 31);
    t -= __shfl_sync(~0u, upto - sum, p);
    const int c = (l * per + p) * 32 + lane, i0 = s.first(c);
    float z[E];
    unpack<T>(s.chunk(c), z);
    uint32_t q[E];
    sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) sum += q[e] = mass(z[e], i0 + e);
    upto = warp_scan(sum);
    if (t >= upto - sum && t < upto) {  // this lane's chunk has the element
      t -= upto - sum;
      float value = 0.0f;
      int at = -1;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (at < 0 && t < q[e]) {
          at = e;
          value = z[e];
        }
        t -= at < 0 ? q[e] : 0;
      }
      found(value, i0 + at);
    }
    __syncwarp();
  }

  // the first CTA: draws from the top-k list that settle() left
  __device__ __forceinline__ void draw_from_list(const Weigher& weigh, int top_k, u64 p24, float min_p, const float* u, int S,
                                 int32_t* tok, float* prob) {
    TopList& l = shared().top;
    const int n = min(top_k, shared().count);
    ranked([&](int at, u64 key) {
      if (at < n) {
        l.key[at] = key;
        l.q[at] = grid_mass(weigh(order_value(key)));
      }
    });
    __syncthreads();
    for (int i = (int)threadIdx.x; i < n; i += (int)blockDim.x) {
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
    for (int i = (int)threadIdx.x; i < n; i += (int)blockDim.x) {
      const int index = order_index(l.key[i]);
      u64 first = 0;
      for (int j = 0; j < n; ++j)
        if (order_index(l.key[j]) < index) first += l.kept[j];
      l.first[i] = first;
    }
    __syncthreads();
    for (int d = (int)threadIdx.x; d < S; d += (int)blockDim.x) {
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

// ---- the K best
//
// conf = 2^((z - m) c) / sum, one pass from memory with a running maximum, then a few thousand elements from L2.  1,024 rows
// of 126,000 bf16, 32 best: 61 us, 4.2 TB/s, where a copy of the bytes at 6.7 TB/s is 39 us.  What is left: issue slots
// (55 % used; nine instructions an element) and the waits of a row's ranking, which three rows an SM cover in part.
// Two CTAs an SM with 64 registers: 64 us; three have 40 and spill 60 to 72 bytes, in the ways of a full list.  Few rows: a
// call on the host takes 6.8 us, 64 rows of 32,768 on the GPU 6.2.

template <typename T>
struct Propose {
  typedef PickArgs Args;
  const Args& a;
  __device__ explicit Propose(const Args& args) : a(args) {}

  __device__ __forceinline__ void run(Row<T>& row, int r) const {
    constexpr int E = ElemOf<T>::E;
    const int lane = (int)threadIdx.x % 32, warps = (int)blockDim.x / 32, warp = warp_index();
    const float temp = row_temperature(a, r);
    const float c = exponent_scale(temp);
    // one pass: the lane's maximum so far and the sum of its weights relative to it
    LaneTop top;
    float2 sums = make_float2(0.0f, 0.0f);
    row.s.sweep([&](const uint4 (&v)[4], int at) {
      ChunkMax<T, false> batch;
      batch.add(v);
      const float x = batch.value();
      if (x > top.first) {
        const float by = exp2_32((top.first - x) * c);
        sums.x *= by;
        sums.y *= by;
      }
      top.add(x, at);
      if (top.first == -CUDART_INF_F) return;
      const Weigher relative{top.first, c};
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
    const float most = row.top_of(top.first, a.K, &floor);
    const Weigher weigh = weigher(most, c);
    row.collect(floor, top);
    float sum = sums.x + sums.y;
    if (__any_sync(~0u, sum != sum) || most == CUDART_INF_F) {  // NaN or +inf among the warp's elements or the row's
      sum = 0.0f;
      row.each([&](float z, int) {
        const float w = weigh(z);
        sum += w > 0.0f ? w : 0.0f;
      });
    } else {
      sum = top.first == -CUDART_INF_F ? 0.0f : sum * exp2_32((top.first - weigh.m) * weigh.c);
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) *row.group.at(&shared().sums[row.group.rank * warps + warp], 0) = sum;
    row.group.sync();
    row.settle(a.K, most);
    if (row.group.rank != 0) return;
    sum = 0.0f;
    for (int i = 0; i < (int)row.group.n * warps; ++i) sum += shared().sums[i];
    int32_t* cand = a.cand + (long long)r * a.K;
    float* conf = a.conf + (long long)r * a.K;
    const bool good = temp >= 0.0f;
    for (int i = (int)threadIdx.x; i < a.K; i += (int)blockDim.x)
      if (!good || i >= shared().count) {
        cand[i] = -1;
        conf[i] = 0.0f;
      }
    if (good)
      row.ranked([&](int at, u64 key) {
        if (at >= a.K) return;
        cand[at] = order_index(key);
        conf[at] = temp == 0.0f ? (at == 0 ? 1.0f : 0.0f) : weigh(order_value(key)) / sum;
      });
    if (row.group.n > 1) row.group.sync();  // the others have looked at the count
  }
};

// ---- draws
//
// A pass from memory for the maximum, one from L2 for the masses by part, a chunk a lane for each draw; with a nucleus or a
// long top-k a pass for the histogram and one for the bin's elements and the kept masses in place of that of masses.
// 1,024 rows of 126,000 bf16: 100 us by temperature, 303 us with top-p.  17 and 54 instructions an element use 56 and 66 % of
// the issue slots; the rest is waits that two rows an SM (46 % of its warps) leave open.  Of the nucleus's instructions the
// histogram's two additions to shared memory are the slowest: one of 64 bits took 570 us in all.  Two CTAs an SM have 64
// registers and spill 188 bytes; three have 40 and spill 304: 115 us by temperature, 320 with top-p.  With 512, 384 and 256
// threads: 100, 117, 111 us and 303, 336, 321.

template <typename T>
struct Sample {
  typedef PickArgs Args;
  const Args& a;
  __device__ explicit Sample(const Args& args) : a(args) {}

  __device__ __forceinline__ void run(Row<T>& row, int r) const {
    const int lane = (int)threadIdx.x % 32;
    const int b = r / a.rows.k;
    const float temp = row_temperature(a, r);
    float top_p = a.top_p ? a.top_p[b] : 1.0f;
    const float min_p = a.min_p ? a.min_p[b] : 0.0f;
    int top_k = a.top_k ? a.top_k[b] : 0;
    const bool good = temp >= 0.0f && top_p == top_p && min_p == min_p;
    top_p = fminf(fmaxf(top_p, 0.0f), 1.0f);
    const u64 p24 = __float2uint_rn(top_p * 16777216.0f);
    if (temp == 0.0f || p24 == 0 || min_p > 1.0f || !good) top_k = 1;
    if (top_k <= 0 || top_k > a.rows.V) top_k = a.rows.V;
    const bool by_list = top_k <= kMaxK;
    const float* u = a.u + (long long)r * a.S;
    const int warp = warp_index(), warps = (int)blockDim.x / 32;
    const float first_u = warp < a.S ? u[warp] : 0.0f;  // on its way during the passes
    int32_t* tok = a.tok + (long long)r * a.S;
    float* prob = a.prob + (long long)r * a.S;
    float floor;
    const LaneTop top = row.lane_top();
    const float most = row.top_of(top.first, by_list ? top_k : 0, &floor);
    const Weigher weigh = weigher(most, exponent_scale(temp));
    if (by_list) {
      row.collect(floor, top);
      row.group.sync();
      row.settle(top_k, most);
      if (row.group.rank != 0) return;
      row.draw_from_list(weigh, good ? top_k : 0, p24, min_p, u, a.S, tok, prob);
      if (row.group.n > 1) row.group.sync();  // the others have looked at the count
      return;
    }
    // T = inf: the exponents of -inf, which also fills the last chunks up, are -inf times 0
    row.special = row.special || fabsf(weigh.m) == CUDART_INF_F || weigh.c == 0.0f;
    const bool by_mass = p24 < (1u << 24);
    Kept kept{no_floor(), fmaxf(min_p, 0.0f)};
    if (top_k < a.rows.V)
      kept.floor = floor_of(Row<T>::threshold(row, weigh, kept.floor, top_k - 1, false, by_mass ? -1.0f : kept.min_p));
    if (by_mass) kept.floor = floor_of(Row<T>::threshold(row, weigh, kept.floor, p24, true, kept.min_p));
    if (top_k == a.rows.V && !by_mass) {
      Row<T>::masses(row, weigh, kept);
      row.group.sync();
    }
    u64 mine, ahead;
    const u64 all = row.all_mass(&mine, &ahead);
    for (int i = warp; i < a.S; i += warps) {
      const float x = i == warp ? first_u : u[i];
      if (all == 0 || !(x >= 0.0f && x <= 1.0f)) {
        if (row.group.rank == 0 && lane == 0) {
          tok[i] = -1;
          prob[i] = 0.0f;
        }
        continue;
      }
      const u64 t = min(share24((u64)(x * 16777216.0f), all), all - 1);
      if (t >= ahead && t < ahead + mine) Row<T>::draw(row, t - ahead, weigh, kept, all, &tok[i], &prob[i]);
    }
    if (row.group.n > 1) row.group.sync();  // no CTA leaves while its masses are read
  }
};

// a cluster of CTAs for each row
template <typename T, template <typename> class Op, int kPerSm>
__global__ void __launch_bounds__(kRowThreads, kPerSm) k_rows(PickArgs a) {
  Row<T> row;
  row.per_cta = a.rows.per;
  const int r = (int)(blockIdx.x / row.group.n);
  row.s.open(row_address<T>(a.rows, r), a.rows, row.group.rank, shared().ends);
  Op<T>(a).run(row, r);
}

template <typename T, template <typename> class Op, int kPerSm>
epic_status launch(PickArgs& a, long long rows, cudaStream_t st) {
  const RowShape p = row_shape(rows, a.rows.V, sizeof(T), kPickThreadsMin, kRowThreads);
  a.rows.per = p.per;
  return launch_rows((const void*)k_rows<T, Op, kPerSm>, p, rows, &a, st);
}

template <typename T>
epic_status launch(PickArgs& a, long long rows, bool sample, cudaStream_t st) {
  return sample ? launch<T, Sample, 2>(a, rows, st) : launch<T, Propose, 3>(a, rows, st);
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
  if (K > kMaxK || V > kMaxV) return EPIC_ERR_CAPACITY;
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
  if (V > kMaxV) return EPIC_ERR_CAPACITY;
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
