// The matrix products of the head's loss, on the tensor units: logits = h W^T,
// gradients dh = e W and dW = e^T hs.
//
// A tile of 256 x 256 is a pair of CTAs': each copies 128 rows of both operands in steps of 64 of the sum (TMA, five steps
// ahead), one thread of the pair issues the products, sums lie in tensor memory, twice, so that eight warps a CTA work on
// one tile's sums while the next tile's are made.  Operands are read as they lie: e along and across its rows, the head by
// tokens and by hidden dimensions.
//
// A step of a tile takes the tensor units 512 clocks and 64 bytes a clock and SM from L2, about what L2 gives: a CTA's own
// tile of 128 x 256 would need 96.  Of 4,096 rows through 32,768 x 2,048 the tensor pipe is active 95 % of the time for logits
// alone, 84 % with exponentials, 88 % for both gradients (261, 289 and 582 us); of 4,096 through 126,000 x 4,096 they take 2.08,
// 2.22 and 4.64 ms (2.03, 1.90 and 1.82 PFLOP/s) from rest, both calls 9.1 ms, and 10.1 one after another, at the power limit.  With
// few rows the head's bytes are the time: 32 through 126,000 x 4,096 185 us (5.6 TB/s) for logits, 400 for the gradients, which
// read it once and write as much.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "head_launch.cuh"
#include "head_loss.h"
#include "head_rows.cuh"
#include "tensor_tiles.cuh"

namespace epic {
namespace {

constexpr int kTile = 256, kHalf = 128;  // a pair's tile, a CTA's share of an operand
constexpr int kStepK = 64, kStages = 5;
constexpr int kOperand = kHalf * kStepK * 2, kStage = 2 * kOperand;  // bytes
constexpr int kWorkWarps = 8, kThreads = 128 + 32 * kWorkWarps;
constexpr int kPairs = 76;  // of the GB300's 152 SMs
constexpr int kTurn = 2 * 32 * 128;  // bytes of a warp's two turning buffers: 64 elements of 32 rows each
constexpr int kShared = kStages * kStage + kWorkWarps * kTurn + 1024;

struct Bars {
  uint64_t full[kStages], empty[kStages], sums_full[2], sums_empty[2];
  uint32_t sums, gave_up;
};

// One tile of a product: where its operands' boxes lie and how many steps its sum has
struct Task {
  int m0, n0;      // rows of A and B
  int k0, steps;   // first step
  int job;         // 0: logits, or gradient of hidden states; 1: gradient of the head
  int part;        // of a sum in several parts
};

struct TileArgs {
  HeadPlan p;
  LogitsPass pass;
  HiddenGrad out;
  void* grad_head;
  long long grad_head_stride;
  HeadSum sum;
  int bf16;
  int pairs;  // of CTAs
  long long wait;  // limit of a wait, in clocks
};

__device__ __forceinline__ int up_div(int a, int b) { return (a + b - 1) / b; }

// Division by a number that stays
struct Divisor {
  uint32_t by, inverse;
  __device__ __forceinline__ explicit Divisor(int n) : by(n), inverse(0xffffffffu / (uint32_t)n) {}
  __device__ __forceinline__ int of(int x, int& rest) const {
    uint32_t q = __umulhi(x, inverse), left = x - q * by;  // q is at most 2 too small
    while (left >= by) left -= by, q++;
    rest = (int)left;
    return (int)q;
  }
};

// The tiles of a pair, one after another.  (Each warp role goes through them for itself; worked out anew for every tile, with
// its divisions, a tile of one step took 5,400 clocks.)
//
// Logits: the rows' tiles of one column of tiles after another, so that the head is read once.
struct LogitsTasks {
  Divisor row_tiles;
  int at, tiles, steps, pairs;
  __device__ __forceinline__ LogitsTasks(const TileArgs& a, int n, int pair)
      : row_tiles(max(1, up_div(n, kTile))), at(pair), tiles(up_div(n, kTile) * up_div(a.p.V, kTile)),
        steps(up_div(a.p.d, kStepK)), pairs(a.pairs) {}
  __device__ __forceinline__ bool next(Task& t) {
    if (at >= tiles) return false;
    int m;
    const int column = row_tiles.of(at, m);
    t = {m * kTile, column * kTile, 0, steps, 0, 0};
    at += pairs;
    return true;
  }
};

// Gradients: first all tiles of hidden states (long sums), then the head's.  Where the former do not come out even, the pairs
// without a last one take as many of the latter as it is worth before the rest is dealt to all.
struct GradTasks {
  Divisor columns;
  int pairs;
  int row_tiles, head_tiles, hidden_parts, head_parts, v_steps, r_steps;
  int hidden, hidden_left;  // the next tile of hidden states, how many
  int head[2], by[2], left[2];  // the next one of the head's, how far the one after is, how many, in the two rounds
  __device__ __forceinline__ GradTasks(const TileArgs& a, int n, int pair) : columns(up_div(a.p.d, kTile)), pairs(a.pairs) {
    const GradSplit& s = a.p.split;
    const int ct = columns.by;
    row_tiles = up_div(n, kTile) * ct;
    head_tiles = up_div(a.p.V, kTile) * ct;
    hidden_parts = s.hidden_parts;
    head_parts = s.head_parts;
    v_steps = up_div(a.p.V, kStepK);
    r_steps = up_div(n, kStepK);
    const int all_hidden = hidden_parts * row_tiles, all_head = head_parts * head_tiles, last = all_hidden % pairs;
    hidden = pair;
    hidden_left = all_hidden / pairs + (pair < last);
    // (an estimate in floats is as good, and the same for all)
    const float worth = __fdividef((float)(up_div(v_steps, max(1, hidden_parts)) + s.tile_cost),
                                   (float)(up_div(r_steps, max(1, head_parts)) + s.tile_cost));
    const int idle = last ? pairs - last : 0, first = idle ? min(all_head / idle, (int)worth) : 0;
    head[0] = pair - last, by[0] = idle, left[0] = pair >= last ? first : 0;
    head[1] = first * idle + pair, by[1] = pairs;
    left[1] = head[1] < all_head ? (all_head - head[1] + pairs - 1) / pairs : 0;
  }
  __device__ __forceinline__ void sum(Task& t, int job, int at, int tiles, int parts, int steps) const {
    int part = 0, c;
    t.k0 = 0;
    t.steps = steps;
    if (parts > 1) {
      part = at / tiles;
      at -= part * tiles;
      t.k0 = (int)((long long)steps * part / parts);
      t.steps = (int)((long long)steps * (part + 1) / parts) - t.k0;
    }
    t.m0 = columns.of(at, c) * kTile;
    t.n0 = c * kTile;
    t.job = job;
    t.part = part;
  }
  __device__ __forceinline__ bool next(Task& t) {
    if (hidden_left > 0) {
      sum(t, 0, hidden, row_tiles, hidden_parts, v_steps);
      hidden += pairs;
      hidden_left--;
      return true;
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
      if (left[i] <= 0) continue;
      sum(t, 1, head[i], head_tiles, head_parts, r_steps);
      head[i] += by[i];
      left[i]--;
      return true;
    }
    return false;
  }
};

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *(const uint32_t*)&h;
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&h;
}

// A warp's sums on their way out: 64 elements of its 32 rows, a lane a row, turned in shared memory so that they leave by
// whole runs of a row (1 GB of a gradient leaves at 4.9 TB/s by 32 bytes of every lane's own row, at 6.6 by runs).  Rows
// of 128 bytes, chunks of 16 swizzled by the row's number in 8: as boxes are, and without conflicts either way.  Two buffers,
// so that one fence (some 500 clocks) is for two boxes.
struct Turn {
  uint32_t at, other;
  int lane;
  __device__ __forceinline__ uint32_t chunk(int row, int c) const { return at + row * 128 + ((c ^ row) & 7) * 16; }
  // the lane's elements 32 half ..
  template <typename T>
  __device__ __forceinline__ void put(const float (&v)[32], int half) const {
#pragma unroll
    for (int c = 0; c < 4; c++)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk(lane, half * 4 + c)),
                   "r"(pack2<T>(v[8 * c], v[8 * c + 1])), "r"(pack2<T>(v[8 * c + 2], v[8 * c + 3])),
                   "r"(pack2<T>(v[8 * c + 4], v[8 * c + 5])), "r"(pack2<T>(v[8 * c + 6], v[8 * c + 7]))
                   : "memory");
  }
  // all 64, or from the second on
  template <typename T>
  __device__ __forceinline__ void put(const float (&v)[32], const float (&w)[32], bool second) const {
    float x[65];
#pragma unroll
    for (int i = 0; i < 32; i++) x[i] = v[i], x[32 + i] = w[i];
    x[64] = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; c++) {
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; i++)
        o[i] = pack2<T>(second ? x[8 * c + 2 * i + 1] : x[8 * c + 2 * i], second ? x[8 * c + 2 * i + 2] : x[8 * c + 2 * i + 1]);
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk(lane, c)), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3])
                   : "memory");
    }
  }
  // 32 numbers of 32 bits of the lane's row
  __device__ __forceinline__ void put_floats(const float (&v)[32]) const {
#pragma unroll
    for (int c = 0; c < 8; c++)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk(lane, c)), "f"(v[4 * c]), "f"(v[4 * c + 1]),
                   "f"(v[4 * c + 2]), "f"(v[4 * c + 3])
                   : "memory");
  }
  // to the other buffer
  __device__ __forceinline__ void next() {
    const uint32_t now = other;
    other = at;
    at = now;
  }
  // before the first put: the boxes before have left
  __device__ __forceinline__ void free() const {
    if (lane == 0) boxes_read<0>();
    __syncwarp();
  }
  // the other buffer's box and, if x2 >= 0, this one's at x2
  __device__ __forceinline__ void store(const CUtensorMap* map, int x, int x2, int y) const {
    shared_to_boxes();
    __syncwarp();
    if (lane == 0) {
      store_box(map, other, x, y);
      if (x2 >= 0) store_box(map, at, x2, y);
    }
  }
  // to each lane's row `to` (NULL from row `rows` on), which starts at a multiple of 16 bytes, 64 elements: 8 lanes a row
  __device__ __forceinline__ void store_whole(uint16_t* to) const {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int row = i * 4 + lane / 8;
      uint16_t* p = (uint16_t*)__shfl_sync(~0u, (unsigned long long)to, row);
      uint4 v;
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                   : "r"(chunk(row, lane % 8))
                   : "memory");
      if (p) *(uint4*)(p + lane % 8 * 8) = v;
    }
  }
  // the same of rows that start anywhere, `count` elements of up to 64 (the same in all lanes): a warp a row, two elements a
  // lane.  Rows that start at an odd element were put from the second on; lanes write their own row's ends.
  __device__ __forceinline__ void store_runs(uint16_t* to, int rows, int count, uint32_t first) const {
    const bool odd = (uintptr_t)to & 2;
    const uint32_t odds = __ballot_sync(~0u, odd);
    __syncwarp();
    if (to && odd) *to = (uint16_t)first;
    const int last = count - 1 - odd;  // in what was put
    if (to && last >= 0 && last % 2 == 0) {
      uint16_t v;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(chunk(lane, last / 8) + last % 8 * 2) : "memory");
      to[count - 1] = v;
    }
    to += odd;
#pragma unroll 1
    for (int row0 = 0; row0 < min(rows, 32); row0 += 8) {
      uint32_t two[8];
#pragma unroll
      for (int i = 0; i < 8; i++)
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(two[i]) : "r"(at + (row0 + i) * 128 + ((lane / 4) ^ i) * 16 + lane % 4 * 4) : "memory");
#pragma unroll
      for (int i = 0; i < 8; i++) {
        uint32_t* p = (uint32_t*)__shfl_sync(~0u, (unsigned long long)to, row0 + i);
        if (row0 + i < rows && 2 * lane + 1 < count - (int)(odds >> (row0 + i) & 1)) p[lane] = two[i];
      }
    }
  }
};

__device__ __forceinline__ float sum32(const float (&v)[32]) {
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; j++) s[j] = (v[j] + v[j + 8]) + (v[j + 16] + v[j + 24]);
  return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
}

__device__ __forceinline__ float max32(const float (&v)[32]) {
  float m = v[0];
#pragma unroll
  for (int j = 1; j < 32; j++) m = fmaxf(m, v[j]);
  return m;
}

// What a row's logits are made into, read before they are there
struct LogitsRow {
  int target;
  float ref, mul, at;
  __device__ __forceinline__ LogitsRow(const TileArgs& a, bool probs, int n, int row) : target(-1), ref(0.0f), mul(1.0f), at(0.0f) {
    if (row >= n) return;
    const HeadPlan& p = a.p;
    target = p.tgt[row];
    if (!probs) return;
    ref = a.pass.known ? p.known_ref[row] : p.ref[row];
    if (a.pass.known) mul = p.known_mul[row];
    if (a.pass.only_again) at = p.e_target[row];
  }
};

// Logits of one row, kRecCols columns from `sums`: the record, and with `probs` the exponentials.  z is only ever in registers.
template <typename T, bool kProbs>
__device__ __forceinline__ void logits_rows(const TileArgs& a, const HeadMaps& maps, int n, const LogitsRow& is, uint32_t sums,
                                            int row, int col, Turn& turn) {
  const HeadPlan& p = a.p;
  const bool real = row < n, known = a.pass.known;
  const int y = real ? is.target - col : -1;
  const float ref = is.ref, mul = is.mul;
  float to = kProbs ? (known ? 0.0f : ref) : kNoRef, s = 0.0f;
#pragma unroll 1
  for (int c = 0; c < kRecCols; c += 32) {
    if (col + c >= p.lde) break;
    float z[32];
    sums_load(sums + c, z);
    sums_loaded(z);
    const int here = y - c;
    if (col + c + 32 > p.V) {
#pragma unroll
      for (int j = 0; j < 32; j++)
        if (col + c + j >= p.V) z[j] = -CUDART_INF_F;
    }
    if (here >= 0 && here < 32) {  // the target is left out
      float zt = 0.0f;
#pragma unroll
      for (int j = 0; j < 32; j++)
        if (j == here) zt = z[j], z[j] = -CUDART_INF_F;
      if (a.pass.sums) p.zt[row] = zt;
    }
    if (kProbs) {
#pragma unroll
      for (int j = 0; j < 32; j++) z[j] = ex2(fmaf(z[j], kLog2E, -ref)) * mul;
      s += sum32(z);
      if (is.at != 0.0f && here >= 0 && here < 32) {
#pragma unroll
        for (int j = 0; j < 32; j++)
          if (j == here) z[j] = is.at;
        p.at_target[row] = lost<T>(is.at) * *p.post;
      }
      if (!real) {
#pragma unroll
        for (int j = 0; j < 32; j++) z[j] = 0.0f;
      }
      if (c == 0) turn.free();
      if (c % 64 == 0) turn.next();
      turn.put<T>(z, c / 32 % 2);
    } else {
      const float top = whole_ref(max32(z));
#pragma unroll
      for (int j = 0; j < 32; j++) z[j] = ex2(fmaf(z[j], kLog2E, -top));
      meet(to, s, top, sum32(z));
    }
  }
  if (kProbs && col < p.lde) {
    if (col + 64 >= p.lde) turn.next();  // one box only
    turn.store(&maps.e_out, col, col + 64 < p.lde ? col + 64 : -1, row - turn.lane);
  }
  if (!a.pass.sums || col >= p.V) return;
  // exponentials past the window: once more, relative to the largest
  const bool past = kProbs && !known && real && !(s <= 1.2e18f);
  if (kProbs && __any_sync(~0u, past)) {
    float to2 = kNoRef, s2 = 0.0f;
#pragma unroll 1
    for (int c = 0; c < kRecCols; c += 32) {
      float z[32];
      sums_load(sums + c, z);
      sums_loaded(z);
#pragma unroll
      for (int j = 0; j < 32; j++)
        if (col + c + j >= p.V || j == y - c) z[j] = -CUDART_INF_F;
      const float top = whole_ref(max32(z));
#pragma unroll
      for (int j = 0; j < 32; j++) z[j] = ex2(fmaf(z[j], kLog2E, -top));
      meet(to2, s2, top, sum32(z));
    }
    if (past) to = to2, s = s2;
  }
  if (real) p.rec[(long long)(col / kRecCols) * p.cap + row] = record(to, s);
}

__device__ __forceinline__ void store_floats(float* part, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) ((float4*)part)[j / 4] = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
}

// What a row of a gradient needs beside its sums, read before they are there
struct GradRow {
  long long begin;  // of a hidden state's gradient
  float coef;       // what its sums are multiplied with
  int4 with;        // of a hidden state: its target; of the head: the listed rows with that target; or -1
  float4 f;         // what they are multiplied with
  // a tile ahead
  __device__ __forceinline__ GradRow(const TileArgs& a, int n, bool again, float post, const Task& t, int row_of_tile)
      : begin(0), coef(post), with(make_int4(-1, -1, -1, -1)), f(make_float4(0.0f, 0.0f, 0.0f, 0.0f)) {
    const HeadPlan& p = a.p;
    const int row = t.m0 + row_of_tile;
    if (t.job == 0 && row < n) {
      begin = p.to[row];
      if (!again) coef = p.coef[row];
      f.x = p.at_target[row];
      with.x = p.tgt[row];
    } else if (t.job == 1 && row < p.V) {
      with = p.list[row];
    }
  }
  // before the tile's sums are waited for
  __device__ __forceinline__ void factors(const TileArgs& a, const Task& t) {
    if (t.job == 0) {
      if (f.x == 0.0f) with.x = -1;
      return;
    }
    const float* at = a.p.at_target;
    if (with.x >= 0) f.x = at[with.x];
    if (with.y >= 0) f.y = at[with.y];
    if (with.z >= 0) f.z = at[with.z];
    if (with.w >= 0) f.w = at[with.w];
  }
};

// v += f x[0..31], of which those before `end` are used, at a multiple of 16 bytes
template <typename T>
__device__ __forceinline__ void add_row(float (&v)[32], float f, const T* x, int end) {
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
    if (j >= end) break;
    const uint4 w = *(const uint4*)(x + j);
    const T* t = (const T*)&w;
#pragma unroll
    for (int i = 0; i < 8; i++) v[j + i] = fmaf(f, as_float(t[i]), v[j + i]);
  }
}

// Sums of a gradient's tile: kHalf columns of each lane's row, 64 at a time
template <typename T>
__device__ __forceinline__ void grad_rows(const TileArgs& a, const HeadMaps& maps, int n, float post, const GradRow& is,
                                          const Task& t, uint32_t sums, int row, int col, Turn& turn) {
  const HeadPlan& p = a.p;
  const GradSplit& sp = a.p.split;
  const bool hidden = t.job == 0;
  const bool parts = (hidden ? sp.hidden_parts : sp.head_parts) > 1;
  const int end = hidden ? n : p.V;
  if (row - turn.lane >= end) return;
  const bool there = row < end, out = !parts && (hidden || a.sum == kOnly || a.sum == kLast), box = out && !hidden && maps.boxes;
  uint16_t* to = nullptr;
  if (there && out) to = hidden ? (uint16_t*)a.out.grad + is.begin : (uint16_t*)a.grad_head + row * a.grad_head_stride;
  const float scale = hidden ? is.coef : post;
  const bool whole = __all_sync(~0u, ((uintptr_t)to & 15) == 0);
  const CUtensorMap* part = hidden ? &maps.hidden_parts : &maps.head_parts;
  const int part_row = t.part * (hidden ? p.cap : (int)sp.tokens) + row - turn.lane;
  float* acc = p.acc + (long long)row * p.ldp;
  auto load = [&](float(&v)[32], float(&w)[32], int c) {
    if (t.steps > 0) {
      sums_load(sums + (c - col), v);
      sums_load(sums + (c - col) + 32, w);
      sums_loaded(v);
      sums_loaded(w);
    } else {
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] = w[j] = 0.0f;
    }
  };
  auto pass = [&](float(&v)[32], int c) {
    if (!hidden && a.sum != kOnly && there && c < p.d) {
      if (a.sum != kFirst) {
#pragma unroll
        for (int j = 0; j < 32; j++) v[j] += acc[c + j];
      }
      if (a.sum != kLast) store_floats(acc + c, v);
    }
  };
#pragma unroll 1
  for (int c = col; c < col + kHalf && c < p.d; c += 64) {
    float v[32], w[32];
    load(v, w, c);
    if (c == col || parts) turn.free();
    if (parts) {
      turn.next();
      turn.put_floats(v);
      turn.next();
      turn.put_floats(w);
      turn.store(part, c, c + 32 < p.d ? c + 32 : -1, part_row);
      continue;
    }
    if (scale != 1.0f) {
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] *= scale, w[j] *= scale;
    }
    const T* x = hidden ? (const T*)p.head + c : (const T*)p.hc + c;
    const long long ld = hidden ? p.ldw : p.ldh;
    int4 q = is.with;
    float4 f = is.f;
#pragma unroll 1
    while (__any_sync(~0u, q.x >= 0)) {
      if (q.x >= 0) {
        add_row(v, f.x, x + q.x * ld, p.d - c);
        add_row(w, f.x, x + q.x * ld + 32, p.d - c - 32);
      }
      q = make_int4(q.y, q.z, q.w, -1);
      f = make_float4(f.y, f.z, f.w, 0.0f);
    }
    pass(v, c);
    pass(w, c + 32);
    if (!out) continue;
    uint16_t* here = to ? to + c : nullptr;
    if (!box && !(whole && p.d - c >= 64)) {
      turn.next();
      turn.put<T>(v, w, (uintptr_t)here & 2);
      turn.store_runs(here, end - (row - turn.lane), min(p.d - c, 64), pack2<T>(v[0], v[0]) & 0xffff);
      continue;
    }
    turn.next();
    turn.put<T>(v, 0);
    turn.put<T>(w, 1);
    if (!box) turn.store_whole(here);
  }
  if (box && col < p.d) {
    if (col + 64 >= p.d) turn.next();  // one box only
    turn.store(&maps.grad_out, col, col + 64 < p.d ? col + 64 : -1, row - turn.lane);
  }
}

// NaN to a row's half, kHalf columns from `half` on, of all of a pair's tiles: whatever comes of them is NaN, too
template <typename T, int kForm>
__device__ __noinline__ void spoil_tiles(const TileArgs& a, int n, int pair, int row_of_tile, int half) {
  const HeadPlan& p = a.p;
  typename std::conditional<kForm == 2, GradTasks, LogitsTasks>::type tasks(a, n, pair);
  Task t;
  while (tasks.next(t)) {
    const long long row = t.m0 + row_of_tile;
    const int col = t.n0 + half;
    if (kForm != 2) {
      if (row >= n) continue;
      if (a.pass.sums && col < p.V) p.rec[(long long)(col / kRecCols) * p.cap + row] = make_float2(0.0f, CUDART_NAN_F);
      if (kForm == 1)
        for (long long c = col; c < min(col + (long long)kHalf, p.lde); c++) ((T*)p.e)[row * p.lde + c] = of_float<T>(CUDART_NAN_F);
      continue;
    }
    const GradSplit& sp = p.split;
    const bool hidden = t.job == 0;
    if (row >= (hidden ? n : p.V)) continue;
    float* sums = nullptr;
    if ((hidden ? sp.hidden_parts : sp.head_parts) > 1)
      sums = (hidden ? sp.hidden + t.part * (long long)p.cap * p.ldp : sp.head + t.part * sp.tokens * p.ldp) + row * p.ldp;
    else if (!hidden && a.sum != kOnly && a.sum != kLast)
      sums = p.acc + row * p.ldp;
    T* to = hidden ? (T*)a.out.grad + p.to[row] : (T*)a.grad_head + row * a.grad_head_stride;
    for (int c = col; c < min(col + kHalf, p.d); c++) {
      if (sums) sums[c] = CUDART_NAN_F;
      else to[c] = of_float<T>(CUDART_NAN_F);
    }
  }
}

// kForm 0: records; 1: exponentials (and records); 2: gradients
template <typename T, int kForm>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_head_tiles(const __grid_constant__ HeadMaps maps, const __grid_constant__ TileArgs a) {
  extern __shared__ uint8_t shared_raw[];
  __shared__ Bars bars;
  uint8_t* shared = (uint8_t*)(((uintptr_t)shared_raw + 1023) / 1024 * 1024);
  const uint32_t stages = smem_address(shared);
  const int warp = warp_of_thread(), lane = threadIdx.x % 32, pair = blockIdx.x / 2;
  const uint32_t rank = cluster_rank();
  const uint32_t full = smem_address(bars.full), empty = smem_address(bars.empty);
  const uint32_t sums_full = smem_address(bars.sums_full), sums_empty = smem_address(bars.sums_empty);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; s++) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < 2; s++) {
      bar_init(sums_full + 8 * s, 1);
      bar_init(sums_empty + 8 * s, 2 * kWorkWarps);
    }
    bars.gave_up = 0;
    bar_init_visible();
  }
  if (threadIdx.x == 32)
    for (const CUtensorMap* m : {&maps.hc, &maps.hs, &maps.head, &maps.e, &maps.e_out, &maps.grad_out, &maps.hidden_parts,
                                 &maps.head_parts})
      prefetch_map(m);
  if (kForm != 2 && a.pass.only_again) {  // mostly there is nothing to do
    follow();
    if (*a.p.again == 0) return;
  }
  if (warp == 1) sums_take_pair(smem_address(&bars.sums));
  products_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  const uint32_t sums = bars.sums;
  follow();
  let_next();
  const bool again = *a.p.again != 0;
  const int n = *a.p.count;
  typename std::conditional<kForm == 2, GradTasks, LogitsTasks>::type tasks(a, n, pair);
  bool ok = a.wait > 0;
  if (warp == 0) {
    if (lane == 0) {  // copies
      const uint32_t full0 = at_rank(full, 0);
      int s = 0;
      uint32_t turn = 0;
      Task t;
      while (ok && tasks.next(t)) {
        const int m = t.m0 + rank * kHalf, c = t.n0 + rank * kHalf;
        for (int k = t.k0; k < t.k0 + t.steps; k++) {
          if (!(ok = bar_wait(empty + 8 * s, turn ^ 1, a.wait))) break;
          if (rank == 0) bar_expect(full + 8 * s, 2 * kStage);
          const uint32_t A = stages + s * kStage, B = A + kOperand, bar = full0 + 8 * s;
          // 128 rows of 64 along the sum, or 64 of the sum by 128 across it: two boxes each
          const CUtensorMap* ma = kForm == 2 ? &maps.e : &maps.hc;
          const CUtensorMap* mb = kForm != 2 || t.job == 0 ? &maps.head : again ? &maps.hc : &maps.hs;
          const bool a_across = kForm == 2 && t.job == 1, b_across = kForm == 2;
          const int at = k * kStepK;
#pragma unroll
          for (int i = 0; i < 2; i++) {
            load_box_pair(ma, A + i * kOperand / 2, bar, a_across ? m + 64 * i : at, a_across ? at : m + 64 * i);
            load_box_pair(mb, B + i * kOperand / 2, bar, b_across ? c + 64 * i : at, b_across ? at : c + 64 * i);
          }
          if (++s == kStages) s = 0, turn ^= 1;
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {  // products
      int s = 0, use = 0;
      uint32_t turn = 0;
      Task t;
      while (ok && tasks.next(t)) {
        if (t.steps <= 0) continue;
        const int half = use & 1;
        if (!(ok = bar_wait_warp(sums_empty + 8 * half, (use >> 1 & 1) ^ 1, a.wait))) break;
        products_fence_after();
        const bool a_across = kForm == 2 && t.job == 1, b_across = kForm == 2;
        const uint32_t kind = product_kind(a.bf16, a_across, b_across, kTile, kTile);
        const uint32_t to = sums + half * kTile;
        for (int k = 0; k < t.steps; k++) {
          if (!(ok = bar_wait_warp(full + 8 * s, turn, a.wait))) break;
          products_fence_after();
          if (one_lane()) {
            const uint32_t A = stages + s * kStage, B = A + kOperand;
            const uint64_t da = a_across ? operand_mn(A) : operand_k(A), db = b_across ? operand_mn(B) : operand_k(B);
            const uint32_t na = a_across ? kNextMN : kNextK, nb = b_across ? kNextMN : kNextK;
#pragma unroll
            for (int j = 0; j < kStepK / 16; j++) product_pair(to, da + j * na, db + j * nb, kind, k > 0 || j > 0);
            products_arrive_pair(empty + 8 * s);
          }
          __syncwarp();
          if (++s == kStages) s = 0, turn ^= 1;
        }
        if (!ok) break;
        if (one_lane()) products_arrive_pair(sums_full + 8 * half);
        __syncwarp();
        use++;
      }
    }
  } else if (warp < 4) {
    if (kForm != 2 && a.p.list && !a.pass.only_again)  // empty lists, for the kernel behind this one
      for (long long v = blockIdx.x * 64ll + threadIdx.x - 64; v < a.p.V; v += gridDim.x * 64ll)
        a.p.list[v] = make_int4(-1, -1, -1, -1);
  } else {
    const int part = warp - 4, quarter = warp % 4;
    const uint32_t turns = stages + kStages * kStage + part * kTurn;
    Turn turn = {turns, turns + kTurn / 2, lane};
    const float post = kForm == 2 && again ? *a.p.post : 1.0f;
    int use = 0;
    const int row_of_tile = rank * kHalf + quarter * 32 + lane, off = part / 4 * kHalf;
    // one tile's sums, by `rows`; false: gave up
    auto tile = [&](const Task& t, auto rows) {
      const int half = use & 1;
      const uint32_t from = sums + half * kTile + off + ((uint32_t)quarter * 32 << 16);
      if (t.steps > 0) {
        if (!(ok = bar_wait_warp(sums_full + 8 * half, use >> 1 & 1, a.wait))) return false;
        products_fence_after();
      }
      rows(from);
      if (t.steps > 0) {
        products_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(at_rank(sums_empty + 8 * half, 0));
        use++;
      }
      return true;
    };
    Task t;
    if constexpr (kForm == 2) {
      Task ahead = {a.p.V, 0, 0, 0, 1, 0};
      bool more = tasks.next(ahead);
      GradRow with_ahead(a, n, again, post, ahead, row_of_tile);  // a tile before it is needed
      while (ok && more) {
        t = ahead;
        GradRow with = with_ahead;
        with.factors(a, t);
        more = tasks.next(ahead);
        if (more) with_ahead = GradRow(a, n, again, post, ahead, row_of_tile);
        if (!tile(t, [&](uint32_t from) { grad_rows<T>(a, maps, n, post, with, t, from, t.m0 + row_of_tile, t.n0 + off, turn); }))
          break;
      }
    } else {
      while (ok && tasks.next(t)) {
        const int row = t.m0 + row_of_tile;
        const LogitsRow is(a, kForm == 1, n, row);
        if (!tile(t, [&](uint32_t from) {
              if (row - lane < up_div(n, kStepK) * kStepK)
                logits_rows<T, kForm == 1>(a, maps, n, is, from, row, t.n0 + off, turn);
            }))
          break;
      }
    }
    if (lane == 0) boxes_read<0>();
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
    if (warp >= 4 && lane == 0) boxes_stored();
    __syncthreads();
    if (warp >= 4) spoil_tiles<T, kForm>(a, n, pair, rank * kHalf + threadIdx.x % kHalf, threadIdx.x / kHalf % 2 * kHalf);
    __syncthreads();
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) sums_free_pair(sums);
}

// v += f x[0..3], at a multiple of 8 bytes; of a row's last four those past it are not used
template <typename T>
__device__ __forceinline__ void add_four(float (&v)[4], float f, const T* x) {
  const uint2 w = *(const uint2*)x;
  const T* t = (const T*)&w;
#pragma unroll
  for (int i = 0; i < 4; i++) v[i] = fmaf(f, as_float(t[i]), v[i]);
}

// Parts of a gradient's sums, in order
template <typename T>
__global__ void __launch_bounds__(256) k_head_parts(const __grid_constant__ TileArgs a) {
  follow();
  let_next();
  const HeadPlan& p = a.p;
  const GradSplit& sp = a.p.split;
  const bool hidden = blockIdx.y == 0 && sp.hidden_parts > 1;
  const int parts = hidden ? sp.hidden_parts : sp.head_parts, chunks = up_div(p.d, 4);
  const long long rows = hidden ? *p.count : p.V, room = hidden ? p.cap : sp.tokens;
  const float* from = hidden ? sp.hidden : sp.head;
  const bool again = *p.again != 0;
  const float post = again ? *p.post : 1.0f;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < rows * chunks; i += gridDim.x * 256ll) {
    const long long row = i / chunks;
    const int c = (int)(i % chunks) * 4;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < parts; k++) {
      const float4 v = *(const float4*)(from + (k * room + row) * p.ldp + c);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    const float scale = hidden && !again ? p.coef[row] : post;
    float v[4] = {s.x * scale, s.y * scale, s.z * scale, s.w * scale};
    const int end = min(4, p.d - c);
    T* to;
    if (hidden) {
      to = (T*)a.out.grad + p.to[row];
      const float f = p.at_target[row];
      if (f != 0.0f) add_four(v, f, (const T*)p.head + p.tgt[row] * p.ldw + c);
    } else {
      to = (T*)a.grad_head + row * a.grad_head_stride;
      const int4 list = p.list[row];
      for (const int q : {list.x, list.y, list.z, list.w}) {
        if (q < 0) break;
        add_four(v, p.at_target[q], (const T*)p.hc + q * p.ldh + c);
      }
    }
    float* acc = p.acc + row * p.ldp + c;
    for (int j = 0; j < end; j++) {
      float x = v[j];
      if (!hidden && (a.sum == kMiddle || a.sum == kLast)) x += acc[j];
      if (!hidden && (a.sum == kFirst || a.sum == kMiddle)) acc[j] = x;
      else to[c + j] = of_float<T>(x);
    }
  }
}

// ---------------------------------------------------------------- host

long long up_tiles(long long n) { return (n + kTile - 1) / kTile; }
// No more than there are tiles
int pairs_for(long long tiles) { return (int)std::min<long long>(kPairs, std::max(1ll, tiles)); }

template <typename T, int kForm>
epic_status launch_tiles(const HeadMaps& maps, const TileArgs& a, cudaStream_t st) {
  return launch_next(k_head_tiles<T, kForm>, 2 * a.pairs, kThreads, kShared, kShared, st, maps, a);
}

}  // namespace

GradSplit split_grads(int rows, int d, int V) {
  GradSplit s = {};
  const long long ct = (d + kTile - 1) / kTile, mt = (rows + kTile - 1) / kTile, vt = (V + (long long)kTile - 1) / kTile;
  const long long kv = (V + (long long)kStepK - 1) / kStepK, kr = (rows + kStepK - 1) / kStepK;
  s.tile_cost = 4;  // epilogue and first loads of a tile, some 2,000 clocks, in steps of 512
  s.tokens = vt * kTile;
  const long long all = mt * ct * (kv + s.tile_cost) + vt * ct * (kr + s.tile_cost), unit = std::max(8ll, all / kPairs);
  s.hidden_parts = (int)std::min<long long>(kMostParts, (kv + unit - 1) / unit);
  s.head_parts = (int)std::min<long long>(kMostParts, (kr + unit - 1) / unit);
  return s;
}

epic_status make_head_maps(HeadMaps& maps, const HeadPlan& p, int dtype, bool grads, void* grad_head, long long stride) {
  const bool bf16 = dtype == EPIC_BF16;
  if (!make_map(&maps.hc, bf16, p.hc, p.ldh, p.cap, p.ldh, 64) || !make_map(&maps.head, bf16, p.head, p.d, p.V, p.ldw, 64))
    return EPIC_ERR_CUDA;
  maps.hs = maps.e = maps.e_out = maps.grad_out = maps.hidden_parts = maps.head_parts = maps.hc;
  if (p.V == 1) stride = p.ldh;
  maps.boxes = grad_head && p.d % 8 == 0 && (uintptr_t)grad_head % 16 == 0 && stride % 8 == 0 && stride < 1ll << 38;
  if (!grads) return EPIC_OK;
  if (!make_map(&maps.e, bf16, p.e, p.lde, p.cap, p.lde, 64) || !make_map(&maps.e_out, bf16, p.e, p.lde, p.cap, p.lde, 32) ||
      (p.hs && !make_map(&maps.hs, bf16, p.hs, p.ldh, p.cap, p.ldh, 64)) ||
      (maps.boxes && !make_map(&maps.grad_out, bf16, grad_head, p.d, p.V, stride, 32)))
    return EPIC_ERR_CUDA;
  const GradSplit& s = p.split;
  if ((s.hidden_parts > 1 && !make_float_map(&maps.hidden_parts, s.hidden, p.ldp, (long long)s.hidden_parts * p.cap, p.ldp)) ||
      (s.head_parts > 1 && !make_float_map(&maps.head_parts, s.head, p.ldp, s.head_parts * s.tokens, p.ldp)))
    return EPIC_ERR_CUDA;
  return EPIC_OK;
}

epic_status launch_head_logits(const HeadPlan& p, const HeadMaps& maps, int dtype, const LogitsPass& pass, cudaStream_t st) {
  TileArgs a = {};
  a.p = p;
  a.pass = pass;
  a.bf16 = dtype == EPIC_BF16;
  a.wait = wait_limit();
  a.pairs = pairs_for(up_tiles(p.rows) * up_tiles(p.V));
  if (pass.probs) return a.bf16 ? launch_tiles<__nv_bfloat16, 1>(maps, a, st) : launch_tiles<__half, 1>(maps, a, st);
  return a.bf16 ? launch_tiles<__nv_bfloat16, 0>(maps, a, st) : launch_tiles<__half, 0>(maps, a, st);
}

epic_status launch_head_grads(const HeadPlan& p, const HeadMaps& maps, int dtype, const HiddenGrad& out, void* grad_head,
                              long long stride, HeadSum sum, cudaStream_t st) {
  TileArgs a = {};
  a.p = p;
  a.out = out;
  a.grad_head = grad_head;
  a.grad_head_stride = stride;
  a.sum = sum;
  a.bf16 = dtype == EPIC_BF16;
  a.wait = wait_limit();
  if (!out.grad) a.p.split.hidden_parts = 0;
  if (!grad_head) a.p.split.head_parts = 0;
  a.pairs = pairs_for(up_tiles(p.d) * (a.p.split.hidden_parts * up_tiles(p.rows) + a.p.split.head_parts * up_tiles(p.V)));
  const epic_status s = a.bf16 ? launch_tiles<__nv_bfloat16, 2>(maps, a, st) : launch_tiles<__half, 2>(maps, a, st);
  if (s != EPIC_OK) return s;
  const bool hidden = a.p.split.hidden_parts > 1, head = a.p.split.head_parts > 1;
  if (!hidden && !head) return EPIC_OK;
  const long long most = std::max(hidden ? (long long)p.rows : 0, head ? (long long)p.V : 0) * ((p.d + 3) / 4);
  const dim3 grid((unsigned)std::min(1216ll, (most + 255) / 256), hidden && head ? 2 : 1);
  return launch_next(a.bf16 ? k_head_parts<__nv_bfloat16> : k_head_parts<__half>, grid, 256, 0, kNoCache, st, a);
}

}  // namespace epic
