// The matrix products of the head's loss, on the tensor units: logits = h W^T,
// gradients dh = e W and dW = e^T hs.
//
// A tile of 256 x 256 is a pair of CTAs': each copies 128 rows of both operands in steps of 64 of the sum (TMA, six steps
// ahead), one thread of the pair issues the products, sums lie in tensor memory, twice, so that eight warps a CTA work on
// one tile's sums while the next tile's are made.  Operands are read as they lie: e along and across its rows, the head by
// tokens and by hidden dimensions.
#include <cuda.h>

#include <algorithm>

#include "head_loss.h"
#include "head_rows.cuh"
#include "tensor_tiles.cuh"

namespace epic {
namespace {

constexpr int kTile = 256, kHalf = 128;  // a pair's tile, a CTA's share of an operand
constexpr int kStepK = 64, kStages = 6;
constexpr int kOperand = kHalf * kStepK * 2, kStage = 2 * kOperand;  // bytes
constexpr int kWorkWarps = 8, kThreads = 128 + 32 * kWorkWarps;
constexpr int kPairs = 76;  // of the GB300's 152 SMs
constexpr int kTurnRow = 34;  // 16-bit elements from row to row of a warp's turning buffer
constexpr int kTurn = 32 * kTurnRow * 2;
constexpr int kShared = kStages * kStage + kWorkWarps * kTurn + 1024;

struct Bars {
  uint64_t full[kStages], empty[kStages], sums_full[2], sums_empty[2];
  uint32_t sums;
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
};

struct Maps {
  CUtensorMap hc, hc_mn, hs, head_k, head_mn, e_k, e_mn;
};

__device__ __forceinline__ int up_div(int a, int b) { return (a + b - 1) / b; }

// The i-th tile of pair `pair`, or false.  Logits: the rows' tiles of one column of tiles after another, so that the head is
// read once.
__device__ __forceinline__ bool logits_task(const TileArgs& a, int n, int pair, int i, Task& t) {
  const int mt = up_div(n, kTile), at = pair + i * kPairs;
  if (at >= mt * up_div(a.p.V, kTile)) return false;
  t = {at % mt * kTile, at / mt * kTile, 0, up_div(a.p.d, kStepK), 0, 0};
  return true;
}

// Gradients: first all tiles of hidden states' (long sums), then the head's.  Where the former do not come out even, the
// pairs without a last one take as many of the latter as it is worth before the rest is dealt to all.
__device__ __forceinline__ bool grads_task(const TileArgs& a, int n, int pair, int i, Task& t) {
  const GradSplit& s = a.p.split;
  const int ct = up_div(a.p.d, kTile);
  const int mt = up_div(n, kTile), vt = up_div(a.p.V, kTile);
  const int hidden = s.hidden_parts * mt * ct, head = s.head_parts * vt * ct;
  const int own = hidden / kPairs + (pair < hidden % kPairs);
  if (i < own) {
    const int at = pair + i * kPairs, part = at / (mt * ct), tile = at % (mt * ct);
    const int all = up_div(a.p.V, kStepK), k0 = (int)((long long)all * part / s.hidden_parts);
    t = {tile / ct * kTile, tile % ct * kTile, k0, (int)((long long)all * (part + 1) / s.hidden_parts) - k0, 0, part};
    return true;
  }
  i -= own;
  const int all = up_div(n, kStepK), last = hidden % kPairs, idle = last ? kPairs - last : 0;
  int at;
  const int per = up_div(all, max(1, s.head_parts)) + s.tile_cost;
  const int first = idle ? min(head / idle, (up_div(up_div(a.p.V, kStepK), s.hidden_parts) + s.tile_cost) / per) : 0;
  if (pair >= last && idle) {
    if (i < first) at = pair - last + i * idle;
    else at = first * idle + pair + (i - first) * kPairs;
  } else {
    at = first * idle + pair + i * kPairs;
  }
  if (at >= head) return false;
  const int part = at / (vt * ct), tile = at % (vt * ct), k0 = (int)((long long)all * part / s.head_parts);
  t = {tile / ct * kTile, tile % ct * kTile, k0, (int)((long long)all * (part + 1) / s.head_parts) - k0, 1, part};
  return true;
}

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

// 32 bytes at a multiple of 32
__device__ __forceinline__ void store_sector(void* to, const uint32_t (&v)[16], int at) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[at]), "r"(v[at + 1]), "r"(v[at + 2]),
               "r"(v[at + 3]), "r"(v[at + 4]), "r"(v[at + 5]), "r"(v[at + 6]), "r"(v[at + 7])
               : "memory");
}

// 32 elements of each lane's row to `to` (NULL: none), of which the first `count` exist (the same in all lanes).  Rows that
// start at any element are turned in shared memory, so that lanes write one row's elements: half a warp a row, two elements a
// lane from the row's first multiple of 4 bytes on.  The loop has no branches but predicates: waits for one row's
// elements are no waits for the next's.
template <typename T>
__device__ __forceinline__ void store_rows(T* to, const float (&v)[32], int count, bool whole, uint16_t* turn, int lane) {
  uint32_t w[16];
#pragma unroll
  for (int j = 0; j < 16; j++) w[j] = pack2<T>(v[2 * j], v[2 * j + 1]);
  if (whole && count >= 32) {
    if (to) {
      store_sector(to, w, 0);
      store_sector(to + 16, w, 8);
    }
    return;
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 16; j++) ((uint32_t*)(turn + lane * kTurnRow))[j] = w[j];
  __syncwarp();
  const int at = lane % 16;
  count = min(count, 32);
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += 8) {
    uint16_t* row[4];
    uint32_t two[4];
    int j[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = r0 + 2 * i + lane / 16;
      row[i] = (uint16_t*)__shfl_sync(~0u, (unsigned long long)to, r);
      j[i] = 2 * at + (int)((uintptr_t)row[i] / 2 % 2);
      two[i] = turn[r * kTurnRow + j[i]] | (uint32_t)turn[r * kTurnRow + j[i] + 1] << 16;
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (row[i] && j[i] + 1 < count) *(uint32_t*)(row[i] + j[i]) = two[i];
      if (row[i] && j[i] + 1 == count) row[i][j[i]] = (uint16_t)two[i];
      if (row[i] && j[i] == 1) row[i][0] = turn[(r0 + 2 * i + lane / 16) * kTurnRow];
    }
  }
}

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

// Logits of one row, kRecCols columns from `sums`: the record, and with `probs` the exponentials.  z is only ever in registers.
template <typename T, bool kProbs>
__device__ __forceinline__ void logits_rows(const TileArgs& a, int n, uint32_t sums, int row, int col, int lane) {
  const HeadPlan& p = a.p;
  const bool real = row < n;
  const int y = real ? p.tgt[row] - col : -1;
  const bool known = a.pass.known;
  const float ref = !kProbs || !real ? 0.0f : known ? p.known_ref[row] : p.ref[row];
  const float mul = kProbs && real && known ? p.known_mul[row] : 1.0f;
  const float at = kProbs && real && a.pass.only_again ? p.known_at[row] : 0.0f;
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
    float zt = 0.0f;
    const bool target = here >= 0 && here < 32;
    if (target) {
#pragma unroll
      for (int j = 0; j < 32; j++)
        if (j == here) zt = z[j], z[j] = -CUDART_INF_F;
      if (a.pass.sums) p.zt[row] = zt;
    }
    if (kProbs) {
#pragma unroll
      for (int j = 0; j < 32; j++) z[j] = ex2(fmaf(z[j], kLog2E, -ref)) * mul;
      s += sum32(z);
      if (target) {
        const float e = a.pass.only_again ? at : ex2(fmaf(zt, kLog2E, -ref)) * mul;
#pragma unroll
        for (int j = 0; j < 32; j++)
          if (j == here) z[j] = e;
      }
      if (row < up_div(n, kStepK) * kStepK) {
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 16; j++) w[j] = real ? pack2<T>(z[2 * j], z[2 * j + 1]) : 0u;
        T* e = (T*)p.e + (long long)row * p.lde + col + c;
        store_sector(e, w, 0);
        store_sector(e + 16, w, 8);
      }
    } else {
      const float top = whole_ref(max32(z));
#pragma unroll
      for (int j = 0; j < 32; j++) z[j] = ex2(fmaf(z[j], kLog2E, -top));
      meet(to, s, top, sum32(z));
    }
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

template <typename T>
__device__ __forceinline__ void store_part(float* part, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) ((float4*)part)[j / 4] = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
}

// Sums of a gradient's tile: kHalf columns of each lane's row, two loads of 32 at a time
template <typename T>
__device__ __forceinline__ void grad_rows(const TileArgs& a, int n, bool again, float post, const Task& t, uint32_t sums,
                                          int row, int col, uint16_t* turn, int lane) {
  const HeadPlan& p = a.p;
  const GradSplit& sp = a.p.split;
  const bool hidden = t.job == 0;
  const bool parts = (hidden ? sp.hidden_parts : sp.head_parts) > 1;
  const bool there = row < (hidden ? n : p.V);
  T* to = nullptr;
  float scale = post;
  if (there && !parts) {
    if (hidden) {
      const long long r = a.out.r0 + p.src[row];
      to = (T*)a.out.grad + (r / a.out.n) * a.out.stride_b + (r % a.out.n) * a.out.stride_n;
      if (!again) scale = p.coef[row];
    } else {
      to = (T*)a.grad_head + row * a.grad_head_stride;
    }
  }
  const bool whole = __all_sync(~0u, ((uintptr_t)(to + col) & 31) == 0 || !to);
  float* part = hidden ? sp.hidden + ((long long)t.part * p.cap + row) * p.ldp : sp.head + ((long long)t.part * p.V + row) * p.ldp;
  float* acc = p.acc + (long long)row * p.ldp;
  auto store = [&](float(&v)[32], int c) {
    if (c >= p.d) return;
    if (t.steps <= 0) {
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] = 0.0f;
    }
    if (parts) {
      if (there) store_part<T>(part + c, v);
      return;
    }
    if (hidden || post != 1.0f) {
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] *= scale;
    }
    if (!hidden && a.sum != kOnly && there) {
      if (a.sum != kFirst) {
#pragma unroll
        for (int j = 0; j < 32; j++) v[j] += acc[c + j];
      }
      if (a.sum != kLast) store_part<T>(acc + c, v);
    }
    if (hidden || a.sum == kOnly || a.sum == kLast) store_rows<T>(to ? to + c : nullptr, v, p.d - c, whole, turn, lane);
  };
#pragma unroll 1
  for (int c = col; c < col + kHalf && c < p.d; c += 64) {
    float v[32], w[32];
    if (t.steps > 0) {
      sums_load(sums + (c - col), v);
      sums_load(sums + (c - col) + 32, w);
      sums_loaded(v);
      sums_loaded(w);
    }
    store(v, c);
    store(w, c + 32);
  }
}

// kForm 0: records; 1: exponentials (and records); 2: gradients
template <typename T, int kForm>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_head_tiles(const __grid_constant__ Maps maps, const __grid_constant__ TileArgs a) {
  extern __shared__ uint8_t shared_raw[];
  __shared__ Bars bars;
  const bool again = *a.p.again != 0;
  if (kForm != 2 && a.pass.only_again && !again) return;
  const int n = *a.p.count;
  uint8_t* shared = (uint8_t*)(((uintptr_t)shared_raw + 1023) / 1024 * 1024);
  const uint32_t stages = smem_address(shared);
  uint16_t* turns = (uint16_t*)(shared + kStages * kStage);
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
    bar_init_visible();
  }
  if (warp == 1) sums_take_pair(smem_address(&bars.sums));
  products_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  const uint32_t sums = bars.sums;

  auto task = [&](int i, Task& t) {
    return kForm == 2 ? grads_task(a, n, pair, i, t) : logits_task(a, n, pair, i, t);
  };
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {  // copies
      const uint32_t full0 = at_rank(full, 0);
      int s = 0;
      uint32_t turn = 0;
      Task t;
      for (int i = 0; ok && task(i, t); i++) {
        const int m = t.m0 + rank * kHalf, c = t.n0 + rank * kHalf;
        for (int k = t.k0; k < t.k0 + t.steps; k++) {
          if (!(ok = bar_wait(empty + 8 * s, turn ^ 1))) break;
          if (rank == 0) bar_expect(full + 8 * s, 2 * kStage);
          const uint32_t A = stages + s * kStage, B = A + kOperand, bar = full0 + 8 * s;
          if (kForm != 2) {
            load_box_pair(&maps.hc, A, bar, k * kStepK, m);
            load_box_pair(&maps.head_k, B, bar, k * kStepK, c);
          } else if (t.job == 0) {
            load_box_pair(&maps.e_k, A, bar, k * kStepK, m);
            load_box_pair(&maps.head_mn, B, bar, c, k * kStepK);
            load_box_pair(&maps.head_mn, B + kOperand / 2, bar, c + 64, k * kStepK);
          } else {
            load_box_pair(&maps.e_mn, A, bar, m, k * kStepK);
            load_box_pair(&maps.e_mn, A + kOperand / 2, bar, m + 64, k * kStepK);
            const CUtensorMap* h = again ? &maps.hc_mn : &maps.hs;
            load_box_pair(h, B, bar, c, k * kStepK);
            load_box_pair(h, B + kOperand / 2, bar, c + 64, k * kStepK);
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
      for (int i = 0; ok && task(i, t); i++) {
        if (t.steps <= 0) continue;
        const int half = use & 1;
        if (!(ok = bar_wait(sums_empty + 8 * half, (use >> 1 & 1) ^ 1))) break;
        products_fence_after();
        const bool a_across = kForm == 2 && t.job == 1, b_across = kForm == 2;
        const uint32_t kind = product_kind(a.bf16, a_across, b_across, kTile, kTile);
        const uint32_t to = sums + half * kTile;
        for (int k = 0; k < t.steps; k++) {
          if (!(ok = bar_wait(full + 8 * s, turn))) break;
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
  } else if (warp >= 4) {
    const int part = warp - 4, quarter = warp % 4;
    uint16_t* turn = turns + part * 32 * kTurnRow;
    const float post = kForm == 2 && again ? *a.p.post : 1.0f;
    int use = 0;
    Task t;
    for (int i = 0; task(i, t); i++) {
      const int half = use & 1;
      const int row = t.m0 + rank * kHalf + quarter * 32 + lane, off = part / 4 * kHalf;
      const uint32_t from = sums + half * kTile + off + ((uint32_t)quarter * 32 << 16);
      if (t.steps > 0) {
        if (!(ok = bar_wait(sums_full + 8 * half, use >> 1 & 1))) break;
        products_fence_after();
      }
      if (kForm == 2) {
        grad_rows<T>(a, n, again, post, t, from, row, t.n0 + off, turn, lane);
      } else if (row - lane < up_div(n, kStepK) * kStepK) {
        logits_rows<T, kForm == 1>(a, n, from, row, t.n0 + off, lane);
      }
      if (t.steps > 0) {
        products_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(at_rank(sums_empty + 8 * half, 0));
        use++;
      }
    }
  }
  if (!ok) {
    *a.p.failed = 1;
    let_copies_land();
  }
  products_fence_before();
  __syncwarp();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  products_fence_after();
  if (warp == 1) sums_free_pair(sums);
}

// Parts of a gradient's sums, in order
template <typename T>
__global__ void __launch_bounds__(256) k_head_parts(const __grid_constant__ TileArgs a) {
  const HeadPlan& p = a.p;
  const GradSplit& sp = a.p.split;
  const bool hidden = blockIdx.y == 0 && sp.hidden_parts > 1;
  const int parts = hidden ? sp.hidden_parts : sp.head_parts, chunks = up_div(p.d, 4);
  const long long rows = hidden ? *p.count : p.V, room = hidden ? p.cap : p.V;
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
    float v[4] = {s.x, s.y, s.z, s.w};
    T* to;
    if (hidden) {
      const long long r = a.out.r0 + p.src[row];
      to = (T*)a.out.grad + (r / a.out.n) * a.out.stride_b + (r % a.out.n) * a.out.stride_n;
    } else {
      to = (T*)a.grad_head + row * a.grad_head_stride;
    }
    const float scale = hidden && !again ? p.coef[row] : post;
    float* acc = p.acc + row * p.ldp + c;
    for (int j = 0; j < 4 && c + j < p.d; j++) {
      float x = v[j] * scale;
      if (!hidden && (a.sum == kMiddle || a.sum == kLast)) x += acc[j];
      if (!hidden && (a.sum == kFirst || a.sum == kMiddle)) acc[j] = x;
      else to[c + j] = of_float<T>(x);
    }
  }
}

// ---------------------------------------------------------------- host

epic_status launched() { return cudaGetLastError() == cudaSuccess ? EPIC_OK : EPIC_ERR_CUDA; }

template <typename T, int kForm>
epic_status launch_tiles(const Maps& maps, const TileArgs& a, cudaStream_t st) {
  if (cudaFuncSetAttribute(k_head_tiles<T, kForm>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared) != cudaSuccess)
    return cudaGetLastError(), EPIC_ERR_CUDA;
  k_head_tiles<T, kForm><<<2 * kPairs, kThreads, kShared, st>>>(maps, a);
  return launched();
}

}  // namespace

GradSplit split_grads(int rows, int d, int V) {
  GradSplit s = {};
  const long long ct = (d + kTile - 1) / kTile, mt = (rows + kTile - 1) / kTile, vt = (V + (long long)kTile - 1) / kTile;
  const long long kv = (V + (long long)kStepK - 1) / kStepK, kr = (rows + kStepK - 1) / kStepK;
  s.tile_cost = 4;
  const long long all = mt * ct * (kv + s.tile_cost) + vt * ct * (kr + s.tile_cost), unit = std::max(8ll, all / (3 * kPairs));
  s.hidden_parts = (int)std::min<long long>(kMostParts, (kv + unit - 1) / unit);
  s.head_parts = (int)std::min<long long>(kMostParts, (kr + unit - 1) / unit);
  return s;
}

epic_status launch_head_logits(const HeadPlan& p, int dtype, const LogitsPass& pass, cudaStream_t st) {
  Maps maps = {};
  TileArgs a = {};
  a.p = p;
  a.pass = pass;
  a.bf16 = dtype == EPIC_BF16;
  if (!make_map(&maps.hc, a.bf16, p.hc, p.ldh, p.cap, p.ldh, kHalf) ||
      !make_map(&maps.head_k, a.bf16, p.head, p.d, p.V, p.ldw, kHalf))
    return EPIC_ERR_CUDA;
  if (pass.probs) return dtype == EPIC_F16 ? launch_tiles<__half, 1>(maps, a, st) : launch_tiles<__nv_bfloat16, 1>(maps, a, st);
  return dtype == EPIC_F16 ? launch_tiles<__half, 0>(maps, a, st) : launch_tiles<__nv_bfloat16, 0>(maps, a, st);
}

epic_status launch_head_grads(const HeadPlan& p, int dtype, const HiddenGrad& out, void* grad_head, long long stride,
                              HeadSum sum, cudaStream_t st) {
  Maps maps = {};
  TileArgs a = {};
  a.p = p;
  a.out = out;
  a.grad_head = grad_head;
  a.grad_head_stride = stride;
  a.sum = sum;
  a.bf16 = dtype == EPIC_BF16;
  if (!out.grad) a.p.split.hidden_parts = 0;
  if (!grad_head) a.p.split.head_parts = 0;
  if (!make_map(&maps.hc_mn, a.bf16, p.hc, p.ldh, p.cap, p.ldh, 64) ||
      !make_map(&maps.hs, a.bf16, p.hs ? p.hs : p.hc, p.ldh, p.cap, p.ldh, 64) || !make_map(&maps.e_k, a.bf16, p.e, p.lde, p.cap, p.lde, kHalf) ||
      !make_map(&maps.e_mn, a.bf16, p.e, p.lde, p.cap, p.lde, 64) ||
      !make_map(&maps.head_mn, a.bf16, p.head, p.d, p.V, p.ldw, 64))
    return EPIC_ERR_CUDA;
  const epic_status s = dtype == EPIC_F16 ? launch_tiles<__half, 2>(maps, a, st) : launch_tiles<__nv_bfloat16, 2>(maps, a, st);
  if (s != EPIC_OK) return s;
  const bool hidden = a.p.split.hidden_parts > 1, head = a.p.split.head_parts > 1;
  if (!hidden && !head) return EPIC_OK;
  const long long most = std::max(hidden ? (long long)p.rows : 0, head ? (long long)p.V : 0) * ((p.d + 3) / 4);
  const dim3 grid((unsigned)std::min(1216ll, (most + 255) / 256), hidden && head ? 2 : 1);
  if (dtype == EPIC_F16) k_head_parts<__half><<<grid, 256, 0, st>>>(a);
  else k_head_parts<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
  return launched();
}

}  // namespace epic
