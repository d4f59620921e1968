// Tensor-core tiles of two CTAs: barriers in shared memory, copies of boxes of
// tensors (TMA), products into tensor memory (tcgen05), for kernels that compute
// tiles of 256 x 256 by pairs of CTAs.
//
// Every wait gives up after a limit, in clocks; a limit of 0 is up before the first one.
// A thread whose wait gave up tells both CTAs of its pair and leaves its loops; when all
// threads of the pair have left theirs, what is in flight has time to end, the pair writes
// NaN to all that it was to write, and tensor memory is freed.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include <algorithm>

namespace epic {
namespace {

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// the thread's warp, known to be the same in all its lanes
__device__ __forceinline__ int warp_of_thread() { return __shfl_sync(~0u, threadIdx.x / 32, 0); }
// true in one lane of a whole warp.  Products are issued so, from loops that the warp goes through together: their operands
// then are in uniform registers (from one lane's loop a step of four products took 560 clocks to issue).
__device__ __forceinline__ bool one_lane() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p;
}
// the same place in the shared memory of the cluster's CTA `rank`
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_visible() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// of a barrier in any CTA of the cluster.  What it orders is in shared memory and told to the tensor units by a proxy fence,
// or in tensor memory and fenced by tcgen05.fence: a release to the whole cluster would wait for much more.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done;
}
// false: gave up
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, long long limit) {
  if (bar_try(bar, parity)) return true;
  const long long t = clock64();
  while (!bar_try(bar, parity))
    if (clock64() - t > limit) return false;
  return true;
}
// The lanes of a warp that wait together go on or give up as one: their clocks need not agree on a wait that ends near the limit,
// and elections, loads and stores of tensor memory want all of them.
__device__ __forceinline__ bool all_came(bool ok) { return __all_sync(~0u, ok); }
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, long long limit) {
  if (all_came(bar_try(bar, parity))) return true;
  const long long t = clock64();
  do {
    if (all_came(bar_try(bar, parity))) return true;
  } while (!__any_sync(~0u, clock64() - t > limit));
  return false;
}

// A box of a tensor in two dimensions at (x, y) into this CTA's shared memory; its bytes are counted at `bar`, which may be
// the pair's other CTA's.
__device__ __forceinline__ void load_box_pair(const CUtensorMap* map, uint32_t dst, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::
          "r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
// the same, counted in this CTA
__device__ __forceinline__ void load_box(const CUtensorMap* map, uint32_t dst, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
// A box from shared memory to (x, y), x and y not negative; rows past the tensor's end are left out, and columns
// but for those that begin in the last one's 16 bytes.
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(from), "r"(x), "r"(y)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// the thread's stores have read their boxes, but for the last kLeft
template <int kLeft>
__device__ __forceinline__ void boxes_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory");
}
// the thread's stores are done
__device__ __forceinline__ void boxes_stored() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void shared_to_boxes() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- operands in shared memory: rows of 128 bytes, their chunks of 16 swizzled by the row's number in 8

constexpr uint64_t kSwizzle128 = (uint64_t)2 << 61 | (uint64_t)1 << 46;
// [rows][64 elements] along the product's sum: the next 8 rows are 1,024 bytes on; 16 elements of the sum, 32 bytes
__device__ __forceinline__ uint64_t operand_k(uint32_t addr) {
  return kSwizzle128 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 16 | (addr >> 4 & 0x3fff);
}
constexpr uint32_t kNextK = 32 >> 4;
// [64 of the sum][64 elements] blocks across the sum: the next 8 of the sum are 1,024 bytes on, the next block 8,192; 16 of
// the sum, 2,048 bytes
__device__ __forceinline__ uint64_t operand_mn(uint32_t addr) {
  return kSwizzle128 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)(8192 >> 4) << 16 | (addr >> 4 & 0x3fff);
}
constexpr uint32_t kNextMN = 2048 >> 4;

// What a product is: 16-bit operands (bf16 or fp16) along or across the sum, 32-bit sums, m x n
__host__ __device__ constexpr uint32_t product_kind(bool bf16, bool a_across, bool b_across, int m, int n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u) |
         (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

__device__ __forceinline__ void product_pair(uint32_t sums, uint64_t a, uint64_t b, uint32_t kind, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(sums),
      "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
      : "memory");
}
// the same with the first operand in tensor memory: a lane a row, 16 of the sum in 8 columns
__device__ __forceinline__ void product_pair_in(uint32_t sums, uint32_t a, uint64_t b, uint32_t kind, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(sums),
      "r"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
      : "memory");
}
// an arrival at that barrier of both CTAs once all products so far are done
__device__ __forceinline__ void products_arrive_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"((uint16_t)3)
               : "memory");
}

// all of tensor memory, by one warp of each CTA of the pair
__device__ __forceinline__ void sums_take_pair(uint32_t dst) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(dst) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void sums_free_pair(uint32_t sums) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(sums) : "memory");
}
__device__ __forceinline__ void products_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void products_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// columns of the warp's 32 rows, a lane a row; there after sums_loaded(v)
__device__ __forceinline__ void sums_load(uint32_t sums, float (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
      : "r"(sums));
}
__device__ __forceinline__ void sums_loaded(float (&v)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7])::"memory");
}
__device__ __forceinline__ void sums_load(uint32_t sums, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(sums));
}
__device__ __forceinline__ void sums_loaded(float (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])::"memory");
}
__device__ __forceinline__ void sums_load(uint32_t sums, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(sums));
}
__device__ __forceinline__ void sums_loaded(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])::"memory");
}

// 16 columns of the warp's 32 lanes; there after operand_stored()
__device__ __forceinline__ void operand_store(uint32_t to, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(to),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void operand_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A thread's wait gave up: noted in `flag` of both CTAs, which the pair's next barrier makes known
__device__ __forceinline__ void give_up(uint32_t flag) {
  for (uint32_t r = 0; r < 2; r++) asm volatile("st.shared::cluster.u32 [%0], 1;" ::"r"(at_rank(flag, r)) : "memory");
}
// a microsecond's worth of waiting for copies and products in flight, many times over: after a wait that gave up, when no thread
// of the pair starts others
__device__ __noinline__ void let_all_end() {
  for (int i = 0; i < 2000; i++) __nanosleep(1000);
}

// ---- on the host

// EPIC_HEAD_WAIT_MS [4000] in clocks of some 2.1 GHz
inline long long wait_limit() {
  const char* e = getenv("EPIC_HEAD_WAIT_MS");
  char* end = nullptr;
  const long long ms = e ? strtoll(e, &end, 10) : 0;
  return (e && end != e ? std::min(std::max(ms, 0ll), 1ll << 31) : 4000) * 2100000;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      return (EncodeTiled)nullptr;
    return (EncodeTiled)p;
  }();
  return f;
}

// [rows][cols] of bytes, `ld` apart: boxes of 64 columns and `box` rows, chunks of 16 swizzled by the row's number / 2 in 4
inline bool make_byte_map(CUtensorMap* map, const void* base, long long cols, long long rows, long long ld, int box) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld};
  const cuuint32_t part[2] = {64, (cuuint32_t)box}, step[2] = {1, 1};
  return encode_tiled() &&
         encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)base, size, stride, part, step,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// [rows][cols] of 32-bit floats, `ld` apart: boxes of 32 columns and 32 rows
inline bool make_float_map(CUtensorMap* map, const void* base, long long cols, long long rows, long long ld) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld * 4};
  const cuuint32_t part[2] = {32, 32}, step[2] = {1, 1};
  return encode_tiled() &&
         encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, (void*)base, size, stride, part, step,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// [rows][cols] of 16-bit elements, `ld` apart: boxes of 64 columns and `box` rows
inline bool make_map(CUtensorMap* map, bool bf16, const void* base, long long cols, long long rows, long long ld, int box) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t part[2] = {64, (cuuint32_t)box}, step[2] = {1, 1};
  return encode_tiled() &&
         encode_tiled()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                        (void*)base, size, stride, part, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace epic
