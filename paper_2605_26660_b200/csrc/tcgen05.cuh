// Thin wrappers around the sm_100a instructions the projection kernel is built from: mbarriers, tensor-map copies,
// tcgen05 matrix products with accumulators in tensor memory, clusters, and launches that overlap their predecessor.
#pragma once

#include <cuda.h>

#include "windq_internal.cuh"

namespace windq {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Every wait on a barrier ends: after about two seconds, or as soon as another wait of its thread block has given up, it
// raises *dead (a word of shared memory) and falls through.  The roles then run to their ends without issuing copies.
// Between two looks at most kLookCycles count: a context that is switched out, for however long, comes back with the time
// that it had left, and looks again first.
//
// The loop stays inside the asm block on purpose: a branch the compiler saw would make the control flow of the issuing
// warps look divergent, and with it every operand of the tcgen05 and TMA instructions, which want uniform registers; a
// product then took 70 cycles to issue, more than most of them run.  It is in line a dozen times, so it is kept short: six
// instructions more cost 48 single tokens with 32 adapters 0.9 us of 29.
constexpr unsigned kWaitCycles = 4000000000u, kLookCycles = 1u << 26;
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, uint32_t dead) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .u32 spent, last, now, d;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t"
      "@p bra DONE;\n\t"
      "mov.u32 spent, 0;\n\t"
      "mov.u32 last, %%clock;\n\t"
      "AGAIN:\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t"
      "@p bra DONE;\n\t"
      "ld.volatile.shared.u32 d, [%2];\n\t"
      "setp.ne.u32 p, d, 0;\n\t"
      "@p bra DONE;\n\t"
      "mov.u32 now, %%clock;\n\t"
      "sub.u32 d, now, last;\n\t"
      "mov.u32 last, now;\n\t"
      "min.u32 d, d, %4;\n\t"
      "add.u32 spent, spent, d;\n\t"
      "setp.lt.u32 p, spent, %3;\n\t"
      "@p bra AGAIN;\n\t"
      "st.volatile.shared.u32 [%2], 1;\n\t"
      "DONE:\n\t}" ::"r"(bar),
      "r"(parity), "r"(dead), "n"(kWaitCycles), "n"(kLookCycles)
      : "memory");
}
static_assert(kWaitCycles + (uint64_t)kLookCycles < 1ull << 32, "32-bit sums");
// After a wait has given up, by all threads of the block: lets copies and products that were issued come to their ends
// before the memory they use is given back, counts the block and tells the host.
__device__ __forceinline__ void settle(const Stalls& stalls) {
  const long long begin = clock64();
  while (clock64() - begin < 4000000) {
  }
  if (threadIdx.x == 0) {
    atomicAdd(stalls.blocks, 1ull);
    *stalls.gave_up = 1;
    __threadfence_system();
  }
}
// One lane of a converged warp, the same every time.
__device__ __forceinline__ bool elect_one() {
  uint32_t on;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(on));
  return on != 0;
}
// The warp's index, and a value all lanes agree on, in a form the compiler knows to be uniform.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Tensor-map copies into this block's shared memory; `bar` may, with PAIR, be a barrier of the other block of the pair.
template <bool PAIR>
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
// A box from shared memory into the array; what lies outside the array is not written.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
               : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>  // all but the last N groups of this thread's stores have read their shared memory
__device__ __forceinline__ void tma_store_wait() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: rows of 64 16-bit values (128 bytes), groups of 8 rows
// 1024 bytes apart.  MN-major: blocks of 64 values along M or N, `block` bytes apart, each [k][64], 8 k 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t block) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)((block >> 4) & 0x3fff) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor of kind::f16 with binary32 accumulation; type 0 = fp16, 1 = bf16 for both operands.
__host__ __device__ inline uint32_t instr_desc(int type, bool a_mn, bool b_mn, int m, int n) {
  return 1u << 4 | (uint32_t)type << 7 | (uint32_t)type << 10 | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 |
         (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

// PAIR: the two thread blocks of a cluster whose ranks differ in the last bit work on one product; the even one issues it.
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {  // one whole warp (of both blocks)
  if (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
  if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// Arrives on `bar` when the products issued so far are done: of this block, or (PAIR) at this offset in the blocks of `mask`.
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint32_t bar, uint32_t mask) {
  if (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)mask)
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 lanes x 16 columns of binary32 accumulators, one lane a thread.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's window, of this block's shared address in the block of that rank.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
  return remote;
}
__device__ __forceinline__ void cluster_arrive(uint32_t remote_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote_bar) : "memory");
}
// Sums over the blocks of a cluster, in the order of their ranks: `U` quads of binary32 values, at base + offset[u] in each
// of n (a power of two, at most 8) blocks of ranks first, first + stride, ...  Distributed shared memory answers after the
// better part of a microsecond, so the loads of several blocks are in flight together.
template <int U>
__device__ __forceinline__ void cluster_sum(uint32_t base, const uint32_t (&offset)[U], int n, int first, int stride, float4 (&x)[U]) {
  constexpr int Q = U >= 4 ? 4 : 8;
#pragma unroll
  for (int u = 0; u < U; u++) x[u] = make_float4(0, 0, 0, 0);
  for (int q0 = 0; q0 < n; q0 += Q) {
    float4 y[Q][U];
#pragma unroll
    for (int q = 0; q < Q; q++) {
      if (q0 + q < n) {
        const uint32_t from = cluster_addr(base, first + (q0 + q) * stride);
#pragma unroll
        for (int u = 0; u < U; u++)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(y[q][u].x), "=f"(y[q][u].y), "=f"(y[q][u].z), "=f"(y[q][u].w)
                       : "r"(from + offset[u]));
      }
    }
#pragma unroll
    for (int q = 0; q < Q; q++) {
      if (q0 + q < n) {
#pragma unroll
        for (int u = 0; u < U; u++) x[u].x += y[q][u].x, x[u].y += y[q][u].y, x[u].z += y[q][u].z, x[u].w += y[q][u].w;
      }
    }
  }
}

// Programmatic dependent launch: the kernel may start before its predecessor in the stream has ended; it waits here
// before it reads what the predecessor writes.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }


using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return (EncodeTiled)p;
  }();
  return fn;
}

// A row-major array of 16-bit values [planes][rows][inner], copied in boxes of box_rows x 64 with the 128-byte swizzle;
// what lies outside the array reads as zero.
inline bool make_map(CUtensorMap* map, int dtype, const void* base, int64_t inner, int64_t rows, int64_t planes, int64_t row_stride,
              int64_t plane_stride, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)(2 * row_stride), (cuuint64_t)(2 * plane_stride)};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
  return encode_tiled()(map, dtype == WINDQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                        planes > 0 ? 3 : 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace windq
