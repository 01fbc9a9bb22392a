// Gradients of the two weights of a gated block: dWg = dG^T X, dWu = dU^T X, on the tensor cores (tcgen05, accumulators in tensor
// memory, operands by TMA).  Both operands are transposed: K is the tokens, which are the rows of D (see
// ProductKind) and of X; where D has two terms, X goes by twice.
//
// A tile is 256 rows (outputs of the block) x up to 256 columns (channels) on a pair of thread blocks (cta_group::2: each holds half
// of either operand); persistent over tiles with two accumulators, so that storing a tile overlaps the next.  Warps: one issues TMA
// copies, one issues matrix products, eight read the accumulators and store (with four, storing took longer than the products of a
// short K: 333 tokens x 8191 x 2048 30 us, now 27).  Bound by power for a long K, by writing the gradients for a short one (HBM takes
// 3.9 TB/s of pure writes).
//
// Where the tiles do not fill the GPU, `splits` pairs (a cluster) share a tile along K and add their accumulators through
// distributed shared memory, in rank order: equal calls give equal bits.
#include <algorithm>

#include "feed_forward.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kStorers = 8;  // warps
constexpr int kThreads = 64 + 32 * kStorers;
constexpr int kMaxStages = 8;
constexpr int kSmemLimit = 227 * 1024 - 2048;  // dynamic shared memory of one thread block per SM
constexpr int kPitch = 260;                    // sums of a split tile, 32 bits each, rows free of bank conflicts
constexpr int kStaging = kStorers * 4096;      // a box of 32 rows x 64 columns each
constexpr int kABytes = 2 * 8192;              // of a stage: 128 rows x 64 tokens

struct Args {
  int F, N, dtype;
  int chunks, token_chunks;       // of K (64 tokens each, once a term of D); of the tokens
  int block_cols;                 // columns of a thread block's half
  int row_tiles, col_tiles, group;
  int half_tiles, half;           // row tiles of the first gradient, columns of each half of [dG | dU]
  int splits, stages, accumulators, columns;  // columns: of tensor memory
  const uint32_t* top;
  void* O[2];
  int64_t ldo;
  Stalls stalls;
};

struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], done[2], free[2];
};

// Tiles in an order that keeps a group of row tiles in L2 while the columns stream by.
__device__ __forceinline__ void tile_at(const Args& p, int tile, int& rt, int& ct) {
  const int per = p.group * p.col_tiles, g = tile / per, rest = tile - g * per;
  const int rows = min(p.group, p.row_tiles - g * p.group);
  ct = rest / rows;
  rt = g * p.group + rest - ct * rows;
}

// Adds the sums of a tile's splits, which lie as [row][column] in the shared memory of their blocks, and stores this block's
// share of the rows: those of local index split, split + splits, ...
__device__ __forceinline__ void join(const Args& p, uint32_t base, int rt, int ct, int split, int me) {
  constexpr int U = 4;
  const int quads = p.block_cols / 2;
  const bool second = rt >= p.half_tiles;
  if (second) rt -= p.half_tiles;
  const int m0 = (rt * 2 + me) * 128, n0 = ct * 2 * p.block_cols;
  const int items = max(0, (min(128, p.F - m0) - split + p.splits - 1) / p.splits) * quads;
  const float unscale = p.top ? gradient_power(*p.top, -1) : 1.0f;
  for (int i = threadIdx.x; i < items; i += U * kThreads) {
    uint32_t offset[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int q = min(i + u * kThreads, items - 1);
      offset[u] = (uint32_t)((split + q / quads * p.splits) * kPitch + q % quads * 4) * 4;
    }
    cluster_sum<U>(base, offset, p.splits, me, 2, x);
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int q = i + u * kThreads, m = m0 + split + q / quads * p.splits, n = n0 + q % quads * 4;
      if (q >= items || n >= p.N) continue;
      const float v[4] = {x[u].x * unscale, x[u].y * unscale, x[u].z * unscale, x[u].w * unscale};
      uint16_t* out = static_cast<uint16_t*>(p.O[second]) + m * p.ldo + n;
      if (n + 4 <= p.N) {
        *reinterpret_cast<uint2*>(out) = make_uint2(pack2(v[0], v[1], p.dtype), pack2(v[2], v[3], p.dtype));
      } else {
#pragma unroll
        for (int k = 0; k < 4; k++)
          if (n + k < p.N) store1(out, k, p.dtype, v[k]);
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads, 1)
    weight_gradient_kernel(const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap,
                           const __grid_constant__ CUtensorMap omap0, const __grid_constant__ CUtensorMap omap1,
                           const __grid_constant__ Args p) {
  extern __shared__ uint8_t raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank(), me = rank & 1, leader = rank & ~1u;
  const int b_boxes = (p.block_cols + 63) / 64;
  const uint32_t stage_bytes = kABytes + b_boxes * 8192;
  const uint32_t dead_ = smem_addr(&dead);
  auto full = [&](int s) { return smem_addr(&bars.full[s]); };
  auto empty = [&](int s) { return smem_addr(&bars.empty[s]); };
  auto done = [&](int b) { return smem_addr(&bars.done[b]); };
  auto free_ = [&](int b) { return smem_addr(&bars.free[b]); };

  if (threadIdx.x == 0) {
    prefetch_map(&amap);
    prefetch_map(&bmap);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int b = 0; b < 2; b++) {
      mbar_init(done(b), 1);
      mbar_init(free_(b), 2 * kStorers);
    }
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<true>(smem_addr(&tmem_slot), p.columns);
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the other block's barriers are ready
  tc_fence_after();
  launch_dependents();  // tensor memory is in hand
  wait_for_predecessor();
  const uint32_t tmem = tmem_slot;

  const int team = 2 * p.splits;  // thread blocks of a tile
  const int split = (blockIdx.x % team) / 2, step = gridDim.x / team, tiles = p.row_tiles * p.col_tiles;
  const int c0 = (int)((int64_t)p.chunks * split / p.splits), c1 = (int)((int64_t)p.chunks * (split + 1) / p.splits);

  if (warp == 0) {
    Ring at(p.stages);
    const uint32_t to = cluster_addr(full(0), leader);  // barriers of the issuing block
    for (int tile = blockIdx.x / team; tile < tiles; tile += step) {
      int rt, ct;
      tile_at(p, tile, rt, ct);
      const int m0 = (rt < p.half_tiles ? rt * 256 : p.half + (rt - p.half_tiles) * 256) + me * 128, n0 = (ct * 2 + me) * p.block_cols;
      for (int c = c0; c < c1; c++) {
        mbar_wait(empty(at.s), at.phase ^ 1, dead_);
        const uint32_t dst = base + at.s * stage_bytes, bar = to + at.s * 8;
        if (elect_one() && !*(volatile int*)&dead) {
          if (me == 0) mbar_expect(full(at.s), 2 * stage_bytes);
          const bool second = c >= p.token_chunks;
          const int x = m0 + (second ? 2 * p.half : 0), y = (second ? c - p.token_chunks : c) * 64;
          for (int b = 0; b < 2; b++) tma_load_2d<true>(dst + b * 8192, &amap, x + b * 64, y, bar);
          for (int b = 0; b < b_boxes; b++) tma_load_2d<true>(dst + kABytes + b * 8192, &bmap, n0 + b * 64, y, bar);
        }
        __syncwarp();
        at.next();
      }
    }
  } else if (warp == 1) {
    if (me == 0) {
      const uint32_t idesc = instr_desc(p.dtype, true, true, 256, 2 * p.block_cols), mask = 3u << leader;
      constexpr uint32_t k_step = 2048 >> 4;  // 16 tokens further: two groups of 8 rows
      const uint64_t a_desc = smem_desc(base, 8192), b_desc = smem_desc(base + kABytes, 8192);
      Ring at(p.stages);
      int turn = 0;
      for (int tile = blockIdx.x / team; tile < tiles; tile += step, turn++) {
        const int b = p.accumulators == 2 ? turn & 1 : 0, use = p.accumulators == 2 ? turn >> 1 : turn;
        mbar_wait(free_(b), (use & 1) ^ 1, dead_);
        tc_fence_after();
        const uint32_t d = tmem + b * 256;
        for (int c = c0; c < c1; c++) {
          mbar_wait(full(at.s), at.phase, dead_);
          tc_fence_after();
          const uint64_t off = (uint64_t)(at.s * stage_bytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; k++) mma_f16<true>(d, a_desc + off + k * k_step, b_desc + off + k * k_step, idesc, c > c0 || k > 0);
            mma_commit<true>(empty(at.s), mask);
          }
          __syncwarp();
          at.next();
        }
        if (elect_one()) mma_commit<true>(done(b), mask);
        __syncwarp();
      }
    }
  } else {
    const int quarter = warp & 3, group = (warp - 2) >> 2, at = quarter * 32 + lane;
    const uint32_t staging = base + p.stages * stage_bytes;
    const float unscale = p.top ? gradient_power(*p.top, -1) : 1.0f;
    int turn = 0;
    for (int tile = blockIdx.x / team; tile < tiles; tile += step, turn++) {
      int rt, ct;
      tile_at(p, tile, rt, ct);
      const bool second = rt >= p.half_tiles;
      if (second) rt -= p.half_tiles;
      const int m0 = (rt * 2 + me) * 128, m = m0 + at, n0 = ct * 2 * p.block_cols;
      const int b = p.accumulators == 2 ? turn & 1 : 0, use = p.accumulators == 2 ? turn >> 1 : turn;
      const uint32_t d = tmem + b * 256 + ((uint32_t)(quarter * 32) << 16);
      mbar_wait(done(b), use & 1, dead_);
      tc_fence_after();
      if (p.splits == 1) {
        // 32 rows x 64 columns at a time through shared memory (128-byte swizzle) and out by TMA
        for (int c = group * 64; c < 2 * p.block_cols; c += 128) {
          const uint32_t box = staging + (warp - 2) * 4096, to = box + lane * 128;
          uint32_t r[4][16];
#pragma unroll
          for (int h = 0; h < 4; h++) tmem_load16(d + c + h * 16, r[h]);
          if (lane == 0) tma_store_wait<0>();
          tmem_load_wait();
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 8; q++) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
              const uint32_t* at = &r[q >> 1][(q & 1) * 8 + 2 * k];
              w[k] = pack2(__uint_as_float(at[0]) * unscale, __uint_as_float(at[1]) * unscale, p.dtype);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((q ^ (lane & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                         : "memory");
          }
          fence_async_shared();
          __syncwarp();
          const int n = n0 + c;
          // not by TMA: a box that ends in the middle of 16 bytes, which the copy would write whole
          const bool whole = n + 64 <= p.N || p.N % 8 == 0;
          if (lane == 0) {
            if (whole && m0 + quarter * 32 < p.F && n < p.N)
              tma_store_2d(second ? &omap1 : &omap0, n, m0 + quarter * 32, box);
            tma_store_commit();
          }
          if (!whole && m < p.F) {
            for (int g = 0; g < 8; g++) {
              uint32_t v[4];
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                           : "r"(to + ((g ^ (lane & 7)) << 4))
                           : "memory");
              uint16_t* out = static_cast<uint16_t*>(p.O[second]) + m * p.ldo + n + g * 8;
              if (n + g * 8 + 8 <= p.N) {
                *reinterpret_cast<uint4*>(out) = make_uint4(v[0], v[1], v[2], v[3]);
              } else {
                for (int k = 0; k < 8; k++)
                  if (n + g * 8 + k < p.N) out[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
              }
            }
          }
        }
      } else {
        for (int c = group * 16; c < 2 * p.block_cols; c += 32) {
          uint32_t r[16];
          tmem_load16(d + c, r);
          tmem_load_wait();
#pragma unroll
          for (int k = 0; k < 16; k += 4)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (at * kPitch + c + k) * 4), "r"(r[k]),
                         "r"(r[k + 1]), "r"(r[k + 2]), "r"(r[k + 3])
                         : "memory");
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) cluster_arrive(cluster_addr(free_(b), leader));
    }
    if (lane == 0) tma_store_wait<0>();
  }
  __syncwarp();
  __syncthreads();
  if (dead) settle(p.stalls);
  __syncwarp();
  cluster_sync();  // no more arrivals from other blocks; their sums are in shared memory
  if (warp == 1) {
    tc_fence_after();
    tmem_free<true>(tmem, p.columns);
  }
  if (p.splits > 1) {
    int rt, ct;
    tile_at(p, blockIdx.x / team, rt, ct);  // one tile a team
    join(p, base, rt, ct, split, me);
    __syncwarp();
    cluster_sync();  // no block leaves while another reads its shared memory
  }
}

}  // namespace

windq_status launch_weight_gradient(windq_ctx* ctx, const WeightGradient& q, cudaStream_t st) {
  Args p = {};
  p.F = (int)q.F;
  p.N = (int)q.C;
  p.dtype = q.dtype;
  p.token_chunks = (int)((q.T + 63) / 64);
  p.chunks = q.terms * p.token_chunks;
  p.half = (int)q.half;
  p.half_tiles = (int)((q.F + 255) / 256);
  p.row_tiles = 2 * p.half_tiles;
  p.top = q.top;
  p.O[0] = q.dWg;
  p.O[1] = q.dWu;
  p.ldo = q.ldw;
  p.stalls = stalls_of(ctx);
  // The width that takes the least time in rounds over the GPU (a chunk of K: 0.23 us at width 128, 0.27 at 192, 0.36 at 256;
  // a tile 2 us more, 5 where it is split along K).  Tiles that fill less than half of the GPU are split, as far as clusters of
  // whole SMs find room: 33 of four blocks, 15 of eight.
  const int64_t slots = ctx->sm_count / 2;
  int64_t best = INT64_MAX;
  for (int cols = 128; cols >= 64; cols -= 32) {
    const int width = 2 * cols;
    const int64_t tiles = p.row_tiles * ((q.C + width - 1) / width);
    int splits = 1;
    while (splits < 4 && tiles * splits * 2 <= slots * (splits == 1 ? 8 : 7) / 9 && p.chunks >= splits * 2 * 4) splits *= 2;
    const int64_t waves = (tiles * splits + slots - 1) / slots;
    const int chunk = std::max(210 + width / 5, width * 139 / 100) * (1256 - width) / 1000;
    const int64_t cost = waves * ((int64_t)(p.chunks + splits - 1) / splits * chunk + (splits > 1 ? 5000 : 2000));
    if (cost < best) {
      best = cost;
      p.block_cols = cols;
      p.splits = splits;
    }
  }
  p.col_tiles = (int)((q.C + 2 * p.block_cols - 1) / (2 * p.block_cols));
  p.group = (int)std::max<int64_t>(1, std::min<int64_t>(p.row_tiles, (24ll << 20) / (512 * q.T)));
  const int stage = kABytes + (p.block_cols + 63) / 64 * 8192, staging = p.splits > 1 ? 0 : kStaging;
  p.stages = std::min(kMaxStages, (kSmemLimit - 1024 - staging) / stage);
  p.accumulators = p.splits == 1 ? 2 : 1;
  p.columns = 256 * p.accumulators;
  const int64_t tiles = (int64_t)p.row_tiles * p.col_tiles;
  const int64_t blocks = (p.splits > 1 ? tiles * p.splits : std::min(tiles, slots)) * 2;
  const int smem = 1024 + std::max(p.stages * stage + staging, p.splits > 1 ? 128 * kPitch * 4 : 0);

  CUtensorMap a, b, o[2];
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  const bool ok = make_map_2d(&a, q.dtype, q.D, q.terms * 2 * q.half, q.T, q.terms * 4 * q.half, 64) && make_map_2d(&b, q.dtype, q.X, q.C, q.T, 2 * q.ldx, 64) &&
                  make_map_2d(&o[0], q.dtype, q.dWg, q.C, q.F, 2 * q.ldw, 32) && make_map_2d(&o[1], q.dtype, q.dWu, q.C, q.F, 2 * q.ldw, 32);
  WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  const windq_status ready = prepare_kernel(ctx, kWeightGradient, weight_gradient_kernel, kThreads, kSmemLimit, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  overlapped_launch(cfg, attrs, (int)blocks, kThreads, 2 * p.splits, smem, st);
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, weight_gradient_kernel, a, b, o[0], o[1], p));
  return WINDQ_OK;
}

}  // namespace windq
