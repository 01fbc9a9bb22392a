// Few tokens times the weights of a feed-forward block: the shape of decoding, bound by the bytes of the weights.  The formulas
// and what follows the products are those of product_kernel; its pairs of thread blocks, one tile at a time on a whole SM, start and
// balance too coarsely here (33 tokens x 2 x 11008 x 4096 codes: 26.6 us against 18.5; 80 x 2 x 2048 x 2048 13.0 against 9.3).  Up to 64
// tokens, or 128 of a gated product, whose tiles have half as many outputs to join (128 x 2048 x 2048 codes, not gated: 12.4 us, on
// pairs 9.9).
//
// A tile is 128 rows of weights x all tokens, one a thread block and two blocks an SM, so that the loads of one run while another
// starts or ends.  A gated tile has 64 rows of each weight, lanes n and n + 64 of the accumulators.  Sums leave through shared memory,
// where they lie as the result does; where the tiles do not fill the GPU, `splits` blocks (a cluster) share a tile along K and add their
// sums through distributed shared memory, in rank order: equal calls give equal bits.
//
// A block starts while the stream's kernel before ends and first brings its first weights into L2.
//
// Warps: one issues TMA copies, one issues matrix products, four read the accumulators; all of them finish the tile.
#include <algorithm>

#include "feed_forward.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kThreads = 192;
constexpr int kMaxStages = 8;
constexpr int kSmemLimit = 112 * 1024;  // dynamic shared memory of one of two thread blocks an SM
constexpr int kPitch = 132;             // sums of a tile, 32 bits each, rows free of bank conflicts
constexpr int kChunkBytes = 128;        // of K: 64 16-bit values or 128 codes
constexpr int kWeightBytes = 128 * kChunkBytes;

struct Args {
  int T, N, dtype, act;
  int chunks, half_chunks;  // of K; of the first weight (kInputGrad)
  int tokens;               // of the tile: all of them, rounded up, and once more where D has two terms
  int second, half;         // kInputGrad: row of the second terms in the tile, or 0; columns of dG in D
  int splits, stages, columns;  // columns: of tensor memory
  const float* row_scale;
  const float* col_scale[2];
  const uint32_t* top;
  void* O[3];
  int64_t ldo[3];
  Stalls stalls;
};

struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], done;
};

// (Not __ldg, which wants memory that nothing writes while the kernel lives: the kernel before may still write scales when this one comes.)
__device__ __forceinline__ float scale_of(const float* s, int i, int n) { return i < n ? s[i] : 0.0f; }
// Sums over a cluster's n blocks, in the order of their ranks, of U quads at base + offset[u] in each.  Distributed
// shared memory answers after the better part of a microsecond: the loads of up to four blocks are in flight together.
template <int U, bool CODES>
__device__ __forceinline__ void sum_quads(uint32_t base, const uint32_t (&offset)[U], int n, uint32_t (&x)[U][4]) {
  if (n == 1) {
#pragma unroll
    for (int u = 0; u < U; u++)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(x[u][0]), "=r"(x[u][1]), "=r"(x[u][2]), "=r"(x[u][3])
                   : "r"(base + offset[u])
                   : "memory");
    return;
  }
#pragma unroll
  for (int u = 0; u < U; u++)
#pragma unroll
    for (int k = 0; k < 4; k++) x[u][k] = 0;
  for (int q0 = 0; q0 < n; q0 += 4) {
    uint32_t y[4][U][4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
      if (q0 + q < n) {
        const uint32_t from = cluster_addr(base, q0 + q);
#pragma unroll
        for (int u = 0; u < U; u++)
          asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(y[q][u][0]), "=r"(y[q][u][1]), "=r"(y[q][u][2]), "=r"(y[q][u][3])
                       : "r"(from + offset[u])
                       : "memory");
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int k = 0; k < 4; k++)
#pragma unroll
        for (int q = 0; q < 4; q++)
          if (q0 + q < n) x[u][k] = CODES ? x[u][k] + y[q][u][k] : __float_as_uint(__uint_as_float(x[u][k]) + __uint_as_float(y[q][u][k]));
  }
}

// Four neighbouring values of an output row, the last of which may lie beyond its end.
__device__ __forceinline__ void store_quad(void* O, int64_t ldo, int64_t m, int n, int N, int dtype, const float (&v)[4]) {
  uint16_t* out = static_cast<uint16_t*>(O) + m * ldo + n;
  if (n + 4 <= N) {
    *reinterpret_cast<uint2*>(out) = make_uint2(pack2(v[0], v[1], dtype), pack2(v[2], v[3], dtype));
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (n + k < N) store1(out, k, dtype, v[k]);
  }
}

// Adds the sums of a tile's splits, which lie as [token][output] in the shared memory of their blocks, and stores this block's
// share of the tokens: split, split + splits, ...
template <int KIND>
__device__ __forceinline__ void join(const Args& p, uint32_t base, int wt, int split) {
  using K = Kind<KIND>;
  constexpr int U = K::kGate || K::kTransposed ? 2 : 4, outputs = K::kGate ? 64 : 128, quads = outputs / 4;
  const int n0 = wt * outputs, items = max(0, (p.T - split + p.splits - 1) / p.splits) * quads;
  const float unscale = p.top ? gradient_power(*p.top, -1) : 1.0f;
  for (int i = threadIdx.x; i < items; i += U * kThreads) {
    uint32_t offset[U], x[U][4], y[U][4];
    float row[U], col[U][K::kGate ? 2 : 1][4];  // scales, on their way while the sums are read
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int q = min(i + u * kThreads, items - 1), t = split + q / quads * p.splits, n = n0 + q % quads * 4;
      offset[u] = (uint32_t)(t * kPitch + q % quads * 4) * 4;
      row[u] = K::kCodes ? p.row_scale[t] : unscale;
#pragma unroll
      for (int w = 0; w < (K::kGate ? 2 : 1); w++)
#pragma unroll
        for (int k = 0; k < 4; k++) col[u][w][k] = K::kCodes ? scale_of(p.col_scale[w], n + k, p.N) : 1.0f;
    }
    sum_quads<U, K::kCodes>(base, offset, p.splits, x);
    if (K::kTransposed && p.second) {
#pragma unroll
      for (int u = 0; u < U; u++) offset[u] += p.second * kPitch * 4;
      sum_quads<U, false>(base, offset, p.splits, y);
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int k = 0; k < 4; k++) x[u][k] = __float_as_uint(__uint_as_float(x[u][k]) + __uint_as_float(y[u][k]));
    }
    if (K::kGate) {
#pragma unroll
      for (int u = 0; u < U; u++) offset[u] += 64 * 4;
      sum_quads<U, K::kCodes>(base, offset, p.splits, y);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int q = i + u * kThreads, t = split + q / quads * p.splits, n = n0 + q % quads * 4;
      if (q >= items || n >= p.N) continue;
      float a[4], b[4], h[4];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        a[k] = value_of<K::kCodes>(x[u][k], row[u], col[u][0][k]);
        if (K::kGate) {
          b[k] = value_of<K::kCodes>(y[u][k], row[u], col[u][1][k]);
          h[k] = gated(a[k], b[k], p.act);
        }
      }
      if (K::kGate) {
        if (KIND != kGated || p.O[0]) store_quad(p.O[0], p.ldo[0], t, n, p.N, p.dtype, h);
        if (KIND == kGated && p.O[1]) {
          store_quad(p.O[1], p.ldo[1], t, n, p.N, p.dtype, a);
          store_quad(p.O[2], p.ldo[2], t, n, p.N, p.dtype, b);
        }
      } else {
        store_quad(p.O[0], p.ldo[0], t, n, p.N, p.dtype, a);
      }
    }
  }
}

// One tile (or, split, a part of its K) a thread block.
template <int KIND>
__global__ void __launch_bounds__(kThreads, 2)
    few_tokens_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap0,
                const __grid_constant__ CUtensorMap wmap1, const __grid_constant__ Args p) {
  using K = Kind<KIND>;
  extern __shared__ uint8_t raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t stage_bytes = kWeightBytes + p.tokens * kChunkBytes, dead_ = smem_addr(&dead), done = smem_addr(&bars.done);
  auto full = [&](int s) { return smem_addr(&bars.full[s]); };
  auto empty = [&](int s) { return smem_addr(&bars.empty[s]); };

  if (threadIdx.x == 0) {
    prefetch_map(&xmap);
    prefetch_map(&wmap0);
    prefetch_map(&wmap1);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    mbar_init(done, 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<false>(smem_addr(&tmem_slot), p.columns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  launch_dependents();  // tensor memory is in hand
  const uint32_t tmem = tmem_slot;

  const int split = blockIdx.x % p.splits;
  const int c0 = (int)((int64_t)p.chunks * split / p.splits), c1 = (int)((int64_t)p.chunks * (split + 1) / p.splits);
  const int wt = blockIdx.x / p.splits;

  if (warp == 0) {
    const int n0 = wt * (K::kGate ? 64 : 128);
    auto weights = [&](int c, auto take) {  // the two boxes of a chunk
      if (K::kTransposed) {
        const bool other = c >= p.half_chunks;
        const int k0 = (other ? c - p.half_chunks : c) * 64;
        take(0, other ? &wmap1 : &wmap0, n0, k0);
        take(1, other ? &wmap1 : &wmap0, n0 + 64, k0);
      } else {
        take(0, &wmap0, c * K::kStepK, n0);
        take(1, K::kGate ? &wmap1 : &wmap0, c * K::kStepK, K::kGate ? n0 : n0 + 64);
      }
    };
    if (elect_one())
      for (int c = c0; c < min(c1, c0 + p.stages); c++)
        weights(c, [&](int, const CUtensorMap* map, int x, int y) { tma_prefetch_2d(map, x, y); });
    __syncwarp();
    wait_for_predecessor();
    Ring at(p.stages);
    for (int c = c0; c < c1; c++) {
      mbar_wait(empty(at.s), at.phase ^ 1, dead_);
      const uint32_t dst = base + at.s * stage_bytes, bar = full(at.s);
      if (elect_one() && !*(volatile int*)&dead) {
        mbar_expect(bar, stage_bytes);
        weights(c, [&](int k, const CUtensorMap* map, int x, int y) { tma_load_2d<false>(dst + k * 8192, map, x, y, bar); });
        tma_load_2d<false>(dst + kWeightBytes, &xmap, c * K::kStepK, 0, bar);
        if (K::kTransposed && p.second) tma_load_2d<false>(dst + kWeightBytes + p.second * kChunkBytes, &xmap, c * 64 + 2 * p.half, 0, bar);
      }
      __syncwarp();
      at.next();
    }
  } else if (warp == 1) {
    wait_for_predecessor();
    const uint32_t idesc = K::kCodes ? instr_desc_i8(128, p.tokens) : instr_desc(p.dtype, K::kTransposed, false, 128, p.tokens);
    constexpr uint32_t w_step = (K::kTransposed ? 2048 : 32) >> 4, t_step = 32 >> 4;
    const uint64_t w_desc = smem_desc(base, K::kTransposed ? 8192 : 16), t_desc = smem_desc(base + kWeightBytes, 16);
    Ring at(p.stages);
    for (int c = c0; c < c1; c++) {
      mbar_wait(full(at.s), at.phase, dead_);
      tc_fence_after();
      const uint64_t off = (uint64_t)(at.s * stage_bytes >> 4);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 4; k++) {
          if (K::kCodes) mma_i8<false>(tmem, w_desc + off + k * w_step, t_desc + off + k * t_step, idesc, c > c0 || k > 0);
          else mma_f16<false>(tmem, w_desc + off + k * w_step, t_desc + off + k * t_step, idesc, c > c0 || k > 0);
        }
        mma_commit<false>(empty(at.s), 0);
      }
      __syncwarp();
      at.next();
    }
    if (elect_one()) mma_commit<false>(done, 0);
    __syncwarp();
  } else {
    wait_for_predecessor();
    const int quarter = warp & 3, n = quarter * 32 + lane;
    mbar_wait(done, 0, dead_);
    tc_fence_after();
    // as the result lies: [token][output], the outputs being the lanes; the copies and products of all stages have ended
    for (int c = 0; c < p.tokens; c += 16) {
      uint32_t r[16];
      tmem_load16(tmem + c + ((uint32_t)(quarter * 32) << 16), r);
      tmem_load_wait();
#pragma unroll
      for (int k = 0; k < 16; k++)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + ((c + k) * kPitch + n) * 4), "r"(r[k]) : "memory");
    }
    tc_fence_before();
  }
  __syncwarp();
  __syncthreads();
  if (dead) settle(p.stalls);
  __syncwarp();
  if (warp == 1) {  // given back before this block waits for its cluster
    tc_fence_after();
    tmem_free<false>(tmem, p.columns);
  }
  __syncwarp();
  if (p.splits > 1) cluster_sync();
  join<KIND>(p, base, wt, split);
  if (p.splits > 1) {
    __syncwarp();
    cluster_sync();  // no block leaves while another reads its shared memory
  }
}

template <int KIND>
windq_status launch(windq_ctx* ctx, const CUtensorMap& x, const CUtensorMap (&w)[2], const Args& p, int blocks, int smem, cudaStream_t st) {
  const windq_status ready = prepare_kernel(ctx, kFewTokens + KIND, few_tokens_kernel<KIND>, kThreads, kSmemLimit, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  overlapped_launch(cfg, attrs, blocks, kThreads, p.splits, smem, st);
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, few_tokens_kernel<KIND>, x, w[0], w[1], p));
  return WINDQ_OK;
}

}  // namespace

windq_status launch_few_tokens(windq_ctx* ctx, const Product& q, cudaStream_t st) {
  const bool codes = q.kind == kInt8 || q.kind == kInt8Gated, gate = q.kind == kInt8Gated || q.kind == kGated;
  const bool transposed = q.kind == kInputGrad;
  const int step = codes ? 128 : 64;
  Args p = {};
  p.T = (int)q.T;
  p.N = (int)q.N;
  p.dtype = q.dtype;
  p.act = q.act;
  p.half_chunks = (int)((q.K + step - 1) / step);
  p.chunks = transposed ? 2 * p.half_chunks : p.half_chunks;
  const int rows = (int)round_up(q.T, 16);
  p.second = transposed && q.terms == 2 ? rows : 0;  // two terms of a token are two tokens: the weights are read once
  p.tokens = rows + p.second;
  p.half = (int)q.half;
  p.row_scale = q.row_scale;
  p.top = q.top;
  for (int k = 0; k < 2; k++) p.col_scale[k] = q.col_scale[k];
  for (int k = 0; k < 3; k++) p.O[k] = q.O[k], p.ldo[k] = q.ldo[k];
  p.stalls = stalls_of(ctx);
  const int outputs = gate ? 64 : 128;
  const int64_t tiles = (q.N + outputs - 1) / outputs;
  // As many as two blocks an SM hold: 48 tokens x 4096 x 11008 codes in two splits 20.3 us, in four 16.4; 33 tokens x 2 x 11008 x 4096,
  // 172 tiles, whole 20.4, in two 27.9.  Clusters of four do not fill the last slots of every GPC (60 tokens x 2 x 4700 x 5056, 74
  // tiles: in four splits, 296 blocks, 30.0 us, in two 22.1).  Clusters of eight start and join slowly: for few tiles and a long K alone
  // (8 x 2 x 1024 x 8192 11.8 -> 9.8, but 48 x 4096 x 11008 codes 16.3 -> 17.8).
  p.splits = 1;
  for (int splits = 2; splits <= 4; splits *= 2)
    if (tiles * splits <= ctx->sm_count * 2 * (splits == 4 ? 9 : 10) / 10 && p.chunks >= splits * 4) p.splits = splits;
  if (tiles * 8 <= ctx->sm_count && p.chunks >= 8 * 12) p.splits = 8;
  const int stage = kWeightBytes + p.tokens * kChunkBytes;
  p.stages = std::min(kMaxStages, (kSmemLimit - 1024) / stage);
  p.columns = p.tokens <= 32 ? 32 : p.tokens <= 64 ? 64 : 128;
  const int smem = 1024 + std::max(p.stages * stage, p.tokens * kPitch * 4);

  CUtensorMap x, w[2];
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  const int type = codes ? -1 : q.dtype, bytes = codes ? 1 : 2;
  bool ok = make_map_2d(&x, type, q.X, transposed ? q.terms * 2 * q.half : q.K, q.T, q.ldx * bytes, rows);
  for (int k = 0; ok && k < (q.W[1] ? 2 : 1); k++)
    ok = make_map_2d(&w[k], type, q.W[k], transposed ? q.N : q.K, transposed ? q.K : q.N, q.ldw[k] * bytes, 64);
  if (!q.W[1]) w[1] = w[0];
  WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  const int blocks = (int)(tiles * p.splits);
  switch (q.kind) {
    case kInt8: return launch<kInt8>(ctx, x, w, p, blocks, smem, st);
    case kInt8Gated: return launch<kInt8Gated>(ctx, x, w, p, blocks, smem, st);
    case kGated: return launch<kGated>(ctx, x, w, p, blocks, smem, st);
    default: return launch<kInputGrad>(ctx, x, w, p, blocks, smem, st);
  }
}

}  // namespace windq
