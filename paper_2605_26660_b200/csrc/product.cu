// The matrix products of the feed-forward calls on the tensor cores (tcgen05, accumulators in tensor memory, operands by
// TMA), with what follows a product done on its accumulators: scales of codes, the gate, the rounding.
//
// Warps: one issues TMA copies, one issues matrix products, four read the accumulators and store.  Two layouts of a tile:
//   wide  256 rows x up to 256 columns on a pair of thread blocks (cta_group::2: each holds half of either operand, so that a
//         block's shared memory feeds a product twice as large); persistent over tiles with two accumulators, so that storing
//         a tile overlaps the next
//   tall  (few tokens) 128 outputs x up to 256 tokens: the weight is read once and the tokens cost little -- the shape of
//         decoding, bound by the bytes of the weight
// A gated tile has both products of the same outputs: half of its weight rows are the gate's, half the other's.  In a wide
// tile the two blocks of a pair hold one each, and a row's two accumulators are columns c and c + block_cols; in a tall one
// they are lanes n and n + 64.
//
// Where the tiles do not fill the GPU, `splits` thread blocks (a cluster) share a tile along K and add their accumulators
// through distributed shared memory, in rank order: equal calls give equal bits.
#include <algorithm>

#include "feed_forward.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kThreads = 192;
constexpr int kMaxStages = 8;
constexpr int kSmemLimit = 227 * 1024 - 2048;      // dynamic shared memory of one thread block per SM
constexpr int kSmemLimitTwo = 112 * 1024;          // of two
constexpr int kTallPitch = 132, kWidePitch = 260;  // sums of a tile, 32 bits each, rows free of bank conflicts
constexpr int kStaging = 4 * 2 * 4096;             // of the four storing warps of a wide tile
constexpr int kChunkBytes = 128;                   // of K: 64 16-bit values or 128 codes

struct Args {
  int M, N, dtype, act;
  int chunks, half_chunks;         // of K; of the first weight (kInputGrad)
  int block_rows, block_cols;      // of a thread block: wide 128 rows x half of the columns; tall tokens x weight rows of a box
  int row_tiles, col_tiles, group;
  int half_tiles, half;            // kWeightGrad: row tiles of the first output, columns of each half of A
  int splits, stages, accumulators, columns;  // columns: of tensor memory
  const float* row_scale;
  const float* col_scale[2];
  const uint32_t* top;
  void* O[3];
  int64_t ldo[3];
  Stalls stalls;
};

struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], done[2], free[2];
};

template <int KIND>
struct Kind {
  static constexpr bool kCodes = KIND == kInt8 || KIND == kInt8Gated, kGate = KIND == kInt8Gated || KIND == kGated;
  static constexpr bool kTransA = KIND == kWeightGrad, kTransB = KIND == kInputGrad || KIND == kWeightGrad;
  static constexpr int kStepK = kCodes ? 128 : 64;  // values of a chunk
};

// Tiles in an order that keeps a group of row tiles in L2 while the columns stream by.
__device__ __forceinline__ void tile_at(const Args& p, int tile, int& rt, int& ct) {
  const int per = p.group * p.col_tiles, g = tile / per, rest = tile - g * per;
  const int rows = min(p.group, p.row_tiles - g * p.group);
  ct = rest / rows;
  rt = g * p.group + rest - ct * rows;
}

__device__ __forceinline__ float scale_of(const float* s, int i, int n) { return i < n ? __ldg(s + i) : 0.0f; }
// What an accumulator stands for.
template <bool CODES>
__device__ __forceinline__ float value_of(uint32_t acc, float row, float col) {
  if (CODES) return __int2float_rn((int)acc) * row * col;
  return __uint_as_float(acc) * row;
}
__device__ __forceinline__ float gated(float g, float u, int act) { return g * logistic(gate_exponent(g, act)) * u; }

// Sums over the n blocks of ranks first, first + stride, ... of U quads at base + offset[u] in each, in that order.  Distributed
// shared memory answers after the better part of a microsecond: the loads of up to four blocks are in flight together.
template <int U, bool CODES>
__device__ __forceinline__ void sum_quads(uint32_t base, const uint32_t (&offset)[U], int n, int first, int stride, uint32_t (&x)[U][4]) {
  if (n == 1) {
#pragma unroll
    for (int u = 0; u < U; u++)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(x[u][0]), "=r"(x[u][1]), "=r"(x[u][2]), "=r"(x[u][3])
                   : "r"(base + offset[u])
                   : "memory");
    return;
  }
  uint32_t y[4][U][4];
#pragma unroll
  for (int q = 0; q < 4; q++) {
    if (q < n) {
      const uint32_t from = cluster_addr(base, first + q * stride);
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
    for (int k = 0; k < 4; k++) {
      x[u][k] = y[0][u][k];
#pragma unroll
      for (int q = 1; q < 4; q++)
        if (q < n) x[u][k] = CODES ? x[u][k] + y[q][u][k] : __float_as_uint(__uint_as_float(x[u][k]) + __uint_as_float(y[q][u][k]));
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

// Adds the sums of a tile's splits, which lie as [row][column] in the shared memory of their blocks, and stores this block's
// share of the rows: those of local index split, split + splits, ...
template <int KIND, bool TALL>
__device__ __forceinline__ void join(const Args& p, uint32_t base, int rt, int ct, int split, int me) {
  using K = Kind<KIND>;
  constexpr int pitch = TALL ? kTallPitch : kWidePitch, U = K::kGate ? 2 : 4;
  const int outputs = TALL ? (K::kGate ? 64 : 128) : (K::kGate ? 1 : 2) * p.block_cols, quads = outputs / 4;
  const bool second = KIND == kWeightGrad && rt >= p.half_tiles;
  if (second) rt -= p.half_tiles;
  const int m0 = TALL ? rt * p.block_rows : (rt * 2 + me) * 128, n0 = ct * outputs;
  const int rows = min(TALL ? p.block_rows : 128, p.M - m0);
  const int items = max(0, (rows - split + p.splits - 1) / p.splits) * quads;
  const int shift = (TALL ? 64 : p.block_cols) * 4;  // bytes from g to u
  const float unscale = p.top ? gradient_power(*p.top, -1) : 1.0f;
  for (int i = threadIdx.x; i < items; i += U * kThreads) {
    uint32_t offset[U], x[U][4], y[U][4];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int q = min(i + u * kThreads, items - 1);
      offset[u] = (uint32_t)((split + q / quads * p.splits) * pitch + q % quads * 4) * 4;
    }
    sum_quads<U, K::kCodes>(base, offset, p.splits, me, TALL ? 1 : 2, x);
    if (K::kGate) {
#pragma unroll
      for (int u = 0; u < U; u++) offset[u] += shift;
      sum_quads<U, K::kCodes>(base, offset, p.splits, me, TALL ? 1 : 2, y);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int q = i + u * kThreads, m = m0 + split + q / quads * p.splits, n = n0 + q % quads * 4;
      if (q >= items || n >= p.N) continue;
      const float row = K::kCodes ? __ldg(p.row_scale + m) : unscale;
      float a[4], b[4], h[4];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        a[k] = value_of<K::kCodes>(x[u][k], row, K::kCodes ? scale_of(p.col_scale[0], n + k, p.N) : 1.0f);
        if (K::kGate) {
          b[k] = value_of<K::kCodes>(y[u][k], row, K::kCodes ? scale_of(p.col_scale[1], n + k, p.N) : 1.0f);
          h[k] = gated(a[k], b[k], p.act);
        }
      }
      if (K::kGate) {
        if (KIND != kGated || p.O[0]) store_quad(p.O[0], p.ldo[0], m, n, p.N, p.dtype, h);
        if (KIND == kGated && p.O[1]) {
          store_quad(p.O[1], p.ldo[1], m, n, p.N, p.dtype, a);
          store_quad(p.O[2], p.ldo[2], m, n, p.N, p.dtype, b);
        }
      } else {
        store_quad(p.O[second], p.ldo[second], m, n, p.N, p.dtype, a);
      }
    }
  }
}

template <int KIND>
__global__ void __launch_bounds__(kThreads, 1)
    wide_kernel(const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap0,
                const __grid_constant__ CUtensorMap bmap1, const __grid_constant__ CUtensorMap omap0,
                const __grid_constant__ CUtensorMap omap1, const __grid_constant__ CUtensorMap omap2,
                const __grid_constant__ Args p) {
  using K = Kind<KIND>;
  extern __shared__ uint8_t raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank(), me = rank & 1, leader = rank & ~1u;
  constexpr uint32_t a_bytes = 128 * kChunkBytes;
  const int b_boxes = (p.block_cols + 63) / 64;  // of a transposed weight
  const uint32_t b_bytes = K::kTransB ? b_boxes * 8192 : p.block_cols * kChunkBytes, stage_bytes = a_bytes + b_bytes;
  const uint32_t dead_ = smem_addr(&dead);
  auto full = [&](int s) { return smem_addr(&bars.full[s]); };
  auto empty = [&](int s) { return smem_addr(&bars.empty[s]); };
  auto done = [&](int b) { return smem_addr(&bars.done[b]); };
  auto free_ = [&](int b) { return smem_addr(&bars.free[b]); };

  if (threadIdx.x == 0) {
    prefetch_map(&amap);
    prefetch_map(&bmap0);
    prefetch_map(&bmap1);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int b = 0; b < 2; b++) {
      mbar_init(done(b), 1);
      mbar_init(free_(b), 8);
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
      const bool second = KIND == kWeightGrad && rt >= p.half_tiles;
      const int m0 = (second ? p.half + (rt - p.half_tiles) * 256 : rt * 256) + me * 128;
      const int n0 = K::kGate ? ct * p.block_cols : (ct * 2 + me) * p.block_cols;
      for (int c = c0; c < c1; c++) {
        mbar_wait(empty(at.s), at.phase ^ 1, dead_);
        const uint32_t dst = base + at.s * stage_bytes, bar = to + at.s * 8;
        if (elect_one() && !*(volatile int*)&dead) {
          if (me == 0) mbar_expect(full(at.s), 2 * stage_bytes);
          if (K::kTransA) {
            tma_load_2d<true>(dst, &amap, m0, c * 64, bar);
            tma_load_2d<true>(dst + 8192, &amap, m0 + 64, c * 64, bar);
          } else {
            tma_load_2d<true>(dst, &amap, c * K::kStepK, m0, bar);
          }
          if (K::kTransB) {
            const bool other = KIND == kInputGrad && c >= p.half_chunks;
            const int k0 = (other ? c - p.half_chunks : c) * 64;
            for (int b = 0; b < b_boxes; b++)
              tma_load_2d<true>(dst + a_bytes + b * 8192, other ? &bmap1 : &bmap0, n0 + b * 64, k0, bar);
          } else {
            tma_load_2d<true>(dst + a_bytes, K::kGate && me ? &bmap1 : &bmap0, c * K::kStepK, n0, bar);
          }
        }
        __syncwarp();
        at.next();
      }
    }
  } else if (warp == 1) {
    if (me == 0) {
      const uint32_t idesc = K::kCodes ? instr_desc_i8(256, 2 * p.block_cols)
                                       : instr_desc(p.dtype, K::kTransA, K::kTransB, 256, 2 * p.block_cols);
      const uint32_t mask = 3u << leader;
      // a step of K further: 32 bytes in a K-major tile, two groups of 8 rows in an MN-major one
      constexpr uint32_t a_step = (K::kTransA ? 2048 : 32) >> 4, b_step = (K::kTransB ? 2048 : 32) >> 4;
      const uint64_t a_desc = smem_desc(base, K::kTransA ? 8192 : 16), b_desc = smem_desc(base + a_bytes, K::kTransB ? 8192 : 16);
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
            for (int k = 0; k < 4; k++) {
              if (K::kCodes) mma_i8<true>(d, a_desc + off + k * a_step, b_desc + off + k * b_step, idesc, c > c0 || k > 0);
              else mma_f16<true>(d, a_desc + off + k * a_step, b_desc + off + k * b_step, idesc, c > c0 || k > 0);
            }
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
    const int quarter = warp & 3, at = quarter * 32 + lane;
    const uint32_t staging = base + p.stages * stage_bytes;
    const float unscale = p.top ? gradient_power(*p.top, -1) : 1.0f;
    uint32_t buffer = 0;
    int turn = 0;
    for (int tile = blockIdx.x / team; tile < tiles; tile += step, turn++) {
      int rt, ct;
      tile_at(p, tile, rt, ct);
      const bool second = KIND == kWeightGrad && rt >= p.half_tiles;
      if (second) rt -= p.half_tiles;
      const int m0 = (rt * 2 + me) * 128, m = m0 + at, n0 = ct * (K::kGate ? 1 : 2) * p.block_cols;
      const float row = K::kCodes ? scale_of(p.row_scale, m, p.M) : unscale;
      const int b = p.accumulators == 2 ? turn & 1 : 0, use = p.accumulators == 2 ? turn >> 1 : turn;
      const uint32_t d = tmem + b * 256 + ((uint32_t)(quarter * 32) << 16);
      mbar_wait(done(b), use & 1, dead_);
      tc_fence_after();
      if (p.splits == 1) {
        // 32 rows x 64 columns at a time through shared memory (128-byte swizzle, two buffers a warp) and out by TMA
        const int outputs = (K::kGate ? 1 : 2) * p.block_cols;
        // output 0 (h), 1 (g) or 2 (u); the plain kinds have one, of the accumulators at c
        auto box = [&](int o, int c, void* O, int64_t ldo, const CUtensorMap* map) {
          const uint32_t to = staging + ((quarter * 2 + buffer) * 32 + lane) * 128;
          if (lane == 0) tma_store_wait<1>();
          __syncwarp();
#pragma unroll
          for (int h = 0; h < 4; h++) {
            uint32_t r[16], s[16], w[8];
            if (!K::kGate || o != 2) tmem_load16(d + c + h * 16, r);
            if (K::kGate && o != 1) tmem_load16(d + p.block_cols + c + h * 16, s);
            tmem_load_wait();
            float x[16];
#pragma unroll
            for (int k = 0; k < 16; k++) {
              const int n = n0 + c + h * 16 + k;
              if (!K::kGate) {
                x[k] = value_of<K::kCodes>(r[k], row, K::kCodes ? scale_of(p.col_scale[0], n, p.N) : 1.0f);
              } else {
                const float g = o == 2 ? 0.0f : value_of<K::kCodes>(r[k], row, K::kCodes ? scale_of(p.col_scale[0], n, p.N) : 1.0f);
                const float u = o == 1 ? 0.0f : value_of<K::kCodes>(s[k], row, K::kCodes ? scale_of(p.col_scale[1], n, p.N) : 1.0f);
                x[k] = o == 1 ? g : o == 2 ? u : gated(g, u, p.act);
              }
            }
#pragma unroll
            for (int q = 0; q < 8; q++) w[q] = pack2(x[2 * q], x[2 * q + 1], p.dtype);
#pragma unroll
            for (int q = 0; q < 2; q++)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((h * 2 + q) ^ (lane & 7)) << 4)), "r"(w[4 * q]),
                           "r"(w[4 * q + 1]), "r"(w[4 * q + 2]), "r"(w[4 * q + 3])
                           : "memory");
          }
          fence_async_shared();
          __syncwarp();
          const int n = n0 + c;
          // not by TMA: a box that ends in the middle of 16 bytes, which the copy would write whole
          const bool whole = n + 64 <= p.N || p.N % 8 == 0;
          if (lane == 0) {
            if (whole && m0 + quarter * 32 < p.M && n < p.N) tma_store_2d(map, n, m0 + quarter * 32, staging + (quarter * 2 + buffer) * 4096);
            tma_store_commit();
          }
          if (!whole && m < p.M) {
            for (int g = 0; g < 8; g++) {
              uint32_t v[4];
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                           : "r"(to + ((g ^ (lane & 7)) << 4))
                           : "memory");
              uint16_t* out = static_cast<uint16_t*>(O) + (int64_t)m * ldo + n + g * 8;
              if (n + g * 8 + 8 <= p.N) {
                *reinterpret_cast<uint4*>(out) = make_uint4(v[0], v[1], v[2], v[3]);
              } else {
                for (int k = 0; k < 8; k++)
                  if (n + g * 8 + k < p.N) out[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
              }
            }
          }
          buffer ^= 1;
        };
        for (int c = 0; c < outputs; c += 64) {
          if (KIND == kGated) {
            if (p.O[0]) box(0, c, p.O[0], p.ldo[0], &omap0);
            if (p.O[1]) {
              box(1, c, p.O[1], p.ldo[1], &omap1);
              box(2, c, p.O[2], p.ldo[2], &omap2);
            }
          } else if (KIND == kWeightGrad) {
            box(0, c, second ? p.O[1] : p.O[0], second ? p.ldo[1] : p.ldo[0], second ? &omap1 : &omap0);
          } else {
            box(0, c, p.O[0], p.ldo[0], &omap0);
          }
        }
      } else {
        for (int c = 0; c < 2 * p.block_cols; c += 16) {
          uint32_t r[16];
          tmem_load16(d + c, r);
          tmem_load_wait();
#pragma unroll
          for (int k = 0; k < 16; k += 4)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (at * kWidePitch + c + k) * 4), "r"(r[k]),
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
    join<KIND, false>(p, base, rt, ct, split, me);
    __syncwarp();
    cluster_sync();  // no block leaves while another reads its shared memory
  }
}

// One tile (or, split, a part of its K) a thread block.
template <int KIND>
__global__ void __launch_bounds__(kThreads, 2)
    tall_kernel(const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap0,
                const __grid_constant__ CUtensorMap bmap1, const __grid_constant__ Args p) {
  using K = Kind<KIND>;
  extern __shared__ uint8_t raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t a_bytes = p.block_rows * kChunkBytes;
  constexpr uint32_t b_bytes = 128 * kChunkBytes;
  const uint32_t stage_bytes = a_bytes + b_bytes, dead_ = smem_addr(&dead), done = smem_addr(&bars.done[0]);
  auto full = [&](int s) { return smem_addr(&bars.full[s]); };
  auto empty = [&](int s) { return smem_addr(&bars.empty[s]); };

  if (threadIdx.x == 0) {
    prefetch_map(&amap);
    prefetch_map(&bmap0);
    prefetch_map(&bmap1);
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
  wait_for_predecessor();
  const uint32_t tmem = tmem_slot;

  const int split = blockIdx.x % p.splits;
  const int c0 = (int)((int64_t)p.chunks * split / p.splits), c1 = (int)((int64_t)p.chunks * (split + 1) / p.splits);
  int rt, ct;
  tile_at(p, blockIdx.x / p.splits, rt, ct);

  if (warp == 0) {
    Ring at(p.stages);
    const int m0 = rt * p.block_rows, n0 = ct * (K::kGate ? 64 : 128);
    for (int c = c0; c < c1; c++) {
      mbar_wait(empty(at.s), at.phase ^ 1, dead_);
      const uint32_t dst = base + at.s * stage_bytes, bar = full(at.s);
      if (elect_one() && !*(volatile int*)&dead) {
        mbar_expect(bar, stage_bytes);
        if (K::kTransB) {
          const bool other = c >= p.half_chunks;
          const int k0 = (other ? c - p.half_chunks : c) * 64;
          tma_load_2d<false>(dst, other ? &bmap1 : &bmap0, n0, k0, bar);
          tma_load_2d<false>(dst + 8192, other ? &bmap1 : &bmap0, n0 + 64, k0, bar);
        } else {
          tma_load_2d<false>(dst, &bmap0, c * K::kStepK, n0, bar);
          tma_load_2d<false>(dst + 8192, K::kGate ? &bmap1 : &bmap0, c * K::kStepK, K::kGate ? n0 : n0 + 64, bar);
        }
        tma_load_2d<false>(dst + b_bytes, &amap, c * K::kStepK, m0, bar);
      }
      __syncwarp();
      at.next();
    }
  } else if (warp == 1) {
    const uint32_t idesc = K::kCodes ? instr_desc_i8(128, p.block_rows) : instr_desc(p.dtype, K::kTransB, false, 128, p.block_rows);
    constexpr uint32_t w_step = (K::kTransB ? 2048 : 32) >> 4, t_step = 32 >> 4;
    const uint64_t w_desc = smem_desc(base, K::kTransB ? 8192 : 16), t_desc = smem_desc(base + b_bytes, 16);
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
    const int quarter = warp & 3, n = quarter * 32 + lane;
    mbar_wait(done, 0, dead_);
    tc_fence_after();
    // as the result lies: [token][output], the outputs being the lanes; the copies and products of all stages have ended
    for (int c = 0; c < p.block_rows; c += 16) {
      uint32_t r[16];
      tmem_load16(tmem + c + ((uint32_t)(quarter * 32) << 16), r);
      tmem_load_wait();
#pragma unroll
      for (int k = 0; k < 16; k++)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + ((c + k) * kTallPitch + n) * 4), "r"(r[k]) : "memory");
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
  join<KIND, true>(p, base, rt, ct, split, 0);
  if (p.splits > 1) {
    __syncwarp();
    cluster_sync();  // no block leaves while another reads its shared memory
  }
}

void configure(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attrs)[2], int blocks, int cluster, int smem, cudaStream_t st) {
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = cluster;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
}

template <int KIND>
windq_status launch_wide(windq_ctx* ctx, const CUtensorMap& a, const CUtensorMap (&b)[2], const CUtensorMap (&o)[3], const Args& p,
                         int blocks, int smem, cudaStream_t st) {
  const windq_status ready = prepare_kernel(ctx, kProductWide + KIND, wide_kernel<KIND>, kThreads, kSmemLimit, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  configure(cfg, attrs, blocks, 2 * p.splits, smem, st);
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, wide_kernel<KIND>, a, b[0], b[1], o[0], o[1], o[2], p));
  return WINDQ_OK;
}
template <int KIND>
windq_status launch_tall(windq_ctx* ctx, const CUtensorMap& a, const CUtensorMap (&b)[2], const Args& p, int blocks, int smem,
                         cudaStream_t st) {
  const windq_status ready = prepare_kernel(ctx, kProductTall + KIND, tall_kernel<KIND>, kThreads, kSmemLimit, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  configure(cfg, attrs, blocks, p.splits, smem, st);
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, tall_kernel<KIND>, a, b[0], b[1], p));
  return WINDQ_OK;
}

}  // namespace

windq_status launch_product(windq_ctx* ctx, const Product& q, cudaStream_t st) {
  const bool codes = q.kind == kInt8 || q.kind == kInt8Gated, gate = q.kind == kInt8Gated || q.kind == kGated;
  const bool grad_w = q.kind == kWeightGrad, trans_b = q.kind == kInputGrad || grad_w;
  const bool tall = !grad_w && q.M <= 320;
  const int step = codes ? 128 : 64;
  Args p = {};
  p.M = (int)q.M;
  p.N = (int)q.N;
  p.dtype = q.dtype;
  p.act = q.act;
  p.half_chunks = (int)((q.K + step - 1) / step);
  p.chunks = q.kind == kInputGrad ? 2 * p.half_chunks : p.half_chunks;
  p.half = (int)q.half;
  p.row_scale = q.row_scale;
  p.top = q.top;
  for (int k = 0; k < 2; k++) p.col_scale[k] = q.col_scale[k];
  for (int k = 0; k < 3; k++) p.O[k] = q.O[k], p.ldo[k] = q.ldo[k];
  p.stalls = stalls_of(ctx);

  int smem, blocks;
  if (tall) {
    const int64_t tiles_of = std::max<int64_t>(1, (q.M + 255) / 256);
    p.block_rows = (int)round_up((q.M + tiles_of - 1) / tiles_of, 16);
    p.block_cols = 64;
    p.row_tiles = (int)((q.M + p.block_rows - 1) / p.block_rows);
    const int outputs = gate ? 64 : 128;
    p.col_tiles = (int)((q.N + outputs - 1) / outputs);
    const int64_t tiles = (int64_t)p.row_tiles * p.col_tiles;
    auto splits_for = [&](int64_t slots) {
      int splits = 1;
      while (splits < 4 && tiles * splits * 2 <= slots && p.chunks >= splits * 2 * 4) splits *= 2;
      return splits;
    };
    const bool two = p.block_rows * kTallPitch * 4 <= kSmemLimitTwo - 1024 &&
                     (p.block_rows <= 64 || tiles * splits_for(ctx->sm_count) * 5 < ctx->sm_count * 4);
    p.splits = splits_for((int64_t)ctx->sm_count * (two ? 2 : 1));
    const int stage = (p.block_rows + 128) * kChunkBytes, limit = two ? kSmemLimitTwo : kSmemLimit;
    p.stages = std::min(kMaxStages, (limit - 1024) / stage);
    p.columns = p.block_rows <= 32 ? 32 : p.block_rows <= 64 ? 64 : p.block_rows <= 128 ? 128 : 256;
    p.group = p.row_tiles;
    blocks = (int)(tiles * p.splits);
    smem = 1024 + std::max(p.stages * stage, p.block_rows * kTallPitch * 4);
  } else {
    p.block_rows = 128;
    p.half_tiles = (int)((q.M + 255) / 256);
    p.row_tiles = (grad_w ? 2 : 1) * p.half_tiles;
    const int64_t slots = ctx->sm_count / 2;
    // The width that takes the least time in rounds over the GPU (a chunk of K: 0.23 us at width 128, 0.27 at 192, 0.36 at 256;
    // a tile 2 us more, 5 where it is split along K).  Tiles that fill less than half of the GPU are split.
    int64_t best = INT64_MAX;
    for (int cols = 128; cols >= 64; cols -= gate ? 64 : 32) {
      const int64_t outputs = gate ? cols : 2 * cols, tiles = p.row_tiles * ((q.N + outputs - 1) / outputs);
      int splits = 1;
      while (splits < 4 && tiles * splits * 2 <= slots && p.chunks >= splits * 2 * 4) splits *= 2;
      const int64_t waves = (tiles * splits + slots - 1) / slots;
      const int width = 2 * cols, chunk = std::max(210 + width / 5, width * 139 / 100) * (1256 - width) / 1000;
      const int64_t cost = waves * ((int64_t)(p.chunks + splits - 1) / splits * chunk + (splits > 1 ? 5000 : 2000));
      if (cost < best) {
        best = cost;
        p.block_cols = cols;
        p.splits = splits;
      }
    }
    const int outputs = (gate ? 1 : 2) * p.block_cols;
    p.col_tiles = (int)((q.N + outputs - 1) / outputs);
    p.group = (int)std::max<int64_t>(1, std::min<int64_t>(p.row_tiles, (48ll << 20) / ((int64_t)p.chunks * kChunkBytes * 256)));
    const int stage = 128 * kChunkBytes + (trans_b ? (p.block_cols + 63) / 64 * 8192 : p.block_cols * kChunkBytes);
    const int staging = p.splits > 1 ? 0 : kStaging;
    p.stages = std::min(kMaxStages, (kSmemLimit - 1024 - staging) / stage);
    p.accumulators = p.splits == 1 ? 2 : 1;
    p.columns = 256 * p.accumulators;
    const int64_t tiles = (int64_t)p.row_tiles * p.col_tiles;
    blocks = (int)(p.splits > 1 ? tiles * p.splits : std::min(tiles, slots)) * 2;
    smem = 1024 + std::max(p.stages * stage + staging, p.splits > 1 ? 128 * kWidePitch * 4 : 0);
  }

  CUtensorMap a, b[2], o[3];
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  const int type = codes ? -1 : q.dtype, bytes = codes ? 1 : 2;
  bool ok;
  if (grad_w) {
    ok = make_map_2d(&a, type, q.A, 2 * q.half, q.K, q.lda * 2, 64) && make_map_2d(&b[0], type, q.B[0], q.N, q.K, q.ldb[0] * 2, 64);
    b[1] = b[0];
  } else {
    const int b_rows = trans_b ? 64 : p.block_cols;
    ok = make_map_2d(&a, type, q.A, q.kind == kInputGrad ? 2 * q.half : q.K, q.M, q.lda * bytes, p.block_rows);
    for (int k = 0; ok && k < (q.B[1] ? 2 : 1); k++)
      ok = make_map_2d(&b[k], type, q.B[k], trans_b ? q.N : q.K, trans_b ? q.K : q.N, q.ldb[k] * bytes, b_rows);
    if (!q.B[1]) b[1] = b[0];
  }
  if (!tall) {
    const CUtensorMap* any = nullptr;
    for (int k = 0; ok && k < 3; k++) {
      if (!q.O[k]) continue;
      ok = make_map_2d(&o[k], q.dtype, q.O[k], q.N, q.M, q.ldo[k] * 2, 32);
      any = &o[k];
    }
    for (int k = 0; ok && k < 3; k++)
      if (!q.O[k]) o[k] = *any;  // not used
  }
  WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  switch (q.kind) {
    case kInt8: return tall ? launch_tall<kInt8>(ctx, a, b, p, blocks, smem, st) : launch_wide<kInt8>(ctx, a, b, o, p, blocks, smem, st);
    case kInt8Gated:
      return tall ? launch_tall<kInt8Gated>(ctx, a, b, p, blocks, smem, st) : launch_wide<kInt8Gated>(ctx, a, b, o, p, blocks, smem, st);
    case kGated: return tall ? launch_tall<kGated>(ctx, a, b, p, blocks, smem, st) : launch_wide<kGated>(ctx, a, b, o, p, blocks, smem, st);
    case kInputGrad:
      return tall ? launch_tall<kInputGrad>(ctx, a, b, p, blocks, smem, st) : launch_wide<kInputGrad>(ctx, a, b, o, p, blocks, smem, st);
    default: return launch_wide<kWeightGrad>(ctx, a, b, o, p, blocks, smem, st);
  }
}

}  // namespace windq
