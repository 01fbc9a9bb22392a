// Tokens times the weights of a feed-forward block on the tensor cores (tcgen05, accumulators in tensor memory, operands by
// TMA), with what follows a product done on its accumulators: scales of codes, the gate, the rounding.
//
// A tile is 256 rows of weights x up to 256 tokens on a pair of thread blocks (cta_group::2: each holds half of either operand, so
// that a block's shared memory feeds a product twice as large).  The weights are the rows of the accumulators and the tokens their
// columns because the tokens are what is ragged: a tile takes as many as there are, in steps of 32, where rows come in 256 (777
// tokens x 2 x 13821 x 5120: 193 us, with the tokens as rows 209).  A gated tile has both products of the same 128 outputs, 16 rows
// of one weight and 16 of the other in turns: a storing warp's 32 lanes hold g and u of 16 outputs, and read as 16 x 8 fragments a
// thread has both in its registers.
//
// Outputs leave transposed, [token][output]: fragments go to shared memory by stmatrix.trans and on by TMA.
//
// Persistent over tiles with two accumulators, so that storing a tile overlaps the next.  Tiles that do not fill the GPU are cut along
// K into equal shares, one a pair, where that saves more than it costs.  The pieces of a tile then go to scratch memory, and a second
// kernel adds them, in order, and finishes the tile: nobody waits for another, and equal calls give equal bits.  (Tiles shared by a
// cluster, with sums through distributed shared memory, came out slower: clusters of eight whole SMs fill few of a GPC's.  So did one
// block that adds all of a tile's pieces: 100 tokens x 1024 x 4096 codes 19.5 us, now 10.)
//
// What bounds it: from about 2000 tokens on power (8192 x 14336 x 4096 codes: 305 us in a burst, 338 in a long run), below that the
// copies from L2 (32 KB a chunk of K and block at 256 tokens, 13 TB/s over the GPU) and rounds that are not full.
//
// Warps: one issues TMA copies, one issues matrix products, four or eight read the accumulators and store, 64 tokens a group of four
// at a time.  A block sets itself up, and brings its first weights
// into L2, while the stream's kernel before ends, where that leaves room on the SM.
#include <algorithm>

#include "feed_forward.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kMaxThreads = 64 + 2 * 128;      // the copying and the issuing warp, one or two groups of four that store
constexpr int kMaxStages = 12;
constexpr int kSmemLimit = 227 * 1024 - 2048;  // dynamic shared memory of one thread block per SM
constexpr int kChunkBytes = 128;               // of K: 64 16-bit values or 128 codes
constexpr int kWeightBytes = 128 * kChunkBytes;
constexpr int kBoxBytes = 64 * 128;            // of a store: up to 64 tokens x 64 outputs
constexpr int kBoxes = 2, kBoxesSaved = 3;     // of a set (three: H, g and u); there are two sets
constexpr int kMaxPairs = 74;
constexpr int kLeastShare = 4;                 // chunks of K a pair, where tiles are cut

struct Args {
  int T, N, dtype, act;
  int chunks, half_chunks;      // of K; of the first weight (kInputGrad)
  int tokens;                   // of a tile
  int token_tiles, weight_tiles, group;
  int pairs;
  bool cut;                     // tiles, along K, into a share for each pair; otherwise whole ones are dealt out
  int stages;
  const float* row_scale;
  const float* col_scale[2];
  const uint32_t* top;
  void* O[3];
  int64_t ldo[3];
  uint32_t* partials;
  Stalls stalls;
};

struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], done[2], free[2];
};

// Tiles in an order that keeps a group of token tiles in L2 while the weights stream by.
__device__ __forceinline__ void tile_at(const Args& p, int tile, int& tt, int& wt) {
  const int per = p.group * p.weight_tiles, g = tile / per, rest = tile - g * per;
  const int rows = min(p.group, p.token_tiles - g * p.group);
  wt = rest / rows;
  tt = g * p.group + rest - wt * rows;
}

// Cut tiles as units of a chunk of a tile, tile by tile: where the share of pair i begins.
__device__ __forceinline__ int share(const Args& p, int i) { return (int)((int64_t)p.token_tiles * p.weight_tiles * p.chunks * i / p.pairs); }
// Where a pair's piece lies: its share has at most two, the first, and one that begins a tile later.  As the threads hold it: 32
// tokens as eight times 16 bytes a lane of the accumulators.
__device__ __forceinline__ uint32_t* piece_of(const Args& p, int pair, int later, int me) {
  return p.partials + ((int64_t)(2 * pair + later) * 2 + me) * p.tokens * 128;
}

// What a pair does, in order; every warp walks through the same.
struct Walk {
  const Args& p;
  const int pair;
  int begin = 0, at = 0, end = 0;  // of its share of units
  int next_tile;                   // of its whole tiles
  int tile, c0, c1;                // now
  __device__ explicit Walk(const Args& p) : p(p), pair(blockIdx.x >> 1), next_tile(blockIdx.x >> 1) {
    if (p.cut) {
      at = begin = share(p, pair);
      end = share(p, pair + 1);
    }
  }
  __device__ __forceinline__ bool next() {
    if (p.cut) {
      if (at >= end) return false;
      tile = at / p.chunks;
      c0 = at - tile * p.chunks;
      c1 = min(p.chunks, end - tile * p.chunks);
      at += c1 - c0;
      return true;
    }
    tile = next_tile;
    next_tile += p.pairs;
    c0 = 0;
    c1 = p.chunks;
    return tile < p.token_tiles * p.weight_tiles;
  }
  __device__ __forceinline__ bool later() const { return tile * p.chunks + c0 != begin; }
};

// The four warps of a group that stores.
__device__ __forceinline__ void barrier(int group) { asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory"); }

// 16 lanes x 32 columns of accumulators: of every 8 columns a thread has lanes t / 4 and t / 4 + 8, columns 2 (t % 4) and the next.
__device__ __forceinline__ void tmem_load_fragments(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
// 16 outputs x 32 tokens as fragments x to a box in shared memory, [token][64 outputs] with the 128-byte swizzle: tokens from c
// on, outputs from 8 * chunk on.
__device__ __forceinline__ void put_fragments(uint32_t box, int c, int chunk, int lane, int dtype, const float (&x)[16]) {
#pragma unroll
  for (int h = 0; h < 2; h++) {
    uint32_t w[4];
#pragma unroll
    for (int m = 0; m < 4; m++) w[m] = pack2(x[8 * h + 2 * m], x[8 * h + 2 * m + 1], dtype);
    const int token = c + 16 * h + 8 * (lane >> 4) + (lane & 7), at = chunk + ((lane >> 3) & 1);
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(box + token * 128 + ((at ^ (token & 7)) << 4)),
                 "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                 : "memory");
  }
}
// A box of finished values to O: outputs n0 .. n0 + 63, tokens t0 .. t0 + live - 1; by the storing threads, of whom the first issues.
__device__ __forceinline__ void send_box(const Args& p, uint32_t box, int k, const CUtensorMap* map, int n0, int t0, int live, int thread) {
  if (n0 + 64 <= p.N || p.N % 8 == 0) {
    if (thread == 0 && n0 < p.N) {
      tma_store_2d(map, n0, t0, box);
      if (live > 32) tma_store_2d(map, n0, t0 + 32, box + 32 * 128);
    }
    return;
  }
  // not by TMA: a box that ends in the middle of 16 bytes, which the copy would write whole
  const int n = n0 + (thread & 63);
  for (int i = thread >> 6; i < min(live, 64); i += 2) {
    uint16_t v;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(box + i * 128 + ((((thread & 63) >> 3) ^ (i & 7)) << 4) + (thread & 7) * 2) : "memory");
    if (n < p.N) static_cast<uint16_t*>(p.O[k])[(t0 + i) * p.ldo[k] + n] = v;
  }
}

// 32 tokens of a warp's accumulators, from column d on: 16 lanes, and the 16 others.
__device__ __forceinline__ void load_unit(uint32_t d, uint32_t (&r)[2][16]) {
  tmem_load_fragments(d, r[0]);
  tmem_load_fragments(d + (16u << 16), r[1]);
}
template <bool CODES>
__device__ __forceinline__ void add_quad(uint32_t* x, const uint4& y) {
  const uint32_t v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int e = 0; e < 4; e++) x[e] = CODES ? x[e] + v[e] : __float_as_uint(__uint_as_float(x[e]) + __uint_as_float(v[e]));
}

// What is done with whole sums, by a group of four storing warps.  (Scales are not read by __ldg, which wants memory that nothing writes
// while the kernel lives: the kernel before may still have been writing them when this one came.)
template <int KIND>
struct Finish {
  using K = Kind<KIND>;
  const Args& p;
  const CUtensorMap *omap0, *omap1, *omap2;
  uint32_t boxes;        // the set in use
  const int other;       // from it to the other one, which a group of its own takes in turns with it
  const int group, thread, lane, quarter;
  const bool saved, wanted;
  const float unscale;
  int flip = other;
  int n0, t0, tokens;  // of the tile
  float col[2][2];
  __device__ Finish(const Args& p, const CUtensorMap* o0, const CUtensorMap* o1, const CUtensorMap* o2, uint32_t sets, int groups, int group, int first)
      : p(p), omap0(o0), omap1(o1), omap2(o2), boxes(sets + group * set_bytes(p)), other(groups == 1 ? set_bytes(p) : 0), group(group),
        thread(threadIdx.x - first), lane(threadIdx.x & 31), quarter((threadIdx.x >> 5) & 3),
        saved(KIND == kGated && p.O[1]), wanted(KIND != kGated || p.O[0]), unscale(p.top ? gradient_power(*p.top, -1) : 1.0f) {}
  static __device__ __forceinline__ int set_bytes(const Args& p) { return (KIND == kGated && p.O[1] ? kBoxesSaved : kBoxes) * kBoxBytes; }
  __device__ __forceinline__ void open(int tile, int me) {
    int tt, wt;
    tile_at(p, tile, tt, wt);
    t0 = tt * p.tokens;
    tokens = min(p.tokens, p.T - t0);
    n0 = (2 * wt + me) * (K::kGate ? 64 : 128);
    // the thread's rows: two of each half of the warp's lanes, outputs 8 apart; gated, the halves are the two weights' same outputs
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int e = 0; e < 2; e++) {
        const int n = n0 + (K::kGate ? quarter * 16 : quarter * 32 + h * 16) + e * 8 + (lane >> 2);
        col[h][e] = K::kCodes && n < p.N ? p.col_scale[K::kGate ? h : 0][n] : 0.0f;
      }
  }
  // `units` times 32 tokens of the tile from c on.
  template <int UNITS>
  __device__ __forceinline__ void put(const uint32_t (&r)[UNITS][2][16], int c, int units) {
    if (thread == 0) {  // what was sent from this set before has been read
      if (other) tma_store_wait<1>();
      else tma_store_wait<0>();
    }
    barrier(group);
#pragma unroll
    for (int u = 0; u < UNITS; u++) {
      if (u >= units) break;
      float row[8], x[2][16];
#pragma unroll
      for (int k = 0; k < 8; k++) {
        const int t = t0 + c + u * 32 + (k >> 1) * 8 + (lane & 3) * 2 + (k & 1);
        row[k] = K::kCodes ? (t < p.T ? p.row_scale[t] : 0.0f) : unscale;
      }
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int k = 0; k < 16; k++) x[h][k] = value_of<K::kCodes>(r[u][h][k], row[(k >> 2) * 2 + (k & 1)], col[h][(k >> 1) & 1]);
      if (K::kGate) {
        if (saved) {
          put_fragments(boxes + kBoxBytes, u * 32, quarter * 2, lane, p.dtype, x[0]);
          put_fragments(boxes + 2 * kBoxBytes, u * 32, quarter * 2, lane, p.dtype, x[1]);
        }
        if (wanted) {
#pragma unroll
          for (int k = 0; k < 16; k++) x[0][k] = gated(x[0][k], x[1][k], p.act);
          put_fragments(boxes, u * 32, quarter * 2, lane, p.dtype, x[0]);
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; h++) put_fragments(boxes + (quarter >> 1) * kBoxBytes, u * 32, (quarter & 1) * 4 + h * 2, lane, p.dtype, x[h]);
      }
    }
    fence_async_shared();
    barrier(group);
    const int t = t0 + c, live = min(tokens - c, units * 32);
    if (K::kGate) {
      if (wanted) send_box(p, boxes, 0, omap0, n0, t, live, thread);
      if (saved) {
        send_box(p, boxes + kBoxBytes, 1, omap1, n0, t, live, thread);
        send_box(p, boxes + 2 * kBoxBytes, 2, omap2, n0, t, live, thread);
      }
    } else {
      send_box(p, boxes, 0, omap0, n0, t, live, thread);
      send_box(p, boxes + kBoxBytes, 0, omap0, n0 + 64, t, live, thread);
    }
    if (thread == 0) tma_store_commit();
    boxes += flip;
    flip = -flip;
  }
};

template <int KIND>
__global__ void __launch_bounds__(kMaxThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap0,
                   const __grid_constant__ CUtensorMap wmap1, const __grid_constant__ CUtensorMap omap0,
                   const __grid_constant__ CUtensorMap omap1, const __grid_constant__ CUtensorMap omap2,
                   const __grid_constant__ Args p) {
  using K = Kind<KIND>;
  extern __shared__ uint8_t raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t me = cluster_rank();
  const uint32_t stage_bytes = kWeightBytes + p.tokens / 2 * kChunkBytes;
  const uint32_t dead_ = smem_addr(&dead);
  auto full = [&](int s) { return smem_addr(&bars.full[s]); };
  auto empty = [&](int s) { return smem_addr(&bars.empty[s]); };
  auto done = [&](int b) { return smem_addr(&bars.done[b]); };
  auto free_ = [&](int b) { return smem_addr(&bars.free[b]); };

  if (threadIdx.x == 0) {
    prefetch_map(&xmap);
    prefetch_map(&wmap0);
    prefetch_map(&wmap1);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int b = 0; b < 2; b++) {
      mbar_init(done(b), 1);
      mbar_init(free_(b), 2 * (blockDim.x / 32 - 2));
    }
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<true>(smem_addr(&tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the other block's barriers are ready
  tc_fence_after();
  launch_dependents();  // tensor memory is in hand
  const uint32_t tmem = tmem_slot, boxes = base + p.stages * stage_bytes;

  if (warp == 0) {
    int tt, wt, n0;
    auto open = [&](int tile) {
      tile_at(p, tile, tt, wt);
      n0 = (2 * wt + me) * (K::kGate ? 64 : 128);
    };
    auto weights = [&](int c, auto take) {  // the boxes of a chunk: where in the stage, and where from
      if (K::kTransposed) {
        int k = c;
        bool other = false;
        for (; k >= p.half_chunks; k -= p.half_chunks) other = !other;  // the weights again for the second terms
        for (int b = 0; b < 2; b++) take(b * 8192, other ? &wmap1 : &wmap0, n0 + b * 64, k * 64);
      } else if (K::kGate) {
#pragma unroll
        for (int b = 0; b < 4; b++) {
          take(b * 4096, &wmap0, c * K::kStepK, n0 + b * 16);
          take(b * 4096 + 2048, &wmap1, c * K::kStepK, n0 + b * 16);
        }
      } else {
        take(0, &wmap0, c * K::kStepK, n0);
      }
    };
    {
      Walk first(p);
      first.next();
      open(first.tile);
      if (elect_one())
        for (int c = first.c0; c < min(first.c1, first.c0 + p.stages); c++)
          weights(c, [&](int, const CUtensorMap* map, int x, int y) { tma_prefetch_2d(map, x, y); });
      __syncwarp();
    }
    wait_for_predecessor();
    Ring at(p.stages);
    const uint32_t to = cluster_addr(full(0), 0);  // barriers of the issuing block
    for (Walk walk(p); walk.next();) {
      open(walk.tile);
      const int t0 = tt * p.tokens + me * (p.tokens / 2);
      for (int c = walk.c0; c < walk.c1; c++) {
        mbar_wait(empty(at.s), at.phase ^ 1, dead_);
        const uint32_t dst = base + at.s * stage_bytes, bar = to + at.s * 8;
        if (elect_one() && !*(volatile int*)&dead) {
          if (me == 0) mbar_expect(full(at.s), 2 * stage_bytes);
          weights(c, [&](int at, const CUtensorMap* map, int x, int y) { tma_load_2d<true>(dst + at, map, x, y, bar); });
          tma_load_2d<true>(dst + kWeightBytes, &xmap, c * K::kStepK, t0, bar);
        }
        __syncwarp();
        at.next();
      }
    }
  } else if (warp == 1) {
    wait_for_predecessor();
    if (me == 0) {
      const uint32_t idesc = K::kCodes ? instr_desc_i8(256, p.tokens) : instr_desc(p.dtype, K::kTransposed, false, 256, p.tokens);
      // a step of K further: 32 bytes in a K-major tile, two groups of 8 rows in an MN-major one
      constexpr uint32_t w_step = (K::kTransposed ? 2048 : 32) >> 4, x_step = 32 >> 4;
      const uint64_t w_desc = smem_desc(base, K::kTransposed ? 8192 : 16), x_desc = smem_desc(base + kWeightBytes, 16);
      Ring at(p.stages);
      int turn = 0;
      for (Walk walk(p); walk.next(); turn++) {
        const int b = turn & 1;
        mbar_wait(free_(b), ((turn >> 1) & 1) ^ 1, dead_);
        tc_fence_after();
        const uint32_t d = tmem + b * 256;
        for (int c = walk.c0; c < walk.c1; c++) {
          mbar_wait(full(at.s), at.phase, dead_);
          tc_fence_after();
          const uint64_t off = (uint64_t)(at.s * stage_bytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; k++) {
              if (K::kCodes) mma_i8<true>(d, w_desc + off + k * w_step, x_desc + off + k * x_step, idesc, c > walk.c0 || k > 0);
              else mma_f16<true>(d, w_desc + off + k * w_step, x_desc + off + k * x_step, idesc, c > walk.c0 || k > 0);
            }
            mma_commit<true>(empty(at.s), 3);
          }
          __syncwarp();
          at.next();
        }
        if (elect_one()) mma_commit<true>(done(b), 3);
        __syncwarp();
      }
    }
  } else {
    wait_for_predecessor();
    const int group = (warp - 2) >> 2, groups = (blockDim.x - 64) / 128;
    Finish<KIND> out(p, &omap0, &omap1, &omap2, boxes, groups, group, 64 + group * 128);
    int turn = 0;
    for (Walk walk(p); walk.next(); turn++) {
      const int b = turn & 1;
      const uint32_t d = tmem + b * 256 + ((uint32_t)(out.quarter * 32) << 16);
      out.open(walk.tile, me);
      mbar_wait(done(b), (turn >> 1) & 1, dead_);
      tc_fence_after();
      if (walk.c1 - walk.c0 == p.chunks) {
        for (int c = group * 64; c < out.tokens; c += groups * 64) {
          const int units = c + 32 < out.tokens ? 2 : 1;
          uint32_t r[2][2][16];
#pragma unroll
          for (int u = 0; u < 2; u++)
            if (u < units) load_unit(d + c + u * 32, r[u]);
          tmem_load_wait();
          out.put(r, c, units);
        }
      } else {
        uint32_t* piece = piece_of(p, walk.pair, walk.later(), me) + (out.quarter * 32 + lane) * 4;
        for (int c = group * 32; c < out.tokens; c += groups * 32) {
          uint32_t r[2][16];
          load_unit(d + c, r);
          tmem_load_wait();
#pragma unroll
          for (int k = 0; k < 8; k++) {
            const uint32_t* x = &r[k >> 2][(k & 3) * 4];
            __stcg(reinterpret_cast<uint4*>(piece + c * 128 + k * 512), make_uint4(x[0], x[1], x[2], x[3]));
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) cluster_arrive(cluster_addr(free_(b), 0));
    }
    if (out.thread == 0) tma_store_wait<0>();
  }
  __syncwarp();
  __syncthreads();
  if (dead) settle(p.stalls);
  __syncwarp();
  cluster_sync();  // no more arrivals from the other block
  if (warp == 1) {
    tc_fence_after();
    tmem_free<true>(tmem, 512);
  }
}

// Adds the pieces of the cut tiles and finishes them: one block for 32 tokens of a block's half of a tile.
template <int KIND>
__global__ void __launch_bounds__(128)
    combine_kernel(const __grid_constant__ CUtensorMap omap0, const __grid_constant__ CUtensorMap omap1,
                   const __grid_constant__ CUtensorMap omap2, const __grid_constant__ Args p) {
  __shared__ __align__(1024) uint8_t boxes[kBoxesSaved * kBoxBytes];
  const int me = blockIdx.x & 1, tile = blockIdx.x >> 1, c = blockIdx.y * 32, s = tile * p.chunks;
  launch_dependents();
  wait_for_predecessor();
  Finish<KIND> out(p, &omap0, &omap1, &omap2, smem_addr(boxes), 2, 0, 0);
  out.open(tile, me);
  int q = (int)((int64_t)p.pairs * tile / (p.token_tiles * p.weight_tiles));  // near the pair that holds the first unit
  while (share(p, q + 1) <= s) q++;
  while (share(p, q) > s) q--;
  if (share(p, q + 1) >= s + p.chunks || c >= out.tokens) return;  // one pair had all of it; or no such tokens
  uint32_t r[1][2][16];
#pragma unroll
  for (int k = 0; k < 32; k++) r[0][k >> 4][k & 15] = 0;
  bool more = true;
  while (more) {
    uint4 y[4][8];
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (!more) break;
      const int begin = share(p, q);
      const uint4* from = reinterpret_cast<const uint4*>(piece_of(p, q, begin < s, me) + c * 128 + threadIdx.x * 4);
#pragma unroll
      for (int k = 0; k < 8; k++) y[i][k] = __ldcg(from + k * 128);
      q++;
      n++;
      more = share(p, q) < s + p.chunks;
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) {
#pragma unroll
        for (int k = 0; k < 8; k++) add_quad<Kind<KIND>::kCodes>(&r[0][k >> 2][(k & 3) * 4], y[i][k]);
      }
  }
  out.put(r, c, 1);
  if (out.thread == 0) tma_store_wait<0>();
}

// How the tokens are tiled, and whether the tiles are cut.
struct Plan {
  int tokens, pairs;
  bool cut;
};

// The way that takes the least time.  A chunk of K takes max(200, 110 + tokens) ns: the copies from L2.  Whole tiles take rounds over
// the pairs; up to three more token tiles than there need to be, narrower ones, may fill a round better (200 tokens x 2 x 4096 x 4096
// 25.2 -> 23.2 us, 1500 x 4096 x 4096 codes 34.0 -> 29.5, 600 x 2048 x 8192 codes, which then need no cutting, 30.3 -> 23.1), but mostly
// do not where there are several (777 tokens x 2 x 13821 x 5120 in five tiles 208 us, in four 194).  Cutting, below one round, gives every
// pair an equal share and costs another kernel, about 8 us with what it starts up, and the pieces' way to memory and back, two for a
// pair at most (333 tokens x 2048 x 16382: 30 + 7 us instead of 70); with a whole round and more it loses, because pairs at different
// places of K do not meet in L2 (8192 x 14336 x 4096 codes: 356 us instead of 339).
Plan plan_of(int64_t T, int64_t weight_tiles, int64_t chunks, int64_t slots) {
  const int64_t least = std::max<int64_t>(1, (T + 255) / 256);
  Plan best = {};
  int64_t best_cost = INT64_MAX;
  for (int64_t n = least; n < least + 4; n++) {
    const int64_t tokens = std::max<int64_t>(round_up((T + n - 1) / n, 32), 32), tiles = (T + tokens - 1) / tokens * weight_tiles;
    if (n > least && tokens == best.tokens) continue;
    const int64_t chunk = std::max<int64_t>(200, 110 + tokens), rounds = (tiles + slots - 1) / slots;
    const int64_t whole = 2000 + rounds * (chunks * chunk + 1000);
    if (whole < best_cost - best_cost / 20) {
      best = {(int)tokens, (int)std::min(tiles, slots), false};
      best_cost = whole;
    }
    if (tiles >= slots) continue;
    const int64_t pairs = std::min(slots, std::max(tiles, tiles * chunks / kLeastShare));
    const int64_t cut = (tiles * chunks + pairs - 1) / pairs * chunk + 8000 + (pairs + tiles) * tokens / 2;
    if (pairs > tiles && cut < best_cost - best_cost / 20) {
      best = {(int)tokens, (int)pairs, true};
      best_cost = cut;
    }
  }
  return best;
}

template <int KIND>
windq_status launch(windq_ctx* ctx, const CUtensorMap& x, const CUtensorMap (&w)[2], const CUtensorMap (&o)[3], const Args& p, int blocks,
                    int threads, int smem, cudaStream_t st) {
  const windq_status ready = prepare_kernel(ctx, kProduct + KIND, product_kernel<KIND>, kMaxThreads, kSmemLimit, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  overlapped_launch(cfg, attrs, blocks, threads, 2, smem, st);
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, product_kernel<KIND>, x, w[0], w[1], o[0], o[1], o[2], p));
  if (p.cut) {
    cudaLaunchConfig_t second = {};
    overlapped_launch(second, attrs, p.token_tiles * p.weight_tiles * 2, 128, 1, 0, st);
    second.gridDim.y = (p.tokens + 31) / 32;
    WINDQ_CUDA(ctx, cudaLaunchKernelEx(&second, combine_kernel<KIND>, o[0], o[1], o[2], p));
  }
  return WINDQ_OK;
}

}  // namespace

int64_t product_scratch(int64_t T) {  // never less for more tokens
  const int64_t tokens = std::min<int64_t>(std::max<int64_t>(round_up(T, 32), 32), 256);
  return round_up((int64_t)kMaxPairs * 2 * 2 * tokens * 128 * 4, 256);
}

windq_status launch_product(windq_ctx* ctx, const Product& q, cudaStream_t st) {
  const bool codes = q.kind == kInt8 || q.kind == kInt8Gated, gate = q.kind == kInt8Gated || q.kind == kGated;
  if (q.T <= (gate ? kMostFewGated : kMostFew)) return launch_few_tokens(ctx, q, st);
  const bool transposed = q.kind == kInputGrad;
  const int step = codes ? 128 : 64;
  Args p = {};
  p.T = (int)q.T;
  p.N = (int)q.N;
  p.dtype = q.dtype;
  p.act = q.act;
  p.half_chunks = (int)((q.K + step - 1) / step);
  p.chunks = transposed ? q.terms * 2 * p.half_chunks : p.half_chunks;
  const int outputs = gate ? 128 : 256;
  p.weight_tiles = (int)((q.N + outputs - 1) / outputs);
  const Plan plan = plan_of(q.T, p.weight_tiles, p.chunks, std::min(ctx->sm_count / 2, kMaxPairs));
  p.tokens = plan.tokens;
  p.pairs = plan.pairs;
  p.cut = plan.cut;
  p.token_tiles = (int)((q.T + p.tokens - 1) / p.tokens);
  // 24 MB of tokens: 4096 x 4096 x 22016 and its weights' gradients together 1205 us, with 48 MB 1240, with 96 1305
  p.group = (int)std::max<int64_t>(1, std::min<int64_t>(p.token_tiles, (24ll << 20) / ((int64_t)p.chunks * kChunkBytes * p.tokens)));
  p.row_scale = q.row_scale;
  p.top = q.top;
  for (int k = 0; k < 2; k++) p.col_scale[k] = q.col_scale[k];
  for (int k = 0; k < 3; k++) p.O[k] = q.O[k], p.ldo[k] = q.ldo[k];
  p.partials = (uint32_t*)q.partials;
  p.stalls = stalls_of(ctx);

  const int stage = kWeightBytes + p.tokens / 2 * kChunkBytes, extra = 2 * (q.kind == kGated && q.O[1] ? kBoxesSaved : kBoxes) * kBoxBytes;
  p.stages = std::min(kMaxStages, (kSmemLimit - 1024 - extra) / stage);
  // Of a short K storing a tile takes longer than its products: two groups of warps then (3000 tokens x 2 x 8192 x 2048 codes 107 ->
  // 94 us, 700 x 2048 x 2048 16.4 -> 14.8).  Of a long one they only draw power (4096 x 2 x 8192 x 2048, 16 bits, 204 -> 208).
  const int threads = p.chunks <= (codes ? 16 : 8) ? 64 + 256 : 64 + 128;
  const int smem = kSmemLimit;  // all of it, whatever is used: no block that wants tensor memory fits beside this one

  CUtensorMap x, w[2], o[3];
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  const int type = codes ? -1 : q.dtype, bytes = codes ? 1 : 2;
  bool ok = make_map_2d(&x, type, q.X, transposed ? q.terms * 2 * q.half : q.K, q.T, q.ldx * bytes, p.tokens / 2);
  for (int k = 0; ok && k < (q.W[1] ? 2 : 1); k++)
    ok = transposed ? make_map_2d(&w[k], type, q.W[k], q.N, q.K, q.ldw[k] * bytes, 64)
                    : make_map_2d(&w[k], type, q.W[k], q.K, q.N, q.ldw[k] * bytes, gate ? 16 : 128);
  if (!q.W[1]) w[1] = w[0];
  const CUtensorMap* any = nullptr;
  for (int k = 0; ok && k < 3; k++) {
    if (!q.O[k]) continue;
    ok = make_map_2d(&o[k], q.dtype, q.O[k], q.N, q.T, q.ldo[k] * 2, 32);
    any = &o[k];
  }
  WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  for (int k = 0; k < 3; k++)
    if (!q.O[k]) o[k] = *any;  // not used
  switch (q.kind) {
    case kInt8: return launch<kInt8>(ctx, x, w, o, p, p.pairs * 2, threads, smem, st);
    case kInt8Gated: return launch<kInt8Gated>(ctx, x, w, o, p, p.pairs * 2, threads, smem, st);
    case kGated: return launch<kGated>(ctx, x, w, o, p, p.pairs * 2, threads, smem, st);
    default: return launch<kInputGrad>(ctx, x, w, o, p, p.pairs * 2, threads, smem, st);
  }
}

}  // namespace windq
