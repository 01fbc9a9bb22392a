// The product of the adapter calls: tokens times the shared weight, plus every token's low-rank term, in one kernel on
// the tensor cores (tcgen05, accumulators in tensor memory, operands by TMA).
//
// A low-rank term is more reduction dimension: after the chunks of K the accumulator takes, for every adapter a that the
// tile's tokens use, S (tokens x rank, zero in the rows of other tokens' adapters) times P[a].  So a tile whose tokens
// share an adapter costs rank / K more than the bare product, any mix of adapters is right, and there is no second pass
// over the output.  S enters as the sum of two 16-bit values (22 bits for fp16, 16 for bf16; written by the low-rank
// kernel), which keeps the rounding of the low-rank term below that of the result.
//
// fp16 pairs of tokens whose S is very small or large are scaled by a power of two (shift_of in the low-rank kernel).  In a
// tile that has such tokens the adapters come after all of K, and between the two the accumulators are multiplied by the same
// powers, token by token (exact, in tensor memory, by the warps that store); storing takes them off again.
//
// The low-rank stages come in the second half of a tile's reduction, one adapter after each chunk of K: their handshakes and
// loads then hide behind the chunks' (at the end of 203 tokens with 48 adapters they took 14 us of 75), and the low-rank
// kernel, which this one overlaps at its start, has long ended.
//
// Warps: one issues TMA copies, one issues matrix products, four write the S tiles and, after the tile, read the
// accumulators and store.  Two layouts of a tile:
//   wide  256 tokens x up to 256 outputs on a pair of thread blocks (cta_group::2: each holds half of either operand, so
//         that a block's shared memory feeds a product twice as large); persistent over tiles with two accumulators, so
//         that storing a tile overlaps the next
//   tall  (few tokens) 128 outputs x up to 256 tokens: the weight is read once and the tokens cost little -- the shape of
//         decoding, bound by the bytes of W
// Where the tiles do not fill the GPU, `splits` thread blocks (a cluster) share a tile along K and add their
// accumulators through distributed shared memory, in rank order: equal calls give equal bits.
#include <algorithm>

#include "lora.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kThreads = 192;
constexpr int kMaxStages = 8;
constexpr int kSmemLimit = 227 * 1024 - 2048;       // dynamic shared memory of one thread block per SM
constexpr int kTallPitch = 132, kWidePitch = 260;    // binary32 sums of a split tile, rows free of bank conflicts
constexpr int kSmemLimitTwo = 112 * 1024;           // of two
static_assert(kSmemLimitTwo + 2048 <= kProjectShare, "what the low-rank kernel leaves");

struct ProjectArgs {
  int T, N, chunks, rank, n_adapters, dtype;
  const int32_t* adapter_of;
  const uint16_t* pair;
  const int8_t* shift;
  const int* lists;
  void* O;
  int64_t ldo;
  int token_rows, weight_rows, token_tiles, weight_tiles, group;
  int splits, stages, accumulators, columns;  // columns: of tensor memory
  Stalls stalls;
};

struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], granted[kMaxStages], written[kMaxStages], done[2], free[2], whole, shifted;
};

// The adapters of a tile that are this split's, for a converged warp: 32 of them in its lanes at a time (one load from L2 an
// adapter, even when issued one adapter ahead, took longer than the adapter's products).
struct Adapters {
  const int* list;
  int first, step, lane, count = 0, held = 0;
  bool late = false;  // some of the tile's tokens are scaled: the adapters come after all of K
  unsigned shifts[2] = {};  // of four tokens each: 4 lane and 128 + 4 lane of the tile
  __device__ Adapters(const int* list, int first, int step, int lane) : list(list + 1), first(first), step(step), lane(lane) {}
  __device__ __forceinline__ void open(const ProjectArgs& p, int t0, int rows) {  // the tile's tokens
    if (p.shift) {
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int i = (h * 32 + lane) * 4;  // (the low-rank kernel fills the last four up with zeros)
        shifts[h] = i < rows && t0 + i < p.T ? __ldcg(reinterpret_cast<const unsigned*>(p.shift + t0 + i)) : 0;
      }
    }
    const int n = uniform(__ldcg(list - 1));
    count = n > first ? (n - first + step - 1) / step : 0;
    fetch(0);
    late = count > 0 && __any_sync(0xffffffffu, (shifts[0] | shifts[1]) != 0);
  }
  // 2^shift (or, with sign = -1, its inverse) of token `i` of the tile: of one that all lanes agree on, or of each lane's own.
  __device__ __forceinline__ float power(int i, int sign) {
    const int a = __shfl_sync(0xffffffffu, (int)shifts[0], (i >> 2) & 31), b = __shfl_sync(0xffffffffu, (int)shifts[1], (i >> 2) & 31);
    const int shift = (int)(int8_t)((i < 128 ? a : b) >> (8 * (i & 3)));
    return __uint_as_float((uint32_t)(127 + sign * shift) << 23);
  }
  __device__ __forceinline__ void fetch(int k) { held = k + lane < count ? __ldcg(list + first + (k + lane) * step) : 0; }
  __device__ __forceinline__ int at(int k) {
    if (k && (k & 31) == 0) fetch(k);
    return __shfl_sync(0xffffffffu, held, k & 31);
  }
};

// A warp's quarter of the accumulators times the powers of their tokens (sign = 1) or divided by them (-1).  The tokens are the
// columns of a tall tile; of a wide one they are the rows, `token` this thread's.  Out of line, away from what tiles without
// scaled tokens run (in line it cost 48 single tokens with 32 adapters 0.9 us of 29).
template <bool TALL>
__device__ __noinline__ void rescale(Adapters adapters, uint32_t d, int columns, int token, int sign) {
  const float row = adapters.power(token, sign);
#pragma unroll 1
  for (int c = 0; c < columns; c += 16) {
    uint32_t r[16];
    tmem_load16(d + c, r);
    tmem_load_wait();
#pragma unroll
    for (int k = 0; k < 16; k++) r[k] = __float_as_uint(__uint_as_float(r[k]) * (TALL ? adapters.power(c + k, sign) : row));
    tmem_store16(d + c, r);
  }
  tmem_store_wait();
}

// Tiles in an order that keeps a group of token tiles in L2 while the weight streams by.
__device__ __forceinline__ void tile_at(const ProjectArgs& p, int tile, int& tt, int& wt) {
  const int per = p.group * p.weight_tiles, g = tile / per, rest = tile - g * per;
  const int rows = min(p.group, p.token_tiles - g * p.group);
  wt = rest / rows;
  tt = g * p.group + rest - wt * rows;
}

template <bool TALL, bool TRANS>
__global__ void __launch_bounds__(kThreads, TALL ? 2 : 1)
    project_kernel(const __grid_constant__ CUtensorMap zmap, const __grid_constant__ CUtensorMap wmap,
                   const __grid_constant__ CUtensorMap pmap, const __grid_constant__ CUtensorMap omap,
                   const __grid_constant__ ProjectArgs p) {
  extern __shared__ uint8_t raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
  constexpr bool PAIR = !TALL;
  constexpr int kBlocks = PAIR ? 2 : 1;  // thread blocks that share a tile's products
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR || p.splits > 1 ? cluster_rank() : 0, me = PAIR ? rank & 1 : 0, leader = rank & ~1u;
  const uint32_t token_bytes = p.token_rows * 128;
  const int weight_boxes = (p.weight_rows + 63) / 64;  // of a transposed weight
  const uint32_t weight_bytes = TRANS ? weight_boxes * 8192 : p.weight_rows * 128, stage_bytes = token_bytes + weight_bytes;
  const uint32_t dead_ = smem_addr(&dead);
  auto full = [&](int s) { return smem_addr(&bars.full[s]); };
  auto empty = [&](int s) { return smem_addr(&bars.empty[s]); };
  auto granted = [&](int s) { return smem_addr(&bars.granted[s]); };
  auto written = [&](int s) { return smem_addr(&bars.written[s]); };
  auto done = [&](int b) { return smem_addr(&bars.done[b]); };
  auto free_ = [&](int b) { return smem_addr(&bars.free[b]); };
  const uint32_t whole = smem_addr(&bars.whole), shifted = smem_addr(&bars.shifted);

  if (threadIdx.x == 0) {
    prefetch_map(&zmap);
    prefetch_map(&wmap);
    prefetch_map(&pmap);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
      mbar_init(granted(s), 1);
      mbar_init(written(s), 4 * kBlocks);
    }
    for (int b = 0; b < 2; b++) {
      mbar_init(done(b), 1);
      mbar_init(free_(b), 4 * kBlocks);
    }
    mbar_init(whole, 1);
    mbar_init(shifted, 4 * kBlocks);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<PAIR>(smem_addr(&tmem_slot), p.columns);
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();  // the other block's barriers are ready
  tc_fence_after();
  launch_dependents();  // the next call's low-rank kernel may set itself up while the last tiles finish
  const uint32_t tmem = tmem_slot;

  const int team = kBlocks * p.splits;  // thread blocks of a tile
  const int split = (blockIdx.x % team) / kBlocks, step = gridDim.x / team, tiles = p.token_tiles * p.weight_tiles;
  const int c0 = (int)((int64_t)p.chunks * split / p.splits), c1 = (int)((int64_t)p.chunks * (split + 1) / p.splits);
  const int middle = c0 + (c1 - c0) / 2;  // the chunk after which the first adapter comes
  const int rank_chunks = (p.rank + 63) >> 6;
  const bool paired = p.rank <= 32;  // both halves of S in one stage, at columns 0 and 32
  const int parts = paired ? 1 : 2;

  if (warp == 0) {
    Ring at(p.stages);
    const uint32_t to = PAIR ? cluster_addr(full(0), leader) : full(0);  // barriers of the issuing block
    for (int tile = blockIdx.x / team; tile < tiles; tile += step) {
      int tt, wt;
      tile_at(p, tile, tt, wt);
      const int t0 = (tt * kBlocks + me) * p.token_rows, n0 = (wt * kBlocks + me) * p.weight_rows;
      Adapters adapters(p.lists + (int64_t)tt * (kBlocks * p.token_rows + 1), split, p.splits, lane);
      auto load_adapter = [&](int k) {
        const int a = adapters.at(k);
        for (int e = 0; e < rank_chunks * parts; e++, at.next()) {
          const int rc = e / parts;
          mbar_wait(empty(at.s), at.phase ^ 1, dead_);
          const uint32_t dst = base + at.s * stage_bytes + token_bytes, bar = to + at.s * 8;
          if (elect_one() && !*(volatile int*)&dead) {
            mbar_arrive(granted(at.s));  // the stage's token tile is the writers' now
            if (me == 0) mbar_expect(full(at.s), kBlocks * weight_bytes);
            if (TRANS) {
              for (int b = 0; b < weight_boxes; b++) tma_load_3d<PAIR>(dst + b * 8192, &pmap, n0 + b * 64, rc * 64, a, bar);
            } else {
              tma_load_3d<PAIR>(dst, &pmap, rc * 64, n0, a, bar);
            }
          }
          __syncwarp();
        }
      };
      auto load_chunk = [&](int c) {
        mbar_wait(empty(at.s), at.phase ^ 1, dead_);
        const uint32_t dst = base + at.s * stage_bytes, bar = to + at.s * 8;
        if (elect_one() && !*(volatile int*)&dead) {
          if (me == 0) mbar_expect(full(at.s), kBlocks * stage_bytes);
          tma_load_2d<PAIR>(dst, &zmap, c * 64, t0, bar);
          if (TRANS) {
            for (int b = 0; b < weight_boxes; b++) tma_load_2d<PAIR>(dst + token_bytes + b * 8192, &wmap, n0 + b * 64, c * 64, bar);
          } else {
            tma_load_2d<PAIR>(dst + token_bytes, &wmap, c * 64, n0, bar);
          }
        }
        __syncwarp();
        at.next();
      };
      for (int c = c0; c <= middle; c++) load_chunk(c);
      wait_for_predecessor();
      adapters.open(p, tt * kBlocks * p.token_rows, kBlocks * p.token_rows);
      int c = middle + 1;
      if (adapters.late) {
#pragma unroll 1
        for (; c < c1; c++) load_chunk(c);
      }
      for (int k = 0; k < adapters.count; k++) {
        if (k && c < c1) load_chunk(c++);
        load_adapter(k);
      }
      for (; c < c1; c++) load_chunk(c);
    }
  } else if (warp == 1) {
    if (me == 0) {
      const uint32_t idesc = TALL ? instr_desc(p.dtype, TRANS, false, 128, p.token_rows)
                                  : instr_desc(p.dtype, false, TRANS, 256, 2 * p.weight_rows);
      const uint32_t mask = 3u << leader;
      // 16 values of K further: 32 bytes in a K-major tile, two groups of 8 rows in an MN-major one
      constexpr uint32_t weight_step = TRANS ? 2048 >> 4 : 32 >> 4, token_step = 32 >> 4;
      const uint64_t z_desc = smem_desc(base, 16), w_desc = smem_desc(base + token_bytes, TRANS ? 8192 : 16);
      Ring at(p.stages);
      int turn = 0;
      uint32_t written_phase = 0, shifted_phase = 0;
      for (int tile = blockIdx.x / team; tile < tiles; tile += step, turn++) {
        int tt, wt;
        tile_at(p, tile, tt, wt);
        const int b = p.accumulators == 2 ? turn & 1 : 0, use = p.accumulators == 2 ? turn >> 1 : turn;
        mbar_wait(free_(b), (use & 1) ^ 1, dead_);
        tc_fence_after();
        const uint32_t d = tmem + b * 256;
        auto product = [&](uint64_t z, uint64_t w, bool accumulate) { mma_f16<PAIR>(d, TALL ? w : z, TALL ? z : w, idesc, accumulate); };
        auto multiply_adapter = [&] {
          for (int e = 0; e < rank_chunks * parts; e++, at.next()) {
            const int rc = e / parts;
            mbar_wait(full(at.s), at.phase, dead_);
            mbar_wait(written(at.s), (written_phase >> at.s) & 1, dead_);
            written_phase ^= 1u << at.s;
            tc_fence_after();
            const uint64_t off = (uint64_t)(at.s * stage_bytes >> 4);
            const int steps = (min(64, p.rank - rc * 64) + 15) >> 4;
            if (elect_one()) {
              for (int k = 0; k < steps; k++) product(z_desc + off + k * token_step, w_desc + off + k * weight_step, true);
              if (paired)
                for (int k = 0; k < steps; k++) product(z_desc + off + (k + 2) * token_step, w_desc + off + k * weight_step, true);
              mma_commit<PAIR>(empty(at.s), mask);
            }
            __syncwarp();
          }
        };
        auto multiply_chunk = [&](bool accumulate) {
          mbar_wait(full(at.s), at.phase, dead_);
          tc_fence_after();
          const uint64_t off = (uint64_t)(at.s * stage_bytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; k++) product(z_desc + off + k * token_step, w_desc + off + k * weight_step, accumulate || k > 0);
            mma_commit<PAIR>(empty(at.s), mask);
          }
          __syncwarp();
          at.next();
        };
        for (int c = c0; c <= middle; c++) multiply_chunk(c > c0);
        wait_for_predecessor();
        Adapters adapters(p.lists + (int64_t)tt * (kBlocks * p.token_rows + 1), split, p.splits, lane);
        adapters.open(p, tt * kBlocks * p.token_rows, kBlocks * p.token_rows);
        int c = middle + 1;
        if (adapters.late) {
#pragma unroll 1
          for (; c < c1; c++) multiply_chunk(true);
          if (elect_one()) mma_commit<PAIR>(whole, mask);
          __syncwarp();
          mbar_wait(shifted, shifted_phase, dead_);
          shifted_phase ^= 1;
          tc_fence_after();
        }
        for (int k = 0; k < adapters.count; k++) {
          if (k && c < c1) multiply_chunk(true), c++;
          multiply_adapter();
        }
        for (; c < c1; c++) multiply_chunk(true);
        if (elect_one()) mma_commit<PAIR>(done(b), mask);
        __syncwarp();
      }
    }
  } else {
    const int e = threadIdx.x - 64, quarter = warp & 3;
    // The writers take part in few of a stage's rounds, so they cannot follow its `empty` barrier by parity; the copying
    // warp, which follows every round, grants them the stage.
    Ring ring(p.stages);
    int turn = 0;
    uint32_t granted_phase = 0, whole_phase = 0, buffer = 0;
    const uint32_t staging = base + p.stages * stage_bytes;
    auto tell = [&](uint32_t bar) {  // the block that issues the products
      if (PAIR) cluster_arrive(cluster_addr(bar, leader));
      else mbar_arrive(bar);
    };
    for (int tile = blockIdx.x / team; tile < tiles; tile += step, turn++) {
      int tt, wt;
      tile_at(p, tile, tt, wt);
      int passed = middle - c0 + 1;  // chunks of K that the ring has seen
      ring.skip(passed);
      wait_for_predecessor();
      const int t0 = (tt * kBlocks + me) * p.token_rows;
      // S: a thread writes rows e and e + 128 of the token tile, 16-byte pieces of eight values
      constexpr int kRows = TALL ? 2 : 1;
      int mine[kRows];
      uint4 pieces[kRows][8];  // paired: the first terms, then the second; otherwise one of them
      const uint16_t* src[kRows];
#pragma unroll
      for (int h = 0; h < kRows; h++) {
        const int row = e + h * 128, t = t0 + row;
        mine[h] = row < p.token_rows && t < p.T ? p.adapter_of[t] : -1;
        if (mine[h] >= p.n_adapters) mine[h] = -1;
        src[h] = p.pair + (int64_t)(mine[h] >= 0 ? t : 0) * 2 * p.rank;
      }
      auto load = [&](int rc, int part) {
#pragma unroll
        for (int h = 0; h < kRows; h++)
#pragma unroll
          for (int g = 0; g < 8; g++) {
            const int j = paired ? (g & 3) * 8 : rc * 64 + g * 8;
            pieces[h][g] = mine[h] >= 0 && j < p.rank
                               ? __ldcg(reinterpret_cast<const uint4*>(src[h] + (paired ? g >> 2 : part) * p.rank + j))
                               : make_uint4(0, 0, 0, 0);
          }
      };
      Adapters adapters(p.lists + (int64_t)tt * (kBlocks * p.token_rows + 1), split, p.splits, lane);
      adapters.open(p, tt * kBlocks * p.token_rows, kBlocks * p.token_rows);
      if (adapters.count && paired) load(0, 0);
      const int b = p.accumulators == 2 ? turn & 1 : 0, use = p.accumulators == 2 ? turn >> 1 : turn;
      const uint32_t d = tmem + b * 256 + ((uint32_t)(quarter * 32) << 16);
      const int columns = TALL ? p.token_rows : 2 * p.weight_rows, at = quarter * 32 + lane;
      if (adapters.late) {
        ring.skip(c1 - c0 - passed);
        passed = c1 - c0;
        mbar_wait(whole, whole_phase, dead_);
        whole_phase ^= 1;
        tc_fence_after();
        rescale<TALL>(adapters, d, columns, me * 128 + at, 1);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) tell(shifted);
      }
      for (int k = 0; k < adapters.count; k++) {
        const int a = adapters.at(k);
        if (k && passed < c1 - c0) {
          ring.next();
          passed++;
        }
        for (int x = 0; x < rank_chunks * parts; x++, ring.next()) {
          const int rc = x / parts, s = ring.s;
          if (!paired) load(rc, x & 1);
          mbar_wait(granted(s), (granted_phase >> s) & 1, dead_);
          granted_phase ^= 1u << s;
          const int wide = ((min(64, p.rank - rc * 64) + 15) & ~15) >> 3;  // pieces of whole steps of K
#pragma unroll
          for (int h = 0; h < kRows; h++) {
            const int row = e + h * 128;
            if (row >= p.token_rows) continue;
            const uint32_t dst = base + s * stage_bytes + row * 128;
#pragma unroll
            for (int g = 0; g < 8; g++) {
              if ((paired ? g & 3 : g) >= wide) continue;
              const uint4 v = mine[h] == a ? pieces[h][g] : make_uint4(0, 0, 0, 0);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + ((g ^ (row & 7)) << 4)), "r"(v.x), "r"(v.y), "r"(v.z),
                           "r"(v.w)
                           : "memory");
            }
          }
          fence_async_shared();
          __syncwarp();
          if (lane == 0) tell(written(s));
        }
      }
      ring.skip(c1 - c0 - passed);
      // the accumulators of the tile
      mbar_wait(done(b), use & 1, dead_);
      tc_fence_after();
      if (adapters.late) rescale<TALL>(adapters, d, columns, me * 128 + at, -1);
      if (!TALL && p.splits == 1) {
        // 32 rows x 64 columns at a time through shared memory (128-byte swizzle, two buffers a warp) and out by TMA: rows
        // are far apart, and 16-byte stores straight from the registers took as long as a third of the tile's products
        for (int c = 0; c < columns; c += 64, buffer ^= 1) {
          uint32_t r[4][16];
#pragma unroll
          for (int h = 0; h < 4; h++)
            if (c + h * 16 < columns) tmem_load16(d + c + h * 16, r[h]);
          tmem_load_wait();
          const uint32_t to = staging + ((quarter * 2 + buffer) * 32 + lane) * 128;
          if (lane == 0) tma_store_wait<1>();
          __syncwarp();
#pragma unroll
          for (int h = 0; h < 4; h++)
            if (c + h * 16 < columns) {
#pragma unroll
              for (int k = 0; k < 16; k += 8) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; q++)
                  w[q] = pack2(__uint_as_float(r[h][k + 2 * q]), __uint_as_float(r[h][k + 2 * q + 1]), p.dtype);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((h * 2 + (k >> 3)) ^ (lane & 7)) << 4)), "r"(w[0]),
                             "r"(w[1]), "r"(w[2]), "r"(w[3])
                             : "memory");
              }
            }
          fence_async_shared();
          __syncwarp();
          const int n = wt * 2 * p.weight_rows + c, t = t0 + quarter * 32;
          // not by TMA: a box wider than what is left of the tile, whose other columns are the next tile's, and a box that
          // ends in the middle of 16 bytes, which the copy would write whole
          const bool whole = c + 64 <= columns && (n + 64 <= p.N || p.N % 8 == 0);
          if (lane == 0) {
            if (whole && t < p.T && n < p.N) tma_store_2d(&omap, n, t, staging + (quarter * 2 + buffer) * 4096);
            tma_store_commit();
          }
          if (!whole && t0 + at < p.T) {
            for (int g = 0; c + g * 8 < columns; g++) {
              uint4 w;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                           : "r"(to + ((g ^ (lane & 7)) << 4))
                           : "memory");
              uint16_t* out = static_cast<uint16_t*>(p.O) + (t0 + at) * p.ldo + n + g * 8;
              if (n + g * 8 + 8 <= p.N) {
                *reinterpret_cast<uint4*>(out) = w;
              } else {
                const uint32_t v[4] = {w.x, w.y, w.z, w.w};
                for (int k = 0; k < 8; k++)
                  if (n + g * 8 + k < p.N) out[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
              }
            }
          }
        }
      } else {
        for (int c = 0; c < columns; c += 16) {
          uint32_t r[16];
          tmem_load16(d + c, r);
          tmem_load_wait();
          if (p.splits > 1) {
            // as the result lies: [token][output], the outputs of a tall tile being the lanes
            if (TALL) {
#pragma unroll
              for (int k = 0; k < 16; k++)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + ((c + k) * kTallPitch + at) * 4), "r"(r[k]) : "memory");
            } else {
#pragma unroll
              for (int k = 0; k < 16; k += 4)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (at * kWidePitch + c + k) * 4), "r"(r[k]),
                             "r"(r[k + 1]), "r"(r[k + 2]), "r"(r[k + 3])
                             : "memory");
            }
          } else {
            const int n = wt * 128 + at;
            if (n < p.N) {
#pragma unroll
              for (int k = 0; k < 16; k++) {
                const int t = t0 + c + k;
                if (t < p.T) store1(p.O, t * p.ldo + n, p.dtype, __uint_as_float(r[k]));
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tell(free_(b));
    }
    if (!TALL && lane == 0) tma_store_wait<0>();
  }
  __syncwarp();
  __syncthreads();
  if (dead) settle(p.stalls);
  __syncwarp();
  // A block of its own gives its tensor memory back before it waits for the cluster (see low_rank_kernel).  A pair frees it
  // together, when neither is at work any more; what may share an SM with a pair of split tiles (256 columns, at least 180 KB)
  // is one low-rank block of at most 128 columns; beside a pair of whole tiles (512 columns, at least 202 KB) none fits.
  if (!PAIR && warp == 1) {
    tc_fence_after();
    tmem_free<PAIR>(tmem, p.columns);
  }
  __syncwarp();
  if (team > 1) cluster_sync();  // no more arrivals from other blocks; their sums are in shared memory
  if (PAIR && warp == 1) {
    tc_fence_after();
    tmem_free<PAIR>(tmem, p.columns);
  }
  if (p.splits > 1) {
    // one tile a team: this block adds and stores its share of it
    int tt, wt;
    tile_at(p, blockIdx.x / team, tt, wt);
    const int outputs = TALL ? 128 : 2 * p.weight_rows, quads = outputs / 4, pitch = TALL ? kTallPitch : kWidePitch;
    const int t0 = TALL ? tt * p.token_rows : (tt * 2 + me) * 128, n0 = wt * outputs;
    const int rows = min(TALL ? p.token_rows : 128, p.T - t0), items = max(0, (rows - split + p.splits - 1) / p.splits) * quads;
    constexpr int U = 4;
    for (int i = threadIdx.x; i < items; i += U * kThreads) {
      uint32_t offset[U];
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int q = min(i + u * kThreads, items - 1);
        offset[u] = (uint32_t)((split + q / quads * p.splits) * pitch + q % quads * 4) * 4;
      }
      cluster_sum<U>(base, offset, p.splits, me, kBlocks, x);
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int q = i + u * kThreads, t = t0 + split + q / quads * p.splits, n = n0 + q % quads * 4;
        if (q >= items || n >= p.N) continue;
        if (n + 4 <= p.N) {
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.O) + t * p.ldo + n) =
              make_uint2(pack2(x[u].x, x[u].y, p.dtype), pack2(x[u].z, x[u].w, p.dtype));
        } else {
          const float v[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
          for (int k = 0; k < 4; k++)
            if (n + k < p.N) store1(p.O, t * p.ldo + n + k, p.dtype, v[k]);
        }
      }
    }
    __syncwarp();
    cluster_sync();  // no block leaves while another reads its shared memory
  }
}

template <bool TALL, bool TRANS>
windq_status launch(windq_ctx* ctx, const CUtensorMap& z, const CUtensorMap& w, const CUtensorMap& pm, const CUtensorMap& o, const ProjectArgs& p,
                    int blocks, int smem, cudaStream_t st) {
  const windq_status ready = prepare_kernel(ctx, kProject + 2 * TALL + TRANS, project_kernel<TALL, TRANS>, kThreads, kSmemLimit, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = (TALL ? 1 : 2) * p.splits;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = attrs[1].val.clusterDim.x > 1 ? 2 : 1;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, project_kernel<TALL, TRANS>, z, w, pm, o, p));
  return WINDQ_OK;
}

}  // namespace

// Up to 320 tokens the tiles are tall: a wide tile has 256 tokens whether they are there or not.  (300 tokens: 46 against
// 53 us for 11008 x 4096, 67 against 78 us for 5120 x 13824; 400 tokens: 64 against 55 us and 91 against 80 us.)
static bool is_tall(int64_t T) { return T <= 320; }

int token_tile(int64_t T) {
  if (!is_tall(T)) return 256;
  const int64_t tiles = std::max<int64_t>(1, (T + 255) / 256);
  return (int)round_up(std::max<int64_t>((T + tiles - 1) / tiles, 1), 16);
}

windq_status launch_projection(windq_ctx* ctx, const Projection& q, cudaStream_t st) {
  const bool tall = is_tall(q.T);
  ProjectArgs p = {};
  p.T = (int)q.T;
  p.N = (int)q.N;
  p.chunks = (int)((q.K + 63) / 64);
  p.rank = q.rank;
  p.n_adapters = (int)q.n_adapters;
  p.dtype = q.dtype;
  p.adapter_of = q.adapter_of;
  p.pair = (const uint16_t*)q.pair;
  p.shift = q.shift;
  p.lists = q.lists;
  p.O = q.O;
  p.ldo = q.ldo;
  p.stalls = stalls_of(ctx);
  const int blocks_of_tile = tall ? 1 : 2;
  p.token_rows = tall ? token_tile(q.T) : 128;
  p.weight_rows = 128;
  p.token_tiles = (int)((q.T + p.token_rows * blocks_of_tile - 1) / (p.token_rows * blocks_of_tile));
  // Tall tiles: one thread block an SM, with many stages, where tiles split along K then fill most of the GPU (203 tokens x
  // 8192 x 8192, 128 blocks: 64 against 72 us); otherwise two, if the sums of a split tile fit into half of the shared memory
  // (150 tokens x 11008 x 4096, 86 blocks against 172: 52 against 46 us).  Up to 64 tokens two blocks have stages enough.
  // Four splits at most: clusters of eight start and join slowly (192 tokens x 2048 x 8192: 42 us, with four 34).
  const int64_t tall_tiles = (int64_t)p.token_tiles * ((q.N + 127) / 128);
  auto tall_splits = [&](int64_t slots) {
    int splits = 1;
    while (splits < 4 && tall_tiles * splits * 2 <= slots && p.chunks >= splits * 2 * 4) splits *= 2;
    return splits;
  };
  const bool two = tall && p.token_rows * kTallPitch * 4 <= kSmemLimitTwo - 1024 &&
                   (p.token_rows <= 64 || tall_tiles * tall_splits(ctx->sm_count) * 5 < ctx->sm_count * 4);
  const int64_t slots = tall ? (int64_t)ctx->sm_count * (two ? 2 : 1) : ctx->sm_count / 2;
  p.splits = tall ? tall_splits(slots) : 1;
  if (!tall) {
    // Outputs of a tile: the width that takes the least time in rounds over the GPU.  Measured, a chunk of K takes 0.23 us at
    // width 128, 0.24 at 160, 0.27 at 192, 0.31 at 224 and 0.36 at 256 (max(210 + w / 5, 1.39 w) ns), a tile 2 us more, and 5
    // where it is split along K; a narrow tile moves more bytes a product, which tells where power is the limit.  Tiles that
    // fill less than half of the GPU are split.
    int64_t best = INT64_MAX;
    for (int rows = 128; rows >= 48; rows -= 16) {
      const int64_t tiles = p.token_tiles * ((q.N + 2 * rows - 1) / (2 * rows));
      int splits = 1;
      while (splits < 4 && tiles * splits * 2 <= slots && p.chunks >= splits * 2 * 4) splits *= 2;
      const int64_t waves = (tiles * splits + slots - 1) / slots;
      const int width = 2 * rows, chunk = std::max(210 + width / 5, width * 139 / 100) * (1256 - width) / 1000;
      const int64_t cost = waves * ((int64_t)(p.chunks + splits - 1) / splits * chunk + (splits > 1 ? 5000 : 2000));
      if (cost < best) {
        best = cost;
        p.weight_rows = rows;
        p.splits = splits;
      }
    }
  }
  p.weight_tiles = (int)((q.N + p.weight_rows * blocks_of_tile - 1) / (p.weight_rows * blocks_of_tile));
  p.group = (int)std::max<int64_t>(1, std::min<int64_t>(p.token_tiles, (48ll << 20) / (2 * q.K * p.token_rows * blocks_of_tile)));
  const int stage = p.token_rows * 128 + (q.transposed ? (p.weight_rows + 63) / 64 * 8192 : p.weight_rows * 128);
  const int limit = two ? kSmemLimitTwo : kSmemLimit;
  const int staging = tall || p.splits > 1 ? 0 : 4 * 2 * 4096;
  p.stages = std::min(kMaxStages, (limit - 1024 - staging) / stage);
  const int64_t tiles = (int64_t)p.token_tiles * p.weight_tiles;
  p.accumulators = !tall && p.splits == 1 ? 2 : 1;
  p.columns = tall ? (p.token_rows <= 32 ? 32 : p.token_rows <= 64 ? 64 : p.token_rows <= 128 ? 128 : 256) : 256 * p.accumulators;
  const int64_t blocks = (p.splits > 1 ? tiles * p.splits : std::min(tiles, slots)) * blocks_of_tile;
  const int sums = p.splits > 1 ? (tall ? p.token_rows * kTallPitch : 128 * kWidePitch) * 4 : 0;
  const int smem = 1024 + std::max(p.stages * stage + staging, sums);

  CUtensorMap z, w, pm, o;
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  bool ok = make_map(&z, q.dtype, q.Z, q.K, q.T, 0, q.ldz, 0, p.token_rows);
  if (q.transposed) {
    ok = ok && make_map(&w, q.dtype, q.W, q.N, q.K, 0, q.ldw, 0, 64);
    ok = ok && make_map(&pm, q.dtype, q.P, q.N, q.rank, q.n_adapters, q.N, q.N * q.rank, 64);
  } else {
    ok = ok && make_map(&w, q.dtype, q.W, q.K, q.N, 0, q.ldw, 0, p.weight_rows);
    ok = ok && make_map(&pm, q.dtype, q.P, q.rank, q.N, q.n_adapters, q.rank, q.N * q.rank, p.weight_rows);
  }
  if (tall) o = z;  // not used
  else ok = ok && make_map(&o, q.dtype, q.O, q.N, q.T, 0, q.ldo, 0, 32);
  WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  if (tall) return q.transposed ? launch<true, true>(ctx, z, w, pm, o, p, (int)blocks, smem, st)
                                : launch<true, false>(ctx, z, w, pm, o, p, (int)blocks, smem, st);
  return q.transposed ? launch<false, true>(ctx, z, w, pm, o, p, (int)blocks, smem, st)
                      : launch<false, false>(ctx, z, w, pm, o, p, (int)blocks, smem, st);
}

}  // namespace windq
