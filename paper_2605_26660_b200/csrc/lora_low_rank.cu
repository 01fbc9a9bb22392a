// S[t][j] = scaling[a] * sum_k Z[t][k] P[a](j, k) with a = adapter_of[t]: the low-rank product of the adapter calls, whose
// result (rank values a token) the projection and the gradients take.  Bound by reading Z and the used P once.
//
// A tile of up to 128 tokens (rows of the accumulator, whether there are that many or not) times the P of the adapters its
// tokens use (columns), on tcgen05 with operands by TMA; of the product every token keeps its own adapter's columns.  For
// prompts, whose neighbours share an adapter, that is one pass over Z.  For single tokens with many adapters most of the
// product is thrown away, but it is the bytes of P that count, and TMA keeps all of them in flight: 203 tokens with 48
// adapters of 32 x 8192 took warps with register operands 57 us.
#include <limits.h>

#include <algorithm>

#include "lora.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kLowWarps = 8, kLowThreads = 256;

struct LowJob {
  const uint16_t* Z;
  int64_t ldz;
  const uint16_t* P;  // [a][j][k], or transposed [a][k][j]
  float* S;        // binary32, or NULL
  uint16_t* pair;  // [t][2][j]: the two 16-bit values whose sum stands for S, or NULL
  int8_t* shift;   // fp16 pairs: the power of two by which the token's are scaled
  float* top;      // largest |S[t][j]| of a token, or NULL
  int K, transposed;
};
struct LowRankArgs {
  LowJob job[2];
  int T, rank, n_adapters, dtype, jobs, slots, splits, stages;
  int rows, pack[2], stage_bytes;  // tokens of a tile; adapters of a pass, plain and transposed
  const float* scaling;
  const int32_t* adapter_of;
  int* lists;  // adapters of the projection's token tiles, or NULL
  int list_rows, list_tiles;
  Stalls stalls;
};

// Thread i's id of `count` (at most 256, one a thread): its place among the different ids in the order of their first
// occurrence if it is that occurrence, -1 otherwise; *all = how many there are.  ids < 0 do not count.  Only the first of a
// run of equal ids has to look back.
__device__ int first_place(int id, int count, int* ids, int* taken, int* all) {
  const int i = threadIdx.x;
  ids[i] = i < count ? id : -1;
  __syncthreads();
  bool first = i < count && id >= 0 && (i == 0 || ids[i - 1] != id);
  for (int k = 0; k < i && first; k++) first = ids[k] != id;
  const unsigned vote = __ballot_sync(0xffffffffu, first);
  if ((i & 31) == 0) taken[i >> 5] = __popc(vote);
  __syncthreads();
  int before = __popc(vote & ((1u << (i & 31)) - 1)), sum = 0;
  for (int w = 0; w < kLowWarps; w++) {
    if (w < i >> 5) before += taken[w];
    sum += taken[w];
  }
  *all = sum;
  return first ? before : -1;
}

__device__ __forceinline__ int valid_id(const LowRankArgs& p, int64_t t) {
  const int id = t < p.T ? p.adapter_of[t] : -1;
  return id < p.n_adapters ? id : -1;
}

// The list of one token tile of the projection.
__device__ void write_list(const LowRankArgs& p, int tile, int* ids, int* taken) {
  int all;
  const int id = threadIdx.x < p.list_rows ? valid_id(p, (int64_t)tile * p.list_rows + threadIdx.x) : -1;
  const int place = first_place(id, p.list_rows, ids, taken, &all);
  int* list = p.lists + (int64_t)tile * (p.list_rows + 1);
  if (place >= 0) list[1 + place] = id;
  if (threadIdx.x == 0) list[0] = all;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __int_as_float(0x7f800000); }
// x in [-most, most]; infinities and NaN as they are (fminf and fmaxf would make a number of NaN).
__device__ __forceinline__ float clamp(float x, float most) { return finite(x) ? fminf(fmaxf(x, -most), most) : x; }

// The power of two by which the fp16 pairs of a token are scaled, from its largest |S|.  Two fp16 values lie on the grid
// 2^-24 of their type's smallest step, which leaves 22 bits of the largest |S| where that is 2^-3 or more and 16, as bf16
// pairs have, at 2^-9; they hold up to 2 * 65504.  Within [2^-9, 2^16) nothing is scaled: the projection has less to do then (us
// without and with scaled tokens: 48 single tokens with 32 adapters x 11008 x 4096 29.7 and 32.6, 203 with 48 x 8192 x 8192 67.6
// and 74.3, the backward pass of 8192 x 4096 x 4096 303 and 310).  Outside, the largest goes to [2^12, 2^13), as far as 2^40
// reaches: what lies below after that is less than any result of 16 bits, 128 products with values up to 65504 included, and
// what lies above is more.
__device__ __forceinline__ int shift_of(float top) {
  const int e = (int)(__float_as_uint(top) >> 23) - 127;  // 2^e <= top < 2^(e + 1)
  return top == 0.0f || (e >= -9 && e <= 15) ? 0 : max(-40, min(40, 12 - e));
}

// The two 16-bit values of four values of S: 22 bits of fp16, 16 of bf16.  What is not finite stays so, in the first.
__device__ __forceinline__ void write_pair(const LowRankArgs& p, const LowJob& job, int t, int j, const float (&v)[4]) {
  uint32_t hi[2], lo[2];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    float a = v[2 * k], b = v[2 * k + 1];
    if (p.dtype == WINDQ_F16) {
      a = clamp(a, 131008.0f);
      b = clamp(b, 131008.0f);
      hi[k] = pack2(clamp(a, 65504.0f), clamp(b, 65504.0f), p.dtype);
    } else {
      hi[k] = pack2(a, b, p.dtype);
    }
    const float2 back = unpack2(hi[k], p.dtype);
    lo[k] = pack2(finite(a) ? a - back.x : 0.0f, finite(b) ? b - back.y : 0.0f, p.dtype);
  }
  uint16_t* out = job.pair + (int64_t)t * 2 * p.rank + j;
  *reinterpret_cast<uint2*>(out) = make_uint2(hi[0], hi[1]);
  *reinterpret_cast<uint2*>(out + p.rank) = make_uint2(lo[0], lo[1]);
}

// S of the tokens of this block from the sums of the cluster's blocks, [token][pitch] at `sums`: four values a thread.
// kept(i) tells whether token t0 + i is to be written; tops: one word a token, zero.
template <class Kept>
__device__ __forceinline__ void finish_tokens(const LowRankArgs& p, const LowJob& job, int t0, int tokens, uint32_t sums, int pitch,
                                              int split, const int* ids, int* tops, Kept kept) {
  const int quads = p.rank / 4, share = (tokens - split + p.splits - 1) / p.splits;
  for (int x = threadIdx.x; x < share * quads; x += kLowThreads) {
    const int i = split + x / quads * p.splits, j = x % quads * 4;
    if (!kept(i)) continue;
    const uint32_t offset[1] = {(uint32_t)(i * pitch + j) * 4};
    float4 y[1];
    if (p.splits > 1) cluster_sum<1>(sums, offset, p.splits, 0, 1, y);
    else asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(y[0].x), "=f"(y[0].y), "=f"(y[0].z), "=f"(y[0].w) : "r"(sums + offset[0]) : "memory");
    const float scale = p.scaling[ids[i]];
    const float v[4] = {y[0].x * scale, y[0].y * scale, y[0].z * scale, y[0].w * scale};
    if (job.S) *reinterpret_cast<float4*>(job.S + (int64_t)(t0 + i) * p.rank + j) = make_float4(v[0], v[1], v[2], v[3]);
    if (job.top || job.shift) {
      // of the finite values: the others come through any scaling, and must not set it
      float most = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; k++) most = fmaxf(most, finite(v[k]) ? fabsf(v[k]) : 0.0f);
      atomicMax(&tops[i], __float_as_int(most));
    }
    if (job.shift)  // in the place of the sums, which no other block reads in this one's rows
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(sums + offset[0]), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
    else if (job.pair)
      write_pair(p, job, t0 + i, j, v);
  }
  if (!job.top && !job.shift) return;
  __syncthreads();
  if (job.top) {
    for (int x = threadIdx.x; x < share; x += kLowThreads) {
      const int i = split + x * p.splits;
      if (kept(i)) job.top[t0 + i] = __int_as_float(tops[i]);
    }
  }
  if (job.shift) {
    for (int x = threadIdx.x; x < share * quads; x += kLowThreads) {
      const int i = split + x / quads * p.splits, j = x % quads * 4;
      if (!kept(i)) continue;
      float v[4];
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(sums + (uint32_t)(i * pitch + j) * 4) : "memory");
      const int e = shift_of(__int_as_float(tops[i]));
      const float up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
      for (int k = 0; k < 4; k++) v[k] *= up;
      write_pair(p, job, t0 + i, j, v);
      if (j == 0) job.shift[t0 + i] = (int8_t)e;
    }
  }
}

constexpr int kStages = 16, kRows = 128;
constexpr int kGroup = 4;  // chunks of K that one accumulator takes
constexpr int kLowSmem = 227 * 1024 - 3072;

// Passes: `pack` adapters at a time, as many as 128 columns hold (transposed, where an adapter takes a block of 64 columns
// of shared memory: two), so that a tile in which one prompt ends and the next begins still takes one pass over Z; with one
// adapter a pass such tiles took twice as long and with them the whole kernel (41 against 22 us for 8192 tokens of 4096
// values, rank 64).  `slots` blocks share the passes of a tile, `splits` blocks of a cluster K.  Warps: one issues TMA
// copies, one the products, four take the rows of their own adapter out of tensor memory.
//
// The tensor cores cut a sum off where they add to an accumulator; over 256 steps of K that was 7e-6 of S, and of the
// gradients S goes into (which are binary32; a plain binary32 product is 1e-6 off).  So an accumulator takes four chunks of
// K (16 steps), then its values are added, rounded, to sums in shared memory while the other accumulator fills.
__global__ void __launch_bounds__(kLowThreads)
    low_rank_kernel(const __grid_constant__ CUtensorMap z0, const __grid_constant__ CUtensorMap p0,
                       const __grid_constant__ CUtensorMap z1, const __grid_constant__ CUtensorMap p1,
                       const __grid_constant__ LowRankArgs p) {
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t full_[kStages], empty_[kStages], done_[2], free_[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int dead, ids[256], used[kRows], tops[kRows], taken[kLowWarps];
  __shared__ bool mine[kRows];
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const int split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
  if (blockIdx.y == p.jobs * p.slots) {
    wait_for_predecessor();
    launch_dependents();
    if (split == 0 && tile < p.list_tiles) write_list(p, tile, ids, taken);
    return;  // of a whole cluster
  }
  const bool other = blockIdx.y >= p.slots;
  const int slot = blockIdx.y - (other ? p.slots : 0);
  const LowJob& job = p.job[other];
  const bool trans = job.transposed;
  const int r = p.rank, wide = (r + 15) & ~15;
  const int pack = p.pack[trans];
  const uint32_t token_bytes = p.rows * 128, stage_bytes = p.stage_bytes;
  const uint32_t columns = pack * wide <= 32 ? 32 : pack * wide <= 64 ? 64 : 128;  // of an accumulator
  // the product reads 128 rows whatever the tile holds; what follows a short tile gives rows that nobody keeps
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u, sums = base + p.stages * stage_bytes + (kRows - p.rows) * 128;
  auto full = [&](int s) { return smem_addr(&full_[s]); };
  auto empty = [&](int s) { return smem_addr(&empty_[s]); };
  const uint32_t dead_ = smem_addr(&dead);
  auto done = [&](int g) { return smem_addr(&done_[g & 1]); };  // of group g's accumulator
  auto free = [&](int g) { return smem_addr(&free_[g & 1]); };
  const int t0 = tile * p.rows;

  if (tid == 0) {
    prefetch_map(other ? &z1 : &z0);
    prefetch_map(other ? &p1 : &p0);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int g = 0; g < 2; g++) {
      mbar_init(done(g), 1);
      mbar_init(free(g), 4);
    }
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<false>(smem_addr(&tmem_slot), 2 * columns);
  __syncthreads();
  // Nothing of this call is read or written before the stream's earlier work has ended -- and the kernels that follow may
  // not start before that either: the projection reads its operands without waiting for this kernel.  Nor may they start
  // before this block has its tensor memory: the projection holds its own while it waits for this kernel.
  wait_for_predecessor();
  launch_dependents();
  int n_used;
  const int id = tid < p.rows ? valid_id(p, t0 + tid) : -1, place = first_place(id, p.rows, ids, taken, &n_used);
  if (place >= 0) used[place] = id;
  if (job.shift && slot == 0 && split == 0 && tid < p.rows && id < 0) job.shift[t0 + tid] = 0;  // nobody else's tokens
  if (tid < kRows) tops[tid] = 0, mine[tid] = false;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int chunks = (job.K + 63) >> 6, c0 = (int)((int64_t)chunks * split / p.splits), c1 = (int)((int64_t)chunks * (split + 1) / p.splits);
  n_used = uniform(n_used);
  const int passes = (n_used + pack - 1) / pack;

  if (warp == 0) {
    // (a copy of the loop for each job's maps: an address that is picked at run time takes three times as long to issue)
    auto copy = [&](const CUtensorMap& zmap, const CUtensorMap& pmap) {
      int s = 0;
      uint32_t phase = 0;
      for (int pass = slot; pass < passes; pass += p.slots) {
        const int count = min(pack, n_used - pass * pack), first = uniform(used[pass * pack]);
        const uint32_t bytes = token_bytes + (trans ? (r > 64 ? 16384 : count * 8192) : count * wide * 128);
        for (int c = c0; c < c1; c++) {
          mbar_wait(empty(s), phase ^ 1, dead_);
          const uint32_t at = base + s * stage_bytes, bar = full(s);
          if (elect_one() && !*(volatile int*)&dead) {
            mbar_expect(bar, bytes);
            tma_load_2d<false>(at, &zmap, c * 64, t0, bar);
            if (trans) {
              tma_load_3d<false>(at + token_bytes, &pmap, 0, c * 64, first, bar);
              if (r > 64) tma_load_3d<false>(at + token_bytes + 8192, &pmap, 64, c * 64, first, bar);
              else if (count > 1) tma_load_3d<false>(at + token_bytes + 8192, &pmap, 0, c * 64, used[pass * pack + 1], bar);
            } else {
              tma_load_3d<false>(at + token_bytes, &pmap, c * 64, 0, first, bar);
              for (int u = 1; u < count; u++)
                tma_load_3d<false>(at + token_bytes + u * wide * 128, &pmap, c * 64, 0, used[pass * pack + u], bar);
            }
          }
          __syncwarp();
          if (++s == p.stages) s = 0, phase ^= 1;
        }
      }
    };
    if (other) copy(z1, p1);
    else copy(z0, p0);
  } else if (warp == 1) {
    const uint64_t z_desc = smem_desc(base, 16), p_desc = smem_desc(base + token_bytes, trans ? 8192 : 16);
    const uint32_t p_step = trans ? 2048 >> 4 : 32 >> 4;
    int s = 0, g = 0;
    uint32_t phase = 0;
    for (int pass = slot; pass < passes; pass += p.slots) {
      const int count = min(pack, n_used - pass * pack);
      const uint32_t idesc = instr_desc(p.dtype, false, trans, 128, trans ? wide : count * wide);
      for (int c = c0; c < c1; g++) {
        const uint32_t d = tmem + (g & 1) * columns;
        mbar_wait(free(g), ((g >> 1) & 1) ^ 1, dead_);
        tc_fence_after();
        const int end = min(c + kGroup, c1);
        for (const int begin = c; c < end; c++) {
          mbar_wait(full(s), phase, dead_);
          tc_fence_after();
          const uint64_t off = (uint64_t)(s * stage_bytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; k++)
              mma_f16<false>(d, z_desc + off + k * (32 >> 4), p_desc + off + k * p_step, idesc, c > begin || k > 0);
            if (trans && count > 1) {
#pragma unroll
              for (int k = 0; k < 4; k++)
                mma_f16<false>(d + wide, z_desc + off + k * (32 >> 4), p_desc + off + (8192 >> 4) + k * p_step, idesc, c > begin || k > 0);
            }
            mma_commit<false>(empty(s), 0);
          }
          __syncwarp();
          if (++s == p.stages) s = 0, phase ^= 1;
        }
        if (elect_one()) mma_commit<false>(done(g), 0);
        __syncwarp();
      }
    }
  } else if (warp < 6) {
    const int quarter = warp & 3, row = quarter * 32 + lane, own = ids[row];
    int g = 0;
    for (int pass = slot; pass < passes; pass += p.slots) {
      const int count = min(pack, n_used - pass * pack);
      for (int c = c0; c < c1; c += kGroup, g++) {
        mbar_wait(done(g), (g >> 1) & 1, dead_);
        tc_fence_after();
        for (int i = 0; i < count; i++) {
          const bool keep = own == used[pass * pack + i];
          if (!__any_sync(0xffffffffu, keep)) continue;
          if (keep) mine[row] = true;
          for (int j = 0; j < wide; j += 16) {
            uint32_t x[16];
            tmem_load16(tmem + (g & 1) * columns + ((uint32_t)(quarter * 32) << 16) + i * wide + j, x);
            tmem_load_wait();
            if (keep) {
#pragma unroll
              for (int k = 0; k < 16; k += 4)
                if (j + k < r) {
                  const uint32_t at = sums + (row * (r + 4) + j + k) * 4;
                  float4 y = make_float4(0, 0, 0, 0);
                  if (c > c0) asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(y.x), "=f"(y.y), "=f"(y.z), "=f"(y.w) : "r"(at) : "memory");
                  y.x += __uint_as_float(x[k]), y.y += __uint_as_float(x[k + 1]), y.z += __uint_as_float(x[k + 2]), y.w += __uint_as_float(x[k + 3]);
                  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(y.x), "f"(y.y), "f"(y.z), "f"(y.w) : "memory");
                }
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(free(g));
      }
    }
  }
  __syncwarp();
  __syncthreads();
  if (dead) settle(p.stalls);
  __syncwarp();
  // Before the cluster's barrier: a block that waits for its peers holds no tensor memory, so that whoever waits for columns
  // (a peer's allocation behind a block of another stream, say) waits only for blocks that run to this point by themselves.
  if (warp == 1) {
    tc_fence_after();
    tmem_free<false>(tmem, 2 * columns);
  }
  __syncwarp();
  if (p.splits > 1) cluster_sync();
  finish_tokens(p, job, t0, p.rows, sums, r + 4, split, ids, tops, [&](int i) { return mine[i]; });
  __syncwarp();
  if (p.splits > 1) cluster_sync();
}

windq_status launch(windq_ctx* ctx, LowRankArgs p, cudaStream_t st) {
  const int wide = (p.rank + 15) & ~15;
  p.rows = std::min(kRows, (p.T + 15) & ~15);
  const int tiles = (p.T + p.rows - 1) / p.rows, most = std::min(p.rows, p.n_adapters);  // adapters of a tile
  int least = INT_MAX;
  bool trans = false, plain = false;
  for (int k = 0; k < p.jobs; k++) {
    least = std::min(least, (p.job[k].K + 63) / 64);
    (p.job[k].transposed ? trans : plain) = true;
  }
  auto blocks = [&](int pack) { return (int64_t)tiles * p.jobs * ((most + pack - 1) / pack); };
  if (p.T <= 256) {
    // few tokens: the GPU is filled along K first, then by fewer adapters a pass
    p.splits = 8;
    while (p.splits > 1 && least < p.splits * 2) p.splits /= 2;
    int pack = 128 / wide;
    while (pack > 1 && blocks(pack) * p.splits < ctx->sm_count) pack /= 2;
    while (p.splits > 1 && blocks(pack) * p.splits > 4 * ctx->sm_count) p.splits /= 2;
    p.pack[0] = pack;
    p.pack[1] = p.rank > 64 ? 1 : std::min(2, pack);
    p.slots = (most + p.pack[trans] - 1) / p.pack[trans];
  } else {
    p.pack[0] = 128 / wide;
    p.pack[1] = p.rank > 64 ? 1 : 2;
    p.splits = 1;
    while (p.splits < 8 && (int64_t)tiles * p.jobs * p.splits * 2 <= ctx->sm_count && least >= p.splits * 2 * 4) p.splits *= 2;
    p.slots = (int)std::max<int64_t>(1, std::min<int64_t>((most + p.pack[trans] - 1) / p.pack[trans], ctx->sm_count / ((int64_t)tiles * p.jobs * p.splits)));
  }
  const int sums = p.rows * (p.rank + 4) * 4 + (kRows - p.rows) * 128;
  p.stage_bytes = p.rows * 128 + std::max(plain ? p.pack[0] * wide * 128 : 0, trans ? (p.rank > 64 ? 16384 : p.pack[1] * 8192) : 0);
  // All blocks at once where they can be: an SM's share of its memory (228 KB, of which a block takes 1 KB and 2.4 KB beside
  // the stages) bounds the stages.  Up to 256 tokens a block of the projection, which may start while this kernel runs,
  // finds room beside them where it takes half of an SM's (not where launch_projection gives it the whole, see `two` there).
  const int64_t all = (int64_t)tiles * p.splits * p.jobs * p.slots, each = (all + ctx->sm_count - 1) / ctx->sm_count;
  const int room = (228 * 1024 - (p.T <= 256 ? kProjectShare : 0)) / (int)std::min<int64_t>(each, 4) - 3584;
  const int chunks = (std::max(p.job[0].K, p.job[p.jobs - 1].K) + 63) / 64;
  p.stages = std::max(2, std::min({kStages, (room - 1024 - sums) / p.stage_bytes, (chunks + p.splits - 1) / p.splits}));
  while (p.stages > 2 && 1024 + p.stages * p.stage_bytes + sums > kLowSmem) p.stages--;
  // No more blocks an SM than its 512 columns of tensor memory serve: another would hold shared memory only to wait.
  const int columns = p.pack[0] * wide <= 32 ? 32 : p.pack[0] * wide <= 64 ? 64 : 128;  // at least those of the transposed job
  const int smem = std::max(1024 + p.stages * p.stage_bytes + sums, 228 * 1024 / (512 / (2 * columns) + 1) + 1);
  const windq_status ready = prepare_kernel(ctx, kLowRank, low_rank_kernel, kLowThreads, kLowSmem, false);
  if (ready != WINDQ_OK) return ready;
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  CUtensorMap z[2], pm[2];
  for (int k = 0; k < 2; k++) {
    const LowJob& j = p.job[k < p.jobs ? k : 0];
    bool ok = make_map(&z[k], p.dtype, j.Z, j.K, p.T, 0, j.ldz, 0, p.rows);
    if (j.transposed) ok = ok && make_map(&pm[k], p.dtype, j.P, p.rank, j.K, p.n_adapters, p.rank, (int64_t)j.K * p.rank, 64);
    else ok = ok && make_map(&pm[k], p.dtype, j.P, j.K, p.rank, p.n_adapters, j.K, (int64_t)j.K * p.rank, (p.rank + 15) & ~15);
    WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)(p.jobs * p.slots + (p.lists ? 1 : 0)));
  cfg.blockDim = dim3(kLowThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = p.splits;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = p.splits > 1 ? 2 : 1;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, low_rank_kernel, z[0], pm[0], z[1], pm[1], p));
  return WINDQ_OK;
}

}  // namespace

windq_status launch_low_rank(windq_ctx* ctx, const LowRank& q, cudaStream_t st) {
  LowRankArgs p = {};
  for (int k = 0; k < q.jobs; k++) {
    const LowRankJob& j = q.job[k];
    p.job[k] = LowJob{(const uint16_t*)j.Z, j.ldz, (const uint16_t*)j.P, j.S, (uint16_t*)j.pair, j.shift, j.top, (int)j.K, j.transposed};
  }
  p.jobs = q.jobs;
  p.T = (int)q.T;
  p.rank = q.rank;
  p.n_adapters = (int)q.n_adapters;
  p.dtype = q.dtype;
  p.scaling = q.scaling;
  p.adapter_of = q.adapter_of;
  p.lists = q.lists;
  p.list_rows = token_tile(q.T);
  p.list_tiles = (int)((q.T + p.list_rows - 1) / p.list_rows);
  p.stalls = stalls_of(ctx);
  return launch(ctx, p, st);
}

}  // namespace windq
