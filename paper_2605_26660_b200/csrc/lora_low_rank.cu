// S[t][j] = scaling[a] * sum_k Z[t][k] P[a](j, k) with a = adapter_of[t]: the low-rank product of the adapter calls, whose
// result (rank values a token) the projection and the gradients take.  Bound by reading Z and the used P once.
//
// Two kernels.  Above 256 tokens neighbours share adapters and a tile of 128 tokens times the P of its adapters goes to the
// tensor cores by TMA (many_tokens_kernel).  Up to 256 tokens every token may have its own adapter; what counts then is
// to have all of the P in flight at once, and warps with register operands do that (few_tokens_kernel).
#include <algorithm>

#include "lora.cuh"
#include "tcgen05.cuh"
#include "warp_mma.cuh"

namespace windq {
namespace {

constexpr int kLowWarps = 8, kLowThreads = 256;

struct LowJob {
  const uint16_t* Z;
  int64_t ldz;
  const uint16_t* P;  // [a][j][k], or transposed [a][k][j]
  float* S;        // binary32, or NULL
  uint16_t* pair;  // [t][2][j]: the two 16-bit values whose sum stands for S, or NULL
  float* top;      // largest |S[t][j]| of a token, or NULL
  int K, transposed;
};
struct LowRankArgs {
  LowJob job[2];
  int T, rank, n_adapters, dtype, jobs, slots, splits, stages;
  const float* scaling;
  const int32_t* adapter_of;
  int* lists;  // adapters of the projection's token tiles, or NULL
  int list_rows, list_tiles;
  unsigned long long* stalls;
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
    float v[4] = {y[0].x * scale, y[0].y * scale, y[0].z * scale, y[0].w * scale};
    const int64_t at = (int64_t)(t0 + i) * p.rank + j;
    if (job.S) *reinterpret_cast<float4*>(job.S + at) = make_float4(v[0], v[1], v[2], v[3]);
    if (job.top) atomicMax(&tops[i], __float_as_int(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])))));
    if (job.pair) {
      // 22 bits of fp16 (saturating: the first value takes what it can, the second up to as much again), 16 of bf16
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int k = 0; k < 2; k++) {
        float a = v[2 * k], b = v[2 * k + 1];
        if (p.dtype == WINDQ_F16) {
          a = fminf(fmaxf(a, -131008.0f), 131008.0f);
          b = fminf(fmaxf(b, -131008.0f), 131008.0f);
          hi[k] = pack2(fminf(fmaxf(a, -65504.0f), 65504.0f), fminf(fmaxf(b, -65504.0f), 65504.0f), p.dtype);
        } else {
          hi[k] = pack2(a, b, p.dtype);
        }
        const float2 back = unpack2(hi[k], p.dtype);
        lo[k] = pack2(a - back.x, b - back.y, p.dtype);
      }
      uint16_t* out = job.pair + (int64_t)(t0 + i) * 2 * p.rank + j;
      *reinterpret_cast<uint2*>(out) = make_uint2(hi[0], hi[1]);
      *reinterpret_cast<uint2*>(out + p.rank) = make_uint2(lo[0], lo[1]);
    }
  }
  if (job.top) {
    __syncthreads();
    for (int x = threadIdx.x; x < share; x += kLowThreads) {
      const int i = split + x * p.splits;
      if (kept(i)) job.top[t0 + i] = __int_as_float(tops[i]);
    }
  }
}

// ---- up to 256 tokens ----------------------------------------------------------------------------------------------

constexpr int kFew = 16;  // tokens of a thread block
__host__ __device__ constexpr int few_batch(int nb) { return nb <= 4 ? 4 : nb <= 8 ? 2 : 1; }

// A thread block takes 16 tokens and, one after another, the adapters they use (every slots-th of them): for each the whole
// tile times P[a], of which the rows of its own tokens are kept -- the product's rows would be idle anyway.  The eight warps
// split K in blocks of 32 and so do the `splits` blocks of a cluster; sums are joined in a fixed order.  A warp loads a
// batch of blocks before it multiplies them: one memory latency a batch is most of the time.
//
// The order of K inside a block of 32 does not matter as long as both operands share it: a lane takes eight consecutive
// values (16 bytes) of a row as its part of two k16 steps, so both operands are loaded straight into the layout of the
// matrix product with 64-byte pieces of every row.  Transposed P[a] (k rows of j) goes through shared memory.
template <int NB, bool TRANS>
__device__ __forceinline__ void few_tokens(const LowRankArgs& p, const LowJob& job, uint4* shared, const int* ids, const int* used,
                                           int* tops, int n_used, int t0, int split) {
  constexpr int kBatch = few_batch(NB);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
  const bool bf = p.dtype == WINDQ_BF16;
  const int blocks = (job.K + 31) >> 5, step = kLowWarps * p.splits, r = p.rank;
  const int pitch = r * 2 + 16;                                               // bytes of a row of transposed P[a]
  const uint32_t stage = smem_addr(shared) + warp * kBatch * 32 * pitch;      // a batch a warp
  float* sums = reinterpret_cast<float*>(shared);                             // after the products: partial sums
  auto row_part = [&](const uint16_t* row, int k) {  // values k .. k + 7 of a row of K, zeros past its end
    uint4 x = make_uint4(0, 0, 0, 0);
    if (k + 8 <= job.K) {
      x = *reinterpret_cast<const uint4*>(row + k);
    } else if (k < job.K) {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (k + i < job.K) w[i >> 1] |= (uint32_t)row[k + i] << (16 * (i & 1));
      x = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return x;
  };
  for (int d = blockIdx.y; d < n_used; d += p.slots) {
    const int a = used[d];
    const uint16_t* P = job.P + (int64_t)a * r * job.K;
    float acc[NB][4];
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int k = 0; k < 4; k++) acc[n][k] = 0.0f;
    for (int kb0 = split * kLowWarps + warp; kb0 < blocks; kb0 += kBatch * step) {
      uint4 z[kBatch][2], b[kBatch][TRANS ? 1 : NB];
#pragma unroll
      for (int e = 0; e < kBatch; e++) {
        const int kb = kb0 + e * step, k = kb * 32 + q * 8;
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const int t = t0 + h * 8 + g;
          z[e][h] = t < p.T ? row_part(job.Z + t * job.ldz, k) : make_uint4(0, 0, 0, 0);
        }
        if (TRANS) {
          // lane = row of the block; rows are kept in the order of the matrix product: (step, half, pair, element)
          const int row = kb * 32 + lane, slot = ((lane >> 1) & 3) * 8 + (lane >> 3) * 2 + (lane & 1);
          const uint16_t* src = P + (int64_t)(row < job.K ? row : 0) * r;
          for (int n = 0; n < r / 8; n++) copy16(stage + (e * 32 + slot) * pitch + n * 16, src + n * 8, row < job.K ? 16 : 0);
        } else {
#pragma unroll
          for (int n = 0; n < NB; n++)
            if (n * 8 < r) b[e][n] = row_part(P + (int64_t)(n * 8 + g) * job.K, k);
        }
      }
      if (TRANS) {
        copy_commit();
        copy_wait<0>();
        __syncwarp();
      }
#pragma unroll
      for (int e = 0; e < kBatch; e++) {
        const uint32_t first[4] = {z[e][0].x, z[e][1].x, z[e][0].y, z[e][1].y}, second[4] = {z[e][0].z, z[e][1].z, z[e][0].w, z[e][1].w};
#pragma unroll
        for (int n = 0; n < NB; n++) {
          if (n * 8 < r) {
            uint32_t w[4];
            if (TRANS) {
              ldmatrix_trans(stage + (e * 32 + lane) * pitch + n * 16, w);
            } else {
              const uint4& x = b[e][TRANS ? 0 : n];
              w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
            }
            mma16816(acc[n], first, w[0], w[1], bf);
            mma16816(acc[n], second, w[2], w[3], bf);
          }
        }
      }
      if (TRANS) __syncwarp();
    }
    // join the warps: 4 + 4, 2 + 2, 1 + 1
    __syncthreads();
#pragma unroll
    for (int half = kLowWarps / 2; half >= 1; half >>= 1) {
      if (warp >= half && warp < 2 * half) {
        float* out = sums + (warp - half) * NB * 128 + lane;
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int k = 0; k < 4; k++) out[(n * 4 + k) * 32] = acc[n][k];
      }
      __syncthreads();
      if (warp < half) {
        const float* in = sums + warp * NB * 128 + lane;
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int k = 0; k < 4; k++) acc[n][k] += in[(n * 4 + k) * 32];
      }
      __syncthreads();
    }
    constexpr int kRow = NB * 8 + 4;  // [token][j]
    if (warp == 0) {
#pragma unroll
      for (int n = 0; n < NB; n++)
#pragma unroll
        for (int k = 0; k < 4; k++) sums[(g + (k >> 1) * 8) * kRow + n * 8 + q * 2 + (k & 1)] = acc[n][k];
    }
    __syncwarp();
    if (p.splits > 1) cluster_sync();
    else __syncthreads();
    finish_tokens(p, job, t0, kFew, smem_addr(sums), kRow, split, ids, tops, [&](int i) { return ids[i] == a; });
    __syncwarp();
    if (p.splits > 1) cluster_sync();
    else __syncthreads();
  }
}

template <int NB>
__global__ void __launch_bounds__(kLowThreads) few_tokens_kernel(const __grid_constant__ LowRankArgs p) {
  extern __shared__ uint4 shared[];
  __shared__ int ids[256], used[kFew], tops[kFew], taken[kLowWarps];
  launch_dependents();
  const int split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
  if (blockIdx.y == p.slots) {
    if (split == 0 && blockIdx.z == 0 && tile < p.list_tiles) write_list(p, tile, ids, taken);
    return;  // of a whole cluster: it has no other barrier
  }
  const int t0 = tile * kFew;
  int n_used;
  const int id = threadIdx.x < kFew ? valid_id(p, t0 + threadIdx.x) : -1, place = first_place(id, kFew, ids, taken, &n_used);
  if (place >= 0) used[place] = id;
  if (threadIdx.x < kFew) tops[threadIdx.x] = 0;
  __syncthreads();
  const LowJob& job = p.job[blockIdx.z];
  if (job.transposed) few_tokens<NB, true>(p, job, shared, ids, used, tops, n_used, t0, split);
  else few_tokens<NB, false>(p, job, shared, ids, used, tops, n_used, t0, split);
}

template <int NB>
windq_status launch_few(windq_ctx* ctx, int id, LowRankArgs p, cudaStream_t st) {
  const int tiles = (p.T + kFew - 1) / kFew;
  // blocks for the GPU to hold four times over: first over the adapters of a tile, then along K
  p.slots = std::max(1, std::min({kFew, p.T, p.n_adapters}));
  p.splits = 1;
  const int most = std::max(p.job[0].K, p.jobs > 1 ? p.job[1].K : 0);
  while (p.splits < 8 && (int64_t)tiles * p.slots * p.jobs * p.splits * 2 <= 4 * ctx->sm_count &&
         (most + 31) / 32 >= 2 * kLowWarps * p.splits)
    p.splits *= 2;
  const int sums = std::max(kLowWarps / 2 * NB * 128, kFew * (NB * 8 + 4)) * 4;
  const bool trans = p.job[0].transposed || (p.jobs > 1 && p.job[1].transposed);
  const int smem = std::max(sums, trans ? kLowWarps * few_batch(NB) * 32 * (p.rank * 2 + 16) : 0);
  constexpr int kMost = 128 * 1024;
  static_assert(kLowWarps * few_batch(NB) * 32 * (NB * 16 + 16) <= kMost, "a batch of every warp");
  const windq_status ready = prepare_kernel(ctx, id, few_tokens_kernel<NB>, kLowThreads, kMost, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)(p.slots + (p.lists ? 1 : 0)), (unsigned)p.jobs);
  cfg.blockDim = dim3(kLowThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = p.splits;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = p.splits > 1 ? 1 : 0;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, few_tokens_kernel<NB>, p));
  return WINDQ_OK;
}

// ---- more tokens ---------------------------------------------------------------------------------------------------

constexpr int kMany = 128;  // tokens of a tile
constexpr int kManyStages = 8;
constexpr int kManySmem = 227 * 1024 - 3072;

// A tile of 128 tokens (rows of the accumulator) times the P of its adapters (columns, 16-padded): as many adapters at a
// time as 128 columns hold (transposed, where an adapter takes a block of 64 columns of shared memory: two), one pass over
// K each.  A tile in which one prompt ends and the next begins then still takes one pass; with one adapter a pass such
// tiles took twice as long and with them the whole kernel (41 against 22 us for 8192 tokens of 4096 values, rank 64).  Blocks of a cluster share K.  Warps: one issues TMA
// copies, one the products, four take the rows of their own adapter out of tensor memory.
__global__ void __launch_bounds__(kLowThreads, 1)
    many_tokens_kernel(const __grid_constant__ CUtensorMap z0, const __grid_constant__ CUtensorMap p0,
                       const __grid_constant__ CUtensorMap z1, const __grid_constant__ CUtensorMap p1,
                       const __grid_constant__ LowRankArgs p) {
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t full_[kManyStages], empty_[kManyStages], done_, free_;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead, ids[256], used[kMany], tops[kMany], taken[kLowWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  launch_dependents();
  const int split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
  if (blockIdx.y == p.jobs) {
    if (split == 0 && tile < p.list_tiles) write_list(p, tile, ids, taken);
    return;  // of a whole cluster
  }
  const LowJob& job = p.job[blockIdx.y];
  const CUtensorMap* zmap = blockIdx.y ? &z1 : &z0;
  const CUtensorMap* pmap = blockIdx.y ? &p1 : &p0;
  const bool trans = job.transposed;
  const int r = p.rank, wide = (r + 15) & ~15;
  const int pack = trans ? (r > 64 ? 1 : 2) : 128 / wide;      // adapters of a pass
  const int apart = trans ? 64 : wide;                          // their columns
  constexpr uint32_t stage_bytes = kMany * 128 + 16384, columns = 128;
  const uint32_t base = (smem_addr(raw) + 1023) & ~1023u, sums = base + p.stages * stage_bytes;
  auto full = [&](int s) { return smem_addr(&full_[s]); };
  auto empty = [&](int s) { return smem_addr(&empty_[s]); };
  const uint32_t done = smem_addr(&done_), free = smem_addr(&free_);
  const int t0 = tile * kMany;

  if (tid == 0) {
    prefetch_map(zmap);
    prefetch_map(pmap);
    for (int s = 0; s < p.stages; s++) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    mbar_init(done, 1);
    mbar_init(free, 4);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<false>(smem_addr(&tmem_slot), columns);
  int n_used;
  const int id = tid < kMany ? valid_id(p, t0 + tid) : -1, place = first_place(id, kMany, ids, taken, &n_used);
  if (place >= 0) used[place] = id;
  if (tid < kMany) tops[tid] = 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int chunks = (job.K + 63) >> 6, c0 = (int)((int64_t)chunks * split / p.splits), c1 = (int)((int64_t)chunks * (split + 1) / p.splits);
  const int passes = (n_used + pack - 1) / pack;

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int pass = 0; ok && pass < passes; pass++) {
        const int count = min(pack, n_used - pass * pack);
        const uint32_t bytes = kMany * 128 + (trans ? (r > 64 ? 16384 : count * 8192) : count * wide * 128);
        // every block begins elsewhere in its part of K: rows are a power of two apart in most models, and blocks that
        // walk them in step would meet on few memory channels
        int c = c0 + (tile * 5 + split * 3) % max(1, c1 - c0);
        for (int i = c0; i < c1; i++, c = c + 1 < c1 ? c + 1 : c0) {
          if (!(ok = mbar_wait(empty(s), phase ^ 1, &dead))) break;
          const uint32_t at = base + s * stage_bytes;
          mbar_expect(full(s), bytes);
          tma_load_2d<false>(at, zmap, c * 64, t0, full(s));
          if (trans) {
            for (int u = 0; u < count; u++) tma_load_3d<false>(at + kMany * 128 + u * 8192, pmap, 0, c * 64, used[pass * pack + u], full(s));
            if (r > 64) tma_load_3d<false>(at + kMany * 128 + 8192, pmap, 64, c * 64, used[pass], full(s));
          } else {
            for (int u = 0; u < count; u++)
              tma_load_3d<false>(at + kMany * 128 + u * wide * 128, pmap, c * 64, 0, used[pass * pack + u], full(s));
          }
          if (++s == p.stages) s = 0, phase ^= 1;
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint64_t z_desc = smem_desc(base, 16), p_desc = smem_desc(base + kMany * 128, trans ? 8192 : 16);
      const uint32_t p_step = trans ? 2048 >> 4 : 32 >> 4;
      int s = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int pass = 0; ok && pass < passes; pass++) {
        const int count = min(pack, n_used - pass * pack);
        const uint32_t idesc = instr_desc(p.dtype, false, trans, 128, trans ? wide : count * wide);
        if (!(ok = mbar_wait(free, (pass & 1) ^ 1, &dead))) break;
        tc_fence_after();
        for (int c = c0; c < c1; c++) {
          if (!(ok = mbar_wait(full(s), phase, &dead))) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)(s * stage_bytes >> 4);
#pragma unroll
          for (int k = 0; k < 4; k++)
            mma_f16<false>(tmem, z_desc + off + k * (32 >> 4), p_desc + off + k * p_step, idesc, c > c0 || k > 0);
          if (trans && count > 1) {
#pragma unroll
            for (int k = 0; k < 4; k++)
              mma_f16<false>(tmem + 64, z_desc + off + k * (32 >> 4), p_desc + off + (8192 >> 4) + k * p_step, idesc, c > c0 || k > 0);
          }
          mma_commit<false>(empty(s), 0);
          if (++s == p.stages) s = 0, phase ^= 1;
        }
        if (ok) mma_commit<false>(done, 0);
      }
    }
  } else if (warp < 6) {
    const int quarter = warp & 3, row = quarter * 32 + lane, mine = ids[row];
    for (int pass = 0; pass < passes; pass++) {
      const bool ok = mbar_wait(done, pass & 1, &dead);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const int count = min(pack, n_used - pass * pack);
      for (int i = 0; i < count; i++) {
        const bool keep = mine == used[pass * pack + i];
        if (!__any_sync(0xffffffffu, keep)) continue;
        for (int c = 0; c < wide; c += 16) {
          uint32_t x[16];
          tmem_load16(tmem + ((uint32_t)(quarter * 32) << 16) + i * apart + c, x);
          tmem_load_wait();
          if (keep) {
#pragma unroll
            for (int k = 0; k < 16; k++)
              if (c + k < r) asm volatile("st.shared.b32 [%0], %1;" ::"r"(sums + (row * (r + 4) + c + k) * 4), "r"(x[k]) : "memory");
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(free);
    }
  }
  __syncwarp();
  __syncthreads();
  if (dead && tid == 0) {
    const long long begin = clock64();
    while (clock64() - begin < 4000000) {
    }
    atomicAdd(p.stalls, 1ull);
  }
  __syncwarp();
  if (p.splits > 1) cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_free<false>(tmem, columns);
  }
  finish_tokens(p, job, t0, kMany, sums, r + 4, split, ids, tops, [&](int i) { return ids[i] >= 0; });
  __syncwarp();
  if (p.splits > 1) cluster_sync();
}

windq_status launch_many(windq_ctx* ctx, LowRankArgs p, cudaStream_t st) {
  const int tiles = (p.T + kMany - 1) / kMany;
  int least = (p.job[0].K + 63) / 64;
  if (p.jobs > 1) least = std::min(least, (p.job[1].K + 63) / 64);
  p.splits = 1;
  while (p.splits < 8 && (int64_t)tiles * p.jobs * p.splits * 2 <= ctx->sm_count && least >= p.splits * 2 * 4) p.splits *= 2;
  const int stage = kMany * 128 + 16384, sums = kMany * (p.rank + 4) * 4;
  p.stages = std::min(kManyStages, (kManySmem - 1024 - sums) / stage);
  const windq_status ready = prepare_kernel(ctx, kLowRankMany, many_tokens_kernel, kLowThreads, kManySmem, false);
  if (ready != WINDQ_OK) return ready;
  WINDQ_REQUIRE(ctx, encode_tiled(), WINDQ_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  CUtensorMap z[2], pm[2];
  for (int k = 0; k < 2; k++) {
    const LowJob& j = p.job[k < p.jobs ? k : 0];
    bool ok = make_map(&z[k], p.dtype, j.Z, j.K, p.T, 0, j.ldz, 0, kMany);
    if (j.transposed) ok = ok && make_map(&pm[k], p.dtype, j.P, p.rank, j.K, p.n_adapters, p.rank, (int64_t)j.K * p.rank, 64);
    else ok = ok && make_map(&pm[k], p.dtype, j.P, j.K, p.rank, p.n_adapters, j.K, (int64_t)j.K * p.rank, (p.rank + 15) & ~15);
    WINDQ_REQUIRE(ctx, ok, WINDQ_ERR_CUDA, "a tensor map could not be made");
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)(p.jobs + (p.lists ? 1 : 0)));
  cfg.blockDim = dim3(kLowThreads);
  cfg.dynamicSmemBytes = 1024 + p.stages * stage + sums;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = p.splits;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = p.splits > 1 ? 1 : 0;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, many_tokens_kernel, z[0], pm[0], z[1], pm[1], p));
  return WINDQ_OK;
}

}  // namespace

windq_status launch_low_rank(windq_ctx* ctx, const LowRank& q, cudaStream_t st) {
  LowRankArgs p = {};
  for (int k = 0; k < q.jobs; k++) {
    const LowRankJob& j = q.job[k];
    p.job[k] = LowJob{(const uint16_t*)j.Z, j.ldz, (const uint16_t*)j.P, j.S, (uint16_t*)j.pair, j.top, (int)j.K, j.transposed};
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
  p.stalls = stall_counter(ctx);
  if (q.T > 256) return launch_many(ctx, p, st);
  if (q.rank <= 8) return launch_few<1>(ctx, kLowRankFew, p, st);
  if (q.rank <= 16) return launch_few<2>(ctx, kLowRankFew + 1, p, st);
  if (q.rank <= 32) return launch_few<4>(ctx, kLowRankFew + 2, p, st);
  if (q.rank <= 64) return launch_few<8>(ctx, kLowRankFew + 3, p, st);
  return launch_few<16>(ctx, kLowRankFew + 4, p, st);
}

}  // namespace windq
