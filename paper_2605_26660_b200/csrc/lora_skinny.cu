// The skinny products of the adapter calls: S (tokens x rank) and the gradients of A and B.
//
// Both read a token matrix once and have a result of rank values per token or per channel; they are bound by that read
// (HBM or L2) and use warp-level matrix products (mma.sync m16n8k16), whose operands come straight from where the loads
// put them -- tcgen05 would need whole 128-row tiles of one adapter, and there is nothing to gain from its rate.
#include <algorithm>

#include "lora.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool bf) {
  if (bf)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// 16 bytes of which the first `bytes` are read and the rest is zero.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ---- S[t][j] = scaling[a] * sum_k Z[t][k] P[a](j, k), a = adapter_of[t] --------------------------------------------

constexpr int kLowWarps = 8;

struct LowRankArgs {
  const uint16_t* Z;
  int64_t ldz;
  const uint16_t* P;  // [a][j][k], or transposed [a][k][j]
  int T, K, rank, n_adapters, bf, tiles, slots, splits;
  const float* scaling;
  const int32_t* adapter_of;
  float* S;
  float* top;  // largest |S[t][j]| of a token, or NULL
  int* lists;  // adapters of the projection's token tiles, or NULL
  int list_rows, list_tiles;
};

// Adapters of the tokens of one tile in the order of their first token; one thread a token, blockDim.x >= rows.
__device__ void write_list(const LowRankArgs& p, int tile, int* ids, int* taken) {
  const int i = threadIdx.x;
  const int64_t at = (int64_t)tile * p.list_rows + i;
  int id = i < p.list_rows && at < p.T ? p.adapter_of[at] : -1;
  if (id >= p.n_adapters) id = -1;
  ids[i] = id;
  __syncthreads();
  bool first = id >= 0;
  for (int k = 0; k < i && first; k++) first = ids[k] != id;
  const unsigned vote = __ballot_sync(0xffffffffu, first);
  if ((i & 31) == 0) taken[i >> 5] = __popc(vote);
  __syncthreads();
  int before = __popc(vote & ((1u << (i & 31)) - 1)), all = 0;
  for (int w = 0; w < kLowWarps; w++) {
    if (w < i >> 5) before += taken[w];
    all += taken[w];
  }
  int* list = p.lists + (int64_t)tile * (p.list_rows + 1);
  if (first) list[1 + before] = id;
  if (i == 0) list[0] = all;
}

// A thread block takes 16 MT tokens and, one after another, the adapters they use (every slots-th of them): for each the
// whole tile times P[a], of which the rows of its own tokens are kept -- one pass for prompts, whose neighbours share an
// adapter, and cheap for single tokens, whose matrix-product rows would be idle anyway.  The eight warps split K in blocks
// of 32 and so do the `splits` blocks of a cluster; sums are joined in a fixed order.
//
// The order of K inside a block of 32 does not matter as long as both operands share it: a lane takes eight consecutive
// values (16 bytes) of a row as its part of two k16 steps, so both operands are loaded straight into the layout of the
// matrix product with 64-byte pieces of every row.  Transposed P[a] (k rows of j) goes through shared memory.
template <int MT, int NB, bool TRANS>
__global__ void __launch_bounds__(kLowWarps * 32) low_rank_kernel(const __grid_constant__ LowRankArgs p) {
  extern __shared__ uint4 shared[];
  __shared__ int ids[256], used[16 * MT], n_used, taken[kLowWarps];
  constexpr int kTokens = 16 * MT;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
  launch_dependents();
  const int split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
  if (blockIdx.y == p.slots) {
    if (split == 0 && tile < p.list_tiles) write_list(p, tile, ids, taken);
    return;  // of a whole cluster: it has no other barrier
  }
  const int t0 = tile * kTokens;
  if (tid < kTokens) {
    const int t = t0 + tid;
    const int id = t < p.T ? p.adapter_of[t] : -1;
    ids[tid] = id < p.n_adapters ? id : -1;
  }
  __syncthreads();
  if (warp == 0) {
    int n = 0;
#pragma unroll
    for (int h = 0; h < kTokens; h += 32) {
      const int i = h + lane;
      bool first = i < kTokens && ids[i] >= 0;
      for (int k = 0; k < i && first; k++) first = ids[k] != ids[i];
      const unsigned vote = __ballot_sync(0xffffffffu, first);
      if (first) used[n + __popc(vote & ((1u << lane) - 1))] = ids[i];
      n += __popc(vote);
    }
    if (lane == 0) n_used = n;
  }
  __syncthreads();

  const int blocks = (p.K + 31) >> 5, step = kLowWarps * p.splits;
  const int pitch = p.rank * 2 + 16;                                    // bytes of a row of transposed P[a] in shared memory
  const uint32_t stage = smem_addr(shared) + warp * 2 * 32 * pitch;     // two stages a warp
  float* sums = reinterpret_cast<float*>(shared);                       // after the products: partial sums
  const int r = p.rank;

  for (int d = blockIdx.y; d < n_used; d += p.slots) {
    const int a = used[d];
    const uint16_t* P = p.P + (int64_t)a * r * p.K;
    float acc[MT][NB][4];
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
      for (int n = 0; n < NB; n++)
#pragma unroll
        for (int k = 0; k < 4; k++) acc[m][n][k] = 0.0f;

    auto row_part = [&](const uint16_t* row, int k) {  // values k .. k + 7 of a row of K, zeros past its end
      uint4 x = make_uint4(0, 0, 0, 0);
      if (k + 8 <= p.K) {
        x = *reinterpret_cast<const uint4*>(row + k);
      } else if (k < p.K) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; i++)
          if (k + i < p.K) w[i >> 1] |= (uint32_t)row[k + i] << (16 * (i & 1));
        x = make_uint4(w[0], w[1], w[2], w[3]);
      }
      return x;
    };
    uint4 z[MT][2], b[TRANS ? 1 : NB], z_next[MT][2], b_next[TRANS ? 1 : NB];
    auto fetch = [&](int kb, uint4 (&zz)[MT][2], uint4 (&bb)[TRANS ? 1 : NB], int buffer) {
      const int k = kb * 32 + q * 8;
#pragma unroll
      for (int m = 0; m < MT; m++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const int t = t0 + m * 16 + h * 8 + g;
          zz[m][h] = t < p.T ? row_part(p.Z + t * p.ldz, k) : make_uint4(0, 0, 0, 0);
        }
      if (TRANS) {
        // lane = row of the block; rows are kept in the order of the matrix product: (step, half, pair, element)
        const int row = kb * 32 + lane, slot = ((lane >> 1) & 3) * 8 + (lane >> 3) * 2 + (lane & 1);
        const uint16_t* src = P + (int64_t)(row < p.K ? row : 0) * r;
        for (int n = 0; n < r / 8; n++)
          copy16(stage + buffer * 32 * pitch + slot * pitch + n * 16, src + n * 8, row < p.K ? 16 : 0);
        copy_commit();
      } else {
#pragma unroll
        for (int n = 0; n < NB; n++)
          if (n * 8 < r) bb[n] = row_part(P + (int64_t)(n * 8 + g) * p.K, k);
      }
    };
    int kb = split * kLowWarps + warp, buffer = 0;
    if (kb < blocks) fetch(kb, z, b, 0);
    for (; kb < blocks; kb += step, buffer ^= 1) {
      const bool more = kb + step < blocks;
      if (more) fetch(kb + step, z_next, b_next, buffer ^ 1);
      if (TRANS) {
        if (more) copy_wait<1>();
        else copy_wait<0>();
        __syncwarp();
      }
#pragma unroll
      for (int n = 0; n < NB; n++) {
        if (n * 8 < r) {
          uint32_t w[4];
          if (TRANS) {
            ldmatrix_trans(stage + buffer * 32 * pitch + lane * pitch + n * 16, w);
          } else {
            w[0] = b[TRANS ? 0 : n].x, w[1] = b[TRANS ? 0 : n].y, w[2] = b[TRANS ? 0 : n].z, w[3] = b[TRANS ? 0 : n].w;
          }
#pragma unroll
          for (int m = 0; m < MT; m++) {
            const uint32_t first[4] = {z[m][0].x, z[m][1].x, z[m][0].y, z[m][1].y}, second[4] = {z[m][0].z, z[m][1].z, z[m][0].w, z[m][1].w};
            mma16816(acc[m][n], first, w[0], w[1], p.bf);
            mma16816(acc[m][n], second, w[2], w[3], p.bf);
          }
        }
      }
      if (TRANS) __syncwarp();
      if (more) {
#pragma unroll
        for (int m = 0; m < MT; m++) z[m][0] = z_next[m][0], z[m][1] = z_next[m][1];
#pragma unroll
        for (int n = 0; n < (TRANS ? 1 : NB); n++) b[n] = b_next[n];
      }
    }
    // join the warps: 4 + 4, 2 + 2, 1 + 1
    __syncthreads();
#pragma unroll
    for (int half = kLowWarps / 2; half >= 1; half >>= 1) {
      if (warp >= half && warp < 2 * half) {
        float* out = sums + (warp - half) * MT * NB * 128 + lane;
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
          for (int n = 0; n < NB; n++)
#pragma unroll
            for (int k = 0; k < 4; k++) out[((m * NB + n) * 4 + k) * 32] = acc[m][n][k];
      }
      __syncthreads();
      if (warp < half) {
        const float* in = sums + warp * MT * NB * 128 + lane;
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
          for (int n = 0; n < NB; n++)
#pragma unroll
            for (int k = 0; k < 4; k++) acc[m][n][k] += in[((m * NB + n) * 4 + k) * 32];
      }
      __syncthreads();
    }
    // [token][j]
    constexpr int kRow = NB * 8 + 1;
    if (warp == 0) {
#pragma unroll
      for (int m = 0; m < MT; m++)
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int k = 0; k < 4; k++) sums[(m * 16 + g + (k >> 1) * 8) * kRow + n * 8 + q * 2 + (k & 1)] = acc[m][n][k];
    }
    if (p.splits > 1) cluster_sync();
    else __syncthreads();
    const float scale = p.scaling[a];
    for (int i = split + warp * p.splits; i < kTokens; i += kLowWarps * p.splits) {
      if (ids[i] != a) continue;  // the same for the whole warp
      float top = 0.0f;
      for (int j = lane; j < r; j += 32) {
        float x = 0.0f;
        if (p.splits > 1) {
          for (int s = 0; s < p.splits; s++) x += cluster_load(smem_addr(&sums[i * kRow + j]), s);
        } else {
          x = sums[i * kRow + j];
        }
        x *= scale;
        p.S[(int64_t)(t0 + i) * r + j] = x;
        top = fmaxf(top, fabsf(x));
      }
      if (p.top) {
#pragma unroll
        for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        if (lane == 0) p.top[t0 + i] = top;
      }
    }
    __syncwarp();
    if (p.splits > 1) cluster_sync();
    else __syncthreads();
  }
}

template <int MT, int NB, bool TRANS>
windq_status launch_low_rank(windq_ctx* ctx, int id, LowRankArgs p, cudaStream_t st) {
  p.tiles = (p.T + 16 * MT - 1) / (16 * MT);
  // as many blocks as fill the GPU twice: first over the adapters of a tile, then along K
  const int room = 2 * ctx->sm_count;
  p.slots = std::max(1, std::min({16 * MT, p.T, p.n_adapters, MT == 1 ? 16 : room / p.tiles}));
  p.splits = 1;
  while (p.splits < 8 && (int64_t)p.tiles * p.slots * p.splits * 2 <= room && (p.K + 31) / 32 >= 2 * kLowWarps * p.splits) p.splits *= 2;
  const int sums = std::max(kLowWarps / 2 * MT * NB * 128, 16 * MT * (NB * 8 + 1)) * 4;
  const int smem = std::max(sums, TRANS ? kLowWarps * 2 * 32 * (p.rank * 2 + 16) : 0);
  constexpr int kMost = 160 * 1024;
  const windq_status ready = prepare_kernel(ctx, id, low_rank_kernel<MT, NB, TRANS>, kLowWarps * 32, kMost, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.tiles * p.splits), (unsigned)(p.slots + (p.lists ? 1 : 0)));
  cfg.blockDim = dim3(kLowWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = p.splits;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = p.splits > 1 ? 1 : 0;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, low_rank_kernel<MT, NB, TRANS>, p));
  return WINDQ_OK;
}

// ---- D[a][j][c] = sum over the tokens t of a of S[t][j] Z[t][c] ----------------------------------------------------

constexpr int kGradWarps = 8, kGradCols = 128, kGradTokens = 64, kGradStages = 3;
constexpr int kZPitch = kGradCols * 2 + 16;  // bytes
constexpr int kWindow = 1024;                // blocks of tokens whose activity is looked up at a time

struct GradJob {
  const uint16_t* Z;
  int64_t ldz;
  const float* S;
  const float* top;
  float* D;
  int cols, tiles;
  bool j_first;  // D[a][c][j] instead of D[a][j][c]
};
struct GradArgs {
  GradJob job[2];
  int T, rank, n_adapters, splits;
  const int32_t* adapter_of;
};

// A thread block owns 128 columns of Z for one adapter; a cluster of `splits` shares the tokens.  The tokens that are not
// the adapter's are left out as rows of zeros (copied with size zero, so that what they hold cannot spoil a sum), blocks
// of 64 tokens without any of its tokens are skipped.  Z is the transposed left operand (ldmatrix.trans); S enters as two
// fp16 or three bf16 values whose sum is S to 22 or 24 bits -- fp16 ones after a scaling by a power of two that puts the
// block's largest |S| near 2^13, undone at the end, so that small gradients keep their bits.
template <int NB, bool BF>
__global__ void __launch_bounds__(kGradWarps * 32) gradient_kernel(const __grid_constant__ GradArgs p) {
  constexpr int kTerms = BF ? 3 : 2;
  extern __shared__ uint4 shared[];
  __shared__ short active[kWindow];
  __shared__ unsigned short flags[kWindow];
  __shared__ int n_active;
  __shared__ float tops[kGradWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
  const int split = blockIdx.x % p.splits, a = blockIdx.y, r = p.rank;
  int tile = blockIdx.x / p.splits;
  const bool second = tile >= p.job[0].tiles;
  const GradJob& job = p.job[second];
  if (second) tile -= p.job[0].tiles;
  const int c0 = tile * kGradCols;
  const int all = (p.T + kGradTokens - 1) / kGradTokens;
  const int b0 = (int)((int64_t)all * split / p.splits), b1 = (int)((int64_t)all * (split + 1) / p.splits);
  wait_for_predecessor();

  float up = 1.0f, down = 1.0f;
  if (!BF) {
    float top = 0.0f;
    const int end = min(p.T, b1 * kGradTokens);
    for (int t = b0 * kGradTokens + tid; t < end; t += kGradWarps * 32)
      if (p.adapter_of[t] == a) top = fmaxf(top, job.top[t]);
#pragma unroll
    for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    if (lane == 0) tops[warp] = top;
    __syncthreads();
    for (int w = 0; w < kGradWarps; w++) top = fmaxf(top, tops[w]);
    // 2^e <= top < 2^(e + 1); both factors are kept normal
    const int e = (int)((__float_as_uint(top) >> 23) & 255) - 127, k = max(-100, min(100, 13 - e));
    up = __uint_as_float((uint32_t)(127 + k) << 23);
    down = __uint_as_float((uint32_t)(127 - k) << 23);
  }

  const int s_pitch = r * 2 + 16;
  const uint32_t z_base = smem_addr(shared), s_base = z_base + kGradStages * kGradTokens * kZPitch;
  float acc[NB][4];
#pragma unroll
  for (int n = 0; n < NB; n++)
#pragma unroll
    for (int k = 0; k < 4; k++) acc[n][k] = 0.0f;

  for (int w0 = b0; w0 < b1; w0 += kWindow) {
    const int count = min(kWindow, b1 - w0);
    __syncthreads();
    for (int b = warp; b < count; b += kGradWarps) {
      const int t = (w0 + b) * kGradTokens + lane;
      const bool mine = (t < p.T && p.adapter_of[t] == a) || (t + 32 < p.T && p.adapter_of[t + 32] == a);
      const unsigned vote = __ballot_sync(0xffffffffu, mine);
      if (lane == 0) flags[b] = vote != 0;
    }
    __syncthreads();
    if (warp == 0) {
      int n = 0;
      for (int h = 0; h < count; h += 32) {
        const bool on = h + lane < count && flags[h + lane];
        const unsigned vote = __ballot_sync(0xffffffffu, on);
        if (on) active[n + __popc(vote & ((1u << lane) - 1))] = (short)(h + lane);
        n += __popc(vote);
      }
      if (lane == 0) n_active = n;
    }
    __syncthreads();
    const int n_blocks = n_active;
    auto copy_z = [&](int i) {
      if (i < n_blocks) {
        const int t0 = (w0 + active[i]) * kGradTokens;
        const uint32_t at = z_base + (i % kGradStages) * kGradTokens * kZPitch;
#pragma unroll
        for (int h = 0; h < 4; h++) {
          const int x = h * kGradWarps * 32 + tid, row = x >> 4, piece = x & 15, t = t0 + row, c = c0 + piece * 8;
          const bool on = t < p.T && c < job.cols && p.adapter_of[t] == a;
          const int bytes = on ? min(16, (job.cols - c) * 2) : 0;
          copy16(at + row * kZPitch + piece * 16, on ? job.Z + t * job.ldz + c : job.Z, bytes);
        }
      }
      copy_commit();
    };
    // S of a block: pieces of eight values, kGradTokens * rank / 8 of them over 256 threads
    constexpr int kPieces = (kGradTokens * NB + kGradWarps * 32 - 1) / (kGradWarps * 32);
    float4 s_next[kPieces][2];
    auto load_s = [&](int i) {
      if (i >= n_blocks) return;
      const int t0 = (w0 + active[i]) * kGradTokens;
#pragma unroll
      for (int h = 0; h < kPieces; h++) {
        const int x = h * kGradWarps * 32 + tid, row = x / NB, piece = x % NB, t = t0 + row;
        s_next[h][0] = s_next[h][1] = make_float4(0, 0, 0, 0);
        if (row < kGradTokens && piece * 8 < r && t < p.T && p.adapter_of[t] == a) {
          const float4* src = reinterpret_cast<const float4*>(job.S + (int64_t)t * r + piece * 8);
          s_next[h][0] = src[0];
          s_next[h][1] = src[1];
        }
      }
    };
    auto write_s = [&] {
#pragma unroll
      for (int h = 0; h < kPieces; h++) {
        const int x = h * kGradWarps * 32 + tid, row = x / NB, piece = x % NB;
        if (row >= kGradTokens || piece * 8 >= r) continue;
        float y[8] = {s_next[h][0].x, s_next[h][0].y, s_next[h][0].z, s_next[h][0].w,
                      s_next[h][1].x, s_next[h][1].y, s_next[h][1].z, s_next[h][1].w};
#pragma unroll
        for (int k = 0; k < 8; k++) y[k] *= up;
#pragma unroll
        for (int term = 0; term < kTerms; term++) {
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; k++) {
            w[k] = pack2(y[2 * k], y[2 * k + 1], BF ? WINDQ_BF16 : WINDQ_F16);
            const float2 back = unpack2(w[k], BF ? WINDQ_BF16 : WINDQ_F16);
            y[2 * k] -= back.x;
            y[2 * k + 1] -= back.y;
          }
          const uint32_t at = s_base + (term * kGradTokens + row) * s_pitch + piece * 16;
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        }
      }
    };
    copy_z(0);
    copy_z(1);
    load_s(0);
    for (int i = 0; i < n_blocks; i++) {
      write_s();
      copy_wait<1>();
      __syncthreads();
      copy_z(i + 2);
      load_s(i + 1);
      const uint32_t z_at = z_base + (i % kGradStages) * kGradTokens * kZPitch;
#pragma unroll
      for (int k = 0; k < kGradTokens / 16; k++) {
        // left operand: columns 16 warp .. + 15 (rows of the product), tokens 16 k .. + 15
        uint32_t za[4];
        ldmatrix_trans(z_at + (k * 16 + (lane & 7) + (lane >> 4) * 8) * kZPitch + (warp * 16 + ((lane >> 3) & 1) * 8) * 2, za);
#pragma unroll
        for (int term = 0; term < kTerms; term++) {
          const uint32_t s_at = s_base + (term * kGradTokens + k * 16 + (lane & 15)) * s_pitch + (lane >> 4) * 16;
#pragma unroll
          for (int n = 0; n < NB; n += 2) {
            if (n * 8 < r) {
              uint32_t sb[4];
              // an odd last block has no right neighbour: its lanes read the left one again
              ldmatrix_trans((n + 1) * 8 < r ? s_at + n * 16 : s_at + n * 16 - (lane >> 4) * 16, sb);
              mma16816(acc[n], za, sb[0], sb[1], BF);
              if (n + 1 < NB && (n + 1) * 8 < r) mma16816(acc[n + 1 < NB ? n + 1 : n], za, sb[2], sb[3], BF);
            }
          }
        }
      }
      __syncthreads();
    }
    copy_wait<0>();
  }
  // join the cluster, [j][column] 129 apart
  __syncthreads();
  float* out = reinterpret_cast<float*>(shared);
#pragma unroll
  for (int n = 0; n < NB; n++)
    if (n * 8 < r) {
#pragma unroll
      for (int k = 0; k < 4; k++) out[(n * 8 + q * 2 + (k & 1)) * 129 + warp * 16 + g + (k >> 1) * 8] = acc[n][k] * down;
    }
  if (p.splits > 1) cluster_sync();
  else __syncthreads();
  const int cols = min(kGradCols, job.cols - c0);
  float* D = job.D + (int64_t)a * r * job.cols;
  for (int i = split * kGradWarps * 32 + tid; i < cols * r; i += p.splits * kGradWarps * 32) {
    const int j = job.j_first ? i % r : i / cols, c = job.j_first ? i / r : i % cols;
    float x = 0.0f;
    if (p.splits > 1) {
      for (int s = 0; s < p.splits; s++) x += cluster_load(smem_addr(&out[j * 129 + c]), s);
    } else {
      x = out[j * 129 + c];
    }
    D[job.j_first ? (int64_t)(c0 + c) * r + j : (int64_t)j * job.cols + c0 + c] = x;
  }
  __syncwarp();
  if (p.splits > 1) cluster_sync();
}

template <int NB, bool BF>
windq_status launch_gradients(windq_ctx* ctx, int id, GradArgs p, cudaStream_t st) {
  const int tiles = p.job[0].tiles + p.job[1].tiles, blocks = (p.T + kGradTokens - 1) / kGradTokens;
  // most adapters have a share of the tokens, so the work of one column tile is about that of one adapter with all of them
  p.splits = 1;
  while (p.splits < 8 && tiles * p.splits * 2 <= 4 * ctx->sm_count && blocks >= p.splits * 2 * 4) p.splits *= 2;
  const int loop = kGradStages * kGradTokens * kZPitch + (BF ? 3 : 2) * kGradTokens * (p.rank * 2 + 16);
  const int smem = std::max(loop, p.rank * 129 * 4);
  constexpr int kMost = 112 * 1024;
  const windq_status ready = prepare_kernel(ctx, id, gradient_kernel<NB, BF>, kGradWarps * 32, kMost, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)p.n_adapters);
  cfg.blockDim = dim3(kGradWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = p.splits;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = p.splits > 1 ? 1 : 0;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, gradient_kernel<NB, BF>, p));
  return WINDQ_OK;
}

}  // namespace

windq_status launch_low_rank(windq_ctx* ctx, const LowRank& q, cudaStream_t st) {
  LowRankArgs p = {};
  p.Z = (const uint16_t*)q.Z;
  p.ldz = q.ldz;
  p.P = (const uint16_t*)q.P;
  p.T = (int)q.T;
  p.K = (int)q.K;
  p.rank = q.rank;
  p.n_adapters = (int)q.n_adapters;
  p.bf = q.dtype == WINDQ_BF16;
  p.scaling = q.scaling;
  p.adapter_of = q.adapter_of;
  p.S = q.S;
  p.top = q.top;
  p.lists = q.lists;
  p.list_rows = token_tile(q.T);
  p.list_tiles = (int)((q.T + p.list_rows - 1) / p.list_rows);
  const bool few = q.T <= 256;
#define WINDQ_LOW(index, mt, nb)                                                                     \
  return q.transposed ? launch_low_rank<mt, nb, true>(ctx, kLowRank + 9 + (index), p, st)            \
                      : launch_low_rank<mt, nb, false>(ctx, kLowRank + (index), p, st)
  if (q.rank > 64) WINDQ_LOW(0, 1, 16);
  if (few) {
    if (q.rank <= 8) WINDQ_LOW(1, 1, 1);
    if (q.rank <= 16) WINDQ_LOW(2, 1, 2);
    if (q.rank <= 32) WINDQ_LOW(3, 1, 4);
    WINDQ_LOW(4, 1, 8);
  }
  if (q.rank <= 8) WINDQ_LOW(5, 4, 1);
  if (q.rank <= 16) WINDQ_LOW(6, 4, 2);
  if (q.rank <= 32) WINDQ_LOW(7, 4, 4);
  WINDQ_LOW(8, 2, 8);
#undef WINDQ_LOW
}

windq_status launch_gradients(windq_ctx* ctx, const Gradient* dA, const Gradient* dB, int dtype, int64_t T, int rank,
                              int64_t n_adapters, const int32_t* adapter_of, cudaStream_t st) {
  GradArgs p = {};
  int k = 0;
  for (const Gradient* q : {dA, dB}) {
    if (!q) continue;
    GradJob& j = p.job[k++];
    j.Z = (const uint16_t*)q->Z;
    j.ldz = q->ldz;
    j.S = q->S;
    j.top = q->top;
    j.D = q->D;
    j.cols = (int)q->cols;
    j.tiles = (int)((q->cols + kGradCols - 1) / kGradCols);
    j.j_first = q == dB;
  }
  p.T = (int)T;
  p.rank = rank;
  p.n_adapters = (int)n_adapters;
  p.adapter_of = adapter_of;
#define WINDQ_GRAD(index, nb)                                                                     \
  return dtype == WINDQ_BF16 ? launch_gradients<nb, true>(ctx, kGradient + 5 + (index), p, st)    \
                             : launch_gradients<nb, false>(ctx, kGradient + (index), p, st)
  if (rank <= 8) WINDQ_GRAD(0, 1);
  if (rank <= 16) WINDQ_GRAD(1, 2);
  if (rank <= 32) WINDQ_GRAD(2, 4);
  if (rank <= 64) WINDQ_GRAD(3, 8);
  WINDQ_GRAD(4, 16);
#undef WINDQ_GRAD
}

}  // namespace windq
