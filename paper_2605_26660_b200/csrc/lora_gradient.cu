// The gradients of A and B of the adapter calls.
//
// They read X and dY once and have a result of rank values per channel; they are bound by that read (HBM or L2) and use
// warp-level matrix products (mma.sync m16n8k16): the reduction runs over the tokens of one adapter, which may be any
// subset, and there is nothing to gain from the rate of tcgen05.
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

// D[a][j][c] = sum over the tokens t of a of S[t][j] Z[t][c]

constexpr int kGradWarps = 8, kGradThreads = 256, kGradCols = 256;
constexpr int kZPitch = kGradCols * 2 + 16;  // bytes
constexpr int kGradTokens = 32;              // of a block
constexpr int kWindow = 128;                 // blocks of tokens whose adapters are looked up at a time

// Values j of S that a thread block takes: all of rank 32, and blocks of 32 of a larger one (Z is then read again, from L2).
constexpr int kGradRank = 32;
constexpr int kGradStages = 4, kGradBlocks = 2;  // stages of copies in flight; thread blocks an SM
// The products cut a sum off where they add to it: over 1024 tokens 1.2e-6 of a gradient with S in one term, and more with
// the small second and third terms, where a plain binary32 product is 1e-6 off.  So the sums of four blocks of tokens (128)
// are added, rounded, to a second set of registers, which is also why the rank is taken in blocks.
constexpr int kFlush = 4;

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

// A thread block owns 256 columns of Z for one adapter, a warp 32 of them; a cluster of `splits` shares the tokens.  What
// bounds it once the loads flow is shared memory: every warp reads all of S, so few warps with many columns each are better
// than many with few (with 128 columns a block and 16 a warp the backward pass of 8192 x 4096 x 4096 took 308 us, with these
// 298; both with 23 us of products of S before and 205 of dX after).
//
// The tokens that are not the adapter's are left out as rows of zeros (copied with size zero, so that what they hold cannot
// spoil a sum), blocks of tokens without any of its tokens are skipped.  Z is the transposed left operand (ldmatrix.trans);
// S enters as two fp16 or three bf16 values whose sum is S to 22 or 24 bits -- fp16 ones after a scaling by a power of two
// that puts the largest |S| of the adapter's tokens so far near 2^13, so that small gradients keep their bits (the sums are
// rescaled, exactly, where a later window of tokens holds a larger one).
template <int NB, bool BF>
__global__ void __launch_bounds__(kGradThreads, kGradBlocks) gradient_kernel(const __grid_constant__ GradArgs p) {
  constexpr int kTerms = BF ? 3 : 2, kTokens = kGradTokens, kStages = kGradStages;
  constexpr int kPieces = (kTokens * NB + kGradThreads - 1) / kGradThreads;              // of eight values of S, a thread
  extern __shared__ uint4 shared[];
  __shared__ unsigned masks[kWindow];  // tokens of the adapter
  __shared__ short active[kWindow];
  __shared__ int n_active;
  __shared__ float tops[kGradWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
  const int split = blockIdx.x % p.splits, a = blockIdx.y, j0 = blockIdx.z * kGradRank, r = min(p.rank - j0, kGradRank);
  int tile = blockIdx.x / p.splits;
  const bool second = tile >= p.job[0].tiles;
  const GradJob& job = p.job[second];
  if (second) tile -= p.job[0].tiles;
  const int c0 = tile * kGradCols;
  const int all = (p.T + kTokens - 1) / kTokens;
  launch_dependents();
  wait_for_predecessor();

  float top = 0.0f, up = 1.0f, down = 1.0f;  // largest |S| so far; scaling of S and its inverse

  // a stage: Z [token][column], then S [token][j] in binary32; after the stages two buffers of S in 16-bit terms
  const int s_pitch = r * 2 + 16, s_raw = kTokens * r * 4, s_terms = kTerms * kTokens * s_pitch;
  const int stage_bytes = kTokens * kZPitch + s_raw;
  const uint32_t base = smem_addr(shared), terms = base + kStages * stage_bytes;
  float acc[2][NB][4];
#pragma unroll
  for (int h = 0; h < 2; h++)
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int k = 0; k < 4; k++) acc[h][n][k] = 0.0f;
  float kept[2][NB][4] = {};
  auto flush = [&] {
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int n = 0; n < NB; n++)
#pragma unroll
        for (int k = 0; k < 4; k++) {
          kept[h][n][k] += acc[h][n][k];
          acc[h][n][k] = 0.0f;
        }
  };

  for (int w0 = 0; w0 < all; w0 += kWindow) {
    const int count = min(kWindow, all - w0);
    __syncthreads();
    float most = 0.0f;
#pragma unroll 8
    for (int i = warp; i < count; i += kGradWarps) {
      const int t = w0 * kTokens + i * 32 + lane;
      const int id = t < p.T ? p.adapter_of[t] : -1;
      const float x = !BF && t < p.T ? job.top[t] : 0.0f;
      const unsigned vote = __ballot_sync(0xffffffffu, id == a);
      if (lane == 0) masks[i] = vote;
      if (!BF && id == a) most = fmaxf(most, x);
    }
    if (!BF) {
      most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));  // values >= 0 order like their bits
      if (lane == 0) tops[warp] = most;
    }
    __syncthreads();
    if (!BF) {
      for (int w = 0; w < kGradWarps; w++) most = fmaxf(most, tops[w]);
      if (most > top) {
        top = most;
        // 2^e <= top < 2^(e + 1); both factors are kept normal
        const int e = (int)((__float_as_uint(top) >> 23) & 255) - 127, k = max(-100, min(100, 13 - e));
        const float next = __uint_as_float((uint32_t)(127 + k) << 23), change = next * down;
        up = next;
        down = __uint_as_float((uint32_t)(127 - k) << 23);
        if (w0 > 0) {
          flush();
#pragma unroll
          for (int h = 0; h < 2; h++)
#pragma unroll
            for (int n = 0; n < NB; n++)
#pragma unroll
              for (int q = 0; q < 4; q++) kept[h][n][q] *= change;
        }
      }
    }
    if (warp == 0) {
      int n = 0;
      for (int h = 0; h < count; h += 32) {
        const bool on = h + lane < count && masks[h + lane];
        const unsigned vote = __ballot_sync(0xffffffffu, on);
        if (on) active[n + __popc(vote & ((1u << lane) - 1))] = (short)(h + lane);
        n += __popc(vote);
      }
      if (lane == 0) n_active = n;
    }
    __syncthreads();
    const int n_blocks = (n_active - split + p.splits - 1) / p.splits;  // every splits-th of them is this block's
    auto copy_block = [&](int i) {
      if (i < n_blocks) {
        const int b = active[split + i * p.splits], t0 = (w0 + b) * kTokens;
        const uint32_t at = base + (i % kStages) * stage_bytes;
#pragma unroll
        for (int h = 0; h < kTokens * 32 / kGradThreads; h++) {
          const int x = h * kGradThreads + tid, row = x >> 5, piece = x & 31, c = c0 + piece * 8;
          const bool on = c < job.cols && (masks[b] >> row & 1);
          copy16(at + row * kZPitch + piece * 16, on ? job.Z + (t0 + row) * job.ldz + c : job.Z, on ? min(16, (job.cols - c) * 2) : 0);
        }
#pragma unroll
        for (int h = 0; h < kPieces; h++) {
          const int x = h * kGradThreads + tid, row = x / NB, piece = x % NB;
          if (row >= kTokens || piece * 8 >= r) continue;
          const bool on = masks[b] >> row & 1;
          const float* src = on ? job.S + (int64_t)(t0 + row) * p.rank + j0 + piece * 8 : job.S;
          const uint32_t dst = at + kTokens * kZPitch + (row * r + piece * 8) * 4;
          copy16(dst, src, on ? 16 : 0);
          copy16(dst + 16, src + 4, on ? 16 : 0);
        }
      }
      copy_commit();
    };
    // The thread that copied a piece of S also splits it into terms.
    auto split_s = [&](int i) {
      const uint32_t at = base + (i % kStages) * stage_bytes + kTokens * kZPitch, to = terms + (i & 1) * s_terms;
#pragma unroll
      for (int h = 0; h < kPieces; h++) {
        const int x = h * kGradThreads + tid, row = x / NB, piece = x % NB;
        if (row >= kTokens || piece * 8 >= r) continue;
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; k += 4)
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(y[k]), "=f"(y[k + 1]), "=f"(y[k + 2]), "=f"(y[k + 3])
                       : "r"(at + (row * r + piece * 8 + k) * 4)
                       : "memory");
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
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (term * kTokens + row) * s_pitch + piece * 16), "r"(w[0]),
                       "r"(w[1]), "r"(w[2]), "r"(w[3])
                       : "memory");
        }
      }
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; i++) copy_block(i);
    for (int i = 0; i < n_blocks; i++) {
      if (i % kFlush == 0 && i) flush();
      copy_wait<kStages - 2>();
      split_s(i);
      __syncthreads();
      copy_block(i + kStages - 1);  // into the stage that every warp left before the barrier
      const uint32_t z_at = base + (i % kStages) * stage_bytes, s_at0 = terms + (i & 1) * s_terms;
#pragma unroll
      for (int k = 0; k < kTokens / 16; k++) {
        // left operand: columns 32 warp + 16 h .. + 15 (rows of the product), tokens 16 k .. + 15
        uint32_t za[2][4];
#pragma unroll
        for (int h = 0; h < 2; h++)
          ldmatrix_trans(z_at + (k * 16 + (lane & 7) + (lane >> 4) * 8) * kZPitch + (warp * 32 + h * 16 + ((lane >> 3) & 1) * 8) * 2, za[h]);
#pragma unroll
        for (int term = 0; term < kTerms; term++) {
          const uint32_t s_at = s_at0 + (term * kTokens + k * 16 + (lane & 15)) * s_pitch + (lane >> 4) * 16;
#pragma unroll
          for (int n = 0; n < NB; n += 2) {
            if (n * 8 < r) {
              uint32_t sb[4];
              // an odd last block has no right neighbour: its lanes read the left one again
              ldmatrix_trans((n + 1) * 8 < r ? s_at + n * 16 : s_at + n * 16 - (lane >> 4) * 16, sb);
#pragma unroll
              for (int h = 0; h < 2; h++) {
                mma16816(acc[h][n], za[h], sb[0], sb[1], BF);
                if (n + 1 < NB && (n + 1) * 8 < r) mma16816(acc[h][n + 1 < NB ? n + 1 : n], za[h], sb[2], sb[3], BF);
              }
            }
          }
        }
      }
    }
    copy_wait<0>();
  }
  __syncthreads();
  flush();
  // join the cluster: [column][j] for dB, [j][column] for dA, as the result lies
  const int pitch = job.j_first ? r + 4 : kGradCols + 4;
#pragma unroll
  for (int h = 0; h < 2; h++)
#pragma unroll
    for (int n = 0; n < NB; n++)
      if (n * 8 < r) {
#pragma unroll
        for (int k = 0; k < 4; k++) {
          const int j = n * 8 + q * 2 + (k & 1), c = warp * 32 + h * 16 + g + (k >> 1) * 8;
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(base + (job.j_first ? c * pitch + j : j * pitch + c) * 4),
                       "f"(kept[h][n][k] * down)
                       : "memory");
        }
      }
  __syncwarp();
  if (p.splits > 1) cluster_sync();
  else __syncthreads();
  const int cols = min(kGradCols, job.cols - c0);
  const int quads = (job.j_first ? r : cols) / 4, items = (job.j_first ? cols : r) * quads;  // four values each
  float* D = job.D + (int64_t)a * p.rank * job.cols + (job.j_first ? j0 : (int64_t)j0 * job.cols);
  constexpr int U = 4;
  for (int i = split * kGradThreads + tid; i < items; i += U * p.splits * kGradThreads) {
    uint32_t offset[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int e = min(i + u * p.splits * kGradThreads, items - 1);
      offset[u] = (uint32_t)(e / quads * pitch + e % quads * 4) * 4;
    }
    cluster_sum<U>(base, offset, p.splits, 0, 1, x);
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int e = i + u * p.splits * kGradThreads;
      if (e >= items) continue;
      const int row = e / quads, col = e % quads * 4;
      *reinterpret_cast<float4*>(D + (job.j_first ? (int64_t)(c0 + row) * p.rank + col : (int64_t)row * job.cols + c0 + col)) = x[u];
    }
  }
  __syncwarp();
  if (p.splits > 1) cluster_sync();
}

template <int NB, bool BF>
windq_status launch_gradients(windq_ctx* ctx, int id, GradArgs p, cudaStream_t st) {
  const int tiles = p.job[0].tiles + p.job[1].tiles, blocks = (p.T + kGradTokens - 1) / kGradTokens;
  // every token has one adapter, so the work of a column tile over all adapters is about one pass over the tokens; as many
  // thread blocks as fit, counting on two adapters with tokens where there are so many
  const int ranks = (p.rank + kGradRank - 1) / kGradRank, r = std::min(p.rank, kGradRank);
  p.splits = 1;
  while (p.splits < 8 && (int64_t)tiles * ranks * std::min(p.n_adapters, 2) * p.splits * 2 <= kGradBlocks * ctx->sm_count &&
         blocks >= p.splits * 2 * 4)
    p.splits *= 2;
  const int loop = kGradStages * kGradTokens * (kZPitch + r * 4) + 2 * (BF ? 3 : 2) * kGradTokens * (r * 2 + 16);
  const int smem = std::max(loop, std::max(kGradCols * (r + 4), r * (kGradCols + 4)) * 4);
  constexpr int kMost = 224 * 1024 / kGradBlocks - 2048;
  static_assert(kGradStages * kGradTokens * (kZPitch + NB * 32) + 6 * kGradTokens * (NB * 16 + 16) <= kMost &&
                    (kGradCols + 4) * (NB * 8 + 4) * 4 <= kMost, "kGradBlocks an SM");
  const windq_status ready = prepare_kernel(ctx, id, gradient_kernel<NB, BF>, kGradThreads, kMost, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)p.n_adapters, (unsigned)ranks);
  cfg.blockDim = dim3(kGradThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = p.splits;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, gradient_kernel<NB, BF>, p));
  return WINDQ_OK;
}

}  // namespace

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
  return dtype == WINDQ_BF16 ? launch_gradients<nb, true>(ctx, kGradient + 3 + (index), p, st)    \
                             : launch_gradients<nb, false>(ctx, kGradient + (index), p, st)
  if (rank <= 8) WINDQ_GRAD(0, 1);
  if (rank <= 16) WINDQ_GRAD(1, 2);
  WINDQ_GRAD(2, 4);
#undef WINDQ_GRAD
}

}  // namespace windq
