// The gradients of A and B of the adapter calls.
//
// They read X and dY once and have a result of rank values per channel; they are bound by that read (HBM or L2) and use
// warp-level matrix products (mma.sync m16n8k16): the reduction runs over the tokens of one adapter, which may be any
// subset, and there is nothing to gain from the rate of tcgen05.
#include <algorithm>

#include "lora.cuh"
#include "tcgen05.cuh"
#include "warp_mma.cuh"

namespace windq {
namespace {

// ---- D[a][j][c] = sum over the tokens t of a of S[t][j] Z[t][c] ----------------------------------------------------

constexpr int kGradWarps = 8, kGradCols = 128, kGradTokens = 64, kGradStages = 3;
constexpr int kZPitch = kGradCols * 2 + 16;  // bytes
constexpr int kWindow = 64;                  // blocks of tokens whose adapters are looked up at a time

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
  __shared__ int ids[kWindow * kGradTokens];
  __shared__ short active[kWindow], flags[kWindow];
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
  launch_dependents();
  wait_for_predecessor();

  float up = 1.0f, down = 1.0f;
  if (!BF) {
    float top = 0.0f;
    for (int t = tid; t < p.T; t += kGradWarps * 32) {
      const float x = job.top[t];
      if (p.adapter_of[t] == a) top = fmaxf(top, x);
    }
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

  for (int w0 = 0; w0 < all; w0 += kWindow) {
    const int count = min(kWindow, all - w0);
    __syncthreads();
    for (int b = warp; b < count; b += kGradWarps) {
      const int i = b * kGradTokens + lane, t = w0 * kGradTokens + i;
      const int x = t < p.T ? p.adapter_of[t] : -1, y = t + 32 < p.T ? p.adapter_of[t + 32] : -1;
      ids[i] = x;
      ids[i + 32] = y;
      const unsigned vote = __ballot_sync(0xffffffffu, x == a || y == a);
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
    const int n_blocks = (n_active - split + p.splits - 1) / p.splits;  // every splits-th of them is this block's
    auto block_at = [&](int i) { return (int)active[split + i * p.splits]; };
    auto copy_z = [&](int i) {
      if (i < n_blocks) {
        const int b = block_at(i), t0 = (w0 + b) * kGradTokens;
        const uint32_t at = z_base + (i % kGradStages) * kGradTokens * kZPitch;
#pragma unroll
        for (int h = 0; h < 4; h++) {
          const int x = h * kGradWarps * 32 + tid, row = x >> 4, piece = x & 15, t = t0 + row, c = c0 + piece * 8;
          const bool on = c < job.cols && ids[b * kGradTokens + row] == a;
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
      const int b = block_at(i), t0 = (w0 + b) * kGradTokens;
#pragma unroll
      for (int h = 0; h < kPieces; h++) {
        const int x = h * kGradWarps * 32 + tid, row = x / NB, piece = x % NB, t = t0 + row;
        s_next[h][0] = s_next[h][1] = make_float4(0, 0, 0, 0);
        if (row < kGradTokens && piece * 8 < r && ids[b * kGradTokens + row] == a) {
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
  // every token has one adapter, so the work of a column tile over all adapters is about one pass over the tokens
  p.splits = 1;
  while (p.splits < 8 && tiles * p.splits * 2 <= 3 * ctx->sm_count && blocks >= p.splits * 2 * 4) p.splits *= 2;
  const int loop = kGradStages * kGradTokens * kZPitch + (BF ? 3 : 2) * kGradTokens * (p.rank * 2 + 16);
  const int smem = std::max(loop, p.rank * 129 * 4);
  constexpr int kMost = 108 * 1024;
  const windq_status ready = prepare_kernel(ctx, id, gradient_kernel<NB, BF>, kGradWarps * 32, kMost, false);
  if (ready != WINDQ_OK) return ready;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)p.n_adapters);
  cfg.blockDim = dim3(kGradWarps * 32);
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
