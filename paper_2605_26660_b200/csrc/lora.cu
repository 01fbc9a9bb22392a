// The shared projection with one low-rank adapter per token, and its gradients.
#include "lora.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

__device__ __forceinline__ float value(const void* base, int64_t i, int dt) { return load1(base, i, dt); }

// S[t][j] = scaling[a] * sum_k Z[t][k] * P[a](k, j), P[a](k, j) = P[a * pa + k * pk + j * pj]; zeros without an adapter.
// The blocks past the tokens write the lists of adapters of the token tiles.
__global__ void low_rank_kernel(const void* Z, int64_t ldz, int64_t T, int64_t K, const void* P, int64_t pa, int64_t pk, int64_t pj,
                                int dt, int64_t n_adapters, int rank, const float* scaling, const int32_t* adapter_of, float* S,
                                int* lists, int rows) {
  launch_dependents();
  const int64_t t = blockIdx.x;
  if (t >= T) {
    // adapters in the order of their first token; a thread per token (blockDim.x >= rows)
    __shared__ int ids[256], taken[8];
    const int tile = (int)(t - T), i = threadIdx.x;
    const int64_t at = (int64_t)tile * rows + i;
    int id = i < rows && at < T ? adapter_of[at] : -1;
    if (id >= n_adapters) id = -1;
    ids[i] = id;
    __syncthreads();
    bool first = id >= 0;
    for (int k = 0; k < i && first; k++) first = ids[k] != id;
    const unsigned vote = __ballot_sync(0xffffffffu, first);
    if ((i & 31) == 0) taken[i >> 5] = __popc(vote);
    __syncthreads();
    int before = __popc(vote & ((1u << (i & 31)) - 1)), all = 0;
    for (int w = 0; w < 8; w++) {
      if (w < i >> 5) before += taken[w];
      all += taken[w];
    }
    int* list = lists + (int64_t)tile * (rows + 1);
    if (first) list[1 + before] = id;
    if (i == 0) list[0] = all;
    return;
  }
  const int a = adapter_of[t];
  for (int j = threadIdx.x >> 5; j < rank; j += blockDim.x >> 5) {
    float acc = 0.0f;
    if (a >= 0 && a < n_adapters) {
      for (int64_t k = threadIdx.x & 31; k < K; k += 32)
        acc = fmaf(value(Z, t * ldz + k, dt), value(P, a * pa + k * pk + j * pj, dt), acc);
      for (int d = 16; d; d >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, d);
      acc *= scaling[a];
    }
    if ((threadIdx.x & 31) == 0) S[t * rank + j] = acc;
  }
}

// D[a][..] = sum over the tokens of a of S[t][j] * Z[t][c]; j contiguous (dB) or c contiguous (dA).
__global__ void gradient_kernel(const void* Z, int64_t ldz, int64_t T, int64_t K, const float* S, int rank, int dt,
                                const int32_t* adapter_of, float* D, int64_t dj, int64_t dc) {
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  const int j = blockIdx.y * 8 + threadIdx.y, a = blockIdx.z;
  if (c >= K) return;
  float acc = 0.0f;
  for (int64_t t = 0; t < T; t++)
    if (adapter_of[t] == a) acc = fmaf(S[t * rank + j], value(Z, t * ldz + c, dt), acc);
  D[a * (int64_t)rank * K + j * dj + c * dc] = acc;
}

struct LoraArgs {
  const char* who;
  int dtype;
  const void* X;
  int64_t T, C, ldx;
  const void* W;
  int64_t R, ldw;
  const void *A, *B;
  int64_t n_adapters;
  int rank;
  const float* scaling;
  const int32_t* adapter_of;
};

windq_status check_lora(windq_ctx* ctx, const LoraArgs& q) {
  const char* who = q.who;
  WINDQ_REQUIRE(ctx, q.dtype == WINDQ_F16 || q.dtype == WINDQ_BF16, WINDQ_ERR_ARG, "%s: dtype = %d is neither fp16 nor bf16", who,
                q.dtype);
  WINDQ_REQUIRE(ctx, q.W && q.A && q.B && q.scaling, WINDQ_ERR_NULL, "%s: W, A, B or scaling is NULL", who);
  WINDQ_REQUIRE(ctx, q.T >= 0 && q.T < (1ll << 31) - 256, WINDQ_ERR_SHAPE, "%s: T = %lld", who, (long long)q.T);
  WINDQ_REQUIRE(ctx, q.T == 0 || (q.X && q.adapter_of), WINDQ_ERR_NULL, "%s: X or adapter_of is NULL", who);
  WINDQ_REQUIRE(ctx, q.R > 0 && q.C > 0 && q.R < (1ll << 31) - 256 && q.C < (1ll << 31) - 256, WINDQ_ERR_SHAPE,
                "%s: R = %lld, C = %lld", who, (long long)q.R, (long long)q.C);
  WINDQ_REQUIRE(ctx, q.C % 8 == 0, WINDQ_ERR_SHAPE, "%s: C = %lld is not a multiple of 8", who, (long long)q.C);
  WINDQ_REQUIRE(ctx, q.n_adapters >= 1 && q.n_adapters <= 65535, WINDQ_ERR_SHAPE, "%s: n_adapters = %lld is outside [1, 65535]",
                who, (long long)q.n_adapters);
  WINDQ_REQUIRE(ctx, q.rank >= 8 && q.rank <= 128 && q.rank % 8 == 0, WINDQ_ERR_ARG,
                "%s: rank = %d is not a multiple of 8 in [8, 128]", who, q.rank);
  WINDQ_REQUIRE(ctx, q.ldx >= q.C && q.ldw >= q.C, WINDQ_ERR_SHAPE, "%s: ldx = %lld or ldw = %lld is below C = %lld", who,
                (long long)q.ldx, (long long)q.ldw, (long long)q.C);
  WINDQ_REQUIRE(ctx, q.ldx % 8 == 0 && q.ldw % 8 == 0, WINDQ_ERR_ALIGN, "%s: ldx = %lld or ldw = %lld is not a multiple of 8", who,
                (long long)q.ldx, (long long)q.ldw);
  WINDQ_REQUIRE(ctx, aligned16(q.X) && aligned16(q.W) && aligned16(q.A) && aligned16(q.B) && aligned16(q.scaling) &&
                         aligned16(q.adapter_of),
                WINDQ_ERR_ALIGN, "%s: X, W, A, B, scaling or adapter_of is not 16-byte aligned", who);
  return WINDQ_OK;
}

}  // namespace
}  // namespace windq

extern "C" {

int64_t windq_scratch_bytes_lora_forward(int64_t T, int64_t R, int64_t C, int rank) {
  if (T < 0 || R <= 0 || C <= 0 || rank <= 0) return 0;
  return windq::round_up(4 * T * rank, 256) + windq::list_bytes(T);
}

windq_status windq_lora_forward(windq_ctx* ctx, int dtype, const void* X, int64_t T, int64_t C, int64_t ldx, const void* W,
                                int64_t R, int64_t ldw, const void* A, const void* B, int64_t n_adapters, int rank,
                                const float* scaling, const int32_t* adapter_of, void* Y, int64_t ldy, void* stream) {
  using namespace windq;
  const char* who = "windq_lora_forward";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  const windq_status bad = check_lora(ctx, LoraArgs{who, dtype, X, T, C, ldx, W, R, ldw, A, B, n_adapters, rank, scaling, adapter_of});
  if (bad != WINDQ_OK) return bad;
  WINDQ_REQUIRE(ctx, T == 0 || Y, WINDQ_ERR_NULL, "%s: Y is NULL", who);
  WINDQ_REQUIRE(ctx, ldy >= R, WINDQ_ERR_SHAPE, "%s: ldy = %lld is below R = %lld", who, (long long)ldy, (long long)R);
  WINDQ_REQUIRE(ctx, ldy % 8 == 0 && aligned16(Y), WINDQ_ERR_ALIGN, "%s: Y is not 16-byte aligned or ldy no multiple of 8", who);
  if (T == 0) return WINDQ_OK;
  DeviceGuard guard(ctx->device);
  const windq_status room = ensure_scratch(ctx, windq_scratch_bytes_lora_forward(T, R, C, rank));
  if (room != WINDQ_OK) return room;
  cudaStream_t st = (cudaStream_t)stream;
  float* U = (float*)ctx->scratch;
  int* lists = (int*)((char*)ctx->scratch + round_up(4 * T * rank, 256));
  const int rows = token_tile(T), tiles = (int)((T + rows - 1) / rows);
  low_rank_kernel<<<(unsigned)(T + tiles), 256, 0, st>>>(X, ldx, T, C, A, rank * C, 1, C, dtype, n_adapters, rank, scaling, adapter_of,
                                                         U, lists, rows);
  WINDQ_CUDA(ctx, cudaGetLastError());
  return launch_projection(ctx, Projection{dtype, false, X, T, C, R, ldx, W, ldw, B, n_adapters, rank, adapter_of, U, lists, Y, ldy}, st);
}

int64_t windq_scratch_bytes_lora_backward(int64_t T, int64_t R, int64_t C, int64_t n_adapters, int rank) {
  if (T < 0 || R <= 0 || C <= 0 || rank <= 0 || n_adapters <= 0) return 0;
  return 2 * windq::round_up(4 * T * rank, 256) + windq::list_bytes(T);
}

windq_status windq_lora_backward(windq_ctx* ctx, int dtype, const void* X, int64_t T, int64_t C, int64_t ldx, const void* W,
                                 int64_t R, int64_t ldw, const void* A, const void* B, int64_t n_adapters, int rank,
                                 const float* scaling, const int32_t* adapter_of, const void* dY, int64_t lddy, void* dX,
                                 int64_t lddx, float* dA, float* dB, void* stream) {
  using namespace windq;
  const char* who = "windq_lora_backward";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  const windq_status bad = check_lora(ctx, LoraArgs{who, dtype, X, T, C, ldx, W, R, ldw, A, B, n_adapters, rank, scaling, adapter_of});
  if (bad != WINDQ_OK) return bad;
  WINDQ_REQUIRE(ctx, T == 0 || dY, WINDQ_ERR_NULL, "%s: dY is NULL", who);
  WINDQ_REQUIRE(ctx, lddy >= R, WINDQ_ERR_SHAPE, "%s: lddy = %lld is below R = %lld", who, (long long)lddy, (long long)R);
  WINDQ_REQUIRE(ctx, lddy % 8 == 0 && aligned16(dY), WINDQ_ERR_ALIGN, "%s: dY is not 16-byte aligned or lddy no multiple of 8", who);
  WINDQ_REQUIRE(ctx, dX || dA || dB, WINDQ_ERR_NULL, "%s: dX, dA and dB are all NULL", who);
  WINDQ_REQUIRE(ctx, !dX || lddx >= C, WINDQ_ERR_SHAPE, "%s: lddx = %lld is below C = %lld", who, (long long)lddx, (long long)C);
  WINDQ_REQUIRE(ctx, !dX || lddx % 8 == 0, WINDQ_ERR_ALIGN, "%s: lddx = %lld is not a multiple of 8", who, (long long)lddx);
  WINDQ_REQUIRE(ctx, aligned16(dX) && aligned16(dA) && aligned16(dB), WINDQ_ERR_ALIGN, "%s: dX, dA or dB is not 16-byte aligned", who);
  DeviceGuard guard(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  if (T == 0) {
    if (dA) WINDQ_CUDA(ctx, cudaMemsetAsync(dA, 0, (size_t)(4 * n_adapters * rank * C), st));
    if (dB) WINDQ_CUDA(ctx, cudaMemsetAsync(dB, 0, (size_t)(4 * n_adapters * rank * R), st));
    return WINDQ_OK;
  }
  const windq_status room = ensure_scratch(ctx, windq_scratch_bytes_lora_backward(T, R, C, n_adapters, rank));
  if (room != WINDQ_OK) return room;
  float* U = (float*)ctx->scratch;
  float* V = (float*)((char*)ctx->scratch + round_up(4 * T * rank, 256));
  int* lists = (int*)((char*)V + round_up(4 * T * rank, 256));
  const int rows = token_tile(T), tiles = (int)((T + rows - 1) / rows);
  if (dB)
    low_rank_kernel<<<(unsigned)T, 256, 0, st>>>(X, ldx, T, C, A, rank * C, 1, C, dtype, n_adapters, rank, scaling, adapter_of, U,
                                                 nullptr, rows);
  if (dX || dA)
    low_rank_kernel<<<(unsigned)(T + tiles), 256, 0, st>>>(dY, lddy, T, R, B, R * rank, rank, 1, dtype, n_adapters, rank, scaling,
                                                           adapter_of, V, lists, rows);
  WINDQ_CUDA(ctx, cudaGetLastError());
  if (dX) {
    const windq_status done = launch_projection(
        ctx, Projection{dtype, true, dY, T, R, C, lddy, W, ldw, A, n_adapters, rank, adapter_of, V, lists, dX, lddx}, st);
    if (done != WINDQ_OK) return done;
  }
  if (dA)
    gradient_kernel<<<dim3((unsigned)((C + 31) / 32), rank / 8, (unsigned)n_adapters), dim3(32, 8), 0, st>>>(
        X, ldx, T, C, V, rank, dtype, adapter_of, dA, C, 1);
  if (dB)
    gradient_kernel<<<dim3((unsigned)((R + 31) / 32), rank / 8, (unsigned)n_adapters), dim3(32, 8), 0, st>>>(
        dY, lddy, T, R, U, rank, dtype, adapter_of, dB, 1, rank);
  WINDQ_CUDA(ctx, cudaGetLastError());
  return WINDQ_OK;
}

}  // extern "C"
