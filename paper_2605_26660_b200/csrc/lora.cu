// The shared projection with one low-rank adapter per token, and its gradients: checks and the order of the kernels.
#include "lora.cuh"

namespace windq {
namespace {

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
  WINDQ_REQUIRE(ctx, !*ctx->gave_up, WINDQ_ERR_CUDA, "%s: a wait of an earlier call gave up, its results are invalid (windq_stalls)", who);
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
  WINDQ_REQUIRE(ctx, aligned16(q.X) && aligned16(q.W) && aligned16(q.A) && aligned16(q.B), WINDQ_ERR_ALIGN,
                "%s: X, W, A or B is not 16-byte aligned", who);
  WINDQ_REQUIRE(ctx, (((uintptr_t)q.scaling | (uintptr_t)q.adapter_of) & 3) == 0, WINDQ_ERR_ALIGN,
                "%s: scaling or adapter_of is misaligned", who);
  return WINDQ_OK;
}

}  // namespace
}  // namespace windq

extern "C" {

int64_t windq_scratch_bytes_lora_forward(int64_t T, int64_t R, int64_t C, int rank) {
  if (T < 0 || R <= 0 || C <= 0 || rank <= 0) return 0;
  return windq::round_up(4 * T * rank, 256) + windq::round_up(T, 256) + windq::list_bytes(T);
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
  void* U = ctx->scratch;
  int8_t* shift = (int8_t*)ctx->scratch + round_up(4 * T * rank, 256);
  int* lists = (int*)(shift + round_up(T, 256));
  if (dtype == WINDQ_BF16) shift = nullptr;
  const windq_status low = launch_low_rank(
      ctx, LowRank{dtype, T, n_adapters, rank, scaling, adapter_of, lists, 1, {{false, X, C, ldx, A, nullptr, U, shift, nullptr}}}, st);
  if (low != WINDQ_OK) return low;
  return launch_projection(
      ctx, Projection{dtype, false, X, T, C, R, ldx, W, ldw, B, n_adapters, rank, adapter_of, U, shift, lists, Y, ldy}, st);
}

int64_t windq_scratch_bytes_lora_backward(int64_t T, int64_t R, int64_t C, int64_t n_adapters, int rank) {
  if (T < 0 || R <= 0 || C <= 0 || rank <= 0 || n_adapters <= 0) return 0;
  return 3 * windq::round_up(4 * T * rank, 256) + 2 * windq::round_up(4 * T, 256) + windq::round_up(T, 256) + windq::list_bytes(T);
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
  char* at = (char*)ctx->scratch;
  auto take = [&](int64_t bytes) {
    char* p = at;
    at += round_up(bytes, 256);
    return p;
  };
  float* U = (float*)take(4 * T * rank);
  float* V = (float*)take(4 * T * rank);
  void* V_pair = take(4 * T * rank);
  float* top_u = (float*)take(4 * T);
  float* top_v = (float*)take(4 * T);
  int8_t* shift = (int8_t*)take(T);
  int* lists = (int*)at;
  if (dtype == WINDQ_BF16) shift = nullptr;
  LowRank low = {dtype, T, n_adapters, rank, scaling, adapter_of, dX ? lists : nullptr, 0, {}};
  if (dB) low.job[low.jobs++] = LowRankJob{false, X, C, ldx, A, U, nullptr, nullptr, top_u};
  if (dX || dA)
    low.job[low.jobs++] = LowRankJob{true, dY, R, lddy, B, dA ? V : nullptr, dX ? V_pair : nullptr, dX ? shift : nullptr, dA ? top_v : nullptr};
  windq_status done = launch_low_rank(ctx, low, st);
  // the gradients before dX: the projection's first tiles then start while the last of them finish
  if (done == WINDQ_OK && (dA || dB)) {
    const Gradient ga{X, C, ldx, V, top_v, dA}, gb{dY, R, lddy, U, top_u, dB};
    done = launch_gradients(ctx, dA ? &ga : nullptr, dB ? &gb : nullptr, dtype, T, rank, n_adapters, adapter_of, st);
  }
  if (done == WINDQ_OK && dX)
    done = launch_projection(
        ctx, Projection{dtype, true, dY, T, R, C, lddy, W, ldw, A, n_adapters, rank, adapter_of, V_pair, shift, lists, dX, lddx}, st);
  return done;
}

}  // extern "C"
