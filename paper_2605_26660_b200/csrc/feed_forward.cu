// The feed-forward block of a quantised model: checks, the gradients of its two products, and the order of the kernels.
#include <algorithm>

#include "feed_forward.cuh"
#include "tcgen05.cuh"

namespace windq {
namespace {

constexpr int kThreads = 256;
__device__ constexpr float kInfinity = __builtin_huge_valf();

struct GateArgs {
  const void *gate, *up, *dH;
  int64_t T, ldg, lddh, half;
  int F, act, terms;
  uint16_t* D;     // [T][terms * 2 * half]: dG, dU, and of two terms what rounding took off each; columns of a half behind F are zeros
  uint32_t* top;   // fp16: bits of the largest finite |dG|, |dU|; bf16: NULL
  uint32_t* tops;  // of every block, before that
};

// dU = dH g s, dG = dH u (s + g s (1 - s) y'(g)): see act.
__device__ __forceinline__ void gate_gradient(float g, float u, float dh, int act, float& dg, float& du) {
  const float s = logistic(gate_exponent(g, act)), t = s * (1.0f - s);
  // a gate far out has no slope, and the polynomial of its exponent may have left binary32
  const float slope = act == WINDQ_SILU ? g : g * (kGeluA * fmaf(3.0f * kGeluB * g, g, 1.0f));
  du = dh * (g * s);
  dg = dh * u * (t == 0.0f ? s : fmaf(slope, t, s));
}
// The same where that is not finite.  A shut gate (s = 0) passes nothing on, however far out, and no gradient of H leaves none: of fp16
// sums beyond its range the forward pass kept infinities in gate and up, which stand for numbers.
__device__ __forceinline__ void gate_gradient_far_out(float g, float u, float dh, int act, float& dg, float& du) {
  if (logistic(gate_exponent(g, act)) == 0.0f || dh == 0.0f) {
    du = g != g ? g : dh * 0.0f;
    dg = u != u ? u : du;
  } else {
    gate_gradient(g, u, dh, act, dg, du);
  }
}

// What rounding took off x; nothing where it left infinity or NaN, which then stand for themselves.
__device__ __forceinline__ float rest_of(float x, float rounded) { return fabsf(rounded) < kInfinity ? x - rounded : 0.0f; }

// Eight columns a thread, rows gridDim.y apart.  Bound by memory: 6 bytes read and 4 written a value.  fp16's range does not hold
// what small losses leave, so its values are stored times a power of two (see gradient_power) that a launch with TOP finds
// first: another 6 bytes read, 4 % of a long backward pass.  (Registers for four blocks an SM, five with TOP: with 78 instead of 58 and 48
// 1000 x 4096 x 512 took 59 us instead of 55.5.)
template <int DT, bool TOP>
__global__ void __launch_bounds__(kThreads, TOP ? 5 : 4) gate_gradient_kernel(const GateArgs p) {
  __shared__ uint32_t warps[kThreads / 32];
  auto most = [&](uint32_t x) {  // of the block, in every thread
    x = __reduce_max_sync(0xffffffffu, x);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = x;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kThreads / 32; k++) x = max(x, warps[k]);
    return x;
  };
  launch_dependents();
  wait_for_predecessor();
  uint32_t top = 0;
  float power = 1.0f, largest = 0.0f;
  if (!TOP && p.top) {
    const int blocks = gridDim.x * gridDim.y;
    for (int i = threadIdx.x; i < blocks; i += kThreads) top = max(top, __ldcg(p.tops + i));
    top = most(top);
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) *p.top = top;
    power = gradient_power(top, 1);
  }
  for (int f = (blockIdx.x * kThreads + threadIdx.x) * 8; f < p.half; f += gridDim.x * kThreads * 8) {
    const int live = min(8, p.F - f);
    for (int64_t t = blockIdx.y; t < p.T; t += gridDim.y) {
      float g[8], u[8], dh[8], dg[8], du[8];
      if (live == 8) {
        load8(p.gate, t * p.ldg + f, DT, g);
        load8(p.up, t * p.ldg + f, DT, u);
        load8(p.dH, t * p.lddh + f, DT, dh);
      } else {
        load_some(p.gate, t * p.ldg + f, DT, live, g);
        load_some(p.up, t * p.ldg + f, DT, live, u);
        load_some(p.dH, t * p.lddh + f, DT, live, dh);
      }
      float spoilt = 0.0f;  // NaN if a value is not finite (tests of every value took 3 % of 1000 x 4096 x 512, this 1 %)
#pragma unroll
      for (int k = 0; k < 8; k++) {
        gate_gradient(g[k], u[k], dh[k], p.act, dg[k], du[k]);
        spoilt = fmaf(dg[k], 0.0f, fmaf(du[k], 0.0f, spoilt));
      }
      if (spoilt != 0.0f) {
#pragma unroll
        for (int k = 0; k < 8; k++) {  // reads them again, which costs no registers where all is well
          if (k >= live) break;
          gate_gradient_far_out(load1(p.gate, t * p.ldg + f + k, DT), load1(p.up, t * p.ldg + f + k, DT), load1(p.dH, t * p.lddh + f + k, DT), p.act,
                                dg[k], du[k]);
          // an infinity or a NaN spoils its own token and output, not the power of two of all others
          if (TOP && !(fabsf(dg[k]) < kInfinity)) dg[k] = 0.0f;
          if (TOP && !(fabsf(du[k]) < kInfinity)) du[k] = 0.0f;
        }
      }
#pragma unroll
      for (int k = 0; k < 8; k++) {
        if (TOP) {
          largest = fmaxf(largest, fmaxf(fabsf(dg[k]), fabsf(du[k])));
        } else {
          dg[k] *= power;
          du[k] *= power;
        }
      }
      if (!TOP) {
        const int64_t at = t * p.terms * 2 * p.half + f;
        store8(p.D, at, DT, dg);
        store8(p.D, at + p.half, DT, du);
        if (p.terms == 2) {
#pragma unroll
          for (int k = 0; k < 8; k += 2) {
            const float2 g2 = unpack2(pack2(dg[k], dg[k + 1], DT), DT), u2 = unpack2(pack2(du[k], du[k + 1], DT), DT);
            dg[k] = rest_of(dg[k], g2.x);
            dg[k + 1] = rest_of(dg[k + 1], g2.y);
            du[k] = rest_of(du[k], u2.x);
            du[k + 1] = rest_of(du[k + 1], u2.y);
          }
          store8(p.D, at + 2 * p.half, DT, dg);
          store8(p.D, at + 3 * p.half, DT, du);
        }
      }
    }
  }
  if (TOP) {
    top = most(__float_as_uint(largest));
    if (threadIdx.x == 0) p.tops[blockIdx.y * gridDim.x + blockIdx.x] = top;
  }
}

constexpr int kBlocksPerSm = 24;   // over the whole launch: short blocks come out even (with 8, 4096 x 11008 took 1210 instead of 1200 us in all)
constexpr int kMostBlocks = 8192;  // of the kernel above
constexpr int64_t kTopBytes = 256 + 4 * kMostBlocks;
template <int DT, bool TOP>
windq_status launch_gate_gradient(windq_ctx* ctx, const GateArgs& a, cudaStream_t st) {
  const int64_t across = std::min<int64_t>((a.half + 8 * kThreads - 1) / (8 * kThreads), kMostBlocks);
  const int64_t down = std::max<int64_t>(1, std::min<int64_t>({a.T, (int64_t)ctx->sm_count * kBlocksPerSm / across, kMostBlocks / across}));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  overlapped_launch(cfg, attrs, 1, kThreads, 1, 0, st);
  cfg.gridDim = dim3((unsigned)across, (unsigned)down);
  WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, gate_gradient_kernel<DT, TOP>, a));
  return WINDQ_OK;
}

windq_status check_common(windq_ctx* ctx, const char* who, const void* X, int64_t T, int64_t C, int64_t ldx, int64_t R, int step) {
  WINDQ_REQUIRE(ctx, !*ctx->gave_up, WINDQ_ERR_CUDA, "%s: a wait of an earlier call gave up, its results are invalid (windq_stalls)", who);
  WINDQ_REQUIRE(ctx, T >= 0 && T < (1ll << 31) - 256, WINDQ_ERR_SHAPE, "%s: T = %lld", who, (long long)T);
  // (a sum that ran for seconds would look like a stall)
  WINDQ_REQUIRE(ctx, R > 0 && C > 0 && R < (1ll << 26) && C < (1ll << 26), WINDQ_ERR_SHAPE, "%s: %lld outputs of %lld channels", who,
                (long long)R, (long long)C);
  WINDQ_REQUIRE(ctx, T == 0 || X, WINDQ_ERR_NULL, "%s: the tokens are NULL", who);
  WINDQ_REQUIRE(ctx, ldx >= C, WINDQ_ERR_SHAPE, "%s: ldx = %lld is below C = %lld", who, (long long)ldx, (long long)C);
  WINDQ_REQUIRE(ctx, ldx % step == 0 && aligned16(X), WINDQ_ERR_ALIGN, "%s: the tokens are not 16-byte aligned or ldx = %lld is no multiple of %d",
                who, (long long)ldx, step);
  return WINDQ_OK;
}
windq_status check_weight(windq_ctx* ctx, const char* who, const char* name, const void* W, int64_t ldw, int64_t C, int step) {
  WINDQ_REQUIRE(ctx, W, WINDQ_ERR_NULL, "%s: %s is NULL", who, name);
  WINDQ_REQUIRE(ctx, ldw >= C, WINDQ_ERR_SHAPE, "%s: the leading dimension %lld of %s is below C = %lld", who, (long long)ldw, name, (long long)C);
  WINDQ_REQUIRE(ctx, ldw % step == 0 && aligned16(W), WINDQ_ERR_ALIGN,
                "%s: %s is not 16-byte aligned or its leading dimension %lld no multiple of %d", who, name, (long long)ldw, step);
  return WINDQ_OK;
}
windq_status check_rows(windq_ctx* ctx, const char* who, const char* name, const void* O, int64_t ld, int64_t width) {
  WINDQ_REQUIRE(ctx, ld >= width, WINDQ_ERR_SHAPE, "%s: the leading dimension %lld of %s is below %lld", who, (long long)ld, name, (long long)width);
  WINDQ_REQUIRE(ctx, ld % 8 == 0 && aligned16(O), WINDQ_ERR_ALIGN, "%s: %s is not 16-byte aligned or its leading dimension %lld no multiple of 8",
                who, name, (long long)ld);
  return WINDQ_OK;
}
windq_status check_scale(windq_ctx* ctx, const char* who, const char* name, const float* s) {
  WINDQ_REQUIRE(ctx, s, WINDQ_ERR_NULL, "%s: %s is NULL", who, name);
  WINDQ_REQUIRE(ctx, ((uintptr_t)s & 3) == 0, WINDQ_ERR_ALIGN, "%s: %s is misaligned", who, name);
  return WINDQ_OK;
}
windq_status check_16bit(windq_ctx* ctx, const char* who, int dtype) {
  WINDQ_REQUIRE(ctx, dtype == WINDQ_F16 || dtype == WINDQ_BF16, WINDQ_ERR_ARG, "%s: dtype = %d is neither fp16 nor bf16", who, dtype);
  return WINDQ_OK;
}
windq_status check_act(windq_ctx* ctx, const char* who, int act) {
  WINDQ_REQUIRE(ctx, act == WINDQ_SILU || act == WINDQ_GELU_TANH, WINDQ_ERR_ARG, "%s: activation = %d", who, act);
  return WINDQ_OK;
}
#define WINDQ_TRY(call)                    \
  do {                                     \
    const windq_status s_ = (call);        \
    if (s_ != WINDQ_OK) return s_;         \
  } while (0)

// Terms of dG and dU on the tensor cores.  One costs dX, dWg and dWu about as much precision as their own rounding does (1.41 times its
// error; of few tokens, or where one hot channel has most of a gradient's norm, up to 1.8).  With two their own rounding is all there
// is.  Two is what few tokens take, where they cost next to nothing, and up to 2^30 products, whose time is mostly that of starting kernels
// (10 x 1000 x 800 13.8 -> 16.5 us, 1000 x 1000 x 1000 27.5 -> 41).
int64_t two_term_tokens(int64_t C, int64_t F) { return std::max<int64_t>(kMostFew, (1ll << 30) / (C * F)); }

// Sums of products of two codes stay in 32-bit integers up to here.
constexpr int64_t kMaxCodes = 131071;

}  // namespace
}  // namespace windq

extern "C" {

int64_t windq_scratch_bytes_int8_forward(int64_t T, int64_t R, int64_t C) { return T < 0 || R <= 0 || C <= 0 ? 0 : windq::product_scratch(T); }
int64_t windq_scratch_bytes_gated_forward(int64_t T, int64_t C, int64_t F) { return T < 0 || C <= 0 || F <= 0 ? 0 : windq::product_scratch(T); }

windq_status windq_int8_forward(windq_ctx* ctx, const int8_t* X, int64_t T, int64_t C, int64_t ldx, const float* x_scale,
                                const int8_t* W, int64_t R, int64_t ldw, const float* w_scale, int dtype, void* Y, int64_t ldy,
                                void* stream) {
  using namespace windq;
  const char* who = "windq_int8_forward";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_TRY(check_common(ctx, who, X, T, C, ldx, R, 16));
  WINDQ_REQUIRE(ctx, C <= kMaxCodes, WINDQ_ERR_SHAPE, "%s: C = %lld is above %lld", who, (long long)C, (long long)kMaxCodes);
  WINDQ_TRY(check_16bit(ctx, who, dtype));
  WINDQ_TRY(check_weight(ctx, who, "W", W, ldw, C, 16));
  WINDQ_TRY(check_scale(ctx, who, "w_scale", w_scale));
  WINDQ_TRY(check_rows(ctx, who, "Y", Y, ldy, R));
  if (T == 0) return WINDQ_OK;
  WINDQ_TRY(check_scale(ctx, who, "x_scale", x_scale));
  WINDQ_REQUIRE(ctx, Y, WINDQ_ERR_NULL, "%s: Y is NULL", who);
  DeviceGuard guard(ctx->device);
  WINDQ_TRY(ensure_scratch(ctx, product_scratch(T)));
  Product q = {kInt8, dtype, 0, T, R, C, X, ldx, {W, nullptr}, {ldw, 0}, 0, 0, x_scale, {w_scale, nullptr}, nullptr, {Y, nullptr, nullptr}, {ldy, 0, 0},
               ctx->scratch};
  return launch_product(ctx, q, (cudaStream_t)stream);
}

windq_status windq_gated_int8_forward(windq_ctx* ctx, int activation, const int8_t* X, int64_t T, int64_t C, int64_t ldx,
                                      const float* x_scale, const int8_t* Wg, int64_t ldwg, const float* wg_scale, const int8_t* Wu,
                                      int64_t ldwu, const float* wu_scale, int64_t F, int dtype, void* H, int64_t ldh, void* stream) {
  using namespace windq;
  const char* who = "windq_gated_int8_forward";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_TRY(check_common(ctx, who, X, T, C, ldx, F, 16));
  WINDQ_REQUIRE(ctx, C <= kMaxCodes, WINDQ_ERR_SHAPE, "%s: C = %lld is above %lld", who, (long long)C, (long long)kMaxCodes);
  WINDQ_TRY(check_act(ctx, who, activation));
  WINDQ_TRY(check_16bit(ctx, who, dtype));
  WINDQ_TRY(check_weight(ctx, who, "Wg", Wg, ldwg, C, 16));
  WINDQ_TRY(check_weight(ctx, who, "Wu", Wu, ldwu, C, 16));
  WINDQ_TRY(check_scale(ctx, who, "wg_scale", wg_scale));
  WINDQ_TRY(check_scale(ctx, who, "wu_scale", wu_scale));
  WINDQ_TRY(check_rows(ctx, who, "H", H, ldh, F));
  if (T == 0) return WINDQ_OK;
  WINDQ_TRY(check_scale(ctx, who, "x_scale", x_scale));
  WINDQ_REQUIRE(ctx, H, WINDQ_ERR_NULL, "%s: H is NULL", who);
  DeviceGuard guard(ctx->device);
  WINDQ_TRY(ensure_scratch(ctx, product_scratch(T)));
  Product q = {kInt8Gated, dtype, activation, T, F, C, X, ldx, {Wg, Wu}, {ldwg, ldwu}, 0, 0, x_scale, {wg_scale, wu_scale}, nullptr,
               {H, nullptr, nullptr}, {ldh, 0, 0}, ctx->scratch};
  return launch_product(ctx, q, (cudaStream_t)stream);
}

windq_status windq_gated_forward(windq_ctx* ctx, int dtype, int activation, const void* X, int64_t T, int64_t C, int64_t ldx,
                                 const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, int64_t F, void* H, int64_t ldh,
                                 void* gate_out, void* up_out, int64_t ldg, void* stream) {
  using namespace windq;
  const char* who = "windq_gated_forward";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_TRY(check_common(ctx, who, X, T, C, ldx, F, 8));
  WINDQ_TRY(check_16bit(ctx, who, dtype));
  WINDQ_TRY(check_act(ctx, who, activation));
  WINDQ_TRY(check_weight(ctx, who, "Wg", Wg, ldwg, C, 8));
  WINDQ_TRY(check_weight(ctx, who, "Wu", Wu, ldwu, C, 8));
  WINDQ_TRY(check_rows(ctx, who, "H", H, ldh, F));
  WINDQ_REQUIRE(ctx, !gate_out == !up_out, WINDQ_ERR_NULL, "%s: one of gate_out and up_out is NULL", who);
  if (gate_out) {
    WINDQ_TRY(check_rows(ctx, who, "gate_out", gate_out, ldg, F));
    WINDQ_TRY(check_rows(ctx, who, "up_out", up_out, ldg, F));
  }
  if (T == 0) return WINDQ_OK;
  WINDQ_REQUIRE(ctx, H, WINDQ_ERR_NULL, "%s: H is NULL", who);
  DeviceGuard guard(ctx->device);
  WINDQ_TRY(ensure_scratch(ctx, product_scratch(T)));
  Product q = {kGated, dtype, activation, T, F, C, X, ldx, {Wg, Wu}, {ldwg, ldwu}, 0, 0, nullptr, {nullptr, nullptr}, nullptr,
               {H, gate_out, up_out}, {ldh, ldg, ldg}, ctx->scratch};
  return launch_product(ctx, q, (cudaStream_t)stream);
}

int64_t windq_scratch_bytes_gated_backward(int64_t T, int64_t C, int64_t F, int recompute) {
  if (T < 0 || C <= 0 || F <= 0 || C >= 1ll << 26 || F >= 1ll << 26) return 0;
  const int64_t half = windq::round_up(F, 64);
  // never less for more tokens
  const int64_t rows = std::max<int64_t>(T, 2 * std::min<int64_t>(T, windq::two_term_tokens(C, F)));
  return windq::kTopBytes + windq::round_up(4 * rows * half, 256) + (recompute ? windq::round_up(4 * T * half, 256) : 0) +
         windq::product_scratch(T);
}

windq_status windq_gated_backward(windq_ctx* ctx, int dtype, int activation, const void* X, int64_t T, int64_t C, int64_t ldx,
                                  const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, int64_t F, const void* gate,
                                  const void* up, int64_t ldg, const void* dH, int64_t lddh, void* dX, int64_t lddx, void* dWg,
                                  void* dWu, int64_t lddw, void* stream) {
  using namespace windq;
  const char* who = "windq_gated_backward";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_TRY(check_common(ctx, who, X, T, C, ldx, F, 8));
  WINDQ_TRY(check_16bit(ctx, who, dtype));
  WINDQ_TRY(check_act(ctx, who, activation));
  WINDQ_TRY(check_weight(ctx, who, "Wg", Wg, ldwg, C, 8));
  WINDQ_TRY(check_weight(ctx, who, "Wu", Wu, ldwu, C, 8));
  WINDQ_REQUIRE(ctx, T < (1ll << 28), WINDQ_ERR_SHAPE, "%s: T = %lld", who, (long long)T);
  WINDQ_REQUIRE(ctx, !gate == !up, WINDQ_ERR_NULL, "%s: one of gate and up is NULL", who);
  if (gate) {
    WINDQ_TRY(check_rows(ctx, who, "gate", gate, ldg, F));
    WINDQ_TRY(check_rows(ctx, who, "up", up, ldg, F));
  }
  WINDQ_TRY(check_rows(ctx, who, "dH", dH, lddh, F));
  WINDQ_REQUIRE(ctx, !dWg == !dWu, WINDQ_ERR_NULL, "%s: one of dWg and dWu is NULL", who);
  WINDQ_REQUIRE(ctx, dX || dWg, WINDQ_ERR_NULL, "%s: dX, dWg and dWu are all NULL", who);
  if (dX) WINDQ_TRY(check_rows(ctx, who, "dX", dX, lddx, C));
  if (dWg) {
    WINDQ_TRY(check_rows(ctx, who, "dWg", dWg, lddw, C));
    WINDQ_TRY(check_rows(ctx, who, "dWu", dWu, lddw, C));
  }
  DeviceGuard guard(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  if (T == 0) {
    if (dWg) WINDQ_CUDA(ctx, cudaMemset2DAsync(dWg, 2 * lddw, 0, 2 * C, F, st));
    if (dWg) WINDQ_CUDA(ctx, cudaMemset2DAsync(dWu, 2 * lddw, 0, 2 * C, F, st));
    return WINDQ_OK;
  }
  WINDQ_REQUIRE(ctx, dH, WINDQ_ERR_NULL, "%s: dH is NULL", who);
  WINDQ_TRY(ensure_scratch(ctx, windq_scratch_bytes_gated_backward(T, C, F, !gate)));
  const int64_t half = round_up(F, 64);
  char* at = (char*)ctx->scratch;
  auto take = [&](int64_t bytes) {
    char* p = at;
    at += round_up(bytes, 256);
    return p;
  };
  uint32_t* top = (uint32_t*)take(kTopBytes);
  const int terms = T <= two_term_tokens(C, F) ? 2 : 1;
  uint16_t* D = (uint16_t*)take(4 * T * half * terms);
  uint16_t* kept = gate ? nullptr : (uint16_t*)take(4 * T * half);
  void* partials = at;
  if (!gate) {
    gate = kept;
    up = kept + T * half;
    ldg = half;
    Product q = {kGated, dtype, activation, T, F, C, X, ldx, {Wg, Wu}, {ldwg, ldwu}, 0, 0, nullptr, {nullptr, nullptr}, nullptr,
                 {nullptr, kept, kept + T * half}, {0, half, half}, partials};
    WINDQ_TRY(launch_product(ctx, q, st));
  }
  GateArgs a = {gate, up, dH, T, ldg, lddh, half, (int)F, activation, terms, D, dtype == WINDQ_F16 ? top : nullptr, top + 64};
  if (a.top) {
    WINDQ_TRY((launch_gate_gradient<WINDQ_F16, true>(ctx, a, st)));
    WINDQ_TRY((launch_gate_gradient<WINDQ_F16, false>(ctx, a, st)));
  } else {
    WINDQ_TRY((launch_gate_gradient<WINDQ_BF16, false>(ctx, a, st)));
  }
  if (dX) {
    Product q = {kInputGrad, dtype, 0, T, C, F, D, terms * 2 * half, {Wg, Wu}, {ldwg, ldwu}, half, terms, nullptr, {nullptr, nullptr}, a.top,
                 {dX, nullptr, nullptr}, {lddx, 0, 0}, partials};
    WINDQ_TRY(launch_product(ctx, q, st));
  }
  if (dWg) WINDQ_TRY(launch_weight_gradient(ctx, WeightGradient{dtype, terms, T, F, C, half, D, X, ldx, a.top, dWg, dWu, lddw}, st));
  return WINDQ_OK;
}

}  // extern "C"
