// One AdamW step over many tensors, states in 32 or in 8 bits, and the values of 8-bit states.
//
// Every element is read once and written once, so the step is bound by HBM: 28 bytes an element with fp32 parameter,
// gradient and states, 16 (12 + two codes read and written) with 8-bit states.  At the measured copy rate that leaves an
// SM about 90 instructions an element with 8-bit states, and a plain version of that kernel took 119 (three square roots
// and a quotient among them), so its arithmetic is written for few instructions; see adamw8_kernel.
//
// A warp owns 256 consecutive elements of one tensor -- the block that shares the scales of 8-bit states, so that their
// two maxima are warp reductions -- and a lane eight of them, loaded as 128-bit words.  A thread block takes eight such
// blocks of one tensor and finds its tensor by bisection in the table of first blocks, which travels with the launch as
// a kernel parameter: any mix of tensor sizes is one launch, and nothing is copied to the device before it.
#include <math.h>

#include "fit_device.cuh"
#include "tcgen05.cuh"
#include "typed.cuh"

namespace windq {
namespace {

constexpr int kBlock = 256;                   // elements that share a state scale; elements of a warp
constexpr int kWarps = 8;                     // warps of a thread block
constexpr int kChunk = kBlock * kWarps;       // elements of a thread block

struct AdamwEntry {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* r_scale;
  void* copy;
  int64_t n;
};
// The tensors of one launch: as many as 4 KB of kernel parameters hold.  (Tables of 448 tensors in 32 KB gained nothing for
// 448 tensors, whose 8 launches overlap, and cost the host 5 us more for 14 or 120.)
constexpr int kTable = 56;
struct AdamwTable {
  AdamwEntry e[kTable];
  int first[kTable];  // first chunk of every tensor
  int count;
};

struct AdamwFactors {
  float beta1, one_minus_beta1, beta2, one_minus_beta2, keep, rate, unbias, eps, one;
  const float* grad_scale;
  int param_dtype, grad_dtype, copy_dtype;
};

__device__ __forceinline__ int find_entry(const AdamwTable& tab, int chunk) {
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

constexpr float kPerM = (float)(1.0 / 127), kPerR = (float)(1.0 / 255);
constexpr float kTiny = 0x1p-100f;

__device__ __forceinline__ float decode_m(int q, float scale) {
  const float u = (float)q * kPerM;
  return (u * fabsf(u)) * scale;
}
__device__ __forceinline__ float decode_r(int q, float scale) {
  const float u = (float)q * kPerR;
  return (u * u) * scale;
}

// The eight codes of a lane, little-endian in two words.
__device__ __forceinline__ uint2 load_codes(const void* base, int64_t i, int live) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + i;
  if (live == 8) return *reinterpret_cast<const uint2*>(p);
  uint2 w = make_uint2(0, 0);
#pragma unroll
  for (int k = 0; k < 8; k++)
    if (k < live) {
      if (k < 4) w.x |= (uint32_t)p[k] << (8 * k);
      else w.y |= (uint32_t)p[k] << (8 * (k - 4));
    }
  return w;
}
__device__ __forceinline__ void store_codes(void* base, int64_t i, int live, uint2 w) {
  uint8_t* p = static_cast<uint8_t*>(base) + i;
  if (live == 8) {
    *reinterpret_cast<uint2*>(p) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; k++)
      if (k < live) p[k] = (uint8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
  }
}
__device__ __forceinline__ void load_any(const void* base, int64_t i, int dt, int live, float (&x)[8]) {
  if (live == 8) load8(base, i, dt, x);
  else load_some(base, i, dt, live, x);
}
__device__ __forceinline__ void store_any(void* base, int64_t i, int dt, int live, const float (&x)[8]) {
  if (live == 8) store8(base, i, dt, x);
  else store_some(base, i, dt, live, x);
}

__global__ void __launch_bounds__(kWarps * 32) adamw32_kernel(const __grid_constant__ AdamwTable tab,
                                                              const __grid_constant__ AdamwFactors f) {
  launch_dependents();
  const int j = find_entry(tab, blockIdx.x);
  const AdamwEntry& e = tab.e[j];
  const int64_t block = (int64_t)(blockIdx.x - tab.first[j]) * kWarps + (threadIdx.x >> 5);
  const int64_t n = e.n, i = block * kBlock + (threadIdx.x & 31) * 8;
  if (i >= n) return wait_for_predecessor();
  const int live = i + 8 <= n ? 8 : (int)(n - i);
  float p[8], g[8], m[8], v[8];
  load_any(e.grad, i, f.grad_dtype, live, g);
  load_any(e.param, i, f.param_dtype, live, p);
  load_any(e.m, i, WINDQ_F32, live, m);
  load_any(e.v, i, WINDQ_F32, live, v);
  const float scale = f.grad_scale ? *f.grad_scale : 1.0f;  // a product with 1 is exact
#pragma unroll
  for (int k = 0; k < 8; k++) {
    const float gk = g[k] * scale;
    m[k] = m[k] * f.beta1 + gk * f.one_minus_beta1;
    v[k] = v[k] * f.beta2 + (gk * gk) * f.one_minus_beta2;
    p[k] = p[k] * f.keep - (m[k] * f.rate) / (sqrtf(v[k]) * f.unbias + f.eps);
  }
  store_any(e.param, i, f.param_dtype, live, p);
  if (e.copy) store_any(e.copy, i, f.copy_dtype, live, p);
  store_any(e.m, i, WINDQ_F32, live, m);
  store_any(e.v, i, WINDQ_F32, live, v);
  wait_for_predecessor();
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Byte k of a word of codes as a binary32 value, offset by 2^23: the byte becomes the low end of a significand.
__device__ __forceinline__ float code_bits(uint32_t w, int k) { return __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7550 | k)); }
constexpr float kShift = 8388608.0f;   // 2^23
constexpr float kRound = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer (to nearest even), kept in the low bits

// rint(sqrt(|x|) * levels) of eight values in [-1, 1], with the sign of x where SIGNED, plus kRound.  The hardware's square
// root is off by 2^-22 of itself at most, the product by another 2^-24: less than `guard` of a code.  Only where that could
// cross a rounding boundary is the correctly rounded root taken.
template <bool SIGNED>
__device__ __forceinline__ float with_sign(float y, float x) {  // y >= 0
  return SIGNED ? __uint_as_float(__float_as_uint(y) | (__float_as_uint(x) & 0x80000000u)) : y;
}
template <bool SIGNED>
__device__ __forceinline__ void encode8(const float (&x)[8], float levels, float guard, float (&out)[8]) {
  float worst = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    float2 y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fabsf(x[k])));
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fabsf(x[k + 1])));
    y = mul2(y, both(levels));
    y = make_float2(with_sign<SIGNED>(y.x, x[k]), with_sign<SIGNED>(y.y, x[k + 1]));
    const float2 r = add2(y, both(kRound)), off = fma2(add2(r, both(-kRound)), both(-1.0f), y);
    worst = fmaxf(worst, fmaxf(fabsf(off.x), fabsf(off.y)));
    out[k] = r.x;
    out[k + 1] = r.y;
  }
  if (worst > 0.5f - guard) {
#pragma unroll
    for (int k = 0; k < 8; k++) out[k] = with_sign<SIGNED>(sqrtf(fabsf(x[k])) * levels, x[k]) + kRound;
  }
}
// The low bytes of eight such values.
__device__ __forceinline__ uint2 low_bytes(const float (&x)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const uint32_t a = __byte_perm(__float_as_uint(x[4 * h]), __float_as_uint(x[4 * h + 1]), 0x0040);
    const uint32_t b = __byte_perm(__float_as_uint(x[4 * h + 2]), __float_as_uint(x[4 * h + 3]), 0x0040);
    w[h] = __byte_perm(a, b, 0x5410);
  }
  return make_uint2(w[0], w[1]);
}

// What keeps the instructions few: pairs of binary32 operations in one (each half rounded like the scalar one), codes turned
// into values and back by adding constants instead of conversions, and square roots for codes taken from the approximate
// instruction wherever that decides the code.  All results are those of the formulas, bit for bit.
__global__ void __launch_bounds__(kWarps * 32) adamw8_kernel(const __grid_constant__ AdamwTable tab,
                                                             const __grid_constant__ AdamwFactors f) {
  launch_dependents();
  const int j = find_entry(tab, blockIdx.x);
  const AdamwEntry& e = tab.e[j];
  const int64_t block = (int64_t)(blockIdx.x - tab.first[j]) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const int64_t n = e.n;
  if (block * kBlock >= n) return wait_for_predecessor();  // whole warps only: the block's largest values are warp reductions
  const int64_t i = block * kBlock + lane * 8;
  const int live = i + 8 <= n ? 8 : i < n ? (int)(n - i) : 0;

  float p[8], g[8], m[8], r[8];
  const uint2 qm = load_codes(e.m, i, live), qr = load_codes(e.v, i, live);
  const float ms = e.m_scale[block], rs = e.r_scale[block];
  load_any(e.grad, i, f.grad_dtype, live, g);
  load_any(e.param, i, f.param_dtype, live, p);
  const float2 scale = both(f.grad_scale ? *f.grad_scale : 1.0f);  // a product with 1 is exact
  // The assembler joins a packed product and a packed sum into one rounding; a product with a one that it cannot see keeps
  // both roundings of x + y.
  const float2 one = both(f.one);
  const uint32_t wm[2] = {qm.x ^ 0x80808080u, qm.y ^ 0x80808080u}, wr[2] = {qr.x, qr.y};
  float top_m = 0.0f;
  uint32_t top_r_bits = 0;  // values >= 0 order like their bit patterns, and NaN comes out largest
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    float2 um = make_float2(code_bits(wm[k >> 2], k & 3), code_bits(wm[k >> 2], (k & 3) + 1));
    float2 ur = make_float2(code_bits(wr[k >> 2], k & 3), code_bits(wr[k >> 2], (k & 3) + 1));
    um = mul2(add2(um, both(-kShift - 128.0f)), both(kPerM));
    ur = mul2(add2(ur, both(-kShift)), both(kPerR));
    const float2 mk = mul2(make_float2(um.x * fabsf(um.x), um.y * fabsf(um.y)), both(ms));
    const float2 rk = mul2(mul2(ur, ur), both(rs));
    const float2 gk = mul2(make_float2(g[k], g[k + 1]), scale);
    const float2 mn = fma2(mul2(mk, both(f.beta1)), one, mul2(gk, both(f.one_minus_beta1)));
    const float2 v = fma2(mul2(mul2(rk, rk), both(f.beta2)), one, mul2(mul2(gk, gk), both(f.one_minus_beta2)));
    const float2 rn = make_float2(sqrtf(v.x), sqrtf(v.y));
    const float2 up = mul2(mn, both(f.rate)), down = fma2(mul2(rn, both(f.unbias)), one, both(f.eps));
    const float2 pn = fma2(make_float2(up.x / down.x, up.y / down.y), both(-1.0f), mul2(make_float2(p[k], p[k + 1]), both(f.keep)));
    p[k] = pn.x, p[k + 1] = pn.y;
    m[k] = mn.x, m[k + 1] = mn.y;
    r[k] = rn.x, r[k + 1] = rn.y;
    top_m = fmaxf(top_m, fmaxf(fabsf(mn.x), fabsf(mn.y)));
    top_r_bits = max(top_r_bits, max(__float_as_uint(rn.x), __float_as_uint(rn.y)));
  }
  store_any(e.param, i, f.param_dtype, live, p);
  if (e.copy) store_any(e.copy, i, f.copy_dtype, live, p);
  top_r_bits = __reduce_max_sync(0xffffffffu, top_r_bits);
  if (top_r_bits >= 0x7f800000u) {
    // Some r is not finite (m is wherever r is): its element starts anew, so that the scales stay those of the others.
    top_m = 0.0f;
    top_r_bits = 0;
#pragma unroll
    for (int k = 0; k < 8; k++) {
      if (__float_as_uint(r[k]) >= 0x7f800000u) m[k] = r[k] = 0.0f;
      top_m = fmaxf(top_m, fabsf(m[k]));
      top_r_bits = max(top_r_bits, __float_as_uint(r[k]));
    }
    top_r_bits = __reduce_max_sync(0xffffffffu, top_r_bits);
  }
  top_m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top_m)));
  float top_r = __uint_as_float(top_r_bits);
  top_m = top_m >= kTiny ? top_m : 0.0f;
  top_r = top_r >= kTiny ? top_r : 0.0f;
  const float inv_m = top_m > 0.0f ? 1.0f / top_m : 0.0f, inv_r = top_r > 0.0f ? 1.0f / top_r : 0.0f;
  float x[8], c[8];
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    const float2 y = mul2(make_float2(m[k], m[k + 1]), both(inv_m));
    x[k] = y.x, x[k + 1] = y.y;
  }
  encode8<true>(x, 127.0f, 0x1p-14f, c);
  store_codes(e.m, i, live, low_bytes(c));
  const float least = top_r > 0.0f ? kRound + 1.0f : kRound;  // the code an r above zero gets at least
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    const float2 y = mul2(make_float2(r[k], r[k + 1]), both(inv_r));
    x[k] = y.x, x[k + 1] = y.y;
  }
  encode8<false>(x, 255.0f, 0x1p-13f, c);
#pragma unroll
  for (int k = 0; k < 8; k++) c[k] = r[k] > 0.0f ? fmaxf(c[k], least) : c[k];
  store_codes(e.v, i, live, low_bytes(c));
  if (lane == 0) {
    e.m_scale[block] = top_m;
    e.r_scale[block] = top_r;
  }
  wait_for_predecessor();
}

// param and copy of the table hold the two outputs.
__global__ void __launch_bounds__(kWarps * 32) adamw_states_kernel(const __grid_constant__ AdamwTable tab) {
  launch_dependents();
  const int j = find_entry(tab, blockIdx.x);
  const AdamwEntry& e = tab.e[j];
  const int64_t block = (int64_t)(blockIdx.x - tab.first[j]) * kWarps + (threadIdx.x >> 5);
  const int64_t n = e.n;
  if (block * kBlock >= n) return wait_for_predecessor();
  const int64_t i = block * kBlock + (threadIdx.x & 31) * 8;
  const int live = i + 8 <= n ? 8 : i < n ? (int)(n - i) : 0;
  const uint2 qm = load_codes(e.m, i, live), qr = load_codes(e.v, i, live);
  const float ms = e.m_scale[block], rs = e.r_scale[block];
  float x[8];
#pragma unroll
  for (int k = 0; k < 8; k++) x[k] = decode_m((int)(int8_t)((k < 4 ? qm.x : qm.y) >> (8 * (k & 3))), ms);
  store_any(e.param, i, WINDQ_F32, live, x);
#pragma unroll
  for (int k = 0; k < 8; k++) {
    x[k] = decode_r((int)(uint8_t)((k < 4 ? qr.x : qr.y) >> (8 * (k & 3))), rs);
    x[k] = x[k] * x[k];
  }
  store_any(e.copy, i, WINDQ_F32, live, x);
  wait_for_predecessor();
}

// Launches `kernel` over the entries, kTable tensors and at most 2^30 chunks at a time.  The launches touch different
// tensors: all but the first may start before their predecessor has ended, and end after it.
template <class Fill, class... Kernel, class... More>
windq_status over_tables(windq_ctx* ctx, int n_jobs, Fill fill, cudaStream_t st, void (*kernel)(Kernel...), const More&... more) {
  int j = 0;
  bool first = true;
  while (j < n_jobs) {
    AdamwTable tab;
    int64_t chunks = 0;
    tab.count = 0;
    while (j < n_jobs && tab.count < kTable) {
      const AdamwEntry e = fill(j);
      const int64_t c = (e.n + kChunk - 1) / kChunk;
      if (c > 0) {
        if (chunks + c > (1ll << 30)) break;
        tab.e[tab.count] = e;
        tab.first[tab.count] = (int)chunks;
        tab.count++;
        chunks += c;
      }
      j++;
    }
    if (tab.count == 0) continue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)chunks);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = first ? 0 : 1;
    WINDQ_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, tab, more...));
    first = false;
  }
  return WINDQ_OK;
}

bool valid_dtype(int dt) { return dt == WINDQ_F16 || dt == WINDQ_BF16 || dt == WINDQ_F32; }

// Checks shared by the two calls.
windq_status check_states(windq_ctx* ctx, const char* who, const windq_adamw_job& b, int j, int state_bits) {
  WINDQ_REQUIRE(ctx, b.n >= 0 && b.n < (1ll << 40), WINDQ_ERR_SHAPE, "%s: job %d: n = %lld", who, j, (long long)b.n);
  if (b.n == 0) return WINDQ_OK;
  WINDQ_REQUIRE(ctx, b.m && b.v, WINDQ_ERR_NULL, "%s: job %d: m or v is NULL", who, j);
  WINDQ_REQUIRE(ctx, aligned16(b.m) && aligned16(b.v), WINDQ_ERR_ALIGN, "%s: job %d: m or v is not 16-byte aligned", who, j);
  if (state_bits == 8) {
    WINDQ_REQUIRE(ctx, b.m_scale && b.r_scale, WINDQ_ERR_NULL, "%s: job %d: m_scale or r_scale is NULL", who, j);
    WINDQ_REQUIRE(ctx, ((uintptr_t)b.m_scale & 3) == 0 && ((uintptr_t)b.r_scale & 3) == 0, WINDQ_ERR_ALIGN,
                  "%s: job %d: m_scale or r_scale is misaligned", who, j);
  }
  return WINDQ_OK;
}

}  // namespace
}  // namespace windq

extern "C" {

windq_status windq_adamw_step(windq_ctx* ctx, const windq_adamw_job* jobs, int n_jobs, int param_dtype, int grad_dtype,
                              int copy_dtype, int state_bits, int64_t step, double lr, double beta1, double beta2, double eps,
                              double weight_decay, const float* grad_scale, void* stream) {
  using namespace windq;
  const char* who = "windq_adamw_step";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_REQUIRE(ctx, jobs, WINDQ_ERR_NULL, "%s: jobs is NULL", who);
  WINDQ_REQUIRE(ctx, n_jobs >= 1, WINDQ_ERR_SHAPE, "%s: n_jobs = %d", who, n_jobs);
  WINDQ_REQUIRE(ctx, valid_dtype(param_dtype) && valid_dtype(grad_dtype), WINDQ_ERR_ARG, "%s: param_dtype = %d, grad_dtype = %d",
                who, param_dtype, grad_dtype);
  WINDQ_REQUIRE(ctx, state_bits == 8 || state_bits == 32, WINDQ_ERR_ARG, "%s: state_bits = %d is neither 8 nor 32", who,
                state_bits);
  WINDQ_REQUIRE(ctx, step >= 1, WINDQ_ERR_ARG, "%s: step = %lld must be at least 1", who, (long long)step);
  WINDQ_REQUIRE(ctx, lr >= 0 && isfinite(lr) && weight_decay >= 0 && isfinite(weight_decay), WINDQ_ERR_ARG,
                "%s: lr = %g, weight_decay = %g", who, lr, weight_decay);
  WINDQ_REQUIRE(ctx, beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1, WINDQ_ERR_ARG, "%s: beta1 = %g, beta2 = %g", who, beta1,
                beta2);
  WINDQ_REQUIRE(ctx, (float)eps > 0 && isfinite((float)eps), WINDQ_ERR_ARG, "%s: eps = %g is not a positive binary32 value", who,
                eps);
  WINDQ_REQUIRE(ctx, ((uintptr_t)grad_scale & 3) == 0, WINDQ_ERR_ALIGN, "%s: grad_scale is misaligned", who);
  for (int j = 0; j < n_jobs; j++) {
    const windq_adamw_job& b = jobs[j];
    const windq_status st = check_states(ctx, who, b, j, state_bits);
    if (st != WINDQ_OK) return st;
    if (b.n == 0) continue;
    WINDQ_REQUIRE(ctx, b.param && b.grad, WINDQ_ERR_NULL, "%s: job %d: param or grad is NULL", who, j);
    WINDQ_REQUIRE(ctx, aligned16(b.param) && aligned16(b.grad) && aligned16(b.copy), WINDQ_ERR_ALIGN,
                  "%s: job %d: param, grad or copy is not 16-byte aligned", who, j);
    WINDQ_REQUIRE(ctx, !b.copy || copy_dtype == WINDQ_F16 || copy_dtype == WINDQ_BF16, WINDQ_ERR_ARG, "%s: copy_dtype = %d", who,
                  copy_dtype);
  }
  AdamwFactors f;
  f.beta1 = (float)beta1;
  f.one_minus_beta1 = (float)(1.0 - beta1);
  f.beta2 = (float)beta2;
  f.one_minus_beta2 = (float)(1.0 - beta2);
  f.keep = (float)(1.0 - lr * weight_decay);
  f.rate = (float)(lr / (1.0 - pow(beta1, (double)step)));
  f.unbias = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  f.eps = (float)eps;
  f.one = 1.0f;
  f.grad_scale = grad_scale;
  f.param_dtype = param_dtype;
  f.grad_dtype = grad_dtype;
  f.copy_dtype = copy_dtype;
  DeviceGuard guard(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  auto fill = [&](int j) {
    const windq_adamw_job& b = jobs[j];
    return AdamwEntry{b.param, b.grad, b.m, b.v, b.m_scale, b.r_scale, b.copy, b.n};
  };
  return over_tables(ctx, n_jobs, fill, st, state_bits == 8 ? adamw8_kernel : adamw32_kernel, f);
}

windq_status windq_adamw_states(windq_ctx* ctx, const windq_adamw_job* jobs, int n_jobs, float* const* m_out,
                                float* const* v_out, void* stream) {
  using namespace windq;
  const char* who = "windq_adamw_states";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_REQUIRE(ctx, jobs && m_out && v_out, WINDQ_ERR_NULL, "%s: jobs, m_out or v_out is NULL", who);
  WINDQ_REQUIRE(ctx, n_jobs >= 1, WINDQ_ERR_SHAPE, "%s: n_jobs = %d", who, n_jobs);
  for (int j = 0; j < n_jobs; j++) {
    const windq_status st = check_states(ctx, who, jobs[j], j, 8);
    if (st != WINDQ_OK) return st;
    if (jobs[j].n == 0) continue;
    WINDQ_REQUIRE(ctx, m_out[j] && v_out[j], WINDQ_ERR_NULL, "%s: job %d: an output is NULL", who, j);
    WINDQ_REQUIRE(ctx, aligned16(m_out[j]) && aligned16(v_out[j]), WINDQ_ERR_ALIGN, "%s: job %d: an output is not 16-byte aligned",
                  who, j);
  }
  DeviceGuard guard(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  auto fill = [&](int j) {
    const windq_adamw_job& b = jobs[j];
    return AdamwEntry{m_out[j], nullptr, b.m, b.v, b.m_scale, b.r_scale, v_out[j], b.n};
  };
  return over_tables(ctx, n_jobs, fill, st, adamw_states_kernel);
}

}  // extern "C"
