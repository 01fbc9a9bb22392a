// One AdamW step over many tensors, states in 32 or in 8 bits, and the values of 8-bit states.
//
// Every element is read once and written once, so the step is bound by HBM: 28 bytes an element with fp32 parameter,
// gradient and states, 16 (12 + two codes read and written) with 8-bit states.
//
// A warp owns 256 consecutive elements of one tensor -- the block that shares the scales of 8-bit states, so that their
// two maxima are warp reductions -- and a lane eight of them, loaded as 128-bit words.  A thread block takes eight such
// blocks of one tensor and finds its tensor by bisection in the table of first blocks, which travels with the launch as
// a kernel parameter: any mix of tensor sizes is one launch, and nothing is copied to the device before it.
#include <math.h>

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
// Kernel parameters may hold 32764 bytes; the small table keeps the launches of a few tensors cheap.
template <int N>
struct AdamwTable {
  AdamwEntry e[N];
  int first[N];  // first chunk of every tensor
  int count;
};
constexpr int kSmallTable = 32, kLargeTable = 448;
static_assert(sizeof(AdamwTable<kLargeTable>) + 128 < 32764, "kernel parameters");

struct AdamwFactors {
  float beta1, one_minus_beta1, beta2, one_minus_beta2, keep, rate, unbias, eps;
  const float* grad_scale;
  int param_dtype, grad_dtype, copy_dtype;
};

template <int N>
__device__ __forceinline__ int find_entry(const AdamwTable<N>& tab, int chunk) {
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
  return x;
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
__device__ __forceinline__ void split_bytes(uint2 w, int (&q)[8], bool is_signed) {
#pragma unroll
  for (int k = 0; k < 8; k++) {
    const uint32_t b = ((k < 4 ? w.x : w.y) >> (8 * (k & 3))) & 0xffu;
    q[k] = is_signed ? (int)(int8_t)b : (int)b;
  }
}
__device__ __forceinline__ uint2 join_bytes(const int (&q)[8]) {
  uint2 w = make_uint2(0, 0);
#pragma unroll
  for (int k = 0; k < 8; k++) {
    const uint32_t b = ((uint32_t)q[k] & 0xffu) << (8 * (k & 3));
    if (k < 4) w.x |= b;
    else w.y |= b;
  }
  return w;
}
__device__ __forceinline__ void load_codes(const void* base, int64_t i, int live, bool is_signed, int (&q)[8]) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + i;
  uint2 w = make_uint2(0, 0);
  if (live == 8) {
    w = *reinterpret_cast<const uint2*>(p);
  } else {
#pragma unroll
    for (int k = 0; k < 8; k++)
      if (k < live) {
        if (k < 4) w.x |= (uint32_t)p[k] << (8 * k);
        else w.y |= (uint32_t)p[k] << (8 * (k - 4));
      }
  }
  split_bytes(w, q, is_signed);
}
__device__ __forceinline__ void store_codes(void* base, int64_t i, int live, const int (&q)[8]) {
  uint8_t* p = static_cast<uint8_t*>(base) + i;
  if (live == 8) {
    *reinterpret_cast<uint2*>(p) = join_bytes(q);
  } else {
#pragma unroll
    for (int k = 0; k < 8; k++)
      if (k < live) p[k] = (uint8_t)q[k];
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

template <int N, bool BITS8>
__global__ void __launch_bounds__(kWarps * 32) adamw_kernel(const __grid_constant__ AdamwTable<N> tab,
                                                            const __grid_constant__ AdamwFactors f) {
  const int j = find_entry(tab, blockIdx.x);
  const AdamwEntry& e = tab.e[j];
  const int64_t block = (int64_t)(blockIdx.x - tab.first[j]) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const int64_t n = e.n;
  if (block * kBlock >= n) return;  // whole warps only
  const int64_t i = block * kBlock + lane * 8;
  const int live = i + 8 <= n ? 8 : i < n ? (int)(n - i) : 0;

  float p[8], g[8], m[8], r[8];
  load_any(e.grad, i, f.grad_dtype, live, g);
  load_any(e.param, i, f.param_dtype, live, p);
  if (BITS8) {
    int q[8];
    const float ms = e.m_scale[block], rs = e.r_scale[block];
    load_codes(e.m, i, live, true, q);
#pragma unroll
    for (int k = 0; k < 8; k++) m[k] = decode_m(q[k], ms);
    load_codes(e.v, i, live, false, q);
#pragma unroll
    for (int k = 0; k < 8; k++) {
      r[k] = decode_r(q[k], rs);
      r[k] = r[k] * r[k];
    }
  } else {
    load_any(e.m, i, WINDQ_F32, live, m);
    load_any(e.v, i, WINDQ_F32, live, r);
  }
  const float scale = f.grad_scale ? *f.grad_scale : 1.0f;  // a product with 1 is exact
  float top_m = 0.0f, top_r = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; k++) {
    const float gk = g[k] * scale;
    m[k] = m[k] * f.beta1 + gk * f.one_minus_beta1;
    const float v = r[k] * f.beta2 + (gk * gk) * f.one_minus_beta2;
    r[k] = sqrtf(v);
    p[k] = p[k] * f.keep - (m[k] * f.rate) / (r[k] * f.unbias + f.eps);
    if (BITS8) {
      top_m = fmaxf(top_m, fabsf(m[k]));
      top_r = fmaxf(top_r, r[k]);
    } else {
      r[k] = v;
    }
  }
  store_any(e.param, i, f.param_dtype, live, p);
  if (e.copy) store_any(e.copy, i, f.copy_dtype, live, p);
  if (BITS8) {
    top_m = warp_max(top_m);
    top_r = warp_max(top_r);
    top_m = top_m >= kTiny ? top_m : 0.0f;
    top_r = top_r >= kTiny ? top_r : 0.0f;
    const float inv_m = top_m > 0.0f ? 1.0f / top_m : 0.0f, inv_r = top_r > 0.0f ? 1.0f / top_r : 0.0f;
    int q[8];
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const int c = min(__float2int_rn(sqrtf(fabsf(m[k]) * inv_m) * 127.0f), 127);
      q[k] = m[k] < 0.0f ? -c : c;
    }
    store_codes(e.m, i, live, q);
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const int c = min(__float2int_rn(sqrtf(r[k] * inv_r) * 255.0f), 255);
      q[k] = (r[k] > 0.0f && top_r > 0.0f) ? max(c, 1) : c;
    }
    store_codes(e.v, i, live, q);
    if (lane == 0) {
      e.m_scale[block] = top_m;
      e.r_scale[block] = top_r;
    }
  } else {
    store_any(e.m, i, WINDQ_F32, live, m);
    store_any(e.v, i, WINDQ_F32, live, r);
  }
}

// param and copy of the table hold the two outputs.
template <int N>
__global__ void __launch_bounds__(kWarps * 32) adamw_states_kernel(const __grid_constant__ AdamwTable<N> tab) {
  const int j = find_entry(tab, blockIdx.x);
  const AdamwEntry& e = tab.e[j];
  const int64_t block = (int64_t)(blockIdx.x - tab.first[j]) * kWarps + (threadIdx.x >> 5);
  const int64_t n = e.n;
  if (block * kBlock >= n) return;
  const int64_t i = block * kBlock + (threadIdx.x & 31) * 8;
  const int live = i + 8 <= n ? 8 : i < n ? (int)(n - i) : 0;
  int q[8];
  float x[8];
  const float ms = e.m_scale[block], rs = e.r_scale[block];
  load_codes(e.m, i, live, true, q);
#pragma unroll
  for (int k = 0; k < 8; k++) x[k] = decode_m(q[k], ms);
  store_any(e.param, i, WINDQ_F32, live, x);
  load_codes(e.v, i, live, false, q);
#pragma unroll
  for (int k = 0; k < 8; k++) {
    x[k] = decode_r(q[k], rs);
    x[k] = x[k] * x[k];
  }
  store_any(e.copy, i, WINDQ_F32, live, x);
}

// Launches `go` over the entries in tables of at most kLargeTable tensors and 2^30 chunks.
template <class Fill, class Small, class Large>
windq_status over_tables(windq_ctx* ctx, int n_jobs, Fill fill, Small small, Large large) {
  int j = 0;
  while (j < n_jobs) {
    AdamwTable<kLargeTable> tab;
    int64_t chunks = 0;
    tab.count = 0;
    while (j < n_jobs && tab.count < kLargeTable) {
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
    if (tab.count <= kSmallTable) {
      AdamwTable<kSmallTable> less;
      for (int k = 0; k < tab.count; k++) {
        less.e[k] = tab.e[k];
        less.first[k] = tab.first[k];
      }
      less.count = tab.count;
      small(less, (unsigned)chunks);
    } else {
      large(tab, (unsigned)chunks);
    }
    WINDQ_CUDA(ctx, cudaGetLastError());
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
  f.grad_scale = grad_scale;
  f.param_dtype = param_dtype;
  f.grad_dtype = grad_dtype;
  f.copy_dtype = copy_dtype;
  DeviceGuard guard(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  const int threads = kWarps * 32;
  return over_tables(
      ctx, n_jobs,
      [&](int j) {
        const windq_adamw_job& b = jobs[j];
        return AdamwEntry{b.param, b.grad, b.m, b.v, b.m_scale, b.r_scale, b.copy, b.n};
      },
      [&](const AdamwTable<kSmallTable>& tab, unsigned chunks) {
        if (state_bits == 8) adamw_kernel<kSmallTable, true><<<chunks, threads, 0, st>>>(tab, f);
        else adamw_kernel<kSmallTable, false><<<chunks, threads, 0, st>>>(tab, f);
      },
      [&](const AdamwTable<kLargeTable>& tab, unsigned chunks) {
        if (state_bits == 8) adamw_kernel<kLargeTable, true><<<chunks, threads, 0, st>>>(tab, f);
        else adamw_kernel<kLargeTable, false><<<chunks, threads, 0, st>>>(tab, f);
      });
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
  return over_tables(
      ctx, n_jobs,
      [&](int j) {
        const windq_adamw_job& b = jobs[j];
        return AdamwEntry{m_out[j], nullptr, b.m, b.v, b.m_scale, b.r_scale, v_out[j], b.n};
      },
      [&](const AdamwTable<kSmallTable>& tab, unsigned chunks) {
        adamw_states_kernel<kSmallTable><<<chunks, kWarps * 32, 0, st>>>(tab);
      },
      [&](const AdamwTable<kLargeTable>& tab, unsigned chunks) {
        adamw_states_kernel<kLargeTable><<<chunks, kWarps * 32, 0, st>>>(tab);
      });
}

}  // extern "C"
