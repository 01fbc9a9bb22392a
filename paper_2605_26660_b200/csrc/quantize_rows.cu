// Rows of 16-bit values as 8-bit codes with one scale a row.
//
//   q = round(127 x / a), ties to even, of the exact quotient;  a = max |x| of the row;  scale = a / 127
// One pass: a row is held in registers between its maximum and its codes (up to 16384 values; of a longer one the rest is
// read again, from L2).  Bound by memory: 2 bytes read, 1 written a value, 2 more with the values the codes stand for (4096 x 14336
// with them: 46 us, 0.98 of the copy rate).  W warps share a row: as few as hold it where there are many rows, more where there are
// few and the time is one row's latency (one row of 2048: 2.5 us).
#include <algorithm>

#include "fit_device.cuh"
#include "tcgen05.cuh"
#include "typed.cuh"

namespace windq {
namespace {

constexpr int kThreads = 256, kHeld = 8;  // 16-byte pieces of a row in a lane's registers

struct QuantizeArgs {
  const uint16_t* X;
  int64_t T, ldx;
  int C;
  int8_t* q;
  int64_t ldq;
  float* scale;
  uint16_t* values;
  int64_t ldv;
};

// Eight values of a row as they are stored; what lies behind its end reads as zero and is not touched.  (Not __ldg, which wants memory
// that nothing writes while the kernel lives: this one is there before the kernel that writes X has ended.)
__device__ __forceinline__ uint4 load_piece(const uint16_t* row, int i, int C) {
  if (i * 8 + 8 <= C) return reinterpret_cast<const uint4*>(row)[i];
  uint32_t w[4] = {0, 0, 0, 0};
  for (int k = 0; i * 8 + k < C; k++) w[k >> 1] |= (uint32_t)row[i * 8 + k] << (16 * (k & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The largest magnitudes as bit patterns, two to a word: they order as the numbers do, infinities and then NaN above them all.
__device__ __forceinline__ uint32_t top_of(uint32_t top, const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; k++) top = __vmaxu2(top, w[k] & 0x7fff7fffu);
  return top;
}

// Codes of eight values.  y = x * inv is within 2^-23 of 127 x / a.  That quotient either is a border between two codes (8 bits) or
// is at least 2^-19 of itself away from one (the closest: 127 * 2025 / 2033 = 126.50025, 2^-18.97), and rounding y to 20 bits first --
// c - (c - y), c = 17 y -- moves it by 2^-20 at most: a border comes out as itself, what is not one stays on its side.  Two values an
// instruction: with one, the kernel was bound by issue (8192 x 8192 5 us more of 43).
// LIFT: rows of tiny values, whose 127 / a would overflow, are multiplied by 2^60 first.
template <int DT, bool VALUES, bool LIFT>
__device__ __forceinline__ void encode(const uint4& v, float inv, float scale, uint2& codes, uint4& values) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float t[8];
#pragma unroll
  for (int k = 0; k < 4; k++) {
    float2 x = unpack2(w[k], DT);
    if (LIFT) x = make_float2(x.x * 0x1p60f, x.y * 0x1p60f);
    const float2 y = mul2(x, make_float2(inv, inv)), c = fma2(y, make_float2(16.0f, 16.0f), y);
    const float2 minus = make_float2(-1.0f, -1.0f), rest = fma2(y, minus, c);
    const float2 q = add2(fma2(rest, minus, c), make_float2(12582912.0f, 12582912.0f));  // 1.5 * 2^23: the integer in the low bits
    t[2 * k] = q.x;
    t[2 * k + 1] = q.y;
  }
  uint32_t b[8];
#pragma unroll
  for (int k = 0; k < 8; k++) b[k] = __float_as_uint(t[k]);
  codes.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  codes.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
  if (VALUES) {
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 4; k++) o[k] = pack2((t[2 * k] - 12582912.0f) * scale, (t[2 * k + 1] - 12582912.0f) * scale, DT);
    values = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

template <int DT, int W, bool VALUES>
__global__ void __launch_bounds__(kThreads) quantize_kernel(const QuantizeArgs p) {
  __shared__ uint32_t tops[kThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % W;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 32 / W) + warp / W;
  const bool live = t < p.T;
  launch_dependents();
  wait_for_predecessor();
  const uint16_t* row = p.X + (live ? t : 0) * p.ldx;
  const int pieces = live ? (p.C + 7) / 8 : 0, first = part * 32 + lane, step = W * 32;
  uint4 held[kHeld];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < kHeld; k++) held[k] = first + k * step < pieces ? load_piece(row, first + k * step, p.C) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int k = 0; k < kHeld; k++) top = top_of(top, held[k]);
  for (int i = first + kHeld * step; i < pieces; i += step) top = top_of(top, load_piece(row, i, p.C));
  top = __reduce_max_sync(0xffffffffu, max(top & 0xffff, top >> 16));
  if (W > 1) {
    if (lane == 0) tops[warp] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < W; k++) top = max(top, tops[warp / W * W + k]);
  }
  if (!live) return;
  // a row with an infinity or a NaN: codes of zero and a scale of NaN, which spoil its row of every product
  const bool finite = top < (DT == WINDQ_F16 ? 0x7c00u : 0x7f80u);
  const float a = finite ? unpack2(top, DT).x : 0.0f;
  const bool lift = DT == WINDQ_BF16 && a < 0x1p-60f;
  const float scale = finite ? __fdiv_rn(a, 127.0f) : __uint_as_float(0x7fffffffu);
  const float inv = a > 0.0f ? __fdiv_rn(127.0f, lift ? a * 0x1p60f : a) : 0.0f;
  if (first == 0) p.scale[t] = scale;
  int8_t* q = p.q + t * p.ldq;
  uint16_t* out = VALUES ? p.values + t * p.ldv : nullptr;
  auto write = [&](int i, uint4 v) {
    uint2 codes;
    uint4 values = make_uint4(0, 0, 0, 0);
    if (!finite) v = make_uint4(0, 0, 0, 0);
    if (lift) encode<DT, VALUES, true>(v, inv, scale, codes, values);
    else encode<DT, VALUES, false>(v, inv, scale, codes, values);
    if (i * 8 + 8 <= p.C) {
      reinterpret_cast<uint2*>(q)[i] = codes;
      if (VALUES) reinterpret_cast<uint4*>(out)[i] = values;
    } else {
      const uint32_t o[4] = {values.x, values.y, values.z, values.w};
      for (int k = 0; i * 8 + k < p.C; k++) {
        q[i * 8 + k] = (int8_t)((k < 4 ? codes.x : codes.y) >> (8 * (k & 3)));
        if (VALUES) out[i * 8 + k] = (uint16_t)(o[k >> 1] >> (16 * (k & 1)));
      }
    }
  };
#pragma unroll
  for (int k = 0; k < kHeld; k++)
    if (first + k * step < pieces) write(first + k * step, held[k]);
  for (int i = first + kHeld * step; i < pieces; i += step) write(i, load_piece(row, i, p.C));
}

template <int DT, int W>
cudaError_t launch(const QuantizeArgs& p, cudaStream_t st) {
  const int64_t rows = kThreads / 32 / W;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attrs[2];
  overlapped_launch(cfg, attrs, (int)((p.T + rows - 1) / rows), kThreads, 1, 0, st);
  return p.values ? cudaLaunchKernelEx(&cfg, quantize_kernel<DT, W, true>, p) : cudaLaunchKernelEx(&cfg, quantize_kernel<DT, W, false>, p);
}
template <int DT>
cudaError_t launch(const QuantizeArgs& p, int warps, cudaStream_t st) {
  switch (warps) {
    case 1: return launch<DT, 1>(p, st);
    case 2: return launch<DT, 2>(p, st);
    case 4: return launch<DT, 4>(p, st);
    default: return launch<DT, 8>(p, st);
  }
}

}  // namespace
}  // namespace windq

extern "C" windq_status windq_quantize_rows(windq_ctx* ctx, int dtype, const void* X, int64_t T, int64_t C, int64_t ldx,
                                            int8_t* codes_out, int64_t ldq, float* scale_out, void* values_out, int64_t ldv,
                                            void* stream) {
  using namespace windq;
  const char* who = "windq_quantize_rows";
  if (!ctx) return fail(nullptr, WINDQ_ERR_NULL, "%s: ctx is NULL", who);
  WINDQ_REQUIRE(ctx, dtype == WINDQ_F16 || dtype == WINDQ_BF16, WINDQ_ERR_ARG, "%s: dtype = %d is neither fp16 nor bf16", who, dtype);
  WINDQ_REQUIRE(ctx, T >= 0 && T < (1ll << 31) - 256, WINDQ_ERR_SHAPE, "%s: T = %lld", who, (long long)T);
  WINDQ_REQUIRE(ctx, C > 0 && C < (1ll << 31) - (1 << 20), WINDQ_ERR_SHAPE, "%s: C = %lld", who, (long long)C);
  WINDQ_REQUIRE(ctx, T == 0 || (X && codes_out && scale_out), WINDQ_ERR_NULL, "%s: X, codes_out or scale_out is NULL", who);
  WINDQ_REQUIRE(ctx, ldx >= C && ldq >= C && (!values_out || ldv >= C), WINDQ_ERR_SHAPE, "%s: ldx = %lld, ldq = %lld or ldv = %lld is below C = %lld",
                who, (long long)ldx, (long long)ldq, (long long)ldv, (long long)C);
  WINDQ_REQUIRE(ctx, ldx % 8 == 0 && ldq % 16 == 0 && (!values_out || ldv % 8 == 0), WINDQ_ERR_ALIGN,
                "%s: ldx = %lld or ldv = %lld is not a multiple of 8, or ldq = %lld of 16", who, (long long)ldx, (long long)ldv, (long long)ldq);
  WINDQ_REQUIRE(ctx, aligned16(X) && aligned16(codes_out) && aligned16(values_out), WINDQ_ERR_ALIGN,
                "%s: X, codes_out or values_out is not 16-byte aligned", who);
  WINDQ_REQUIRE(ctx, ((uintptr_t)scale_out & 3) == 0, WINDQ_ERR_ALIGN, "%s: scale_out is misaligned", who);
  if (T == 0) return WINDQ_OK;
  DeviceGuard guard(ctx->device);
  QuantizeArgs p = {(const uint16_t*)X, T, ldx, (int)C, codes_out, ldq, scale_out, (uint16_t*)values_out, ldv};
  int warps = 1;
  while (warps < 8 && (C > warps * 32 * 8 * kHeld || (T * warps < ctx->sm_count * 16 && C > warps * 32 * 8))) warps *= 2;
  WINDQ_CUDA(ctx, dtype == WINDQ_F16 ? launch<WINDQ_F16>(p, warps, (cudaStream_t)stream) : launch<WINDQ_BF16>(p, warps, (cudaStream_t)stream));
  return WINDQ_OK;
}
