// Declarations shared by the translation units of the feed-forward calls.
#pragma once

#include "typed.cuh"

namespace windq {

// act(g) = g s(y(g)) with the logistic function s; y(g) = g (silu) or 2 sqrt(2 / pi) (g + 0.044715 g^3), the tanh form of gelu.
constexpr float kGeluA = 1.5957691216057308f, kGeluB = 0.044715f;
__device__ __forceinline__ float gate_exponent(float g, int act) {
  return act == WINDQ_SILU ? g : kGeluA * fmaf(kGeluB * g * g, g, g);
}
// 1 / (1 + exp(-y)) from exp(-|y|), which cannot overflow.  Relative to the result the two fast functions are off by a few 2^-23
// and by |y| 2^-24 through the exponent's argument, far below the rounding to 16 bits that follows.
__device__ __forceinline__ float logistic(float y) {
  const float e = __expf(-fabsf(y));
  return __fdividef(y < 0.0f ? e : 1.0f, 1.0f + e);
}

// The power of two that the gradients of the two products are multiplied with before they are rounded to fp16 (and its
// inverse, for the products formed from them): their largest then is in [2^14, 2^15).  `top`: bits of the largest finite |value|.
__device__ __forceinline__ float gradient_power(uint32_t top, int sign) {
  if (top == 0) return 1.0f;
  const int shift = min(max(14 + 127 - (int)(top >> 23), -112), 112);
  return __uint_as_float((uint32_t)(127 + sign * shift) << 23);
}

// Tokens times weights, D(t, n) = sum_k X[t][k] W(n, k), and what follows:
//   kInt8        codes of tokens x codes of a weight: O = D * row_scale[t] * col_scale[n]
//   kInt8Gated   two weights: O = act(g) u, with g and u such products
//   kGated       the same of 16-bit tokens and weights; optionally g and u are stored too
//   kInputGrad   dX: D of the tokens x the two weights, transposed: W(n, k) = W[k][n].  D is [dG | dU], or, of two terms, [dG | dU |
//                what rounding took off dG | off dU]
enum ProductKind { kInt8, kInt8Gated, kGated, kInputGrad };

template <int KIND>
struct Kind {
  static constexpr bool kCodes = KIND == kInt8 || KIND == kInt8Gated, kGate = KIND == kInt8Gated || KIND == kGated;
  static constexpr bool kTransposed = KIND == kInputGrad;
  static constexpr int kStepK = kCodes ? 128 : 64;  // values of a chunk
};

// What an accumulator stands for.
template <bool CODES>
__device__ __forceinline__ float value_of(uint32_t acc, float row, float col) {
  if (CODES) return __int2float_rn((int)acc) * row * col;
  return __uint_as_float(acc) * row;
}
__device__ __forceinline__ float gated(float g, float u, int act) { return g * logistic(gate_exponent(g, act)) * u; }

struct Product {
  int kind, dtype, act;
  int64_t T, N, K;        // tokens, outputs, length of the sum (kInputGrad: of each of its two halves)
  const void* X;
  int64_t ldx;
  const void* W[2];
  int64_t ldw[2];
  int64_t half;           // kInputGrad: columns of dG in D, a multiple of 64
  int terms;              // kInputGrad: of D
  const float* row_scale;
  const float* col_scale[2];
  const uint32_t* top;    // fp16 gradients: see gradient_power; nullable
  void* O[3];             // the output; kGated: nullable, and g and u, nullable
  int64_t ldo[3];
  void* partials;         // product_scratch(T) bytes
};
windq_status launch_product(windq_ctx* ctx, const Product& q, cudaStream_t st);
int64_t product_scratch(int64_t T);
// The same for up to so many tokens, gated or not: see product_few.cu.
constexpr int64_t kMostFewGated = 128, kMostFew = 64;
windq_status launch_few_tokens(windq_ctx* ctx, const Product& q, cudaStream_t st);

// dWg = dG^T X, dWu = dU^T X from D, [T][terms * 2 * half].
struct WeightGradient {
  int dtype, terms;
  int64_t T, F, C, half;
  const void* D;
  const void* X;
  int64_t ldx;
  const uint32_t* top;
  void *dWg, *dWu;
  int64_t ldw;
};
windq_status launch_weight_gradient(windq_ctx* ctx, const WeightGradient& q, cudaStream_t st);

}  // namespace windq
