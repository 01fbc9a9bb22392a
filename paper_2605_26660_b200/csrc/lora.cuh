// Declarations shared by the translation units of the adapter calls.
#pragma once

#include "typed.cuh"

namespace windq {

// O[t][n] = sum_k Z[t][k] W(n, k) + sum_j S[t][j] P[a](n, j), a = adapter_of[t]; S is already scaled.
//   forward:  Z = X,  W(n, k) = W[n][k], P[a](n, j) = B[a][n][j]     (k and j contiguous)
//   backward: Z = dY, W(n, k) = W[k][n], P[a](n, j) = A[a][j][n]     (n contiguous: transposed)
struct Projection {
  int dtype;
  bool transposed;
  const void* Z;
  int64_t T, K, N, ldz;
  const void* W;
  int64_t ldw;
  const void* P;
  int64_t n_adapters;
  int rank;
  const int32_t* adapter_of;
  const void* pair;  // S as launch_low_rank leaves it
  const int8_t* shift;
  const int* lists;  // see token_tile
  void* O;
  int64_t ldo;
};

// Rows of the token tiles of a projection over T tokens; the kernel that writes S also writes, for every tile, the
// adapters its tokens use: lists[tile * (rows + 1)] their number, then their indices.
int token_tile(int64_t T);
inline int64_t list_bytes(int64_t T) {
  const int64_t rows = token_tile(T);
  return round_up(4 * ((T + rows - 1) / rows) * (rows + 1), 256);
}

// S[t][j] = scaling[a] * sum_k Z[t][k] P[a](j, k): forward P[a](j, k) = A[a][j][k], backward (transposed) B[a][k][j].
// One or two of them for the same tokens.  Rows of tokens without an adapter are not written.
struct LowRankJob {
  bool transposed;
  const void* Z;
  int64_t K, ldz;
  const void* P;
  float* S;    // nullable
  void* pair;  // 16-bit [T][2][rank]: first and second term of S, for the projection; nullable
  // With pair, fp16: [T rounded up to 256], S of a token is kept as S * 2^shift (see shift_of).  bf16: NULL.
  int8_t* shift;
  float* top;  // fp32 [T], the largest |S[t][j]| of every token; nullable
};
struct LowRank {
  int dtype;
  int64_t T, n_adapters;
  int rank;
  const float* scaling;
  const int32_t* adapter_of;
  int* lists;  // nullable
  int jobs;
  LowRankJob job[2];
};
windq_status launch_low_rank(windq_ctx* ctx, const LowRank& q, cudaStream_t st);

// D[a] = sum over the tokens of a of S[t] (x) Z[t]; dA is [a][j][c], dB is [a][c][j].  Either may be NULL.
struct Gradient {
  const void* Z;
  int64_t cols, ldz;
  const float* S;
  const float* top;
  float* D;
};
windq_status launch_gradients(windq_ctx* ctx, const Gradient* dA, const Gradient* dB, int dtype, int64_t T, int rank,
                              int64_t n_adapters, const int32_t* adapter_of, cudaStream_t st);

constexpr int kProjectShare = 114 * 1024;  // shared memory of a thread block of the projection of few tokens, all told
windq_status launch_projection(windq_ctx* ctx, const Projection& q, cudaStream_t st);

}  // namespace windq
