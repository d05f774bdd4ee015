// Dense products of two 16-bit matrices: what the launchers of a layer's product and of its gradients share.
#pragma once

#include "hinm_internal.h"
#include "linear_epilogue.h"

namespace hinm {

// How an operand lies: the values that are summed over follow one another, or the ones that become rows or columns of the result.
enum OperandForm { kAlong, kAcross };

// result [M][N] = sum over K of a(m, k) b(k, n).  Operands along: a at A[m][k], b at B[n][k]; across: a at A[k][m], b at B[k][n].
struct DenseProduct {
  int M, N, K, dtype;
  OperandForm form_a, form_b;
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb;
  LinearEpilogue to;
  void* workspace;
  LaunchPlan* plan = nullptr;  // set: record what would be launched instead
};
inline bool is_layer(OperandForm form_a, OperandForm form_b) { return form_a == kAlong && form_b == kAcross; }
size_t dense_product_workspace_bytes(int M, int N, int K, OperandForm form_a, OperandForm form_b);  // a multiple of 256
hipError_t launch_dense_product(const DenseProduct& p, hipStream_t stream);
// Of one layer's gradients w is the product dW [M][K], x dX [K][N]: whether one launch of both is sooner than two.  That launch also sums
// the rows of w's A, as they are, to sums [M] unless it is NULL.
bool dense_pair_serves(const DenseProduct& w, const DenseProduct& x);
hipError_t launch_dense_pair(const DenseProduct& w, const DenseProduct& x, float* sums, hipStream_t stream);
// rows of any pitch and address to rows of `pitch` (a multiple of 8) from an aligned address on, zeros behind them
hipError_t launch_row_copy(const void* from, int64_t ld, void* to, int64_t pitch, int rows, int row, hipStream_t stream);
// a layer's product (A along, B across) on up to kFewTokens tokens
constexpr int kFewTokens = 16;
hipError_t launch_linear_few(const DenseProduct& p, hipStream_t stream);
// the weights' gradient (both along) of up to kOuterTokens
constexpr int kOuterTokens = 32;
inline bool is_outer(OperandForm form_a, OperandForm form_b, int K) { return form_a == kAlong && form_b == kAlong && K <= kOuterTokens; }
hipError_t launch_linear_outer(const DenseProduct& p, hipStream_t stream);

// dZ [M][ldz] = dY act'(Z), zero in columns from N on to the next multiple of 8 (ldz is one), and dbias [M] = its sums over N
// columns; either may be NULL.  Z NULL: no activation.
struct SlopeArgs {
  int M, N;
  const uint16_t *Z, *dY;
  int64_t ldy;  // of both
  Pieces rows;  // of both
  int act;
  uint16_t* dZ;
  int64_t ldz;
  float* dbias;
};
hipError_t launch_linear_slope(const SlopeArgs& a, int dtype, hipStream_t stream);

}  // namespace hinm
