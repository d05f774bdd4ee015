// What follows a dense product: Z = product + bias, Y = act(Z) + residual, rounded once (include/hinm.h, hinm_linear).
#pragma once

#include "activations.h"
#include "eight_values.h"

namespace hinm {

struct LinearEpilogue {
  int M, N;  // of the result
  const float* bias;
  const uint16_t* residual;
  int64_t ldr;
  Pieces residual_rows;
  uint16_t* Z;
  void* Y;
  int64_t ldy;  // of Z and Y
  int act;
  bool out_f32;  // Y holds the float32 values themselves
};

// Eight consecutive columns of row m from n on, `left` >= 1 of them in the row, from their sums.  `r`: the residual's eight as
// load_residual left them; apart, so that the load is under way before the sums are.
template <int DT>
__device__ __forceinline__ u32x4 load_residual(const LinearEpilogue& e, int m, int n, int left) {
  return e.residual ? draw_eight(e.residual + m * e.ldr + n, left, e.residual_rows) : u32x4{0, 0, 0, 0};
}
template <int DT>
__device__ __forceinline__ void finish_eight(const LinearEpilogue& e, int m, int n, int left, float bias, u32x4 r, float (&v)[8]) {
  const int64_t at = m * e.ldy + n;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] += bias;
  if (e.Z) {
    u32x4 z;
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = floats_to_bits<DT>(v[2 * j], v[2 * j + 1]);
    store_eight(e.Z + at, z, left);
  }
  activate(v, e.act);
  if (e.residual) {
    r = place_eight(r, left, e.residual_rows);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] += low_half<DT>(r[j]);
      v[2 * j + 1] += high_half<DT>(r[j]);
    }
  }
  if (e.out_f32) {
    float* to = static_cast<float*>(e.Y) + at;
    if (left >= 8) {
      *reinterpret_cast<u32x4_a4*>(to) = __builtin_bit_cast(u32x4, (f32x4{v[0], v[1], v[2], v[3]}));
      *reinterpret_cast<u32x4_a4*>(to + 4) = __builtin_bit_cast(u32x4, (f32x4{v[4], v[5], v[6], v[7]}));
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) to[j] = v[j];
    return;
  }
  u32x4 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = floats_to_bits<DT>(v[2 * j], v[2 * j + 1]);
  store_eight(static_cast<uint16_t*>(e.Y) + at, y, left);
}

}  // namespace hinm
