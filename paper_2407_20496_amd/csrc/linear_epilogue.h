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

// A row's last columns go one by one, in loops that stay loops: a tile's code holds them for each of its pieces.
__device__ __forceinline__ u32x4 draw_piece(const uint16_t* p, int left, Pieces rows) {
  if (left >= 8 || rows == kAligned) return *reinterpret_cast<const u32x4_a2*>(p);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll 1
  for (int j = left - 1; j >= 0; --j) v = u32x4{v[0] << 16 | p[j], v[1] << 16 | v[0] >> 16, v[2] << 16 | v[1] >> 16, v[3] << 16 | v[2] >> 16};
  return v;
}
__device__ __forceinline__ void store_piece(uint16_t* p, u32x4 v, int left) {
  if (left >= 8) {
    *reinterpret_cast<u32x4_a2*>(p) = v;
    return;
  }
#pragma unroll 1
  for (int j = 0; j < left; ++j) {
    p[j] = (uint16_t)v[0];
    v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  }
}

// Eight consecutive columns of row m from n on, `left` >= 1 of them in the row, from their sums with the bias.  `r`: the
// residual's eight as draw_residual left them; apart, so that the load can be under way before the sums are there.
__device__ __forceinline__ u32x4 draw_residual(const LinearEpilogue& e, int m, int n, int left) {
  return draw_piece(e.residual + m * e.ldr + n, left, e.residual_rows);
}
// WHOLE: all eight exist, and the result is 16-bit.
template <int DT, Epilogue E, bool WHOLE>
__device__ __forceinline__ void finish_eight(const LinearEpilogue& e, int m, int n, int left, u32x4 r, float (&v)[8]) {
  const int64_t at = m * e.ldy + n;
  auto rounded = [&]() __attribute__((always_inline)) {
    return u32x4{floats_to_bits<DT>(v[0], v[1]), floats_to_bits<DT>(v[2], v[3]), floats_to_bits<DT>(v[4], v[5]), floats_to_bits<DT>(v[6], v[7])};
  };
  if constexpr (E != kEpiBare) {
    if (e.Z) store_piece(e.Z + at, rounded(), WHOLE ? 8 : left);
    activate<E>(v, e.act);
    if (e.residual) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] += low_half<DT>(r[j]);
        v[2 * j + 1] += high_half<DT>(r[j]);
      }
    }
  }
  if (WHOLE || !e.out_f32) {
    store_piece(static_cast<uint16_t*>(e.Y) + at, rounded(), WHOLE ? 8 : left);
    return;
  }
  float* const to = static_cast<float*>(e.Y) + at;
  if (left >= 8) {
    *reinterpret_cast<u32x4_a4*>(to) = __builtin_bit_cast(u32x4, (f32x4{v[0], v[1], v[2], v[3]}));
    *reinterpret_cast<u32x4_a4*>(to + 4) = __builtin_bit_cast(u32x4, (f32x4{v[4], v[5], v[6], v[7]}));
    return;
  }
#pragma unroll 1
  for (int j = 0; j < left; ++j) {
    to[j] = v[0];
#pragma unroll
    for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
  }
}

}  // namespace hinm
