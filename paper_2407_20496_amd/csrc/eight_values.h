// Pieces of eight consecutive 16-bit values of a row, whole or cut short at the row's end.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hinm_internal.h"
#include "mfma_types.h"

namespace hinm {

// How the pieces of a matrix's rows are read and written.  Any address does for the hardware's 16 bytes; only a row's end asks
// for care, as nothing beyond it may be touched unless it lies in the same aligned 16 bytes, hence in the same page.
enum Pieces {
  kAligned,   // every piece begins at a multiple of 16 bytes: a row's end is read whole
  kAnywhere,  // a row's end is read as the eight values that end there, and shifted
  kFew,       // rows of fewer than eight values: one by one
};
inline Pieces pieces_of_rows(const void* p, int64_t ld, int cols) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 ? kAligned : cols >= 8 ? kAnywhere : kFew;
}
// ... of two matrices that one rule serves
inline Pieces lesser(Pieces a, Pieces b) { return a > b ? a : b; }

// Eight consecutive 16-bit values as they are read, `valid` >= 1 of them in the row; place_eight or trim_eight has to
// follow.  Apart, so that no load waits for the one before it.
__device__ __forceinline__ u32x4 draw_eight(const uint16_t* p, int valid, Pieces rows) {
  if (rows != kFew) return *reinterpret_cast<const u32x4_a2*>(p - (rows == kAnywhere ? max(8 - valid, 0) : 0));
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (j < valid) v[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
  return v;
}
// The values in the row at their places; what stands behind them is anything.
__device__ __forceinline__ u32x4 place_eight(u32x4 v, int valid, Pieces rows) {
  if (valid >= 8 || rows != kAnywhere) return v;
  const int back = 8 - valid;
  if (back & 4) v = u32x4{v[2], v[3], 0, 0};
  if (back & 2) v = u32x4{v[1], v[2], v[3], 0};
  if (back & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  return v;
}
// ... and zero behind them
__device__ __forceinline__ u32x4 trim_eight(u32x4 v, int valid, Pieces rows) {
  if (valid >= 8 || rows != kAligned) return place_eight(v, valid, rows);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] &= valid >= 2 * j + 2 ? 0xffffffffu : valid == 2 * j + 1 ? 0xffffu : 0u;
  return v;
}
// PAST: whole pieces go around the caches (for rows of whole cache lines).  A template parameter: of two stores that differ in
// this alone the compiler keeps one.
template <bool PAST = false>
__device__ __forceinline__ void store_eight(uint16_t* p, u32x4 v, int valid) {
  if (valid >= 8) {
    if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4_a2*>(p) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {  // a row's end: pairs, and the last one if it has none
    if (valid >= 2 * j + 2) *reinterpret_cast<u32_a2*>(p + 2 * j) = v[j];
    else if (valid == 2 * j + 1) p[2 * j] = (uint16_t)v[j];
  }
}

// The two values of a word.
template <int DT>
__device__ __forceinline__ float low_half(uint32_t w) { return bits_to_float<DT>((uint16_t)w); }
template <int DT>
__device__ __forceinline__ float high_half(uint32_t w) {
  if constexpr (DT == HINM_BF16) return __builtin_bit_cast(float, w & 0xffff0000u);
  return bits_to_float<DT>((uint16_t)(w >> 16));
}

}  // namespace hinm
