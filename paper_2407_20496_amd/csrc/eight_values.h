// Pieces of eight consecutive 16-bit values of a row, whole or cut short at the row's end.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hinm_internal.h"
#include "mfma_types.h"

namespace hinm {

// Eight consecutive 16-bit values; `valid` >= 1 of them exist, the rest reads as zero.  vec: the first is 16-byte aligned; then
// all eight are read whenever one exists (an aligned piece lies in one page) and those beyond are cleared.
__device__ __forceinline__ u32x4 load_eight(const uint16_t* p, int valid, bool vec) {
  u32x4 v = {0, 0, 0, 0};
  if (vec) {
    v = *reinterpret_cast<const u32x4*>(p);
    if (valid < 8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] &= valid >= 2 * j + 2 ? 0xffffffffu : valid == 2 * j + 1 ? 0xffffu : 0u;
    }
    return v;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < valid) v[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
  return v;
}
// PAST: whole pieces go around the caches (for rows of whole cache lines).  A template parameter: of two stores that differ in
// this alone the compiler keeps one.
template <bool PAST = false>
__device__ __forceinline__ void store_eight(uint16_t* p, u32x4 v, int valid, bool vec) {
  if (vec && valid >= 8) {
    if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = v;
    return;
  }
  if (vec) {  // a row's end: pairs, and the last one if it has none
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (valid >= 2 * j + 2) reinterpret_cast<uint32_t*>(p)[j] = v[j];
      else if (valid == 2 * j + 1) p[2 * j] = (uint16_t)v[j];
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < valid) p[j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
}

// The two values of a word.
template <int DT>
__device__ __forceinline__ float low_half(uint32_t w) { return bits_to_float<DT>((uint16_t)w); }
template <int DT>
__device__ __forceinline__ float high_half(uint32_t w) {
  if constexpr (DT == HINM_BF16) return __builtin_bit_cast(float, w & 0xffff0000u);
  return bits_to_float<DT>((uint16_t)(w >> 16));
}

// Whether every row of a matrix begins at a multiple of 16 bytes.
inline bool rows_in_pieces(const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0; }

}  // namespace hinm
