// Microscaled 4-bit form (include/hinm.h): where codes and scales lie, and the conversions in both directions.
//
// 32 consecutive values share the power of two 2^(e - 127) (e = scale byte); a code is a sign and a place in
// 0, .5, 1, 1.5, 2, 3, 4, 6.  The form lies in memory as the scaled 32x32x64 matrix instruction takes it: 32 rows x 64 values
// are 1 KB, lane after lane, so that every kernel reads operands in whole contiguous kilobytes, through LDS or straight into
// registers.
//
// Operand layout of the instruction on 4-bit values, established on MI355X with random codes and scales: lane l holds row
// l % 32 and 32 values of block l / 32, in order, low nibble first; one byte of its scale register (chosen per instruction)
// scales them; 255 makes a result NaN whatever the codes.  D: lane l holds column l % 32, rows 8 (register / 4) +
// 4 (l / 32) + register % 4.  Which two blocks of a row an instruction takes is free as long as both operands agree.  Here a
// line of 256 values = 8 blocks is four instructions, instruction i = 0..3 taking blocks 4 (i / 2) + i % 2 (lower lanes) and 2
// further (upper lanes); 16 scale bytes of 512 values lie so that word q of a lane's two holds the bytes of its blocks in
// instructions with i % 2 = q: byte i / 2 in the first line, 2 + i / 2 in the second.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eight_values.h"

namespace hinm {

constexpr int kMx4Line = 256;    // values of a row in a line: 128 bytes of codes
constexpr int kMx4Group = 512;   // values whose 16 scale bytes lie together
constexpr int kMx4Rows = 32;     // rows of a block of rows
constexpr int kMx4BlockBytes = kMx4Rows * 128;  // of a line

__host__ __device__ constexpr int mx4_lines(int length) { return (int)(((int64_t)length + 255) / 256); }
__host__ __device__ constexpr int mx4_groups(int length) { return (int)(((int64_t)length + 511) / 512); }
__host__ __device__ constexpr int mx4_row_blocks(int rows) { return (int)(((int64_t)rows + 31) / 32); }
__host__ __device__ constexpr int64_t mx4_code_bytes(int rows, int length) {
  return (int64_t)mx4_lines(length) * mx4_row_blocks(rows) * kMx4BlockBytes;
}
__host__ __device__ constexpr int64_t mx4_scale_bytes(int rows, int length) {
  return (int64_t)mx4_groups(length) * mx4_row_blocks(rows) * (kMx4Rows * 16);
}
// where a block of rows begins in a line of codes and in a group of scales
__host__ __device__ constexpr int64_t mx4_codes_at(int line, int row_blocks, int block) {
  return ((int64_t)line * row_blocks + block) * kMx4BlockBytes;
}
__host__ __device__ constexpr int64_t mx4_scales_at(int group, int row_blocks, int block) {
  return ((int64_t)group * row_blocks + block) * (kMx4Rows * 16);
}
// which 512 bytes (16 of each of 32 rows) of a line's block of rows hold block p = 0..7 of 32 values
__host__ __device__ constexpr int mx4_chunk_of(int p) { return 2 * (2 * (p >> 2) + (p & 1)) + ((p >> 1) & 1); }
// place of the scale byte of block j = 0..15 of a group
__host__ __device__ constexpr int mx4_scale_place(int j) { return 4 * (j & 3) + (j >> 2); }

// Larger of the magnitudes in both halves (sign bits cleared): 16-bit formats order like their bit patterns, NaN highest.
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Scale byte of a block whose largest magnitude is the given pattern: its binary exponent less two, clamped at the bottom;
// 255 for infinities and NaN.
template <int DT>
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t magnitude) {
  const uint32_t e = __builtin_bit_cast(uint32_t, bits_to_float<DT>((uint16_t)magnitude)) >> 23;
  return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}
// What a value is multiplied with before it is rounded to a code: 2^(127 - e), a normal number for every finite block.
__device__ __forceinline__ float mx4_inverse_scale(uint32_t e) { return __builtin_bit_cast(float, (254u - e) << 23); }
// ... and a code's value after: 2^(e - 127).
__device__ __forceinline__ float mx4_scale_value(uint32_t e) {
  return __builtin_bit_cast(float, e == 255 ? 0x7fc00000u : e == 0 ? 0x00400000u : e << 23);
}

// ... of both halves with those of another lane of the row of 16, which the control word names.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with_lane(uint32_t m) {
  return max_halves(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true));
}

}  // namespace hinm
