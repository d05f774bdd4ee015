// Microscaled 4-bit form (include/hinm.h): where codes and scales lie, and the conversions in both directions.
//
// 32 consecutive values share the power of two 2^(e - 127) (e = scale byte); a code is a sign and a place in
// 0, .5, 1, 1.5, 2, 3, 4, 6.  Lines of 256 values = 128 bytes of codes and groups of 512 values = 16 scale bytes come first
// in the order, rows second: what a workgroup takes of neighbouring rows at one place of the summed axis is one contiguous
// piece.  (Rows after one another instead: a group's scale bytes of 256 rows lay in 256 cache lines, which were fetched again
// for every group.)  Byte 4 b + s of a group's scales belongs to block 4 s + b.
//
// Operand layout of the scaled matrix instructions on 4-bit values, established on MI355X with random codes and scales:
// lane l of the 16x16x128 form holds row l % 16 and the 32 values of block l / 16, in order, low nibble first; of the
// 32x32x64 form row l % 32 and block l / 32.  One byte of its scale register (chosen per instruction) scales the
// lane's 32 values; 255 makes a result NaN whatever the codes.  D: lane l holds column l % 16, rows 4 (l / 16) + register
// (16x16), or column l % 32, rows 8 (register / 4) + 4 (l / 32) + register % 4 (32x32).  Which 32 values meet is
// free as long as both operands agree: with the scale bytes in the order above a lane's 4-byte word serves four k-steps of
// the 16x16x128 form (block 4 s + lane / 16 in step s), and two words serve eight instructions of the 32x32x64 form.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eight_values.h"

namespace hinm {

constexpr int kMx4Step = 128;    // values of a 16x16x128 instruction: 64 bytes of codes
constexpr int kMx4Line = 256;    // values of a line of codes
constexpr int kMx4Group = 512;   // values whose 16 scale bytes lie together

__host__ __device__ constexpr int mx4_lines(int length) { return (int)(((int64_t)length + 255) / 256); }
__host__ __device__ constexpr int mx4_groups(int length) { return (int)(((int64_t)length + 511) / 512); }
__host__ __device__ constexpr int64_t mx4_code_bytes(int rows, int length) { return (int64_t)mx4_lines(length) * rows * 128; }
__host__ __device__ constexpr int64_t mx4_scale_bytes(int rows, int length) { return (int64_t)mx4_groups(length) * rows * 16; }
// where a row's line of codes and its group of scales begin
__host__ __device__ constexpr int64_t mx4_line_at(int line, int rows, int64_t row) { return ((int64_t)line * rows + row) * 128; }
__host__ __device__ constexpr int64_t mx4_group_at(int group, int rows, int64_t row) { return ((int64_t)group * rows + row) * 16; }
// of block j among its group's 16
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

}  // namespace hinm
