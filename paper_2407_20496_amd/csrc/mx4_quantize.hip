// 16-bit matrices to the microscaled 4-bit form and back (include/hinm.h, mx4_form.h).
//
// A block's scale needs the largest of 32 magnitudes, its codes one multiplication by a power of two (exact) and the
// hardware's conversion (nearest, ties to the even code, beyond 6 to 6) a value: 2 bytes in and 17/32 out, bound by memory.
#include "mx4_form.h"

namespace hinm {

namespace {

constexpr int kThreads = 256;

template <int CTRL>
__device__ __forceinline__ uint32_t max_with_lane(uint32_t m) {
  return max_halves(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true));
}

// ---- blocks along the rows --------------------------------------------------------------------------
// A wave takes 512 consecutive values of a row (eight a lane, four lanes a block): one contiguous kilobyte in, two lines of
// codes and the group's 16 scale bytes out.
template <int DT>
__global__ __launch_bounds__(kThreads) void mx4_rows_kernel(const uint16_t* src, int64_t ld, int rows, int cols, bool vec,
                                                            uint8_t* codes, uint8_t* scales) {
  const int lane = threadIdx.x & 63;
  const int groups = (cols + kMx4Group - 1) / kMx4Group;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (item >= (int64_t)rows * groups) return;
  const int64_t row = item / groups;
  const int g = (int)(item - row * groups);
  const int k = g * kMx4Group + 8 * lane;
  const u32x4 v = k < cols ? load_eight(src + row * ld + k, cols - k, vec) : u32x4{0, 0, 0, 0};
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) m = max_halves(m, v[j] & 0x7fff7fffu);
  m = max_with_lane<0xB1>(m);  // lane ^ 1
  m = max_with_lane<0x4E>(m);  // lane ^ 2
  m = max_halves(m, m >> 16) & 0xffffu;
  const bool beyond = (k & ~31) >= cols;
  const uint32_t e = mx4_scale_of<DT>(m);
  const float s = mx4_inverse_scale(e);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[0]) * s, high_half<DT>(v[0]) * s, 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[1]) * s, high_half<DT>(v[1]) * s, 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[2]) * s, high_half<DT>(v[2]) * s, 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[3]) * s, high_half<DT>(v[3]) * s, 1.0f, 3);
  if (e == 255) c = 0;
  const int line = 2 * g + (lane >> 5);
  if (line < mx4_lines(cols)) *reinterpret_cast<uint32_t*>(codes + mx4_line_at(line, rows, row) + 4 * (lane & 31)) = c;
  if ((lane & 3) == 0) scales[mx4_group_at(g, rows, row) + mx4_scale_place(lane >> 2)] = (uint8_t)(beyond ? 127 : e);
}

// ---- blocks down the columns ------------------------------------------------------------------------
// A workgroup takes 64 columns x 512 rows.  A wave reads a block's 32 rows in four loads of eight 128-byte segments: lane l
// holds columns 8 (l % 8) .. + 7 of rows 4 (l / 8) .. + 3, so it has two bytes of codes for each of its columns.  They
// meet in LDS and leave as two runs of 8 KB.
constexpr int kTileCols = 64;
constexpr int kColumnPitch = 256 + 16;  // bytes of a column's codes in LDS: the pad spreads the columns over the banks

template <int DT>
__global__ __launch_bounds__(kThreads) void mx4_columns_kernel(const uint16_t* src, int64_t ld, int rows, int cols, bool vec,
                                                               uint8_t* codes, uint8_t* scales) {
  __shared__ __align__(16) uint8_t tile[kTileCols * kColumnPitch];
  __shared__ __align__(16) uint8_t tile_scales[kTileCols * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tiles = (cols + kTileCols - 1) / kTileCols;
  const int g = blockIdx.x / tiles;
  const int n0 = (blockIdx.x - g * tiles) * kTileCols;
  const int c8 = lane & 7, rg = lane >> 3;
  const int n = n0 + 8 * c8;
  u32x4 v[4][4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int k = g * kMx4Group + 32 * (wave + 4 * q) + 4 * rg;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[q][i] = (k + i < rows && n < cols) ? load_eight(src + (int64_t)(k + i) * ld + n, cols - n, vec) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int block = wave + 4 * q;
    const bool beyond = g * kMx4Group + 32 * block >= rows;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max_halves(m, v[q][i][w] & 0x7fff7fffu);
      m = max_with_lane<0x128>(m);  // lane ^ 8
      m = max_halves(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max_halves(m, (uint32_t)__shfl_xor((int)m, 32));
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t e = mx4_scale_of<DT>(half ? m >> 16 : m & 0xffffu);
        const float s = mx4_inverse_scale(e);
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (half ? high_half<DT>(v[q][i][w]) : low_half<DT>(v[q][i][w])) * s;
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], 1.0f, 1);
        if (e == 255) c = 0;
        const int col = 8 * c8 + 2 * w + half;
        *reinterpret_cast<uint16_t*>(tile + col * kColumnPitch + 16 * block + 2 * rg) = (uint16_t)c;
        if (rg == 0) tile_scales[16 * col + mx4_scale_place(block)] = (uint8_t)(beyond ? 127 : e);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int piece = threadIdx.x + kThreads * q;  // of 2 lines x 64 columns x 8
    const int line = 2 * g + (piece >> 9), col = (piece >> 3) & 63, at = 16 * (piece & 7);
    if (n0 + col < cols && line < mx4_lines(rows))
      *reinterpret_cast<u32x4*>(codes + mx4_line_at(line, cols, n0 + col) + at) =
          *reinterpret_cast<const u32x4*>(tile + col * kColumnPitch + 128 * (piece >> 9) + at);
  }
  if (threadIdx.x < kTileCols && n0 + (int)threadIdx.x < cols)
    *reinterpret_cast<u32x4*>(scales + mx4_group_at(g, cols, n0 + threadIdx.x)) =
        *reinterpret_cast<const u32x4*>(tile_scales + 16 * threadIdx.x);
}

// ---- back -------------------------------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(kThreads) void mx4_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int rows, int length,
                                                              uint16_t* dst, int64_t ld, bool vec) {
  const int lane = threadIdx.x & 63;
  const int groups = (length + kMx4Group - 1) / kMx4Group;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (item >= (int64_t)rows * groups) return;
  const int64_t row = item / groups;
  const int g = (int)(item - row * groups);
  const int k = g * kMx4Group + 8 * lane;
  if (k >= length) return;
  const uint32_t c = *reinterpret_cast<const uint32_t*>(codes + mx4_line_at(2 * g + (lane >> 5), rows, row) + 4 * (lane & 31));
  const float s = mx4_scale_value(scales[mx4_group_at(g, rows, row) + mx4_scale_place(lane >> 2)]);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
  u32x4 out;
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = floats_to_bits<DT>(f[j][0] * s, f[j][1] * s);
  store_eight(dst + row * ld + k, out, length - k, vec);
}

}  // namespace

hipError_t launch_mx4_quantize(int rows, int cols, int dtype, const void* src, int64_t ld, bool columns, uint8_t* codes,
                               uint8_t* scales, hipStream_t stream) {
  // one column without a stride is one row
  if (columns && cols == 1 && ld == 1) return launch_mx4_quantize(1, rows, dtype, src, rows, false, codes, scales, stream);
  const uint16_t* p = static_cast<const uint16_t*>(src);
  const bool vec = rows_in_pieces(src, ld) || (rows == 1 && (reinterpret_cast<uintptr_t>(src) & 15) == 0);
  if (columns) {
    const int64_t tiles = (cols + kTileCols - 1) / kTileCols, groups = (rows + kMx4Group - 1) / kMx4Group;
    const dim3 grid((uint32_t)(tiles * groups));
    if (dtype == HINM_F16) mx4_columns_kernel<HINM_F16><<<grid, kThreads, 0, stream>>>(p, ld, rows, cols, vec, codes, scales);
    else mx4_columns_kernel<HINM_BF16><<<grid, kThreads, 0, stream>>>(p, ld, rows, cols, vec, codes, scales);
  } else {
    const int64_t items = (int64_t)rows * ((cols + kMx4Group - 1) / kMx4Group);
    const dim3 grid((uint32_t)((items + kThreads / 64 - 1) / (kThreads / 64)));
    if (dtype == HINM_F16) mx4_rows_kernel<HINM_F16><<<grid, kThreads, 0, stream>>>(p, ld, rows, cols, vec, codes, scales);
    else mx4_rows_kernel<HINM_BF16><<<grid, kThreads, 0, stream>>>(p, ld, rows, cols, vec, codes, scales);
  }
  return hipGetLastError();
}

hipError_t launch_mx4_unpack(int rows, int length, int dtype, const uint8_t* codes, const uint8_t* scales, void* dst, int64_t ld,
                             hipStream_t stream) {
  const int64_t items = (int64_t)rows * ((length + kMx4Group - 1) / kMx4Group);
  const dim3 grid((uint32_t)((items + kThreads / 64 - 1) / (kThreads / 64)));
  uint16_t* p = static_cast<uint16_t*>(dst);
  const bool vec = rows_in_pieces(dst, ld);
  if (dtype == HINM_F16) mx4_unpack_kernel<HINM_F16><<<grid, kThreads, 0, stream>>>(codes, scales, rows, length, p, ld, vec);
  else mx4_unpack_kernel<HINM_BF16><<<grid, kThreads, 0, stream>>>(codes, scales, rows, length, p, ld, vec);
  return hipGetLastError();
}

}  // namespace hinm
