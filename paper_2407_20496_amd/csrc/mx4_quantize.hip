// 16-bit matrices to the microscaled 4-bit form and back (include/hinm.h, mx4_form.h).
//
// A block's scale needs the largest of 32 magnitudes, its codes one multiplication by a power of two (exact) and the
// hardware's conversion (nearest, ties to the even code, beyond 6 to 6) a value: 2 bytes in and 17/32 out, bound by memory.
// A workgroup takes what becomes whole 4 KB blocks of the form, puts the codes together in LDS and writes them contiguously.
// bf16, sources that lie in memory, reading 2 and writing 17/32 bytes a value: 11008x4096 along the rows 22.7 us (5.0 TB/s, a
// large copy 4.8), down the columns 24.0 (4.8), back 24 (4.8); 4096x4096 10.6 and 11.3; rows at odd addresses (11008x4095)
// 23 along the rows and 31 back.  Below some 4096x1000 a launch is most of it: 256x256 3.4.
#include "mx4_form.h"

namespace hinm {

namespace {

constexpr int kThreads = 256;
// A 512-byte chunk of a block of rows takes 528 bytes in LDS: codes of one row lie in one place of every chunk, and without
// the pad all of them would fall on the same banks.
constexpr int kChunkPitch = 512 + 16;

// Workgroups that share cache lines of the source (rows that do not begin at multiples of 128 bytes) run on one XCD, in
// contiguous runs of the list; otherwise neighbours of the list run side by side (down the columns 11008x1571 14.3 -> 12.4 us and
// 11008x4095 30.9 -> 24.9 in runs; whole lines, 11008x4096 along the rows, 22.7 -> 23.4).
__device__ __forceinline__ int item_of_workgroup(bool whole_lines) {
  return whole_lines ? (int)blockIdx.x : (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
}

// ---- blocks along the rows --------------------------------------------------------------------------
// A workgroup takes 32 rows x 256 values, a line of a block of rows; a wave eight rows in four loads of two rows each, a lane
// eight values, four lanes a block.
template <int DT>
__global__ __launch_bounds__(kThreads) void mx4_rows_kernel(const uint16_t* src, int64_t ld, int rows, int cols, Pieces pieces,
                                                            bool whole_lines, uint8_t* codes, uint8_t* scales) {
  __shared__ __align__(16) uint8_t tile[8 * kChunkPitch];
  __shared__ __align__(16) uint8_t tile_scales[kMx4Rows][8];  // byte 2 (p % 4) + p / 4 of block p
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lines = mx4_lines(cols), blocks = mx4_row_blocks(rows);
  const int item = item_of_workgroup(whole_lines);
  const int rb = item / lines, line = item - rb * lines;
  if (rb >= blocks) return;
  const int in_line = 8 * (lane & 31), k = line * kMx4Line + in_line, p = in_line >> 5;
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = rb * kMx4Rows + 8 * wave + 2 * i + (lane >> 5);
    v[i] = r < rows && k < cols ? draw_eight(src + (int64_t)r * ld + k, cols - k, pieces) : u32x4{0, 0, 0, 0};
  }
  const bool beyond = (k & ~31) >= cols;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = trim_eight(v[i], cols - k, pieces);
    const int r = 8 * wave + 2 * i + (lane >> 5);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max_halves(m, v[i][j] & 0x7fff7fffu);
    m = max_with_lane<0xB1>(m);  // lane ^ 1
    m = max_with_lane<0x4E>(m);  // lane ^ 2
    m = max_halves(m, m >> 16) & 0xffffu;
    const uint32_t e = mx4_scale_of<DT>(m);
    const float s = mx4_inverse_scale(e);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[i][0]) * s, high_half<DT>(v[i][0]) * s, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[i][1]) * s, high_half<DT>(v[i][1]) * s, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[i][2]) * s, high_half<DT>(v[i][2]) * s, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(v[i][3]) * s, high_half<DT>(v[i][3]) * s, 1.0f, 3);
    if (e == 255) c = 0;
    *reinterpret_cast<uint32_t*>(tile + mx4_chunk_of(p) * kChunkPitch + 16 * r + 4 * (lane & 3)) = c;
    if ((lane & 3) == 0) tile_scales[r][2 * (p & 3) + (p >> 2)] = (uint8_t)(beyond ? 127 : e);
  }
  __syncthreads();
  const int here = min(kMx4Rows, rows - rb * kMx4Rows), r = threadIdx.x & 31;
  if (r >= here) return;
  *reinterpret_cast<u32x4*>(codes + mx4_codes_at(line, blocks, rb) + 16 * threadIdx.x) =
      *reinterpret_cast<const u32x4*>(tile + (threadIdx.x >> 5) * kChunkPitch + 16 * r);
  // two bytes of each of four words; a group's last line writes the absent one's too
  const int word = threadIdx.x >> 5;
  if (word >= 4) return;
  uint8_t* to = scales + mx4_scales_at(line >> 1, blocks, rb) + 16 * r + 4 * word;
  const uint16_t bytes = *reinterpret_cast<const uint16_t*>(&tile_scales[r][2 * word]);
  if (line & 1) *reinterpret_cast<uint16_t*>(to + 2) = bytes;
  else if (line == lines - 1) *reinterpret_cast<uint32_t*>(to) = 0x7f7f0000u | bytes;
  else *reinterpret_cast<uint16_t*>(to) = bytes;
}

// ---- blocks down the columns ------------------------------------------------------------------------
// A workgroup takes 64 columns x 128 rows, half a line; a wave a block's 32 rows, in four loads of eight 128-byte segments: lane
// l holds columns 8 (l % 8) .. + 7 of rows 4 (l / 8) .. + 3, so it has two bytes of codes for each of its columns.  Small
// pieces: a workgroup reads, converts and writes one after the other, and with 512 rows each, all of them did so together
// (4096x4096: 15.2 us).
constexpr int kTileCols = 64, kTileRows = 128;

template <int DT>
__global__ __launch_bounds__(kThreads) void mx4_columns_kernel(const uint16_t* src, int64_t ld, int rows, int cols, Pieces pieces,
                                                               bool whole_lines, uint8_t* codes, uint8_t* scales) {
  __shared__ __align__(16) uint8_t tile[2][4 * kChunkPitch];  // two blocks of 32 columns
  __shared__ uint8_t tile_scales[4 * kTileCols];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tiles = (cols + kTileCols - 1) / kTileCols, blocks = mx4_row_blocks(cols), units = 2 * mx4_lines(rows);
  const int item = item_of_workgroup(whole_lines);
  const int unit = item / tiles, n0 = (item - unit * tiles) * kTileCols;
  if (unit >= units) return;
  const int c8 = lane & 7, rg = lane >> 3, n = n0 + 8 * c8, k0 = unit * kTileRows + 32 * wave, k = k0 + 4 * rg;
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = k + i < rows && n < cols ? draw_eight(src + (int64_t)(k + i) * ld + n, cols - n, pieces) : u32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = trim_eight(v[i], cols - n, pieces);
  const bool beyond = k0 >= rows;
  const int chunk = 2 * (wave & 1) + (wave >> 1);  // of block p = 4 (unit % 2) + wave, within the half line
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max_halves(m, v[i][w] & 0x7fff7fffu);
    m = max_with_lane<0x128>(m);  // lane ^ 8
    m = max_halves(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max_halves(m, (uint32_t)__shfl_xor((int)m, 32));
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t e = mx4_scale_of<DT>(half ? m >> 16 : m & 0xffffu);
      const float s = mx4_inverse_scale(e);
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = (half ? high_half<DT>(v[i][w]) : low_half<DT>(v[i][w])) * s;
      uint32_t c = 0;
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], 1.0f, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], 1.0f, 1);
      if (e == 255) c = 0;
      const int col = 8 * c8 + 2 * w + half;
      *reinterpret_cast<uint16_t*>(&tile[col >> 5][chunk * kChunkPitch + 16 * (col & 31) + 2 * rg]) = (uint16_t)c;
      if (rg == 2 * w + half) tile_scales[4 * col + wave] = (uint8_t)(beyond ? 127 : e);
    }
  }
  __syncthreads();
  // gathered first: written by the lanes that found them, eight at a time, these bytes cost a fifth of the kernel (11008x4096
  // 29.7 us for 24.0).  A byte of each of a column's four words; the last unit writes those of blocks that do not exist too
  const int col = threadIdx.x >> 2, step = unit & 3;
  if (n0 + col < cols) {
    uint8_t* to = scales + mx4_scales_at(unit >> 2, blocks, (n0 + col) >> 5) + 16 * (col & 31) + 4 * (threadIdx.x & 3) + step;
    to[0] = tile_scales[threadIdx.x];
    for (int q = 1; q <= (unit == units - 1 && step == 1 ? 2 : 0); ++q) to[q] = 127;
  }
  const int b = threadIdx.x >> 7, r = threadIdx.x & 31;
  if (n0 + 32 * b + r >= cols) return;
  *reinterpret_cast<u32x4*>(codes + mx4_codes_at(unit >> 1, blocks, n0 / 32 + b) + 2048 * (unit & 1) + 16 * (threadIdx.x & 127)) =
      *reinterpret_cast<const u32x4*>(&tile[b][((threadIdx.x >> 5) & 3) * kChunkPitch + 16 * r]);
}

// ---- back -------------------------------------------------------------------------------------------
// Byte of an LDS tile that holds block j = 0..15 (512 values) of row r in a block of rows.
__device__ __forceinline__ int lds_place(int j, int r) { return (8 * (j >> 3) + mx4_chunk_of(j & 7)) * kChunkPitch + 16 * r; }

template <int DT>
__global__ __launch_bounds__(kThreads) void mx4_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int rows, int length,
                                                              uint16_t* dst, int64_t ld) {
  __shared__ __align__(16) uint8_t tile[16 * kChunkPitch];
  __shared__ __align__(16) uint8_t tile_scales[kMx4Rows * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int groups = mx4_groups(length), blocks = mx4_row_blocks(rows);
  const int rb = blockIdx.x / groups, g = blockIdx.x - rb * groups;
  const int here = min(kMx4Rows, rows - rb * kMx4Rows);
  const int chunk = threadIdx.x >> 5, r = threadIdx.x & 31;
  if (r < here) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
      if (2 * g + q < mx4_lines(length))
        *reinterpret_cast<u32x4*>(tile + (8 * q + chunk) * kChunkPitch + 16 * r) =
            *reinterpret_cast<const u32x4*>(codes + mx4_codes_at(2 * g + q, blocks, rb) + 16 * threadIdx.x);
    if (chunk == 0)
      *reinterpret_cast<u32x4*>(tile_scales + 16 * r) = *reinterpret_cast<const u32x4*>(scales + mx4_scales_at(g, blocks, rb) + 16 * r);
  }
  __syncthreads();
  const int k = g * kMx4Group + 8 * lane;
  if (k >= length) return;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  for (int i = 8 * wave; i < min(8 * wave + 8, here); ++i) {
    const uint32_t c = *reinterpret_cast<const uint32_t*>(tile + lds_place(lane >> 2, i) + 4 * (lane & 3));
    const float s = mx4_scale_value(tile_scales[16 * i + mx4_scale_place(lane >> 2)]);
    const f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
    u32x4 out;
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = floats_to_bits<DT>(f[j][0] * s, f[j][1] * s);
    store_eight(dst + (int64_t)(rb * kMx4Rows + i) * ld + k, out, length - k);
  }
}

}  // namespace

hipError_t launch_mx4_quantize(int rows, int cols, int dtype, const void* src, int64_t ld, bool columns, uint8_t* codes,
                               uint8_t* scales, hipStream_t stream) {
  // one column without a stride is one row
  if (columns && cols == 1 && ld == 1) return launch_mx4_quantize(1, rows, dtype, src, rows, false, codes, scales, stream);
  const uint16_t* p = static_cast<const uint16_t*>(src);
  const Pieces pieces = pieces_of_rows(src, rows == 1 ? 8 : ld, cols);
  const bool whole_lines = (reinterpret_cast<uintptr_t>(src) & 127) == 0 && ld % 64 == 0;
  const int64_t items = columns ? (int64_t)((cols + kTileCols - 1) / kTileCols) * 2 * mx4_lines(rows)
                                : (int64_t)mx4_row_blocks(rows) * mx4_lines(cols);
  const dim3 grid((uint32_t)((items + 7) / 8 * 8));
  auto launch = [&](auto kernel) {
    kernel<<<grid, kThreads, 0, stream>>>(p, ld, rows, cols, pieces, whole_lines, codes, scales);
  };
  if (columns) launch(dtype == HINM_F16 ? mx4_columns_kernel<HINM_F16> : mx4_columns_kernel<HINM_BF16>);
  else launch(dtype == HINM_F16 ? mx4_rows_kernel<HINM_F16> : mx4_rows_kernel<HINM_BF16>);
  return hipGetLastError();
}

hipError_t launch_mx4_unpack(int rows, int length, int dtype, const uint8_t* codes, const uint8_t* scales, void* dst, int64_t ld,
                             hipStream_t stream) {
  const dim3 grid((uint32_t)((int64_t)mx4_row_blocks(rows) * mx4_groups(length)));
  uint16_t* p = static_cast<uint16_t*>(dst);
  if (dtype == HINM_F16) mx4_unpack_kernel<HINM_F16><<<grid, kThreads, 0, stream>>>(codes, scales, rows, length, p, ld);
  else mx4_unpack_kernel<HINM_BF16><<<grid, kThreads, 0, stream>>>(codes, scales, rows, length, p, ld);
  return hipGetLastError();
}

}  // namespace hinm
