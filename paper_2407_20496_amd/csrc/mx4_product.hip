// Products of two matrices in microscaled 4-bit form, Y = A B^T, on the scaled matrix instructions (include/hinm.h).
#include "direct_lds.h"
#include "mx4_form.h"
#include "workgroup_items.h"

#include <type_traits>

namespace hinm {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// The instructions' register forms take 8 words; 4-bit operands use the first four.
__device__ __forceinline__ i32x8 operand(u32x4 v) {
  return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}
constexpr int kFp4 = 4;  // operand format code of 4-bit values
template <int BYTE_A, int BYTE_B = BYTE_A>
__device__ __forceinline__ f32x16 mfma_32x32x64(u32x4 a, uint32_t a_scale, u32x4 b, uint32_t b_scale, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, kFp4, kFp4, BYTE_A, (int)a_scale, BYTE_B,
                                                         (int)b_scale);
}

struct ProductShape {
  int M, N, K;
  int64_t ldy;
  bool relu;
};

// Four consecutive columns of a row of Y from n on, those below N, rounded.
template <int OUT>  // HINM_F16, HINM_BF16, 2 = float32
__device__ __forceinline__ void store_four(void* Y, int64_t row_at, int n, f32x4 v, const ProductShape& p) {
  if (p.relu) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] < 0 ? 0 : v[e];  // keeps NaN
  }
  if constexpr (OUT == 2) {
    float* to = static_cast<float*>(Y) + row_at + n;
    if (n + 4 <= p.N) {
      *reinterpret_cast<u32x4_a4*>(to) = __builtin_bit_cast(u32x4, v);
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < p.N) to[e] = v[e];
  } else {
    uint16_t* to = static_cast<uint16_t*>(Y) + row_at + n;
    const u32x2 w = {floats_to_bits<OUT>(v[0], v[1]), floats_to_bits<OUT>(v[2], v[3])};
    if (n + 4 <= p.N) {
      *reinterpret_cast<u32x2_a2*>(to) = w;
      return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < p.N) to[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
  }
}

// ---- operands straight into registers, the summed axis split over the waves ------------------------------
// A workgroup owns 32 WM rows of A times 32 WN rows of B; its waves take lines of 256 values in turn, each for the whole tile,
// with no barrier between them, and add their tiles in LDS in a fixed order.  The operands of a line are loaded while the
// line before it multiplies.  B is the instruction's row operand, so that a lane ends with four consecutive columns of Y.
//   Rows of B beyond N lie beyond the buffer descriptor's bytes for their lanes: they read as zero and cost no traffic.
//   Few columns are bound by A's 17/32 bytes a value, which every workgroup has under way at once: 4096x11008 of 16 columns
// 6.3 us (3.8 TB/s; 128 workgroups), 16384x11008 of 8, quantising included, 23 us (4.2 TB/s); more columns by what a compute unit
// draws from L2: 4096x4096 of 256 7.4 us.
constexpr int slab_pitch(int WN) { return 32 * WN + 4; }
template <int OUT, int WN, int WAVES>
__device__ __forceinline__ void add_slabs(const float (*slabs)[32 * slab_pitch(WN)], int count, int block_m, int block_n,
                                          void* Y, const ProductShape& p) {
  for (int t = threadIdx.x; t < 32 * 8 * WN; t += 64 * WAVES) {
    const int row = t / (8 * WN), at = 4 * (t % (8 * WN));
    const int m = 32 * block_m + row, n = 32 * block_n + at;
    if (m >= p.M || n >= p.N) continue;
    f32x4 v = *reinterpret_cast<const f32x4*>(slabs[0] + row * slab_pitch(WN) + at);
    for (int w = 1; w < count; ++w) v += *reinterpret_cast<const f32x4*>(slabs[w] + row * slab_pitch(WN) + at);
    store_four<OUT>(Y, (int64_t)m * p.ldy, n, v, p);
  }
}

template <int OUT, int WM, int WN, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 8 / WAVES) void mx4_stream_kernel(const uint8_t* a_codes, const uint8_t* a_scales,
                                                                           const uint8_t* b_codes, const uint8_t* b_scales,
                                                                           void* Y, ProductShape p) {
  constexpr int kPitch = slab_pitch(WN);
  __shared__ __align__(16) float slabs[WAVES][32 * kPitch];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks_a = mx4_row_blocks(p.M), blocks_b = mx4_row_blocks(p.N);
  const int tiles_m = (blocks_a + WM - 1) / WM, tiles_n = (blocks_b + WN - 1) / WN;
  const int item = item_of_workgroup(tiles_m * tiles_n);
  if (item < 0) return;
  const int block_m = item / tiles_n * WM, block_n = item % tiles_n * WN;
  const int half = lane >> 5, r = lane & 31;
  const int lines = mx4_lines(p.K);
  // where the tile's blocks of rows lie from its first on; beyond the matrices the last one repeats (not stored)
  uint32_t at_a[WM], at_b[WN], scales_at_a[WM], scales_at_b[WN];
  constexpr uint32_t kNowhere = 0x7fffff00u;
#pragma unroll
  for (int i = 0; i < WM; ++i) {
    const int b = min(i, blocks_a - 1 - block_m);
    at_a[i] = kMx4BlockBytes * b + 16 * lane;
    scales_at_a[i] = kMx4Rows * 16 * b + 16 * r + 8 * half;
  }
#pragma unroll
  for (int i = 0; i < WN; ++i) {
    const int b = min(i, blocks_b - 1 - block_n);
    const bool row = 32 * (block_n + b) + r < p.N;
    at_b[i] = row ? kMx4BlockBytes * b + 16 * lane : kNowhere;
    scales_at_b[i] = row ? kMx4Rows * 16 * b + 16 * r + 8 * half : kNowhere;
  }
  struct Line {
    u32x4 a[4][WM], b[4][WN];
    u32x2 scale_a[WM], scale_b[WN];
  };
  struct Sources {
    __amdgpu_buffer_rsrc_t a, b;
  };
  auto sources_of = [&](int line) {
    return Sources{buffer_of(a_codes + mx4_codes_at(line, blocks_a, block_m), WM * kMx4BlockBytes),
                   buffer_of(b_codes + mx4_codes_at(line, blocks_b, block_n), WN * kMx4BlockBytes)};
  };
  auto load_scales = [&](int line, Line& f) {
    const __amdgpu_buffer_rsrc_t a = buffer_of(a_scales + mx4_scales_at(line >> 1, blocks_a, block_m), WM * kMx4Rows * 16);
    const __amdgpu_buffer_rsrc_t b = buffer_of(b_scales + mx4_scales_at(line >> 1, blocks_b, block_n), WN * kMx4Rows * 16);
#pragma unroll
    for (int i = 0; i < WM; ++i) f.scale_a[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(a, scales_at_a[i], 0, 0));
#pragma unroll
    for (int i = 0; i < WN; ++i) f.scale_b[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, scales_at_b[i], 0, 0));
  };
  auto load_step = [&](const Sources& src, int q, Line& f) {
#pragma unroll
    for (int i = 0; i < WM; ++i)
      f.a[q][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src.a, at_a[i], 1024 * q, 0));
#pragma unroll
    for (int i = 0; i < WN; ++i)
      f.b[q][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src.b, at_b[i], 1024 * q, 0));
  };
  f32x16 acc[WN][WM];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;
  // scale words of the line that multiplies: the second line of a group has its bytes two places up
  u32x2 scale_a[WM], scale_b[WN];
  auto take_scales = [&](int line, const Line& f) {
    const uint32_t down = 16 * (line & 1);
#pragma unroll
    for (int i = 0; i < WM; ++i) scale_a[i] = u32x2{f.scale_a[i][0] >> down, f.scale_a[i][1] >> down};
#pragma unroll
    for (int i = 0; i < WN; ++i) scale_b[i] = u32x2{f.scale_b[i][0] >> down, f.scale_b[i][1] >> down};
  };
  auto multiply = [&](auto which, const Line& f) {
    constexpr int q = decltype(which)::value;
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
      for (int j = 0; j < WM; ++j)
        acc[i][j] = mfma_32x32x64<q / 2>(f.b[q][i], scale_b[i][q & 1], f.a[q][j], scale_a[j][q & 1], acc[i][j]);
  };

  Line f;
  if (wave < lines) {
    const Sources src = sources_of(wave);
    load_scales(wave, f);
    load_step(src, 0, f);
    load_step(src, 1, f);
    load_step(src, 2, f);
    load_step(src, 3, f);
    int line = wave;
    for (; line + WAVES < lines; line += WAVES) {
      const Sources next = sources_of(line + WAVES);
      take_scales(line, f);
      load_scales(line + WAVES, f);
      multiply(std::integral_constant<int, 0>{}, f);
      load_step(next, 0, f);
      multiply(std::integral_constant<int, 1>{}, f);
      load_step(next, 1, f);
      multiply(std::integral_constant<int, 2>{}, f);
      load_step(next, 2, f);
      multiply(std::integral_constant<int, 3>{}, f);
      load_step(next, 3, f);
    }
    take_scales(line, f);
    multiply(std::integral_constant<int, 0>{}, f);
    multiply(std::integral_constant<int, 1>{}, f);
    multiply(std::integral_constant<int, 2>{}, f);
    multiply(std::integral_constant<int, 3>{}, f);
  }
  // 32 rows of Y at a time: every wave's part to its slab, then all of them added
  const int count = min(WAVES, lines);  // waves that had a line
#pragma unroll
  for (int j = 0; j < WM; ++j) {
    if (j > 0) __syncthreads();
    if (wave < count) {
#pragma unroll
      for (int i = 0; i < WN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(slabs[wave] + r * kPitch + 32 * i + 8 * q + 4 * half) =
              f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    }
    __syncthreads();
    add_slabs<OUT, WN, WAVES>(slabs, count, block_m + j, block_n, Y, p);
  }
}

template <int OUT, int WM, int WN, int WAVES>
hipError_t launch_stream(const Mx4ProductArgs& a, const ProductShape& p, hipStream_t stream) {
  const int64_t items = (int64_t)((p.M + 32 * WM - 1) / (32 * WM)) * ((p.N + 32 * WN - 1) / (32 * WN));
  if (a.plan) {
    plan_record(a.plan, "mx4_stream_kernel<OUT=%d,WM=%d,WN=%d,WAVES=%d> grid=%u block=%d", OUT, WM, WN, WAVES, grid_of_items(items), 64 * WAVES);
    return hipSuccess;
  }
  mx4_stream_kernel<OUT, WM, WN, WAVES><<<dim3(grid_of_items(items)), 64 * WAVES, 0, stream>>>(a.a_codes, a.a_scales, a.b_codes,
                                                                                             a.b_scales, a.Y, p);
  return hipGetLastError();
}

// ---- one token, quantised on the way ---------------------------------------------------------------------
// The form above for 32 rows of A, eight waves and one row of B that comes as 16-bit values: a wave quantises the line it is
// about to multiply, four values a lane, and passes the codes through LDS to the two lanes that hold the row.  One launch
// where quantising apart takes two; sums in the same order, so the same result bit for bit.  11008x4096: 6.0 us, 4.0 TB/s of
// weights; a launch's start and the trip to memory are half of it.
template <int OUT, int DT>
__global__ __launch_bounds__(512) void mx4_token_kernel(const uint8_t* codes, const uint8_t* scales, const uint16_t* x, int64_t ldx,
                                                        void* Y, ProductShape p) {
  constexpr int kWaves = 8, kLinePlace = 8 * 16 + 16;  // a line's codes and its eight scale bytes
  __shared__ __align__(16) uint8_t places[kWaves][kLinePlace + 16];  // ... and zeros
  __shared__ __align__(16) float sums[kWaves][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = mx4_row_blocks(p.M), block = item_of_workgroup(blocks);
  if (block < 0) return;
  const int half = lane >> 5, r = lane & 31, lines = mx4_lines(p.K);
  uint8_t* const place = places[wave];
  struct Line {
    u32x4 a[4];
    u32x2 scale_a, x;
  };
  auto load_line = [&](int line, Line& f) {
    const uint8_t* c = codes + mx4_codes_at(line, blocks, block) + 16 * lane;
#pragma unroll
    for (int q = 0; q < 4; ++q) f.a[q] = *reinterpret_cast<const u32x4*>(c + 1024 * q);
    f.scale_a = *reinterpret_cast<const u32x2*>(scales + mx4_scales_at(line >> 1, blocks, block) + 16 * r + 8 * half);
    const int k = line * kMx4Line + 4 * lane;
    f.x = u32x2{0, 0};
    if (ldx == 1 && k + 4 <= p.K) {
      f.x = *reinterpret_cast<const u32x2_a2*>(x + k);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k + j < p.K) f.x[j >> 1] |= (uint32_t)x[(k + j) * ldx] << (16 * (j & 1));
    }
  };
  f32x16 acc;
#pragma unroll
  for (int q = 0; q < 16; ++q) acc[q] = 0;
  auto multiply = [&](int line, const Line& f) {
    uint32_t m = max_halves(f.x[0] & 0x7fff7fffu, f.x[1] & 0x7fff7fffu);
    m = max_with_lane<0xB1>(m);   // lane ^ 1
    m = max_with_lane<0x4E>(m);   // lane ^ 2
    m = max_with_lane<0x141>(m);  // the other four of eight
    m = max_halves(m, m >> 16) & 0xffffu;
    const uint32_t e = mx4_scale_of<DT>(m);
    const float s = mx4_inverse_scale(e);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(f.x[0]) * s, high_half<DT>(f.x[0]) * s, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, low_half<DT>(f.x[1]) * s, high_half<DT>(f.x[1]) * s, 1.0f, 1);
    if (e == 255) c = 0;
    // LDS operations of a wave are done in order; the compiler is held to it
    *reinterpret_cast<uint16_t*>(place + 2 * lane) = (uint16_t)c;
    if ((lane & 7) == 0) place[128 + (lane >> 3)] = (uint8_t)e;
    asm volatile("" ::: "memory");
    u32x4 b[4];
    uint32_t scale_b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int of = 4 * (q >> 1) + 2 * half + (q & 1);
      b[q] = *reinterpret_cast<const u32x4*>(place + (r == 0 ? 16 * of : kLinePlace));
      scale_b[q] = place[128 + of];
    }
    asm volatile("" ::: "memory");
    const uint32_t down = 16 * (line & 1);
    const u32x2 scale_a = {f.scale_a[0] >> down, f.scale_a[1] >> down};
    acc = mfma_32x32x64<0, 0>(b[0], scale_b[0], f.a[0], scale_a[0], acc);
    acc = mfma_32x32x64<0, 0>(b[1], scale_b[1], f.a[1], scale_a[1], acc);
    acc = mfma_32x32x64<0, 1>(b[2], scale_b[2], f.a[2], scale_a[0], acc);
    acc = mfma_32x32x64<0, 1>(b[3], scale_b[3], f.a[3], scale_a[1], acc);
  };
  if (lane < 4) *reinterpret_cast<uint32_t*>(place + kLinePlace + 4 * lane) = 0;
  Line f;
  if (wave < lines) {
    load_line(wave, f);
    int line = wave;
    for (; line + kWaves < lines; line += kWaves) {
      Line next;
      load_line(line + kWaves, next);
      multiply(line, f);
      f = next;
    }
    multiply(line, f);
  }
  // D: row 0 is register 0 of the lower lanes, lane l column l of D = row l of A
  if (half == 0) sums[wave][r] = acc[0];
  __syncthreads();
  const int m = 32 * block + (int)threadIdx.x;
  if (threadIdx.x >= 32 || m >= p.M) return;
  float v = sums[0][threadIdx.x];
  const int count = min(kWaves, lines);
  for (int w = 1; w < count; ++w) v += sums[w][threadIdx.x];
  store_four<OUT>(Y, (int64_t)m * p.ldy, 0, f32x4{v, 0, 0, 0}, p);
}

// ---- a few tokens, quantised on the way ------------------------------------------------------------------
// The same for 32 tokens a workgroup, or all of 2 .. 31, in P = 1, 2 or 4 pieces of a row of X, at most 4096 / P channels.  The
// waves first quantise those tokens into LDS, in passes of 256 / P channels: a lane takes four channels of eight tokens, as the
// kernel that quantises columns, so eight lanes hold a block.  Every workgroup does that, which pays for small products only,
// but there a launch less is 2.6 us of the caller's time.  On the device, in a graph, us in two launches and here:
//   up to 32 tokens, 16 passes: 8192x256 of 16 5.9 and 3.7, 4096x1024 of 8 6.6 and 4.4, 4096x2048 of 16 7.2 and 7.3;
//   more, by workgroups (at most 768, which run at once) and lines: 752 of one line 6.7 and 6.9, 512 of two 6.5 and 5.9, 611 of
//   two 6.7 and 8.1, 256 of four 6.9 and 7.0, 329 of four 6.8 and 8.7; 512x500 of 200 tokens 6.2 and 4.2.
// The forms that would serve such products apart (64x128 and smaller) add their lines in the same order.  Tokens that do not
// exist come out of what happens to lie there: a row of the instruction's operand has no part in another row's result.
constexpr int kFewPasses = 16;
template <int OUT, int DT, int P>
__global__ __launch_bounds__(512) void mx4_few_kernel(const uint8_t* codes, const uint8_t* scales, const uint16_t* x, int64_t ldx,
                                                      Pieces pieces, void* Y, ProductShape p) {
  constexpr int kWaves = 8, kTokens = 8 * P, kLanes = 64 / P, kPitch = slab_pitch(1), kRounds = kFewPasses / kWaves;
  __shared__ __align__(16) uint8_t x_codes[kFewPasses * 1024];  // [block][token][16]
  __shared__ uint8_t x_scales[kFewPasses * 64];                 // [block][token]
  __shared__ __align__(16) float slabs[kWaves][32 * kPitch];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = mx4_row_blocks(p.M), blocks_n = (p.N + 31) / 32;
  const int item = item_of_workgroup(blocks * blocks_n);
  if (item < 0) return;
  const int block = item / blocks_n, block_n = item - block * blocks_n;
  const int half = lane >> 5, r = lane & 31, lines = mx4_lines(p.K);
  const int n = 8 * (lane / kLanes), left = p.N - 32 * block_n - n, k4 = 4 * (lane % kLanes);  // this lane's tokens; its channels of a pass
  u32x4 v[kRounds][4];
#pragma unroll
  for (int s = 0; s < kRounds; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = 4 * kLanes * (wave + kWaves * s) + k4 + i;
      v[s][i] = k < p.K && left > 0 ? draw_eight(x + (int64_t)k * ldx + 32 * block_n + n, left, pieces) : u32x4{0, 0, 0, 0};
    }
  struct Line {
    u32x4 a[4];
    u32x2 scale_a;
  };
  auto load_line = [&](int line, Line& f) {
    const uint8_t* c = codes + mx4_codes_at(line, blocks, block) + 16 * lane;
#pragma unroll
    for (int q = 0; q < 4; ++q) f.a[q] = *reinterpret_cast<const u32x4*>(c + 1024 * q);
    f.scale_a = *reinterpret_cast<const u32x2*>(scales + mx4_scales_at(line >> 1, blocks, block) + 16 * r + 8 * half);
  };
  Line f;
  if (wave < lines) load_line(wave, f);
#pragma unroll
  for (int s = 0; s < kRounds; ++s) {
    const int pass = wave + kWaves * s, k = 4 * kLanes * pass + k4, in_block = (k >> 2) & 7;
    if (pass >= lines * P) break;
    uint8_t* const to = x_codes + ((k >> 5) * kTokens + n) * 16 + 2 * in_block;
    uint8_t* const to_scale = x_scales + (k >> 5) * kTokens + n;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[s][i] = place_eight(v[s][i], left, pieces);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max_halves(m, v[s][i][w] & 0x7fff7fffu);
      m = max_with_lane<0xB1>(m);   // lane ^ 1
      m = max_with_lane<0x4E>(m);   // lane ^ 2
      m = max_with_lane<0x141>(m);  // the other four of eight
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t e = mx4_scale_of<DT>(h ? m >> 16 : m & 0xffffu);
        const float inverse = mx4_inverse_scale(e);
        float g[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = (h ? high_half<DT>(v[s][i][w]) : low_half<DT>(v[s][i][w])) * inverse;
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, g[0], g[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, g[2], g[3], 1.0f, 1);
        if (e == 255) c = 0;
        *reinterpret_cast<uint16_t*>(to + 16 * (2 * w + h)) = (uint16_t)c;
        if (in_block == 2 * w + h) to_scale[2 * w + h] = (uint8_t)e;
      }
    }
  }
  __syncthreads();
  f32x16 acc;
#pragma unroll
  for (int q = 0; q < 16; ++q) acc[q] = 0;
  auto multiply = [&](int line, const Line& f) {
    u32x4 b[4];
    uint32_t scale_b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = (8 * line + 4 * (q >> 1) + 2 * half + (q & 1)) * kTokens + (r & (kTokens - 1));
      b[q] = *reinterpret_cast<const u32x4*>(x_codes + 16 * at);
      scale_b[q] = x_scales[at];
    }
    const uint32_t down = 16 * (line & 1);
    const u32x2 scale_a = {f.scale_a[0] >> down, f.scale_a[1] >> down};
    acc = mfma_32x32x64<0, 0>(b[0], scale_b[0], f.a[0], scale_a[0], acc);
    acc = mfma_32x32x64<0, 0>(b[1], scale_b[1], f.a[1], scale_a[1], acc);
    acc = mfma_32x32x64<0, 1>(b[2], scale_b[2], f.a[2], scale_a[0], acc);
    acc = mfma_32x32x64<0, 1>(b[3], scale_b[3], f.a[3], scale_a[1], acc);
  };
  if (wave < lines) {
    Line next;
    if (wave + kWaves < lines) load_line(wave + kWaves, next);
    multiply(wave, f);
    if (wave + kWaves < lines) multiply(wave + kWaves, next);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(slabs[wave] + r * kPitch + 8 * q + 4 * half) =
          f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
  }
  __syncthreads();
  add_slabs<OUT, 1, kWaves>(slabs, min(kWaves, lines), block, block_n, Y, p);
}

// ---- many rows of both: tiles through LDS ---------------------------------------------------------------
// A workgroup of four waves (2 x 2) owns TM = 64 WM rows of A and TN = 64 WN rows of B; a wave owns half of each, in 32x32
// tiles.  A stage is a line of 256 values, copied straight into LDS, RING (2 or 4) stages in turn; the 16 scale bytes a row has
// for 512 values come with every second stage.  A stage is four instructions for every 32x32 tile; a wave reads the operands of the
// next one while it multiplies.
//   Waits (large tiles): copies of a wave land in order.  Before the last quarter of stage p those of stages p + 2 .. p + RING - 1 may be
// outstanding, all earlier ones are waited for, and so are the wave's LDS reads of stage p; past the barrier that holds for all
// waves, so stage p + 1 is there and the place of stage p takes stage p + RING: half of its copies during the last quarter of
// p, the others during the first of p + 1.  Scales of group g + RING / 2 are copied in the last quarter of stage 2 g, ahead of
// stage 2 g + RING, and read after stage 2 g + RING - 1; their place held group g - RING / 2.  Beyond the last stage the last
// one is copied again; nobody reads it.
//   What bounds it: 16384x16384x8192 takes 0.93 to 1.0 ms, 4.4 to 4.7 PFLOP/s, at a clock that the power limit holds at 1.5 to
// 1.6 GHz (a loop of nothing but the instruction reaches 6.3 PFLOP/s on such operands, 8.7 on zeros).  Tiles of 128 rows wait:
// a stage is 512 clocks of products and takes some 1400, as one wave a SIMD stands at its copies, the barrier and its LDS reads in
// turn (matrix units busy 36 % of its life; 36 KB a stage and unit are half of what L2 gives): 4096x4096 of 1000 columns 13.4 to
// 15.8 us (2.1 to 2.5 PFLOP/s).  Two workgroups a unit, 2048 columns: busy half of the time, 23 us (3.0); with operands of zeros
// 18.5.  Tiles of 256x128 measured the same there (22.2) and less elsewhere.

template <int WM, int WN, int RING>
struct TileSizes {
  static constexpr int TM = 64 * WM, TN = 64 * WN;
  static constexpr int kStageBytes = (TM + TN) * 128;
  static constexpr int kScaleBytes = (TM + TN) * 16;               // of two stages
  static constexpr int kCopies = (TM + TN) / 32;                   // of a wave and stage: 8 rows each
  static constexpr int kLds = RING * (kStageBytes + kScaleBytes);
  static_assert(RING == 2 || RING == 4, "places by masks");
  static_assert(TM == TN && (TM == 128 || TM == 256), "whole copies for every wave");
};

template <int OUT, int WM, int WN, int RING>
__global__ __launch_bounds__(256, WM * WN > 8 ? 1 : 2) void mx4_tile_kernel(const uint8_t* a_codes, const uint8_t* a_scales,
                                                                            const uint8_t* b_codes, const uint8_t* b_scales,
                                                                            void* Y, ProductShape p) {
  using T = TileSizes<WM, WN, RING>;
  extern __shared__ __align__(16) uint8_t lds[];
  uint8_t* const lds_scales = lds + RING * T::kStageBytes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the list of tiles: panels of eight tiles of A times all of B, so that the 32 tiles an XCD works on share eight and four
  // operand tiles
  const int tiles_m = (p.M + T::TM - 1) / T::TM, tiles_n = (p.N + T::TN - 1) / T::TN;
  const int item = item_of_workgroup(tiles_m * tiles_n);
  if (item < 0) return;
  const int panel = item / (8 * tiles_n), in_panel = item - panel * 8 * tiles_n;
  const int height = min(8, tiles_m - 8 * panel);
  const int m0 = (8 * panel + in_panel % height) * T::TM, n0 = in_panel / height * T::TN;
  const int stages = mx4_lines(p.K), groups = mx4_groups(p.K);
  // A wave copies a quarter of A's blocks of rows, then one of B's, a kilobyte at a time; blocks beyond the matrices repeat the
  // last one (what they give is not stored).
  constexpr int kOfA = T::TM / 32;
  const int blocks_a = mx4_row_blocks(p.M), blocks_b = mx4_row_blocks(p.N), block_m = m0 / 32, block_n = n0 / 32;
  const uint32_t lane_at = 16 * lane;
  uint32_t from[T::kCopies];  // uniform
#pragma unroll
  for (int c = 0; c < T::kCopies; ++c) {
    const int kb = c < kOfA ? wave * kOfA + c : wave * (T::TN / 32) + c - kOfA;
    from[c] = kMx4BlockBytes * min(kb >> 2, (c < kOfA ? blocks_a - block_m : blocks_b - block_n) - 1) + 1024 * (kb & 3);
  }
  struct Source {
    __amdgpu_buffer_rsrc_t a, b;
  };
  auto source_of = [&](int stage) {
    const int line = min(stage, stages - 1);
    return Source{buffer_of(a_codes + mx4_codes_at(line, blocks_a, block_m), T::TM * 128),
                  buffer_of(b_codes + mx4_codes_at(line, blocks_b, block_n), T::TN * 128)};
  };
  auto copy_rows = [&](const Source& src, int stage, int c) {  // one of the wave's copies of a stage
    const int kb = c < kOfA ? wave * kOfA + c : T::TM / 8 + wave * (T::TN / 32) + c - kOfA;
    copy16_to_lds(c < kOfA ? src.a : src.b, lane_at, from[c], lds + (stage & (RING - 1)) * T::kStageBytes + kb * 1024);
  };
  // scales: two blocks of rows a copy; with 256 rows of each matrix every wave copies both, with 128 two waves A and two B
  constexpr bool kBoth = T::TM == 256;
  const bool scales_of_a = kBoth || wave < 2;
  const int scale_block = 2 * (kBoth ? wave : wave & 1);
  uint8_t* const scale_place = lds_scales + (scales_of_a ? 0 : T::TM * 16) + scale_block * 512;
  const int lane_block = scale_block + (lane >> 5);
  const uint32_t scale_from_a = 512 * min(lane_block, blocks_a - block_m - 1) + 16 * (lane & 31);
  const uint32_t scale_from_b = 512 * min(lane_block, blocks_b - block_n - 1) + 16 * (lane & 31);
  auto copy_scales = [&](int g) {
    const int group = min(g, groups - 1);
    const uint8_t* of_a = a_scales + mx4_scales_at(group, blocks_a, block_m);
    const uint8_t* of_b = b_scales + mx4_scales_at(group, blocks_b, block_n);
    uint8_t* to = scale_place + (g & (RING - 1)) * T::kScaleBytes;
    copy16_to_lds(buffer_of(scales_of_a ? of_a : of_b, T::TM * 16), scales_of_a ? scale_from_a : scale_from_b, 0, to);
    if constexpr (kBoth) copy16_to_lds(buffer_of(of_b, T::TN * 16), scale_from_b, 0, to + T::TM * 16);
  };

  const int half = lane >> 5, r = lane & 31;
  const int wave_m = (wave & 1) * 32 * WM, wave_n = (wave >> 1) * 32 * WN;
  const int at_a = wave_m * 128 + lane_at, at_b = (T::TM + wave_n) * 128 + lane_at;

  // one operand set: what a quarter of a stage multiplies
  struct Operands {
    u32x4 a[WM], b[WN];
  };
  auto read_one = [&](int stage, int quarter, int t, Operands& f) {
    const uint8_t* base = lds + (stage & (RING - 1)) * T::kStageBytes + 1024 * quarter;
    if (t < WM) f.a[t] = *reinterpret_cast<const u32x4*>(base + at_a + kMx4BlockBytes * t);
    else f.b[t - WM] = *reinterpret_cast<const u32x4*>(base + at_b + kMx4BlockBytes * (t - WM));
  };
  u32x2 scale_a[WM], scale_b[WN];  // word q: quarters with h % 2 = q, two bytes a stage
  auto read_scales = [&](int g) {
    const uint8_t* base = lds_scales + (g & (RING - 1)) * T::kScaleBytes + 8 * half;
#pragma unroll
    for (int i = 0; i < WM; ++i) scale_a[i] = *reinterpret_cast<const u32x2*>(base + 16 * (wave_m + 32 * i + r));
#pragma unroll
    for (int i = 0; i < WN; ++i) scale_b[i] = *reinterpret_cast<const u32x2*>(base + 16 * (T::TM + wave_n + 32 * i + r));
  };

  f32x16 acc[WN][WM];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;
  // Small tiles: a wave holds the operands of a whole stage and reads those of the next one meanwhile (a quarter's products,
  // 128 clocks, do not cover the way through LDS).  The barrier then stands before the stage, at which every wave has read it.
  constexpr bool kWhole = WM * WN <= 4;
  // A quarter of a stage: the products of one operand set, and between them, one at a time so that neither the wave's issue nor
  // the units behind it back up, the LDS reads of the next set (from the first product on: the compiler waits there for every
  // read before it) and, in the quarters that have them, half of a stage's copies.
  auto quarter_stage = [&](auto byte, auto which, const Operands& now, Operands& next, int read_stage, int copied_stage) {
    constexpr int kTiles = WM * WN, kReads = WM + WN, kHalf = T::kCopies / 2, h = decltype(which)::value;
    constexpr bool kCopying = h == 3 || h == 0;
    const Source src = source_of(copied_stage);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int i = t / WM, j = t % WM;
      acc[i][j] = mfma_32x32x64<decltype(byte)::value>(now.b[i], scale_b[i][h & 1], now.a[j], scale_a[j][h & 1], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = t * kReads * 2 / kTiles; e < (t + 1) * kReads * 2 / kTiles && e < kReads; ++e)
        read_one(read_stage, (h + 1) & 3, e, next);
#pragma unroll
      for (int c = t * kHalf / kTiles; kCopying && c < (t + 1) * kHalf / kTiles; ++c)
        copy_rows(src, copied_stage, (h == 0 ? kHalf : 0) + c);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

#pragma unroll
  for (int g = 0; g < RING / 2; ++g) copy_scales(g);
#pragma unroll
  for (int q = 0; q < RING; ++q) {
    const Source src = source_of(q);
#pragma unroll
    for (int c = 0; c < (kWhole || q < RING - 1 ? T::kCopies : T::kCopies / 2); ++c) copy_rows(src, q, c);
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kWhole ? (RING - 1) * T::kCopies : (RING - 2) * T::kCopies + T::kCopies / 2) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  // FIRST: the first stage of its group, with scale bytes 0 and 1; the other one has 2 and 3
  int p0 = 0;
  if constexpr (kWhole) {
    struct Stage {
      Operands q[4];
    };
    Stage even, odd;
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int t = 0; t < WM + WN; ++t) read_one(0, h, t, even.q[h]);
    read_scales(0);
    auto stage = [&](auto is_first, int p, const Stage& now, Stage& next) {
      constexpr bool kFirst = decltype(is_first)::value;
      constexpr int kTiles = WM * WN, kReads = WM + WN, kPart = T::kCopies / 4;
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((RING - 2) * T::kCopies) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (kFirst) copy_scales((p >> 1) + RING / 2);
      const Source src = source_of(p + RING);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          const int i = t / WM, j = t % WM;
          if (h < 2)
            acc[i][j] = mfma_32x32x64<kFirst ? 0 : 2>(now.q[h].b[i], scale_b[i][h & 1], now.q[h].a[j], scale_a[j][h & 1], acc[i][j]);
          else
            acc[i][j] = mfma_32x32x64<kFirst ? 1 : 3>(now.q[h].b[i], scale_b[i][h & 1], now.q[h].a[j], scale_a[j][h & 1], acc[i][j]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = t * kReads / kTiles; e < (t + 1) * kReads / kTiles; ++e) read_one(p + 1, h, e, next.q[h]);
#pragma unroll
          for (int c = t * kPart / kTiles; c < (t + 1) * kPart / kTiles; ++c) copy_rows(src, p + RING, h * kPart + c);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    for (; p0 + 2 <= stages; p0 += 2) {
      stage(std::true_type{}, p0, even, odd);
      stage(std::false_type{}, p0 + 1, odd, even);
      read_scales((p0 >> 1) + 1);
    }
    if (p0 < stages) stage(std::true_type{}, p0, even, odd);
  } else {
    Operands first, second;
#pragma unroll
    for (int t = 0; t < WM + WN; ++t) read_one(0, 0, t, first);
    read_scales(0);
    auto stage = [&](auto is_first, int p) {
      constexpr bool kFirst = decltype(is_first)::value;
      constexpr std::integral_constant<int, kFirst ? 0 : 2> lower{};
      constexpr std::integral_constant<int, kFirst ? 1 : 3> upper{};
      quarter_stage(lower, std::integral_constant<int, 0>{}, first, second, p, p + RING - 1);
      quarter_stage(lower, std::integral_constant<int, 1>{}, second, first, p, 0);
      quarter_stage(upper, std::integral_constant<int, 2>{}, first, second, p, 0);
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((RING - 2) * T::kCopies) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (kFirst) copy_scales((p >> 1) + RING / 2);
      quarter_stage(upper, std::integral_constant<int, 3>{}, second, first, p + 1, p + RING);
    };
    for (; p0 + 2 <= stages; p0 += 2) {
      stage(std::true_type{}, p0);
      stage(std::false_type{}, p0 + 1);
      read_scales((p0 >> 1) + 1);
    }
    if (p0 < stages) stage(std::true_type{}, p0);
  }
  // every copy has landed and every wave has read its operands: the ring becomes the waves' slabs
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  // 32 rows of Y at a time: to the wave's slab, and from there in whole pieces of 16 bytes
  constexpr int kElem = OUT == 2 ? 4 : 2;
  constexpr int kRowBytes = 32 * WN * kElem, kRowPitch = kRowBytes + 16, kPer = 16 / kElem;
  static_assert(4 * 32 * kRowPitch <= T::kLds, "slabs");
  uint8_t* slab = lds + wave * 32 * kRowPitch;
#pragma unroll
  for (int j = 0; j < WM; ++j) {
#pragma unroll
    for (int i = 0; i < WN; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        if (p.relu) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = v[e] < 0 ? 0 : v[e];  // keeps NaN
        }
        uint8_t* to = slab + r * kRowPitch + (32 * i + 8 * q + 4 * half) * kElem;
        if constexpr (OUT == 2) *reinterpret_cast<f32x4*>(to) = v;
        else *reinterpret_cast<u32x2*>(to) = u32x2{floats_to_bits<OUT>(v[0], v[1]), floats_to_bits<OUT>(v[2], v[3])};
      }
    }
    asm volatile("" ::: "memory");  // LDS operations of a wave are done in order; the compiler is held to it
    constexpr int kPieces = kRowBytes / 16;
#pragma unroll
    for (int c = 0; c < 32 * kPieces / 64; ++c) {
      const int row = (64 * c + lane) / kPieces, piece = (64 * c + lane) % kPieces;
      const int m = m0 + wave_m + 32 * j + row, n = n0 + wave_n + piece * kPer;
      const u32x4 v = *reinterpret_cast<const u32x4*>(slab + row * kRowPitch + 16 * piece);
      if (m >= p.M || n >= p.N) continue;
      uint8_t* to = static_cast<uint8_t*>(Y) + ((int64_t)m * p.ldy + n) * kElem;
      if (n + kPer <= p.N) {
        *reinterpret_cast<u32x4_a2*>(to) = v;
      } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if (n + e >= p.N) break;
          if constexpr (OUT == 2) reinterpret_cast<uint32_t*>(to)[e] = v[e];
          else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    asm volatile("" ::: "memory");
  }
}

template <int OUT, int WM, int WN, int RING>
hipError_t launch_tile(const Mx4ProductArgs& a, const ProductShape& p, hipStream_t stream) {
  using T = TileSizes<WM, WN, RING>;
  const int64_t tiles = (int64_t)((p.M + T::TM - 1) / T::TM) * ((p.N + T::TN - 1) / T::TN);
  if (a.plan) {
    plan_record(a.plan, "mx4_tile_kernel<OUT=%d,WM=%d,WN=%d,RING=%d> grid=%u block=256 lds=%d", OUT, WM, WN, RING, grid_of_items(tiles), T::kLds);
    return hipSuccess;
  }
  const hipError_t e = raise_lds_limit<mx4_tile_kernel<OUT, WM, WN, RING>>(T::kLds);
  if (e != hipSuccess) return e;
  mx4_tile_kernel<OUT, WM, WN, RING><<<dim3(grid_of_items(tiles)), 256, T::kLds, stream>>>(a.a_codes, a.a_scales, a.b_codes,
                                                                                              a.b_scales, a.Y, p);
  return hipGetLastError();
}

// Which form serves a shape: the least of estimates in microseconds, fitted to launches with weights from memory at 134
// shapes (M, K of 128 .. 16384, 1 .. 8192 columns), of which the form chosen was the best one or at most 10 % behind it.  Both sides
// of each line: 4096x4096 of 256 columns 7.5 us from registers, 9.8 as tiles of 128 rows; of 1000 columns 15.3 and 12.0; of 2048
// columns 22 as tiles of 128 rows with a ring of four stages, 21.4 with two stages and two workgroups a unit; of 4096 columns
// 40 as tiles of 128 rows, 37 of 256; 8254x1280 of 3533 columns, where writing counts, 32 and 34.
struct Form {
  int rows, cols;      // of a workgroup
  int waves;           // registers: that share the lines; 0: tiles
  int at_once;         // tiles: workgroups that the chip holds
  double start;        // us of a launch and of what does not overlap
  double line;         // registers: us of a wave's line
  double alone, full;  // tiles: us of a stage, with few workgroups and with all places taken; registers: KB/us that a compute
                       // unit draws with one workgroup, and with two or more
  double writing;      // tiles: us that all places take to write 16-bit results while nothing multiplies
};
constexpr Form kForms[] = {
    {32, 32, 8, 0, 4.0, 0.40, 122, 98, 0},           {32, 64, 8, 0, 4.0, 0.80, 117, 87, 0},
    {64, 64, 8, 0, 4.0, 1.29, 99, 58, 0},            {64, 128, 4, 0, 4.0, 1.18, 84, 63, 0},
    {128, 128, 0, 256, 4.6, 0, 0.30, 0.61, 1.0}, {128, 128, 0, 512, 3.9, 0, 0.52, 1.14, 1.5},
    {256, 256, 0, 256, 8.2, 0, 0.92, 1.77, 4.0},
};
constexpr int64_t kMostGroups = 1 << 22;  // of up to 512 threads in a launch
double estimate_us(const Form& f, const ProductShape& p, bool out_f32) {
  const int64_t groups = (int64_t)((p.M + f.rows - 1) / f.rows) * ((p.N + f.cols - 1) / f.cols);
  const double lines = mx4_lines(p.K);
  if (f.waves) {
    if (groups > kMostGroups) return 1e30;
    const double each = lines * 0.128 * (f.rows + (p.N < f.cols ? p.N : f.cols));  // KB
    const double share = groups <= 256 ? 1 : groups / 256.0;                       // workgroups of a compute unit
    const double rate = share >= 2 ? f.full : f.alone + (f.full - f.alone) * (share - 1);
    const double drawn = (double)((groups + 255) / 256) * each / rate;
    const double in_turn = (double)((mx4_lines(p.K) + f.waves - 1) / f.waves) * f.line, weights = lines * 128.0 * p.M / 5.5e6;
    const double most = drawn > in_turn ? drawn : in_turn;
    return f.start + (most > weights ? most : weights) + drawn / 8;
  }
  const int64_t full = groups / f.at_once;
  const double left = (double)(groups - full * f.at_once) / f.at_once;
  const double rounds = (double)groups / f.at_once, written = rounds > 0.5 ? (rounds - 0.5) * (out_f32 ? 2 : 1) : 0;
  return f.start + lines * ((double)full * f.full + (left > 0 ? f.alone + (f.full - f.alone) * left : 0)) + f.writing * written;
}

int form_of(const ProductShape& p, bool out_f32) {
  int best = 0;  // one column: as mx4_token_kernel adds it
  for (int i = 1; p.N > 1 && i < (int)(sizeof kForms / sizeof kForms[0]); ++i)
    if (estimate_us(kForms[i], p, out_f32) < estimate_us(kForms[best], p, out_f32)) best = i;
  return best;
}

template <int OUT>
hipError_t launch_out(const Mx4ProductArgs& a, hipStream_t stream) {
  const ProductShape p{a.M, a.N, a.K, a.ldy, a.relu};
  switch (form_of(p, OUT == 2)) {
    case 0: return launch_stream<OUT, 1, 1, 8>(a, p, stream);
    case 1: return launch_stream<OUT, 1, 2, 8>(a, p, stream);
    case 2: return launch_stream<OUT, 2, 2, 8>(a, p, stream);
    case 3: return launch_stream<OUT, 2, 4, 4>(a, p, stream);
    case 4: return launch_tile<OUT, 2, 2, 4>(a, p, stream);
    case 5: return launch_tile<OUT, 2, 2, 2>(a, p, stream);
    default: return launch_tile<OUT, 4, 4, 2>(a, p, stream);
  }
}

template <int OUT, int DT>
hipError_t launch_token(const Mx4ProductArgs& a, const void* x, int64_t ldx, hipStream_t stream) {
  const ProductShape p{a.M, a.N, a.K, a.ldy, a.relu};
  if (a.plan) {
    plan_record(a.plan, "mx4_token_kernel<OUT=%d,DT=%d> grid=%u block=512", OUT, DT, grid_of_items(mx4_row_blocks(a.M)));
    return hipSuccess;
  }
  mx4_token_kernel<OUT, DT><<<dim3(grid_of_items(mx4_row_blocks(a.M))), 512, 0, stream>>>(
      a.a_codes, a.a_scales, static_cast<const uint16_t*>(x), ldx, a.Y, p);
  return hipGetLastError();
}

template <int OUT, int DT>
hipError_t launch_few(const Mx4ProductArgs& a, const void* x, int64_t ldx, hipStream_t stream) {
  const ProductShape p{a.M, a.N, a.K, a.ldy, a.relu};
  const dim3 grid(grid_of_items((int64_t)mx4_row_blocks(a.M) * ((a.N + 31) / 32)));
  if (a.plan) {
    plan_record(a.plan, "mx4_few_kernel<OUT=%d,DT=%d,P=%d> grid=%u block=512", OUT, DT, a.N <= 8 ? 1 : a.N <= 16 ? 2 : 4, grid.x);
    return hipSuccess;
  }
  const Pieces pieces = pieces_of_rows(x, ldx, a.N);
  auto launch = [&](auto kernel) {
    kernel<<<grid, 512, 0, stream>>>(a.a_codes, a.a_scales, static_cast<const uint16_t*>(x), ldx, pieces, a.Y, p);
  };
  if (a.N <= 8) launch(mx4_few_kernel<OUT, DT, 1>);
  else if (a.N <= 16) launch(mx4_few_kernel<OUT, DT, 2>);
  else launch(mx4_few_kernel<OUT, DT, 4>);
  return hipGetLastError();
}

}  // namespace

bool mx4_quantises_on_the_way(const Mx4ProductArgs& a) {
  if (a.N == 1) return true;
  const int pieces = a.N <= 8 ? 1 : a.N <= 16 ? 2 : 4;
  const int64_t lines = mx4_lines(a.K), groups = (int64_t)mx4_row_blocks(a.M) * ((a.N + 31) / 32);
  if (lines * pieces > kFewPasses) return false;
  const int form = form_of(ProductShape{a.M, a.N, a.K, a.ldy, a.relu}, a.out_f32);
  return a.N <= 32 ? form == 0 : form <= 3 && groups <= 768 && groups * lines <= 1024;
}

hipError_t launch_mx4_product(const Mx4ProductArgs& a, hipStream_t stream) {
  if (a.out_f32) return launch_out<2>(a, stream);
  return a.dtype == HINM_F16 ? launch_out<HINM_F16>(a, stream) : launch_out<HINM_BF16>(a, stream);
}

hipError_t launch_mx4_on_the_way(const Mx4ProductArgs& a, const void* x, int64_t ldx, hipStream_t stream) {
  if (a.N > 1) {
    if (a.dtype == HINM_F16)
      return a.out_f32 ? launch_few<2, HINM_F16>(a, x, ldx, stream) : launch_few<HINM_F16, HINM_F16>(a, x, ldx, stream);
    return a.out_f32 ? launch_few<2, HINM_BF16>(a, x, ldx, stream) : launch_few<HINM_BF16, HINM_BF16>(a, x, ldx, stream);
  }
  if (a.dtype == HINM_F16)
    return a.out_f32 ? launch_token<2, HINM_F16>(a, x, ldx, stream) : launch_token<HINM_F16, HINM_F16>(a, x, ldx, stream);
  return a.out_f32 ? launch_token<2, HINM_BF16>(a, x, ldx, stream) : launch_token<HINM_BF16, HINM_BF16>(a, x, ldx, stream);
}

}  // namespace hinm
