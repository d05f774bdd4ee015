// Products of two matrices in microscaled 4-bit form, Y = A B^T, on the scaled matrix instructions (include/hinm.h).
#include "direct_lds.h"
#include "mx4_form.h"

#include <type_traits>

namespace hinm {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// The instructions' register forms take 8 words; 4-bit operands use the first four.
__device__ __forceinline__ i32x8 operand(u32x4 v) {
  return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}
constexpr int kFp4 = 4;  // operand format code of 4-bit values
template <int BYTE>
__device__ __forceinline__ f32x4 mfma_16x16x128(u32x4 a, uint32_t a_scale, u32x4 b, uint32_t b_scale, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), c, kFp4, kFp4, BYTE, (int)a_scale, BYTE,
                                                          (int)b_scale);
}

template <int BYTE>
__device__ __forceinline__ f32x16 mfma_32x32x64(u32x4 a, uint32_t a_scale, u32x4 b, uint32_t b_scale, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, kFp4, kFp4, BYTE, (int)a_scale, BYTE,
                                                         (int)b_scale);
}

struct ProductShape {
  int M, N, K;
  int64_t ldy;
  bool relu;
};

template <int OUT>  // HINM_F16, HINM_BF16, 2 = float32
__device__ __forceinline__ void store_one(void* Y, int64_t at, float v) {
  if constexpr (OUT == 2) static_cast<float*>(Y)[at] = v;
  else static_cast<uint16_t*>(Y)[at] = float_to_bits<OUT>(v);
}

// ---- few rows of B: the summed axis split over the waves of a workgroup ---------------------------------
// A workgroup owns 16 rows of A and 16 NT rows of B; its waves take groups of 512 values in turn, straight from memory into
// registers, and add their tiles in LDS in a fixed order.  B is the instructions' row operand, so that a lane ends with four
// consecutive columns of one row of Y.
template <int OUT, int NT>
__global__ __launch_bounds__(512) void mx4_split_kernel(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                                                        const uint8_t* b_scales, void* Y, ProductShape p) {
  extern __shared__ __align__(16) float slabs[];  // [waves][16][16 NT + 4]
  constexpr int kPitch = 16 * NT + 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r = lane & 15, b = lane >> 4;
  const int blocks_n = (p.N + 16 * NT - 1) / (16 * NT);
  const int m0 = (int)(blockIdx.x / blocks_n) * 16, n0 = (int)(blockIdx.x % blocks_n) * 16 * NT;
  const int lines = mx4_lines(p.K), groups = mx4_groups(p.K);
  // rows beyond the matrices repeat the last one: what they give is not stored
  const int64_t ra = min(m0 + r, p.M - 1);
  const uint8_t* ac = a_codes + ra * 128 + 16 * b;
  const uint8_t* as = a_scales + ra * 16 + 4 * b;
  const int64_t a_line = (int64_t)p.M * 128, b_line = (int64_t)p.N * 128, a_group = (int64_t)p.M * 16, b_group = (int64_t)p.N * 16;
  const uint8_t *bc[NT], *bs[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t rb = min(n0 + 16 * t + r, p.N - 1);
    bc[t] = b_codes + rb * 128 + 16 * b;
    bs[t] = b_scales + rb * 16 + 4 * b;
  }
  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4{0, 0, 0, 0};
  for (int g = wave; g < groups; g += waves) {
    const uint32_t sa = *reinterpret_cast<const uint32_t*>(as + g * a_group);
    uint32_t sb[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) sb[t] = *reinterpret_cast<const uint32_t*>(bs[t] + g * b_group);
    auto step = [&](auto s_) {
      constexpr int s = decltype(s_)::value;
      const int line = 2 * g + s / 2;
      if (line >= lines) return;
      const u32x4 a = *reinterpret_cast<const u32x4*>(ac + line * a_line + 64 * (s & 1));
#pragma unroll
      for (int t = 0; t < NT; ++t)
        acc[t] = mfma_16x16x128<s>(*reinterpret_cast<const u32x4*>(bc[t] + line * b_line + 64 * (s & 1)), sb[t], a, sa, acc[t]);
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }
  float* slab = slabs + wave * 16 * kPitch;
#pragma unroll
  for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(slab + r * kPitch + 16 * t + 4 * b) = acc[t];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * 16 * NT; i += blockDim.x) {
    const int row = i / (16 * NT), col = i % (16 * NT);
    if (m0 + row >= p.M || n0 + col >= p.N) continue;
    float v = 0;
    for (int w = 0; w < waves; ++w) v += slabs[(w * 16 + row) * kPitch + col];
    if (p.relu) v = v < 0 ? 0 : v;  // keeps NaN
    store_one<OUT>(Y, (int64_t)(m0 + row) * p.ldy + n0 + col, v);
  }
}

template <int OUT, int NT>
hipError_t launch_split(const Mx4ProductArgs& a, const ProductShape& p, hipStream_t stream) {
  const int groups = (p.K + kMx4Group - 1) / kMx4Group;
  const int waves = groups >= 8 ? 8 : groups >= 4 ? 4 : groups >= 2 ? 2 : 1;
  const size_t lds = (size_t)waves * 16 * (16 * NT + 4) * sizeof(float);
  const int64_t grid = (int64_t)((p.M + 15) / 16) * ((p.N + 16 * NT - 1) / (16 * NT));
  if (lds > 65536) {
    const hipError_t e = raise_lds_limit<mx4_split_kernel<OUT, NT>>((int)lds);
    if (e != hipSuccess) return e;
  }
  mx4_split_kernel<OUT, NT><<<dim3((uint32_t)grid), 64 * waves, lds, stream>>>(a.a_codes, a.a_scales, a.b_codes, a.b_scales, a.Y, p);
  return hipGetLastError();
}

// ---- many rows of both: tiles through LDS ---------------------------------------------------------------
// A workgroup of four waves (2 x 2) owns TM = 64 WM rows of A and TN = 64 WN rows of B; a wave owns half of each, in 32x32
// tiles.  A stage is 256 values = one 128-byte line of every row, copied straight into LDS, two stages in turn; the 16 scale
// bytes a row has for 512 values come with every second stage.  A stage is four instructions for every 32x32 tile; a wave
// reads the operands of the next one while it multiplies.  (Stages of 128 values, four in turn: copies of half lines run at
// 20 bytes a clock and compute unit and took 885 us of 16384x16384x8192's 1176 us by themselves.)
//   Swizzle: the eight 16-byte pieces of a row sit at piece ^ (row / 2 % 8), applied on the copy's source side, so that 16
// consecutive lanes (16 rows, one piece) read 16 different 16-byte units of 256 bytes.
//   Waits: before the last quarter of stage p every copy of the wave's has landed, stage p + 1 among them, and its LDS reads of
// stage p are done; past the barrier that holds for all waves, so the place of stage p takes stage p + 2: half of its copies
// during the last quarter of p, the others during the first of p + 1.  Scales of group g + 1 (stages 2 g + 2 and 2 g + 3) are
// copied in the last quarter of stage 2 g into the half that group g - 1 used.  Beyond the last stage the last one is
// copied again; nobody reads it.

template <int WM, int WN>
struct TileSizes {
  static constexpr int TM = 64 * WM, TN = 64 * WN;
  static constexpr int kStageBytes = (TM + TN) * 128;
  static constexpr int kScaleBytes = (TM + TN) * 16;               // of two stages
  static constexpr int kCopies = (TM + TN) / 32;                   // of a wave and stage: 8 rows each
  static constexpr int kLds = 2 * (kStageBytes + kScaleBytes);
  static_assert(TM == TN && (TM == 128 || TM == 256), "whole copies for every wave");
};

template <int OUT, int WM, int WN>
__global__ __launch_bounds__(256, WM * WN > 8 ? 1 : 2) void mx4_tile_kernel(const uint8_t* a_codes, const uint8_t* a_scales,
                                                                            const uint8_t* b_codes, const uint8_t* b_scales,
                                                                            void* Y, ProductShape p) {
  using T = TileSizes<WM, WN>;
  extern __shared__ __align__(16) uint8_t lds[];
  uint8_t* const lds_scales = lds + 2 * T::kStageBytes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroups go to the eight XCDs in turn: each XCD takes a contiguous run of the list of tiles, panels of eight tiles of A
  // times all of B, so that the 32 tiles it works on share eight and four operand tiles in its L2
  const int tiles_m = (p.M + T::TM - 1) / T::TM, tiles_n = (p.N + T::TN - 1) / T::TN;
  const int per = gridDim.x >> 3;
  const int item = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (item >= tiles_m * tiles_n) return;
  const int panel = item / (8 * tiles_n), in_panel = item - panel * 8 * tiles_n;
  const int height = min(8, tiles_m - 8 * panel);
  const int m0 = (8 * panel + in_panel % height) * T::TM, n0 = in_panel / height * T::TN;
  const int stages = mx4_lines(p.K), groups = mx4_groups(p.K);

  // Where this lane's part of each copy comes from, from the first of the tile's rows in a line or group on; rows beyond the
  // matrices repeat the last one (what they give is not stored).  A wave copies a quarter of A's rows, then one of B's.
  constexpr int kOfA = T::TM / 32;
  const int rows_a = min(T::TM, p.M - m0), rows_b = min(T::TN, p.N - n0);
  uint32_t from[T::kCopies];
#pragma unroll
  for (int c = 0; c < T::kCopies; ++c) {
    const int row = (c < kOfA ? wave * (T::TM / 4) + 8 * c : wave * (T::TN / 4) + 8 * (c - kOfA)) + (lane >> 3);
    const int piece = (lane & 7) ^ ((row >> 1) & 7);
    from[c] = 128 * min(row, (c < kOfA ? rows_a : rows_b) - 1) + 16 * piece;
  }
  struct Source {
    __amdgpu_buffer_rsrc_t a, b;
  };
  auto source_of = [&](int stage) {
    const int line = min(stage, stages - 1);
    return Source{buffer_of(a_codes + mx4_line_at(line, p.M, m0), 128u * rows_a),
                  buffer_of(b_codes + mx4_line_at(line, p.N, n0), 128u * rows_b)};
  };
  auto copy_rows = [&](const Source& src, int stage, int c) {  // one of the wave's copies of a stage
    const int row0 = c < kOfA ? wave * (T::TM / 4) + 8 * c : T::TM + wave * (T::TN / 4) + 8 * (c - kOfA);
    copy16_to_lds(c < kOfA ? src.a : src.b, from[c], lds + (stage & 1) * T::kStageBytes + row0 * 128);
  };
  // scales: 64 rows a copy; with 256 rows of each matrix every wave copies both, with 128 two waves A and two B
  constexpr bool kBoth = T::TM == 256;
  const bool scales_of_a = kBoth || wave < 2;
  const uint8_t* const scale_rows = scales_of_a ? a_scales + 16 * (int64_t)m0 : b_scales + 16 * (int64_t)n0;
  const int64_t scale_group = 16 * (int64_t)(scales_of_a ? p.M : p.N);
  const int scale_count = scales_of_a ? rows_a : rows_b;
  const int scale_row0 = 64 * (kBoth ? wave : wave & 1);
  uint8_t* const scale_place = lds_scales + (scales_of_a ? 0 : T::TM * 16) + scale_row0 * 16;
  const uint32_t scale_from = 16 * min(scale_row0 + lane, scale_count - 1), scale_from_b = 16 * min(scale_row0 + lane, rows_b - 1);
  auto copy_scales = [&](int g) {
    const int group = min(g, groups - 1);
    copy16_to_lds(buffer_of(scale_rows + group * scale_group, 16u * scale_count), scale_from, scale_place + (g & 1) * T::kScaleBytes);
    if constexpr (kBoth)
      copy16_to_lds(buffer_of(b_scales + mx4_group_at(group, p.N, n0), 16u * rows_b), scale_from_b,
                    scale_place + T::TM * 16 + (g & 1) * T::kScaleBytes);
  };

  const int half = lane >> 5, r = lane & 31;
  const int wave_m = (wave & 1) * 32 * WM, wave_n = (wave >> 1) * 32 * WN;
  // byte offset of this lane's piece of a row in the first quarter (the others differ in its bits 0 and 2), and of its first rows
  const int piece0 = 16 * ((2 * half) ^ ((r >> 1) & 7));
  const int row_a = (wave_m + r) * 128, row_b = (T::TM + wave_n + r) * 128;

  // one operand set: what a quarter of a stage multiplies
  struct Operands {
    u32x4 a[WM], b[WN];
  };
  auto read_one = [&](int stage, int quarter, int t, Operands& f) {
    const uint8_t* base = lds + (stage & 1) * T::kStageBytes + (piece0 ^ 16 * (4 * (quarter >> 1) + (quarter & 1)));
    if (t < WM) f.a[t] = *reinterpret_cast<const u32x4*>(base + row_a + 4096 * t);
    else f.b[t - WM] = *reinterpret_cast<const u32x4*>(base + row_b + 4096 * (t - WM));
  };
  u32x2 scale_a[WM], scale_b[WN];  // word q: the lane's blocks 2 half + q of four steps
  auto read_scales = [&](int g) {
    const uint8_t* base = lds_scales + (g & 1) * T::kScaleBytes + 8 * half;
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

  copy_scales(0);
#pragma unroll
  for (int c = 0; c < T::kCopies; ++c) copy_rows(source_of(0), 0, c);
#pragma unroll
  for (int c = 0; c < T::kCopies / 2; ++c) copy_rows(source_of(1), 1, c);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(T::kCopies / 2) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  Operands first, second;
#pragma unroll
  for (int t = 0; t < WM + WN; ++t) read_one(0, 0, t, first);
  read_scales(0);

  // FIRST: the first stage of its group, with scale bytes 0 and 1; the other one has 2 and 3
  auto stage = [&](auto is_first, int p) {
    constexpr bool kFirst = decltype(is_first)::value;
    constexpr std::integral_constant<int, kFirst ? 0 : 2> lower{};
    constexpr std::integral_constant<int, kFirst ? 1 : 3> upper{};
    quarter_stage(lower, std::integral_constant<int, 0>{}, first, second, p, p + 1);
    quarter_stage(lower, std::integral_constant<int, 1>{}, second, first, p, 0);
    quarter_stage(upper, std::integral_constant<int, 2>{}, first, second, p, 0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (kFirst) copy_scales((p >> 1) + 1);
    quarter_stage(upper, std::integral_constant<int, 3>{}, second, first, p + 1, p + 2);
  };
  int p0 = 0;
  for (; p0 + 2 <= stages; p0 += 2) {
    stage(std::true_type{}, p0);
    stage(std::false_type{}, p0 + 1);
    read_scales((p0 >> 1) + 1);
  }
  if (p0 < stages) stage(std::true_type{}, p0);
  // every copy has landed and every wave has read its operands: the ring becomes the waves' slabs
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  // 32 rows of Y at a time: to the wave's slab, and from there in whole pieces of 16 bytes
  constexpr int kElem = OUT == 2 ? 4 : 2;
  constexpr int kRowBytes = 32 * WN * kElem, kRowPitch = kRowBytes + 16, kPer = 16 / kElem;
  static_assert(4 * 32 * kRowPitch <= T::kLds, "slabs");
  uint8_t* slab = lds + wave * 32 * kRowPitch;
  const bool vec = (reinterpret_cast<uintptr_t>(Y) & 15) == 0 && p.ldy % kPer == 0;
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
    __builtin_amdgcn_wave_barrier();
    constexpr int kPieces = kRowBytes / 16;
#pragma unroll
    for (int c = 0; c < 32 * kPieces / 64; ++c) {
      const int row = (64 * c + lane) / kPieces, piece = (64 * c + lane) % kPieces;
      const int m = m0 + wave_m + 32 * j + row, n = n0 + wave_n + piece * kPer;
      const u32x4 v = *reinterpret_cast<const u32x4*>(slab + row * kRowPitch + 16 * piece);
      if (m >= p.M || n >= p.N) continue;
      uint8_t* to = static_cast<uint8_t*>(Y) + ((int64_t)m * p.ldy + n) * kElem;
      if (vec && n + kPer <= p.N) {
        *reinterpret_cast<u32x4*>(to) = v;
      } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if (n + e >= p.N) break;
          if constexpr (OUT == 2) reinterpret_cast<uint32_t*>(to)[e] = v[e];
          else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int OUT, int WM, int WN>
hipError_t launch_tile(const Mx4ProductArgs& a, const ProductShape& p, hipStream_t stream) {
  using T = TileSizes<WM, WN>;
  const int64_t tiles = (int64_t)((p.M + T::TM - 1) / T::TM) * ((p.N + T::TN - 1) / T::TN);
  const hipError_t e = raise_lds_limit<mx4_tile_kernel<OUT, WM, WN>>(T::kLds);
  if (e != hipSuccess) return e;
  mx4_tile_kernel<OUT, WM, WN><<<dim3((uint32_t)((tiles + 7) / 8 * 8)), 256, T::kLds, stream>>>(a.a_codes, a.a_scales, a.b_codes,
                                                                                              a.b_scales, a.Y, p);
  return hipGetLastError();
}

template <int OUT>
hipError_t launch_out(const Mx4ProductArgs& a, hipStream_t stream) {
  const ProductShape p{a.M, a.N, a.K, a.ldy, a.relu};
  if (a.M > 512 && a.N > 512) return launch_tile<OUT, 4, 4>(a, p, stream);
  if (a.M > 256 && a.N > 256) return launch_tile<OUT, 2, 2>(a, p, stream);
  if (a.N <= 16) return launch_split<OUT, 1>(a, p, stream);
  if (a.N <= 32) return launch_split<OUT, 2>(a, p, stream);
  if (a.N <= 64) return launch_split<OUT, 4>(a, p, stream);
  return launch_split<OUT, 8>(a, p, stream);
}

}  // namespace

hipError_t launch_mx4_product(const Mx4ProductArgs& a, hipStream_t stream) {
  if (a.out_f32) return launch_out<2>(a, stream);
  return a.dtype == HINM_F16 ? launch_out<HINM_F16>(a, stream) : launch_out<HINM_BF16>(a, stream);
}

}  // namespace hinm
