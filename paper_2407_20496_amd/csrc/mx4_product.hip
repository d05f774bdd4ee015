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
  const int64_t cp = mx4_code_pitch(p.K), sp = mx4_scale_pitch(p.K);
  const int steps = (p.K + kMx4Step - 1) / kMx4Step, groups = (steps + 3) / 4;
  // rows beyond the matrices repeat the last one: what they give is not stored
  const int64_t ra = min(m0 + r, p.M - 1);
  const uint8_t* ac = a_codes + ra * cp + 16 * b;
  const uint8_t* as = a_scales + ra * sp + 4 * b;
  const uint8_t *bc[NT], *bs[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t rb = min(n0 + 16 * t + r, p.N - 1);
    bc[t] = b_codes + rb * cp + 16 * b;
    bs[t] = b_scales + rb * sp + 4 * b;
  }
  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4{0, 0, 0, 0};
  for (int g = wave; g < groups; g += waves) {
    const uint32_t sa = *reinterpret_cast<const uint32_t*>(as + 16 * (int64_t)g);
    uint32_t sb[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) sb[t] = *reinterpret_cast<const uint32_t*>(bs[t] + 16 * (int64_t)g);
    auto step = [&](auto s_) {
      constexpr int s = decltype(s_)::value;
      if (4 * g + s >= steps) return;
      const int64_t at = 256 * (int64_t)g + 64 * s;
      const u32x4 a = *reinterpret_cast<const u32x4*>(ac + at);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        acc[t] = mfma_16x16x128<s>(*reinterpret_cast<const u32x4*>(bc[t] + at), sb[t], a, sa, acc[t]);
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
// tiles.  A stage is one k-step: 64 bytes of every row, copied straight into LDS, kStages stages in a ring; the 16 scale
// bytes a row has for four k-steps come with every fourth stage.  A wave holds the operands of the stage it multiplies and
// reads those of the next meanwhile.
//   Swizzle: the four 16-byte pieces of a row sit at piece ^ (row / 4 % 4), applied on the copy's source side, so that 16
// consecutive lanes (16 rows, one piece) read 16 different 16-byte units of 256 bytes.
//   Waits: copies of a wave land in order.  In the middle of step s the copies of stages s + 2 and s + 3 may be outstanding,
// all earlier ones are waited for; past the barrier stage s + 1 is there for everyone, and everyone has read stage s (its
// LDS reads are waited for before the barrier), so its place takes stage s + 4: half of its copies in the second half of step
// s, the others in the first half of step s + 1.  Scales of group g + 1 are copied in the first
// step of group g into the half that group g - 1 used, and have landed by its last step, before stage 4 g + 4.  Beyond the last step the last stage is
// copied again, which keeps the count the same; nobody reads it.
constexpr int kStages = 4;

template <int WM, int WN>
struct TileSizes {
  static constexpr int TM = 64 * WM, TN = 64 * WN;
  static constexpr int kStageBytes = (TM + TN) * 64;
  static constexpr int kScaleBytes = (TM + TN) * 16;               // of a group of four steps
  static constexpr int kCopies = (TM + TN) / 64;                   // of a wave and stage: 16 rows each
  static constexpr int kScaleCopies = (TM + TN) / 256;             // of a wave and group: 64 rows each
  static constexpr int kLds = kStages * kStageBytes + 2 * kScaleBytes;
  static_assert((TM + TN) % 256 == 0 && TM % 64 == 0, "whole copies for every wave");
};

template <int OUT, int WM, int WN>
__global__ __launch_bounds__(256, WM * WN > 8 ? 1 : 2) void mx4_tile_kernel(const uint8_t* a_codes, const uint8_t* a_scales,
                                                                            const uint8_t* b_codes, const uint8_t* b_scales,
                                                                            void* Y, ProductShape p) {
  using T = TileSizes<WM, WN>;
  extern __shared__ __align__(16) uint8_t lds[];
  uint8_t* const lds_scales = lds + kStages * T::kStageBytes;
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
  const int64_t cp = mx4_code_pitch(p.K), sp = mx4_scale_pitch(p.K);
  const int steps = (p.K + kMx4Step - 1) / kMx4Step, groups = (steps + 3) >> 2;

  // where this lane's part of each copy comes from; rows beyond the matrices repeat the last one (what they give is not stored)
  const uint8_t* from[T::kCopies];
  const uint8_t* scales_from[T::kScaleCopies];
#pragma unroll
  for (int c = 0; c < T::kCopies; ++c) {
    const int row = 16 * (wave * T::kCopies + c) + (lane >> 2);
    const int piece = (lane & 3) ^ ((lane >> 4) & 3);
    from[c] = (row < T::TM ? a_codes + min(m0 + row, p.M - 1) * cp : b_codes + min(n0 + row - T::TM, p.N - 1) * cp) + 16 * piece;
  }
#pragma unroll
  for (int c = 0; c < T::kScaleCopies; ++c) {
    const int row = 64 * (wave * T::kScaleCopies + c) + lane;
    scales_from[c] = row < T::TM ? a_scales + min(m0 + row, p.M - 1) * sp : b_scales + min(n0 + row - T::TM, p.N - 1) * sp;
  }
  auto copy_rows = [&](int s, int c) {  // one of the wave's copies of a stage
    copy16_to_lds(from[c] + 64 * (int64_t)min(s, steps - 1),
                  lds + (s & (kStages - 1)) * T::kStageBytes + (wave * T::kCopies + c) * 1024);
  };
  auto copy_scales = [&](int g) {
    const int64_t at = 16 * (int64_t)min(g, groups - 1);
    uint8_t* to = lds_scales + (g & 1) * T::kScaleBytes + wave * T::kScaleCopies * 1024;
#pragma unroll
    for (int c = 0; c < T::kScaleCopies; ++c) copy16_to_lds(scales_from[c] + at, to + 1024 * c);
  };

  const int half = lane >> 5, r = lane & 31;
  const int wave_m = (wave & 1) * 32 * WM, wave_n = (wave >> 1) * 32 * WN;
  // byte offsets of this lane's two pieces of a row, and of its first rows
  const int piece0 = 16 * ((2 * half) ^ ((r >> 2) & 3)), piece1 = 16 * ((2 * half + 1) ^ ((r >> 2) & 3));
  const int row_a = (wave_m + r) * 64, row_b = (T::TM + wave_n + r) * 64;

  // one operand set: piece q of this lane's blocks of a stage (the first or second instruction of a step)
  struct Operands {
    u32x4 a[WM], b[WN];
  };
  auto read_one = [&](int s, int q, int t, Operands& f) {
    const uint8_t* base = lds + (s & (kStages - 1)) * T::kStageBytes + (q ? piece1 : piece0);
    if (t < WM) f.a[t] = *reinterpret_cast<const u32x4*>(base + row_a + 2048 * t);
    else f.b[t - WM] = *reinterpret_cast<const u32x4*>(base + row_b + 2048 * (t - WM));
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
  // Half a step: the products of one operand set, and between them, one at a time so that neither the wave's issue nor the
  // units behind it back up, the LDS reads of the next set (from the first product on: the compiler waits there for every
  // read before it) and half of a stage's copies.
  auto half_step = [&](auto byte, auto which, const Operands& now, Operands& next, int read_stage, int copied_stage) {
    constexpr int kTiles = WM * WN, kReads = WM + WN, kHalfCopies = T::kCopies / 2, q = decltype(which)::value;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int i = t / WM, j = t % WM;
      acc[i][j] = mfma_32x32x64<decltype(byte)::value>(now.b[i], scale_b[i][q], now.a[j], scale_a[j][q], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = t * kReads * 2 / kTiles; e < (t + 1) * kReads * 2 / kTiles && e < kReads; ++e) read_one(read_stage, 1 - q, e, next);
#pragma unroll
      for (int c = t * kHalfCopies / kTiles; c < (t + 1) * kHalfCopies / kTiles; ++c) copy_rows(copied_stage, (1 - q) * kHalfCopies + c);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  copy_scales(0);
#pragma unroll
  for (int s = 0; s < kStages; ++s)
#pragma unroll
    for (int c = 0; c < T::kCopies; ++c)
      if (s < kStages - 1 || c < T::kCopies / 2) copy_rows(s, c);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * T::kCopies - T::kCopies / 2) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  Operands first, second;
#pragma unroll
  for (int t = 0; t < WM + WN; ++t) read_one(0, 0, t, first);
  read_scales(0);

  auto step = [&](auto byte, int s, bool with_scales) {
    half_step(byte, std::integral_constant<int, 0>{}, first, second, s, s + kStages - 1);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * T::kCopies) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (with_scales) copy_scales((s >> 2) + 1);
    half_step(byte, std::integral_constant<int, 1>{}, second, first, s + 1, s + kStages);
  };
  int s = 0;
  for (; s + 4 <= steps; s += 4) {
    step(std::integral_constant<int, 0>{}, s, true);
    step(std::integral_constant<int, 1>{}, s + 1, false);
    step(std::integral_constant<int, 2>{}, s + 2, false);
    step(std::integral_constant<int, 3>{}, s + 3, false);
    read_scales((s >> 2) + 1);
  }
  for (; s < steps; ++s) {  // up to three steps: the scale bytes move down instead
    step(std::integral_constant<int, 0>{}, s, false);
#pragma unroll
    for (int i = 0; i < WM; ++i) scale_a[i] = u32x2{scale_a[i][0] >> 8, scale_a[i][1] >> 8};
#pragma unroll
    for (int i = 0; i < WN; ++i) scale_b[i] = u32x2{scale_b[i][0] >> 8, scale_b[i][1] >> 8};
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
