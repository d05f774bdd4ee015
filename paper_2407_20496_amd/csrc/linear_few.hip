// A dense layer on few tokens (include/hinm.h, hinm_linear): the weights stream through registers once.
//
// A workgroup owns 16 rows of W and all tokens, at most 16; its waves take runs of 64 channels in turn, each
// for the whole of that, with no barrier between them, and their sums meet in LDS in a fixed order.  The 16x16x32 instruction
// takes W as it lies (a lane 16 bytes of a row, four lanes 64 consecutive bytes); X, whose channels lie apart, goes through a
// place in LDS of the wave's own and comes back by transposing reads; a single token's vector needs no turning and comes
// from memory as it is.  A run's loads are under way while the run before it multiplies.
//   Bound by the weights' bytes: 11008x4096 of one token 17.4 us (5.2 TB/s, in part from the memory-side cache; through tiles in LDS 55),
// 4096x11008 of 16 tokens 21.1 (4.3 TB/s; 38).  Weights of
// odd rows are turned in LDS, from whole runs of 256 bytes a row: 11008x4095 of one token 26 us, 43.5 where a lane draws 16 bytes of each row.
#include "linear_tile.h"

#include <type_traits>

#include "workgroup_items.h"

namespace hinm {

namespace {

struct FewArgs {
  const uint16_t* W;
  int64_t ldw;
  const uint16_t* X;
  int64_t ldx;
  int K;
  Pieces rows_w, rows_x;
};

template <int DT>
__device__ __forceinline__ f32x4 mfma_16x16x32(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (DT == HINM_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// VECTOR: one token, its channels one after the other.  PIECES: rows of W at multiples of 16 bytes.
template <int DT, Epilogue E, bool VECTOR, bool PIECES, int RB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_few_kernel(FewArgs a, LinearEpilogue e) {
  constexpr int kRun = PIECES ? 64 : 128, kSteps = kRun / 32, kFewRows = 16 * RB;
  static_assert(PIECES || RB == 1, "a place for 16 rows");
  constexpr int kTokens = 16, kPitch = kTokens + 4;
  constexpr int kTurnedX = VECTOR ? 0 : kRun * kTokens * 2, kTurned = kTurnedX + (PIECES ? 0 : 16 * kRun * 2);  // bytes
  constexpr int kSums = kFewRows * kPitch * 4;
  constexpr int kPlace = kTurned > kSums ? kTurned : kSums;  // of a wave: a run of X and of W, and in the end its sums
  __shared__ __align__(16) uint8_t places[WAVES][kPlace];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = item_of_workgroup((e.M + kFewRows - 1) / kFewRows);
  if (item < 0) return;
  const int m0 = item * kFewRows, r = lane & 15, g = lane >> 4;
  const int runs = (a.K + kRun - 1) / kRun;
  constexpr int kPointers = PIECES ? RB : 4;
  const uint16_t* w[kPointers];
#pragma unroll
  for (int b = 0; b < kPointers; ++b)
    w[b] = a.W + (int64_t)min(m0 + (PIECES ? 16 * b + r : 4 * b + g), e.M - 1) * a.ldw + (PIECES ? 8 * g : 8 * r);
  const u32x4 none = {0, 0, 0, 0};
  struct Run {
    u32x4 w[RB][kSteps], x[kRun / 32];  // w: not of pieces, rows 4 i + lane / 16, eight channels each
  };
  auto load = [&](int run, Run& f) __attribute__((always_inline)) {
    const int k0 = run * kRun;
    if (k0 + kRun <= a.K) {
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) f.w[b][s] = *reinterpret_cast<const u32x4_a2*>(PIECES ? w[b] + k0 + 32 * s : w[s] + k0);
      if constexpr (VECTOR) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) f.x[s] = r == 0 ? u32x4(*reinterpret_cast<const u32x4_a2*>(a.X + k0 + 32 * s + 8 * g)) : none;
      }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int left = a.K - k0 - 32 * s - 8 * g;
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const int of_w = PIECES ? left : a.K - k0 - 8 * r;
          f.w[b][s] = of_w > 0 ? trim_eight(draw_eight(PIECES ? w[b] + k0 + 32 * s : w[s] + k0, of_w, a.rows_w), of_w, a.rows_w) : none;
        }
        if constexpr (VECTOR) f.x[s] = r == 0 && left > 0 ? trim_eight(draw_eight(a.X + k0 + 32 * s + 8 * g, left, a.rows_x), left, a.rows_x) : none;
      }
    }
    if constexpr (!VECTOR) {
#pragma unroll
      for (int t = 0; t < kRun / 32; ++t) {
        const int k = k0 + lane + 64 * (t >> 1), left = e.N - 8 * (t & 1);
        f.x[t] = k < a.K && left > 0 ? draw_eight(a.X + k * a.ldx + 8 * (t & 1), left, a.rows_x) : none;
      }
    }
  };
  f32x4 acc[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) acc[b] = f32x4{0, 0, 0, 0};
  uint8_t* const place = places[wave];
  auto multiply = [&](Run& f) __attribute__((always_inline)) {
    u32x4 x[kSteps];
    asm volatile("" ::: "memory");  // LDS operations of a wave are done in order; the compiler is held to it
    if constexpr (!PIECES) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        *reinterpret_cast<u32x4*>(place + kTurnedX + (4 * s + g) * kRun * 2 + 16 * (r ^ (4 * s + g))) = f.w[0][s];
    }
    if constexpr (!VECTOR) {
#pragma unroll
      for (int t = 0; t < kRun / 32; ++t)
        *reinterpret_cast<u32x4*>(place + (lane + 64 * (t >> 1)) * kTokens * 2 + 16 * (t & 1)) = place_eight(f.x[t], e.N - 8 * (t & 1), a.rows_x);
    }
    asm volatile("" ::: "memory");
    if constexpr (!PIECES) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) f.w[0][s] = *reinterpret_cast<const u32x4*>(place + kTurnedX + r * kRun * 2 + 16 * ((4 * s + g) ^ r));
    }
    if constexpr (VECTOR) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) x[s] = f.x[s];
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const uint8_t* from = place + (32 * s + 8 * g + (r >> 2)) * kTokens * 2 + 8 * (r & 3);
        const u32x2 low = lds_read_tr16(from), high = lds_read_tr16(from + 4 * kTokens * 2);
        x[s] = u32x4{low[0], low[1], high[0], high[1]};
      }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int b = 0; b < RB; ++b) acc[b] = mfma_16x16x32<DT>(x[s], f.w[b][s], acc[b]);
  };
  Run f;
  if (wave < runs) {
    load(wave, f);
    int run = wave;
    for (; run + WAVES < runs; run += WAVES) {
      Run next;
      load(run + WAVES, next);
      multiply(f);
      f = next;
    }
    multiply(f);
  }
  // a lane holds rows 16 b + lane % 16, tokens 4 (lane / 16) + 0 .. 3
  auto sums = [&](int q) __attribute__((always_inline)) { return reinterpret_cast<float*>(places[q]); };
  asm volatile("" ::: "memory");
#pragma unroll
  for (int b = 0; b < RB; ++b) *reinterpret_cast<f32x4*>(sums(wave) + (16 * b + r) * kPitch + 4 * g) = acc[b];
  __syncthreads();
  const int count = min(WAVES, runs);
  for (int i = threadIdx.x; i < kFewRows * kTokens; i += 64 * WAVES) {
    const int at = i / kTokens * kPitch + i % kTokens;
    float v = sums(0)[at];
    for (int q = 1; q < count; ++q) v += sums(q)[at];
    sums(0)[at] = v;
  }
  __syncthreads();
  const int row = threadIdx.x >> 1, n = 8 * (threadIdx.x & 1), m = m0 + row, left = e.N - n;
  if (row >= kFewRows || m >= e.M || left <= 0) return;
  u32x4 residual = none;
  if (e.residual) residual = draw_residual(e, m, n, min(left, 8));
  const float b = e.bias ? e.bias[m] : 0.0f;
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = sums(0)[row * kPitch + n + j] + b;
  finish_eight<DT, E, false>(e, m, n, min(left, 8), residual, v);
}

template <int DT, Epilogue E, bool VECTOR, bool PIECES, int RB, int WAVES>
hipError_t launch_few_as(const DenseProduct& d, const FewArgs& a, hipStream_t stream) {
  const dim3 grid(grid_of_items(((int64_t)d.M + 16 * RB - 1) / (16 * RB)));
  if (d.plan) {
    plan_record(d.plan, "linear_few_kernel<DT=%d,E=%d,VECTOR=%d,PIECES=%d,RB=%d,WAVES=%d> grid=%u block=%d", DT, (int)E, (int)VECTOR, (int)PIECES, RB, WAVES, grid.x, 64 * WAVES);
    return hipSuccess;
  }
  linear_few_kernel<DT, E, VECTOR, PIECES, RB, WAVES><<<grid, 64 * WAVES, 0, stream>>>(a, d.to);
  return hipGetLastError();
}
template <int DT, Epilogue E>
hipError_t launch_few_tokens(const DenseProduct& d, hipStream_t stream) {
  const bool vector = d.N == 1 && d.ldb == 1;
  const FewArgs a{static_cast<const uint16_t*>(d.A), d.lda, static_cast<const uint16_t*>(d.B), d.ldb, d.K, pieces_of_rows(d.A, d.lda, d.K),
                  vector ? pieces_of_rows(d.B, 8, d.K) : pieces_of_rows(d.B, d.ldb, d.N)};
  if (a.rows_w != kAligned) return vector ? launch_few_as<DT, E, true, false, 1, 8>(d, a, stream) : launch_few_as<DT, E, false, false, 1, 8>(d, a, stream);
  if (vector) return launch_few_as<DT, E, true, true, 1, 16>(d, a, stream);
  // More rows share what a workgroup draws of X, which every workgroup draws, where they are many enough to fill the chip all
  // the same: 16384x16384 of 16 tokens 121 us with 16 rows and 98 with 64, 11008x4096 27.6 and 22.9, 4096x11008 25.4 and 50.7.
  return (d.M + 63) / 64 >= 160 ? launch_few_as<DT, E, false, true, 4, 16>(d, a, stream) : launch_few_as<DT, E, false, true, 1, 16>(d, a, stream);
}
template <int DT>
hipError_t launch_few_dtype(const DenseProduct& d, hipStream_t stream) {
  switch (epilogue_of(d.to.act)) {
    case kEpiGelu: return launch_few_tokens<DT, kEpiGelu>(d, stream);
    case kEpiSigmoid: return launch_few_tokens<DT, kEpiSigmoid>(d, stream);
    default: return launch_few_tokens<DT, kEpiLinear>(d, stream);
  }
}

// The weights' gradient of up to 32 tokens: dW = dZ X^T in one step of the instruction, bound by dW's bytes, which leave straight from
// registers.  A wave owns 64 rows and 128 columns, a workgroup 512 columns; there is nothing in LDS and nothing to wait for but
// the first loads.  X is the row operand, its rows in such an order that a lane ends with eight consecutive columns: row
// i of instruction t is column 8 (i / 4) + 4 t + i % 4 of 32.  11008x4096 of 16 tokens 18.8 us (4.8 TB/s; in tiles of 256 through LDS 32.0),
// 4096x4096 of 16 9.8 (13.8), 5482x5960 of 3 15.9 (28.3).
constexpr int kOuterRows = 64, kOuterColumns = 128;
template <int DT>
__global__ __launch_bounds__(256) void linear_outer_kernel(FewArgs a, LinearEpilogue e) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int across = (e.N + 4 * kOuterColumns - 1) / (4 * kOuterColumns);
  const int item = item_of_workgroup((e.M + kOuterRows - 1) / kOuterRows * across);
  if (item < 0) return;
  const int m0 = item / across * kOuterRows, k0 = (item % across * 4 + wave) * kOuterColumns, left = a.K - 8 * g;
  if (k0 >= e.N) return;
  constexpr int kBlocks = kOuterRows / 16, kParts = kOuterColumns / 32;
  const u32x4 none = {0, 0, 0, 0};
  u32x4 z[kBlocks], x[kParts][2];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) z[b] = left > 0 ? draw_eight(a.W + min(m0 + 16 * b + r, e.M - 1) * a.ldw + 8 * g, left, a.rows_w) : none;
#pragma unroll
  for (int s = 0; s < kParts; ++s)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int k = k0 + 32 * s + 8 * (r >> 2) + 4 * t + (r & 3);
      x[s][t] = left > 0 && k < e.N ? draw_eight(a.X + k * a.ldx + 8 * g, left, a.rows_x) : none;
    }
  if (left > 0) {
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) z[b] = trim_eight(z[b], left, a.rows_w);
#pragma unroll
    for (int s = 0; s < kParts; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) x[s][t] = trim_eight(x[s][t], left, a.rows_x);
  }
  auto store = [&](auto whole_tag) __attribute__((always_inline)) {
    constexpr bool kWhole = decltype(whole_tag)::value;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int s = 0; s < kParts; ++s) {
        const f32x4 zero = {0, 0, 0, 0}, low = mfma_16x16x32<DT>(x[s][0], z[b], zero), high = mfma_16x16x32<DT>(x[s][1], z[b], zero);
        float v[8] = {low[0], low[1], low[2], low[3], high[0], high[1], high[2], high[3]};
        const int m = m0 + 16 * b + r, n = k0 + 32 * s + 8 * g;
        if (kWhole || (m < e.M && n < e.N)) finish_eight<DT, kEpiBare, kWhole>(e, m, n, min(e.N - n, 8), none, v);
      }
  };
  if (!e.out_f32 && m0 + kOuterRows <= e.M && k0 + kOuterColumns <= e.N) store(std::true_type{});
  else store(std::false_type{});
}

template <int DT>
hipError_t launch_outer(const DenseProduct& d, hipStream_t stream) {
  const FewArgs a{static_cast<const uint16_t*>(d.A), d.lda, static_cast<const uint16_t*>(d.B), d.ldb, d.K, pieces_of_rows(d.A, d.lda, d.K),
                  pieces_of_rows(d.B, d.ldb, d.K)};
  const dim3 grid(grid_of_items(((int64_t)d.M + kOuterRows - 1) / kOuterRows * ((d.N + 4 * kOuterColumns - 1) / (4 * kOuterColumns))));
  if (d.plan) {
    plan_record(d.plan, "linear_outer_kernel<DT=%d> grid=%u block=256", DT, grid.x);
    return hipSuccess;
  }
  linear_outer_kernel<DT><<<grid, 256, 0, stream>>>(a, d.to);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_outer(const DenseProduct& d, hipStream_t stream) {
  return d.dtype == HINM_F16 ? launch_outer<HINM_F16>(d, stream) : launch_outer<HINM_BF16>(d, stream);
}
hipError_t launch_linear_few(const DenseProduct& d, hipStream_t stream) {
  return d.dtype == HINM_F16 ? launch_few_dtype<HINM_F16>(d, stream) : launch_few_dtype<HINM_BF16>(d, stream);
}

}  // namespace hinm
