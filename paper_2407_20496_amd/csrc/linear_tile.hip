// Dense products of two 16-bit matrices on the matrix cores, tiles through LDS (include/hinm.h, hinm_linear and its gradients).
#include "linear_tile.h"

#include <algorithm>
#include <utility>

#include "column_strips.h"
#include "direct_lds.h"
#include "lds_in_flight.h"
#include "wave_reduce.h"
#include "workgroup_items.h"

namespace hinm {

namespace {

struct TileArgs {
  const uint16_t* A;
  int64_t lda;
  const uint16_t* B;
  int64_t ldb;
  int K;
  int whole_tiles;              // that one workgroup each has; the others are shared by `splits`, with so many stages each
  int splits, stages_of_split;
  Pieces rows_a, rows_b;
  float* partials;  // of workgroups that share a tile
};

// A stage of one operand in LDS: T rows (or columns) of the result, BK values that are summed over, in pieces of 16 bytes.
// Along: T LDS rows of BK values; across: BK LDS rows of T values, from which transposing reads draw.  A piece's place in its
// row is exchanged by a key of the row, so that the rows a read touches at a time lie on different banks: 16 rows of a
// fragment at pitches of 128 or 64 bytes; four rows, 64 bytes of each, for a transposing read.
template <int T, int BK, OperandForm F>
struct OperandStage {
  static constexpr int kRowBytes = F == kAlong ? 2 * BK : 2 * T;
  static constexpr int kBytes = 2 * T * BK;
  static constexpr int kCopies = kBytes / 1024;  // of a wave: 64 pieces
  static_assert(BK == 64 || BK == 32, "keys of rows");
  static_assert(T == 32 || T == 64 || T == 128 || T == 256, "keys of rows");

  // of pieces along, of 32-byte units across
  static __device__ __forceinline__ int key(int row) {
    if constexpr (F == kAlong) return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
    return T >= 128 ? swizzle_of_row(row) : T == 64 ? row & 2 : 0;
  }
  // The piece of the stage that lies at copy c, lane l: its LDS row, and its first value in the row.
  static __device__ __forceinline__ void piece_of(int c, int lane, int& row, int& value) {
    const int at = 1024 * c + 16 * lane;
    row = at / kRowBytes;
    const int place = at % kRowBytes / 16;
    if constexpr (F == kAlong) value = 8 * (place ^ key(row));
    else value = 8 * ((((place >> 1) ^ key(row)) << 1) | (place & 1));
  }
  // Zeros behind a stage's end within a piece: what a row holds there is not a number of the sum.
  static __device__ __forceinline__ void clear_behind(uint8_t* stage, int left_k, int threads) {
    for (int row = threadIdx.x; row < T; row += threads) {
      u32x4* const piece = reinterpret_cast<u32x4*>(stage + row * kRowBytes + ((left_k >> 3) ^ key(row)) * 16);
      *piece = trim_eight(*piece, left_k & 7, kAligned);
    }
  }
};

constexpr uint32_t kWholeBuffer = 0x7fffffffu;  // offsets into it stay within the matrix by themselves
constexpr uint32_t kNowhere = 0x80000000u;      // beyond it

// One operand of a workgroup: where its pieces come from.
template <int T, int BK, OperandForm F, int COPIES>  // copies of this wave
struct OperandSource {
  using S = OperandStage<T, BK, F>;
  const uint16_t* base;  // the tile's first value at the first k
  int64_t ld;
  int first_copy;
  uint32_t from[COPIES];  // bytes from a stage's first value, for whole stages

  __device__ __forceinline__ void init(const uint16_t* matrix, int64_t ld_, int tile0, int size, int k0, int wave_copy, int lane) {
    ld = ld_;
    base = F == kAlong ? matrix + tile0 * ld + k0 : matrix + k0 * ld + tile0;
    first_copy = wave_copy;
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      int row, value;
      S::piece_of(first_copy + c, lane, row, value);
      // beyond the result's rows and columns the tile's last row, or its first columns, repeat: what they give is not stored
      if constexpr (F == kAlong) row = min(row, size - 1 - tile0);
      else value = tile0 + value < size ? value : 0;
      from[c] = (uint32_t)((row * ld + value) * 2);
    }
  }
  __device__ __forceinline__ const uint16_t* of_stage(int stage) const {
    return base + (F == kAlong ? (int64_t)stage * BK : (int64_t)stage * BK * ld);
  }
  // straight into LDS
  __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t stage, int c, uint8_t* to) const {
    copy16_to_lds(stage, from[c], 0, to + 1024 * (first_copy + c));
  }
  // From here on a stage that ends early: what lies beyond its end is beyond the buffer's, and zeros are written.
  __device__ __forceinline__ void cut(int lane, int left_k) {
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      int row, value;
      S::piece_of(first_copy + c, lane, row, value);
      if ((F == kAlong ? value : row) >= left_k) from[c] = kNowhere;
    }
  }
  // ... or through registers, where rows lie at any address: drawn, then trimmed
  __device__ __forceinline__ u32x4 draw(int stage, int c, int lane, int left_k, int tile0, int size, Pieces rows, int& valid) const {
    int row, value;
    S::piece_of(first_copy + c, lane, row, value);
    if constexpr (F == kAlong) {
      row = min(row, size - 1 - tile0);
      valid = left_k - value;
    } else {
      valid = row < left_k ? size - tile0 - value : 0;
    }
    return valid > 0 ? draw_eight(of_stage(stage) + row * ld + value, valid, rows) : u32x4{0, 0, 0, 0};
  }
};

// 32 rows of a wave's part of a tile to the result, from their registers.  acc[i]: columns 32 i .. of the wave; a lane holds row
// lane % 32, columns 8 q + 4 (lane / 32) + 0 .. 3 in four registers of each q.  The halves of a wave exchange every second four: a
// lower lane then holds columns 8 q .. 8 q + 7, its partner above those of q + 1, whole pieces of 16 bytes.  (By way of LDS, in
// pieces of whole lines, a wave of four tiles each way took 29000 clocks for what takes some 6000 here.)
// ACCUMULATION: the sums stand in accumulation registers, and leave them when their turn comes (the compiler would move all of
// them at once, and spill).
template <bool ACCUMULATION>
__device__ __forceinline__ float taken(float sum) {
  if constexpr (ACCUMULATION) {
    float v;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(sum));
    return v;
  }
  return sum;
}
template <int WN, bool ACCUMULATION>
struct RowStore {
  u32x4 residual[2 * WN];

  // the residual's pieces, under way ahead of their sums
  template <bool WHOLE>
  __device__ __forceinline__ void draw(const LinearEpilogue& e, int m0, int n0) {
    if (!e.residual) return;
    const int lane = threadIdx.x & 63, m = m0 + (lane & 31);
#pragma unroll
    for (int t = 0; t < 2 * WN; ++t) {
      const int n = n0 + 16 * t + 8 * (lane >> 5), left = e.N - n;
      if (WHOLE) residual[t] = draw_residual(e, m, n, 8);
      else residual[t] = m < e.M && left > 0 ? draw_residual(e, m, n, left) : u32x4{0, 0, 0, 0};
    }
  }
  template <int DT, Epilogue E, bool WHOLE>
  __device__ __forceinline__ void store(const f32x16 (&acc)[WN], float bias, int m0, int n0, const LinearEpilogue& e) {
    const int lane = threadIdx.x & 63, m = m0 + (lane & 31);
#pragma unroll
    for (int t = 0; t < 2 * WN; ++t) {
      float v[8];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t a = __builtin_bit_cast(uint32_t, taken<ACCUMULATION>(acc[t >> 1][8 * (t & 1) + c]) + bias);
        uint32_t b = __builtin_bit_cast(uint32_t, taken<ACCUMULATION>(acc[t >> 1][8 * (t & 1) + 4 + c]) + bias);
        swap_lanes<32>(a, b);
        v[c] = __builtin_bit_cast(float, a);
        v[4 + c] = __builtin_bit_cast(float, b);
      }
      const int n = n0 + 16 * t + 8 * (lane >> 5), left = e.N - n;
      if (WHOLE || (m < e.M && left > 0)) finish_eight<DT, E, WHOLE>(e, m, n, left, residual[t], v);
    }
  }
};
// The bias of the row that a lane holds of 32.
template <Epilogue E>
__device__ __forceinline__ float bias_of_row(const LinearEpilogue& e, int m0) {
  const int m = m0 + (threadIdx.x & 31);
  return E != kEpiBare && e.bias && m < e.M ? e.bias[m] : 0.0f;
}

template <OperandForm FA, OperandForm FB, int WM, int WN, int GM, int GN, int BK, int RING>
struct TileSizes {
  static constexpr int kWaves = GM * GN, kThreads = 64 * kWaves;
  static constexpr int TM = 32 * WM * GM, TN = 32 * WN * GN;
  using StageA = OperandStage<TM, BK, FA>;
  using StageB = OperandStage<TN, BK, FB>;
  static constexpr int kStageBytes = StageA::kBytes + StageB::kBytes;
  static constexpr int kCopiesA = StageA::kCopies / kWaves, kCopiesB = StageB::kCopies / kWaves, kCopies = kCopiesA + kCopiesB;
  static constexpr int kLds = RING * kStageBytes;
  static_assert(StageA::kCopies % kWaves == 0 && StageB::kCopies % kWaves == 0, "whole copies for every wave");
  static_assert(RING >= 2 && (RING - 2) * kCopies + kCopies / 2 < 64 && kLds <= 160 * 1024, "copies in flight are counted; LDS of a unit");
};

// Which tile an item of the list is: panels of eight tiles of rows times all columns, so that the tiles an XCD works on at a time
// share operands.
struct TilePlace {
  int m0, n0;
  __device__ __forceinline__ TilePlace(int tile, int TM, int TN, int M, int N) {
    const int tiles_m = (M + TM - 1) / TM, tiles_n = (N + TN - 1) / TN;
    const int panel = tile / (8 * tiles_n), in_panel = tile - panel * 8 * tiles_n;
    const int height = min(8, tiles_m - 8 * panel);
    m0 = (8 * panel + in_panel % height) * TM;
    n0 = in_panel / height * TN;
  }
};

// A workgroup of GM x GN waves owns TM rows and TN columns of the result; a wave owns 32 WM x 32 WN of them.  A stage is BK
// values of the summed axis; RING of them lie in LDS in turn.  A step is 16 of these values: WM WN matrix instructions; a wave
// reads the operands of the next step while it multiplies, one read between two instructions.  B is the instruction's row
// operand, so that a lane ends with four consecutive columns of the result.
//   Waits: copies of a wave land in order.  Before the last step of stage p those of stages p + 2 .. p + RING - 1 may be
// outstanding, all earlier ones are waited for, and so are the wave's LDS reads of stage p; past the barrier that holds for all
// waves, so stage p + 1 is there and the place of stage p takes stage p + RING: half of its copies during the last step of p, the
// others during the first of p + 1.
//   What bounds it, at rates of bf16: tiles of 256 the power (16384x16384 of 8192 columns 3.47 ms, 1270 TFLOP/s: matrix units busy 74 % of the
// clocks at 1.6 GHz, some 2700 a stage for 2048 of products; 8192x8192 of 8192 0.81 to 0.86 ms, 1280 to 1360).  Tiles of 256x128 and 128 with few
// workgroups the LDS: 0.63 and 0.32 us a stage, whose reads (98 and 66 KB) and copies (49 and 33 KB) take 0.48 and 0.32 at 128 bytes a clock of
// 2.4 GHz.  On a full chip such a stage takes 0.95 and 0.60 us (11008x4096 of 1571 columns 164 us, 863 TFLOP/s; 4096x4096 of 2048 columns 67 us,
// 1025, matrix units busy 46 %): the LDS moves some 75 of its 128 bytes a clock then, the copies draw 13 TB/s from the L2s, and what holds them
// (these, or the waits between waves) was not taken apart.  Small products: a start of 2.5 to 3 us, the first stage's way from memory.
template <int DT, OperandForm FA, OperandForm FB, Epilogue E, int WM, int WN, int GM, int GN, int BK, int RING, bool GUARDED>
__device__ __forceinline__ void multiply_tile(const TileArgs& a, const LinearEpilogue& e, int group, int groups) {
  using T = TileSizes<FA, FB, WM, WN, GM, GN, BK, RING>;
  constexpr int kSteps = BK / 16;
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = ((e.M + T::TM - 1) / T::TM) * ((e.N + T::TN - 1) / T::TN), shared = tiles - a.whole_tiles;
  const int whole_groups = (a.whole_tiles + 7) & ~7;
  const bool alone = group < whole_groups;
  const int item = alone ? item_of(group, whole_groups, a.whole_tiles) : item_of(group - whole_groups, groups - whole_groups, shared * a.splits);
  if (item < 0) return;
  const int split = alone ? 0 : item / shared, tile = alone ? item : a.whole_tiles + item - split * shared;
  const TilePlace place(tile, T::TM, T::TN, e.M, e.N);
  const int all_stages = (a.K + BK - 1) / BK, first = split * a.stages_of_split;
  const int stages = alone ? all_stages : min(a.stages_of_split, all_stages - first), k0 = first * BK;
  // stages that copies fill; the last one of all may be cut short
  const int whole = GUARDED ? 0 : min(stages, a.K / BK - first);

  OperandSource<T::TM, BK, FA, T::kCopiesA> of_a;
  OperandSource<T::TN, BK, FB, T::kCopiesB> of_b;
  of_a.init(a.A, a.lda, place.m0, e.M, k0, wave * T::kCopiesA, lane);
  of_b.init(a.B, a.ldb, place.n0, e.N, k0, wave * T::kCopiesB, lane);
  struct Buffers {
    __amdgpu_buffer_rsrc_t a, b;
  };
  auto buffers_of = [&](int stage) __attribute__((always_inline)) {
    const uint32_t bytes = stage < stages ? kWholeBuffer : 0;  // a stage that does not exist: zeros, which nobody reads
    return Buffers{buffer_of(of_a.of_stage(stage), bytes), buffer_of(of_b.of_stage(stage), bytes)};
  };
  // places of the ring, as bytes from its beginning
  auto place_after = [](uint32_t place) { return place == (RING - 1) * T::kStageBytes ? 0u : place + T::kStageBytes; };
  auto place_before = [](uint32_t place) { return place == 0 ? (RING - 1) * T::kStageBytes : place - T::kStageBytes; };
  auto copy_one = [&](const Buffers& from, uint32_t place, int c) __attribute__((always_inline)) {
    if (c < T::kCopiesA) of_a.copy(from.a, c, lds + place);
    else of_b.copy(from.b, c - T::kCopiesA, lds + place + T::StageA::kBytes);
  };
  // stages through registers
  struct Held {
    u32x4 v[T::kCopies];
  };
  auto draw_stage = [&](int stage, Held& h) __attribute__((always_inline)) {
    const int left_k = a.K - k0 - stage * BK;
#pragma unroll
    for (int c = 0; c < T::kCopies; ++c) {
      int valid;
      h.v[c] = c < T::kCopiesA ? of_a.draw(stage, c, lane, left_k, place.m0, e.M, a.rows_a, valid)
                               : of_b.draw(stage, c - T::kCopiesA, lane, left_k, place.n0, e.N, a.rows_b, valid);
    }
  };
  auto put_stage = [&](int stage, uint32_t place_of_it, const Held& h) __attribute__((always_inline)) {
    const int left_k = a.K - k0 - stage * BK;
    uint8_t* const slot = lds + place_of_it;
#pragma unroll
    for (int c = 0; c < T::kCopies; ++c) {
      const bool is_a = c < T::kCopiesA;
      int row, value, valid;
      uint8_t* to;
      if (is_a) {
        T::StageA::piece_of(of_a.first_copy + c, lane, row, value);
        valid = FA == kAlong ? left_k - value : row < left_k ? e.M - place.m0 - value : 0;
        to = slot + 1024 * (of_a.first_copy + c);
      } else {
        T::StageB::piece_of(of_b.first_copy + c - T::kCopiesA, lane, row, value);
        valid = FB == kAlong ? left_k - value : row < left_k ? e.N - place.n0 - value : 0;
        to = slot + T::StageA::kBytes + 1024 * (of_b.first_copy + c - T::kCopiesA);
      }
      *reinterpret_cast<u32x4*>(to + 16 * lane) = valid > 0 ? trim_eight(h.v[c], valid, is_a ? a.rows_a : a.rows_b) : u32x4{0, 0, 0, 0};
    }
  };

  // the last stage where it is cut short is cleared behind its end once it is there
  const int left_k = a.K - k0 - whole * BK;
  auto cut_offsets = [&]() __attribute__((always_inline)) {
    of_a.cut(lane, left_k);
    of_b.cut(lane, left_k);
  };
  auto clear_cut_stage = [&](uint32_t at) __attribute__((always_inline)) {
    if ((FA == kAcross && FB == kAcross) || whole == stages || !(left_k & 7)) return;
    if constexpr (FA == kAlong) T::StageA::clear_behind(lds + at, left_k, T::kThreads);
    if constexpr (FB == kAlong) T::StageB::clear_behind(lds + at + T::StageA::kBytes, left_k, T::kThreads);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  const int wave_m = (wave % GM) * 32 * WM, wave_n = (wave / GM) * 32 * WN;
  float bias[WM];
#pragma unroll
  for (int j = 0; j < WM; ++j) bias[j] = bias_of_row<E>(e, place.m0 + wave_m + 32 * j);

  // LDS reads: by step along, by tile of 32 across
  const int half = lane >> 5, r = lane & 31, in16 = lane & 15;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  constexpr int kAddressesA = FA == kAlong ? kSteps : WM, kAddressesB = FB == kAlong ? kSteps : WN;
  uint32_t at_a[kAddressesA], at_b[kAddressesB];
#pragma unroll
  for (int i = 0; i < kAddressesA; ++i)
    at_a[i] = lds_base + (FA == kAlong ? (wave_m + r) * T::StageA::kRowBytes + ((2 * i + half) ^ T::StageA::key(r)) * 16
                                       : (8 * half + (in16 >> 2)) * T::StageA::kRowBytes +
                                             (((wave_m + 32 * i) / 16 + ((lane >> 4) & 1)) ^ T::StageA::key(in16 >> 2)) * 32 + (in16 & 3) * 8);
#pragma unroll
  for (int i = 0; i < kAddressesB; ++i)
    at_b[i] = lds_base + T::StageA::kBytes +
              (FB == kAlong ? (wave_n + r) * T::StageB::kRowBytes + ((2 * i + half) ^ T::StageB::key(r)) * 16
                            : (8 * half + (in16 >> 2)) * T::StageB::kRowBytes +
                                  (((wave_n + 32 * i) / 16 + ((lane >> 4) & 1)) ^ T::StageB::key(in16 >> 2)) * 32 + (in16 & 3) * 8);
  // the operands of a step while their reads are in flight: one read each along, two across
  struct Operands {
    u32x4 a[WM], b[WN];
    uint64_t part_a[WM][2], part_b[WN][2];
  };
  auto read_one = [&](auto step_tag, auto tile_tag, uint32_t slot, Operands& f) __attribute__((always_inline)) {
    constexpr int s = decltype(step_tag)::value, t = decltype(tile_tag)::value;
    if constexpr (t < WM) {
      if constexpr (FA == kAlong) {
        lds_read_b128<t * 32 * T::StageA::kRowBytes>(at_a[s] + slot, f.a[t]);
      } else {
        lds_read_tr16<16 * s * T::StageA::kRowBytes>(at_a[t] + slot, f.part_a[t][0]);
        lds_read_tr16<(16 * s + 4) * T::StageA::kRowBytes>(at_a[t] + slot, f.part_a[t][1]);
      }
    } else {
      constexpr int u = t - WM;
      if constexpr (FB == kAlong) {
        lds_read_b128<u * 32 * T::StageB::kRowBytes>(at_b[s] + slot, f.b[u]);
      } else {
        lds_read_tr16<16 * s * T::StageB::kRowBytes>(at_b[u] + slot, f.part_b[u][0]);
        lds_read_tr16<(16 * s + 4) * T::StageB::kRowBytes>(at_b[u] + slot, f.part_b[u][1]);
      }
    }
  };
  auto wait_operands = [&](Operands& f) __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)");
    typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
    if constexpr (FA == kAlong) {
#pragma unroll
      for (int t = 0; t < WM; ++t) pin(f.a[t]);
    } else {
#pragma unroll
      for (int t = 0; t < WM; ++t) {
        pin(f.part_a[t][0]);
        pin(f.part_a[t][1]);
        f.a[t] = __builtin_bit_cast(u32x4, (u64x2{f.part_a[t][0], f.part_a[t][1]}));
      }
    }
    if constexpr (FB == kAlong) {
#pragma unroll
      for (int t = 0; t < WN; ++t) pin(f.b[t]);
    } else {
#pragma unroll
      for (int t = 0; t < WN; ++t) {
        pin(f.part_b[t][0]);
        pin(f.part_b[t][1]);
        f.b[t] = __builtin_bit_cast(u32x4, (u64x2{f.part_b[t][0], f.part_b[t][1]}));
      }
    }
  };

  f32x16 acc[WN][WM];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;

  // the first stages, of the last one half: the other half follows in the first step
  Held held;
  constexpr int kHalf = T::kCopies / 2;
  // Small tiles: a step's products do not cover the way through LDS, so a wave holds the operands of a whole stage and reads those
  // of the next one meanwhile.
  constexpr bool kWholeStages = !GUARDED && WM * WN <= 4;
  if constexpr (GUARDED) {
    for (int q = 0; q < min(RING, stages); ++q) {
      draw_stage(q, held);
      put_stage(q, q * T::kStageBytes, held);
    }
    if (RING < stages) draw_stage(RING, held);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  } else {
#pragma unroll
    for (int q = 0; q < RING; ++q) {
      if (q == whole) cut_offsets();
      const Buffers from = buffers_of(q);
#pragma unroll
      for (int c = 0; c < (kWholeStages || q < RING - 1 ? T::kCopies : kHalf); ++c) copy_one(from, q * T::kStageBytes, c);
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kWholeStages ? (RING - 1) * T::kCopies : (RING - 2) * T::kCopies + kHalf) : "memory");
  }
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if (!GUARDED && whole == 0) clear_cut_stage(0);

  uint32_t at = 0;  // the place of stage p, and of stage p + RING
  Operands sets[kWholeStages ? 2 * kSteps : 2];
  if constexpr (kWholeStages) {
    // The barrier stands ahead of a stage's products: past it every wave has read the stage, whose place takes stage p + RING, and
    // stage p + 1 is there.
    unroll<0, kSteps>([&](auto s) __attribute__((always_inline)) {
      unroll<0, WM + WN>([&](auto t) __attribute__((always_inline)) { read_one(s, t, 0, sets[decltype(s)::value]); });
    });
    auto stage = [&](auto odd_tag, int p) __attribute__((always_inline)) {
      constexpr int now = decltype(odd_tag)::value ? kSteps : 0, next = kSteps - now;
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((RING - 2) * T::kCopies) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const uint32_t after = place_after(at);
      if (p + RING == whole) cut_offsets();
      if (p + 1 == whole) clear_cut_stage(after);
      const Buffers from = buffers_of(p + RING);
      unroll<0, kSteps>([&](auto step_tag) __attribute__((always_inline)) {
        constexpr int s = decltype(step_tag)::value, kTiles = WM * WN, kReads = WM + WN;
        constexpr int c0 = s * T::kCopies / kSteps, c1 = (s + 1) * T::kCopies / kSteps;
        unroll<0, kTiles>([&](auto t_tag) __attribute__((always_inline)) {
          constexpr int t = decltype(t_tag)::value, i = t / WM, j = t % WM;
          acc[i][j] = mfma_32x32x16<DT>(sets[now + s].b[i], sets[now + s].a[j], acc[i][j]);
          __builtin_amdgcn_sched_barrier(0);
          // all reads of the next stage during three quarters of the products, waited for behind the last
          constexpr int kAll = kSteps * kReads, kOver = kSteps * kTiles * 3 / 4, n = s * kTiles + t;
          constexpr int r0 = n * kAll / kOver, r1 = (n + 1) * kAll / kOver;
          unroll<(r0 < kAll ? r0 : kAll), (r1 < kAll ? r1 : kAll)>([&](auto u) __attribute__((always_inline)) {
            constexpr int v = decltype(u)::value;
            read_one(std::integral_constant<int, v / kReads>{}, std::integral_constant<int, v % kReads>{}, after, sets[next + v / kReads]);
          });
#pragma unroll
          for (int c = c0 + t * (c1 - c0) / kTiles; c < c0 + (t + 1) * (c1 - c0) / kTiles; ++c) copy_one(from, at, c);
          __builtin_amdgcn_sched_barrier(0);
        });
      });
      at = after;
      unroll<0, kSteps>([&](auto s) __attribute__((always_inline)) { wait_operands(sets[next + decltype(s)::value]); });
    };
    unroll<0, kSteps>([&](auto s) __attribute__((always_inline)) { wait_operands(sets[decltype(s)::value]); });
    int p = 0;
    for (; p + 2 <= stages; p += 2) {
      stage(std::false_type{}, p);
      stage(std::true_type{}, p + 1);
    }
    if (p < stages) stage(std::false_type{}, p);
  } else {
    unroll<0, WM + WN>([&](auto t) { read_one(std::integral_constant<int, 0>{}, t, 0, sets[0]); });

    for (int p = 0; p < stages; ++p) {
      const uint32_t after = place_after(at), before = place_before(at);
      unroll<0, kSteps>([&](auto step_tag) __attribute__((always_inline)) {
        constexpr int s = decltype(step_tag)::value;
        constexpr bool kEnds = s == kSteps - 1, kCopying = !GUARDED && (s == 0 || kEnds);
        constexpr int kTiles = WM * WN, kReads = WM + WN, kCount = kEnds ? kHalf : T::kCopies - kHalf;
        Operands &now = sets[s & 1], &next = sets[(s + 1) & 1];
        wait_operands(now);
        if constexpr (kEnds) {
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(GUARDED ? 0 : (RING - 2) * T::kCopies) : "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          if constexpr (GUARDED) {
            if (p + RING < stages) put_stage(p + RING, at, held);
            if (p + RING + 1 < stages) draw_stage(p + RING + 1, held);
          } else {
            if (p + RING == whole) cut_offsets();
            if (p + 1 == whole) clear_cut_stage(after);
          }
        }
        const Buffers from = buffers_of(kEnds ? p + RING : p + RING - 1);
        unroll<0, kTiles>([&](auto t_tag) __attribute__((always_inline)) {
          constexpr int t = decltype(t_tag)::value, i = t / WM, j = t % WM;
          acc[i][j] = mfma_32x32x16<DT>(now.b[i], now.a[j], acc[i][j]);
          __builtin_amdgcn_sched_barrier(0);
          constexpr int b = t * kReads * 2 / kTiles, to = (t + 1) * kReads * 2 / kTiles;
          unroll<(b < kReads ? b : kReads), (to < kReads ? to : kReads)>([&](auto u) __attribute__((always_inline)) {
            read_one(std::integral_constant<int, (s + 1) % kSteps>{}, u, kEnds ? after : at, next);
          });
          if constexpr (kCopying) {
  #pragma unroll
            for (int c = t * kCount / kTiles; c < (t + 1) * kCount / kTiles; ++c) copy_one(from, kEnds ? at : before, (kEnds ? 0 : kHalf) + c);
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      });
      at = after;
    }
    // what was read of the stage beyond the last one is not used, but has to be there before its registers are
    wait_operands(sets[0]);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // copies of stages that do not exist: they write to this workgroup's LDS

  if (!alone) {
    float* const to = a.partials + (int64_t)item * (T::TM * T::TN) + wave * (WM * WN * 1024) + 4 * lane;
#pragma unroll
    for (int j = 0; j < WM; ++j)
#pragma unroll
      for (int i = 0; i < WN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(to + ((j * WN + i) * 4 + q) * 256) =
              f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    return;
  }
  // the sums are read by instructions that the compiler does not look into: it sees no need to wait for the last products
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
  auto store = [&](auto whole_tag) __attribute__((always_inline)) {
    constexpr bool kWhole = decltype(whole_tag)::value;
    RowStore<WN, (WM * WN > 8)> to[2];
    if constexpr (E != kEpiBare) to[0].template draw<kWhole>(e, place.m0 + wave_m, place.n0 + wave_n);
    unroll<0, WM>([&](auto j_tag) __attribute__((always_inline)) {
      constexpr int j = decltype(j_tag)::value;
      if constexpr (E != kEpiBare && j + 1 < WM) to[(j + 1) & 1].template draw<kWhole>(e, place.m0 + wave_m + 32 * (j + 1), place.n0 + wave_n);
      f32x16 rows[WN];
#pragma unroll
      for (int i = 0; i < WN; ++i) rows[i] = acc[i][j];
      to[j & 1].template store<DT, E, kWhole>(rows, bias[j], place.m0 + wave_m + 32 * j, place.n0 + wave_n, e);
    });
  };
  if (!e.out_f32 && place.m0 + T::TM <= e.M && place.n0 + T::TN <= e.N) store(std::true_type{});
  else store(std::false_type{});
}

template <int DT, OperandForm FA, OperandForm FB, Epilogue E, int WM, int WN, int GM, int GN, int BK, int RING, bool GUARDED>
__global__ __launch_bounds__(64 * GM * GN, WM * WN > 8 ? 1 : 2) void linear_tile_kernel(TileArgs a, LinearEpilogue e) {
  multiply_tile<DT, FA, FB, E, WM, WN, GM, GN, BK, RING, GUARDED>(a, e, blockIdx.x, gridDim.x);
}

// Sums of A's rows (whole pieces), a wave each.
struct RowSums {
  float* to;
  int first;  // workgroup of the launch
};
template <int DT>
__device__ __forceinline__ void add_rows(const TileArgs& a, int M, float* to, int group) {
  const int lane = threadIdx.x & 63, m = 4 * group + (threadIdx.x >> 6);
  if (m >= M) return;
  constexpr int kAtOnce = 4;
  const uint16_t* const row = a.A + m * a.lda;
  float sum = 0;
  for (int k0 = 8 * lane; k0 < a.K; k0 += 512 * kAtOnce) {
    u32x4 v[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int k = k0 + 512 * i;
      v[i] = k < a.K ? trim_eight(*reinterpret_cast<const u32x4*>(row + k), a.K - k, kAligned) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      float x[8];
      widen<DT>(v[i], x);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += x[j];
    }
  }
  sum = add_lanes_by_8(add_eight_lanes(sum));
  if (lane == 0) to[m] = sum;
}

// Both gradients of a layer in one launch: each fills a chip badly alone, and the beginning of one hides the other's end.  The product with
// more stages has the first workgroups; the bias's gradient, where dZ is dY, the last ones (768x768 of 4096 columns: instead of a launch
// of 3 to 4 us ahead).
template <int DT, int WM, int WN>
__global__ __launch_bounds__(256, 2) void linear_pair_kernel(TileArgs w, LinearEpilogue to_w, TileArgs x, LinearEpilogue to_x, int first, bool w_first, RowSums sums) {
  const int block = blockIdx.x;
  if (block >= sums.first) return add_rows<DT>(w, to_w.M, sums.to, block - sums.first);
  const bool in_first = block < first;
  const int group = in_first ? block : block - first, groups = in_first ? first : sums.first - first;
  if (in_first == w_first) multiply_tile<DT, kAlong, kAlong, kEpiBare, WM, WN, 2, 2, 64, 4, false>(w, to_w, group, groups);
  else multiply_tile<DT, kAcross, kAcross, kEpiBare, WM, WN, 2, 2, 64, 4, false>(x, to_x, group, groups);
}

// Tiles that several workgroups have summed parts of: the parts added in order, 32 rows of every wave a workgroup.
template <int DT, Epilogue E, int WM, int WN, int GM, int GN>
__global__ __launch_bounds__(64 * GM * GN) void linear_join_kernel(const float* partials, int whole_tiles, int splits, LinearEpilogue e) {
  constexpr int TM = 32 * WM * GM, TN = 32 * WN * GN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int shared = ((e.M + TM - 1) / TM) * ((e.N + TN - 1) / TN) - whole_tiles;
  const int item = item_of_workgroup(shared * WM);
  if (item < 0) return;
  const int tile = item / WM, j = item - tile * WM;
  const TilePlace place(whole_tiles + tile, TM, TN, e.M, e.N);
  const int m0 = place.m0 + (wave % GM) * 32 * WM + 32 * j, n0 = place.n0 + (wave / GM) * 32 * WN;
  if (m0 >= e.M || n0 >= e.N) return;
  const float* from = partials + (int64_t)tile * (TM * TN) + wave * (WM * WN * 1024) + j * (WN * 1024) + 4 * lane;
  RowStore<WN, false> to;
  if constexpr (E != kEpiBare) to.template draw<false>(e, m0, n0);
  const float bias = bias_of_row<E>(e, m0);
  f32x16 acc[WN];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[i][q] = 0;
#pragma unroll 4
  for (int s = 0; s < splits; ++s, from += (int64_t)shared * (TM * TN)) {
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(from + (i * 4 + q) * 256);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][4 * q + c] += v[c];
      }
  }
  to.template store<DT, E, false>(acc, bias, m0, n0, e);
}

// Which form serves a shape, and by how many workgroups the tiles of its last round are shared: the least of estimates in
// microseconds, fitted to launches at 74 shapes (M, N, K of 128 .. 16384, some from 4 on; operands from memory) with every form and up to
// 16 workgroups a tile.  What they choose is the best of these or at most 11 % behind it.  Both sides of
// each line: 2048x2048 of 2048 columns 22.2 us in tiles of 128, 27.8 of 256x128, 33.4 of 64; 4096x4096 of 2048 67, 82 and 124,
// in tiles of 256 100; of 4096 in those 113 (1208 TFLOP/s); 1024x1024 of 1024 6.9 in tiles of 64, 11.0 of 128; 11008x4096 of 1571
// columns, 559 tiles of 256x128, 162 us with a third round of 47 workgroups and 152 where four share each of its tiles;
// 4096x4096 of 200, 256 tiles of 64 unshared, 21 us; 64 tiles of 128 take 42 alone and 23 in four parts.
struct TileForm {
  int rows, cols, at_once;         // of a tile; workgroups that the chip holds, one or two to a compute unit
  double start;                    // us of a launch and of what does not overlap
  double alone, one_each, full;    // us of a stage: with few workgroups, with one to each unit, with all places taken
  double tile;                     // us of a tile's beginning and end
  double join, join_rate;          // sharing: us of the second launch, MB/us that the parts are written and read at
};
enum { kFormGuarded, kFormLarge, kFormWide, kFormMiddle, kFormSmall, kTileFormCount };
constexpr TileForm kTileForms[kTileFormCount] = {
    {128, 128, 512, 2.9, 1.1, 1.3, 2.3, 3.0, 3.1, 6.5},
    {256, 256, 256, 3.41, 1.172, 1.786, 1.786, 5.88, 2.73, 5.88},
    {256, 128, 256, 2.41, 0.628, 0.955, 0.955, 4.40, 2.50, 7.40},
    {128, 128, 256, 2.95, 0.319, 0.600, 0.600, 2.69, 3.14, 6.52},
    {64, 64, 512, 2.18, 0.179, 0.273, 0.499, 1.63, 2.78, 6.39},
};
constexpr int kUnits = 256;
constexpr int kStage = 64;  // summed values, of every form
constexpr int kShares[] = {2, 3, 4, 6, 8, 12, 16};

int64_t tiles_of(const TileForm& f, int M, int N) { return (int64_t)((M + f.rows - 1) / f.rows) * ((N + f.cols - 1) / f.cols); }
// of a stage with `groups` of at most f.at_once workgroups
double stage_us(const TileForm& f, int64_t groups) {
  // a unit with two decides, so half of the way from one each to all places is taken with the first of them
  return groups <= kUnits ? f.alone + (f.one_each - f.alone) * (double)groups / kUnits
                          : f.one_each + (f.full - f.one_each) * (0.6 + 0.8 * ((double)groups / f.at_once - 0.5));
}
double rounds_us(const TileForm& f, int64_t groups, int stages) {
  const int64_t rounds = groups / f.at_once, left = groups - rounds * f.at_once;
  return (double)rounds * (stages * f.full + f.tile) + (left ? stages * stage_us(f, left) + f.tile : 0);
}
struct TilePlan {
  int form, whole_tiles, splits, stages_of_split;
  double us;
};
TilePlan plan_of(int M, int N, int K, bool guarded) {
  const int stages = (K + kStage - 1) / kStage;
  TilePlan best{};
  double least = 1e300;
  for (int i = guarded ? kFormGuarded : kFormGuarded + 1; i < (guarded ? kFormGuarded + 1 : (int)kTileFormCount); ++i) {
    const TileForm& f = kTileForms[i];
    const int64_t tiles = tiles_of(f, M, N);
    auto take = [&](double us, int64_t whole, int splits, int each) {
      if (us >= least) return;
      least = us;
      best = TilePlan{i, (int)whole, splits, each, us};
    };
    take(f.start + rounds_us(f, tiles, stages), tiles, 1, stages);
    const int64_t whole = tiles / f.at_once * f.at_once, shared = tiles - whole;
    if (shared == 0 || stages < 2) continue;
    for (int splits : kShares) {
      const int each = (stages + splits - 1) / splits, parts = (stages + each - 1) / each;
      const int64_t groups = shared * parts;
      if (parts < 2 || (splits > 2 && groups > 2 * f.at_once)) break;
      const double moved = (double)groups * f.rows * f.cols * 8e-6;  // MB of parts written and read
      take(f.start + rounds_us(f, whole, stages) + rounds_us(f, groups, each) + f.join + moved / f.join_rate, whole, parts, each);
    }
  }
  return best;
}
// Both gradients' products in one launch, no tiles shared: its form by estimates from the same table, or kFormGuarded where two launches
// are sooner.  The longer workgroups begin, the shorter ones take the places beside them, and what is left of the longer ones goes on
// with fewer on the chip.  us of two launches, of one in tiles of 128, in tiles of 64: 768x768 of 4096 columns 24.1, 24.8, 20.1, of 1000
// 13.2, 13.4, 10.1; 256x256 of 64 6.9, 5.8, 3.8; 2304x768 of 512 13.9, 9.6, 10.5; 2048x2048 of 1024 29.8, 22.0, 29.9; 4096x4096 of 256
// 43, 47, 49; 8192x128 of 512 16, 46, 29.  Of 33 such shapes the choice is the best or at most 7 % behind it.
double pair_us(const TileForm& f, int M, int K, int N) {
  int64_t longer = tiles_of(f, M, K), shorter = tiles_of(f, K, N);
  int stages = (N + kStage - 1) / kStage, less = (M + kStage - 1) / kStage;
  if (less > stages) {
    std::swap(longer, shorter);
    std::swap(stages, less);
  }
  const double stage = stage_us(f, std::min<int64_t>(longer + shorter, f.at_once));
  const double long_us = stages * stage + f.tile, short_us = less * stage + f.tile;
  if (longer < f.at_once) {
    const double beside = short_us * std::max(1.0, (double)shorter / (double)(f.at_once - longer));
    if (beside <= long_us) return f.start + beside + (long_us - beside) / stage * stage_us(f, longer);
  }
  return f.start + (longer * long_us + shorter * short_us) / f.at_once + 0.5 * short_us;
}
// the weights' gradient of few tokens by itself
double outer_us(int M, int K) { return 2.5 + 2e-6 / 4.5 * M * K; }
int pair_form(int M, int K, int N) {
  int form = kFormGuarded;
  double least = (N <= kOuterTokens ? outer_us(M, K) : plan_of(M, K, N, false).us) + plan_of(K, N, M, false).us;
  for (int i : {kFormMiddle, kFormSmall}) {
    const double us = pair_us(kTileForms[i], M, K, N);
    if (us < least) {
      least = us;
      form = i;
    }
  }
  return form;
}
size_t partial_bytes(const TilePlan& p, int M, int N) {
  const TileForm& f = kTileForms[p.form];
  return (size_t)p.splits * (tiles_of(f, M, N) - p.whole_tiles) * f.rows * f.cols * sizeof(float);
}

// Rows of A that follow one another at any address (their length is not a multiple of 8) lie apart in the workspace first, in whole
// pieces, where that and the product from there take less than the product through registers: 4095x4095 of 1000 columns 85 us as
// they lie.
struct CopyOfA {
  int rows, row;  // how many, and their length
  int64_t pitch() const { return ((int64_t)row + 7) / 8 * 8; }
  size_t bytes() const { return ((size_t)rows * pitch() * 2 + 255) & ~size_t{255}; }
  double us() const { return 2.5 + 4e-6 / 4.5 * rows * row; }
};
// Weights alone: the other operands have rows of whole pieces where a program uses this package's buffers.
bool may_copy(int M, int K, OperandForm form_a, OperandForm form_b) { return form_b == kAcross && (form_a == kAlong ? K : M) % 8 != 0; }
CopyOfA copy_of(int M, int K, OperandForm form_a) { return form_a == kAlong ? CopyOfA{M, K} : CopyOfA{K, M}; }
__global__ __launch_bounds__(256) void linear_copy_kernel(const uint16_t* from, int64_t ld, uint16_t* to, int64_t pitch, int rows, int row, Pieces pieces) {
  const int per_row = (int)(pitch / 8);
  const int64_t all = (int64_t)rows * per_row, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
    const int r = (int)(i / per_row), at = 8 * (int)(i - (int64_t)r * per_row), left = row - at;
    *reinterpret_cast<u32x4*>(to + r * pitch + at) = trim_eight(draw_eight(from + r * ld + at, left, pieces), left, pieces);
  }
}

// How the operands of a product lie.  Copies into LDS take whole pieces at multiples of 16 bytes, from offsets of 31 bits within a stage.
struct Operands {
  Pieces rows_a, rows_b;
  bool far_a, far_b;
  explicit Operands(const DenseProduct& d)
      : rows_a(pieces_of_rows(d.A, d.lda, d.form_a == kAlong ? d.K : d.M)), rows_b(pieces_of_rows(d.B, d.ldb, d.form_b == kAlong ? d.K : d.N)),
        far_a(d.lda > (1 << 21)), far_b(d.ldb > (1 << 21)) {}
  bool guarded() const { return rows_a != kAligned || rows_b != kAligned || far_a || far_b; }
  TilePlan plan(const DenseProduct& d) const { return plan_of(d.M, d.N, d.K, guarded()); }
  // whether the product is sooner from a copy of A
  bool copies(const DenseProduct& d) const {
    if (rows_a == kAligned || rows_b != kAligned || far_b || !may_copy(d.M, d.K, d.form_a, d.form_b)) return false;
    const CopyOfA c = copy_of(d.M, d.K, d.form_a);
    return c.pitch() <= 1 << 21 && plan_of(d.M, d.N, d.K, false).us + c.us() < plan(d).us;
  }
};

template <int DT, OperandForm FA, OperandForm FB, Epilogue E, int WM, int WN, int GM, int GN, int BK, int RING, bool GUARDED>
hipError_t launch_tiles(const DenseProduct& d, const TileArgs& a, int64_t tiles, hipStream_t stream) {
  using T = TileSizes<FA, FB, WM, WN, GM, GN, BK, RING>;
  const int shared = (int)(tiles - a.whole_tiles);
  const dim3 grid(grid_of_items(a.whole_tiles) + grid_of_items((int64_t)shared * a.splits)), join(grid_of_items((int64_t)shared * WM));
  if (d.plan) {
    plan_record(d.plan, "linear_tile_kernel<DT=%d,FA=%d,FB=%d,E=%d,WM=%d,WN=%d,GM=%d,GN=%d,BK=%d,RING=%d,GUARDED=%d> grid=%u block=%d lds=%d whole=%d splits=%d",
                DT, (int)FA, (int)FB, (int)E, WM, WN, GM, GN, BK, RING, (int)GUARDED, grid.x, T::kThreads, T::kLds, a.whole_tiles, a.splits);
    if (shared) plan_record(d.plan, "linear_join_kernel<DT=%d,E=%d,WM=%d,WN=%d,GM=%d,GN=%d> grid=%u block=%d", DT, (int)E, WM, WN, GM, GN, join.x, T::kThreads);
    return hipSuccess;
  }
  const hipError_t e = raise_lds_limit<linear_tile_kernel<DT, FA, FB, E, WM, WN, GM, GN, BK, RING, GUARDED>>(T::kLds);
  if (e != hipSuccess) return e;
  linear_tile_kernel<DT, FA, FB, E, WM, WN, GM, GN, BK, RING, GUARDED><<<grid, T::kThreads, T::kLds, stream>>>(a, d.to);
  if (shared) linear_join_kernel<DT, E, WM, WN, GM, GN><<<join, T::kThreads, 0, stream>>>(a.partials, a.whole_tiles, a.splits, d.to);
  return hipGetLastError();
}

template <int DT, OperandForm FA, OperandForm FB, Epilogue E>
hipError_t launch_form(const DenseProduct& d, hipStream_t stream) {
  const Operands o(d);
  const TilePlan plan = o.plan(d);
  const TileArgs a{static_cast<const uint16_t*>(d.A), d.lda, static_cast<const uint16_t*>(d.B), d.ldb, d.K, plan.whole_tiles, plan.splits,
                   plan.stages_of_split, o.rows_a, o.rows_b, static_cast<float*>(d.workspace)};
  const int64_t tiles = tiles_of(kTileForms[plan.form], d.M, d.N);
  switch (plan.form) {
    case kFormGuarded: return launch_tiles<DT, FA, FB, E, 2, 2, 2, 2, 64, 2, true>(d, a, tiles, stream);
    case kFormLarge: return launch_tiles<DT, FA, FB, E, 4, 4, 2, 2, 64, 2, false>(d, a, tiles, stream);
    case kFormWide: return launch_tiles<DT, FA, FB, E, 4, 2, 2, 2, 64, 3, false>(d, a, tiles, stream);
    case kFormMiddle: return launch_tiles<DT, FA, FB, E, 2, 2, 2, 2, 64, 4, false>(d, a, tiles, stream);
    default: return launch_tiles<DT, FA, FB, E, 1, 1, 2, 2, 64, 4, false>(d, a, tiles, stream);
  }
}
template <int DT>
hipError_t launch_dtype(const DenseProduct& d, hipStream_t stream) {
  // the gradients' products have nothing behind them
  if (d.form_b == kAlong) return launch_form<DT, kAlong, kAlong, kEpiBare>(d, stream);
  if (d.form_a == kAcross) return launch_form<DT, kAcross, kAcross, kEpiBare>(d, stream);
  switch (epilogue_of(d.to.act)) {
    case kEpiGelu: return launch_form<DT, kAlong, kAcross, kEpiGelu>(d, stream);
    case kEpiSigmoid: return launch_form<DT, kAlong, kAcross, kEpiSigmoid>(d, stream);
    default: return launch_form<DT, kAlong, kAcross, kEpiLinear>(d, stream);
  }
}

template <int DT, int WM, int WN>
hipError_t launch_pair(const TileForm& f, const DenseProduct& w, const DenseProduct& x, float* sums, hipStream_t stream) {
  constexpr int kLds = TileSizes<kAlong, kAlong, WM, WN, 2, 2, 64, 4>::kLds;
  static_assert(kLds == TileSizes<kAcross, kAcross, WM, WN, 2, 2, 64, 4>::kLds, "of either product");
  auto args = [&](const DenseProduct& d) {
    const int stages = (d.K + kStage - 1) / kStage;
    return TileArgs{static_cast<const uint16_t*>(d.A), d.lda, static_cast<const uint16_t*>(d.B), d.ldb, d.K, (int)tiles_of(f, d.M, d.N), 1, stages,
                    kAligned, kAligned, nullptr};
  };
  const TileArgs of_w = args(w), of_x = args(x);
  const bool w_first = w.K >= x.K;
  const uint32_t groups_w = grid_of_items(of_w.whole_tiles), groups_x = grid_of_items(of_x.whole_tiles);
  const uint32_t tiles = groups_w + groups_x, rows = sums ? (uint32_t)((w.M + 3) / 4) : 0;
  if (w.plan) {
    plan_record(w.plan, "linear_pair_kernel<DT=%d,WM=%d,WN=%d> grid=%u block=256 lds=%d", DT, WM, WN, tiles + rows, kLds);
    return hipSuccess;
  }
  const hipError_t e = raise_lds_limit<linear_pair_kernel<DT, WM, WN>>(kLds);
  if (e != hipSuccess) return e;
  linear_pair_kernel<DT, WM, WN><<<tiles + rows, 256, kLds, stream>>>(of_w, w.to, of_x, x.to, (int)(w_first ? groups_w : groups_x), w_first, {sums, (int)tiles});
  return hipGetLastError();
}
template <int DT>
hipError_t launch_pair_of(const DenseProduct& w, const DenseProduct& x, float* sums, hipStream_t stream) {
  const int form = pair_form(w.M, w.N, w.K);
  const TileForm& f = kTileForms[form];
  return form == kFormMiddle ? launch_pair<DT, 2, 2>(f, w, x, sums, stream) : launch_pair<DT, 1, 1>(f, w, x, sums, stream);
}

}  // namespace

size_t dense_product_workspace_bytes(int M, int N, int K, OperandForm form_a, OperandForm form_b) {
  if ((is_layer(form_a, form_b) && N <= kFewTokens) || is_outer(form_a, form_b, K)) return 0;
  const size_t guarded = partial_bytes(plan_of(M, N, K, true), M, N);
  const size_t whole = partial_bytes(plan_of(M, N, K, false), M, N) + (may_copy(M, K, form_a, form_b) ? copy_of(M, K, form_a).bytes() : 0);
  return whole > guarded ? whole : guarded;
}

hipError_t launch_row_copy(const void* from, int64_t ld, void* to, int64_t pitch, int rows, int row, hipStream_t stream) {
  const int64_t groups = (rows * (pitch / 8) + 1023) / 1024;  // four pieces a thread
  linear_copy_kernel<<<dim3((uint32_t)(groups < 1 << 20 ? groups : 1 << 20)), 256, 0, stream>>>(
      static_cast<const uint16_t*>(from), ld, static_cast<uint16_t*>(to), pitch, rows, row, pieces_of_rows(from, ld, row));
  return hipGetLastError();
}

hipError_t launch_dense_product(const DenseProduct& p, hipStream_t stream) {
  if (is_layer(p.form_a, p.form_b) && p.N <= kFewTokens) return launch_linear_few(p, stream);
  if (is_outer(p.form_a, p.form_b, p.K)) return launch_linear_outer(p, stream);
  DenseProduct d = p;
  const Operands o(p);
  if (o.copies(p)) {
    const CopyOfA c = copy_of(p.M, p.K, p.form_a);
    d.A = p.workspace;
    d.lda = c.pitch();
    d.workspace = static_cast<uint8_t*>(p.workspace) + c.bytes();
    if (p.plan) {
      plan_record(p.plan, "linear_copy_kernel block=256");
    } else {
      const hipError_t e = launch_row_copy(p.A, p.lda, p.workspace, c.pitch(), c.rows, c.row, stream);
      if (e != hipSuccess) return e;
    }
  }
  return d.dtype == HINM_F16 ? launch_dtype<HINM_F16>(d, stream) : launch_dtype<HINM_BF16>(d, stream);
}

bool dense_pair_serves(const DenseProduct& w, const DenseProduct& x) {
  return !Operands(w).guarded() && !Operands(x).guarded() && pair_form(w.M, w.N, w.K) != kFormGuarded;
}
hipError_t launch_dense_pair(const DenseProduct& w, const DenseProduct& x, float* sums, hipStream_t stream) {
  return w.dtype == HINM_F16 ? launch_pair_of<HINM_F16>(w, x, sums, stream) : launch_pair_of<HINM_BF16>(w, x, sums, stream);
}

}  // namespace hinm
