// Dense products of two 16-bit matrices on the matrix cores, tiles through LDS (include/hinm.h, hinm_linear and its gradients).
#include "linear_tile.h"

#include "direct_lds.h"
#include "lds_in_flight.h"
#include "workgroup_items.h"

namespace hinm {

namespace {

struct TileArgs {
  const uint16_t* A;
  int64_t lda;
  const uint16_t* B;
  int64_t ldb;
  int K, splits, stages_of_split;
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
  // ... of a stage that ends early: what lies beyond its end is beyond the buffer's, and zeros are written
  __device__ __forceinline__ void copy_cut(__amdgpu_buffer_rsrc_t stage, int c, int lane, int left_k, uint8_t* to) const {
    int row, value;
    S::piece_of(first_copy + c, lane, row, value);
    copy16_to_lds(stage, (F == kAlong ? value : row) < left_k ? from[c] : kNowhere, 0, to + 1024 * (first_copy + c));
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

template <OperandForm FA, OperandForm FB, int WM, int WN, int GM, int GN, int BK, int RING>
struct TileSizes {
  static constexpr int kWaves = GM * GN, kThreads = 64 * kWaves;
  static constexpr int TM = 32 * WM * GM, TN = 32 * WN * GN;
  using StageA = OperandStage<TM, BK, FA>;
  using StageB = OperandStage<TN, BK, FB>;
  static constexpr int kStageBytes = StageA::kBytes + StageB::kBytes;
  static constexpr int kCopiesA = StageA::kCopies / kWaves, kCopiesB = StageB::kCopies / kWaves, kCopies = kCopiesA + kCopiesB;
  static constexpr int kSlabPitch = 32 * WN * 4 + 16, kSlabBytes = 32 * kSlabPitch;  // of a wave: 32 rows of sums
  static constexpr int kLds = RING * kStageBytes > kWaves * kSlabBytes ? RING * kStageBytes : kWaves * kSlabBytes;
  static_assert(StageA::kCopies % kWaves == 0 && StageB::kCopies % kWaves == 0, "whole copies for every wave");
  static_assert(RING == 2 || RING == 4, "places by masks");
};

// Rows 32 j .. of a wave's part of a tile: its sums to the wave's slab, and from there to the result in whole pieces.
// acc[i]: columns 32 i .. of the wave; a lane holds row lane % 32, columns 8 (e / 4) + 4 (lane / 32) + e % 4.  Pieces are finished
// two at a time, in a loop that stays one (a tile's code would outgrow the instruction cache), while the next two residuals
// are on their way.
template <int DT, int WN>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[WN], uint8_t* slab, int m0, int n0, const LinearEpilogue& e) {
  constexpr int kPitch = 32 * WN * 4 + 16, kPieces = 4 * WN, kRows = 64 / kPieces, kGroup = 2;
  const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
  const int piece = lane % kPieces, n = n0 + 8 * piece, left = min(8, e.N - n);
  const int most = left > 0 ? min(32, e.M - m0) : 0;  // rows of this lane's columns that exist
  struct Group {
    u32x4 residual[kGroup];
    float bias[kGroup];
  };
  auto load = [&](int row0, Group& g) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
      const int row = row0 + c * kRows;
      g.residual[c] = row < most ? load_residual<DT>(e, m0 + row, n, left) : u32x4{0, 0, 0, 0};
      g.bias[c] = row < most && e.bias ? e.bias[m0 + row] : 0.0f;
    }
  };
  Group now;
  load(lane / kPieces, now);
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(slab + r * kPitch + (32 * i + 8 * q + 4 * half) * 4) =
          f32x4{acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
  asm volatile("" ::: "memory");  // LDS operations of a wave are done in order; the compiler is held to it
#pragma unroll 1
  for (int row0 = lane / kPieces; row0 < most; row0 += kGroup * kRows) {
    Group next;
    load(row0 + kGroup * kRows, next);
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
      const int row = row0 + c * kRows;
      if (row >= most) break;
      const float* from = reinterpret_cast<const float*>(slab + row * kPitch + 32 * piece);
      const f32x4 low = *reinterpret_cast<const f32x4*>(from), high = *reinterpret_cast<const f32x4*>(from + 4);
      float v[8] = {low[0], low[1], low[2], low[3], high[0], high[1], high[2], high[3]};
      finish_eight<DT>(e, m0 + row, n, left, now.bias[c], now.residual[c], v);
    }
    now = next;
  }
  asm volatile("" ::: "memory");
}

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
template <int DT, OperandForm FA, OperandForm FB, int WM, int WN, int GM, int GN, int BK, int RING, bool GUARDED>
__global__ __launch_bounds__(64 * GM * GN, WM * WN > 8 ? 1 : 2) void linear_tile_kernel(TileArgs a, LinearEpilogue e) {
  using T = TileSizes<FA, FB, WM, WN, GM, GN, BK, RING>;
  constexpr int kSteps = BK / 16;
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = ((e.M + T::TM - 1) / T::TM) * ((e.N + T::TN - 1) / T::TN);
  const int item = item_of_workgroup(tiles * a.splits);
  if (item < 0) return;
  const int split = item / tiles, tile = item - split * tiles;
  const TilePlace place(tile, T::TM, T::TN, e.M, e.N);
  const int first = split * a.stages_of_split;
  const int stages = min(a.stages_of_split, (a.K + BK - 1) / BK - first), k0 = first * BK;
  // stages that copies fill; the last one of all may be cut short
  const int whole = GUARDED ? 0 : min(stages, a.K / BK - first);

  OperandSource<T::TM, BK, FA, T::kCopiesA> of_a;
  OperandSource<T::TN, BK, FB, T::kCopiesB> of_b;
  of_a.init(a.A, a.lda, place.m0, e.M, k0, wave * T::kCopiesA, lane);
  of_b.init(a.B, a.ldb, place.n0, e.N, k0, wave * T::kCopiesB, lane);
  struct Buffers {
    __amdgpu_buffer_rsrc_t a, b;
  };
  auto buffers_of = [&](int stage) __attribute__((always_inline)) { return Buffers{buffer_of(of_a.of_stage(stage), kWholeBuffer), buffer_of(of_b.of_stage(stage), kWholeBuffer)}; };
  auto slot_of = [&](int stage) __attribute__((always_inline)) { return lds + (stage & (RING - 1)) * T::kStageBytes; };
  auto copy_one = [&](const Buffers& from, int stage, int c) __attribute__((always_inline)) {
    if (c < T::kCopiesA) of_a.copy(from.a, c, slot_of(stage));
    else of_b.copy(from.b, c - T::kCopiesA, slot_of(stage) + T::StageA::kBytes);
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
  auto put_stage = [&](int stage, const Held& h) __attribute__((always_inline)) {
    const int left_k = a.K - k0 - stage * BK;
    uint8_t* const slot = slot_of(stage);
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

  // the last stage where it is cut short: copied whole at a time, and cleared behind its end once it is there
  const int left_k = a.K - k0 - whole * BK;
  auto copy_cut_stage = [&]() __attribute__((always_inline)) {
    const Buffers from = buffers_of(whole);
#pragma unroll
    for (int c = 0; c < T::kCopies; ++c) {
      if (c < T::kCopiesA) of_a.copy_cut(from.a, c, lane, left_k, slot_of(whole));
      else of_b.copy_cut(from.b, c - T::kCopiesA, lane, left_k, slot_of(whole) + T::StageA::kBytes);
    }
  };
  auto clear_cut_stage = [&]() __attribute__((always_inline)) {
    if ((FA == kAcross && FB == kAcross) || !(left_k & 7)) return;
    if constexpr (FA == kAlong) T::StageA::clear_behind(slot_of(whole), left_k, T::kThreads);
    if constexpr (FB == kAlong) T::StageB::clear_behind(slot_of(whole) + T::StageA::kBytes, left_k, T::kThreads);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // LDS reads: by step along, by tile of 32 across
  const int half = lane >> 5, r = lane & 31, in16 = lane & 15;
  const int wave_m = (wave % GM) * 32 * WM, wave_n = (wave / GM) * 32 * WN;
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
  auto read_one = [&](auto step_tag, auto tile_tag, int stage, Operands& f) __attribute__((always_inline)) {
    constexpr int s = decltype(step_tag)::value, t = decltype(tile_tag)::value;
    const uint32_t slot = (stage & (RING - 1)) * T::kStageBytes;
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

  // the first stages
  Held held;
  const int ahead = min(RING, stages);
  if constexpr (GUARDED) {
    for (int q = 0; q < ahead; ++q) {
      draw_stage(q, held);
      put_stage(q, held);
    }
    if (RING < stages) draw_stage(RING, held);
  } else {
    // beyond RING - 1 whole ones only half of the last: the other half follows in the first step
    for (int q = 0; q < min(RING, whole); ++q) {
      const Buffers from = buffers_of(q);
#pragma unroll
      for (int c = 0; c < T::kCopies; ++c)
        if (q < RING - 1 || c < T::kCopies / 2 || whole < RING) copy_one(from, q, c);
    }
    if (whole < ahead) copy_cut_stage();
  }
  // stage 0 is waited for, and all of them where they are few
  if (!GUARDED && whole >= RING) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((RING - 2) * T::kCopies + T::kCopies / 2) : "memory");
  else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if (!GUARDED && whole == 0) clear_cut_stage();

  Operands sets[2];
  unroll<0, WM + WN>([&](auto t) { read_one(std::integral_constant<int, 0>{}, t, 0, sets[0]); });

  // SECOND / FIRST: the second half of stage p + RING - 1 and the first of p + RING are copied; LAST: no stage follows
  auto stage = [&](auto second_tag, auto first_tag, auto last_tag, int p) __attribute__((always_inline)) {
    constexpr bool kSecond = decltype(second_tag)::value, kFirst = decltype(first_tag)::value, kLast = decltype(last_tag)::value;
    unroll<0, kSteps>([&](auto step_tag) __attribute__((always_inline)) {
      constexpr int s = decltype(step_tag)::value;
      constexpr bool kEnds = s == kSteps - 1;
      constexpr bool kCopying = (s == 0 && kSecond) || (kEnds && kFirst), kReading = !(kEnds && kLast);
      constexpr int kTiles = WM * WN, kReads = WM + WN, kHalf = T::kCopies / 2, kOthers = T::kCopies - kHalf;
      Operands &now = sets[s & 1], &next = sets[(s + 1) & 1];
      wait_operands(now);
      if constexpr (kEnds && !kLast) {
        if constexpr (kSecond) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((RING - 2) * T::kCopies) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if constexpr (GUARDED) {
          if (p + RING < stages) put_stage(p + RING, held);
          if (p + RING + 1 < stages) draw_stage(p + RING + 1, held);
        } else if constexpr (!kFirst) {
          if (whole < stages) {
            if (p + RING == whole) copy_cut_stage();
            if (!kSecond && p + 1 == whole) clear_cut_stage();
          }
        }
      }
      const int copied = kEnds ? p + RING : p + RING - 1;
      const Buffers from = buffers_of(kCopying ? copied : 0);
      unroll<0, kTiles>([&](auto t_tag) __attribute__((always_inline)) {
        constexpr int t = decltype(t_tag)::value, i = t / WM, j = t % WM;
        acc[i][j] = mfma_32x32x16<DT>(now.b[i], now.a[j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kReading) {
          constexpr int b = t * kReads * 2 / kTiles, to = (t + 1) * kReads * 2 / kTiles;
          unroll<(b < kReads ? b : kReads), (to < kReads ? to : kReads)>([&](auto u) __attribute__((always_inline)) {
            read_one(std::integral_constant<int, (s + 1) % kSteps>{}, u, kEnds ? p + 1 : p, next);
          });
        }
        if constexpr (kCopying) {
          constexpr int kCount = kEnds ? kHalf : kOthers;
#pragma unroll
          for (int c = t * kCount / kTiles; c < (t + 1) * kCount / kTiles; ++c) copy_one(from, copied, (kEnds ? 0 : kHalf) + c);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  int p = 0;
  if constexpr (!GUARDED) {
    for (; p + RING < whole; ++p) stage(yes, yes, no, p);
    if (p + RING == whole && p + 1 < stages) stage(yes, no, no, p++);
  }
  for (; p + 1 < stages; ++p) stage(no, no, no, p);
  stage(no, no, yes, p);
  // every wave has read its operands: the ring becomes the waves' slabs
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  if (a.splits > 1) {
    float* const to = a.partials + ((int64_t)split * tiles + tile) * (T::TM * T::TN) + wave * (WM * WN * 1024) + 4 * lane;
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
  uint8_t* const slab = lds + wave * T::kSlabBytes;
  unroll<0, WM>([&](auto j_tag) __attribute__((always_inline)) {
    constexpr int j = decltype(j_tag)::value;
    f32x16 rows[WN];
#pragma unroll
    for (int i = 0; i < WN; ++i) rows[i] = acc[i][j];
    store_rows<DT, WN>(rows, slab, place.m0 + wave_m + 32 * j, place.n0 + wave_n, e);
  });
}

// Tiles that several workgroups have summed parts of: the parts added in order, 32 rows of every wave a workgroup.
template <int DT, int WM, int WN, int GM, int GN>
__global__ __launch_bounds__(64 * GM * GN) void linear_join_kernel(const float* partials, int splits, LinearEpilogue e) {
  constexpr int TM = 32 * WM * GM, TN = 32 * WN * GN, kSlabBytes = 32 * (32 * WN * 4 + 16);
  __shared__ __align__(16) uint8_t slabs[GM * GN * kSlabBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = ((e.M + TM - 1) / TM) * ((e.N + TN - 1) / TN);
  const int item = item_of_workgroup(tiles * WM);
  if (item < 0) return;
  const int tile = item / WM, j = item - tile * WM;
  const TilePlace place(tile, TM, TN, e.M, e.N);
  const int m0 = place.m0 + (wave % GM) * 32 * WM + 32 * j, n0 = place.n0 + (wave / GM) * 32 * WN;
  if (m0 >= e.M || n0 >= e.N) return;
  const float* from = partials + (int64_t)tile * (TM * TN) + wave * (WM * WN * 1024) + j * (WN * 1024) + 4 * lane;
  f32x16 acc[WN];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[i][q] = 0;
#pragma unroll 4
  for (int s = 0; s < splits; ++s, from += (int64_t)tiles * (TM * TN)) {
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(from + (i * 4 + q) * 256);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][4 * q + c] += v[c];
      }
  }
  store_rows<DT, WN>(acc, slabs + wave * kSlabBytes, m0, n0, e);
}

// Which form serves a shape.
struct TileForm {
  int rows, cols;
};
constexpr int kFormGuarded = 0, kFormSmall = 1, kFormLarge = 2;
constexpr TileForm kTileForms[] = {{128, 128}, {128, 128}, {256, 256}};
constexpr int kStage = 64;  // summed values, of every form

int64_t tiles_of(int form, int M, int N) {
  return (int64_t)((M + kTileForms[form].rows - 1) / kTileForms[form].rows) * ((N + kTileForms[form].cols - 1) / kTileForms[form].cols);
}
struct TilePlan {
  int form, splits, stages_of_split;
};
TilePlan plan_of(int M, int N, int K, bool guarded) {
  TilePlan p{guarded ? kFormGuarded : kFormSmall, 1, 0};
  const int stages = (K + kStage - 1) / kStage;
  if (!guarded && tiles_of(kFormLarge, M, N) >= 224) p.form = kFormLarge;
  const int64_t tiles = tiles_of(p.form, M, N);
  if (p.form != kFormLarge && tiles < 256 && stages > 4) {
    const int most = (int)(512 / tiles), least = stages / 4;
    p.splits = most < least ? most : least;
    if (p.splits < 1) p.splits = 1;
  }
  p.stages_of_split = (stages + p.splits - 1) / p.splits;
  p.splits = (stages + p.stages_of_split - 1) / p.stages_of_split;
  return p;
}
size_t partial_bytes(const TilePlan& p, int M, int N) {
  return p.splits < 2 ? 0 : (size_t)p.splits * tiles_of(p.form, M, N) * kTileForms[p.form].rows * kTileForms[p.form].cols * sizeof(float);
}

template <int DT, OperandForm FA, OperandForm FB, int WM, int WN, int GM, int GN, int BK, int RING, bool GUARDED>
hipError_t launch_tiles(const DenseProduct& d, const TileArgs& a, int64_t tiles, hipStream_t stream) {
  using T = TileSizes<FA, FB, WM, WN, GM, GN, BK, RING>;
  const dim3 grid(grid_of_items(tiles * a.splits));
  if (d.plan) {
    plan_record(d.plan, "linear_tile_kernel<DT=%d,FA=%d,FB=%d,WM=%d,WN=%d,GM=%d,GN=%d,BK=%d,RING=%d,GUARDED=%d> grid=%u block=%d lds=%d splits=%d", DT,
                (int)FA, (int)FB, WM, WN, GM, GN, BK, RING, (int)GUARDED, grid.x, T::kThreads, T::kLds, a.splits);
  } else {
    const hipError_t e = raise_lds_limit<linear_tile_kernel<DT, FA, FB, WM, WN, GM, GN, BK, RING, GUARDED>>(T::kLds);
    if (e != hipSuccess) return e;
    linear_tile_kernel<DT, FA, FB, WM, WN, GM, GN, BK, RING, GUARDED><<<grid, T::kThreads, T::kLds, stream>>>(a, d.to);
  }
  if (a.splits > 1) {
    if constexpr (WN <= 2) {
      const dim3 join(grid_of_items(tiles * WM));
      if (d.plan) plan_record(d.plan, "linear_join_kernel<DT=%d,WM=%d,WN=%d,GM=%d,GN=%d> grid=%u block=%d", DT, WM, WN, GM, GN, join.x, T::kThreads);
      else linear_join_kernel<DT, WM, WN, GM, GN><<<join, T::kThreads, 0, stream>>>(a.partials, a.splits, d.to);
    }
  }
  return d.plan ? hipSuccess : hipGetLastError();
}

template <int DT, OperandForm FA, OperandForm FB>
hipError_t launch_form(const DenseProduct& d, hipStream_t stream) {
  // copies take whole pieces at multiples of 16 bytes, from offsets of 31 bits within a stage
  const Pieces rows_a = pieces_of_rows(d.A, d.lda, FA == kAlong ? d.K : d.M), rows_b = pieces_of_rows(d.B, d.ldb, FB == kAlong ? d.K : d.N);
  const bool guarded = rows_a != kAligned || rows_b != kAligned || d.lda > (1 << 21) || d.ldb > (1 << 21);
  const TilePlan plan = plan_of(d.M, d.N, d.K, guarded);
  const TileArgs a{static_cast<const uint16_t*>(d.A), d.lda, static_cast<const uint16_t*>(d.B), d.ldb, d.K, plan.splits, plan.stages_of_split,
                   rows_a, rows_b, static_cast<float*>(d.workspace)};
  const int64_t tiles = tiles_of(plan.form, d.M, d.N);
  switch (plan.form) {
    case kFormGuarded: return launch_tiles<DT, FA, FB, 2, 2, 2, 2, 64, 2, true>(d, a, tiles, stream);
    case kFormSmall: return launch_tiles<DT, FA, FB, 2, 2, 2, 2, 64, 2, false>(d, a, tiles, stream);
    default: return launch_tiles<DT, FA, FB, 4, 4, 2, 2, 64, 2, false>(d, a, tiles, stream);
  }
}
template <int DT>
hipError_t launch_dtype(const DenseProduct& d, hipStream_t stream) {
  if (d.form_b == kAlong) return launch_form<DT, kAlong, kAlong>(d, stream);
  return d.form_a == kAlong ? launch_form<DT, kAlong, kAcross>(d, stream) : launch_form<DT, kAcross, kAcross>(d, stream);
}

}  // namespace

size_t dense_product_workspace_bytes(int M, int N, int K) {
  const size_t a = partial_bytes(plan_of(M, N, K, false), M, N), b = partial_bytes(plan_of(M, N, K, true), M, N);
  return a > b ? a : b;
}

hipError_t launch_dense_product(const DenseProduct& p, hipStream_t stream) {
  return p.dtype == HINM_F16 ? launch_dtype<HINM_F16>(p, stream) : launch_dtype<HINM_BF16>(p, stream);
}

}  // namespace hinm
