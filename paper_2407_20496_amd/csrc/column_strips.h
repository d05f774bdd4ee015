// Sums down the columns of channels x tokens matrices, for norms: strips of 64 columns, their rows by chunks.
#pragma once

#include "eight_values.h"
#include "wave_reduce.h"

namespace hinm {

constexpr int kThreads = 256;
constexpr int kStrip = 64;                 // columns of a workgroup: eight lanes of eight
constexpr int kRowsAtOnce = kThreads / 8;  // rows that its lanes cover together: a round
constexpr int kRounds = 4;                 // rounds whose loads are in flight together
constexpr int kPatch = kRounds * kRowsAtOnce;
constexpr int kGradRounds = 2;             // ... of the gradients' four inputs
constexpr int kGradPatch = kGradRounds * kRowsAtOnce;
constexpr int kWaves = kThreads / 64;

inline int strip_count(int N) { return (N + kStrip - 1) / kStrip; }
// Patches of a workgroup where `at_once` of them run at a time: the fewest with which all of them do.  (One round and a part
// costs two: 16384x4000 forward 214 -> 190 us, 11008x1571 66 -> 56; gradients 4096x2048 45 -> 40.)
inline int patches_of_workgroup(int patches, int N, int at_once) {
  const int most = at_once / strip_count(N);
  return most < 1 ? patches : (patches + most - 1) / most;
}
// Patches of a chunk: four workgroups to a compute unit, at most 64 chunks, so that adding a strip's chunks stays small beside
// its rows.
inline int chunk_patches(int K, int N) {
  const int patches = (K + kPatch - 1) / kPatch, per = patches_of_workgroup(patches, N, 1024), least = (patches + 63) / 64;
  return per > least ? per : least;
}
inline int chunk_count(int K, int N) {
  const int rows = kPatch * chunk_patches(K, N);
  return (K + rows - 1) / rows;
}

// What a kernel knows of its matrices' rows: whole cache lines; pieces of 16 bytes at multiples of 16; nothing (the registers
// that a row's end at any address takes cost the other two their occupancy: 4096x2048 24 -> 27 us).
enum Layout { kLines, kPieces, kAny };
template <Layout L>
__device__ __forceinline__ Pieces known(Pieces rows) { return L == kAny ? rows : kAligned; }

// Which strip and chunk a workgroup has.  Workgroups go to the eight XCDs in turn.  Rows of whole cache lines: neighbouring
// workgroups take neighbouring strips of the same rows.  Otherwise neighbouring strips share lines and each XCD takes a
// contiguous run of the list (chunk, strip), so that the parts of a line meet in one L2 (16384x1000: 68 -> 48 us; at
// 4096x8192, whole lines, the run costs 87 -> 100 us).  Whole lines are also written around the caches, where the partial
// ones wait for their other half (16384x4096: 187 -> 141 us; 11008x1571, partial lines, 67 -> 80 us).
struct Place {
  int n0, n, left, row0, rows, chunk, strip;  // first column; this lane's first column, how many it has; rows of the chunk
  __device__ __forceinline__ bool none() const { return rows <= 0; }  // beyond the list
  __device__ __forceinline__ Place(int K, int N, int rows_per_chunk, bool whole_lines) {
    const int strips = (N + kStrip - 1) / kStrip;
    const int item = whole_lines ? (int)blockIdx.x : (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
    chunk = item / strips;
    strip = item - chunk * strips;
    n0 = strip * kStrip;
    n = n0 + 8 * (threadIdx.x & 7);
    left = min(8, N - n);
    row0 = chunk * rows_per_chunk;
    rows = min(rows_per_chunk, K - row0);
  }
};

template <int DT>
__device__ __forceinline__ void widen(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[2 * j] = low_half<DT>(v[j]);
    f[2 * j + 1] = high_half<DT>(v[j]);
  }
}
template <int DT>
__device__ __forceinline__ u32x4 narrow(const float (&f)[8]) {
  return u32x4{floats_to_bits<DT>(f[0], f[1]), floats_to_bits<DT>(f[2], f[3]), floats_to_bits<DT>(f[4], f[5]),
               floats_to_bits<DT>(f[6], f[7])};
}

// Sum over each eight neighbouring lanes.
template <int CTRL>
__device__ __forceinline__ float plus_moved(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float add_eight_lanes(float v) {
  v = plus_moved<0xB1>(v);      // lane ^ 1
  v = plus_moved<0x4E>(v);      // lane ^ 2
  return plus_moved<0x141>(v);  // the other four
}

// Sum over a wave's lanes with the same lane % 8.
__device__ __forceinline__ float add_lanes_by_8(float v) {
  v = plus_moved<0x128>(v);  // lane ^ 8
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Eight values of every lane, added over the lanes with the same lane % 8 and left one to a lane: value j = lane / 8 with its
// three bits turned round (lane / 32 the highest).  Each step adds what two halves of the lanes hold of half of the values:
// swaps of register halves, no LDS.
template <int LANES>
__device__ __forceinline__ float swapped_sum(float a, float b) {
  uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
  swap_lanes<LANES>(x, y);
  return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}
template <int LANES>
__device__ __forceinline__ double swapped_sum(double a, double b) {
  u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
  uint32_t x0 = x[0], x1 = x[1], y0 = y[0], y1 = y[1];
  swap_lanes<LANES>(x0, y0);
  swap_lanes<LANES>(x1, y1);
  return __builtin_bit_cast(double, (u32x2{x0, x1})) + __builtin_bit_cast(double, (u32x2{y0, y1}));
}
__device__ __forceinline__ uint32_t from_lane_8(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true); }
__device__ __forceinline__ float from_lane_8(float v) { return __builtin_bit_cast(float, from_lane_8(__builtin_bit_cast(uint32_t, v))); }
__device__ __forceinline__ double from_lane_8(double v) {
  const u32x2 x = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, (u32x2{from_lane_8(x[0]), from_lane_8(x[1])}));
}
template <class T>
__device__ __forceinline__ T add_columns(const T (&v)[8]) {
  T w[4], x[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = swapped_sum<32>(v[i], v[i + 4]);
#pragma unroll
  for (int i = 0; i < 2; ++i) x[i] = swapped_sum<16>(w[i], w[i + 2]);
  const bool second = threadIdx.x & 8;
  const T kept = second ? x[1] : x[0], given = second ? x[0] : x[1];
  return kept + from_lane_8(given);
}

// QUANTITIES sums of the workgroup's 64 columns, added over its threads in a fixed order, to partial[quantity][chunk][N].
template <int QUANTITIES, class T>
__device__ __forceinline__ void store_sums(const T (&sum)[QUANTITIES][8], const Place& p, T* partial, int chunks, int N) {
  __shared__ T by_wave[QUANTITIES][kWaves][kStrip];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j = 4 * (lane >> 5) + 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1);
#pragma unroll
  for (int q = 0; q < QUANTITIES; ++q) by_wave[q][wave][8 * (lane & 7) + j] = add_columns(sum[q]);
  __syncthreads();
  const int col = threadIdx.x & (kStrip - 1), n = p.n0 + col;
  for (int q = threadIdx.x / kStrip; q < QUANTITIES; q += kThreads / kStrip) {
    T t = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += by_wave[q][w][col];
    if (n < N) partial[((int64_t)q * chunks + p.chunk) * N + n] = t;
  }
}

// ... and their totals over the chunks, to total[quantity][64].  The caller waits at a barrier.
constexpr int kChunksAtOnce = 8;
template <int QUANTITIES, class T>
__device__ __forceinline__ void add_chunks(const T* partial, int chunks, int N, const Place& p, T (*total)[kStrip]) {
  static_assert(QUANTITIES <= kThreads / kStrip, "a thread for each");
  const int col = threadIdx.x & (kStrip - 1), n = p.n0 + col, q = threadIdx.x / kStrip;
  if (q >= QUANTITIES || n >= N) return;
  const T* at = partial + (int64_t)q * chunks * N + n;
  T t = 0;
  for (int c = 0; c < chunks; c += kChunksAtOnce) {
    T v[kChunksAtOnce];
#pragma unroll
    for (int j = 0; j < kChunksAtOnce; ++j) v[j] = at[(int64_t)min(c + j, chunks - 1) * N];
#pragma unroll
    for (int j = 0; j < kChunksAtOnce; ++j) t += c + j < chunks ? v[j] : T(0);
  }
  total[q][col] = t;
}

// Rows of a workgroup in the second launches: the gradients' has three to a compute unit.
inline int rows_of_apply(int K, int N) { return kPatch * patches_of_workgroup((K + kPatch - 1) / kPatch, N, 1024); }
inline int rows_of_grad_apply(int K, int N) { return kGradPatch * patches_of_workgroup((K + kGradPatch - 1) / kGradPatch, N, 768); }

template <int THREADS>
__device__ __forceinline__ float add_workgroup(float v, float* by_wave) {
  v = add_lanes_by_8(add_eight_lanes(v));
  if ((threadIdx.x & 63) == 0) by_wave[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) t += by_wave[w];
  return t;
}
// eight floats from k on, `valid` of them (the rest: zero); absent: ones.  WHOLE: all eight exist, at a multiple of 16 bytes
template <bool WHOLE>
__device__ __forceinline__ void load_factors(const float* p, int k, int valid, float (&f)[8]) {
  f32x4 low = {1, 1, 1, 1}, high = {1, 1, 1, 1};
  if (p && (WHOLE || (valid >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0))) {
    low = *reinterpret_cast<const f32x4*>(p + k);
    high = *reinterpret_cast<const f32x4*>(p + k + 4);
  } else if (!WHOLE && p) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      low[j] = j < valid ? p[k + j] : 0.0f;
      high[j] = j + 4 < valid ? p[k + j + 4] : 0.0f;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[j] = low[j];
    f[4 + j] = high[j];
  }
}

// Workgroups for the list (chunk, strip), a multiple of the XCDs.
inline dim3 grid_of(int chunks, int N) { return dim3((uint32_t)(((int64_t)chunks * strip_count(N) + 7) / 8 * 8)); }
inline bool at_16_bytes(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool in_lines(const void* p, int64_t ld) { return !p || ((reinterpret_cast<uintptr_t>(p) & 127) == 0 && ld % 64 == 0); }

}  // namespace hinm
