// Layer norm over the channels of channels x tokens matrices, and its gradients (include/hinm.h).
//
// As the norms around a block (block_norm.hip): sums run down the columns, so columns are split over workgroups and two launches
// draw whole cache lines, the first for the sums, by chunks of rows, the second for the results.  Forward, a column's mean and
// variance come from sum x and sum x^2 in binary64: products of two 16-bit values are exact there, and the difference
// sum x^2 / K - mean^2 keeps its digits down to 2^-50 of mean^2, far below what 16-bit values around such a mean can differ by.
// Where one workgroup holds a column, its deviations are squared themselves.  Backward, with xn = (x - mean) rstd and g = w du:
//   dx = dh + rstd (g - sum_k g / K - xn sum_k g xn / K),   dw = sum_n du xn,   db = sum_n du.
// Bound by memory, which the second launch reads again (in part from the memory-side cache): 4096x2047 13.0 us (sums 5.2, results 8.2 on
// the device; 2.6 TB/s of what is read once and written), 16384x1000 with its gradients 41.6 (17.5, 22.7 and 3.9 for dw and db: 2.4 TB/s, rows
// of 2000 bytes that share lines), 768x4096 with dh 15.2 (6.0, 7.2, 2.3).  One token of 4096 channels: 2.4 us on the device.
#include "column_strips.h"

namespace hinm {

namespace {

// ---- forward ------------------------------------------------------------------------------------------

struct LayerNorm {
  int K, N, rows_per_chunk, chunks, rows_of_apply;
  float eps;
  const uint16_t* x;
  int64_t ldx;
  const float *w, *b;
  uint16_t* u;
  int64_t ldu;
  float *mean, *rstd;
  double* sums;  // [2][chunks][N]: x, x^2
  Pieces rows;
  Layout layout;
};

__device__ __forceinline__ float root_of(double variance, float eps) { return 1.0f / sqrtf((float)variance + eps); }

// Sums in float32 are of 2^-14 of the values, of which there are at most 2^14: as many bf16 values of any size do not leave its range.
constexpr float kSumScale = 0x1p-14f;
__device__ __forceinline__ float mean_of_sum(float sum, int K) { return sum / ((float)K * kSumScale); }

// kRounds rows of a lane's columns, from row k on in steps of a round
template <Layout L>
__device__ __forceinline__ void load_rows(const uint16_t* x, int64_t ld, const Place& p, int k, int end, Pieces rows, u32x4 (&v)[kRounds]) {
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    v[i] = r < end && p.left > 0 ? draw_eight(x + (int64_t)r * ld + p.n, p.left, known<L>(rows)) : u32x4{0, 0, 0, 0};
  }
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads) void layer_norm_sums_kernel(LayerNorm a) {
  const Place p(a.K, a.N, a.rows_per_chunk, L == kLines);
  if (p.none()) return;
  double sum[2][8] = {};
  const int end = p.row0 + p.rows;
  for (int k = p.row0 + (threadIdx.x >> 3); k < end; k += kPatch) {
    u32x4 v[kRounds];
    load_rows<L>(a.x, a.ldx, p, k, end, a.rows, v);
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      float x[8];
      widen<DT>(place_eight(v[i], p.left, known<L>(a.rows)), x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double wide = x[j];
        sum[0][j] += wide;
        sum[1][j] += wide * wide;
      }
    }
  }
  store_sums<2>(sum, p, a.sums, a.chunks, a.N);
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads, 4) void layer_norm_apply_kernel(LayerNorm a) {
  __shared__ double total[2][kStrip];
  __shared__ float mean_of[kStrip], root[kStrip];
  const Place p(a.K, a.N, a.rows_of_apply, L == kLines);
  if (p.none()) return;
  const int end = p.row0 + p.rows, first = p.row0 + (threadIdx.x >> 3), at = 8 * (threadIdx.x & 7);
  u32x4 v[kRounds];
  load_rows<L>(a.x, a.ldx, p, first, end, a.rows, v);  // on their way while the sums are added
  add_chunks<2>(a.sums, a.chunks, a.N, p, total);
  __syncthreads();
  if (threadIdx.x < kStrip) {
    const int n = p.n0 + threadIdx.x;
    float m = 0, r = 0;
    if (n < a.N) {
      const double mean = total[0][threadIdx.x] / a.K;
      double variance = total[1][threadIdx.x] / a.K - mean * mean;
      if (variance < 0) variance = 0;  // all of it cancelled
      m = (float)mean;
      r = root_of(variance, a.eps);
      if (p.chunk == 0) {
        if (a.mean) a.mean[n] = m;
        if (a.rstd) a.rstd[n] = r;
      }
    }
    mean_of[threadIdx.x] = m;
    root[threadIdx.x] = r;
  }
  __syncthreads();
  if (p.left <= 0) return;
  float m[8], r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    m[j] = mean_of[at + j];
    r[j] = root[at + j];
  }
  for (int k = first; k < end; k += kPatch) {
    u32x4 next[kRounds];
    if (k + kPatch < end) load_rows<L>(a.x, a.ldx, p, k + kPatch, end, a.rows, next);
    float w[kRounds], b[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int row = k + i * kRowsAtOnce;
      w[i] = row < end && a.w ? a.w[row] : 1.0f;
      b[i] = row < end && a.b ? a.b[row] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int row = k + i * kRowsAtOnce;
      if (row >= end) break;
      float x[8];
      widen<DT>(place_eight(v[i], p.left, known<L>(a.rows)), x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (x[j] - m[j]) * (r[j] * w[i]) + b[i];
      store_eight<L == kLines>(a.u + (int64_t)row * a.ldu + p.n, narrow<DT>(x), p.left);
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i) v[i] = next[i];
  }
}

// Few channels, or a few tokens: one launch.  A workgroup of 512 threads owns eight columns, a row a lane, and holds all their
// rows in registers (ROUNDS rows a thread) through both sums.
constexpr int kHeldThreads = 512;

// Sums over the workgroup of every thread's eight columns.
template <int QUANTITIES>
__device__ __forceinline__ void add_held(float (&sum)[QUANTITIES][8], float (*by_wave)[kHeldThreads / 64][8], float (*total)[8]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < QUANTITIES; ++q) {
    const float t = add_eight_lanes(add_columns(sum[q]));
    if ((lane & 7) == 0) by_wave[q][threadIdx.x >> 6][4 * (lane >> 5) + 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1)] = t;
  }
  __syncthreads();
  if (threadIdx.x < 8 * QUANTITIES) {
    const int q = threadIdx.x >> 3, j = threadIdx.x & 7;
    float t = 0;
#pragma unroll
    for (int w = 0; w < kHeldThreads / 64; ++w) t += by_wave[q][w][j];
    total[q][j] = t;
  }
  __syncthreads();
}

template <int DT, int ROUNDS>
__global__ __launch_bounds__(kHeldThreads) void layer_norm_held_kernel(LayerNorm a) {
  __shared__ float by_wave[1][kHeldThreads / 64][8], total[2][1][8];
  // neighbouring columns, which share lines, on one XCD
  const int n = 8 * ((int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3)), left = min(8, a.N - n);
  if (left <= 0) return;
  u32x4 v[ROUNDS];
  float w[ROUNDS], b[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    const bool in = k < a.K;
    v[i] = in ? draw_eight(a.x + (int64_t)k * a.ldx + n, left, a.rows) : u32x4{0, 0, 0, 0};
    w[i] = in && a.w ? a.w[k] : 1.0f;
    b[i] = in && a.b ? a.b[k] : 0.0f;
  }
  float sum[1][8] = {}, m[8], r[8];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    v[i] = place_eight(v[i], left, a.rows);
    float x[8];
    widen<DT>(v[i], x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[0][j] = fmaf(x[j], kSumScale, sum[0][j]);
  }
  add_held<1>(sum, by_wave, total[0]);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    m[j] = mean_of_sum(total[0][0][j], a.K);
    sum[0][j] = 0;
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    if ((int)threadIdx.x + i * kHeldThreads >= a.K) break;
    float x[8];
    widen<DT>(v[i], x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[0][j] += (x[j] - m[j]) * (x[j] - m[j]);
  }
  add_held<1>(sum, by_wave, total[1]);
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = 1.0f / sqrtf(total[1][0][j] / (float)a.K + a.eps);
  if (threadIdx.x < left) {
    const float mean = mean_of_sum(total[0][0][threadIdx.x], a.K);
    if (a.mean) a.mean[n + threadIdx.x] = mean;
    if (a.rstd) a.rstd[n + threadIdx.x] = 1.0f / sqrtf(total[1][0][threadIdx.x] / (float)a.K + a.eps);
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    if (k >= a.K) break;
    float x[8];
    widen<DT>(v[i], x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (x[j] - m[j]) * (r[j] * w[i]) + b[i];
    store_eight(a.u + (int64_t)k * a.ldu + n, narrow<DT>(x), left);
  }
}

// One token without a stride: a vector, held by one workgroup, eight channels a thread and round.  WHOLE: whole pieces at
// multiples of 16 bytes (channels and factors).  Sums of more than 2^13 values of 11 bits may need more than float32's 24, and a
// mean off by one of its steps counts where the deviations are no larger (equal channels of 65504: 0.004 beside a root of eps of
// 0.003): there what the deviations' own mean is beside zero is taken off them (16384 channels 4.3 us a call, without it 3.9).
constexpr int kVectorMost = 2 * 8 * 1024;  // channels

template <int DT, int THREADS, int ROUNDS, bool WHOLE>
__global__ __launch_bounds__(THREADS) void layer_norm_vector_kernel(LayerNorm a) {
  constexpr bool kLong = 8 * THREADS * ROUNDS > 1 << 13;
  __shared__ __align__(16) float by_wave[3][THREADS / 64];
  float x[ROUNDS][8], w[ROUNDS][8], b[ROUNDS][8];
  u32x4 of_x[ROUNDS];
  const u32x4 none = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = 8 * (threadIdx.x + i * THREADS), left = a.K - k;
    const int at = WHOLE && left <= 0 ? 0 : k;  // threads beyond the vector read its beginning, and drop it
    of_x[i] = WHOLE ? draw_eight(a.x + at, 8, kAligned) : left > 0 ? draw_eight(a.x + k, left, a.rows) : none;
    load_factors<WHOLE>(a.w, at, left, w[i]);
    if (a.b) load_factors<WHOLE>(a.b, at, left, b[i]);
  }
  float sum = 0;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int left = a.K - 8 * (int)(threadIdx.x + i * THREADS);
    widen<DT>(WHOLE ? (left > 0 ? of_x[i] : none) : left > 0 ? trim_eight(of_x[i], left, a.rows) : none, x[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fmaf(x[i][j], kSumScale, sum);
  }
  const float mean = mean_of_sum(add_workgroup<THREADS>(sum, by_wave[0]), a.K);
  float rest = 0;
  sum = 0;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int left = a.K - 8 * (int)(threadIdx.x + i * THREADS);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[i][j] = j < left ? x[i][j] - mean : 0.0f;
      sum += x[i][j] * x[i][j];
      if constexpr (kLong) rest += x[i][j];
    }
  }
  if constexpr (kLong) {  // read behind the barrier of the squares' sum
    const float of_wave = add_lanes_by_8(add_eight_lanes(rest));
    if ((threadIdx.x & 63) == 0) by_wave[2][threadIdx.x >> 6] = of_wave;
  }
  float variance = add_workgroup<THREADS>(sum, by_wave[1]) / (float)a.K;
  if constexpr (kLong) {
    rest = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) rest += by_wave[2][w];
    rest /= (float)a.K;
    variance -= rest * rest;
    if (variance < 0) variance = 0;  // all of it cancelled; keeps NaN
  }
  const float r = 1.0f / sqrtf(variance + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[0] = mean + rest;
    if (a.rstd) a.rstd[0] = r;
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = 8 * (threadIdx.x + i * THREADS), left = a.K - k;
    if (left <= 0) break;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] = (x[i][j] - rest) * (r * w[i][j]) + (a.b ? b[i][j] : 0.0f);
    store_eight(a.u + k, narrow<DT>(x[i]), left);
  }
}

// ---- gradients ----------------------------------------------------------------------------------------
// The second launch writes dx and adds every row of its strip; where there are several strips, a third adds them.

struct LayerNormGrad {
  int K, N, rows_per_chunk, chunks, rows_of_apply;
  const uint16_t* x;
  int64_t ldx;
  const float *w, *mean, *rstd;
  const uint16_t* du;
  int64_t ldu;
  const uint16_t* dh;
  uint16_t* dx;  // of ldx, as dh
  float *dw, *db;
  float* sums;      // [2][chunks][N]: g, g xn
  float* row_sums;  // [2][row_strips][K]: du xn, du
  int row_strips;   // of 64 columns, or of eight
  Pieces rows_x, rows_u;  // of x and dh; of du
  Layout layout;
};

__device__ __forceinline__ void store_row_sums(const LayerNormGrad& a, int strip, int k, float of_w, float of_b) {
  if (a.row_strips == 1) {
    if (a.dw) a.dw[k] = of_w;
    if (a.db) a.db[k] = of_b;
  } else {
    a.row_sums[(int64_t)strip * a.K + k] = of_w;
    a.row_sums[(int64_t)(a.row_strips + strip) * a.K + k] = of_b;
  }
}

// Rows in flight together: x, du and dh of each.
struct PatchGrad {
  u32x4 x[kGradRounds], du[kGradRounds], dh[kGradRounds];
  float w[kGradRounds];
};
template <Layout L, bool ALL>  // without dh where only the sums are wanted
__device__ __forceinline__ void load_patch(const LayerNormGrad& a, const Place& p, int k, int end, PatchGrad& v) {
  const u32x4 none = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kGradRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    const bool in = r < end && p.left > 0;
    const int64_t at = (int64_t)r * a.ldx + p.n;
    v.x[i] = in ? draw_eight(a.x + at, p.left, known<L>(a.rows_x)) : none;
    v.du[i] = in ? draw_eight(a.du + (int64_t)r * a.ldu + p.n, p.left, known<L>(a.rows_u)) : none;
    if (ALL) v.dh[i] = in && a.dh ? draw_eight(a.dh + at, p.left, known<L>(a.rows_x)) : none;
  }
#pragma unroll
  for (int i = 0; i < kGradRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    v.w[i] = r >= end ? 0.0f : a.w ? a.w[r] : 1.0f;
  }
}

template <int DT>
__device__ __forceinline__ void add_grad_sums(u32x4 of_x, u32x4 of_du, float w, const float (&m)[8], const float (&r)[8],
                                              float (&sum)[2][8]) {
  float x[8], g[8];
  widen<DT>(of_x, x);
  widen<DT>(of_du, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] *= w;
    sum[0][j] += g[j];
    sum[1][j] += g[j] * ((x[j] - m[j]) * r[j]);
  }
}
// A row's results and its eight columns' part of the channel's two sums.  c0, c1: sums of g and of g xn over K.
template <int DT>
__device__ __forceinline__ void grad_row(u32x4 of_x, u32x4 of_du, u32x4 of_dh, float w, const float (&m)[8], const float (&r)[8],
                                         const float (&c0)[8], const float (&c1)[8], float (&dx)[8], float& of_w, float& of_b) {
  float x[8], du[8];
  widen<DT>(of_x, x);
  widen<DT>(of_du, du);
  widen<DT>(of_dh, dx);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float xn = (x[j] - m[j]) * r[j];
    of_w += du[j] * xn;
    of_b += du[j];
    dx[j] += r[j] * (w * du[j] - c0[j] - xn * c1[j]);
  }
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads) void layer_norm_grad_sums_kernel(LayerNormGrad a) {
  const Place p(a.K, a.N, a.rows_per_chunk, L == kLines);
  if (p.none()) return;
  float sum[2][8] = {}, m[8], r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    m[j] = j < p.left ? a.mean[p.n + j] : 0.0f;
    r[j] = j < p.left ? a.rstd[p.n + j] : 0.0f;
  }
  const int end = p.row0 + p.rows;
  for (int k = p.row0 + (threadIdx.x >> 3); k < end; k += kGradPatch) {
    PatchGrad v;
    load_patch<L, false>(a, p, k, end, v);
#pragma unroll
    for (int i = 0; i < kGradRounds; ++i)
      add_grad_sums<DT>(trim_eight(v.x[i], p.left, known<L>(a.rows_x)), trim_eight(v.du[i], p.left, known<L>(a.rows_u)), v.w[i], m, r, sum);
  }
  store_sums<2>(sum, p, a.sums, a.chunks, a.N);
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads, 3) void layer_norm_grad_apply_kernel(LayerNormGrad a) {
  __shared__ float total[2][kStrip];
  const Place p(a.K, a.N, a.rows_of_apply, L == kLines);
  if (p.none()) return;
  const int end = p.row0 + p.rows, first = p.row0 + (threadIdx.x >> 3), at = 8 * (threadIdx.x & 7);
  PatchGrad v;
  load_patch<L, true>(a, p, first, end, v);
  add_chunks<2>(a.sums, a.chunks, a.N, p, total);
  float m[8], r[8], c0[8], c1[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    m[j] = j < p.left ? a.mean[p.n + j] : 0.0f;
    r[j] = j < p.left ? a.rstd[p.n + j] : 0.0f;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    c0[j] = total[0][at + j] / (float)a.K;
    c1[j] = total[1][at + j] / (float)a.K;
  }
  // whole patches: the lanes of a row add their columns together
  for (int k = first; k - first < p.rows; k += kGradPatch) {
    PatchGrad next;
    if (k - first + kGradPatch < p.rows) load_patch<L, true>(a, p, k + kGradPatch, end, next);
#pragma unroll
    for (int i = 0; i < kGradRounds; ++i) {
      const int row = k + i * kRowsAtOnce;
      const bool in = row < end;
      float dx[8], of_w = 0, of_b = 0;
      grad_row<DT>(trim_eight(v.x[i], p.left, known<L>(a.rows_x)), trim_eight(v.du[i], p.left, known<L>(a.rows_u)),
                   trim_eight(v.dh[i], p.left, known<L>(a.rows_x)), v.w[i], m, r, c0, c1, dx, of_w, of_b);
      if (in && p.left > 0 && a.dx) store_eight<L == kLines>(a.dx + (int64_t)row * a.ldx + p.n, narrow<DT>(dx), p.left);
      of_w = add_eight_lanes(of_w);
      of_b = add_eight_lanes(of_b);
      if (in && (threadIdx.x & 7) == 0) store_row_sums(a, p.strip, row, of_w, of_b);
    }
    v = next;
  }
}

// Few channels or tokens: the sums and the results in one launch, as layer_norm_held_kernel.
template <int DT, int ROUNDS>
__global__ __launch_bounds__(kHeldThreads) void layer_norm_grad_held_kernel(LayerNormGrad a) {
  __shared__ float by_wave[2][kHeldThreads / 64][8], total[2][8];
  const int strip = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  const int n = 8 * strip, left = min(8, a.N - n);
  if (left <= 0) return;
  const u32x4 none = {0, 0, 0, 0};
  u32x4 x[ROUNDS], du[ROUNDS], dh[ROUNDS];
  float w[ROUNDS], m[8], r[8], sum[2][8] = {};
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    const bool in = k < a.K;
    const int64_t at = (int64_t)k * a.ldx + n;
    x[i] = in ? draw_eight(a.x + at, left, a.rows_x) : none;
    du[i] = in ? draw_eight(a.du + (int64_t)k * a.ldu + n, left, a.rows_u) : none;
    dh[i] = in && a.dh ? draw_eight(a.dh + at, left, a.rows_x) : none;
    w[i] = !in ? 0.0f : a.w ? a.w[k] : 1.0f;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    m[j] = j < left ? a.mean[n + j] : 0.0f;
    r[j] = j < left ? a.rstd[n + j] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    x[i] = trim_eight(x[i], left, a.rows_x);
    du[i] = trim_eight(du[i], left, a.rows_u);
    dh[i] = trim_eight(dh[i], left, a.rows_x);
    if ((int)threadIdx.x + i * kHeldThreads < a.K) add_grad_sums<DT>(x[i], du[i], w[i], m, r, sum);
  }
  add_held<2>(sum, by_wave, total);
  float c0[8], c1[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    c0[j] = total[0][j] / (float)a.K;
    c1[j] = total[1][j] / (float)a.K;
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    if (k >= a.K) break;
    float dx[8], of_w = 0, of_b = 0;
    grad_row<DT>(x[i], du[i], dh[i], w[i], m, r, c0, c1, dx, of_w, of_b);
    if (a.dx) store_eight(a.dx + (int64_t)k * a.ldx + n, narrow<DT>(dx), left);
    store_row_sums(a, strip, k, of_w, of_b);
  }
}

// Strips added in a fixed order, kAdders threads a channel, 32 channels (a cache line) a workgroup.
constexpr int kAdders = 32;
__global__ __launch_bounds__(32 * kAdders) void layer_norm_grad_weights_kernel(LayerNormGrad a) {
  __shared__ float part[2][kAdders][32];
  const int col = threadIdx.x & 31, q = threadIdx.x >> 5, k = blockIdx.x * 32 + col;
  float of_w = 0, of_b = 0;
  if (k < a.K) {
#pragma unroll 8
    for (int t = q; t < a.row_strips; t += kAdders) {
      of_w += a.row_sums[(int64_t)t * a.K + k];
      of_b += a.row_sums[(int64_t)(a.row_strips + t) * a.K + k];
    }
  }
  part[0][q][col] = of_w;
  part[1][q][col] = of_b;
  __syncthreads();
  if (q > 0 || k >= a.K) return;
#pragma unroll
  for (int t = 1; t < kAdders; ++t) {
    of_w += part[0][t][col];
    of_b += part[1][t][col];
  }
  if (a.dw) a.dw[k] = of_w;
  if (a.db) a.db[k] = of_b;
}

// Rounds of the forward kernel that holds all rows, or 0.  One launch that reads x once, but only a workgroup to eight columns: us held |
// in strips, 512x64 4.4 | 5.8, 1024x256 4.8 | 5.9, 1024x2048 7.1 | 7.3, 768x4096 8.5 | 8.0, 512x8000 11.2 | 9.1; of four rounds 2048x128
// 5.9 | 6.5, 2048x512 6.5 | 6.3; of eight 4096x17 7.1 | 7.8, 4096x64 11.3 | 7.5.
int rounds_held(int K, int N) {
  if (K <= 2 * kHeldThreads) return (int64_t)K * N <= 2 << 20 ? 2 : 0;
  if (K <= 4 * kHeldThreads) return N <= 256 ? 4 : 0;
  return K <= 8 * kHeldThreads && N <= 16 ? 8 : 0;
}
// Backward, where a launch adds up the workgroups' shares of dw and db in either way: 512x64 6.4 | 7.4, 1024x256 7.3 | 9.4, 1024x2048
// 11.6 | 12.6, and with dh 12.8 | 13.1; 768x4096 14.4 | 15.0, but with dh 17.2 | 15.6; 1024x8000 30.9 | 24.2; of four rounds 2048x32
// 8.4 | 7.5.  At most eight columns have no shares.
int grad_rounds_held(int K, int N) {
  if (K <= 2 * kHeldThreads) return (int64_t)K * N <= 2 << 20 ? 2 : 0;
  return K <= 4 * kHeldThreads && N <= 8 ? 4 : 0;
}

template <int DT, Layout L>
hipError_t launch_strips(const LayerNorm& a, hipStream_t stream) {
  layer_norm_sums_kernel<DT, L><<<grid_of(a.chunks, a.N), kThreads, 0, stream>>>(a);
  layer_norm_apply_kernel<DT, L><<<grid_of((a.K + a.rows_of_apply - 1) / a.rows_of_apply, a.N), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <int DT, bool WHOLE>
void launch_vector(const LayerNorm& a, hipStream_t stream) {
  if (a.K <= 4096) layer_norm_vector_kernel<DT, 512, 1, WHOLE><<<1, 512, 0, stream>>>(a);
  else if (a.K <= 8192) layer_norm_vector_kernel<DT, 1024, 1, WHOLE><<<1, 1024, 0, stream>>>(a);
  else layer_norm_vector_kernel<DT, 1024, 2, WHOLE><<<1, 1024, 0, stream>>>(a);
}

template <int DT>
hipError_t launch_forward(const LayerNorm& a, hipStream_t stream) {
  if (a.N == 1 && a.ldx == 1 && a.ldu == 1 && a.K <= kVectorMost) {
    LayerNorm v = a;
    v.rows = pieces_of_rows(a.x, 8, a.K);
    const bool whole = a.K % 8 == 0 && v.rows == kAligned && at_16_bytes(a.w) && at_16_bytes(a.b);
    if (whole) launch_vector<DT, true>(v, stream);
    else launch_vector<DT, false>(v, stream);
    return hipGetLastError();
  }
  if (const int rounds = rounds_held(a.K, a.N)) {
    const dim3 held((uint32_t)(((a.N + 7) / 8 + 7) / 8 * 8));
    if (rounds == 2) layer_norm_held_kernel<DT, 2><<<held, kHeldThreads, 0, stream>>>(a);
    else if (rounds == 4) layer_norm_held_kernel<DT, 4><<<held, kHeldThreads, 0, stream>>>(a);
    else layer_norm_held_kernel<DT, 8><<<held, kHeldThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  if (a.layout == kLines) return launch_strips<DT, kLines>(a, stream);
  if (a.layout == kPieces) return launch_strips<DT, kPieces>(a, stream);
  return launch_strips<DT, kAny>(a, stream);
}

hipError_t launch_grad_weights(const LayerNormGrad& a, hipStream_t stream) {
  if (a.row_strips > 1 && (a.dw || a.db))
    layer_norm_grad_weights_kernel<<<dim3((uint32_t)((a.K + 31) / 32)), 32 * kAdders, 0, stream>>>(a);
  return hipGetLastError();
}

template <int DT, Layout L>
hipError_t launch_grad_strips(const LayerNormGrad& a, hipStream_t stream) {
  layer_norm_grad_sums_kernel<DT, L><<<grid_of(a.chunks, a.N), kThreads, 0, stream>>>(a);
  layer_norm_grad_apply_kernel<DT, L><<<grid_of((a.K + a.rows_of_apply - 1) / a.rows_of_apply, a.N), kThreads, 0, stream>>>(a);
  return launch_grad_weights(a, stream);
}

template <int DT>
hipError_t launch_backward(const LayerNormGrad& a, hipStream_t stream) {
  if (const int rounds = grad_rounds_held(a.K, a.N)) {
    LayerNormGrad held = a;
    held.row_strips = (a.N + 7) / 8;
    held.row_sums = a.sums;
    const dim3 grid((uint32_t)((held.row_strips + 7) / 8 * 8));
    if (rounds == 2) layer_norm_grad_held_kernel<DT, 2><<<grid, kHeldThreads, 0, stream>>>(held);
    else layer_norm_grad_held_kernel<DT, 4><<<grid, kHeldThreads, 0, stream>>>(held);
    return launch_grad_weights(held, stream);
  }
  if (a.layout == kLines) return launch_grad_strips<DT, kLines>(a, stream);
  if (a.layout == kPieces) return launch_grad_strips<DT, kPieces>(a, stream);
  return launch_grad_strips<DT, kAny>(a, stream);
}

}  // namespace

size_t layer_norm_workspace_bytes(int K, int N) {
  return rounds_held(K, N) ? 0 : (size_t)2 * chunk_count(K, N) * N * sizeof(double);
}
hipError_t launch_layer_norm(const LayerNormArgs& b, hipStream_t stream) {
  LayerNorm a{b.K, b.N, kPatch * chunk_patches(b.K, b.N), chunk_count(b.K, b.N), rows_of_apply(b.K, b.N), b.eps,
              static_cast<const uint16_t*>(b.x), b.ldx, b.w, b.b, static_cast<uint16_t*>(b.u), b.ldu, b.mean, b.rstd,
              reinterpret_cast<double*>(b.workspace), pieces_of_rows(b.x, b.ldx, b.N), kAny};
  a.layout = in_lines(a.x, a.ldx) && in_lines(a.u, a.ldu) ? kLines : a.rows == kAligned ? kPieces : kAny;
  return b.dtype == HINM_F16 ? launch_forward<HINM_F16>(a, stream) : launch_forward<HINM_BF16>(a, stream);
}

size_t layer_norm_grad_workspace_bytes(int K, int N) {
  if (grad_rounds_held(K, N)) return N <= 8 ? 0 : (size_t)2 * ((N + 7) / 8) * K * sizeof(float);
  return ((size_t)2 * chunk_count(K, N) * N + (size_t)2 * strip_count(N) * K) * sizeof(float);
}
hipError_t launch_layer_norm_grad(const LayerNormGradArgs& b, hipStream_t stream) {
  LayerNormGrad a{b.K, b.N, kPatch * chunk_patches(b.K, b.N), chunk_count(b.K, b.N), rows_of_grad_apply(b.K, b.N),
                  static_cast<const uint16_t*>(b.x), b.ldx, b.w, b.mean, b.rstd, static_cast<const uint16_t*>(b.du), b.ldu,
                  static_cast<const uint16_t*>(b.dh), static_cast<uint16_t*>(b.dx), b.dw, b.db, b.workspace,
                  b.workspace + (int64_t)2 * chunk_count(b.K, b.N) * b.N, strip_count(b.N),
                  lesser(pieces_of_rows(b.x, b.ldx, b.N), pieces_of_rows(b.dh, b.ldx, b.N)), pieces_of_rows(b.du, b.ldu, b.N), kAny};
  const bool lines = in_lines(a.x, a.ldx) && in_lines(a.dh, a.ldx) && in_lines(a.dx, a.ldx) && in_lines(a.du, a.ldu);
  a.layout = lines ? kLines : a.rows_x == kAligned && a.rows_u == kAligned ? kPieces : kAny;
  return b.dtype == HINM_F16 ? launch_backward<HINM_F16>(a, stream) : launch_backward<HINM_BF16>(a, stream);
}

}  // namespace hinm
