// Norms on both sides of a block with gates and residual, and their gradients (include/hinm.h).
//
// Matrices are channels x tokens, so a norm's sums run down the columns, and only a workgroup that draws whole cache lines
// (64 columns) of many rows keeps enough of memory in flight: columns are split over workgroups.  Two launches: the first
// adds what every column needs over its rows, by chunks; the second adds the chunks in a fixed order and writes the results.
// The second norm's sum is there after the first launch because h is linear in x and y with factors known per column:
//   h = s x + r t (c y)   with c = gate w_post per channel, t = token_gate, r = rstd_y per token:
//   sum h^2 = s^2 sum x^2 + 2 s r t sum x (c y) + (r t)^2 sum (c y)^2.
// The three may cancel (a block whose output undoes its residual), so they are added in binary64: the products of two floats
// are exact there and the sum keeps its digits down to 2^-50 of what cancels; what h itself loses is its own rounding.
// Infinities do not meet in these sums as they do in h, so the cross term leaves them out (cross_of_finite).  The gradients'
// correction S = sum_k c y d is linear in the gradient d in the same way.
//
// Bound by memory: read twice (the second time from the caches behind L2 where they hold it), written once.  bf16, a channel
// factor and a token's gate, us against what reading and writing once takes at 4.8 TB/s: 4096x2048 23.5 against 14, 4096x8192
// 76 against 56, 16384x1000 (rows that share lines) 53 against 27; gradients 4096x2048 38 against 21, 4096x8192 138 against
// 84, 16384x1000 85 against 41.  Kernels alone: 4096x8192 sums at 5.1 TB/s, results at 6.0; gradients at 4.8 and 4.9.
#include "column_strips.h"

namespace hinm {

namespace {

// ---- forward ------------------------------------------------------------------------------------------

struct Forward {
  int K, N, rows_per_chunk, chunks, rows_of_apply;
  float scale, eps;
  const uint16_t *x, *y;
  const float *w_post, *gate, *token_gate, *w_pre;
  uint16_t* h;
  int64_t ld_stream;
  uint16_t* u;
  int64_t ld_block;
  float *rstd_y, *rstd_h;
  double* sums;  // [4][chunks][N]: y^2, x^2, x c y, (c y)^2
  Pieces stream, block;
  Layout layout;
};

__device__ __forceinline__ float channel_factor(const float* w_post, const float* gate, int k) {
  return (w_post ? w_post[k] : 1.0f) * (gate ? gate[k] : 1.0f);
}

// kRounds rows of x and y of a lane's columns, from row k on in steps of a round, with their channels' factors
struct PatchXY {
  u32x4 x[kRounds], y[kRounds];
  float c[kRounds], w[kRounds];  // gate w_post; w_pre
};
template <Layout L>
__device__ __forceinline__ void load_patch(const Forward& a, const Place& p, int k, int end, PatchXY& v) {
  const u32x4 none = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    const bool in = r < end && p.left > 0;
    v.x[i] = in ? draw_eight(a.x + (int64_t)r * a.ld_stream + p.n, p.left, known<L>(a.stream)) : none;
    v.y[i] = in && a.y ? draw_eight(a.y + (int64_t)r * a.ld_block + p.n, p.left, known<L>(a.block)) : none;
  }
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    v.c[i] = r < end ? channel_factor(a.w_post, a.gate, r) : 0.0f;
    v.w[i] = r < end && a.w_pre ? a.w_pre[r] : 0.0f;
  }
}

// A thread's sums x c y once more, for columns that hold what is not finite: over elements of which both are.  An infinity in x or
// in c y is in its own square's sum, which makes sum h^2 infinite as h is; only where both are infinite and of opposite signs in
// h, h is not a number, and neither is its sum.  (With the products the sum would hold inf - inf, or 0 inf, where h has none.)
template <int DT, Layout L>
__device__ __forceinline__ void cross_of_finite(const Forward& a, const Place& p, double (&squares)[8], double (&cross)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) cross[j] = 0;
#pragma unroll 1
  for (int k = p.row0 + (threadIdx.x >> 3); k < p.row0 + p.rows; k += kRowsAtOnce) {
    const float c = channel_factor(a.w_post, a.gate, k);
    float x[8], y[8];
    widen<DT>(place_eight(draw_eight(a.x + (int64_t)k * a.ld_stream + p.n, p.left, known<L>(a.stream)), p.left, known<L>(a.stream)), x);
    widen<DT>(place_eight(draw_eight(a.y + (int64_t)k * a.ld_block + p.n, p.left, known<L>(a.block)), p.left, known<L>(a.block)), y);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float b = c * y[j];
      const bool x_finite = fabsf(x[j]) < INFINITY, b_finite = fabsf(b) < INFINITY;
      if (x_finite && b_finite) cross[j] += (double)x[j] * b;
      if (x_finite || b_finite || j >= p.left) continue;
      const float t = a.token_gate ? a.token_gate[p.n + j] : 1.0f;
      if ((x[j] < 0) ^ (b < 0) ^ (a.scale < 0) ^ (t < 0)) squares[j] = NAN;
    }
  }
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads) void block_norm_sums_kernel(Forward a) {
  const Place p(a.K, a.N, a.rows_per_chunk, L == kLines);
  if (p.none()) return;
  double sum[4][8] = {};
  float y_squares[8] = {};  // nothing cancels there
  const int end = p.row0 + p.rows;
  for (int k = p.row0 + (threadIdx.x >> 3); k < end; k += kPatch) {
    PatchXY v;
    load_patch<L>(a, p, k, end, v);
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      float x[8], y[8];
      widen<DT>(place_eight(v.x[i], p.left, known<L>(a.stream)), x);
      widen<DT>(place_eight(v.y[i], p.left, known<L>(a.block)), y);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double wide = x[j], b = v.c[i] * y[j];  // c y is rounded to a float as in h
        y_squares[j] += y[j] * y[j];
        sum[1][j] += wide * wide;
        sum[2][j] += wide * b;
        sum[3][j] += b * b;
      }
    }
  }
  bool finite = true;  // squares of floats and sums of them are, in binary64
#pragma unroll
  for (int j = 0; j < 8; ++j) finite = finite && (j >= p.left || sum[1][j] + sum[3][j] < INFINITY);
  if (a.y && !finite) cross_of_finite<DT, L>(a, p, sum[1], sum[2]);
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[0][j] = y_squares[j];
  store_sums<4>(sum, p, a.sums, a.chunks, a.N);
}

template <int DT>
__device__ __forceinline__ void row_of_h(const Forward& a, u32x4 x, u32x4 y, float c, const float (&branch)[8], float (&h)[8]) {
  float v[8];
  widen<DT>(x, h);
  widen<DT>(y, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] = h[j] * a.scale + branch[j] * (c * v[j]);
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads, 4) void block_norm_apply_kernel(Forward a) {
  __shared__ double total[4][kStrip];
  __shared__ float branch[kStrip], root[kStrip];
  const Place p(a.K, a.N, a.rows_of_apply, L == kLines);
  if (p.none()) return;
  const int end = p.row0 + p.rows, first = p.row0 + (threadIdx.x >> 3), at = 8 * (threadIdx.x & 7);
  PatchXY v;
  load_patch<L>(a, p, first, end, v);  // on their way while the sums are added
  if (a.w_post || a.w_pre) add_chunks<4>(a.sums, a.chunks, a.N, p, total);
  __syncthreads();
  if (threadIdx.x < kStrip) {
    const int n = p.n0 + threadIdx.x;
    float b = 1, r = 0;
    if (n < a.N) {
      if (a.token_gate) b = a.token_gate[n];
      if (a.w_post) {
        const float ry = 1.0f / sqrtf((float)(total[0][threadIdx.x] / a.K) + a.eps);
        b *= ry;
        if (a.rstd_y && p.chunk == 0) a.rstd_y[n] = ry;
      }
      if (a.w_pre) {
        const double s = a.scale;
        double sum = s * s * total[1][threadIdx.x];
        if (a.y) sum += 2 * s * b * total[2][threadIdx.x] + (double)b * b * total[3][threadIdx.x];
        if (sum < 0) sum = 0;  // all of it cancelled
        r = 1.0f / sqrtf((float)(sum / a.K) + a.eps);
        if (a.rstd_h && p.chunk == 0) a.rstd_h[n] = r;
      }
    }
    branch[threadIdx.x] = b;
    root[threadIdx.x] = r;
  }
  __syncthreads();
  float of_token[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) of_token[j] = branch[at + j];
  if (p.left <= 0) return;
  float of_u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) of_u[j] = root[at + j];
  for (int k = first; k < end; k += kPatch) {
    PatchXY next;
    if (k + kPatch < end) load_patch<L>(a, p, k + kPatch, end, next);
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int r = k + i * kRowsAtOnce;
      if (r >= end) break;
      float h[8];
      row_of_h<DT>(a, place_eight(v.x[i], p.left, known<L>(a.stream)), place_eight(v.y[i], p.left, known<L>(a.block)), v.c[i],
                   of_token, h);
      if (a.h) store_eight<L == kLines>(a.h + (int64_t)r * a.ld_stream + p.n, narrow<DT>(h), p.left);
      if (a.w_pre) {
        const float w = v.w[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] *= w * of_u[j];
        store_eight<L == kLines>(a.u + (int64_t)r * a.ld_block + p.n, narrow<DT>(h), p.left);
      }
    }
    v = next;
  }
}

// Few channels, or a few tokens: one launch.  A workgroup of 512 threads owns eight columns, a row a lane, and holds x and y of
// all their rows in registers (ROUNDS rows a thread) through both sums.  It draws 16 bytes of each line, so it loses where
// there is much to draw (4096 channels: 8 tokens 10 us against 14.5 in two launches, 64 tokens 20 against 14; 1024 channels:
// 2048 tokens 10.6 against 12.8, 4096 tokens 16.7 against 14.8).
constexpr int kHeldThreads = 512;

// Reciprocal roots of eight columns from every thread's sums of squares.
__device__ __forceinline__ void held_roots(float (&sum)[8], float (*by_wave)[8], float* root, const Forward& a, int n0,
                                           float* out) {
  const int lane = threadIdx.x & 63;
  const float t = add_eight_lanes(add_columns(sum));
  if ((lane & 7) == 0) by_wave[threadIdx.x >> 6][4 * (lane >> 5) + 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1)] = t;
  __syncthreads();
  if (threadIdx.x < 8) {
    float t = 0;
#pragma unroll
    for (int w = 0; w < kHeldThreads / 64; ++w) t += by_wave[w][threadIdx.x];
    const float r = 1.0f / sqrtf(t / (float)a.K + a.eps);
    root[threadIdx.x] = r;
    if (out && n0 + (int)threadIdx.x < a.N) out[n0 + threadIdx.x] = r;
  }
  __syncthreads();
}

template <int DT, int ROUNDS>
__global__ __launch_bounds__(kHeldThreads) void block_norm_held_kernel(Forward a) {
  __shared__ float by_wave[kHeldThreads / 64][8], root[8];
  // neighbouring columns, which share lines, on one XCD
  const int n = 8 * ((int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3)), left = min(8, a.N - n);
  if (left <= 0) return;
  const u32x4 none = {0, 0, 0, 0};
  u32x4 x[ROUNDS], y[ROUNDS];
  float c[ROUNDS], w[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    const bool in = k < a.K;
    x[i] = in ? draw_eight(a.x + (int64_t)k * a.ld_stream + n, left, a.stream) : none;
    y[i] = in && a.y ? draw_eight(a.y + (int64_t)k * a.ld_block + n, left, a.block) : none;
    c[i] = in ? channel_factor(a.w_post, a.gate, k) : 0.0f;
    w[i] = in && a.w_pre ? a.w_pre[k] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    x[i] = place_eight(x[i], left, a.stream);
    y[i] = place_eight(y[i], left, a.block);
  }
  float of_token[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) of_token[j] = a.token_gate && j < left ? a.token_gate[n + j] : 1.0f;
  float sum[8] = {};
  if (a.w_post) {
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      float v[8];
      widen<DT>(y[i], v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j] * v[j];
    }
    held_roots(sum, by_wave, root, a, n, a.rstd_y);
#pragma unroll
    for (int j = 0; j < 8; ++j) of_token[j] *= root[j];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    if (k >= a.K) break;
    float h[8];
    row_of_h<DT>(a, x[i], y[i], c[i], of_token, h);
    if (a.h) store_eight(a.h + (int64_t)k * a.ld_stream + n, narrow<DT>(h), left);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += h[j] * h[j];
  }
  if (!a.w_pre) return;
  held_roots(sum, by_wave, root, a, n, a.rstd_h);
  float of_u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) of_u[j] = root[j];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    if (k >= a.K) break;
    float h[8];
    row_of_h<DT>(a, x[i], y[i], c[i], of_token, h);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] *= w[i] * of_u[j];
    store_eight(a.u + (int64_t)k * a.ld_block + n, narrow<DT>(h), left);
  }
}

// One token without a stride: a vector, held by one workgroup, eight channels a thread and round.  Most of it is a launch and one
// trip to memory, so nothing stands between the loads: WHOLE, whole pieces at multiples of 16 bytes (channels and factors),
// has no row's end to look after (4096 channels in a graph 3.5 us without, 2.7 with; on 1024 threads for 512 3.9 and 3.5).  A
// call: 4096 channels 12.2 us with the kernel above and 8.0 here, 16384 channels 19.9 in two launches and 7.4.
constexpr int kVectorMost = 2 * 8 * 1024;  // channels

template <int DT, int THREADS, int ROUNDS, bool WHOLE>
__global__ __launch_bounds__(THREADS) void block_norm_vector_kernel(Forward a) {
  __shared__ __align__(16) float by_wave[2][THREADS / 64];
  float x[ROUNDS][8], y[ROUNDS][8], c[ROUNDS][8], g[ROUNDS][8], w[ROUNDS][8];
  u32x4 of_x[ROUNDS], of_y[ROUNDS];
  const u32x4 none = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = 8 * (threadIdx.x + i * THREADS), left = a.K - k;
    const int at = WHOLE && left <= 0 ? 0 : k;  // threads beyond the vector read its beginning, and drop it
    of_x[i] = WHOLE ? draw_eight(a.x + at, 8, kAligned) : left > 0 ? draw_eight(a.x + k, left, a.stream) : none;
    of_y[i] = none;
    if (a.y) of_y[i] = WHOLE ? draw_eight(a.y + at, 8, kAligned) : left > 0 ? draw_eight(a.y + k, left, a.block) : none;
    load_factors<WHOLE>(a.w_post, at, left, c[i]);
    load_factors<WHOLE>(a.gate, at, left, g[i]);
    load_factors<WHOLE>(a.w_pre, at, left, w[i]);
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int left = a.K - 8 * (int)(threadIdx.x + i * THREADS);
    widen<DT>(WHOLE ? (left > 0 ? of_x[i] : none) : trim_eight(of_x[i], left, a.stream), x[i]);
    widen<DT>(WHOLE ? (left > 0 ? of_y[i] : none) : trim_eight(of_y[i], left, a.block), y[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) c[i][j] *= g[i][j];
  }
  float token = a.token_gate ? a.token_gate[0] : 1.0f;
  if (a.w_post) {
    float sum = 0;
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += y[i][j] * y[i][j];
    const float r = 1.0f / sqrtf(add_workgroup<THREADS>(sum, by_wave[0]) / (float)a.K + a.eps);
    if (a.rstd_y && threadIdx.x == 0) a.rstd_y[0] = r;
    token *= r;
  }
  float sum = 0;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[i][j] = x[i][j] * a.scale + token * (c[i][j] * y[i][j]);  // h from here on
      sum += x[i][j] * x[i][j];
    }
  if (a.h) {
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      const int k = 8 * (threadIdx.x + i * THREADS), left = a.K - k;
      if (left > 0) store_eight(a.h + k, narrow<DT>(x[i]), left);
    }
  }
  if (!a.w_pre) return;
  const float r = 1.0f / sqrtf(add_workgroup<THREADS>(sum, by_wave[1]) / (float)a.K + a.eps);
  if (a.rstd_h && threadIdx.x == 0) a.rstd_h[0] = r;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = 8 * (threadIdx.x + i * THREADS), left = a.K - k;
    if (left <= 0) break;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] *= w[i][j] * r;
    store_eight(a.u + k, narrow<DT>(x[i]), left);
  }
}

// ---- gradients ----------------------------------------------------------------------------------------
// The second norm's correction needs S = sum_k c d y with d the gradient of h, which itself holds the first correction:
//   s1 = sum_k w_pre du h,   S = sum_k c y dh + rstd_h sum_k c y w_pre du - rstd_h^3 s1 / K sum_k c y h.
// The second launch writes dx and dy and adds every row of its strip; where there are several, a third adds them (4096x3
// 14.7 -> 12 us without it).  Few channels or tokens: one launch, and one that adds the strips where there are several.

struct Backward {
  int K, N, rows_per_chunk, chunks, rows_of_apply;
  float scale;
  const uint16_t *h, *y;
  const float *w_post, *gate, *token_gate, *w_pre, *rstd_y, *rstd_h;
  const uint16_t *dh, *du;
  uint16_t* dx;
  int64_t ld_stream;
  uint16_t* dy;
  int64_t ld_block;
  float *dw_post, *dgate, *dtoken_gate, *dw_pre;
  float* sums;      // [4][chunks][N]
  float* row_sums;  // [2][row_strips][K]
  int row_strips;   // of 64 columns, or of eight
  Pieces stream, block;
  Layout layout;
};

// Channel k's, from its sums over all tokens of du h rstd_h and of d y rstd_y token_gate.
__device__ __forceinline__ void store_weight_gradients(const Backward& a, int k, float of_w_pre, float of_branch) {
  if (a.dw_pre) a.dw_pre[k] = of_w_pre;
  if (a.dw_post) a.dw_post[k] = (a.gate ? a.gate[k] : 1.0f) * of_branch;
  if (a.dgate) a.dgate[k] = (a.w_post ? a.w_post[k] : 1.0f) * of_branch;
}

// ... of a strip's columns
__device__ __forceinline__ void store_row_sums(const Backward& a, int strip, int k, float of_w_pre, float of_branch) {
  if (a.row_strips == 1) {
    store_weight_gradients(a, k, of_w_pre, of_branch);
  } else {
    a.row_sums[(int64_t)strip * a.K + k] = of_w_pre;
    a.row_sums[(int64_t)(a.row_strips + strip) * a.K + k] = of_branch;
  }
}

struct PatchGrad {
  u32x4 h[kGradRounds], dh[kGradRounds], du[kGradRounds], y[kGradRounds];
  float c[kGradRounds], w[kGradRounds];
};
template <Layout L>
__device__ __forceinline__ void load_patch(const Backward& a, const Place& p, int k, int end, PatchGrad& v) {
  const u32x4 none = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kGradRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    const bool in = r < end && p.left > 0;
    const int64_t stream = (int64_t)r * a.ld_stream + p.n, block = (int64_t)r * a.ld_block + p.n;
    v.h[i] = in && a.w_pre ? draw_eight(a.h + stream, p.left, known<L>(a.stream)) : none;
    v.dh[i] = in && a.dh ? draw_eight(a.dh + stream, p.left, known<L>(a.stream)) : none;
    v.du[i] = in && a.w_pre ? draw_eight(a.du + block, p.left, known<L>(a.block)) : none;
    v.y[i] = in && a.y ? draw_eight(a.y + block, p.left, known<L>(a.block)) : none;
  }
#pragma unroll
  for (int i = 0; i < kGradRounds; ++i) {
    const int r = k + i * kRowsAtOnce;
    v.c[i] = r < end ? channel_factor(a.w_post, a.gate, r) : 0.0f;
    v.w[i] = r < end && a.w_pre ? a.w_pre[r] : 0.0f;
  }
}

// A row's part of a column's four sums.
template <int DT>
__device__ __forceinline__ void add_grad_sums(u32x4 of_h, u32x4 of_dh, u32x4 of_du, u32x4 of_y, float c, float w,
                                              float (&sum)[4][8]) {
  float h[8], dh[8], g[8], y[8];
  widen<DT>(of_h, h);
  widen<DT>(of_dh, dh);
  widen<DT>(of_du, g);
  widen<DT>(of_y, y);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] *= w;
    y[j] *= c;
    sum[0][j] += g[j] * h[j];
    sum[1][j] += y[j] * dh[j];
    sum[2][j] += y[j] * g[j];
    sum[3][j] += y[j] * h[j];
  }
}
// From their totals: the factors of h and of y in the corrections, rstd_h^3 s1 / K and rstd_y^2 S / K.  first: the one that
// writes the token's gradient.
__device__ __forceinline__ void corrections(const Backward& a, int n, bool first, float s0, float s1, float s2, float s3, float& f1,
                                            float& f2) {
  f1 = f2 = 0;
  if (n >= a.N) return;
  const float r = a.w_pre ? a.rstd_h[n] : 0.0f, ry = a.w_post ? a.rstd_y[n] : 1.0f;
  // one factor after the other: the cube of a reciprocal root leaves float32 where the root of a token of 10^13 does not
  f1 = r * (r * (r * (s0 / (float)a.K)));
  const float S = s1 + r * s2 - f1 * s3;
  f2 = a.w_post ? ry * (ry * (S / (float)a.K)) : 0.0f;
  if (a.dtoken_gate && first) a.dtoken_gate[n] = S * ry;
}
// A row's results and its eight columns' part of the channel's two sums.
template <int DT>
__device__ __forceinline__ void grad_row(const Backward& a, u32x4 of_h, u32x4 of_dh, u32x4 of_du, u32x4 of_y, float c, float w,
                                         const float (&rh)[8], const float (&token)[8], const float (&f1)[8], const float (&f2)[8],
                                         float (&dx)[8], float (&dy)[8], float& of_w_pre, float& of_branch) {
  float h[8], g[8];
  widen<DT>(of_h, h);
  widen<DT>(of_dh, dx);
  widen<DT>(of_du, g);
  widen<DT>(of_y, dy);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    of_w_pre += g[j] * h[j] * rh[j];
    const float d = dx[j] + w * g[j] * rh[j] - h[j] * f1[j];
    of_branch += d * dy[j] * token[j];
    dx[j] = a.scale * d;
    dy[j] = token[j] * (c * d - dy[j] * f2[j]);
  }
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads) void block_norm_grad_sums_kernel(Backward a) {
  const Place p(a.K, a.N, a.rows_per_chunk, L == kLines);
  if (p.none()) return;
  float sum[4][8] = {};
  const int end = p.row0 + p.rows;
  for (int k = p.row0 + (threadIdx.x >> 3); k < end; k += kGradPatch) {
    PatchGrad v;
    load_patch<L>(a, p, k, end, v);
#pragma unroll
    for (int i = 0; i < kGradRounds; ++i)
      add_grad_sums<DT>(trim_eight(v.h[i], p.left, known<L>(a.stream)), trim_eight(v.dh[i], p.left, known<L>(a.stream)),
                        trim_eight(v.du[i], p.left, known<L>(a.block)), trim_eight(v.y[i], p.left, known<L>(a.block)), v.c[i],
                        v.w[i], sum);
  }
  store_sums<4>(sum, p, a.sums, a.chunks, a.N);
}

template <int DT, Layout L>
__global__ __launch_bounds__(kThreads, 3) void block_norm_grad_apply_kernel(Backward a) {
  __shared__ float total[4][kStrip], first_of[kStrip], second_of[kStrip];  // corrections: rstd_h^3 s1 / K; rstd_y^2 S / K
  const Place p(a.K, a.N, a.rows_of_apply, L == kLines);
  if (p.none()) return;
  const int end = p.row0 + p.rows, first = p.row0 + (threadIdx.x >> 3), at = 8 * (threadIdx.x & 7);
  PatchGrad v;
  load_patch<L>(a, p, first, end, v);
  add_chunks<4>(a.sums, a.chunks, a.N, p, total);
  float rh[8], token[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool in = j < p.left;
    rh[j] = in && a.w_pre ? a.rstd_h[p.n + j] : 0.0f;
    token[j] = !in ? 0.0f : (a.token_gate ? a.token_gate[p.n + j] : 1.0f) * (a.w_post ? a.rstd_y[p.n + j] : 1.0f);
  }
  __syncthreads();
  if (threadIdx.x < kStrip) {
    float f1, f2;
    corrections(a, p.n0 + (int)threadIdx.x, p.chunk == 0, total[0][threadIdx.x], total[1][threadIdx.x], total[2][threadIdx.x],
                total[3][threadIdx.x], f1, f2);
    first_of[threadIdx.x] = f1;
    second_of[threadIdx.x] = f2;
  }
  __syncthreads();
  float f1[8], f2[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f1[j] = first_of[at + j];
    f2[j] = second_of[at + j];
  }
  // whole patches: the lanes of a row add their columns together
  for (int k = first; k - first < p.rows; k += kGradPatch) {
    PatchGrad next;
    if (k - first + kGradPatch < p.rows) load_patch<L>(a, p, k + kGradPatch, end, next);
#pragma unroll
    for (int i = 0; i < kGradRounds; ++i) {
      const int r = k + i * kRowsAtOnce;
      const bool in = r < end;
      float dx[8], dy[8], of_w_pre = 0, of_branch = 0;
      grad_row<DT>(a, trim_eight(v.h[i], p.left, known<L>(a.stream)), trim_eight(v.dh[i], p.left, known<L>(a.stream)),
                   trim_eight(v.du[i], p.left, known<L>(a.block)), trim_eight(v.y[i], p.left, known<L>(a.block)), v.c[i], v.w[i],
                   rh, token, f1, f2, dx, dy, of_w_pre, of_branch);
      if (in && p.left > 0) {
        if (a.dx) store_eight<L == kLines>(a.dx + (int64_t)r * a.ld_stream + p.n, narrow<DT>(dx), p.left);
        if (a.dy) store_eight<L == kLines>(a.dy + (int64_t)r * a.ld_block + p.n, narrow<DT>(dy), p.left);
      }
      of_w_pre = add_eight_lanes(of_w_pre);
      of_branch = add_eight_lanes(of_branch);
      if (in && (threadIdx.x & 7) == 0) {
        store_row_sums(a, p.strip, r, of_w_pre, of_branch);
      }
    }
    v = next;
  }
}

// Few channels or tokens: the sums and the results in one launch, as block_norm_held_kernel.
template <int DT, int ROUNDS>
__global__ __launch_bounds__(kHeldThreads) void block_norm_grad_held_kernel(Backward a) {
  __shared__ float by_wave[4][kHeldThreads / 64][8], first_of[8], second_of[8];
  const int strip = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  const int n = 8 * strip, left = min(8, a.N - n);
  if (left <= 0) return;
  const u32x4 none = {0, 0, 0, 0};
  u32x4 h[ROUNDS], dh[ROUNDS], du[ROUNDS], y[ROUNDS];
  float c[ROUNDS], w[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    const bool in = k < a.K;
    const int64_t stream = (int64_t)k * a.ld_stream + n, block = (int64_t)k * a.ld_block + n;
    h[i] = in && a.w_pre ? draw_eight(a.h + stream, left, a.stream) : none;
    dh[i] = in && a.dh ? draw_eight(a.dh + stream, left, a.stream) : none;
    du[i] = in && a.w_pre ? draw_eight(a.du + block, left, a.block) : none;
    y[i] = in && a.y ? draw_eight(a.y + block, left, a.block) : none;
    c[i] = in ? channel_factor(a.w_post, a.gate, k) : 0.0f;
    w[i] = in && a.w_pre ? a.w_pre[k] : 0.0f;
  }
  float rh[8], token[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    rh[j] = j < left && a.w_pre ? a.rstd_h[n + j] : 0.0f;
    token[j] = j >= left ? 0.0f : (a.token_gate ? a.token_gate[n + j] : 1.0f) * (a.w_post ? a.rstd_y[n + j] : 1.0f);
  }
  float sum[4][8] = {};
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    h[i] = trim_eight(h[i], left, a.stream);
    dh[i] = trim_eight(dh[i], left, a.stream);
    du[i] = trim_eight(du[i], left, a.block);
    y[i] = trim_eight(y[i], left, a.block);
    add_grad_sums<DT>(h[i], dh[i], du[i], y[i], c[i], w[i], sum);
  }
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float t = add_eight_lanes(add_columns(sum[q]));
    if ((lane & 7) == 0) by_wave[q][threadIdx.x >> 6][4 * (lane >> 5) + 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1)] = t;
  }
  __syncthreads();
  if (threadIdx.x < 8) {
    float t[4] = {};
#pragma unroll
    for (int v = 0; v < kHeldThreads / 64; ++v)
#pragma unroll
      for (int q = 0; q < 4; ++q) t[q] += by_wave[q][v][threadIdx.x];
    corrections(a, n + (int)threadIdx.x, true, t[0], t[1], t[2], t[3], first_of[threadIdx.x], second_of[threadIdx.x]);
  }
  __syncthreads();
  float f1[8], f2[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f1[j] = first_of[j];
    f2[j] = second_of[j];
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int k = threadIdx.x + i * kHeldThreads;
    if (k >= a.K) break;
    float dx[8], dy[8], of_w_pre = 0, of_branch = 0;
    grad_row<DT>(a, h[i], dh[i], du[i], y[i], c[i], w[i], rh, token, f1, f2, dx, dy, of_w_pre, of_branch);
    if (a.dx) store_eight(a.dx + (int64_t)k * a.ld_stream + n, narrow<DT>(dx), left);
    if (a.dy) store_eight(a.dy + (int64_t)k * a.ld_block + n, narrow<DT>(dy), left);
    store_row_sums(a, strip, k, of_w_pre, of_branch);
  }
}

// Strips added in a fixed order, kAdders threads a channel, 32 channels (a cache line) a workgroup: 2 to 5 us, a launch and a trip
// to memory (768x1000, 125 strips: 3.0 us, with 8 threads a channel 4.2).
constexpr int kAdders = 32;
__global__ __launch_bounds__(32 * kAdders) void block_norm_grad_weights_kernel(Backward a) {
  __shared__ float part[2][kAdders][32];
  const int col = threadIdx.x & 31, q = threadIdx.x >> 5, k = blockIdx.x * 32 + col;
  float of_w_pre = 0, of_branch = 0;
  if (k < a.K) {
#pragma unroll 8
    for (int t = q; t < a.row_strips; t += kAdders) {
      of_w_pre += a.row_sums[(int64_t)t * a.K + k];
      of_branch += a.row_sums[(int64_t)(a.row_strips + t) * a.K + k];
    }
  }
  part[0][q][col] = of_w_pre;
  part[1][q][col] = of_branch;
  __syncthreads();
  if (q > 0 || k >= a.K) return;
#pragma unroll
  for (int t = 1; t < kAdders; ++t) {
    of_w_pre += part[0][t][col];
    of_branch += part[1][t][col];
  }
  store_weight_gradients(a, k, of_w_pre, of_branch);
}

}  // namespace

// Rounds of the forward kernel that holds all rows, or 0.
static int rounds_held(int K, int N) {
  if (K <= 2 * kHeldThreads && (int64_t)K * N <= 3 << 20) return 2;
  return K <= 8 * kHeldThreads && N <= 16 ? 8 : 0;
}
size_t block_norm_workspace_bytes(int K, int N) {
  return rounds_held(K, N) ? 0 : (size_t)4 * chunk_count(K, N) * N * sizeof(double);
}

template <int DT, Layout L>
static hipError_t launch_forward_strips(const Forward& a, hipStream_t stream) {
  if (a.w_post || a.w_pre) block_norm_sums_kernel<DT, L><<<grid_of(a.chunks, a.N), kThreads, 0, stream>>>(a);
  block_norm_apply_kernel<DT, L><<<grid_of((a.K + a.rows_of_apply - 1) / a.rows_of_apply, a.N), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <int DT, bool WHOLE>
static void launch_vector(const Forward& a, hipStream_t stream) {
  if (a.K <= 4096) block_norm_vector_kernel<DT, 512, 1, WHOLE><<<1, 512, 0, stream>>>(a);
  else if (a.K <= 8192) block_norm_vector_kernel<DT, 1024, 1, WHOLE><<<1, 1024, 0, stream>>>(a);
  else block_norm_vector_kernel<DT, 1024, 2, WHOLE><<<1, 1024, 0, stream>>>(a);
}

template <int DT>
static hipError_t launch_forward(const Forward& a, hipStream_t stream) {
  if (a.N == 1 && a.ld_stream == 1 && (a.ld_block == 1 || (!a.y && !a.w_pre)) && a.K <= kVectorMost) {
    Forward v = a;
    v.stream = pieces_of_rows(a.x, 8, a.K);
    v.block = pieces_of_rows(a.y, 8, a.K);
    const bool whole = a.K % 8 == 0 && v.stream == kAligned && v.block == kAligned && at_16_bytes(a.w_post) &&
                       at_16_bytes(a.gate) && at_16_bytes(a.w_pre);
    if (whole) launch_vector<DT, true>(v, stream);
    else launch_vector<DT, false>(v, stream);
    return hipGetLastError();
  }
  if (const int rounds = rounds_held(a.K, a.N)) {
    const dim3 held((uint32_t)(((a.N + 7) / 8 + 7) / 8 * 8));
    if (rounds == 2) block_norm_held_kernel<DT, 2><<<held, kHeldThreads, 0, stream>>>(a);
    else block_norm_held_kernel<DT, 8><<<held, kHeldThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  if (a.layout == kLines) return launch_forward_strips<DT, kLines>(a, stream);
  if (a.layout == kPieces) return launch_forward_strips<DT, kPieces>(a, stream);
  return launch_forward_strips<DT, kAny>(a, stream);
}

hipError_t launch_block_norm(const BlockNormArgs& b, hipStream_t stream) {
  Forward a{b.K, b.N, kPatch * chunk_patches(b.K, b.N), chunk_count(b.K, b.N), rows_of_apply(b.K, b.N), b.residual_scale, b.eps,
            static_cast<const uint16_t*>(b.x), static_cast<const uint16_t*>(b.y), b.w_post, b.gate, b.token_gate, b.w_pre,
            static_cast<uint16_t*>(b.h), b.ld_stream, static_cast<uint16_t*>(b.u), b.ld_block, b.rstd_y, b.rstd_h,
            reinterpret_cast<double*>(b.workspace), kAligned, kAligned, kAny};
  a.stream = pieces_of_rows(a.x, a.ld_stream, a.N);
  a.block = pieces_of_rows(a.y, a.ld_block, a.N);
  const bool lines = in_lines(a.x, a.ld_stream) && in_lines(a.h, a.ld_stream) && in_lines(a.y, a.ld_block) &&
                     in_lines(a.u, a.ld_block);
  a.layout = lines ? kLines : a.stream == kAligned && a.block == kAligned ? kPieces : kAny;
  return b.dtype == HINM_F16 ? launch_forward<HINM_F16>(a, stream) : launch_forward<HINM_BF16>(a, stream);
}

// Rounds of the kernel that holds all rows, or 0 (us in two launches and three, and there): one launch for up to eight tokens
// (256x1 16.7 and 8.5, 2048x8 12.2 and 9.0); two for few channels and not too much to draw in pieces of 16 bytes (768x200 14.6 and
// 11.5, 768x1000 15.1 and 14.1, 1024x1000 15.1 and 15.8, 768x4096 20 and 26), nor too many strips to add (64x4096 14.7
// and 12.1, 64x16000 15.6 and 37).
static int grad_rounds_held(int K, int N) {
  if (N <= 8) return K <= 2 * kHeldThreads ? 2 : K <= 4 * kHeldThreads ? 4 : 0;
  return K <= 2 * kHeldThreads && N <= 4096 && (int64_t)K * N <= 3 << 18 ? 2 : 0;
}
size_t block_norm_grad_workspace_bytes(int K, int N) {
  if (grad_rounds_held(K, N)) return N <= 8 ? 0 : (size_t)2 * ((N + 7) / 8) * K * sizeof(float);
  return ((size_t)4 * chunk_count(K, N) * N + (size_t)2 * strip_count(N) * K) * sizeof(float);
}

static hipError_t launch_grad_weights(const Backward& a, hipStream_t stream) {
  if (a.row_strips > 1 && (a.dw_pre || a.dw_post || a.dgate))
    block_norm_grad_weights_kernel<<<dim3((uint32_t)((a.K + 31) / 32)), 32 * kAdders, 0, stream>>>(a);
  return hipGetLastError();
}

template <int DT, Layout L>
static hipError_t launch_backward_strips(const Backward& a, hipStream_t stream) {
  block_norm_grad_sums_kernel<DT, L><<<grid_of(a.chunks, a.N), kThreads, 0, stream>>>(a);
  block_norm_grad_apply_kernel<DT, L><<<grid_of((a.K + a.rows_of_apply - 1) / a.rows_of_apply, a.N), kThreads, 0, stream>>>(a);
  return launch_grad_weights(a, stream);
}

template <int DT>
static hipError_t launch_backward(const Backward& a, hipStream_t stream) {
  if (const int rounds = grad_rounds_held(a.K, a.N)) {
    Backward held = a;
    held.row_strips = (a.N + 7) / 8;
    held.row_sums = a.sums;
    const dim3 grid((uint32_t)((held.row_strips + 7) / 8 * 8));
    if (rounds == 2) block_norm_grad_held_kernel<DT, 2><<<grid, kHeldThreads, 0, stream>>>(held);
    else block_norm_grad_held_kernel<DT, 4><<<grid, kHeldThreads, 0, stream>>>(held);
    return launch_grad_weights(held, stream);
  }
  if (a.layout == kLines) return launch_backward_strips<DT, kLines>(a, stream);
  if (a.layout == kPieces) return launch_backward_strips<DT, kPieces>(a, stream);
  return launch_backward_strips<DT, kAny>(a, stream);
}

hipError_t launch_block_norm_grad(const BlockNormGradArgs& b, hipStream_t stream) {
  Backward a{b.K, b.N, kPatch * chunk_patches(b.K, b.N), chunk_count(b.K, b.N), rows_of_grad_apply(b.K, b.N), b.residual_scale,
             static_cast<const uint16_t*>(b.h), static_cast<const uint16_t*>(b.y), b.w_post, b.gate, b.token_gate, b.w_pre,
             b.rstd_y, b.rstd_h, static_cast<const uint16_t*>(b.dh), static_cast<const uint16_t*>(b.du),
             static_cast<uint16_t*>(b.dx), b.ld_stream, static_cast<uint16_t*>(b.dy), b.ld_block, b.dw_post, b.dgate,
             b.dtoken_gate, b.dw_pre, b.workspace, b.workspace + (int64_t)4 * chunk_count(b.K, b.N) * b.N,
             strip_count(b.N), kAligned, kAligned, kAny};
  a.stream = lesser(pieces_of_rows(a.h, a.ld_stream, a.N), pieces_of_rows(a.dh, a.ld_stream, a.N));
  a.block = lesser(pieces_of_rows(a.y, a.ld_block, a.N), pieces_of_rows(a.du, a.ld_block, a.N));
  const bool lines = in_lines(a.h, a.ld_stream) && in_lines(a.dh, a.ld_stream) && in_lines(a.dx, a.ld_stream) &&
                     in_lines(a.y, a.ld_block) && in_lines(a.du, a.ld_block) && in_lines(a.dy, a.ld_block);
  a.layout = lines ? kLines : a.stream == kAligned && a.block == kAligned ? kPieces : kAny;
  return b.dtype == HINM_F16 ? launch_backward<HINM_F16>(a, stream) : launch_backward<HINM_BF16>(a, stream);
}

}  // namespace hinm
