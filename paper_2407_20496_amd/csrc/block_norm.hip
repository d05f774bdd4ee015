// Norms on both sides of a block with gates and residual, and their gradients (include/hinm.h).
//
// Matrices are channels x tokens, so a norm's sums run down the columns.  A workgroup owns a strip of 64 columns (eight
// lanes of eight) and a chunk of rows; partial sums of the chunks meet in the workspace and every later pass adds them in the
// same order.
#include "eight_values.h"

namespace hinm {

namespace {

constexpr int kThreads = 256;
constexpr int kStrip = 64;                      // columns of a workgroup
constexpr int kRowsAtOnce = kThreads / 8;       // rows that its lanes cover together
constexpr int kWaves = kThreads / 64;

// Rows of a chunk: at least 128, and at most 64 chunks.
int chunk_rows(int K) {
  const int least = (K + 63) / 64;
  return least <= 128 ? 128 : (least + kRowsAtOnce - 1) / kRowsAtOnce * kRowsAtOnce;
}
int chunk_count(int K) { return (K + chunk_rows(K) - 1) / chunk_rows(K); }
int strip_count(int N) { return (N + kStrip - 1) / kStrip; }

struct Strip {
  int n0, n, left, row0, rows, chunk;  // first column; this lane's first column and how many it has; rows of the chunk
  __device__ __forceinline__ Strip(int K, int N, int rows_per_chunk) {
    const int strips = (N + kStrip - 1) / kStrip;
    chunk = blockIdx.x / strips;
    n0 = (blockIdx.x - chunk * strips) * kStrip;
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

// Sums of the workgroup's 64 columns over its threads: `s` eight columns of this thread, the result (fixed order) in
// total[0..63] after the call's last barrier.
__device__ __forceinline__ void add_strip(float (&s)[8], float* by_wave, float* total) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    s[j] += __shfl_xor(s[j], 8);
    s[j] += __shfl_xor(s[j], 16);
    s[j] += __shfl_xor(s[j], 32);
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) by_wave[wave * kStrip + 8 * lane + j] = s[j];
  }
  __syncthreads();
  if (threadIdx.x < kStrip) {
    float t = 0;
    for (int w = 0; w < kWaves; ++w) t += by_wave[w * kStrip + threadIdx.x];
    total[threadIdx.x] = t;
  }
  __syncthreads();
}

// Sum over the chunks of one column's partial sums.
__device__ __forceinline__ float add_chunks(const float* partial, int chunks, int N, int n) {
  float t = 0;
  for (int c = 0; c < chunks; ++c) t += partial[(int64_t)c * N + n];
  return t;
}

// ---- forward ------------------------------------------------------------------------------------------

struct Forward {
  int K, N, rows_per_chunk, chunks;
  float scale, eps;
  const uint16_t *x, *y;
  const float *w_post, *gate, *token_gate, *w_pre;
  uint16_t* h;
  int64_t ld_stream;
  uint16_t* u;
  int64_t ld_block;
  float *rstd_y, *rstd_h;
  float *sum_y, *sum_h;  // [chunks][N]
  bool vec_stream, vec_block;
};

// eight columns of h in one row
template <int DT>
__device__ __forceinline__ void row_of_h(const Forward& a, int k, int n, int left, const float (&token)[8], float (&h)[8]) {
  widen<DT>(load_eight(a.x + (int64_t)k * a.ld_stream + n, left, a.vec_stream), h);
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] *= a.scale;
  if (a.y) {
    float y[8];
    widen<DT>(load_eight(a.y + (int64_t)k * a.ld_block + n, left, a.vec_block), y);
    const float c = (a.w_post ? a.w_post[k] : 1.0f) * (a.gate ? a.gate[k] : 1.0f);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] += c * (token[j] * y[j]);
  }
}

// token_gate rstd_y of a lane's columns
__device__ __forceinline__ void factors_of_tokens(const Forward& a, const Strip& s, const float* rstd, float (&token)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    token[j] = j < s.left && a.token_gate ? a.token_gate[s.n + j] : 1.0f;
    if (a.w_post) token[j] *= rstd[s.n - s.n0 + j];
  }
}

// rstd of the strip's columns from the chunks' sums, to LDS and (by the first chunk's workgroups) to memory
__device__ __forceinline__ void finish_rstd(const Forward& a, const Strip& s, const float* sums, float* out, float* rstd) {
  if (threadIdx.x < kStrip) {
    const int n = s.n0 + threadIdx.x;
    float r = 0;
    if (n < a.N) {
      r = 1.0f / sqrtf(add_chunks(sums, a.chunks, a.N, n) / (float)a.K + a.eps);
      if (out && s.chunk == 0) out[n] = r;
    }
    rstd[threadIdx.x] = r;
  }
  __syncthreads();
}

// PASS 0: sums of y^2.  1: sums of h^2.  2: h and u.
template <int DT, int PASS>
__global__ __launch_bounds__(kThreads) void block_norm_pass_kernel(Forward a) {
  __shared__ float by_wave[kWaves * kStrip], total[kStrip], rstd_y[kStrip], rstd_h[kStrip];
  const Strip s(a.K, a.N, a.rows_per_chunk);
  if constexpr (PASS > 0) {
    if (a.w_post) finish_rstd(a, s, a.sum_y, PASS == 2 ? a.rstd_y : nullptr, rstd_y);
    if (PASS == 2 && a.w_pre) finish_rstd(a, s, a.sum_h, a.rstd_h, rstd_h);
  }
  float token[8], sum[8] = {};
  if constexpr (PASS > 0) factors_of_tokens(a, s, rstd_y, token);
  if (s.left > 0) {
    for (int i = threadIdx.x >> 3; i < s.rows; i += kRowsAtOnce) {
      const int k = s.row0 + i;
      float v[8];
      if constexpr (PASS == 0) {
        widen<DT>(load_eight(a.y + (int64_t)k * a.ld_block + s.n, s.left, a.vec_block), v);
      } else {
        row_of_h<DT>(a, k, s.n, s.left, token, v);
      }
      if constexpr (PASS < 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j] * v[j];
      } else {
        if (a.h) store_eight(a.h + (int64_t)k * a.ld_stream + s.n, narrow<DT>(v), s.left, a.vec_stream);
        if (a.w_pre) {
          const float w = a.w_pre[k];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= w * rstd_h[s.n - s.n0 + j];
          store_eight(a.u + (int64_t)k * a.ld_block + s.n, narrow<DT>(v), s.left, a.vec_block);
        }
      }
    }
  }
  if constexpr (PASS < 2) {
    add_strip(sum, by_wave, total);
    const int n = s.n0 + threadIdx.x;
    if (threadIdx.x < kStrip && n < a.N) (PASS == 0 ? a.sum_y : a.sum_h)[(int64_t)s.chunk * a.N + n] = total[threadIdx.x];
  }
}

// ---- gradients ----------------------------------------------------------------------------------------
// The second norm's correction needs S = sum_k c d y with c = gate w_post and d the gradient of h, which itself holds the
// first correction.  S is linear in d, so one pass over the inputs gives both:
//   s1 = sum_k w_pre du h,   S = sum_k c y dh + rstd_h sum_k c y w_pre du - rstd_h^3 s1 / K sum_k c y h.
// A second pass writes dx and dy and adds every row of its strip; a third adds the strips.

struct Backward {
  int K, N, rows_per_chunk, chunks;
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
  float* row_sums;  // [2][strips][K]
  bool vec_stream, vec_block;
};

template <int DT>
__device__ __forceinline__ void grad_row(const Backward& a, int k, int n, int left, float (&h)[8], float (&dh)[8], float (&g)[8],
                                         float (&y)[8]) {
  const int64_t at_stream = (int64_t)k * a.ld_stream + n, at_block = (int64_t)k * a.ld_block + n;
  const u32x4 none = {0, 0, 0, 0};
  widen<DT>(a.w_pre ? load_eight(a.h + at_stream, left, a.vec_stream) : none, h);
  widen<DT>(a.dh ? load_eight(a.dh + at_stream, left, a.vec_stream) : none, dh);
  widen<DT>(a.w_pre ? load_eight(a.du + at_block, left, a.vec_block) : none, g);
  widen<DT>(a.y ? load_eight(a.y + at_block, left, a.vec_block) : none, y);
}
__device__ __forceinline__ float factor_of_channel(const Backward& a, int k) {
  return (a.w_post ? a.w_post[k] : 1.0f) * (a.gate ? a.gate[k] : 1.0f);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void block_norm_grad_sums_kernel(Backward a) {
  __shared__ float by_wave[kWaves * kStrip], total[kStrip];
  const Strip s(a.K, a.N, a.rows_per_chunk);
  float sum[4][8] = {};
  if (s.left > 0) {
    for (int i = threadIdx.x >> 3; i < s.rows; i += kRowsAtOnce) {
      const int k = s.row0 + i;
      float h[8], dh[8], g[8], y[8];
      grad_row<DT>(a, k, s.n, s.left, h, dh, g, y);
      const float w = a.w_pre ? a.w_pre[k] : 0.0f, c = factor_of_channel(a, k);
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
  }
  const int n = s.n0 + threadIdx.x;
  for (int q = 0; q < 4; ++q) {
    add_strip(sum[q], by_wave, total);
    if (threadIdx.x < kStrip && n < a.N) a.sums[((int64_t)q * a.chunks + s.chunk) * a.N + n] = total[threadIdx.x];
  }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void block_norm_grad_rows_kernel(Backward a) {
  __shared__ float first[kStrip], second[kStrip];  // corrections per column: rstd_h^3 s1 / K; rstd_y^2 S / K
  const Strip s(a.K, a.N, a.rows_per_chunk);
  const int strips = (a.N + kStrip - 1) / kStrip, strip = s.n0 / kStrip;
  if (threadIdx.x < kStrip) {
    const int n = s.n0 + threadIdx.x;
    float f1 = 0, f2 = 0;
    if (n < a.N) {
      float t[4];
      for (int q = 0; q < 4; ++q) t[q] = add_chunks(a.sums + (int64_t)q * a.chunks * a.N, a.chunks, a.N, n);
      const float rh = a.w_pre ? a.rstd_h[n] : 0.0f, ry = a.w_post ? a.rstd_y[n] : 1.0f;
      f1 = rh * rh * rh * (t[0] / (float)a.K);
      const float S = t[1] + rh * t[2] - f1 * t[3];
      f2 = a.w_post ? ry * ry * (S / (float)a.K) : 0.0f;
      if (a.dtoken_gate && s.chunk == 0) a.dtoken_gate[n] = S * ry;
    }
    first[threadIdx.x] = f1;
    second[threadIdx.x] = f2;
  }
  __syncthreads();
  float rh[8], token[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool in = j < s.left;
    rh[j] = in && a.w_pre ? a.rstd_h[s.n + j] : 0.0f;
    token[j] = !in ? 0.0f : (a.token_gate ? a.token_gate[s.n + j] : 1.0f) * (a.w_post ? a.rstd_y[s.n + j] : 1.0f);
  }
  // whole rounds of rows: the lanes of a row add their columns together
  for (int i0 = 0; i0 < s.rows; i0 += kRowsAtOnce) {
    const int i = i0 + (threadIdx.x >> 3), k = s.row0 + i;
    float of_w_pre = 0, of_branch = 0;
    if (i < s.rows && s.left > 0) {
      float h[8], dh[8], g[8], y[8];
      grad_row<DT>(a, k, s.n, s.left, h, dh, g, y);
      const float w = a.w_pre ? a.w_pre[k] : 0.0f, c = factor_of_channel(a, k);
      const int at = s.n - s.n0;
      float dx[8], dy[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        of_w_pre += g[j] * h[j] * rh[j];
        const float d = dh[j] + w * g[j] * rh[j] - h[j] * first[at + j];
        of_branch += d * y[j] * token[j];
        dx[j] = a.scale * d;
        dy[j] = token[j] * (c * d - y[j] * second[at + j]);
      }
      if (a.dx) store_eight(a.dx + (int64_t)k * a.ld_stream + s.n, narrow<DT>(dx), s.left, a.vec_stream);
      if (a.dy) store_eight(a.dy + (int64_t)k * a.ld_block + s.n, narrow<DT>(dy), s.left, a.vec_block);
    }
#pragma unroll
    for (int q = 1; q < 8; q *= 2) {
      of_w_pre += __shfl_xor(of_w_pre, q);
      of_branch += __shfl_xor(of_branch, q);
    }
    if (i < s.rows && (threadIdx.x & 7) == 0) {
      a.row_sums[(int64_t)strip * a.K + k] = of_w_pre;
      a.row_sums[(int64_t)(strips + strip) * a.K + k] = of_branch;
    }
  }
}

__global__ __launch_bounds__(kThreads) void block_norm_grad_weights_kernel(Backward a) {
  const int strips = (a.N + kStrip - 1) / kStrip;
  const int k = blockIdx.x * kThreads + threadIdx.x;
  if (k >= a.K) return;
  float of_w_pre = 0, of_branch = 0;
  for (int t = 0; t < strips; ++t) {
    of_w_pre += a.row_sums[(int64_t)t * a.K + k];
    of_branch += a.row_sums[(int64_t)(strips + t) * a.K + k];
  }
  if (a.dw_pre) a.dw_pre[k] = of_w_pre;
  if (a.dw_post) a.dw_post[k] = (a.gate ? a.gate[k] : 1.0f) * of_branch;
  if (a.dgate) a.dgate[k] = (a.w_post ? a.w_post[k] : 1.0f) * of_branch;
}

}  // namespace

size_t block_norm_workspace_bytes(int K, int N) { return (size_t)2 * chunk_count(K) * N * sizeof(float); }

template <int DT>
static hipError_t launch_forward(const Forward& a, hipStream_t stream) {
  const dim3 grid((uint32_t)(a.chunks * strip_count(a.N)));
  if (a.w_post) block_norm_pass_kernel<DT, 0><<<grid, kThreads, 0, stream>>>(a);
  if (a.w_pre) block_norm_pass_kernel<DT, 1><<<grid, kThreads, 0, stream>>>(a);
  block_norm_pass_kernel<DT, 2><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_block_norm(const BlockNormArgs& b, hipStream_t stream) {
  Forward a{b.K, b.N, chunk_rows(b.K), chunk_count(b.K), b.residual_scale, b.eps,
            static_cast<const uint16_t*>(b.x), static_cast<const uint16_t*>(b.y), b.w_post, b.gate, b.token_gate, b.w_pre,
            static_cast<uint16_t*>(b.h), b.ld_stream, static_cast<uint16_t*>(b.u), b.ld_block, b.rstd_y, b.rstd_h,
            b.workspace, b.workspace + (int64_t)chunk_count(b.K) * b.N, false, false};
  a.vec_stream = rows_in_pieces(a.x, a.ld_stream) && (!a.h || rows_in_pieces(a.h, a.ld_stream));
  a.vec_block = (!a.y || rows_in_pieces(a.y, a.ld_block)) && (!a.u || rows_in_pieces(a.u, a.ld_block));
  return b.dtype == HINM_F16 ? launch_forward<HINM_F16>(a, stream) : launch_forward<HINM_BF16>(a, stream);
}

size_t block_norm_grad_workspace_bytes(int K, int N) {
  return ((size_t)4 * chunk_count(K) * N + (size_t)2 * strip_count(N) * K) * sizeof(float);
}

template <int DT>
static hipError_t launch_backward(const Backward& a, hipStream_t stream) {
  const dim3 grid((uint32_t)(a.chunks * strip_count(a.N)));
  block_norm_grad_sums_kernel<DT><<<grid, kThreads, 0, stream>>>(a);
  block_norm_grad_rows_kernel<DT><<<grid, kThreads, 0, stream>>>(a);
  if (a.dw_pre || a.dw_post || a.dgate)
    block_norm_grad_weights_kernel<<<dim3((uint32_t)((a.K + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_block_norm_grad(const BlockNormGradArgs& b, hipStream_t stream) {
  Backward a{b.K, b.N, chunk_rows(b.K), chunk_count(b.K), b.residual_scale, static_cast<const uint16_t*>(b.h),
             static_cast<const uint16_t*>(b.y), b.w_post, b.gate, b.token_gate, b.w_pre, b.rstd_y, b.rstd_h,
             static_cast<const uint16_t*>(b.dh), static_cast<const uint16_t*>(b.du), static_cast<uint16_t*>(b.dx), b.ld_stream,
             static_cast<uint16_t*>(b.dy), b.ld_block, b.dw_post, b.dgate, b.dtoken_gate, b.dw_pre,
             b.workspace, b.workspace + (int64_t)4 * chunk_count(b.K) * b.N, false, false};
  auto in_pieces = [](const void* p, int64_t ld) { return !p || rows_in_pieces(p, ld); };
  a.vec_stream = in_pieces(a.h, a.ld_stream) && in_pieces(a.dh, a.ld_stream) && in_pieces(a.dx, a.ld_stream);
  a.vec_block = in_pieces(a.y, a.ld_block) && in_pieces(a.du, a.ld_block) && in_pieces(a.dy, a.ld_block);
  return b.dtype == HINM_F16 ? launch_backward<HINM_F16>(a, stream) : launch_backward<HINM_BF16>(a, stream);
}

}  // namespace hinm
