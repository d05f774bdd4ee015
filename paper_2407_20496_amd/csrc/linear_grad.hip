// The gradient that reaches a layer's product: dZ = dY act'(Z), rounded, and its sums over the tokens (include/hinm.h).
#include "linear_tile.h"

#include <algorithm>

#include "column_strips.h"

namespace hinm {

namespace {

// A row is shared by LANES threads, eight columns each at a time; 256 / LANES rows a workgroup.  Bound by memory: Z and dY read
// once, dZ written once in rows of whole pieces, zeros behind the last column.  dZ is rounded to 16 bits because the matrix
// instructions take it so; the sums are of the values before that.  4096x2048 with gelu 12.8 us, 3.9 TB/s.  8, 64 or 256 lanes a row, so
// that a row of N columns has few lanes without a piece and a long one does not wait for one wave.
template <int DT, int LANES>
__global__ __launch_bounds__(256) void linear_slope_kernel(SlopeArgs a) {
  __shared__ float by_wave[4];
  const int t = threadIdx.x % LANES;
  constexpr int kAtOnce = 2, kRows = 256 / LANES;
  const u32x4 none = {0, 0, 0, 0};
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.M; first += (int64_t)gridDim.x * kRows) {
    const int64_t m = first + threadIdx.x / LANES;
    const bool in = m < a.M;
    float sum = 0;
    for (int n0 = 8 * t; in && n0 < a.N; n0 += 8 * LANES * kAtOnce) {
      u32x4 dy[kAtOnce], z[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int n = n0 + 8 * LANES * i, left = a.N - n;
        const int64_t at = m * a.ldy + n;
        dy[i] = left > 0 ? draw_eight(a.dY + at, left, a.rows) : none;
        z[i] = left > 0 && a.Z ? draw_eight(a.Z + at, left, a.rows) : none;
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int n = n0 + 8 * LANES * i, left = a.N - n;
        if (left <= 0) break;
        float g[8], v[8];
        widen<DT>(trim_eight(dy[i], left, a.rows), g);
        widen<DT>(trim_eight(z[i], left, a.rows), v);
        if (a.Z) {
          switch (a.act) {
#define HINM_SLOPE(act)                                                                \
  case act:                                                                            \
    _Pragma("unroll") for (int j = 0; j < 8; ++j) g[j] *= activation_slope(v[j], act); \
    break;
            HINM_SLOPE(kActRelu)
            HINM_SLOPE(kActGelu)
            HINM_SLOPE(kActGeluTanh)
            HINM_SLOPE(kActSilu)
#undef HINM_SLOPE
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += g[j];
        if (a.dZ) *reinterpret_cast<u32x4*>(a.dZ + m * a.ldz + n) = narrow<DT>(g);
      }
    }
    if (!a.dbias) continue;
    if constexpr (LANES == 8) {
      sum = add_eight_lanes(sum);
    } else {
      sum = add_lanes_by_8(add_eight_lanes(sum));
      if constexpr (LANES == 256) {
        __syncthreads();  // the last row's sums have been read
        if ((threadIdx.x & 63) == 0) by_wave[threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = by_wave[0] + by_wave[1] + by_wave[2] + by_wave[3];
      }
    }
    if (in && t == 0) a.dbias[m] = sum;
  }
}

template <int DT>
hipError_t launch_lanes(const SlopeArgs& a, hipStream_t stream) {
  auto groups = [&](int rows) { return dim3((uint32_t)std::min<int64_t>(((int64_t)a.M + rows - 1) / rows, 1 << 20)); };
  if (a.N <= 64) linear_slope_kernel<DT, 8><<<groups(32), 256, 0, stream>>>(a);
  else if (a.N <= 1024) linear_slope_kernel<DT, 64><<<groups(4), 256, 0, stream>>>(a);
  else linear_slope_kernel<DT, 256><<<groups(1), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_slope(const SlopeArgs& a, int dtype, hipStream_t stream) {
  return dtype == HINM_F16 ? launch_lanes<HINM_F16>(a, stream) : launch_lanes<HINM_BF16>(a, stream);
}

}  // namespace hinm
