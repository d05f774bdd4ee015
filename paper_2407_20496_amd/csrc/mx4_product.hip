// Products of two matrices in microscaled 4-bit form, Y = A B^T, on the scaled matrix instructions (include/hinm.h).
#include "mx4_form.h"

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

template <int OUT>
hipError_t launch_out(const Mx4ProductArgs& a, hipStream_t stream) {
  const ProductShape p{a.M, a.N, a.K, a.ldy, a.relu};
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
