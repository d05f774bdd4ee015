// Activations of a layer's epilogue and their slopes, in float32 (include/hinm.h, HINM_EPI_*).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hinm.h"

namespace hinm {

enum Activation { kActNone, kActRelu, kActGelu, kActGeluTanh, kActSilu };
constexpr uint32_t kActFlags = HINM_EPI_RELU | HINM_EPI_GELU | HINM_EPI_GELU_TANH | HINM_EPI_SILU;
// ... that a call's flags name; -1 where they name several
inline int activation_of(uint32_t flags) {
  switch (flags & kActFlags) {
    case 0: return kActNone;
    case HINM_EPI_RELU: return kActRelu;
    case HINM_EPI_GELU: return kActGelu;
    case HINM_EPI_GELU_TANH: return kActGeluTanh;
    case HINM_EPI_SILU: return kActSilu;
  }
  return -1;
}

constexpr float kLog2e = 1.4426950408889634f;

// Phi(x), the normal distribution's probability of less than x, and exp(-x^2 / 2).  For x >= 0, 1 - Phi(x) = exp(-x^2 / 2) R(x)
// with R(x) = erfcx(x / sqrt 2) / 2, a smooth falling function, taken as a polynomial of degree eight in t = 1 / (1 + 0.3 x)
// without a constant term (R ~ 1 / x far out).  Coefficients: least squares of the relative error, reweighted until its peaks are
// level, 1.5e-7 over 0 .. 14.  In float32 Phi is 5e-7 off, and below zero, relative to itself, more the farther out: the rounding of
// x^2, times x^2 / 2 (8e-7 to -4, 2.1e-6 to -6, 5.2e-6 to -10, 7.7e-6 to -13), still far below half a step of 16 bits.
__device__ __forceinline__ float normal_probability(float x, float& bell) {
  const float a = fabsf(x), t = __builtin_amdgcn_rcpf(fmaf(0.3f, a, 1.0f));
  bell = __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2e));
  float r = 0.03567543998360634f;
  r = fmaf(r, t, -0.157205730676651f);
  r = fmaf(r, t, 0.20635786652565002f);
  r = fmaf(r, t, -0.05368749052286148f);
  r = fmaf(r, t, 0.12856358289718628f);
  r = fmaf(r, t, 0.09991291910409927f);
  r = fmaf(r, t, 0.12075404822826385f);
  r = fmaf(r, t, 0.11962929368019104f);
  const float beyond = r * t * bell;
  return x < 0 ? beyond : 1.0f - beyond;
}
__device__ __forceinline__ float sigmoid(float q) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(q * -kLog2e));
}
constexpr float kTanhScale = 1.5957691216057308f;  // 2 sqrt(2 / pi): (1 + tanh q) / 2 = sigmoid(2 q)
constexpr float kTanhCube = 0.044715f;

// What an epilogue's code holds of them, one of these: no function of the sum at all; nothing or relu; gelu; z sigmoid(scale z +
// cube z^3), which serves two.
enum Epilogue { kEpiBare, kEpiLinear, kEpiGelu, kEpiSigmoid };
inline Epilogue epilogue_of(int act) { return act == kActGelu ? kEpiGelu : act >= kActGeluTanh ? kEpiSigmoid : kEpiLinear; }

template <Epilogue E, int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
  if constexpr (E == kEpiLinear) {
    if (act != kActRelu) return;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = v[j] < 0 ? 0.0f : v[j];  // keeps NaN
  } else if constexpr (E == kEpiGelu) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float bell;
      v[j] *= normal_probability(v[j], bell);
    }
  } else if constexpr (E == kEpiSigmoid) {
    const float scale = act == kActSilu ? 1.0f : kTanhScale, cube = act == kActSilu ? 0.0f : kTanhScale * kTanhCube;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      // where the square leaves float32, beside a cube of zero too, the sigmoid is at its end: a scale of its own for infinity
      const float x = v[j], square = fminf(x * x, 3.0e38f);
      v[j] = x * sigmoid(x * fmaf(cube, square, scale));
    }
  }
}

// An infinite v has the limit, 0 or 1 (a sum beyond 16 bits is kept as one): far out the factor beside v is zero, and their product
// would be no number.
__device__ __forceinline__ float activation_slope(float v, int act) {
  switch (act) {
    case kActRelu: return v > 0 ? 1.0f : v <= 0 ? 0.0f : v;
    case kActGelu: {
      float bell;
      const float p = normal_probability(v, bell);
      return bell == 0 ? p : fmaf(v, bell * 0.3989422804014327f, p);
    }
    case kActGeluTanh: {
      const float s = sigmoid(kTanhScale * fmaf(kTanhCube * v * v, v, v)), both = s * (1.0f - s);
      return both > 0 ? fmaf(v * both, kTanhScale * fmaf(3.0f * kTanhCube, v * v, 1.0f), s) : s;
    }
    case kActSilu: {
      const float s = sigmoid(v), rest = 1.0f - s;
      return s * rest == 0 ? s : s * fmaf(v, rest, 1.0f);
    }
  }
  return 1.0f;
}

}  // namespace hinm
