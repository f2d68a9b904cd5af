// Shared device building blocks of the operators that read or write rows in 8 bits,
// and the activations and their derivatives.
//
// A row in 8 bits is C e4m3 values q and an fp32 scale; it stands for q * scale.  With
// top the row's largest magnitude, at least 2^-100, scale = top / 448 (448 is the largest
// e4m3 number) and q = v * (448 / top) rounded to nearest even: off by at most 2^-4 of a
// value, or half of the smallest step (2^-10 scale) near zero.  One scale a row, so that a
// product can take it out of the sum over the row.
#pragma once

#include <type_traits>

#include "rows.h"

namespace spc {
namespace {

constexpr float kE4m3Max = 448.0f;

// The order of magnitudes as unsigned numbers: NaN above infinity above the rest.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ float larger_magnitude(float a, float b) {
  return __float_as_uint(a) > __float_as_uint(b) ? a : b;      // (of values without signs)
}
// The scale of a row whose largest magnitude is `top`, and what its values are
// multiplied by: NaN and 0 for a row with an infinity or NaN.
__device__ __forceinline__ void scale_of(float top, float* scale, float* inverse) {
  const bool fine = __float_as_uint(top) < 0x7f800000u;
  const float t = fine ? fmaxf(top, 0x1p-100f) : 1.0f;
  *scale = fine ? t / kE4m3Max : __uint_as_float(0x7fc00000u);
  *inverse = fine ? kE4m3Max / t : 0.0f;
}
// Four values to e4m3.  (Those of a row that is not finite: `inverse` is 0, and so are
// they, NaN too.)
__device__ __forceinline__ uint32_t pack_e4m3(const float* v, float inverse) {
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = inverse == 0.0f ? 0.0f : v[i] * inverse;
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false);
  u = __builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], u, true);
  return static_cast<uint32_t>(u);
}
__device__ __forceinline__ void unpack_e4m3(uint32_t u, float* v) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), false);
  const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), true);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
}

// Elements [c, c + N) of a row of C e4m3 values at p, those past the end 0 (N 4 or 8, a
// piece of the other rows of a call); TAIL as for load_row.
template <int N, bool TAIL>
__device__ __forceinline__ void load_row8(const uint8_t* p, int64_t c, int64_t C, float (&v)[N]) {
  uint32_t u[N / 4] = {};
  if (!TAIL || c + N <= C) {
    __builtin_memcpy(u, p + c, N);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < C) u[i / 4] |= static_cast<uint32_t>(p[c + i]) << (8 * (i % 4));
  }
#pragma unroll
  for (int q = 0; q < N / 4; ++q) unpack_e4m3(u[q], v + 4 * q);
}
template <int N, bool TAIL>
__device__ __forceinline__ void store_row8(uint8_t* p, int64_t c, int64_t C, const float (&v)[N],
                                           float inverse) {
  uint32_t u[N / 4];
#pragma unroll
  for (int q = 0; q < N / 4; ++q) u[q] = pack_e4m3(v + 4 * q, inverse);
  if (!TAIL || c + N <= C) {
    __builtin_memcpy(p + c, u, N);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < C) p[c + i] = static_cast<uint8_t>(u[i / 4] >> (8 * (i % 4)));
  }
}

// Activations and their derivatives, in few operations: they are a third of the time of a
// finished tile (348,208 x 1024 through the GELU's derivative, 26 operations an element: 144
// of 593 us).  1 / (1 + 2^t) by the hardware's exp2 and reciprocal, off by a unit of fp32 each and
// by the rounding of t: 0 and 1 where 2^t leaves fp32's range.
__device__ __forceinline__ float logistic2(float t) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}
constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596303e-8f;
// The logistic function of z.  Rounding z log2(e) is off by up to |z| units of exp's value, which
// counts where that is the result, far below 0; FINE (fp32 results: bf16 ones have no place for it)
// puts it back.  (Both ends are reached long before +-120, and nothing is infinite within.)
template <bool FINE> __device__ __forceinline__ float logistic(float z) {
  if constexpr (FINE) {
    const float c = __builtin_amdgcn_fmed3f(z, -120.0f, 120.0f), t = c * -kLog2e;
    const float lost = fmaf(c, -kLog2eLow, fmaf(c, -kLog2e, -t));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t) * fmaf(lost, 0.693147181f, 1.0f));
  } else {
    return logistic2(z * -kLog2e);
  }
}
// GELU in its tanh form: z (1 + tanh u) / 2 = z / (1 + exp(-2 u)), u = sqrt(2 / pi) (z + 0.044715
// z^3): -2 u log2(e) = z (G + G3 z^2).
constexpr float kG = -2.30220819f, kG3 = -0.102943240f;
template <int ACT, bool FINE> __device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == SPCONV_ACT_RELU) return z < 0.0f ? 0.0f : z;
  if constexpr (ACT == SPCONV_ACT_GELU) return z * logistic2(z * fmaf(kG3, z * z, kG));
  if constexpr (ACT == SPCONV_ACT_SILU) return z * logistic<FINE>(z);
  return z;
}
// With s the logistic function's value: s + s (1 - s) z (2 u)', and 1 - s as s - s s (off by
// half a unit of 1).
template <int ACT, bool FINE> __device__ __forceinline__ float slope(float z) {
  if constexpr (ACT == SPCONV_ACT_RELU) return z <= 0.0f ? 0.0f : 1.0f;
  if constexpr (ACT == SPCONV_ACT_GELU) {
    const float z2 = z * z, s = logistic2(z * fmaf(kG3, z2, kG));
    // (2 sqrt(2 / pi) (1 + 3 * 0.044715 z^2), kept finite: s (1 - s) is 0 there)
    const float w = __builtin_amdgcn_fmed3f(z * fmaf(0.214064449f, z2, 1.59576912f), -0x1p100f, 0x1p100f);
    return fmaf(fmaf(-s, s, s), w, s);
  }
  if constexpr (ACT == SPCONV_ACT_SILU) {
    const float s = logistic<FINE>(z);
    return fmaf(fmaf(-s, s, s), z, s);
  }
  return 1.0f;
}

// f(integral constant of the activation).
template <typename F> __device__ __host__ __forceinline__ auto by_act(int act, F f) {
  switch (act) {
    case SPCONV_ACT_RELU: return f(std::integral_constant<int, SPCONV_ACT_RELU>());
    case SPCONV_ACT_GELU: return f(std::integral_constant<int, SPCONV_ACT_GELU>());
    case SPCONV_ACT_SILU: return f(std::integral_constant<int, SPCONV_ACT_SILU>());
    default: return f(std::integral_constant<int, SPCONV_ACT_NONE>());
  }
}
inline bool act_ok(int act) { return act >= SPCONV_ACT_NONE && act <= SPCONV_ACT_SILU; }

}  // namespace
}  // namespace spc
