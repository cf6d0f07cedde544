// Activations of the gated block and their derivatives, of the product z itself.
// Written without cancellation: gelu's and gelu_tanh's 1 + erf and 1 + tanh are
// erfc and a sigmoid, so that values below 0 are off by about as many units of the
// last place as their exponent is large (silu's, of z itself, by a few).  This ends
// where the factor of z leaves fp32's normal numbers: values are within 2^-119 of 0
// there (silu from -87 on, gelu from -12.9, gelu_tanh from -10), and soon are 0.
#pragma once

#include <type_traits>

#include "gated_internal.h"

namespace hfk {
namespace {

// EXACT: to fp32's last bits; else to about 2^-20, for values rounded to bf16
template <bool EXACT>
__device__ __forceinline__ float sigmoid_of(float z) {
  if constexpr (EXACT) return 1.0f / (1.0f + expf(-z));
  else return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
}
// phi(z), ACT one of GA_*
template <int ACT, bool EXACT>
__device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == GA_SIGMOID) return sigmoid_of<EXACT>(z);
  if constexpr (ACT == GA_TANH) return tanhf(z);
  if constexpr (ACT == GA_RELU) return z <= 0.0f ? 0.0f : z;        // (NaN stays)
  if constexpr (ACT == GA_SILU) return z * sigmoid_of<EXACT>(z);
  if constexpr (ACT == GA_GELU) return 0.5f * z * erfcf(-0.70710678f * z);
  // 1.5957...: 2 sqrt(2 / pi); z^2 stays finite (the sigmoid is 0 or 1 by 1e4)
  return z * sigmoid_of<EXACT>(1.59576912f * z * (1.0f + 0.044715f * fminf(z * z, 1e4f)));
}
// and its slope
template <int ACT, bool EXACT>
__device__ __forceinline__ void act_and_slope(float z, float& a, float& d) {
  if constexpr (ACT == GA_SIGMOID) {
    a = sigmoid_of<EXACT>(z);
    d = a * (1.0f - a);
  } else if constexpr (ACT == GA_TANH) {
    a = tanhf(z);
    d = 1.0f - a * a;
  } else if constexpr (ACT == GA_RELU) {
    a = z <= 0.0f ? 0.0f : z;
    d = z > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == GA_SILU) {
    const float p = sigmoid_of<EXACT>(z);
    a = z * p;
    d = p + a * (1.0f - p);
  } else if constexpr (ACT == GA_GELU) {
    const float p = 0.5f * erfcf(-0.70710678f * z);
    const float q = -0.5f * z * z;
    a = z * p;
    d = p + z * 0.39894228f * (EXACT ? expf(q) : __expf(q));     // 1 / sqrt(2 pi)
  } else {
    const float z2 = fminf(z * z, 1e4f);
    const float p = sigmoid_of<EXACT>(1.59576912f * z * (1.0f + 0.044715f * z2));
    a = z * p;
    d = p + a * (1.0f - p) * 1.59576912f * (1.0f + 0.134145f * z2);
  }
}
// f with the activation as a constant: what f does for many values is compiled
// for each activation, with no branch between the values
template <class Fn>
__device__ __forceinline__ void with_act(int act, Fn f) {
  switch (act) {
    case GA_SIGMOID: f(std::integral_constant<int, GA_SIGMOID>()); break;
    case GA_TANH: f(std::integral_constant<int, GA_TANH>()); break;
    case GA_RELU: f(std::integral_constant<int, GA_RELU>()); break;
    case GA_SILU: f(std::integral_constant<int, GA_SILU>()); break;
    case GA_GELU: f(std::integral_constant<int, GA_GELU>()); break;
    default: f(std::integral_constant<int, GA_GELU_TANH>());
  }
}

// The scale byte of a block whose largest magnitude is `big`: 127 + e - 6, with
// 2^e the power of two at or below it, one more where its code would round to
// 128; 255 where a number is not finite.  The numbers are codes times
// 2^(byte - 127), the codes within 127.
__device__ __forceinline__ int block_byte(float big) {
  const uint32_t b = __float_as_uint(big);
  if (b >= 0x7f800000u) return 255;
  const int e = (int)((b + 0x10000u) >> 23) - 6;
  return e > 0 ? e : 0;
}
// 2^(127 - byte), and 2^(byte - 127)
__device__ __forceinline__ float code_factor(int byte) {
  // byte 0 .. 249: exponents 127 .. -122
  return __uint_as_float((uint32_t)(254 - byte) << 23);
}
__device__ __forceinline__ float code_step(int byte) {
  return byte == 255 ? __uint_as_float(0x7fc00000u)
                     : byte ? __uint_as_float((uint32_t)byte << 23) : __uint_as_float(0x400000u);
}

}  // namespace
}  // namespace hfk
