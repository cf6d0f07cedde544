// Activations of the gated block and their derivatives, of the product z itself.
// Written without cancellation: gelu's and gelu_tanh's 1 + erf and 1 + tanh are
// erfc and a sigmoid, so that values far below 0 keep their digits.
#pragma once

#include "gated_internal.h"

namespace hfk {
namespace {

// EXACT: to fp32's last bits; else to about 2^-20, for values rounded to bf16
template <bool EXACT>
__device__ __forceinline__ float sigmoid_of(float z) {
  if constexpr (EXACT) return 1.0f / (1.0f + expf(-z));
  else return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
}
template <bool EXACT>
__device__ __forceinline__ float act_of(int act, float z) {
  switch (act) {
    case GA_SIGMOID: return sigmoid_of<EXACT>(z);
    case GA_TANH: return tanhf(z);
    case GA_RELU: return z <= 0.0f ? 0.0f : z;        // (NaN stays)
    case GA_SILU: return z * sigmoid_of<EXACT>(z);
    case GA_GELU: return 0.5f * z * erfcf(-0.70710678f * z);
    default: {
      const float z2 = fminf(z * z, 1e4f);       // (finite; the sigmoid is 0 or 1 by then)
      return z * sigmoid_of<EXACT>(1.59576912f * z * (1.0f + 0.044715f * z2));
    }
  }
}
template <bool EXACT>
__device__ __forceinline__ void act_and_slope(int act, float z, float& a, float& d) {
  switch (act) {
    case GA_SIGMOID:
      a = sigmoid_of<EXACT>(z);
      d = a * (1.0f - a);
      break;
    case GA_TANH:
      a = tanhf(z);
      d = 1.0f - a * a;
      break;
    case GA_RELU:
      a = z <= 0.0f ? 0.0f : z;
      d = z > 0.0f ? 1.0f : 0.0f;
      break;
    case GA_SILU: {
      const float p = sigmoid_of<EXACT>(z);
      a = z * p;
      d = p + a * (1.0f - p);
      break;
    }
    case GA_GELU: {
      const float p = 0.5f * erfcf(-0.70710678f * z);
      const float q = -0.5f * z * z;
      a = z * p;
      d = p + z * 0.39894228f * (EXACT ? expf(q) : __expf(q));     // 1 / sqrt(2 pi)
      break;
    }
    default: {
      const float z2 = fminf(z * z, 1e4f);       // 1.5957...: 2 sqrt(2 / pi)
      const float p = sigmoid_of<EXACT>(1.59576912f * z * (1.0f + 0.044715f * z2));
      a = z * p;
      d = p + a * (1.0f - p) * 1.59576912f * (1.0f + 0.134145f * z2);
    }
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
