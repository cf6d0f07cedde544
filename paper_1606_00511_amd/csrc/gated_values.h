// Eight neighbours of a row, the work of a lane in the gated block's kernels: their
// loads and stores in every type and as the codes of a checkpoint.
#pragma once

#include "gated_act.h"
#include "mfma_tile.h"

namespace hfk {
namespace {

// two values rounded to bf16, in one instruction (one by one they take four: unpacking
// 16,384 x 8,192 98 -> 81 us)
__device__ __forceinline__ uint32_t f2bf2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}
__device__ __forceinline__ u32x4 f2bf8(const float (&v)[8]) {
  return u32x4{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
}
// sum sa sb of a sum of codes, as ((sum a) sb) c with sa = a c.  The scales' product on its
// own may leave fp32's normal numbers where the result does not; the sum, 0 or at least 1,
// times a scale gets no smaller than the scale (and is exact below the normal numbers), and
// too large only of a scale above 2^97, which waits for the other one.  (8,192 rows, 16,384
// x 4,096: 504 -> 507 us by the third product; with a choice by a row's or a tile's scales
// in its place 508 to 509.)
struct RowFactor {
  float a, c;
  __device__ __forceinline__ explicit RowFactor(float sa) {
    const bool large = fabsf(sa) > 0x1p64f;
    a = large ? 1.0f : sa;
    c = large ? sa : 1.0f;
  }
  __device__ __forceinline__ float scaled(int sum, float sb) const {
    return (float)sum * a * sb * c;
  }
};
// What v's rounding to the bf16 number b left; 0 where that is not finite (beside an
// infinity its rest would be one of the other sign, or NaN).
__device__ __forceinline__ float rest_of(float v, uint32_t b) {
  return (b & 0x7f80u) == 0x7f80u ? 0.0f : v - bf2f(b);
}
// 8 values to p, of any alignment, the first `have` of them, and from it
// (STREAM: past the caches)
template <bool STREAM = false>
__device__ __forceinline__ void put(float* p, const float (&v)[8], int have) {
  if (have >= 8) {
    put16<STREAM>(p, __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}));
    put16<STREAM>(p + 4, __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < have) p[j] = v[j];
  }
}
template <bool STREAM = false>
__device__ __forceinline__ void put(bf16_t* p, const float (&v)[8], int have) {
  if (have >= 8) {
    put16<STREAM>(p, f2bf8(v));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < have) store1(p + j, v[j]);
  }
}
__device__ __forceinline__ void get(const float* p, float (&v)[8], int have) {
  if (have >= 8) {
    f32x4 a, b;
    __builtin_memcpy(&a, p, 16);
    __builtin_memcpy(&b, p + 4, 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < have ? p[j] : 0.0f;
  }
}
__device__ __forceinline__ void get(const bf16_t* p, float (&v)[8], int have) {
  if (have >= 8) {
    u32x4 w;
    __builtin_memcpy(&w, p, 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = bf2f(w[j] & 0xffffu);
      v[2 * j + 1] = bf2f(w[j] >> 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < have ? bf2f(p[j]) : 0.0f;
  }
}
// 8 codes times step
__device__ __forceinline__ void get_codes(const int8_t* p, float step, float (&v)[8], int have) {
  if (have >= 8) {
    uint32_t w[2];
    __builtin_memcpy(w, p, 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(w[j >> 2] >> (8 * (j & 3))) * step;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < have ? (float)p[j] * step : 0.0f;
  }
}
// 8 values of a block of 32, which 4 neighbouring lanes share, to codes: their
// scale byte; values past `have` count 0
template <bool STREAM = false>
__device__ __forceinline__ int put_codes(int8_t* p, const float (&v)[8], int have) {
  // (of magnitudes as whole numbers the largest: NaN is above all, where fmaxf
  // would lose it)
  uint32_t big = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < have) big = max(big, __float_as_uint(v[j]) & 0x7fffffffu);
  big = max(big, (uint32_t)__shfl_xor((int)big, 1, 64));
  big = max(big, (uint32_t)__shfl_xor((int)big, 2, 64));
  const int byte = block_byte(__uint_as_float(big));
  const float f = byte == 255 ? 0.0f : code_factor(byte);
  // (bytes of the code + 128, and then their highest bits turned)
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float q = byte == 255 ? 0.0f : rintf(v[j] * f);
    w[j >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(q + 128.0f, j & 3, w[j >> 2]);
  }
  w[0] ^= 0x80808080u;
  w[1] ^= 0x80808080u;
  if (have >= 8) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef u32x2 __attribute__((aligned(1))) loose;
    if (STREAM) __builtin_nontemporal_store(u32x2{w[0], w[1]}, (loose*)p);
    else *(loose*)p = u32x2{w[0], w[1]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < have) p[j] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
  return byte;
}

}  // namespace
}  // namespace hfk
