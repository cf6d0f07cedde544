// Row kernels of the gated block: copies of operands with zeros around, sums of
// split products, checkpoints in 8 bits and codes with a scale for each row.  All
// are bound by memory.
#include <algorithm>

#include "gated_act.h"
#include "gated_values.h"
#include "mfma_tile.h"

namespace hfk {
namespace {

// ------------------------------------------------------------------- padding
// 16 bytes of a destination row from chunk c: elements of the source row, zeros
// past `cols`
template <class E>
__device__ __forceinline__ u32x4 padded(const E* src, int c, int cols) {
  constexpr int N = 16 / (int)sizeof(E);
  const int at = c * N;
  u32x4 w = u32x4{0u, 0u, 0u, 0u};
  if (at + N <= cols) {
    __builtin_memcpy(&w, src + at, 16);
  } else if (at < cols) {
    E v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = at + j < cols ? src[at + j] : E(0);
    __builtin_memcpy(&w, v, 16);
  }
  return w;
}

// the same of a checkpoint
__device__ __forceinline__ u32x4 unpacked(const GPad& p, int row, int c) {
  const int n = 16 / p.es, at = c * n, have = p.cols - at;
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = 0.0f;
  if (have > 0)
    get_codes((const int8_t*)p.src + (size_t)row * p.ld + at,
              code_step(p.scale[(size_t)row * p.lds + at / CODE_BLOCK]), v, min(have, n));
  if (p.es == 4) return __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
  return f2bf8(v);
}

// ------------------------------------------------- sums of split products
struct FinishOne {
  GFinish f;
  int rows, chunks, first;     // rows of out (both), 8 columns each; first workgroup
  long long stride;            // of partials
  int rm, rn, gx, gy, blocks;  // with shares: the tiles, and K blocks of each
};
struct FinishAll {
  FinishOne one[3];
  int n;
};
// f's outputs by `groups` workgroups, of which this is the b-th
template <class E, class O>
__device__ __forceinline__ void finish_body(const FinishOne& one, uint32_t b, uint32_t groups) {
  const GGemm& g = one.f.g;
  const GEpi& e = one.f.e;
  const int dup = one.f.dup, end = min(e.mout, g.M);
  const uint32_t chunks = one.chunks;
  const long long stride = one.stride;
  // (at most 2^31 chunks, of 262,144 rows of 65,536, and 2^28 a step: below 2^32)
  const uint32_t total = (uint32_t)one.rows * chunks;
  for (uint32_t i = b * 256u + threadIdx.x; i < total; i += groups * 256u) {
    const int row = (int)(i / chunks), m = g.m0 + 8 * (int)(i % chunks);
    const bool second = row >= e.nout;
    const int n = second ? e.n1 + row - e.nout : row, have = end - m;
    const float* p = e.part + (size_t)n * e.ldp + (m - g.m0);
    int parts = g.splits;
    if (one.f.share) {
      // the tile's units; of the first one the place where its share ends, of the others
      // where they begin
      const int rm = one.rm, rn = one.rn, tm = m / rm, tn = n / rn;
      const int at = one.f.work + tile_place(tm, tn, one.gx, one.gy) * one.blocks;
      const int u0 = at / one.f.share, u1 = (at + one.blocks - 1) / one.f.share;
      parts = u1 - u0 + 1;
      if (parts == 1) continue;            // (written by its unit)
      p = e.part + (size_t)(2 * u0 + 1) * rm * rn + (n - tn * rn) * rm + m - tm * rm;
    }
    // partial s of the sum
    auto from = [&](const float* q, int s) {
      return one.f.share && s ? q + (2 * s - 1) * stride : q + s * stride;
    };
    float v[8];
    if constexpr (sizeof(E) == 1) {
      int t[8] = {};
#pragma unroll 4
      for (int s = 0; s < parts; ++s) {
        const float* w = from(p, s);
        const i32x4 a = *(const i32x4*)w, b = *(const i32x4*)(w + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          t[j] += a[j];
          t[4 + j] += b[j];
        }
      }
      const RowFactor sn(e.sn[n]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = sn.scaled(t[j], e.sm[min(m + j, e.mout - 1)]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
      for (int h = 0; h < (dup ? 2 : 1); ++h) {
        const float* q = p + (size_t)h * dup * e.ldp;
#pragma unroll 4
        for (int s = 0; s < parts; ++s) {
          const float* w = from(q, s);
          const f32x4 a = *(const f32x4*)w, b = *(const f32x4*)(w + 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j] += a[j];
            v[4 + j] += b[j];
          }
        }
      }
    }
    O* out = (O*)(second ? e.out1 : e.out) +
             (size_t)(second ? row - e.nout : row) * (second ? e.ldo1 : e.ldo) + m;
    if (e.accumulate) {
      float o[8];
      get(out, o, have);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += o[j];
    }
    put(out, v, have);
  }
}

// ------------------------------------------------------------- checkpoints
template <class E, bool STREAM>
__device__ __forceinline__ void pack_body(const E* X, long long ldx, uint32_t total, int cols,
                                          uint32_t per, int8_t* codes, long long ldc,
                                          uint8_t* scale, long long lds) {
  // (whole blocks of 32: the 4 lanes of one are all here or none is)
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= total) return;
  const uint32_t row = i / per, c = i % per;
  const int at = 8 * (int)c, have = cols - at;
  float v[8];
  get(X + (size_t)row * ldx + at, v, have);
  const int byte = put_codes<STREAM>(codes + (size_t)row * ldc + at, v, have);
  if ((c & 3) == 0) scale[(size_t)row * lds + c / 4] = (uint8_t)byte;
}

template <class E, bool STREAM>
__device__ __forceinline__ void unpack_body(const int8_t* codes, long long ldc,
                                            const uint8_t* scale, long long lds,
                                            int cols, E* X, long long ldx, uint32_t per,
                                            uint32_t total) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= total) return;
  const uint32_t row = i / per, c = i % per;
  const int at = 8 * (int)c, have = cols - at;
  float v[8];
  get_codes(codes + (size_t)row * ldc + at, code_step(scale[(size_t)row * lds + c / 4]), v, have);
  put<STREAM>(X + (size_t)row * ldx + at, v, have);
}

// --------------------------------------------------------- codes of rows
// q = round(x / s) to even where x inv is next to a border between two codes: what is
// left of x beside q s decides, which an fma gives exactly
__device__ __forceinline__ float border_code(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), half = 0.5f * s;
  const bool odd = (int)q & 1;
  if (r > half || (r == half && odd)) q += 1.0f;
  else if (-r > half || (-r == half && odd)) q -= 1.0f;
  return q;
}
struct RowScale {
  float s;       // what is stored
  float f, ss, inv;   // x f / ss, with f a power of two that keeps 1 / ss finite
};
__device__ __forceinline__ RowScale row_scale(uint32_t big) {
  RowScale r;
  const float amax = __uint_as_float(big);
  r.s = big >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : amax / 127.0f;
  const bool none = big >= 0x7f800000u || r.s == 0.0f;
  r.f = none ? 0.0f : r.s < 1e-30f ? 0x1p64f : 1.0f;
  r.ss = none ? 1.0f : r.s * r.f;
  r.inv = 1.0f / r.ss;
  return r;
}
// (EVEN: all 8 are there; have, room: how many are, and how many are written)
template <bool EVEN>
__device__ __forceinline__ void put_row_codes(int8_t* p, const float (&v)[8], const RowScale& r,
                                              int have, int room) {
  if (r.f == 0.0f) have = 0;                   // (a row without codes)
  else if (EVEN) have = 8;
  // x inv is off by less than 2^-15 of a step: only next to a border, 2^-13 of all
  // places, does it not tell the code (a branch for each number: 49 us for 8,192 rows
  // of 4,096, for 8 at once 30)
  float q[8], near = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float t = (j < have ? v[j] * r.f : 0.0f) * r.inv;
    q[j] = rintf(t);
    near = fmaxf(near, fabsf(t - q[j]));
  }
  if (near > 0.5f - 0x1p-14f) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < have) q[j] = border_code(v[j] * r.f, r.ss, r.inv);
  }
  // (bytes of q + 128, and then their highest bits turned)
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    w[j >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(
        __builtin_amdgcn_fmed3f(q[j], -127.0f, 127.0f) + 128.0f, j & 3, w[j >> 2]);
  w[0] ^= 0x80808080u;
  w[1] ^= 0x80808080u;
  if (EVEN || room >= 8) {
    __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < room) p[j] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// the largest of W waves'
template <int W>
__device__ __forceinline__ uint32_t group_max(uint32_t big) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) big = max(big, (uint32_t)__shfl_xor((int)big, d, 64));
  if constexpr (W > 1) {
    __shared__ uint32_t part[W];
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = big;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) big = max(big, part[w]);
  }
  return big;
}
// A row by W waves, of a workgroup of 4.  C > 0: cols is a multiple of 8, and a lane's C
// chunks stay in registers between the two passes (zcols <= 512 W C); else the row is
// read twice.  (Chunks that may be cut are four times the code, which a row or two
// wait for: 32 rows of 4,096 took 10.7 us with them and 4.6 without.)
template <class E, int W, int C>
__device__ __forceinline__ void codes_body(const E* X, long long ldx, int rows, int cols,
                                           int8_t* codes, long long ldc, int zcols, float* scale) {
  const int row = W == 4 ? blockIdx.x : 4 * blockIdx.x + threadIdx.x / 64;
  if (row >= rows) return;                    // (W == 1: a whole wave)
  const int t = W == 4 ? threadIdx.x : threadIdx.x % 64;
  const E* x = X + (size_t)row * ldx;
  int8_t* out = codes + (size_t)row * ldc;
  uint32_t big = 0;
  float keep[C > 0 ? C : 1][8];
  if constexpr (C > 0) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int at = 8 * (t + 64 * W * i);
#pragma unroll
      for (int j = 0; j < 8; ++j) keep[i][j] = 0.0f;
      if (at < cols) get(x + at, keep[i], 8);
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) big = max(big, magnitude(keep[i][j]));
  } else {
    for (int at = 8 * t; at < cols; at += 512 * W) {
      float v[8];
      get(x + at, v, cols - at);
#pragma unroll
      for (int j = 0; j < 8; ++j) big = max(big, magnitude(v[j]));
    }
  }
  const RowScale r = row_scale(group_max<W>(big));
  if (t == 0) scale[row] = r.s;
  if constexpr (C > 0) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int at = 8 * (t + 64 * W * i);
      if (at < zcols) put_row_codes<true>(out + at, keep[i], r, 8, 8);
    }
  } else {
    for (int at = 8 * t; at < zcols; at += 512 * W) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
      if (at < cols) get(x + at, v, cols - at);
      put_row_codes<false>(out + at, v, r, cols - at, zcols - at);
    }
  }
}

}  // namespace

extern "C" __global__ __launch_bounds__(256) void hf_gated_pad(GPads all, int chunks0, int chunks1,
                                                               int chunks2, int chunks3,
                                                               int chunks4) {
  // the copy that this workgroup belongs to
  int b = blockIdx.x, k = 0;
  const int n[GPADS - 1] = {chunks0, chunks1, chunks2, chunks3, chunks4};
#pragma unroll
  for (int j = 0; j < GPADS - 1; ++j)
    if (k == j && b >= n[j]) {
      b -= n[j];
      k = j + 1;
    }
  const GPad p = all.p[k];
  const uint32_t per = (uint32_t)(p.pcols * p.es / 16);
  const uint32_t rows = (uint32_t)p.prows * p.times;
  // 4 rows of chunks a workgroup and step: 1,024 chunks
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t i = (uint32_t)b * 1024u + 256u * u + threadIdx.x;
    const uint32_t to = i / per, c = i % per;
    if (to >= rows) return;
    const uint32_t row = to % (uint32_t)p.prows;
    u32x4 w = u32x4{0u, 0u, 0u, 0u};
    if ((int)row < p.rows) {
      const char* src = (const char*)p.src + (size_t)row * p.ld * p.es;
      if (p.scale) w = unpacked(p, (int)row, (int)c);
      else w = p.es == 4 ? padded((const float*)src, (int)c, p.cols)
                    : p.es == 2 ? padded((const uint16_t*)src, (int)c, p.cols)
                                : padded((const int8_t*)src, (int)c, p.cols);
    }
    *(u32x4*)((char*)p.dst + (size_t)i * 16) = w;
  }
}

#define HF_FINISH(SUF, E, O)                                                                     \
  extern "C" __global__ __launch_bounds__(256) void hf_gated_finish_##SUF(FinishAll a) {         \
    const int b = blockIdx.x;                                                                    \
    if (a.n > 2 && b >= a.one[2].first)                                                          \
      finish_body<E, O>(a.one[2], b - a.one[2].first, gridDim.x - a.one[2].first);               \
    else if (a.n > 1 && b >= a.one[1].first)                                                     \
      finish_body<E, O>(a.one[1], b - a.one[1].first,                                            \
                        (a.n > 2 ? a.one[2].first : gridDim.x) - a.one[1].first);                \
    else                                                                                         \
      finish_body<E, O>(a.one[0], b, a.n > 1 ? a.one[1].first : gridDim.x);                      \
  }
HF_FINISH(f32, float, float)
HF_FINISH(bf16, bf16_t, bf16_t)
HF_FINISH(codes_f32, int8_t, float)
HF_FINISH(codes_bf16, int8_t, bf16_t)

#define HF_ROW_CODES(NAME, E, W, C)                                                             \
  extern "C" __global__ __launch_bounds__(256) void NAME(                                       \
      const E* X, long long ldx, int rows, int cols, int8_t* codes, long long ldc, int zcols,    \
      float* scale) {                                                                            \
    codes_body<E, W, C>(X, ldx, rows, cols, codes, ldc, zcols, scale);                           \
  }
#define HF_PACK(SUF, E, STREAM)                                                                  \
  extern "C" __global__ __launch_bounds__(256) void hf_gated_pack_##SUF(                         \
      const E* X, long long ldx, uint32_t total, int cols, uint32_t per, int8_t* codes,          \
      long long ldc, uint8_t* scale, long long lds) {                                            \
    pack_body<E, STREAM>(X, ldx, total, cols, per, codes, ldc, scale, lds);                      \
  }                                                                                              \
  extern "C" __global__ __launch_bounds__(256) void hf_gated_unpack_##SUF(                       \
      const int8_t* codes, long long ldc, const uint8_t* scale, long long lds, int cols, E* X,   \
      long long ldx, uint32_t per, uint32_t total) {                                             \
    unpack_body<E, STREAM>(codes, ldc, scale, lds, cols, X, ldx, per, total);                    \
  }
HF_PACK(f32, float, false)
HF_PACK(bf16, bf16_t, false)
HF_PACK(f32_s, float, true)
HF_PACK(bf16_s, bf16_t, true)
#define HF_CODES(SUF, E)                                                                         \
  HF_ROW_CODES(hf_gated_codes_##SUF, E, 4, 0)                                                    \
  HF_ROW_CODES(hf_gated_codes_##SUF##_c1, E, 1, 2)                                               \
  HF_ROW_CODES(hf_gated_codes_##SUF##_c4, E, 4, 2)                                               \
  HF_ROW_CODES(hf_gated_codes_##SUF##_c16, E, 4, 8)
HF_CODES(f32, float)
HF_CODES(bf16, bf16_t)

// 2,048 columns of a row a workgroup, which finds the row's largest among the
// products' parts of it first
extern "C" __global__ __launch_bounds__(256) void hf_gated_codes_h(const float* H, long long ldh,
                                                                   const float* hmax,
                                                                   long long ldmax, int nmax,
                                                                   int cols, int8_t* codes,
                                                                   long long ldc, int zcols,
                                                                   int chunks, float* scale) {
  const size_t row = blockIdx.x / (uint32_t)chunks;
  const int at = 2048 * (int)(blockIdx.x % (uint32_t)chunks) + 8 * (int)threadIdx.x;
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = 0.0f;
  if (at < cols) get(H + row * ldh + at, v, cols - at);
  uint32_t big = 0;
#pragma unroll 8
  for (int i = threadIdx.x; i < nmax; i += 256) big = max(big, magnitude(hmax[row * ldmax + i]));
  const RowScale r = row_scale(group_max<4>(big));
  if (at == 0) scale[row] = r.s;
  if (at < zcols) put_row_codes<false>(codes + row * ldc + at, v, r, cols - at, zcols - at);
}

// ------------------------------------------------------------- launchers
#define HF_LAUNCH(NAME, K, GRID, BLOCK, ...)                                       \
  do {                                                                             \
    prof_begin(L, NAME);                                                           \
    hipExtLaunchKernelGGL(K, dim3((unsigned)(GRID)), dim3(BLOCK), 0, L.stream,     \
                          prof_a(L), prof_b(L), 0, __VA_ARGS__);                   \
    prof_end(L, NAME, 0.0, 0.0);                                                   \
  } while (0)

void gated_pad(const Launch& L, const GPads& p) {
  if (p.n < 1) return;
  int c[GPADS] = {};
  long long grid = 0;
  for (int i = 0; i < p.n; ++i) {
    const long long chunks = (long long)p.p[i].prows * p.p[i].times * (p.p[i].pcols * p.p[i].es / 16);
    c[i] = (int)((chunks + 1023) / 1024);
    grid += c[i];
  }
  // (the copies after the last one have no workgroups)
  for (int i = p.n; i < GPADS; ++i) c[i] = 0;
  HF_LAUNCH("hf_gated_pad", hf_gated_pad, grid, 256, p, c[0], c[1], c[2], c[3], c[4]);
}

void gated_finish(const Launch& L, int type, int out_type, const GFinish* f, int n) {
  FinishAll a = {};
  int grid = 0;
  for (int i = 0; i < n; ++i) {
    const GGemm& g = f[i].g;
    const GEpi& e = f[i].e;
    const int chunks = (std::min(e.mout, g.M) - g.m0 + 7) / 8, rn = tile_n(g.tile);
    const int rows = (e.n1 < g.N ? 2 : 1) * e.nout;
    if (chunks < 1 || rows < 1) continue;
    const int rm = tile_m(g.tile), gy = (g.N + rn - 1) / rn;
    a.one[a.n++] = FinishOne{f[i], rows, chunks, grid,
                             f[i].share ? (long long)rm * rn : (long long)gy * rn * e.ldp, rm, rn,
                             (g.M + rm - 1) / rm, gy, g.K / (type == VT_F32 ? 32 : 64)};
    grid += (int)std::min<long long>(((long long)rows * chunks + 255) / 256, 1 << 20);
  }
  if (grid < 1) return;
  if (type == VT_I8) {
    if (out_type == VT_F32)
      HF_LAUNCH("hf_gated_finish", hf_gated_finish_codes_f32, grid, 256, a);
    else
      HF_LAUNCH("hf_gated_finish", hf_gated_finish_codes_bf16, grid, 256, a);
  } else if (type == VT_F32) {
    HF_LAUNCH("hf_gated_finish", hf_gated_finish_f32, grid, 256, a);
  } else {
    HF_LAUNCH("hf_gated_finish", hf_gated_finish_bf16, grid, 256, a);
  }
}

void gated_pack(const Launch& L, int type, const void* X, long long ldx, long long rows, int cols,
                int8_t* codes, long long ldc, uint8_t* scale, long long lds) {
  const uint32_t per = (uint32_t)((cols + CODE_BLOCK - 1) / CODE_BLOCK * (CODE_BLOCK / 8));
  const uint32_t total = (uint32_t)rows * per;      // at most 2^31: 262,144 rows of 65,536
  if (!total) return;
  const bool much = rows * cols > L3_BYTES / 4;
  if (type == VT_F32)
    HF_LAUNCH("hf_gated_pack", (much ? hf_gated_pack_f32_s : hf_gated_pack_f32), (total + 255) / 256, 256, (const float*)X, ldx,
              total, cols, per, codes, ldc, scale, lds);
  else
    HF_LAUNCH("hf_gated_pack", (much ? hf_gated_pack_bf16_s : hf_gated_pack_bf16), (total + 255) / 256, 256, (const bf16_t*)X, ldx,
              total, cols, per, codes, ldc, scale, lds);
}

void gated_unpack(const Launch& L, int type, const int8_t* codes, long long ldc,
                  const uint8_t* scale, long long lds, long long rows, int cols, void* X,
                  long long ldx) {
  const uint32_t per = (uint32_t)((cols + 7) / 8);
  const uint32_t total = (uint32_t)rows * per;
  if (!total) return;
  const bool much = rows * cols * (type == VT_F32 ? 4 : 2) > L3_BYTES / 2;
  if (type == VT_F32)
    HF_LAUNCH("hf_gated_unpack", (much ? hf_gated_unpack_f32_s : hf_gated_unpack_f32),
              (total + 255) / 256, 256, codes, ldc, scale, lds, cols, (float*)X, ldx, per, total);
  else
    HF_LAUNCH("hf_gated_unpack", (much ? hf_gated_unpack_bf16_s : hf_gated_unpack_bf16),
              (total + 255) / 256, 256, codes, ldc, scale, lds, cols, (bf16_t*)X, ldx, per, total);
}

namespace {
// a row by a wave or by 4, whose lanes hold up to 16 or 64 numbers of it; what no lane
// can hold, or has cut chunks, is read twice (8,192 rows of 4,096, bf16: 39 us read
// twice, 30 held)
template <class E>
void codes_of(const Launch& L, void (*const (&k)[4])(const E*, long long, int, int, int8_t*,
                                                     long long, int, float*),
              const E* X, long long ldx, int rows, int cols, int8_t* codes, long long ldc,
              int zcols, float* scale) {
  const bool even = cols % 8 == 0 && zcols % 8 == 0;
  const int i = !even ? 0 : zcols <= 1024 ? 1 : zcols <= 4096 ? 2 : zcols <= 16384 ? 3 : 0;
  HF_LAUNCH("hf_gated_codes", k[i], i == 1 ? (rows + 3) / 4 : rows, 256, X, ldx, rows,
            cols, codes, ldc, zcols, scale);
}
}  // namespace

void gated_codes(const Launch& L, int type, const void* X, long long ldx, long long rows, int cols,
                 int8_t* codes, long long ldc, int zcols, float* scale) {
  if (rows < 1) return;
#define HF_CK(SUF) {hf_gated_codes_##SUF, hf_gated_codes_##SUF##_c1, hf_gated_codes_##SUF##_c4, \
                    hf_gated_codes_##SUF##_c16}
  if (type == VT_F32)
    codes_of<float>(L, HF_CK(f32), (const float*)X, ldx, (int)rows, cols, codes, ldc, zcols, scale);
  else
    codes_of<bf16_t>(L, HF_CK(bf16), (const bf16_t*)X, ldx, (int)rows, cols, codes, ldc, zcols,
                     scale);
}

void gated_codes_h(const Launch& L, const float* H, long long ldh, const float* hmax,
                   long long ldmax, int nmax, int rows, int cols, int8_t* codes, long long ldc, int zcols, float* scale) {
  if (rows < 1) return;
  const int chunks = (zcols + 2047) / 2048;
  HF_LAUNCH("hf_gated_codes_h", hf_gated_codes_h, (long long)rows * chunks, 256, H, ldh, hmax,
            ldmax, nmax, cols, codes, ldc, zcols, chunks, scale);
}

}  // namespace hfk
