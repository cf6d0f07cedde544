// Products of few rows of X (a new token of each of some users), in fp32, bf16 and
// 8-bit codes: bound by reading the matrices once.
//
// A workgroup has 16 or 32 rows of a matrix ("up": of both) and all rows of X, and
// its waves share K: groups of U steps of 64 bytes a row, in turn.  Fragments go
// from memory straight into registers, 16 rows of 64 bytes an instruction, the
// next group's on their way during a group's MFMAs (16 x 16, so that one to 16
// tokens cost one product); nothing waits for another wave before the sums of all
// waves are joined in LDS, in the order of the waves.  Loads need no alignment and
// the last group reads element by element past K's last whole chunk, so odd widths
// are read in place.
// Against tiles of 128 x 128 with partials in memory (bf16): 1 row, 1,024 x 4,096:
// 32 -> 14 us; 24 rows, 4,096 x 16,384: up 74 -> 54; 15 rows, 1,507 x 2,494, copied for
// tiles: 34 -> 25.
#include "gated_act.h"
#include "gated_values.h"
#include "mfma_tile.h"

namespace hfk {
namespace {

template <class E>
struct Step;                       // 64 bytes a row: K values, a lane 16 bytes
template <>
struct Step<bf16_t> {
  typedef f32x4 Sum;
  __device__ static __forceinline__ Sum mma(u32x4 a, u32x4 b, Sum c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Step<int8_t> {
  typedef i32x4 Sum;
  __device__ static __forceinline__ Sum mma(u32x4 a, u32x4 b, Sum c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};
template <>
struct Step<float> {
  typedef f32x4 Sum;
  // (value j of the 4 lanes that share a row is k = 4 lane + j, of A and B alike)
  __device__ static __forceinline__ Sum mma(u32x4 a, u32x4 b, Sum c) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
};

__device__ __forceinline__ u32x4 load16(const void* p) {
  u32x4 w;
  __builtin_memcpy(&w, p, 16);
  return w;
}
// the first `have` elements, zeros behind them
template <class E>
__device__ __forceinline__ u32x4 load_some(const E* p, int have) {
  constexpr int N = 16 / (int)sizeof(E);
  if (have >= N) return load16(p);
  E v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = j < have ? p[j] : E(0);
  u32x4 w;
  __builtin_memcpy(&w, v, 16);
  return w;
}

// RB blocks of 16 rows of a matrix, NB of X; TWO: X's rows have a second term
template <class E, class O, bool UP, int RB, int NB, int U, int WMAX, bool TWO>
__device__ __forceinline__ void few_body(const GGemm& s, const GEpi& e) {
  constexpr int EPC = 16 / (int)sizeof(E), KS = 4 * EPC;
  constexpr int NA = UP ? 2 * RB : RB, NX = TWO ? 2 * NB : NB;
  typedef typename Step<E>::Sum Sum;
  const int lane = threadIdx.x & 63, l = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6;
  const int m0 = blockIdx.x * 16 * RB;
  const int K = s.K, groups = (K + U * KS - 1) / (U * KS), whole = K / (U * KS);

  const E *a[NA], *x[NX];
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const size_t row = (size_t)min(m0 + 16 * i + l, s.alim - 1);
    a[i] = (const E*)s.A + row * s.lda + EPC * q;
    if constexpr (UP) a[RB + i] = (const E*)s.A1 + row * s.lda1 + EPC * q;
  }
#pragma unroll
  for (int i = 0; i < NX; ++i)
    x[i] = (const E*)s.B + (size_t)(min(16 * (i % NB) + l, s.blim - 1) + (i < NB ? 0 : e.dup)) * s.ldb +
           EPC * q;

  Sum acc[NA][NB];
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][j][r] = 0;
  struct Group {
    u32x4 a[U][NA], x[U][NX];
  };
  auto fetch = [&](Group& f, int g) {
    const int k0 = g * U * KS;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < NA; ++i) f.a[u][i] = load16(a[i] + k0 + u * KS);
#pragma unroll
      for (int i = 0; i < NX; ++i) f.x[u][i] = load16(x[i] + k0 + u * KS);
    }
    // (all of them ahead of the products, between which the compiler would spread
    // them: up of 1 row, 4,096 x 16,384: 52 -> 49 us)
    __builtin_amdgcn_sched_barrier(0);
  };
  auto mma = [&](const Group& f) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NX; ++j)
          acc[i][j % NB] = Step<E>::mma(f.a[u][i], f.x[u][j], acc[i][j % NB]);
  };
  // This wave's whole groups, two at a time; no branch comes between a group's loads
  // and the products of the one before, where the compiler would wait for all.
  // (All workgroups in one order: what they read of X at a time is then one cache's
  // lines; started at different places, 24 rows, 4,096 x 16,384: down 45 -> 51 us.)
  const int mine = wave < whole ? (whole - wave + W - 1) / W : 0;
  Group f, n;
  if (mine > 0) {
    auto group = [&](int i) { return wave + i * W; };
    fetch(f, group(0));
    int i = 0;
    for (; i + 2 < mine; i += 2) {
      fetch(n, group(i + 1));
      mma(f);
      fetch(f, group(i + 2));
      mma(n);
    }
    if (i + 1 < mine) {
      fetch(n, group(i + 1));
      mma(f);
      mma(n);
    } else {
      mma(f);
    }
  }
  if (whole < groups && whole % W == wave) {
    const int k0 = whole * U * KS;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int have = K - k0 - u * KS - EPC * q;
#pragma unroll
      for (int i = 0; i < NA; ++i) f.a[u][i] = load_some(a[i] + k0 + u * KS, have);
#pragma unroll
      for (int i = 0; i < NX; ++i) f.x[u][i] = load_some(x[i] + k0 + u * KS, have);
    }
    mma(f);
  }

  // the waves' sums, joined by a wave for each pair of blocks
  __shared__ Sum part[WMAX][NA * NB][64];
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) part[wave][i * NB + j][lane] = acc[i][j];
  __syncthreads();
  auto join = [&](auto act, int p) {
    const int i = p / NB, j = p % NB;
    Sum g, u;
#pragma unroll
    for (int r = 0; r < 4; ++r) g[r] = u[r] = 0;
#pragma unroll 4
    for (int w = 0; w < W; ++w) {
      g += part[w][i * NB + j][lane];
      if constexpr (UP) u += part[w][(RB + i) * NB + j][lane];
    }
    // lane (l, q), register r: row n = l of X, row m = 4 q + r of the matrix
    const int n = 16 * j + l, m = m0 + 16 * i + 4 * q;
    if constexpr (UP) {
      float v[4];
      const bool keep = sizeof(E) != 1 && e.keep != KEEP_NONE && n < e.T;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int mm = min(m + r, e.F - 1);
        float gr, ur;
        if constexpr (sizeof(E) == 1) {
          const RowFactor sn(e.sn[min(n, e.T - 1)]);
          gr = sn.scaled(g[r], e.sm[mm]);
          ur = sn.scaled(u[r], e.sm1[mm]);
        } else {
          gr = g[r];
          ur = u[r];
        }
        if (keep && m + r < e.F) {
          // (what becomes codes is kept in fp32)
          const size_t at = (size_t)n * e.ldk + m + r;
          if (sizeof(E) == 4 || e.keep == KEEP_CODES) {
            ((float*)e.kept)[at] = gr;
            ((float*)e.kept)[at + e.F] = ur;
          } else {
            store1((bf16_t*)e.kept + at, gr);
            store1((bf16_t*)e.kept + at + e.F, ur);
          }
        }
        v[r] = m + r < e.F ? act_of<act.value, sizeof(E) != 2>(gr) * ur : 0.0f;
      }
      if constexpr (sizeof(E) == 1) {
        uint32_t big = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) big = max(big, __float_as_uint(v[r]) & 0x7fffffffu);
        big = max(big, (uint32_t)__shfl_xor((int)big, 16, 64));
        big = max(big, (uint32_t)__shfl_xor((int)big, 32, 64));
        if (q == 0 && n < e.T && m < e.F) e.hmax[(size_t)n * e.ldmax + m / 16] = __uint_as_float(big);
      }
      if (n < e.T && m < e.Fp) {
        if (sizeof(E) == 2 && !e.h32) {
          uint32_t b[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) b[r] = f2bf(v[r]);
          bf16_t* h = (bf16_t*)e.h + (size_t)n * e.ldh + m;
          *(uint2*)h = uint2{b[0] | b[1] << 16, b[2] | b[3] << 16};
          if (e.dup) {
#pragma unroll
            for (int r = 0; r < 4; ++r) b[r] = f2bf(rest_of(v[r], b[r]));
            *(uint2*)(h + e.dup * e.ldh) = uint2{b[0] | b[1] << 16, b[2] | b[3] << 16};
          }
        } else {
          *(f32x4*)((float*)e.h + (size_t)n * e.ldh + m) = f32x4{v[0], v[1], v[2], v[3]};
        }
      }
    } else if (n < e.nout) {
      O* out = (O*)e.out + (size_t)n * e.ldo + m;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (m + r < e.mout) {
          if constexpr (sizeof(E) == 1) store1(out + r, RowFactor(e.sn[n]).scaled(g[r], e.sm[m + r]));
          else store1(out + r, g[r]);
        }
    }
  };
  for (int p = wave; p < RB * NB; p += W) {
    if constexpr (UP) with_act(e.act, [&](auto act) { join(act, p); });
    else join(std::integral_constant<int, 0>(), p);
  }
}

}  // namespace

// up to 16, 32 and 64 rows of X; "up" with 16 rows of both matrices a workgroup, and of
// more than 16 rows of X with 32 where that leaves no unit without a workgroup (half
// the reads of X: 24 rows, 4,096 x 16,384: 63 -> 54 us; 28 rows, 2,981 x 3,115, fp32, 98
// workgroups: 54 us, 195: 36).  With second terms a wave has half as much on its way and
// up to twice as many share K (24 rows, 300 x 900: 14.5 -> 13.0 us; 869 x 3,110: 23.7 ->
// 22.0).
#define HF_FEW(NAME, E, O, UP, RB, U32, U64, W, TWO)                                            \
  extern "C" __global__ __launch_bounds__(64 * W) void NAME##_32(GGemm s, GEpi e) {             \
    few_body<E, O, UP, RB, 2, U32, W, TWO>(s, e);                                               \
  }                                                                                             \
  extern "C" __global__ __launch_bounds__(64 * W) void NAME##_64(GGemm s, GEpi e) {             \
    few_body<E, O, UP, RB, 4, U64, W, TWO>(s, e);                                               \
  }
#define HF_FEW_ALL(NAME, E, O, UP, U32, U64, W, TWO)                                            \
  extern "C" __global__ __launch_bounds__(1024) void NAME##_16(GGemm s, GEpi e) {               \
    few_body<E, O, UP, 1, 1, 4, 16, TWO>(s, e);                                                 \
  }                                                                                             \
  HF_FEW(NAME, E, O, UP, 1, U32, U64, W, TWO)
HF_FEW_ALL(hf_gated_few_up_f32, float, float, true, 4, 2, 8, false)
HF_FEW_ALL(hf_gated_few_up_bf16, bf16_t, bf16_t, true, 4, 2, 8, false)
HF_FEW_ALL(hf_gated_few_up_codes, int8_t, float, true, 4, 2, 8, false)
HF_FEW(hf_gated_few_up2_f32, float, float, true, 2, 2, 2, 8, false)
HF_FEW(hf_gated_few_up2_bf16, bf16_t, bf16_t, true, 2, 2, 2, 8, false)
HF_FEW(hf_gated_few_up2_codes, int8_t, float, true, 2, 2, 2, 8, false)
HF_FEW_ALL(hf_gated_few_down_f32, float, float, false, 4, 2, 8, false)
HF_FEW_ALL(hf_gated_few_down_bf16, bf16_t, bf16_t, false, 2, 1, 16, true)
HF_FEW_ALL(hf_gated_few_down_codes_f32, int8_t, float, false, 4, 2, 8, false)
HF_FEW_ALL(hf_gated_few_down_codes_bf16, int8_t, bf16_t, false, 4, 2, 8, false)

namespace {
#define HF_FK(NAME) {NAME##_16, NAME##_32, NAME##_64}
#define HF_FK2(NAME) {nullptr, NAME##_32, NAME##_64}
// by type (codes: and the output's) and rows
const GKernel few_up[3][3] = {HF_FK(hf_gated_few_up_f32), HF_FK(hf_gated_few_up_bf16),
                              HF_FK(hf_gated_few_up_codes)};
const GKernel few_up2[3][3] = {HF_FK2(hf_gated_few_up2_f32), HF_FK2(hf_gated_few_up2_bf16),
                               HF_FK2(hf_gated_few_up2_codes)};
const GKernel few_down[4][3] = {HF_FK(hf_gated_few_down_f32), HF_FK(hf_gated_few_down_bf16),
                                HF_FK(hf_gated_few_down_codes_f32),
                                HF_FK(hf_gated_few_down_codes_bf16)};
inline int size_of(int type) { return type == VT_F32 ? 4 : type == VT_BF16 ? 2 : 1; }

// two: the kernels with 32 rows a workgroup, or null; rest: X's rows have second terms
void launch(const Launch& L, const char* name, const GKernel* one, const GKernel* two, int es,
            bool rest, const GGemm& g, const GEpi& e) {
  const int i = g.N <= 16 ? 0 : g.N <= 32 ? 1 : 2;
  const bool rows32 = i > 0 && two && g.M > 255 * 32;
  const int rb = rows32 ? 2 : 1, most = i == 0 || rest ? 16 : 8;
  const int u = (i == 2 || rows32 ? 2 : 4) / (i > 0 && rest ? 2 : 1);
  const int grid = (g.M + 16 * rb - 1) / (16 * rb);
  // enough waves for 8 a compute unit, each with a group of K at least
  const int groups = (g.K * es + 64 * u - 1) / (64 * u);
  int w = 1;
  while (w < most && 2 * w <= groups && (w < 4 || (long long)grid * w < 2048)) w *= 2;
  prof_begin(L, name);
  hipExtLaunchKernelGGL((rows32 ? two : one)[i], dim3(grid), dim3(64 * w), 0, L.stream, prof_a(L),
                        prof_b(L), 0, g, e);
  prof_end(L, name, 2.0 * g.M * (double)g.N * g.K, 0.0);
}
}  // namespace

void gated_few_up(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  launch(L, "hf_gated_few_up", few_up[type], few_up2[type], size_of(type), false, g, e);
}
void gated_few_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e) {
  launch(L, "hf_gated_few_down", few_down[type == VT_I8 ? 2 + out_type : type], nullptr,
         size_of(type), type == VT_BF16, g, e);
}

}  // namespace hfk
