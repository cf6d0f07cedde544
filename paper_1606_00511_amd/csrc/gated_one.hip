// Products of one row of X (a single token), in fp32, bf16 and 8-bit codes: bound by
// reading the matrices once, and for small ones by what a launch takes.
//
// A wave has a row of a matrix ("up": the same row of both), whose 1,024-byte pieces
// its lanes read 16 bytes each, U of them on their way at a time; the multiply-adds
// with X's row, which all waves read, are the vector units', and the lanes' sums are
// joined in a fixed tree.  A small matrix is so spread over
// the whole card, which 16 rows a workgroup would not fill, and a large one is read
// evenly (bf16: 1,024 x 4,096: down 7.9 -> 4.6 us; 4,096 x 16,384: up 49 -> 46, down 34
// -> 27, 403 MB at 5.6 TB/s; with two rows of X the second one's products cost what
// the even reads gain: 87 us in gated_few.hip, 89 so).
// Rows of one or two pieces leave a wave too little to do: theirs is gated_few.hip (1,024
// x 4,096: up 5.9 us, 7.2 to 7.9 here).  h stays in fp32 between the two products.
// Loads need no alignment.
#include "gated_act.h"
#include "gated_values.h"
#include "mfma_tile.h"

namespace hfk {
namespace {

// 16 bytes of a row as numbers, and their products with X's
template <class E>
struct Piece;
template <>
struct Piece<bf16_t> {
  static constexpr int N = 8;
  typedef float Sum;
  u32x4 w;
  __device__ __forceinline__ float value(int j) const {
    return j & 1 ? __uint_as_float(w[j / 2] & 0xffff0000u) : __uint_as_float(w[j / 2] << 16);
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  typedef float Sum;
  u32x4 w;
  __device__ __forceinline__ float value(int j) const { return __uint_as_float(w[j]); }
};
template <>
struct Piece<int8_t> {
  static constexpr int N = 16;
  typedef int Sum;
  u32x4 w;
};
// as many numbers of X: of its own type, or fp32 (h)
template <int N>
struct Numbers {
  f32x4 v[N / 4];
  __device__ __forceinline__ float value(int j) const { return v[j / 4][j % 4]; }
};
template <class E, class P>
__device__ __forceinline__ void fma_piece(typename Piece<E>::Sum& s, const Piece<E>& a, const P& x) {
  if constexpr (sizeof(E) == 1) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_sdot4((int)a.w[j], (int)x.w[j], s, false);
  } else {
#pragma unroll
    for (int j = 0; j < Piece<E>::N; ++j) s = fmaf(a.value(j), x.value(j), s);
  }
}
// the first `have` elements of N, zeros behind them; all of them where EVEN
template <class T, int N, class P, bool EVEN>
__device__ __forceinline__ void load_piece(P& p, const T* at, int have) {
  static_assert(sizeof(P) == N * sizeof(T), "piece");
  if (EVEN || have >= N) {
    __builtin_memcpy(&p, at, sizeof(P));
  } else {
    T v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < have ? at[j] : T(0);
    __builtin_memcpy(&p, v, sizeof(P));
  }
}

// E: the matrix's type, XT: X's
template <class E, class XT, class O, bool UP, int U>
__device__ __forceinline__ void one_body(const GGemm& s, const GEpi& e) {
  typedef Piece<E> A;
  typedef typename A::Sum Sum;
  typedef typename std::conditional<std::is_same<E, XT>::value, Piece<E>, Numbers<A::N>>::type X;
  constexpr int N = A::N, NA = UP ? 2 : 1;
  const int lane = threadIdx.x & 63;
  const int m = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (m >= s.M) return;
  const E* a[NA];
  a[0] = (const E*)s.A + (size_t)m * s.lda + N * lane;
  if constexpr (UP) a[1] = (const E*)s.A1 + (size_t)m * s.lda1 + N * lane;
  const XT* x = (const XT*)s.B + N * lane;

  Sum acc[NA];
#pragma unroll
  for (int i = 0; i < NA; ++i) acc[i] = 0;
  struct Group {
    A a[U][NA];
    X x[U];
  };
  constexpr int STEP = 64 * N;            // a piece of every lane
  auto products = [&](const Group& f) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NA; ++i) fma_piece<E>(acc[i], f.a[u][i], f.x[u]);
  };
  auto fetch = [&](Group& f, int k0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < NA; ++i) load_piece<E, N, A, true>(f.a[u][i], a[i] + k0 + u * STEP, N);
      load_piece<XT, N, X, true>(f.x[u], x + k0 + u * STEP, N);
    }
    // (all of them ahead of the products, between which the compiler would spread them)
    __builtin_amdgcn_sched_barrier(0);
  };
  const int whole = s.K / (U * STEP);
  int k0 = 0;
  if (whole > 0) {
    Group f, n;
    fetch(f, 0);
    int i = 0;
    for (; i + 2 < whole; i += 2) {
      fetch(n, (i + 1) * U * STEP);
      products(f);
      fetch(f, (i + 2) * U * STEP);
      products(n);
    }
    if (i + 1 < whole) {
      fetch(n, (i + 1) * U * STEP);
      products(f);
      products(n);
    } else {
      products(f);
    }
    k0 = whole * U * STEP;
  }
  if (k0 < s.K) {
    // fewer pieces than a group, the last one cut
    Group f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int have = s.K - k0 - u * STEP - N * lane;
#pragma unroll
      for (int i = 0; i < NA; ++i) load_piece<E, N, A, false>(f.a[u][i], a[i] + k0 + u * STEP, have);
      load_piece<XT, N, X, false>(f.x[u], x + k0 + u * STEP, have);
    }
    products(f);
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < NA; ++i) acc[i] += __shfl_xor(acc[i], d, 64);

  if (lane) return;
  float gr = (float)acc[0], ur = (float)acc[NA - 1];
  if constexpr (sizeof(E) == 1) {
    const RowFactor sn(e.sn[0]);
    gr = sn.scaled(acc[0], e.sm[m]);
    if constexpr (UP) ur = sn.scaled(acc[1], e.sm1[m]);
  }
  if constexpr (UP) {
    if (sizeof(E) != 1 && e.keep != KEEP_NONE) {
      // (what becomes codes is kept in fp32)
      if (sizeof(E) == 4 || e.keep == KEEP_CODES) {
        ((float*)e.kept)[m] = gr;
        ((float*)e.kept)[m + e.F] = ur;
      } else {
        store1((bf16_t*)e.kept + m, gr);
        store1((bf16_t*)e.kept + m + e.F, ur);
      }
    }
    float h = 0.0f;
    with_act(e.act, [&](auto act) { h = act_of<act.value, true>(gr) * ur; });
    ((float*)e.h)[m] = h;
  } else {
    store1((O*)e.out + m, gr);
  }
}

}  // namespace

#define HF_ONE(NAME, E, XT, O, UP)                                                     \
  extern "C" __global__ __launch_bounds__(256) void NAME(GGemm s, GEpi e) {            \
    one_body<E, XT, O, UP, 4>(s, e);                                                   \
  }
HF_ONE(hf_gated_one_up_f32, float, float, float, true)
HF_ONE(hf_gated_one_up_bf16, bf16_t, bf16_t, float, true)
HF_ONE(hf_gated_one_up_codes, int8_t, int8_t, float, true)
HF_ONE(hf_gated_one_down_f32, float, float, float, false)
HF_ONE(hf_gated_one_down_bf16, bf16_t, float, bf16_t, false)
HF_ONE(hf_gated_one_down_codes_f32, int8_t, int8_t, float, false)
HF_ONE(hf_gated_one_down_codes_bf16, int8_t, int8_t, bf16_t, false)

namespace {
void launch(const Launch& L, const char* name, GKernel k, const GGemm& g, const GEpi& e) {
  prof_begin(L, name);
  hipExtLaunchKernelGGL(k, dim3((g.M + 3) / 4), dim3(256), 0, L.stream, prof_a(L), prof_b(L), 0, g,
                        e);
  prof_end(L, name, 2.0 * g.M * (double)g.K, 0.0);
}
}  // namespace

void gated_one_up(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  static const GKernel k[3] = {hf_gated_one_up_f32, hf_gated_one_up_bf16, hf_gated_one_up_codes};
  launch(L, "hf_gated_one_up", k[type], g, e);
}
void gated_one_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e) {
  static const GKernel k[4] = {hf_gated_one_down_f32, hf_gated_one_down_bf16,
                               hf_gated_one_down_codes_f32, hf_gated_one_down_codes_bf16};
  launch(L, "hf_gated_one_down", k[type == VT_I8 ? 2 + out_type : type], g, e);
}

}  // namespace hfk
