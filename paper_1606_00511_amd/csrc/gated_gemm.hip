// The products of the gated block without an activation, and the launches of all.
#include "gated_gemm.h"

namespace hfk {

#define HF_GGEMM_T(NAME, MODE)                              \
  HF_GGEMM_FEW(NAME##_f32, float, float, MODE, GA_RELU)     \
  HF_GGEMM_FEW(NAME##_bf16, bf16_t, bf16_t, MODE, GA_RELU)
HF_GGEMM_T(hf_gated_down, DOWN)
// dh = dY Wd of few rows, by partials (a product like dX's of one matrix), and what "dh"
// makes of their sum: a tile's whole K on one unit is a chain of reads that wait for
// memory, 0.7 us a block of 128 bytes, and few rows have few tiles
HF_GGEMM_T(hf_gated_dh_part, DX)
template <class E>
__device__ __forceinline__ void dh_sum_body(const GGemm& g, const GEpi& e, long long stride) {
  const uint32_t chunks = (uint32_t)e.Fp / 8, i = blockIdx.x * 256u + threadIdx.x;
  const int n = (int)(i / chunks), f = 8 * (int)(i % chunks);
  if (n >= g.N) return;
  const int have = n < e.T ? e.F - f : 0;
  const float* p = e.part + (size_t)n * e.ldp + f;
  float d[8], gv[8], u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) d[j] = 0.0f;
  get_kept<E>(e, n, f, have, gv, u);
#pragma unroll 4
  for (int s = 0; s < g.splits; ++s) {
    const f32x4 a = *(const f32x4*)(p + s * stride), b = *(const f32x4*)(p + s * stride + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      d[j] += a[j];
      d[4 + j] += b[j];
    }
  }
  with_act(e.act, [&](auto act) { dh_chunk<E, act.value, false>(e, n, f, have, d, gv, u); });
}
extern "C" __global__ __launch_bounds__(256) void hf_gated_dh_sum_f32(GGemm g, GEpi e,
                                                                      long long stride) {
  dh_sum_body<float>(g, e, stride);
}
extern "C" __global__ __launch_bounds__(256) void hf_gated_dh_sum_bf16(GGemm g, GEpi e,
                                                                       long long stride) {
  dh_sum_body<bf16_t>(g, e, stride);
}
// dX, dWd and dWg with dWu in one launch, its workgroups in this order: they need
// nothing of each other, and the last ones of a product leave no unit idle while
// another's begin
template <class E, int WM, int WN, int GM, int GN>
__device__ __forceinline__ void grads_body(const GGrads& a) {
  const int L = blockIdx.x;
  if (L < a.first[1]) {
    ggemm_body<E, E, DX, GA_RELU, WM, WN, GM, GN, 2>(a.g[0], a.e[0], L);
  } else {
    const bool last = L >= a.first[2];
    const GGemm g = last ? a.g[2] : a.g[1];
    const GEpi e = last ? a.e[2] : a.e[1];
    ggemm_body<E, E, DW, GA_RELU, WM, WN, GM, GN, 2>(g, e, L - (last ? a.first[2] : a.first[1]));
  }
}
// The same by units that have equal shares of the K blocks of all tiles in a row: a
// share ends inside a tile, whose partials the units that have a share of it leave in
// parts 2 u (that began in another unit's share) and 2 u + 1 of the workspace.
template <class E, int WM, int WN, int GM, int GN>
__device__ __forceinline__ void shares_body(const GGrads& a) {
  constexpr int RM = 32 * WM * GM, RN = 32 * WN * GN, BK = 128 / (int)sizeof(E);
  // (an XCD's units have neighbouring tiles)
  const int L = blockIdx.x, u = L % 8 * (gridDim.x / 8) + L / 8;
  const int end = min((u + 1) * a.share, a.work[3]);
  for (int at = u * a.share; at < end;) {
    const int i = at >= a.work[2] ? 2 : at >= a.work[1] ? 1 : 0;
    const GGemm g = a.g[i];
    const GEpi e = a.e[i];
    const int gx = (g.M + RM - 1) / RM, gy = (g.N + RN - 1) / RN, nvb = g.K / BK;
    const int r = (at - a.work[i]) / nvb;
    Piece p;
    // (what follows from the thread is worked out for each tile: kept over the loop it
    // takes registers that the products need)
    p.tid = threadIdx.x;
    asm("" : "+v"(p.tid));
    tile_in(r, gx, gy, p.tm, p.tn);
    p.vb0 = at - a.work[i] - r * nvb;
    p.nblk = min(nvb - p.vb0, end - at);
    p.part = p.nblk == nvb ? nullptr : a.part + (size_t)(2 * u + (p.vb0 == 0)) * (RM * RN);
    if (i == 0) ggemm_body<E, E, DX, GA_RELU, WM, WN, GM, GN, 2, true>(g, e, 0, p);
    else ggemm_body<E, E, DW, GA_RELU, WM, WN, GM, GN, 2, true>(g, e, 0, p);
    at += p.nblk;
    __syncthreads();       // the stages are free
  }
}
#define HF_GRADS(SUF, E)                                                                        \
  extern "C" __global__ __launch_bounds__(512, 1) void hf_gated_grads_##SUF##_big(GGrads a) {   \
    grads_body<E, 4, 2, 2, 4>(a);                                                               \
  }                                                                                             \
  extern "C" __global__ __launch_bounds__(256, 2) void hf_gated_grads_##SUF(GGrads a) {         \
    grads_body<E, 2, 2, 2, 2>(a);                                                               \
  }
HF_GRADS(f32, float)
HF_GRADS(bf16, bf16_t)
extern "C" __global__ __launch_bounds__(512, 1) void hf_gated_shares_f32_big(GGrads a) {
  shares_body<float, 4, 2, 2, 4>(a);
}
extern "C" __global__ __launch_bounds__(256, 2) void hf_gated_shares_f32(GGrads a) {
  shares_body<float, 2, 2, 2, 2>(a);
}
HF_GGEMM_FEW(hf_gated_down_codes_f32, int8_t, float, DOWN, GA_RELU)
HF_GGEMM_FEW(hf_gated_down_codes_bf16, int8_t, bf16_t, DOWN, GA_RELU)

extern const GActKernels gated_sigmoid, gated_tanh, gated_relu, gated_silu, gated_gelu,
    gated_gelu_tanh;

namespace {
const GActKernels& act_kernels(int act) {
  switch (act) {
    case GA_SIGMOID: return gated_sigmoid;
    case GA_TANH: return gated_tanh;
    case GA_RELU: return gated_relu;
    case GA_SILU: return gated_silu;
    case GA_GELU: return gated_gelu;
    default: return gated_gelu_tanh;
  }
}
void launch(const Launch& L, const char* name, const GKernel* k, const GGemm& g, const GEpi& e) {
  const int grid = gated_tiles(g) * g.splits;
  if (grid < 1) return;
  prof_begin(L, name);
  hipExtLaunchKernelGGL(k[g.tile], dim3(grid), dim3(g.tile == TILE_BIG ? 512 : 256), 0, L.stream,
                        prof_a(L), prof_b(L), 0, g, e);
  prof_end(L, name, 2.0 * (g.M - g.m0) * (double)g.N * g.K, 0.0);
}
}  // namespace

void gated_up(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  launch(L, "hf_gated_up", act_kernels(e.act).up[type], g, e);
}
void gated_dh(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  launch(L, "hf_gated_dh", act_kernels(e.act).dh[type], g, e);
}
void gated_dh_split(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  static const GKernel k[2][4] = {HF_GK_FEW(hf_gated_dh_part_f32), HF_GK_FEW(hf_gated_dh_part_bf16)};
  launch(L, "hf_gated_dh_part", k[type], g, e);
  const int rn = tile_n(g.tile), grid = (int)(((long long)g.N * (e.Fp / 8) + 255) / 256);
  prof_begin(L, "hf_gated_dh_sum");
  hipExtLaunchKernelGGL((type == VT_F32 ? hf_gated_dh_sum_f32 : hf_gated_dh_sum_bf16), dim3(grid),
                        dim3(256), 0, L.stream, prof_a(L), prof_b(L), 0, g, e,
                        (long long)((g.N + rn - 1) / rn) * rn * e.ldp);
  prof_end(L, "hf_gated_dh_sum", 0.0, 0.0);
}
void gated_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e) {
  static const GKernel k[2][4] = {HF_GK_FEW(hf_gated_down_f32), HF_GK_FEW(hf_gated_down_bf16)};
  static const GKernel c[2][4] = {HF_GK_FEW(hf_gated_down_codes_f32),
                                  HF_GK_FEW(hf_gated_down_codes_bf16)};
  launch(L, "hf_gated_down", type == VT_I8 ? c[out_type] : k[type], g, e);
}
void gated_grads(const Launch& L, int type, GGrads a) {
  a.first[0] = 0;
  for (int i = 0; i < 3; ++i)
    a.first[i + 1] = a.first[i] + (a.e[i].out ? gated_tiles(a.g[i]) * a.g[i].splits : 0);
  if (a.first[3] < 1) return;
  static void (*const k[3][2])(GGrads) = {{hf_gated_grads_f32, hf_gated_grads_f32_big},
                                          {hf_gated_grads_bf16, hf_gated_grads_bf16_big},
                                          {hf_gated_shares_f32, hf_gated_shares_f32_big}};
  const int tile = a.g[0].tile;
  prof_begin(L, "hf_gated_grads");
  hipExtLaunchKernelGGL(k[a.share ? 2 : type][tile], dim3(a.share ? units_of(tile) : a.first[3]),
                        dim3(tile == TILE_BIG ? 512 : 256), 0, L.stream, prof_a(L), prof_b(L), 0, a);
  prof_end(L, "hf_gated_grads", 0.0, 0.0);
}

}  // namespace hfk
