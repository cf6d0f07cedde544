// The products of the gated block without an activation, and the launches of all.
#include "gated_gemm.h"

namespace hfk {

#define HF_GGEMM_T(NAME, MODE)                              \
  HF_GGEMM_FEW(NAME##_f32, float, float, MODE, GA_RELU)     \
  HF_GGEMM_FEW(NAME##_bf16, bf16_t, bf16_t, MODE, GA_RELU)
HF_GGEMM_T(hf_gated_down, DOWN)
HF_GGEMM_T(hf_gated_dx, DX)
HF_GGEMM_WIDE(hf_gated_dw_f32, float, float, DW, GA_RELU)
HF_GGEMM_WIDE(hf_gated_dw_bf16, bf16_t, bf16_t, DW, GA_RELU)
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
  if (g.M <= g.m0 || g.N < 1) return;
  const int RM = tile_m(g.tile), RN = tile_n(g.tile);
  const dim3 grid((g.M - g.m0 + RM - 1) / RM, (g.N + RN - 1) / RN, g.splits);
  prof_begin(L, name);
  hipExtLaunchKernelGGL(k[g.tile], grid, dim3(g.tile == TILE_BIG ? 512 : 256), 0, L.stream,
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
void gated_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e) {
  static const GKernel k[2][4] = {HF_GK_FEW(hf_gated_down_f32), HF_GK_FEW(hf_gated_down_bf16)};
  static const GKernel c[2][4] = {HF_GK_FEW(hf_gated_down_codes_f32),
                                  HF_GK_FEW(hf_gated_down_codes_bf16)};
  launch(L, "hf_gated_down", type == VT_I8 ? c[out_type] : k[type], g, e);
}
void gated_dx(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  static const GKernel k[2][4] = {HF_GK_FEW(hf_gated_dx_f32), HF_GK_FEW(hf_gated_dx_bf16)};
  launch(L, "hf_gated_dx", k[type], g, e);
}
void gated_dw(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  static const GKernel k[2][2] = {{hf_gated_dw_f32, hf_gated_dw_f32_big},
                                  {hf_gated_dw_bf16, hf_gated_dw_bf16_big}};
  launch(L, "hf_gated_dw", k[type], g, e);
}

}  // namespace hfk
