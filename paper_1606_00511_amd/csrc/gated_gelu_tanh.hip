// The gated block's products with gelu_tanh.
#include "gated_gemm.h"

HF_GATED_ACT(gelu_tanh, GA_GELU_TANH)
