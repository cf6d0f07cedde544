// The gated block's products with tanh.
#include "gated_gemm.h"

HF_GATED_ACT(tanh, GA_TANH)
