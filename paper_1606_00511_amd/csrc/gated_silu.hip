// The gated block's products with silu.
#include "gated_gemm.h"

HF_GATED_ACT(silu, GA_SILU)
