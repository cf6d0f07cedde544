// The gated block's products with gelu.
#include "gated_gemm.h"

HF_GATED_ACT(gelu, GA_GELU)
