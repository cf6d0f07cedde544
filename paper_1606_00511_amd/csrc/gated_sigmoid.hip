// The gated block's products with sigmoid.
#include "gated_gemm.h"

HF_GATED_ACT(sigmoid, GA_SIGMOID)
