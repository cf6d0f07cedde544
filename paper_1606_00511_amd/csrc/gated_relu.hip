// The gated block's products with relu.
#include "gated_gemm.h"

HF_GATED_ACT(relu, GA_RELU)
