// Products of f32 operands, A stored by rows, B by rows.
#define RSC_T float
#define RSC_AC 0
#define RSC_BC 0
#define RSC_NAME f32_rr
#include "gemm_inst.h"
