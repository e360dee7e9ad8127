// Products of f32 operands, A stored by rows, B by columns.
#define RSC_T float
#define RSC_AC 0
#define RSC_BC 1
#define RSC_NAME f32_rc
#include "gemm_inst.h"
