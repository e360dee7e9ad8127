// Products of f32 operands, A stored by columns, B by columns.
#define RSC_T float
#define RSC_AC 1
#define RSC_BC 1
#define RSC_NAME f32_cc
#include "gemm_inst.h"
