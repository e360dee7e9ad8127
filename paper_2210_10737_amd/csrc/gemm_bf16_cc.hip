// Products of bf16 operands, A stored by columns, B by columns.
#define RSC_T __bf16
#define RSC_AC 1
#define RSC_BC 1
#define RSC_NAME bf16_cc
#include "gemm_inst.h"
