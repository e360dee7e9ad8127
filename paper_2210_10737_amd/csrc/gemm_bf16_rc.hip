// Products of bf16 operands, A stored by rows, B by columns.
#define RSC_T __bf16
#define RSC_AC 0
#define RSC_BC 1
#define RSC_NAME bf16_rc
#include "gemm_inst.h"
