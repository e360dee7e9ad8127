// Products of f16 operands, A stored by columns, B by columns.
#define RSC_T _Float16
#define RSC_AC 1
#define RSC_BC 1
#define RSC_NAME f16_cc
#include "gemm_inst.h"
