// Products of f16 operands, A stored by rows, B by columns.
#define RSC_T _Float16
#define RSC_AC 0
#define RSC_BC 1
#define RSC_NAME f16_rc
#include "gemm_inst.h"
