// Products of f16 operands, A stored by rows, B by rows.
#define RSC_T _Float16
#define RSC_AC 0
#define RSC_BC 0
#define RSC_NAME f16_rr
#include "gemm_inst.h"
