// The optimizer step (adamw.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "rsc.h"

namespace rsc {

struct AdamwRates {
    double lr, beta1, beta2;
    float b1, b2, c1, c2, keep, eps;  // c = 1 - b, keep = 1 - lr weight_decay, rounded once
    uint64_t seed;
};

size_t adamw_ws_bytes();
hipError_t adamw_launch(int32_t dtype, int32_t codes, const rsc_adamw_tensor_t *t, int32_t count, const AdamwRates &a,
                        int64_t *step, void *ws, hipStream_t stream);
hipError_t adamw_moments_launch(const rsc_adamw_tensor_t *t, int32_t count, float *const *m, float *const *v,
                                hipStream_t stream);

}  // namespace rsc
