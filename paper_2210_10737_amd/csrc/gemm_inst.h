// The launches of one operand type and layout: each gemm_*.hip defines RSC_T,
// RSC_AC, RSC_BC (operands stored by columns) and RSC_NAME and includes this.
#include "gemm.h"

namespace rsc {
namespace {

template <typename F>
hipError_t with_shape(int shape, F f) {
    switch (shape) {
        case 0: return f(std::integral_constant<int, 256>(), std::integral_constant<int, 256>(),
                         std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
        case 1: return f(std::integral_constant<int, 128>(), std::integral_constant<int, 128>(),
                         std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
        case 2: return f(std::integral_constant<int, 128>(), std::integral_constant<int, 64>(),
                         std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 32>(), std::integral_constant<int, 128>(),
                         std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
    }
    return hipErrorInvalidValue;
}

unsigned blocks_of(const Product &p, int bm, int bn) {
    return (unsigned)(ceil_div(p.m, bm) * ceil_div(p.n, bn) * p.splits);
}

}  // namespace

#define RSC_CAT2(a, b) a##b
#define RSC_CAT(a, b) RSC_CAT2(a, b)

hipError_t RSC_CAT(product_, RSC_NAME)(int shape, const Product &p, const Epilogue &e, hipStream_t stream) {
    return with_shape(shape, [&](auto bm, auto bn, auto wm, auto wn) {
        gemm::product_kernel<RSC_T, RSC_AC, RSC_BC, bm.value, bn.value, wm.value, wn.value>
            <<<blocks_of(p, bm.value, bn.value), 64 * wm.value * wn.value, 0, stream>>>(p, e);
        if (p.splits > 1) {
            const int64_t waves = ceil_div(p.m, bm.value) * ceil_div(p.n, bn.value) * (bm.value * bn.value / 1024);
            gemm::join_kernel<RSC_T><<<(unsigned)ceil_div(waves, 4), 256, 0, stream>>>(p, e, bm.value, bn.value);
        }
        return hipGetLastError();
    });
}

#if !RSC_AC
hipError_t RSC_CAT(stats_, RSC_NAME)(int shape, const Product &p, const Classes &c, hipStream_t stream) {
    return with_shape(shape, [&](auto bm, auto bn, auto wm, auto wn) {
        gemm::stats_kernel<RSC_T, RSC_BC, bm.value, bn.value, wm.value, wn.value>
            <<<blocks_of(p, bm.value, bn.value), 64 * wm.value * wn.value, 0, stream>>>(p, c);
        return hipGetLastError();
    });
}
hipError_t RSC_CAT(grad_, RSC_NAME)(int shape, const Product &p, const Classes &c, hipStream_t stream) {
    return with_shape(shape, [&](auto bm, auto bn, auto wm, auto wn) {
        gemm::grad_kernel<RSC_T, RSC_BC, bm.value, bn.value, wm.value, wn.value>
            <<<blocks_of(p, bm.value, bn.value), 64 * wm.value * wn.value, 0, stream>>>(p, c);
        return hipGetLastError();
    });
}
#endif

}  // namespace rsc
