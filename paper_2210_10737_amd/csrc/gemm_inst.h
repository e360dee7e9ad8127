// The launches of one operand type and layout: each gemm_*.hip defines RSC_T,
// RSC_AC, RSC_BC (operands stored by columns) and RSC_NAME and includes this.
#include <type_traits>

#include "gemm.h"

namespace rsc {
namespace {

// f(the shape's configuration). The largest has eight waves of 128 x 64 for 16
// bits, and four of 128 x 128 for fp32, which split each value half as often
// (8192^3: 209 TFLOP/s against 151 to 157 with eight). Tiles of 64 bytes of k
// in a ring of four were within 4 % for 16 bits (1,259 against 1,231 at
// 8192^3, 1,200 against 1,261 at 4096 x 4096 x 8192), and 16 % slower
// where the operands' rows are 32 KiB apart.
template <typename F>
hipError_t with_shape(int shape, F f) {
    using namespace gemm;
    using Largest = std::conditional_t<sizeof(RSC_T) == 2, Config<256, 256, 2, 4, 128, 2>, Config<256, 256, 2, 2, 128, 2>>;
    switch (shape) {
        case 0: return f(Largest());
        case 1: return f(Config<128, 128, 2, 2, 128, 2>());
        case 2: return f(Config<128, 64, 2, 2, 128, 2>());
        case 3: return f(Config<32, 128, 1, 4, 128, 4>());
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
#if !RSC_AC && !RSC_BC
    if (shape == kFewRowsShape) {
        const unsigned blocks = (unsigned)ceil_div(p.n, 8);
        switch (p.m) {
            case 1: gemm::few_rows_kernel<RSC_T, 1><<<blocks, 256, 0, stream>>>(p, e); break;
            case 2: gemm::few_rows_kernel<RSC_T, 2><<<blocks, 256, 0, stream>>>(p, e); break;
            default: return hipErrorInvalidValue;
        }
        return hipGetLastError();
    }
#endif
    return with_shape(shape, [&](auto config) {
        using C = decltype(config);
        gemm::product_kernel<RSC_T, RSC_AC, RSC_BC, C><<<blocks_of(p, C::BM, C::BN), C::THREADS, 0, stream>>>(p, e);
        if (p.splits > 1) {
            const int64_t threads = p.m * ceil_div(p.n, gemm::kWidth<RSC_T>);
            if (threads < 8192 && p.splits > 32)
                gemm::join_kernel<RSC_T, 32><<<(unsigned)ceil_div(threads * 32, 256), 256, 0, stream>>>(p, e);
            else if (threads < 32768 && p.splits > 4)
                gemm::join_kernel<RSC_T, 8><<<(unsigned)ceil_div(threads * 8, 256), 256, 0, stream>>>(p, e);
            else
                gemm::join_kernel<RSC_T, 1><<<(unsigned)ceil_div(threads, 256), 256, 0, stream>>>(p, e);
        }
        return hipGetLastError();
    });
}

#if !RSC_AC
hipError_t RSC_CAT(stats_, RSC_NAME)(int shape, const Product &p, const Classes &c, hipStream_t stream) {
    return with_shape(shape, [&](auto config) {
        using C = decltype(config);
        gemm::stats_kernel<RSC_T, RSC_BC, C><<<blocks_of(p, C::BM, C::BN), C::THREADS, 0, stream>>>(p, c);
        return hipGetLastError();
    });
}
hipError_t RSC_CAT(grad_, RSC_NAME)(int shape, const Product &p, const Classes &c, hipStream_t stream) {
    return with_shape(shape, [&](auto config) {
        using C = decltype(config);
        gemm::grad_kernel<RSC_T, RSC_BC, C><<<blocks_of(p, C::BM, C::BN), C::THREADS, 0, stream>>>(p, c);
        return hipGetLastError();
    });
}
#endif

}  // namespace rsc
