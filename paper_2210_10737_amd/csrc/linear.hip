// A layer's product Y = act(alpha X W + bias + beta R) and its gradients, and
// the choice of tiles and splits for every product of the update phase.
#include <cmath>

#include "rsc_internal.h"
#include "update.h"

namespace rsc {
namespace {

constexpr int kCus = 256;

template <typename T>
struct Val;
template <>
struct Val<float> {
    static constexpr int W = 4;
};
template <>
struct Val<__bf16> {
    static constexpr int W = 8;
};
template <>
struct Val<_Float16> {
    static constexpr int W = 8;
};

// act'(z) from what the forward pass kept: the output for a ReLU (positive
// where the argument was), the argument itself, in fp32, for the others: rounded
// to 16 bits it added a tenth to a gradient's error.
__device__ __forceinline__ float slope_of(float s, int act) {
    switch (act) {
        case kRelu: return s > 0.f ? 1.f : (s != s ? s : 0.f);
        case kGelu: {
            const float cdf = 0.5f * erfcf(-0.70710678118654752f * s);
            return cdf + s * 0.39894228040143268f * expf(-0.5f * s * s);
        }
        case kSilu: {
            const float p = 1.f / (1.f + expf(-s));
            // s p (1 - p) without 0 * inf far below zero, where p is 0
            return p + (s < -88.f ? 0.f : s * p * (1.f - p));
        }
        default: return 1.f;
    }
}

// One pass over dY: dz = dY act'(saved), dr = beta dz, and the column sums of
// dz over this block's rows, in fp64 (the additions hide behind the loads). dz is
// rounded to the operands' type, for the matrix instructions: for 16 bits dX and dW are
// then off by sqrt(2) times their own rounding, behind GELU and SiLU (a ReLU's
// dz is dY or 0). A second product for the rest would double the pass. Bound by
// memory: 232,965 x 256 fp32 with GELU 164 us, 4.4 TB/s.
// A block takes `strip` columns, as groups of W values a thread, and the rows
// of its chunk; any of dz, dr and part may be missing.
struct Pass {
    const void *dy, *saved;
    int64_t lddy, ldsaved;
    void *dz, *dr;
    int64_t lddz, lddr;
    double *part;  // part[chunk * m + column]
    int64_t n;
    int32_t m, act, groups, rows_a_chunk;  // groups: threads along the columns, a power of two
    float beta;
};

template <typename T>
__device__ __forceinline__ void write_row(T *p, int count, const float (&v)[Val<T>::W], float by) {
    constexpr int W = Val<T>::W;
    typedef T vec __attribute__((ext_vector_type(W)));
    if (count >= W) {
        vec x;
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = (T)(by * v[i]);
        *(vec *)p = x;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < count) p[i] = (T)(by * v[i]);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void pass_kernel(Pass p) {
    constexpr int W = Val<T>::W;
    __shared__ double sum[256 * W];
    const int g = threadIdx.x & (p.groups - 1), lanes = 256 / p.groups, lane = threadIdx.x / p.groups;
    const int c = (blockIdx.x * p.groups + g) * W, count = p.m - c;
    const int64_t r0 = (int64_t)blockIdx.y * p.rows_a_chunk, r1 = min(p.n, r0 + p.rows_a_chunk);
    double acc[W];
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] = 0.0;
    if (count > 0) {
        const auto take = [&](int64_t row, float (&v)[W], const float (&s)[W]) {
            if (p.act != kNone) {
#pragma unroll
                for (int i = 0; i < W; ++i) v[i] *= slope_of(s[i], p.act);
            }
            if (p.dz) write_row<T>((T *)p.dz + row * p.lddz + c, count, v, 1.f);
            if (p.dr) write_row<T>((T *)p.dr + row * p.lddr + c, count, v, p.beta);
            if (p.part) {
#pragma unroll
                for (int i = 0; i < W; ++i) acc[i] += (double)v[i];
            }
        };
        // four rows a turn, all read before the first is converted or anything
        // is written. Whole 16 bytes are read also where the row ends inside
        // them (rows are whole 16-byte units apart) and zeroed from there on.
        typedef T vec __attribute__((ext_vector_type(W)));
        for (int64_t r = r0 + lane; r < r1; r += 4 * lanes) {
            vec y[4], z[4];
            float4 zf[4][W / 4];
            // kept in T (a ReLU's output) or in fp32
            const bool same = p.act == kRelu || (p.act != kNone && sizeof(T) == 4);
            const bool wide = p.act != kNone && !same;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t row = min(r + u * lanes, r1 - 1);
                y[u] = *(const vec *)((const T *)p.dy + row * p.lddy + c);
                if (same) z[u] = *(const vec *)((const T *)p.saved + row * p.ldsaved + c);
                if (wide) {
                    // (the row's 16-byte units; past the last one it is read again)
                    const float4 *const from = (const float4 *)((const float *)p.saved + row * p.ldsaved + c);
#pragma unroll
                    for (int q = 0; q < W / 4; ++q) zf[u][q] = from[count > 4 * q ? q : 0];
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (r + u * lanes >= r1) break;
                float v[W], s[W];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    v[i] = i < count ? (float)y[u][i] : 0.f;
                    s[i] = 0.f;
                    if (same) s[i] = i < count ? (float)z[u][i] : 0.f;
                    if (wide) s[i] = i < count ? (&zf[u][i / 4].x)[i % 4] : 0.f;
                }
                take(r + u * lanes, v, s);
            }
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int i = 0; i < W; ++i) sum[i * 256 + threadIdx.x] = acc[i];
    __syncthreads();
    for (int j = threadIdx.x; j < p.groups * W; j += 256) {
        const int col = (blockIdx.x * p.groups) * W + j;
        if (col >= p.m) continue;
        double s = 0.0;
        for (int l = 0; l < lanes; ++l) s += sum[(j % W) * 256 + l * p.groups + j / W];
        p.part[(int64_t)blockIdx.y * p.m + col] = s;
    }
}

// out[col] = scale * the chunks' sums: 64 threads a column, each every 64th
// chunk in order, then over a fixed tree. (16 threads a column took 31 to 42
// us for 2,048 chunks.)
template <typename T>
__global__ __launch_bounds__(1024) void column_total_kernel(const double *part, int32_t chunks, int32_t m, float scale,
                                                           const float *scale_dev, T *out) {
    __shared__ double sum[1024];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), s = threadIdx.x >> 4;
    double acc = 0.0;
    if (c < m) {
        int i = s;
        for (; i + 192 < chunks; i += 256) {
            const double *p = part + (int64_t)i * m + c;
            const double x = p[0], y = p[64 * (int64_t)m], z = p[128 * (int64_t)m], w = p[192 * (int64_t)m];
            acc += (x + y) + (z + w);
        }
        for (; i < chunks; i += 64) acc += part[(int64_t)i * m + c];
    }
    sum[threadIdx.x] = acc;
    __syncthreads();
#pragma unroll
    for (int h = 32; h > 0; h /= 2) {
        if (s < h) sum[threadIdx.x] += sum[threadIdx.x + h * 16];
        __syncthreads();
    }
    if (s == 0 && c < m) {
        acc = sum[threadIdx.x];
        const double by = scale_dev ? (double)scale * (double)*scale_dev : (double)scale;
        out[c] = (T)(float)(by * acc);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T *p, int64_t ld, int64_t rows, int64_t cols) {
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += step)
        p[(i / cols) * ld + i % cols] = (T)0.f;
}

struct Chunks {
    int32_t groups, strips, rows, count;
};
// about 2,048 blocks, and at least 8 rows for each thread of a column
Chunks chunks_of(int32_t dtype, int64_t n, int64_t m) {
    const int64_t w = dtype == kF32 ? 4 : 8, need = ceil_div(m, w);
    Chunks c;
    c.groups = 1;
    while (c.groups < 64 && c.groups < need) c.groups *= 2;
    c.strips = (int32_t)ceil_div(need, c.groups);
    const int64_t lanes = 256 / c.groups;
    const int64_t blocks = std::max<int64_t>(1, 2048 / c.strips);
    c.rows = (int32_t)std::min<int64_t>(std::max<int64_t>(ceil_div(ceil_div(n, blocks), lanes) * lanes, 8 * lanes),
                                        int64_t(1) << 30);
    c.count = (int32_t)ceil_div(std::max<int64_t>(n, 1), c.rows);
    return c;
}

hipError_t pass_launch(int32_t dtype, Pass p, const Chunks &c, hipStream_t stream) {
    p.groups = c.groups;
    p.rows_a_chunk = c.rows;
    // a row's strips next to each other: blocks that run together read whole
    // rows (strips of rows 4 KiB apart alone are in a quarter of the channels)
    const dim3 grid((unsigned)c.strips, (unsigned)c.count);
    if (dtype == kF32) pass_kernel<float><<<grid, 256, 0, stream>>>(p);
    else if (dtype == kBf16) pass_kernel<__bf16><<<grid, 256, 0, stream>>>(p);
    else pass_kernel<_Float16><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t column_total_launch(int32_t dtype, const double *part, int32_t chunks, int32_t m, float scale,
                               const float *scale_dev, void *out, int32_t out_f32, hipStream_t stream) {
    const unsigned grid = (unsigned)ceil_div(m, 16);
    if (dtype == kF32 || out_f32)
        column_total_kernel<float><<<grid, 1024, 0, stream>>>(part, chunks, m, scale, scale_dev, (float *)out);
    else if (dtype == kBf16)
        column_total_kernel<__bf16><<<grid, 1024, 0, stream>>>(part, chunks, m, scale, scale_dev, (__bf16 *)out);
    else
        column_total_kernel<_Float16><<<grid, 1024, 0, stream>>>(part, chunks, m, scale, scale_dev, (_Float16 *)out);
    return hipGetLastError();
}

hipError_t zero_launch(int32_t dtype, void *p, int64_t ld, int64_t rows, int64_t cols, hipStream_t stream) {
    if (rows <= 0 || cols <= 0) return hipSuccess;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(rows * cols, 256), 4096);
    if (dtype == kF32) zero_kernel<float><<<grid, 256, 0, stream>>>((float *)p, ld, rows, cols);
    else zero_kernel<_Float16><<<grid, 256, 0, stream>>>((_Float16 *)p, ld, rows, cols);
    return hipGetLastError();
}

// ---- tile shape and splits ----------------------------------------------------
// A model of the time in nanoseconds: blocks run in rounds of as many as the
// 256 CUs hold, a block's tiles of k at the rate its shape reaches and a fixed
// part for its first loads and its results; splits add a launch and the
// writing and reading of their partial sums. The rates are those of products
// forced to each shape, 1 to 700,000 rows. For 5003 x 1021 x 2045 fp16 it picks 256 x 256
// (38 us; 44 with 128 x 128, 41 with 128 x 64), for dX of the same layer 128 x 64 (36 us).
namespace {
Cut cut_of(int32_t dtype, int64_t m, int64_t n, int64_t k, bool may_split) {
    // flops per ns of a CU with all its blocks, blocks a CU, ns of a block
    // besides its tiles of k
    struct Rate {
        double rate;
        int per_cu;
        double fixed;
    };
    static const Rate kBf[kShapeCount] = {{5000, 1, 9000}, {3900, 2, 5000}, {3000, 3, 4000}, {1100, 2, 2500}};
    static const Rate kFp32[kShapeCount] = {{850, 1, 26000}, {720, 2, 9000}, {650, 3, 5000}, {300, 2, 2500}};
    const int64_t bk = 128 / (int64_t)value_size(dtype), kt = ceil_div(k, bk);
    Cut best{0, 1, (int32_t)(kt * bk), 0};
    double best_ns = 1e300;
    for (int s = 0; s < kShapeCount; ++s) {
        const Rate &r = dtype == kF32 ? kFp32[s] : kBf[s];
        const int64_t tiles = ceil_div(m, kShapes[s].bm) * ceil_div(n, kShapes[s].bn);
        const int64_t slots = (int64_t)kCus * r.per_cu;
        const double step_ns = 2.0 * kShapes[s].bm * kShapes[s].bn * (double)bk * r.per_cu / r.rate;
        // as many splits as fill 1/4, 1/2, 1 or 2 rounds of blocks
        int64_t last = 0;
        for (int f = -3; f <= (may_split ? 1 : -3); ++f) {
            const int64_t fill = f < 0 ? slots >> -f : slots << f;
            const int64_t want = f == -3 ? 1 : std::min(kt, std::max<int64_t>(fill / tiles, 1));
            const int64_t per = ceil_div(kt, want), splits = ceil_div(kt, per);
            if (splits <= last) continue;
            last = splits;
            const int64_t blocks = tiles * splits, rounds = ceil_div(blocks, slots);
            // a CU that holds fewer blocks than it could runs each faster, a single one at most 1.6 times
            const double share = rounds > 1 ? (double)rounds
                                            : std::max((double)std::min<int64_t>(r.per_cu, ceil_div(blocks, kCus)) / r.per_cu,
                                                       r.per_cu > 1 ? 1.0 / 1.6 : 1.0);
            double ns = share * (double)per * step_ns + (double)rounds * r.fixed;
            if (splits > 1)
                ns += 2500.0 + 2.0 * 4.0 * (double)m * (double)n * (double)splits / 8000.0 + 25.0 * (double)splits;
            if (ns < best_ns) {
                best_ns = ns;
                best = Cut{s, (int32_t)splits, (int32_t)(per * bk), 0};
            }
        }
    }
    if (best.splits > 1)
        best.bytes = sizeof(float) * (size_t)best.splits * (size_t)m * (size_t)((n + 7) / 8 * 8);
    return best;
}
}  // namespace

Cut product_cut(int32_t dtype, int32_t layout, int64_t m, int64_t n, int64_t k) {
    if (layout == kRowsRows && m <= kFewRows) return Cut{kFewRowsShape, 1, 0, 0};
    return cut_of(dtype, m, n, k, true);
}

// the loss's products take every logit of a tile at once, so k is not split
int loss_shape(int32_t dtype, int64_t m, int64_t n, int64_t k) { return cut_of(dtype, m, n, k, false).shape; }

hipError_t product_launch(int32_t dtype, int32_t layout, Product p, Epilogue e, void *ws, hipStream_t stream) {
    if (p.m <= 0 || p.n <= 0) return hipSuccess;
    // results far beyond the L2s (32 MiB in all) only push the operands out of
    // them: 200,000 x 300 x 512 fp32 494 us, 445 with streaming stores; 232,964 x 256 x 600 560, 532
    e.stream = (double)p.m * p.n * (double)value_size(dtype) > 128.0 * 1024 * 1024;
    const Cut c = product_cut(dtype, layout, p.m, p.n, p.k);
    p.splits = c.splits;
    p.split_k = c.split_k;
    p.partial = (float *)ws;
    using F = hipError_t (*)(int, const Product &, const Epilogue &, hipStream_t);
    static const F kProducts[3][3] = {{product_f32_rr, product_f32_rc, product_f32_cc},
                                      {product_bf16_rr, product_bf16_rc, product_bf16_cc},
                                      {product_f16_rr, product_f16_rc, product_f16_cc}};
    return kProducts[dtype][layout](c.shape, p, e, stream);
}

// ---- layer ----------------------------------------------------------------------
size_t linear_ws_bytes(const Linear &l) {
    return align_up(product_cut(l.dtype, l.out_major ? kRowsRows : kRowsCols, l.n, l.m, l.k).bytes, 256);
}

hipError_t linear_launch(const Linear &l, const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias,
                         int32_t bias_f32, const void *r, int64_t ldr, void *y, int64_t ldy, float *pre, int64_t ldpre,
                         void *ws, hipStream_t stream) {
    Product p;
    p.a = x;
    p.lda = ldx;
    p.b = w;
    p.ldb = ldw;
    p.m = l.n;
    p.n = l.m;
    p.k = l.k;
    Epilogue e;
    e.alpha = l.alpha;
    e.beta = l.beta;
    e.bias = bias;
    e.bias_f32 = bias_f32;
    e.act = l.act;
    e.r = r;
    e.ldr = ldr;
    e.y = y;
    e.ldy = ldy;
    e.pre = pre;
    e.ldpre = ldpre;
    e.sure = l.sure;
    e.b_cols = !l.out_major;
    return product_launch(l.dtype, l.out_major ? kRowsRows : kRowsCols, p, e, ws, stream);
}

namespace {
// dz's place in the workspace: rows a whole number of 16 bytes apart
int64_t dz_ld(const Linear &l) { return (int64_t)align_up((size_t)l.m, 16 / value_size(l.dtype)); }
size_t dz_bytes(const Linear &l) {
    return l.act == kNone ? 0 : align_up((size_t)l.n * dz_ld(l) * value_size(l.dtype), 256);
}
size_t cut_bytes(const Linear &l, bool dx, bool dw) {
    size_t b = 0;
    if (dx) b = std::max(b, product_cut(l.dtype, l.out_major ? kRowsCols : kRowsRows, l.n, l.k, l.m).bytes);
    if (dw) b = std::max(b, l.out_major ? product_cut(l.dtype, kColsCols, l.m, l.k, l.n).bytes
                                        : product_cut(l.dtype, kColsCols, l.k, l.m, l.n).bytes);
    return align_up(b, 256);
}
}  // namespace

size_t linear_backward_ws_bytes(const Linear &l, bool dx, bool dw, bool db) {
    return dz_bytes(l) + (db ? column_sum_ws_bytes(l.n, l.m) : 0) + (l.n > 0 ? cut_bytes(l, dx, dw) : 0);
}

size_t column_sum_ws_bytes(int64_t n, int64_t m) {
    // chunks * m: at most 2,048 blocks of 64 groups of 8 columns, and a chunk
    // has 8 rows or more (the bound grows with m, so a narrower sum fits too)
    const int64_t most = std::max<int64_t>(m, std::min<int64_t>(2048 * 512, ceil_div(std::max<int64_t>(n, 1), 8) * m));
    return align_up(sizeof(double) * (size_t)most, 256);
}

hipError_t column_sum_launch(int32_t dtype, const void *a, int64_t lda, int64_t n, int64_t m, float scale,
                             const float *scale_dev, void *out, int32_t out_f32, void *ws, hipStream_t stream) {
    const Chunks c = chunks_of(dtype, n, m);
    Pass p{};
    p.dy = a;
    p.lddy = lda;
    p.part = (double *)ws;
    p.n = n;
    p.m = (int32_t)m;
    hipError_t e = pass_launch(dtype, p, c, stream);
    if (e == hipSuccess) e = column_total_launch(dtype, p.part, c.count, (int32_t)m, scale, scale_dev, out, out_f32, stream);
    return e;
}

hipError_t linear_backward_launch(const Linear &l, const void *dy, int64_t lddy, const void *saved, int64_t ldsaved,
                                  const void *x, int64_t ldx, const void *w, int64_t ldw, const LinearGrads &g,
                                  void *ws, hipStream_t stream) {
    char *at = (char *)ws;
    void *dz_ws = at;
    at += dz_bytes(l);
    double *part = (double *)at;
    if (g.db) at += column_sum_ws_bytes(l.n, l.m);
    hipError_t e = hipSuccess;
    if (l.n == 0) {  // no rows: the sums over them are zero
        if (g.dw) e = zero_launch(l.dtype, g.dw, g.lddw, l.out_major ? l.m : l.k, l.out_major ? l.k : l.m, stream);
        if (g.db && e == hipSuccess) e = zero_launch(g.db_f32 ? (int32_t)kF32 : l.dtype, g.db, l.m, 1, l.m, stream);
        return e;
    }
    const void *dz = dy;
    int64_t lddz = lddy;
    if (l.act != kNone || g.db || g.dr) {
        Pass p{};
        p.dy = dy;
        p.lddy = lddy;
        p.saved = saved;
        p.ldsaved = ldsaved;
        p.act = l.act;
        p.n = l.n;
        p.m = l.m;
        p.beta = l.beta;
        if (l.act != kNone && (g.dx || g.dw)) {
            // with beta = 1 the residual's gradient is dz itself
            const bool shared = g.dr && l.beta == 1.f;
            p.dz = shared ? g.dr : dz_ws;
            p.lddz = shared ? g.lddr : dz_ld(l);
            dz = p.dz;
            lddz = p.lddz;
        }
        if (g.dr && p.dz != g.dr) {
            p.dr = g.dr;
            p.lddr = g.lddr;
        }
        if (g.db) p.part = part;
        const Chunks c = chunks_of(l.dtype, l.n, l.m);
        e = pass_launch(l.dtype, p, c, stream);
        if (g.db && e == hipSuccess)
            e = column_total_launch(l.dtype, part, c.count, l.m, 1.f, nullptr, g.db, g.db_f32, stream);
    }
    if (g.dx && e == hipSuccess) {
        // dX = alpha dZ W^T
        Product p;
        p.a = dz;
        p.lda = lddz;
        p.b = w;
        p.ldb = ldw;
        p.m = l.n;
        p.n = l.k;
        p.k = l.m;
        Epilogue o;
        o.alpha = l.alpha;
        o.y = g.dx;
        o.ldy = g.lddx;
        e = product_launch(l.dtype, l.out_major ? kRowsCols : kRowsRows, p, o, at, stream);
    }
    if (g.dw && e == hipSuccess) {
        // dW = alpha X^T dZ, or its transpose where W is stored so
        Product p;
        p.a = l.out_major ? dz : x;
        p.lda = l.out_major ? lddz : ldx;
        p.b = l.out_major ? x : dz;
        p.ldb = l.out_major ? ldx : lddz;
        p.m = l.out_major ? l.m : l.k;
        p.n = l.out_major ? l.k : l.m;
        p.k = l.n;
        Epilogue o;
        o.alpha = l.alpha;
        o.y = g.dw;
        o.ldy = g.lddw;
        e = product_launch(l.dtype, kColsCols, p, o, at, stream);
    }
    return e;
}

}  // namespace rsc
