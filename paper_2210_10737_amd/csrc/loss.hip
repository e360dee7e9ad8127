// Softmax cross entropy of the logits X W + bias against one class a row, and
// its gradients, with the logits in tiles.
//
// Forward: one product whose epilogue keeps, for each row and tile of classes,
// the largest logit and the sum of exp(logit - largest); the tiles are joined
// row by row into lse = log sum exp, and loss = lse - own logit.
// Backward: the classes are taken in pieces; each piece's logits are computed
// again and leave as G = weight (exp(logit - lse) - [own class]) in the
// operands' type, from which dX += G W^T and dW = X^T G of the piece follow, and
// as its columns' sums from before that rounding, for db. Only one piece of G is
// ever held.
//
// G has no small factors in it (1/count, the upstream gradient): those go into
// the products' fp32 epilogues. fp16's G is scaled by 2^10 as well, so that
// probabilities down to 2^-34 are not lost. Gradients of single rows (reduction
// "none") may differ by any factor, too: under the largest one's scale a row 2^24
// times smaller would lose bits of its dX. So in fp16 each row is formed at a
// scale of its own, dX at that scale, and dX's and, for dW, G's rows are then taken to
// the common one by powers of two: exact, but for dX's own subnormal values, which
// are rounded twice, and for rows of G that are nothing beside the others in dW.
//
// Up to 64 classes (n x 64 values beside the n x k of X) the forward pass can
// leave G, since it has all of a row's logits in one tile: the backward pass then
// reads X once less (232,965 x 256 fp32, 41 classes: 92 us).
#include <cmath>

#include "rsc_internal.h"
#include "update.h"

namespace rsc {
namespace {

struct Rows {
    Classes c;
    int32_t n, v, tiles;
    float *loss_row;       // reduction 0: the rows' losses
    double *sum;           // per block: sum and count
    double *count;
};

// lse of each row from its tiles' statistics, and its loss. 256 / S rows a
// block, S threads a row.
template <int S>
__global__ __launch_bounds__(256) void rows_kernel(Rows a, float *lse_out) {
    constexpr int R = 256 / S;
    __shared__ float top[S][R], sum[S][R];
    const int r = threadIdx.x % R, s = threadIdx.x / R;
    const int m = blockIdx.x * R + r;
    float mx = -INFINITY, acc = 0.f;
    if (m < a.n) {
        for (int j = s; j < a.tiles; j += S) {
            const float2 v = a.c.stats[(int64_t)j * a.n + m];
            const float up = fmaxf(mx, v.x), base = up == -INFINITY ? 0.f : up;
            acc = acc * expf(mx - base) + v.y * expf(v.x - base);
            mx = up;
        }
    }
    top[s][r] = mx;
    sum[s][r] = acc;
    __syncthreads();
    double loss = 0.0, count = 0.0;
    if (s == 0 && m < a.n) {
        for (int i = 1; i < S; ++i) {
            const float x = top[i][r], up = fmaxf(mx, x), base = up == -INFINITY ? 0.f : up;
            acc = acc * expf(mx - base) + sum[i][r] * expf(x - base);
            mx = up;
        }
        const float lse = mx + logf(acc);
        lse_out[m] = lse;
        const int64_t t = a.c.targets_i32 ? (int64_t)((const int32_t *)a.c.targets)[m]
                                          : ((const int64_t *)a.c.targets)[m];
        float l = 0.f;
        if (t != a.c.ignore) {
            // a class outside 0 .. v-1 shows as NaN
            l = t >= 0 && t < a.v ? (mx - a.c.own_logit[m]) + logf(acc) : NAN;
            loss = (double)l;
            count = 1.0;
        }
        if (a.loss_row) a.loss_row[m] = l;
    }
    if (!a.sum) return;
    __shared__ double ls[R], lc[R];
    if (s == 0) {
        ls[r] = loss;
        lc[r] = count;
    }
    __syncthreads();
    for (int h = R / 2; h > 0; h /= 2) {
        if ((int)threadIdx.x < h) {
            ls[threadIdx.x] += ls[threadIdx.x + h];
            lc[threadIdx.x] += lc[threadIdx.x + h];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.sum[blockIdx.x] = ls[0];
        a.count[blockIdx.x] = lc[0];
    }
}

// loss = the blocks' sum (over the count of rows that are not left out, 0 if
// there is none); count = that count, at least 1, or 1 for a plain sum
__global__ __launch_bounds__(1024) void total_kernel(const double *sum, const double *count, int32_t blocks,
                                                     int32_t mean, float *loss, float *count_out) {
    __shared__ double a[1024], b[1024];
    double x = 0.0, y = 0.0;
    for (int i = threadIdx.x; i < blocks; i += 1024) {
        x += sum[i];
        y += count[i];
    }
    a[threadIdx.x] = x;
    b[threadIdx.x] = y;
    __syncthreads();
    for (int h = 512; h > 0; h /= 2) {
        if ((int)threadIdx.x < h) {
            a[threadIdx.x] += a[threadIdx.x + h];
            b[threadIdx.x] += b[threadIdx.x + h];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const double c = mean && b[0] > 1.0 ? b[0] : 1.0;
        if (loss) *loss = (float)(a[0] / c);
        if (count_out) *count_out = (float)c;
    }
}

// The scalar factor of all gradients: upstream / count, or for gradients of
// single rows a power of two near the largest of them (1 if that is 0 or not
// finite), by which the rows' weights are divided.
__global__ __launch_bounds__(1024) void factor_kernel(Classes c, const float *dloss, const float *count, int32_t n,
                                                      int32_t by_row, float *factor) {
    if (!by_row) {
        if (threadIdx.x == 0) *factor = *dloss / *count;
        return;
    }
    __shared__ float top[1024];
    float mx = 0.f;
    for (int m = threadIdx.x; m < n; m += 1024)
        if (c.target(m) != -1) mx = fmaxf(mx, fabsf(dloss[m]));
    top[threadIdx.x] = mx;
    __syncthreads();
    for (int h = 512; h > 0; h /= 2) {
        if ((int)threadIdx.x < h) top[threadIdx.x] = fmaxf(top[threadIdx.x], top[threadIdx.x + h]);
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        mx = top[0];
        *factor = mx > 0.f && mx <= 3.4e38f ? ldexpf(1.f, max(-120, min(120, ilogbf(mx)))) : 1.f;
    }
}

// A row's weight: 0 for one that is left out, NaN for a class out of range.
// row_scale (nullable): the row's own power of two, by which its weight is divided
// to 1/4 .. 1/2 in magnitude in place of the factor (non-finite ones stay).
__global__ __launch_bounds__(256) void weight_kernel(Classes c, const float *dloss, const float *factor, int32_t n,
                                                     int32_t v, int32_t by_row, float *weight, float *row_scale) {
    const int m = blockIdx.x * 256 + threadIdx.x;
    if (m >= n) return;
    const int64_t t = c.targets_i32 ? (int64_t)((const int32_t *)c.targets)[m] : ((const int64_t *)c.targets)[m];
    float by = by_row ? *factor : 1.f;
    if (row_scale) {
        const float up = fabsf(dloss[m]);
        by = up > 0.f && up <= 3.4e38f ? ldexpf(4.f, max(-120, min(120, ilogbf(up)))) : 1.f;
        row_scale[m] = by;
    }
    float w = 0.f;
    if (t != c.ignore) w = t >= 0 && t < v ? (by_row ? dloss[m] / by : 1.f) : NAN;
    weight[m] = w;
}

// Rows times powers of two: row_scale[m], over *over if that is given
__global__ __launch_bounds__(256) void scale_rows_kernel(_Float16 *p, int64_t ld, int32_t rows, int32_t cols,
                                                         const float *row_scale, const float *over) {
    const int64_t chunks = (cols + 7) / 8, step = (int64_t)gridDim.x * 256;
    typedef _Float16 vec __attribute__((ext_vector_type(8)));
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks * rows; i += step) {
        const int64_t m = i / chunks;
        const int c = (int)(i % chunks) * 8;
        const float by = over ? row_scale[m] / *over : row_scale[m];
        _Float16 *const at = p + m * ld + c;
        if (cols - c >= 8) {
            vec x = *(const vec *)at;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (_Float16)((float)x[j] * by);
            *(vec *)at = x;
        } else {
            for (int j = 0; j < cols - c; ++j) at[j] = (_Float16)((float)at[j] * by);
        }
    }
}
hipError_t scale_rows(void *p, int64_t ld, int32_t rows, int32_t cols, const float *row_scale, const float *over,
                      hipStream_t stream) {
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div((int64_t)rows * ((cols + 7) / 8), 256), 8192);
    scale_rows_kernel<<<grid, 256, 0, stream>>>((_Float16 *)p, ld, rows, cols, row_scale, over);
    return hipGetLastError();
}

constexpr size_t kPieceBytes = size_t(256) << 20;

// classes of a piece: a multiple of 256 such that G stays within 256 MiB, or
// 2,048 where that is more, and a row of G within 4 MiB; all pieces alike, since a
// small last one would leave most of the chip idle
int64_t piece_of(const Loss &l) {
    const int64_t row = (int64_t)std::max(l.n, 1) * (int64_t)value_size(l.dtype);
    const int64_t fit = (int64_t)kPieceBytes / row / 256 * 256;
    const int64_t most = std::min<int64_t>(std::max<int64_t>(fit, 2048), int64_t(1) << 20);
    if (l.v <= most) return l.v;
    return (int64_t)align_up((size_t)ceil_div(l.v, ceil_div(l.v, most)), 256);
}

float grad_scale(const Loss &l) { return l.dtype == kF16 ? 1024.f : 1.f; }

using StatsFn = hipError_t (*)(int, const Product &, const Classes &, hipStream_t);
StatsFn stats_fn(const Loss &l) {
    static const StatsFn f[3][2] = {{stats_f32_rc, stats_f32_rr}, {stats_bf16_rc, stats_bf16_rr}, {stats_f16_rc, stats_f16_rr}};
    return f[l.dtype][l.out_major ? 1 : 0];
}
StatsFn grad_fn(const Loss &l) {
    static const StatsFn f[3][2] = {{grad_f32_rc, grad_f32_rr}, {grad_bf16_rc, grad_bf16_rr}, {grad_f16_rc, grad_f16_rr}};
    return f[l.dtype][l.out_major ? 1 : 0];
}

int rows_split(int64_t tiles) { return tiles >= 4 ? 16 : 1; }

}  // namespace

size_t loss_ws_bytes(const Loss &l) {
    const int64_t n = std::max(l.n, 1), tiles = ceil_div(l.v, kShapes[loss_shape(l.dtype, l.n, l.v, l.k)].bn);
    return align_up(sizeof(float2) * (size_t)(tiles * n), 256) + align_up(sizeof(float) * (size_t)n, 256) +
           2 * align_up(sizeof(double) * (size_t)ceil_div(n, 256 / rows_split(tiles)), 256);
}

hipError_t loss_launch(const Loss &l, const void *x, int64_t ldx, const void *w, int64_t ldw, const Classes &classes,
                       float *loss, float *lse, float *count, void *ws, hipStream_t stream) {
    const int shape = loss_shape(l.dtype, l.n, l.v, l.k);
    const int64_t tiles = ceil_div(l.v, kShapes[shape].bn), n = std::max(l.n, 1);
    const int split = rows_split(tiles);
    const unsigned blocks = (unsigned)ceil_div(l.n, 256 / split);
    Classes c = classes;
    c.scale = grad_scale(l);
    char *at = (char *)ws;
    c.stats = (float2 *)at;
    at += align_up(sizeof(float2) * (size_t)(tiles * n), 256);
    c.own_logit = (float *)at;
    at += align_up(sizeof(float) * (size_t)n, 256);
    double *sum = (double *)at;
    at += align_up(sizeof(double) * (size_t)ceil_div(n, 256 / split), 256);
    double *cnt = (double *)at;
    Rows r{};
    if (l.n > 0) {
        Product p;
        p.a = x;
        p.lda = ldx;
        p.b = w;
        p.ldb = ldw;
        p.m = l.n;
        p.n = l.v;
        p.k = l.k;
        hipError_t e = stats_fn(l)(shape, p, c, stream);
        if (e != hipSuccess) return e;
        r.c = c;
        r.n = l.n;
        r.v = l.v;
        r.tiles = (int32_t)tiles;
        r.loss_row = l.reduction == 0 ? loss : nullptr;
        r.sum = l.reduction == 0 ? nullptr : sum;
        r.count = cnt;
        if (split == 16) rows_kernel<16><<<blocks, 256, 0, stream>>>(r, lse);
        else rows_kernel<1><<<blocks, 256, 0, stream>>>(r, lse);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (l.reduction != 0)
        total_kernel<<<1, 1024, 0, stream>>>(sum, cnt, (int32_t)blocks, l.reduction == 2, loss, count);
    return hipGetLastError();
}

namespace {
size_t piece_cuts(const Loss &l, bool dx, bool dw) {
    // over the two widths that pieces have: the full one and the last one's
    const int64_t piece = piece_of(l), rest = l.v % piece;
    size_t b = 0;
    for (int64_t v : {piece, rest}) {
        if (v == 0) continue;
        if (dx) b = std::max(b, product_cut(l.dtype, l.out_major ? kRowsCols : kRowsRows, l.n, l.k, v).bytes);
        if (dw) b = std::max(b, l.out_major ? product_cut(l.dtype, kColsCols, v, l.k, l.n).bytes
                                            : product_cut(l.dtype, kColsCols, l.k, v, l.n).bytes);
    }
    return align_up(b, 256);
}
// the columns' partial sums: of each row of tiles where the gradient pass forms
// G, of column_sum_launch's chunks where G is given
size_t sums_bytes(const Loss &l, bool kept) {
    const int64_t piece = piece_of(l), rest = l.v % piece;
    if (kept) return column_sum_ws_bytes(l.n, piece);
    size_t b = 0;
    for (int64_t v : {piece, rest})
        if (v > 0) b = std::max(b, sizeof(double) * (size_t)(v * ceil_div(l.n, kShapes[loss_shape(l.dtype, l.n, v, l.k)].bm)));
    return align_up(b, 256);
}
// do rows have scales of their own?
bool own_scales(const Loss &l, bool dx) { return dx && l.dtype == kF16 && l.reduction == 0; }
int64_t grad_ld(const Loss &l) { return (int64_t)align_up((size_t)piece_of(l), 16 / value_size(l.dtype)); }
int64_t acc_ld(const Loss &l) { return (int64_t)align_up((size_t)l.k, 4); }
}  // namespace

size_t loss_backward_ws_bytes(const Loss &l, bool dx, bool dw, bool kept) {
    if (l.n == 0) return 256;
    size_t b = 256 + sums_bytes(l, kept) + piece_cuts(l, dx, dw);
    if (!kept)
        b += align_up((size_t)l.n * grad_ld(l) * value_size(l.dtype), 256) + align_up(sizeof(float) * (size_t)l.n, 256);
    if (dx && piece_of(l) < l.v) b += align_up(sizeof(float) * (size_t)l.n * acc_ld(l), 256);
    if (own_scales(l, dx)) b += align_up(sizeof(float) * (size_t)l.n, 256);
    return b;
}

hipError_t loss_backward_launch(const Loss &l, const float *dloss, const void *x, int64_t ldx, const void *w,
                                int64_t ldw, Classes c, const float *count, const LossGrads &g, bool kept,
                                void *ws, hipStream_t stream) {
    hipError_t e = hipSuccess;
    const int32_t db_type = g.db_f32 ? (int32_t)kF32 : l.dtype;
    if (l.n == 0) {
        if (g.dw) e = zero_launch(l.dtype, g.dw, g.lddw, l.out_major ? l.v : l.k, l.out_major ? l.k : l.v, stream);
        if (g.db && e == hipSuccess) e = zero_launch(db_type, g.db, l.v, 1, l.v, stream);
        return e;
    }
    const int64_t piece = piece_of(l), es = (int64_t)value_size(l.dtype);
    char *at = (char *)ws;
    float *weight = nullptr;
    if (!kept) {
        c.grad = at;
        c.ldgrad = grad_ld(l);
        at += align_up((size_t)l.n * c.ldgrad * es, 256);
        weight = (float *)at;
        at += align_up(sizeof(float) * (size_t)l.n, 256);
    }
    float *factor = (float *)at;
    at += 256;
    void *sums = at;
    at += sums_bytes(l, kept);
    float *acc = nullptr;
    if (g.dx && piece < l.v) {
        acc = (float *)at;
        at += align_up(sizeof(float) * (size_t)l.n * acc_ld(l), 256);
    }
    float *row_scale = nullptr;
    if (own_scales(l, g.dx != nullptr)) {
        row_scale = (float *)at;
        at += align_up(sizeof(float) * (size_t)l.n, 256);
    }
    void *cut = at;
    factor_kernel<<<1, 1024, 0, stream>>>(c, dloss, count, l.n, l.reduction == 0, factor);
    if (!kept)
        weight_kernel<<<(unsigned)ceil_div(l.n, 256), 256, 0, stream>>>(c, dloss, factor, l.n, l.v, l.reduction == 0,
                                                                        weight, row_scale);
    e = hipGetLastError();
    c.weight = weight;
    c.scale = grad_scale(l) * (row_scale ? 4.f : 1.f);
    c.row_scale = row_scale;
    c.over = factor;
    c.sums = g.db && !kept ? (double *)sums : nullptr;
    const void *bias = c.bias;
    for (int64_t v0 = 0; v0 < l.v && e == hipSuccess; v0 += piece) {
        const int32_t vc = (int32_t)std::min(piece, l.v - v0);
        const char *wp = (const char *)w + (l.out_major ? v0 * ldw : v0) * es;
        c.first = v0;
        c.bias = bias ? (const char *)bias + v0 * (c.bias_f32 ? 4 : es) : nullptr;
        Product p;
        p.a = x;
        p.lda = ldx;
        p.b = wp;
        p.ldb = ldw;
        p.m = l.n;
        p.n = vc;
        p.k = l.k;
        const int shape = loss_shape(l.dtype, l.n, vc, l.k);
        if (!kept) e = grad_fn(l)(shape, p, c, stream);
        if (g.dx && e == hipSuccess) {
            Product q;
            q.a = c.grad;
            q.lda = c.ldgrad;
            q.b = wp;
            q.ldb = ldw;
            q.m = l.n;
            q.n = l.k;
            q.k = vc;
            const bool last = v0 + vc >= l.v;
            Epilogue o;
            o.alpha = 1.f / c.scale;
            o.alpha_dev = row_scale ? nullptr : factor;
            if (v0 > 0) {
                o.r = acc;
                o.ldr = acc_ld(l);
                o.r_f32 = 1;
            }
            o.y = last ? g.dx : (void *)acc;
            o.ldy = last ? g.lddx : acc_ld(l);
            o.y_f32 = last ? 0 : 1;
            e = product_launch(l.dtype, l.out_major ? kRowsCols : kRowsRows, q, o, cut, stream);
            if (row_scale && last && e == hipSuccess) e = scale_rows(g.dx, g.lddx, l.n, l.k, row_scale, nullptr, stream);
        }
        if (row_scale && g.dw && e == hipSuccess) e = scale_rows(c.grad, c.ldgrad, l.n, vc, row_scale, factor, stream);
        if (g.dw && e == hipSuccess) {
            Product q;
            q.a = l.out_major ? c.grad : x;
            q.lda = l.out_major ? c.ldgrad : ldx;
            q.b = l.out_major ? x : c.grad;
            q.ldb = l.out_major ? ldx : c.ldgrad;
            q.m = l.out_major ? vc : l.k;
            q.n = l.out_major ? l.k : vc;
            q.k = l.n;
            Epilogue o;
            o.alpha = 1.f / c.scale;
            o.alpha_dev = factor;
            o.y = (char *)g.dw + (l.out_major ? v0 * g.lddw : v0) * es;
            o.ldy = g.lddw;
            e = product_launch(l.dtype, kColsCols, q, o, cut, stream);
        }
        if (g.db && e == hipSuccess) {
            void *const db = (char *)g.db + v0 * (g.db_f32 ? 4 : es);
            if (kept)
                e = column_sum_launch(l.dtype, c.grad, c.ldgrad, l.n, vc, 1.f / c.scale, factor, db, g.db_f32, sums, stream);
            else
                e = column_total_launch(l.dtype, c.sums, (int32_t)ceil_div(l.n, kShapes[shape].bm), vc, 1.f / c.scale,
                                        factor, db, g.db_f32, stream);
        }
    }
    return e;
}

}  // namespace rsc
