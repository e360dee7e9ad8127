// C ABI of the update phase (declared in include/rsc.h): argument checks in
// front of linear.hip, loss.hip and adamw.hip.
#include <cmath>

#include "adamw.h"
#include "api_checks.h"
#include "rsc.h"
#include "rsc_internal.h"
#include "update.h"

namespace {

using namespace rsc::api;

rsc_status_t check_dtype(int32_t dtype, const char *name) {
    if (dtype != RSC_F32 && dtype != RSC_BF16 && dtype != RSC_F16)
        return fail(RSC_ERR_INVALID_ARGUMENT, "%s = %d is no rsc_dtype_t", name, dtype);
    return RSC_OK;
}

// A rows x cols matrix of the update phase. The 4 MiB rows keep every byte
// offset inside a tile of 256 rows below 2^31.
rsc_status_t check_matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, const char *name) {
    const int64_t size = (int64_t)rsc::value_size(dtype);
    if (ld < cols) return fail(RSC_ERR_INVALID_ARGUMENT, "%s: ld %lld < %lld", name, (long long)ld, (long long)cols);
    if (ld > (int64_t(1) << 22) / size)
        return fail(RSC_ERR_UNSUPPORTED, "%s: rows of %lld values are over 4 MiB", name, (long long)ld);
    if (ld * size % 16 != 0)
        return fail(RSC_ERR_UNSUPPORTED, "%s: ld %lld is not a whole number of 16 bytes", name, (long long)ld);
    if (rows > 0 && !p) return fail(RSC_ERR_INVALID_ARGUMENT, "%s is NULL", name);
    if (!aligned(p, 16)) return fail(RSC_ERR_UNSUPPORTED, "%s is not 16-byte aligned", name);
    return RSC_OK;
}

rsc_status_t check_vector(const void *p, int32_t vec_dtype, int32_t dtype, const char *name) {
    if (!p) return RSC_OK;
    if (vec_dtype != RSC_F32 && vec_dtype != dtype)
        return fail(RSC_ERR_INVALID_ARGUMENT, "%s: dtype %d (the operands' or RSC_F32)", name, vec_dtype);
    if (!aligned(p, rsc::value_size(vec_dtype))) return fail(RSC_ERR_UNSUPPORTED, "%s is misaligned", name);
    return RSC_OK;
}

// Every shape's thread blocks then stay within 2^31 threads a launch, and row
// numbers, with the last tile's, within int32.
rsc_status_t check_tiles(int64_t a, int64_t b, const char *what) {
    if (rsc::ceil_div(a, 32) * rsc::ceil_div(b, 64) > (int64_t(1) << 24))
        return fail(RSC_ERR_UNSUPPORTED, "%s: a product of %lld x %lld", what, (long long)a, (long long)b);
    return RSC_OK;
}

rsc_status_t check_sizes(int32_t n, int32_t k, int32_t m, const char *what) {
    if (n < 0 || k < 1 || m < 1) return fail(RSC_ERR_INVALID_ARGUMENT, "%s: n = %d, k = %d, m or v = %d", what, n, k, m);
    RSC_TRY(check_tiles(n, m, what));
    RSC_TRY(check_tiles(n, k, what));
    RSC_TRY(check_tiles(m, n, what));
    RSC_TRY(check_tiles(k, n, what));
    RSC_TRY(check_tiles(k, m, what));
    return check_tiles(m, k, what);
}

// An operand or result in memory: rows of `cols` bytes, `pitch` bytes apart.
struct Area {
    const void *p;
    int64_t rows, cols, pitch;
    const char *name;
};
Area area(const void *p, int64_t rows, int64_t cols, int64_t ld, size_t size, const char *name) {
    return Area{p, rows, cols * (int64_t)size, ld * (int64_t)size, name};
}
Area line(const void *p, int64_t count, size_t size, const char *name) { return area(p, 1, count, count, size, name); }

// Do they share a byte? Rows of the same pitch may lie in each other's gaps
// (column ranges of one matrix); where pitches differ, ranges that meet count.
bool meet(Area a, Area b) {
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.cols <= 0 || b.cols <= 0) return false;
    const int64_t from_a = (int64_t)(uintptr_t)a.p, from_b = (int64_t)(uintptr_t)b.p;
    if (from_a + (a.rows - 1) * a.pitch + a.cols <= from_b || from_b + (b.rows - 1) * b.pitch + b.cols <= from_a)
        return false;
    if (a.rows == 1) a.pitch = b.pitch;
    if (b.rows == 1) b.pitch = a.pitch;
    if (a.pitch != b.pitch || (a.rows == 1 && b.rows == 1) || a.cols > a.pitch || b.cols > b.pitch) return true;
    const int64_t at = ((from_b - from_a) % a.pitch + a.pitch) % a.pitch;  // of b's rows in a's
    return at < a.cols || at + b.cols > a.pitch;
}

// No result lies on an operand or on another result.
template <int O, int I>
rsc_status_t check_apart(const Area (&outs)[O], const Area (&ins)[I], const char *what) {
    for (int i = 0; i < O; ++i) {
        for (int j = i + 1; j < O; ++j)
            if (meet(outs[i], outs[j]))
                return fail(RSC_ERR_INVALID_ARGUMENT, "%s: %s overlaps %s", what, outs[i].name, outs[j].name);
        for (const Area &in : ins)
            if (meet(outs[i], in))
                return fail(RSC_ERR_INVALID_ARGUMENT, "%s: %s overlaps %s", what, outs[i].name, in.name);
    }
    return RSC_OK;
}

rsc_status_t check_linear(const rsc_linear_t *p) {
    if (!p) return fail(RSC_ERR_INVALID_ARGUMENT, "the layer is NULL");
    RSC_TRY(check_dtype(p->dtype, "dtype"));
    if (p->act < RSC_ACT_NONE || p->act > RSC_ACT_SILU)
        return fail(RSC_ERR_INVALID_ARGUMENT, "act = %d is no rsc_act_t", p->act);
    return check_sizes(p->n, p->k, p->m, "linear");
}

rsc::Linear layer_of(const rsc_linear_t *p) {
    return rsc::Linear{p->dtype, p->act, p->n, p->k, p->m, p->w_out_major != 0, p->alpha, p->beta,
                       p->for_gradients != 0};
}

rsc_status_t check_xent(const rsc_xent_t *p) {
    if (!p) return fail(RSC_ERR_INVALID_ARGUMENT, "the loss is NULL");
    RSC_TRY(check_dtype(p->dtype, "dtype"));
    if (p->reduction < 0 || p->reduction > 2)
        return fail(RSC_ERR_INVALID_ARGUMENT, "reduction = %d (0, 1 or 2)", p->reduction);
    return check_sizes(p->n, p->k, p->v, "xent");
}

rsc::Loss loss_of(const rsc_xent_t *p) {
    return rsc::Loss{p->dtype, p->n, p->k, p->v, p->w_out_major != 0, p->reduction};
}

rsc_status_t check_xent_operands(const rsc_xent_t *p, const void *X, int64_t ldx, const void *W, int64_t ldw,
                                 const void *bias, const void *targets) {
    RSC_TRY(check_matrix(X, p->n, p->k, ldx, p->dtype, "X"));
    RSC_TRY(check_matrix(W, 1, p->w_out_major ? p->k : p->v, ldw, p->dtype, "W"));
    RSC_TRY(check_vector(bias, p->bias_dtype, p->dtype, "bias"));
    if (p->n > 0 && !targets) return fail(RSC_ERR_INVALID_ARGUMENT, "targets is NULL");
    if (!aligned(targets, p->targets_i32 ? 4 : 8)) return fail(RSC_ERR_UNSUPPORTED, "targets is misaligned");
    return RSC_OK;
}

Area xent_weights(const rsc_xent_t *p, const void *W, int64_t ldw) {
    const size_t size = rsc::value_size(p->dtype);
    return p->w_out_major ? area(W, p->v, p->k, ldw, size, "W") : area(W, p->k, p->v, ldw, size, "W");
}

rsc_status_t check_kept(const rsc_xent_t *p, const void *G, int64_t ldg) {
    if (p->v > rsc::kKeptClasses || p->reduction == 0)
        return fail(RSC_ERR_UNSUPPORTED, "G: %d classes (at most %d), reduction %d (1 or 2)", p->v, rsc::kKeptClasses,
                    p->reduction);
    return check_matrix(G, p->n, p->v, ldg, p->dtype, "G");
}

rsc::Classes classes_of(const rsc_xent_t *p, const void *bias, const void *targets) {
    rsc::Classes c;
    c.targets = targets;
    c.targets_i32 = p->targets_i32 != 0;
    c.ignore = p->ignore_index;
    c.bias = bias;
    c.bias_f32 = p->bias_dtype == RSC_F32;
    return c;
}

rsc_status_t check_scalar(const void *p, const char *name) {
    if (!p) return fail(RSC_ERR_INVALID_ARGUMENT, "%s is NULL", name);
    if (!aligned(p, 4)) return fail(RSC_ERR_UNSUPPORTED, "%s is not 4-byte aligned", name);
    return RSC_OK;
}

rsc_status_t check_moments(const rsc_adamw_tensor_t &t, int32_t i, bool codes) {
    if (t.n < 0) return fail(RSC_ERR_INVALID_ARGUMENT, "tensor %d: n = %lld < 0", i, (long long)t.n);
    if (t.n >= int64_t(1) << 34) return fail(RSC_ERR_UNSUPPORTED, "tensor %d: n = %lld", i, (long long)t.n);
    if (t.n == 0) return RSC_OK;
    if (!t.exp_avg || !t.exp_avg_sq || (codes && (!t.exp_avg_scale || !t.exp_avg_sq_scale)))
        return fail(RSC_ERR_INVALID_ARGUMENT, "tensor %d: a moment or its scale is NULL", i);
    if (!codes && (!aligned(t.exp_avg, 4) || !aligned(t.exp_avg_sq, 4)))
        return fail(RSC_ERR_UNSUPPORTED, "tensor %d: moments are not 4-byte aligned", i);
    if (codes && (!aligned(t.exp_avg_scale, 4) || !aligned(t.exp_avg_sq_scale, 4)))
        return fail(RSC_ERR_UNSUPPORTED, "tensor %d: scales are not 4-byte aligned", i);
    return RSC_OK;
}

}  // namespace

extern "C" {

size_t rsc_linear_workspace_bytes(const rsc_linear_t *p) {
    if (check_linear(p) != RSC_OK || p->n == 0) return 0;
    return rsc::linear_ws_bytes(layer_of(p));
}

rsc_status_t rsc_linear(const rsc_linear_t *p, const void *X, int64_t ldx, const void *W, int64_t ldw,
                        const void *bias, int32_t bias_dtype, const void *R, int64_t ldr, void *Y, int64_t ldy,
                        float *pre, int64_t ldpre, void *ws, size_t ws_bytes, hipStream_t stream) {
    RSC_TRY(check_linear(p));
    RSC_TRY(check_matrix(X, p->n, p->k, ldx, p->dtype, "X"));
    RSC_TRY(check_matrix(W, 1, p->w_out_major ? p->k : p->m, ldw, p->dtype, "W"));
    RSC_TRY(check_vector(bias, bias_dtype, p->dtype, "bias"));
    if (R) RSC_TRY(check_matrix(R, p->n, p->m, ldr, p->dtype, "R"));
    RSC_TRY(check_matrix(Y, p->n, p->m, ldy, p->dtype, "Y"));
    if (pre) RSC_TRY(check_matrix(pre, p->n, p->m, ldpre, RSC_F32, "pre"));
    if (p->n == 0) return RSC_OK;
    RSC_TRY(check_ws(ws, ws_bytes, rsc_linear_workspace_bytes(p), "linear"));
    const size_t size = rsc::value_size(p->dtype);
    const bool in_place = R == Y && (ldr == ldy || p->n == 1);
    const Area outs[] = {area(Y, p->n, p->m, ldy, size, "Y"), area(pre, p->n, p->m, ldpre, 4, "pre")};
    const Area ins[] = {area(X, p->n, p->k, ldx, size, "X"),
                        p->w_out_major ? area(W, p->m, p->k, ldw, size, "W") : area(W, p->k, p->m, ldw, size, "W"),
                        line(bias, p->m, rsc::value_size(bias_dtype), "bias"),
                        area(in_place ? nullptr : R, p->n, p->m, ldr, size, "R")};
    RSC_TRY(check_apart(outs, ins, "linear"));
    RSC_TRY(check_device());
    RSC_HIP(rsc::linear_launch(layer_of(p), X, ldx, W, ldw, bias, bias_dtype == RSC_F32, R, ldr, Y, ldy, pre, ldpre,
                               ws, stream),
            "linear launch");
    return RSC_OK;
}

size_t rsc_linear_backward_workspace_bytes(const rsc_linear_t *p, int32_t with_dx, int32_t with_dw,
                                           int32_t with_dbias) {
    if (check_linear(p) != RSC_OK) return 0;
    return rsc::linear_backward_ws_bytes(layer_of(p), with_dx != 0, with_dw != 0, with_dbias != 0);
}

rsc_status_t rsc_linear_backward(const rsc_linear_t *p, const void *dY, int64_t lddy, const void *saved,
                                 int64_t ldsaved, const void *X, int64_t ldx, const void *W, int64_t ldw, void *dX,
                                 int64_t lddx, void *dW, int64_t lddw, void *dbias, int32_t bias_dtype, void *dR,
                                 int64_t lddr, void *ws, size_t ws_bytes, hipStream_t stream) {
    RSC_TRY(check_linear(p));
    const int64_t w_rows = p->w_out_major ? p->m : p->k, w_cols = p->w_out_major ? p->k : p->m;
    RSC_TRY(check_matrix(dY, p->n, p->m, lddy, p->dtype, "dY"));
    if (p->act != RSC_ACT_NONE) RSC_TRY(check_matrix(saved, p->n, p->m, ldsaved, p->act == RSC_ACT_RELU ? p->dtype : RSC_F32, "saved"));
    if (dW) {
        RSC_TRY(check_matrix(X, p->n, p->k, ldx, p->dtype, "X"));
        RSC_TRY(check_matrix(dW, w_rows, w_cols, lddw, p->dtype, "dW"));
    }
    if (dX) {
        RSC_TRY(check_matrix(W, w_rows, w_cols, ldw, p->dtype, "W"));
        RSC_TRY(check_matrix(dX, p->n, p->k, lddx, p->dtype, "dX"));
    }
    RSC_TRY(check_vector(dbias, bias_dtype, p->dtype, "dbias"));
    if (dR) RSC_TRY(check_matrix(dR, p->n, p->m, lddr, p->dtype, "dR"));
    RSC_TRY(check_ws(ws, ws_bytes, rsc_linear_backward_workspace_bytes(p, dX != nullptr, dW != nullptr,
                                                                       dbias != nullptr),
                     "linear backward"));
    const size_t size = rsc::value_size(p->dtype);
    const Area outs[] = {area(dX, p->n, p->k, lddx, size, "dX"), area(dW, w_rows, w_cols, lddw, size, "dW"),
                         line(dbias, p->m, rsc::value_size(bias_dtype), "dbias"), area(dR, p->n, p->m, lddr, size, "dR")};
    const Area ins[] = {area(dY, p->n, p->m, lddy, size, "dY"),
                        area(p->act != RSC_ACT_NONE ? saved : nullptr, p->n, p->m, ldsaved,
                             p->act == RSC_ACT_RELU ? size : 4, "saved"),
                        area(dW ? X : nullptr, p->n, p->k, ldx, size, "X"),
                        area(dX ? W : nullptr, w_rows, w_cols, ldw, size, "W")};
    RSC_TRY(check_apart(outs, ins, "linear backward"));
    RSC_TRY(check_device());
    rsc::LinearGrads g;
    g.dx = dX;
    g.lddx = lddx;
    g.dw = dW;
    g.lddw = lddw;
    g.db = dbias;
    g.db_f32 = bias_dtype == RSC_F32;
    g.dr = dR;
    g.lddr = lddr;
    RSC_HIP(rsc::linear_backward_launch(layer_of(p), dY, lddy, saved, ldsaved, X, ldx, W, ldw, g, ws, stream),
            "linear backward launch");
    return RSC_OK;
}

size_t rsc_xent_workspace_bytes(const rsc_xent_t *p) {
    if (check_xent(p) != RSC_OK) return 0;
    return rsc::loss_ws_bytes(loss_of(p));
}

rsc_status_t rsc_xent(const rsc_xent_t *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const void *bias,
                      const void *targets, float *loss, float *lse, float *count, void *G, int64_t ldg, void *ws,
                      size_t ws_bytes, hipStream_t stream) {
    RSC_TRY(check_xent(p));
    RSC_TRY(check_xent_operands(p, X, ldx, W, ldw, bias, targets));
    if (p->n > 0 || p->reduction != 0) RSC_TRY(check_scalar(loss, "loss"));
    if (p->n > 0) RSC_TRY(check_scalar(lse, "lse"));
    if (p->reduction != 0) RSC_TRY(check_scalar(count, "count"));
    if (G) RSC_TRY(check_kept(p, G, ldg));
    RSC_TRY(check_ws(ws, ws_bytes, rsc_xent_workspace_bytes(p), "xent"));
    const size_t size = rsc::value_size(p->dtype);
    const Area outs[] = {line(loss, p->reduction == 0 ? p->n : 1, 4, "loss"), line(lse, p->n, 4, "lse"),
                         line(p->reduction == 0 ? nullptr : count, 1, 4, "count"), area(G, p->n, p->v, ldg, size, "G")};
    const Area ins[] = {area(X, p->n, p->k, ldx, size, "X"), xent_weights(p, W, ldw),
                        line(bias, p->v, rsc::value_size(p->bias_dtype), "bias"),
                        line(targets, p->n, p->targets_i32 ? 4 : 8, "targets")};
    RSC_TRY(check_apart(outs, ins, "xent"));
    RSC_TRY(check_device());
    rsc::Classes c = classes_of(p, bias, targets);
    c.grad = G;
    c.ldgrad = ldg;
    RSC_HIP(rsc::loss_launch(loss_of(p), X, ldx, W, ldw, c, loss, lse, count, ws, stream), "xent launch");
    return RSC_OK;
}

size_t rsc_xent_backward_workspace_bytes(const rsc_xent_t *p, int32_t with_dx, int32_t with_dw, int32_t with_g) {
    if (check_xent(p) != RSC_OK) return 0;
    return rsc::loss_backward_ws_bytes(loss_of(p), with_dx != 0, with_dw != 0, with_g != 0);
}

rsc_status_t rsc_xent_backward(const rsc_xent_t *p, const float *dloss, const void *X, int64_t ldx, const void *W,
                               int64_t ldw, const void *bias, const void *targets, const float *lse,
                               const float *count, const void *G, int64_t ldg, void *dX, int64_t lddx, void *dW,
                               int64_t lddw, void *dbias, void *ws, size_t ws_bytes, hipStream_t stream) {
    RSC_TRY(check_xent(p));
    RSC_TRY(check_xent_operands(p, X, ldx, W, ldw, bias, targets));
    if (p->n > 0 || p->reduction != 0) RSC_TRY(check_scalar(dloss, "dloss"));
    if (p->n > 0) RSC_TRY(check_scalar(lse, "lse"));
    if (p->reduction != 0) RSC_TRY(check_scalar(count, "count"));
    if (dX) RSC_TRY(check_matrix(dX, p->n, p->k, lddx, p->dtype, "dX"));
    if (dW)
        RSC_TRY(check_matrix(dW, p->w_out_major ? p->v : p->k, p->w_out_major ? p->k : p->v, lddw, p->dtype, "dW"));
    RSC_TRY(check_vector(dbias, p->bias_dtype, p->dtype, "dbias"));
    if (G) RSC_TRY(check_kept(p, G, ldg));
    RSC_TRY(check_ws(ws, ws_bytes,
                     rsc_xent_backward_workspace_bytes(p, dX != nullptr, dW != nullptr, G != nullptr),
                     "xent backward"));
    const size_t size = rsc::value_size(p->dtype);
    Area w_grad = xent_weights(p, dW, lddw);
    w_grad.name = "dW";
    const Area outs[] = {area(dX, p->n, p->k, lddx, size, "dX"), w_grad,
                         line(dbias, p->v, rsc::value_size(p->bias_dtype), "dbias")};
    const Area ins[] = {area(X, p->n, p->k, ldx, size, "X"), xent_weights(p, W, ldw),
                        line(bias, p->v, rsc::value_size(p->bias_dtype), "bias"),
                        line(targets, p->n, p->targets_i32 ? 4 : 8, "targets"),
                        line(dloss, p->reduction == 0 ? p->n : 1, 4, "dloss"), line(lse, p->n, 4, "lse"),
                        line(p->reduction == 0 ? nullptr : count, 1, 4, "count"), area(G, p->n, p->v, ldg, size, "G")};
    RSC_TRY(check_apart(outs, ins, "xent backward"));
    RSC_TRY(check_device());
    rsc::LossGrads g;
    g.dx = dX;
    g.lddx = lddx;
    g.dw = dW;
    g.lddw = lddw;
    g.db = dbias;
    g.db_f32 = p->bias_dtype == RSC_F32;
    rsc::Classes c = classes_of(p, bias, targets);
    c.lse = lse;
    c.grad = const_cast<void *>(G);  // (read only)
    c.ldgrad = ldg;
    RSC_HIP(rsc::loss_backward_launch(loss_of(p), dloss, X, ldx, W, ldw, c, count, g, G != nullptr, ws, stream),
            "xent backward launch");
    return RSC_OK;
}

size_t rsc_adamw_workspace_bytes(void) { return rsc::adamw_ws_bytes(); }

rsc_status_t rsc_adamw_step(const rsc_adamw_t *p, const rsc_adamw_tensor_t *tensors_host, int32_t count,
                            int64_t *step, void *ws, size_t ws_bytes, hipStream_t stream) {
    if (!p) return fail(RSC_ERR_INVALID_ARGUMENT, "the options are NULL");
    RSC_TRY(check_dtype(p->dtype, "dtype"));
    if (p->state_bits != 32 && p->state_bits != 8)
        return fail(RSC_ERR_INVALID_ARGUMENT, "state_bits = %d (32 or 8)", p->state_bits);
    if (!(p->beta1 >= 0 && p->beta1 < 1 && p->beta2 >= 0 && p->beta2 < 1 && p->eps >= 0) || !std::isfinite(p->lr) ||
        !std::isfinite(p->weight_decay) || !std::isfinite(p->eps))
        return fail(RSC_ERR_INVALID_ARGUMENT, "need 0 <= beta < 1, eps >= 0, finite lr and weight_decay");
    if (count < 0 || (count > 0 && !tensors_host)) return fail(RSC_ERR_INVALID_ARGUMENT, "tensors: count %d", count);
    if (!step) return fail(RSC_ERR_INVALID_ARGUMENT, "step is NULL");
    if (!aligned(step, 8)) return fail(RSC_ERR_UNSUPPORTED, "step is not 8-byte aligned");
    const bool codes = p->state_bits == 8;
    const size_t size = rsc::value_size(p->dtype);
    for (int32_t i = 0; i < count; ++i) {
        const rsc_adamw_tensor_t &t = tensors_host[i];
        RSC_TRY(check_moments(t, i, codes));
        if (t.n == 0) continue;
        if (!t.param || !t.grad) return fail(RSC_ERR_INVALID_ARGUMENT, "tensor %d: param or grad is NULL", i);
        if (!aligned(t.param, size) || !aligned(t.grad, size) || !aligned(t.master, 4))
            return fail(RSC_ERR_UNSUPPORTED, "tensor %d: param, grad or master is misaligned", i);
    }
    RSC_TRY(check_ws(ws, ws_bytes, rsc::adamw_ws_bytes(), "adamw"));
    RSC_TRY(check_device());
    rsc::AdamwRates a;
    a.lr = p->lr;
    a.beta1 = p->beta1;
    a.beta2 = p->beta2;
    a.b1 = (float)p->beta1;
    a.b2 = (float)p->beta2;
    a.c1 = (float)(1.0 - p->beta1);
    a.c2 = (float)(1.0 - p->beta2);
    a.keep = (float)(1.0 - p->lr * p->weight_decay);
    a.eps = (float)p->eps;
    a.seed = p->seed;
    RSC_HIP(rsc::adamw_launch(p->dtype, codes, tensors_host, count, a, step, ws, stream), "adamw launch");
    return RSC_OK;
}

rsc_status_t rsc_adamw_moments(const rsc_adamw_tensor_t *tensors_host, int32_t count,
                               float *const *exp_avg_out_host, float *const *exp_avg_sq_out_host,
                               hipStream_t stream) {
    if (count < 0 || (count > 0 && (!tensors_host || !exp_avg_out_host || !exp_avg_sq_out_host)))
        return fail(RSC_ERR_INVALID_ARGUMENT, "tensors: count %d", count);
    for (int32_t i = 0; i < count; ++i) {
        RSC_TRY(check_moments(tensors_host[i], i, true));
        if (tensors_host[i].n == 0) continue;
        RSC_TRY(check_scalar(exp_avg_out_host[i], "exp_avg_out"));
        RSC_TRY(check_scalar(exp_avg_sq_out_host[i], "exp_avg_sq_out"));
    }
    RSC_TRY(check_device());
    RSC_HIP(rsc::adamw_moments_launch(tensors_host, count, exp_avg_out_host, exp_avg_sq_out_host, stream),
            "adamw moments launch");
    return RSC_OK;
}

}  // extern "C"
