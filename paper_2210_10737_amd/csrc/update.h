// The update phase's kernels: layer products, class loss, optimizer step.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rsc {

enum : int32_t { kF32 = 0, kBf16 = 1, kF16 = 2 };           // rsc_dtype_t
enum : int32_t { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };  // rsc_act_t
enum : int32_t { kRowsRows = 0, kRowsCols = 1, kColsCols = 2 };  // operand storage of a product (A, B)

// C[m][n] = sum_k A(m, k) B(k, n); leading dimensions in values
struct Product {
    const void *a = nullptr, *b = nullptr;
    int64_t lda = 0, ldb = 0;
    int32_t m = 0, n = 0, k = 0;
    // the launch's own: k is cut into `splits` ranges of split_k values, a
    // multiple of every shape's tile
    int32_t splits = 1, split_k = 0;
    float *partial = nullptr;
};

// y = act(alpha alpha_dev acc + bias + beta r); alpha_dev, bias, r, pre (the
// value before act) nullable
struct Epilogue {
    float alpha = 1.f, beta = 1.f;
    const float *alpha_dev = nullptr;
    const void *bias = nullptr;
    int32_t bias_f32 = 0;
    int32_t act = kNone;
    const void *r = nullptr;
    int64_t ldr = 0;
    int32_t r_f32 = 0;
    int32_t y_f32 = 0;
    void *y = nullptr;
    int64_t ldy = 0;
    float *pre = nullptr;
    int64_t ldpre = 0;
    // results go past the caches (set by the launch for large ones)
    bool stream = false;
    // ReLU: signs next to zero are decided in 64 bits; B's storage then
    bool sure = false;
    int32_t b_cols = 0;
};

// What the loss's products need besides X and W
struct Classes {
    const void *targets = nullptr;  // int64 or int32
    int32_t targets_i32 = 0;
    int64_t ignore = 0;
    const void *bias = nullptr;
    int32_t bias_f32 = 0;
    // statistics pass: (largest, sum of exp) of row m over tile j of classes at
    // stats[j * rows + m]; the logit of the row's own class
    float2 *stats = nullptr;
    float *own_logit = nullptr;
    // gradient pass, and the statistics pass where it leaves the gradient too
    const float *lse = nullptr, *weight = nullptr;
    float scale = 1.f;
    int64_t first = 0;  // the piece's first class
    void *grad = nullptr;
    int64_t ldgrad = 0;
    // fp16, nullable: what the rows' weights are divided by, and the factor that the
    // columns' sums are under
    const float *row_scale = nullptr, *over = nullptr;
    double *sums = nullptr;  // gradient pass, nullable: each row of tiles' column sums, the piece's width apart

    __device__ __forceinline__ int64_t raw(int m) const {
        return targets_i32 ? (int64_t)((const int32_t *)targets)[m] : ((const int64_t *)targets)[m];
    }
    __device__ __forceinline__ bool left_out(int m) const { return raw(m) == ignore; }
    // the row's class; -1 for a row that is left out
    __device__ __forceinline__ int64_t target(int m) const { return left_out(m) ? -1 : raw(m); }
};

// ---- products (gemm_*.hip) ----------------------------------------------------
// shape: an index into kShapes
struct Shape {
    int32_t bm, bn;
};
constexpr Shape kShapes[] = {{256, 256}, {128, 128}, {128, 64}, {32, 128}};
constexpr int kShapeCount = 4;
// a kernel of its own: up to this many rows against weights stored by rows
constexpr int kFewRowsShape = 4, kFewRows = 2;

#define RSC_PRODUCT_DECL(name)                                                                       \
    hipError_t product_##name(int shape, const Product &p, const Epilogue &e, hipStream_t stream);
#define RSC_CLASSES_DECL(name)                                                                       \
    hipError_t stats_##name(int shape, const Product &p, const Classes &c, hipStream_t stream);      \
    hipError_t grad_##name(int shape, const Product &p, const Classes &c, hipStream_t stream);
RSC_PRODUCT_DECL(f32_rr) RSC_PRODUCT_DECL(f32_rc) RSC_PRODUCT_DECL(f32_cc)
RSC_PRODUCT_DECL(bf16_rr) RSC_PRODUCT_DECL(bf16_rc) RSC_PRODUCT_DECL(bf16_cc)
RSC_PRODUCT_DECL(f16_rr) RSC_PRODUCT_DECL(f16_rc) RSC_PRODUCT_DECL(f16_cc)
RSC_CLASSES_DECL(f32_rr) RSC_CLASSES_DECL(f32_rc)
RSC_CLASSES_DECL(bf16_rr) RSC_CLASSES_DECL(bf16_rc)
RSC_CLASSES_DECL(f16_rr) RSC_CLASSES_DECL(f16_rc)
#undef RSC_PRODUCT_DECL
#undef RSC_CLASSES_DECL

// Tile shape and number of splits for a product of this size, and the bytes of
// partial sums that the splits take (0 for one)
struct Cut {
    int32_t shape, splits, split_k;
    size_t bytes;
};
Cut product_cut(int32_t dtype, int32_t layout, int64_t m, int64_t n, int64_t k);
int loss_shape(int32_t dtype, int64_t m, int64_t n, int64_t k);
// runs it; ws holds the cut's bytes
hipError_t product_launch(int32_t dtype, int32_t layout, Product p, Epilogue e, void *ws, hipStream_t stream);

inline size_t value_size(int32_t dtype) { return dtype == kF32 ? 4 : 2; }

// ---- layer (linear.hip) ----------------------------------------------------------
struct Linear {
    int32_t dtype, act, n, k, m, out_major;
    float alpha, beta;
    bool sure;  // forward: Y is kept for the backward pass
};
size_t linear_ws_bytes(const Linear &l);
size_t linear_backward_ws_bytes(const Linear &l, bool dx, bool dw, bool db);
hipError_t linear_launch(const Linear &l, const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias,
                         int32_t bias_f32, const void *r, int64_t ldr, void *y, int64_t ldy, float *pre, int64_t ldpre,
                         void *ws, hipStream_t stream);
struct LinearGrads {
    void *dx = nullptr, *dw = nullptr, *db = nullptr, *dr = nullptr;
    int64_t lddx = 0, lddw = 0, lddr = 0;
    int32_t db_f32 = 0;
};
hipError_t linear_backward_launch(const Linear &l, const void *dy, int64_t lddy, const void *saved, int64_t ldsaved,
                                  const void *x, int64_t ldx, const void *w, int64_t ldw, const LinearGrads &g,
                                  void *ws, hipStream_t stream);
// out[j] = scale * scale_dev * sum over rows of a[i][j] (fp32 sums in one fixed order); scale_dev nullable
size_t column_sum_ws_bytes(int64_t n, int64_t m);
// out[j] = scale * scale_dev * the sum of part[i * m + j] over the chunks
hipError_t column_total_launch(int32_t dtype, const double *part, int32_t chunks, int32_t m, float scale,
                               const float *scale_dev, void *out, int32_t out_f32, hipStream_t stream);
hipError_t zero_launch(int32_t dtype, void *p, int64_t ld, int64_t rows, int64_t cols, hipStream_t stream);
hipError_t column_sum_launch(int32_t dtype, const void *a, int64_t lda, int64_t n, int64_t m, float scale,
                             const float *scale_dev, void *out, int32_t out_f32, void *ws, hipStream_t stream);

// ---- class loss (loss.hip) ---------------------------------------------------------
struct Loss {
    int32_t dtype, n, k, v, out_major, reduction;  // reduction: 0 none, 1 sum, 2 mean
};
// up to this many classes the statistics pass can leave the logits' gradient
// (they are one tile of every shape)
constexpr int kKeptClasses = 64;
size_t loss_ws_bytes(const Loss &l);
// kept: the gradient that the statistics pass left is given
size_t loss_backward_ws_bytes(const Loss &l, bool dx, bool dw, bool kept);
hipError_t loss_launch(const Loss &l, const void *x, int64_t ldx, const void *w, int64_t ldw, const Classes &c,
                       float *loss, float *lse, float *count, void *ws, hipStream_t stream);
struct LossGrads {
    void *dx = nullptr, *dw = nullptr, *db = nullptr;
    int64_t lddx = 0, lddw = 0;
    int32_t db_f32 = 0;
};
hipError_t loss_backward_launch(const Loss &l, const float *dloss, const void *x, int64_t ldx, const void *w,
                                int64_t ldw, Classes c, const float *count, const LossGrads &g, bool kept,
                                void *ws, hipStream_t stream);

}  // namespace rsc
