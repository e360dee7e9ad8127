// Matrix product of the update phase: C = A B with an epilogue, for row-major
// fp32, bf16 and fp16 operands of any size, sums in fp32.
//
//   C[m][n] = sum_k A(m, k) B(k, n)
//
// A is stored [m][k] (kRows: a row's k values lie together) or [k][m]
// (kCols); B is stored [n][k] (kRows) or [k][n] (kCols). The products of a
// layer need (rows, rows) and (rows, cols) for Y = X W and dX = dZ W^T, and
// (cols, cols) for dW = X^T dZ.
//
// One block computes a BM x BN tile with WM x WN waves, each a grid of 32x32
// matrix-core tiles. The operands' tiles are BK = 128 bytes of k deep and go
// from memory to LDS directly (16 bytes a lane, through buffer descriptors
// that return zero past a matrix's end), double-buffered: the next tile is in
// flight while the waves work on the present one.
//
// LDS layouts, both free of bank conflicts:
//   kRows: 128 bytes a row, its eight 16-byte chunks at chunk ^ (row & 7); a
//     lane reads its eight k values by one (fp32: two) 16-byte reads.
//   kCols: BK rows of BM (BN) values as they lie in memory, chunks XORed with
//     a few bits of k; 16-bit fragments come by the transposing LDS read
//     (ds_read_b64_tr_b16), fp32 ones by eight 4-byte reads.
//
// The matrix instruction is fed (B, A), so that a lane holds one row m and
// four consecutive columns n per register quad: stores and row sums are along
// n.
//
// fp32 operands: the fp32 matrix instruction runs at 1/16 of the bf16 one, so
// each value is split into three bf16 parts (x = hi + mid + lo, exact for
// normal values below bf16's largest) and the six products whose weight is at least 2^-16
// of the first are summed in fp32, the smallest first; the three left out are
// below 2^-25 relative, under fp32's own rounding. An infinite operand gives
// NaN (inf - inf in the split).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "rsc_internal.h"
#include "update.h"

namespace rsc {
namespace gemm {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr uint32_t kOutside = 0x80000000u;  // past every descriptor's range

// 16 bytes a lane from the descriptor's buffer to 64 consecutive places in LDS.
// Written as assembly since the compiler waits for a load to LDS that it knows
// of before the next LDS read, whichever buffer that is for; the load has no
// register result, and wait_loads() stands before the barrier that hands a
// buffer over. (m0, the place in LDS, is a reserved register: the compiler
// keeps nothing in it, and no other instruction of these kernels reads it.)
__device__ __forceinline__ void load_to_lds(v4i rsrc, uint32_t lds, uint32_t off, uint32_t soff) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 4\n\t"
        "buffer_load_dwordx4 %1, %2, %3 offen lds"
        :
        : "s"(lds), "v"(off), "s"(rsrc), "s"(soff)
        : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <typename T>
struct Type;
template <>
struct Type<float> {
    using frag = float __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Type<__bf16> {
    using frag = v8bf;
    static __device__ __forceinline__ float get(__bf16 v) { return (float)v; }
    static __device__ __forceinline__ __bf16 put(float v) { return (__bf16)v; }
};
template <>
struct Type<_Float16> {
    using frag = v8h;
    static __device__ __forceinline__ float get(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 put(float v) { return (_Float16)v; }
};

// ---- one operand's tile: R rows (or columns) by 128 bytes of k -------------
template <typename T, bool COLS, int R, int WAVES>
struct Operand {
    static constexpr int ES = (int)sizeof(T);
    static constexpr int BK = 128 / ES;
    static constexpr int CH = 16 / ES;              // values a chunk
    static constexpr int BYTES = R * 128;
    static constexpr int N = BYTES / 1024 / WAVES;  // loads of a wave
    static_assert(BYTES % (1024 * WAVES) == 0, "whole wave loads");
    static constexpr int CPR = COLS ? R / CH : 8;   // chunks an LDS row

    // XOR of a chunk's place in LDS row k of the kCols form: 16 bits: four
    // rows of one transposing read fall into four 64-byte bank groups; fp32:
    // the two half-waves, eight rows apart, into two 128-byte ones
    static __device__ __forceinline__ int swizzle(int k) {
        if (ES == 2) return CPR >= 16 ? (k & 3) << 2 : CPR == 8 ? ((k >> 1) & 1) << 2 : 0;
        return CPR >= 16 ? ((k >> 3) & 1) << 3 : 0;
    }

    const char *base;       // of the tile's first row (kRows) or column (kCols)
    int64_t bytes;          // from base to the end of the matrix
    int64_t step;           // kCols: bytes from one k tile to the next
    uint32_t off[N];        // a lane's byte offsets in its loads
    int k_at;               // kRows: k of a lane's chunk within the tile, the same in all its loads

    __device__ __forceinline__ void init(const void *p, int64_t ld, int first, int count, int K, int wave, int lane) {
        const int64_t ldb = ld * ES;
        if (COLS) {
            base = (const char *)p + (int64_t)first * ES;
            bytes = ((int64_t)(K - 1) * ldb + (int64_t)(count - first) * ES + 15) & ~(int64_t)15;
            step = (int64_t)BK * ldb;
        } else {
            base = (const char *)p + (int64_t)first * ldb;
            bytes = ((int64_t)(count - first - 1) * ldb + (int64_t)K * ES + 15) & ~(int64_t)15;
            step = 0;
        }
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int lin = (q * WAVES + wave) * 64 + lane;
            const int row = lin / CPR, slot = lin % CPR;
            if (COLS)
                off[q] = (uint32_t)(row * ldb) + (uint32_t)((slot ^ swizzle(row)) * 16);
            else
                off[q] = (uint32_t)(row * ldb) + (uint32_t)((slot ^ (row & 7)) * 16);
        }
        k_at = COLS ? 0 : ((lane & 7) ^ ((lane >> 3) & 7)) * CH;
    }

    // tile t's loads into LDS at `to`; last: it holds K's end
    __device__ __forceinline__ void load(char *to, int t, int K, bool last, int wave) const {
        const char *from = base;
        int64_t left = bytes;
        uint32_t so = 0;
        if (COLS) {
            from += t * step;
            left -= t * step;
        } else {
            so = (uint32_t)t * 128u;
        }
        const uint32_t n = left <= 0 ? 0u : (uint32_t)(left < (int64_t)0x7ffffff0 ? left : (int64_t)0x7ffffff0);
        const uint64_t at = (uint64_t)from;
        const v4i rs = {(int)(uint32_t)at, (int)(uint32_t)((at >> 32) & 0xffffu), (int)n, 0x00027000};
        const bool outside = !COLS && last && t * BK + k_at >= K;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const uint32_t o = outside ? kOutside : off[q];
            load_to_lds(rs, (uint32_t)(uintptr_t)(lds_void *)(to + (q * WAVES + wave) * 1024), o, so);
        }
    }

    // kRows, the tile that ends inside a chunk: zeroes that chunk's values from
    // k = kn on (they hold what lies behind K in memory)
    static __device__ __forceinline__ void clear_tail(char *at, int kn, int threads) {
        if (COLS) return;
        for (int row = threadIdx.x; row < R; row += threads) {
            T *chunk = (T *)(at + row * 128 + (((kn / CH) ^ (row & 7)) * 16));
            for (int j = kn % CH; j < CH; ++j) chunk[j] = (T)0.f;
        }
    }

    // the fragment of 32 rows from `r0`, k = 16 s .. 16 s + 15 of the tile:
    // lane l has row r0 + l % 32, k = 16 s + 8 (l / 32) + 0..7
    static __device__ __forceinline__ typename Type<T>::frag frag(const char *at, int r0, int s, int lane) {
        typename Type<T>::frag f;
        if constexpr (ES == 2) {
            if constexpr (COLS) {
                const int i = lane & 15, g = lane >> 4;
                const int k = 16 * s + 8 * (g >> 1) + (i >> 2);
                const int c = (r0 + (g & 1) * 16) / 8 + ((i & 3) >> 1);
                const int sub = (i & 1) * 8;
                const char *p0 = at + k * (R * ES) + ((c ^ swizzle(k)) * 16) + sub;
                const char *p1 = at + (k + 4) * (R * ES) + ((c ^ swizzle(k + 4)) * 16) + sub;
                v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)p0);
                v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)p1);
                const v8s v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
                f = __builtin_bit_cast(typename Type<T>::frag, v);
            } else {
                const int row = r0 + (lane & 31), c = 2 * s + (lane >> 5);
                f = *(const typename Type<T>::frag *)(at + row * 128 + ((c ^ (row & 7)) * 16));
            }
        } else {
            if constexpr (COLS) {
                const int row = r0 + (lane & 31);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = 16 * s + 8 * (lane >> 5) + j;
                    f[j] = *(const float *)(at + k * (R * ES) + (((row >> 2) ^ swizzle(k)) * 16) + (row & 3) * 4);
                }
            } else {
                const int row = r0 + (lane & 31), c = 4 * s + 2 * (lane >> 5);
                const v4f a = *(const v4f *)(at + row * 128 + ((c ^ (row & 7)) * 16));
                const v4f b = *(const v4f *)(at + row * 128 + (((c + 1) ^ (row & 7)) * 16));
                f = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        }
        return f;
    }
};

__device__ __forceinline__ v16f mfma(v8bf a, v8bf b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v16f mfma(v8h a, v8h b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// x = part[0] + part[1] + part[2]
struct Split {
    v8bf part[3];
    __device__ __forceinline__ explicit Split(Type<float>::frag x) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = x[j];
            const __bf16 h = (__bf16)v;
            v -= (float)h;
            const __bf16 m = (__bf16)v;
            v -= (float)m;
            part[0][j] = h;
            part[1][j] = m;
            part[2][j] = (__bf16)v;
        }
    }
};

// ---- the work of one block ------------------------------------------------
template <typename T, bool AC, bool BC, int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int WAVES = WM * WN;
    static constexpr int THREADS = 64 * WAVES;
    static constexpr int TA = BM / WM / 32, TB = BN / WN / 32;
    using A = Operand<T, AC, BM, WAVES>;
    using B = Operand<T, BC, BN, WAVES>;
    static constexpr int BK = A::BK;
    static constexpr int LDS = 2 * (A::BYTES + B::BYTES);

    static __device__ __forceinline__ void compute(v16f (&acc)[TA][TB], const char *sa, const char *sb, int wm, int wn,
                                                   int lane) {
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            if constexpr (sizeof(T) == 2) {
                typename Type<T>::frag a[TA], b[TB];
#pragma unroll
                for (int i = 0; i < TA; ++i) a[i] = A::frag(sa, (wm * TA + i) * 32, s, lane);
#pragma unroll
                for (int j = 0; j < TB; ++j) b[j] = B::frag(sb, (wn * TB + j) * 32, s, lane);
#pragma unroll
                for (int i = 0; i < TA; ++i)
#pragma unroll
                    for (int j = 0; j < TB; ++j) acc[i][j] = mfma(b[j], a[i], acc[i][j]);
            } else {
                v8bf b[TB][3];
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    const Split v(B::frag(sb, (wn * TB + j) * 32, s, lane));
#pragma unroll
                    for (int u = 0; u < 3; ++u) b[j][u] = v.part[u];
                }
#pragma unroll
                for (int i = 0; i < TA; ++i) {
                    const Split a(A::frag(sa, (wm * TA + i) * 32, s, lane));
                    constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                    for (int u = 0; u < 6; ++u)
#pragma unroll
                        for (int j = 0; j < TB; ++j) acc[i][j] = mfma(b[j][pb[u]], a.part[pa[u]], acc[i][j]);
                }
            }
        }
    }

    // acc = A(m0.., k) B(k, n0..) over the k tiles t0 .. t1 - 1
    static __device__ __forceinline__ void product(v16f (&acc)[TA][TB], const Product &p, char *lds, int m0, int n0,
                                                   int t0, int t1) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        const int wm = wave / WN, wn = wave % WN;
        A a;
        B b;
        a.init(p.a, p.lda, m0, p.m, p.k, wave, lane);
        b.init(p.b, p.ldb, n0, p.n, p.k, wave, lane);
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        char *const la = lds, *const lb = lds + 2 * A::BYTES;
        const int last = (p.k - 1) / BK;
        a.load(la, t0, p.k, t0 == last, wave);
        b.load(lb, t0, p.k, t0 == last, wave);
        int buf = 0;
        for (int t = t0; t < t1; ++t) {
            wait_loads();
            __syncthreads();  // tile t has landed, and nobody reads the other buffer any more
            const int nb = buf ^ 1;
            if (t + 1 < t1) {
                a.load(la + nb * A::BYTES, t + 1, p.k, t + 1 == last, wave);
                b.load(lb + nb * B::BYTES, t + 1, p.k, t + 1 == last, wave);
            }
            if ((!AC || !BC) && t == last && p.k % A::CH != 0) {
                A::clear_tail(la + buf * A::BYTES, p.k - t * BK, THREADS);
                B::clear_tail(lb + buf * B::BYTES, p.k - t * BK, THREADS);
                __syncthreads();
            }
            compute(acc, la + buf * A::BYTES, lb + buf * B::BYTES, wm, wn, lane);
            buf = nb;
        }
    }
};

// the block's tile and range of k: neighbouring tiles go to one XCD (blocks
// are dealt to the 8 XCDs in turn), eight rows of tiles after another, so that
// the tiles in work at one time on an XCD share their operands in its L2
struct Place {
    int m, n, split;
};
__device__ __forceinline__ Place place(int tiles_m, int tiles_n, int splits) {
    const int tiles = tiles_m * tiles_n, total = tiles * splits;
    const int x = blockIdx.x & 7, q = total >> 3, r = total & 7;
    const int at = x * q + (x < r ? x : r) + (blockIdx.x >> 3);
    Place o;
    o.split = at / tiles;
    const int t = at - o.split * tiles;
    const int per = 8 * tiles_n, g = t / per, in = t - g * per;
    const int rows = min(8, tiles_m - g * 8);
    o.n = in / rows;
    o.m = g * 8 + (in - o.n * rows);
    return o;
}

// ---- epilogues --------------------------------------------------------------
__device__ __forceinline__ float act_of(float z, int act) {
    switch (act) {
        case kRelu: return z > 0.f ? z : (z != z ? z : 0.f);
        case kGelu: return 0.5f * z * erfcf(-0.70710678118654752f * z);
        case kSilu: return z / (1.f + expf(-z));
        default: return z;
    }
}

// exp of a difference of logits: to the rounding of fp32 where the result is
// fp32, the hardware's (2 ulp and the argument's rounding) for 16-bit results
template <typename T>
__device__ __forceinline__ float exp_of(float x) {
    return sizeof(T) == 4 ? expf(x) : __expf(x);
}

template <typename T>
__device__ __forceinline__ void load4(const T *p, int count, float (&v)[4]) {
    typedef T v4 __attribute__((ext_vector_type(4)));
    if (count >= 4) {
        const v4 x = *(const v4 *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = Type<T>::get(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < count ? Type<T>::get(p[i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T *p, int count, const float (&v)[4]) {
    typedef T v4 __attribute__((ext_vector_type(4)));
    if (count >= 4) {
        v4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = Type<T>::put(v[i]);
        *(v4 *)p = x;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) p[i] = Type<T>::put(v[i]);
    }
}
template <typename T>
__device__ __forceinline__ float bias_at(const void *bias, int f32, int n) {
    return f32 ? ((const float *)bias)[n] : Type<T>::get(((const T *)bias)[n]);
}

// y = act(alpha acc + bias + beta r) of one 32x32 tile at (m0, n0)
template <typename T>
__device__ __forceinline__ void finish(const v16f &acc, const Product &p, const Epilogue &e, int m0, int n0, int lane) {
    const int m = m0 + (lane & 31);
    if (m >= p.m) return;
    const float alpha = e.alpha_dev ? e.alpha * *e.alpha_dev : e.alpha;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int n = n0 + 8 * q + 4 * (lane >> 5), count = p.n - n;
        if (count <= 0) continue;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = alpha * acc[4 * q + i];
        if (e.bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) v[i] += bias_at<T>(e.bias, e.bias_f32, n + i);
        }
        if (e.r) {
            float r[4];
            if (e.r_f32)
                load4((const float *)e.r + (int64_t)m * e.ldr + n, count, r);
            else
                load4((const T *)e.r + (int64_t)m * e.ldr + n, count, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf(e.beta, r[i], v[i]);
        }
        if (e.pre) store4((T *)e.pre + (int64_t)m * e.ldpre + n, count, v);
        if (e.act != kNone) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = act_of(v[i], e.act);
        }
        if (e.y_f32)
            store4((float *)e.y + (int64_t)m * e.ldy + n, count, v);
        else
            store4((T *)e.y + (int64_t)m * e.ldy + n, count, v);
    }
}

// The product with the linear epilogue; with more than one split the raw sums
// go to p.partial (in the order that the joining kernel reads them back).
template <typename T, bool AC, bool BC, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM *WN, 1) void product_kernel(Product p, Epilogue e) {
    using G = Tile<T, AC, BC, BM, BN, WM, WN>;
    __shared__ __attribute__((aligned(1024))) char lds[G::LDS];
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const Place o = place(tm, tn, p.splits);
    const int tiles = (p.k + G::BK - 1) / G::BK;
    const int t0 = o.split * p.split_tiles, t1 = min(tiles, t0 + p.split_tiles);
    v16f acc[G::TA][G::TB];
    G::product(acc, p, lds, o.m * BM, o.n * BN, t0, t1);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    if (p.splits > 1) {
        float *to = p.partial + ((int64_t)o.split * tm * tn + o.m * tn + o.n) * (BM * BN);
#pragma unroll
        for (int i = 0; i < G::TA; ++i)
#pragma unroll
            for (int j = 0; j < G::TB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v4f v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r];
                    const int sub = ((wm * G::TA + i) * (BN / 32) + wn * G::TB + j) * 4 + q;
                    *(v4f *)(to + (int64_t)sub * 256 + lane * 4) = v;
                }
        return;
    }
#pragma unroll
    for (int i = 0; i < G::TA; ++i)
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
            finish<T>(acc[i][j], p, e, o.m * BM + (wm * G::TA + i) * 32, o.n * BN + (wn * G::TB + j) * 32, lane);
}

// The sum of the splits' partial tiles, in split order, and the epilogue: a
// wave for each 32x32 tile.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(Product p, Epilogue e, int bm, int bn) {
    const int tm = (p.m + bm - 1) / bm, tn = (p.n + bn - 1) / bn;
    const int sub_n = bn / 32, subs = (bm / 32) * sub_n;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (w >= (int64_t)tm * tn * subs) return;
    const int tile = (int)(w / subs), sub = (int)(w % subs);
    const int m0 = (tile / tn) * bm + (sub / sub_n) * 32, n0 = (tile % tn) * bn + (sub % sub_n) * 32;
    if (m0 >= p.m || n0 >= p.n) return;
    const float *from = p.partial + (int64_t)tile * (bm * bn) + sub * 1024 + lane * 4;
    const int64_t step = (int64_t)tm * tn * bm * bn;
    v16f acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    for (int s = 0; s < p.splits; ++s) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const v4f v = *(const v4f *)(from + s * step + q * 256);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[4 * q + r] += v[r];
        }
    }
    finish<T>(acc, p, e, m0, n0, lane);
}

// Softmax statistics of the logits X W + b over one tile of classes, for every
// row the largest and the sum of exp(logit - largest): the logits stay in
// registers. The lane that holds a row's own class writes its logit.
template <typename T, bool BC, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM *WN, 1) void stats_kernel(Product p, Classes c) {
    using G = Tile<T, false, BC, BM, BN, WM, WN>;
    __shared__ __attribute__((aligned(1024))) char lds[G::LDS];
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const Place o = place(tm, tn, 1);
    v16f acc[G::TA][G::TB];
    G::product(acc, p, lds, o.m * BM, o.n * BN, 0, (p.k + G::BK - 1) / G::BK);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    float *const top = (float *)lds, *const sum = top + WN * BM;
    __syncthreads();  // the operand tiles are read out
#pragma unroll
    for (int i = 0; i < G::TA; ++i) {
        const int row = (wm * G::TA + i) * 32 + (lane & 31), m = o.m * BM + row;
        const int64_t t = m < p.m ? c.target(m) : -1;
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = o.n * BN + (wn * G::TB + j) * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
                float v = acc[i][j][r];
                if (c.bias && n < p.n) v += bias_at<T>(c.bias, c.bias_f32, n);
                if (n >= p.n) v = -INFINITY;
                else if (n == t) c.own_logit[m] = v;
                acc[i][j][r] = v;
                mx = fmaxf(mx, v);
            }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        float s = 0.f;
        const float base = mx == -INFINITY ? 0.f : mx;  // no class left: exp(-inf) = 0 each
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) s += exp_of<T>(acc[i][j][r] - base);
        s += __shfl_xor(s, 32);
        if (lane < 32) {
            top[wn * BM + row] = mx;
            sum[wn * BM + row] = s;
        }
    }
    __syncthreads();
    for (int row = threadIdx.x; row < BM; row += G::THREADS) {
        const int m = o.m * BM + row;
        if (m >= p.m) continue;
        float mx = -INFINITY, s = 0.f;
#pragma unroll
        for (int w = 0; w < WN; ++w) mx = fmaxf(mx, top[w * BM + row]);
        const float base = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int w = 0; w < WN; ++w) s += sum[w * BM + row] * expf(top[w * BM + row] - base);
        c.stats[(int64_t)o.n * p.m + m] = make_float2(mx, s);
    }
}

// The logits' gradient over one piece of the classes, from recomputed logits:
// g = weight (exp(logit - lse) - [own class]) c.scale, zero for rows left out.
template <typename T, bool BC, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM *WN, 1) void grad_kernel(Product p, Classes c) {
    using G = Tile<T, false, BC, BM, BN, WM, WN>;
    __shared__ __attribute__((aligned(1024))) char lds[G::LDS];
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const Place o = place(tm, tn, 1);
    v16f acc[G::TA][G::TB];
    G::product(acc, p, lds, o.m * BM, o.n * BN, 0, (p.k + G::BK - 1) / G::BK);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < G::TA; ++i) {
        const int m = o.m * BM + (wm * G::TA + i) * 32 + (lane & 31);
        if (m >= p.m) continue;
        const int64_t t = c.target(m) - c.first;
        const float w = c.weight[m] * c.scale, lse = c.lse[m];
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = o.n * BN + (wn * G::TB + j) * 32 + 8 * q + 4 * (lane >> 5), count = p.n - n;
                if (count <= 0) continue;
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float l = acc[i][j][4 * q + r];
                    if (c.bias && r < count) l += bias_at<T>(c.bias, c.bias_f32, n + r);
                    const float g = w * (exp_of<T>(l - lse) - (n + r == t ? 1.f : 0.f));
                    v[r] = w == 0.f ? 0.f : g;
                }
                store4((T *)c.grad + (int64_t)m * c.ldgrad + n, count, v);
            }
    }
}

}  // namespace gemm
}  // namespace rsc
