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
// matrix-core tiles. The operands' tiles are DEPTH bytes of k deep and go from
// memory to LDS directly (16 bytes a lane, through buffer descriptors that
// return zero past a matrix's end) into a ring of STAGES buffers.
//
// LDS layouts, both free of bank conflicts:
//   kRows: DEPTH bytes a row, its 16-byte chunks XORed with a few bits of the
//     row; a lane reads its eight k values by one (fp32: two) 16-byte reads.
//   kCols: BK rows of BM (BN) values as they lie in memory, chunks XORed with
//     a few bits of k; 16-bit fragments come by the transposing LDS read
//     (ds_read_b64_tr_b16), fp32 ones by eight 4-byte reads.
//
// The matrix instruction is fed (B, A), so that a lane holds one row m and
// four consecutive columns n per register quad: row sums stay in the lane.
// Results leave through LDS, 32 rows of a wave at a time, so that each store
// (and each read of a residual) covers whole 128-byte lines: written straight
// from the accumulators, 16 bytes a row, a 256 x 256 bf16 tile took 10 us more.
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

#include <type_traits>

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
// register result, and wait_but() stands before the barrier that hands a
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

// ---- one operand's tile: R rows (or columns) by DEPTH bytes of k -----------
template <typename T, bool COLS, int R, int WAVES, int DEPTH>
struct Operand {
    static constexpr int ES = (int)sizeof(T);
    static constexpr int BK = DEPTH / ES;
    static constexpr int CH = 16 / ES;              // values a chunk
    static constexpr int BYTES = R * DEPTH;
    static constexpr int N = BYTES / 1024 / WAVES;  // loads of a wave
    static_assert(BYTES % (1024 * WAVES) == 0, "whole wave loads");
    static_assert(WAVES % 2 == 0, "a lane's chunk of k is the same in all its loads");
    static constexpr int CPR = COLS ? R / CH : DEPTH / 16;  // chunks an LDS row

    // kRows: XOR of a chunk's place in its row. A 16-byte read takes 16 lanes,
    // here 16 consecutive rows, a cycle from 64 banks: rows that start at the
    // same bank (every second one of 128 bytes, every fourth of 64) get their
    // chunk of k from different places.
    static __device__ __forceinline__ int turn(int row) { return DEPTH == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }
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
                off[q] = (uint32_t)(row * ldb) + (uint32_t)((slot ^ turn(row)) * 16);
        }
        k_at = COLS ? 0 : ((lane % CPR) ^ turn((wave * 64 + lane) / CPR)) * CH;
    }

    // what a tile's loads share
    struct Source {
        v4i rsrc;
        uint32_t soff;
        bool outside;
    };
    // tile t; last: it holds K's end; !live: a tile past the end, its loads write zeros
    __device__ __forceinline__ Source source(int t, int K, bool last, bool live) const {
        const char *from = base;
        int64_t left = bytes;
        Source o;
        o.soff = 0;
        if (COLS) {
            from += t * step;
            left -= t * step;
        } else {
            o.soff = (uint32_t)t * DEPTH;
        }
        const uint32_t n = left <= 0 || !live ? 0u : (uint32_t)(left < (int64_t)0x7ffffff0 ? left : (int64_t)0x7ffffff0);
        const uint64_t at = (uint64_t)from;
        o.rsrc = v4i{(int)(uint32_t)at, (int)(uint32_t)((at >> 32) & 0xffffu), (int)n, 0x00027000};
        o.outside = !COLS && last && t * BK + k_at >= K;
        return o;
    }
    // load q of the wave
    __device__ __forceinline__ void load(const Source &o, int q, char *to, int wave) const {
        load_to_lds(o.rsrc, (uint32_t)(uintptr_t)(lds_void *)(to + (q * WAVES + wave) * 1024),
                    o.outside ? kOutside : off[q], o.soff);
    }

    // kRows, the tile that ends inside a chunk: zeroes that chunk's values from
    // k = kn on (they hold what lies behind K in memory)
    static __device__ __forceinline__ void clear_tail(char *at, int kn, int threads) {
        if (COLS) return;
        for (int row = threadIdx.x; row < R; row += threads) {
            T *chunk = (T *)(at + row * DEPTH + (((kn / CH) ^ turn(row)) * 16));
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
                f = *(const typename Type<T>::frag *)(at + row * DEPTH + ((c ^ turn(row)) * 16));
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
                const v4f a = *(const v4f *)(at + row * DEPTH + ((c ^ turn(row)) * 16));
                const v4f b = *(const v4f *)(at + row * DEPTH + (((c + 1) ^ turn(row)) * 16));
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
// BM x BN by WM x WN waves, tiles DEPTH bytes of k deep, STAGES of them in LDS
template <int BM_, int BN_, int WM_, int WN_, int DEPTH_, int STAGES_>
struct Config {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, DEPTH = DEPTH_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
};

template <int N>
__device__ __forceinline__ void wait_but() {  // all loads but the N youngest have landed
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <typename T, bool AC, bool BC, typename C>
struct Tile {
    static constexpr int BM = C::BM, BN = C::BN, WN = C::WN, THREADS = C::THREADS, STAGES = C::STAGES;
    static constexpr int TA = BM / C::WM / 32, TB = BN / WN / 32;
    using A = Operand<T, AC, BM, C::WAVES, C::DEPTH>;
    using B = Operand<T, BC, BN, C::WAVES, C::DEPTH>;
    static constexpr int BK = A::BK, STEPS = BK / 16;
    static_assert(STEPS % 2 == 0, "fragments alternate between two sets");
    static constexpr int STAGE = A::BYTES + B::BYTES, LDS = STAGES * STAGE;
    static constexpr int LOADS = A::N + B::N;  // of a wave for a tile

    struct Frags {
        typename Type<T>::frag a[TA], b[TB];
        // fragment x of TA + TB, in the order in which multiply() needs them
        __device__ __forceinline__ void read(int x, const char *at, int wm, int wn, int s, int lane) {
            if (x == 0) a[0] = A::frag(at, wm * TA * 32, s, lane);
            else if (x <= TB) b[x - 1] = B::frag(at + A::BYTES, (wn * TB + x - 1) * 32, s, lane);
            else a[x - TB] = A::frag(at, (wm * TA + x - TB) * 32, s, lane);
        }
    };

    // acc = A(m0.., k) B(k, n0..) over the k tiles t0 .. t1 - 1. STAGES - 1
    // tiles are in flight; the fragments of a step of 16 k are read while the
    // step before is multiplied, across tiles too, and the loads of a later
    // tile go out between the matrix instructions. For 16-bit operands the
    // order is fixed by hand (a read or a load, then a matrix instruction):
    // left to itself the compiler puts each read right before its use.
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
        const int last = (p.k - 1) / BK;
        const bool cut = (!AC || !BC) && p.k % A::CH != 0 && t1 > last;  // K ends inside a chunk
        // tile t is in LDS for every wave, and every wave is done with the one before
        const auto arrive = [&](int t, char *at) {
            wait_but<(STAGES - 2) * LOADS>();
            __syncthreads();
            if (cut && t == last) {
                A::clear_tail(at, p.k - t * BK, THREADS);
                B::clear_tail(at + A::BYTES, p.k - t * BK, THREADS);
                __syncthreads();
            }
        };
        typename A::Source sa;
        typename B::Source sb;
        const auto aim = [&](int t) {
            sa = a.source(t, p.k, t == last, t < t1);
            sb = b.source(t, p.k, t == last, t < t1);
        };
        const auto load = [&](int x, char *to) {
            if (x < A::N) a.load(sa, x, to, wave);
            else b.load(sb, x - A::N, to + A::BYTES, wave);
        };
#pragma unroll
        for (int u = 0; u < STAGES - 1; ++u) {
            aim(t0 + u);
#pragma unroll
            for (int x = 0; x < LOADS; ++x) load(x, lds + u * STAGE);
        }
        char *at = lds, *const end = lds + STAGES * STAGE;
        arrive(t0, at);
        Frags f[2];
#pragma unroll
        for (int x = 0; x < TA + TB; ++x) f[0].read(x, at, wm, wn, 0, lane);
        for (int t = t0; t < t1; ++t) {
            char *const to = at == lds ? end - STAGE : at - STAGE;
            char *const next = at + STAGE == end ? lds : at + STAGE;
            aim(t + STAGES - 1);
            // the tile's matrix instructions but the last step's, and how many of them pass between two loads
            constexpr int MULS = TA * TB, ROOM = (STEPS - 1) * MULS, EVERY = STAGES > 2 && ROOM / LOADS > 1 ? ROOM / LOADS : 1;
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const bool over = s + 1 == STEPS;  // reads on are the next tile's (zero or stale after the last)
                    if (over) arrive(t + 1, next);
#pragma unroll
                    for (int x = 0; x < MULS; ++x) {
                        __builtin_amdgcn_sched_barrier(0);
                        // reads in the first matrix instructions, evenly if there are more of them
#pragma unroll
                        for (int y = 0; y < TA + TB; ++y)
                            if (y * MULS / (TA + TB > MULS ? TA + TB : MULS) == x)
                                f[(s + 1) & 1].read(y, over ? next : at, wm, wn, over ? 0 : s + 1, lane);
                        const int m = s * MULS + x;
                        if (!over) {
#pragma unroll
                            for (int y = 0; y < LOADS; ++y)
                                if (min(y * EVERY, ROOM - 1) == m) load(y, to);
                        }
                        acc[x / TB][x % TB] = mfma(f[s & 1].b[x % TB], f[s & 1].a[x / TB], acc[x / TB][x % TB]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int x = 0; x < LOADS; ++x) load(x, to);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const bool over = s + 1 == STEPS;
                    if (over) arrive(t + 1, next);
#pragma unroll
                    for (int x = 0; x < TA + TB; ++x)
                        f[(s + 1) & 1].read(x, over ? next : at, wm, wn, over ? 0 : s + 1, lane);
                    multiply_split(acc, f[s & 1]);
                }
            }
            at = next;
        }
        wait_but<0>();
        __syncthreads();  // nothing is in flight to LDS any more
    }

    static __device__ __forceinline__ void multiply_split(v16f (&acc)[TA][TB], const Frags &f) {
        v8bf b[TB][3];
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            const Split v(f.b[j]);
#pragma unroll
            for (int u = 0; u < 3; ++u) b[j][u] = v.part[u];
        }
#pragma unroll
        for (int i = 0; i < TA; ++i) {
            const Split a(f.a[i]);
            constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
            for (int u = 0; u < 6; ++u)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = mfma(b[j][pb[u]], a.part[pa[u]], acc[i][j]);
        }
    }
};

// the block's tile and range of k: neighbouring tiles go to one XCD (blocks
// are dealt to the 8 XCDs in turn), four rows of tiles after another, so that
// the 32 tiles in work at one time on an XCD, four by eight, share their
// operands in its L2 (16384 x 4096 x 8192 bf16: 918 us, 960 with eight rows, 990 with 16)
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
    const int per = 4 * tiles_n, g = t / per, in = t - g * per;
    const int rows = min(4, tiles_m - g * 4);
    o.n = in / rows;
    o.m = g * 4 + (in - o.n * rows);
    return o;
}

// ---- epilogues --------------------------------------------------------------
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if (ACT == kRelu) return z > 0.f ? z : (z != z ? z : 0.f);
    if (ACT == kGelu) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    if (ACT == kSilu) return z / (1.f + expf(-z));
    return z;
}

// exp(v - base). For fp32 results to the rounding of fp32; for 16-bit ones by the
// hardware's power of two (2 ulp). The difference comes first: log2(e) times a
// logit of fp32's lowest values, as masks have them, is past its range.
template <typename T>
__device__ __forceinline__ float exp_below(float v, float base) {
    return sizeof(T) == 4 ? expf(v - base) : __builtin_amdgcn_exp2f((v - base) * 1.44269504089f);
}

template <typename T>
__device__ __forceinline__ float bias_at(const void *bias, int f32, int64_t n) {
    return f32 ? ((const float *)bias)[n] : Type<T>::get(((const T *)bias)[n]);
}

// values a lane takes of a row in the epilogue: 16 bytes of the result
template <typename T>
constexpr int kWidth = 16 / (int)sizeof(T);

// the first `count` (at least 1) of a row's 16 bytes, zeros behind them. All
// are read: rows are whole 16-byte units apart, so they lie with the first one.
template <typename T>
__device__ __forceinline__ void load_row(const T *p, int count, float (&v)[kWidth<T>]) {
    constexpr int W = kWidth<T>;
    typedef T vec __attribute__((ext_vector_type(W)));
    const vec x = *(const vec *)p;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = i < count ? Type<T>::get(x[i]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_row(T *p, int count, const float (&v)[kWidth<T>], bool stream = false) {
    constexpr int W = kWidth<T>;
    typedef T vec __attribute__((ext_vector_type(W)));
    if (count >= W) {
        vec x;
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = Type<T>::put(v[i]);
        if (stream) __builtin_nontemporal_store(x, (vec *)p);
        else *(vec *)p = x;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < count) p[i] = Type<T>::put(v[i]);
    }
}
// the same for W fp32 values at a place that is 16-byte aligned
template <int W>
__device__ __forceinline__ void load_f32(const float *p, int count, float (&v)[W]) {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (count > 4 * q) load_row(p + 4 * q, count - 4 * q, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * q + i] = x[i];
    }
}
template <int W>
__device__ __forceinline__ void store_f32(float *p, int count, const float (&v)[W], bool stream = false) {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) {
        const float x[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        store_row(p + 4 * q, count - 4 * q, x, stream);
    }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// the bias of a lane's columns, 0 without one or past the end
template <typename T>
__device__ __forceinline__ void load_bias(const void *bias, int f32, int n, int count, float (&v)[kWidth<T>]) {
#pragma unroll
    for (int i = 0; i < kWidth<T>; ++i) v[i] = bias && i < count ? bias_at<T>(bias, f32, n + i) : 0.f;
}

// A lane's place in the epilogue: its first row, and its columns n .. n +
// count - 1, the same in every row that it takes (`down` rows further on,
// the same for the whole wave).
struct Spot {
    int m, n, count;
};

// What the residual adds to a lane's columns, as read: fp32, or the operands' type
// in x[0].
template <int W>
struct Rest {
    v4f x[W / 4];
};
template <typename T>
__device__ __forceinline__ Rest<kWidth<T>> fetch_rest(const Epilogue &e, const Spot &at, int down) {
    constexpr int W = kWidth<T>;
    Rest<W> g = {};
    if (at.count <= 0) return g;
    if (e.r_f32 && sizeof(T) != 4) {
        const float *const p = (const float *)e.r + (at.m * e.ldr + at.n) + down * e.ldr;
#pragma unroll
        for (int q = 0; q < W / 4; ++q)
            if (at.count > 4 * q) g.x[q] = *(const v4f *)(p + 4 * q);
    } else {
        g.x[0] = *(const v4f *)((const T *)e.r + (at.m * e.ldr + at.n) + down * e.ldr);
    }
    return g;
}

// z = alpha sum + bias (+ beta r)
template <typename T>
__device__ __forceinline__ void argument(float (&v)[kWidth<T>], const float (&bias)[kWidth<T>], float alpha) {
#pragma unroll
    for (int i = 0; i < kWidth<T>; ++i) v[i] = fmaf(alpha, v[i], bias[i]);
}
template <typename T>
__device__ __forceinline__ void argument(float (&v)[kWidth<T>], const float (&bias)[kWidth<T>], const Epilogue &e,
                                         float alpha, const Spot &at, const Rest<kWidth<T>> &g, float (&r)[kWidth<T>]) {
    constexpr int W = kWidth<T>;
    typedef T vec __attribute__((ext_vector_type(W)));
    if (e.r_f32 && sizeof(T) != 4) {
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] = i < at.count ? g.x[i / 4][i % 4] : 0.f;
    } else {
        const vec x = __builtin_bit_cast(vec, g.x[0]);
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] = i < at.count ? Type<T>::get(x[i]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = fmaf(e.beta, r[i], fmaf(alpha, v[i], bias[i]));
}
// a positive value that its type would round to 0: the type's smallest (see mend())
template <typename T>
constexpr float kSmallest = std::is_same_v<T, _Float16> ? 0x1p-24f : 0x1p-126f;
template <typename T>
__device__ __forceinline__ float above_zero(float y) {
    return y > 0.f && Type<T>::get(Type<T>::put(y)) == 0.f ? kSmallest<T> : y;
}

// y = act(z)
template <typename T, int ACT>
__device__ __forceinline__ void leave(float (&v)[kWidth<T>], const Epilogue &e, const Spot &at, int down) {
    constexpr int W = kWidth<T>;
    if (e.pre) store_f32(e.pre + (at.m * e.ldpre + at.n) + down * e.ldpre, at.count, v, e.stream);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = act_of<ACT>(v[i]);
    if (e.y_f32) store_f32((float *)e.y + (at.m * e.ldy + at.n) + down * e.ldy, at.count, v);
    else store_row((T *)e.y + (at.m * e.ldy + at.n) + down * e.ldy, at.count, v, e.stream);
}

// ---- the sign of a ReLU's argument ------------------------------------------
// A ReLU's gradient hangs on the sign of its argument. A sum in fp32 that comes
// out next to zero may have the other sign, which takes in or leaves out a whole
// term of every gradient: among 10 million results of 1,021 terms about one. For results
// that a backward pass will read (e.sure) those few are formed again in 64
// bits, and a positive one that its type would round to 0 stays at the type's
// smallest value.
// sum over k of A(m, k) B(k, n) in 64 bits (products of the operands' types are
// exact there), by the whole wave; A stored by rows
template <typename T>
__device__ __forceinline__ double dot64(const Product &p, int b_cols, int m, int n) {
    constexpr int W = kWidth<T>;
    const int lane = threadIdx.x & 63;
    const T *const a = (const T *)p.a + m * p.lda;
    double sum = 0.0;
    for (int k = lane * W; k < p.k; k += 64 * W) {
        float x[W], y[W];
        load_row(a + k, p.k - k, x);
        if (b_cols) {
#pragma unroll
            for (int i = 0; i < W; ++i) y[i] = Type<T>::get(((const T *)p.b)[min(k + i, p.k - 1) * p.ldb + n]);
#pragma unroll
            for (int i = 0; i < W; ++i) y[i] = k + i < p.k ? y[i] : 0.f;
        } else {
            load_row((const T *)p.b + n * p.ldb + k, p.k - k, y);
        }
#pragma unroll
        for (int i = 0; i < W; ++i) sum = fma((double)x[i], (double)y[i], sum);
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    return sum;
}

// How far a sum of k terms may be off, from the largest sum around it: a random
// walk of roundings takes it 2^-24 sqrt(k / 16) of that, this is more than ten
// times as far.
__device__ __forceinline__ float doubt_of(float largest, int k) { return largest * 0x1p-24f * (8.f + sqrtf((float)k)); }

// The largest sum around one of a row: the wave's, which sees the scale of every
// column, unless the row's own is 2^10 times smaller, as beside a row of another
// scale in A: then ordinary results would count as next to zero, too many of them
// for the list (up to that factor some 16 of 8,192). From fewer than kScaleOf
// columns a row's own scale does not show, since all of them may be next to zero.
constexpr int kScaleOf = 8;
__device__ __forceinline__ float largest_around(float row, float wave, int columns) {
    return columns >= kScaleOf && row * 1024.f < wave ? row : wave;
}

// Is an argument next to zero? `others`: the magnitudes added to the sum. A sum
// of exactly 0 is taken as such (a row of zeros).
__device__ __forceinline__ bool unsure(float z, float sum, float others, float doubt) {
    return sum != 0.f && fabsf(z) < fmaf(others, 0x1p-22f, doubt);
}
// what one wave forms again at most: operands of few different values can cancel
// everywhere, but then their sums are exact
constexpr int kBudget = 32;

// A place to form again, and the residual's value there: Y may lie on R, and is
// written by then.
struct Again {
    uint32_t place;
    float r;
};
// Row m, column n once more, by the whole wave.
template <typename T>
__device__ __forceinline__ void mend(const Product &p, const Epilogue &e, float alpha, int m, int n, float r) {
    double s = (double)alpha * dot64<T>(p, e.b_cols, m, n);
    if (e.bias) s += (double)bias_at<T>(e.bias, e.bias_f32, n);
    if (e.r) s += (double)e.beta * (double)r;
    if ((threadIdx.x & 63) != 0) return;
    const float z = (float)s, y = above_zero<T>(fmaxf(z, 0.f));
    if (e.pre) e.pre[m * e.ldpre + n] = z;
    if (e.y_f32) ((float *)e.y)[m * e.ldy + n] = y;
    else ((T *)e.y)[m * e.ldy + n] = Type<T>::put(y);
}

// A wave's list of unsure places, in LDS. They are formed again when the wave's
// rows are done: the accumulators are free by then. (Within the rows' loop the
// 256 x 256 kernel spilled, and every product took 4 to 15 times as long.)
struct Unsure {
    Again *list;
    int count = 0;  // the same in all lanes
    // Values above zero also leave as such (above_zero). All lanes call it; most,
    // eight values at a time, with nothing near zero.
    template <typename T>
    __device__ __forceinline__ void note(float (&z)[kWidth<T>], const float (&sum)[kWidth<T>],
                                         const float (&bias)[kWidth<T>], const float (&r)[kWidth<T>],
                                         const Epilogue &e, float doubt, uint32_t place, int width) {
        constexpr int W = kWidth<T>;
        float low = INFINITY, added = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            low = fminf(low, fabsf(z[i]));
            added = fmaxf(added, fmaf(fabsf(e.beta), fabsf(r[i]), fabsf(bias[i])));
        }
        if (!__ballot(width > 0 && low < fmaxf(fmaf(added, 0x1p-22f, doubt), kSmallest<T>))) return;
        uint32_t todo = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (i < width && unsure(z[i], sum[i], fabsf(bias[i]) + fabsf(e.beta * r[i]), doubt)) todo |= 1u << i;
            z[i] = above_zero<T>(z[i]);
        }
        while (const uint64_t who = __ballot(todo != 0)) {
            const int at = count + __popcll(who & ((1ull << (threadIdx.x & 63)) - 1));
            const int first = __ffs((int)todo) - 1;
            float residual = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) residual = i == first ? r[i] : residual;
            if (todo && at < kBudget) list[at] = Again{place + first, residual};
            todo &= todo - 1;
            count = min(count + __popcll(who), kBudget);
        }
    }
};

// f(the activation as a constant): one test a block; GRADIENT: a product of the
// backward pass, which has none
template <bool GRADIENT = false, typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (GRADIENT ? kNone : act) {
        case kRelu: return f(std::integral_constant<int, kRelu>());
        case kGelu: return f(std::integral_constant<int, kGelu>());
        case kSilu: return f(std::integral_constant<int, kSilu>());
        default: return f(std::integral_constant<int, kNone>());
    }
}
__device__ __forceinline__ float alpha_of(const Epilogue &e) { return e.alpha_dev ? e.alpha * *e.alpha_dev : e.alpha; }

// f(down, v) for the accumulators' rows, W consecutive columns of the row
// `down` below the lane's spot a call. Through the wave's own part
// of LDS, which nothing else uses then; rows are 16 bytes more than a multiple of 128
// apart, so that 16 rows' writes and a row's reads fall into different banks.
template <typename G, int W>
__device__ __forceinline__ Spot spot_of(const Product &p, int m0, int n0) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int COLS = G::TB * 32, LANES = COLS / W;
    Spot s;
    s.m = m0 + (wave / G::WN) * G::TA * 32 + lane / LANES;
    s.n = n0 + (wave % G::WN) * COLS + (lane % LANES) * W;
    s.count = p.n - s.n;
    return s;
}
// What fetch(down) reads for f goes out for four calls together, the first four
// before the rows pass through LDS: one by one behind the stores of the row before (which
// the compiler must keep in order) a residual took 6.5 us of 43 at 5003 x 1021 x 2045.
template <typename G, int W, typename Fetch, typename F>
__device__ __forceinline__ void by_rows(const v16f (&acc)[G::TA][G::TB], char *lds, Fetch fetch, F f) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int COLS = G::TB * 32, LD = COLS + 4;
    static_assert(32 * LD * 4 * (G::THREADS / 64) <= G::LDS, "the waves' rows");
    float *const slab = (float *)lds + wave * (32 * LD);
    constexpr int LANES = COLS / W, ROWS = 64 / LANES;  // lanes a row, rows at a time
    constexpr int CALLS = 32 / ROWS, AHEAD = CALLS < 4 ? CALLS : 4;
    const int c = (lane % LANES) * W;
#pragma unroll
    for (int i = 0; i < G::TA; ++i) {
        decltype(fetch(0)) got[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) got[u] = fetch(i * 32 + u * ROWS);
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v4f x;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = acc[i][j][4 * q + r];
                *(v4f *)(slab + (lane & 31) * LD + j * 32 + 8 * q + 4 * (lane >> 5)) = x;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int u0 = 0; u0 < CALLS; u0 += AHEAD) {
            if (u0 > 0) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) got[u] = fetch(i * 32 + (u0 + u) * ROWS);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int row = (u0 + u) * ROWS + lane / LANES;
                float v[W];
#pragma unroll
                for (int q = 0; q < W / 4; ++q) {
                    const v4f x = *(const v4f *)(slab + row * LD + c + 4 * q);
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[4 * q + r] = x[r];
                }
                f(i * 32 + (u0 + u) * ROWS, v, got[u]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}
struct Nothing {};
template <typename G, int W, typename F>
__device__ __forceinline__ void by_rows(const v16f (&acc)[G::TA][G::TB], char *lds, F f) {
    by_rows<G, W>(acc, lds, [](int) { return Nothing(); }, [&](int down, float (&v)[W], Nothing) { f(down, v); });
}

// The product with the linear epilogue; with more than one split the raw sums
// go to p.partial, a matrix of p.m rows ld_partial(p.n) apart for each split.
__host__ __device__ inline int64_t ld_partial(int n) { return ((int64_t)n + 7) & ~(int64_t)7; }

template <typename T, bool AC, bool BC, typename C>
__global__ __launch_bounds__(C::THREADS, 1) void product_kernel(Product p, Epilogue e) {
    using G = Tile<T, AC, BC, C>;
    constexpr int BM = C::BM, BN = C::BN, W = kWidth<T>;
    __shared__ __attribute__((aligned(1024))) char lds[G::LDS];
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const Place o = place(tm, tn, p.splits);
    const int tiles = (p.k + G::BK - 1) / G::BK;
    const int t0 = o.split * (p.split_k / G::BK), t1 = min(tiles, t0 + p.split_k / G::BK);
    v16f acc[G::TA][G::TB];
    G::product(acc, p, lds, o.m * BM, o.n * BN, t0, t1);
    if (p.splits > 1) {
        const Spot at = spot_of<G, 4>(p, o.m * BM, o.n * BN);
        const int64_t ld = ld_partial(p.n);
        float *const to = p.partial + (int64_t)o.split * p.m * ld + at.m * ld + at.n;
        by_rows<G, 4>(acc, lds, [&](int down, const float (&v)[4]) {
            if (at.count > 0 && at.m + down < p.m) store_row(to + down * ld, at.count, v);
        });
        return;
    }
    const float alpha = alpha_of(e);
    const Spot at = spot_of<G, W>(p, o.m * BM, o.n * BN);
    float bias[W];
    load_bias<T>(e.bias, e.bias_f32, at.n, at.count, bias);
    const bool sure = !AC && e.act == kRelu && e.sure;  // (the forward pass)
    // in LDS behind the waves' rows: each wave's list, and its rows' bounds
    constexpr int SLABS = 32 * (G::TB * 32 + 4) * 4 * (C::THREADS / 64), LISTS = kBudget * (int)sizeof(Again) * (C::THREADS / 64);
    static_assert(SLABS + LISTS + G::TA * 32 * 4 * (C::THREADS / 64) <= G::LDS, "the waves' rows, lists and bounds");
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Unsure again{(Again *)(lds + SLABS) + kBudget * wave};
    float *const doubts = (float *)(lds + SLABS + LISTS) + G::TA * 32 * wave;
    if (sure) {
        // Columns past the last take no part: with B stored by columns they are sums
        // of what lies beside a row in memory.
        const int left = p.n - (o.n * BN + (wave % C::WN) * G::TB * 32 + 4 * (lane >> 5));
        float largest[G::TA], all = 0.f;
#pragma unroll
        for (int i = 0; i < G::TA; ++i) {
            largest[i] = 0.f;
#pragma unroll
            for (int j = 0; j < G::TB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    largest[i] = j * 32 + 8 * (r >> 2) + (r & 3) < left ? fmaxf(largest[i], fabsf(acc[i][j][r])) : largest[i];
            largest[i] = fmaxf(largest[i], __shfl_xor(largest[i], 32));
            all = fmaxf(all, largest[i]);
        }
        all = wave_max(all);
        const int columns = p.n - (o.n * BN + (wave % C::WN) * G::TB * 32);
#pragma unroll
        for (int i = 0; i < G::TA; ++i)
            doubts[i * 32 + (lane & 31)] = doubt_of(fabsf(alpha) * largest_around(largest[i], all, columns), p.k);
    }
    with_act<AC>(e.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        // whole: no residual, and all rows and columns of the tile exist, which is
        // one test a block instead of several a row (716,847 x 300 x 512 fp32: 1,580
        // us, 1,632 with them). Not for the activations whose arithmetic is the time.
        const auto rows = [&](auto whole, auto fetch) {
            by_rows<G, W>(acc, lds, fetch, [&](int down, float (&v)[W], const auto &rest) {
                const Spot spot{at.m, at.n, whole ? W : at.count};
                const bool live = whole || (at.count > 0 && at.m + down < p.m);
                if (ACT != kRelu && !live) return;
                float sum[W], r[W];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    sum[i] = v[i];
                    r[i] = 0.f;
                }
                if constexpr (std::is_same_v<decltype(rest), const Nothing &>) argument<T>(v, bias, alpha);
                else argument<T>(v, bias, e, alpha, spot, rest, r);
                if (!AC && ACT == kRelu && sure)
                    again.note<T>(v, sum, bias, r, e, doubts[at.m + down - o.m * BM - (wave / C::WN) * G::TA * 32],
                                  (uint32_t)(at.m + down - o.m * BM) << 16 | (at.n - o.n * BN), live ? spot.count : 0);
                if (live) leave<T, ACT>(v, e, spot, down);
            });
        };
        if constexpr (ACT == kNone || ACT == kRelu) {
            if (!e.r && (o.m + 1) * BM <= p.m && (o.n + 1) * BN <= p.n)
                return rows(std::true_type(), [](int) { return Nothing(); });
        }
        rows(std::false_type(),
             [&](int down) { return e.r && at.m + down < p.m ? fetch_rest<T>(e, at, down) : Rest<W>{}; });
    });
    if (!AC && again.count > 0) {
        // behind the rows' own stores
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        for (int i = 0; i < again.count; ++i) {
            const Again x = again.list[i];
            mend<T>(p, e, alpha, o.m * BM + (int)(x.place >> 16), o.n * BN + (int)(x.place & 0xffff), x.r);
        }
    }
}

// The sum of the splits' partial sums and the epilogue: L neighbouring threads
// take W columns of one row, each every L-th split, and add up over a fixed
// tree. One thread is enough where the results fill the chip; with few of them
// (a single row) the splits' reads, one after another, were the time: 16.5 us
// for 4,096 results of 64 splits.
template <typename T, int L>
__global__ __launch_bounds__(256) void join_kernel(Product p, Epilogue e) {
    constexpr int W = kWidth<T>;
    const int64_t ld = ld_partial(p.n), chunks = (p.n + W - 1) / W;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int part = threadIdx.x % L;
    bool live = at < chunks * p.m;
    const int m = live ? (int)(at / chunks) : 0, n = live ? (int)(at % chunks) * W : 0, count = p.n - n;
    const float *from = p.partial + m * ld + n;
    const int64_t step = (int64_t)p.m * ld;
    float v[W], bias[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = 0.f;
    int s = live ? part : p.splits;
    for (; s + 3 * L < p.splits; s += 4 * L) {
        float x[4][W];
#pragma unroll
        for (int u = 0; u < 4; ++u) load_f32(from + (s + u * L) * step, count, x[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] += x[u][i];
    }
    for (; s < p.splits; s += L) {
        float x[W];
        load_f32(from + s * step, count, x);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += x[i];
    }
#pragma unroll
    for (int d = 1; d < L; d *= 2)
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += __shfl_xor(v[i], d);
    live = live && part == 0;
    const float alpha = alpha_of(e);
    const Spot spot{m, n, count};
    float r[W], sum[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        sum[i] = v[i];
        r[i] = bias[i] = 0.f;
    }
    if (live) {
        load_bias<T>(e.bias, e.bias_f32, n, count, bias);
        if (e.r) argument<T>(v, bias, e, alpha, spot, fetch_rest<T>(e, spot, 0), r);
        else argument<T>(v, bias, alpha);
    }
    const bool sure = e.act == kRelu && e.sure;
    __shared__ Again lists[4][kBudget];
    Unsure again{lists[threadIdx.x >> 6]};
    if (sure) {
        float largest = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) largest = fmaxf(largest, fabsf(sum[i]));
        // over the wave's chunks of the same row, which are next to each other
        // (places past the last have sums of 0)
        const float all = wave_max(largest);
        const int64_t first = ((int64_t)blockIdx.x * 256 + (threadIdx.x & ~63)) / L;
        const int from_chunk = (int)max((int64_t)0, first - m * chunks), to_chunk = (int)min(chunks, first + 64 / L - m * chunks);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const float below = __shfl_up(largest, d);
            const int row = __shfl_up(m, d);
            if ((int)(threadIdx.x & 63) >= d && row == m) largest = fmaxf(largest, below);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const float above = __shfl_down(largest, d);
            const int row = __shfl_down(m, d);
            if ((int)(threadIdx.x & 63) + d < 64 && row == m) largest = fmaxf(largest, above);
        }
        const int columns = min(to_chunk * W, p.n) - from_chunk * W;
        const float doubt = doubt_of(fabsf(alpha) * largest_around(largest, all, columns), p.k);
        // places: the value's number among the wave's
        again.note<T>(v, sum, bias, r, e, doubt, (threadIdx.x & 63) * W, live ? count : 0);
    }
    if (live) with_act(e.act, [&](auto act) { leave<T, decltype(act)::value>(v, e, spot, 0); });
    if (again.count > 0) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        for (int i = 0; i < again.count; ++i) {
            const Again x = again.list[i];
            const int from = (int)x.place / W;
            mend<T>(p, e, alpha, __shfl(m, from), __shfl(n, from) + (int)x.place % W, x.r);
        }
    }
}

// Few rows (R of them, 1 to kFewRows) against weights stored by rows: bound by
// reading the weights once, so a wave takes two columns, 16 bytes of their rows
// a lane and turn, sums in the lane and then over a fixed tree. Neither tiles nor
// splits nor a joining launch: 4096 x 4096 bf16 (33.5 MB of weights) one row
// 5.3 us against 9.4 by tiles, two 9.5 against 10.4; 4096 x 4096 fp32 12.3
// against 19.6 and 13.2 against 20, all with the weights in the caches. From memory
// one row of bf16 takes 8.0 us, two 15.8 against 12.6 by tiles. fp32 operands are
// multiplied as they are.
template <typename T, int R>
__global__ __launch_bounds__(256) void few_rows_kernel(Product p, Epilogue e) {
    constexpr int W = kWidth<T>, AHEAD = 4, COLUMNS = 2;
    typedef T vec __attribute__((ext_vector_type(W)));
    const int n0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * COLUMNS, lane = threadIdx.x & 63;
    if (n0 >= p.n) return;
    const T *w[COLUMNS];
#pragma unroll
    for (int j = 0; j < COLUMNS; ++j) w[j] = (const T *)p.b + min(n0 + j, p.n - 1) * p.ldb;
    float acc[COLUMNS][R];
#pragma unroll
    for (int j = 0; j < COLUMNS; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[j][r] = 0.f;
    int k0 = lane * W;
    for (; k0 + (AHEAD - 1) * 64 * W + W <= p.k; k0 += 64 * W * AHEAD) {
        vec a[AHEAD][R], b[AHEAD][COLUMNS];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
#pragma unroll
            for (int j = 0; j < COLUMNS; ++j) b[u][j] = *(const vec *)(w[j] + k0 + u * 64 * W);
#pragma unroll
            for (int r = 0; r < R; ++r) a[u][r] = *(const vec *)((const T *)p.a + r * p.lda + k0 + u * 64 * W);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < COLUMNS; ++j)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        acc[j][r] = fmaf(Type<T>::get(a[u][r][i]), Type<T>::get(b[u][j][i]), acc[j][r]);
    }
    for (; k0 < p.k; k0 += 64 * W) {
        float b[COLUMNS][W];
#pragma unroll
        for (int j = 0; j < COLUMNS; ++j) load_row(w[j] + k0, p.k - k0, b[j]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float a[W];
            load_row((const T *)p.a + r * p.lda + k0, p.k - k0, a);
#pragma unroll
            for (int j = 0; j < COLUMNS; ++j)
#pragma unroll
                for (int i = 0; i < W; ++i) acc[j][r] = fmaf(a[i], b[j][i], acc[j][r]);
        }
    }
    // lane j R + r finishes column j of row r
    const bool sure = e.act == kRelu && e.sure;
    float v = 0.f;
    double exact = 0.0;
#pragma unroll
    for (int j = 0; j < COLUMNS; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int d = 32; d > 0; d /= 2) acc[j][r] += __shfl_xor(acc[j][r], d);
            if (lane == j * R + r) v = acc[j][r];
            if (sure) {  // (the weights are in the caches now)
                const double s = dot64<T>(p, 0, r, min(n0 + j, p.n - 1));
                if (lane == j * R + r) exact = s;
            }
        }
    const int n = n0 + lane / R, m = lane % R;
    if (lane >= COLUMNS * R || n >= p.n) return;
    const float alpha = alpha_of(e), bias = e.bias ? bias_at<T>(e.bias, e.bias_f32, n) : 0.f;
    v = fmaf(alpha, v, bias);
    exact = (double)alpha * exact + (double)bias;
    if (e.r) {
        const int64_t at = m * e.ldr + n;
        const float r = e.r_f32 ? ((const float *)e.r)[at] : Type<T>::get(((const T *)e.r)[at]);
        v = fmaf(e.beta, r, v);
        exact += (double)e.beta * (double)r;
    }
    if (sure) v = (float)exact;
    if (e.pre) e.pre[m * e.ldpre + n] = v;
    with_act(e.act, [&](auto act) { v = act_of<decltype(act)::value>(v); });
    if (sure) v = above_zero<T>(v);
    if (e.y_f32) ((float *)e.y)[m * e.ldy + n] = v;
    else ((T *)e.y)[m * e.ldy + n] = Type<T>::put(v);
}

// Softmax statistics of the logits X W + b over one tile of classes, for every
// row the largest and the sum of exp(logit - largest): the logits stay in
// registers. The lane that holds a row's own class writes its logit. Bound by the
// matrix instructions where k is long (8192 x 4096 x 131,072 bf16: 7.6 ms, 1,160
// TFLOP/s), by a tile's fixed part where it is short: 3001 x 1000 x 50,021 fp16 399 us,
// 456 with a test and a select for each logit's bias and class.
template <typename T, bool BC, typename C>
__global__ __launch_bounds__(C::THREADS, 1) void stats_kernel(Product p, Classes c) {
    using G = Tile<T, false, BC, C>;
    constexpr int BM = C::BM, BN = C::BN, WN = C::WN;
    __shared__ __attribute__((aligned(1024))) char lds[G::LDS];
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const Place o = place(tm, tn, 1);
    static_assert(G::THREADS >= BM && G::THREADS >= BN, "a row and a class each");
    const int tid = threadIdx.x;
    // a row's class and a class's bias, on their way while the logits are formed
    int64_t own_class = -1;
    float class_bias = 0.f;
    if (tid < BM && o.m * BM + tid < p.m) own_class = c.target(o.m * BM + tid);
    if (tid < BN && o.n * BN + tid < p.n && c.bias) class_bias = bias_at<T>(c.bias, c.bias_f32, o.n * BN + tid);
    v16f acc[G::TA][G::TB];
    G::product(acc, p, lds, o.m * BM, o.n * BN, 0, (p.k + G::BK - 1) / G::BK);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    float *const top = (float *)lds, *const sum = top + WN * BM, *const biases = sum + WN * BM;
    int *const owns = (int *)(biases + BN);  // the row's own class, counted from the tile's first
    static_assert((2 * WN * BM + BN + BM) * 4 <= G::LDS, "rows and classes");
    if (tid < BM) {
        const int64_t t = own_class - (int64_t)o.n * BN;
        owns[tid] = own_class < p.n && t >= 0 && t < BN ? (int)t : -1;
    }
    // what is past the last class takes no part
    if (tid < BN) biases[tid] = o.n * BN + tid < p.n ? class_bias : -INFINITY;
    __syncthreads();
    const int n0 = o.n * BN + wn * G::TB * 32 + 4 * (lane >> 5);  // column of a lane's r = 0, j = 0
    const bool whole = o.n * BN + BN <= p.n;
    const float *const bias = biases + (n0 - o.n * BN);
#pragma unroll
    for (int i = 0; i < G::TA; ++i) {
        const int row = (wm * G::TA + i) * 32 + (lane & 31), m = o.m * BM + row;
        if (!whole) {
#pragma unroll
            for (int j = 0; j < G::TB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const v4f b = *(const v4f *)(bias + j * 32 + 8 * q);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[i][j][4 * q + r] = b[r] == -INFINITY ? -INFINITY : acc[i][j][4 * q + r] + b[r];
                }
        } else if (c.bias) {
#pragma unroll
            for (int j = 0; j < G::TB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const v4f b = *(const v4f *)(bias + j * 32 + 8 * q);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][4 * q + r] += b[r];
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, acc[i][j][r]);
        // the own class, counted from n0, if it is one of this lane's columns: in few tiles
        const int at = owns[row] - (n0 - o.n * BN);
        const bool mine = owns[row] >= 0 && at >= 0 && at < G::TB * 32 && ((at >> 2) & 1) == 0;
        if (__ballot(mine)) {
            float own = 0.f;
#pragma unroll
            for (int j = 0; j < G::TB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) own = at == j * 32 + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : own;
            if (mine) c.own_logit[m] = own;
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        float s = 0.f;
        const float base = mx == -INFINITY ? 0.f : mx;  // no class left: exp(-inf) = 0 each
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) s += exp_below<T>(acc[i][j][r], base);
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
    if (!c.grad) return;
    // All classes are in this tile (the caller's one condition for c.grad): the
    // logits' gradient for weight 1 leaves with them
#pragma unroll
    for (int i = 0; i < G::TA; ++i) {
        const int row = (wm * G::TA + i) * 32 + (lane & 31), m = o.m * BM + row;
        float mx = -INFINITY, s = 0.f;
#pragma unroll
        for (int w = 0; w < WN; ++w) mx = fmaxf(mx, top[w * BM + row]);
        const float base = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int w = 0; w < WN; ++w) s += sum[w * BM + row] * expf(top[w * BM + row] - base);
        const float lse = mx + logf(s);
        const int64_t t = m < p.m ? c.target(m) : -1;
        const bool left_out = m >= p.m || c.left_out(m), bad = !left_out && (t < 0 || t >= p.n);
#pragma unroll
        for (int j = 0; j < G::TB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = n0 + j * 32 + 8 * (r >> 2) + (r & 3);
                const float g = c.scale * (exp_below<T>(acc[i][j][r], lse) - (n == t ? 1.f : 0.f));
                acc[i][j][r] = left_out ? 0.f : bad ? NAN : g;
            }
    }
    __syncthreads();  // top and sum are read out
    constexpr int W = kWidth<T>;
    const Spot at = spot_of<G, W>(p, o.m * BM, o.n * BN);
    by_rows<G, W>(acc, lds, [&](int down, float (&v)[W]) {
        if (at.count > 0 && at.m + down < p.m)
            store_row((T *)c.grad + (at.m * c.ldgrad + at.n) + down * c.ldgrad, at.count, v);
    });
}

// The logits' gradient over one piece of the classes, from recomputed logits:
// g = weight (exp(logit - lse) - [own class]) c.scale, zero for rows left out.
// Bound as the statistics are: 3001 x 1000 x 25,088 fp16 227 us with the columns'
// sums (222 without them; a pass over G takes 32), 252 with the rows' values read
// behind each store.
template <typename T, bool BC, typename C>
__global__ __launch_bounds__(C::THREADS, 1) void grad_kernel(Product p, Classes c) {
    using G = Tile<T, false, BC, C>;
    constexpr int BM = C::BM, BN = C::BN, W = kWidth<T>;
    __shared__ __attribute__((aligned(1024))) char lds[G::LDS];
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const Place o = place(tm, tn, 1);
    static_assert(G::THREADS >= BM && G::THREADS >= BN, "a row and a column each");
    const int tid = threadIdx.x;
    // a row's class, factor and log-sum-exp, on their way while the logits are formed
    int64_t own_class = -1;
    float weight = 0.f, lse = 0.f, rel = 1.f;
    if (tid < BM && o.m * BM + tid < p.m) {
        own_class = c.target(o.m * BM + tid);
        weight = c.weight[o.m * BM + tid];
        lse = c.lse[o.m * BM + tid];
        if (c.row_scale) rel = c.row_scale[o.m * BM + tid] / *c.over;
    }
    v16f acc[G::TA][G::TB];
    G::product(acc, p, lds, o.m * BM, o.n * BN, 0, (p.k + G::BK - 1) / G::BK);
    struct Row {
        float weight, base;
        int own;    // counted from the tile's first class
        float rel;  // of the row's scale to the columns' sums'
    };
    constexpr int SLABS = 32 * (G::TB * 32 + 4) * 4 * (C::THREADS / 64);
    static_assert(SLABS + BM * (int)sizeof(Row) <= G::LDS, "the waves' rows and theirs");
    Row *const rows = (Row *)(lds + SLABS);
    if (tid < BM) {
        const int64_t t = own_class - c.first - (int64_t)o.n * BN;
        rows[tid] = Row{weight * c.scale, lse, own_class >= 0 && t >= 0 && t < BN ? (int)t : -1, rel};
    }
    __syncthreads();
    const Spot at = spot_of<G, W>(p, o.m * BM, o.n * BN);
    float bias[W];
    load_bias<T>(c.bias, c.bias_f32, at.n, at.count, bias);
    // the columns' sums, from before G is rounded (fp32: 19 additions to a lane's
    // rows and its neighbours', the rest in 64 bits)
    using Sum = std::conditional_t<sizeof(T) == 4, double, float>;
    Sum column[W] = {};
    by_rows<G, W>(acc, lds, [&](int down, float (&v)[W]) {
        const int m = at.m + down;
        if (m >= p.m || at.count <= 0) return;
        const Row row = rows[m - o.m * BM];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = row.weight == 0.f ? 0.f : row.weight * exp_below<T>(v[i] + bias[i], row.base);
        const int own = row.own - (at.n - o.n * BN);  // the own class among the lane's columns
        if (row.own >= 0 && own >= 0 && own < W) {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (i == own) v[i] -= row.weight;
        }
        if (c.sums) {
#pragma unroll
            for (int i = 0; i < W; ++i) column[i] += (Sum)(v[i] * row.rel);
        }
        store_row((T *)c.grad + (at.m * c.ldgrad + at.n) + down * c.ldgrad, at.count, v);
    });
    if (!c.sums) return;
    // over the lanes that hold other rows of the same columns, then over the waves
    constexpr int LANES = G::TB * 32 / W;
    const int wave = tid >> 6, lane = tid & 63;
    Sum *const part = (Sum *)(lds + SLABS + BM * sizeof(Row));
    static_assert(SLABS + BM * (int)sizeof(Row) + C::WM * BN * (int)sizeof(Sum) <= G::LDS, "and the waves' sums");
    static_assert((SLABS + BM * sizeof(Row)) % sizeof(Sum) == 0, "aligned");
#pragma unroll
    for (int i = 0; i < W; ++i) {
#pragma unroll
        for (int d = LANES; d < 64; d *= 2) column[i] += __shfl_xor(column[i], d);
        if (lane < LANES) part[(wave / C::WN) * BN + (wave % C::WN) * G::TB * 32 + lane * W + i] = column[i];
    }
    __syncthreads();
    if (tid < BN && o.n * BN + tid < p.n) {
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < C::WM; ++w) sum += (double)part[w * BN + tid];
        c.sums[(int64_t)o.m * p.n + o.n * BN + tid] = sum;
    }
}

}  // namespace gemm
}  // namespace rsc
