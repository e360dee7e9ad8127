// One AdamW step over many tensors at once, the moments in 32 bits or in 8.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8 bits: blocks of 256 elements with their largest value s. The first moment
// is s (q / 127) |q / 127|, q in -127 .. 127; the second is held as its root,
// s (q / 255)^2, q in 0 .. 255, so that both resolve values far below the
// block's largest (6e-5 and 1.5e-5 of it). A step changes v by a thousandth,
// less than a code: codes are rounded up or down at random in proportion
// (SplitMix64 of seed, step and element), so that the changes add up. A root
// above zero keeps a code of at least 1, which bounds m / sqrt(v).
//
// Bound by memory (400M fp32 parameters with 8 bits 1.55 ms, 4.1 TB/s; 381M bf16
// ones with masters, 28 bytes each, 2.09 ms, 5.1 TB/s, parts of them in the caches) and, for
// small steps, by the launch: every value is read and written once, 256 threads take
// 4,096 consecutive elements of a tensor, a wave 256 at a time (one block of
// codes: its largest value is a reduction over the wave). All tensors of a
// launch are in its arguments, so that a captured launch holds them.
//
// Each operation rounds by itself (no contraction): the step is defined to the
// bit, and codes next to a border do not hang on the compiler.
#include "rsc_internal.h"
#include "adamw.h"

namespace rsc {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int8_t v4c __attribute__((ext_vector_type(4)));
typedef uint8_t v4u __attribute__((ext_vector_type(4)));

struct AdamwTensor : rsc_adamw_tensor_t {
    int32_t aligned;  // every pointer to 16 bytes
};

constexpr int kTensors = 44;  // of a launch: their descriptors fit 4 KB of arguments
constexpr int kChunk = 4096;  // elements a thread block

struct Batch {
    AdamwTensor t[kTensors];
    uint64_t first[kTensors];      // number of the tensor's first random word
    int32_t end[kTensors];         // thread blocks up to and with the tensor
    int32_t count;
};
static_assert(sizeof(Batch) + sizeof(AdamwRates) + 64 <= 4096, "kernel arguments");

// what depends on the step's number
struct Now {
    float rate, unbias;
    int64_t step;
};

__device__ __forceinline__ Now now_of(int64_t t, const AdamwRates &a) {
    Now now;
    now.step = t;
    now.rate = (float)(a.lr / (1.0 - pow(a.beta1, (double)t)));
    now.unbias = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)t)));
    return now;
}

// step += 1, and the bias corrections for it
__global__ void begin_kernel(int64_t *step, AdamwRates a, Now *now) {
    const int64_t t = *step + 1;
    *step = t;
    *now = now_of(t, a);
}

// SplitMix64 (Steele, Lea and Flood 2014): output `number` is mix(seed + number kGamma)
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;
__device__ __forceinline__ uint64_t mix(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// the largest of the wave's non-negative values; as integers, so that a NaN is
// above all and is kept
__device__ __forceinline__ float wave_max(float x) {
    uint32_t v = __float_as_uint(x);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return __uint_as_float(v);
}

__device__ __forceinline__ float decode(float code, float by) {
#pragma clang fp contract(off)
    const float w = code * by;
    return w * fabsf(w);
}

// The code by its definition, every operation rounded: min(floor(sqrt(x /
// scale) levels + u), levels), scale taken as 1 where it is 0.
__device__ __noinline__ float encode_exactly(float x, float scale, float levels, float u) {
#pragma clang fp contract(off)
    const float share = x / (scale > 0.f ? scale : 1.f);
    return fminf(floorf(sqrtf(share) * levels + u), levels);
}
// The same from the hardware's reciprocal and root (1 ulp each, so within
// levels 2^-21 with the roundings), and by the definition only where that
// could be on the other side of a whole number: 2 levels 2^-21 of all values.
// `inverse`: about 1 / scale. (The exact divisions and roots of two codes made
// the step bound by instructions: 1,888 us for 400M parameters.)
__device__ __forceinline__ float encode(float x, float scale, float inverse, float levels, uint32_t bits) {
    const float u = (float)bits * 0x1p-24f;
    const float a = fmaf(__builtin_amdgcn_sqrtf(x * inverse), levels, u);
    const float f = floorf(a), part = a - f, near = levels * 0x1p-21f;
    // written so that a NaN goes the exact way too
    if (!(part > near && part < 1.f - near)) return encode_exactly(x, scale, levels, u);
    return fminf(f, levels);
}

template <typename T, int COUNT>
__device__ __forceinline__ void get4(const T *p, int n, bool vec, T (&v)[COUNT]) {
    typedef T v4 __attribute__((ext_vector_type(4)));
    if (vec) {
        const v4 x = *(const v4 *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : (T)0;
    }
}
// STREAM: past the caches
template <bool STREAM, typename T, int COUNT>
__device__ __forceinline__ void put4(T *p, int n, bool vec, const T (&v)[COUNT]) {
    typedef T v4 __attribute__((ext_vector_type(4)));
    if (vec) {
        v4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
        if (STREAM) __builtin_nontemporal_store(x, (v4 *)p);
        else *(v4 *)p = x;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = v[i];
    }
}

// the tensor of a thread block (the first one whose last block is not before
// it) and the block's number within it
__device__ __forceinline__ int tensor_of(const Batch &b, int64_t *chunk) {
    int lo = 0, hi = b.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if ((int)blockIdx.x < b.end[mid]) hi = mid;
        else lo = mid + 1;
    }
    *chunk = (int64_t)blockIdx.x - (lo ? b.end[lo - 1] : 0);
    return lo;
}

// what a thread reads for four elements
template <typename T, bool CODES>
struct Four {
    // the value that the step is applied to: master, or for 16-bit parameters
    // without masters param
    T grad[4], param[4];
    float master[4], m[4], v[4], qs, rs;
    int8_t q[4];
    uint8_t c[4];
    int n;  // of the four that exist, 0 or less past the end
    bool vec;

    __device__ __forceinline__ void read(const AdamwTensor &t, int64_t at) {
        n = (int)max((int64_t)0, min((int64_t)4, t.n - at));
        vec = t.aligned && n == 4;
        get4((const T *)t.grad + at, n, vec, grad);
        if constexpr (sizeof(T) == 4) {
            get4(t.master ? t.master + at : (const float *)t.param + at, n, vec, master);
        } else {
            if (t.master) get4(t.master + at, n, vec, master);
            else get4((const T *)t.param + at, n, vec, param);
        }
        if (CODES) {
            get4((const int8_t *)t.exp_avg + at, n, vec, q);
            get4((const uint8_t *)t.exp_avg_sq + at, n, vec, c);
            qs = t.exp_avg_scale[at >> 8];
            rs = t.exp_avg_sq_scale[at >> 8];
        } else {
            get4((const float *)t.exp_avg + at, n, vec, m);
            get4((const float *)t.exp_avg_sq + at, n, vec, v);
        }
    }
};

constexpr int kTurns = kChunk / 1024;  // times that a wave takes 256 elements
constexpr uint64_t kArrival = 1ull << 40;

// ONE: the only launch of a step, which counts it as well: every block adds an
// arrival in the upper 24 bits of *step (the lower 40 are the steps until now,
// unchanged until all have arrived) and forms the bias corrections itself, the
// last one takes the arrivals off and adds the step. Saves the launch of
// begin_kernel where a step is no longer than launches are.
template <typename T, bool CODES, bool ONE>
__global__ __launch_bounds__(256) void step_kernel(Batch b, AdamwRates a, const Now *now_dev, int64_t *step) {
#pragma clang fp contract(off)
    int64_t chunk;
    const int which = tensor_of(b, &chunk);
    const AdamwTensor t = b.t[which];
    const int64_t wave_from = chunk * kChunk + (int64_t)(threadIdx.x >> 6) * 256;
    const int64_t from = wave_from + (threadIdx.x & 63) * 4;
    // ONE: all reads go out first, behind them the step's number. A long step is
    // faster with a turn's reads at a time and twice the waves (8 bits: 515 us
    // for 133M parameters against 645).
    Four<T, CODES> x[ONE ? kTurns : 1];
    if (ONE) {
#pragma unroll
        for (int k = 0; k < kTurns; ++k)
            if (wave_from + k * 1024 < t.n) x[ONE ? k : 0].read(t, from + k * 1024);
    }
    float rate, unbias;
    int64_t number;
    if (ONE) {
        __shared__ Now shared;
        if (threadIdx.x == 0) {
            const uint64_t old = atomicAdd((unsigned long long *)step, (unsigned long long)kArrival);
            if ((old >> 40) == gridDim.x - 1)
                atomicAdd((unsigned long long *)step, (unsigned long long)(1 - kArrival * gridDim.x));
            shared = now_of((int64_t)(old & (kArrival - 1)) + 1, a);
        }
        __syncthreads();
        rate = shared.rate;
        unbias = shared.unbias;
        number = shared.step;
    } else {
        rate = now_dev->rate;
        unbias = now_dev->unbias;
        number = now_dev->step;
    }
    const uint64_t base = (uint64_t)number * (1ull << 40) + b.first[which] + 1;
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
        const int64_t at = from + k * 1024;
        if (wave_from + k * 1024 >= t.n) break;  // the whole wave is past the end
        if (!ONE) x[0].read(t, at);
        const Four<T, CODES> &f = x[ONE ? k : 0];
        float p[4], m[4], r[4], v[4];
        uint32_t m_bits = 0, r_bits = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float g = (float)f.grad[i];
            if constexpr (sizeof(T) == 4) p[i] = f.master[i];
            else p[i] = t.master ? f.master[i] : (float)f.param[i];
            if (CODES) {
                m[i] = decode((float)f.q[i], (float)(1.0 / 127)) * f.qs;
                const float root = decode((float)f.c[i], (float)(1.0 / 255)) * f.rs;
                v[i] = root * root;
            } else {
                m[i] = f.m[i];
                v[i] = f.v[i];
            }
            m[i] = m[i] * a.b1 + g * a.c1;
            v[i] = v[i] * a.b2 + (g * a.c2) * g;
            r[i] = sqrtf(v[i]);
            p[i] = p[i] * a.keep - (m[i] * rate) / (r[i] * unbias + a.eps);
            if (CODES && i < f.n) {
                m_bits = max(m_bits, __float_as_uint(fabsf(m[i])));
                r_bits = max(r_bits, __float_as_uint(r[i]) & 0x7fffffffu);
            }
        }
        if (t.master) put4<!ONE>(t.master + at, f.n, f.vec, p);
        {
            T y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (T)p[i];
            put4<!ONE>((T *)t.param + at, f.n, f.vec, y);
        }
        if (CODES) {
            const float m_top = wave_max(__uint_as_float(m_bits)), r_top = wave_max(__uint_as_float(r_bits));
            const float m_inv = __builtin_amdgcn_rcpf(m_top > 0.f ? m_top : 1.f);
            const float r_inv = __builtin_amdgcn_rcpf(r_top > 0.f ? r_top : 1.f);
            int8_t q[4];
            uint8_t c[4];
            uint64_t word = a.seed + (base + (uint64_t)at) * kGamma;
#pragma unroll
            for (int i = 0; i < 4; ++i, word += kGamma) {
                const uint64_t z = mix(word);
                const float qm = encode(fabsf(m[i]), m_top, m_inv, 127.f, (uint32_t)(z & 0xffffffu));
                q[i] = (int8_t)(m[i] < 0.f ? -qm : qm);
                const float qr = encode(r[i], r_top, r_inv, 255.f, (uint32_t)((z >> 24) & 0xffffffu));
                c[i] = (uint8_t)(r[i] > 0.f ? fmaxf(qr, 1.f) : qr);
            }
            put4<!ONE>((int8_t *)t.exp_avg + at, f.n, f.vec, q);
            put4<!ONE>((uint8_t *)t.exp_avg_sq + at, f.n, f.vec, c);
            if ((threadIdx.x & 63) == 0) {
                t.exp_avg_scale[at >> 8] = m_top;
                t.exp_avg_sq_scale[at >> 8] = r_top;
            }
        } else {
            put4<!ONE>((float *)t.exp_avg + at, f.n, f.vec, m);
            put4<!ONE>((float *)t.exp_avg_sq + at, f.n, f.vec, v);
        }
    }
}

// the values that 8-bit moments stand for
__global__ __launch_bounds__(256) void moments_kernel(Batch b) {
#pragma clang fp contract(off)
    int64_t chunk;
    const AdamwTensor t = b.t[tensor_of(b, &chunk)];
    const int64_t from = chunk * kChunk + threadIdx.x * 4;
    int8_t q[kTurns][4];
    uint8_t c[kTurns][4];
    float qs[kTurns], rs[kTurns];
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
        const int64_t at = from + k * 1024;
        if (at >= t.n) break;
        const int n = (int)min((int64_t)4, t.n - at);
        get4((const int8_t *)t.exp_avg + at, n, t.aligned && n == 4, q[k]);
        get4((const uint8_t *)t.exp_avg_sq + at, n, t.aligned && n == 4, c[k]);
        qs[k] = t.exp_avg_scale[at >> 8];
        rs[k] = t.exp_avg_sq_scale[at >> 8];
    }
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
        const int64_t at = from + k * 1024;
        if (at >= t.n) break;
        const int n = (int)min((int64_t)4, t.n - at);
        const bool vec = t.aligned && n == 4;
        float m[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = decode((float)q[k][i], (float)(1.0 / 127)) * qs[k];
            const float root = decode((float)c[k][i], (float)(1.0 / 255)) * rs[k];
            v[i] = root * root;
        }
        put4<true>(t.master + at, n, vec, m);
        put4<true>((float *)t.param + at, n, vec, v);
    }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// f(batch, thread blocks) for the tensors in groups that fit a launch
template <typename F>
hipError_t in_batches(const rsc_adamw_tensor_t *t, int32_t count, F f) {
    Batch b;
    b.count = 0;
    int64_t blocks = 0;
    uint64_t first = 0;
    hipError_t e = hipSuccess;
    auto flush = [&] {
        if (b.count && e == hipSuccess) e = f(b, (unsigned)blocks);
        b.count = 0;
        blocks = 0;
    };
    for (int32_t i = 0; i < count; ++i) {
        const rsc_adamw_tensor_t &x = t[i];
        if (x.n == 0) continue;
        const int64_t need = ceil_div(x.n, kChunk);
        if (b.count == kTensors || blocks + need > (int64_t(1) << 23)) flush();  // 2^31 threads a launch
        blocks += need;
        static_cast<rsc_adamw_tensor_t &>(b.t[b.count]) = x;
        // 16-bit parameters and codes move by 8 and 4 bytes, which 16 covers
        b.t[b.count].aligned = aligned16(x.param) && aligned16(x.grad) && aligned16(x.exp_avg) &&
                               aligned16(x.exp_avg_sq) && aligned16(x.master);
        b.first[b.count] = first;
        b.end[b.count] = (int32_t)blocks;
        ++b.count;
        first += (uint64_t)ceil_div(x.n, 256) * 256;
    }
    flush();
    return e;
}

}  // namespace

size_t adamw_ws_bytes() { return 256; }
static_assert(sizeof(Now) <= 256, "workspace");

namespace {
template <bool ONE>
hipError_t step_launch(int32_t dtype, int32_t codes, const Batch &b, unsigned blocks, const AdamwRates &a,
                       const Now *now, int64_t *step, hipStream_t stream) {
    if (dtype == 0 && codes) step_kernel<float, true, ONE><<<blocks, 256, 0, stream>>>(b, a, now, step);
    else if (dtype == 0) step_kernel<float, false, ONE><<<blocks, 256, 0, stream>>>(b, a, now, step);
    else if (dtype == 1 && codes) step_kernel<__bf16, true, ONE><<<blocks, 256, 0, stream>>>(b, a, now, step);
    else if (dtype == 1) step_kernel<__bf16, false, ONE><<<blocks, 256, 0, stream>>>(b, a, now, step);
    else if (codes) step_kernel<_Float16, true, ONE><<<blocks, 256, 0, stream>>>(b, a, now, step);
    else step_kernel<_Float16, false, ONE><<<blocks, 256, 0, stream>>>(b, a, now, step);
    return hipGetLastError();
}
// a step of at most this many thread blocks, in one launch, counts itself
constexpr unsigned kOneLaunch = 1024;
}  // namespace

hipError_t adamw_launch(int32_t dtype, int32_t codes, const rsc_adamw_tensor_t *t, int32_t count, const AdamwRates &a,
                        int64_t *step, void *ws, hipStream_t stream) {
    Now *now = (Now *)ws;
    int64_t blocks = 0, tensors = 0;
    for (int32_t i = 0; i < count; ++i) {
        blocks += ceil_div(t[i].n, kChunk);
        tensors += t[i].n > 0;
    }
    const bool one = blocks > 0 && blocks <= kOneLaunch && tensors <= kTensors;
    if (!one) {
        begin_kernel<<<1, 1, 0, stream>>>(step, a, now);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return in_batches(t, count, [&](const Batch &b, unsigned n) {
        return one ? step_launch<true>(dtype, codes, b, n, a, now, step, stream)
                   : step_launch<false>(dtype, codes, b, n, a, now, step, stream);
    });
}

hipError_t adamw_moments_launch(const rsc_adamw_tensor_t *t, int32_t count, float *const *m, float *const *v,
                                hipStream_t stream) {
    for (int32_t i = 0; i < count;) {
        // the outputs stand where the parameters do in a step
        rsc_adamw_tensor_t some[kTensors];
        int32_t have = 0;
        for (; i < count && have < kTensors; ++i) {
            some[have] = t[i];
            some[have].param = v[i];
            some[have].grad = nullptr;
            some[have].master = m[i];
            ++have;
        }
        const hipError_t e = in_batches(some, have, [&](const Batch &b, unsigned blocks) {
            moments_kernel<<<blocks, 256, 0, stream>>>(b);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rsc
