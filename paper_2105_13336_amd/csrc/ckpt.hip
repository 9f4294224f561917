// Elementwise operators on 8-bit checkpoints: pack, unpack, GELU (which leaves a checkpoint of its input) and its
// backward pass (which reads it, and may leave one of the output).
//
// All four are bound by HBM: 3 to 10 bytes an element (16 or 32 bits) against 4 instructions (unpack) to 24 (GELU).  A lane holds 8 consecutive
// columns (one 16-byte load in 16 bits, 8 bytes of a checkpoint), four neighbouring lanes a group, so that a group's largest
// magnitude is two moves between lanes away and no element is read twice.
//
// Kernel time and bytes moved: pack and unpack of 16384 x 3136 in 32 bits, one after the other, 62 + 42 us (258 MB each, together 5.0
// TB/s: the pack waits for what the unpack before it has left in the 256 MB cache; by itself it takes 42); gelu 8192 x 3072 bf16 with
// a checkpoint 27 us (127 MB, 4.7 TB/s; its instructions alone would take 15 of them); gelu_backward 16384 x 16384 bf16 with a checkpoint
// of the output 290 us (1.63 GB, 5.6 TB/s); unpack of that 129 us (0.81 GB, 6.3 TB/s).  A large copy reaches 4.9 to 5.4 TB/s.
#include "ops_device.h"

#include <type_traits>

namespace tensile {

namespace {

constexpr int kEachThreads = 256;
constexpr int kAtOnce = 2;            // slots of a thread whose loads are under way together

// Where a thread works.  kDense: the matrices' rows follow each other without a gap and are whole groups, so all of it is one row:
// slot k is columns 8k .. 8k+7, all there.  Else slots are numbered row by row, 4 * ceil(cols / 32) to a row.  (The same sizes
// in bf16, dense against rows 32 columns further apart: 8192 x 3072 gelu 20.7 against 24.4 us, gelu_backward 24.0 against 28.9;
// 16384 x 16384 pack 137 against 149 us, gelu 232 against 266; 300 x 512 3.8 against 4.0.)
struct Walk {
    int64_t cols;
    int64_t total;                    // slots
    int64_t per_row;
};
template <bool kDense>
struct Slot {
    int64_t row, col;
    int left;                         // columns of the slot's eight that exist; below 1: none (the last group's end)
    __device__ __forceinline__ bool whole() const { return kDense || left >= kChunk; }
    __device__ __forceinline__ bool any() const { return kDense || left > 0; }
    template <typename T>
    __device__ __forceinline__ T *in(const Matrix &m) const {
        return static_cast<T *>(m.p) + (kDense ? col : row * m.ld + col);
    }
    __device__ __forceinline__ int8_t *q(const Ckpt &c) const { return c.q + (kDense ? col : row * c.ld_q + col); }
    __device__ __forceinline__ uint8_t *scale(const Ckpt &c) const { return c.scale + (kDense ? col / kGroup : row * c.ld_scale + col / kGroup); }
    __device__ __forceinline__ int count() const { return kDense ? kChunk : left; }
};

// A workgroup takes kAtOnce * 256 consecutive slots: first all loads, then the rest.
template <bool kDense, typename Load, typename Finish>
__device__ __forceinline__ void walk(const Walk &w, Load load, Finish finish) {
    constexpr int64_t kBlock = kAtOnce * kEachThreads;
    auto place = [&](int64_t slot) __attribute__((always_inline)) -> Slot<kDense> {
        if constexpr (kDense) {
            return {0, slot * kChunk, kChunk};
        } else {
            int64_t row, k;
            if (w.total <= UINT32_MAX) {
                const uint32_t r = static_cast<uint32_t>(slot) / static_cast<uint32_t>(w.per_row);
                row = r;
                k = static_cast<uint32_t>(slot) - r * static_cast<uint32_t>(w.per_row);
            } else {
                row = slot / w.per_row;
                k = slot - row * w.per_row;
            }
            const int64_t left = w.cols - k * kChunk;
            return {row, k * kChunk, left < kChunk ? static_cast<int>(left) : kChunk};
        }
    };
    for (int64_t base = blockIdx.x * kBlock; base < w.total; base += gridDim.x * kBlock) {
        if (base + kBlock <= w.total) {
            Slot<kDense> at[kAtOnce];
            decltype(load(at[0])) raw[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                at[u] = place(base + u * kEachThreads + threadIdx.x);
                raw[u] = load(at[u]);
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) finish(at[u], raw[u]);
        } else {
            for (int64_t slot = base + threadIdx.x; slot < w.total; slot += kEachThreads) {   // (a group's four lanes leave together)
                const Slot<kDense> at = place(slot);
                finish(at, load(at));
            }
        }
    }
}

template <typename T, bool kDense>
__device__ __forceinline__ Raw8<T> read_raw(const Matrix &m, const Slot<kDense> &s) {
    if (s.any()) return load_raw(s.template in<const T>(m), s.count());
    return Raw8<T>{};
}
template <typename T, bool kDense>
__device__ __forceinline__ void write8(const Matrix &m, const Slot<kDense> &s, const float (&f)[8]) {
    if (s.any()) store8(s.template in<T>(m), f, s.count());
}
struct Held {
    u32x2 q;
    uint32_t code;
};
template <bool kDense>
__device__ __forceinline__ Held read_ckpt(const Ckpt &c, const Slot<kDense> &s) {
    Held h{u32x2{0, 0}, *s.scale(c)};
    if (s.any()) h.q = load_q(s.q(c), s.count());
    return h;
}
template <bool kDense>
__device__ __forceinline__ void write_ckpt(const Ckpt &c, const Slot<kDense> &s, float (&f)[8], uint32_t cap) {
    uint32_t code;
    const u32x2 w = pack8(f, cap, code);
    if (s.any()) store_q(s.q(c), w, s.count());
    if ((threadIdx.x & 3) == 0) *s.scale(c) = static_cast<uint8_t>(code);
}
// Columns that do not exist take no part in a group's largest magnitude.
template <bool kDense>
__device__ __forceinline__ void blank(float (&f)[8], const Slot<kDense> &s) {
    if (!s.whole()) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= s.left) f[j] = 0.0f;
    }
}

// GELU in 16 bits: from the distribution function to 1e-7, absolutely.  A result's rounding is larger, but for x < -5.5 in bf16, where the result is below 2e-7
// and off by up to 1 %.  (The forms for 32 bits further down are 10 to 20 % slower where the data lie in the cache: 8192 x 3072 f16
// forward 17.5 and 21.4 us, bf16 backward with a checkpoint 24.5 and 27.3.)
// The normal distribution's tail by Abramowitz and Stegun 7.1.26 (error below 7.5e-8) from one exponential and one reciprocal:
// 1 - Phi(|x|) = t*(a1 + ... + a5 t^4)*exp(-x^2/2)/2, t = 1/(1 + p|x|/sqrt 2).  e: exp(-x^2/2).
__device__ __forceinline__ float normal_tail(float x, float &e) {
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.23164189f, __builtin_fabsf(x), 1.0f));
    float s = __builtin_fmaf(0.5307027145f, t, -0.7265760135f);
    s = __builtin_fmaf(s, t, 0.7107068705f);
    s = __builtin_fmaf(s, t, -0.142248368f);
    s = __builtin_fmaf(s, t, 0.127414796f);
    return s * t * e;
}
// The tanh form: (1 + tanh u)/2 = 1/(1 + exp(-2u)).
__device__ __forceinline__ float tanh_cdf(float x, float x2) {
    const float u2 = x * __builtin_fmaf(0.071354816272f, x2, 1.5957691216f);            // 2u
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u2));
}
// (from |x| = 100 on the distribution function is 0 or 1: no overflow on the way)
__device__ __forceinline__ float capped_square(float x) { return __builtin_amdgcn_fmed3f(x * x, 0.0f, 1e4f); }

// x*P(x) = max(x, 0) - |x|*(1 - P(|x|)), in which neither a small tail nor a small x cancels.  x_capped is x, or 100 where that is larger: inf
// stays out of the product, while -inf * 0 is NaN.  (By hand: fmin and fmax cost one and two more, to quiet a NaN; `tail` brings it in.)
__device__ __forceinline__ float capped(float x) {
    float least;
    asm("v_min_f32 %0, 0x42c80000, %1" : "=v"(least) : "v"(x));
    return least;
}
__device__ __forceinline__ float from_tail(float x, float x_capped, float tail) {
    float above;
    asm("v_max_f32 %0, 0, %1" : "=v"(above) : "v"(x));
    return __builtin_fmaf(-__builtin_fabsf(x_capped), tail, above);
}

// GELU in 32 bits, to a few units of the result (the product with a distribution function that is within 1e-7 absolutely is not, where x is below
// 0 or large).  The kernels wait for memory, so that it costs little: 8192 x 8192 94 us forward and 108 backward, 94 and 105 by the form above.
// Relative norm of the error, this and that (elementary operations in 32 bits: 3.3e-8, 3.8e-8, 3.2e-8, 5.3e-8): y 2.4e-8 and 7.0e-8, dx 3.5e-8 and
// 1.1e-7; tanh y 2.4e-8 and 4.0e-8, dx 3.6e-8 and 9.6e-8.
// 1 - Phi(|x|) = R*exp(-x^2/2): R falls slowly from 1/2, a polynomial in v = |x|/(1 + 0.35|x|), whose coefficients are fitted to the least
// relative error for |x| <= 14.5 (3.1e-8; beyond, exp(-x^2/2) is 0 in 32 bits).  The 1/2 is exact and added last: a small |x| keeps all
// its bits.  capped: x, no larger than 100.
struct Normal {
    float r, e;                       // R and exp(-x^2/2)
};
__device__ __forceinline__ Normal normal(float x, float capped) {
    const float a = __builtin_fabsf(capped), v = a * __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, a, 1.0f));
    float s = __builtin_fmaf(2.196936572e-06f, v, -2.552021214e-05f);
    s = __builtin_fmaf(s, v, 9.320835806e-05f);
    s = __builtin_fmaf(s, v, -7.410841436e-05f);
    s = __builtin_fmaf(s, v, 0.0002308475395f);
    s = __builtin_fmaf(s, v, -0.002482980739f);
    s = __builtin_fmaf(s, v, -0.006802681071f);
    s = __builtin_fmaf(s, v, 0.1103606986f);
    s = __builtin_fmaf(s, v, -0.3989416219f);
    return {__builtin_fmaf(s, v, 0.5f), __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x)};
}
// The tanh form's tail: E*t with E = exp(-2|u|) <= 1 and t = 1/(1 + E).
struct Logistic {
    float tail, t;
};
__device__ __forceinline__ Logistic logistic(float x, float x2) {
    const float e = __builtin_amdgcn_exp2f(-__builtin_fabsf(x) * __builtin_fmaf(0.10294324f, x2, 2.3022082f));   // -2|u|/ln 2
    const float t = __builtin_amdgcn_rcpf(1.0f + e);
    return {e * t, t};
}

template <typename T>
constexpr bool kRoundsTo32 = sizeof(T) == 4;

template <bool kTanh, bool kTo32>
__device__ __forceinline__ float gelu(float x) {
    if constexpr (kTanh) {
        if constexpr (kTo32) return from_tail(x, capped(x), logistic(x, capped_square(x)).tail);
        return x * tanh_cdf(x, capped_square(x));
    } else {
        if constexpr (kTo32) {
            const float c = capped(x);
            const Normal n = normal(x, c);
            return from_tail(x, c, n.r * n.e);
        }
        float e;
        return from_tail(x, capped(x), normal_tail(x, e));
    }
}
// y and dy/dx = P + x*P', P the distribution function.  To 32 bits P is the tail where x is negative and 1 - tail elsewhere, and the tail is
// taken out of all but the 1, so that one rounding is the last: e*(x/sqrt(2 pi) -+ R), and of the tanh form tail*(x*t*d(2u)/dx -+ 1).
template <bool kTanh, bool kTo32>
__device__ __forceinline__ float gelu_slope(float x, float &y) {
    if constexpr (kTo32) {
        const bool negative = as_u32(x) >> 31;
        const float one = negative ? 0.0f : 1.0f;
        if constexpr (kTanh) {
            const float x2 = capped_square(x);
            const Logistic l = logistic(x, x2);
            y = from_tail(x, x, l.tail);                    // (a checkpoint holds no infinity: a tail of 0 wins over any x)
            const float m = __builtin_amdgcn_fmed3f(x, -100.0f, 100.0f) * l.t;
            return __builtin_fmaf(l.tail, __builtin_fmaf(m, __builtin_fmaf(0.214064448816f, x2, 1.5957691216f), negative ? 1.0f : -1.0f), one);
        } else {
            const float c = __builtin_amdgcn_fmed3f(x, -100.0f, 100.0f);
            const Normal n = normal(x, c);
            y = from_tail(x, c, n.r * n.e);
            return __builtin_fmaf(n.e, __builtin_fmaf(c, 0.39894228040143268f, negative ? n.r : -n.r), one);
        }
    } else if constexpr (kTanh) {
        const float x2 = capped_square(x), p = tanh_cdf(x, x2);
        const float dp = p * (1.0f - p) * __builtin_fmaf(0.214064448816f, x2, 1.5957691216f);   // p(1-p) * d(2u)/dx
        y = x * p;
        return __builtin_fmaf(x, dp, p);
    } else {
        float e;
        const float tail = normal_tail(x, e), p = x < 0.0f ? tail : 1.0f - tail;
        y = x * p;
        return __builtin_fmaf(x, 0.39894228040143268f * e, p);
    }
}

template <typename T, bool kDense>
__global__ __launch_bounds__(kEachThreads) void pack_kernel(Walk w, Matrix x, Ckpt c, uint32_t cap) {
    using S = Slot<kDense>;
    walk<kDense>(
        w, [&](const S &s) { return read_raw<T>(x, s); },
        [&](const S &s, const Raw8<T> &raw) {
            float f[8];
            widen(raw, f);
            write_ckpt(c, s, f, cap);
        });
}

template <typename T, bool kDense>
__global__ __launch_bounds__(kEachThreads) void unpack_kernel(Walk w, Ckpt c, Matrix y) {
    using S = Slot<kDense>;
    walk<kDense>(
        w, [&](const S &s) { return read_ckpt(c, s); },
        [&](const S &s, const Held &h) {
            float f[8];
            unpack8(h.q, scale_of(h.code), f);
            write8<T>(y, s, f);
        });
}

template <typename T, bool kDense, bool kTanh>
__global__ __launch_bounds__(kEachThreads) void gelu_kernel(Walk w, Matrix x, Matrix y, Ckpt c, uint32_t cap) {
    using S = Slot<kDense>;
    walk<kDense>(
        w, [&](const S &s) { return read_raw<T>(x, s); },
        [&](const S &s, const Raw8<T> &raw) {
            float f[8], g[8];
            widen(raw, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = gelu<kTanh, kRoundsTo32<T>>(f[j]);
            write8<T>(y, s, g);
            if (c.q) write_ckpt(c, s, f, cap);
        });
}

template <typename T, bool kDense, bool kTanh>
__global__ __launch_bounds__(kEachThreads) void gelu_backward_kernel(Walk w, Matrix dy, Ckpt c, Matrix dx, Ckpt y, uint32_t cap) {
    using S = Slot<kDense>;
    struct Both {
        Raw8<T> dy;
        Held x;
    };
    walk<kDense>(
        w, [&](const S &s) { return Both{read_raw<T>(dy, s), read_ckpt(c, s)}; },
        [&](const S &s, const Both &raw) {
            float f[8], g[8], v[8];
            widen(raw.dy, g);
            unpack8(raw.x.q, scale_of(raw.x.code), f);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] *= gelu_slope<kTanh, kRoundsTo32<T>>(f[j], v[j]);
            write8<T>(dx, s, g);
            if (y.q) {
                blank(v, s);           // (a NaN group's missing columns)
                write_ckpt(y, s, v, cap);
            }
        });
}

Walk make_walk(const EachArgs &a, bool *dense, uint32_t *blocks) {
    auto tight = [&](const Matrix &m) { return !m.p || m.ld == a.cols || a.rows == 1; };
    auto tight_c = [&](const Ckpt &c) { return !c.q || (c.ld_q == a.cols && c.ld_scale == a.cols / kGroup) || a.rows == 1; };
    *dense = a.cols % kGroup == 0 && tight(a.a) && tight(a.b) && tight_c(a.c) && tight_c(a.d);
    Walk w{};
    w.cols = a.cols;
    w.per_row = (a.cols + kGroup - 1) / kGroup * (kGroup / kChunk);
    w.total = a.rows * w.per_row;
    const int64_t want = (w.total + kAtOnce * kEachThreads - 1) / (kAtOnce * kEachThreads);
    *blocks = static_cast<uint32_t>(want < (1 << 23) ? want : 1 << 23);
    return w;
}

// f(element, dense)
template <typename F>
int by_type(int type, bool dense, F f) {
    auto with = [&](auto t) {
        if (dense) f(t, std::true_type{});
        else f(t, std::false_type{});
    };
    if (type == TENSILE_F32) with(float{});
    else if (type == TENSILE_BF16) with(bf16_t{});
    else with(f16_t{});
    TS_HIP(hipGetLastError());
    return TENSILE_OK;
}

}  // namespace

int launch_pack(const ::tensile_ops *, hipStream_t s, const EachArgs &a, int type) {
    uint32_t blocks;
    bool dense;
    const Walk w = make_walk(a, &dense, &blocks);
    return by_type(type, dense, [&](auto t, auto d) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(pack_kernel<decltype(t), decltype(d)::value>), dim3(blocks), dim3(kEachThreads), 0, s, w, a.a, a.c,
                           static_cast<uint32_t>(a.cap));
    });
}

int launch_unpack(const ::tensile_ops *, hipStream_t s, const EachArgs &a, int type) {
    uint32_t blocks;
    bool dense;
    const Walk w = make_walk(a, &dense, &blocks);
    return by_type(type, dense, [&](auto t, auto d) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<decltype(t), decltype(d)::value>), dim3(blocks), dim3(kEachThreads), 0, s, w, a.c, a.b);
    });
}

int launch_gelu(const ::tensile_ops *, hipStream_t s, const EachArgs &a, int type, bool tanh_form) {
    uint32_t blocks;
    bool dense;
    const Walk w = make_walk(a, &dense, &blocks);
    return by_type(type, dense, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr bool kD = decltype(d)::value;
        auto kernel = tanh_form ? gelu_kernel<T, kD, true> : gelu_kernel<T, kD, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kEachThreads), 0, s, w, a.a, a.b, a.c, static_cast<uint32_t>(a.cap));
    });
}

int launch_gelu_backward(const ::tensile_ops *, hipStream_t s, const EachArgs &a, int type, bool tanh_form) {
    uint32_t blocks;
    bool dense;
    const Walk w = make_walk(a, &dense, &blocks);
    return by_type(type, dense, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr bool kD = decltype(d)::value;
        auto kernel = tanh_form ? gelu_backward_kernel<T, kD, true> : gelu_backward_kernel<T, kD, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kEachThreads), 0, s, w, a.a, a.c, a.b, a.d, static_cast<uint32_t>(a.cap));
    });
}

}  // namespace tensile
