// Elementwise operators on 8-bit checkpoints: pack, unpack, GELU (which leaves a checkpoint of its input) and its
// backward pass (which reads it, and may leave one of the output).
//
// All four are bound by HBM: 2 to 5 bytes an element against some 10 to 45 instructions.  A lane holds 8 consecutive
// columns (one 16-byte load in 16 bits, 8 bytes of a checkpoint), four neighbouring lanes a group, so that a group's largest
// magnitude is two moves between lanes away and no element is read twice.
#include "ops_device.h"

namespace tensile {

namespace {

constexpr int kEachThreads = 256;

// Slots are numbered row by row.  A grid that has to go on advances by `drow` rows and `dslot` slots: one division a thread.
struct Walk {
    int64_t rows, cols;
    int64_t total;                    // slots
    int64_t per_row;
    int64_t drow, dslot;
};

template <typename F>
__device__ __forceinline__ void walk(const Walk &w, F f) {
    int64_t slot = static_cast<int64_t>(blockIdx.x) * kEachThreads + threadIdx.x;
    if (slot >= w.total) return;
    int64_t row, k;
    if (w.rows == 1) {
        row = 0;
        k = slot;
    } else if (w.total <= UINT32_MAX) {
        const uint32_t r = static_cast<uint32_t>(slot) / static_cast<uint32_t>(w.per_row);
        row = r;
        k = static_cast<uint32_t>(slot) - r * static_cast<uint32_t>(w.per_row);
    } else {
        row = slot / w.per_row;
        k = slot - row * w.per_row;
    }
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kEachThreads;
    for (;;) {
        const int64_t col = k * kChunk, left = w.cols - col;
        f(row, col, left < kChunk ? static_cast<int>(left) : kChunk);
        slot += stride;
        if (slot >= w.total) return;   // (a group's four lanes leave together)
        row += w.drow;
        k += w.dslot;
        if (k >= w.per_row) {
            k -= w.per_row;
            ++row;
        }
    }
}

template <typename T>
__device__ __forceinline__ T *at(const Matrix &m, int64_t row, int64_t col) {
    return static_cast<T *>(m.p) + row * m.ld + col;
}
// (left <= 0: the slot lies behind the row's end, in its last group)
template <typename T>
__device__ __forceinline__ void read8(const Matrix &m, int64_t row, int64_t col, int left, float (&f)[8]) {
    if (left > 0) {
        load8(at<T>(m, row, col), left, f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void write8(const Matrix &m, int64_t row, int64_t col, int left, const float (&f)[8]) {
    if (left > 0) store8(at<T>(m, row, col), f, left);
}
__device__ __forceinline__ void read_ckpt(const Ckpt &c, int64_t row, int64_t col, int left, float (&f)[8]) {
    u32x2 w = {0, 0};
    if (left > 0) w = load_q(c.q + row * c.ld_q + col, left);
    unpack8(w, scale_of(c.scale[row * c.ld_scale + col / kGroup]), f);
}
__device__ __forceinline__ void write_ckpt(const Ckpt &c, int64_t row, int64_t col, int left, float (&f)[8], uint32_t cap) {
    uint32_t code;
    const u32x2 w = pack8(f, cap, code);
    if (left > 0) store_q(c.q + row * c.ld_q + col, w, left);
    if (col % kGroup == 0) c.scale[row * c.ld_scale + col / kGroup] = static_cast<uint8_t>(code);
}
// Columns that do not exist take no part in a group's largest magnitude.
__device__ __forceinline__ void blank(float (&f)[8], int left) {
    if (left < kChunk) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= left) f[j] = 0.0f;
    }
}

// Phi(x) and phi(x) from one exponential and one reciprocal: the normal distribution's tail by Abramowitz and Stegun
// 7.1.26 (error below 7.5e-8), 1 - Phi(|x|) = t*(a1 + ... + a5 t^4)*exp(-x^2/2)/2, t = 1/(1 + p|x|/sqrt 2).
__device__ __forceinline__ void normal_cdf(float x, float &cdf, float &pdf) {
    const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x);     // exp(-x^2/2)
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.23164189f, __builtin_fabsf(x), 1.0f));
    float s = __builtin_fmaf(0.5307027145f, t, -0.7265760135f);
    s = __builtin_fmaf(s, t, 0.7107068705f);
    s = __builtin_fmaf(s, t, -0.142248368f);
    s = __builtin_fmaf(s, t, 0.127414796f);
    const float tail = s * t * e;
    cdf = x < 0.0f ? tail : 1.0f - tail;
    pdf = 0.39894228040143268f * e;
}

// What y = x*p and dy/dx = p + x*dp are made of.  The tanh form: (1 + tanh u)/2 = 1/(1 + exp(-2u)).
template <bool kTanh>
__device__ __forceinline__ void gelu_parts(float x, float &p, float &dp) {
    if constexpr (kTanh) {
        const float x2 = __builtin_fminf(x * x, 1e4f);      // (from |x| = 100 on p is 0 or 1; no overflow on the way)
        const float u2 = x * __builtin_fmaf(0.071354816272f, x2, 1.5957691216f);            // 2u
        const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * u2);
        p = __builtin_amdgcn_rcpf(1.0f + e);
        dp = p * (1.0f - p) * __builtin_fmaf(0.214064448816f, x2, 1.5957691216f);           // p(1-p) * d(2u)/dx
    } else {
        normal_cdf(x, p, dp);
    }
}

template <typename T>
__global__ __launch_bounds__(kEachThreads) void pack_kernel(Walk w, Matrix x, Ckpt c, uint32_t cap) {
    walk(w, [&](int64_t row, int64_t col, int left) {
        float f[8];
        read8<T>(x, row, col, left, f);
        write_ckpt(c, row, col, left, f, cap);
    });
}

template <typename T>
__global__ __launch_bounds__(kEachThreads) void unpack_kernel(Walk w, Ckpt c, Matrix y) {
    walk(w, [&](int64_t row, int64_t col, int left) {
        float f[8];
        read_ckpt(c, row, col, left, f);
        write8<T>(y, row, col, left, f);
    });
}

template <typename T, bool kTanh>
__global__ __launch_bounds__(kEachThreads) void gelu_kernel(Walk w, Matrix x, Matrix y, Ckpt c, uint32_t cap) {
    walk(w, [&](int64_t row, int64_t col, int left) {
        float f[8], g[8];
        read8<T>(x, row, col, left, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float p, dp;
            gelu_parts<kTanh>(f[j], p, dp);
            g[j] = f[j] * p;
        }
        write8<T>(y, row, col, left, g);
        if (c.q) write_ckpt(c, row, col, left, f, cap);
    });
}

template <typename T, bool kTanh>
__global__ __launch_bounds__(kEachThreads) void gelu_backward_kernel(Walk w, Matrix dy, Ckpt c, Matrix dx, Ckpt y, uint32_t cap) {
    walk(w, [&](int64_t row, int64_t col, int left) {
        float f[8], g[8];
        read8<T>(dy, row, col, left, g);
        read_ckpt(c, row, col, left, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float p, dp;
            gelu_parts<kTanh>(f[j], p, dp);
            g[j] *= __builtin_fmaf(f[j], dp, p);
            f[j] *= p;
        }
        write8<T>(dx, row, col, left, g);
        if (y.q) {
            blank(f, left);            // (a NaN group's missing columns)
            write_ckpt(y, row, col, left, f, cap);
        }
    });
}

// Rows that follow each other without a gap are one row: no slot is left empty and none has to be found by division.
Walk make_walk(const ::tensile_ops *ops, const EachArgs &a, uint32_t *blocks) {
    Walk w{};
    w.rows = a.rows;
    w.cols = a.cols;
    const bool whole = a.cols % kGroup == 0;
    auto dense = [&](const Matrix &m) { return !m.p || m.ld == a.cols; };
    auto dense_c = [&](const Ckpt &c) { return !c.q || (c.ld_q == a.cols && c.ld_scale == a.cols / kGroup); };
    if (whole && dense(a.a) && dense(a.b) && dense_c(a.c) && dense_c(a.d)) {
        w.rows = 1;
        w.cols = a.rows * a.cols;
    }
    w.per_row = (w.cols + kGroup - 1) / kGroup * (kGroup / kChunk);
    w.total = w.rows * w.per_row;
    const int64_t want = (w.total + kEachThreads - 1) / kEachThreads;
    const int64_t most = int64_t{ops->num_cus} * 8;
    const int64_t n = want < most ? want : most;
    const int64_t stride = n * kEachThreads;
    w.drow = stride / w.per_row;
    w.dslot = stride % w.per_row;
    *blocks = static_cast<uint32_t>(n);
    return w;
}

template <typename F>
int by_type(int type, F f) {
    if (type == TENSILE_F32) f(float{});
    else if (type == TENSILE_BF16) f(bf16_t{});
    else f(f16_t{});
    TS_HIP(hipGetLastError());
    return TENSILE_OK;
}

}  // namespace

int launch_pack(const ::tensile_ops *ops, hipStream_t s, const EachArgs &a, int type) {
    uint32_t blocks;
    const Walk w = make_walk(ops, a, &blocks);
    return by_type(type, [&](auto t) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(pack_kernel<decltype(t)>), dim3(blocks), dim3(kEachThreads), 0, s, w, a.a, a.c,
                           static_cast<uint32_t>(a.cap));
    });
}

int launch_unpack(const ::tensile_ops *ops, hipStream_t s, const EachArgs &a, int type) {
    uint32_t blocks;
    const Walk w = make_walk(ops, a, &blocks);
    return by_type(type, [&](auto t) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<decltype(t)>), dim3(blocks), dim3(kEachThreads), 0, s, w, a.c, a.b);
    });
}

int launch_gelu(const ::tensile_ops *ops, hipStream_t s, const EachArgs &a, int type, bool tanh_form) {
    uint32_t blocks;
    const Walk w = make_walk(ops, a, &blocks);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto kernel = tanh_form ? gelu_kernel<T, true> : gelu_kernel<T, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kEachThreads), 0, s, w, a.a, a.b, a.c, static_cast<uint32_t>(a.cap));
    });
}

int launch_gelu_backward(const ::tensile_ops *ops, hipStream_t s, const EachArgs &a, int type, bool tanh_form) {
    uint32_t blocks;
    const Walk w = make_walk(ops, a, &blocks);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        auto kernel = tanh_form ? gelu_backward_kernel<T, true> : gelu_backward_kernel<T, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kEachThreads), 0, s, w, a.a, a.c, a.b, a.d, static_cast<uint32_t>(a.cap));
    });
}

}  // namespace tensile
