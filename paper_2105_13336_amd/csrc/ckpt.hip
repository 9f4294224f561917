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
#include "act_device.h"
#include "each_device.h"

namespace tensile {

namespace {

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
