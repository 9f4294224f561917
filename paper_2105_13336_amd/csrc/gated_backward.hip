// The gated layer, backward: the gradients of gate and up from the checkpoints, elementwise, and that of the layer's input, a product
// over both (see gated_body.h).
#include "each_device.h"
#include "gated_body.h"

namespace tensile {

namespace {

// dgate = dh*u*act'(g), dup = dh*act(g), and act(g)*u in 8 bits.  Bound by HBM: 9.1 bytes an element (bf16, with a checkpoint of h), 8192 x 2048 23 us (6.6 TB/s), 8192 x
// 10944 127 (6.4).  dx is summed from dgate and dup as they are rounded here, which the weights' gradients read too: with 16 bits that is an error of the size of dx's own
// rounding (bf16 0.0023 of its norm instead of 0.0017, f16 2.9e-4 instead of 2.1e-4 within its range), and twice the matrix instructions without it.
template <typename T, bool kDense, typename A>
__global__ __launch_bounds__(kEachThreads) void gated_grad_kernel(Walk w, Matrix dh, Ckpt gate, Ckpt up, Matrix dgate, Matrix dup, Ckpt h, uint32_t cap) {
    using S = Slot<kDense>;
    struct All {
        Raw8<T> dh;
        Held g, u;
    };
    walk<kDense>(
        w, [&](const S &s) { return All{read_raw<T>(dh, s), read_ckpt(gate, s), read_ckpt(up, s)}; },
        [&](const S &s, const All &raw) {
            float d[8], g[8], u[8], v[8];
            widen(raw.dh, d);
            unpack8(raw.g.q, scale_of(raw.g.code), g);
            unpack8(raw.u.q, scale_of(raw.u.code), u);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float value;
                const float slope = A::template slope<kRoundsTo32<T>>(g[j], value);
                v[j] = value * u[j];
                g[j] = d[j] * u[j] * slope;
                u[j] = d[j] * value;
            }
            write8<T>(dgate, s, g);
            write8<T>(dup, s, u);
            if (h.q) {
                blank(v, s);           // (a NaN group's missing columns)
                write_ckpt(h, s, v, cap);
            }
        });
}

template <typename T>
int choose(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &a) {
    const int64_t cus = ops->num_cus;
    if (a.M <= 32) {
        const int64_t tiles = (a.R + 63) / 64, steps = 2 * static_cast<int64_t>(a.C) * static_cast<int64_t>(sizeof(T)) / kRow;
        int64_t split = 2 * cus / tiles;
        if (split > steps / 4) split = steps / 4;
        if (split < 1) split = 1;
        // Four wavefronts, one workgroup to a CU, or two and two: a round of the former takes half as long, one of the latter hides where workgroups begin and end.
        // Four and two, us, bf16, tiles x length of each sum: 625 x 60 15.5 and 13.2; 750 x 512 25.2 and 23.2; 750 x 1024 38.3 and 37.5; 750 x 1500 64 and 66.5; 625 x 2048
        // 69 and 76; 1250 x 2048 128 and 132; 1024 x 512 31.5 and 27.5; 2048 x 1024 115 and 108; f32 625 x 2048 140 and 164, 1024 x 512 71 and 60.
        const int64_t n = tiles * split;
        const bool four = n <= cus || (steps >= 40 && rounds(n, cus) < 2 * rounds(n, 2 * cus));
        return run_rows<T, false>(ops, s, a, is_far<T, Rows, false>(a), split, four);
    }
    const int64_t small = tiles_of<Small, false>(a);
    const bool far = is_far<T, Few, false>(a);                           // (tiles of Small and Middle are as many tokens)
    if (small <= cus || far) return run_tiles<T, Few, false>(ops, s, a, far, parts_of(small, cus, steps_of<T, false>(a)));
    // A round of tiles, as many as the card has places for, takes 1 where they are large, 0.47 of middle size and 0.65 where they are small (two to a CU).
    // Large, middle and small (us, dx alone): 8192 x 4096 x 10944 1113, 1497 and 1442; 8192 x 768 x 2048 88, 52 and 58.
    // (In 32 bits, where the matrix instructions take 16 times as long, small tiles do, which have the registers to add up by steps.)
    if constexpr (sizeof(T) == 2) {
        const int64_t l = 100 * rounds(tiles_of<Large, false>(a), cus), m = 47 * rounds(tiles_of<Middle, false>(a), cus), n = 65 * rounds(small, 2 * cus);
        if (l <= m && l <= n && !is_far<T, Large, false>(a)) return run_tiles<T, Large, false>(ops, s, a);
        if (m <= n) return run_tiles<T, Middle, false>(ops, s, a);
    }
    return run_tiles<T, Small, false>(ops, s, a);
}

}  // namespace

int launch_gated_backward(const ::tensile_ops *ops, hipStream_t s, const GatedArgs &g, int type) {
    bool dense, dense2;
    uint32_t blocks;
    const Walk w = make_walk({g.M, g.F, g.h, g.dgate, g.gate, g.up, 0}, &dense, &blocks);
    make_walk({g.M, g.F, g.dup, {}, g.h_c, {}, 0}, &dense2, &blocks);
    const int rc = by_type(type, dense && dense2, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr bool kD = decltype(d)::value;
        auto kernel = g.act == TENSILE_SILU ? gated_grad_kernel<T, kD, Silu> : g.act == TENSILE_GELU ? gated_grad_kernel<T, kD, Gelu<false>>
                                                                                                      : gated_grad_kernel<T, kD, Gelu<true>>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kEachThreads), 0, s, w, g.h, g.gate, g.up, g.dgate, g.dup, g.h_c, static_cast<uint32_t>(g.cap));
    });
    if (rc != TENSILE_OK || !g.x.p) return rc;
    ProductArgs a{};
    a.M = g.M;
    a.C = g.F;
    a.R = g.K;
    a.q[0] = g.dgate;
    a.q[1] = g.dup;
    a.p[0] = g.w_gate;
    a.p[1] = g.w_up;
    a.out = g.x;
    if (type == TENSILE_F32) return choose<float>(ops, s, a);
    if (type == TENSILE_BF16) return choose<bf16_t>(ops, s, a);
    return choose<f16_t>(ops, s, a);
}

}  // namespace tensile
