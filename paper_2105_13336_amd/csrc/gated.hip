// The gated layer, forward: two projections, the activation and the product in one kernel (see gated_body.h).
#include "gated_body.h"

namespace tensile {

namespace {

template <typename T>
int choose(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &a) {
    if (a.M <= 32) {
        // Few features and long sums: these are split, four wavefronts to a part, where that saves more than adding them up and its launch take (4 us, and 2.5 on the
        // host).  Whole and split, us, one call after the other: f32 (from 1536 columns) 32 x 784 x 512 14 and 9 + 4, 32 x 1024 x 512 15.4 and 11.6, 32 x 1568 x 512 20.8 and 12.8; bf16
        // (from 8192) 32 x 4096 x 800 12.9 and 12.8, 32 x 6272 x 800 17.3 and 14.0, 32 x 8192 x 800 20.0 and 14.4, 32 x 16384 x 512 51 and 17.7, 8 x 8192 x 2000 28.4 and 23.3.  Up to
        // 2.5 us of the difference a host pays that waits for each call.
        const int64_t tiles = (a.R + 31) / 32, each = steps_of<T, true>(a) / 4, fill = ops->num_cus / tiles;
        constexpr int64_t kLong = sizeof(T) == 2 ? 32 : 12, kLeast = sizeof(T) == 2 ? 4 : 2;
        const int64_t most = each >= kLong ? each / kLeast : 1;
        return run_rows<T, true>(ops, s, a, is_far<T, Rows, true>(a), fill < most ? fill : most, tiles <= ops->num_cus);
    }
    const int64_t cus = ops->num_cus, small = tiles_of<Small, true>(a);
    const bool far = is_far<T, Few, true>(a);                            // (tiles of Small are as large)
    if (small <= cus || far) return run_tiles<T, Few, true>(ops, s, a, far, parts_of(small, cus, steps_of<T, true>(a)));
    // A round of tiles, as many as the card has places for, takes 1 where they are large and 0.65 where they are small (two to a CU).  Large and small (us, with
    // checkpoints): 8192 x 4096 x 10944 1180 and 1450; 8192 x 768 x 2048 67 and 81 (both before stores went past the caches); 4096 x 768 x 2048 33 and 37; 2048 x 768 x 2048 28 and 20.
    // (In 32 bits, where the matrix instructions take 16 times as long, small tiles do, which have the registers to add up by steps.)
    if constexpr (sizeof(T) == 2) {
        if (!is_far<T, Large, true>(a) && 20 * rounds(tiles_of<Large, true>(a), cus) <= 13 * rounds(small, 2 * cus)) return run_tiles<T, Large, true>(ops, s, a);
    }
    return run_tiles<T, Small, true>(ops, s, a);
}

}  // namespace

int launch_gated(const ::tensile_ops *ops, hipStream_t s, const GatedArgs &g, int type) {
    ProductArgs a{};
    a.M = g.M;
    a.C = g.K;
    a.R = g.F;
    a.q[0] = a.q[1] = g.x;
    a.p[0] = g.w_gate;
    a.p[1] = g.w_up;
    a.bias[0] = g.b_gate;
    a.bias[1] = g.b_up;
    a.param_type = g.param_type;
    a.act = g.act;
    a.cap = g.cap;
    a.out = g.h;
    a.kept[0] = g.gate;
    a.kept[1] = g.up;
    if (type == TENSILE_F32) return choose<float>(ops, s, a);
    if (type == TENSILE_BF16) return choose<bf16_t>(ops, s, a);
    return choose<f16_t>(ops, s, a);
}

}  // namespace tensile
