// The gated layer, forward: two projections, the activation and the product in one kernel (see gated_body.h).
#include "gated_body.h"

namespace tensile {

namespace {

template <typename T>
int choose(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &a) {
    const bool far = is_far(a.q[0], sizeof(T)) || is_far(a.p[0], sizeof(T)) || is_far(a.p[1], sizeof(T));
    if (a.M <= 32) return run_rows<T, true>(ops, s, a, far, 1, (a.R + 31) / 32 <= ops->num_cus);
    const int64_t large = ((a.M + Large::kTok - 1) / Large::kTok) * ((a.R + Large::kP / 2 - 1) / (Large::kP / 2));
    if (large >= ops->num_cus) return run_tiles<T, Large, true>(ops, s, a, far, 1);
    const int64_t small = ((a.M + Small::kTok - 1) / Small::kTok) * ((a.R + Small::kP / 2 - 1) / (Small::kP / 2));
    int64_t split = 2 * static_cast<int64_t>(ops->num_cus) / small;
    const int64_t most = a.C * static_cast<int64_t>(sizeof(T)) / 1024;
    if (split > most) split = most;
    return run_tiles<T, Small, true>(ops, s, a, far, split);
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
