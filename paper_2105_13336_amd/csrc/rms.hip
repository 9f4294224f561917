// Root-mean-square norm and its backward pass (see norm_body.h).
#include "norm_body.h"

namespace tensile {

int launch_rms_norm(const ::tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type) {
    return norm_forward<false>(ops, s, a, type, param_type);
}

int launch_rms_norm_backward(const ::tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type, void *dgamma) {
    return norm_backward<false>(ops, s, a, type, param_type, dgamma, nullptr);
}

}  // namespace tensile
