// Layer norm and its backward pass (see norm_body.h).
#include "norm_body.h"

namespace tensile {

int launch_norm(const ::tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type) {
    return norm_forward<true>(ops, s, a, type, param_type);
}

int launch_norm_backward(const ::tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type, void *dgamma, void *dbeta) {
    return norm_backward<true>(ops, s, a, type, param_type, dgamma, dbeta);
}

}  // namespace tensile
