// Declarations shared by the operators on 8-bit checkpoints of activations (ops.hip: handle and entry points,
// ckpt.hip: pack, unpack and GELU, norm.hip: layer norm, rms.hip: root-mean-square norm, gated.hip and gated_backward.hip: the gated layer,
// linear_grad.hip: the weight gradient).
#pragma once

#include "common.h"

#include <tuple>

namespace tensile {

constexpr int kGroup = 32;            // columns that share a scale
constexpr int kChunk = 8;             // columns a lane holds at a time: four lanes hold a group
constexpr uint32_t kNanCode = 255;

// Scratch memory of the operators on one queue (see Workspace in common.h for the rules).
struct OpsScratch {
    std::mutex mu;
    DevBuf<float> buf;
    std::vector<void *> retired;
    bool captured = false;            // belongs to a capture: it is provided while the stream is being captured
    ~OpsScratch();
    int provide(size_t floats, const char *what);
};

// The queue whose calls run one after the other and share scratch.  A stream's handle names it, but for two cases:
//   hipStreamPerThread is another queue in every host thread: `thread` is that thread's number, never given twice, else 0;
//   what is captured runs wherever the graph is launched, beside other graphs captured on that stream and beside its eager calls:
//   `capture` is the capture's number, 0 outside of one.
struct ScratchKey {
    hipStream_t stream;
    uint64_t thread;
    unsigned long long capture;
    bool operator<(const ScratchKey &o) const { return std::tie(stream, thread, capture) < std::tie(o.stream, o.thread, o.capture); }
};

struct Matrix {
    void *p;
    int64_t ld;
};

struct Ckpt {
    int8_t *q;
    uint8_t *scale;
    int64_t ld_q, ld_scale;
};

// Elementwise calls: rows x cols walked in slots of kChunk columns, 4 * ceil(cols / kGroup) slots a row.
struct EachArgs {
    int64_t rows, cols;
    Matrix a, b;                      // in, out (unused: null)
    Ckpt c, d;                        // in or out
    int32_t cap;                      // largest code
};

struct NormArgs {
    int64_t rows;
    int32_t cols;
    Matrix x, r, y, t;                // forward: input, residual, output, sum; backward: dy, dresidual, dx, -
    Ckpt c;
    float *rstd;
    const void *gamma, *beta;
    float eps;
    int32_t cap;
    float *part;                      // backward: [workgroup][2][cols], of the root-mean-square norm [workgroup][cols]
};

// The gated layer; backward h is dh and x is dx (null: not wanted).
struct GatedArgs {
    int64_t M;
    int32_t K, F;
    Matrix x, w_gate, w_up, h;
    const void *b_gate, *b_up;
    int32_t param_type, act, cap;
    Ckpt gate, up;
    Matrix dgate, dup;
    Ckpt h_c;
};

struct LinearArgs {
    int64_t M;
    int32_t N, K;
    Matrix dy;
    Ckpt c;
    const void *gamma, *beta;
    int32_t param_type;
    Matrix dw;
    int32_t dw_type;
    void *dbias;
};

// Each enqueues on the stream; types are checked by the caller.
int launch_pack(const tensile_ops *ops, hipStream_t s, const EachArgs &a, int type);
int launch_unpack(const tensile_ops *ops, hipStream_t s, const EachArgs &a, int type);
int launch_gelu(const tensile_ops *ops, hipStream_t s, const EachArgs &a, int type, bool tanh_form);
int launch_gelu_backward(const tensile_ops *ops, hipStream_t s, const EachArgs &a, int type, bool tanh_form);
int launch_norm(const tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type);
int launch_norm_backward(const tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type, void *dgamma, void *dbeta);
int launch_rms_norm(const tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type);
int launch_rms_norm_backward(const tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type, void *dgamma);
int launch_gated(const tensile_ops *ops, hipStream_t s, const GatedArgs &g, int type);
int launch_gated_backward(const tensile_ops *ops, hipStream_t s, const GatedArgs &g, int type);
int launch_linear_grad(const tensile_ops *ops, hipStream_t s, const LinearArgs &a, int type);

}  // namespace tensile

struct tensile_ops {
    int device = 0;
    int num_cus = 256;
    mutable std::mutex mu;            // guards the map
    mutable std::map<tensile::ScratchKey, std::unique_ptr<tensile::OpsScratch>> scratch;
};

namespace tensile {
// The scratch of (handle, queue), created on first use; the caller locks it while it sizes it and enqueues.
OpsScratch &ops_scratch(const tensile_ops *ops, hipStream_t stream);
}  // namespace tensile
