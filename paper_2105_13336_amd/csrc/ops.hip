// Entry points of the operators on 8-bit checkpoints: the handle, its scratch memory and the checks of the arguments.
#include "ops.h"

#include <atomic>
#include <cfloat>
#include <new>

namespace tensile {

OpsScratch::~OpsScratch() {
    for (void *p : retired) (void)hipFree(p);
}

namespace {

// While it lives, the calling thread may allocate although a stream is being captured (the allocation is no part of the graph).
struct AllocateInCapture {
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    const bool on;
    explicit AllocateInCapture(bool wanted) : on(wanted && hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess) {}
    ~AllocateInCapture() {
        if (on) (void)hipThreadExchangeStreamCaptureMode(&mode);
    }
};

uint64_t thread_number() {
    static std::atomic<uint64_t> last{0};
    thread_local const uint64_t own = ++last;
    return own;
}

// 0: not being captured (the default stream never is).
unsigned long long capture_number(hipStream_t stream) {
    if (stream == nullptr) return 0;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    unsigned long long id = 0;
    if (hipStreamGetCaptureInfo(stream, &status, &id) != hipSuccess) {
        (void)hipGetLastError();
        return 0;
    }
    return status == hipStreamCaptureStatusActive ? id : 0;
}

}  // namespace

int OpsScratch::provide(size_t floats, const char *what) {
    if (buf.p && floats <= buf.n) return TENSILE_OK;
    size_t want = floats ? floats : 1;
    const size_t least = want;
    if (want < 2 * buf.n) want = 2 * buf.n;   // at least doubled: what is parked in `retired` stays below what is in use
    retired.reserve(retired.size() + 1);
    const AllocateInCapture allowed(captured);
    float *fresh = nullptr;
    hipError_t e = device_malloc(reinterpret_cast<void **>(&fresh), want * sizeof(float));
    if (e != hipSuccess && want > least) {    // (memory for what is needed may still be there)
        (void)hipGetLastError();
        want = least;
        e = device_malloc(reinterpret_cast<void **>(&fresh), want * sizeof(float));
    }
    if (e != hipSuccess) return hip_fail(e, what);
    if (buf.p) retired.push_back(buf.p);
    buf.p = fresh;
    buf.n = want;
    buf.owned = true;
    return TENSILE_OK;
}

OpsScratch &ops_scratch(const tensile_ops *ops, hipStream_t stream) {
    const ScratchKey key{stream, stream == hipStreamPerThread ? thread_number() : 0, capture_number(stream)};
    std::lock_guard<std::mutex> g(ops->mu);
    std::unique_ptr<OpsScratch> &slot = ops->scratch[key];
    if (!slot) {
        slot.reset(new OpsScratch());
        slot->captured = key.capture != 0;
    }
    return *slot;
}

namespace {

constexpr int64_t kMostCols = int64_t{1} << 30;   // columns are counted in 32 bits
constexpr int64_t kMostRows = int64_t{1} << 40;

size_t element_size(int type) { return type == TENSILE_F32 ? 4 : 2; }
bool known_type(int type) { return type == TENSILE_F32 || type == TENSILE_BF16 || type == TENSILE_F16; }
int32_t largest_code(int type) { return type == TENSILE_F16 ? 136 : 248; }

int refuse(const char *who, const char *name, const char *why) {
    set_error("%s: %s %s", who, name, why);
    return TENSILE_E_INVAL;
}

int check_ops(const tensile_ops *ops, const char *who) {
    if (!ops) { set_error("%s: NULL handle", who); return TENSILE_E_INVAL; }
    int device = -1;
    TS_HIP(hipGetDevice(&device));
    if (device != ops->device) {
        set_error("%s: the handle belongs to device %d, the current device is %d", who, ops->device, device);
        return TENSILE_E_INVAL;
    }
    return TENSILE_OK;
}

int check_shape(int64_t rows, int64_t cols, int64_t ld, const char *who, const char *name) {
    if (rows < 0 || cols < 1) return refuse(who, name, "needs rows >= 0 and cols >= 1");
    if (rows > kMostRows || cols > kMostCols) {
        set_error("%s: %s has more than 2^40 rows or 2^30 columns", who, name);
        return TENSILE_E_RANGE;
    }
    int64_t span;
    if (ld < cols) return refuse(who, name, "has rows that overlap (ld < cols)");
    if (__builtin_mul_overflow(rows, ld, &span) || span > (int64_t{1} << 60)) {
        set_error("%s: %s spans more than 2^60 elements", who, name);
        return TENSILE_E_RANGE;
    }
    return TENSILE_OK;
}

int check_matrix(const tensile_matrix *m, const char *who, const char *name) {
    if (!m) return refuse(who, name, "is NULL");
    if (!known_type(m->type)) return refuse(who, name, "has an unknown type");
    const int rc = check_shape(m->rows, m->cols, m->ld, who, name);
    if (rc != TENSILE_OK) return rc;
    if (m->rows > 0 && !m->data) return refuse(who, name, "has no data (NULL)");
    if (reinterpret_cast<uintptr_t>(m->data) % element_size(m->type)) return refuse(who, name, "is not aligned to its elements");
    return TENSILE_OK;
}

int check_like(const tensile_matrix *m, const tensile_matrix *x, const char *who, const char *name) {
    const int rc = check_matrix(m, who, name);
    if (rc != TENSILE_OK) return rc;
    if (m->rows != x->rows || m->cols != x->cols || m->type != x->type) return refuse(who, name, "differs in shape or type");
    return TENSILE_OK;
}

int check_ckpt(const tensile_ckpt *c, int64_t rows, int64_t cols, const char *who, const char *name) {
    if (!c) return refuse(who, name, "is NULL");
    int rc = check_shape(c->rows, c->cols, c->ld_q, who, name);
    if (rc != TENSILE_OK) return rc;
    if (c->rows != rows || c->cols != cols) return refuse(who, name, "differs in shape");
    rc = check_shape(c->rows, (c->cols + kGroup - 1) / kGroup, c->ld_scale, who, name);
    if (rc != TENSILE_OK) return rc;
    if (c->rows > 0 && (!c->q || !c->scale)) return refuse(who, name, "has no data (NULL)");
    return TENSILE_OK;
}

int check_param(const void *p, int param_type, int type, const char *who, const char *name) {
    if (param_type != TENSILE_F32 && param_type != type) return refuse(who, "param_type", "is neither TENSILE_F32 nor the activations' type");
    if (!p) return refuse(who, name, "is NULL");
    if (reinterpret_cast<uintptr_t>(p) % element_size(param_type)) return refuse(who, name, "is not aligned to its elements");
    return TENSILE_OK;
}

Matrix view(const tensile_matrix *m) { return m ? Matrix{m->data, m->ld} : Matrix{nullptr, 0}; }
Ckpt view(const tensile_ckpt *c) { return c ? Ckpt{c->q, c->scale, c->ld_q, c->ld_scale} : Ckpt{nullptr, nullptr, 0, 0}; }

// What the entry points have in common: no exception leaves them.
template <typename F>
int guarded(const char *who, F f) {
    try {
        return f();
    } catch (const std::bad_alloc &) {
        set_error("%s: out of host memory", who);
        return TENSILE_E_NOMEM;
    } catch (...) {
        set_error("%s: unexpected failure", who);
        return TENSILE_E_HIP;
    }
}

#define TS_TRY(call)                          \
    do {                                      \
        const int rc_ = (call);               \
        if (rc_ != TENSILE_OK) return rc_;    \
    } while (0)

}  // namespace

}  // namespace tensile

using namespace tensile;

extern "C" {

int tensile_ops_create(tensile_ops **out) {
    return guarded("ops_create", [&]() -> int {
        if (!out) { set_error("ops_create: out is NULL"); return TENSILE_E_INVAL; }
        *out = nullptr;
        int device = 0, cus = 0;
        TS_HIP(hipGetDevice(&device));
        TS_HIP(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device));
        std::unique_ptr<tensile_ops> h(new tensile_ops());
        h->device = device;
        h->num_cus = cus > 0 ? cus : 256;
        *out = h.release();
        return TENSILE_OK;
    });
}

void tensile_ops_free(tensile_ops *ops) {
    if (!ops) return;
    (void)hipDeviceSynchronize();
    delete ops;
}

int tensile_ckpt_pack(tensile_ops *ops, const tensile_matrix *x, const tensile_ckpt *c, void *hip_stream) {
    return guarded("ckpt_pack", [&]() -> int {
        const char *who = "ckpt_pack";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(x, who, "x"));
        TS_TRY(check_ckpt(c, x->rows, x->cols, who, "c"));
        if (x->rows == 0) return TENSILE_OK;
        EachArgs a{x->rows, x->cols, view(x), {}, view(c), {}, largest_code(x->type)};
        return launch_pack(ops, static_cast<hipStream_t>(hip_stream), a, x->type);
    });
}

int tensile_ckpt_unpack(tensile_ops *ops, const tensile_ckpt *c, const tensile_matrix *y, void *hip_stream) {
    return guarded("ckpt_unpack", [&]() -> int {
        const char *who = "ckpt_unpack";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(y, who, "y"));
        TS_TRY(check_ckpt(c, y->rows, y->cols, who, "c"));
        if (y->rows == 0) return TENSILE_OK;
        EachArgs a{y->rows, y->cols, {}, view(y), view(c), {}, 0};
        return launch_unpack(ops, static_cast<hipStream_t>(hip_stream), a, y->type);
    });
}

int tensile_layer_norm(tensile_ops *ops, const tensile_matrix *x, const tensile_matrix *residual, const void *gamma,
                       const void *beta, int32_t param_type, double eps, const tensile_matrix *y,
                       const tensile_matrix *total, const tensile_ckpt *xhat, float *rstd, void *hip_stream) {
    return guarded("layer_norm", [&]() -> int {
        const char *who = "layer_norm";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(x, who, "x"));
        if (residual) TS_TRY(check_like(residual, x, who, "residual"));
        TS_TRY(check_like(y, x, who, "y"));
        if (total) TS_TRY(check_like(total, x, who, "total"));
        if (total && x->rows > 0 && total->data == y->data) return refuse(who, "total", "is y");
        if (xhat) TS_TRY(check_ckpt(xhat, x->rows, x->cols, who, "xhat"));
        TS_TRY(check_param(gamma, param_type, x->type, who, "gamma"));
        TS_TRY(check_param(beta, param_type, x->type, who, "beta"));
        if (!(eps >= 0.0 && eps <= FLT_MAX)) return refuse(who, "eps", "is negative or not a finite 32-bit number");
        if (x->rows == 0) return TENSILE_OK;
        NormArgs a{};
        a.rows = x->rows;
        a.cols = static_cast<int32_t>(x->cols);
        a.x = view(x); a.r = view(residual); a.y = view(y); a.t = view(total);
        a.c = view(xhat);
        a.rstd = rstd;
        a.gamma = gamma; a.beta = beta;
        a.eps = static_cast<float>(eps);
        if (eps > 0.0 && a.eps == 0.0f) a.eps = FLT_TRUE_MIN;             // (a constant row has no NaN then)
        a.cap = largest_code(x->type);
        return launch_norm(ops, static_cast<hipStream_t>(hip_stream), a, x->type, param_type);
    });
}

int tensile_layer_norm_backward(tensile_ops *ops, const tensile_matrix *dy, const tensile_ckpt *xhat, const float *rstd,
                                const void *gamma, int32_t param_type, const tensile_matrix *dresidual,
                                const tensile_matrix *dx, void *dgamma, void *dbeta, void *hip_stream) {
    return guarded("layer_norm_backward", [&]() -> int {
        const char *who = "layer_norm_backward";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(dy, who, "dy"));
        TS_TRY(check_ckpt(xhat, dy->rows, dy->cols, who, "xhat"));
        if (dy->rows > 0 && !rstd) return refuse(who, "rstd", "is NULL");
        if (dresidual) TS_TRY(check_like(dresidual, dy, who, "dresidual"));
        TS_TRY(check_like(dx, dy, who, "dx"));
        TS_TRY(check_param(gamma, param_type, dy->type, who, "gamma"));
        if (!dgamma != !dbeta) return refuse(who, "dgamma, dbeta", "are given one without the other");
        if (dgamma) {
            TS_TRY(check_param(dgamma, param_type, dy->type, who, "dgamma"));
            TS_TRY(check_param(dbeta, param_type, dy->type, who, "dbeta"));
        }
        if (dy->rows == 0 && !dgamma) return TENSILE_OK;
        NormArgs a{};
        a.rows = dy->rows;
        a.cols = static_cast<int32_t>(dy->cols);
        a.x = view(dy); a.r = view(dresidual); a.y = view(dx);
        a.c = view(xhat);
        a.rstd = const_cast<float *>(rstd);
        a.gamma = gamma;
        return launch_norm_backward(ops, static_cast<hipStream_t>(hip_stream), a, dy->type, param_type, dgamma, dbeta);
    });
}

int tensile_gelu(tensile_ops *ops, const tensile_matrix *x, const tensile_matrix *y, const tensile_ckpt *c,
                 int32_t tanh_form, void *hip_stream) {
    return guarded("gelu", [&]() -> int {
        const char *who = "gelu";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(x, who, "x"));
        TS_TRY(check_like(y, x, who, "y"));
        if (c) TS_TRY(check_ckpt(c, x->rows, x->cols, who, "c"));
        if (x->rows == 0) return TENSILE_OK;
        EachArgs a{x->rows, x->cols, view(x), view(y), view(c), {}, largest_code(x->type)};
        return launch_gelu(ops, static_cast<hipStream_t>(hip_stream), a, x->type, tanh_form != 0);
    });
}

int tensile_gelu_backward(tensile_ops *ops, const tensile_matrix *dy, const tensile_ckpt *c, const tensile_matrix *dx,
                          const tensile_ckpt *y_c, int32_t tanh_form, void *hip_stream) {
    return guarded("gelu_backward", [&]() -> int {
        const char *who = "gelu_backward";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(dy, who, "dy"));
        TS_TRY(check_ckpt(c, dy->rows, dy->cols, who, "c"));
        TS_TRY(check_like(dx, dy, who, "dx"));
        if (y_c) TS_TRY(check_ckpt(y_c, dy->rows, dy->cols, who, "y_c"));
        if (dy->rows == 0) return TENSILE_OK;
        EachArgs a{dy->rows, dy->cols, view(dy), view(dx), view(c), view(y_c), largest_code(dy->type)};
        return launch_gelu_backward(ops, static_cast<hipStream_t>(hip_stream), a, dy->type, tanh_form != 0);
    });
}

int tensile_linear_grad(tensile_ops *ops, const tensile_matrix *dy, const tensile_ckpt *c, const void *gamma,
                        const void *beta, int32_t param_type, const tensile_matrix *dw, void *dbias, void *hip_stream) {
    return guarded("linear_grad", [&]() -> int {
        const char *who = "linear_grad";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(dy, who, "dy"));
        if (!c) return refuse(who, "c", "is NULL");
        TS_TRY(check_ckpt(c, dy->rows, c->cols, who, "c"));
        TS_TRY(check_matrix(dw, who, "dw"));
        if (dw->rows != dy->cols || dw->cols != c->cols) return refuse(who, "dw", "is not (columns of dy) x (columns of c)");
        if (dw->type != TENSILE_F32 && dw->type != dy->type) return refuse(who, "dw", "is of neither TENSILE_F32 nor dy's type");
        if (!gamma != !beta) return refuse(who, "gamma, beta", "are given one without the other");
        if (gamma) {
            TS_TRY(check_param(gamma, param_type, dy->type, who, "gamma"));
            TS_TRY(check_param(beta, param_type, dy->type, who, "beta"));
        }
        if (dbias && reinterpret_cast<uintptr_t>(dbias) % element_size(dw->type)) return refuse(who, "dbias", "is not aligned to its elements");
        LinearArgs a{};
        a.M = dy->rows;
        a.N = static_cast<int32_t>(dy->cols);
        a.K = static_cast<int32_t>(c->cols);
        a.dy = view(dy); a.c = view(c);
        a.gamma = gamma; a.beta = beta;
        a.param_type = param_type;
        a.dw = view(dw);
        a.dw_type = dw->type;
        a.dbias = dbias;
        return launch_linear_grad(ops, static_cast<hipStream_t>(hip_stream), a, dy->type);
    });
}

}  // extern "C"
