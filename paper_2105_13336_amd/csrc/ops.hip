// Entry points of the operators on 8-bit checkpoints: the handle, its scratch memory and the checks of the arguments.
#include "ops.h"

#include <atomic>
#include <cfloat>
#include <initializer_list>
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

#define TS_TRY(call)                          \
    do {                                      \
        const int rc_ = (call);               \
        if (rc_ != TENSILE_OK) return rc_;    \
    } while (0)

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

int check_eps(double eps, const char *who) {
    return eps >= 0.0 && eps <= FLT_MAX ? TENSILE_OK : refuse(who, "eps", "is negative or not a finite 32-bit number");
}
float held_eps(double eps) {
    const float e = static_cast<float>(eps);
    return eps > 0.0 && e == 0.0f ? FLT_TRUE_MIN : e;                     // (a row of zeros, or a constant one, has no NaN then)
}

int check_activation(int32_t activation, const char *who) {
    const bool known = activation == TENSILE_SILU || activation == TENSILE_GELU || activation == TENSILE_GELU_TANH;
    return known ? TENSILE_OK : refuse(who, "activation", "is not one of TENSILE_SILU, TENSILE_GELU, TENSILE_GELU_TANH");
}

// Where a matrix lies, in bytes: `rows` times `wide` bytes, `pitch` apart.  A result must not meet anything else that the call reads or writes: it is
// written while others read.
struct Span {
    const char *name;
    int64_t at, rows, wide, pitch;     // rows 0: nothing there
};
Span span(const tensile_matrix *m, const char *name) {
    if (!m || m->rows == 0) return {name, 0, 0, 0, 0};
    const int64_t size = static_cast<int64_t>(element_size(m->type));
    return {name, reinterpret_cast<int64_t>(m->data), m->rows, m->cols * size, m->ld * size};
}
Span span(const tensile_ckpt *c, const char *name) {
    if (!c || c->rows == 0) return {name, 0, 0, 0, 0};
    return {name, reinterpret_cast<int64_t>(c->q), c->rows, c->cols, c->ld_q};
}
Span scale_span(const tensile_ckpt *c, const char *name) {
    if (!c || c->rows == 0) return {name, 0, 0, 0, 0};
    return {name, reinterpret_cast<int64_t>(c->scale), c->rows, (c->cols + kGroup - 1) / kGroup, c->ld_scale};
}
bool identical(const Span &a, const Span &b) { return a.at == b.at && a.rows == b.rows && a.wide == b.wide && (a.rows < 2 || a.pitch == b.pitch); }

int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }        // (b > 0)
// Rows j of b, first to last of b.rows, of which a byte lies in [from, from + wide).
bool meets_row(const Span &b, int64_t from, int64_t wide) {
    const int64_t first = floor_div(from - b.wide - b.at, b.pitch) + 1, last = -floor_div(-(from + wide - b.at), b.pitch) - 1;
    return (first > 0 ? first : 0) <= (last < b.rows - 1 ? last : b.rows - 1);
}
// Whether a byte belongs to both.  Exact: rows of one may lie between those of the other, as the halves of a matrix's columns do.
bool meet(const Span &a, const Span &b) {
    if (a.rows == 0 || b.rows == 0) return false;
    if (a.at + (a.rows - 1) * a.pitch + a.wide <= b.at || b.at + (b.rows - 1) * b.pitch + b.wide <= a.at) return false;
    if (a.rows == 1) return meets_row(b, a.at, a.wide);
    if (b.rows == 1) return meets_row(a, b.at, b.wide);
    if (a.pitch == b.pitch) {
        // the first row of a, moved by the differences of row numbers that there are, against b's first
        const Span moved{b.name, b.at - (a.rows - 1) * b.pitch, a.rows + b.rows - 1, b.wide, b.pitch};
        return meets_row(moved, a.at, a.wide);
    }
    const Span &few = a.rows < b.rows ? a : b, &many = a.rows < b.rows ? b : a;
    for (int64_t i = 0; i < few.rows; ++i)
        if (meets_row(many, few.at + i * few.pitch, few.wide)) return true;
    return false;
}
// out, a result, against `others` - of which `may_be` are those that it may be itself, row for row
int check_apart(const char *who, const Span &out, std::initializer_list<Span> others, std::initializer_list<Span> may_be = {}) {
    auto refused = [&](const Span &s) {
        set_error("%s: %s overlaps %s", who, out.name, s.name);
        return TENSILE_E_INVAL;
    };
    for (const Span &s : others)
        if (meet(out, s)) return refused(s);
    for (const Span &s : may_be)
        if (!identical(out, s) && meet(out, s)) return refused(s);
    return TENSILE_OK;
}

int check_ckpt_apart(const char *who, const tensile_ckpt *c, const char *name, const char *scale_name, std::initializer_list<Span> others) {
    const Span scales = scale_span(c, scale_name);
    TS_TRY(check_apart(who, span(c, name), others));
    TS_TRY(check_apart(who, span(c, name), {scales}));
    return check_apart(who, scales, others);
}
bool same_ckpt(const tensile_ckpt *a, const tensile_ckpt *b) { return identical(span(a, ""), span(b, "")) && identical(scale_span(a, ""), scale_span(b, "")); }

int check_norm_places(const char *who, const tensile_matrix *x, const tensile_matrix *residual, const tensile_matrix *y, const tensile_matrix *total,
                      const tensile_ckpt *xhat) {
    const Span x_at = span(x, "x"), r_at = span(residual, "residual"), y_at = span(y, "y"), t_at = span(total, "total"), c_at = span(xhat, "xhat"),
               scales = scale_span(xhat, "xhat.scale");
    TS_TRY(check_apart(who, y_at, {t_at, c_at, scales}, {x_at, r_at}));
    TS_TRY(check_apart(who, t_at, {c_at, scales}, {x_at, r_at}));
    return xhat ? check_ckpt_apart(who, xhat, "xhat", "xhat.scale", {x_at, r_at}) : TENSILE_OK;
}
int check_norm_backward_places(const char *who, const tensile_matrix *dy, const tensile_ckpt *xhat, const tensile_matrix *dresidual, const tensile_matrix *dx) {
    return check_apart(who, span(dx, "dx"), {span(xhat, "xhat"), scale_span(xhat, "xhat.scale")}, {span(dy, "dy"), span(dresidual, "dresidual")});
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
        TS_TRY(check_ckpt_apart(who, c, "c", "c.scale", {span(x, "x")}));
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
        TS_TRY(check_apart(who, span(y, "y"), {span(c, "c"), scale_span(c, "c.scale")}));
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
        TS_TRY(check_eps(eps, who));
        if (x->rows == 0) return TENSILE_OK;
        TS_TRY(check_norm_places(who, x, residual, y, total, xhat));
        NormArgs a{};
        a.rows = x->rows;
        a.cols = static_cast<int32_t>(x->cols);
        a.x = view(x); a.r = view(residual); a.y = view(y); a.t = view(total);
        a.c = view(xhat);
        a.rstd = rstd;
        a.gamma = gamma; a.beta = beta;
        a.eps = held_eps(eps);
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
        TS_TRY(check_norm_backward_places(who, dy, xhat, dresidual, dx));
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

int tensile_rms_norm(tensile_ops *ops, const tensile_matrix *x, const tensile_matrix *residual, const void *gamma,
                     int32_t param_type, double eps, const tensile_matrix *y, const tensile_matrix *total,
                     const tensile_ckpt *xhat, float *rstd, void *hip_stream) {
    return guarded("rms_norm", [&]() -> int {
        const char *who = "rms_norm";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(x, who, "x"));
        if (residual) TS_TRY(check_like(residual, x, who, "residual"));
        TS_TRY(check_like(y, x, who, "y"));
        if (total) TS_TRY(check_like(total, x, who, "total"));
        if (total && x->rows > 0 && total->data == y->data) return refuse(who, "total", "is y");
        if (xhat) TS_TRY(check_ckpt(xhat, x->rows, x->cols, who, "xhat"));
        TS_TRY(check_param(gamma, param_type, x->type, who, "gamma"));
        TS_TRY(check_eps(eps, who));
        if (x->rows == 0) return TENSILE_OK;
        TS_TRY(check_norm_places(who, x, residual, y, total, xhat));
        NormArgs a{};
        a.rows = x->rows;
        a.cols = static_cast<int32_t>(x->cols);
        a.x = view(x); a.r = view(residual); a.y = view(y); a.t = view(total);
        a.c = view(xhat);
        a.rstd = rstd;
        a.gamma = gamma;
        a.eps = held_eps(eps);
        a.cap = largest_code(x->type);
        return launch_rms_norm(ops, static_cast<hipStream_t>(hip_stream), a, x->type, param_type);
    });
}

int tensile_rms_norm_backward(tensile_ops *ops, const tensile_matrix *dy, const tensile_ckpt *xhat, const float *rstd,
                              const void *gamma, int32_t param_type, const tensile_matrix *dresidual,
                              const tensile_matrix *dx, void *dgamma, void *hip_stream) {
    return guarded("rms_norm_backward", [&]() -> int {
        const char *who = "rms_norm_backward";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(dy, who, "dy"));
        TS_TRY(check_ckpt(xhat, dy->rows, dy->cols, who, "xhat"));
        if (dy->rows > 0 && !rstd) return refuse(who, "rstd", "is NULL");
        if (dresidual) TS_TRY(check_like(dresidual, dy, who, "dresidual"));
        TS_TRY(check_like(dx, dy, who, "dx"));
        TS_TRY(check_param(gamma, param_type, dy->type, who, "gamma"));
        if (dgamma) TS_TRY(check_param(dgamma, param_type, dy->type, who, "dgamma"));
        if (dy->rows == 0 && !dgamma) return TENSILE_OK;
        TS_TRY(check_norm_backward_places(who, dy, xhat, dresidual, dx));
        NormArgs a{};
        a.rows = dy->rows;
        a.cols = static_cast<int32_t>(dy->cols);
        a.x = view(dy); a.r = view(dresidual); a.y = view(dx);
        a.c = view(xhat);
        a.rstd = const_cast<float *>(rstd);
        a.gamma = gamma;
        return launch_rms_norm_backward(ops, static_cast<hipStream_t>(hip_stream), a, dy->type, param_type, dgamma);
    });
}

int tensile_gated_linear(tensile_ops *ops, const tensile_matrix *x, const tensile_matrix *w_gate, const tensile_matrix *w_up,
                         const void *b_gate, const void *b_up, int32_t param_type, int32_t activation,
                         const tensile_matrix *h, const tensile_ckpt *gate, const tensile_ckpt *up, void *hip_stream) {
    return guarded("gated_linear", [&]() -> int {
        const char *who = "gated_linear";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(x, who, "x"));
        TS_TRY(check_matrix(w_gate, who, "w_gate"));
        TS_TRY(check_like(w_up, w_gate, who, "w_up"));
        if (w_gate->type != x->type) return refuse(who, "w_gate", "is not of x's type");
        if (w_gate->cols != x->cols) return refuse(who, "w_gate", "has not the columns of x");
        if (w_gate->rows < 1) return refuse(who, "w_gate", "has no rows");
        if (w_gate->rows > kMostCols) { set_error("gated_linear: w_gate has more than 2^30 rows"); return TENSILE_E_RANGE; }
        TS_TRY(check_matrix(h, who, "h"));
        if (h->rows != x->rows || h->cols != w_gate->rows || h->type != x->type) return refuse(who, "h", "is not (rows of x) x (rows of w_gate), or not of x's type");
        if (h->rows > 0 && (h->data == x->data || h->data == w_gate->data || h->data == w_up->data)) return refuse(who, "h", "is x or a weight matrix");
        if (!b_gate != !b_up) return refuse(who, "b_gate, b_up", "are given one without the other");
        if (b_gate) {
            TS_TRY(check_param(b_gate, param_type, x->type, who, "b_gate"));
            TS_TRY(check_param(b_up, param_type, x->type, who, "b_up"));
        }
        TS_TRY(check_activation(activation, who));
        if (gate) TS_TRY(check_ckpt(gate, h->rows, h->cols, who, "gate"));
        if (up) TS_TRY(check_ckpt(up, h->rows, h->cols, who, "up"));
        if (gate && up && h->rows > 0 && (gate->q == up->q || gate->scale == up->scale)) return refuse(who, "up", "is gate");
        if (x->rows == 0) return TENSILE_OK;
        const Span x_at = span(x, "x"), wg_at = span(w_gate, "w_gate"), wu_at = span(w_up, "w_up"), h_at = span(h, "h"), g_at = span(gate, "gate"),
                   g_scales = scale_span(gate, "gate.scale"), u_at = span(up, "up"), u_scales = scale_span(up, "up.scale");
        TS_TRY(check_apart(who, h_at, {x_at, wg_at, wu_at, g_at, g_scales, u_at, u_scales}));
        if (gate) TS_TRY(check_ckpt_apart(who, gate, "gate", "gate.scale", {x_at, wg_at, wu_at, u_at, u_scales}));
        if (up) TS_TRY(check_ckpt_apart(who, up, "up", "up.scale", {x_at, wg_at, wu_at}));
        GatedArgs a{};
        a.M = x->rows;
        a.K = static_cast<int32_t>(x->cols);
        a.F = static_cast<int32_t>(w_gate->rows);
        a.x = view(x); a.w_gate = view(w_gate); a.w_up = view(w_up); a.h = view(h);
        a.b_gate = b_gate; a.b_up = b_up;
        a.param_type = param_type;
        a.act = activation;
        a.cap = largest_code(x->type);
        a.gate = view(gate); a.up = view(up);
        return launch_gated(ops, static_cast<hipStream_t>(hip_stream), a, x->type);
    });
}

int tensile_gated_linear_backward(tensile_ops *ops, const tensile_matrix *dh, const tensile_ckpt *gate, const tensile_ckpt *up,
                                  int32_t activation, const tensile_matrix *dgate, const tensile_matrix *dup,
                                  const tensile_ckpt *h_c, const tensile_matrix *w_gate, const tensile_matrix *w_up,
                                  const tensile_matrix *dx, void *hip_stream) {
    return guarded("gated_linear_backward", [&]() -> int {
        const char *who = "gated_linear_backward";
        TS_TRY(check_ops(ops, who));
        TS_TRY(check_matrix(dh, who, "dh"));
        TS_TRY(check_ckpt(gate, dh->rows, dh->cols, who, "gate"));
        TS_TRY(check_ckpt(up, dh->rows, dh->cols, who, "up"));
        TS_TRY(check_activation(activation, who));
        TS_TRY(check_like(dgate, dh, who, "dgate"));
        TS_TRY(check_like(dup, dh, who, "dup"));
        if (dh->rows > 0 && dgate->data == dup->data) return refuse(who, "dup", "is dgate");
        if (h_c) TS_TRY(check_ckpt(h_c, dh->rows, dh->cols, who, "h_c"));
        if (!w_gate != !dx || !w_up != !dx) return refuse(who, "w_gate, w_up, dx", "are given one without the others");
        if (dx) {
            TS_TRY(check_matrix(w_gate, who, "w_gate"));
            TS_TRY(check_like(w_up, w_gate, who, "w_up"));
            if (w_gate->rows != dh->cols || w_gate->type != dh->type) return refuse(who, "w_gate", "has not a row for each column of dh, or is not of dh's type");
            TS_TRY(check_matrix(dx, who, "dx"));
            if (dx->rows != dh->rows || dx->cols != w_gate->cols || dx->type != dh->type) return refuse(who, "dx", "is not (rows of dh) x (columns of w_gate), or not of dh's type");
            if (dx->rows > 0 && (dx->data == dgate->data || dx->data == dup->data || dx->data == w_gate->data || dx->data == w_up->data))
                return refuse(who, "dx", "is dgate, dup or a weight matrix");
        }
        if (dh->rows == 0) return TENSILE_OK;
        const Span dh_at = span(dh, "dh"), g_at = span(gate, "gate"), g_scales = scale_span(gate, "gate.scale"), u_at = span(up, "up"),
                   u_scales = scale_span(up, "up.scale"), wg_at = span(w_gate, "w_gate"), wu_at = span(w_up, "w_up"), dgate_at = span(dgate, "dgate"),
                   dup_at = span(dup, "dup"), dx_at = span(dx, "dx"), h_at = span(h_c, "h_c"), h_scales = scale_span(h_c, "h_c.scale");
        TS_TRY(check_apart(who, dgate_at, {g_at, g_scales, u_at, u_scales, wg_at, wu_at, dup_at, dx_at, h_at, h_scales}, {dh_at}));
        TS_TRY(check_apart(who, dup_at, {g_at, g_scales, u_at, u_scales, wg_at, wu_at, dx_at, h_at, h_scales}, {dh_at}));
        TS_TRY(check_apart(who, dx_at, {g_at, g_scales, u_at, u_scales, wg_at, wu_at, h_at, h_scales}, {dh_at}));
        if (h_c) {
            TS_TRY(check_ckpt_apart(who, h_c, "h_c", "h_c.scale", {dh_at, wg_at, wu_at}));
            if (!same_ckpt(h_c, gate)) TS_TRY(check_ckpt_apart(who, h_c, "h_c", "h_c.scale", {g_at, g_scales}));
            if (!same_ckpt(h_c, up)) TS_TRY(check_ckpt_apart(who, h_c, "h_c", "h_c.scale", {u_at, u_scales}));
        }
        GatedArgs a{};
        a.M = dh->rows;
        a.F = static_cast<int32_t>(dh->cols);
        a.h = view(dh); a.gate = view(gate); a.up = view(up); a.dgate = view(dgate); a.dup = view(dup); a.h_c = view(h_c);
        a.act = activation;
        a.cap = largest_code(dh->type);
        if (dx) {
            a.K = static_cast<int32_t>(dx->cols);
            a.w_gate = view(w_gate); a.w_up = view(w_up); a.x = view(dx);
        }
        return launch_gated_backward(ops, static_cast<hipStream_t>(hip_stream), a, dh->type);
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
        TS_TRY(check_apart(who, span(y, "y"), {}, {span(x, "x")}));
        if (c) TS_TRY(check_ckpt_apart(who, c, "c", "c.scale", {span(x, "x"), span(y, "y")}));
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
        TS_TRY(check_apart(who, span(dx, "dx"), {span(c, "c"), scale_span(c, "c.scale")}, {span(dy, "dy")}));
        if (y_c) TS_TRY(check_ckpt_apart(who, y_c, "y_c", "y_c.scale", {span(dy, "dy"), span(dx, "dx")}));
        if (y_c && !same_ckpt(y_c, c)) TS_TRY(check_ckpt_apart(who, y_c, "y_c", "y_c.scale", {span(c, "c"), scale_span(c, "c.scale")}));
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
        TS_TRY(check_apart(who, span(dw, "dw"), {span(dy, "dy"), span(c, "c"), scale_span(c, "c.scale")}));
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
