// Elementwise operators on matrices and checkpoints: which eight columns a thread works on, their loads and stores, and the launch.
#pragma once

#include "ops_device.h"

#include <type_traits>

namespace tensile {

namespace {

constexpr int kEachThreads = 256;
constexpr int kAtOnce = 2;            // slots of a thread whose loads are under way together

// Where a thread works.  kDense: the matrices' rows follow each other without a gap and are whole groups, so all of it is one row:
// slot k is columns 8k .. 8k+7, all there.  Else slots are numbered row by row, 4 * ceil(cols / 32) to a row.  (The same sizes
// in bf16, dense against rows 32 columns further apart: 8192 x 3072 gelu 20.7 against 24.4 us, gelu_backward 24.0 against 28.9;
// 16384 x 16384 pack 137 against 149 us, gelu 232 against 266; 300 x 512 3.8 against 4.0.)
struct Walk {
    int64_t cols;
    int64_t total;                    // slots
    int64_t per_row;
};
template <bool kDense>
struct Slot {
    int64_t row, col;
    int left;                         // columns of the slot's eight that exist; below 1: none (the last group's end)
    __device__ __forceinline__ bool whole() const { return kDense || left >= kChunk; }
    __device__ __forceinline__ bool any() const { return kDense || left > 0; }
    template <typename T>
    __device__ __forceinline__ T *in(const Matrix &m) const {
        return static_cast<T *>(m.p) + (kDense ? col : row * m.ld + col);
    }
    __device__ __forceinline__ int8_t *q(const Ckpt &c) const { return c.q + (kDense ? col : row * c.ld_q + col); }
    __device__ __forceinline__ uint8_t *scale(const Ckpt &c) const { return c.scale + (kDense ? col / kGroup : row * c.ld_scale + col / kGroup); }
    __device__ __forceinline__ int count() const { return kDense ? kChunk : left; }
};

// A workgroup takes kAtOnce * 256 consecutive slots: first all loads, then the rest.
template <bool kDense, typename Load, typename Finish>
__device__ __forceinline__ void walk(const Walk &w, Load load, Finish finish) {
    constexpr int64_t kBlock = kAtOnce * kEachThreads;
    auto place = [&](int64_t slot) __attribute__((always_inline)) -> Slot<kDense> {
        if constexpr (kDense) {
            return {0, slot * kChunk, kChunk};
        } else {
            int64_t row, k;
            if (w.total <= UINT32_MAX) {
                const uint32_t r = static_cast<uint32_t>(slot) / static_cast<uint32_t>(w.per_row);
                row = r;
                k = static_cast<uint32_t>(slot) - r * static_cast<uint32_t>(w.per_row);
            } else {
                row = slot / w.per_row;
                k = slot - row * w.per_row;
            }
            const int64_t left = w.cols - k * kChunk;
            return {row, k * kChunk, left < kChunk ? static_cast<int>(left) : kChunk};
        }
    };
    for (int64_t base = blockIdx.x * kBlock; base < w.total; base += gridDim.x * kBlock) {
        if (base + kBlock <= w.total) {
            Slot<kDense> at[kAtOnce];
            decltype(load(at[0])) raw[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                at[u] = place(base + u * kEachThreads + threadIdx.x);
                raw[u] = load(at[u]);
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) finish(at[u], raw[u]);
        } else {
            for (int64_t slot = base + threadIdx.x; slot < w.total; slot += kEachThreads) {   // (a group's four lanes leave together)
                const Slot<kDense> at = place(slot);
                finish(at, load(at));
            }
        }
    }
}

template <typename T, bool kDense>
__device__ __forceinline__ Raw8<T> read_raw(const Matrix &m, const Slot<kDense> &s) {
    if (s.any()) return load_raw(s.template in<const T>(m), s.count());
    return Raw8<T>{};
}
template <typename T, bool kDense>
__device__ __forceinline__ void write8(const Matrix &m, const Slot<kDense> &s, const float (&f)[8]) {
    if (s.any()) store8(s.template in<T>(m), f, s.count());
}
struct Held {
    u32x2 q;
    uint32_t code;
};
template <bool kDense>
__device__ __forceinline__ Held read_ckpt(const Ckpt &c, const Slot<kDense> &s) {
    Held h{u32x2{0, 0}, *s.scale(c)};
    if (s.any()) h.q = load_q(s.q(c), s.count());
    return h;
}
template <bool kDense>
__device__ __forceinline__ void write_ckpt(const Ckpt &c, const Slot<kDense> &s, float (&f)[8], uint32_t cap) {
    uint32_t code;
    const u32x2 w = pack8(f, cap, code);
    if (s.any()) store_q(s.q(c), w, s.count());
    if ((threadIdx.x & 3) == 0) *s.scale(c) = static_cast<uint8_t>(code);
}
// Columns that do not exist take no part in a group's largest magnitude.
template <bool kDense>
__device__ __forceinline__ void blank(float (&f)[8], const Slot<kDense> &s) {
    if (!s.whole()) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= s.left) f[j] = 0.0f;
    }
}

Walk make_walk(const EachArgs &a, bool *dense, uint32_t *blocks) {
    auto tight = [&](const Matrix &m) { return !m.p || m.ld == a.cols || a.rows == 1; };
    auto tight_c = [&](const Ckpt &c) { return !c.q || (c.ld_q == a.cols && c.ld_scale == a.cols / kGroup) || a.rows == 1; };
    *dense = a.cols % kGroup == 0 && tight(a.a) && tight(a.b) && tight_c(a.c) && tight_c(a.d);
    Walk w{};
    w.cols = a.cols;
    w.per_row = (a.cols + kGroup - 1) / kGroup * (kGroup / kChunk);
    w.total = a.rows * w.per_row;
    const int64_t want = (w.total + kAtOnce * kEachThreads - 1) / (kAtOnce * kEachThreads);
    *blocks = static_cast<uint32_t>(want < (1 << 23) ? want : 1 << 23);
    return w;
}

// f(element, dense)
template <typename F>
int by_type(int type, bool dense, F f) {
    auto with = [&](auto t) {
        if (dense) f(t, std::true_type{});
        else f(t, std::false_type{});
    };
    if (type == TENSILE_F32) with(float{});
    else if (type == TENSILE_BF16) with(bf16_t{});
    else with(f16_t{});
    TS_HIP(hipGetLastError());
    return TENSILE_OK;
}

}  // namespace

}  // namespace tensile
