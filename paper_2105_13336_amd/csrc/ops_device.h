// Device code shared by the operators: eight columns of a row in a lane's registers, in each element type, and the
// packing of a group of 32 by four neighbouring lanes.
#pragma once

#include "ops.h"

namespace tensile {

struct bf16_t {
    uint16_t bits;
};
struct f16_t {
    uint16_t bits;
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight elements as they lie in memory.
template <typename T>
struct Raw8 {
    u32x4 v;
};
template <>
struct Raw8<float> {
    u32x4 v, w;
};

// Loads and stores take any alignment that suits the element (the hardware splits what crosses a line); `left` is how
// many of the eight exist, at least 1.  Elements beyond are zero.
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw(const T *p, int left) {
    Raw8<T> r;
    if (left >= kChunk) {
        __builtin_memcpy(&r, p, sizeof r);
    } else {
        T e[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            T z{};
            if (j < left) z = p[j];
            e[j] = z;
        }
        __builtin_memcpy(&r, e, sizeof r);
    }
    return r;
}

__device__ __forceinline__ float as_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }

__device__ __forceinline__ void widen(const Raw8<float> &r, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[j] = as_f32(r.v[j]);
        f[4 + j] = as_f32(r.w[j]);
    }
}
__device__ __forceinline__ void widen(const Raw8<bf16_t> &r, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = as_f32(r.v[j] << 16);
        f[2 * j + 1] = as_f32(r.v[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const Raw8<f16_t> &r, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f16x2 h = __builtin_bit_cast(f16x2, static_cast<uint32_t>(r.v[j]));
        f[2 * j] = static_cast<float>(h[0]);
        f[2 * j + 1] = static_cast<float>(h[1]);
    }
}

// Rounded to nearest, ties to even.
__device__ __forceinline__ void narrow(const float (&f)[8], Raw8<float> &r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        r.v[j] = as_u32(f[j]);
        r.w[j] = as_u32(f[4 + j]);
    }
}
__device__ __forceinline__ void narrow(const float (&f)[8], Raw8<bf16_t> &r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x2 p = {f[2 * j], f[2 * j + 1]};
        r.v[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
    }
}
__device__ __forceinline__ void narrow(const float (&f)[8], Raw8<f16_t> &r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x2 p = {f[2 * j], f[2 * j + 1]};
        r.v[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2));
    }
}

template <typename T>
__device__ __forceinline__ void store_raw(T *p, const Raw8<T> &r, int left) {
    if (left >= kChunk) {
        __builtin_memcpy(p, &r, sizeof r);
    } else {
        T e[kChunk];
        __builtin_memcpy(e, &r, sizeof r);
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < left) p[j] = e[j];
    }
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, int left, float (&f)[8]) {
    widen(load_raw(p, left), f);
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&f)[8], int left) {
    Raw8<T> r;
    narrow(f, r);
    store_raw(p, r, left);
}

// One element, for what is not a hot path.
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return as_f32(static_cast<uint32_t>(x.bits) << 16); }
__device__ __forceinline__ float to_f32(f16_t x) { return static_cast<float>(__builtin_bit_cast(_Float16, x.bits)); }
__device__ __forceinline__ void from_f32(float f, float &x) { x = f; }
__device__ __forceinline__ void from_f32(float f, bf16_t &x) { x.bits = __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ __forceinline__ void from_f32(float f, f16_t &x) { x.bits = __builtin_bit_cast(uint16_t, static_cast<_Float16>(f)); }

// ------------------------------------------------------------------ checkpoints

__device__ __forceinline__ u32x2 load_q(const int8_t *p, int left) {
    u32x2 w = {0, 0};
    if (left >= kChunk) {
        __builtin_memcpy(&w, p, 8);
    } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < left) w[j / 4] |= static_cast<uint32_t>(static_cast<uint8_t>(p[j])) << (8 * (j % 4));
    }
    return w;
}
__device__ __forceinline__ void store_q(int8_t *p, u32x2 w, int left) {
    if (left >= kChunk) {
        __builtin_memcpy(p, &w, 8);
    } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < left) p[j] = static_cast<int8_t>(w[j / 4] >> (8 * (j % 4)));
    }
}

// 2^(code-127): the code is the scale's exponent field; 255 stands for NaN.
__device__ __forceinline__ float scale_of(uint32_t code) { return as_f32(code == kNanCode ? 0x7fc00000u : code << 23); }

__device__ __forceinline__ void unpack8(u32x2 w, float scale, float (&f)[8]) {
    uint32_t v[2] = {w[0], w[1]};
    asm("" : "+v"(v[0]), "+v"(v[1]));  // (or the bytes are taken apart where they are loaded, by two more instructions each)
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = static_cast<float>(static_cast<int8_t>(v[j / 4] >> (8 * (j % 4)))) * scale;
}

template <int kCtrl>
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    const uint32_t y = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, 0xf, 0xf, true));
    return x > y ? x : y;
}

// The largest magnitude of a lane's eight, as the bits of a 32-bit number.  Magnitudes are compared as integers: the order is that
// of the numbers, and infinities and NaN are above all others.
__device__ __forceinline__ uint32_t largest(const float (&f)[8]) {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t m = as_u32(f[j]) & 0x7fffffffu;
        a = a > m ? a : m;
    }
    return a;
}

// The four lanes 4k .. 4k+3 hold a group's 32 values (zero where there are none) and all of them call this.
__device__ __forceinline__ u32x2 pack8(const float (&f)[8], uint32_t cap, uint32_t &code) {
    uint32_t a = largest(f);
    a = quad_max<0xB1>(a);             // quad_perm [1,0,3,2]
    a = quad_max<0x4E>(a);             // quad_perm [2,3,0,1]
    // a = m * 2^E, 1 <= m < 2: the scale is 2^(E-6), or 2^(E-5) where m >= 127.5/64 (the quotient would round to 128)
    const uint32_t up = (a + 0x10000u) >> 23;
    uint32_t c = up > 7 ? up - 6 : 1;
    const bool cut = c > cap;
    if (cut) c = cap;
    // f / scale is exact, so the one rounding is that of the sum with 1.5 * 2^23, whose low byte is the integer
    constexpr float kMiddle = 12582912.0f;
    const float inv = as_f32((254u - c) << 23);
    float b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = __builtin_fmaf(f[j], inv, kMiddle);
    if (cut) {                         // 127 scales are the most that is held
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = __builtin_amdgcn_fmed3f(b[j], kMiddle - 127.0f, kMiddle + 127.0f);
    }
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t lo = __builtin_amdgcn_perm(as_u32(b[4 * k + 1]), as_u32(b[4 * k]), 0x0c0c0400);
        const uint32_t hi = __builtin_amdgcn_perm(as_u32(b[4 * k + 3]), as_u32(b[4 * k + 2]), 0x04000c0c);
        w[k] = lo | hi;
    }
    if (a >= 0x7f800000u) {
        c = kNanCode;
        w = u32x2{0, 0};
    }
    code = c;
    return w;
}

// ------------------------------------------------------------------ sums over lanes

template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp_f32(float x) {
    return as_f32(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(as_u32(x)), kCtrl, kRowMask, 0xf, false)));
}

// The sum over a row of 16 lanes, in every lane of it (rotations by 8, 4, 2, 1).
__device__ __forceinline__ float sum16(float x) {
    x += dpp_f32<0x128, 0xf>(x);
    x += dpp_f32<0x124, 0xf>(x);
    x += dpp_f32<0x122, 0xf>(x);
    x += dpp_f32<0x121, 0xf>(x);
    return x;
}

// The sum over the 64 lanes, wave-uniform: rows 0 and 2 are added to rows 1 and 3, then lane 31 to the upper half.
__device__ __forceinline__ float sum64(float x) {
    x = sum16(x);
    x += dpp_f32<0x142, 0xa>(x);
    x += dpp_f32<0x143, 0xc>(x);
    return as_f32(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(as_u32(x)), 63)));
}

}  // namespace tensile
