// The matrix products of the gated layer, forward (gated.hip) and backward (gated_backward.hip):
//   g[m,f] = sum_k x[m,k]*Wg[f,k],  u[m,f] = sum_k x[m,k]*Wu[f,k]          (and from both act(g)*u, in the registers that hold them)
//   dx[m,k] = sum_f dgate[m,f]*Wg[f,k] + sum_f dup[m,f]*Wu[f,k]
//
// Long batches are bound by the matrix instructions and the clock that the chip can keep up with them (1.6 to 1.7 GHz, 64 to 72 % of its cycles): 8192 x 4096 x
// 10944 bf16 1084 to 1089 us (1350 TFLOP/s; a library's product of the same size alone 1115 to 1124), with checkpoints 1115 to 1133; backward 1090 to 1107 after 143 for the
// elementwise part (a library's product alone, weights as they lie, 1040 to 1080).  These are the best of loops over the one call; with inputs in turn and other kernels
// between, on a chip that is warm, the products take 1200 to 1260 and 1110 to 1250.  f32 2048 x 4096 x 4096 970 us (141 TFLOP/s of 157), backward 1005 + 20.6
// (137).  Single tokens are bound by the weights' bytes: 1 x 4096 x 10944 38 us (4.7 TB/s), 1 x 4096 x 43776 120 (6.0).
//
// On the matrix instructions with 32-bit sums: bf16 and f16 as they are, f32 on those for 32 bits (products and sums as in ordinary arithmetic).
// A block of the result is 32 x 32; its rows are weights (f, or k backward) and its columns tokens, so that a lane holds 16 of the 32
// features of one token, and gate and up of the same f and m lie in the same register of two blocks.
#pragma once

#include "act_device.h"

#include <type_traits>

namespace tensile {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// (the LDS-direct loads below take their target from m0, which the compiler counts as its own and says so)
#pragma clang diagnostic ignored "-Winline-asm"

typedef const __attribute__((address_space(1))) char *global_bytes;
typedef __attribute__((address_space(3))) char lds_char;

constexpr uint32_t kXcds = 8;

template <typename T>
constexpr int kPer16 = 16 / static_cast<int>(sizeof(T));   // elements of 16 bytes

// c += the product of what 16 bytes of each lane hold: lane l has row (or column) l % 32 and of the summed index the values
// (l / 32) * kPer16 onwards.
__device__ __forceinline__ f32x16 multiply_add(bf16_t, u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply_add(f16_t, u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply_add(float, u32x4 a, u32x4 b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(as_f32(a[j]), as_f32(b[j]), c, 0, 0, 0);
    return c;
}

// 16 bytes of a row of `n` elements (kPer16 at least) from element c on, zeros behind the last one: the load takes what exists, and as many before, which are
// shifted out.
template <typename T>
__device__ __forceinline__ u32x4 load_end(const T *row, int64_t c, int64_t n, bool keep) {
    constexpr int kPer = kPer16<T>;
    const int64_t left = n - c;
    const int over = left < kPer && left > 0 ? kPer - static_cast<int>(left) : 0;
    u32x4 r;
    __builtin_memcpy(&r, row + (left > 0 ? c - over : 0), 16);
    r = shift_out(r, over * static_cast<int>(sizeof(T)));
    const u32x4 none = {0, 0, 0, 0};
    return keep && left > 0 ? r : none;
}
// The same of any row, element by element.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T *p, int64_t left) {
    constexpr int kPer = kPer16<T>;
    u32x4 r = {0, 0, 0, 0};
    if (left >= kPer) {
        __builtin_memcpy(&r, p, 16);
    } else if (left > 0) {
        T e[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            T z{};
            if (j < left) z = p[j];
            e[j] = z;
        }
        __builtin_memcpy(&r, e, 16);
    }
    return r;
}

// ------------------------------------------------------------------ what the kernels are given

struct ProductArgs {
    int64_t M;                        // tokens
    int32_t C;                        // length of a sum (backward: of each of the two)
    int32_t R;                        // features of the result
    int32_t n_whole;                  // steps of a sum that can be brought whole (of each of the two)
    Matrix q[2];                      // tokens x C: x, or dgate and dup
    Matrix p[2];                      // Wg, Wu: R x C forward, C x R backward
    // forward
    const void *bias[2];
    int32_t param_type, act, cap;
    Matrix out;                       // h, or dx
    Ckpt kept[2];
    // how the work is cut: tiles of tokens and features, and the steps of a sum among `split` workgroups a tile
    uint32_t tiles_m, tiles_r, split;
    float *part;                      // split > 1: [tile][split][gate, up][token][feature]
};

template <typename T>
__device__ __forceinline__ float param_at(int type, const void *p, int64_t at) {
    return type == TENSILE_F32 ? static_cast<const float *>(p)[at] : to_f32(static_cast<const T *>(p)[at]);
}

// What becomes of the sums of a wavefront's kPB blocks (32 rows each) of 32 tokens.  They go through the LDS, so that a lane has eight features of a token and a
// store whole lines of memory, in a loop: in registers it takes a copy of all of this for every block, and spills (8192 x 4096 x 10944 with checkpoints 1356 us against
// 1278, the rest unchanged).  It takes 7 us a tile of 256 x 128, 10 with checkpoints, of which the stores are most and the activation 2: 8192 x 256 x 2048, two tiles
// to a CU, 32 and 39 us, without all of this 17.
template <int kPB_, bool kForward>
struct Exchange {
    static constexpr int kPB = kPB_, kWide = kForward ? kPB * 16 : kPB * 32;           // features
    static constexpr int kPitch = kWide + 4;                                           // floats from a token to the next: 16 lanes' 16 bytes lie in different banks
    static constexpr int kBytes = 32 * kPitch * 4 * (kForward ? 2 : 1);                // of a wavefront
    static constexpr int kLanes = kWide / 8, kAtOnce = 64 / kLanes;                    // a token's lanes, tokens at once
    static constexpr int kPasses = (32 + kAtOnce - 1) / kAtOnce;
    static constexpr bool kEven = kLanes * kAtOnce == 64 && 32 % kAtOnce == 0;         // every lane has a token in every pass

    // Block b of the blocks, as the matrix instructions leave it: a lane has rows 8q + 4 (lane / 32) .. + 3 of token lane % 32.
    static __device__ __forceinline__ void put(float *region, int b, const f32x16 &acc) {
        const int lane = threadIdx.x & 63, plane = kForward ? b & 1 : 0, at = (kForward ? b / 2 : b) * 32;
        float *const to = region + plane * 32 * kPitch + (lane & 31) * kPitch + at + 4 * (lane >> 5);
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4 *>(to + 8 * q) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    }
    // Eight features of a token, kRegions wavefronts' sums added up.
    template <int kRegions>
    static __device__ __forceinline__ void get(const float *region, int plane, int token, float (&v)[8]) {
        const int lane = threadIdx.x & 63;
        const float *from = region + plane * 32 * kPitch + token * kPitch + lane % kLanes * 8;
        f32x4 lo = *reinterpret_cast<const f32x4 *>(from), hi = *reinterpret_cast<const f32x4 *>(from + 4);
#pragma unroll
        for (int k = 1; k < kRegions; ++k) {
            from += kBytes / 4;
            lo += *reinterpret_cast<const f32x4 *>(from);
            hi += *reinterpret_cast<const f32x4 *>(from + 4);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = lo[j];
            v[4 + j] = hi[j];
        }
    }
    // (a wavefront's LDS accesses are in order; this keeps the compiler from changing it)
    static __device__ __forceinline__ void order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
};

// Where a token's eight features go, h or dx and their places in the checkpoints.
template <typename T, bool kForward>
struct Target {
    T *out;
    int8_t *q[2] = {};
    uint8_t *scale[2] = {};
    __device__ __forceinline__ Target(const ProductArgs &a, int64_t token, int r) : out(static_cast<T *>(a.out.p) + token * a.out.ld + r) {
        if constexpr (kForward) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (a.kept[k].q) {
                    q[k] = a.kept[k].q + token * a.kept[k].ld_q + r;
                    scale[k] = a.kept[k].scale + token * a.kept[k].ld_scale + r / kGroup;
                }
        }
    }
    __device__ __forceinline__ void go_on(const ProductArgs &a, int tokens) {
        out += tokens * a.out.ld;
        if constexpr (kForward) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (a.kept[k].q) {
                    q[k] += tokens * a.kept[k].ld_q;
                    scale[k] += tokens * a.kept[k].ld_scale;
                }
        }
    }
};
template <typename T>
__device__ __forceinline__ void load_bias(const ProductArgs &a, int r, int left, float (&bias)[2][8]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[k][j] = a.bias[0] && j < left ? param_at<T>(a.param_type, a.bias[k], r + j) : 0.0f;
}
// Gate and up, v and u, of a token's eight features, of which `left` exist (kWhole: all): biases, checkpoints, activation, product.  Four neighbouring lanes
// hold a group and call this together, `there` or not.  kPast: stores past the caches.
template <typename T, bool kWhole, bool kPast>
__device__ __forceinline__ void finish_gated(const ProductArgs &a, float (&v)[8], float (&u)[8], const float (&bias)[2][8], const Target<T, true> &to, int left, bool there) {
    const int n = kWhole ? kChunk : left;
    if (a.bias[0]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] += bias[0][j];
            u[j] += bias[1][j];
        }
    }
    // (Features that do not exist hold copies of the last one, without its bias: they take no part.)
    if (!kWhole && left < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= left) v[j] = u[j] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!a.kept[k].q) continue;
        uint32_t code;
        const u32x2 w = pack8(k ? u : v, static_cast<uint32_t>(a.cap), code);
        if (there) {
            if constexpr (kPast) store_q_past(to.q[k], w, n);
            else store_q(to.q[k], w, n);
        }
        if (there && (threadIdx.x & 3) == 0) *to.scale[k] = static_cast<uint8_t>(code);
    }
    auto apply = [&](auto act) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = decltype(act)::template value<kRoundsTo32<T>>(v[j]) * u[j];
    };
    if (a.act == TENSILE_SILU) apply(Silu{});
    else if (a.act == TENSILE_GELU) apply(Gelu<false>{});
    else apply(Gelu<true>{});
    if (there) {
        if constexpr (kPast) store8_past(to.out, v, n);
        else store8(to.out, v, n);
    }
}

// Tokens from first_token on, 32 at a time, `times` times, and features from r0 on: write(t) puts what belongs to the t-th 32 tokens into the region (kRegions of
// them: each wavefront's part of the sums).  A wavefront goes through them from pass `start` on, every `stride`-th one.
template <typename T, int kPB, bool kForward, int kRegions, bool kPast, typename Write>
__device__ __forceinline__ void finish(const ProductArgs &a, float *region, int64_t first_token, int r0, int times, int start, int stride, Write write) {
    using E = Exchange<kPB, kForward>;
    static_assert(!kForward || E::kEven, "");
    const int lane = threadIdx.x & 63;
    const int r = r0 + lane % E::kLanes * 8, left = a.R - r;
    float bias[2][8];
    if constexpr (kForward) load_bias<T>(a, r, left, bias);
    // (Addresses go on by additions: a product of 64 bits for each store is a quarter of all of this.)
    int64_t token = first_token + start * E::kAtOnce + lane / E::kLanes;
    Target<T, kForward> to(a, token, r);
    auto all = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool kWhole = decltype(whole)::value;
#pragma unroll 1
        for (int t = 0; t < times; ++t) {
            E::order();
            write(t);
            E::order();
#pragma unroll 2
            for (int pass = start; pass < E::kPasses; pass += stride) {
                const int in = pass * E::kAtOnce + lane / E::kLanes;
                const bool mine = E::kEven || (lane / E::kLanes < E::kAtOnce && in < 32), there = mine && (kWhole || (token < a.M && left > 0));
                float v[8];
                E::template get<kRegions>(region, 0, mine ? in : 0, v);
                if constexpr (kForward) {
                    float u[8];
                    E::template get<kRegions>(region, 1, in, u);
                    finish_gated<T, kWhole, kPast>(a, v, u, bias, to, left, there);
                } else if (there) {
                    if constexpr (kPast) store8_past(to.out, v, kWhole ? kChunk : left);
                    else store8(to.out, v, kWhole ? kChunk : left);
                }
                to.go_on(a, stride * E::kAtOnce);
                token += stride * E::kAtOnce;
            }
            if constexpr (!E::kEven) {
                to.go_on(a, 32 - E::kPasses * E::kAtOnce);
                token += 32 - E::kPasses * E::kAtOnce;
            }
        }
    };
    // (The same for all lanes of the wavefront, and asked once: else a tenth of this is questions.)
    const bool whole = r0 + E::kWide <= a.R && first_token + 32 * times <= a.M;
    if (whole) all(std::true_type{});
    else all(std::false_type{});
}

// Where the sums are split: a part's sums as they are, [tile][split][gate, up][token][feature].  base: of the (tile, split)'s first, wide: the tile's features.
template <int kPB, bool kForward, int kRegions, typename Write>
__device__ __forceinline__ void leave_part(float *base, int tokens, int wide, int first_token, int r0, float *region, int times, int start, int stride, Write write) {
    using E = Exchange<kPB, kForward>;
    static_assert(E::kEven, "");
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int t = 0; t < times; ++t) {
        E::order();
        write(t);
        E::order();
#pragma unroll
        for (int k = 0; k < (kForward ? 2 : 1); ++k)
#pragma unroll 1
            for (int pass = start; pass < E::kPasses; pass += stride) {
                const int in = pass * E::kAtOnce + lane / E::kLanes;
                float v[8];
                E::template get<kRegions>(region, k, in, v);
                store8(base + (k * tokens + first_token + 32 * t + in) * wide + r0 + lane % E::kLanes * 8, v, kChunk);
            }
    }
}

// ------------------------------------------------------------------ tiles

// A workgroup's tile: kWP x kWT wavefronts of 32 kPB rows of the weights x 32 kTB tokens each.  Forward the weights' rows are gate and up by turns, 32 each: the
// tile is half as many features wide.
template <int kPB_, int kTB_, int kWP_, int kWT_, int kPerCu_, int kSlots_>
struct Tile {
    static constexpr int kPB = kPB_, kTB = kTB_, kWP = kWP_, kWT = kWT_, kPerCu = kPerCu_, kSlots = kSlots_;   // kSlots: steps in the LDS
    static constexpr int kWaves = kWP * kWT, kThreads = 64 * kWaves;
    static constexpr int kP = 32 * kPB * kWP, kTok = 32 * kTB * kWT;
    // Large tiles end at about the same time, each with 64 KB of h and as much of the checkpoints; together that is what the L2 holds, and there it displaces what
    // the next tiles share (8192 x 4096 x 10944 with checkpoints 1198 us, past the caches 1160; 8192 x 768 x 2048 65 and 59; backward 96.5 and 93.8 in all).  It is no
    // cost put off to the reader: the layer and the product that reads h together, through the caches and past them, us: 4096 x 768 x 2048, whose h is 16 MB, 61.1 and 57.6, 8192 x
    // 768 x 2048 104 and 95, 8192 x 4096 x 10944 1642 and 1633; the backward pass and the norm's that reads dx, of 13 and 67 MB, 98.3 and 97.0, 1279 and 1277.
    static constexpr bool kPast = kP * kTok >= 192 * 128;
    static constexpr bool kSplit = kSlots > 3;                           // what is split, or far, takes tiles of this kind (Few, which alone has the LDS for a fourth step)
};

// A step takes kRow bytes of a row, a line of the caches (with half a line to a step the L2 is asked twice as often, and answers a line or half of one in the same
// time: 8192 x 4096 x 10944 1230 us against 1183): kParts fragments.
constexpr int kRow = 128, kParts = kRow / 32;

// Of staged rows the 16-byte chunks are stored in an order that depends on the row, so that 16 rows' chunks of the same number lie in different banks.
__device__ __forceinline__ int stored_chunk(int row, int chunk) { return chunk ^ (row >> 1 & 7); }

// Where a workgroup works.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD gets a run of consecutive tiles, and consecutive
// tiles lie in bands kBand tiles high, so that those under way on an XCD share rows of both operands.
constexpr uint32_t kBand = 8;
struct Place {
    uint32_t tile, split;
    int r0;
    int64_t m0;
};
template <typename G, bool kForward>
__device__ __forceinline__ Place place_of(const ProductArgs &a, uint32_t tile) {
    const uint32_t per_band = kBand * a.tiles_r, band = tile / per_band, in_band = tile - band * per_band;
    const uint32_t rest = a.tiles_m - band * kBand, high = rest < kBand ? rest : kBand, r = in_band / high;
    Place w;
    w.tile = tile;
    w.split = 0;
    w.m0 = static_cast<int64_t>(band * kBand + (in_band - r * high)) * G::kTok;
    w.r0 = static_cast<int>(r) * (kForward ? G::kP / 2 : G::kP);
    return w;
}
template <typename G, bool kForward>
__device__ __forceinline__ Place place(const ProductArgs &a) {
    const uint32_t total = gridDim.x, xcd = blockIdx.x % kXcds;
    const uint32_t at = xcd * (total / kXcds) + (xcd < total % kXcds ? xcd : total % kXcds) + blockIdx.x / kXcds;
    Place w = place_of<G, kForward>(a, at / a.split);
    w.split = at - w.tile * a.split;
    return w;
}

// From memory to the LDS without a register in between, 16 bytes of each lane in the order of the lanes.  (By hand: of the builtin the compiler waits for every
// one under way before the next LDS read, whatever it reads.  They write no register; the kernels wait.)
__device__ __forceinline__ void bring_16(uint32_t to, global_bytes from, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(from) : "memory", "m0");
}

// A tile's steps: what is brought to the LDS, read from there and multiplied.  kWaves wavefronts, of which this is number `wave`, share slots at `lds`;
// kFar: rows too far apart for 32-bit offsets; every step goes by way of registers.
template <typename T, typename G, bool kForward, bool kFar>
struct Steps {
    static constexpr int kPB = G::kPB, kTB = G::kTB, kPer = kPer16<T>, kStep = kRow / static_cast<int>(sizeof(T));   // elements of a sum in a step
    static constexpr int kSums = kForward ? 1 : 2;
    static constexpr int kSlotP = G::kP * kRow, kSlot = kSlotP + G::kTok * kRow;
    static constexpr int kLoadsP = G::kP / 8 / G::kWaves, kLoadsQ = G::kTok / 8 / G::kWaves;                         // a wave's, of 1024 bytes each
    static_assert(kLoadsP * G::kWaves * 8 == G::kP && kLoadsQ * G::kWaves * 8 == G::kTok, "");
    static constexpr int kRowP = G::kP * static_cast<int>(sizeof(T));                                                // backward: bytes of a staged row of the weights
    static constexpr int64_t kSize = sizeof(T);

    const ProductArgs &a;
    char *const lds;
    const int64_t m0;
    const int r0, lane, wave, wave_p, wave_t;
    // What a lane multiplies of a part of a step, and the sums.  (Not members: the compiler would keep them in memory.)
    struct Fragments {
        u32x4 p[kPB], q[kTB];
    };
    using Sums = f32x16[kPB][kTB];
    // In 32 bits nothing is rounded but the sums themselves: every step's is taken by itself and then added to the others', so that a term passes through 32 +
    // (steps) roundings instead of one for every term behind it.  (In 16 bits a matrix instruction adds 16 products at once, and results are rounded to 16 bits.)
    static constexpr bool kByStep = sizeof(T) == 4;
    static __device__ __forceinline__ void add_step(Sums &acc, Sums &total) {
        if constexpr (kByStep) {
#pragma unroll
            for (int b = 0; b < kPB; ++b)
#pragma unroll
                for (int t = 0; t < kTB; ++t) {
                    total[b][t] += acc[b][t];
                    acc[b][t] = f32x16{};
                }
        }
    }
    static __device__ __forceinline__ const Sums &result(const Sums &acc, const Sums &total) {
        if constexpr (kByStep) return total;
        else return acc;
    }

    __device__ __forceinline__ Steps(const ProductArgs &args, const Place &w, char *slots, int number)
        : a(args), lds(slots), m0(w.m0), r0(w.r0), lane(threadIdx.x & 63), wave(number), wave_p(number / G::kWT), wave_t(number % G::kWT) {
        places();
        if constexpr (!kFar) offsets();
    }

    // What a lane brings of a step, 16 bytes a load.  Tokens, and forward the weights: 8 rows x 8 chunks to a load.  Backward the weights lie with the summed
    // index outermost: whole rows of the tile's columns, staged as they are (16 bits: their 32-byte blocks in an order that depends on the row, so
    // that the 4 rows x 2 blocks that half a wavefront reads at a time lie in different banks).  What does not exist is replaced by something that does.
    struct Piece {
        int64_t row;                  // of the matrix (backward, weights: of the step)
        int col;                      // element
    };
    // (rows of a multiple of 256 bytes begin at the same bank, others in the one or the other half of the banks by turns)
    static __device__ __forceinline__ int turned(int row) { return kRowP % 256 == 0 ? 2 * (row & 3) : 2 * (row >> 1 & 1); }
    __device__ __forceinline__ Piece piece_p(int i) const {
        if constexpr (kForward) {
            const int row = (wave * kLoadsP + i) * 8 + lane / 8, f = r0 + row / 64 * 32 + row % 32;
            return {f < a.R ? f : a.R - 1, stored_chunk(row, lane & 7) * kPer};
        } else {
            const int at = ((wave * kLoadsP + i) * 64 + lane) * 16, row = at / kRowP, in = at % kRowP;
            const int col = sizeof(T) == 2 ? ((in / 32) ^ turned(row)) * 16 + in % 32 / 2 : in / 4;
            return {row, r0 + col};
        }
    }
    __device__ __forceinline__ Piece piece_q(int i) const {
        const int row = (wave * kLoadsQ + i) * 8 + lane / 8;
        const int64_t m = m0 + row;
        return {m < a.M ? m : a.M - 1, stored_chunk(row, lane & 7) * kPer};
    }
    __device__ __forceinline__ int matrix_of(int i) const { return kForward ? ((wave * kLoadsP + i) >> 2) & 1 : 0; }

    uint32_t off_p[kLoadsP], off_q[kSums][kLoadsQ];
    const char *base_p[2], *base_q[kSums];
    __device__ __forceinline__ void offsets() {
#pragma unroll
        for (int k = 0; k < 2; ++k) base_p[k] = static_cast<const char *>(a.p[k].p) + (kForward ? r0 * a.p[k].ld : static_cast<int64_t>(r0)) * kSize;
#pragma unroll
        for (int i = 0; i < kLoadsP; ++i) {
            const Piece c = piece_p(i);
            if constexpr (kForward) off_p[i] = static_cast<uint32_t>(((c.row - r0) * (matrix_of(i) ? a.p[1].ld : a.p[0].ld) + c.col) * kSize);
            else off_p[i] = static_cast<uint32_t>((c.col < a.R ? c.col - r0 : 0) * kSize);
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            base_q[k] = static_cast<const char *>(a.q[k].p) + m0 * a.q[k].ld * kSize;
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i) {
                const Piece c = piece_q(i);
                off_q[k][i] = static_cast<uint32_t>(((c.row - m0) * a.q[k].ld + c.col) * kSize);
            }
        }
    }
    // Load i of step s, of 2 * n_whole backward (gate, then up).
    static constexpr int kLoads = kLoadsP + kLoadsQ;
    __device__ __forceinline__ void bring_part(int s, int slot, int i) const {
        const bool second = !kForward && s >= a.n_whole;
        const int64_t at = static_cast<int64_t>(second ? s - a.n_whole : s) * kStep;
        const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)lds)) + slot * kSlot;
        if (i >= kLoadsP) {
            const int k = i - kLoadsP;
            const char *const from = (kForward || !second ? base_q[0] : base_q[kSums - 1]) + at * kSize;
            bring_16(to + kSlotP + (wave * kLoadsQ + k) * 1024, (global_bytes)from, kForward || !second ? off_q[0][k] : off_q[kSums - 1][k]);
        } else if constexpr (kForward) {
            bring_16(to + (wave * kLoadsP + i) * 1024, (global_bytes)((matrix_of(i) ? base_p[1] : base_p[0]) + at * kSize), off_p[i]);
        } else {
            const int64_t pitch = (second ? a.p[1].ld : a.p[0].ld) * kSize;
            const char *const from = second ? base_p[1] : base_p[0];
            const uint32_t row = static_cast<uint32_t>(((wave * kLoadsP + i) * 64 + lane) * 16 / kRowP);
            bring_16(to + (wave * kLoadsP + i) * 1024, (global_bytes)(from + at * pitch), row * static_cast<uint32_t>(pitch) + off_p[i]);
        }
    }
    // All of them; kQ: of the tokens' loads the first ones only
    template <int kQ = kLoadsQ>
    __device__ __forceinline__ void bring(int s, int slot) const {
#pragma unroll
        for (int i = 0; i < kLoadsP + kQ; ++i) bring_part(s, slot, i);
    }

    // Where a lane's fragments lie, part e of the step in the first slot.  (Two chunks on are an exclusive or, in the order of the chunks.)
    int p_at[kForward ? 1 : kPB], q_at;
    __device__ __forceinline__ void places() {
        const int half = lane >> 5, in_row = (lane & 31) * kRow + stored_chunk(lane & 31, half) * 16;
        q_at = kSlotP + wave_t * kTB * 32 * kRow + in_row;
        if constexpr (kForward) {
            p_at[0] = wave_p * kPB * 32 * kRow + in_row;
        } else {
            // 16 bits: 16 lanes read four rows of 16 columns and each gets the four values of its column
            const int t_row = half * 8 + (lane & 15) / 4;
#pragma unroll
            for (int b = 0; b < kPB; ++b) {
                if constexpr (sizeof(T) == 2)
                    p_at[b] = t_row * kRowP + ((((wave_p * kPB + b) * 2 + (lane >> 4 & 1)) ^ turned(t_row)) * 32) + (lane & 3) * 8;
                else p_at[b] = 4 * half * kRowP + ((wave_p * kPB + b) * 32 + (lane & 31)) * 4;
            }
        }
    }
    __device__ __forceinline__ void read(Fragments &f, int e, int slot) const {
#pragma unroll
        for (int b = 0; b < kPB; ++b) {
            if constexpr (kForward) {
                f.p[b] = *reinterpret_cast<const u32x4 *>(lds + ((p_at[0] ^ (32 * e)) + slot * kSlot) + b * 32 * kRow);
            } else if constexpr (sizeof(T) == 2) {
                typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                lds_char *const from = (lds_char *)lds + (p_at[b] + slot * kSlot) + 16 * e * kRowP;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)from);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + 4 * kRowP));
                f.p[b] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) f.p[b][j] = *reinterpret_cast<const uint32_t *>(lds + (p_at[b] + slot * kSlot) + (8 * e + j) * kRowP);
            }
        }
#pragma unroll
        for (int t = 0; t < kTB; ++t) f.q[t] = *reinterpret_cast<const u32x4 *>(lds + ((q_at ^ (32 * e)) + slot * kSlot) + t * 32 * kRow);
    }
    static __device__ __forceinline__ void multiply(const Fragments &f, Sums &acc, int from = 0, int to = kPB * kTB) {
#pragma unroll
        for (int k = 0; k < kPB * kTB; ++k)
            if (k >= from && k < to) acc[k / kTB][k % kTB] = multiply_add(T{}, f.p[k / kTB], f.q[k % kTB], acc[k / kTB][k % kTB]);
    }
    // LDS instructions of a read
    static constexpr int kReads = kTB + (kForward ? 1 : sizeof(T) == 2 ? 2 : 4) * kPB;

    // Elements from c0 on of sum k, less than a step or the matrices' last rows, by way of registers, to the first slot.  `meet`: what the wavefronts that share
    // the slots do before and behind.
    template <typename Meet>
    __device__ __forceinline__ void rest(int k, int64_t c0, Sums &acc, Meet meet) const {
        meet();
        auto bring_all = [&](auto load) __attribute__((always_inline)) {
            u32x4 v[kLoadsP + kLoadsQ];
#pragma unroll
            for (int i = 0; i < kLoadsP; ++i) {
                const Piece c = piece_p(i);
                const Matrix m = (kForward ? matrix_of(i) : k) ? a.p[1] : a.p[0];
                if constexpr (kForward) v[i] = load(static_cast<const T *>(m.p) + c.row * m.ld, c0 + c.col, a.C, true);
                else v[i] = load(static_cast<const T *>(m.p) + (c0 + c.row < a.C ? c0 + c.row : a.C - 1) * m.ld, c.col, a.R, c0 + c.row < a.C);
            }
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i) {
                const Piece c = piece_q(i);
                const Matrix m = k ? a.q[1] : a.q[0];
                v[kLoadsP + i] = load(static_cast<const T *>(m.p) + c.row * m.ld, c0 + c.col, a.C, true);
            }
#pragma unroll
            for (int i = 0; i < kLoadsP; ++i) *reinterpret_cast<u32x4 *>(lds + (wave * kLoadsP + i) * 1024 + lane * 16) = v[i];
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i) *reinterpret_cast<u32x4 *>(lds + kSlotP + (wave * kLoadsQ + i) * 1024 + lane * 16) = v[kLoadsP + i];
        };
        // (one load after the other, each behind a question, takes 1 us a load)
        if (a.C >= kPer && (kForward || a.R >= kPer)) bring_all([](const T *row, int64_t c, int64_t n, bool keep) __attribute__((always_inline)) { return load_end(row, c, n, keep); });
        else bring_all([](const T *row, int64_t c, int64_t n, bool keep) __attribute__((always_inline)) { return load_chunk(row + c, keep ? n - c : 0); });
        meet();
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
            Fragments f;
            read(f, e, 0);
            multiply(f, acc);
        }
    }
};

// The steps, whole ones and behind them the rest, are the splits' by equal parts.
template <typename T, typename G, bool kForward, bool kFar>
__global__ __launch_bounds__(G::kThreads, G::kPerCu * G::kWaves / 4) void product_kernel(ProductArgs a) {
    using S = Steps<T, G, kForward, kFar>;
    using E = Exchange<G::kPB, kForward>;
    constexpr int kExchange = E::kBytes * G::kWaves, kSlots = G::kSlots, kLoads = S::kLoads, kProducts = G::kPB * G::kTB;
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * S::kSlot > kExchange ? kSlots * S::kSlot : kExchange];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place w = place<G, kForward>(a);
    const S st(a, w, lds, wave);
    typename S::Sums acc = {}, total = {};
    typename S::Fragments f[2];
    const int whole = S::kSums * a.n_whole, rest_from = a.n_whole * S::kStep, rests = (a.C - rest_from + S::kStep - 1) / S::kStep;
    int from = 0, to = whole + S::kSums * rests;                         // (at most 2^26: a step is 32 elements at least)
    if (a.split > 1) {                                                   // (a division of 64 bits is some hundred instructions)
        const int64_t n = to;
        from = static_cast<int>(n * w.split / a.split);
        to = static_cast<int>(n * (w.split + 1) / a.split);
    }
    const int begin = from, end = to < whole ? to : whole;
    if constexpr (!kFar) {
        // Forward, in 16 bits, matrix instructions by turns with LDS reads, and in the last part of a step with loads: 8192 x 4096 x 10944 with checkpoints 1153 ->
        // 1133 us, 8192 x 768 x 2048 58.2 -> 57.2.  (Backward, where a fragment is two reads, 1248 -> 1261.)
        constexpr bool kInTurn = kForward && sizeof(T) == 2;
        static_assert(kProducts % 2 == 0 || !kInTurn, "");
        auto between = [&](auto products) __attribute__((always_inline)) {
            constexpr int kThese = decltype(products)::value;
            if constexpr (kInTurn) {
#pragma unroll
                for (int k = 0; k < kThese; ++k) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, (S::kReads + kThese - 1) / kThese, 0);
                }
            }
        };
        // Step s multiplies while the kSlots - 1 steps behind it are on their way or there.  Behind its barrier every wave has the last fragments of step s in
        // registers and its share of step s+1 in the LDS: step s + kSlots is sent for in its place.  At the barrier all but step s+1 may be under way.
        auto step = [&](int s, int slot, auto steady) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < kParts - 1; ++e) {
                st.read(f[(e + 1) & 1], e + 1, slot);
                S::multiply(f[e & 1], acc);
                between(std::integral_constant<int, kProducts>{});
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (decltype(steady)::value) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kSlots - 2) * kLoads) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            st.read(f[0], 0, (slot + 1) % kSlots);
            if constexpr (decltype(steady)::value && kInTurn) {
                S::multiply(f[(kParts - 1) & 1], acc, 0, kProducts / 2);
                between(std::integral_constant<int, kProducts / 2>{});
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    st.bring_part(s + kSlots, slot, i);
                    S::multiply(f[(kParts - 1) & 1], acc, kProducts / 2 + i * (kProducts / 2) / kLoads, kProducts / 2 + (i + 1) * (kProducts / 2) / kLoads);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                if (decltype(steady)::value || s + kSlots < end) st.bring(s + kSlots, slot);
                S::multiply(f[(kParts - 1) & 1], acc);
            }
            S::add_step(acc, total);
            __builtin_amdgcn_sched_barrier(0);
        };
        if (begin < end) {
#pragma unroll
            for (int s = 0; s < kSlots; ++s)
                if (begin + s < end) st.bring(begin + s, s);
            if (begin + kSlots <= end) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kSlots - 1) * kLoads) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
            st.read(f[0], 0, 0);
            int s = begin;
            for (; s + 2 * kSlots <= end; s += kSlots) {
#pragma unroll
                for (int k = 0; k < kSlots; ++k) step(s + k, k, std::true_type{});
            }
            for (; s < end; s += kSlots) {
#pragma unroll
                for (int k = 0; k < kSlots; ++k)
                    if (s + k < end) step(s + k, k, std::false_type{});
            }
        }
    }
    for (int s = from < whole ? whole : from; s < to; ++s) {
        const int k = s - whole >= rests;
        st.rest(k, rest_from + static_cast<int64_t>(s - whole - (k ? rests : 0)) * S::kStep, acc, [] { __syncthreads(); });
        S::add_step(acc, total);
    }
    const typename S::Sums &sums = S::result(acc, total);
    __syncthreads();
    float *const region = reinterpret_cast<float *>(lds + wave * E::kBytes);
    auto write = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int tt = 0; tt < G::kTB; ++tt)
            if (t == tt) {
#pragma unroll
                for (int b = 0; b < G::kPB; ++b) E::put(region, b, sums[b][tt]);
            }
    };
    if constexpr (G::kSplit) {
        if (a.split > 1) {
            leave_part<G::kPB, kForward, 1>(a.part + (static_cast<int64_t>(w.tile) * a.split + w.split) * (G::kP * G::kTok), G::kTok, kForward ? G::kP / 2 : G::kP,
                                            st.wave_t * G::kTB * 32, st.wave_p * E::kWide, region, G::kTB, 0, 1, write);
            return;
        }
    }
    finish<T, G::kPB, kForward, 1, G::kPast>(a, region, w.m0 + st.wave_t * G::kTB * 32, w.r0 + st.wave_p * E::kWide, G::kTB, 0, 1, write);
}

// Up to 32 tokens: the weights are read once and that is what it costs.  A workgroup has 32 features (backward 64), of whose sums each wavefront takes every
// kWaves-th step, by itself: it brings its own steps, kRing of them, and waits for nobody.  The wavefronts' sums are added up where they go through
// the LDS.  kQ: loads of eight tokens (more rows of the staged 32 than that are left as they are; their columns of the result are not used).
constexpr int kRing = 3;
using Rows = Tile<2, 1, 1, 1, 1, kRing>;
template <typename T, bool kForward, bool kFar, int kWaves, int kQ>
__global__ __launch_bounds__(64 * kWaves) void product_rows_kernel(ProductArgs a) {
    using S = Steps<T, Rows, kForward, kFar>;
    using E = Exchange<Rows::kPB, kForward>;
    static_assert(kWaves * E::kBytes <= kWaves * kRing * S::kSlot, "");
    __shared__ __attribute__((aligned(1024))) char lds[kWaves * kRing * S::kSlot];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place w = place<Rows, kForward>(a);
    const S st(a, w, lds + wave * kRing * S::kSlot, 0);
    typename S::Sums acc = {}, total = {};
    if constexpr (!kFar) {
        // the wavefront's steps: first, first + stride, ... : n of them
        const int stride = kWaves * static_cast<int>(a.split), first = static_cast<int>(w.split) * kWaves + wave, whole = S::kSums * a.n_whole;
        const int n = whole > first ? (whole - first + stride - 1) / stride : 0;
        // (Forward each workgroup begins elsewhere in its sums: at the same place of rows that lie a power of two apart all of them would ask the same few memory
        // channels.  1 x 4096 x 16384 52 -> 47 us, 24 tokens x 4096 x 10944 f16 40.6 -> 39.6; backward, where neighbours share lines, 36 -> 39.)
        const int turn = kForward && n > 0 ? static_cast<int>((w.tile * 37u) % static_cast<uint32_t>(n)) : 0;
        auto at = [&](int i) __attribute__((always_inline)) { return first + (i + turn < n ? i + turn : i + turn - n) * stride; };
        auto step = [&](int i, int slot, auto steady) __attribute__((always_inline)) {
            if constexpr (decltype(steady)::value) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kRing - 1) * (S::kLoadsP + kQ)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            typename S::Fragments f[2];
            st.read(f[0], 0, slot);
#pragma unroll
            for (int e = 0; e < kParts; ++e) {
                if (e + 1 < kParts) st.read(f[(e + 1) & 1], e + 1, slot);
                S::multiply(f[e & 1], acc);
            }
            S::add_step(acc, total);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (decltype(steady)::value || i + kRing < n) st.template bring<kQ>(at(i + kRing), slot);
        };
#pragma unroll
        for (int k = 0; k < kRing; ++k)
            if (k < n) st.template bring<kQ>(at(k), k);
        int i = 0;
        for (; i + 2 * kRing <= n; i += kRing) {
#pragma unroll
            for (int k = 0; k < kRing; ++k) step(i + k, k, std::true_type{});
        }
        for (; i < n; i += kRing) {
#pragma unroll
            for (int k = 0; k < kRing; ++k)
                if (i + k < n) step(i + k, k, std::false_type{});
        }
    }
    // (the rest goes on in turn behind the whole steps: kFar all of it)
    {
        // (in 32 bits: for a comparison of two 64-bit numbers, uniform as they are, hipcc of ROCm 7.2 has put a vector comparison in front of a scalar selection)
        const int from = a.n_whole * S::kStep, per = (a.C - from + S::kStep - 1) / S::kStep, stride = kWaves * static_cast<int>(a.split);
        const int own = static_cast<int>(w.split) * kWaves + wave;
        for (int s = (own + stride - S::kSums * a.n_whole % stride) % stride; s < S::kSums * per; s += stride) {
            const int k = s >= per;
            st.rest(k, from + static_cast<int64_t>(s - (k ? per : 0)) * S::kStep, acc, [] { E::order(); });
            S::add_step(acc, total);
        }
    }
    __syncthreads();
    float *const region = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int b = 0; b < Rows::kPB; ++b) E::put(reinterpret_cast<float *>(lds + wave * E::kBytes), b, S::result(acc, total)[b][0]);
    __syncthreads();
    if (a.split > 1)
        leave_part<Rows::kPB, kForward, kWaves>(a.part + (static_cast<int64_t>(w.tile) * a.split + w.split) * (Rows::kP * Rows::kTok), Rows::kTok, E::kWide, 0, 0, region,
                                                1, wave, kWaves, [](int) {});
    else finish<T, Rows::kPB, kForward, kWaves, false>(a, region, w.m0, w.r0, 1, wave, kWaves, [](int) {});
}

// split > 1: the parts of a sum added up in a fixed order, then as above.  Eight features of a token to a thread.
template <typename G, bool kForward>
struct Join {
    static constexpr int kWide = kForward ? G::kP / 2 : G::kP, kPlane = G::kTok * kWide, kUnits = kPlane / 8;
    static constexpr int kThreads = kUnits < 256 ? kUnits : 256, kBlocks = kUnits / kThreads;    // of a tile
    static_assert(kUnits % kThreads == 0, "");
};
template <typename T, typename G, bool kForward>
__global__ __launch_bounds__((Join<G, kForward>::kThreads)) void product_join_kernel(ProductArgs a) {
    using J = Join<G, kForward>;
    constexpr int kWide = J::kWide, kPlane = J::kPlane, kPart = G::kP * G::kTok;
    const uint32_t tile = blockIdx.x / J::kBlocks;
    const int unit = blockIdx.x % J::kBlocks * J::kThreads + threadIdx.x;
    const Place w = place_of<G, kForward>(a, tile);
    const int64_t token = w.m0 + unit / (kWide / 8);
    const int r = w.r0 + unit % (kWide / 8) * 8, left = a.R - r;
    const bool there = token < a.M && left > 0;
    float sum[2][8] = {};
    if (there) {                                                         // (four parts' loads under way)
        const float *from = a.part + static_cast<int64_t>(tile) * a.split * kPart + unit * 8;
#pragma unroll 4
        for (uint32_t s = 0; s < a.split; ++s, from += kPart)
#pragma unroll
            for (int k = 0; k < (kForward ? 2 : 1); ++k) {
                float v[8];
                load8(from + k * kPlane, kChunk, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[k][j] += v[j];
            }
    }
    const Target<T, kForward> to(a, token, r);
    if constexpr (kForward) {
        float bias[2][8];
        load_bias<T>(a, r, left, bias);
        finish_gated<T, false, false>(a, sum[0], sum[1], bias, to, left, there);
    } else if (there) {
        store8(to.out, sum[0], left);
    }
}

// Cuts the result into tiles of G and launches for them.  A launch takes kMost tiles each way at most (it has room for 2^32 threads, and wraps silently beyond).
constexpr int64_t kMost = 1 << 11;
template <typename T, typename G, bool kForward, typename Launch>
int run(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &whole, bool far, int64_t split, Launch launch) {
    constexpr int64_t kWide = kForward ? G::kP / 2 : G::kP, kSize = sizeof(T);
    const int64_t tiles_m = (whole.M + G::kTok - 1) / G::kTok, tiles_r = (whole.R + kWide - 1) / kWide;
    const int64_t steps = (kForward ? 1 : 2) * ((static_cast<int64_t>(whole.C) * kSize + kRow - 1) / kRow);
    if (split > steps) split = steps;
    if (split < 1) split = 1;
    std::unique_lock<std::mutex> lock;
    float *part = nullptr;
    if (split > 1) {                                                     // (where there are few tiles: one launch)
        OpsScratch &scratch = ops_scratch(ops, s);
        lock = std::unique_lock<std::mutex>(scratch.mu);
        const int rc = scratch.provide(static_cast<size_t>(tiles_m * tiles_r * split) * G::kP * G::kTok,
                                       kForward ? "gated_linear: partial sums" : "gated_linear_backward: partial sums");
        if (rc != TENSILE_OK) return rc;
        part = scratch.buf.p;
    }
    // Backward a load of columns reads what lies behind the row's last one, up to the end of the row's last chunk: not where that is behind the matrix.
    constexpr int64_t kPer = kPer16<T>, kStep = kRow / kSize;
    int64_t behind = 0;                                                  // rows at the end that are not brought whole
    if (!kForward && whole.R % kPer) {
        const int64_t least = whole.p[0].ld < whole.p[1].ld ? whole.p[0].ld : whole.p[1].ld;
        behind = (kPer - 1 + least - 1) / least;
    }
    const int64_t n_whole = far || whole.C < behind ? 0 : (whole.C - behind) / kStep;
    auto moved = [](Matrix m, int64_t rows, int64_t cols) {
        return Matrix{m.p ? static_cast<char *>(m.p) + (rows * m.ld + cols) * kSize : nullptr, m.ld};
    };
    for (int64_t r = 0; r < tiles_r; r += kMost)
        for (int64_t m = 0; m < tiles_m; m += kMost) {
            ProductArgs a = whole;
            const int64_t r0 = r * kWide, m0 = m * G::kTok;
            a.tiles_r = static_cast<uint32_t>(tiles_r - r < kMost ? tiles_r - r : kMost);
            a.tiles_m = static_cast<uint32_t>(tiles_m - m < kMost ? tiles_m - m : kMost);
            a.split = static_cast<uint32_t>(split);
            a.part = part;
            a.n_whole = static_cast<int32_t>(n_whole);
            a.M -= m0;
            a.R -= static_cast<int32_t>(r0);
            a.out = moved(a.out, m0, r0);
            for (int k = 0; k < 2; ++k) {
                a.q[k] = moved(a.q[k], m0, 0);
                a.p[k] = kForward ? moved(a.p[k], r0, 0) : moved(a.p[k], 0, r0);
                if (a.bias[k]) a.bias[k] = static_cast<const char *>(a.bias[k]) + r0 * (a.param_type == TENSILE_F32 ? 4 : 2);
                if (a.kept[k].q) {
                    a.kept[k].q += m0 * a.kept[k].ld_q + r0;
                    a.kept[k].scale += m0 * a.kept[k].ld_scale + r0 / kGroup;
                }
            }
            launch(a, dim3(a.tiles_m * a.tiles_r * a.split), a.tiles_m * a.tiles_r);
            TS_HIP(hipGetLastError());
        }
    return TENSILE_OK;
}

template <typename T, typename G, bool kForward>
int run_tiles(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &whole, bool far = false, int64_t split = 1) {
    return run<T, G, kForward>(ops, s, whole, far, split, [&](const ProductArgs &a, dim3 grid, uint32_t tiles) {
        const dim3 block(G::kThreads);
        if constexpr (G::kSplit) {
            if (far) hipLaunchKernelGGL(HIP_KERNEL_NAME(product_kernel<T, G, kForward, true>), grid, block, 0, s, a);
        }
        if (!far) hipLaunchKernelGGL(HIP_KERNEL_NAME(product_kernel<T, G, kForward, false>), grid, block, 0, s, a);
        if constexpr (G::kSplit) {
            if (a.split > 1)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(product_join_kernel<T, G, kForward>), dim3(tiles * Join<G, kForward>::kBlocks),
                                   dim3(Join<G, kForward>::kThreads), 0, s, a);
        }
    });
}
template <typename T, bool kForward>
int run_rows(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &whole, bool far, int64_t split, bool four) {
    return run<T, Rows, kForward>(ops, s, whole, far, split, [&](const ProductArgs &a, dim3 grid, uint32_t tiles) {
        auto with = [&](auto waves, auto q) {
            constexpr int kWaves = decltype(waves)::value, kQ = decltype(q)::value;
            hipLaunchKernelGGL(HIP_KERNEL_NAME(product_rows_kernel<T, kForward, false, kWaves, kQ>), grid, dim3(64 * kWaves), 0, s, a);
        };
        using Two = std::integral_constant<int, 2>;
        using Four = std::integral_constant<int, 4>;
        using One = std::integral_constant<int, 1>;
        if (far) hipLaunchKernelGGL(HIP_KERNEL_NAME(product_rows_kernel<T, kForward, true, 4, 4>), grid, dim3(256), 0, s, a);
        else if (four && a.M <= 8) with(Four{}, One{});
        else if (four) with(Four{}, Four{});
        else if (a.M <= 8) with(Two{}, One{});
        else with(Two{}, Four{});
        if (a.split > 1)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(product_join_kernel<T, Rows, kForward>), dim3(tiles * Join<Rows, kForward>::kBlocks),
                               dim3(Join<Rows, kForward>::kThreads), 0, s, a);
    });
}

// (Four wavefronts of 128 x 128, one to a SIMD, read the LDS a third less and are slower all the same, 1461 us against 1138 at 8192 x 4096 x 10944: nothing runs while
// one waits.  256 x 128 with three steps of half lines, two workgroups to a CU: 1399 against 1230 then.)
using Large = Tile<4, 2, 2, 4, 1, 2>;    // 256 x 256
using Middle = Tile<3, 1, 2, 4, 1, 3>;   // 192 x 128
using Small = Tile<2, 2, 2, 2, 2, 2>;    // 128 x 128
using Few = Tile<2, 2, 2, 2, 1, 4>;      // 128 x 128, for splits: four steps in the LDS

// Whether the rows that a tile of G reads from one scalar address lie too far apart for offsets of 32 bits (kept below 2^31): its tokens, its features forward, a
// step's rows of the weights backward.  They are reached by 64-bit addresses then, and every step goes by way of registers.  24 x 4096 x 10944 bf16, us: tokens 8 KB, 16 MB and
// 64 MB apart 42.1, 43.5 and 43.0; 96 MB apart, which is too far, 73.6.
constexpr int64_t kFarBytes = (int64_t{1} << 31) - (1 << 12);            // (less than a row's part of a step)
inline bool is_far(const Matrix &m, int64_t rows, int64_t at_once, int64_t size) {
    return (rows < at_once ? rows - 1 : at_once - 1) * m.ld * size >= kFarBytes;
}
template <typename T, typename G, bool kForward>
bool is_far(const ProductArgs &a) {
    constexpr int64_t kSize = sizeof(T);
    bool far = false;
    for (int k = 0; k < 2; ++k)
        far = far || is_far(a.q[k], a.M, G::kTok, kSize) || is_far(a.p[k], kForward ? a.R : a.C, kForward ? G::kP / 2 : kRow / kSize, kSize);
    return far;
}

inline int64_t rounds(int64_t tiles, int64_t places) { return (tiles + places - 1) / places; }
template <typename T, bool kForward>
int64_t steps_of(const ProductArgs &a) {
    return (kForward ? 1 : 2) * rounds(static_cast<int64_t>(a.C) * static_cast<int64_t>(sizeof(T)), kRow);
}
// Few tiles: their sums are split until the card is full, but not below 12 steps (adding up is another launch, 4 us).  1, 2, 4 and 8 parts, us:
// backward 64 x 4096 x 10944 (32 tiles, 342 steps) 142, 82, 51, 44; 512 x 768 x 2048 (24, 64) 37, 28, 22, 22; 301 x 1000 x 1500 f16 (24, 48) 38, 30, 26.5, 26;
// forward 64 x 4096 x 2048 (32, 64) 35, 25, 20, 21; 301 x 1000 x 1500 (72, 16) 17, 19, 26; 64 x 4096 x 10944 (171, 64) 47, 61.
inline int64_t parts_of(int64_t tiles, int64_t places, int64_t steps) {
    const int64_t fill = places / tiles, most = steps / 12;
    return fill < most ? fill : most;
}
template <typename G, bool kForward>
int64_t tiles_of(const ProductArgs &a) {
    constexpr int64_t kWide = kForward ? G::kP / 2 : G::kP;
    return ((a.M + G::kTok - 1) / G::kTok) * ((a.R + kWide - 1) / kWide);
}

}  // namespace

}  // namespace tensile
