// The matrix products of the gated layer, forward (gated.hip) and backward (gated_backward.hip):
//   g[m,f] = sum_k x[m,k]*Wg[f,k],  u[m,f] = sum_k x[m,k]*Wu[f,k]          (and from both act(g)*u, in the registers that hold them)
//   dx[m,k] = sum_f dgate[m,f]*Wg[f,k] + sum_f dup[m,f]*Wu[f,k]
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

// Up to 16 bytes of a row, `left` elements of which exist (0 or fewer: none); zeros behind them.
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
    Matrix q[2];                      // tokens x C: x, or dgate and dup
    Matrix p[2];                      // Wg, Wu: R x C forward, C x R backward
    // forward
    const void *bias[2];
    int32_t param_type, act, cap;
    Matrix out;                       // h, or dx
    Ckpt kept[2];
    // how the work is cut: tiles of tokens and features, and the steps of a sum among `split` workgroups a tile
    uint32_t tiles_m, tiles_r, split;
    float *part;                      // split > 1: [tile][split][wavefront][block][register][lane]
};

template <typename T>
__device__ __forceinline__ float param_at(int type, const void *p, int64_t at) {
    return type == TENSILE_F32 ? static_cast<const float *>(p)[at] : to_f32(static_cast<const T *>(p)[at]);
}

// What becomes of the sums of a wavefront's kPB blocks (32 rows each) of 32 tokens.  They go through the LDS, so that a lane has eight features of a token and a
// store whole lines of memory, in a loop: in registers it takes a copy of all of this for every block, which the instruction cache does not hold
// (8192 x 4096 x 10944 with checkpoints 1356 us, so LATER).
template <int kPB_, bool kForward>
struct Exchange {
    static constexpr int kPB = kPB_, kWide = kForward ? kPB * 16 : kPB * 32;           // features
    static constexpr int kPitch = kWide + 4;                                           // floats from a token to the next: 16 lanes' 16 bytes lie in different banks
    static constexpr int kBytes = 32 * kPitch * 4 * (kForward ? 2 : 1);                // of a wavefront
    static constexpr int kLanes = kWide / 8, kAtOnce = 64 / kLanes;                    // a token's lanes, tokens at once

    // Block b of the blocks, as the matrix instructions leave it: a lane has rows 8q + 4 (lane / 32) .. + 3 of token lane % 32.
    static __device__ __forceinline__ void put(float *region, int b, const f32x16 &acc) {
        const int lane = threadIdx.x & 63, plane = kForward ? b & 1 : 0, at = (kForward ? b / 2 : b) * 32;
        float *const to = region + plane * 32 * kPitch + (lane & 31) * kPitch + at + 4 * (lane >> 5);
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4 *>(to + 8 * q) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    }
    static __device__ __forceinline__ void get(const float *region, int plane, int token, float (&v)[8]) {
        const int lane = threadIdx.x & 63;
        const float *const from = region + plane * 32 * kPitch + token * kPitch + lane % kLanes * 8;
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(from), hi = *reinterpret_cast<const f32x4 *>(from + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = lo[j];
            v[4 + j] = hi[j];
        }
    }
    // (a wavefront's LDS accesses are in order; this keeps the compiler from changing it)
    static __device__ __forceinline__ void order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
};

// Tokens from first_token on, 32 at a time, `times` times, and the wavefront's features from r0 on: write(t) puts what belongs to the t-th 32 tokens into the region.
template <typename T, int kPB, bool kForward, typename Write>
__device__ __forceinline__ void finish(const ProductArgs &a, float *region, int64_t first_token, int r0, int times, Write write) {
    using E = Exchange<kPB, kForward>;
    const int lane = threadIdx.x & 63;
    const int r = r0 + lane % E::kLanes * 8, left = a.R - r;
    float bias[kForward ? 2 : 1][8] = {};
    if constexpr (kForward) {
        if (a.bias[0]) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) bias[k][j] = param_at<T>(a.param_type, a.bias[k], r + j);
        }
    }
    // (Addresses go on by additions: a product of 64 bits for each store is a quarter of all of this.)
    int64_t token = first_token + lane / E::kLanes;
    T *out = static_cast<T *>(a.out.p) + token * a.out.ld + r;
    int8_t *q[2] = {};
    uint8_t *scale[2] = {};
    if constexpr (kForward) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (a.kept[k].q) {
                q[k] = a.kept[k].q + token * a.kept[k].ld_q + r;
                scale[k] = a.kept[k].scale + token * a.kept[k].ld_scale + r / kGroup;
            }
    }
    auto all = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool kWhole = decltype(whole)::value;
#pragma unroll 1
        for (int t = 0; t < times; ++t) {
            E::order();
            write(t);
            E::order();
#pragma unroll 2
            for (int pass = 0; pass < 32 / E::kAtOnce; ++pass) {
                const int in = pass * E::kAtOnce + lane / E::kLanes, n = kWhole ? kChunk : left;
                const bool there = kWhole || (token < a.M && left > 0);
                float v[8];
                E::get(region, 0, in, v);
                if constexpr (kForward) {
                    float u[8];
                    E::get(region, 1, in, u);
                    if (a.bias[0]) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            v[j] += bias[0][j];
                            u[j] += bias[1][j];
                        }
                    }
                    // (Rows that do not exist hold copies of the last one, without its bias: they take no part.)
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
                        if (there) store_q(q[k], w, n);
                        if (there && (lane & 3) == 0) *scale[k] = static_cast<uint8_t>(code);
                        q[k] += E::kAtOnce * a.kept[k].ld_q;
                        scale[k] += E::kAtOnce * a.kept[k].ld_scale;
                    }
                    auto apply = [&](auto act) __attribute__((always_inline)) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = decltype(act)::template value<kRoundsTo32<T>>(v[j]) * u[j];
                    };
                    if (a.act == TENSILE_SILU) apply(Silu{});
                    else if (a.act == TENSILE_GELU) apply(Gelu<false>{});
                    else apply(Gelu<true>{});
                }
                if (there) store8(out, v, n);
                out += E::kAtOnce * a.out.ld;
                token += E::kAtOnce;
            }
        }
    };
    // (The same for all lanes of the wavefront, and asked once: else a tenth of this is questions.)
    const bool whole = r0 + E::kWide <= a.R && first_token + 32 * times <= a.M;
    if (whole) all(std::true_type{});
    else all(std::false_type{});
}

// ------------------------------------------------------------------ tiles

// A workgroup's tile: kWP x kWT wavefronts of 32 kPB rows of the weights x 32 kTB tokens each.  Forward the weights' rows are gate and up by turns, 32 each: the
// tile is half as many features wide.
template <int kPB_, int kTB_, int kWP_, int kWT_, int kPerCu_>
struct Tile {
    static constexpr int kPB = kPB_, kTB = kTB_, kWP = kWP_, kWT = kWT_, kPerCu = kPerCu_;
    static constexpr int kWaves = kWP * kWT, kThreads = 64 * kWaves;
    static constexpr int kP = 32 * kPB * kWP, kTok = 32 * kTB * kWT;
};

// A step takes kRow bytes of a row, a line of the caches (with half a line to a step the L2 is asked twice as often: it answers a line or half of one in the same
// time); two steps are in the LDS, kParts fragments long each.
constexpr int kRow = 128, kSlots = 2, kParts = kRow / 32;

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

// kFar: rows too far apart for 32-bit offsets; every step goes by way of registers.
template <typename T, typename G, bool kForward, bool kFar>
__global__ __launch_bounds__(G::kThreads, G::kPerCu * G::kWaves / 4) void product_kernel(ProductArgs a) {
    constexpr int kPB = G::kPB, kTB = G::kTB, kPer = kPer16<T>, kStep = kRow / static_cast<int>(sizeof(T));      // elements of a sum in a step
    constexpr int kSlotP = G::kP * kRow, kSlot = kSlotP + G::kTok * kRow;
    constexpr int kLoadsP = G::kP / 8 / G::kWaves, kLoadsQ = G::kTok / 8 / G::kWaves;   // a wave's, of 1024 bytes each
    static_assert(kLoadsP * G::kWaves * 8 == G::kP && kLoadsQ * G::kWaves * 8 == G::kTok, "");
    constexpr int kRowP = G::kP * static_cast<int>(sizeof(T));                         // backward: bytes of a staged row of the weights
    constexpr int kExchange = Exchange<kPB, kForward>::kBytes * G::kWaves;
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * kSlot > kExchange ? kSlots * kSlot : kExchange];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave_p = wave / G::kWT, wave_t = wave % G::kWT;
    const Place w = place<G, kForward>(a);

    // What a lane brings of a step, 16 bytes a load.  Tokens, and forward the weights: 8 rows x 8 chunks to a load.  Backward the weights lie with the summed
    // index outermost: whole rows of the tile's columns, staged as they are (16 bits: their 32-byte blocks in an order that depends on the row, so
    // that the 4 rows x 2 blocks that half a wavefront reads at a time lie in different banks).  What does not exist is replaced by something that does.
    struct Piece {
        int64_t row;                  // of the matrix (backward, weights: of the step)
        int col;                      // element
    };
    auto row_of = [&](int i) __attribute__((always_inline)) { return (wave * kLoadsP + i) * 8 + lane / 8; };       // of the tile's weights, forward
    auto piece_p = [&](int i) __attribute__((always_inline)) -> Piece {
        if constexpr (kForward) {
            const int row = row_of(i), f = w.r0 + row / 64 * 32 + row % 32;
            return {f < a.R ? f : a.R - 1, stored_chunk(row, lane & 7) * kPer};
        } else {
            const int at = ((wave * kLoadsP + i) * 64 + lane) * 16, row = at / kRowP, in = at % kRowP;
            int col = sizeof(T) == 2 ? ((in / 32) ^ (2 * (row & 3))) * 16 + in % 32 / 2 : in / 4;
            col += w.r0;
            return {row, col};
        }
    };
    auto piece_q = [&](int i) __attribute__((always_inline)) -> Piece {
        const int row = (wave * kLoadsQ + i) * 8 + lane / 8;
        const int64_t m = w.m0 + row;
        return {m < a.M ? m : a.M - 1, stored_chunk(row, lane & 7) * kPer};
    };
    auto matrix_of = [&](int i) __attribute__((always_inline)) { return kForward ? ((wave * kLoadsP + i) >> 2) & 1 : 0; };

    f32x16 acc[kPB][kTB] = {};
    u32x4 fp[2][kPB], fq[2][kTB];
    // Where a lane's fragments lie, part e of the step in the first slot.  (Two chunks on are an exclusive or, in the order of the chunks.)
    const int half = lane >> 5, in_row = (lane & 31) * kRow + stored_chunk(lane & 31, half) * 16;
    // backward, 16 bits: 16 lanes read four rows of 16 columns and each gets the four values of its column
    const int t_row = half * 8 + (lane & 15) / 4;
    int p_at[kForward ? 1 : kPB];
    if constexpr (kForward) {
        p_at[0] = wave_p * kPB * 32 * kRow + in_row;
    } else {
#pragma unroll
        for (int b = 0; b < kPB; ++b) {
            if constexpr (sizeof(T) == 2)
                p_at[b] = t_row * kRowP + ((((wave_p * kPB + b) * 2 + (lane >> 4 & 1)) ^ (2 * (t_row & 3))) * 32) + (lane & 3) * 8;
            else p_at[b] = 4 * half * kRowP + ((wave_p * kPB + b) * 32 + (lane & 31)) * 4;
        }
    }
    const int q_at = kSlotP + wave_t * kTB * 32 * kRow + in_row;
    auto read = [&](int e, int slot) __attribute__((always_inline)) {
        const int to = e & 1;
#pragma unroll
        for (int b = 0; b < kPB; ++b) {
            if constexpr (kForward) {
                fp[to][b] = *reinterpret_cast<const u32x4 *>(lds + ((p_at[0] ^ (32 * e)) + slot * kSlot) + b * 32 * kRow);
            } else if constexpr (sizeof(T) == 2) {
                typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                lds_char *const from = (lds_char *)lds + (p_at[b] + slot * kSlot) + 16 * e * kRowP;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)from);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + 4 * kRowP));
                fp[to][b] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) fp[to][b][j] = *reinterpret_cast<const uint32_t *>(lds + (p_at[b] + slot * kSlot) + (8 * e + j) * kRowP);
            }
        }
#pragma unroll
        for (int t = 0; t < kTB; ++t) fq[to][t] = *reinterpret_cast<const u32x4 *>(lds + ((q_at ^ (32 * e)) + slot * kSlot) + t * 32 * kRow);
    };
    auto multiply = [&](int e) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < kPB; ++b)
#pragma unroll
            for (int t = 0; t < kTB; ++t) acc[b][t] = multiply_add(T{}, fp[e & 1][b], fq[e & 1][t], acc[b][t]);
    };

    // Whole steps.  Backward a load of columns reads what lies behind the row's last one, up to the end of the row's last chunk: not where that is behind
    // the matrix.  Of those steps, 2 * n_whole backward (gate, then up), the split takes a part; the rest, by way of registers, its last one.
    constexpr int kSums = kForward ? 1 : 2;
    int n_whole = 0;
    if constexpr (!kFar) {
        if constexpr (kForward) {
            n_whole = a.C / kStep;
        } else {
            const int64_t least = a.p[0].ld < a.p[1].ld ? a.p[0].ld : a.p[1].ld;
            const int64_t behind = a.R % kPer == 0 ? 0 : (kPer - 1 + least - 1) / least;   // rows at the end that are not read whole
            n_whole = a.C > behind ? static_cast<int>((a.C - behind) / kStep) : 0;
        }
    }
    int begin = 0, end = kSums * n_whole;                                // (at most 2^25: a step is 32 elements at least)
    if (a.split > 1) {                                                   // (a division of 64 bits is some hundred instructions)
        const int64_t n = end;
        begin = static_cast<int>(n * w.split / a.split);
        end = static_cast<int>(n * (w.split + 1) / a.split);
    }

    if constexpr (!kFar) {
        const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)lds));
        // From memory to the LDS without a register in between, 16 bytes of each lane in the order of the lanes.  (By hand: of the builtin the compiler waits
        // for every one under way before the next LDS read, whatever it reads.  They write no register; the waits are at the barriers below.)
        auto bring_16 = [&](uint32_t to, global_bytes from, uint32_t off) __attribute__((always_inline)) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(from) : "memory", "m0");
        };
        uint32_t off_p[kLoadsP], off_q[kSums][kLoadsQ];
        const char *base_p[2], *base_q[kSums];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            base_p[k] = static_cast<const char *>(a.p[k].p) + (kForward ? w.r0 * a.p[k].ld : static_cast<int64_t>(w.r0)) * static_cast<int64_t>(sizeof(T));
#pragma unroll
        for (int k = 0; k < kSums; ++k) base_q[k] = static_cast<const char *>(a.q[k].p) + w.m0 * a.q[k].ld * static_cast<int64_t>(sizeof(T));
#pragma unroll
        for (int i = 0; i < kLoadsP; ++i) {
            const Piece c = piece_p(i);
            if constexpr (kForward) off_p[i] = static_cast<uint32_t>(((c.row - w.r0) * a.p[matrix_of(i)].ld + c.col) * static_cast<int64_t>(sizeof(T)));
            else off_p[i] = static_cast<uint32_t>((c.col < a.R ? c.col - w.r0 : 0) * static_cast<int64_t>(sizeof(T)));
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i) {
                const Piece c = piece_q(i);
                off_q[k][i] = static_cast<uint32_t>(((c.row - w.m0) * a.q[k].ld + c.col) * static_cast<int64_t>(sizeof(T)));
            }
        auto bring = [&](int s, int slot) __attribute__((always_inline)) {
            const bool second = !kForward && s >= n_whole;
            const int64_t at = static_cast<int64_t>(second ? s - n_whole : s) * kStep;
            const uint32_t to = lds_at + slot * kSlot;
            if constexpr (kForward) {
#pragma unroll
                for (int i = 0; i < kLoadsP; ++i)
                    bring_16(to + (wave * kLoadsP + i) * 1024, (global_bytes)(base_p[matrix_of(i)] + at * static_cast<int64_t>(sizeof(T))), off_p[i]);
            } else {
                const int64_t pitch = (second ? a.p[1].ld : a.p[0].ld) * static_cast<int64_t>(sizeof(T));
                const char *const from = second ? base_p[1] : base_p[0];
#pragma unroll
                for (int i = 0; i < kLoadsP; ++i) {
                    const uint32_t row = static_cast<uint32_t>(((wave * kLoadsP + i) * 64 + lane) * 16 / kRowP);
                    bring_16(to + (wave * kLoadsP + i) * 1024, (global_bytes)(from + at * pitch), row * static_cast<uint32_t>(pitch) + off_p[i]);
                }
            }
            const char *const from = (kForward || !second ? base_q[0] : base_q[kSums - 1]) + at * static_cast<int64_t>(sizeof(T));
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i)
                bring_16(to + kSlotP + (wave * kLoadsQ + i) * 1024, (global_bytes)from, kForward || !second ? off_q[0][i] : off_q[kSums - 1][i]);
        };
        // Step s multiplies while step s+1 is on its way.  Behind its barrier every wave has the last fragments of step s in registers and its share of step s+1
        // in the LDS: step s+2 is sent for in the place of step s.
        auto step = [&](int s, int slot, auto steady) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < kParts - 1; ++e) {
                read(e + 1, slot);
                multiply(e);
                __builtin_amdgcn_sched_barrier(0);
            }
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            read(0, slot ^ 1);
            if (decltype(steady)::value || s + kSlots < end) bring(s + kSlots, slot);
            multiply(kParts - 1);
            __builtin_amdgcn_sched_barrier(0);
        };
        if (begin < end) {
#pragma unroll
            for (int s = 0; s < kSlots; ++s)
                if (begin + s < end) bring(begin + s, s);
            if (begin + 1 < end) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoadsP + kLoadsQ) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
            read(0, 0);
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
    // What is left of the sums, less than a step or the matrices' last rows (kFar: all of them, split by steps), by way of registers.
    auto rest = [&](int k, int64_t c0) __attribute__((always_inline)) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoadsP; ++i) {
            const Piece c = piece_p(i);
            u32x4 v;
            if constexpr (kForward) {
                const Matrix &m = a.p[matrix_of(i)];
                v = load_chunk(static_cast<const T *>(m.p) + c.row * m.ld + c0 + c.col, a.C - c0 - c.col);
            } else {
                const Matrix &m = a.p[k];
                const int64_t row = c0 + c.row;
                v = load_chunk(static_cast<const T *>(m.p) + row * m.ld + c.col, row < a.C ? a.R - c.col : 0);
            }
            *reinterpret_cast<u32x4 *>(lds + (wave * kLoadsP + i) * 1024 + lane * 16) = v;
        }
#pragma unroll
        for (int i = 0; i < kLoadsQ; ++i) {
            const Piece c = piece_q(i);
            const Matrix &m = a.q[k];
            const u32x4 v = load_chunk(static_cast<const T *>(m.p) + c.row * m.ld + c0 + c.col, a.C - c0 - c.col);
            *reinterpret_cast<u32x4 *>(lds + kSlotP + (wave * kLoadsQ + i) * 1024 + lane * 16) = v;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
            read(e, 0);
            multiply(e);
        }
    };
    if constexpr (kFar) {
        const int64_t per = (a.C + kStep - 1) / kStep, n = per * kSums;
        for (int64_t s = n * w.split / a.split; s < n * (w.split + 1) / a.split; ++s) rest(s >= per, (s >= per ? s - per : s) * kStep);
    } else if (w.split == a.split - 1) {
        for (int k = 0; k < kSums; ++k)
            for (int64_t c0 = static_cast<int64_t>(n_whole) * kStep; c0 < a.C; c0 += kStep) rest(k, c0);
    }
    if (a.split > 1) {
        float *const out = a.part + ((static_cast<int64_t>(w.tile) * a.split + w.split) * G::kWaves + wave) * (kPB * kTB * 1024) + lane;
#pragma unroll
        for (int b = 0; b < kPB; ++b)
#pragma unroll
            for (int t = 0; t < kTB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) out[((b * kTB + t) * 16 + r) * 64] = acc[b][t][r];
        return;
    }
    __syncthreads();
    using E = Exchange<kPB, kForward>;
    float *const region = reinterpret_cast<float *>(lds + wave * E::kBytes);
    finish<T, kPB, kForward>(a, region, w.m0 + wave_t * kTB * 32, w.r0 + wave_p * E::kWide, kTB, [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int tt = 0; tt < kTB; ++tt)
            if (t == tt) {
#pragma unroll
                for (int b = 0; b < kPB; ++b) E::put(region, b, acc[b][tt]);
            }
    });
}

// split > 1: the parts of a sum added up in a fixed order, then as above.  A wavefront takes what one of the tile's had of 32 tokens.
template <typename T, typename G, bool kForward>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a) {
    using E = Exchange<G::kPB, kForward>;
    constexpr int kUnits = G::kTB * G::kWaves;                           // of a tile
    __shared__ __attribute__((aligned(16))) char lds[4 * E::kBytes];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t at = blockIdx.x * 4 + own, tile = at / kUnits;
    if (tile >= a.tiles_m * a.tiles_r) return;
    const int unit = static_cast<int>(at - tile * kUnits), wave = unit / G::kTB, t = unit % G::kTB;
    const Place w = place_of<G, kForward>(a, tile);
    float *const region = reinterpret_cast<float *>(lds + own * E::kBytes);
    f32x16 acc[G::kPB] = {};
    const float *from = a.part + (static_cast<int64_t>(tile) * a.split * G::kWaves + wave) * (G::kPB * G::kTB * 1024) + lane;
    for (uint32_t s = 0; s < a.split; ++s, from += G::kWaves * G::kPB * G::kTB * 1024)
#pragma unroll
        for (int b = 0; b < G::kPB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] += from[((b * G::kTB + t) * 16 + r) * 64];
    finish<T, G::kPB, kForward>(a, region, w.m0 + (wave % G::kWT * G::kTB + t) * 32, w.r0 + wave / G::kWT * E::kWide, 1, [&](int) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < G::kPB; ++b) E::put(region, b, acc[b]);
    });
}

// Launches a tile's kernels.  A launch takes kMost tiles each way at most (it has room for 2^32 threads, and wraps silently beyond).
constexpr int64_t kMost = 1 << 11;
template <typename T, typename G, bool kForward>
int run_tiles(const ::tensile_ops *ops, hipStream_t s, const ProductArgs &whole, bool far, int64_t split, const char *what) {
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
        const int rc = scratch.provide(static_cast<size_t>(tiles_m * tiles_r * split) * G::kP * G::kTok, what);
        if (rc != TENSILE_OK) return rc;
        part = scratch.buf.p;
    }
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
            const dim3 grid(a.tiles_m * a.tiles_r * a.split), block(G::kThreads);
            if (far) hipLaunchKernelGGL(HIP_KERNEL_NAME(product_kernel<T, G, kForward, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL(HIP_KERNEL_NAME(product_kernel<T, G, kForward, false>), grid, block, 0, s, a);
            TS_HIP(hipGetLastError());
            if (split > 1) {
                const uint32_t units = a.tiles_m * a.tiles_r * (G::kTB * G::kWaves);
                hipLaunchKernelGGL(HIP_KERNEL_NAME(product_join_kernel<T, G, kForward>), dim3((units + 3) / 4), dim3(256), 0, s, a);
                TS_HIP(hipGetLastError());
            }
        }
    return TENSILE_OK;
}

// Rows further apart than this are reached by 64-bit addresses only (256 of them, or 32 of a step, from a scalar one).
constexpr int64_t kFarBytes = 1 << 23;
inline bool is_far(const Matrix &m, int64_t size) { return m.ld * size >= kFarBytes; }

using Large = Tile<4, 2, 2, 4, 1>;    // 256 x 256
using Small = Tile<2, 2, 2, 2, 2>;    // 128 x 128

}  // namespace

}  // namespace tensile
