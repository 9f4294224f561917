// Gradients of a linear layer's parameters from an 8-bit checkpoint of its input:
//   dw[n,k] = sum_m dy[m,n] * X[m,k],   dbias[n] = sum_m dy[m,n]
// and, where the checkpoint holds a layer norm's xhat, X = xhat*gamma + beta, which leaves the product as it is:
//   dw[n,k] = gamma[k] * sum_m dy[m,n]*xhat[m,k] + beta[k] * dbias[n].
//
// The product runs on the bf16 matrix instructions with 32-bit sums.  A checkpoint's value (7 bits times a power of two) is
// a bf16 number, and dy is one, or the exact sum of two (f16) or three (f32): each piece is a product of its own, so no
// operand is rounded.
//
// Both operands lie in memory with the summed index (the row) outermost, while a matrix instruction wants eight consecutive
// values of it in a lane: rows are staged in the LDS as they are and read transposed (ds_read_tr16_b64: 16 lanes read four
// rows of 16 columns and each gets the four values of its column).
#include "ops_device.h"

#include <type_traits>

namespace tensile {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// (the LDS-direct loads below take their target from m0, which the compiler counts as its own and says so)
#pragma clang diagnostic ignored "-Winline-asm"

// (16 bytes at any alignment)
typedef u32x4 u32x4_anywhere __attribute__((aligned(1)));
typedef const __attribute__((address_space(1))) char *global_bytes;
typedef const __attribute__((address_space(1))) u32x4_anywhere *global_16;

constexpr uint32_t kXcds = 8, kBand = 8;

// How many bf16 numbers add up to an element of dy.
template <typename T> struct Pieces;
template <> struct Pieces<bf16_t> { static constexpr int n = 1; };
template <> struct Pieces<f16_t> { static constexpr int n = 2; };
template <> struct Pieces<float> { static constexpr int n = 3; };

struct GradArgs {
    LinearArgs a;
    int32_t tiles_n, tiles_k, split;
    int64_t rows_per_split;
    // split > 1: the sums as the tiles' lanes hold them, [tile][split][wavefront][block][register][lane], then [split][N] sums of dy
    float *part;
};

// A staged row's 16-column blocks (32 bytes) are stored in an order that depends on the row: the 4 rows x 2 blocks
// that half a wavefront reads at a time lie in different banks.
template <int kRowBytes>
__device__ __forceinline__ int swizzle(int row, int block) { return row * kRowBytes + ((block ^ (2 * (row & 3))) * 32); }

// x = p[0] + p[1] + ...: each piece the leading 8 bits of what is left (exact); infinities and NaN are all in the first.  (Quieted: a
// NaN whose bits are all in the lower half would be an infinity.)
template <int kPieces>
__device__ __forceinline__ void split_bf16(float x, uint32_t (&p)[kPieces]) {
    x = __builtin_canonicalizef(x);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const uint32_t top = as_u32(x) & 0xffff0000u;
        p[k] = top;
        const float rest = x - as_f32(top);
        x = k == 0 && (top & 0x7f800000u) == 0x7f800000u ? 0.0f : rest;
    }
}

// The 16 bytes moved down by `bytes` (0 .. 15), zeros behind them.
__device__ __forceinline__ u32x4 shift_out(u32x4 w, int bytes) {
    const u32x4 two = bytes & 8 ? u32x4{w[2], w[3], 0, 0} : w;
    const u32x4 one = bytes & 4 ? u32x4{two[1], two[2], two[3], 0} : two;
    const uint32_t b = bytes & 3;
    return u32x4{__builtin_amdgcn_alignbyte(one[1], one[0], b), __builtin_amdgcn_alignbyte(one[2], one[1], b),
                 __builtin_amdgcn_alignbyte(one[3], one[2], b), __builtin_amdgcn_alignbyte(0, one[3], b)};
}
// Eight elements without their first n (0 .. 7), zeros behind them; all zero unless `keep`.
template <typename T>
__device__ __forceinline__ void drop_front(Raw8<T> &r, int n, bool keep) {
    r.v = keep ? shift_out(r.v, 2 * n) : u32x4{0, 0, 0, 0};
}
__device__ __forceinline__ void drop_front(Raw8<float> &r, int n, bool keep) {
    const u32x4 none = {0, 0, 0, 0};
    const u32x4 v = n & 4 ? r.w : r.v, w = n & 4 ? none : r.w;
    const u32x4 v2 = n & 2 ? u32x4{v[2], v[3], w[0], w[1]} : v, w2 = n & 2 ? u32x4{w[2], w[3], 0, 0} : w;
    const u32x4 v3 = n & 1 ? u32x4{v2[1], v2[2], v2[3], w2[0]} : v2, w3 = n & 1 ? u32x4{w2[1], w2[2], w2[3], 0} : w2;
    r.v = keep ? v3 : none;
    r.w = keep ? w3 : none;
}

// A workgroup's tile: kWN x kWK wavefronts of 32 kNB columns of dy x 32 kKB columns of the checkpoint each, two wavefronts to a
// SIMD in all; 32 rows to a step.  kByHalves: the columns of the checkpoint lie in the tile in the order that the streaming
// kernel's staging gives them, of 128 the first halves of eight sixteens and then the second.  A wavefront takes one block of
// each: of four sixteens both halves.
template <int kNB_, int kKB_, int kWN_, int kWK_, bool kByHalves_ = false>
struct Tile {
    static constexpr int kNB = kNB_, kKB = kKB_, kWN = kWN_, kWK = kWK_;
    static constexpr bool kByHalves = kByHalves_;
    static constexpr int kThreads = 64 * kWN * kWK, kN = 32 * kNB * kWN, kK = 32 * kKB * kWK;
    static constexpr int kPerCu = 512 / kThreads;
    // The sums of dy are taken by the kWK wavefronts that share its columns: every second one takes the same 16 rows of a step
    // (see the kernels), and of these each a part of the blocks, kSum, which are its first.
    static constexpr int kSum = 2 * kNB / kWK;
    static_assert(kNB % kSum == 0 && (kNB & (kNB - 1)) == 0, "");
    static __device__ __forceinline__ int block(int wave, int i) { return i ^ (wave % kWK / 2 * kSum); }
    // row and column of the tile that a lane's register r of block (i, j) is
    static __device__ __forceinline__ int row(int wave, int lane, int i, int r) {
        return (wave / kWK * kNB + block(wave, i)) * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
    }
    static __device__ __forceinline__ int column_block(int wave, int j) {
        return kByHalves ? wave % kWK / 2 * 4 + wave % 2 + 2 * j : wave % kWK * kKB + j;
    }
    // (kByHalves: as `by_columns` leaves them)
    static __device__ __forceinline__ int column(int wave, int lane, int j) {
        const int in = lane & 31;
        return (wave % kWK * kKB + j) * 32 + (kByHalves ? (in >> 3) % 2 * 16 + (in >> 4) * 8 + in % 8 : in);
    }
    // kByHalves: block 0 is given the first two of the wavefront's four sixteens, block 1 the others, so that a store has 32 columns
    // of a row to itself: the second row of 16 lanes of block 0 and the first of block 1 change places.  (A store of eight times 8
    // columns is twice the requests: 100 x 4096 x 4096 22.6 us against 19.9, 64 x 8192 x 8192, 268 MB of dw, 59 against 55.)
    static __device__ __forceinline__ void by_columns(f32x16 (&acc)[kNB][kKB]) {
        if constexpr (kByHalves) {
            static_assert(kKB == 2 && kWK % 2 == 0, "");
#pragma unroll
            for (int i = 0; i < kNB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const auto v = __builtin_amdgcn_permlane16_swap(as_u32(acc[i][0][r]), as_u32(acc[i][1][r]), false, false);
                    acc[i][0][r] = as_f32(v[0]);
                    acc[i][1][r] = as_f32(v[1]);
                }
        }
    }
};
using Staged = Tile<2, 2, 2, 2>;             // 128 x 128, two workgroups to a CU, by way of registers
using StagedWide = Tile<2, 2, 2, 4>;         // 128 x 256, one workgroup to a CU
using Narrow = Tile<2, 2, 2, 2, true>;       // the same for the kernel of 16-bit brain floats
using Wide = Tile<4, 2, 2, 4, true>;         // 256 x 256, one workgroup to a CU
constexpr int kRows = 32;
constexpr int kPartRows = 256;               // of a part at least, where the rows are split

// Where a workgroup works.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD gets a run of consecutive
// tiles, and consecutive tiles lie in bands kBand tiles high, so that those under way on an XCD share their rows of both operands.
struct Place {
    int split, tile, n0, k0;
    bool last;                        // of the splits
    int64_t m_begin, m_end;
};
template <typename G>
__device__ __forceinline__ Place place(const GradArgs &g) {
    const uint32_t total = gridDim.x, xcd = blockIdx.x % kXcds;
    const uint32_t at = xcd * (total / kXcds) + (xcd < total % kXcds ? xcd : total % kXcds) + blockIdx.x / kXcds;
    const uint32_t tiles = static_cast<uint32_t>(g.tiles_n) * g.tiles_k, tile = at % tiles;
    const uint32_t band = tile / (kBand * g.tiles_k), in_band = tile % (kBand * g.tiles_k);
    const uint32_t high = g.tiles_n - band * kBand < kBand ? g.tiles_n - band * kBand : kBand;
    Place w;
    w.split = static_cast<int>(at / tiles);
    const uint32_t n = band * kBand + in_band % high, k = in_band / high;
    w.tile = static_cast<int>(n * g.tiles_k + k);
    w.n0 = static_cast<int>(n) * G::kN;
    w.k0 = static_cast<int>(k) * G::kK;
    w.m_begin = w.split * g.rows_per_split;
    // (The end is chosen by a 32-bit comparison, not as the smaller of two 64-bit rows: for that, uniform as it is, hipcc of ROCm 7.2 has put a
    // vector comparison in front of a scalar selection, which then goes by the carry of an addition: every part ran to the last row.)
    w.last = w.split == g.split - 1;
    w.m_end = w.last ? g.a.M : w.m_begin + g.rows_per_split;
    return w;
}

template <typename T>
__device__ __forceinline__ void put_as(int type, void *p, int64_t at, float v) {
    if (type == TENSILE_F32) static_cast<float *>(p)[at] = v;
    else from_f32(v, static_cast<T *>(p)[at]);
}
template <typename T>
__device__ __forceinline__ float get_as(int type, const void *p, int64_t at) {
    return type == TENSILE_F32 ? static_cast<const float *>(p)[at] : to_f32(static_cast<const T *>(p)[at]);
}

// What a workgroup does with its tile's sums: dbias, and dw with the norm's parameters, or all as they are where the rows are split.
// `sums` is LDS for two rows of the tile's width.
template <typename T, typename G>
__device__ __forceinline__ void finish(const GradArgs &g, const Place &w, f32x16 (&acc)[G::kNB][G::kKB], const float (&bias)[G::kSum],
                                       bool use_bias, float *sums) {
    constexpr int kNB = G::kNB, kKB = G::kKB;
    const LinearArgs &a = g.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    G::by_columns(acc);
    // sums of dy: over the two halves of the wavefront, then over the two halves of the steps
    if (use_bias) {
#pragma unroll
        for (int i = 0; i < G::kSum; ++i) {
            const float s = bias[i] + __shfl_xor(bias[i], 32);
            if (lane < 32) sums[wave % 2 * G::kN + (wave / G::kWK * kNB + G::block(wave, i)) * 32 + lane] = s;
        }
        __syncthreads();
        if (tid < G::kN) sums[tid] = sums[tid] + sums[G::kN + tid];
        __syncthreads();
    }
    if (g.split > 1) {
        constexpr int64_t kElements = static_cast<int64_t>(G::kN) * G::kK;
        float *out = g.part + (static_cast<int64_t>(w.tile) * g.split + w.split) * kElements + wave * (kNB * kKB * 1024) + lane;
#pragma unroll
        for (int i = 0; i < kNB; ++i)
#pragma unroll
            for (int j = 0; j < kKB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) out[((i * kKB + j) * 16 + r) * 64] = acc[i][j][r];
        if (w.k0 == 0 && use_bias && tid < G::kN && w.n0 + tid < a.N)
            g.part[static_cast<int64_t>(g.tiles_n) * g.tiles_k * g.split * kElements + static_cast<int64_t>(w.split) * a.N + w.n0 + tid] = sums[tid];
        return;
    }
    if (w.k0 == 0 && a.dbias && tid < G::kN && w.n0 + tid < a.N) put_as<T>(a.dw_type, a.dbias, w.n0 + tid, sums[tid]);
    float gamma[kKB], beta[kKB];
#pragma unroll
    for (int j = 0; j < kKB; ++j) {
        const int k = w.k0 + G::column(wave, lane, j);
        gamma[j] = a.gamma && k < a.K ? get_as<T>(a.param_type, a.gamma, k) : 1.0f;
        beta[j] = a.gamma && k < a.K ? get_as<T>(a.param_type, a.beta, k) : 0.0f;
    }
    // (What is asked for every element costs as much as the store: whether it exists, which type it has.)
    auto write = [&](auto whole, auto wide) __attribute__((always_inline)) {
        using Out = typename std::conditional<decltype(wide)::value, float, T>::type;
#pragma unroll
        for (int i = 0; i < kNB; ++i) {
            // (the sums of the lane's sixteen rows first, four at a time: an LDS read before every store costs 12 us a tile)
            float own[16] = {};
            if (a.gamma) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 s = *reinterpret_cast<const f32x4 *>(sums + G::row(wave, lane, i, r));
#pragma unroll
                    for (int u = 0; u < 4; ++u) own[r + u] = s[u];
                }
            }
#pragma unroll
            for (int j = 0; j < kKB; ++j) {
                const int k = w.k0 + G::column(wave, lane, j);
                if (!decltype(whole)::value && k >= a.K) continue;
                Out *const to = static_cast<Out *>(a.dw.p) + k;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int n = w.n0 + G::row(wave, lane, i, r);
                    if (!decltype(whole)::value && n >= a.N) continue;
                    from_f32(__builtin_fmaf(acc[i][j][r], gamma[j], beta[j] * own[r]), to[static_cast<int64_t>(n) * a.dw.ld]);
                }
            }
        }
    };
    const bool whole = w.n0 + G::kN <= a.N && w.k0 + G::kK <= a.K;
    if (a.dw_type == TENSILE_F32) {
        if (whole) write(std::true_type{}, std::true_type{});
        else write(std::false_type{}, std::true_type{});
    } else {
        if (whole) write(std::true_type{}, std::false_type{});
        else write(std::false_type{}, std::false_type{});
    }
}

// The product for any type; 32 and 16-bit gradients are three and two pieces, each a product of its own, and bound by those:
// 6000 x 8192 x 8192 2350 us (f32) and 1780 us (f16), 1030 and 900 TFLOP/s in pieces; 4096 x 4096 x 4096 391 and 307 us.  Beside the
// products it is ordinary instructions that count: to a matrix instruction 5.5 on vectors (f32), of which 3.2 take dy apart.
// kByElement: matrices with rows shorter than a load, or too far apart for 32-bit offsets.
template <typename T, typename G, bool kByElement>
__global__ __launch_bounds__(G::kThreads, 2) void linear_grad_kernel(GradArgs g) {
    constexpr int kNB = G::kNB, kKB = G::kKB, kP = Pieces<T>::n;
    constexpr int kTileN = G::kN, kTileK = G::kK;
    constexpr int kRowN = 2 * kTileN, kRowK = 2 * kTileK;                // bytes of a staged row
    constexpr int kPlane = kRows * kRowN;                                // of a staged piece of dy
    constexpr int kBuffer = kP * kPlane + kRows * kRowK;
    constexpr int kDyPer = 8 * G::kThreads / kTileN, kXPer = 16 * G::kThreads / kTileK;   // rows that the workgroup loads at once
    constexpr int kDyLoads = kRows / kDyPer, kXLoads = kRows / kXPer;    // per thread and step
    static_assert(kDyPer % 4 == 0 && kXPer % 4 == 0 && kRows % kXPer == 0 && kRows % kDyPer == 0, "");
    __shared__ __attribute__((aligned(16))) char lds[2 * kBuffer];
    const LinearArgs &a = g.a;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wave_n = wave / G::kWK, wave_k = wave % G::kWK;
    const Place w = place<G>(g);
    const int n0 = w.n0, k0 = w.k0;
    const int64_t m_begin = w.m_begin, m_end = w.m_end;

    // staging: a thread loads 8 columns of dy, 16 of the checkpoint, of a row at a time
    const int dy_row = tid / (kTileN / 8), dy_col = tid % (kTileN / 8) * 8;
    const int x_row = tid / (kTileK / 16), x_col = tid % (kTileK / 16) * 16;
    const int dy_left = a.N - n0 - dy_col, x_left = a.K - k0 - x_col;
    // (threads without a column load the first ones: they end in columns of the tile that are not stored)
    const int dy_from = dy_left > 0 ? n0 + dy_col : 0, x_from = x_left > 0 ? k0 + x_col : 0;
    uint32_t dy_off[kDyLoads], x_off[kXLoads], s_off[kXLoads];           // from the step's first row
#pragma unroll
    for (int i = 0; i < kDyLoads; ++i)
        dy_off[i] = static_cast<uint32_t>(((dy_row + kDyPer * i) * a.dy.ld + dy_from) * static_cast<int64_t>(sizeof(T)));
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
        x_off[i] = static_cast<uint32_t>((x_row + kXPer * i) * a.c.ld_q + x_from);
        s_off[i] = static_cast<uint32_t>((x_row + kXPer * i) * a.c.ld_scale + x_from / kGroup);
    }
    const char *const dy_base = static_cast<const char *>(a.dy.p);
    const int64_t dy_pitch = a.dy.ld * static_cast<int64_t>(sizeof(T));

    Raw8<T> dy_raw[kDyLoads];
    u32x4 x_raw[kXLoads];
    uint32_t x_code[kXLoads];
    // Whole rows: what lies behind a row's last column is read along (it is the next row's, or between the rows).  (The asm keeps
    // the step's address in scalar registers, beside 32-bit offsets: else every load has a 64-bit pointer of its own.)
    auto request_dy = [&](int64_t m) __attribute__((always_inline)) {
        global_bytes from = (global_bytes)(dy_base + m * dy_pitch);
        asm volatile("" : "+s"(from));
#pragma unroll
        for (int i = 0; i < kDyLoads; ++i) {
            dy_raw[i].v = *(global_16)(from + dy_off[i]);
            if constexpr (sizeof(T) == 4) dy_raw[i].w = *(global_16)(from + dy_off[i] + 16);
        }
    };
    auto request_x = [&](int64_t m) __attribute__((always_inline)) {
        global_bytes from = (global_bytes)(a.c.q + m * a.c.ld_q), codes = (global_bytes)(a.c.scale + m * a.c.ld_scale);
        asm volatile("" : "+s"(from), "+s"(codes));
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            x_raw[i] = *(global_16)(from + x_off[i]);
            x_code[i] = static_cast<uint8_t>(codes[s_off[i]]);
        }
    };
    // The same where rows may be missing or be the matrix's last: a thread whose columns do not all exist reads as many
    // before them and shifts those out; a missing row reads the last one and becomes zero.
    const int dy_over = dy_left > 0 && dy_left < 8 ? 8 - dy_left : 0, x_over = x_left > 0 && x_left < 16 ? 16 - x_left : 0;
    auto last_dy = [&](int64_t m) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kDyLoads; ++i) {
            const int64_t r = m + dy_row + kDyPer * i;
            if constexpr (kByElement) {
                dy_raw[i] = Raw8<T>{};
                if (r < m_end && dy_left > 0) dy_raw[i] = load_raw(static_cast<const T *>(a.dy.p) + r * a.dy.ld + dy_from, dy_left);
                continue;
            }
            const char *const from = dy_base + (r < m_end ? r : m_end - 1) * dy_pitch;
            __builtin_memcpy(&dy_raw[i], from + static_cast<int64_t>(dy_from - dy_over) * static_cast<int64_t>(sizeof(T)), sizeof dy_raw[i]);
            drop_front(dy_raw[i], dy_over, r < m_end);
        }
    };
    auto last_x = [&](int64_t m) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            const int64_t r = m + x_row + kXPer * i, rr = r < m_end ? r : m_end - 1;
            if constexpr (kByElement) {
                x_raw[i] = u32x4{0, 0, 0, 0};
                x_code[i] = 0;
                if (r < m_end && x_left > 0) {
                    const int8_t *const from = a.c.q + r * a.c.ld_q + x_from;
                    const u32x2 lo = load_q(from, x_left), hi = x_left > 8 ? load_q(from + 8, x_left - 8) : u32x2{0, 0};
                    x_raw[i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                    x_code[i] = a.c.scale[r * a.c.ld_scale + x_from / kGroup];
                }
                continue;
            }
            __builtin_memcpy(&x_raw[i], a.c.q + rr * a.c.ld_q + (x_from - x_over), 16);
            x_raw[i] = shift_out(x_raw[i], x_over);
            x_code[i] = r < m_end ? a.c.scale[rr * a.c.ld_scale + x_from / kGroup] : 0;
            if (r >= m_end) x_raw[i] = u32x4{0, 0, 0, 0};
        }
    };
    const int dy_at = swizzle<kRowN>(dy_row, dy_col / 16) + (dy_col % 16) * 2;
    const int x_at = kP * kPlane + swizzle<kRowK>(x_row, x_col / 16);
    auto stage_dy = [&](char *to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kDyLoads; ++i) {
            char *at = to + dy_at + i * kDyPer * kRowN;
            if constexpr (kP == 1) {
                *reinterpret_cast<u32x4 *>(at) = dy_raw[i].v;
            } else {
                float f[8];
                widen(dy_raw[i], f);
                u32x4 w[kP];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t lo[kP], hi[kP];
                    split_bf16<kP>(f[2 * j], lo);
                    split_bf16<kP>(f[2 * j + 1], hi);
#pragma unroll
                    for (int p = 0; p < kP; ++p) w[p][j] = __builtin_amdgcn_perm(hi[p], lo[p], 0x07060302);
                }
#pragma unroll
                for (int p = 0; p < kP; ++p) *reinterpret_cast<u32x4 *>(at + p * kPlane) = w[p];
            }
        }
    };
    auto stage_x = [&](char *to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            char *at = to + x_at + i * kXPer * kRowK;
            const float scale = scale_of(x_code[i]);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float f[8];
                unpack8(u32x2{x_raw[i][2 * half], x_raw[i][2 * half + 1]}, scale, f);
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(as_u32(f[2 * j + 1]), as_u32(f[2 * j]), 0x07060302);
                *reinterpret_cast<u32x4 *>(at + half * 16) = w;
            }
        }
    };

    f32x16 acc[kNB][kKB] = {};
    float bias[G::kSum] = {};
    const bool use_bias = a.gamma || (k0 == 0 && a.dbias);
    // transposed reads: the lanes of a group of 16 read rows 8h .. 8h+3 (and +4) of 16 columns
    const int i16 = lane & 15, group = lane >> 4;
    const int t_row = (group >> 1) * 8 + i16 / 4, t_in = (i16 & 3) * 8;
    // Of a step's two blocks of 16 rows a wave takes first the one of its parity in the row of the tile: the sums of dy are
    // taken of that one only, by the waves that share its columns, without a branch.
    const int turn = wave_k & 1;
    int a_at[2][kNB], b_at[2][kKB];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int row = t_row + 16 * (e ^ turn);
#pragma unroll
        for (int b = 0; b < kNB; ++b) a_at[e][b] = swizzle<kRowN>(row, (wave_n * kNB + G::block(wave, b)) * 2 + (group & 1)) + t_in;
#pragma unroll
        for (int b = 0; b < kKB; ++b) b_at[e][b] = kP * kPlane + swizzle<kRowK>(row, G::column_block(wave, b) * 2 + (group & 1)) + t_in;
    }
    auto fragment = [&](const char *p, int four_rows) __attribute__((always_inline)) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + four_rows));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // A step is a chain of phases, one for each 16 rows and piece.  A phase multiplies the fragments that the phase before it has
    // read and reads those of the next one; the last phase of a step, behind the barrier, reads the first of the next step.
    constexpr int kPhases = 2 * kP;
    bf16x8 fa[2][kNB], fb[2][kKB];
    auto read = [&](int q, const char *from) __attribute__((always_inline)) {
        const int e = q / kP, p = q % kP;
#pragma unroll
        for (int b = 0; b < kNB; ++b) fa[q & 1][b] = fragment(from + p * kPlane + a_at[e][b], 4 * kRowN);
        if (p == 0) {
#pragma unroll
            for (int b = 0; b < kKB; ++b) fb[e][b] = fragment(from + b_at[e][b], 4 * kRowK);
        }
    };
    auto multiply = [&](int q, auto sums) __attribute__((always_inline)) {
        const int e = q / kP;
#pragma unroll
        for (int i = 0; i < kNB; ++i)
#pragma unroll
            for (int j = 0; j < kKB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[q & 1][i], fb[e][j], acc[i][j], 0, 0, 0);
        if constexpr (decltype(sums)::value) {
            if (e == 0) {
                const bf16x2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
                for (int i = 0; i < G::kSum; ++i) {
                    float s = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bf16x2 v = {fa[q & 1][i][2 * j], fa[q & 1][i][2 * j + 1]};
                        s = __builtin_amdgcn_fdot2_f32_bf16(v, one, s, false);
                    }
                    bias[i] += s;
                }
            }
        }
    };
    // (not __syncthreads, which would also wait for the loads from memory that are under way)
    auto lds_barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    // One step: rows m .. m+31 are in `now` and the first fragments in registers.  Before the barrier the next step's rows of
    // dy go to `next`, where its rows of the checkpoint are already; behind it `now` is free, and the rows of the
    // checkpoint after those go there.
    auto step = [&](int64_t m, char *now, char *next, auto whole, auto sums) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < kPhases; ++q) {
            if (q < kPhases - 1) {
                read(q + 1, now);
                if (q == 0) {
                    stage_dy(next);
                    if constexpr (decltype(whole)::value) request_dy(m + 2 * kRows);
                    else last_dy(m + 2 * kRows);
                }
            } else {
                lds_barrier();
                read(0, next);
                stage_x(now);
                if constexpr (decltype(whole)::value) request_x(m + 3 * kRows);
                else last_x(m + 3 * kRows);
            }
            multiply(q, sums);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const int64_t whole_end = w.last ? a.M - 1 : m_end;                  // rows that may be read whole
    auto steps = [&](auto sums) __attribute__((always_inline)) {
        int64_t m = m_begin;
        for (; !kByElement && m + 5 * kRows <= whole_end; m += 2 * kRows) {
            step(m, lds, lds + kBuffer, std::true_type{}, sums);
            step(m + kRows, lds + kBuffer, lds, std::true_type{}, sums);
        }
        char *now = lds, *next = lds + kBuffer;
        for (; m < m_end; m += kRows) {
            step(m, now, next, std::false_type{}, sums);
            char *const other = now;
            now = next;
            next = other;
        }
    };
    if (m_begin < m_end) {
        last_dy(m_begin);
        last_x(m_begin);
        stage_dy(lds);
        stage_x(lds);
        last_x(m_begin + kRows);
        stage_x(lds + kBuffer);
        last_dy(m_begin + kRows);
        last_x(m_begin + 2 * kRows);
        // (vmcnt(0): the compiler would else wait in every step as if the loop had just been entered, for the newest loads too)
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
        read(0, lds);
        if (use_bias) steps(std::true_type{});
        else steps(std::false_type{});
        __syncthreads();
    }

    finish<T, G>(g, w, acc, bias, use_bias, reinterpret_cast<float *>(lds));
}

// The same for a bf16 gradient.  What is on its way from memory lies in the LDS, not in registers: dy three steps ahead and the
// checkpoint four, some 90 KB to a CU.  With registers to hold it one step was all there was room for, and the loads were what
// bounded the kernel (16384 x 8192 x 8192, 256 x 256 tiles: 2230 us, 1480 without them, 1780 so).  Of the LDS's 160 KB a CU's
// workgroups have 136: two wavefronts to a SIMD, which hide about four ordinary instructions behind each matrix instruction; of the
// large tile there are 2.9, and 3.2 where dy is summed.  What is left: the chip lowers its clock to 1.9 to 2.0 GHz.
template <typename G>
__global__ __launch_bounds__(G::kThreads, 2) void linear_grad_stream_kernel(GradArgs g) {
    constexpr int kNB = G::kNB, kKB = G::kKB, kRowN = 2 * G::kN, kRowK = 2 * G::kK;
    constexpr int kSlotN = kRows * kRowN, kSlotK = kRows * kRowK, kRaw = kRows * G::kK;   // a step's rows: staged, and as they are held
    constexpr int kCodes = 4 * G::kThreads;                              // ... a code takes four bytes
    constexpr int kDy = 0, kX = 4 * kSlotN, kQ = kX + 2 * kSlotK, kC = kQ + 4 * kRaw;   // four steps of dy, two of X, four of the checkpoint
    constexpr int kOwn = kRows * 64 / G::kThreads;                       // rows that a wave brings, 64 times 16 bytes at a time:
    constexpr int kDyRows = 64 * 8 / G::kN, kXRows = 64 * 16 / G::kK;    // 8 columns of dy to a lane, 16 of the checkpoint
    static_assert(kOwn == 2 * kDyRows && kOwn == kXRows && G::kByHalves, "");
    __shared__ __attribute__((aligned(1024))) char lds[kC + 4 * kCodes];
    typedef __attribute__((address_space(3))) char lds_char;
    const LinearArgs &a = g.a;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave_n = wave / G::kWK, wave_k = wave % G::kWK;
    const Place w = place<G>(g);
    const int n0 = w.n0, k0 = w.k0;
    const int64_t m_begin = w.m_begin, m_end = w.m_end;

    // The LDS takes 16 bytes of each lane in the order of the lanes, so the staged rows' order of blocks (swizzle) is that of
    // the addresses.
    uint32_t dy_off[2];
    int dy_over[2];                   // columns of the lane's eight that do not exist (only the last rows' loads care)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        constexpr int kLanes = 64 / kDyRows;
        const int row = kOwn * wave + kDyRows * j + lane / kLanes, block = (lane % kLanes >> 1) ^ (2 * (row & 3));
        const int col = n0 + block * 16 + (lane & 1) * 8;
        dy_off[j] = static_cast<uint32_t>((row * a.dy.ld + (col < a.N ? col : 0)) * 2);    // (no such column: any will do)
        dy_over[j] = col < a.N && col + 8 > a.N ? col + 8 - a.N : 0;
    }
    // (a thread dequantises what it has brought)
    const int x_row = kOwn * wave + lane / (64 / kXRows), x_col = lane % (64 / kXRows) * 16;
    const int x_from = k0 + x_col < a.K ? k0 + x_col : 0;
    const uint32_t x_off = static_cast<uint32_t>(x_row * a.c.ld_q + x_from);
    const uint32_t s_off = static_cast<uint32_t>(x_row * a.c.ld_scale + x_from / kGroup);
    // (first the first halves of eight threads' columns, then the second: 128 bytes at a time, without a bank conflict; see Tile)
    int x_at[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int chunk = (lane & 7) + 8 * half + 16 * (x_col / 128);
        x_at[half] = kX + swizzle<kRowK>(x_row, chunk >> 1) + (chunk & 1) * 16;
    }

    // From memory to the LDS without a register in between.  (By hand: of the builtin the compiler waits for every one under way
    // before the next LDS read, whatever it reads.  They write no register; the waits are at the barriers below.)
    auto bring = [&](uint32_t to, global_bytes from, uint32_t off) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(from) : "memory", "m0");
    };
    const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)lds));
    auto bring_dy = [&](int64_t m, int slot) __attribute__((always_inline)) {
        const global_bytes from = (global_bytes)(static_cast<const char *>(a.dy.p) + m * a.dy.ld * 2);
#pragma unroll
        for (int j = 0; j < 2; ++j) bring(lds_at + kDy + slot * kSlotN + (kOwn * wave + kDyRows * j) * kRowN, from, dy_off[j]);
    };
    auto bring_x = [&](int64_t m, int slot) __attribute__((always_inline)) {
        bring(lds_at + kQ + slot * kRaw + wave * 1024, (global_bytes)(a.c.q + m * a.c.ld_q), x_off);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" ::"s"(lds_at + kC + slot * kCodes + wave * 256), "v"(s_off),
                     "s"((global_bytes)(a.c.scale + m * a.c.ld_scale)) : "memory", "m0");
    };
    struct Sixteen {
        u32x4 v[2];
    };
    auto dequantised = [&](u32x4 raw, uint32_t c) __attribute__((always_inline)) {
        const float scale = scale_of(c);
        Sixteen w;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float f[8];
            unpack8(u32x2{raw[2 * half], raw[2 * half + 1]}, scale, f);
#pragma unroll
            for (int j = 0; j < 4; ++j) w.v[half][j] = __builtin_amdgcn_perm(as_u32(f[2 * j + 1]), as_u32(f[2 * j]), 0x07060302);
        }
        return w;
    };
    auto held = [&](int slot) __attribute__((always_inline)) {
        return dequantised(*reinterpret_cast<const u32x4 *>(lds + kQ + slot * kRaw + tid * 16), *reinterpret_cast<const uint8_t *>(lds + kC + slot * kCodes + tid * 4));
    };
    auto put = [&](const Sixteen &w, int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < 2; ++half) *reinterpret_cast<u32x4 *>(lds + x_at[half] + slot * kSlotK) = w.v[half];
    };

    f32x16 acc[kNB][kKB] = {};
    float bias[G::kSum] = {};
    const bool use_bias = a.gamma || (k0 == 0 && a.dbias);
    const int i16 = lane & 15, group = lane >> 4;
    const int t_row = (group >> 1) * 8 + i16 / 4, t_in = (i16 & 3) * 8;
    const int turn = wave_k & 1;                                         // (see above)
    int a_at[2][kNB], b_at[2][kKB];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int row = t_row + 16 * (e ^ turn);
#pragma unroll
        for (int b = 0; b < kNB; ++b) a_at[e][b] = kDy + swizzle<kRowN>(row, (wave_n * kNB + G::block(wave, b)) * 2 + (group & 1)) + t_in;
#pragma unroll
        for (int b = 0; b < kKB; ++b) b_at[e][b] = kX + swizzle<kRowK>(row, G::column_block(wave, b) * 2 + (group & 1)) + t_in;
    }
    auto fragment = [&](int p, int four_rows) __attribute__((always_inline)) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((lds_char *)lds + p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((lds_char *)lds + p + four_rows));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    bf16x8 fa[2][kNB], fb[2][kKB];
    auto read = [&](int e, int dy_slot, int x_slot) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < kNB; ++b) fa[e][b] = fragment(a_at[e][b] + dy_slot * kSlotN, 4 * kRowN);
#pragma unroll
        for (int b = 0; b < kKB; ++b) fb[e][b] = fragment(b_at[e][b] + x_slot * kSlotK, 4 * kRowK);
    };
    auto multiply = [&](int e, auto sums) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kNB; ++i)
#pragma unroll
            for (int j = 0; j < kKB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[e][i], fb[e][j], acc[i][j], 0, 0, 0);
        if constexpr (decltype(sums)::value) {
            if (e == 0) {
                const bf16x2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
                for (int i = 0; i < G::kSum; ++i) {
                    float s = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bf16x2 v = {fa[e][i][2 * j], fa[e][i][2 * j + 1]};
                        s = __builtin_amdgcn_fdot2_f32_bf16(v, one, s, false);
                    }
                    bias[i] += s;
                }
            }
        }
    };

    // Step s multiplies rows m_begin + 32 s onwards.  Before its barrier a wave dequantises its share of step s+2 of the checkpoint.
    // Behind it every wave has the last fragments of step s in registers and its share of step s+1 in the LDS: then step s+2 of X is
    // put there, step s+6 of the checkpoint and step s+4 of dy are sent for.
    // At the barrier the newest 8 requests may be under way: two steps of 4.
    const int64_t whole_end = !w.last || (a.K % 16 == 0 && a.N % 8 == 0) ? m_end : a.M - 1;
    const int64_t n_whole = (whole_end - m_begin) / kRows;
    auto step = [&](int64_t s, int dy_slot, int dy_next, int x_slot, int q_slot, auto steady, auto sums) __attribute__((always_inline)) {
        read(1, dy_slot, x_slot);
        const Sixteen w = held(q_slot);
        multiply(0, sums);
        // (a matrix instruction, two LDS reads, six others, and so on)
#pragma unroll
        for (int k = 0; k < kNB * kKB; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(steady)::value) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        read(0, dy_next, x_slot ^ 1);
        put(w, x_slot);
        if (decltype(steady)::value || s + 4 < n_whole) bring_dy(m_begin + (s + 4) * kRows, dy_slot);
        if (decltype(steady)::value || s + 6 < n_whole) bring_x(m_begin + (s + 6) * kRows, q_slot);
        multiply(1, sums);
#pragma unroll
        for (int k = 0; k < kNB * kKB; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto steps = [&](auto sums) __attribute__((always_inline)) {
        int64_t s = 0;
        for (; s + 10 <= n_whole; s += 4) {
            step(s, 0, 1, 0, 2, std::true_type{}, sums);
            step(s + 1, 1, 2, 1, 3, std::true_type{}, sums);
            step(s + 2, 2, 3, 0, 0, std::true_type{}, sums);
            step(s + 3, 3, 0, 1, 1, std::true_type{}, sums);
        }
        for (; s < n_whole; s += 4) {
            step(s, 0, 1, 0, 2, std::false_type{}, sums);
            if (s + 1 < n_whole) step(s + 1, 1, 2, 1, 3, std::false_type{}, sums);
            if (s + 2 < n_whole) step(s + 2, 2, 3, 0, 0, std::false_type{}, sums);
            if (s + 3 < n_whole) step(s + 3, 3, 0, 1, 1, std::false_type{}, sums);
        }
    };
    auto all = [&](auto sums) __attribute__((always_inline)) {
        if (n_whole > 0) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s < n_whole) {
                    bring_dy(m_begin + s * kRows, s);
                    bring_x(m_begin + s * kRows, s);
                }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s < n_whole) {
                    put(held(s), s);
                    if (s + 4 < n_whole) bring_x(m_begin + (s + 4) * kRows, s);
                }
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            read(0, 0, 0);
            steps(sums);
        }
        // what is left, less than a step or the matrix's last row, by way of registers
        const int64_t m = m_begin + n_whole * kRows;
        if (m < m_end) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = kOwn * wave + kDyRows * j;
                u32x4 v = {0, 0, 0, 0};
                if (m + row + lane / (64 / kDyRows) < m_end)
                    v = shift_out(*(global_16)((global_bytes)(static_cast<const char *>(a.dy.p) + m * a.dy.ld * 2) + dy_off[j] - 2 * dy_over[j]), 2 * dy_over[j]);
                *reinterpret_cast<u32x4 *>(lds + kDy + row * kRowN + lane * 16) = v;
            }
            u32x4 v = {0, 0, 0, 0};
            uint32_t c = 0;
            if (m + x_row < m_end) {
                const int over = k0 + x_col < a.K && k0 + x_col + 16 > a.K ? k0 + x_col + 16 - a.K : 0;
                v = shift_out(*(global_16)((global_bytes)(a.c.q + m * a.c.ld_q) + x_off - over), over);
                c = a.c.scale[m * a.c.ld_scale + s_off];
            }
            put(dequantised(v, c), 0);
            __syncthreads();
            read(0, 0, 0);
            read(1, 0, 0);
            multiply(0, sums);
            multiply(1, sums);
        }
    };
    if (use_bias) all(std::true_type{});
    else all(std::false_type{});
    __syncthreads();
    finish<bf16_t, G>(g, w, acc, bias, use_bias, reinterpret_cast<float *>(lds));
}

// split > 1: the partial sums added up in a fixed order, with the norm's parameters, rounded once.  Four lanes' registers of
// the same number are four columns of a row; kStrands threads take every kStrands-th part of such a four and of the row's sum of dy.
// Bound by the parts' bytes, which the main kernel has just left in the cache: 7 parts of 3072 x 768, 12 us (66 MB, 5.5 TB/s).
template <typename T, typename G, int kStrands>
__global__ __launch_bounds__(256) void linear_join_kernel(GradArgs g) {
    constexpr int kElements = G::kN * G::kK, kQuads = kElements / 4, kOwn = 256 / kStrands;   // fours of a workgroup
    __shared__ f32x4 strand_v[kStrands > 1 ? 256 : 1];
    __shared__ float strand_b[kStrands > 1 ? 256 : 1];
    const LinearArgs &a = g.a;
    const int tid = threadIdx.x, strand = tid / kOwn;
    const int tile = blockIdx.x / (kQuads / kOwn), quad = blockIdx.x % (kQuads / kOwn) * kOwn + tid % kOwn;
    const int lane = quad % 16 * 4, r = quad / 16 % 16, block = quad / 256 % (G::kNB * G::kKB), wave = quad / (256 * G::kNB * G::kKB);
    const int n = tile / g.tiles_k * G::kN + G::row(wave, lane, block / G::kKB, r);
    const int k = tile % g.tiles_k * G::kK + G::column(wave, lane, block % G::kKB);
    const bool there = n < a.N && k < a.K, want_sum = there && (a.gamma || (a.dbias && k == 0));
    const float *from = g.part + static_cast<int64_t>(tile) * g.split * kElements + quad * 4;
    const float *sums = g.part + static_cast<int64_t>(g.tiles_n) * g.tiles_k * g.split * kElements + n;
    f32x4 v = {0, 0, 0, 0};
    float b = 0.0f;
    if (there) {
        for (int s0 = strand; s0 < g.split; s0 += 8 * kStrands) {        // (eight loads under way)
            f32x4 part[8];
            float sum[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int64_t s = s0 + u * kStrands < g.split ? s0 + u * kStrands : s0;
                part[u] = *reinterpret_cast<const f32x4 *>(from + s * kElements);
                sum[u] = want_sum ? sums[s * a.N] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (s0 + u * kStrands < g.split) {
                    v += part[u];
                    b += sum[u];
                }
        }
    }
    if constexpr (kStrands > 1) {
        strand_v[tid] = v;
        strand_b[tid] = b;
        __syncthreads();
        if (strand > 0) return;
#pragma unroll
        for (int y = 1; y < kStrands; ++y) {
            v += strand_v[y * kOwn + tid];
            b += strand_b[y * kOwn + tid];
        }
    }
    if (!there) return;
    if (a.dbias && k == 0) put_as<T>(a.dw_type, a.dbias, n, b);
    if (a.gamma) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + j < a.K) v[j] = __builtin_fmaf(v[j], get_as<T>(a.param_type, a.gamma, k + j), get_as<T>(a.param_type, a.beta, k + j) * b);
    }
    const int64_t at = static_cast<int64_t>(n) * a.dw.ld + k;
    if (a.dw_type == TENSILE_F32 && k + 4 <= a.K) {
        __builtin_memcpy(static_cast<float *>(a.dw.p) + at, &v, sizeof v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + j < a.K) put_as<T>(a.dw_type, a.dw.p, at + j, v[j]);
    }
}

template <typename T, typename G, bool kByElement>
int run(const ::tensile_ops *ops, hipStream_t s, const LinearArgs &a) {
    GradArgs g{};
    g.a = a;
    g.tiles_n = (a.N + G::kN - 1) / G::kN;
    g.tiles_k = (a.K + G::kK - 1) / G::kK;
    const int64_t tiles = static_cast<int64_t>(g.tiles_n) * g.tiles_k;
    // (2^32 threads to a launch)
    if (tiles > UINT32_MAX / G::kThreads) { set_error("linear_grad: dw has more than 2^32 / %d tiles of %d x %d", G::kThreads, G::kN, G::kK); return TENSILE_E_RANGE; }
    // The rows are split where there are fewer tiles than places, but not below kPartRows each.  (8192 x 3072 x 768, 36 tiles: 4 parts
    // are no faster than 7: less to join, but 112 CUs idle.)
    const int64_t slots = G::kPerCu * static_cast<int64_t>(ops->num_cus);
    int64_t split = slots / tiles;
    if (split > a.M / kPartRows) split = a.M / kPartRows;
    if (split < 1) split = 1;
    g.rows_per_split = ((a.M + split - 1) / split + kRows - 1) / kRows * kRows;
    split = g.rows_per_split ? (a.M + g.rows_per_split - 1) / g.rows_per_split : 1;
    g.split = static_cast<int32_t>(split);
    std::unique_lock<std::mutex> lock;
    if (split > 1) {
        OpsScratch &scratch = ops_scratch(ops, s);
        lock = std::unique_lock<std::mutex>(scratch.mu);
        const size_t need = static_cast<size_t>(split) * (static_cast<size_t>(tiles) * G::kN * G::kK + a.N);
        const int rc = scratch.provide(need, "linear_grad: partial sums");
        if (rc != TENSILE_OK) return rc;
        g.part = scratch.buf.p;
    }
    const dim3 grid(static_cast<uint32_t>(tiles * split));
    if constexpr (G::kByHalves) hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_grad_stream_kernel<G>), grid, dim3(G::kThreads), 0, s, g);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_grad_kernel<T, G, kByElement>), grid, dim3(G::kThreads), 0, s, g);
    TS_HIP(hipGetLastError());
    if (split > 1) {
        // (more than 8 parts: eight threads to a four; 16384 x 256 x 256, 64 parts, 19.6 against 23.3 us)
        const uint32_t blocks = static_cast<uint32_t>(tiles * (G::kN * G::kK / 1024));
        if (split <= 8) hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_join_kernel<T, G, 1>), dim3(blocks), dim3(256), 0, s, g);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_join_kernel<T, G, 8>), dim3(blocks * 8), dim3(256), 0, s, g);
        TS_HIP(hipGetLastError());
    }
    return TENSILE_OK;
}

template <typename T>
int choose(const ::tensile_ops *ops, hipStream_t s, const LinearArgs &a) {
    // A load takes 8 columns of dy, 16 of the checkpoint, and reaches them and the scales by 32 bits from the first of a step's 32 rows.
    constexpr int64_t kFar = 1 << 26;
    const bool by_element = a.N < 8 || a.K < 16 || a.dy.ld * static_cast<int64_t>(sizeof(T)) >= kFar || a.c.ld_q >= kFar || a.c.ld_scale >= kFar;
    if (by_element) return run<T, Staged, true>(ops, s, a);
    if constexpr (std::is_same<T, bf16_t>::value) {
        const int64_t wide = static_cast<int64_t>((a.N + Wide::kN - 1) / Wide::kN) * ((a.K + Wide::kK - 1) / Wide::kK);
        const int64_t area = static_cast<int64_t>(a.N) * a.K, padded = wide * Wide::kN * Wide::kK;
        // Large tiles read the LDS half as often for a product; small ones fill the card with fewer parts to join, and the
        // edges of dw with less that is not there.  Wide against Narrow (us): 16384 x 8192 x 8192 1793 and 2491; 2048 x 4096 x 4096 78
        // and 98; 8192 x 3072 x 768 (36 tiles) 62 and 69; 8192 x 768 x 768 (9) 34 and 28; 1000 x 1024 x 1024 (16) 25 and 18;
        // 16384 x 128 x 4096 (16, half of it padding) 53 and 37; 6000 x 300 x 300 (4) 24 and 16.
        if (wide >= 32 && padded <= area + area / 2) return run<T, Wide, false>(ops, s, a);
        return run<T, Narrow, false>(ops, s, a);
    } else {
        // The wider tile takes dy apart once for 256 columns; the other has more workgroups where not even half the CUs get one.
        // StagedWide against Staged (us, f32 and f16): 6000 x 8192 x 8192 2140 and 2545, 1604 and 1718; 8192 x 768 x 768 (18 tiles in
        // 32 parts at most) 46 and 52, 37 and 42; 600 x 3072 x 768 (72 in 2) 32 and 35; 1000 x 1024 x 1024 (32 in 3) 28.9 and 27.9;
        // 6000 x 300 x 300 (2.2 times its size in tiles) 26.3 and 25.5.
        const int64_t wide = static_cast<int64_t>((a.N + StagedWide::kN - 1) / StagedWide::kN) * ((a.K + StagedWide::kK - 1) / StagedWide::kK);
        const int64_t area = static_cast<int64_t>(a.N) * a.K, padded = wide * StagedWide::kN * StagedWide::kK;
        const int64_t parts = a.M < 2 * kPartRows ? 1 : a.M / kPartRows;
        if (2 * wide * parts >= ops->num_cus && padded <= area + area / 2) return run<T, StagedWide, false>(ops, s, a);
        return run<T, Staged, false>(ops, s, a);
    }
}

}  // namespace

int launch_linear_grad(const ::tensile_ops *ops, hipStream_t s, const LinearArgs &a, int type) {
    if (type == TENSILE_F32) return choose<float>(ops, s, a);
    if (type == TENSILE_BF16) return choose<bf16_t>(ops, s, a);
    return choose<f16_t>(ops, s, a);
}

}  // namespace tensile
