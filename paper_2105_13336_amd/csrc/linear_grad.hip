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

namespace tensile {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 128;            // columns of dy and of the checkpoint per workgroup
constexpr int kGradThreads = 256;     // four wavefronts, 64 x 64 of the tile each
constexpr int kRowBytes = kTile * 2;  // of a staged row

// How many bf16 numbers add up to an element of dy, and how many rows a step takes.
template <typename T> struct Pieces;
template <> struct Pieces<bf16_t> { static constexpr int n = 1, rows = 64; };
template <> struct Pieces<f16_t> { static constexpr int n = 2, rows = 32; };
template <> struct Pieces<float> { static constexpr int n = 3, rows = 32; };

struct GradArgs {
    LinearArgs a;
    int32_t tiles_n, tiles_k, split;
    int64_t rows_per_split;           // a multiple of 64
    float *part;                      // split > 1: [split][N][K] sums, then [split][N] sums of dy
};

// A staged row's 16-column blocks (32 bytes) are stored in an order that depends on the row: the 4 rows x 2 blocks
// that half a wavefront reads at a time lie in different banks.
__device__ __forceinline__ int swizzle(int row, int block) { return row * kRowBytes + ((block ^ (2 * (row & 3))) * 32); }

// x = p[0] + p[1] + ...: each piece the leading 8 bits of what is left (exact); infinities and NaN are all in the first.
template <int kPieces>
__device__ __forceinline__ void split_bf16(float x, uint32_t (&p)[kPieces]) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const uint32_t top = as_u32(x) & 0xffff0000u;
        p[k] = top;
        const float rest = x - as_f32(top);
        x = (top & 0x7f800000u) == 0x7f800000u ? 0.0f : rest;
    }
}

template <typename T>
__global__ __launch_bounds__(kGradThreads, 2) void linear_grad_kernel(GradArgs g) {
    constexpr int kP = Pieces<T>::n, kRows = Pieces<T>::rows;
    constexpr int kPlane = kRows * kRowBytes;                            // bytes of a staged plane
    constexpr int kBuffer = (kP + 1) * kPlane;
    constexpr int kDyLoads = kRows / 16, kXLoads = kRows / 32;           // per thread and step
    __shared__ __attribute__((aligned(16))) char lds[2 * kBuffer];
    const LinearArgs &a = g.a;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wave_n = wave >> 1, wave_k = wave & 1;
    const int64_t tile = blockIdx.x;
    const int split = static_cast<int>(tile / (g.tiles_n * g.tiles_k));
    const int in_split = static_cast<int>(tile % (g.tiles_n * g.tiles_k));
    const int n0 = in_split / g.tiles_k * kTile, k0 = in_split % g.tiles_k * kTile;
    const int64_t m_begin = split * g.rows_per_split;
    const int64_t m_end = m_begin + g.rows_per_split < a.M ? m_begin + g.rows_per_split : a.M;

    // staging: 16 threads to a row of dy (8 columns each), 8 threads to a row of the checkpoint (16 columns each)
    const int dy_row = tid >> 4, dy_col = (tid & 15) * 8;
    const int x_row = tid >> 3, x_col = (tid & 7) * 16;
    const int dy_left = a.N - n0 - dy_col, x_left = a.K - k0 - x_col;
    const T *dy = static_cast<const T *>(a.dy.p) + n0 + dy_col;
    const int8_t *xq = a.c.q + k0 + x_col;
    const uint8_t *xs = a.c.scale + (k0 + x_col) / kGroup;

    Raw8<T> dy_raw[kDyLoads];
    u32x2 x_raw[kXLoads][2];
    uint32_t x_code[kXLoads];
    auto request = [&](int64_t m) {
#pragma unroll
        for (int i = 0; i < kDyLoads; ++i) {
            const int64_t r = m + dy_row + 16 * i;
            dy_raw[i] = Raw8<T>{};
            if (r < m_end && dy_left > 0) dy_raw[i] = load_raw(dy + r * a.dy.ld, dy_left);
        }
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            const int64_t r = m + x_row + 32 * i;
            x_raw[i][0] = x_raw[i][1] = u32x2{0, 0};
            x_code[i] = 0;
            if (r < m_end && x_left > 0) {
                x_raw[i][0] = load_q(xq + r * a.c.ld_q, x_left);
                if (x_left > 8) x_raw[i][1] = load_q(xq + r * a.c.ld_q + 8, x_left - 8);
                x_code[i] = xs[r * a.c.ld_scale];
            }
        }
    };
    auto stage = [&](char *to) {
#pragma unroll
        for (int i = 0; i < kDyLoads; ++i) {
            const int r = dy_row + 16 * i;
            char *at = to + swizzle(r, dy_col / 16) + (dy_col % 16) * 2;
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
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            const int r = x_row + 32 * i;
            char *at = to + kP * kPlane + swizzle(r, x_col / 16);
            const float scale = scale_of(x_code[i]);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float f[8];
                unpack8(x_raw[i][half], scale, f);
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(as_u32(f[2 * j + 1]), as_u32(f[2 * j]), 0x07060302);
                *reinterpret_cast<u32x4 *>(at + half * 16) = w;
            }
        }
    };

    f32x16 acc[2][2] = {};
    float bias[2] = {0.0f, 0.0f};
    const bool want_bias = a.gamma || (k0 == 0 && a.dbias);
    // transposed reads: the lanes of a group of 16 read rows 8h .. 8h+3 (and +4) of 16 columns
    const int i16 = lane & 15, group = lane >> 4;
    const int t_row = (group >> 1) * 8 + i16 / 4, t_in = (i16 & 3) * 8;
    int a_at[2], b_at[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        a_at[b] = swizzle(t_row, wave_n * 4 + b * 2 + (group & 1)) + t_in;
        b_at[b] = kP * kPlane + swizzle(t_row, wave_k * 4 + b * 2 + (group & 1)) + t_in;
    }
    auto fragment = [&](const char *p) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * kRowBytes));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto multiply = [&](const char *from) {
        float step_bias[2] = {0.0f, 0.0f};
#pragma unroll
        for (int kk = 0; kk < kRows / 16; ++kk) {
            bf16x8 fb[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) fb[b] = fragment(from + b_at[b] + kk * 16 * kRowBytes);
#pragma unroll
            for (int p = 0; p < kP; ++p) {
                bf16x8 fa[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) fa[b] = fragment(from + p * kPlane + a_at[b] + kk * 16 * kRowBytes);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
                if (want_bias && (kk & 1) == wave_k) {                  // (the two waves of a row of the tile take turns)
                    const bf16x2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bf16x2 v = {fa[i][2 * j], fa[i][2 * j + 1]};
                            step_bias[i] = __builtin_amdgcn_fdot2_f32_bf16(v, one, step_bias[i], false);
                        }
                }
            }
        }
        bias[0] += step_bias[0];
        bias[1] += step_bias[1];
    };

    if (m_begin < m_end) {
        request(m_begin);
        stage(lds);
        __syncthreads();
        int cur = 0;
        for (int64_t m = m_begin; m < m_end; m += kRows) {
            const bool more = m + kRows < m_end;
            if (more) request(m + kRows);
            multiply(lds + cur * kBuffer);
            if (more) stage(lds + (cur ^ 1) * kBuffer);
            __syncthreads();
            cur ^= 1;
        }
    }

    // sums of dy: over the two halves of the wavefront, then over the two waves that took turns
    float *sums = reinterpret_cast<float *>(lds);                         // [2][128]
    if (want_bias) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float s = bias[i] + __shfl_xor(bias[i], 32);
            if (lane < 32) sums[wave_k * kTile + wave_n * 64 + i * 32 + lane] = s;
        }
        __syncthreads();
        if (tid < kTile) sums[tid] = sums[tid] + sums[kTile + tid];
        __syncthreads();
    }

    const int k_lane = k0 + wave_k * 64 + (lane & 31);
    const int n_lane = wave_n * 64 + 4 * (lane >> 5);
    if (g.split > 1) {
        float *out = g.part + static_cast<int64_t>(split) * a.N * a.K;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int n = n0 + n_lane + i * 32 + 8 * (r / 4) + r % 4, k = k_lane + j * 32;
                    if (n < a.N && k < a.K) out[static_cast<int64_t>(n) * a.K + k] = acc[i][j][r];
                }
        if (k0 == 0 && want_bias && tid < kTile && n0 + tid < a.N)
            g.part[static_cast<int64_t>(g.split) * a.N * a.K + static_cast<int64_t>(split) * a.N + n0 + tid] = sums[tid];
        return;
    }
    auto put = [&](void *p, int64_t at, float v) {
        if (a.dw_type == TENSILE_F32) static_cast<float *>(p)[at] = v;
        else from_f32(v, static_cast<T *>(p)[at]);
    };
    auto param = [&](const void *p, int k) {
        return a.param_type == TENSILE_F32 ? static_cast<const float *>(p)[k] : to_f32(static_cast<const T *>(p)[k]);
    };
    if (k0 == 0 && a.dbias && tid < kTile && n0 + tid < a.N) put(a.dbias, n0 + tid, sums[tid]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int k = k_lane + j * 32;
        if (k >= a.K) continue;
        const float ga = a.gamma ? param(a.gamma, k) : 1.0f, be = a.gamma ? param(a.beta, k) : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int in_tile = n_lane + i * 32 + 8 * (r / 4) + r % 4, n = n0 + in_tile;
                if (n >= a.N) continue;
                float v = acc[i][j][r];
                if (a.gamma) v = __builtin_fmaf(v, ga, be * sums[in_tile]);
                put(a.dw.p, static_cast<int64_t>(n) * a.dw.ld + k, v);
            }
    }
}

// split > 1: the partial sums added up in order, with the norm's parameters, rounded once.
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(GradArgs g) {
    const LinearArgs &a = g.a;
    const int64_t plane = static_cast<int64_t>(a.N) * a.K;
    const float *sums = g.part + g.split * plane;
    auto put = [&](void *p, int64_t at, float v) {
        if (a.dw_type == TENSILE_F32) static_cast<float *>(p)[at] = v;
        else from_f32(v, static_cast<T *>(p)[at]);
    };
    auto param = [&](const void *p, int k) {
        return a.param_type == TENSILE_F32 ? static_cast<const float *>(p)[k] : to_f32(static_cast<const T *>(p)[k]);
    };
    const int k = blockIdx.x * 256 + threadIdx.x;
    for (int n = blockIdx.y; n < a.N; n += gridDim.y) {
        float b = 0.0f;
        if (a.gamma || (a.dbias && k == 0))
            for (int s = 0; s < g.split; ++s) b += sums[static_cast<int64_t>(s) * a.N + n];
        if (a.dbias && k == 0) put(a.dbias, n, b);
        if (k < a.K) {
            float v = 0.0f;
            for (int s = 0; s < g.split; ++s) v += g.part[s * plane + static_cast<int64_t>(n) * a.K + k];
            if (a.gamma) v = __builtin_fmaf(v, param(a.gamma, k), param(a.beta, k) * b);
            put(a.dw.p, static_cast<int64_t>(n) * a.dw.ld + k, v);
        }
    }
}

template <typename T>
int run(const ::tensile_ops *ops, hipStream_t s, const LinearArgs &a) {
    GradArgs g{};
    g.a = a;
    g.tiles_n = (a.N + kTile - 1) / kTile;
    g.tiles_k = (a.K + kTile - 1) / kTile;
    const int64_t tiles = static_cast<int64_t>(g.tiles_n) * g.tiles_k;
    if (tiles > INT32_MAX) { set_error("linear_grad: more than 2^31 tiles of 128 x 128"); return TENSILE_E_RANGE; }
    // two workgroups to a CU; the rows are split where there are too few tiles, but not below 256 rows each
    const int64_t slots = 2 * static_cast<int64_t>(ops->num_cus);
    int64_t split = slots / tiles;
    if (split > a.M / 256) split = a.M / 256;
    if (split < 1) split = 1;
    g.rows_per_split = ((a.M + split - 1) / split + 63) / 64 * 64;
    split = g.rows_per_split ? (a.M + g.rows_per_split - 1) / g.rows_per_split : 1;
    if (split < 1) split = 1;
    g.split = static_cast<int32_t>(split);
    std::unique_lock<std::mutex> lock;
    if (split > 1) {
        OpsScratch &scratch = ops_scratch(ops, s);
        lock = std::unique_lock<std::mutex>(scratch.mu);
        const size_t need = static_cast<size_t>(split) * a.N * (static_cast<size_t>(a.K) + 1);
        const int rc = scratch.provide(need, "linear_grad: partial sums");
        if (rc != TENSILE_OK) return rc;
        g.part = scratch.buf.p;
    }
    hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_grad_kernel<T>), dim3(static_cast<uint32_t>(tiles * split)), dim3(kGradThreads), 0, s, g);
    TS_HIP(hipGetLastError());
    if (split > 1) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_join_kernel<T>), dim3((a.K + 255) / 256, a.N < 4096 ? a.N : 4096), dim3(256), 0, s, g);
        TS_HIP(hipGetLastError());
    }
    return TENSILE_OK;
}

}  // namespace

int launch_linear_grad(const ::tensile_ops *ops, hipStream_t s, const LinearArgs &a, int type) {
    if (type == TENSILE_F32) return run<float>(ops, s, a);
    if (type == TENSILE_BF16) return run<bf16_t>(ops, s, a);
    return run<f16_t>(ops, s, a);
}

}  // namespace tensile
