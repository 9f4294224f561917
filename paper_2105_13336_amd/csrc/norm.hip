// Layer norm, forward and backward, with the normalised row kept in 8 bits.
//
// Bound by HBM: forward reads 2 and writes 3.03 bytes an element (bf16, with a checkpoint), backward reads 3.03 and writes 2; a residual
// is 2 more.  Calls with a residual and a checkpoint: forward 16384 x 8192 183 us (5.2 TB/s), 65536 x 768 70 us (5.1), 8192 x 768
// 11 us (4.4; two rows to a wavefront, so that starting and ending count); backward without one 16384 x 8192 143 us (4.7), 65536 x 768
// 57 us (4.4), with one 16381 x 8192 169 + 5 us (5.6 TB/s), 8192 x 768 11 + 4 us, the second the sums over the workgroups.
// A row is held in the registers of its team (16 lanes, a wavefront, or a workgroup) from the one load to the stores: the
// mean, then the centred squares (no cancellation), then the outputs.  A team goes from row to row with the parameters in
// registers and the next row's loads under way.  Backward keeps the two parameter gradients of its columns
// in registers over all its rows; workgroups leave partial sums, which a second kernel adds up in a fixed order.
#include "ops_device.h"

#include <type_traits>

namespace tensile {

namespace {

// (a row's address plus 32 bits: the first is scalar where the row is)
template <typename T>
__device__ __forceinline__ T *at(const Matrix &m, int64_t row, int col) {
    return static_cast<T *>(m.p) + row * m.ld + static_cast<uint32_t>(col);
}

// kEven: rows of a multiple of 8 columns, so that a chunk is there or not, and nothing is asked about its parts.  (The tests for those
// more than double the instructions of a row: 65536 x 768, bf16, backward 68 -> 55 us.)
template <bool kEven, typename T>
__device__ __forceinline__ Raw8<T> get(const T *p, int left) {
    Raw8<T> r;
    if constexpr (kEven) __builtin_memcpy(&r, p, sizeof r);
    else r = load_raw(p, left);
    return r;
}
template <bool kEven, typename T>
__device__ __forceinline__ void put(T *p, const float (&f)[8], int left) {
    store8(p, f, kEven ? kChunk : left);
}
template <bool kEven>
__device__ __forceinline__ void put_packed(const Ckpt &c, int64_t row, uint32_t col, int left, const float (&f)[8], uint32_t cap) {
    uint32_t code;
    const u32x2 w = pack8(f, cap, code);
    if (left > 0) store_q(c.q + row * c.ld_q + col, w, kEven ? kChunk : left);
    if (left > 0 && col % kGroup == 0) (c.scale + row * c.ld_scale)[col / kGroup] = static_cast<uint8_t>(code);
}

// Sum over the lanes of a team, the same value in each of them.  kWaves > 1: `slot` is one of the team's LDS rows,
// which no wave still reads (see the callers).
template <int kLanes, int kWaves>
__device__ __forceinline__ float team_sum(float x, float *slot) {
    if constexpr (kLanes == 16) {
        return sum16(x);
    } else if constexpr (kWaves == 1) {
        return sum64(x);
    } else {
        const float s = sum64(x);
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = s;
        __syncthreads();
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) t += slot[w];
        return t;
    }
}

// A workgroup's teams, kLanes lanes of a wavefront or kWaves wavefronts each.  Of a row chunk n of a thread covers columns
// (n * kThreads + its number in the team) * 8 onwards.
template <int kLanes, int kWaves>
struct Team {
    static constexpr int kThreads = kLanes * kWaves;                    // of a team
    static constexpr int kBlock = kWaves == 1 ? 512 : kThreads;
    static constexpr int kTeams = kBlock / kThreads;                    // of a workgroup
    // the first row of the thread's team: the same for a wavefront's lanes, and the compiler knows, unless it has four teams
    static __device__ __forceinline__ int64_t first_row() {
        const int team = threadIdx.x / kThreads;
        return static_cast<int64_t>(blockIdx.x) * kTeams + (kLanes == 64 ? __builtin_amdgcn_readfirstlane(team) : team);
    }
};

// Forward with rows of at most kThreads * 8 * kChunks columns.
template <typename T, typename P, int kLanes, int kWaves, int kChunks, bool kEven>
__global__ __launch_bounds__((Team<kLanes, kWaves>::kBlock), 4) void norm_kernel(NormArgs a) {
    using G = Team<kLanes, kWaves>;
    __shared__ float sums[2][kWaves];
    const int lane = threadIdx.x % G::kThreads;
    const int64_t teams = static_cast<int64_t>(gridDim.x) * G::kTeams;
    int64_t row = G::first_row();
    if (row >= a.rows) return;
    uint32_t col[kChunks];
    int left[kChunks];
    float gamma[kChunks][8], beta[kChunks][8];
    Raw8<T> x[kChunks], r[kChunks];
#pragma unroll
    for (int n = 0; n < kChunks; ++n) {
        col[n] = (n * G::kThreads + lane) * kChunk;
        left[n] = a.cols - static_cast<int>(col[n]);
        x[n] = r[n] = Raw8<T>{};           // (and so it stays where there is no such column)
#pragma unroll
        for (int j = 0; j < 8; ++j) gamma[n][j] = beta[n][j] = 0.0f;
    }
    const float n_cols = static_cast<float>(a.cols);
    auto request = [&](int64_t at_row) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kChunks; ++n)
            if (left[n] > 0) {
                x[n] = get<kEven>(at<const T>(a.x, at_row, col[n]), left[n]);
                if (a.r.p) r[n] = get<kEven>(at<const T>(a.r, at_row, col[n]), left[n]);
            }
    };
    request(row);
#pragma unroll
    for (int n = 0; n < kChunks; ++n)
        if (left[n] > 0) {
            widen(get<kEven>(static_cast<const P *>(a.gamma) + col[n], left[n]), gamma[n]);
            widen(get<kEven>(static_cast<const P *>(a.beta) + col[n], left[n]), beta[n]);
        }
    for (; row < a.rows; row += teams) {
        float v[kChunks][8];
        float s = 0.0f;
#pragma unroll
        for (int n = 0; n < kChunks; ++n) {
            widen(x[n], v[n]);
            if (a.r.p) {
                float w[8];
                widen(r[n], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[n][j] += w[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[n][j];
        }
        if (row + teams < a.rows) request(row + teams);
        if (a.t.p) {
#pragma unroll
            for (int n = 0; n < kChunks; ++n)
                if (left[n] > 0) put<kEven>(at<T>(a.t, row, col[n]), v[n], left[n]);
        }
        // (divided, not multiplied by 1/cols: the mean of a constant row whose sum is exact is that constant.
        // The two rows of `sums` are written in turn, with a barrier between a row's reading and its next writing)
        const float mean = team_sum<kLanes, kWaves>(s, sums[0]) / n_cols;
        s = 0.0f;
#pragma unroll
        for (int n = 0; n < kChunks; ++n) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[n][j] = (kEven ? left[n] > 0 : j < left[n]) ? v[n][j] - mean : 0.0f;
                s += v[n][j] * v[n][j];
            }
        }
        const float var = team_sum<kLanes, kWaves>(s, sums[1]) / n_cols;
        const float rstd = 1.0f / __builtin_sqrtf(var + a.eps);
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int n = 0; n < kChunks; ++n) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[n][j] *= rstd;
                y[j] = __builtin_fmaf(v[n][j], gamma[n][j], beta[n][j]);
            }
            if (left[n] > 0) put<kEven>(at<T>(a.y, row, col[n]), y, left[n]);
            if (a.c.q) {
#pragma unroll
                for (int j = 0; j < 8; ++j)                             // (0 * inf: a missing column would be NaN)
                    if (kEven ? left[n] <= 0 : j >= left[n]) v[n][j] = 0.0f;
                put_packed<kEven>(a.c, row, col[n], left[n], v[n], static_cast<uint32_t>(a.cap));
            }
        }
    }
}

// Forward with rows too long for the registers (more than 16384 columns): a workgroup of 1024 threads passes over each row three times,
// two of them from the caches (4096 x 20480 bf16, residual, checkpoint: 391 MB read from memory of 336 there, 194 us, 3.0 TB/s of what has to
// move; three quarters of the wavefronts' time is waiting, for one pass's loads after the other).  4096 x 16384 in this form 140 us.
template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
    __shared__ float sums[2][16];
    const float n_cols = static_cast<float>(a.cols);
    const int last = (a.cols + kGroup - 1) / kGroup * kGroup;            // a group's four lanes stay together
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        auto read = [&](int c, float (&v)[8]) {
            const int left = a.cols - c;
            if (left <= 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = 0.0f;
                return;
            }
            load8(at<const T>(a.x, row, c), left, v);
            if (a.r.p) {
                float w[8];
                load8(at<const T>(a.r, row, c), left, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += w[j];
            }
        };
        float s = 0.0f, v[8];
        for (int c = threadIdx.x * kChunk; c < last; c += 1024 * kChunk) {
            read(c, v);
            float p = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) p += v[j];
            s += p;
        }
        const float mean = team_sum<64, 16>(s, sums[0]) / n_cols;
        s = 0.0f;
        for (int c = threadIdx.x * kChunk; c < last; c += 1024 * kChunk) {
            read(c, v);
            float p = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = c + j < a.cols ? v[j] - mean : 0.0f;
                p += d * d;
            }
            s += p;
        }
        const float var = team_sum<64, 16>(s, sums[1]) / n_cols;
        const float rstd = 1.0f / __builtin_sqrtf(var + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        for (int c = threadIdx.x * kChunk; c < last; c += 1024 * kChunk) {
            const int left = a.cols - c;
            read(c, v);
            if (a.t.p && left > 0) store8(at<T>(a.t, row, c), v, left);
            float g[8], b[8], y[8];
            if (left > 0) {
                load8(static_cast<const P *>(a.gamma) + c, left, g);
                load8(static_cast<const P *>(a.beta) + c, left, b);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = j < left ? (v[j] - mean) * rstd : 0.0f;
                y[j] = left > 0 ? __builtin_fmaf(v[j], g[j], b[j]) : 0.0f;
            }
            if (left > 0) store8(at<T>(a.y, row, c), y, left);
            if (a.c.q) {
                uint32_t code;
                const u32x2 w = pack8(v, static_cast<uint32_t>(a.cap), code);
                if (left > 0) store_q(a.c.q + row * a.c.ld_q + c, w, left);
                if (c % kGroup == 0) a.c.scale[row * a.c.ld_scale + c / kGroup] = static_cast<uint8_t>(code);
            }
        }
    }
}

// Backward with rows of at most kThreads * 8 * kChunks columns; a.part: [workgroup][2][cols] or null.  A workgroup of 512 threads (or
// 1024 where a row takes them) is one or more teams that go on together.
template <int kLanes, int kWaves>
struct BackTeam {
    static constexpr int kThreads = kLanes * kWaves, kBlock = kWaves > 8 ? kThreads : 512, kTeams = kBlock / kThreads;
};

template <typename T, typename P, int kLanes, int kWaves, int kChunks, bool kEven>
__global__ __launch_bounds__((BackTeam<kLanes, kWaves>::kBlock), 4) void norm_backward_kernel(NormArgs a) {
    using G = BackTeam<kLanes, kWaves>;
    static_assert(kChunks == 1 || G::kTeams == 1, "");
    constexpr int kSpan = G::kThreads * kChunk;                          // columns of a team (one chunk)
    __shared__ float sums[2][G::kTeams][2][kWaves];                      // [row's parity][team][sum]
    __shared__ float merge[G::kTeams > 1 ? G::kTeams * kSpan : 1];
    const int team = kLanes == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G::kThreads) : threadIdx.x / G::kThreads;
    const int lane = threadIdx.x % G::kThreads, wave = threadIdx.x / 64 % kWaves;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * G::kTeams;
    uint32_t col[kChunks];
    int left[kChunks];
    float gamma[kChunks][8] = {}, dgamma[kChunks][8] = {}, dbeta[kChunks][8] = {};
#pragma unroll
    for (int n = 0; n < kChunks; ++n) {
        col[n] = (n * G::kThreads + lane) * kChunk;
        left[n] = a.cols - static_cast<int>(col[n]);
    }
    const float inv = 1.0f / static_cast<float>(a.cols);
    // A row as it lies in memory: 28 bytes a chunk (bf16) where its numbers would take 64.  What is not there stays zero.
    struct Row {
        Raw8<T> x[kChunks], r[kChunks];
        u32x2 q[kChunks];
        uint32_t code[kChunks];
        float rstd;
    };
    auto request = [&](Row &w, int64_t row) __attribute__((always_inline)) {
        if (row < a.rows) {
#pragma unroll
            for (int n = 0; n < kChunks; ++n)
                if (left[n] > 0) {
                    w.x[n] = get<kEven>(at<const T>(a.x, row, col[n]), left[n]);
                    w.q[n] = load_q(a.c.q + row * a.c.ld_q + col[n], kEven ? kChunk : left[n]);
                    w.code[n] = (a.c.scale + row * a.c.ld_scale)[col[n] / kGroup];
                    if (a.r.p) w.r[n] = get<kEven>(at<const T>(a.r, row, col[n]), left[n]);
                }
            w.rstd = a.rstd[row];
        }
    };
    // (two chunks leave no registers for the next row)
    constexpr bool kAhead = kChunks == 1;
    Row now{}, next{};
    int64_t first = static_cast<int64_t>(blockIdx.x) * G::kTeams;
    if constexpr (kAhead) request(now, first + team);
#pragma unroll
    for (int n = 0; n < kChunks; ++n)
        if (left[n] > 0) widen(get<kEven>(static_cast<const P *>(a.gamma) + col[n], left[n]), gamma[n]);
    int parity = 0;
    for (; first < a.rows; first += stride) {
        const int64_t row = first + team;
        if constexpr (kAhead) request(next, row + stride);
        else request(now, row);
        float s1 = 0.0f, s2 = 0.0f, dy[kChunks][8], xh[kChunks][8];
#pragma unroll
        for (int n = 0; n < kChunks; ++n) {
            widen(now.x[n], dy[n]);
            unpack8(now.q[n], scale_of(now.code[n]), xh[n]);
            if constexpr (!kEven) {
                if (left[n] < kChunk) {                                  // (a NaN group's missing columns belong to no sum)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j >= left[n]) xh[n][j] = 0.0f;
                }
            }
            if (row < a.rows) {                                          // (a team without a row holds an older one)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dgamma[n][j] = __builtin_fmaf(dy[n][j], xh[n][j], dgamma[n][j]);
                    dbeta[n][j] += dy[n][j];
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dy[n][j] *= gamma[n][j];
                s1 += dy[n][j];
                s2 = __builtin_fmaf(dy[n][j], xh[n][j], s2);
            }
        }
        // (one barrier a row: a row's two sums are read before the next row's barrier, and written again behind that)
        float c1, c2;
        if constexpr (kWaves == 1) {
            c1 = team_sum<kLanes, 1>(s1, nullptr) * inv;
            c2 = team_sum<kLanes, 1>(s2, nullptr) * inv;
        } else {
            s1 = sum64(s1);
            s2 = sum64(s2);
            if ((threadIdx.x & 63) == 0) {
                sums[parity][team][0][wave] = s1;
                sums[parity][team][1][wave] = s2;
            }
            __syncthreads();
            c1 = c2 = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                c1 += sums[parity][team][0][w];
                c2 += sums[parity][team][1][w];
            }
            c1 *= inv;
            c2 *= inv;
            parity ^= 1;
        }
        if (row < a.rows) {
#pragma unroll
            for (int n = 0; n < kChunks; ++n) {
                if (left[n] <= 0) continue;
                float d[8];
                if (a.r.p) {
                    widen(now.r[n], d);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = __builtin_fmaf(now.rstd, dy[n][j] - c1 - xh[n][j] * c2, d[j]);
                put<kEven>(at<T>(a.y, row, col[n]), d, left[n]);
            }
        }
        if constexpr (kAhead) now = next;
    }
    if (!a.part) return;
    float *part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
    if constexpr (G::kTeams == 1) {
#pragma unroll
        for (int n = 0; n < kChunks; ++n)
            if (left[n] > 0) {
                store8(part + col[n], dgamma[n], left[n]);
                store8(part + a.cols + col[n], dbeta[n], left[n]);
            }
    } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half) __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) merge[team * kSpan + col[0] + j] = half ? dbeta[0][j] : dgamma[0][j];
            __syncthreads();
            for (int c = threadIdx.x; c < kSpan && c < a.cols; c += G::kBlock) {
                float s = 0.0f;
#pragma unroll
                for (int t = 0; t < G::kTeams; ++t) s += merge[t * kSpan + c];
                part[half * static_cast<int64_t>(a.cols) + c] = s;
            }
        }
    }
}

// Backward with rows too long for the registers, part one: dx.  4096 x 16384 f32 80 us the parameters' sums, 150 dx, 12 the join (604 MB have to
// move: 123 us at the rate of a copy); bf16 4096 x 20480 70, 107 and 14.
template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_backward_long_kernel(NormArgs a) {
    __shared__ float sums[2][16];
    const float inv = 1.0f / static_cast<float>(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        auto read = [&](int c, float (&h)[8], float (&xh)[8]) {
            const int left = a.cols - c;
            float g[8];
            load8(at<const T>(a.x, row, c), left, h);
            load8(static_cast<const P *>(a.gamma) + c, left, g);
            unpack8(load_q(a.c.q + row * a.c.ld_q + c, left), scale_of(a.c.scale[row * a.c.ld_scale + c / kGroup]), xh);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[j] *= g[j];
                if (j >= left) xh[j] = 0.0f;
            }
        };
        float s1 = 0.0f, s2 = 0.0f, h[8], xh[8];
        for (int c = threadIdx.x * kChunk; c < a.cols; c += 1024 * kChunk) {
            read(c, h, xh);
            float p1 = 0.0f, p2 = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p1 += h[j];
                p2 = __builtin_fmaf(h[j], xh[j], p2);
            }
            s1 += p1;
            s2 += p2;
        }
        const float c1 = team_sum<64, 16>(s1, sums[0]) * inv;
        const float c2 = team_sum<64, 16>(s2, sums[1]) * inv;
        const float rstd = a.rstd[row];
        for (int c = threadIdx.x * kChunk; c < a.cols; c += 1024 * kChunk) {
            const int left = a.cols - c;
            read(c, h, xh);
            float d[8];
            if (a.r.p) load8(at<const T>(a.r, row, c), left, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = rstd * (h[j] - c1 - xh[j] * c2);
                d[j] = a.r.p ? d[j] + e : e;
            }
            store8(at<T>(a.y, row, c), d, left);
        }
    }
}

// ... part two, before dx may overwrite dy: partial sums of the parameter gradients, 2048 columns and every gridDim.y-th row
// to a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a) {
    const int c = (blockIdx.x * 256 + threadIdx.x) * kChunk, left = a.cols - c;
    if (left <= 0) return;
    float dgamma[8] = {}, dbeta[8] = {};
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float dy[8], xh[8];
        load8(at<const T>(a.x, row, c), left, dy);
        unpack8(load_q(a.c.q + row * a.c.ld_q + c, left), scale_of(a.c.scale[row * a.c.ld_scale + c / kGroup]), xh);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dgamma[j] = __builtin_fmaf(dy[j], xh[j], dgamma[j]);
            dbeta[j] += dy[j];
        }
    }
    float *part = a.part + static_cast<int64_t>(blockIdx.y) * 2 * a.cols;
    store8(part + c, dgamma, left);
    store8(part + a.cols + c, dbeta, left);
}

// dgamma, dbeta = the partial sums' columns added up: 32 columns and 32 strands to a workgroup, each strand every 32nd
// partial sum, then the strands in order.  Latency: 2.5 to 4 us for 768 columns and 512 partial sums, 5 us for 8192 and 256.
// first: of the 2 * cols columns that a launch takes (a launch has room for 2^32 threads, and wraps silently beyond).
constexpr int64_t kGradientBlocks = 1 << 20;
template <typename P>
__global__ __launch_bounds__(1024) void norm_gradients_kernel(const float *part, int32_t n_part, int32_t cols, P *dgamma, P *dbeta, int64_t first) {
    __shared__ float strand[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = first + static_cast<int64_t>(blockIdx.x) * 32 + x, width = 2 * static_cast<int64_t>(cols);
    float s = 0.0f;
    if (c < width) {
#pragma unroll 8
        for (int k = y; k < n_part; k += 32) s += part[k * width + c];
    }
    strand[y][x] = s;
    __syncthreads();
    if (y == 0 && c < width) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += strand[k][x];
        P out;
        from_f32(s, out);
        if (c < cols) dgamma[c] = out;
        else dbeta[c - cols] = out;
    }
}

// f(element, parameter, even)
template <typename F>
void by_types(int type, int param_type, bool even, F f) {
    auto with = [&](auto t, auto p) {
        if (even) f(t, p, std::true_type{});
        else f(t, p, std::false_type{});
    };
    if (type == TENSILE_F32) with(float{}, float{});
    else if (type == TENSILE_BF16 && param_type == TENSILE_F32) with(bf16_t{}, float{});
    else if (type == TENSILE_BF16) with(bf16_t{}, bf16_t{});
    else if (param_type == TENSILE_F32) with(f16_t{}, float{});
    else with(f16_t{}, f16_t{});
}

uint32_t grid_of(int64_t rows, int64_t teams, int64_t most) {
    const int64_t n = (rows + teams - 1) / teams;
    return static_cast<uint32_t>(n < most ? n : most);
}

}  // namespace

int launch_norm(const ::tensile_ops *ops, hipStream_t s, const NormArgs &a, int type, int param_type) {
    const int64_t cus = ops->num_cus;
    // The smallest team that holds the row: fewer barriers and sums, and no idle lanes.  Against the next larger one (us): 65536 x 128
    // 11.5 and 25.3; 8192 x 512 7.2 and 8.7; x 768 10.1 and 15.2; x 2048 24.5 and 25.6; x 8192 90 and 99; 4096 x 16384 89 and,
    // in three passes, 140.
    by_types(type, param_type, a.cols % kChunk == 0, [&](auto t, auto p, auto even) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr bool kEven = decltype(even)::value;
#define TS_NORM(lanes, waves, chunks, per_cu)                                                                              \
    do {                                                                                                                   \
        using G = Team<lanes, waves>;                                                                              \
        hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<T, P, lanes, waves, chunks, kEven>), dim3(grid_of(a.rows, G::kTeams, cus * per_cu)), \
                           dim3(G::kBlock), 0, s, a);                                                                      \
    } while (0)
        if (a.cols <= 128) TS_NORM(16, 1, 1, 4);
        else if (a.cols <= 512) TS_NORM(64, 1, 1, 4);
        else if (a.cols <= 1024) TS_NORM(64, 1, 2, 2);
        else if (a.cols <= 2048) TS_NORM(64, 4, 1, 8);
        else if (a.cols <= 4096) TS_NORM(64, 4, 2, 4);
        else if (a.cols <= 8192) TS_NORM(64, 8, 2, 2);
        else if (a.cols <= 16384) TS_NORM(64, 16, 2, 1);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_long_kernel<T, P>), dim3(grid_of(a.rows, 1, cus * 2)), dim3(1024), 0, s, a);
#undef TS_NORM
    });
    TS_HIP(hipGetLastError());
    return TENSILE_OK;
}

int launch_norm_backward(const ::tensile_ops *ops, hipStream_t s, const NormArgs &args, int type, int param_type, void *dgamma, void *dbeta) {
    const int64_t cus = ops->num_cus;
    NormArgs a = args;
    // workgroups: what is resident, two of 512 threads to a CU (partial sums take 8 bytes a column each)
    // Teams as above; against the next larger one (us): 65536 x 128 12.7 and 23.3; 8192 x 512 10.0 and 12.0; x 768 12.7 and 17.1; x 2048
    // 21.4 and 26.5; x 4096 41 and 55; 4096 x 16384 113 and, in two passes, 144.
    // (1024 threads have room for two chunks each of 16-bit gradients)
    const bool is_long = a.cols > (type == TENSILE_F32 ? 8192 : 16384);
    const int teams = a.cols <= 128 ? 32 : a.cols <= 512 ? 8 : a.cols <= 1024 ? 4 : a.cols <= 2048 ? 2 : 1, per_cu = a.cols <= 4096 ? 2 : 1;
    const int64_t n_columns = (static_cast<int64_t>(a.cols) + 2047) / 2048;      // (long rows)
    const uint32_t n_part = grid_of(a.rows, is_long ? 1 : teams, is_long ? (8 * cus + n_columns - 1) / n_columns : cus * per_cu);
    std::unique_lock<std::mutex> lock;
    if (dgamma) {
        OpsScratch &scratch = ops_scratch(ops, s);
        lock = std::unique_lock<std::mutex>(scratch.mu);
        const int rc = scratch.provide(static_cast<size_t>(n_part) * 2 * static_cast<size_t>(a.cols), "layer_norm_backward: partial sums");
        if (rc != TENSILE_OK) return rc;
        a.part = scratch.buf.p;
    }
    by_types(type, param_type, a.cols % kChunk == 0, [&](auto t, auto p, auto even) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr bool kEven = decltype(even)::value;
        if (a.rows > 0) {
#define TS_NORM(lanes, waves, chunks)                                                                                      \
    hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_backward_kernel<T, P, lanes, waves, chunks, kEven>), dim3(n_part),             \
                       dim3(BackTeam<lanes, waves>::kBlock), 0, s, a)
            if (a.cols <= 128) TS_NORM(16, 1, 1);
            else if (a.cols <= 512) TS_NORM(64, 1, 1);
            else if (a.cols <= 1024) TS_NORM(64, 2, 1);
            else if (a.cols <= 2048) TS_NORM(64, 4, 1);
            else if (a.cols <= 4096) TS_NORM(64, 8, 1);
            else if (a.cols <= 8192) TS_NORM(64, 16, 1);
            else if (!is_long) {
                if constexpr (sizeof(T) == 2) TS_NORM(64, 16, 2);
            }
            else {
                if (dgamma)
                    hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_columns_kernel<T>), dim3(static_cast<uint32_t>(n_columns), n_part), dim3(256), 0, s, a);
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_backward_long_kernel<T, P>), dim3(grid_of(a.rows, 1, cus * 2)), dim3(1024), 0, s, a);
            }
#undef TS_NORM
        }
        if (dgamma) {
            const int64_t blocks = (2 * static_cast<int64_t>(a.cols) + 31) / 32;
            for (int64_t first = 0; first < blocks; first += kGradientBlocks)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_gradients_kernel<P>), dim3(grid_of(blocks - first, 1, kGradientBlocks)), dim3(1024), 0, s,
                                   a.part, static_cast<int32_t>(n_part), a.cols, static_cast<P *>(dgamma), static_cast<P *>(dbeta), first * 32);
        }
    });
    TS_HIP(hipGetLastError());
    return TENSILE_OK;
}

}  // namespace tensile
