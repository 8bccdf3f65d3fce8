// norm.hip -- layer norm over rows of C values and its backward, for gfx950 (MI355X): what a branch
// has in front of it, between the streams' read and its own products.
//
//     mu = mean x,   s = (mean (x - mu)^2 + eps)^(-1/2),   xh = (x - mu) s,   y = xh w + b
//     g = dy w,   dx = s (g - mean g - xh mean(g xh)),   dw = sum over rows of dy xh,   db = sum of dy
//
// Both passes are bound by HBM: a row is read once into registers (the backward: x and dy), summed over
// and written from there. G threads hold a row, sixteen values each (the backward: eight), and keep their columns' w and b
// (backward: w and the sums of dw and db) in registers over all rows that their group of threads takes.
// 32 K rows of 4096 bf16: forward 96 us, 5.6 TB/s; backward 150, 5.4 (6.1 at its fastest, where nothing is being
// written back from the call before).
// The variance is the mean of (x - mu)^2 with mu known, so a large common offset costs no digits, and sums
// are divided by C, not multiplied by its rounded reciprocal: equal values have no spread.

#include "common.h"

namespace {

typedef uint32_t v4u_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t v4u_at4 __attribute__((ext_vector_type(4), aligned(4)));

// A row of C values in 16-byte chunks; where C is no whole number of them (RAGGED), rows begin at any
// element and the last chunk holds `rem` values.
struct Row {
    int64_t C;
    int nc;   // chunks, the last one included
    int rem;  // values in the last chunk, 1..E
};

template <int DX, bool RAGGED>
__device__ __forceinline__ int chunk_values(const Row& r, int c) {
    constexpr int E = MixChunk<DX>::E;
    if (c >= r.nc) return 0;
    return RAGGED && c == r.nc - 1 ? r.rem : E;
}

// Chunk c as it is asked for: the last one of a ragged row as the sixteen bytes that end with the row, so that no
// load waits for another one (element by element, the wave that has it lost the row ahead: 32 K rows of 4095 bf16
// forward 170 us and now 117, backward 338 and 186; of 4096, 96 and 150). Rows of less than sixteen bytes come element by element.
template <int DX, bool RAGGED>
__device__ __forceinline__ v4u ask_chunk(const char* row, const Row& r, int c) {
    constexpr int E = MixChunk<DX>::E;
    const char* p = row + 16 * static_cast<int64_t>(c);
    if (c >= r.nc) return v4u{0, 0, 0, 0};
    if constexpr (!RAGGED) {
        return __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
    } else if (r.nc > 1) {
        if (c == r.nc - 1) p -= (E - r.rem) * (16 / E);
        if constexpr (DX == BIRKHOFF4_BF16)
            return *reinterpret_cast<const v4u_at2*>(p);
        else
            return *reinterpret_cast<const v4u_at4*>(p);
    } else {
        v4u v = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < E - 1; ++e) {
            if (e >= r.rem) continue;
            if constexpr (DX == BIRKHOFF4_BF16)
                v[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[e]) << (16 * (e & 1));
            else
                v[e] = reinterpret_cast<const uint32_t*>(p)[e];
        }
        return v;
    }
}

// Its values, zeros past the row's end.
template <int DX, bool RAGGED>
__device__ __forceinline__ v4u chunk_of(v4u v, const Row& r, int c) {
    constexpr int E = MixChunk<DX>::E;
    if (RAGGED && r.nc > 1 && c == r.nc - 1 && r.rem < E) {
        const uint64_t lo = v.x | static_cast<uint64_t>(v.y) << 32, hi = v.z | static_cast<uint64_t>(v.w) << 32;
        const int bits = (E - r.rem) * (128 / E);
        const uint64_t a = bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits), b = bits >= 64 ? 0 : hi >> bits;
        v = v4u{static_cast<uint32_t>(a), static_cast<uint32_t>(a >> 32), static_cast<uint32_t>(b), static_cast<uint32_t>(b >> 32)};
    }
    return v;
}

template <int DX, bool RAGGED>
__device__ __forceinline__ v4u load_chunk(const char* row, const Row& r, int c) {
    return chunk_of<DX, RAGGED>(ask_chunk<DX, RAGGED>(row, r, c), r, c);
}

template <int DX, bool RAGGED>
__device__ __forceinline__ void store_chunk(char* row, const Row& r, int c, const v4u v) {
    constexpr int E = MixChunk<DX>::E;
    char* p = row + 16 * static_cast<int64_t>(c);
    if constexpr (!RAGGED) {
        if (c < r.nc) __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(p));
    } else {
        const int n = chunk_values<DX, RAGGED>(r, c);
        if (n == E) {
            if constexpr (DX == BIRKHOFF4_BF16)
                *reinterpret_cast<v4u_at2*>(p) = v;
            else
                *reinterpret_cast<v4u_at4*>(p) = v;
        } else if (n > 0) {
#pragma unroll
            for (int e = 0; e < E - 1; ++e) {
                if (e >= n) continue;
                if constexpr (DX == BIRKHOFF4_BF16)
                    reinterpret_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(v[e / 2] >> (16 * (e & 1)));
                else
                    reinterpret_cast<uint32_t*>(p)[e] = v[e];
            }
        }
    }
}

// The E parameters of chunk c; `none` where there are none (and past the row's end, where it does not matter).
template <int DW, int E>
__device__ __forceinline__ void load_params(const void* w, const Row& r, int c, float none, float out[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = none;
    const int64_t at = static_cast<int64_t>(c) * E;
    if (!w || at >= r.C) return;
    if (at + E <= r.C) {
        if constexpr (DW == BIRKHOFF4_BF16) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(w) + at);
#pragma unroll
            for (int k = 0; k < E / 2; ++k) {
                out[2 * k] = __uint_as_float(p[k] << 16);
                out[2 * k + 1] = __uint_as_float(p[k] & 0xffff0000u);
            }
        } else {
            const v4f* p = reinterpret_cast<const v4f*>(static_cast<const float*>(w) + at);
#pragma unroll
            for (int k = 0; k < E / 4; ++k) {
                const v4f v = p[k];
#pragma unroll
                for (int e = 0; e < 4; ++e) out[4 * k + e] = v[e];
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (at + e >= r.C) continue;
        if constexpr (DW == BIRKHOFF4_BF16)
            out[e] = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(w)[at + e]) << 16);
        else
            out[e] = static_cast<const float*>(w)[at + e];
    }
}

// Sum over the lanes of a group of G <= 64 threads, the same in all of them.
template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma clang fp contract(off)
    x = gsum_lanes<8>(x);
    if constexpr (G >= 16) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xF, 0xF, true));  // row_ror:8
    if constexpr (G >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (G >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// Sums of N values over a group of G threads, the same in all of them. Groups of several waves add
// through `red`, in the order of the waves; the caller gives each sum of a row another part of it (and
// the next row's first sum comes after a barrier that all have passed), so one barrier a sum is enough.
template <int G, int NT, int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float (*red)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<(G < 64 ? G : 64)>(v[k]);
    if constexpr (G > 64) {
        const int wave = threadIdx.x / 64;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) red[wave][k] = v[k];
        }
        __syncthreads();
        const int first = wave / (G / 64) * (G / 64);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float s = red[first][k];
#pragma unroll
            for (int w = 1; w < G / 64; ++w) s += red[first + w][k];
            v[k] = s;
        }
    }
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// Values of a row that a thread holds: 32 K rows of 4096 bf16 97 us with 16 and four blocks of 256 threads a compute unit, 106
// with 8 and eight blocks, 98 with 32; 8191 of 1023 12.3, 13.7 and 15.9 (10.8 since, see ask_chunk). The backward's sums of dw and db leave room for 8.
constexpr int kFwdHeld = 16, kFwdBlocks = 4, kHeld = 8;
constexpr int fwd_threads(int G) { return G > 256 ? G : 256; }

template <int DX, int DW, bool RAGGED, int G>
__global__ __launch_bounds__(fwd_threads(G)) void norm_fwd_kernel(const void* __restrict__ X, const void* __restrict__ weight,
                                                                  const void* __restrict__ bias, float eps, float c,
                                                                  void* __restrict__ Y, float* __restrict__ mean,
                                                                  float* __restrict__ rstd, int64_t B, Row r) {
    constexpr int E = MixChunk<DX>::E, K = kFwdHeld / E, NT = fwd_threads(G), PER = NT / G;
    __shared__ float red[2][NT / 64][1];
    const int t = threadIdx.x % G;
    float w[K][E], b[K][E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_params<DW, E>(weight, r, t + G * k, 1.f, w[k]);
        load_params<DW, E>(bias, r, t + G * k, 0.f, b[k]);
    }
    const int64_t pitch = r.C * (DX == BIRKHOFF4_BF16 ? 2 : 4), step = static_cast<int64_t>(gridDim.x) * PER;
    const char* x = static_cast<const char*>(X);
    char* y = static_cast<char*>(Y);
    int64_t row = static_cast<int64_t>(blockIdx.x) * PER + threadIdx.x / G;
    v4u next[K];
#pragma unroll
    for (int k = 0; k < K; ++k) next[k] = row < B ? ask_chunk<DX, RAGGED>(x + row * pitch, r, t + G * k) : v4u{0, 0, 0, 0};
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * PER; base < B; base += step) {  // uniform over the block
        float v[K][E], sum[1] = {0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            unpack_chunk<DX>(chunk_of<DX, RAGGED>(next[k], r, t + G * k), v[k]);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += v[k][e];
        }
        const int64_t own = row;
        row += step;
        if (row < B) {
#pragma unroll
            for (int k = 0; k < K; ++k) next[k] = ask_chunk<DX, RAGGED>(x + row * pitch, r, t + G * k);
        }
        group_sums<G, NT>(sum, red[0]);
        const float mu = sum[0] / c;
        float sq[1] = {0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int n = chunk_values<DX, RAGGED>(r, t + G * k);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[k][e] -= mu;
                if (e < n) sq[0] = __builtin_fmaf(v[k][e], v[k][e], sq[0]);
            }
        }
        group_sums<G, NT>(sq, red[1]);
        const float s = 1.f / __builtin_sqrtf(sq[0] / c + eps);
        if (own < B) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float o[E];
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(v[k][e] * s, w[k][e], b[k][e]);
                store_chunk<DX, RAGGED>(y + own * pitch, r, t + G * k, pack_chunk<DX>(o));
            }
            if (t == 0) {
                if (mean) mean[own] = mu;
                if (rstd) rstd[own] = s;
            }
        }
    }
}

// Rows of more chunks than threads hold: a block a row, read three times (the second and third from L2).
constexpr int kLongThreads = 1024;

template <int DX, int DW, bool RAGGED>
__global__ __launch_bounds__(kLongThreads) void norm_long_fwd_kernel(const void* __restrict__ X, const void* __restrict__ weight,
                                                                     const void* __restrict__ bias, float eps, float c,
                                                                     void* __restrict__ Y, float* __restrict__ mean,
                                                                     float* __restrict__ rstd, int64_t B, Row r) {
    constexpr int E = MixChunk<DX>::E;
    __shared__ float red[2][kLongThreads / 64][1];
    const int64_t pitch = r.C * (DX == BIRKHOFF4_BF16 ? 2 : 4);
    for (int64_t row = blockIdx.x; row < B; row += gridDim.x) {
        const char* x = static_cast<const char*>(X) + row * pitch;
        float sum[1] = {0.f}, sq[1] = {0.f}, v[E];
        for (int k = threadIdx.x; k < r.nc; k += kLongThreads) {
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(x, r, k), v);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += v[e];
        }
        group_sums<kLongThreads, kLongThreads>(sum, red[0]);
        const float mu = sum[0] / c;
        for (int k = threadIdx.x; k < r.nc; k += kLongThreads) {
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(x, r, k), v);
            const int n = chunk_values<DX, RAGGED>(r, k);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < n) sq[0] = __builtin_fmaf(v[e] - mu, v[e] - mu, sq[0]);
        }
        group_sums<kLongThreads, kLongThreads>(sq, red[1]);
        const float s = 1.f / __builtin_sqrtf(sq[0] / c + eps);
        for (int k = threadIdx.x; k < r.nc; k += kLongThreads) {
            float w[E], b[E];
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(x, r, k), v);
            load_params<DW, E>(weight, r, k, 1.f, w);
            load_params<DW, E>(bias, r, k, 0.f, b);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = __builtin_fmaf((v[e] - mu) * s, w[e], b[e]);
            store_chunk<DX, RAGGED>(static_cast<char*>(Y) + row * pitch, r, k, pack_chunk<DX>(v));
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = s;
        }
    }
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------
// Each block takes every gridDim.x-th set of 1024 / G rows; its threads keep the sums of dw and db of
// their columns over all its rows, and the block's groups are added through LDS at the end: one row of
// 2 C sums a block, which norm_join_kernel adds in the blocks' order.
constexpr int kBwdThreads = 1024;

template <int DX, int DW, bool RAGGED, int G>
__global__ __launch_bounds__(kBwdThreads) void norm_bwd_kernel(const void* __restrict__ X, const void* __restrict__ weight,
                                                               const float* __restrict__ mean, const float* __restrict__ rstd,
                                                               const void* __restrict__ dY, float c, void* __restrict__ dX,
                                                               float* __restrict__ part, int64_t B, Row r) {
    constexpr int E = MixChunk<DX>::E, K = kHeld / E, PER = kBwdThreads / G;
    __shared__ float red[2][kBwdThreads / 64][2];
    __shared__ v4f joint[PER > 1 ? kBwdThreads : 1];
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    float w[K][E], dw[K][E], db[K][E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_params<DW, E>(weight, r, t + G * k, 1.f, w[k]);
#pragma unroll
        for (int e = 0; e < E; ++e) dw[k][e] = db[k][e] = 0.f;
    }
    const int64_t pitch = r.C * (DX == BIRKHOFF4_BF16 ? 2 : 4), step = static_cast<int64_t>(gridDim.x) * PER;
    const char *x = static_cast<const char*>(X), *dy = static_cast<const char*>(dY);
    char* dx = static_cast<char*>(dX);
    int64_t row = static_cast<int64_t>(blockIdx.x) * PER + group;
    v4u nx[K], ny[K];
    float nmu = 0.f, ns = 0.f;
    auto fetch = [&](int64_t at) {
        const bool in = at < B;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            nx[k] = in ? ask_chunk<DX, RAGGED>(x + at * pitch, r, t + G * k) : v4u{0, 0, 0, 0};
            ny[k] = in ? ask_chunk<DX, RAGGED>(dy + at * pitch, r, t + G * k) : v4u{0, 0, 0, 0};
        }
        nmu = in ? mean[at] : 0.f;
        ns = in ? rstd[at] : 0.f;
    };
    fetch(row);
    int turn = 0;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * PER; base < B; base += step, turn ^= 1) {  // uniform
        v4u cx[K], cy[K];
        const float mu = nmu, s = ns;
        const int64_t own = row;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            cx[k] = chunk_of<DX, RAGGED>(nx[k], r, t + G * k);
            cy[k] = chunk_of<DX, RAGGED>(ny[k], r, t + G * k);
        }
        row += step;
        fetch(row);
        float sum[2] = {0.f, 0.f};  // of g and of g xh
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float xv[E], gv[E];
            unpack_chunk<DX>(cx[k], xv);
            unpack_chunk<DX>(cy[k], gv);
            const int n = chunk_values<DX, RAGGED>(r, t + G * k);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float xh = e < n ? (xv[e] - mu) * s : 0.f;  // past the row's end dy is 0, x may make NaN of it
                const float g = gv[e] * w[k][e];
                db[k][e] += gv[e];
                dw[k][e] = __builtin_fmaf(gv[e], xh, dw[k][e]);
                sum[0] += g;
                sum[1] = __builtin_fmaf(g, xh, sum[1]);
            }
        }
        group_sums<G, kBwdThreads>(sum, red[turn]);
        if (dX && own < B) {
            const float m0 = sum[0] / c, m1 = sum[1] / c;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float xv[E], gv[E], o[E];
                unpack_chunk<DX>(cx[k], xv);
                unpack_chunk<DX>(cy[k], gv);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float xh = (xv[e] - mu) * s;
                    o[e] = s * __builtin_fmaf(-xh, m1, __builtin_fmaf(gv[e], w[k][e], -m0));
                }
                store_chunk<DX, RAGGED>(dx + own * pitch, r, t + G * k, pack_chunk<DX>(o));
            }
        }
    }
    if (!part) return;
    float* out = part + static_cast<int64_t>(blockIdx.x) * 2 * r.C;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < E / 4; ++q) {
                const float* a = h ? &db[k][4 * q] : &dw[k][4 * q];
                v4f v = {a[0], a[1], a[2], a[3]};
                if constexpr (PER > 1) {
                    __syncthreads();
                    joint[threadIdx.x] = v;
                    __syncthreads();
                    if (group == 0)
                        for (int j = 1; j < PER; ++j) v += joint[t + G * j];
                }
                const int64_t col = static_cast<int64_t>(t + G * k) * E + 4 * q;
                if (group == 0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e < r.C) out[h * r.C + col + e] = v[e];
                }
            }
}

// Rows of more chunks than threads hold: dx a block a row, from two readings of it; dw and db by blocks
// of a share of the rows and 256 columns each.
template <int DX, int DW, bool RAGGED>
__global__ __launch_bounds__(kLongThreads) void norm_long_bwd_kernel(const void* __restrict__ X, const void* __restrict__ weight,
                                                                     const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                     const void* __restrict__ dY, float c,
                                                                     void* __restrict__ dX, int64_t B, Row r) {
    constexpr int E = MixChunk<DX>::E;
    __shared__ float red[2][kLongThreads / 64][2];
    const int64_t pitch = r.C * (DX == BIRKHOFF4_BF16 ? 2 : 4);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < B; row += gridDim.x, turn ^= 1) {
        const char *x = static_cast<const char*>(X) + row * pitch, *dy = static_cast<const char*>(dY) + row * pitch;
        const float mu = mean[row], s = rstd[row];
        float sum[2] = {0.f, 0.f}, xv[E], gv[E], w[E];
        for (int k = threadIdx.x; k < r.nc; k += kLongThreads) {
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(x, r, k), xv);
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(dy, r, k), gv);
            load_params<DW, E>(weight, r, k, 1.f, w);
            const int n = chunk_values<DX, RAGGED>(r, k);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float g = gv[e] * w[e], xh = e < n ? (xv[e] - mu) * s : 0.f;
                sum[0] += g;
                sum[1] = __builtin_fmaf(g, xh, sum[1]);
            }
        }
        group_sums<kLongThreads, kLongThreads>(sum, red[turn]);
        const float m0 = sum[0] / c, m1 = sum[1] / c;
        for (int k = threadIdx.x; k < r.nc; k += kLongThreads) {
            float o[E];
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(x, r, k), xv);
            unpack_chunk<DX>(load_chunk<DX, RAGGED>(dy, r, k), gv);
            load_params<DW, E>(weight, r, k, 1.f, w);
#pragma unroll
            for (int e = 0; e < E; ++e)
                o[e] = s * __builtin_fmaf(-(xv[e] - mu) * s, m1, __builtin_fmaf(gv[e], w[e], -m0));
            store_chunk<DX, RAGGED>(static_cast<char*>(dX) + row * pitch, r, k, pack_chunk<DX>(o));
        }
    }
}

template <int DX>
__global__ __launch_bounds__(256) void norm_long_sums_kernel(const void* __restrict__ X, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, const void* __restrict__ dY,
                                                             float* __restrict__ part, int64_t B, int64_t C) {
    const int64_t col = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (col >= C) return;
    float dw = 0.f, db = 0.f;
    for (int64_t row = blockIdx.y; row < B; row += gridDim.y) {
        float x, g;
        if constexpr (DX == BIRKHOFF4_BF16) {
            x = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(X)[row * C + col]) << 16);
            g = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(dY)[row * C + col]) << 16);
        } else {
            x = static_cast<const float*>(X)[row * C + col];
            g = static_cast<const float*>(dY)[row * C + col];
        }
        dw = __builtin_fmaf(g, (x - mean[row]) * rstd[row], dw);
        db += g;
    }
    float* out = part + static_cast<int64_t>(blockIdx.y) * 2 * C + col;
    out[0] = dw;
    out[C] = db;
}

// The blocks' sums added in their order, 16 parts of them first: 64 columns a block. Without rows: zeros.
constexpr int kNormJoin = 1024, kNormJoinCols = 64;

template <int DW>
__global__ __launch_bounds__(kNormJoin) void norm_join_kernel(const float* __restrict__ part, int blocks, int64_t C,
                                                              void* __restrict__ dweight, void* __restrict__ dbias) {
    constexpr int PARTS = kNormJoin / kNormJoinCols;
    __shared__ float red[PARTS][kNormJoinCols];
    const int c = threadIdx.x % kNormJoinCols, p = threadIdx.x / kNormJoinCols;
    const int64_t col = static_cast<int64_t>(blockIdx.x) * kNormJoinCols + c;  // of 2 C
    float v = 0.f;
    if (col < 2 * C)
#pragma unroll 8
        for (int k = p; k < blocks; k += PARTS) v += part[static_cast<int64_t>(k) * 2 * C + col];
    red[p][c] = v;
    __syncthreads();
    if (p > 0 || col >= 2 * C) return;
    for (int k = 1; k < PARTS; ++k) v += red[k][c];
    void* out = col < C ? dweight : dbias;
    if (!out) return;
    const int64_t at = col < C ? col : col - C;
    if constexpr (DW == BIRKHOFF4_BF16)
        static_cast<uint16_t*>(out)[at] = static_cast<uint16_t>(pack_bf16(v, 0.f));
    else
        static_cast<float*>(out)[at] = v;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int64_t kNormMaxRows = int64_t(1) << 31;
constexpr int64_t kNormMaxWidth = int64_t(1) << 20;
constexpr int64_t kNormMaxValues = int64_t(1) << 46;

struct NormShape {
    int64_t B;
    Row r;
    bool ragged;
};

int norm_shape(int64_t B, int64_t C, int x_dtype, int w_dtype, NormShape* s) {
    if (B < 0 || B > kNormMaxRows) return BIRKHOFF4_ERR_SIZE;
    if (!dtype_ok(x_dtype) || !dtype_ok(w_dtype)) return BIRKHOFF4_ERR_DTYPE;
    if (C <= 0) return BIRKHOFF4_ERR_CHANNELS;
    if (C > kNormMaxWidth || (B > 0 && C > kNormMaxValues / B)) return BIRKHOFF4_ERR_SIZE;
    const int64_t e = x_dtype == BIRKHOFF4_BF16 ? 8 : 4;
    const int64_t nc = (C + e - 1) / e;
    *s = {B, {C, static_cast<int>(nc), static_cast<int>(C - (nc - 1) * e)}, C % e != 0};
    return BIRKHOFF4_OK;
}

constexpr int64_t kLongRow = 1024 * kHeld;  // values of a row, above which the backward's threads do not hold it
constexpr int64_t kNormBlocks = 256;  // of the backward: one a compute unit (two: 32 K rows of 4096 bf16 164 us instead of 154, 4097 of 1000 fp32 15.6 and 12.7)

// Threads that hold a row: the fewest, 16 at least.
int row_group(int64_t C, int held = kHeld) {
    int g = 16;
    while (g * held < C) g *= 2;
    return g;
}

// Rows of sums that the backward writes and the join reads, none without rows.
int64_t bwd_blocks(const NormShape& s) {
    if (s.B == 0) return 0;
    if (s.r.C > kLongRow) {  // shares of the rows
        const int64_t want = 2048 / ((s.r.C + 255) / 256);
        return want < 1 ? 1 : want < s.B ? want : s.B;
    }
    const int64_t per = kBwdThreads / row_group(s.r.C), want = (s.B + per - 1) / per;
    return want < kNormBlocks ? want : kNormBlocks;
}

template <int DX, int DW, bool RAGGED>
int launch_norm_fwd(const NormShape& s, const void* X, const void* weight, const void* bias, float eps, void* Y, float* mean,
                    float* rstd, int cus, hipStream_t stream) {
    const float c = static_cast<float>(s.r.C);
    auto go = [&](auto kern, int G, int threads) {
        const int64_t want = (s.B * G + threads - 1) / threads, most = int64_t(cus) * kFwdBlocks * 256 / threads;
        launch_kernel(kern, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(threads), 0, stream, X, weight, bias,
                      eps, c, Y, mean, rstd, s.B, s.r);
        return launch_status();
    };
#define FWD(G) \
    case G: return go(norm_fwd_kernel<DX, DW, RAGGED, G>, G, fwd_threads(G))
    switch (s.r.C > 1024 * kFwdHeld ? 0 : row_group(s.r.C, kFwdHeld)) {
        FWD(16);
        FWD(32);
        FWD(64);
        FWD(128);
        FWD(256);
        FWD(512);
        FWD(1024);
    }
#undef FWD
    launch_kernel((norm_long_fwd_kernel<DX, DW, RAGGED>), dim3(static_cast<unsigned>(s.B < 2 * cus ? s.B : 2 * cus)),
                  dim3(kLongThreads), 0, stream, X, weight, bias, eps, c, Y, mean, rstd, s.B, s.r);
    return launch_status();
}

template <int DX, int DW, bool RAGGED>
int launch_norm_bwd(const NormShape& s, const void* X, const void* weight, const float* mean, const float* rstd,
                    const void* dY, void* dX, void* dweight, void* dbias, float* part, int cus, hipStream_t stream) {
    const float c = static_cast<float>(s.r.C);
    const int64_t blocks = bwd_blocks(s);
    if (!dweight && !dbias) part = nullptr;
    if (s.B > 0 && s.r.C <= kLongRow) {
        auto go = [&](auto kern) {
            launch_kernel(kern, dim3(static_cast<unsigned>(blocks)), dim3(kBwdThreads), 0, stream, X, weight, mean, rstd, dY,
                          c, dX, part, s.B, s.r);
        };
#define BWD(G) \
    case G: go(norm_bwd_kernel<DX, DW, RAGGED, G>); break
        switch (row_group(s.r.C)) {
            BWD(16);
            BWD(32);
            BWD(64);
            BWD(128);
            BWD(256);
            BWD(512);
            BWD(1024);
        }
#undef BWD
    } else if (s.B > 0) {
        if (dX)
            launch_kernel((norm_long_bwd_kernel<DX, DW, RAGGED>), dim3(static_cast<unsigned>(s.B < 2 * cus ? s.B : 2 * cus)),
                          dim3(kLongThreads), 0, stream, X, weight, mean, rstd, dY, c, dX, s.B, s.r);
        if (part)
            launch_kernel((norm_long_sums_kernel<DX>), dim3(static_cast<unsigned>((s.r.C + 255) / 256), static_cast<unsigned>(blocks)),
                          dim3(256), 0, stream, X, mean, rstd, dY, part, s.B, s.r.C);
    }
    if (dweight || dbias)
        launch_kernel((norm_join_kernel<DW>), dim3(static_cast<unsigned>((2 * s.r.C + kNormJoinCols - 1) / kNormJoinCols)),
                      dim3(kNormJoin), 0, stream, part, static_cast<int>(blocks), s.r.C, dweight, dbias);
    return launch_status();
}

bool norm_eps_ok(float eps) { return eps >= 0.f && eps < __builtin_inff(); }

}  // namespace

extern "C" {

int birkhoff4_norm_fwd(const void* X, int x_dtype, const void* weight, const void* bias, int w_dtype, float eps, void* Y,
                       float* mean, float* rstd, int64_t B, int64_t C, hipStream_t stream) {
    NormShape s;
    if (int e = norm_shape(B, C, x_dtype, w_dtype, &s)) return e;
    if (!norm_eps_ok(eps)) return BIRKHOFF4_ERR_EPS;
    if (B == 0) return BIRKHOFF4_OK;
    if (!X || !Y) return BIRKHOFF4_ERR_NULL;
    const void* all[] = {X, weight, bias, Y, mean, rstd};
    for (const void* p : all)
        if (misaligned(p)) return BIRKHOFF4_ERR_ALIGN;
    const size_t rows = static_cast<size_t>(B), row = static_cast<size_t>(C) * dtype_bytes(x_dtype),
                 par = static_cast<size_t>(C) * dtype_bytes(w_dtype);
    const Span ins[] = {{X, rows * row}, {weight, par}, {bias, par}};
    const Span outs[] = {{Y, rows * row}, {mean, rows * 4}, {rstd, rows * 4}};
    if (!disjoint(outs, 3, ins, 3)) return BIRKHOFF4_ERR_OVERLAP;
    int cus = 0;
    if (int e = device_cus(stream, &cus)) return e;
    constexpr int F = BIRKHOFF4_F32, H = BIRKHOFF4_BF16;
    auto pick = [&](auto plain, auto ragged) { return s.ragged ? ragged : plain; };
    auto launch = x_dtype == H ? (w_dtype == H ? pick(launch_norm_fwd<H, H, false>, launch_norm_fwd<H, H, true>)
                                               : pick(launch_norm_fwd<H, F, false>, launch_norm_fwd<H, F, true>))
                               : (w_dtype == H ? pick(launch_norm_fwd<F, H, false>, launch_norm_fwd<F, H, true>)
                                               : pick(launch_norm_fwd<F, F, false>, launch_norm_fwd<F, F, true>));
    return launch(s, X, weight, bias, eps, Y, mean, rstd, cus, stream);
}

int64_t birkhoff4_norm_work(int64_t B, int64_t C, int x_dtype) {
    NormShape s;
    if (int e = norm_shape(B, C, x_dtype, BIRKHOFF4_F32, &s)) return e;
    return bwd_blocks(s) * 2 * C * 4;
}

int birkhoff4_norm_bwd(const void* X, int x_dtype, const void* weight, int w_dtype, const float* mean, const float* rstd,
                       const void* dY, void* dX, void* dweight, void* dbias, void* work, int64_t work_bytes, int64_t B,
                       int64_t C, hipStream_t stream) {
    NormShape s;
    if (int e = norm_shape(B, C, x_dtype, w_dtype, &s)) return e;
    const bool sums = dweight || dbias;
    if (B == 0 && !sums) return BIRKHOFF4_OK;
    if (B > 0 && (!X || !mean || !rstd || !dY || (sums && !work))) return BIRKHOFF4_ERR_NULL;
    const int64_t need = sums ? bwd_blocks(s) * 2 * C * 4 : 0;
    if (work_bytes < need) return BIRKHOFF4_ERR_WORK;
    const void* all[] = {X, weight, mean, rstd, dY, dX, dweight, dbias, work};
    for (const void* p : all)
        if (misaligned(p)) return BIRKHOFF4_ERR_ALIGN;
    const size_t rows = static_cast<size_t>(B), row = static_cast<size_t>(C) * dtype_bytes(x_dtype),
                 par = static_cast<size_t>(C) * dtype_bytes(w_dtype);
    const Span ins[] = {{X, rows * row}, {weight, par}, {mean, rows * 4}, {rstd, rows * 4}, {dY, rows * row}};
    const Span outs[] = {{dX, rows * row}, {dweight, par}, {dbias, par}, {work, static_cast<size_t>(need)}};
    if (!disjoint(outs, 4, ins, 5)) return BIRKHOFF4_ERR_OVERLAP;
    if (!sums && !dX) return BIRKHOFF4_OK;
    int cus = 0;
    if (int e = device_cus(stream, &cus)) return e;
    constexpr int F = BIRKHOFF4_F32, H = BIRKHOFF4_BF16;
    auto pick = [&](auto plain, auto ragged) { return s.ragged ? ragged : plain; };
    auto launch = x_dtype == H ? (w_dtype == H ? pick(launch_norm_bwd<H, H, false>, launch_norm_bwd<H, H, true>)
                                               : pick(launch_norm_bwd<H, F, false>, launch_norm_bwd<H, F, true>))
                               : (w_dtype == H ? pick(launch_norm_bwd<F, H, false>, launch_norm_bwd<F, H, true>)
                                               : pick(launch_norm_bwd<F, F, false>, launch_norm_bwd<F, F, true>));
    return launch(s, X, weight, mean, rstd, dY, dX, dweight, dbias, static_cast<float*>(work), cus, stream);
}

}  // extern "C"
