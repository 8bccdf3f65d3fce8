// pre.hip -- how a hyper-connection layer reads its streams (Sec. 2.1), for gfx950 (MI355X).
//
// The layer's update is x <- H^res x + (H^post)^T F(H^pre x) with x a token's n = 4 or 8 streams
// of C channels. Its coefficients come from the streams themselves: with v the token's K = n C
// values, r = (|v|^2 / K + eps)^(-1/2) and W of N = n^2 + 2 n rows,
//     q = r W v,   l = alpha_g q + bias   (g: rows 0..n-1, n..2n-1 and the n^2 others)
//     h^pre = sigmoid(l_pre),   h = 2 sigmoid(l_post),   H = l_res,   U = sum_i h^pre_i X_i
// H are the logits of the residual mixing and U is the branch's input. The backward, from
// dU, dh, dH and optionally E, a gradient of the streams from elsewhere:
//     dl_pre,i = h^pre_i (1 - h^pre_i) <dU, X_i>,  dl_post = dh h (1 - h / 2),  dl_res = dH
//     dbias = sum over tokens of dl,   dalpha_g = sum over tokens and rows of g of dl q
//     G = r alpha_g dl,   dW = sum over tokens of G v^T,   s = (r / K) sum_j G_j q_j
//     dX_i = E_i + h^pre_i dU + (G W)_i - s X_i
//
// Both are bound by HBM: with n = 4 a token of 2-byte values is 2 N operations per 2 bytes, a
// tenth of what the matrix cores do in that time. W (N rows) is used by every token and stays in
// L2; the products run on the matrix cores with the tokens as one side of the tile.

#include <type_traits>

#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int N>
struct Gates {
    static constexpr int rows = N * N + 2 * N;        // 24 or 80: rows of W, coefficients of a token
    static constexpr int tiles = (rows + 15) / 16;    // 16-row tiles of a product
    static constexpr int stride = rows + 4;           // floats per token of the partial sums: rows, |v|^2, 0, 0, 0
    static constexpr int ksteps = (rows + 31) / 32;   // 32-row steps of a product over the rows
};

__device__ __forceinline__ v4f mfma_bf16(const v4u a, const v4u b, const v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
}

__device__ __forceinline__ v4f mfma_f32(float a, float b, const v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// c += a b over 64 bytes of sixteen rows of each side, lane l holding 16-byte chunk l / 16 of row
// l % 16: one product of 32 bf16 values, or four of 4 fp32 values (values m of the four chunks).
template <int DX>
__device__ __forceinline__ v4f mfma_chunks(const v4u a, const v4u b, v4f c) {
    if constexpr (DX == BIRKHOFF4_BF16) {
        return mfma_bf16(a, b, c);
    } else {
#pragma unroll
        for (int m = 0; m < 4; ++m) c = mfma_f32(__uint_as_float(a[m]), __uint_as_float(b[m]), c);
        return c;
    }
}

__device__ __forceinline__ float sigmoid(float x) { return rcp(1.0f + ex2(-kLog2e * x)); }

// alpha's entry for row j of W.
template <int N>
__device__ __forceinline__ float row_scale(const float* __restrict__ alpha, int j) {
    return alpha[j < N ? 0 : j < 2 * N ? 1 : 2];
}

// ---------------------------------------------------------------------------
// Forward: the products W v and |v|^2 of every token
// ---------------------------------------------------------------------------
// Blocks take some tokens and a share of the row, in steps of 64 bytes, two steps (a 128-byte line of
// each token) at a time. Tokens are the columns of the products' tiles, rows of W the rows; |v|^2 is
// the diagonal of the product of the tokens' operand with itself (fp32: plain sums, as the fp32
// matrix rate is nearer to what HBM delivers). A wave loads whole lines, eight lanes a row, and takes
// them to the operands' layout (a lane row's chunk) through LDS of its own while the next are on
// the way: loaded in that layout, sixteen rows of 64 bytes at a time, 32 K tokens of 4 x 4096 bf16 took
// 249 us instead of 195. The shares' sums are added by the reader, in order: no atomics, so a
// token's result does not depend on timing.
template <int DX, int N, int TT>
struct GateSums {  // of a wave's 16 TT tokens: lane (g, c) has rows 16 r + 4 g .. + 3 of token 16 t + c
    static constexpr int RT = Gates<N>::tiles, R = Gates<N>::rows;
    v4f acc[TT][RT], norm[TT];
    float ss[TT];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            norm[t] = v4f{0.f, 0.f, 0.f, 0.f};
            ss[t] = 0.f;
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[t][r] = v4f{0.f, 0.f, 0.f, 0.f};
        }
    }

    // One step: chunk g of row 16 r + c of W, and of token 16 t + c.
    __device__ __forceinline__ void step(const v4u (&wv)[RT], const v4u (&xv)[TT]) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[t][r] = mfma_chunks<DX>(wv[r], xv[t], acc[t][r]);
            if constexpr (DX == BIRKHOFF4_BF16) {
                norm[t] = mfma_bf16(xv[t], xv[t], norm[t]);
            } else {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float v = __uint_as_float(xv[t][m]);
                    ss[t] = __builtin_fmaf(v, v, ss[t]);
                }
            }
        }
    }

    // After the last step: token 16 t + c's |v|^2 is the diagonal's value in lane group c / 4.
    __device__ __forceinline__ void finish(int c) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            float sum;
            if constexpr (DX == BIRKHOFF4_BF16) {
                sum = (c & 3) == 0 ? norm[t].x : (c & 3) == 1 ? norm[t].y : (c & 3) == 2 ? norm[t].z : norm[t].w;
            } else {
                sum = ss[t];
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
            }
            norm[t] = v4f{sum, 0.f, 0.f, 0.f};
        }
    }

    // This lane's quads of the tokens' rows of sums: f(token, quad, value).
    template <typename F>
    __device__ __forceinline__ void each(int g, int c, F&& f) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
                if (16 * r + 4 * g < R) f(16 * t + c, 4 * r + g, acc[t][r]);
            if (g == c >> 2) f(16 * t + c, Gates<N>::stride / 4 - 1, norm[t]);
        }
    }
};

// Offsets of the rows that a lane loads, eight rows at a time, from the wave's first token; past the
// last token: that token again, its sums not stored.
template <int TT>
__device__ __forceinline__ void line_offsets(uint32_t (&off)[2 * TT], int lane, int64_t row_bytes, int64_t last) {
#pragma unroll
    for (int t = 0; t < 2 * TT; ++t) {
        const int64_t row = 8 * t + (lane >> 3);
        off[t] = static_cast<uint32_t>(row_bytes * (row < last ? row : last)) + 16 * (lane & 7);
    }
}

// The lane's chunks of the lines at p: of both steps, or, with the row's end between them, of the first.
template <int TT>
__device__ __forceinline__ void load_lines(v4u (&xr)[2 * TT], const char* p, const uint32_t (&off)[2 * TT], bool two,
                                           int lane) {
    const bool mine = two || (lane & 7) < 4;
#pragma unroll
    for (int t = 0; t < 2 * TT; ++t) {
        xr[t] = v4u{0u, 0u, 0u, 0u};
        if (mine) xr[t] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p + off[t]));
    }
}

// A block's tile of tokens and share of the row. Workgroups go to the eight XCDs in turn; each XCD
// gets neighbouring pairs, tiles first, so that its L2 holds the part of W of its shares (forward of 8 K
// tokens of 8 x 4096 bf16, 5.2 MB of W, 211 -> 202 us, with W's loads behind the streams' 237 -> 204; n = 4, whose
// W an L2 holds whole: 16 K tokens of 4 x 4096 194 -> 190, 2^15 of 4 x 2048 188 -> 204).
struct GatePlace {
    int64_t tile;
    int64_t share;
};

__device__ __forceinline__ GatePlace gate_place(uint32_t tiles, uint32_t per_xcd) {
    const uint32_t k = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    return {k % tiles, k / tiles};
}

// A block's GW waves share its 16 TT tokens and take the lines of its share of the row in turn; their
// sums are added in LDS, the upper half of the waves to the lower.
template <int DX, int N, int TT, int GW>
__global__ __launch_bounds__(64 * GW, GW > 8 ? GW / 4 : 2) void pre_gate_kernel(const v4u* __restrict__ X,
                                                                      const v4u* __restrict__ W,
                                                                      float* __restrict__ part, int64_t B, int64_t steps,
                                                                      int64_t per, uint32_t tiles, uint32_t per_xcd) {
    constexpr int RT = Gates<N>::tiles, R = Gates<N>::rows, S4 = Gates<N>::stride / 4;
    // 128 bytes of a row and 16 that keep the lanes that read one chunk of sixteen rows on different banks
    __shared__ union {
        v4u rows[GW][16 * TT][9];
        v4f red[GW / 2][16 * TT][S4];
    } lds;
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const GatePlace at = gate_place(tiles, per_xcd);
    const int64_t first = at.tile * 16 * TT;
    const int64_t s0 = at.share * per, s1 = s0 + per < steps ? s0 + per : steps;
    if (s0 >= s1) return;  // the whole block
    const char* base = reinterpret_cast<const char*>(X) + 64 * steps * first;
    uint32_t off[2 * TT];
    line_offsets<TT>(off, lane, 64 * steps, B - 1 - first);
    const v4u* wr[RT];  // past the last row: that row, its sums not stored
#pragma unroll
    for (int r = 0; r < RT; ++r) wr[r] = W + 4 * steps * (16 * r + c < R ? 16 * r + c : R - 1) + g;
    GateSums<DX, N, TT> sums;
    sums.clear();
    // blocks begin at different places of the row: begun together, forward of 16 K tokens of 4 x 4096 bf16 212 us
    // instead of 190, 2^15 390 instead of 383
    const int64_t turns = (s1 - s0 + 2 * GW - 1) / (2 * GW);
    int64_t turn = (blockIdx.x >> 3) % turns, next = s0 + 2 * GW * turn + 2 * w;
    v4u xr[2 * TT];
    auto load = [&](int64_t s) {
        if (s < s1) {  // uniform
            load_lines<TT>(xr, base + 64 * s, off, s + 1 < s1, lane);
        } else {
#pragma unroll
            for (int t = 0; t < 2 * TT; ++t) xr[t] = v4u{0u, 0u, 0u, 0u};
        }
    };
    load(next);
    for (int64_t k = 0; k < turns; ++k) {
        const int64_t s = next;
        v4u xv[2][TT], wv[2][RT];
        // W's lines before the next streams' (loads come back in order): a wait for them is for them alone
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int r = 0; r < RT; ++r) wv[u][r] = v4u{0u, 0u, 0u, 0u};
            if (s + u < s1) {  // uniform
#pragma unroll
                for (int r = 0; r < RT; ++r) wv[u][r] = wr[r][4 * (s + u)];
            }
        }
        __builtin_amdgcn_wave_barrier();  // the last turn's reads of the wave's lines come before, this one's after
#pragma unroll
        for (int t = 0; t < 2 * TT; ++t) lds.rows[w][8 * t + (lane >> 3)][lane & 7] = xr[t];
        __builtin_amdgcn_wave_barrier();
        turn = turn + 1 < turns ? turn + 1 : 0;
        next = s0 + 2 * GW * turn + 2 * w;
        if (k + 1 < turns) load(next);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < TT; ++t) xv[u][t] = lds.rows[w][16 * t + c][4 * u + g];
#pragma unroll
        for (int u = 0; u < 2; ++u) sums.step(wv[u], xv[u]);
    }
    sums.finish(c);
    auto put = [&](int k) { sums.each(g, c, [&](int t, int q, v4f& v) { lds.red[k][t][q] = v; }); };
    auto add = [&](int k) { sums.each(g, c, [&](int t, int q, v4f& v) { v += lds.red[k][t][q]; }); };
    __syncthreads();
#pragma unroll
    for (int half = GW / 2; half >= 1; half /= 2) {
        if (w >= half && w < 2 * half) put(w - half);
        __syncthreads();
        if (w < half) add(w);
        __syncthreads();
    }
    if (w == 0) {
        v4f* dst = reinterpret_cast<v4f*>(part) + (at.share * B + first) * S4;
        sums.each(g, c, [&](int t, int q, v4f& v) {
            if (first + t < B) dst[t * S4 + q] = v;
        });
    }
}

// Many tokens with n = 8, whose W is as much as the streams of 80 tokens: a block's waves have 64 tokens
// each and go along the row together, so that a line of W is brought to LDS once for all of them. From
// 2 K tokens on; whole forward in us, without it in brackets: 2049 tokens of 8 x 512 bf16 29 (32), 2049 of 8 x
// 4096 81 (83), 3000 of 8 x 4096 101 (117), 6000 166 (209), 32 K 790 (996), 8000 of 8 x 1024 fp32 178 (228); slower
// at few of the sizes tried (4096 of 8 x 512 37 (33), 2500 of 8 x 4096 fp32 272 (252)). With n = 4 such a form,
// of eight waves, is not there: it was slower at most sizes (20481 tokens of 4 x 4096 297 (256), 2^15 403 (388),
// 65537 of 4 x 512 137 (120)) and faster only where its 512-token blocks came out even (2^15 of 4 x 2048 196
// (206), 2^18 of 4 x 128 128 (139)) or rows were very short (10^6 of 4 x 8 189 (228)).
constexpr int kGateWideWaves = 4;

template <int DX>
__global__ __launch_bounds__(64 * kGateWideWaves, 2) void pre_gate_wide_kernel(const v4u* __restrict__ X,
                                                                               const v4u* __restrict__ W,
                                                                               float* __restrict__ part, int64_t B,
                                                                               int64_t steps, int64_t per, uint32_t tiles,
                                                                               uint32_t per_xcd) {
    constexpr int N = 8, RT = Gates<N>::tiles, R = Gates<N>::rows, S4 = Gates<N>::stride / 4, TT = 4, GW = kGateWideWaves;
    constexpr int kThreads = 64 * GW, WQ = (8 * R + kThreads - 1) / kThreads;
    __shared__ v4u rows[GW][16 * TT][9];
    __shared__ v4u wrow[2][R][9];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const GatePlace at = gate_place(tiles, per_xcd);
    const int64_t first = (at.tile * GW + w) * 16 * TT;
    const int64_t s0 = at.share * per, s1 = s0 + per < steps ? s0 + per : steps;
    if (s0 >= s1) return;  // the whole block
    const int64_t start = first < B ? first : B - 1;  // a wave without tokens goes along on the last one's values
    const char* base = reinterpret_cast<const char*>(X) + 64 * steps * start;
    uint32_t off[2 * TT];
    line_offsets<TT>(off, lane, 64 * steps, B - 1 - start);
    GateSums<DX, N, TT> sums;
    sums.clear();
    const int64_t turns = (s1 - s0 + 1) / 2;
    int64_t turn = (blockIdx.x >> 3) % turns;
    v4u xr[2 * TT], wq[WQ];
    auto load = [&](int64_t s) {
        const bool two = s + 1 < s1;  // uniform
        load_lines<TT>(xr, base + 64 * s, off, two, lane);
#pragma unroll
        for (int q = 0; q < WQ; ++q) {
            const int k = static_cast<int>(threadIdx.x) + kThreads * q;
            wq[q] = v4u{0u, 0u, 0u, 0u};
            if (k < 8 * R && (two || (k & 7) < 4)) wq[q] = W[4 * (steps * (k >> 3) + s) + (k & 7)];
        }
    };
    load(s0 + 2 * turn);
    for (int64_t k = 0; k < turns; ++k) {
        const int buf = static_cast<int>(k & 1);
        __builtin_amdgcn_wave_barrier();  // the last turn's reads of the wave's lines come before
#pragma unroll
        for (int t = 0; t < 2 * TT; ++t) rows[w][8 * t + (lane >> 3)][lane & 7] = xr[t];
#pragma unroll
        for (int q = 0; q < WQ; ++q) {
            const int e = static_cast<int>(threadIdx.x) + kThreads * q;
            if (e < 8 * R) wrow[buf][e >> 3][e & 7] = wq[q];
        }
        // this line of W is there, and everybody has read the one that the next turn overwrites
        __syncthreads();
        turn = turn + 1 < turns ? turn + 1 : 0;
        if (k + 1 < turns) load(s0 + 2 * turn);
        v4u xv[2][TT], wv[2][RT];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int r = 0; r < RT; ++r) wv[u][r] = wrow[buf][16 * r + c < R ? 16 * r + c : R - 1][4 * u + g];
#pragma unroll
            for (int t = 0; t < TT; ++t) xv[u][t] = rows[w][16 * t + c][4 * u + g];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) sums.step(wv[u], xv[u]);
    }
    sums.finish(c);
    v4f* dst = reinterpret_cast<v4f*>(part) + (at.share * B + first) * S4;
    sums.each(g, c, [&](int t, int q, v4f& v) {
        if (first + t < B) dst[t * S4 + q] = v;
    });
}

// ---------------------------------------------------------------------------
// Forward: the coefficients, and U = sum_i h^pre_i X_i
// ---------------------------------------------------------------------------
// Lanes take 16-byte chunks of the rows, L lanes a token and 64 / L tokens a wave. The tokens' partial
// sums are added (lane j row j) while the streams are on the way; the waves of a block of one token
// take shares in turn (added by each of its waves: 32 tokens of 8 x 4096 with 32 shares 17 us).
constexpr int kReadWaves = 8;

template <int DX, int N, int L>
__global__ __launch_bounds__(64 * kReadWaves) void pre_read_kernel(const float* __restrict__ part, const v4u* __restrict__ X,
                                                       const float* __restrict__ alpha, const float* __restrict__ bias,
                                                       float eps, float inv_k, v4u* __restrict__ U,
                                                       float* __restrict__ h, float* __restrict__ H,
                                                       float* __restrict__ Q, float* __restrict__ rms, int64_t B,
                                                       int64_t nc, int splits) {
    constexpr int R = Gates<N>::rows, S = Gates<N>::stride, J = (S + 63) / 64, TW = 64 / L, E = MixChunk<DX>::E;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int W = blockDim.x >> 6;
    // blocks from the last token back: the last ones that the products read are still in the cache. With more
    // of them than one dimension of a grid takes, they lie along z too
    const int64_t block = static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x;
    const int64_t t0 = (static_cast<int64_t>(gridDim.z) * gridDim.x - 1 - block) * TW;
    const int64_t tok = t0 + lane / L;
    const int64_t first = L == 64 ? 64 * (static_cast<int64_t>(blockIdx.y) * W + w) : 0;  // this wave's column
    const int64_t col = first + lane % L;
    v4u x[N];
    const v4u* row = X + N * nc * (tok < B ? tok : B - 1);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = v4u{0u, 0u, 0u, 0u};
    if (col < nc) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_nontemporal_load(row + (i * nc + col));
    }
    __shared__ float psum[L == 64 ? kReadWaves : 1][64 * J];
    float hp[N];
#pragma unroll
    for (int i = 0; i < N; ++i) hp[i] = 0.f;
#pragma unroll
    for (int k = 0; k < TW; ++k) {
        const int64_t t = t0 + k;
        if (t >= B) break;  // uniform
        float sum[J], l[J], gate[J];
#pragma unroll
        for (int m = 0; m < J; ++m) sum[m] = 0.f;
#pragma unroll 8
        for (int s = L == 64 ? w : 0; s < splits; s += L == 64 ? W : 1) {
            const float* p = part + (s * B + t) * S;
#pragma unroll
            for (int m = 0; m < J; ++m)
                if (64 * m + lane < S) sum[m] += p[64 * m + lane];
        }
        if (L == 64 && W > 1 && splits > 1) {  // uniform over the block
#pragma unroll
            for (int m = 0; m < J; ++m) psum[w][64 * m + lane] = sum[m];
            __syncthreads();
            const int most = splits < W ? splits : W;
#pragma unroll
            for (int m = 0; m < J; ++m) {
                sum[m] = psum[0][64 * m + lane];
                for (int q = 1; q < most; ++q) sum[m] += psum[q][64 * m + lane];
            }
        } else if (L == 64 && W > 1 && w > 0) {  // one share: the other waves read it too
#pragma unroll
            for (int m = 0; m < J; ++m)
                if (64 * m + lane < S) sum[m] = part[t * S + 64 * m + lane];
        }
        const float norm2 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sum[R / 64]), R % 64));
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(norm2, inv_k, eps));
#pragma unroll
        for (int m = 0; m < J; ++m) {
            const int j = 64 * m + lane < R ? 64 * m + lane : R - 1;
            sum[m] *= r;  // q
            l[m] = __builtin_fmaf(row_scale<N>(alpha, j), sum[m], bias[j]);
            gate[m] = sigmoid(l[m]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gate[0]), i));
            if (lane / L == k) hp[i] = v;
        }
        if (first == 0) {  // the token's first wave
            if (lane == 0) rms[t] = r;
            if (lane >= N && lane < 2 * N) h[N * t + lane - N] = 2.0f * gate[0];
#pragma unroll
            for (int m = 0; m < J; ++m) {
                const int j = 64 * m + lane;
                if (j < R) Q[R * t + j] = sum[m];
                if (j >= 2 * N && j < R) H[N * N * t + j - 2 * N] = l[m];
            }
        }
    }
    if (col < nc && tok < B) {
        float u[E];
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v[E];
            unpack_chunk<DX>(x[i], v);
#pragma unroll
            for (int e = 0; e < E; ++e) u[e] = __builtin_fmaf(hp[i], v[e], u[e]);
        }
        U[nc * tok + col] = pack_chunk<DX>(u);
    }
}

// ---------------------------------------------------------------------------
// Backward: <dU, X_i> and the coefficients' gradients
// ---------------------------------------------------------------------------
// Tokens are padded to whole stages of 32 (Bp), whose G, h^pre and s are zero, for the products
// below. `share` waves of the block take four consecutive tokens, one after the other, sharing
// their columns; the first of these waves forms G. A block leaves one row of sums for dbias and
// dalpha. Bound: HBM; many short blocks that cover whole tokens stream best (2^15 tokens of 4 x 4096
// bf16 218 us, 6.2 TB/s; a resident grid that loops 254, a wave per token 236).
constexpr int kTokenStep = 32;  // tokens of a stage of the products over tokens
constexpr int kHalf = 16;
constexpr int kDotWaves = 8;

template <int DX, int N>
__device__ __forceinline__ float add_dot(const v4u a, const v4u b, float acc) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DX == BIRKHOFF4_BF16)  // products of bf16 values are exact in fp32
            acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, static_cast<uint32_t>(a[k])),
                                                  __builtin_bit_cast(bf16x2, static_cast<uint32_t>(b[k])), acc, false);
        else
            acc = __builtin_fmaf(__uint_as_float(a[k]), __uint_as_float(b[k]), acc);
    }
    return acc;
}

__device__ __forceinline__ float wave_sum(float x) {
    x = rest_sum<4>(x);
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A stage of G in the operands' layouts, with the tokens' h^pre and s: written by pre_dot_kernel,
// copied to LDS as it is by pre_back_kernel. bf16: G as the sum of three bf16 values, which hold all
// 24 bits of it, so that the products are those of fp32: 0.07 % of dW's values are not the exact result
// rounded to bf16 (2^15 tokens of 4 x 4096; torch's fp32 products 0.2 %), with two (2^-16 of G) it was 0.45 %.
// It costs 1 % of an autograd step there, 3 % of one of 8 K tokens of 8 x 4096.
// Operand rows past the last row of W are zeros.
template <int DX, int N>
struct Stage {
    static constexpr bool H16 = DX == BIRKHOFF4_BF16;
    static constexpr int R = Gates<N>::rows, RT = Gates<N>::tiles, KS = H16 ? Gates<N>::ksteps : R / 4;
    static constexpr int parts = H16 ? 3 : 1;  // bf16 values of one of G
    static constexpr int rows = H16 ? 32 * KS : 16 * RT;  // rows that have a place
    // n = 8: the last step has 16 rows, so that two parts fit one operand of 32 (and the third one with zeros)
    static constexpr bool paired = H16 && R % 32 == 16;
    using T = std::conditional_t<H16, uint16_t, float>;
    static constexpr int KE = H16 ? 8 : KS;  // values per lane of a dX operand
    static constexpr int KO = H16 ? parts * KS - paired : 1;  // dX operands per half
    alignas(16) T w[parts][RT][2][64][4];  // dW: lane (g, j): row j's tokens 4 g .. + 3 of each half
    alignas(16) T x[2][KO][64][KE];        // dX: by halves; lane (g, t): token t's rows of the operand's group g
    alignas(16) float coef[N + 1][kTokenStep];

    // Place among a half's groups of dX operands (four to an operand) of rows 8 octet .. + 7 of a part.
    static __device__ __forceinline__ int group(int part, int octet) {
        if (paired && octet >= 4 * (KS - 1)) return 4 * parts * (KS - 1) + 2 * part + octet - 4 * (KS - 1);
        return 4 * (parts * (octet >> 2) + part) + (octet & 3);
    }
};

// fp32 values as three bf16 ones each, by truncation: the upper eight bits of the significand (no
// rounding, so a large value does not overflow), the next eight and the last eight. Exact, but for
// what lies below fp32's smallest normal value; nothing past the first where it is not finite.
template <int NV>
__device__ __forceinline__ void split_bf16(const float (&v)[NV], uint32_t (&p)[3][NV / 2]) {
    float rest[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) rest[k] = v[k];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
#pragma unroll
        for (int k = 0; k < NV / 2; ++k)
            p[q][k] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * k + 1]), __float_as_uint(rest[2 * k]), 0x07060302u);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const float up = __uint_as_float(__float_as_uint(rest[k]) & 0xffff0000u);
            rest[k] = __builtin_fabsf(rest[k]) < __builtin_inff() ? rest[k] - up : 0.f;
        }
    }
}

// Four tokens' rows (G, then h^pre and s) from a wave's LDS to their places in the stage, in pieces
// of 8 and 16 bytes that lie together (single values written as they come cost 45 of 280 us at
// 2^15 tokens of 4 x 4096). t: the first of them in the stage.
template <int DX, int N, int LEN>
__device__ __forceinline__ void store_stage(Stage<DX, N>& to, const float (&row)[4][LEN], int t, int lane) {
    using St = Stage<DX, N>;
    const int half = t >> 4, g = (t >> 2) & 3;
    for (int j = lane; j < 16 * St::RT; j += 64) {
        const float v[4] = {row[0][j], row[1][j], row[2][j], row[3][j]};
        const int at = 16 * g + (j & 15);
        if constexpr (St::H16) {
            uint32_t p[St::parts][2];
            split_bf16<4>(v, p);
#pragma unroll
            for (int q = 0; q < St::parts; ++q)
                *reinterpret_cast<uint2*>(to.w[q][j >> 4][half][at]) = uint2{p[q][0], p[q][1]};
        } else {
            *reinterpret_cast<v4f*>(to.w[0][j >> 4][half][at]) = v4f{v[0], v[1], v[2], v[3]};
        }
    }
    if constexpr (St::H16) {
        const int k = lane & 3, j8 = lane >> 2;
        if (j8 < St::rows / 8) {
            float v[8];
            uint32_t p[St::parts][4];
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = row[k][8 * j8 + q];
            split_bf16<8>(v, p);
            auto put = [&](int group, int q) {
                *reinterpret_cast<v4u*>(to.x[half][group >> 2][16 * (group & 3) + (t & 15) + k]) =
                    v4u{p[q][0], p[q][1], p[q][2], p[q][3]};
            };
            if (St::paired && 8 * j8 >= St::R) {  // the last operand's two groups of zeros
                put(4 * St::KO - 2 + (j8 & 1), 0);
            } else {
#pragma unroll
                for (int q = 0; q < St::parts; ++q) put(St::group(q, j8), q);
            }
        }
    } else {
        for (int q = lane; q < 2 * St::R; q += 64) {  // pairs of rows
            const int k = q / (St::R / 2), j = 2 * (q % (St::R / 2));
            *reinterpret_cast<f32x2*>(&to.x[half][0][16 * (j / St::KS) + (t & 15) + k][j % St::KS]) =
                f32x2{row[k][j], row[k][j + 1]};
        }
    }
    if (lane <= N) {
        const int j = St::rows + lane;
        *reinterpret_cast<v4f*>(&to.coef[lane][t]) = v4f{row[0][j], row[1][j], row[2][j], row[3][j]};
    }
}

template <int DX, int N>
__global__ __launch_bounds__(64 * kDotWaves) void pre_dot_kernel(
    const v4u* __restrict__ X, const v4u* __restrict__ dU, const float* __restrict__ Q, const float* __restrict__ rms,
    const float* __restrict__ alpha, const float* __restrict__ bias, const float* __restrict__ dh,
    const float* __restrict__ dH, Stage<DX, N>* __restrict__ G, float* __restrict__ sums, int64_t B, int64_t Bp, int64_t nc, float inv_k, int share) {
    constexpr int R = Gates<N>::rows, S = Gates<N>::stride, P = Stage<DX, N>::rows, J = (P + 63) / 64;
    __shared__ float dots[kDotWaves][N];
    __shared__ float total[kDotWaves][S];
    __shared__ float row[kDotWaves][4][P + N + 1];
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int per = kDotWaves / share, sub = w / share, part = w % share;  // share: a power of two
    float sum_dl[J], sum_dq[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < J; ++m) sum_dl[m] = 0.f;
    const int64_t t0 = 4 * (static_cast<int64_t>(blockIdx.x) * per + sub);
    for (int k = 0; k < 4; ++k) {
        const int64_t t = t0 + k;
        float d[N], out[1];
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = 0.f;
        if (dU && t < B) {  // uniform over the wave
            for (int64_t col = 64 * part + lane; col < nc; col += 64 * share) {
                const v4u u = dU[nc * t + col];
                v4u x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = __builtin_nontemporal_load(X + (nc * (N * t + i) + col));
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = add_dot<DX, N>(u, x[i], d[i]);
            }
        }
        lane_sums<32, N>(d, out, lane);
        float dot = rest_sum<N>(out[0]);  // lane: value lane N / 64
        if (share > 1) {  // uniform over the block
            if (lane % (64 / N) == 0) dots[w][lane / (64 / N)] = dot;
            __syncthreads();
            if (part == 0) {
                dot = dots[w][lane / (64 / N)];
                for (int q = 1; q < share; ++q) dot += dots[w + q][lane / (64 / N)];
            }
            __syncthreads();
        }
        if (part == 0) {
            // lane j < N takes <dU, X_j>
            dot = __int_as_float(
                __builtin_amdgcn_ds_bpermute(4 * (lane < N ? lane * (64 / N) : 0), __float_as_int(dot)));
            const float r = t < B ? rms[t] : 0.f;
            float s = 0.f;
#pragma unroll
            for (int m = 0; m < J; ++m) {
                const int j = 64 * m + lane;
                if (j >= P) continue;
                float dl = 0.f, q = 0.f, gate = 0.f;
                const float a = row_scale<N>(alpha, j);
                if (t < B && j < R) {
                    q = Q[R * t + j];
                    if (j < 2 * N) {
                        gate = sigmoid(__builtin_fmaf(a, q, bias[j]));
                        const float up = j < N ? dot : dh ? 2.0f * dh[N * t + j - N] : 0.f;
                        dl = up * gate * (1.0f - gate);
                    } else if (dH) {
                        dl = dH[N * N * t + j - 2 * N];
                    }
                }
                const float gj = r * a * dl, dq = dl * q;
                s = __builtin_fmaf(gj, q, s);
                row[w][k][j] = gj;
                if (j < N) row[w][k][P + j] = gate;
                sum_dl[m] += dl;
                sum_dq[0] += j < N ? dq : 0.f;
                sum_dq[1] += j >= N && j < 2 * N ? dq : 0.f;
                sum_dq[2] += j >= 2 * N ? dq : 0.f;
            }
            s = wave_sum(s);
            if (lane == 0) row[w][k][P + N] = s * r * inv_k;
        }
    }
    __builtin_amdgcn_wave_barrier();  // lanes read what others of the wave have written
    if (part == 0 && t0 < Bp) store_stage<DX, N>(G[t0 / kTokenStep], row[w], static_cast<int>(t0 % kTokenStep), lane);
    // a row of sums for the block: dl's, then the three groups' dl q
#pragma unroll
    for (int m = 0; m < J; ++m)
        if (64 * m + lane < R) total[w][64 * m + lane] = sum_dl[m];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const float v = wave_sum(sum_dq[q]);
        if (lane == 0) total[w][R + q] = v;
    }
    if (lane == 0) total[w][R + 3] = 0.f;
    __syncthreads();
    for (int j = threadIdx.x; j < S; j += 64 * kDotWaves) {
        float v = 0.f;
        for (int q = 0; q < kDotWaves; q += share) v += total[q][j];
        sums[static_cast<int64_t>(blockIdx.x) * S + j] = v;
    }
}

// ---------------------------------------------------------------------------
// Backward: dX and partial sums of dW
// ---------------------------------------------------------------------------
// A wave takes CW channels of a stream, CE of them per lane (lane l: group g = l / 16, channels CE
// (l % 16) .. + CE), over the stages of 32 tokens of its share, in halves of 16 of which lane group g
// has tokens 4 g .. 4 g + 3. The same registers serve everything:
//  * dW: tile of 16 rows of W (G transposed, tokens along k) times the tokens' values, one product
//    per channel c of the lanes: column l % 16 is channel CE (l % 16) + c, and k runs over the
//    stage's tokens as the lanes hold them, four of each half.
//  * dX: the rows of a product are the half's tokens, so that row 4 g + i, which lane group g gets,
//    is the token whose values it holds.
// W and X are exact in bf16, sums are fp32. W's rows stay in LDS or registers throughout; a stage of
// G is copied to LDS once for all waves of a block, a stage ahead, and a half's streams are loaded
// while the other half is worked on.
//
// Bound: HBM, by the width of the rows' pieces. A copy (two arrays read, one written) by waves that
// take 128, 256 or 512 bytes of each row reaches 5.0, 5.5 and 6.5 TB/s here, so a block's waves take
// neighbouring pieces, 512 bytes together, of one or two streams: 2^15 tokens of 4 x 4096 bf16 648 -> 578 us,
// 2^13 of 8 x 4096 388 -> 350 (with G as three bf16 values instead of two 596, 5.9 TB/s, and 370, 4.7 TB/s).
// Loading a whole stage ahead (n = 4 with 128-byte pieces, 681 us) or leaving the offsets' arithmetic out
// of the loop (664) did not help.
template <int DX, int N>
struct Back {
    // n = 8: half as many channels, as the sums of 5 row tiles fill the registers
    static constexpr int CE = (DX == BIRKHOFF4_BF16 ? 8 : 4) / (N == 8 ? 2 : 1);
    static constexpr int CW = 16 * CE;
    static constexpr int words = CE * (DX == BIRKHOFF4_BF16 ? 2 : 4) / 4;  // of a lane's channels
};

template <int WORDS>
struct Words {
    uint32_t v[WORDS];
};

// ONCE: a byte that no other wave reads (non-temporal).
template <int WORDS, bool ONCE = false, typename I>
__device__ __forceinline__ Words<WORDS> load_words(const void* base, I byte) {
    typedef uint32_t vec __attribute__((ext_vector_type(WORDS)));
    const vec* p = reinterpret_cast<const vec*>(static_cast<const char*>(base) + byte);
    const vec q = ONCE ? __builtin_nontemporal_load(p) : *p;
    Words<WORDS> r;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) r.v[k] = q[k];
    return r;
}

template <int WORDS, typename I>
__device__ __forceinline__ void store_words(void* base, I byte, const Words<WORDS>& r) {
    typedef uint32_t vec __attribute__((ext_vector_type(WORDS)));
    vec q;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) q[k] = r.v[k];
    __builtin_nontemporal_store(q, reinterpret_cast<vec*>(static_cast<char*>(base) + byte));
}

// Channel c of a lane's words.
template <int DX, int WORDS>
__device__ __forceinline__ float channel(const Words<WORDS>& r, int c) {
    if constexpr (DX == BIRKHOFF4_BF16)
        return __uint_as_float(c & 1 ? r.v[c / 2] & 0xffff0000u : r.v[c / 2] << 16);
    else
        return __uint_as_float(r.v[c]);
}

// bf16 channel c of two (eight) rows, in order.
template <int WORDS>
__device__ __forceinline__ uint32_t column_pair(const Words<WORDS>& a, const Words<WORDS>& b, int c) {
    // selector bytes 0..3: second operand, 4..7: first
    return __builtin_amdgcn_perm(b.v[c / 2], a.v[c / 2], c & 1 ? 0x07060302u : 0x05040100u);
}

template <int WORDS>
__device__ __forceinline__ v4u column8(const Words<WORDS> r[8], int c) {
    return v4u{column_pair(r[0], r[1], c), column_pair(r[2], r[3], c), column_pair(r[4], r[5], c),
               column_pair(r[6], r[7], c)};
}

typedef uint32_t v2u __attribute__((ext_vector_type(2)));

// W's rows in the dX products' layout are in LDS, or, where they would leave a CU one block (fp32
// with n = 8), in registers.
template <int DX, int N>
struct BackPlan {
    static constexpr bool H16 = DX == BIRKHOFF4_BF16;
    static constexpr bool w_lds = H16 || N == 4;
    static constexpr int waves = 4;  // of a block
    static constexpr int adj = 512 / (Back<DX, N>::CW * (H16 ? 2 : 4));  // neighbouring chunks of a stream in it
    static constexpr int stages = H16 && N == 8 ? 1 : 2;  // of G in LDS
};

template <int DX, int N>
__global__ __launch_bounds__((64 * BackPlan<DX, N>::waves), 2) void pre_back_kernel(
    const void* __restrict__ X, const void* __restrict__ W, const void* __restrict__ dU, const void* __restrict__ E,
    const Stage<DX, N>* __restrict__ G, void* __restrict__ dX, float* __restrict__ dWp, int64_t B, int64_t stages,
    int64_t C, uint32_t cols, uint32_t shares, uint32_t per_xcd) {
    using St = Stage<DX, N>;
    constexpr bool H16 = St::H16;
    constexpr int R = St::R, RT = St::RT, KS = St::KS;
    constexpr int CE = Back<DX, N>::CE, WO = Back<DX, N>::words, SZ = H16 ? 2 : 4;
    constexpr int NW = BackPlan<DX, N>::waves, NS = BackPlan<DX, N>::stages;
    constexpr int kThreads = 64 * NW, kQuads = sizeof(St) / 16, GQ = (kQuads + kThreads - 1) / kThreads;
    static_assert(sizeof(St) % 16 == 0, "copied in 16-byte pieces");
    constexpr bool kLds = BackPlan<DX, N>::w_lds;
    using Row = Words<WO>;
    __shared__ St lds[NS];
    // [channel][four lane groups an operand][lane of the group]: of bf16 eight rows, of fp32 one
    constexpr int WG = 4 * KS - 2 * St::paired;
    __shared__ std::conditional_t<H16, v4u, float> wlds[kLds ? NW : 1][kLds ? CE : 1][WG][16];
    const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
    const int ww = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    constexpr int ADJ = BackPlan<DX, N>::adj;
    // an XCD's blocks are neighbours, streams first (which share dU), then pieces of the row, then shares
    // of the tokens, whose part of G its L2 holds: backward of 4096 tokens of 4 x 4096 bf16 131 -> 121 us
    constexpr uint32_t kSets = N * ADJ / NW;  // blocks over the streams
    const uint32_t place = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3), share = place / (kSets * cols);
    if (share >= shares) return;  // the whole block
    const int w = static_cast<int>(place % kSets) * (NW / ADJ) + ww / ADJ;  // the stream
    const int64_t ch = (static_cast<int64_t>(place / kSets % cols) * ADJ + ww % ADJ) * Back<DX, N>::CW + CE * c16;
    const bool own = ch < C;
    const int64_t at = own ? ch : 0;  // lanes past the end of the row read its start and store nothing
    const int64_t K = N * C;

    v4u gq[GQ];
    auto fetch = [&](int64_t st) {
#pragma unroll
        for (int q = 0; q < GQ; ++q) {
            const int k = static_cast<int>(threadIdx.x) + kThreads * q;
            if (k < kQuads) gq[q] = reinterpret_cast<const v4u*>(G + st)[k];
        }
    };
    auto put = [&](St& to) {
#pragma unroll
        for (int q = 0; q < GQ; ++q) {
            const int k = static_cast<int>(threadIdx.x) + kThreads * q;
            if (k < kQuads) reinterpret_cast<v4u*>(&to)[k] = gq[q];
        }
    };
    // a half's rows start at a uniform address, the lane's four at 32-bit offsets from it; past the
    // last token: that token again
    auto rows_of = [&](int64_t t0, uint32_t off[4], int64_t stride) {
        const int last = B - t0 < kHalf ? static_cast<int>(B - t0) - 1 : kHalf - 1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            off[k] = static_cast<uint32_t>(4 * g + k < last ? 4 * g + k : last) * static_cast<uint32_t>(stride * SZ) +
                     static_cast<uint32_t>(at * SZ);
    };
    auto load_x = [&](Row (&x)[4], int64_t t0) {
        uint32_t off[4];
        rows_of(t0, off, K);
        const char* base = static_cast<const char*>(X) + (K * t0 + w * C) * SZ;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = load_words<WO, true>(base, off[k]);
    };
    auto load_eu = [&](Row (&e)[4], Row (&u)[4], int64_t t0) {
        uint32_t off[4];
        if (E) {
            rows_of(t0, off, K);
            const char* base = static_cast<const char*>(E) + (K * t0 + w * C) * SZ;
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = load_words<WO, true>(base, off[k]);
        }
        if (dU) {
            rows_of(t0, off, C);
            const char* base = static_cast<const char*>(dU) + C * t0 * SZ;
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = load_words<WO>(base, off[k]);
        }
    };

    int64_t st = share;
    fetch(st);
    Row x[2][4] = {}, e[2][4] = {}, u[2][4] = {};
    // a stage has two halves also where the last one is past the end
    auto load = [&](int hf, int64_t t0) {
        if (t0 >= B) return;  // uniform
        load_x(x[hf], t0);
        load_eu(e[hf], u[hf], t0);
    };
    load(0, st * kTokenStep);
    load(1, st * kTokenStep + kHalf);

    // W's rows: operand of the dX products, for each channel c of the lane
    std::conditional_t<H16, v4u, float> wreg[kLds ? 1 : KS][CE];
    // the lane's group of operand k: where two parts of G share it, both halves of the lanes have the same rows
    auto group = [&](int k) { return St::paired && k == KS - 1 ? g & 1 : g; };
    auto keep = [&](int k, int c, auto v) {
        if constexpr (kLds)
            wlds[ww][c][4 * k + group(k)][c16] = v;
        else
            wreg[k][c] = v;
    };
    auto wop = [&](int k, int c) {
        if constexpr (kLds)
            return wlds[ww][c][4 * k + group(k)][c16];
        else
            return wreg[k][c];
    };
    if constexpr (H16) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            Words<WO> rows[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {  // past the last row: that row, which meets zeros of G
                const int row = 32 * k + 8 * group(k) + j;
                rows[j] = load_words<WO>(W, (K * (row < R ? row : R - 1) + w * C + at) * SZ);
            }
#pragma unroll
            for (int c = 0; c < CE; ++c) keep(k, c, column8<WO>(rows, c));
        }
    } else {
#pragma unroll
        for (int k = 0; k < KS; ++k) {  // lane group g has rows g R / 4 ..
            const Words<WO> row = load_words<WO>(W, (K * (g * KS + k) + w * C + at) * SZ);
#pragma unroll
            for (int c = 0; c < CE; ++c) keep(k, c, __uint_as_float(row.v[c]));
        }
    }
    v4f acc[RT][CE];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CE; ++c) acc[r][c] = v4f{0.f, 0.f, 0.f, 0.f};

    // dW += G^T X
    auto sum_w = [&](const St& s) {
        if constexpr (H16) {
            v4u b[CE];
#pragma unroll
            for (int c = 0; c < CE; ++c)
                b[c] = v4u{column_pair(x[0][0], x[0][1], c), column_pair(x[0][2], x[0][3], c),
                           column_pair(x[1][0], x[1][1], c), column_pair(x[1][2], x[1][3], c)};
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int p = 0; p < St::parts; ++p) {
                    const v2u a0 = *reinterpret_cast<const v2u*>(s.w[p][r][0][lane]);
                    const v2u a1 = *reinterpret_cast<const v2u*>(s.w[p][r][1][lane]);
                    const v4u a = {a0.x, a0.y, a1.x, a1.y};
#pragma unroll
                    for (int c = 0; c < CE; ++c) acc[r][c] = mfma_bf16(a, b[c], acc[r][c]);
                }
        } else {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const v4f gr = *reinterpret_cast<const v4f*>(s.w[0][r][hf][lane]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int c = 0; c < CE; ++c)
                            acc[r][c] = mfma_f32(gr[k], __uint_as_float(x[hf][k].v[c]), acc[r][c]);
                }
        }
    };
    auto work = [&](Row (&x)[4], Row (&e)[4], Row (&u)[4], const St& s, int hf, int64_t t0) {
        if (t0 >= B) return;  // uniform
        // dX = E + h^pre dU + G W - s X
        v4f d[CE];
#pragma unroll
        for (int c = 0; c < CE; ++c) d[c] = v4f{0.f, 0.f, 0.f, 0.f};
        if constexpr (H16) {
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                constexpr int NP = St::parts;
                const int np = St::paired && k == KS - 1 ? NP - 1 : NP;
                v4u a[NP];
#pragma unroll
                for (int p = 0; p < np; ++p) a[p] = *reinterpret_cast<const v4u*>(s.x[hf][NP * k + p][lane]);
#pragma unroll
                for (int c = 0; c < CE; ++c) {
                    const v4u b = wop(k, c);
#pragma unroll
                    for (int p = 0; p < np; ++p) d[c] = mfma_bf16(a[p], b, d[c]);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int c = 0; c < CE; ++c) d[c] = mfma_f32(s.x[hf][0][lane][k], wop(k, c), d[c]);
        }
        uint32_t off[4];
        rows_of(t0, off, K);
        char* out = static_cast<char*>(dX) + (K * t0 + w * C) * SZ;
        const v4f hp = *reinterpret_cast<const v4f*>(&s.coef[w][kHalf * hf + 4 * g]);
        const v4f sv = *reinterpret_cast<const v4f*>(&s.coef[N][kHalf * hf + 4 * g]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float o[CE];
#pragma unroll
            for (int c = 0; c < CE; ++c) {
                o[c] = __builtin_fmaf(hp[k], channel<DX, WO>(u[k], c), channel<DX, WO>(e[k], c) + d[c][k]);
                o[c] = __builtin_fmaf(-sv[k], channel<DX, WO>(x[k], c), o[c]);
            }
            Words<WO> r;
#pragma unroll
            for (int q = 0; q < WO; ++q) {
                if constexpr (H16)
                    r.v[q] = pack_bf16(o[2 * q], o[2 * q + 1]);
                else
                    r.v[q] = __float_as_uint(o[q]);
            }
            if (own && t0 + 4 * g + k < B) store_words<WO>(out, off[k], r);
        }
    };

    put(lds[0]);
    for (int cur = 0; st < stages; cur ^= NS - 1) {
        const int64_t t0 = st * kTokenStep;
        st += shares;
        const bool more = st < stages;  // uniform over the block
        __syncthreads();                // this stage's G is there, and nobody reads the other's any more
        if (more) fetch(st);
        if (t0 + kTokenStep > B) {  // tokens past the last one add nothing to dW: zeros, as 0 times their G
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (t0 + kHalf * hf + 4 * g + k >= B) x[hf][k] = Row{};
        }
        sum_w(lds[cur]);
        work(x[0], e[0], u[0], lds[cur], 0, t0);
        if (more) load(0, st * kTokenStep);
        work(x[1], e[1], u[1], lds[cur], 1, t0 + kHalf);
        if (more) {
            load(1, st * kTokenStep + kHalf);
            if constexpr (NS == 1) __syncthreads();
            put(lds[NS == 2 ? cur ^ 1 : 0]);
        }
    }
    if (own) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 16 * r + 4 * g + i;
                if (j >= R) continue;
                v4f* p = reinterpret_cast<v4f*>(dWp + (static_cast<int64_t>(share) * R + j) * K + w * C + ch);
                if constexpr (CE == 2) {
                    *reinterpret_cast<f32x2*>(p) = f32x2{acc[r][0][i], acc[r][1][i]};
                } else {
#pragma unroll
                    for (int q = 0; q < CE / 4; ++q)
                        p[q] = v4f{acc[r][4 * q][i], acc[r][4 * q + 1][i], acc[r][4 * q + 2][i], acc[r][4 * q + 3][i]};
                }
            }
    }
}

// The shares' sums added in a fixed order: dW, four threads to 16 bytes of the fp32 sums, and in the
// grid's last blocks dbias and dalpha, sixteen entries a block.
constexpr int kJoinBlock = 1024;
constexpr int kJoinQuads = kJoinBlock / 4;

template <int N, bool DW16>
__global__ __launch_bounds__(kJoinBlock) void pre_join_kernel(const v4f* __restrict__ dWp, const float* __restrict__ sums,
                                                              void* __restrict__ dW, float* __restrict__ dalpha,
                                                              float* __restrict__ dbias, int64_t quads, int shares,
                                                              int64_t rows, unsigned wblocks) {
    constexpr int R = Gates<N>::rows, S = Gates<N>::stride;
    if (blockIdx.x < wblocks) {
        __shared__ v4f quarter[3][kJoinQuads];
        const int own = threadIdx.x % kJoinQuads, part = threadIdx.x / kJoinQuads;
        for (int64_t base = static_cast<int64_t>(blockIdx.x) * kJoinQuads; base < quads;
             base += static_cast<int64_t>(wblocks) * kJoinQuads) {  // uniform over the block
            const int64_t q = base + own;
            v4f v = {0.f, 0.f, 0.f, 0.f};
            if (q < quads) {
#pragma unroll 4
                for (int k = part; k < shares; k += 4) v += dWp[k * quads + q];
            }
            if (part > 0) quarter[part - 1][own] = v;
            __syncthreads();
            if (part == 0 && q < quads) {
                v = (v + quarter[0][own]) + (quarter[1][own] + quarter[2][own]);
                if constexpr (DW16)
                    static_cast<uint2*>(dW)[q] = uint2{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
                else
                    static_cast<v4f*>(dW)[q] = v;
            }
            __syncthreads();
        }
        return;
    }
    __shared__ float red[kJoinBlock / 16][16];
    const int c = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int j = 16 * static_cast<int>(blockIdx.x - wblocks) + c;
    float v = 0.f;
    if (j < S)
#pragma unroll 16
        for (int64_t k = part; k < rows; k += kJoinBlock / 16) v += sums[k * S + j];
    red[part][c] = v;
    __syncthreads();
    if (part == 0) {
        v = red[0][c];
        for (int k = 1; k < kJoinBlock / 16; ++k) v += red[k][c];
        if (j < R)
            dbias[j] = v;
        else if (j < R + 3)
            dalpha[j - R] = v;
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct PreShape {
    int64_t B, C, nc, steps;  // nc: 16-byte chunks of a stream's row; steps: 64 bytes of a token
};

struct GateLaunch {
    bool wide;                   // pre_gate_wide_kernel (n = 8)
    int tt, waves;               // 16-token tiles and waves of a block
    int64_t tiles, splits, per;  // blocks over tokens, shares of the row, steps per share
};

// Tokens of a block and its waves, and shares of the row, us of the whole forward:
//  * up to 16 tokens one tile and 16 waves: 1 token of 4 x 4096 bf16 8.1, of 8 x 4096 13.7.
//  * n = 4 up to 512 two tiles and 16 waves: 96 tokens of 4 x 4096 11.4, four tiles and 4 waves 11.8; 300
//    14.3 and 15.6; 600 19.3 and 18.6, 1000 of 4 x 1024 12.5 and 14.1. n = 8 up to 64 two tiles and 8 waves
//    (more do not fit the registers): 32 tokens of 8 x 4096 17.0, four tiles 18.4; 64 17.3 and 19.2; 100 of
//    8 x 2048 15.7 and 16.8, 600 of 8 x 4096 47 and 33.5.
//  * else four tiles, each row of W read once for 64 tokens, and 4 waves: 16 K tokens of 4 x 4096
//    190 (two tiles 213), 2^15 384 (430), 1023 of 8 x 4096 40 (49).
//  * shares until 2048 waves (4097 tokens of 4 x 1000 fp32 45.0; 4096 waves 47.6), each wave with a
//    whole line of every token at least; at most 16, as each costs a read of the sums (600 tokens of 8 x
//    4096 33.9, with 32 37.3; 1023 of 8 x 2052 fp32 61.7 and 73.3), 32 where there are few blocks
//    (32 tokens of 8 x 4096 16.9, with 16 28).
constexpr int64_t kGateWant = 2048;

template <int N>
constexpr int gate_waves(int tiles) { return tiles == 1 ? 16 : tiles == 2 ? (N == 4 ? 16 : 8) : 4; }

GateLaunch gate_launch(const PreShape& s, int n) {
    GateLaunch l;
    l.wide = n == 8 && s.B > 2048;
    l.tt = s.B <= 16 ? 1 : s.B <= (n == 4 ? 512 : 64) ? 2 : 4;
    l.waves = n == 4 ? gate_waves<4>(l.tt) : gate_waves<8>(l.tt);
    int64_t lines = l.waves;  // at least, of a share
    if (l.wide) {
        l.waves = kGateWideWaves;
        l.tt *= l.waves;
        lines = 4;
    }
    l.tiles = cdiv(s.B, 16 * l.tt);
    const int64_t most = cdiv(s.steps, 2 * lines), cap = l.tiles <= 4 ? 32 : 16;
    int64_t want = cdiv(kGateWant, l.waves * l.tiles);
    if (want > most) want = most;
    if (want > cap) want = cap;
    l.per = 2 * cdiv(cdiv(s.steps, want), 2);
    l.splits = cdiv(s.steps, l.per);
    return l;
}

struct BackLaunch {
    int64_t Bp;                    // tokens in whole steps
    int share;                     // of pre_dot_kernel
    int64_t dot_blocks;
    int64_t chunks, token_shares;  // of pre_back_kernel
    int64_t g, sums, dw, bytes;  // the workspace's parts: offsets in bytes, and its size
};

constexpr int64_t kBackWaves = 2048;  // two per SIMD

BackLaunch back_launch(const PreShape& s, int n, bool bf16) {
    BackLaunch l;
    const int64_t rows = n * n + 2 * n;
    constexpr int F = BIRKHOFF4_F32, S = BIRKHOFF4_BF16;
    const int64_t stage_bytes = n == 4 ? (bf16 ? sizeof(Stage<S, 4>) : sizeof(Stage<F, 4>))
                                       : (bf16 ? sizeof(Stage<S, 8>) : sizeof(Stage<F, 8>));
    l.Bp = cdiv(s.B, kTokenStep) * kTokenStep;
    l.share = 1;
    while (l.share < kDotWaves && l.share < cdiv(s.nc, 64)) l.share *= 2;
    l.dot_blocks = cdiv(l.Bp / 4, kDotWaves / l.share);
    const int cw = n == 4 ? (bf16 ? Back<S, 4>::CW : Back<F, 4>::CW) : (bf16 ? Back<S, 8>::CW : Back<F, 8>::CW);
    l.chunks = cdiv(s.C, cw);
    const int64_t steps = l.Bp / kTokenStep;
    int64_t shares = kBackWaves / (n * l.chunks);
    if (shares < 1) shares = 1;
    if (shares > steps) shares = steps;
    // the fewest shares whose longest is no longer
    l.token_shares = steps ? cdiv(steps, cdiv(steps, shares)) : 0;
    int64_t at = 0;
    auto take = [&](int64_t floats) {
        const int64_t was = at;
        at += cdiv(4 * floats, 256) * 256;
        return was;
    };
    l.g = take(l.Bp / kTokenStep * (stage_bytes / 4));
    l.sums = take(l.dot_blocks * (rows + 4));
    l.dw = take(l.token_shares * rows * n * s.C);
    l.bytes = at;
    return l;
}

// The dot kernel has 16 lanes a token up to 64 chunks of a row and 128 at most (above 256 chunks, of
// which memory does not hold 2^25 tokens): below a launch's 2^32 lanes. The read splits its grid.
constexpr int64_t kPreMaxTokens = int64_t(1) << 26;
constexpr int64_t kMaxLanes = int64_t(1) << 31;  // along one dimension of a grid
constexpr int64_t kPreMaxValues = int64_t(1) << 46;
constexpr int64_t kPreMaxChannels = int64_t(1) << 20;  // 64 tokens lie within 32-bit offsets

// The checks that both directions and the workspace's size share.
int pre_shape(int n, int64_t B, int64_t C, int x_dtype, PreShape* s) {
    if (B < 0 || B > kPreMaxTokens) return BIRKHOFF4_ERR_SIZE;
    if (!dtype_ok(x_dtype)) return BIRKHOFF4_ERR_DTYPE;
    const int64_t e = x_dtype == BIRKHOFF4_BF16 ? 8 : 4;
    if (C <= 0 || C % e != 0) return BIRKHOFF4_ERR_CHANNELS;
    if (C > kPreMaxChannels || (B > 0 && n * C > kPreMaxValues / B)) return BIRKHOFF4_ERR_SIZE;
    *s = {B, C, C / e, n * (C / e) / 4};
    return BIRKHOFF4_OK;
}

bool eps_ok(float eps) { return eps >= 0.f && eps < __builtin_inff(); }

template <int DX, int N>
int launch_pre_fwd(const PreShape& s, const void* X, const void* W, const float* alpha, const float* bias, float eps,
                   void* U, float* h, float* H, float* q, float* rms, float* part, hipStream_t stream) {
    const GateLaunch l = gate_launch(s, N);
    const v4u *x = static_cast<const v4u*>(X), *w = static_cast<const v4u*>(W);
    auto gate = l.tt == 1   ? pre_gate_kernel<DX, N, 1, gate_waves<N>(1)>
                : l.tt == 2 ? pre_gate_kernel<DX, N, 2, gate_waves<N>(2)> : pre_gate_kernel<DX, N, 4, gate_waves<N>(4)>;
    if constexpr (N == 8)
        if (l.wide) gate = pre_gate_wide_kernel<DX>;
    const uint32_t tiles = static_cast<uint32_t>(l.tiles), per_xcd = static_cast<uint32_t>(cdiv(l.tiles * l.splits, 8));
    launch_kernel(gate, dim3(8 * per_xcd), dim3(64 * l.waves), 0, stream, x, w, part, s.B, s.steps, l.per, tiles,
                  per_xcd);
    const int L = s.nc <= 8 ? 8 : s.nc <= 16 ? 16 : s.nc <= 32 ? 32 : 64;
    auto read = L == 8 ? pre_read_kernel<DX, N, 8> : L == 16 ? pre_read_kernel<DX, N, 16>
                : L == 32 ? pre_read_kernel<DX, N, 32> : pre_read_kernel<DX, N, 64>;
    const int64_t cols = cdiv(s.nc, L), shares = cdiv(cols, kReadWaves), waves = cdiv(cols, shares);
    const int64_t blocks = cdiv(s.B, 64 / L), layers = cdiv(64 * waves * blocks, kMaxLanes);
    launch_kernel(read, dim3(static_cast<unsigned>(cdiv(blocks, layers)), static_cast<unsigned>(shares),
                             static_cast<unsigned>(layers)),
                  dim3(static_cast<unsigned>(64 * waves)), 0, stream, part, x, alpha, bias, eps,
                  static_cast<float>(1.0 / (static_cast<double>(N) * s.C)), static_cast<v4u*>(U), h, H, q, rms, s.B, s.nc,
                  static_cast<int>(l.splits));
    return launch_status();
}

template <int DX, int N>
int launch_pre_bwd(const PreShape& s, const void* X, const void* W, const float* alpha, const float* bias, const float* q,
                   const float* rms, const void* dU, const float* dh, const float* dH, const void* E, void* dX, void* dW,
                   float* dalpha, float* dbias, char* work, hipStream_t stream) {
    const BackLaunch l = back_launch(s, N, DX == BIRKHOFF4_BF16);
    auto at = [&](int64_t o) { return reinterpret_cast<float*>(work + o); };
    Stage<DX, N>* stage = reinterpret_cast<Stage<DX, N>*>(at(l.g));
    if (s.B > 0) {
        launch_kernel((pre_dot_kernel<DX, N>), dim3(static_cast<unsigned>(l.dot_blocks)), dim3(64 * kDotWaves), 0, stream,
                      static_cast<const v4u*>(X), static_cast<const v4u*>(dU), q, rms, alpha, bias, dh, dH, stage,
                      at(l.sums), s.B, l.Bp, s.nc,
                      static_cast<float>(1.0 / (static_cast<double>(N) * s.C)), l.share);
        using Plan = BackPlan<DX, N>;
        const uint32_t cols = static_cast<uint32_t>(cdiv(l.chunks, Plan::adj));
        const uint32_t shares = static_cast<uint32_t>(l.token_shares);
        const uint32_t per_xcd = static_cast<uint32_t>(cdiv(int64_t(N) * Plan::adj / Plan::waves * cols * shares, 8));
        launch_kernel((pre_back_kernel<DX, N>), dim3(8 * per_xcd), dim3(64 * Plan::waves), 0, stream, X, W, dU, E, stage,
                      dX, at(l.dw), s.B, l.Bp / kTokenStep, s.C, cols, shares, per_xcd);
    }
    // without tokens the sums are empty: zeros
    const int64_t quads = Gates<N>::rows * N * s.C / 4;
    const int64_t want = cdiv(quads, kJoinQuads);
    const unsigned wblocks = static_cast<unsigned>(want < 4096 ? want : 4096);
    launch_kernel((pre_join_kernel<N, DX == BIRKHOFF4_BF16>), dim3(wblocks + (Gates<N>::stride + 15) / 16),
                  dim3(kJoinBlock), 0, stream, reinterpret_cast<const v4f*>(at(l.dw)), at(l.sums), dW, dalpha, dbias,
                  quads, static_cast<int>(l.token_shares), l.dot_blocks, wblocks);
    return launch_status();
}

int64_t pre_work(int n, int64_t B, int64_t C, int x_dtype, int backward) {
    PreShape s;
    if (int e = pre_shape(n, B, C, x_dtype, &s)) return e;
    if (B == 0) return 0;
    if (backward) return back_launch(s, n, x_dtype == BIRKHOFF4_BF16).bytes;
    const GateLaunch l = gate_launch(s, n);
    return l.splits * B * (n * n + 2 * n + 4) * 4;
}

template <int N>
int pre_fwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, float eps, void* U, float* h,
            float* H, float* q, float* rms, void* work, int64_t work_bytes, int64_t B, int64_t C, hipStream_t stream) {
    PreShape s;
    if (int e = pre_shape(N, B, C, x_dtype, &s)) return e;
    if (!eps_ok(eps)) return BIRKHOFF4_ERR_EPS;
    if (B == 0) return BIRKHOFF4_OK;
    if (!X || !W || !alpha || !bias || !U || !h || !H || !q || !rms || !work) return BIRKHOFF4_ERR_NULL;
    const int64_t need = pre_work(N, B, C, x_dtype, 0);
    if (work_bytes < need) return BIRKHOFF4_ERR_WORK;
    const void* all[] = {X, W, alpha, bias, U, h, H, q, rms, work};
    for (const void* p : all)
        if (misaligned(p)) return BIRKHOFF4_ERR_ALIGN;
    const size_t row = static_cast<size_t>(C) * dtype_bytes(x_dtype), b = static_cast<size_t>(B), R = Gates<N>::rows;
    const Span ins[] = {{X, b * N * row}, {W, R * N * row}, {alpha, 12}, {bias, 4 * R}};
    const Span outs[] = {{U, b * row}, {h, b * N * 4}, {H, b * N * N * 4}, {q, b * R * 4}, {rms, b * 4},
                         {work, static_cast<size_t>(need)}};
    if (!disjoint(outs, 6, ins, 4)) return BIRKHOFF4_ERR_OVERLAP;
    auto launch = x_dtype == BIRKHOFF4_BF16 ? launch_pre_fwd<BIRKHOFF4_BF16, N> : launch_pre_fwd<BIRKHOFF4_F32, N>;
    return launch(s, X, W, alpha, bias, eps, U, h, H, q, rms, static_cast<float*>(work), stream);
}

template <int N>
int pre_bwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, const float* q,
            const float* rms, const void* dU, const float* dh, const float* dH, const void* E, void* dX, void* dW,
            float* dalpha, float* dbias, void* work, int64_t work_bytes, int64_t B, int64_t C, hipStream_t stream) {
    PreShape s;
    if (int e = pre_shape(N, B, C, x_dtype, &s)) return e;
    if (!dW || !dalpha || !dbias) return BIRKHOFF4_ERR_NULL;
    if (B > 0 && (!X || !W || !alpha || !bias || !q || !rms || !dX || !work)) return BIRKHOFF4_ERR_NULL;
    const int64_t need = pre_work(N, B, C, x_dtype, 1);
    if (work_bytes < need) return BIRKHOFF4_ERR_WORK;
    const void* all[] = {X, W, alpha, bias, q, rms, dU, dh, dH, E, dX, dW, dalpha, dbias, work};
    for (const void* p : all)
        if (misaligned(p)) return BIRKHOFF4_ERR_ALIGN;
    const size_t row = static_cast<size_t>(C) * dtype_bytes(x_dtype), b = static_cast<size_t>(B), R = Gates<N>::rows;
    const Span ins[] = {{X, b * N * row}, {W, R * N * row}, {alpha, 12}, {bias, 4 * R}, {q, b * R * 4}, {rms, b * 4},
                        {dU, b * row}, {dh, b * N * 4}, {dH, b * N * N * 4}, {E, b * N * row}};
    const Span outs[] = {{dX, b * N * row}, {dW, R * N * row}, {dalpha, 12}, {dbias, 4 * R},
                         {work, static_cast<size_t>(need)}};
    if (!disjoint(outs, 5, ins, 10)) return BIRKHOFF4_ERR_OVERLAP;
    auto launch = x_dtype == BIRKHOFF4_BF16 ? launch_pre_bwd<BIRKHOFF4_BF16, N> : launch_pre_bwd<BIRKHOFF4_F32, N>;
    return launch(s, X, W, alpha, bias, q, rms, dU, dh, dH, E, dX, dW, dalpha, dbias, static_cast<char*>(work), stream);
}

}  // namespace

extern "C" {

int64_t birkhoff4_pre_work(int64_t B, int64_t C, int x_dtype, int backward) { return pre_work(4, B, C, x_dtype, backward); }
int64_t birkhoff8_pre_work(int64_t B, int64_t C, int x_dtype, int backward) { return pre_work(8, B, C, x_dtype, backward); }

int birkhoff4_pre_fwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, float eps, void* U,
                      float* h, float* H, float* q, float* rms, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream) {
    return pre_fwd<4>(X, W, x_dtype, alpha, bias, eps, U, h, H, q, rms, work, work_bytes, B, C, stream);
}

int birkhoff8_pre_fwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, float eps, void* U,
                      float* h, float* H, float* q, float* rms, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream) {
    return pre_fwd<8>(X, W, x_dtype, alpha, bias, eps, U, h, H, q, rms, work, work_bytes, B, C, stream);
}

int birkhoff4_pre_bwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, const float* q,
                      const float* rms, const void* dU, const float* dh, const float* dH, const void* E, void* dX,
                      void* dW, float* dalpha, float* dbias, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream) {
    return pre_bwd<4>(X, W, x_dtype, alpha, bias, q, rms, dU, dh, dH, E, dX, dW, dalpha, dbias, work, work_bytes, B, C,
                      stream);
}

int birkhoff8_pre_bwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, const float* q,
                      const float* rms, const void* dU, const float* dh, const float* dH, const void* E, void* dX,
                      void* dW, float* dalpha, float* dbias, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream) {
    return pre_bwd<8>(X, W, x_dtype, alpha, bias, q, rms, dU, dh, dH, E, dX, dW, dalpha, dbias, work, work_bytes, B, C,
                      stream);
}

}  // extern "C"
