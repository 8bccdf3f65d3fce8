// orth.hip -- matrices taken towards their nearest (semi-)orthogonal ones by Newton-Schulz products, and
// the weight update with momentum around it, for gfx950 (MI355X).
//
// With m the smaller side of G and X = G / (|G|_F + eps) seen from it (m rows, n >= m columns):
//     A = X X^T,   E = b A + c A^2,   X <- a X + E X        (a, b, c of each step)
// An odd polynomial of X: it keeps the singular vectors and moves the singular values, p(s) = a s + b s^3 +
// c s^5. Every step is three products, 2 m^2 n + 2 m^3 + 2 m^2 n operations, of which the symmetric A and
// A^2 need one half: bound by the matrix cores but for small m. 4096 x 4096 in bf16 takes 1.6 ms, 0.86 PFLOP/s of
// those operations; 2560 x 10240 in fp32 (three times as many, in fp16) 3.2 ms.
//
// The products run on the matrix cores in fp16 pieces with fp32 sums. A value x is stored as 2^12 x, whose
// fp16 rounding is `hi` and the fp16 rounding of what is left `lo`: 22 bits for values above 2^-14, and
// never further off than 2^-37, for values below 16 (singular values stay below 1.3 in the usual steps).
// Results in fp32 take three products, hi hi + hi lo + lo hi: what fp32 inputs would give (relative error
// of 512 x 512 after five steps 1.4e-6, in fp32 1.3e-6). Results that are rounded to bf16 take hi hi alone,
// and what the rounding to 11 bits would spoil most is kept out of the products:
//   * a X is added from both pieces: it is what E X corrects, and the steps behind amplify its error (a
//     matrix of low rank 1.1e-2 off without that, 2e-4 with it);
//   * the diagonals D of A and F of E, the large entries, whose roundings all go one way where the singular
//     values are near to each other, are fp32 numbers of their own, and zeros in A and E as stored:
//     (A^2)_ij = (D_i + D_j) A_ij + (A A)_ij off the diagonal, D_i^2 + (A A)_ii on it, and X <- (a + F_i) X_i + (E X)_i
//     (a spread 400 x 3200 3.6e-3 off without, 0.45e-3 with them).
// What is left, 0.2e-3 to 1.1e-3, is less than the result's own rounding to bf16, 1.7e-3; of low rank it is up to 5e-3 (81 x
// 81 of rank one). More than five of the usual steps would make more of it; the first of them take two pieces
// (kMostGrowth).
//
// The products are of rows with rows (both operands have the summed index along their rows), so X is kept
// in both orders.

#include <type_traits>
#include <utility>

#include "common.h"

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v4u_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t v2u_at2 __attribute__((ext_vector_type(2), aligned(2)));

constexpr float kUnit = 4096.f;  // what values are stored in multiples of 1 / kUnit of
constexpr int kOrthMaxSteps = 64;
constexpr int kPad = 64;         // rows and columns of the stored matrices are whole multiples

// A stored matrix: panels of 64 bytes of every row, one row behind the other, so that a tile's rows of one
// panel are one piece of memory, which goes to LDS as it is. SPLIT: 16 columns' hi and then their lo;
// otherwise 32 columns' hi, and lo, where it is kept, the same way in a matrix of its own. The 16-byte piece c
// of row r lies at place c ^ (r / 4 mod 4) of its 64 bytes: sixteen lanes that read one piece of sixteen
// neighbouring rows from LDS find it in sixteen different places of its 256 bytes of banks (with r / 2, which is
// right for 128, half of the cycles of LDS were conflicts).
struct Plane {
    char* hi;
    char* lo;
    int64_t rows;    // with zeros around
    int64_t stride;  // bytes from one matrix of the batch to the next
};

constexpr int panel_cols(bool split) { return split ? 16 : 32; }

// Where the eight columns from `col` (a multiple of eight) on of a row begin; SPLIT: their lo is at that ^ 32.
template <bool SPLIT>
__device__ __forceinline__ int64_t place(const Plane& p, int64_t row, int64_t col) {
    constexpr int N = panel_cols(SPLIT);
    const int piece = static_cast<int>(col % N / 8);
    return (col / N * p.rows + row) * 64 + 16 * (piece ^ static_cast<int>(row / 4 & 3));
}

typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// Eight values as hi and lo: two conversions of a pair each, and the rest by one multiply-add of mixed types.
__device__ __forceinline__ void halves(const float v[8], h8* hi, h8* lo) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const h2 x = __builtin_convertvector((f32x2{v[e], v[e + 1]}), h2);
        const h2 y = __builtin_convertvector((f32x2{__builtin_fmaf(static_cast<float>(x[0]), -1.f, v[e]),
                                                    __builtin_fmaf(static_cast<float>(x[1]), -1.f, v[e + 1])}), h2);
        (*hi)[e] = x[0], (*hi)[e + 1] = x[1];
        (*lo)[e] = y[0], (*lo)[e + 1] = y[1];
    }
}

template <bool SPLIT>
__device__ __forceinline__ void store8(const Plane& p, int64_t matrix, int64_t row, int64_t col, const h8& hi, const h8& lo) {
    const int64_t at = matrix * p.stride + place<SPLIT>(p, row, col);
    *reinterpret_cast<h8*>(p.hi + at) = hi;
    if constexpr (SPLIT)
        *reinterpret_cast<h8*>(p.hi + (at ^ 32)) = lo;
    else if (p.lo)
        *reinterpret_cast<h8*>(p.lo + at) = lo;
}

// ---------------------------------------------------------------------------
// Before the products: momentum, norms, and the matrices as stored
// ---------------------------------------------------------------------------
template <int DG>
__device__ __forceinline__ float load_value(const void* p, int64_t at) {
    if constexpr (DG == BIRKHOFF4_BF16)
        return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(p)[at]) << 16);
    else
        return static_cast<const float*>(p)[at];
}

template <int DG>
__device__ __forceinline__ void load4(const void* p, int64_t at, float v[4]) {
    if constexpr (DG == BIRKHOFF4_BF16) {
        const v2u_at2 u = *reinterpret_cast<const v2u_at2*>(static_cast<const uint16_t*>(p) + at);
        v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
        v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
        const v4u_at4 u = *reinterpret_cast<const v4u_at4*>(static_cast<const float*>(p) + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(u[e]);
    }
}

// Four neighbouring values of a row of the caller's array, of which `n` are there.
template <int DO>
__device__ __forceinline__ v4f read4(const void* out, int64_t at, int64_t n) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (n >= 4) {
        load4<DO>(out, at, v);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) v[e] = load_value<DO>(out, at + e);
    }
    return v4f{v[0], v[1], v[2], v[3]};
}

template <int DO>
__device__ __forceinline__ void write4(void* out, int64_t at, int64_t n, const v4f v) {
    if (n >= 4) {
        if constexpr (DO == BIRKHOFF4_BF16) {
            *reinterpret_cast<v2u_at2*>(static_cast<uint16_t*>(out) + at) = v2u_at2{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
        } else {
            *reinterpret_cast<v4u_at4*>(static_cast<float*>(out) + at) =
                v4u_at4{__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e) {
        if (e >= n) continue;
        if constexpr (DO == BIRKHOFF4_BF16)
            static_cast<uint16_t*>(out)[at + e] = static_cast<uint16_t>(pack_bf16(v[e], 0.f));
        else
            static_cast<float*>(out)[at + e] = v[e];
    }
}

// What is orthogonalised: G, or with M, which is renewed before it, the direction G + momentum M or M.
struct Source {
    const void* G;
    float* M;
    float momentum;
    bool nesterov;

    __device__ __forceinline__ float direction(float g, float m) const { return nesterov ? __builtin_fmaf(momentum, m, g) : m; }
};

// M <- momentum M + G where there is one, and the sum of squares of each matrix's direction in 64 bits (no
// finite fp32 matrix leaves its range): gridDim.x partial sums for each of gridDim.y matrices. Bound by memory:
// 10240 x 2560 (bf16 G, fp32 M read and written) 46 us, 5.7 TB/s; four loads of each array in flight.
constexpr int kPrepBlock = 256;

template <int DG, bool MOMENTUM>
__global__ __launch_bounds__(kPrepBlock) void orth_prep_kernel(Source s, double* __restrict__ sums, int64_t values, int64_t first) {
    __shared__ double red[kPrepBlock];
    const int64_t matrix = blockIdx.y, base = (first + matrix) * values;
    double sum = 0.0;
    auto take = [&](float g, float* m) {
        float u = g;
        if constexpr (MOMENTUM) {
            *m = __builtin_fmaf(s.momentum, *m, g);
            u = s.direction(g, *m);
        }
        sum = __builtin_fma(static_cast<double>(u), static_cast<double>(u), sum);
    };
    const int64_t quads = (values + 3) / 4, pace = static_cast<int64_t>(gridDim.x) * kPrepBlock;
    constexpr int N = 4;  // asked for together
    for (int64_t q0 = static_cast<int64_t>(blockIdx.x) * kPrepBlock + threadIdx.x; q0 < quads; q0 += N * pace) {
        v4f g[N], m[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t q = q0 + k * pace, there = values - 4 * q;
            g[k] = read4<DG>(s.G, base + 4 * q, there);
            if constexpr (MOMENTUM) m[k] = read4<BIRKHOFF4_F32>(s.M, base + 4 * q, there);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t q = q0 + k * pace, there = values - 4 * q;
#pragma unroll
            for (int e = 0; e < 4; ++e) {  // zeros where there is nothing
                float x = MOMENTUM ? m[k][e] : 0.f;
                take(g[k][e], &x);
                if constexpr (MOMENTUM) m[k][e] = x;
            }
            if constexpr (MOMENTUM)
                if (there > 0) write4<BIRKHOFF4_F32>(s.M, base + 4 * q, there, m[k]);
        }
    }
    red[threadIdx.x] = sum;
    for (int half = kPrepBlock / 2; half > 0; half /= 2) {
        __syncthreads();
        if (threadIdx.x < half) red[threadIdx.x] += red[threadIdx.x + half];
    }
    if (threadIdx.x == 0) sums[matrix * gridDim.x + blockIdx.x] = red[0];
}

// The directions R x C over their norms, stored in their own order (own) and the other (turned), with zeros
// around: 64 x 64 values a block, turned in LDS (a pitch of 65, so that both directions go over all banks). A NaN
// or infinity anywhere makes the whole matrix NaN. Bound by memory: 4096 x 4096 bf16 28 us, 4.8 TB/s of 2 + 6 bytes a
// value (10240 x 2560 with M, in fp32 pieces, 78 us, 4.7 TB/s).
constexpr int kConvert = 64;

template <int DG, bool MOMENTUM, bool SPLIT>
__global__ __launch_bounds__(256) void orth_convert_kernel(Source s, const double* __restrict__ sums, int parts, double eps,
                                                           Plane own, Plane turned, int64_t R, int64_t C, int64_t first,
                                                           unsigned matrices, unsigned blocks, unsigned across) {
    __shared__ float tile[kConvert][kConvert + 1];
    __shared__ double red[256];
    // `blocks` a matrix, `across` of them along a row. Where an XCD has whole matrices, on the one that takes their products
    // (48 of 512 x 128 16 us without, 10 with; one of 10240 x 2560 78 without, 88 with).
    const unsigned flat = matrices >= 8 ? blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8 : blockIdx.x, block = flat % blocks;
    if (flat / blocks >= matrices) return;  // uniform over the block
    const int64_t matrix = flat / blocks, base = (first + matrix) * R * C;
    const int64_t r0 = static_cast<int64_t>(block / across) * kConvert, c0 = static_cast<int64_t>(block % across) * kConvert;
    constexpr int N = kConvert / 16;
    const int c = 4 * (threadIdx.x % 16);
    v4f u[N], m[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t row = r0 + threadIdx.x / 16 + 16 * k, at = base + row * C + c0 + c, there = row < R ? C - c0 - c : 0;
        u[k] = read4<DG>(s.G, at, there);
        if constexpr (MOMENTUM) m[k] = read4<BIRKHOFF4_F32>(s.M, at, there);
    }
    double norm = 0.0;  // the parts in the order of the threads, then pairs
    for (int k = threadIdx.x; k < parts; k += 256) norm += sums[matrix * parts + k];
    red[threadIdx.x] = norm;
    for (int half = 128; half > 0; half /= 2) {
        __syncthreads();
        if (threadIdx.x < half) red[threadIdx.x] += red[threadIdx.x + half];
    }
    __syncthreads();
    norm = __builtin_sqrt(red[0]);
    const double scale = norm < __builtin_inf() ? kUnit / (norm + eps) : __builtin_nan("");
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int r = threadIdx.x / 16 + 16 * k;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = u[k][e];
            if constexpr (MOMENTUM) v = s.direction(v, m[k][e]);
            // around the values zeros, whatever the scale
            tile[r][c + e] = r0 + r < R && c0 + c + e < C ? static_cast<float>(v * scale) : 0.f;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int task = threadIdx.x + 256 * k, line = task / 8, at = 8 * (task % 8);
        float v[8];
        h8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[line][at + e];
        halves(v, &hi, &lo);
        store8<SPLIT>(own, matrix, r0 + line, c0 + at, hi, lo);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[at + e][line];
        halves(v, &hi, &lo);
        store8<SPLIT>(turned, matrix, c0 + line, r0 + at, hi, lo);
    }
}

// A matrix stored in pieces of 16 columns' hi and lo, into 32 columns' hi (and lo, where it is kept) of another place.
__global__ __launch_bounds__(256) void orth_apart_kernel(Plane from, Plane to, int64_t cols) {
    const int64_t matrix = blockIdx.y, pieces = from.rows * (cols / 8);
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < pieces; k += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = k / 2 % from.rows, col = k / 2 / from.rows * 16 + k % 2 * 8;
        const int64_t at = matrix * from.stride + place<true>(from, row, col);
        store8<false>(to, matrix, row, col, *reinterpret_cast<const h8*>(from.hi + at), *reinterpret_cast<const h8*>(from.hi + (at ^ 32)));
    }
}

// ---------------------------------------------------------------------------
// The products
// ---------------------------------------------------------------------------
enum { GRAM, POLY, PAIR, NEXT, LAST };

// acc_ij = sum_k P_ik Q_jk in units of kUnit^2. Results, stored as own_ij and as turned_ji:
//   GRAM  A = acc
//   POLY  E = keep A + add A^2 with A^2 from acc, src = A and its diagonal as above
//   PAIR  add M N for symmetric M = P and N = Q that commute: add (D_i N_ij + M_ij D'_j + acc), D and D' theirs
//   NEXT  add ((keep + F_i) src_ij + acc), the next X;  LAST: the same, which goes to the caller's array
// All but the last two have a symmetric result: its tiles below the diagonal alone are computed. `plus` is
// added to the diagonal of POLY's.
struct Product {
    Plane P, Q, src, own, turned;
    const float* src_diag;  // D (POLY, PAIR) or F (NEXT, LAST), `side` a matrix
    float* own_diag;        // D (GRAM, PAIR) or F (POLY)
    float keep, add;
    const float* q_diag;    // D' (PAIR)
    float plus;
    int64_t side;
    int panels;             // of P's and Q's rows
    int tiles, tj;          // of the result, and along j
    int matrices;
};

// What becomes of the last step's values: out (rows x cols, `tall`: out_ji), or the weights
// W <- (1 - rate decay) W - rate scale value with rate = lr * *lr_at.
struct Result {
    void* out;
    int64_t rows, cols, first;
    bool tall, update;
    float lr, decay, scale;
    const float* lr_at;
};

// Four waves have (32 W) x (32 W) of a (64 W) x (64 W) tile each; KS groups of four take a KS-th of the panels each and
// add up at the end. A group's `stages` panels of both operands lie in LDS: while one is multiplied the next
// one is there and the others are on their way. At the middle of a stage the block's waves meet: what the
// next stage reads has come then, and the one before is read by nobody any more, whose place the last one
// takes.
// What bounds it: large products the card's power, which takes the clock to 1.6..2 GHz while the matrix cores are busy two
// thirds of the cycles: A X of 2560 x 10240 in fp32 376 us, 1.07 PFLOP/s of fp16 products; 4096 x 4096 in bf16 160
// (0.86), its X X^T 88, half a product. Small ones a block's latency: 5 to 10 us of 48 matrices of 128 x 512.
constexpr int stages(int w) { return w == 3 ? 6 : 5; }
[[maybe_unused]] constexpr int kRawBuffer = 0x00027000;  // a buffer of bytes, addresses outside of it read as zero

template <int W>
constexpr int stage_bytes() { return 2 * 64 * W * 64; }

// The 32 x 32 parts of a stored matrix from a row and a column on, whole multiples of 32: each is four (without
// lo: two) pieces of memory of 1 KB, which a wave reads and writes 16 bytes a lane. An image is their copy
// in LDS: SPLIT: 2 KB of two panels; otherwise 2 KB of hi and of lo.
template <bool SPLIT>
struct Parts {
    char *hi, *lo;
    int64_t across;  // bytes from 32 columns to the next

    __device__ __forceinline__ Parts(const Plane& p, int64_t matrix, int64_t row, int64_t col) {
        const int64_t at = matrix * p.stride + (col / panel_cols(SPLIT) * p.rows + row) * 64;
        hi = p.hi + at;
        lo = SPLIT ? p.hi + at + p.rows * 64 : p.lo + at;
        across = p.rows * (SPLIT ? 128 : 64);
    }
    // kilobyte k of the part `r` parts down and `c` parts across
    __device__ __forceinline__ char* kilobyte(int r, int c, int k) const {
        return (k < 2 ? hi : lo) + c * across + r * 2048 + 1024 * (k & 1);
    }
};

// Where the piece of eight columns from `col` (0, 8, 16, 24) on lies in row `row` of an image.
template <bool SPLIT>
__device__ __forceinline__ int spot(int row, int col, bool lo) {
    if constexpr (SPLIT)
        return 2048 * (col >> 4) + row * 64 + 16 * (((col >> 3 & 1) + (lo ? 2 : 0)) ^ (row >> 2 & 3));
    else
        return (lo ? 2048 : 0) + row * 64 + 16 * ((col >> 3) ^ (row >> 2 & 3));
}

// Of N products, one ahead of each of 2 W reads of LDS and then, where there are LOADS, of the 2 W loads, so that
// the matrix cores do not wait for all of them (the loads write LDS, so they are not put before a read).
template <int W, int N, bool LOADS>
__device__ __forceinline__ void mix_reads() {
    if constexpr (W > 1) {
        constexpr int left = N - 2 * W, each = left >= 2 * W ? 1 : left > 0 ? (2 * W + left - 1) / left : 2 * W;
#pragma unroll
        for (int k = 0; k < 2 * W; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        if constexpr (LOADS) {
#pragma unroll
            for (int k = 0; k < 2 * W; k += each) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x010, each, 0);
            }
        }
        __builtin_amdgcn_sched_group_barrier(0x008, left > 0 ? left : 0, 0);
    }
}

template <bool SPLIT, int KIND, int DO, int W, int KS>
__global__ __launch_bounds__(256 * KS, W * KS == 1 ? 4 : W * KS == 2 ? 2 : KS) void orth_product_kernel(Product g, Result res) {
    constexpr int T = 64 * W;
    constexpr bool SYM = KIND == GRAM || KIND == POLY || KIND == PAIR;
    constexpr int S = stages(W), STAGE = stage_bytes<W>();
    static_assert(KS * S * STAGE >= KS * 4 * W * W * 4096, "the sums take the stages' place");
    __shared__ __attribute__((aligned(128))) char lds[KS * S * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3;
    const int group = KS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
    // Blocks go round the eight XCDs: each XCD takes neighbouring tiles of neighbouring matrices, whose rows its L2 holds.
    const unsigned flat = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    const unsigned of = g.matrices > 1 ? flat / static_cast<unsigned>(g.tiles) : 0;
    const int tile = static_cast<int>(flat - of * g.tiles);
    const int64_t matrix = of;
    if (tile >= g.tiles || of >= static_cast<unsigned>(g.matrices)) return;  // uniform over the block
    int ti, tj;
    if constexpr (SYM) {  // row by row below the diagonal
        ti = static_cast<int>((__builtin_sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > tile) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
        tj = tile - ti * (ti + 1) / 2;
    } else {
        // four rows of tiles, column by column: those of an XCD are as many rows as columns, about
        const int rows = g.tiles / g.tj, band = tile / (4 * g.tj), high = rows - 4 * band < 4 ? rows - 4 * band : 4;
        const int in = tile - band * 4 * g.tj;
        ti = 4 * band + in % high;
        tj = in / high;
    }
    // Rows behind the stored ones, of a tile that hangs over: others in their place, which nothing is made of.
    int pr[W], qr[W];  // bytes from the panel's first row
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const int64_t r = 16 * (W * wave + k), ri = ti * static_cast<int64_t>(T) + r, rj = tj * static_cast<int64_t>(T) + r;
        pr[k] = static_cast<int>((ri < g.P.rows ? ri : g.P.rows - 16) * 64);
        qr[k] = static_cast<int>((rj < g.Q.rows ? rj : g.Q.rows - 16) * 64);
    }
    [[maybe_unused]] char *const p0 = g.P.hi + matrix * g.P.stride, *const q0 = g.Q.hi + matrix * g.Q.stride;
    [[maybe_unused]] const int p_panel = static_cast<int>(g.P.rows * 64), q_panel = static_cast<int>(g.Q.rows * 64);
    [[maybe_unused]] const int lane16 = lane * 16;
    const int panels = g.panels / KS, begin = panels * group;
    char* const own = lds + group * (S * STAGE);
    int asked = begin, room = 1024 * W * wave;  // the next panel and its place
    auto load = [&] {  // past the last panel: the last one again, into a place that is not read
#ifdef __HIP_DEVICE_COMPILE__  // the host's compiler has no such buffers
        const auto pb = __builtin_amdgcn_make_buffer_rsrc(p0 + static_cast<int64_t>(asked) * p_panel, 0, p_panel, kRawBuffer);
        const auto qb = __builtin_amdgcn_make_buffer_rsrc(q0 + static_cast<int64_t>(asked) * q_panel, 0, q_panel, kRawBuffer);
#pragma unroll
        for (int k = 0; k < W; ++k) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(pb, (__attribute__((address_space(3))) void*)(own + room + 1024 * k), 16, lane16,
                                                     pr[k], 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(qb, (__attribute__((address_space(3))) void*)(own + room + T * 64 + 1024 * k), 16,
                                                     lane16, qr[k], 0, 0);
        }
#endif
        asked = asked + 1 < begin + panels ? asked + 1 : asked;
        room = room >= (S - 1) * STAGE ? room - (S - 1) * STAGE : room + STAGE;
    };
    const int wi = 32 * W * (wave >> 1), wj = 32 * W * (wave & 1);
    const int r32 = lane & 31, h = lane >> 5;
    const char* own_rows = own + (wi + r32) * 64;
    const char* col_rows = own + (T + wj + r32) * 64;
    const int swizzle = (r32 >> 2) & 3;
    // pieces 2 part + h: SPLIT: hi (part 0) or lo of 16 columns; otherwise 16 of 32 columns
    auto fetch = [&](int from, int part, h8 (&a)[W], h8 (&b)[W]) {
        const int at = from + 16 * ((2 * part + h) ^ swizzle);
        a[0] = *reinterpret_cast<const h8*>(own_rows + at);  // in the order in which they are multiplied
#pragma unroll
        for (int k = 0; k < W; ++k) b[k] = *reinterpret_cast<const h8*>(col_rows + at + 2048 * k);
#pragma unroll
        for (int k = 1; k < W; ++k) a[k] = *reinterpret_cast<const h8*>(own_rows + at + 2048 * k);
    };
    v16f acc[W][W] = {};
    auto multiply = [&](const h8 (&a)[W], const h8 (&b)[W]) {
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i], b[j], acc[i][j], 0, 0, 0);
    };
    auto meet = [&] {  // the next stage is there; of those behind it 2 W loads each of this wave are on their way
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"((S - 3) * 2 * W) : "memory");
        __builtin_amdgcn_sched_barrier(0);  // what was read before is also multiplied before
    };
    // What the ends of the 32 x 32 parts need from memory is asked for here: behind the sums, and behind the
    // stores of the part before (for which a wait for a later load waits too), its latency would be seen each
    // time (2900 cycles a part).
    const int64_t ib = static_cast<int64_t>(ti) * T + wi, jb = static_cast<int64_t>(tj) * T + wj;
    const float* sd = KIND != GRAM ? g.src_diag + matrix * g.side : nullptr;
    // parts that this group ends: its own half of the columns, or all of them for the first group
    constexpr bool HALVES = KS == 2 && W == 2;
    constexpr int ENDS = HALVES ? W : W * W;
    auto part_a = [&](int k) { return HALVES ? k : k / W; };
    auto part_b = [&](int k) { return HALVES ? group : k % W; };
    auto there = [&](int k) {  // uniform over the wave: rows come in whole 64s
        return ib + 32 * part_a(k) < g.P.rows && jb + 32 * part_b(k) < g.Q.rows &&
               !(SYM && ib + 32 * part_a(k) < jb + 32 * part_b(k));
    };
    v4u src[ENDS][4], src2[KIND == PAIR ? ENDS : 1][4];
    v4f di[W][2][2];
    float dj[W];
    // Places of an image that a lane writes and reads, part by part at constant distances: its pieces of row j
    // (turned order), and, value by value, column j of rows 8 h .. + 3 and 8 h + 4 .. (own order).
    const int lane16b = lane * 16;
    int piece_at[2][2], value_at[2][2];  // [hi, lo][first or second]
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            piece_at[y][u] = spot<SPLIT>(r32, 16 * u + 8 * h, y == 1);
            value_at[y][u] = spot<SPLIT>(8 * h + 4 * u, r32 & 24, y == 1) + 2 * (r32 & 7);
        }
    auto out_at = [&](int k, int t, int64_t* n) {  // LAST: four values of a row of the caller's array, and how many are there
        const int64_t i0 = ib + 32 * part_a(k), j0 = jb + 32 * part_b(k);
        const int64_t row = (res.tall ? j0 : i0) + 8 * t + lane / 8, col = (res.tall ? i0 : j0) + 4 * (lane % 8);
        *n = row < res.rows ? res.cols - col : 0;
        return ((res.first + matrix) * res.rows + row) * res.cols + col;
    };
    const bool ends = HALVES || group == 0;
    if constexpr (KIND != GRAM)
        if (ends) {
            const Parts<SPLIT> from(g.src, matrix, jb, ib);
#pragma unroll
            for (int k = 0; k < ENDS; ++k)
                if (there(k)) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        src[k][u] = *reinterpret_cast<const v4u*>(from.kilobyte(part_b(k), part_a(k), u) + lane16b);
                    if constexpr (KIND == PAIR) {
                        const Parts<SPLIT> other(g.P, matrix, jb, ib);
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            src2[k][u] = *reinterpret_cast<const v4u*>(other.kilobyte(part_b(k), part_a(k), u) + lane16b);
                    }
                }
#pragma unroll
            for (int a = 0; a < W; ++a)
                if (ib + 32 * a < g.P.rows)
#pragma unroll
                    for (int u = 0; u < 4; ++u) di[a][u / 2][u % 2] = *reinterpret_cast<const v4f*>(sd + ib + 32 * a + 16 * (u / 2) + 8 * h + 4 * (u % 2));
            if constexpr (KIND == POLY || KIND == PAIR) {
                const float* qd = KIND == PAIR ? g.q_diag + matrix * g.side : sd;
#pragma unroll
                for (int b = 0; b < W; ++b)
                    if (jb + 32 * b < g.Q.rows) dj[b] = qd[jb + 32 * b + r32];
            }
        }
#pragma unroll
    for (int k = 0; k < S - 1; ++k) load();
    h8 a0[W], b0[W], a1[W], b1[W];
    meet();
    fetch(0, 0, a0, b0);
    int now = 0;
#pragma unroll 1
    for (int stage = 0; stage < panels; ++stage) {
        fetch(now, 1, a1, b1);
        multiply(a0, b0);
        mix_reads<W, W * W, false>();
        meet();
        now = now == (S - 1) * STAGE ? 0 : now + STAGE;
        if constexpr (SPLIT) {
            h8 a2[W], b2[W];
            fetch(now, 0, a2, b2);
            load();
            multiply(a0, b1);
            multiply(a1, b0);
            mix_reads<W, 2 * W * W, true>();
#pragma unroll
            for (int k = 0; k < W; ++k) a0[k] = a2[k], b0[k] = b2[k];
        } else {
            fetch(now, 0, a0, b0);
            load();
            multiply(a1, b1);
            mix_reads<W, W * W, true>();
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);

    // The groups' sums are added through LDS, in their order; two groups end half of the parts each.
    auto slot = [&](int of, int q) { return reinterpret_cast<v4f*>(lds) + ((of * 4 + wave) * W * W + q) * 256; };
    if constexpr (KS > 1) {
#pragma unroll
        for (int q = 0; q < W * W; ++q)
            if (HALVES ? q % W != group : group > 0)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const v16f& c = acc[q / W][q % W];
                    slot(group, q)[r * 64 + lane] = v4f{c[4 * r], c[4 * r + 1], c[4 * r + 2], c[4 * r + 3]};
                }
        __syncthreads();
        if (!ends) return;
#pragma unroll
        for (int q = 0; q < W * W; ++q)
            if (!HALVES || q % W == group)
#pragma unroll
                for (int of = HALVES ? 0 : 1; of < (HALVES ? 1 : KS); ++of)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const v4f x = slot(HALVES ? group ^ 1 : of, q)[r * 64 + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[q / W][q % W][4 * r + e] += x[e];
                    }
    }
    float rate = 0.f;
    v4f old[ENDS][4];
    if constexpr (KIND == LAST)
        if (res.update) {
            rate = res.lr_at ? res.lr * *res.lr_at : res.lr;
#pragma unroll
            for (int k = 0; k < ENDS; ++k)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    int64_t n;
                    const int64_t at = out_at(k, t, &n);
                    old[k][t] = read4<DO>(res.out, at, n);
                }
        }
    const Parts<SPLIT> to_turned(g.turned, matrix, jb, ib), to_own(g.own, matrix, ib, jb);
#pragma unroll
    for (int k = 0; k < ENDS; ++k) {
        if (!there(k)) continue;
        // A lane has column j of 32 x 32 values, rows 8 g + 4 h + 0..3 of it in sum[4 g ..]: exchanged between the wave's
        // halves, eight neighbouring rows, which are one piece of row j in the other order. What src adds is
        // in that order too. Whatever goes to and comes from memory passes the part's place in LDS, so that
        // a wave's accesses are whole kilobytes.
        const int a = part_a(k), b = part_b(k);
        // a group reads what the other one has put into its own slots
        char* image = reinterpret_cast<char*>(HALVES ? slot(group, a * W + group) : slot(0, a * W + b));
        v16f sum;
        if constexpr (HALVES)
            sum = group ? acc[a][W - 1] : acc[a][0];
        else
            sum = acc[k / W][k % W];
        float v[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[8 * u + e]), __float_as_uint(sum[8 * u + 4 + e]), false, false);
                v[u][e] = __uint_as_float(x[0]);
                v[u][4 + e] = __uint_as_float(x[1]);
            }
        const bool across = SYM && ib + 32 * a == jb + 32 * b;  // the diagonal
        float one = 0.f;                                                                  // the product's value on it
        if constexpr (SYM)
            if (across) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) one = 16 * u + 8 * h + e == r32 ? v[u][e] : one;
                one /= kUnit * kUnit;
            }
        if constexpr (KIND != GRAM) {
            auto pieces_of = [&](const v4u (&from)[4], float (&to)[2][8]) {
#pragma unroll
                for (int u = 0; u < 4; ++u) *reinterpret_cast<v4u*>(image + 1024 * u + lane16b) = from[u];
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const h8 hi = *reinterpret_cast<const h8*>(image + piece_at[0][u]);
                    const h8 lo = *reinterpret_cast<const h8*>(image + piece_at[1][u]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) to[u][e] = __builtin_fmaf(static_cast<float>(hi[e]), 1.f, static_cast<float>(lo[e]));
                }
                __builtin_amdgcn_wave_barrier();
            };
            const float djk = HALVES ? (group ? dj[W - 1] : dj[0]) : dj[k % W], add = g.add / kUnit;
            float s[2][8], s2[KIND == PAIR ? 2 : 1][8];
            pieces_of(src[k], s);
            if constexpr (KIND == PAIR) pieces_of(src2[k], s2);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = di[HALVES ? k : k / W][u][e / 4][e % 4];
                    if constexpr (KIND == POLY)
                        v[u][e] = __builtin_fmaf(__builtin_fmaf(g.add, d + djk, g.keep), s[u][e], add * v[u][e]);
                    else if constexpr (KIND == PAIR)
                        v[u][e] = __builtin_fmaf(g.add, __builtin_fmaf(d, s[u][e], djk * s2[u][e]), add * v[u][e]);
                    else
                        v[u][e] = __builtin_fmaf(g.add * (g.keep + d), s[u][e], add * v[u][e]);
                }
            if (KIND == POLY && across) one = g.plus + __builtin_fmaf(g.keep, djk, g.add * __builtin_fmaf(djk, djk, one));
            // row i is column j here, and the first factor's diagonal is asked for along i alone
            if constexpr (KIND == PAIR)
                if (across) {
                    float dd = 0.f;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            dd = 16 * u + 8 * h + e == r32 ? di[HALVES ? k : k / W][u][e / 4][e % 4] : dd;
                    one = g.add * __builtin_fmaf(dd, djk, one);
                }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] /= kUnit;
        }
        if constexpr (KIND == LAST) {
            // rows of the caller's array in LDS, 128 bytes each, whose 16-byte pieces change places by the row
            auto at = [&](int row, int col) { return reinterpret_cast<float*>(image + row * 128 + 16 * ((col >> 2) ^ (row & 7)) + 4 * (col & 3)); };
            const float shrink = 1.f - rate * res.decay, by = rate * res.scale;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = 16 * u + 8 * h + e;
                    *(res.tall ? at(r32, i) : at(i, r32)) = v[u][e] / kUnit;
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                v4f o = *reinterpret_cast<const v4f*>(at(8 * t + lane / 8, 4 * (lane % 8)));
                if (res.update)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(-by, o[e], shrink * old[k][t][e]);
                int64_t n;
                const int64_t to = out_at(k, t, &n);
                write4<DO>(res.out, to, n, o);
            }
        } else {
            constexpr int TURNED = SPLIT || KIND == GRAM || KIND == NEXT ? 4 : 2, OWN = SPLIT || KIND == GRAM ? 4 : 2;
            if (across) {  // the diagonal itself lies elsewhere
                if (r32 / 8 % 2 == h) g.own_diag[matrix * g.side + jb + 32 * b + r32] = one;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = 16 * u + 8 * h + e == r32 ? 0.f : v[u][e];
            }
            h8 hi[2], lo[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                halves(v[u], &hi[u], &lo[u]);
                *reinterpret_cast<h8*>(image + piece_at[0][u]) = hi[u];
                if (TURNED == 4 || OWN == 4) *reinterpret_cast<h8*>(image + piece_at[1][u]) = lo[u];
            }
            __builtin_amdgcn_wave_barrier();
            auto values = [&](bool all) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (!all && 16 * u + 8 * h + e < r32) continue;
                        *reinterpret_cast<_Float16*>(image + value_at[0][e / 4] + 1024 * u + 64 * (e % 4)) = hi[u][e];
                        if (OWN == 4) *reinterpret_cast<_Float16*>(image + value_at[1][e / 4] + 1024 * u + 64 * (e % 4)) = lo[u][e];
                    }
            };
            if (!across) {
                v4u out[TURNED];
#pragma unroll
                for (int u = 0; u < TURNED; ++u) out[u] = *reinterpret_cast<const v4u*>(image + 1024 * u + lane16b);
#pragma unroll
                for (int u = 0; u < TURNED; ++u) *reinterpret_cast<v4u*>(to_turned.kilobyte(b, a, u) + lane16b) = out[u];
                __builtin_amdgcn_wave_barrier();
                values(true);
            } else {
                // Of a symmetric result what lies below the diagonal counts, whatever the tiles (the sum of the
                // pieces' products is not the same bits with the factors exchanged): above it the turned
                // order, which is there, has it.
                values(false);
            }
            __builtin_amdgcn_wave_barrier();
            v4u out[OWN];
#pragma unroll
            for (int u = 0; u < OWN; ++u) out[u] = *reinterpret_cast<const v4u*>(image + 1024 * u + lane16b);
#pragma unroll
            for (int u = 0; u < OWN; ++u) *reinterpret_cast<v4u*>(to_own.kilobyte(a, b, u) + lane16b) = out[u];
        }
    }
}

// ---------------------------------------------------------------------------
// Matrices with a side of at most 80
// ---------------------------------------------------------------------------
// X after any number of steps is F X with F a polynomial in A = X X^T of the beginning, so the steps can run
// on m x m values alone: with p = a I + b A + c A^2, F <- p F and A <- p A p (all of them symmetric, and they
// commute). G is read twice, for the first A and for F X, whatever the steps; the direct form reads X twice a
// step and launches three kernels for it. An error of A is multiplied by up to a^2 = 12 a step where the
// singular value is small, so A and F are 64-bit numbers, from products of the inputs without rounding: the
// result is nearer than fp32 products bring it. LDS is the limit of m: three matrices of 5 x 5 tiles are 150 KB of it. The
// cube of m runs on one compute unit a matrix (m = 80: 36 us of the matrix cores for five steps, of 52 that the kernel takes;
// m = 24: 10), and G G^T of 80 rows takes them half as long as reading fp32 G does. 24 x 16384 fp32 takes 21 us,
// 80 x 32768 97 (10 MB twice: 4 at the memory's rate).
//
// Errors grow with the product g of the steps' largest |p| (for singular values up to sqrt(2), below): A's by g^2, and a
// rounding between F's large and small directions by g^3, which five of the usual steps (g = 485) leave at 2^-26.
// Where g is larger, an eigenvalue that should be zero, of either sign, would run away. There (DEEP):
//   * A and F are made symmetric in every bit: their errors grow by g and g^2 then;
//   * the first steps, to g = 64, are taken as above, then A is formed anew from F G, whose small values are 64 times as large;
//   * from then on A <- p A p + shift I with a shift that is above what the step can have rounded: A stays positive definite, its eigenvalues stay where p keeps them, and F stays below
//     64 / sqrt(2 P^1.5 2^-53) = 2^28. Singular values under 2^-26 of the norm stay behind what 64 bits would make of them (in fp32
//     products they are lost among the roundings).
//   * F X is formed in 64 bits whatever the result's type: F's large values meet zeros.
// 24 x 1024 in fp32 of rank one: 2.5e-8 off after ten steps and 1.2e-5 after 64 (rows that are equal in pairs: 2.5e-8 and
// 2.7e-6), where fp32 products are 1e-2 and 1 off (2e-6 and 4e-6).
constexpr int kNarrow = 80;
constexpr int kSlab = 64;            // columns of X taken at a time
constexpr int kSlabPitch = kSlab + 1;
constexpr double kFar = 0x1p80;      // what bf16 values far from one are multiplied or divided by

typedef double v4d __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4d mfma_f64(double a, double b, v4d c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0); }

// X's rows (16 MT of them, zeros behind the m) and columns j0 .. j0 + 63 of a direction, from the caller's
// R x C array: X = U, or for a tall U its transpose. A thread has MT times four neighbouring values of the
// array, which it asks for (fetch) long before they go to LDS (put).
template <int DG, bool MOMENTUM, int MT>
struct Slab {
    const Source& s;
    int64_t base, C, n;
    int m;
    bool tall;
    v4f g[MT], mo[MT];

    __device__ __forceinline__ Slab(const Source& src, int64_t at, int64_t R, int64_t cols)
        : s(src), base(at), C(cols), n(R > cols ? R : cols), m(static_cast<int>(R > cols ? cols : R)), tall(R > cols) {}
    // where a thread's q-th four values are: in the array, and their place in the slab; how many are there
    __device__ __forceinline__ int64_t where(int q, int64_t j0, int64_t* at, int* line, int* c) const {
        const int left = static_cast<int>(n - j0 < kSlab ? n - j0 : kSlab), task = threadIdx.x + 256 * q;
        if (tall) {
            *line = task / (4 * MT), *c = 4 * (task % (4 * MT));
            *at = base + (j0 + *line) * C + *c;
            return *line < left ? m - *c : 0;
        }
        *line = task / 16, *c = 4 * (task % 16);
        *at = base + *line * C + j0 + *c;
        return *line < m ? left - *c : 0;
    }
    __device__ __forceinline__ float* value(float* slab, int line, int c) const {
        return slab + (tall ? c * kSlabPitch + line : line * kSlabPitch + c);
    }
    __device__ __forceinline__ void fetch(int64_t j0) {
#pragma unroll
        for (int q = 0; q < MT; ++q) {
            int64_t at = base;
            int line, c;
            const int64_t there = j0 < n ? where(q, j0, &at, &line, &c) : 0;
            g[q] = read4<DG>(s.G, at, there);
            if constexpr (MOMENTUM) mo[q] = read4<BIRKHOFF4_F32>(s.M, at, there);
        }
    }
    // RENEW: M on the way; SCALED: the values times `scale`
    template <bool RENEW, bool SCALED>
    __device__ __forceinline__ void put(int64_t j0, float* slab, double scale) {
#pragma unroll
        for (int q = 0; q < MT; ++q) {
            int64_t at;
            int line, c;
            const int64_t there = where(q, j0, &at, &line, &c);
            v4f u = g[q];
            if constexpr (MOMENTUM) {
                v4f m2 = mo[q];
                if constexpr (RENEW) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) m2[e] = __builtin_fmaf(s.momentum, m2[e], u[e]);
                    write4<BIRKHOFF4_F32>(s.M, at, there, m2);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = s.direction(u[e], m2[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) *value(slab, line, c + e) = SCALED ? static_cast<float>(u[e] * scale) : u[e];
        }
    }
};

// Tiles of 16 x 16 on and below the diagonal, row by row.
constexpr int tri(int t) { return t * (t + 1) / 2; }

// Each block's part of U U^T (gridDim.x blocks a matrix), and the momentum's renewal. The block's four
// waves take every fourth tile each, over all columns of a slab.
constexpr int kGramBlock = 256;

template <int DG, bool MOMENTUM, int MT>
__global__ __launch_bounds__(kGramBlock) void orth_narrow_gram_kernel(Source s, double* __restrict__ part, int64_t R, int64_t C,
                                                                      int64_t first) {
    constexpr int TILES = tri(MT), OWN = (TILES + 3) / 4;
    __shared__ float slab[16 * MT * kSlabPitch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y, base = (first + matrix) * R * C, n = R > C ? R : C;
    v4d acc[OWN] = {};
    int ri[OWN], rj[OWN];  // where a lane reads its rows of a tile's sides
#pragma unroll
    for (int q = 0; q < OWN; ++q) {
        const int t = wave + 4 * q < TILES ? wave + 4 * q : 0;
        int i = 0;
        while (tri(i + 1) <= t) ++i;
        ri[q] = (16 * i + (lane & 15)) * kSlabPitch + (lane >> 4);
        rj[q] = (16 * (t - tri(i)) + (lane & 15)) * kSlabPitch + (lane >> 4);
    }
    Slab<DG, MOMENTUM, MT> x(s, base, R, C);
    const int64_t pace = static_cast<int64_t>(gridDim.x) * kSlab;
    x.fetch(static_cast<int64_t>(blockIdx.x) * kSlab);
    for (int64_t j0 = static_cast<int64_t>(blockIdx.x) * kSlab; j0 < n; j0 += pace) {
        __syncthreads();
        x.template put<true, false>(j0, slab, 1.0);
        __syncthreads();
        x.fetch(j0 + pace);
#pragma unroll 4
        for (int k = 0; k < kSlab; k += 4)
#pragma unroll
            for (int q = 0; q < OWN; ++q)  // a tile too many is the first one again: a branch here took four times as long
                acc[q] = mfma_f64(slab[ri[q] + k], slab[rj[q] + k], acc[q]);
    }
    double* out = part + (matrix * gridDim.x + blockIdx.x) * (TILES * 256);
#pragma unroll
    for (int q = 0; q < OWN; ++q)
        if (wave + 4 * q < TILES)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[(wave + 4 * q) * 256 + (4 * r + (lane >> 4)) * 16 + (lane & 15)] = acc[q][r];
}

// The blocks' parts added, 16 entries a block in 16 parts of the order, so that few loads follow one another.
__global__ __launch_bounds__(256) void orth_narrow_join_kernel(const double* __restrict__ part, double* __restrict__ sum, int parts,
                                                               int entries) {
    __shared__ double red[16][16];
    const int c = threadIdx.x & 15, p = threadIdx.x >> 4;
    const int64_t matrix = blockIdx.y, at = static_cast<int64_t>(blockIdx.x) * 16 + c;
    double v = 0.0;
#pragma unroll 8
    for (int k = p; k < parts; k += 16) v += part[(matrix * parts + k) * entries + at];
    red[p][c] = v;
    __syncthreads();
    if (p > 0) return;
    for (int k = 1; k < 16; ++k) v += red[k][c];
    sum[matrix * entries + at] = v;
}

// Each block's part of Y Y^T for Y = F X, formed a slab at a time: four waves take 16 columns each of Y, and then the tiles
// of Y Y^T as above. M is renewed already.
template <int DG, bool MOMENTUM, int MT>
__global__ __launch_bounds__(kGramBlock) void orth_narrow_again_kernel(Source s, const double* __restrict__ F,
                                                                       const double* __restrict__ scales, double* __restrict__ part,
                                                                       int64_t R, int64_t C, int64_t first) {
    constexpr int P = 16 * MT, TILES = tri(MT), OWN = (TILES + 3) / 4;
    __shared__ float slab[P * kSlabPitch];
    __shared__ double f[P * P], y[P * kSlabPitch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y, base = (first + matrix) * R * C, n = R > C ? R : C;
    v4d acc[OWN] = {};
    int ri[OWN], rj[OWN];
#pragma unroll
    for (int q = 0; q < OWN; ++q) {
        const int t = wave + 4 * q < TILES ? wave + 4 * q : 0;
        int i = 0;
        while (tri(i + 1) <= t) ++i;
        ri[q] = (16 * i + (lane & 15)) * kSlabPitch + (lane >> 4);
        rj[q] = (16 * (t - tri(i)) + (lane & 15)) * kSlabPitch + (lane >> 4);
    }
    Slab<DG, MOMENTUM, MT> x(s, base, R, C);
    const int64_t pace = static_cast<int64_t>(gridDim.x) * kSlab;
    x.fetch(static_cast<int64_t>(blockIdx.x) * kSlab);
    for (int k = threadIdx.x; k < P * P; k += kGramBlock) f[k] = F[matrix * P * P + k];
    const double scale = scales[2 * matrix];
    for (int64_t j0 = static_cast<int64_t>(blockIdx.x) * kSlab; j0 < n; j0 += pace) {
        __syncthreads();
        x.template put<false, false>(j0, slab, 1.0);
        __syncthreads();
        x.fetch(j0 + pace);
        v4d z[MT] = {};
#pragma unroll 4
        for (int k = 0; k < P; k += 4) {
            const int at = k + (lane >> 4);
            const double v = slab[at * kSlabPitch + 16 * wave + (lane & 15)];
#pragma unroll
            for (int t = 0; t < MT; ++t) z[t] = mfma_f64(f[at * P + 16 * t + (lane & 15)], v, z[t]);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) y[(16 * t + 4 * r + (lane >> 4)) * kSlabPitch + 16 * wave + (lane & 15)] = z[t][r] * scale;
        __syncthreads();
#pragma unroll 4
        for (int k = 0; k < kSlab; k += 4)
#pragma unroll
            for (int q = 0; q < OWN; ++q) acc[q] = mfma_f64(y[ri[q] + k], y[rj[q] + k], acc[q]);
    }
    double* out = part + (matrix * gridDim.x + blockIdx.x) * (TILES * 256);
#pragma unroll
    for (int q = 0; q < OWN; ++q)
        if (wave + 4 * q < TILES)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[(wave + 4 * q) * 256 + (4 * r + (lane >> 4)) * 16 + (lane & 15)] = acc[q][r];
}

// F of each matrix from its G G^T: one block a matrix, a wave for each 16 x 16 tile on and below the diagonal. What a
// product leaves in a lane, four values of a column every four rows apart, is also what the next one wants from it: as
// the second factor as it stands, as the first one, of a symmetric matrix, from the tile across the diagonal. So tiles lie in
// LDS by lanes, 16 bytes of each in two halves, and a wave puts its own and its transpose.
constexpr int kTile = 2048;  // bytes

typedef double v2d __attribute__((ext_vector_type(2)));

struct Coefs {
    float v[3 * kOrthMaxSteps];
};

// A is of F X for the F that is there (`again`), or of G. Shifts in units of A's trace: of A at the beginning, and after each step.
struct DeepCoefs : Coefs {
    float first, shift[kOrthMaxSteps];
    bool again;
};

template <int MT, bool DEEP>
__global__ __launch_bounds__(64 * tri(MT)) void orth_narrow_poly_kernel(const double* __restrict__ sum, double* __restrict__ F,
                                                                        double* __restrict__ scales, double eps,
                                                                        std::conditional_t<DEEP, DeepCoefs, Coefs> coefs, int steps) {
    constexpr int P = 16 * MT, MATRIX = MT * MT * kTile;
    constexpr bool ROOM = MT <= 3;  // for what would otherwise take the place of something that is still being read
    __shared__ __attribute__((aligned(16))) char lds[(ROOM ? 5 : 3) * MATRIX];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t matrix = blockIdx.x;
    int ti = 0;
    while (tri(ti + 1) <= wave) ++ti;
    const int tj = wave - tri(ti);
    const int row = 16 * ti + (lane >> 4), col = 16 * tj + (lane & 15);  // of value r: row + 4 r
    char *const A = lds, *const S = lds + MATRIX, *const T = ROOM ? lds + 2 * MATRIX : A, *Q = lds + (ROOM ? 3 : 2) * MATRIX,
         *free = ROOM ? lds + 4 * MATRIX : Q;
    auto tile = [&](const char* M, int i, int j) {
        const char* at = M + (i * MT + j) * kTile + 16 * lane;
        const v2d x = *reinterpret_cast<const v2d*>(at), y = *reinterpret_cast<const v2d*>(at + kTile / 2);
        return v4d{x.x, x.y, y.x, y.y};
    };
    // M N as two sums that do not wait for each other, and with two second factors both
    auto product = [&](const char* M, const char* N) {
        v4d x = {}, y = {};
#pragma unroll
        for (int k = 0; k < MT; ++k) {
            const v4d a = tile(M, k, ti), b = tile(N, k, tj);
            x = mfma_f64(a[0], b[0], x);
            y = mfma_f64(a[1], b[1], y);
            x = mfma_f64(a[2], b[2], x);
            y = mfma_f64(a[3], b[3], y);
        }
        return x + y;
    };
    auto products = [&](const char* M, const char* N, const char* O, v4d* by_n, v4d* by_o) {
        v4d x = {}, y = {};
#pragma unroll
        for (int k = 0; k < MT; ++k) {
            const v4d a = tile(M, k, ti), b = tile(N, k, tj), c = tile(O, k, tj);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x = mfma_f64(a[r], b[r], x);
                y = mfma_f64(a[r], c[r], y);
            }
        }
        *by_n = x, *by_o = y;
    };
    auto put = [&](char* M, const v4d& v) {
        char* at = M + (ti * MT + tj) * kTile + 16 * lane;
        // row c of the transpose: value c / 4 of the lanes of c mod 4
        const int c = lane & 15;
        char* across = M + (tj * MT + ti) * kTile + kTile / 2 * (c >> 3) + 256 * (c & 3) + 16 * (lane >> 4) + 8 * (c >> 2 & 1);
        if (DEEP && ti == tj) {  // what lies below the diagonal, on both sides of it
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (row + 4 * r >= col) *reinterpret_cast<double*>(at + kTile / 2 * (r >> 1) + 8 * (r & 1)) = v[r];
                if (row + 4 * r > col) *reinterpret_cast<double*>(across + 64 * r) = v[r];
            }
            return;
        }
        *reinterpret_cast<v2d*>(at) = v2d{v[0], v[1]};
        *reinterpret_cast<v2d*>(at + kTile / 2) = v2d{v[2], v[3]};
        if (ti != tj) {
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<double*>(across + 64 * r) = v[r];
        }
    };
    // scalar loads would make the reads of LDS beside them wait, and each other
    __shared__ double co[3 * kOrthMaxSteps];
    for (int k = threadIdx.x; k < 3 * steps; k += 64 * tri(MT)) co[k] = coefs.v[k];
    v4d a, f = {};
#pragma unroll
    for (int r = 0; r < 4; ++r) a[r] = sum[(matrix * tri(MT) + wave) * 256 + (4 * r + (lane >> 4)) * 16 + (lane & 15)];
    put(A, a);
    __syncthreads();
    auto trace = [&] {  // of what lies in A's place, the same in every wave
        double x = 0.0;
        const int c = lane & 15;
#pragma unroll
        for (int k = 0; k < MT; ++k)
            x += *reinterpret_cast<const double*>(A + k * (MT + 1) * kTile + kTile / 2 * (c >> 3) + 256 * (c & 3) + 16 * c + 8 * (c >> 2 & 1));
#pragma unroll
        for (int k = 1; k < 16; k *= 2) x += __shfl_xor(x, k);
        return x;
    };
    auto shifted = [&](const v4d& v, double by) {
        v4d x = v;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = row + 4 * r == col ? x[r] + by : x[r];
        return x;
    };
    double norm = trace();
    bool fresh = true;  // F is the identity still
    if constexpr (DEEP) fresh = !coefs.again;
    const double square = norm;
    norm = __builtin_sqrt(norm);
    double scale = norm < __builtin_inf() ? 1.0 / (norm + eps) : __builtin_nan("");
    if (!fresh) scale = 1.0;
    a = a * scale * scale;
    double by = scale * scale;  // what A in LDS lacks
    if constexpr (DEEP) {
        a = shifted(a, coefs.first * (square * scale * scale));
        __syncthreads();
        put(A, a);
        if (!fresh) {
            v4d q;
#pragma unroll
            for (int r = 0; r < 4; ++r) q[r] = F[matrix * P * P + (row + 4 * r) * P + col];
            put(Q, q);
        }
        __syncthreads();
        by = 1.0;
    }
    for (int k = 0; k < steps; ++k) {
        const double ca = co[3 * k], cb = co[3 * k + 1], cc = co[3 * k + 2];
        double shift = 0.0;
        if constexpr (DEEP) {
            a = tile(A, ti, tj);  // the same on both sides of the diagonal
            shift = coefs.shift[k] * trace();
        }
        v4d p = product(A, A), t;
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_fma(cc, p[r] * by * by, __builtin_fma(cb, a[r], row + 4 * r == col ? ca : 0.0));
        if (fresh && steps == 1) {
            f = p;
            break;
        }
        put(S, p);
        __syncthreads();
        if (k + 1 == steps) {  // uniform
            f = product(S, Q);
            break;
        }
        if (fresh && k == 0) {
            f = p;
            t = product(S, A) * by;
            by = 1.0;
        } else {
            products(S, Q, A, &f, &t);
        }
        if constexpr (!ROOM) __syncthreads();
        put(free, f);
        put(T, t);
        if constexpr (ROOM) {
            char* const now = free;
            free = Q, Q = now;
        }
        __syncthreads();
        a = product(S, T);
        if constexpr (DEEP) a = shifted(a, shift);
        if constexpr (!ROOM) __syncthreads();
        put(A, a);
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (row + 4 * r >= col)
            F[matrix * P * P + (row + 4 * r) * P + col] = F[matrix * P * P + col * P + row + 4 * r] = f[r];
    if (fresh && threadIdx.x == 0) {
        scales[2 * matrix] = scale;
        scales[2 * matrix + 1] = norm < 0x1p-60 ? kFar : norm > 0x1p60 ? 1.0 / kFar : 1.0;
    }
}

// F X, 64 columns at a time: four waves take 16 each. F has values of a^5 = 485 where X has small singular values,
// whose products with the large ones cancel: an fp32 result is formed in 64 bits, or it would be off by 485
// roundings of X there (one for bf16 in 32, but for the larger F of many steps). 24 x 16384 fp32 4.9 us, which is latency.
template <int DG, int DO, bool MOMENTUM, int MT, bool WIDE>
__global__ __launch_bounds__(256) void orth_narrow_apply_kernel(Source s, const double* __restrict__ F, const double* __restrict__ scales,
                                                                Result res) {
    constexpr int P = 16 * MT;
    using Value = std::conditional_t<WIDE, double, float>;
    using Sums = std::conditional_t<WIDE, v4d, v4f>;
    __shared__ float slab[P * kSlabPitch];
    __shared__ Value f[P * P];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y, base = (res.first + matrix) * res.rows * res.cols;
    const int64_t n = res.tall ? res.rows : res.cols, pace = static_cast<int64_t>(gridDim.x) * kSlab;
    Slab<DG, MOMENTUM, MT> x(s, base, res.rows, res.cols);
    x.fetch(static_cast<int64_t>(blockIdx.x) * kSlab);
    for (int k = threadIdx.x; k < P * P; k += 256) f[k] = static_cast<Value>(F[matrix * P * P + k]);
    const double scale = scales[2 * matrix];
    const float rate = res.update && res.lr_at ? res.lr * *res.lr_at : res.lr;
    const float shrink = 1.f - rate * res.decay, by = rate * res.scale;
    for (int64_t j0 = static_cast<int64_t>(blockIdx.x) * kSlab; j0 < n; j0 += pace) {
        __syncthreads();
        x.template put<false, !WIDE>(j0, slab, scale);
        __syncthreads();
        x.fetch(j0 + pace);
        v4f old[MT];
        if (res.update)
#pragma unroll
            for (int q = 0; q < MT; ++q) {
                int64_t at;
                int line, c;
                const int64_t there = x.where(q, j0, &at, &line, &c);
                old[q] = read4<DO>(res.out, at, there);
            }
        Sums acc[MT] = {};
#pragma unroll 4
        for (int k = 0; k < P; k += 4) {
            const int at = k + (lane >> 4);
            const Value v = slab[at * kSlabPitch + 16 * wave + (lane & 15)];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const Value c = f[at * P + 16 * t + (lane & 15)];
                if constexpr (WIDE)
                    acc[t] = mfma_f64(c, v, acc[t]);
                else
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(c, v, acc[t], 0, 0, 0);
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + (WIDE ? 4 * r + (lane >> 4) : 4 * (lane >> 4) + r);
                slab[row * kSlabPitch + 16 * wave + (lane & 15)] = WIDE ? static_cast<float>(acc[t][r] * scale) : acc[t][r];
            }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < MT; ++q) {
            int64_t at;
            int line, c;
            const int64_t there = x.where(q, j0, &at, &line, &c);
            v4f v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = *x.value(slab, line, c + e);
                if (res.update) v[e] = __builtin_fmaf(-by, v[e], shrink * old[q][e]);
            }
            write4<DO>(res.out, at, there, v);
        }
    }
}

// ---------------------------------------------------------------------------
// The same for bf16 matrices with fewer rows than columns, and a bf16 result
// ---------------------------------------------------------------------------
// The matrix cores take the values as they lie in memory: eight neighbours of a row are what a lane of a product
// of rows has, and products of bf16 values are exact in fp32. Their sums over `run` columns, 64 or 256, are fp32 numbers (off
// by 2^-24 of them at most a few times, at random), the sums of those 64-bit ones: enough for a bf16 result
// where the steps multiply an error by 12 four times. A block whose squares leave fp32's range takes its columns
// again with values far from it (2^80 times or 2^-80 times them, which is exact). 32 matrices of 80 x 32768 take
// 36 us, 4.7 TB/s (by 64-bit products four times as long; with registers for one wave a SIMD 47).
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v4f mfma_b16(const v4u a, const v4u b, const v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

typedef uint32_t v4u_at2 __attribute__((ext_vector_type(4), aligned(2)));

// Eight neighbouring bf16 values, of which `n` are there, zeros behind.
__device__ __forceinline__ v4u read8(const void* G, int64_t at, int64_t n) {
    const uint16_t* p = static_cast<const uint16_t*>(G) + at;
    if (n >= 8) return *reinterpret_cast<const v4u_at2*>(p);
    v4u v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) v[e / 2] |= static_cast<uint32_t>(p[e]) << (16 * (e & 1));
    return v;
}

// The eight values times `by`, a power of two.
__device__ __forceinline__ v4u times(const v4u v, float by) {
    v4u w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(__uint_as_float(v[e] << 16) * by, __uint_as_float(v[e] & 0xffff0000u) * by);
    return w;
}

template <int MT>
__global__ __launch_bounds__(256, 2) void orth_narrow16_gram_kernel(const void* __restrict__ G, double* __restrict__ part, int m, int64_t n,
                                                                 int run, int64_t first) {
    constexpr int TILES = tri(MT);
    __shared__ double joint[TILES * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t matrix = blockIdx.y, base = (first + matrix) * m * n;
    const int64_t pace = static_cast<int64_t>(gridDim.x) * 4 * run;
    v4u x[2][MT];  // 64 columns: each half is asked for again as soon as it has been multiplied
    const uint32_t own = static_cast<uint32_t>(((lane & 15) * n + 8 * (lane >> 4)) * 2);
    const bool there = 16 * (MT - 1) + (lane & 15) < m;  // rows behind the last one are zeros
    auto fetch = [&](int k, int64_t j0) {
        const int64_t j = j0 + 32 * k;  // uniform over the wave
        const char* g = static_cast<const char*>(G) + 2 * (base + j);
        if (j + 32 <= n) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
                x[k][t] = t + 1 < MT || there ? v4u(*reinterpret_cast<const v4u_at2*>(g + 32 * t * n + own)) : v4u{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int row = 16 * t + (lane & 15);
                x[k][t] = read8(G, base + row * n + j + 8 * (lane >> 4), row < m ? n - j - 8 * (lane >> 4) : 0);
            }
        }
    };
    auto sums = [&](auto scaled, float by) {
        v4d acc[TILES] = {};
        int64_t j0 = (static_cast<int64_t>(blockIdx.x) * 4 + wave) * run;
        fetch(0, j0);
        fetch(1, j0);
        for (; j0 < n; j0 += pace) {
            v4f sum[TILES] = {};
#pragma unroll 1
            for (int c = 0; c < run; c += 64) {
                const int64_t j1 = c + 64 < run ? j0 + c + 64 : j0 + pace;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if constexpr (decltype(scaled)::value)
#pragma unroll
                        for (int t = 0; t < MT; ++t) x[k][t] = times(x[k][t], by);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int j = 0; j <= i; ++j) sum[tri(i) + j] = mfma_b16(x[k][i], x[k][j], sum[tri(i) + j]);
                    __builtin_amdgcn_sched_barrier(0);  // or both halves would need registers twice
                    fetch(k, j1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][r] += static_cast<double>(sum[t][r]);
        }
        const double back = 1.0 / (static_cast<double>(by) * by);
        for (int w = 0; w < 4; ++w) {  // the waves' sums, in their order
            if (wave == w) {
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        double* at = &joint[t * 256 + (4 * (lane >> 4) + r) * 16 + (lane & 15)];
                        const double v = decltype(scaled)::value ? acc[t][r] * back : acc[t][r];
                        *at = w == 0 ? v : *at + v;
                    }
            }
            __syncthreads();
        }
    };
    sums(std::false_type{}, 1.f);
    double squares = 0.0;  // the same in every wave
    for (int k = lane; k < 16 * MT; k += 64) squares += joint[(tri(k / 16) + k / 16) * 256 + 17 * (k % 16)];
#pragma unroll
    for (int k = 1; k < 64; k *= 2) squares += __shfl_xor(squares, k);
    // below 2^-80 the up to 2^20 products lost under 2^-126 would be more than 2^-26 of it
    if (!(squares >= 0x1p-80 && squares < __builtin_inf())) {
        __syncthreads();
        sums(std::true_type{}, static_cast<float>(squares < 0x1p-80 ? kFar : 1.0 / kFar));
    }
    for (int k = threadIdx.x; k < TILES * 256; k += 256) part[(matrix * gridDim.x + blockIdx.x) * (TILES * 256) + k] = joint[k];
}

// F X with F as three bf16 values, which are all its fp32 bits. A wave has 128 columns: its lanes read 16 bytes of
// eight rows each, and of eight columns the rows' values are paired for the products, whose results are 16 bytes
// of a row again. 32 matrices of 80 x 32768 69 us, 4.8 TB/s.
template <int MT>
__global__ __launch_bounds__(256) void orth_narrow16_apply_kernel(const void* __restrict__ G, const double* __restrict__ F,
                                                                  const double* __restrict__ scales, void* __restrict__ out, int m,
                                                                  int64_t n, int64_t first) {
    constexpr int P = 16 * MT, KS = (P + 31) / 32;
    __shared__ v4u f[MT][KS][3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y, base = (first + matrix) * m * n;
    const double up = scales[2 * matrix + 1], scale = scales[2 * matrix] / up;
    const bool far = up != 1.0;  // values that many times, and F less by it
    for (int q = wave; q < MT * KS; q += 4) {
        const int t = q / KS, k = q % KS, row = 16 * t + (lane & 15), col = 32 * k + 8 * (lane >> 4);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = col < P ? static_cast<float>(F[matrix * P * P + row * P + col + e] * scale) : 0.f;
#pragma unroll
        for (int part = 0; part < 3; ++part) {
            v4u w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                v[2 * e] -= __uint_as_float(w[e] << 16);
                v[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
            }
            f[t][k][part][lane] = w;
        }
    }
    __syncthreads();
    for (int64_t j0 = (static_cast<int64_t>(blockIdx.x) * 4 + wave) * 128; j0 < n; j0 += static_cast<int64_t>(gridDim.x) * 512) {
        const int64_t j = j0 + 8 * (lane & 15), there = n - j;
        v4u x[KS][8];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int row = 32 * k + 8 * (lane >> 4) + r;
                x[k][r] = read8(G, base + row * n + j, row < m ? there : 0);
            }
        if (far)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int r = 0; r < 8; ++r) x[k][r] = times(x[k][r], static_cast<float>(up));
        // column c of the eight rows: halves of the words c / 2, paired
        auto column = [&](int k, int c) {
            v4u b;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                b[e] = __builtin_amdgcn_perm(x[k][2 * e + 1][c / 2], x[k][2 * e][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
            return b;
        };
        v4u col[KS][8];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int c = 0; c < 8; ++c) col[k][c] = column(k, c);
#pragma unroll 1
        for (int t = 0; t < MT; ++t) {
            v4f acc[8] = {};
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    const v4u a = f[t][k][part][lane];
#pragma unroll
                    for (int c = 0; c < 8; ++c) acc[c] = mfma_b16(a, col[k][c], acc[c]);
                }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * (lane >> 4) + r;
                if (row >= m) continue;
                uint16_t* to = static_cast<uint16_t*>(out) + base + row * n + j;
                v4u_at2 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = pack_bf16(acc[2 * e][r], acc[2 * e + 1][r]);
                if (there >= 8) {
                    *reinterpret_cast<v4u_at2*>(to) = o;
                } else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < there) to[e] = static_cast<uint16_t>(o[e / 2] >> (16 * (e & 1)));
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int64_t kOrthMaxSide = int64_t(1) << 20;
constexpr int64_t kOrthMaxSmall = int64_t(1) << 16;  // of the smaller side: every grid stays below 2^32 threads
constexpr int64_t kOrthMaxValues = int64_t(1) << 46;
constexpr int64_t kOrthMaxMatrices = int64_t(1) << 26;
constexpr int64_t kGroupBytes = int64_t(1) << 30;  // of workspace, which matrices are taken together for
constexpr int kMostParts = 1024;
constexpr int64_t kGramBlocks = 512;

struct OrthShape {
    int64_t B, R, C;         // the caller's matrices
    int64_t m, n, mp, np;    // smaller and larger side, and with zeros around
    int64_t group;           // matrices at a time
    int mt;                  // tiles of 16 of a narrow matrix's smaller side, 0 for the others
    int64_t parts;           // sums of squares of a matrix, or of its blocks' G G^T
    int64_t x, xt, lo, a, e, d, more, bytes;  // bytes of a stored X, its other order, its lo, A, E, a diagonal, and the workspace
};

// split: products of two pieces each, which fp32 results have and the first steps of many for bf16 ones. What those take of
// the workspace is a bf16 result's, and one matrix's at least.
int orth_shape(int64_t B, int64_t R, int64_t C, int dtype, bool split, OrthShape* s) {
    if (B < 0 || R < 0 || C < 0 || B > kOrthMaxMatrices || R > kOrthMaxSide || C > kOrthMaxSide) return BIRKHOFF4_ERR_SIZE;
    if (!dtype_ok(dtype)) return BIRKHOFF4_ERR_DTYPE;
    if (R > 0 && C > 0 && B > kOrthMaxValues / (R * C)) return BIRKHOFF4_ERR_SIZE;
    *s = {};
    s->B = B, s->R = R, s->C = C;
    if (B == 0 || R == 0 || C == 0) return BIRKHOFF4_OK;
    s->m = R < C ? R : C;
    s->n = R < C ? C : R;
    if (s->m > kOrthMaxSmall) return BIRKHOFF4_ERR_SIZE;
    if (s->m <= kNarrow) {
        s->mt = static_cast<int>((s->m + 15) / 16);
        const int64_t slabs = (s->n + kSlab - 1) / kSlab, entries = tri(s->mt) * 256 * 8;
        s->e = entries;               // the sum of the parts
        s->x = s->mt * s->mt * 2048;  // F
        s->group = kGroupBytes / (s->e + s->x + 16);
        if (s->group > B) s->group = B;
        if (s->group > 32768) s->group = 32768;
        s->parts = kGramBlocks / s->group;
        if (s->parts > slabs) s->parts = slabs;
        if (s->parts < 1) s->parts = 1;
        s->a = s->parts > 1 ? s->parts * entries : 0;  // the parts
        s->bytes = s->group * (s->a + s->e + s->x + 16);
        return BIRKHOFF4_OK;
    }
    s->mp = (s->m + kPad - 1) / kPad * kPad;
    s->np = (s->n + kPad - 1) / kPad * kPad;
    s->d = s->mp * 4;
    auto each = [&](bool pieces) {  // bytes of one matrix
        const int64_t size = pieces ? 4 : 2;
        s->x = s->xt = s->mp * s->np * size;
        s->lo = pieces ? 0 : s->mp * s->np * 2;
        s->e = s->mp * s->mp * size;  // E, and A without its lo
        s->a = s->e + (pieces ? 0 : s->e);
        // of steps without X: their products, which an update may take (and never does nearer to a square)
        s->more = dtype == BIRKHOFF4_F32 && 4 * s->np >= 5 * s->mp ? 3 * s->e + 3 * s->mp * 4 : 0;
        return 2 * (s->x + s->xt + s->lo) + s->a + s->e + 2 * s->d + s->more + kMostParts * 8;
    };
    const int64_t turns = (R * C + 16 * kPrepBlock - 1) / (16 * kPrepBlock);
    s->parts = turns < kMostParts ? turns : kMostParts;
    auto fit = [&](int64_t bytes, int64_t one) {
        int64_t group = bytes / one;
        if (group < 1) group = 1;
        if (group > B) group = B;
        return group > 32768 ? 32768 : group;
    };
    const int64_t pieces = each(true), usual = each(dtype == BIRKHOFF4_F32);
    s->group = fit(kGroupBytes, usual);
    s->bytes = s->group * usual > pieces ? s->group * usual : pieces;
    if (split) s->group = fit(s->bytes, each(true));
    return BIRKHOFF4_OK;
}

struct OrthCall {
    Source src;
    Result res;
    const float* coefs;
    int steps;
    double eps;
    bool deep;  // more growth than kMostGrowth
};

// The most of |a + b t + c t^2|, t the square of a singular value from 0 to sqrt(2), and at least one. (A larger
// one that a step leaves below 2 has grown by less than sqrt(2), which the room from 8 to 16 is for.)
double most_of(const float* c) {
    auto at = [&](double t) { return __builtin_fabs(c[0] + t * (c[1] + t * static_cast<double>(c[2]))); };
    double most = 1.0;
    for (const double t : {0.0, 2.0, c[2] != 0.f ? -0.5 * c[1] / c[2] : 0.0})
        if (t >= 0.0 && t <= 2.0 && at(t) > most) most = at(t);
    return most;
}

// What the steps may multiply a small value by (five of the usual ones have 485) where
//   * those of a narrow matrix are taken in one run (24 x 1024 of rank one in fp32: eight of them are 3e-5 off, ten 5e-2);
//   * a bf16 result's products are of one piece each, whose roundings grow by as much: of 1280 x 6000 with singular values
//     from 1 to 1e-7, five are 1.7e-3 off, which is the result's own rounding. The steps in front of the last ones take two
//     pieces, 725 instead of 325 us each of 4096 x 4096: eight of them are 4.0e-3 off (with one piece throughout 5.9e-3) and 25
//     1.7e-3 (1.3e-2), of 150 x 260 of rank one eight 1.9e-3 (4.2e-2; in fp32 products 4e-3).
constexpr double kMostGrowth = 512.0;
constexpr double kNarrowFirst = 64.0;  // in the first run of more

double growth_of(const float* coefs, int steps) {
    double growth = 1.0;
    for (int k = 0; k < steps; ++k) growth *= most_of(coefs + 3 * k);
    return growth;
}

template <int DG, int DO, bool MOMENTUM, int MT>
int launch_narrow(const OrthShape& s, const OrthCall& call, char* work, hipStream_t stream) {
    constexpr bool WIDE = DO == BIRKHOFF4_F32;
    double* sum = reinterpret_cast<double*>(work);
    double* scales = reinterpret_cast<double*>(work + s.group * s.e);
    double* F = reinterpret_cast<double*>(work + s.group * (s.e + 16));
    const bool deep = call.deep;
    int begin = 0;  // steps of the first run
    while (begin < call.steps && growth_of(call.coefs, begin + 1) <= kNarrowFirst) ++begin;
    const bool rows16 = DG == BIRKHOFF4_BF16 && DO == BIRKHOFF4_BF16 && !MOMENTUM && s.R <= s.C && !deep;
    // long sums where they leave a block for every compute unit
    const int run = s.group * ((s.n + 1023) / 1024) >= 256 ? 256 : 64;
    const int64_t most = rows16 ? (s.n + 4 * run - 1) / (4 * run) : s.parts, parts = s.parts < most ? s.parts : most;
    double* part = parts > 1 ? reinterpret_cast<double*>(work + s.group * (s.e + 16 + s.x)) : sum;
    Coefs coefs = {};
    for (int k = 0; k < 3 * call.steps; ++k) coefs.v[k] = call.coefs[k];
    const int64_t slabs = (s.n + kSlab - 1) / kSlab;
    DeepCoefs start = {coefs}, rest = {};
    if (deep) {
        // A's entries are sums of that many products, one after the other. A step is two products of P terms and p itself,
        // of matrices of which |p| may be as large as `most`, and whose Frobenius norms are up to sqrt(P) times their largest value.
        constexpr double P = 16 * MT;
        rest.first = static_cast<float>(((slabs + parts - 1) / parts * kSlab + parts / 16 + 32) * 0x1p-53);
        for (int k = begin; k < call.steps; ++k) {
            const double p = most_of(call.coefs + 3 * k);
            for (int e = 0; e < 3; ++e) rest.v[3 * (k - begin) + e] = call.coefs[3 * k + e];
            rest.shift[k - begin] = static_cast<float>(2.0 * P * __builtin_sqrt(P) * 0x1p-53 * p * p);
        }
        rest.again = begin > 0;
    }
    for (int64_t first = 0; first < s.B; first += s.group) {
        const unsigned L = static_cast<unsigned>(s.B - first < s.group ? s.B - first : s.group);
        auto join = [&] {
            if (parts > 1)
                launch_kernel(orth_narrow_join_kernel, dim3(16 * tri(MT), L), dim3(256), 0, stream, part, sum,
                              static_cast<int>(parts), 256 * tri(MT));
        };
        if (rows16)
            launch_kernel(orth_narrow16_gram_kernel<MT>, dim3(static_cast<unsigned>(parts), L), dim3(256), 0, stream, call.src.G,
                          part, static_cast<int>(s.m), s.n, run, first);
        else
            launch_kernel((orth_narrow_gram_kernel<DG, MOMENTUM, MT>), dim3(static_cast<unsigned>(parts), L), dim3(kGramBlock), 0,
                          stream, call.src, part, s.R, s.C, first);
        join();
        if (!deep) {
            launch_kernel((orth_narrow_poly_kernel<MT, false>), dim3(L), dim3(64 * tri(MT)), 0, stream, sum, F, scales, call.eps, coefs,
                          call.steps);
        } else {
            if (begin > 0) {
                launch_kernel((orth_narrow_poly_kernel<MT, true>), dim3(L), dim3(64 * tri(MT)), 0, stream, sum, F, scales, call.eps,
                              start, begin);
                launch_kernel((orth_narrow_again_kernel<DG, MOMENTUM, MT>), dim3(static_cast<unsigned>(parts), L), dim3(kGramBlock), 0,
                              stream, call.src, F, scales, part, s.R, s.C, first);
                join();
            }
            launch_kernel((orth_narrow_poly_kernel<MT, true>), dim3(L), dim3(64 * tri(MT)), 0, stream, sum, F, scales, call.eps, rest,
                          call.steps - begin);
        }
        Result res = call.res;
        res.first = first;
        const int64_t turns = rows16 ? (s.n + 511) / 512 : slabs;  // what a block takes at a time
        int64_t blocks = kGramBlocks / L;  // two a compute unit (four: 32 of 80 x 32768 bf16 76 us instead of 69)
        if (blocks < 1) blocks = 1;
        if (blocks > turns) blocks = turns;
        if (rows16) {
            launch_kernel(orth_narrow16_apply_kernel<MT>, dim3(static_cast<unsigned>(blocks), L), dim3(256), 0, stream, call.src.G, F,
                          scales, res.out, static_cast<int>(s.m), s.n, first);
        } else {
            auto kern = deep ? orth_narrow_apply_kernel<DG, DO, MOMENTUM, MT, true> : orth_narrow_apply_kernel<DG, DO, MOMENTUM, MT, WIDE>;
            launch_kernel(kern, dim3(static_cast<unsigned>(blocks), L), dim3(256), 0, stream, call.src, F, scales, res);
        }
    }
    return launch_status();
}

// The tile and the groups of a product: the one of least time, by what a block takes for its panels with few and
// with all compute units busy (us a panel; the matrix cores' clock and L2 are shared) and for its beginning
// and end, fitted to products of 128 to 4096 rows. Measured (us): (A X) of 2560 x 10240 in fp32 128 x 128 383, in
// two groups 415, 192 x 192 374, 64 x 64 554; X X^T of it 217, 201, 325, 339, of 1000 x 2565 43, 39, 78, 22; of
// 4096 x 4096 in bf16 107, 112, 84, 167. 64 x 64 in one group is for many small matrices: 100 of 128 x 128 in fp32 183 -> 120
// for all steps, 48 of 128 x 512 in bf16 120 -> 110.
struct Tile {
    int w, groups, slots;  // its side in 64s, and how many blocks run at once
    double few, all, ends;
};
constexpr Tile kTiles[2][5] = {{{1, 2, 512, 0.20, 0.46, 4.0},
                              {2, 1, 512, 0.21, 0.45, 9.0},
                              {2, 2, 256, 0.33, 0.50, 9.0},
                              {1, 1, 1024, 0.20, 0.46, 4.0},
                              {3, 1, 256, 0.36, 0.62, 12.0}},
                             {{1, 4, 256, 0.40, 0.53, 4.0},
                              {2, 1, 512, 0.23, 0.55, 8.0},
                              {2, 2, 256, 0.42, 0.62, 8.5},
                              {1, 1, 1024, 0.25, 0.53, 4.0},
                              {3, 1, 256, 0.44, 0.75, 12.0}}};

int64_t tiles_of(int64_t rows, int64_t cols, bool half, int w, int64_t* tj) {
    const int64_t t = 64 * w, i = (rows + t - 1) / t, j = (cols + t - 1) / t;
    *tj = j;
    return half ? i * (i + 1) / 2 : i * j;
}

int choose_tile(bool split, bool half, bool last, int64_t L, int64_t rows, int64_t cols, int panels, double* time = nullptr) {
    int best = 0;
    double least = 0.0;
    for (int k = 0; k < (last ? 4 : 5); ++k) {  // with more to read at the end the largest tile does not fit the registers
        const Tile& t = kTiles[split][k];
        int64_t tj;
        const int64_t blocks = L * tiles_of(rows, cols, half, t.w, &tj), rest = blocks % t.slots;
        auto round = [&](double busy) { return panels / t.groups * (t.few + (t.all - t.few) * busy) + t.ends; };
        const double cost = blocks / t.slots * round(1.0) + (rest ? round(static_cast<double>(rest) / t.slots) : 0.0);
        if (k == 0 || cost < least) least = cost, best = k;
    }
    if (time) *time = least;
    return best;
}

template <bool SPLIT, int KIND, int DO>
void launch_product(Product g, const Result& res, int64_t group, unsigned L, int64_t rows, int64_t cols, hipStream_t stream) {
    // by the matrices of a full group, so that a batch's last ones are summed like the others
    constexpr bool HALF = KIND == GRAM || KIND == POLY || KIND == PAIR;
    const int k = choose_tile(SPLIT, HALF, KIND == LAST || KIND == PAIR, group, rows, cols, g.panels);
    const Tile& t = kTiles[SPLIT][k];
    int64_t tj;
    const int64_t tiles = tiles_of(rows, cols, HALF, t.w, &tj);
    g.tiles = static_cast<int>(tiles), g.tj = static_cast<int>(tj), g.matrices = static_cast<int>(L);
    auto kern = k == 0   ? orth_product_kernel<SPLIT, KIND, DO, 1, kTiles[SPLIT][0].groups>
                : k == 1 ? orth_product_kernel<SPLIT, KIND, DO, 2, 1>
                : k == 2 ? orth_product_kernel<SPLIT, KIND, DO, 2, 2> : orth_product_kernel<SPLIT, KIND, DO, 1, 1>;
    if constexpr (KIND != LAST && KIND != PAIR)
        if (k == 4) kern = orth_product_kernel<SPLIT, KIND, DO, 3, 1>;
    launch_kernel(kern, dim3(static_cast<unsigned>(8 * ((L * tiles + 7) / 8))), dim3(static_cast<unsigned>(256 * t.groups)), 0, stream, g,
                  res);
}

// Whether an update's steps are taken two or three at a time without X: X <- q X with q the product of the steps'
// p = a I + b A + c A^2, and A' = p A p instead of a new X X^T, all of them symmetric and of X's smaller side. For
// five steps two X X^T and two products with X instead of five, and nine more of the smaller side. An error of A
// is multiplied by up to a^2 = 12 a step, so A is formed anew after three. Directions off,
// with X every step, without it, and in fp32 products: 2560 x 10240 of eight strong directions among weak ones after five
// steps 1.6e-6, 6.5e-6 and 2.7e-6, after eight, whose runs are the worst of 2 to 12, 3.4e-6, 3.8e-5 and 1.1e-5; with independent
// values after five 1.7e-6, 6.8e-7 and 6e-6; of singular values from 1 to 1e-7 after five 5e-6, 2e-5 and 8e-6. An update's
// weights, of which they are a few hundredths, hardly show that, while an orthogonalised matrix would: only updates of fp32 weights
// take it. 2560 x 10240: 3240 -> 2030 us.
bool without_x(int64_t mp, int64_t np, int64_t L, int steps) {
    if (steps < 2) return false;
    const int runs = (steps + 2) / 3, along = static_cast<int>(np / panel_cols(true)), across = static_cast<int>(mp / panel_cols(true));
    double gram, poly, next;
    choose_tile(true, true, false, L, mp, mp, along, &gram);
    choose_tile(true, true, true, L, mp, mp, across, &poly);
    choose_tile(true, false, true, L, mp, np, across, &next);
    // a run of r steps: r polynomials, r - 1 products for q and 2 (r - 1) for A
    return runs * (gram + next) + (steps + 3 * (steps - runs)) * 1.1 * poly < 0.95 * steps * (gram + poly + next);
}

// The stored matrices of one form: X and its other order of this step and the next one's, A and E.
struct Stored {
    Plane x[2], xt[2], a, e;
};

// TWO: products of two pieces, of all steps for fp32 results, of all but the last ones for bf16 results. (The roundings of
// those that follow grow by kMostGrowth at most: five of the usual steps.)
template <int DG, int DO, bool MOMENTUM, bool TWO>
int launch_large(const OrthShape& s, const OrthCall& call, char* work, hipStream_t stream) {
    constexpr std::bool_constant<TWO> begun{};
    constexpr std::true_type two{};
    constexpr std::false_type one{};
    const bool tall = s.R > s.C;
    char* at = work;
    auto take = [&](int64_t bytes) {
        char* p = at;
        at += bytes * s.group;
        return bytes ? p : nullptr;
    };
    Stored p;
    for (int k = 0; k < 2; ++k) {
        p.x[k] = {take(s.x), nullptr, s.mp, s.x};
        p.xt[k] = {take(s.xt), nullptr, s.np, s.xt};
        p.xt[k].lo = take(s.lo);
    }
    p.a = {take(s.e), nullptr, s.mp, s.e};
    p.a.lo = take(TWO ? 0 : s.e);
    p.e = {take(s.e), nullptr, s.mp, s.e};
    Stored q = p;  // the form of one piece in the same places: half of each, and the lo in the other half
    if (TWO) q.xt[0].lo = p.xt[0].hi + s.xt / 2, q.xt[1].lo = p.xt[1].hi + s.xt / 2, q.a.lo = p.a.hi + s.e / 2;
    float* const da = reinterpret_cast<float*>(take(s.d));
    float* const de_first = reinterpret_cast<float*>(take(s.d));
    double* sums = reinterpret_cast<double*>(take(kMostParts * 8));
    char* const rest = at;  // s.more bytes a matrix
    int turn = 0;  // the first step of one piece
    if (DO == BIRKHOFF4_F32) turn = call.steps;
    else if (TWO)
        for (turn = call.steps - 1; turn > 0 && growth_of(call.coefs + 3 * (turn - 1), call.steps - turn + 1) <= kMostGrowth;) --turn;
    auto along = [&](auto split) { return static_cast<int>(s.np / panel_cols(decltype(split)::value)); };
    auto across = [&](auto split) { return static_cast<int>(s.mp / panel_cols(decltype(split)::value)); };
    for (int64_t first = 0; first < s.B; first += s.group) {
        const unsigned L = static_cast<unsigned>(s.B - first < s.group ? s.B - first : s.group);
        launch_kernel((orth_prep_kernel<DG, MOMENTUM>), dim3(static_cast<unsigned>(s.parts), L), dim3(kPrepBlock), 0, stream,
                      call.src, sums, s.R * s.C, first);
        const int64_t Rp = tall ? s.np : s.mp, Cp = tall ? s.mp : s.np;
        const int64_t tiles = Cp / kConvert * (Rp / kConvert);
        launch_kernel((orth_convert_kernel<DG, MOMENTUM, TWO>), dim3(static_cast<unsigned>((L * tiles + 7) / 8 * 8)), dim3(256), 0,
                      stream, call.src, sums, static_cast<int>(s.parts), call.eps, tall ? p.xt[0] : p.x[0], tall ? p.x[0] : p.xt[0], s.R,
                      s.C, first, L, static_cast<unsigned>(tiles), static_cast<unsigned>(Cp / kConvert));
        Result res = call.res;
        res.first = first;
        Plane e = p.e;  // which changes places with others below
        float* de = de_first;
        char* free = rest;
        [[maybe_unused]] auto take_more = [&](int64_t bytes) {
            char* p = free;
            free += bytes * s.group;
            return p;
        };
        auto gram = [&](auto split, const Stored& m, int now) {
            constexpr bool S = decltype(split)::value;
            launch_product<S, GRAM, S ? BIRKHOFF4_F32 : BIRKHOFF4_BF16>({m.x[now], m.x[now], {}, m.a, m.a, nullptr, da, 0.f, 0.f, nullptr, 0.f, s.mp,
                                                                         along(split), 0, 0, 0}, res, s.group, L, s.mp, s.mp, stream);
        };
        auto poly = [&](auto split, const Stored& m, const Plane& e, float* de, const float* c, float plus) {
            constexpr bool S = decltype(split)::value;
            launch_product<S, POLY, S ? BIRKHOFF4_F32 : BIRKHOFF4_BF16>({m.a, m.a, m.a, e, e, da, de, c[1], c[2], nullptr, plus, s.mp, across(split), 0,
                                                                         0, 0}, res, s.group, L, s.mp, s.mp, stream);
        };
        auto next = [&](auto split, const Stored& m, int now, const Plane& by, const float* diag, float keep, float add, bool last) {
            constexpr bool S = decltype(split)::value;
            const Product g = {by, m.xt[now], m.xt[now], m.x[now ^ 1], m.xt[now ^ 1], diag, nullptr, keep, add, nullptr, 0.f, s.mp, across(split), 0, 0, 0};
            if constexpr (S == (DO == BIRKHOFF4_F32))
                if (last) return launch_product<S, LAST, DO>(g, res, s.group, L, s.mp, s.np, stream);
            launch_product<S, NEXT, S ? BIRKHOFF4_F32 : BIRKHOFF4_BF16>(g, res, s.group, L, s.mp, s.np, stream);
        };
        if constexpr (MOMENTUM && DO == BIRKHOFF4_F32) {
            const int runs = (call.steps + 2) / 3;
            if (s.more && without_x(s.mp, s.np, s.group, call.steps)) {
                // q = p_k .. p_1 of a run and A' = p A p of its steps; a power of two keeps q's entries below 16
                const Plane& a = p.a;
                Plane t = e, q[2] = {e, e};
                t.hi = take_more(s.e), q[0].hi = take_more(s.e), q[1].hi = take_more(s.e);
                float* dt = reinterpret_cast<float*>(take_more(s.mp * 4));
                float* dq[2];
                for (float*& d : dq) d = reinterpret_cast<float*>(take_more(s.mp * 4));
                auto pair = [&](const Plane& M, const float* dm, const Plane& N, const float* dn, const Plane& to, float* d, float by) {
                    launch_product<true, PAIR, BIRKHOFF4_F32>({M, N, N, to, to, dm, d, 0.f, by, dn, 0.f, s.mp, across(two), 0, 0, 0}, res, s.group, L, s.mp, s.mp,
                                                    stream);
                };
                for (int run = 0, k = 0; run < runs; ++run) {
                    const int length = (call.steps - k) / (runs - run);  // the shorter ones first
                    gram(two, p, run & 1);
                    double most = 1.0;
                    float scale = 1.f;
                    Plane now = e;
                    float* dnow = de;
                    for (int i = 0; i < length; ++i, ++k) {
                        const float* c = call.coefs + 3 * k;
                        poly(two, p, e, de, c, c[0]);
                        most *= most_of(c);
                        if (i > 0) {
                            float by = 1.f;
                            while (scale * by * most > 8.0) by *= 0.5f;
                            scale *= by;
                            pair(e, de, now, dnow, q[i & 1], dq[i & 1], by);
                            now = q[i & 1], dnow = dq[i & 1];
                        }
                        if (i + 1 < length) {
                            pair(e, de, a, da, t, dt, 1.f);
                            pair(e, de, t, dt, a, da, 1.f);
                            if (i == 0) {  // the first p is q, and the next p comes elsewhere
                                std::swap(e.hi, q[0].hi);
                                std::swap(de, dq[0]);
                                now = q[0], dnow = dq[0];
                            }
                        }
                    }
                    next(two, p, run & 1, now, dnow, 0.f, 1.f / scale, run + 1 == runs);
                }
                continue;
            }
        }
        int now = 0;
        auto step = [&](auto split, const Stored& m, int k) {
            const float* c = call.coefs + 3 * k;
            gram(split, m, now);
            poly(split, m, m.e, de, c, 0.f);
            next(split, m, now, m.e, de, c[0], 1.f, k + 1 == call.steps);
            now ^= 1;
        };
        for (int k = 0; k < turn; ++k) step(begun, p, k);
        if constexpr (DO == BIRKHOFF4_BF16) {
            if (TWO) {
                const int64_t blocks = (s.mp * s.np / 8 + 255) / 256;
                const dim3 grid(static_cast<unsigned>(blocks < 4096 ? blocks : 4096), L);
                launch_kernel(orth_apart_kernel, grid, dim3(256), 0, stream, p.x[now], q.x[now ^ 1], s.np);
                launch_kernel(orth_apart_kernel, grid, dim3(256), 0, stream, p.xt[now], q.xt[now ^ 1], s.mp);
                now ^= 1;
            }
            for (int k = turn; k < call.steps; ++k) step(one, q, k);
        }
    }
    return launch_status();
}

template <int DG, int DO, bool MOMENTUM>
int launch_orth(const OrthShape& s, const OrthCall& call, char* work, hipStream_t stream) {
    switch (s.mt) {
        case 1: return launch_narrow<DG, DO, MOMENTUM, 1>(s, call, work, stream);
        case 2: return launch_narrow<DG, DO, MOMENTUM, 2>(s, call, work, stream);
        case 3: return launch_narrow<DG, DO, MOMENTUM, 3>(s, call, work, stream);
        case 4: return launch_narrow<DG, DO, MOMENTUM, 4>(s, call, work, stream);
        case 5: return launch_narrow<DG, DO, MOMENTUM, 5>(s, call, work, stream);
    }
    if constexpr (DO == BIRKHOFF4_BF16)
        if (!call.deep) return launch_large<DG, DO, MOMENTUM, false>(s, call, work, stream);
    return launch_large<DG, DO, MOMENTUM, true>(s, call, work, stream);
}

int64_t orth_work(int64_t B, int64_t R, int64_t C, int dtype) {
    OrthShape s;
    if (int e = orth_shape(B, R, C, dtype, false, &s)) return e;
    return s.bytes;
}

// The checks that both calls share, and the launches. `out`: what is written, W or the result.
int orth_call(const void* G, int g_dtype, float* M, float momentum, bool nesterov, void* out, int o_dtype, bool update, float lr,
              const float* lr_at, float decay, float scale, const float* coefs, int steps, float eps, void* work,
              int64_t work_bytes, int64_t B, int64_t R, int64_t C, hipStream_t stream) {
    const bool known = coefs && steps >= 1 && steps <= kOrthMaxSteps, deep = known && !(growth_of(coefs, steps) <= kMostGrowth);
    OrthShape s;
    if (int e = orth_shape(B, R, C, o_dtype, o_dtype == BIRKHOFF4_F32 || deep, &s)) return e;
    if (!dtype_ok(g_dtype)) return BIRKHOFF4_ERR_DTYPE;
    if (steps < 1 || steps > kOrthMaxSteps) return BIRKHOFF4_ERR_STEPS;
    if (!(eps >= 0.f && eps < __builtin_inff())) return BIRKHOFF4_ERR_EPS;
    if (!coefs) return BIRKHOFF4_ERR_NULL;
    if (B == 0 || R == 0 || C == 0) return BIRKHOFF4_OK;
    if (!G || !out || !work || (update && !M)) return BIRKHOFF4_ERR_NULL;
    if (work_bytes < s.bytes) return BIRKHOFF4_ERR_WORK;
    // the caller's arrays may begin at any value
    auto off = [](const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; };
    if (off(G, dtype_bytes(g_dtype)) || off(out, dtype_bytes(o_dtype)) || off(M, 4) || off(lr_at, 4) || misaligned(work))
        return BIRKHOFF4_ERR_ALIGN;
    const size_t values = static_cast<size_t>(B) * R * C;
    const Span ins[] = {{G, values * dtype_bytes(g_dtype)}, {lr_at, 4}};
    const Span outs[] = {{out, values * dtype_bytes(o_dtype)}, {M, values * 4}, {work, static_cast<size_t>(s.bytes)}};
    if (!disjoint(outs, 3, ins, 2)) return BIRKHOFF4_ERR_OVERLAP;
    const OrthCall call = {{G, M, momentum, nesterov}, {out, R, C, 0, R > C, update, lr, decay, scale, lr_at}, coefs, steps, eps, deep};
    constexpr int F = BIRKHOFF4_F32, H = BIRKHOFF4_BF16;
    auto pick = [&](auto plain, auto with) { return update ? with : plain; };
    auto launch = g_dtype == H ? (o_dtype == H ? pick(launch_orth<H, H, false>, launch_orth<H, H, true>)
                                               : pick(launch_orth<H, F, false>, launch_orth<H, F, true>))
                               : (o_dtype == H ? pick(launch_orth<F, H, false>, launch_orth<F, H, true>)
                                               : pick(launch_orth<F, F, false>, launch_orth<F, F, true>));
    return launch(s, call, static_cast<char*>(work), stream);
}

}  // namespace

extern "C" {

int64_t birkhoff4_orth_work(int64_t B, int64_t rows, int64_t cols, int out_dtype) { return orth_work(B, rows, cols, out_dtype); }

int birkhoff4_orth(const void* G, int g_dtype, void* out, int out_dtype, const float* coefs, int steps, float eps, void* work,
                   int64_t work_bytes, int64_t B, int64_t rows, int64_t cols, hipStream_t stream) {
    return orth_call(G, g_dtype, nullptr, 0.f, false, out, out_dtype, false, 1.f, nullptr, 0.f, 1.f, coefs, steps, eps, work,
                     work_bytes, B, rows, cols, stream);
}

int birkhoff4_orth_step(void* W, int w_dtype, const void* G, int g_dtype, float* M, float momentum, int nesterov, float lr,
                        const float* lr_at, float decay, float scale, const float* coefs, int steps, float eps, void* work,
                        int64_t work_bytes, int64_t B, int64_t rows, int64_t cols, hipStream_t stream) {
    return orth_call(G, g_dtype, M, momentum, nesterov != 0, W, w_dtype, true, lr, lr_at, decay, scale, coefs, steps,
                     eps, work, work_bytes, B, rows, cols, stream);
}

}  // extern "C"
