// orth.hip -- matrices taken towards their nearest (semi-)orthogonal ones by Newton-Schulz products, and
// the weight update with momentum around it, for gfx950 (MI355X).
//
// With m the smaller side of G and X = G / (|G|_F + eps) seen from it (m rows, n >= m columns):
//     A = X X^T,   E = b A + c A^2,   X <- a X + E X        (a, b, c of each step)
// An odd polynomial of X: it keeps the singular vectors and moves the singular values, p(s) = a s + b s^3 +
// c s^5. Every step is three products, 2 m^2 n + 2 m^3 + 2 m^2 n operations, of which the symmetric A and
// A^2 need one half: bound by the matrix cores but for small m.
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
// What is left, 0.2e-3 to 1.1e-3, is less than the result's own rounding to bf16, 1.7e-3.
//
// The products are of rows with rows (both operands have the summed index along their rows), so X is kept
// in both orders.

#include "common.h"

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v4u_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t v2u_at2 __attribute__((ext_vector_type(2), aligned(2)));

constexpr float kUnit = 4096.f;  // what values are stored in multiples of 1 / kUnit of
constexpr int kOrthMaxSteps = 64;
constexpr int kPad = 128;        // rows and columns of the stored matrices are whole multiples

// A stored matrix: rows of `pitch` bytes. SPLIT: lines of 128 bytes, 32 columns' hi and then their lo;
// otherwise hi alone, and lo, where it is kept, in a matrix of its own.
struct Plane {
    char* hi;
    char* lo;
    int64_t pitch;   // bytes of a row
    int64_t stride;  // bytes from one matrix of the batch to the next
};

template <bool SPLIT>
__device__ __forceinline__ int64_t place(const Plane& p, int64_t row, int64_t col) {
    return row * p.pitch + (SPLIT ? (col >> 5) * 128 + (col & 31) * 2 : col * 2);
}

// Eight columns from `col` (a multiple of eight) on.
template <bool SPLIT>
__device__ __forceinline__ void store8(const Plane& p, int64_t matrix, int64_t row, int64_t col, const float v[8]) {
    h8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        hi[e] = static_cast<_Float16>(v[e]);
        lo[e] = static_cast<_Float16>(v[e] - static_cast<float>(hi[e]));
    }
    const int64_t at = matrix * p.stride + place<SPLIT>(p, row, col);
    *reinterpret_cast<h8*>(p.hi + at) = hi;
    if constexpr (SPLIT)
        *reinterpret_cast<h8*>(p.hi + at + 64) = lo;
    else if (p.lo)
        *reinterpret_cast<h8*>(p.lo + at) = lo;
}

template <bool SPLIT>
__device__ __forceinline__ void load8(const Plane& p, int64_t matrix, int64_t row, int64_t col, float v[8]) {
    const int64_t at = matrix * p.stride + place<SPLIT>(p, row, col);
    const h8 hi = *reinterpret_cast<const h8*>(p.hi + at);
    const h8 lo = *reinterpret_cast<const h8*>(SPLIT ? p.hi + at + 64 : p.lo + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(hi[e]) + static_cast<float>(lo[e]);
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

// What is orthogonalised: G, or with a momentum M the direction G + ahead M (M renewed already).
struct Source {
    const void* G;
    float* M;
    float momentum, ahead;
};

// M <- momentum M + G where there is one, and the sum of squares of each matrix's direction in 64 bits (no
// finite fp32 matrix leaves its range): gridDim.x partial sums for each of gridDim.y matrices.
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
            u = s.ahead < 0.f ? *m : __builtin_fmaf(s.ahead, *m, g);
        }
        sum = __builtin_fma(static_cast<double>(u), static_cast<double>(u), sum);
    };
    const int64_t quads = values / 4;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * kPrepBlock + threadIdx.x; q < quads;
         q += static_cast<int64_t>(gridDim.x) * kPrepBlock) {
        float g[4], m[4] = {0.f, 0.f, 0.f, 0.f};
        load4<DG>(s.G, base + 4 * q, g);
        if constexpr (MOMENTUM) load4<BIRKHOFF4_F32>(s.M, base + 4 * q, m);
#pragma unroll
        for (int e = 0; e < 4; ++e) take(g[e], &m[e]);
        if constexpr (MOMENTUM) {
            v4u_at4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(m[e]);
            *reinterpret_cast<v4u_at4*>(s.M + base + 4 * q) = o;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x < values - 4 * quads) {
        const int64_t at = base + 4 * quads + threadIdx.x;
        float m = 0.f;
        if constexpr (MOMENTUM) m = s.M[at];
        take(load_value<DG>(s.G, at), &m);
        if constexpr (MOMENTUM) s.M[at] = m;
    }
    red[threadIdx.x] = sum;
    for (int half = kPrepBlock / 2; half > 0; half /= 2) {
        __syncthreads();
        if (threadIdx.x < half) red[threadIdx.x] += red[threadIdx.x + half];
    }
    if (threadIdx.x == 0) sums[matrix * gridDim.x + blockIdx.x] = red[0];
}

// The directions R x C over their norms, stored in their own order (own) and the other (turned), with zeros
// around: 64 x 64 values a block. A NaN or infinity anywhere makes the whole matrix NaN.
constexpr int kConvert = 64;

template <int DG, bool MOMENTUM, bool SPLIT>
__global__ __launch_bounds__(256) void orth_convert_kernel(Source s, const double* __restrict__ sums, int parts, double eps,
                                                           Plane own, Plane turned, int64_t R, int64_t C, int64_t first) {
    __shared__ float tile[kConvert][kConvert + 1];
    const int64_t matrix = blockIdx.z, base = (first + matrix) * R * C;
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kConvert, c0 = static_cast<int64_t>(blockIdx.x) * kConvert;
    double norm = 0.0;
    for (int k = 0; k < parts; ++k) norm += sums[matrix * parts + k];
    norm = __builtin_sqrt(norm);
    const double scale = norm < __builtin_inf() ? kUnit / (norm + eps) : __builtin_nan("");
    const int c = 4 * (threadIdx.x % 16);
#pragma unroll
    for (int k = 0; k < kConvert / 16; ++k) {
        const int r = threadIdx.x / 16 + 16 * k;
        const int64_t row = r0 + r, col = c0 + c, at = base + row * C + col;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (row < R && col < C) {
            float m[4] = {0.f, 0.f, 0.f, 0.f};
            if (col + 4 <= C) {
                load4<DG>(s.G, at, v);
                if constexpr (MOMENTUM) load4<BIRKHOFF4_F32>(s.M, at, m);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (col + e < C) {
                        v[e] = load_value<DG>(s.G, at + e);
                        if constexpr (MOMENTUM) m[e] = s.M[at + e];
                    }
            }
            if constexpr (MOMENTUM)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = s.ahead < 0.f ? m[e] : __builtin_fmaf(s.ahead, m[e], v[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = col + e < C ? static_cast<float>(v[e] * scale) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[r][c + e] = v[e];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int task = threadIdx.x + 256 * k, line = task / 8, at = 8 * (task % 8);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[line][at + e];
        store8<SPLIT>(own, matrix, r0 + line, c0 + at, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[at + e][line];
        store8<SPLIT>(turned, matrix, c0 + line, r0 + at, v);
    }
}

// ---------------------------------------------------------------------------
// The products
// ---------------------------------------------------------------------------
enum { GRAM, POLY, NEXT, LAST };

// acc_ij = sum_k P_ik Q_jk in units of kUnit^2. Results, stored as own_ij and as turned_ji:
//   GRAM  A = acc
//   POLY  E = keep A + add A^2 with A^2 from acc, src = A and its diagonal as above
//   NEXT  (keep + F_i) src_ij + acc, the next X;  LAST: the same, which goes to the caller's array
// GRAM and POLY have a symmetric result: its tiles below the diagonal alone are computed.
struct Product {
    Plane P, Q, src, own, turned;
    const float* src_diag;  // D (POLY) or F (NEXT, LAST), `side` a matrix
    float* own_diag;        // D (GRAM) or F (POLY)
    float keep, add;
    int64_t side;
    int lines;    // of 128 bytes in a row of P and Q
    int tj;       // tiles along j
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

constexpr int kTile = 128;
constexpr int kStage = 2 * kTile * 128;           // bytes of one step of both operands
constexpr int kTilePitch = kTile + 1;             // floats of a row of the finished tile
constexpr int kTileBytes = kTile * kTilePitch * 4;

template <bool SPLIT, int KIND, int DO>
__global__ __launch_bounds__(256) void orth_product_kernel(Product g, Result res) {
    static_assert(2 * kStage <= kTileBytes, "the finished tile takes the stages' place");
    __shared__ __attribute__((aligned(128))) char lds[kTileBytes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y;
    int ti, tj;
    if constexpr (KIND == GRAM || KIND == POLY) {  // row by row below the diagonal
        const int t = blockIdx.x;
        ti = static_cast<int>((__builtin_sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > t) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
        tj = t - ti * (ti + 1) / 2;
    } else {
        ti = blockIdx.x / g.tj;
        tj = blockIdx.x % g.tj;
    }
    const char* p = g.P.hi + matrix * g.P.stride + static_cast<int64_t>(ti) * kTile * g.P.pitch;
    const char* q = g.Q.hi + matrix * g.Q.stride + static_cast<int64_t>(tj) * kTile * g.Q.pitch;

    // A step is 128 bytes of 128 rows of both, loaded straight to LDS, eight rows an instruction. The
    // 16-byte piece c of row r lies at place c ^ (r mod 8) of its 128 bytes, so that the eight lanes that
    // read one piece of eight rows together find it in eight places.
    const int row8 = lane / 8, piece = (lane % 8) ^ row8;
    auto load = [&](int step, int buf) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = 8 * (4 * wave + k);
            const char* a = p + static_cast<int64_t>(r + row8) * g.P.pitch + static_cast<int64_t>(step) * 128 + 16 * piece;
            const char* b = q + static_cast<int64_t>(r + row8) * g.Q.pitch + static_cast<int64_t>(step) * 128 + 16 * piece;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)a,
                                             (__attribute__((address_space(3))) void*)(lds + buf * kStage + r * 128), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)b,
                                             (__attribute__((address_space(3))) void*)(lds + buf * kStage + kTile * 128 + r * 128),
                                             16, 0, 0);
        }
    };
    // a wave has 64 x 64 of the tile: 2 x 2 products of 32 x 32
    const int wi = 64 * (wave >> 1), wj = 64 * (wave & 1);
    v16f acc[2][2] = {};
    load(0, 0);
    for (int step = 0; step < g.lines; ++step) {
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this step's lines are there
        __syncthreads();                     // for all waves, and nobody reads the other stage any more
        const char* at = lds + (step & 1) * kStage;
        h8 a[2][4], b[2][4];  // pieces 2 c + lane / 32
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int r = 32 * t + (lane & 31), place = 16 * ((2 * c + (lane >> 5)) ^ (r & 7));
                a[t][c] = *reinterpret_cast<const h8*>(at + (wi + r) * 128 + place);
                b[t][c] = *reinterpret_cast<const h8*>(at + (kTile + wj + r) * 128 + place);
            }
        if (step + 1 < g.lines) load(step + 1, (step + 1) & 1);
#pragma unroll
        for (int c = 0; c < (SPLIT ? 2 : 4); ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][c], b[j][c], acc[i][j], 0, 0, 0);
                    if constexpr (SPLIT) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][c], b[j][c + 2], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][c + 2], b[j][c], acc[i][j], 0, 0, 0);
                    }
                }
    }
    __syncthreads();
    float* tile = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = wi + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, col = wj + 32 * j + (lane & 31);
                tile[row * kTilePitch + col] = acc[i][j][r];
            }
    __syncthreads();
    const int64_t i0 = static_cast<int64_t>(ti) * kTile, j0 = static_cast<int64_t>(tj) * kTile;
    const float* sd = KIND != GRAM ? g.src_diag + matrix * g.side : nullptr;
    float* od = KIND == GRAM || KIND == POLY ? g.own_diag + matrix * g.side : nullptr;
#pragma unroll 1
    for (int task = threadIdx.x; task < kTile * kTile / 8; task += 256) {
        const int r = task / 16, c = 8 * (task % 16);
        const bool diag = (KIND == GRAM || KIND == POLY) && ti == tj && r / 8 == c / 8;
        float v[8], s[8], di = 0.f;
        if constexpr (KIND != GRAM) {
            load8<SPLIT>(g.src, matrix, i0 + r, j0 + c, s);
            di = sd[i0 + r];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = tile[r * kTilePitch + c + e] / kUnit;
            if constexpr (KIND == GRAM) v[e] = t;
            if constexpr (KIND == POLY) v[e] = __builtin_fmaf(__builtin_fmaf(g.add, di + sd[j0 + c + e], g.keep), s[e], g.add * t);
            if constexpr (KIND == NEXT || KIND == LAST) v[e] = __builtin_fmaf(g.keep + di, s[e], t);
            if (diag && e == r % 8) {
                const float one = t / kUnit;
                if constexpr (KIND == GRAM) od[i0 + r] = one;
                if constexpr (KIND == POLY) od[i0 + r] = __builtin_fmaf(g.keep, di, g.add * __builtin_fmaf(di, di, one));
                v[e] = 0.f;
            }
            tile[r * kTilePitch + c + e] = v[e];
        }
        if constexpr (KIND != LAST) store8<SPLIT>(g.own, matrix, i0 + r, j0 + c, v);
    }
    if constexpr (KIND == GRAM || KIND == POLY)
        if (ti == tj) return;
    __syncthreads();
    if constexpr (KIND != LAST) {
#pragma unroll 1
        for (int task = threadIdx.x; task < kTile * kTile / 8; task += 256) {
            const int r = task / 16, c = 8 * (task % 16);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = tile[(c + e) * kTilePitch + r];
            store8<SPLIT>(g.turned, matrix, j0 + r, i0 + c, v);
        }
    } else {
        float rate = res.lr;
        if (res.update && res.lr_at) rate *= *res.lr_at;
        const float shrink = 1.f - rate * res.decay, by = rate * res.scale;
        const int64_t r0 = res.tall ? j0 : i0, c0 = res.tall ? i0 : j0;
        const int64_t base = (res.first + matrix) * res.rows * res.cols;
#pragma unroll 1
        for (int task = threadIdx.x; task < kTile * kTile; task += 256) {
            const int r = task / kTile, c = task % kTile;
            if (r0 + r >= res.rows || c0 + c >= res.cols) continue;
            float v = (res.tall ? tile[c * kTilePitch + r] : tile[r * kTilePitch + c]) / kUnit;
            const int64_t at = base + (r0 + r) * res.cols + c0 + c;
            if (res.update) v = __builtin_fmaf(-by, v, shrink * load_value<DO>(res.out, at));
            if constexpr (DO == BIRKHOFF4_BF16)
                static_cast<uint16_t*>(res.out)[at] = static_cast<uint16_t>(pack_bf16(v, 0.f));
            else
                static_cast<float*>(res.out)[at] = v;
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
// result is nearer than fp32 products bring it. The matrix cores' 64-bit rate is the limit of m: its cube
// runs on one compute unit a matrix (m = 80: 36 us of the matrix cores for five steps), and G G^T of 80 rows
// takes them half as long as reading fp32 G does. F X is formed in fp32.
constexpr int kNarrow = 80;
constexpr int kSlab = 64;            // columns of X taken at a time
constexpr int kSlabPitch = kSlab + 1;

typedef double v4d __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4d mfma_f64(double a, double b, v4d c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0); }

// X's rows (16 MT of them, zeros behind the m) and columns j0 .. j0 + 63 of a direction, from the caller's
// R x C array at `base`: X = U, or for a tall U its transpose. WRITE: renews M on the way.
template <int DG, bool MOMENTUM, bool WRITE, int MT>
__device__ __forceinline__ void load_slab(const Source& s, int64_t base, int64_t R, int64_t C, int64_t j0, float* slab) {
    const bool tall = R > C;
    const int m = static_cast<int>(tall ? C : R);
    const int64_t n = tall ? R : C;
    const int left = static_cast<int>(n - j0 < kSlab ? n - j0 : kSlab);
    // lines of the array: m rows of 64 values, or 64 rows of m, in pieces of four
    const int lines = tall ? kSlab : 16 * MT, quads = tall ? 4 * MT : kSlab / 4;
    const int used = tall ? left : m, width = tall ? m : left;
    for (int task = threadIdx.x; task < lines * quads; task += blockDim.x) {
        const int line = task / quads, c = 4 * (task % quads);
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (line < used && c < width) {
            const int64_t at = base + (tall ? (j0 + line) * C + c : line * C + j0 + c);
            float mv[4] = {0.f, 0.f, 0.f, 0.f};
            const bool whole = c + 4 <= width;
            if (whole) {
                load4<DG>(s.G, at, v);
                if constexpr (MOMENTUM) load4<BIRKHOFF4_F32>(s.M, at, mv);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (c + e < width) {
                        v[e] = load_value<DG>(s.G, at + e);
                        if constexpr (MOMENTUM) mv[e] = s.M[at + e];
                    }
            }
            if constexpr (MOMENTUM) {
                if constexpr (WRITE) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) mv[e] = __builtin_fmaf(s.momentum, mv[e], v[e]);
                    if (whole) {
                        v4u_at4 o;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(mv[e]);
                        *reinterpret_cast<v4u_at4*>(s.M + at) = o;
                    } else {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (c + e < width) s.M[at + e] = mv[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = s.ahead < 0.f ? mv[e] : __builtin_fmaf(s.ahead, mv[e], v[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) slab[tall ? (c + e) * kSlabPitch + line : line * kSlabPitch + c + e] = v[e];
    }
}

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
    for (int64_t j0 = static_cast<int64_t>(blockIdx.x) * kSlab; j0 < n; j0 += static_cast<int64_t>(gridDim.x) * kSlab) {
        __syncthreads();
        load_slab<DG, MOMENTUM, true, MT>(s, base, R, C, j0, slab);
        __syncthreads();
#pragma unroll 4
        for (int k = 0; k < kSlab; k += 4)
#pragma unroll
            for (int q = 0; q < OWN; ++q)
                if (wave + 4 * q < TILES)  // uniform over the wave
                    acc[q] = mfma_f64(slab[ri[q] + k], slab[rj[q] + k], acc[q]);
    }
    double* out = part + (matrix * gridDim.x + blockIdx.x) * (TILES * 256);
#pragma unroll
    for (int q = 0; q < OWN; ++q)
        if (wave + 4 * q < TILES)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[(wave + 4 * q) * 256 + (4 * r + (lane >> 4)) * 16 + (lane & 15)] = acc[q][r];
}

// The blocks' parts added, 64 entries a block in four parts of the order.
__global__ __launch_bounds__(256) void orth_narrow_join_kernel(const double* __restrict__ part, double* __restrict__ sum, int parts,
                                                               int entries) {
    __shared__ double red[4][64];
    const int c = threadIdx.x & 63, p = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y, at = static_cast<int64_t>(blockIdx.x) * 64 + c;
    double v = 0.0;
#pragma unroll 8
    for (int k = p; k < parts; k += 4) v += part[(matrix * parts + k) * entries + at];
    red[p][c] = v;
    __syncthreads();
    if (p == 0) sum[matrix * entries + at] = (v + red[1][c]) + (red[2][c] + red[3][c]);
}

// F of each matrix from its G G^T: one block a matrix, a wave for each tile. A matrix in LDS is
// symmetric, so its rows serve as both factors' columns: the lanes of 16 read 16 neighbours.
constexpr int kPolyBlock = 1024;

struct Coefs {
    float v[3 * kOrthMaxSteps];
};

template <int MT>
__global__ __launch_bounds__(kPolyBlock) void orth_narrow_poly_kernel(const double* __restrict__ sum, float* __restrict__ F,
                                                                      double* __restrict__ scales, double eps, Coefs coefs, int steps) {
    constexpr int P = 16 * MT;
    static_assert(tri(MT) <= kPolyBlock / 64, "a tile a wave");
    __shared__ double A[P * P], S[P * P], Q[P * P];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.x;
    int ti = 0;
    while (tri(ti + 1) <= wave) ++ti;
    const int tj = wave - tri(ti);
    const bool mine = wave < tri(MT);  // uniform over the wave
    const int row = 16 * ti + (lane >> 4), col = 16 * tj + (lane & 15);  // of value r: row + 4 r
    auto product = [&](const double* M, const double* N) {
        v4d acc = {};
        if (mine)
#pragma unroll 4
            for (int k = 0; k < P; k += 4)
                acc = mfma_f64(M[(k + (lane >> 4)) * P + 16 * ti + (lane & 15)], N[(k + (lane >> 4)) * P + 16 * tj + (lane & 15)], acc);
        return acc;
    };
    auto put = [&](double* M, const v4d& v) {
        if (mine)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (row + 4 * r >= col) M[(row + 4 * r) * P + col] = M[col * P + row + 4 * r] = v[r];
    };
    v4d a = {}, f = {};
    if (mine)
#pragma unroll
        for (int r = 0; r < 4; ++r) a[r] = sum[(matrix * tri(MT) + wave) * 256 + (4 * r + (lane >> 4)) * 16 + (lane & 15)];
    put(A, a);
    __syncthreads();
    double norm = 0.0;
    for (int k = 0; k < P; ++k) norm += A[k * P + k];
    norm = __builtin_sqrt(norm);
    const double scale = norm < __builtin_inf() ? 1.0 / (norm + eps) : __builtin_nan("");
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) a[r] = a[r] * scale * scale;
    put(A, a);
    __syncthreads();
    for (int k = 0; k < steps; ++k) {
        const double ca = coefs.v[3 * k], cb = coefs.v[3 * k + 1], cc = coefs.v[3 * k + 2];
        v4d p = product(A, A);
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_fma(cc, p[r], __builtin_fma(cb, a[r], row + 4 * r == col ? ca : 0.0));
        put(S, p);
        __syncthreads();
        const bool last = k + 1 == steps;  // uniform
        f = k == 0 ? p : product(S, Q);
        if (!last) a = product(S, A);
        __syncthreads();
        if (!last) {
            put(Q, f);
            put(A, a);
            __syncthreads();
            a = product(S, A);
            __syncthreads();
            put(A, a);
            __syncthreads();
        }
    }
    if (mine)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (row + 4 * r >= col)
                F[matrix * P * P + (row + 4 * r) * P + col] = F[matrix * P * P + col * P + row + 4 * r] = static_cast<float>(f[r]);
    if (threadIdx.x == 0) scales[matrix] = scale;
}

// F X, 64 columns at a time: four waves take 16 each.
template <int DG, int DO, bool MOMENTUM, int MT>
__global__ __launch_bounds__(256) void orth_narrow_apply_kernel(Source s, const float* __restrict__ F, const double* __restrict__ scales,
                                                                Result res) {
    constexpr int P = 16 * MT;
    __shared__ float slab[P * kSlabPitch];
    __shared__ float f[P * P];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t matrix = blockIdx.y, base = (res.first + matrix) * res.rows * res.cols;
    const int64_t n = res.tall ? res.rows : res.cols;
    const int m = static_cast<int>(res.tall ? res.cols : res.rows);
    for (int k = threadIdx.x; k < P * P; k += 256) f[k] = F[matrix * P * P + k];
    const double scale = scales[matrix];
    float rate = res.lr;
    if (res.update && res.lr_at) rate *= *res.lr_at;
    const float shrink = 1.f - rate * res.decay, by = rate * res.scale;
    for (int64_t j0 = static_cast<int64_t>(blockIdx.x) * kSlab; j0 < n; j0 += static_cast<int64_t>(gridDim.x) * kSlab) {
        __syncthreads();
        load_slab<DG, MOMENTUM, false, MT>(s, base, res.rows, res.cols, j0, slab);
        __syncthreads();
        v4f acc[MT] = {};
#pragma unroll 4
        for (int k = 0; k < P; k += 4) {
            const int at = k + (lane >> 4);
            const float x = static_cast<float>(slab[at * kSlabPitch + 16 * wave + (lane & 15)] * scale);
#pragma unroll
            for (int t = 0; t < MT; ++t)
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[at * P + 16 * t + (lane & 15)], x, acc[t], 0, 0, 0);
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) slab[(16 * t + 4 * (lane >> 4) + r) * kSlabPitch + 16 * wave + (lane & 15)] = acc[t][r];
        __syncthreads();
        const int left = static_cast<int>(n - j0 < kSlab ? n - j0 : kSlab);
        const int lines = res.tall ? left : m, width = res.tall ? m : left;
        for (int task = threadIdx.x; task < lines * width; task += 256) {
            const int line = task / width, c = task % width;
            float v = res.tall ? slab[c * kSlabPitch + line] : slab[line * kSlabPitch + c];
            const int64_t at = base + (res.tall ? (j0 + line) * res.cols + c : line * res.cols + j0 + c);
            if (res.update) v = __builtin_fmaf(-by, v, shrink * load_value<DO>(res.out, at));
            if constexpr (DO == BIRKHOFF4_BF16)
                static_cast<uint16_t*>(res.out)[at] = static_cast<uint16_t>(pack_bf16(v, 0.f));
            else
                static_cast<float*>(res.out)[at] = v;
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
constexpr int kMostParts = 128;
constexpr int64_t kGramBlocks = 512;

struct OrthShape {
    int64_t B, R, C;         // the caller's matrices
    int64_t m, n, mp, np;    // smaller and larger side, and with zeros around
    int64_t group;           // matrices at a time
    int mt;                  // tiles of 16 of a narrow matrix's smaller side, 0 for the others
    int64_t parts;           // sums of squares of a matrix, or of its blocks' G G^T
    int64_t x, xt, lo, a, e, d, bytes;  // bytes of a stored X, its other order, its lo, A, E, a diagonal, and the workspace
};

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
        s->x = s->mt * s->mt * 1024;  // F
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
    const int64_t size = split ? 4 : 2;
    s->x = s->xt = s->mp * s->np * size;
    s->lo = split ? 0 : s->mp * s->np * 2;
    s->a = s->mp * s->mp * 4;  // hi and lo
    s->e = s->mp * s->mp * size;
    s->d = s->mp * 4;
    const int64_t quads = (R * C + 4 * kPrepBlock - 1) / (4 * kPrepBlock);
    s->parts = quads < kMostParts ? quads : kMostParts;
    const int64_t each = 2 * (s->x + s->xt + s->lo) + s->a + s->e + 2 * s->d + kMostParts * 8;
    s->group = kGroupBytes / each;
    if (s->group < 1) s->group = 1;
    if (s->group > B) s->group = B;
    if (s->group > 32768) s->group = 32768;
    s->bytes = s->group * each;
    return BIRKHOFF4_OK;
}

struct OrthCall {
    Source src;
    Result res;
    const float* coefs;
    int steps;
    double eps;
};

template <int DG, int DO, bool MOMENTUM, int MT>
int launch_narrow(const OrthShape& s, const OrthCall& call, char* work, hipStream_t stream) {
    double* sum = reinterpret_cast<double*>(work);
    double* scales = reinterpret_cast<double*>(work + s.group * s.e);
    float* F = reinterpret_cast<float*>(work + s.group * (s.e + 16));
    double* part = s.parts > 1 ? reinterpret_cast<double*>(work + s.group * (s.e + 16 + s.x)) : sum;
    Coefs coefs = {};
    for (int k = 0; k < 3 * call.steps; ++k) coefs.v[k] = call.coefs[k];
    const int64_t slabs = (s.n + kSlab - 1) / kSlab;
    for (int64_t first = 0; first < s.B; first += s.group) {
        const unsigned L = static_cast<unsigned>(s.B - first < s.group ? s.B - first : s.group);
        launch_kernel((orth_narrow_gram_kernel<DG, MOMENTUM, MT>), dim3(static_cast<unsigned>(s.parts), L), dim3(kGramBlock), 0,
                      stream, call.src, part, s.R, s.C, first);
        if (s.parts > 1)
            launch_kernel(orth_narrow_join_kernel, dim3(4 * tri(MT), L), dim3(256), 0, stream, part, sum,
                          static_cast<int>(s.parts), 256 * tri(MT));
        launch_kernel((orth_narrow_poly_kernel<MT>), dim3(L), dim3(kPolyBlock), 0, stream, sum, F, scales, call.eps, coefs,
                      call.steps);
        Result res = call.res;
        res.first = first;
        int64_t blocks = 2 * kGramBlocks / L;
        if (blocks < 1) blocks = 1;
        if (blocks > slabs) blocks = slabs;
        launch_kernel((orth_narrow_apply_kernel<DG, DO, MOMENTUM, MT>), dim3(static_cast<unsigned>(blocks), L), dim3(256), 0,
                      stream, call.src, F, scales, res);
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
    constexpr bool SPLIT = DO == BIRKHOFF4_F32;
    constexpr int64_t W = SPLIT ? 4 : 2;
    const bool tall = s.R > s.C;
    char* at = work;
    auto take = [&](int64_t bytes) {
        char* p = at;
        at += bytes * s.group;
        return bytes ? p : nullptr;
    };
    Plane x[2], xt[2];
    for (int k = 0; k < 2; ++k) {
        x[k] = {take(s.x), nullptr, s.np * W, s.x};
        x[k].lo = take(s.lo);
        xt[k] = {take(s.xt), nullptr, s.mp * W, s.xt};
    }
    Plane a = {take(s.a), nullptr, s.mp * W, s.mp * s.mp * W};
    if (!SPLIT) a.lo = a.hi + s.group * s.mp * s.mp * 2;
    Plane e = {take(s.e), nullptr, s.mp * W, s.mp * s.mp * W};
    float* da = reinterpret_cast<float*>(take(s.d));
    float* de = reinterpret_cast<float*>(take(s.d));
    double* sums = reinterpret_cast<double*>(take(kMostParts * 8));
    for (int64_t first = 0; first < s.B; first += s.group) {
        const unsigned L = static_cast<unsigned>(s.B - first < s.group ? s.B - first : s.group);
        launch_kernel((orth_prep_kernel<DG, MOMENTUM>), dim3(static_cast<unsigned>(s.parts), L), dim3(kPrepBlock), 0, stream,
                      call.src, sums, s.R * s.C, first);
        const int64_t Rp = tall ? s.np : s.mp, Cp = tall ? s.mp : s.np;
        launch_kernel((orth_convert_kernel<DG, MOMENTUM, SPLIT>),
                      dim3(static_cast<unsigned>(Cp / kConvert), static_cast<unsigned>(Rp / kConvert), L), dim3(256), 0, stream,
                      call.src, sums, static_cast<int>(s.parts), call.eps, tall ? xt[0] : x[0], tall ? x[0] : xt[0], s.R, s.C, first);
        const int tm = static_cast<int>(s.mp / kTile), tn = static_cast<int>(s.np / kTile);
        const unsigned half = static_cast<unsigned>(tm) * (tm + 1) / 2;
        Result res = call.res;
        res.first = first;
        for (int k = 0; k < call.steps; ++k) {
            const float* c = call.coefs + 3 * k;
            const int now = k & 1;
            const int along = static_cast<int>(s.np * W / 128), across = static_cast<int>(s.mp * W / 128);
            Product g = {x[now], x[now], {}, a, a, nullptr, da, 0.f, 0.f, s.mp, along, tm};
            launch_kernel((orth_product_kernel<SPLIT, GRAM, DO>), dim3(half, L), dim3(256), 0, stream, g, res);
            g = {a, a, a, e, e, da, de, c[1], c[2], s.mp, across, tm};
            launch_kernel((orth_product_kernel<SPLIT, POLY, DO>), dim3(half, L), dim3(256), 0, stream, g, res);
            g = {e, xt[now], x[now], x[now ^ 1], xt[now ^ 1], de, nullptr, c[0], 0.f, s.mp, across, tn};
            auto last = k + 1 < call.steps ? orth_product_kernel<SPLIT, NEXT, DO> : orth_product_kernel<SPLIT, LAST, DO>;
            launch_kernel(last, dim3(static_cast<unsigned>(tm) * tn, L), dim3(256), 0, stream, g, res);
        }
    }
    return launch_status();
}

int64_t orth_work(int64_t B, int64_t R, int64_t C, int dtype) {
    OrthShape s;
    if (int e = orth_shape(B, R, C, dtype, dtype == BIRKHOFF4_F32, &s)) return e;
    return s.bytes;
}

// The checks that both calls share, and the launches. `out`: what is written, W or the result.
int orth_call(const void* G, int g_dtype, float* M, float momentum, float ahead, void* out, int o_dtype, bool update, float lr,
              const float* lr_at, float decay, float scale, const float* coefs, int steps, float eps, void* work,
              int64_t work_bytes, int64_t B, int64_t R, int64_t C, hipStream_t stream) {
    OrthShape s;
    if (int e = orth_shape(B, R, C, o_dtype, o_dtype == BIRKHOFF4_F32, &s)) return e;
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
    const OrthCall call = {{G, M, momentum, ahead}, {out, R, C, 0, R > C, update, lr, decay, scale, lr_at}, coefs, steps, eps};
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
    return orth_call(G, g_dtype, nullptr, 0.f, 0.f, out, out_dtype, false, 1.f, nullptr, 0.f, 1.f, coefs, steps, eps, work,
                     work_bytes, B, rows, cols, stream);
}

int birkhoff4_orth_step(void* W, int w_dtype, const void* G, int g_dtype, float* M, float momentum, int nesterov, float lr,
                        const float* lr_at, float decay, float scale, const float* coefs, int steps, float eps, void* work,
                        int64_t work_bytes, int64_t B, int64_t rows, int64_t cols, hipStream_t stream) {
    return orth_call(G, g_dtype, M, momentum, nesterov ? momentum : -1.f, W, w_dtype, true, lr, lr_at, decay, scale, coefs, steps,
                     eps, work, work_bytes, B, rows, cols, stream);
}

}  // extern "C"
