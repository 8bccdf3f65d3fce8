/*
 * birkhoff4.h -- batched 4x4 Birkhoff projection on AMD Instinct MI355X (gfx950).
 *
 * The forward pass projects exp(H[b]) onto the Birkhoff polytope of doubly
 * stochastic 4x4 matrices in the KL geometry (eq. birkhoff_projection), by
 * Newton's method on the reduced 3-dimensional entropic-OT dual (Sec. 3.1-3.2,
 * eq. min_fx, eq. grad_hess; cost M = -H, eta = 1, a = b = 1). The backward pass
 * maps dL/dP to dL/dH by implicit differentiation through the optimality
 * conditions (Sec. 4, eq. derivative, with the sign flip for H = -M), reading
 * only P and dP: no iterates or Hessians are stored.
 *
 * Conventions shared by every entry point
 *   - All array arguments are DEVICE pointers on the current HIP device; the
 *     caller owns them. The library never allocates, frees or synchronises.
 *   - Work is enqueued on `stream` (0 = the null stream) and the call returns
 *     at once; errors found on the host are returned before anything is queued.
 *   - 4x4 arrays are [B][4][4] row-major and contiguous: element (b,i,j) is at
 *     16*b + 4*i + j. `dual` is [B][8] = (alpha_1..alpha_4, beta_1..beta_4) with
 *     beta_4 = 0, so that log P_ij - H_ij = alpha_i + beta_j.
 *   - Every array must be 16-byte aligned, and no output may overlap another
 *     argument (in-place use is not supported).
 *   - B = 0 is a no-op returning BIRKHOFF4_OK.
 *   - Numerical outcomes are not errors: a matrix that does not reach `tol`
 *     within `max_iter` iterations returns its last accepted (row-stochastic)
 *     iterate; a matrix with a NaN or infinite entry returns NaN in all its
 *     outputs. The _ex variants report both cases per matrix.
 */
#ifndef BIRKHOFF4_H
#define BIRKHOFF4_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes. */
enum {
    BIRKHOFF4_OK = 0,
    BIRKHOFF4_ERR_NULL = -1,      /* a required pointer is NULL while B > 0 */
    BIRKHOFF4_ERR_SIZE = -2,      /* B < 0, or too large for the index type */
    BIRKHOFF4_ERR_TOL = -3,       /* tol < 0 or NaN */
    BIRKHOFF4_ERR_MAX_ITER = -4,  /* max_iter < 0 or > 10000 */
    BIRKHOFF4_ERR_DTYPE = -5,     /* unknown storage dtype code */
    BIRKHOFF4_ERR_ALIGN = -6,     /* an array is not 16-byte aligned */
    BIRKHOFF4_ERR_OVERLAP = -7,   /* an output overlaps another argument */
    BIRKHOFF4_ERR_STEPS = -8,     /* step count out of range: Sinkhorn's 1..48, the orthogonalisation's 1..64 */
    BIRKHOFF4_ERR_DEVICE = -9,    /* HIP device query failed */
    BIRKHOFF4_ERR_LAUNCH = -10,   /* kernel launch failed (hipGetLastError) */
    BIRKHOFF4_ERR_VARIANT = -11,  /* unknown forward variant */
    BIRKHOFF4_ERR_ETA = -12,      /* eta not positive and finite */
    BIRKHOFF4_ERR_CHANNELS = -13, /* width C negative, or zero or no whole number of 16-byte chunks where that is needed */
    BIRKHOFF4_ERR_EPS = -14,      /* eps negative, infinite or NaN */
    BIRKHOFF4_ERR_WORK = -15,     /* the workspace is smaller than the call's _work says */
    BIRKHOFF4_ERR_DROP = -16      /* dropout probability outside [0, 1) */
};

/* Forward kernel variants (birkhoff4_fwd_ex2). Both compute the same projection to the
 * same tolerance; they differ in how problems map to lanes, so iterates and step counts may
 * differ at the rounding level. */
enum {
    BIRKHOFF4_AUTO = 0,       /* LATENCY for B <= 32768, else THROUGHPUT */
    BIRKHOFF4_THROUGHPUT = 1, /* one problem per lane, with lane-level refill */
    BIRKHOFF4_LATENCY = 2     /* four lanes per problem (one row each), no refill */
};

/* Storage dtypes: of inputs, and of the outputs that a dtype argument names (dH of the _ex2 and
 * _ex backwards, the mixed streams); the others are fp32. Compute is always fp32. */
enum {
    BIRKHOFF4_F32 = 0,
    BIRKHOFF4_BF16 = 1
};

/* Per-matrix status codes written to `iters` by birkhoff4_fwd_ex (values >= 0
 * are the number of Newton trial steps taken, see below). */
enum {
    BIRKHOFF4_NOT_CONVERGED = -1, /* max_iter trial steps did not reach tol */
    BIRKHOFF4_NON_FINITE = -2     /* the input matrix had a NaN or infinite entry */
};

/* Forward projection, fp32 input.
 *
 * H     [B][4][4] fp32 logits (the paper's residual logits, R = -M).
 * P     [B][4][4] fp32 output: the projection, rows summing to one by
 *       construction and every column sum within `tol` of one on return.
 * dual  [B][8] fp32 output, or NULL to skip it: alpha*(beta*) (eq. alpha_opt)
 *       and beta* with beta_4 = 0 (Sec. 3.1 gauge).
 * tol   stopping tolerance on max_j |sum_i P_ij - 1| (the paper uses 1e-6);
 *       tol = 0 stops a matrix only when its fp32 column sums are exactly one,
 *       so in practice most run for max_iter trial steps.
 * max_iter  maximum number of Newton trial steps per matrix, 0..10000 (each is one
 *       evaluation of the dual at a trial point: a damped Newton step, or a
 *       backtracking of it with a larger Levenberg-Marquardt shift). 0 returns T at the initial point, which is the
 *       row softmax of H after the columns are centred (beta_j^(0) = mean of
 *       column 4 minus mean of column j). A step moves the column
 *       potentials apart by at most 8 (natural-log units), so logits whose
 *       solution lies far from the centred start need more: at H ~ N(0, s^2)
 *       64 steps converge every matrix up to s = 100 and leave up to 30 % at
 *       s = 500-1000, where 1000 steps converge them all.
 *   Range: finite logits up to about 5e37 in magnitude are handled; larger
 *       ones can overflow the fp32 scaling by log2(e) and are then reported
 *       like a non-finite input.
 */
int birkhoff4_fwd(const float* H, float* P, float* dual, int64_t B, float tol,
                  int max_iter, hipStream_t stream);

/* Backward (vector-Jacobian product), fp32 upstream gradient.
 *
 * P     [B][4][4] fp32: the projection returned by the forward pass (T*).
 * dual  accepted for symmetry with the forward pass and not read (the 4x4
 *       backward needs only T* and G, Sec. 4.2); may be NULL.
 * dP    [B][4][4] fp32: dL/dP (the paper's G).
 * dH    [B][4][4] fp32 output: dL/dH = -D of eq. derivative, with Delta taken as
 *       the Hessian of the reduced dual at P. Rows and columns of dH sum to zero.
 */
int birkhoff4_bwd(const float* P, const float* dual, const float* dP, float* dH,
                  int64_t B, hipStream_t stream);

/* Forward projection with a storage dtype for H and per-matrix diagnostics.
 * h_dtype is BIRKHOFF4_F32 or BIRKHOFF4_BF16 (H then holds B*16 bf16 values,
 * widened exactly to fp32). iters is NULL or an int32 [B] output receiving the
 * number of trial steps taken, or BIRKHOFF4_NOT_CONVERGED / BIRKHOFF4_NON_FINITE.
 * Other arguments as in birkhoff4_fwd. */
int birkhoff4_fwd_ex(const void* H, int h_dtype, float* P, float* dual, int32_t* iters,
                     int64_t B, float tol, int max_iter, hipStream_t stream);

/* Forward with an explicit kernel variant (BIRKHOFF4_AUTO, _THROUGHPUT or _LATENCY); other
 * arguments as in birkhoff4_fwd_ex, which is this call with BIRKHOFF4_AUTO. The latency
 * variant splits each problem's row-wise work over four lanes (the paper's Sec. 3.3 also
 * spreads one matrix over several lanes), which shortens the serial chain of a Newton step
 * for batches too small to fill the GPU; returns BIRKHOFF4_ERR_VARIANT for other values. */
int birkhoff4_fwd_ex2(const void* H, int h_dtype, float* P, float* dual, int32_t* iters,
                      int64_t B, float tol, int max_iter, int variant, hipStream_t stream);

/* Backward with a storage dtype for dP (BIRKHOFF4_F32 or BIRKHOFF4_BF16). */
int birkhoff4_bwd_ex(const float* P, const void* dP, int dp_dtype, float* dH, int64_t B,
                     hipStream_t stream);

/* Backward with storage dtypes for dP and for dH (BIRKHOFF4_F32 or BIRKHOFF4_BF16 each): a
 * bf16 dH [B][4][4] is the fp32 gradient rounded to nearest even. */
int birkhoff4_bwd_ex2(const float* P, const void* dP, int dp_dtype, void* dH, int dh_dtype,
                      int64_t B, hipStream_t stream);

/* Saved-Hessian variant (Sec. 4.2: at the solution the Hessian of the reduced dual equals
 * the Delta of eq. derivative, so the forward's Hessian can be kept for the backward).
 * birkhoff4_fwd_hess is birkhoff4_fwd_ex (one problem per lane, any B) that also writes,
 * per matrix, the six column weights W_jk = sum_i P_ij P_ik of its output P, whose
 * Laplacian grounded at column 4 is that Hessian: hess [B][8] fp32 =
 * (W_12, W_13, W_14, W_23, W_24, W_34, 0, 0), 32 bytes per matrix, caller-owned, 16-byte
 * aligned, not overlapping the other arrays; dual and iters may be NULL.
 * birkhoff4_bwd_hess is birkhoff4_bwd_ex taking those weights instead of recomputing them
 * from P. Both return the codes of the calls they extend; hess NULL gives
 * BIRKHOFF4_ERR_NULL. This trades 32 bytes of writes and of reads per matrix for the six
 * weight sums of the backward; the default pair above does not use it. */
int birkhoff4_fwd_hess(const void* H, int h_dtype, float* P, float* dual, float* hess, int32_t* iters,
                       int64_t B, float tol, int max_iter, hipStream_t stream);
int birkhoff4_bwd_hess(const float* P, const float* hess, const void* dP, int dp_dtype, float* dH,
                       int64_t B, hipStream_t stream);

/* Baseline: n_steps iterations of Sinkhorn-Knopp (eq. sinkhorn_knopp) from
 * v^(0) = 1 on A = exp(H) (each row shifted by its maximum, which leaves every
 * iterate diag(u) A diag(v) unchanged); P = diag(u^(n)) A diag(v^(n)), whose
 * columns sum to one. 1 <= n_steps <= 48. Denominators are clamped at the
 * smallest normal fp32 so that underflowed rows and columns stay finite. */
int birkhoff4_sk_fwd(const void* H, int h_dtype, float* P, int64_t B, int n_steps,
                     hipStream_t stream);

/* Baseline backward: the exact gradient of the n_steps Sinkhorn-Knopp map at H,
 * applied to dP (reverse mode through the unrolled iterations, recomputed from
 * H in registers; nothing is stored between the passes). */
int birkhoff4_sk_bwd(const void* H, int h_dtype, const void* dP, int dp_dtype, float* dH,
                     int64_t B, int n_steps, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * n = 8 (the mHC layer with eight streams, Sec. 3.1): the same projection and
 * gradient for 8 x 8 matrices, by Newton on the 7-dimensional reduced dual with the
 * general gradient and Hessian (eq. grad_hess with a = b = 1, eta = 1) and the general
 * implicit backward (eq. derivative). Return codes, dtypes and status words as above.
 *
 * H     [B][8][8] (h_dtype fp32 or bf16), row-major, device memory.
 * P     [B][8][8] fp32 output: rows and columns sum to one within tol.
 * dual  NULL or [B][16] fp32 output: (alpha_1..alpha_8, beta_1..beta_7, beta_8 = 0),
 *       natural-log units, log P_ij = H_ij + alpha_i + beta_j.
 * iters NULL or int32 [B] output: trial steps taken, BIRKHOFF4_NOT_CONVERGED or
 *       BIRKHOFF4_NON_FINITE (that matrix's P and dual are then NaN).
 * tol, max_iter as in birkhoff4_fwd. Buffers must not overlap; 16-byte alignment.
 * Asynchronous on `stream`; nothing is allocated. */
int birkhoff8_fwd(const void* H, int h_dtype, float* P, float* dual, int32_t* iters,
                  int64_t B, float tol, int max_iter, hipStream_t stream);

/* Backward for n = 8: dH [B][8][8] fp32 = dL/dH from P (the forward's output) and
 * dP [B][8][8] (dp_dtype fp32 or bf16), eq. derivative with Delta the Hessian of the
 * reduced dual at P. Rows and columns of dH sum to zero. dH must not overlap P or dP. */
int birkhoff8_bwd(const float* P, const void* dP, int dp_dtype, float* dH, int64_t B,
                  hipStream_t stream);

/* birkhoff8_bwd with a storage dtype for dH (as in birkhoff4_bwd_ex2). */
int birkhoff8_bwd_ex(const float* P, const void* dP, int dp_dtype, void* dH, int dh_dtype,
                     int64_t B, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * General entropic OT for 4 x 4 (eq. entropic, Sec. 2.3): for each b,
 *   T = argmin over { T >= 0, T 1 = a, T^T 1 = b } of <T, M> - eta h(T),
 * h(T) = -sum T_ij (log T_ij - 1), by the same Newton iteration on the reduced dual
 * (eq. min_fx with the general eq. grad_hess); the Birkhoff projection is the case
 * M = -H, a = b = 1, eta = 1.
 *
 * M     [B][4][4] fp32 cost, row-major.
 * a, b  [B][4] fp32 marginals: positive, sum(a[b]) = sum(b[b]) for each b (when the
 *       sums differ there is no solution and the status is BIRKHOFF4_NOT_CONVERGED).
 * eta   regulariser > 0 (BIRKHOFF4_ERR_ETA otherwise).
 * T     [B][4][4] fp32 output: rows sum to a exactly up to rounding, columns to b
 *       within tol: |c_j - b_j| <= tol max(1, sum(a) / n, b_j) for every column (n = 4
 *       here): absolute for unit-sized marginals, relative above, where the fp32 resolution
 *       of the column sums grows with the masses; for a = b = 1 this is the Birkhoff test.
 *       The last column, whose potential is fixed, may in addition differ by
 *       |sum a - sum b| as computed in fp32, since fp32 marginals rarely have equal sums.
 * dual  NULL or [B][8] fp32 output: (alpha_1..4, beta_1..3, beta_4 = 0) in the units of
 *       M, with T_ij = exp((alpha_i + beta_j - M_ij) / eta) (eq. dual).
 * iters NULL or int32 [B]: trial steps taken, BIRKHOFF4_NOT_CONVERGED, or
 *       BIRKHOFF4_NON_FINITE for a NaN, infinite or non-positive input (T, dual NaN).
 * tol, max_iter, alignment, overlap rules and asynchrony as in birkhoff4_fwd. */
int birkhoff4_ot_fwd(const float* M, const float* a, const float* b, float eta, float* T,
                     float* dual, int32_t* iters, int64_t B, float tol, int max_iter,
                     hipStream_t stream);

/* Backward of birkhoff4_ot_fwd (eq. derivative): dM [B][4][4] fp32 = dL/dM from the
 * solution T, the row marginals a [B][4] and dT = dL/dT [B][4][4] fp32, with Delta the
 * Hessian of the reduced dual at T. Rows and columns of dM sum to zero. dM must not
 * overlap the inputs. */
int birkhoff4_ot_bwd(const float* T, const float* a, const float* dT, float eta, float* dM,
                     int64_t B, hipStream_t stream);

/* General entropic OT for 8 x 8 problems: birkhoff4_ot_fwd / birkhoff4_ot_bwd with n = m = 8
 * (eq. entropic, eq. grad_hess, eq. derivative). M, T, dT, dM are [B][8][8] fp32 (256 bytes per
 * problem), a and b [B][8] fp32, dual [B][16] = (alpha_1..8, beta_1..7, beta_8 = 0) with
 * T_ij = exp((alpha_i + beta_j - M_ij) / eta); iters as for birkhoff8_fwd. Arguments, return
 * codes, status words and ownership as for the 4 x 4 calls. */
int birkhoff8_ot_fwd(const float* M, const float* a, const float* b, float eta, float* T, float* dual,
                     int32_t* iters, int64_t B, float tol, int max_iter, hipStream_t stream);
int birkhoff8_ot_bwd(const float* T, const float* a, const float* dT, float eta, float* dM, int64_t B,
                     hipStream_t stream);

/* Residual mixing of the mHC layer (Sec. 2.1): each token's n = 4 streams are mixed by its
 * projected matrix, Y = P X with P = proj(exp(H)), the term H^res x_l of the layer's update.
 *
 * H      [B][4][4] logits, h_dtype F32 or BF16 (as in birkhoff4_fwd_ex).
 * X      [B][4][C] streams of each token, row-major (stream i of token b starts at element
 *        (4 b + i) C), x_dtype F32 or BF16; NULL allowed when C = 0.
 * Y      [B][4][C] output in x_dtype: Y_i = sum_j P_ij X_j per token, accumulated in fp32;
 *        bf16 results are rounded to nearest even.
 * P      [B][4][4] fp32 output: the projection, exactly what birkhoff4_fwd_ex would write
 *        for H (the default forward variant); the backward needs it.
 * dual, iters  NULL or outputs as in birkhoff4_fwd_ex.
 * C      channels per stream, >= 0, a multiple of 8 for BF16 streams or 4 for F32
 *        (BIRKHOFF4_ERR_CHANNELS otherwise): every row is whole 16-byte chunks.
 * tol, max_iter as in birkhoff4_fwd. Y must not overlap any input or P, dual or iters; P,
 * dual and iters must not overlap X. Every check is made before anything is queued. */
int birkhoff4_mix_fwd(const void* H, int h_dtype, const void* X, int x_dtype, void* Y, float* P, float* dual,
                      int32_t* iters, int64_t B, int64_t C, float tol, int max_iter, hipStream_t stream);

/* Backward of birkhoff4_mix_fwd: from P (its output), the streams X and dY = dL/dY
 * ([B][4][C], both in x_dtype), writes dX = dL/dX = P^T dY per token ([B][4][C] in x_dtype,
 * fp32 accumulation, bf16 rounded to nearest even) and dH = dL/dH ([B][4][4] fp32): the
 * projection's backward (eq. derivative, as in birkhoff4_bwd) applied to
 * dP_ij = sum_c dY_i[c] X_j[c]. One pass over X and dY. Outputs must not overlap each other
 * or any input. Return codes as for birkhoff4_mix_fwd. */
int birkhoff4_mix_bwd(const float* P, const void* X, const void* dY, int x_dtype, void* dX, float* dH, int64_t B,
                      int64_t C, hipStream_t stream);

/* birkhoff4_mix_bwd with a storage dtype for dH (as in birkhoff4_bwd_ex2). */
int birkhoff4_mix_bwd_ex(const float* P, const void* X, const void* dY, int x_dtype, void* dX, void* dH, int dh_dtype,
                         int64_t B, int64_t C, hipStream_t stream);

/* Residual mixing with n = 8 streams per token: birkhoff4_mix_fwd / birkhoff4_mix_bwd with the
 * 8 x 8 projection (birkhoff8_fwd / birkhoff8_bwd). H and P are [B][8][8], X, Y, dY, dX are
 * [B][8][C] (stream i of token b starts at element (8 b + i) C), dual [B][16] and iters as for
 * birkhoff8_fwd, dH [B][8][8] fp32. Arguments, dtypes, the rule for C, return codes and overlap
 * rules as for the 4 x 4 calls. */
int birkhoff8_mix_fwd(const void* H, int h_dtype, const void* X, int x_dtype, void* Y, float* P, float* dual,
                      int32_t* iters, int64_t B, int64_t C, float tol, int max_iter, hipStream_t stream);
int birkhoff8_mix_bwd(const float* P, const void* X, const void* dY, int x_dtype, void* dX, float* dH, int64_t B,
                      int64_t C, hipStream_t stream);

/* birkhoff8_mix_bwd with a storage dtype for dH. dP [B][8][8] fp32 is an output too: dL/dP,
 * from which dH is formed; with an fp32 dH it may be dH's own memory, and must not overlap
 * anything otherwise. */
int birkhoff8_mix_bwd_ex(const float* P, const void* X, const void* dY, int x_dtype, void* dX, float* dP, void* dH,
                         int dh_dtype, int64_t B, int64_t C, hipStream_t stream);

/* How the layer reads its streams (Sec. 2.1: x <- H^res x + (H^post)^T F(H^pre x)): the
 * coefficients of a token from its streams, and the branch's input U = H^pre x. With v the token's
 * K = n C values (n = 4 here), N = n^2 + 2 n, r = (|v|^2 / K + eps)^(-1/2):
 *   q = r W v,  l_j = alpha_g q_j + bias_j with g = 0 for rows j < n, 1 for n <= j < 2 n, else 2,
 *   h^pre = sigmoid(l_0 .. l_{n-1}),  h = 2 sigmoid(l_n .. l_{2n-1}),  H = the other n^2 (row-major),
 *   U = sum_i h^pre_i X_i.
 *
 * X      [B][n][C] streams in x_dtype (F32 or BF16); W [N][n C] in x_dtype too.
 * alpha  [3] fp32, bias [N] fp32; eps >= 0 and finite (BIRKHOFF4_ERR_EPS).
 * U      [B][C] output in x_dtype (bf16 rounded to nearest even); sums are fp32 throughout.
 * h, H   [B][n], [B][n][n] fp32 outputs: what birkhoff4_post_fwd takes.
 * q, rms [B][N], [B] fp32 outputs: q and r, which the backward needs.
 * work   workspace of work_bytes >= birkhoff4_pre_work(B, C, x_dtype, 0) bytes, in use until the
 *        call's work on `stream` has ended; its contents before and after mean nothing.
 * C      > 0, a multiple of 8 for BF16 or 4 for F32, at most 2^20 (BIRKHOFF4_ERR_CHANNELS, _SIZE);
 *        B at most 2^26.
 * A token with a NaN or infinite value has NaN (or infinite) outputs; the others are not touched
 * by it. |v|^2 is an fp32 sum: where it passes fp32's range, r = 0, and where it is 0 with eps = 0, r is
 * infinite. The result does not depend on timing: no atomics, fixed orders of sums. */
int birkhoff4_pre_fwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, float eps, void* U,
                      float* h, float* H, float* q, float* rms, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream);

/* Backward of birkhoff4_pre_fwd: from its inputs, q and rms, and the gradients dU [B][C] (x_dtype),
 * dh [B][n], dH [B][n][n] (fp32) and E [B][n][C] (x_dtype; a gradient of the streams from
 * elsewhere, added to dX), each of which may be NULL for zero, writes dX [B][n][C] and dW [N][n C]
 * (x_dtype), dalpha [3] and dbias [N] (fp32). With B = 0 these sums are written as zeros, and only
 * dW, dalpha and dbias need be there. work as above, of birkhoff4_pre_work(B, C, x_dtype, 1) bytes. */
int birkhoff4_pre_bwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, const float* q,
                      const float* rms, const void* dU, const float* dh, const float* dH, const void* E, void* dX,
                      void* dW, float* dalpha, float* dbias, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream);

/* Bytes of workspace of the forward (backward = 0) or the backward (1); a negative return code for
 * sizes or a dtype that those calls refuse. */
int64_t birkhoff4_pre_work(int64_t B, int64_t C, int x_dtype, int backward);

/* The same for n = 8 streams: N = 80, H and dH [B][8][8]. */
int birkhoff8_pre_fwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, float eps, void* U,
                      float* h, float* H, float* q, float* rms, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream);
int birkhoff8_pre_bwd(const void* X, const void* W, int x_dtype, const float* alpha, const float* bias, const float* q,
                      const float* rms, const void* dU, const float* dh, const float* dH, const void* E, void* dX,
                      void* dW, float* dalpha, float* dbias, void* work, int64_t work_bytes, int64_t B, int64_t C,
                      hipStream_t stream);
int64_t birkhoff8_pre_work(int64_t B, int64_t C, int x_dtype, int backward);

/* How the layer writes its streams (Sec. 2.1): the residual mixing of birkhoff4_mix_fwd plus the
 * branch's output Z, weighted by h and with dropout,
 *   Y_i = sum_j P_ij X_j + h_i D,  P = proj(exp(H)),  D = Z / (1 - p) where kept, else 0.
 *
 * h    [B][n] fp32 (n = 4 here), Z [B][C] in x_dtype (NULL allowed when C = 0).
 * p    dropout probability, 0 <= p < 1 (BIRKHOFF4_ERR_DROP). rng is two 64-bit words in device
 *      memory, seed and offset; NULL allowed with p = 0. Element e of Z (counted over the whole
 *      array) is kept where word e mod 4 of the Philox 4x32-10 block with counter (e div 4, offset)
 *      and key seed is at least floor(p 2^32); no mask is stored. Neither n, the dtype nor the
 *      launch changes it. The words are read when the work runs: a replayed graph takes what they
 *      are by then, and the backward must find what the forward found.
 * The other arguments as in birkhoff4_mix_fwd; sums are fp32, bf16 results rounded once. */
int birkhoff4_post_fwd(const void* H, int h_dtype, const void* X, const float* h, const void* Z, int x_dtype, double p,
                       const int64_t* rng, void* Y, float* P, float* dual, int32_t* iters, int64_t B, int64_t C,
                       float tol, int max_iter, hipStream_t stream);

/* Backward of birkhoff4_post_fwd: from its P, X, h, Z, p and rng, and dY [B][n][C] (x_dtype), writes
 * dX and dH as birkhoff4_mix_bwd_ex does, dZ [B][C] (x_dtype) and dh [B][n] (fp32), in one pass over
 * X, Z and dY. Outputs must not overlap each other or any input. */
int birkhoff4_post_bwd(const float* P, const void* X, const float* h, const void* Z, const void* dY, int x_dtype, double p,
                       const int64_t* rng, void* dX, void* dZ, float* dh, void* dH, int dh_dtype, int64_t B, int64_t C,
                       hipStream_t stream);

/* The same with n = 8 streams per token; dP [B][8][8] fp32 as in birkhoff8_mix_bwd_ex. */
int birkhoff8_post_fwd(const void* H, int h_dtype, const void* X, const float* h, const void* Z, int x_dtype, double p,
                       const int64_t* rng, void* Y, float* P, float* dual, int32_t* iters, int64_t B, int64_t C,
                       float tol, int max_iter, hipStream_t stream);
int birkhoff8_post_bwd(const float* P, const void* X, const float* h, const void* Z, const void* dY, int x_dtype, double p,
                       const int64_t* rng, void* dX, void* dZ, float* dh, float* dP, void* dH, int dh_dtype, int64_t B,
                       int64_t C, hipStream_t stream);

/* Layer norm over rows of C values, in front of the layer's branch: with mu the mean of a row x and
 * s = (mean((x - mu)^2) + eps)^(-1/2),
 *   y = (x - mu) s weight + bias.
 *
 * X      [B][C] in x_dtype (F32 or BF16); any C from 1 to 2^20, B up to 2^31.
 * weight, bias  [C] in w_dtype (F32 or BF16, whatever x_dtype is); NULL for ones and for zeros.
 * Y      [B][C] output in x_dtype (bf16 rounded to nearest even once); sums are fp32.
 * mean, rstd  [B] fp32 outputs mu and s, which the backward needs; NULL where they are not wanted.
 * eps >= 0 and finite (BIRKHOFF4_ERR_EPS). A row with a NaN or infinite value has NaN outputs; the
 * others are not touched by it. A row whose squares (x - mu)^2 add up past fp32's range (deviations
 * of 1.8e19 / sqrt(C) and more) gets s = 0, so y = bias and dX = 0; one whose sum passes it NaN.
 * Subnormal numbers count as zero: with eps = 0 a row of equal values, or of deviations below 1e-19,
 * has NaN or infinite outputs. The arrays begin at 16 bytes, their rows at any value. */
int birkhoff4_norm_fwd(const void* X, int x_dtype, const void* weight, const void* bias, int w_dtype, float eps, void* Y,
                       float* mean, float* rstd, int64_t B, int64_t C, hipStream_t stream);

/* Backward of birkhoff4_norm_fwd: from X, weight, mean, rstd and dY [B][C] (x_dtype), writes
 * dX [B][C] (x_dtype), dweight and dbias [C] (w_dtype), each where it is not NULL. With B = 0 the
 * sums are written as zeros. work: a workspace of birkhoff4_norm_work(B, C, x_dtype) bytes, needed
 * where dweight or dbias is; its contents before and after mean nothing. The sums over the rows are
 * fp32, in an order that the sizes alone decide: up to 256 blocks' (for C > 8192, shares') own sums,
 * one row behind the other, and then the sums of these. */
int birkhoff4_norm_bwd(const void* X, int x_dtype, const void* weight, int w_dtype, const float* mean, const float* rstd,
                       const void* dY, void* dX, void* dweight, void* dbias, void* work, int64_t work_bytes, int64_t B,
                       int64_t C, hipStream_t stream);
int64_t birkhoff4_norm_work(int64_t B, int64_t C, int x_dtype);

/* Matrices taken towards their nearest orthogonal ones (rows or columns orthonormal, whichever are
 * fewer) by Newton-Schulz products: X = G / (|G|_F + eps), then for each step k, with A = X X^T
 * (for rows > cols the same of the transpose),
 *   X <- a_k X + (b_k A + c_k A^2) X,
 * which keeps the singular vectors and takes each singular value s to a s + b s^3 + c s^5.
 *
 * G      [B][rows][cols] in g_dtype (F32 or BF16); out the same in out_dtype.
 * coefs  host array of 3 * steps floats a, b, c, read before the call returns; 1 <= steps <= 64
 *        (BIRKHOFF4_ERR_STEPS). Entries of X, A and b A + c A^2 have to stay below 16 in magnitude,
 *        as they do where the steps keep the singular values below 2; what does not ends as NaN.
 * eps    >= 0 and finite (BIRKHOFF4_ERR_EPS). The norm is a 64-bit sum: no finite fp32 matrix is
 *        too large or too small. A zero matrix with eps > 0 gives zeros; one with a NaN or infinite
 *        value gives NaN everywhere; the others of the batch are not touched by it.
 * An fp32 result is about what fp32 products give; with a side of at most 80, what 64-bit ones
 * do. For a bf16 result the products' factors are rounded to fp16 (11 bits), but for the diagonals
 * and a X; sums are fp32: off by less than the rounding of the result itself, by up to three times
 * it for matrices of low rank or of singular values that fade away. Steps whose largest
 * |a + b t + c t^2|, t from 0 to 2, multiply to more than 512 (as six of the usual ones do) make
 * more of small values: for a bf16 result those in front of the last that multiply to 512 take
 * the factors of an fp32 one, and with a side of at most 80 singular values under 2^-26 of |G|_F
 * stay behind what 64 bits would make of them. The number of matrices may change the order of
 * sums; within a batch it is the same for all of them.
 * work   workspace of birkhoff4_orth_work(B, rows, cols, out_dtype) bytes, 16-byte aligned, in use until
 *        the call's work on `stream` has ended. The other arrays may begin at any value. No output may
 *        overlap another argument. rows and cols up to 2^20, the smaller of them up to 2^16, B up to
 *        2^26; a zero among them is a no-op. The result does not depend on timing. */
int birkhoff4_orth(const void* G, int g_dtype, void* out, int out_dtype, const float* coefs, int steps, float eps, void* work,
                   int64_t work_bytes, int64_t B, int64_t rows, int64_t cols, hipStream_t stream);

/* A weight update with momentum along orthogonalised directions, in place:
 *   M <- momentum M + G,   U = G + momentum M (nesterov != 0) or M,
 *   W <- (1 - r decay) W - r scale orth(U),   r = lr *lr_at,
 * for any momentum (of either sign).
 *
 * W      [B][rows][cols] in w_dtype (F32 or BF16, rounded to nearest even); M the same in fp32.
 * lr_at  a float in device memory, read when the work runs (a replayed graph takes what it is by
 *        then), or NULL for one.
 * The other arguments as above, with w_dtype for out_dtype. The direction that fp32 weights far from
 * square take may be off by up to eleven times what birkhoff4_orth's is, which is three times what
 * fp32 products give (2560 x 10240: 4e-5 of its size after eight of the usual steps, 7e-6 after five). */
int birkhoff4_orth_step(void* W, int w_dtype, const void* G, int g_dtype, float* M, float momentum, int nesterov, float lr,
                        const float* lr_at, float decay, float scale, const float* coefs, int steps, float eps, void* work,
                        int64_t work_bytes, int64_t B, int64_t rows, int64_t cols, hipStream_t stream);
int64_t birkhoff4_orth_work(int64_t B, int64_t rows, int64_t cols, int out_dtype);

/* Human-readable text for a return code (static storage). */
const char* birkhoff4_strerror(int code);

/* Library version: major * 10000 + minor * 100 + patch. */
int birkhoff4_version(void);

#ifdef __cplusplus
}
#endif

#endif /* BIRKHOFF4_H */
