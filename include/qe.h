/*
 * qe.h -- C ABI of the MI355X (gfx950) QuantEase hot-path library, libqe.so.
 *
 * QuantEase (arXiv 2309.01885) quantizes one linear layer at a time by
 * minimising f(What) = ||W X - What X||_F^2 over a per-output-channel uniform
 * b-bit grid (Sec. 2.1, problem (1)), with cyclic coordinate descent (Sec. 3)
 * and, optionally, a sparse full-precision outlier matrix H chosen by
 * iterative hard thresholding (Sec. 4).
 *
 * Conventions shared by every entry point:
 *  - Matrices are dense, row-major, contiguous fp32 in DEVICE memory (HBM)
 *    unless stated otherwise: W, What, R/E, H are q x p (q output channels,
 *    p input channels); Sigma is p x p and symmetric; X is p x n or n x p.
 *  - The library never allocates or frees caller memory.  Scratch space comes
 *    from the caller as a device workspace `ws` of at least the size returned
 *    by the matching *_workspace_size query; the first 256 bytes of every
 *    workspace hold a device status word.
 *  - All work is enqueued on `stream` (a hipStream_t; NULL = the default
 *    stream) and is asynchronous.  Host-detectable argument errors return
 *    immediately with nothing enqueued.  Data-dependent errors (a
 *    non-positive diagonal entry of Sigma, a non-finite or non-positive grid
 *    scale) are written to the workspace status word, the remaining kernels
 *    of that call become no-ops, and qe_sync_status() reports them.
 *  - Results are bitwise deterministic for a fixed shape, block width and
 *    flag set (no floating-point atomics anywhere).
 *  - Concurrent calls on different streams need disjoint workspaces and
 *    outputs.
 */
#ifndef QE_H
#define QE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int qe_status;

#define QE_OK              0
#define QE_ERR_ARG         1  /* null pointer, bad size, bits outside [1, 8], ... */
#define QE_ERR_DIAG        2  /* some Sigma_jj <= 0 or not finite (Lemma 1 assumes Sigma_jj > 0) */
#define QE_ERR_SCALE       3  /* some grid scale <= 0 or not finite */
#define QE_ERR_WORKSPACE   4  /* workspace null or smaller than the size query */
#define QE_ERR_HIP         5  /* a HIP runtime call failed */
#define QE_ERR_UNSUPPORTED 6  /* a valid request this library does not implement */
#define QE_ERR_TOO_LARGE   7  /* qe_cd_sweep_noalloc: the sizes need more than its fixed scratch */
#define QE_ERR_NONFINITE   8  /* QE_DEBUG_CHECKS found a NaN or infinity in an input */

/* Layouts of X for qe_gram, optionally or-ed with one of QE_GRAM_FP32 and
 * QE_GRAM_BF16X3 (both at once is QE_ERR_ARG). */
#define QE_LAYOUT_PN 0        /* X is p x n: each channel's n tokens contiguous */
#define QE_LAYOUT_NP 1        /* X is n x p: each token's p channels contiguous */
#define QE_GRAM_FP32 0x100    /* products on the fp32 matrix cores instead of split ones */
#define QE_GRAM_BF16X3 0x200  /* the three-way bf16 split everywhere (no fp16 split) */

/* Flags for qe_cd_sweep / qe_cd_outlier_sweep. */
#define QE_INIT_FROM_W 0x1u   /* start from What = W (Sec. 3.1) or What = W - H (Sec. 4.3);
                                 R (or E) is set to 0; codes are not yet valid */
#define QE_R_VALID     0x2u   /* R (or E) already holds (What [+ H] - W) Sigma: resume */
#define QE_CODES_VALID 0x4u   /* codes hold What's grid codes: the keep-current tie rule of the
                                 modified CD (Sec. 3.3) applies from the first sweep */
/* Relaxed sweeps (Sec. 3.2, "Initialization": some iterations skip the
 * quantization).  With period k in [1, 255], sweeps k, 2k, ... of a call
 * (counted from 1) write the unconstrained minimiser beta of Lemma 1 instead
 * of q_i(beta); the last sweep of a call is never relaxed.  After a relaxed
 * sweep What is off the grid, so the next sweep starts with codes invalid;
 * codes are left as they were during a relaxed sweep. */
#define QE_RELAX_PERIOD(k) ((((uint32_t)(k)) & 0xffu) << 8)
#define QE_RELAX_MASK      0xff00u
/* qe_cd_outlier_sweep only: structured outliers ("Structured Outliers",
 * Sec. 4.3): the projection keeps the floor(s / q) whole columns of largest
 * l2 norm instead of the s largest entries (see qe_topk_columns). */
#define QE_OUTLIER_COLUMNS 0x10u
/* Block-update and residual products on the fp32 matrix cores instead of the
 * default exact three-way bf16 split (the split is described at qe_gram). */
#define QE_CD_FP32 0x20u
/* Checks before the sweeps (the paper asks for checks on the inputs before
 * QuantEase runs, footnote to Lemma 1): every input of the call -- W, Sigma,
 * scale, zero, What unless QE_INIT_FROM_W, R (or E) with QE_R_VALID, and H in
 * the outlier-aware call -- is scanned for NaN and infinity, which sets
 * QE_ERR_NONFINITE (reported by qe_sync_status; the rest of the call does
 * nothing).  One extra read of those arrays (about 30 us at 4096 x 4096).
 * Without the flag only Sigma's diagonal and the grid are checked. */
#define QE_DEBUG_CHECKS 0x40u
/* Every block update on the matrix cores.  By default, from the second sweep
 * on (codes valid), a 128 x 128 tile of the block update whose rows changed
 * few codes in the super-block just finished (at most 64 rows, each at most 32
 * codes) applies only those nonzero code differences, as fp32 FMAs; its
 * other rows' update is exactly 0 and is skipped.  Both forms give R up to
 * fp32 rounding; with this flag R's rounding does not depend on how many
 * codes moved. */
#define QE_CD_DENSE 0x10000u
/* qe_cd_sweep only: obj[0] holds, on entry, the objective f of the incoming
 * What and R (e.g. the last value of the previous call), so that chained
 * calls report f without a pass over R.  Needs obj; not with QE_INIT_FROM_W
 * (QE_ERR_ARG). */
#define QE_OBJ_IN 0x80u

/* Human-readable name of a status code (static string). */
const char* qe_status_string(qe_status s);

/* Library ABI version (increases on any signature change). */
int qe_version(void);

/* Synchronises `stream`, then returns the status word of workspace `ws`
 * (QE_OK if no kernel reported a data error).  Also clears the word. */
qe_status qe_sync_status(void* ws, void* stream);

/* ------------------------------------------------------------------------
 * Gram matrix.  Lemma 1 (Sec. 3.2) works with Sigma = X X^T, whose size is
 * independent of the token count n (Sec. 3.2, "Memory Footprint").
 *   Sigma (+)= X X^T; then, if damp > 0, Sigma_jj += damp * mean_j(Sigma_jj).
 * X: p x n (QE_LAYOUT_PN) or n x p (QE_LAYOUT_NP), fp32, device.
 * Sigma: p x p fp32, device; overwritten (accumulate = 0) or added to
 * (accumulate = 1, for token chunks streamed through several calls; pass
 * damp = 0 on all but the last).  The result is exactly symmetric.
 * Products, by default: when p is a multiple of 256 and either X's rows are 16-byte
 * aligned and n is a multiple of 32 or X is token-major, 16-byte aligned and n > 32; or
 * when p > 128 and p p n is at least 3e9 (1e10, and p > 384, where p is a multiple of
 * 128 but not of 256, rows are aligned and n is a multiple of 32); p at
 * most 2^24, and either the split partials fit the workspace or
 * n <= 32768 (at very large p, stream longer token ranges in chunks of at
 * most 32768): each channel i is first scaled by 2^e_i (exact; its largest |x|
 * lands in [2^14, 2^15), a pass over X; e_i at most 127) and each scaled value
 * y is split into two fp16 values
 * (h = fp16(y), m = fp16(y - h)); y_i y_j is formed from the three products
 * h h, h m, m h on the fp16 matrix cores, every product exact in fp32, and
 * the sums are scaled back by 2^-(e_i + e_j).  The dropped terms are below
 * 3 * 2^-22 |y_i y_j| (plus 2^-39 of the channels' largest values for the
 * smallest ones).  Otherwise, or with QE_GRAM_BF16X3, each fp32 value x is
 * split exactly into three bf16 values (h = bf16(x), m = bf16(x - h),
 * l = x - h - m) and x_i x_j is formed from the six products h h, h m, m h,
 * h l, m m, l h on the bf16 matrix cores; the dropped terms are below
 * 2^-23 |x_i x_j| (one fp32 rounding).  With QE_GRAM_FP32 the products run
 * on the fp32 matrix cores.  Accumulation: fp32 over short token chunks,
 * chunk sums added in fp32, split partial sums reduced in fp64.
 * ------------------------------------------------------------------------ */
size_t qe_gram_workspace_size(int64_t p, int64_t n);
qe_status qe_gram(const float* X, int64_t p, int64_t n, int layout, float* Sigma,
                  int accumulate, float damp, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Per-row uniform grid Q_i = { scale_i (k - zero_i) : k = 0 .. 2^bits - 1 }
 * (Sec. 2.1: uniformly spaced levels per output channel).  Asymmetric min/max
 * reading: lo = min(0, min_j W_ij), hi = max(0, max_j W_ij), an all-zero row
 * uses [-1, 1]; scale = (hi - lo) / (2^bits - 1), zero = rint(-lo / scale),
 * all in fp32.  Entries with H_ij != 0 are excluded (outlier-aware grid,
 * Sec. 4.3); H may be NULL.
 * W, H: q x p device.  scale, zero: q floats each, device, written.
 * ------------------------------------------------------------------------ */
qe_status qe_grid_minmax(const float* W, const float* H, int64_t q, int64_t p, int bits,
                         float* scale, float* zero, void* stream);

/* ------------------------------------------------------------------------
 * Blocked cyclic coordinate descent (Sec. 3; Lemma 1; the rank-1 identity of
 * Sec. 3.2; Algorithm "QuantEase").
 * Residual form: R = (What - W) Sigma.  For each column j in order, for all
 * rows i at once:  beta = What_ij - R_ij / Sigma_jj;  What_ij <- q_i(beta)
 * (nearest grid level, half to even, a valid equally-near current level is
 * kept, Sec. 3.3);  R += (What_new - What_old)_{:,j} Sigma_{j,:}.
 * Columns are processed in blocks of `block` (0 = 128; one of 16, 32, 64,
 * 128): inside a block the rank-1 updates touch only the block's columns;
 * the accumulated block update is then applied to every column as one
 * matrix-core GEMM.  A sweep that starts from valid codes and moves few of them
 * runs row by row instead (p <= 16384, no QE_RELAX_PERIOD, none of QE_CD_DENSE and
 * QE_CD_FP32; decided on the device from a sample of the state before the sweep, and
 * then for the rest of the call; after QE_INIT_FROM_W, whose later sweeps move few,
 * at the latest with the fifth sweep, the ninth if q p p is at least 1.5e11): per move
 * one rank-1 update of the row, nothing for a kept code.  The result equals the
 * column-by-column algorithm up to floating-point rounding in either form; R's
 * rounding depends on the form, so a call of K sweeps and K resumed calls agree bit
 * for bit where they make the same choices, and up to rounding otherwise.
 *
 * W:      q x p, device, read (only for R initialisation and the objective).
 * Sigma:  p x p, device, symmetric with Sigma_jj > 0 (else QE_ERR_DIAG).
 * scale, zero: q floats, device (e.g. from qe_grid_minmax); bits in [1, 8].
 * W_hat:  q x p, device, in/out.  codes: q x p uint8, device, in/out.
 * R:      q x p, device, in/out: (What - W) Sigma on exit.
 * sweeps: >= 0 full passes over the columns.
 * flags:  QE_INIT_FROM_W | QE_R_VALID | QE_CODES_VALID | QE_RELAX_PERIOD(k)
 *         | QE_CD_FP32 | QE_CD_DENSE | QE_DEBUG_CHECKS | QE_OBJ_IN.
 *         Without QE_INIT_FROM_W and without QE_R_VALID, R is first
 *         computed as (What - W) Sigma (warm start from any What, Sec. 3.1).
 * obj:    NULL, or device array of `sweeps` doubles receiving
 *         f_k = <What - W, R> = ||(W - What) X||_F^2 after sweep k, formed
 *         as the incoming f plus the exact change of each coordinate move
 *         (Lemma 1's one-dimensional quadratic: delta (2 R_ij + delta
 *         Sigma_jj)), summed in fp64 while the sweep runs, in a fixed order.
 *         The incoming f is 0 with QE_INIT_FROM_W, obj[0] with QE_OBJ_IN,
 *         else one pass <What - W, R> at the start of the call.
 * ------------------------------------------------------------------------ */
size_t qe_cd_workspace_size(int64_t q, int64_t p, int block);
qe_status qe_cd_sweep(const float* W, const float* Sigma, int64_t q, int64_t p, int bits,
                      const float* scale, const float* zero, float* W_hat, uint8_t* codes,
                      float* R, int sweeps, int block, uint32_t flags, double* obj,
                      void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * qe_cd_sweep without allocation or workspace, for callers that cannot
 * allocate device memory: code under stream/graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Arguments and results as for
 * qe_cd_sweep, except:
 *  - the scratch (the status word, 1/Sigma_jj, 1/scale, the two delta
 *    buffers of q x max(256, block) floats, fp64 partial sums) lives in a
 *    library-owned device array of QE_NOALLOC_SCRATCH_BYTES per GPU, held
 *    until the process ends; the call needs qe_cd_workspace_size(q, p, block)
 *    bytes of it and returns QE_ERR_TOO_LARGE, with nothing enqueued, when
 *    that is more (q up to about 30000 rows at the default block);
 *  - status: NULL, or a device int that receives, in stream order at the
 *    end of the call, the call's data-error status (QE_OK, QE_ERR_DIAG,
 *    QE_ERR_SCALE), as qe_sync_status would report it;
 *  - every call on one GPU uses that GPU's one scratch array: calls that
 *    overlap on one GPU (different streams, host threads) race and must be
 *    serialised by the caller.  Each call clears what it needs cleared.
 * No hipMalloc, hipFree or allocating routine is called; the scratch's
 * device address is looked up once per GPU, on the first call there.
 * ------------------------------------------------------------------------ */
#define QE_NOALLOC_SCRATCH_BYTES (64u << 20)
qe_status qe_cd_sweep_noalloc(const float* W, const float* Sigma, int64_t q, int64_t p, int bits,
                              const float* scale, const float* zero, float* W_hat,
                              uint8_t* codes, float* R, int sweeps, int block, uint32_t flags,
                              double* obj, int* status, void* stream);

/* ------------------------------------------------------------------------
 * Outlier-aware QuantEase (Sec. 4, Algorithm "Outlier-Aware QuantEase").
 * Per iteration: one CD sweep on What with H fixed (linear term from
 * W - H, residual E = (What + H - W) Sigma), then one iterative-hard-
 * thresholding step  H <- P_s(H - eta grad_H g),  grad_H g = 2E,
 * eta = 1 / (2 lambda_max), i.e. V = H - E / lambda_max (fp32); P_s keeps
 * the s entries of largest |V| (ties: lower linear index i*p + j; zeros are
 * never kept); then E += (H_new - H_old) Sigma.
 *
 * H:        q x p dense, device, in/out.
 * E:        q x p, device, in/out (the residual).
 * support:  device int64 array of capacity s, in/out: ascending linear
 *           indices of H's nonzeros.  support_nnz: device int64, in/out.
 * s:        outlier budget, 0 <= s <= q*p.  lambda_max > 0 (qe_lambda_max).
 * flags:    QE_INIT_FROM_W: What = W - H (H and support as given, e.g. from
 *           qe_topk_abs on W, Sec. 4.3 initialisation), E = 0.
 *           QE_R_VALID: E already valid.  QE_CODES_VALID as above.
 *           QE_OUTLIER_COLUMNS: structured outliers (whole columns); start
 *           from qe_topk_columns on W.
 *           Without QE_INIT_FROM_W / QE_R_VALID, E = (What + H - W) Sigma.
 *           QE_CD_FP32, QE_CD_DENSE and QE_DEBUG_CHECKS as for qe_cd_sweep.
 * obj:      NULL or device array of 2*sweeps doubles: obj[2k] = g after the
 *           CD sweep of iteration k (g after the previous IHT step, or at
 *           the start, plus the exact change of the sweep's moves, as for
 *           qe_cd_sweep), obj[2k+1] = g after its IHT step (<What + H - W, E>).
 * scale/zero: the outlier-aware grid (qe_grid_minmax with H excluded).
 * ------------------------------------------------------------------------ */
size_t qe_outlier_workspace_size(int64_t q, int64_t p, int block, int64_t s);
qe_status qe_cd_outlier_sweep(const float* W, const float* Sigma, int64_t q, int64_t p,
                              int bits, const float* scale, const float* zero, float* W_hat,
                              uint8_t* codes, float* H, float* E, int64_t s, float lambda_max,
                              int64_t* support, int64_t* support_nnz, int sweeps, int block,
                              uint32_t flags, double* obj, void* ws, size_t ws_bytes,
                              void* stream);

/* ------------------------------------------------------------------------
 * P_s of Sec. 4.3 on a dense array: keep the s entries largest in absolute
 * value (ties: lower index first; exact zeros never kept).
 * V: `count` floats, device.  out: `count` floats, device: P_s(V).
 * support: device int64[s]: kept indices, ascending.  nnz: device int64.
 * ------------------------------------------------------------------------ */
size_t qe_topk_workspace_size(int64_t count, int64_t s);
qe_status qe_topk_abs(const float* V, int64_t count, int64_t s, float* out, int64_t* support,
                      int64_t* nnz, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Structured projection ("Structured Outliers", Sec. 4.3): keep the c whole
 * columns of the q x p matrix V with the largest l2 norm, zero elsewhere.
 * Selection key of column j: sum_i V_ij^2 accumulated in fp64, rounded to
 * fp32; ties go to the lower column; all-zero columns are never kept.
 * out: q x p floats, device.  columns: NULL or device int64[c]: the kept
 * columns, ascending.  support: device int64[q * c]: linear indices of every
 * entry of the kept columns, ascending (the support format of
 * qe_cd_outlier_sweep).  nnz: device int64: number of support entries
 * (q x number of kept columns).
 * ------------------------------------------------------------------------ */
size_t qe_topk_columns_workspace_size(int64_t q, int64_t p);
qe_status qe_topk_columns(const float* V, int64_t q, int64_t p, int64_t c, float* out,
                          int64_t* columns, int64_t* support, int64_t* nnz, void* ws,
                          size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Exact objective and its normaliser (Sec. 2.1 problem (1); Sec. 3.4 relative
 * calibration error), recomputed from scratch, independent of R:
 *   out[0] = <D, D Sigma> = ||(What + H - W) X||_F^2,  D = What + H - W,
 *   out[1] = <W, W Sigma> = ||W X||_F^2.
 * Sigma has to be symmetric: only its lower half is read (and whole tiles of up to 256
 * channels along the diagonal), doubled; another matrix gives another number.
 * The products D Sigma use the exact three-way bf16 split (see qe_gram);
 * <D, D Sigma> is summed in fp64.  H may be NULL.  out: device, 2 doubles.
 * ------------------------------------------------------------------------ */
size_t qe_objective_workspace_size(int64_t q, int64_t p);
qe_status qe_objective(const float* W, const float* W_hat, const float* H, const float* Sigma,
                       int64_t q, int64_t p, double* out, void* ws, size_t ws_bytes,
                       void* stream);

/* ------------------------------------------------------------------------
 * lambda_max(Sigma) by the power method (Sec. 4.3: matrix-vector products
 * only, O(p^2) per iteration), returned as an upper bound, since the IHT step
 * 1 / (2 lambda) of Lemma 3 needs lambda >= lambda_max.  Start vector
 * 1/sqrt(p); iterate v_k = S v_{k-1} / |S v_{k-1}|, quotient
 * rho_k = v_k' S v_k / v_k' v_k.  The iteration used is the first whose
 * quotient changed by at most tol (relative) from the previous one, else
 * iteration max_iters; the result is rho + |S v - rho v| / |v| of that
 * iteration (an eigenvalue lies within that radius of rho; v approximates the
 * leading eigenvector), from fp64 sums, widened by a relative 2^-30 and
 * rounded up to fp32.
 * Synchronises `stream` every 32 iterations.  Up to p = 4096 those 32 run as one
 * cooperative launch that keeps Sigma in registers (where the runtime does not take it
 * or a workgroup waits too long for another, one launch per iteration with the same
 * result; beyond, one launch per iteration).
 * lambda_out: HOST float.
 * ------------------------------------------------------------------------ */
size_t qe_lambda_workspace_size(int64_t p);
qe_status qe_lambda_max(const float* Sigma, int64_t p, int max_iters, float tol,
                        float* lambda_out, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Export for serving.  The paper leaves serving kernels out of scope
 * (Sec. 4.3, "Structured Outliers"); these layouts are this library's.
 *
 * qe_pack_codes: each row of the q x p codes (device uint8, values < 2^bits,
 * bits in [1, 8]) becomes one little-endian bit stream of
 * qe_packed_row_bytes(p, bits) bytes (device, out): code j occupies bits
 * [j*bits, (j+1)*bits), bytes are filled from their least significant bit,
 * rows start on a byte boundary.  Higher code bits are ignored.
 *
 * qe_outliers_csr: the support entries of H (q x p, device) as CSR:
 * support = ascending linear indices (device int64, capacity cap), nnz =
 * device int64 count (clamped to [0, cap]); rowptr: device int64[q + 1],
 * cols: device int32[cap], vals: device float[cap] (out).  Out-of-range
 * indices are clamped into the matrix.
 * ------------------------------------------------------------------------ */
int64_t qe_packed_row_bytes(int64_t p, int bits);
qe_status qe_pack_codes(const uint8_t* codes, int64_t q, int64_t p, int bits, uint8_t* packed,
                        void* stream);
qe_status qe_outliers_csr(const float* H, int64_t q, int64_t p, const int64_t* support,
                          const int64_t* nnz, int64_t cap, int64_t* rowptr, int32_t* cols,
                          float* vals, void* stream);

/* ------------------------------------------------------------------------
 * Key/value cache in 4 bits, for decoders whose layers this library quantizes.
 * The paper covers weights only; grid and layout are this library's.
 *
 * Grid.  The dim channels of a token's key (or value) in one head are cut into
 * groups of `group` consecutive channels.  A group x gets, in fp32,
 *   lo = min(0, min x), hi = max(0, max x),
 *   s = max((hi - lo) * r, 2^-126), r = 1 / 15 rounded, its bit pattern rounded to a
 *   multiple of 16,
 *   z = rint(-lo * (1 / s)),  n = clamp(rint(x * (1 / s)) + z, 0, 15),
 * and is held as the codes n and one word, the bit pattern of s with z in its low
 * four bits; it stands for s (n - z), each element within s / 2 of x (up to rounding).  A
 * group that holds a NaN or an infinity, or whose hi - lo passes the largest fp32
 * number, has a NaN scale: it reads back as NaN, and so does every attention row
 * that sees it.
 *
 * Layout.  dim is a multiple of 8, at most 256; group is 32, 64 or 128; a page
 * holds `page` tokens (a multiple of 32).  The cache is num_pages pages, in each of
 * them kv_heads x page / 32 records of 32 consecutive tokens of one head (pages 16-byte
 * aligned, qe_kv_page_bytes each).  With Dp = dim rounded up to 64, 96, 128, 192 or
 * 256 (channels past dim hold 0), NC = Dp / 32 and NG = ceil(Dp / group), a record is
 *   - 32 key rows of 4 NC words: word j NC + c holds channels 8 (4 c + j) .. + 7,
 *     the lowest channel in the lowest four bits;
 *   - NG x 32 words: the groups' s and z, group-major;
 *   - Dp / 4 x 32 half-words: channels 4 u .. + 3 of the tokens' values;
 *   - NG x 32 words: the value groups' s and z.
 * A token's slot is page number * page + its place in the page.
 *
 * dtype of K, V, Q, out: QE_F32, QE_F16 or QE_BF16; a head's dim channels are
 * contiguous, tokens and heads lie at the given strides (in elements; an output's
 * elements must not overlap).  Pointers are multiples of their elements' size, pages and the
 * workspace of 16 (QE_ERR_ARG otherwise).
 * ------------------------------------------------------------------------ */
#define QE_F32  0
#define QE_F16  1
#define QE_BF16 2

/* Bytes of one page; 0 where the sizes are not supported. */
int64_t qe_kv_page_bytes(int kv_heads, int dim, int group, int page);

/* Quantizes K and V (tokens x kv_heads x dim) into the slots (device int64, one
 * per token; the slots of a call that are not negative must differ).  A negative slot skips
 * its token; so does one past the cache, which also sets QE_ERR_ARG in `status` (NULL, or a
 * device int that the call never clears).  Other tokens of the cache keep their bits.
 * tokens = 0: nothing is done. */
qe_status qe_kv_write(const void* K, const void* V, int dtype, int64_t tokens, int kv_heads, int dim,
                      int64_t k_stride, int64_t k_head_stride, int64_t v_stride, int64_t v_head_stride,
                      const int64_t* slots, int group, void* pages, int64_t num_pages, int page,
                      int* status, void* stream);

/* The values s (n - z) that the cache holds at the slots, rounded once to dtype.
 * Any slots, in any order; a negative one, or one past the cache (QE_ERR_ARG in
 * `status`), gives zeros. */
qe_status qe_kv_read(const void* pages, int64_t num_pages, int page, const int64_t* slots, int64_t tokens,
                     int kv_heads, int dim, int group, void* K, void* V, int dtype, int64_t k_stride,
                     int64_t k_head_stride, int64_t v_stride, int64_t v_head_stride, int* status,
                     void* stream);

/* Pages and slots of a step.  Sequence b has lengths[b] tokens, in the pages table[b * width + j],
 * j < held = max(ceil(lengths[b] / page), keep[b]); the pages that nobody has are free_pages[0] .. [*free_count - 1], a
 * stack whose top is its end, of the num_pages pages 0 .. num_pages - 1.  The call gives every sequence counts[b] more
 * tokens (or takes -counts[b] back, down to none), with new = max(lengths[b] + counts[b], 0) and
 * want = max(ceil(new / page), keep[b]):
 *  - first the pages j = want .. held - 1 of all sequences go back onto the stack, the r-th of them (sequences and
 *    pages in ascending order) to the place r below the new top, and their table entries become -1;
 *  - then the pages j = held .. want - 1 are taken from the top in the same order.  A sequence gets all its pages or none:
 *    those that want any get them as long as the pages wanted up to and including theirs are there, those that want none need
 *    none.  A sequence without its pages keeps its length, and its tokens get the slot -1 (attention with this call's q_start
 *    takes its rows for its last tokens: they mean nothing);
 *  - lengths[b] = new.  keep (NULL: 0): so many of the row's first entries are the caller's, for instance a prefix that
 *    several sequences share.  They are neither pushed, nor taken, nor changed.
 * A next call whose counts are the lengths before this one less those after it restores table, lengths and stack: the
 * opposite counts, but 0 for a sequence that was refused (its pages were not there, its rows passed `total`, its arguments were
 * bad), which has no new tokens to take back and would lose as many of its old ones, and no more than a sequence had
 * where a count took it down to none.
 * Out, all on the device: q_start[b] = the sum of max(counts, 0) before b (batch + 1 entries, cut off at
 * `total`); for row i of the call, which is token lengths[b] + i - q_start[b] (the length before the call) of the
 * sequence with q_start[b] <= i < q_start[b + 1], positions[i] = that token and slots[i] = table page * page + token %
 * page.  Rows from q_start[batch] on, which a graph recorded for `total` rows may have, get -1 in both.
 * lacking (NULL, or one int): the pages that were wanted and not there, 0 where every sequence has its own.
 * QE_ERR_ARG in the workspace's status word (never cleared here) says that the call met
 *  - lengths below 0 or past width * page before or after the call, or keep outside of 0 .. width: such a sequence stays as it
 *    is, and its rows get -1;
 *  - rows past `total`: a sequence that has one stays as it is, its rows before `total` get positions but no slots (a sequence
 *    without new tokens has no rows, wherever it stands);
 *  - a stack outside of 0 .. num_pages, which is cut off, or page numbers outside of the cache that were taken: their tokens get no
 *    slots.
 * batch up to 2^20 (QE_ERR_UNSUPPORTED beyond).  No two rows of table may be the same memory. */
size_t qe_kv_extend_workspace_size(int64_t batch);
qe_status qe_kv_extend(const int32_t* counts, int64_t batch, int32_t* table, int64_t width, int32_t* lengths,
                       const int32_t* keep, int32_t* free_pages, int64_t num_pages, int32_t* free_count, int page,
                       int64_t total, int64_t* slots, int32_t* positions, int32_t* q_start, int32_t* lacking, void* ws,
                       size_t ws_bytes, void* stream);

/* Queries and keys of new tokens, normed and rotated, and keys and values written into the slots, in one
 * pass: out (tokens x heads x dim, may be Q itself, element for element) gets the queries, the cache what qe_kv_write would
 * write for the keys before their rounding to dtype.  For a row x of a head's query (or key), each step one fp32 rounding:
 *   norm (where the weight, dim floats, is not NULL): r = 1 / sqrt(sum x^2 / dim + eps), formed in fp64,
 *     y = (x r) weight;
 *   rotation of the first rot channels (rot even, at most dim; 0: none) by row positions[token] of cos and sin
 *     (rows x rot / 2 floats): a' = a c - b s, b' = b c + a s for the pairs (a, b) of channels (i, i + rot / 2), or
 *     (2 i, 2 i + 1) with interleaved, and c, s the row's entries i;
 * queries are then rounded to dtype.  A token whose position is negative is skipped: its row of out and the
 * cache stay; so is one whose position is not below rows, which also sets QE_ERR_ARG in `status`.  positions
 * may be NULL without rotation.  A token whose slot is negative (or past the cache: QE_ERR_ARG) gets its query alone.
 * Slots, group, pages, strides and status as in qe_kv_write. */
qe_status qe_kv_append(const void* Q, const void* K, const void* V, int dtype, int64_t tokens, int heads, int kv_heads, int dim,
                       int64_t q_stride, int64_t q_head_stride, int64_t k_stride, int64_t k_head_stride, int64_t v_stride,
                       int64_t v_head_stride, const float* q_weight, const float* k_weight, double eps,
                       const int32_t* positions, const float* cos, const float* sin, int64_t rows, int rot, int interleaved,
                       const int64_t* slots, int group, void* pages, int64_t num_pages, int page, void* out, int64_t o_stride,
                       int64_t o_head_stride, int* status, void* stream);

/* Attention over the cache.  Sequence b has lengths[b] cached tokens, token t in
 * page table[b * width + t / page], and the queries q_start[b] .. q_start[b + 1] - 1
 * of the `total` rows of Q (total x heads x dim); with q_start NULL the queries
 * b max_q .. b max_q + max_q - 1.  Its i-th of nq queries stands at token
 * pos = lengths[b] - nq + i, so new tokens are written before the call.  Query head h
 * uses key/value head h / (heads / kv_heads).  The query sees the tokens
 *   t < lengths[b];  causal: t <= pos;  window > 0 (causal only): t > pos - window,
 * and out = sum_t p_t v_t, p the softmax over them of
 *   scale q . k_t + slopes[h] (t - pos)       (slopes NULL: without the last term;
 *                                              causal only).
 * A row that sees no token is 0, its lse -infinity.  lse: NULL or total x heads floats
 * (device): the natural logarithm of the softmax's denominator.  Rows of Q that are no
 * sequence's (before q_start[0], from q_start[batch] on) are neither read nor written.
 * Products run on the fp16 matrix cores: codes are exact there, a query row is
 * scaled by a power of two and rounded to fp16 (exact for fp16 and bf16 inputs up to
 * 2^-25 of the row's largest value; fp32 rows and their probabilities are split into two
 * fp16 parts each), probabilities times value scales are rounded to fp16 (to 2^-11 of
 * themselves, or 2^-35 of the largest such product of the row and channel group where that
 * is more, or 2^-145); statistics and sums are fp32.  Scores whose sum over d of |q_d| times the key
 * scales passes fp32's largest number with the largest |q_d| taken as 2^15 are infinite (keys from about
 * 1e31 on).
 * max_q: at least every nq.  batch * kv_heads * (max_q * heads / kv_heads / 16 + 1) above 2^23 is
 * QE_ERR_UNSUPPORTED.  Lengths past width * page, queries past `total` or max_q and
 * page numbers outside of the cache set QE_ERR_ARG in the workspace's status word (which
 * this call never clears; qe_sync_status does) and count as absent.
 * The lengths are known to the device alone: the work is cut into splits along the tokens, and
 * tiles are chosen, for sequences that fill the table (or the window).  A table much wider than its
 * sequences costs a small call workgroups without work and the launch that joins splits.  Few
 * rows take more splits, so a smaller call may need a larger workspace: ask for each. */
size_t qe_kv_attn_workspace_size(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads,
                                 int dim);
qe_status qe_kv_attn(const void* Q, int dtype, int64_t total, int heads, int dim, int64_t q_stride,
                     int64_t q_head_stride, const int32_t* q_start, int64_t batch, int64_t max_q,
                     const void* pages, int64_t num_pages, int page, int kv_heads, int group,
                     const int32_t* table, int64_t width, const int32_t* lengths, float scale,
                     int causal, int window, const float* slopes, void* out, int64_t o_stride,
                     int64_t o_head_stride, float* lse, void* ws, size_t ws_bytes, void* stream);

/* qe_kv_attn (the same arguments, results and workspace) with the first tokens of every sequence visible beside the window: a
 * query sees the tokens t <= pos with t > pos - window or t < sinks, each once where both hold.  Only the records of the two
 * ranges are read.  window = 0 hides nothing, and sinks then change nothing.  Slopes count the tokens' true distance.
 * sinks >= 0; causal only where not 0 (QE_ERR_ARG). */
qe_status qe_kv_attn_sinks(const void* Q, int dtype, int64_t total, int heads, int dim, int64_t q_stride,
                           int64_t q_head_stride, const int32_t* q_start, int64_t batch, int64_t max_q,
                           const void* pages, int64_t num_pages, int page, int kv_heads, int group,
                           const int32_t* table, int64_t width, const int32_t* lengths, float scale, int causal,
                           int window, int sinks, const float* slopes, void* out, int64_t o_stride, int64_t o_head_stride,
                           float* lse, void* ws, size_t ws_bytes, void* stream);

/* qe_kv_attn without a window for sequences that begin with the same pages (one system prompt, the branches of a request):
 * the sequences groups[g] .. groups[g + 1] - 1 (device, ngroups + 1 ascending entries from 0 to batch; sequences outside of
 * them share nothing) have the same first shared[g] page numbers in their rows of table.  The result is qe_kv_attn's,
 * up to the rounding of sums: the tokens of these pages that every query of the group sees (the whole records of 32 of them)
 * are read through the row of the group's first sequence that has queries, once for the queries of all of them, the others sequence
 * by sequence.  So the shared pages may be filled in part, or be longer than a sequence; sequences without queries do not
 * count, and their rows may hold anything.  A group of one sequence shares nothing.  A call that cannot gain by the sizes that the host
 * knows, rows, heads and the table's width, and one of more than 1024 groups, is qe_kv_attn itself.  Lengths and shared
 * pages are the device's: in a table much wider than the sequences are, or behind short prefixes, the call can be slower than
 * qe_kv_attn (5 to 20 us on an MI355X), and a program that knows them calls that.
 * Beside what qe_kv_attn checks, groups that do not ascend or leave 0 .. batch (then nothing is shared) and
 * shared[g] outside of 0 .. width set QE_ERR_ARG in the workspace's status word.  That the pages are the same is not
 * checked.  The queries of a sequence with a bad range in q_start are not computed. */
size_t qe_kv_attn_shared_workspace_size(int64_t total, int64_t batch, int64_t max_q, int heads, int kv_heads,
                                        int dim, int64_t ngroups);
qe_status qe_kv_attn_shared(const void* Q, int dtype, int64_t total, int heads, int dim, int64_t q_stride,
                            int64_t q_head_stride, const int32_t* q_start, int64_t batch, int64_t max_q,
                            const void* pages, int64_t num_pages, int page, int kv_heads, int group,
                            const int32_t* table, int64_t width, const int32_t* lengths, const int32_t* groups,
                            const int32_t* shared, int64_t ngroups, float scale, int causal, const float* slopes, void* out,
                            int64_t o_stride, int64_t o_head_stride, float* lse, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QE_H */
