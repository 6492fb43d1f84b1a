/*
 * imunpack.h -- C ABI of the MI355X (gfx950) exact low-bit integer GEMM library.
 *
 * The operations are those of "IM-Unpack: Training and Inference with Arbitrarily Low
 * Precision Integers" (arXiv 2403.07339):
 *
 *   Sec. 1, Eq. (gemm)            C = A B^T,  A: n x d,  B: h x d,  C: n x h
 *   Sec. 2, Eq. (quantized_A)     A_q = round(A / scale)            (all entries, no clipping)
 *   Sec. 2, Eq. (quantized_gemm)  C  ~= scale_A * scale_B * (A_q B_q^T)
 *   Sec. 4                        s = 2^(b-1); an entry v is In-Bound iff |v| <= s-1, else
 *                                 Out-of-Bound (OB, a "heavy hitter")
 *   Sec. 4, Eq. (mod)             digits m(v, s, i), each In-Bound, v = sum_i s^i m(v, s, i)
 *   Alg. 1 / 2 / 4 / 5            UnpackRow, UnpackColumn, UnpackBoth and the dispatcher Unpack
 *   Sec. 4 "Combining everything" (A_u, B_e, S_u, Pi_A)    = Unpack(A,   B,   I,   b, strategy_A)
 *                                 (B_eu, A_ue, S_uu, Pi_B) = Unpack(B_e, A_u, S_u, b, strategy_B)
 *                                 A B^T = Pi_A A_ue S_uu B_eu^T Pi_B^T
 *   Alg. 3                        ScaledMatMul: one low-bit GEMM per distinct diagonal entry of S
 *   Sec. 4.2                      unpack ratio r = n' d' h' / (n d h)
 *
 * Throughout, "row" is the non-contracted index (n or h) and "column" the contracted one (d).
 * Digits follow the sign-magnitude reading of floor/mod: digit i of v is
 * sign(v) * ((|v| >> (b-1) i) & (s-1)), which is the only reading under which every digit lies in
 * the symmetric In-Bound interval the paper states.  Rounding is IEEE binary32 division followed
 * by round-half-to-even.  UnpackBoth breaks ties between equal OB counts by the lowest index
 * (rows before columns when the two top counts are equal, as Alg. 4 prints).
 *
 * Conventions
 *   - Every pointer named "device" is GPU memory owned by the caller (hipMalloc / a PyTorch
 *     tensor); "host" pointers are ordinary host memory.  The library owns only plan objects and
 *     batch contexts.
 *   - A plan object belongs to one thread at a time.  Calls that take a const plan only read it;
 *     the others (re-planning, unpack, GEMM, the bound queries and the exports) update state kept in
 *     it (host mirrors of device results, lazily built tables) and must not run concurrently on the
 *     same plan.  Different plans are independent.
 *   - Every function returns IMUNPACK_OK (0) or a negative error code; nothing throws or aborts.
 *   - stream is a hipStream_t passed as void* (NULL = the default stream).  Calls are
 *     asynchronous on it unless stated otherwise.
 *   - All matrices are row-major; ld* is the distance in elements between consecutive rows.
 *   - 2 <= b <= 8: unpacked operands are stored as int8 for every b, or on request as 6-bit
 *     floating-point codes for b <= 4 (imunpack_plan_set_digits).
 */
#ifndef IMUNPACK_H
#define IMUNPACK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void *imunpack_stream_t;
typedef struct imunpack_plan imunpack_plan_t;
typedef struct imunpack_batch imunpack_batch_t;

enum { IMUNPACK_ROW = 0, IMUNPACK_COL = 1, IMUNPACK_BOTH = 2 };

enum {
    IMUNPACK_OK = 0,
    IMUNPACK_EINVAL = -1, /* null pointer, b outside [2,8], unknown strategy, bad sizes or strides */
    IMUNPACK_ERANGE = -2, /* a value or an accumulator bound does not fit (see each call)           */
    IMUNPACK_ENOMEM = -3, /* device or host allocation failed                                       */
    IMUNPACK_EHIP = -4,   /* a HIP call failed; see imunpack_last_hip_error()                       */
    IMUNPACK_ESMALL = -5  /* a caller buffer or workspace is too small                              */
};

/* Heavy-hitter statistics of one integer operand (device pointers, lengths rows / cols):
 * OB count and largest magnitude per row and per column.  (Sec. 4: the IB/OB predicate;
 * Alg. 1 line 3, Alg. 2 line 3, Alg. 4 line 3 consume them.)
 * Optionally also the list of the OB entries themselves, which UnpackBoth (Alg. 4) works on:
 * ob holds 3 * ob_cap int32 laid out as [rows | cols | values], *ob_count (device) the number of
 * OB entries found -- if that exceeds ob_cap the list is incomplete and the planner scans the
 * operand itself.  ob == NULL (ob_cap == 0) skips the list. */
typedef struct {
    int32_t *rowcnt;
    int32_t *colcnt;
    int32_t *rowmax;
    int32_t *colmax;
    int32_t *ob;
    int64_t ob_cap;
    int32_t *ob_count;
} imunpack_stats_t;

/* ---- (0) the range estimate that sets the RTN step ----------------------------------------------
 * Sec. 2, the sentence after Eq. (quantized_A): alpha_p(A), the p-th percentile of the magnitudes of
 * A: the smallest magnitude a such that at least p % of the entries lie in [-a, a], i.e. the k-th
 * smallest |x| with k = ceil(p * rows * cols / 100) (an entry of A, no interpolation).  With beta
 * integers to cover [-alpha_p, alpha_p], Eq. (quantized_A) is imunpack_quantize with
 * scale = alpha_p / (0.5 * beta).
 * X: device, element (r, c) at X[r*sx_r + c*sx_c], strides > 0.  0 < p <= 100; rows * cols < 2^32.
 * alpha: device, one float, written when the stream gets there.  status_flag: device, may be NULL;
 * set to 1 if X holds a NaN (alpha is then meaningless), else 0.  workspace: device,
 * IMUNPACK_PERCENTILE_WORKSPACE_BYTES, contents irrelevant before and after.  Errors: EINVAL. */
#define IMUNPACK_PERCENTILE_WORKSPACE_BYTES 16384
int imunpack_percentile(const float *X, int64_t rows, int64_t cols, int64_t sx_r, int64_t sx_c,
                        double p, float *alpha, int32_t *status_flag, void *workspace,
                        imunpack_stream_t stream);

/* The RTN step of Eq. (quantized_A) itself, formed on the device: beta integers are to cover
 * [-alpha_p, alpha_p], so one step is alpha_p / (0.5 beta) (one binary32 division; Sec. 2, the sentence
 * after Eq. (quantized_A) defines alpha_p).  A matrix whose p-th percentile is 0 (mostly zeros) falls back
 * to its largest magnitude, an all-zero one to the step 1.  Arguments as imunpack_percentile; step:
 * device, one float, written when the stream gets there (imunpack_gemm_batched hands such steps from
 * kernel to kernel without the host reading them).  Errors: EINVAL (also beta not a positive finite number). */
int imunpack_rtn_step(const float *X, int64_t rows, int64_t cols, int64_t sx_r, int64_t sx_c, double p,
                      float beta, float *step, int32_t *status_flag, void *workspace,
                      imunpack_stream_t stream);

/* The same range estimate for callers that cannot allocate device memory or bring a workspace (code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the counters and the
 * selection state live in a fixed array of IMUNPACK_PERCENTILE_WORKSPACE_BYTES of device memory that the
 * library's code object carries, one copy per GPU, held until the process ends.  The call itself
 * allocates and frees nothing.  Arguments, result and errors as imunpack_percentile without the
 * workspace, except that more than IMUNPACK_PERCENTILE_STATIC_MAX_ENTRIES entries (what the array's
 * 32-bit counters can count) return ERANGE.  The array is cleared at the start of every call; all calls
 * on one GPU share it, so two calls that overlap on one GPU (different streams or threads) race: issue
 * them on one stream, or order them with events. */
#define IMUNPACK_PERCENTILE_STATIC_MAX_ENTRIES 4294967295ll
int imunpack_percentile_static(const float *X, int64_t rows, int64_t cols, int64_t sx_r, int64_t sx_c,
                               double p, float *alpha, int32_t *status_flag, imunpack_stream_t stream);

/* ---- (1)+(2) RTN quantisation fused with the heavy-hitter scan --------------------------------
 * Sec. 2, Eq. (quantized_A) with the step supplied by the caller:
 *     Q[r*ldq + c] = rint(X[r*sx_r + c*sx_c] / scale)      (int32, no clipping)
 * The paper prints the scaling as a multiplication by 0.5 beta / alpha_p; the reading taken here is a
 * binary32 division by the step scale = alpha_p / (0.5 beta) (the two can differ in the last bit of
 * the quotient, and so at rounding ties; the oracle the library is checked against divides too).
 * and, in the same pass, the statistics of Q for bit width b (any of the four stats pointers, or
 * stats itself, may be NULL to skip it).  X, Q, stats, status: device.  X may be any strided view
 * with sx_r, sx_c >= 1 (sx_c == 1 and sx_r == 1 have fast paths); Q is written row-major.
 * status (device int32, may be NULL) is set to 0, then to 1 if any input is NaN/Inf or any
 * quotient has magnitude >= 2^31 (such outputs are written as 0); the call itself still returns
 * IMUNPACK_OK -- read status when convenient.
 * Errors: EINVAL (null X/Q, rows/cols < 0, a stride < 1, ldq < cols, scale not finite or <= 0,
 * b outside [2,8]). */
int imunpack_quantize(const float *X, int64_t rows, int64_t cols, int64_t sx_r, int64_t sx_c,
                      float scale, int b, int32_t *Q, int64_t ldq,
                      const imunpack_stats_t *stats, int32_t *status, imunpack_stream_t stream);

/* The same for both operands of one product A B^T (A: n x d, B: h x d, Sec. 2 Eq. (quantized_A) applied to
 * each with its own step): results as two imunpack_quantize calls, issued as one clearing launch and,
 * when both operands take the unit-column-stride fast path, one launch over the rows of both (fewer
 * launches, and the shorter operand fills the tail of the longer one).  status (device, may be NULL):
 * two int32, status[0] for A and status[1] for B.  Errors: as imunpack_quantize. */
int imunpack_quantize_pair(const float *A, int64_t n, int64_t sa_r, int64_t sa_c, float scale_A, int32_t *QA,
                           int64_t ldqa, const imunpack_stats_t *stats_A, const float *B, int64_t h,
                           int64_t sb_r, int64_t sb_c, float scale_B, int32_t *QB, int64_t ldqb,
                           const imunpack_stats_t *stats_B, int64_t d, int b, int32_t *status,
                           imunpack_stream_t stream);

/* ---- (2) stand-alone scan of an integer operand (Sec. 4, IB/OB definition) -------------------- */
int imunpack_scan(const int32_t *Q, int64_t rows, int64_t cols, int64_t ldq, int b,
                  const imunpack_stats_t *stats, imunpack_stream_t stream);

/* ---- strategy choice (Sec. 4.2, unpack ratio r = n'd'h' / (ndh); the "Mix" rows of its tables) -
 * Prices the four pairs of the one-axis strategies from the scan statistics alone, without
 * unpacking: UnpackRow / UnpackColumn append one slot per further digit of the largest magnitude of
 * a row / column, so n', d', h' follow from rowmax / colmax (for UnpackColumn on both operands a
 * column k of A with LA digits meets LB digits of column k of B: LA * LB columns).
 * stats_A, stats_B: device, rowmax and colmax required.  workspace: device, 8-byte aligned,
 * IMUNPACK_PRICE_WORKSPACE_BYTES, contents irrelevant before and after (the call allocates nothing).
 * dims_out (host, may be NULL): [pair][3] = n', d', h' for the pairs (strategy_A, strategy_B) =
 * (ROW,ROW), (ROW,COL), (COL,ROW), (COL,COL); ratio_out (host, may be NULL): their r.  best_A / best_B
 * (host, may be NULL): the pair with the smallest r (first in that order on ties).  UnpackBoth is
 * priced by planning with it (imunpack_plan + imunpack_plan_dims).  Synchronises the stream.
 * Errors: EINVAL, ERANGE (a size does not fit int64), EHIP. */
#define IMUNPACK_PRICE_WORKSPACE_BYTES 64
int imunpack_price(const imunpack_stats_t *stats_A, int64_t n, const imunpack_stats_t *stats_B,
                   int64_t h, int64_t d, int b, void *workspace, int64_t *dims_out, double *ratio_out,
                   int *best_A, int *best_B, imunpack_stream_t stream);

/* ---- (3) unpack plan (Alg. 1, 2, 4, 5 and the two-operand composition of Sec. 4) -------------
 * Decides every row / column split for A (with B as partner) and then for B (with A_u as partner
 * and S_u carried over) without moving the operands.  A: n x d, B: h x d, int32, device.
 * stats_A / stats_B: statistics of A / B for this b as written by imunpack_quantize or
 * imunpack_scan; NULL lets the call scan the operand itself.  For an UnpackBoth operand the OB
 * entry list of its statistics is used if it is complete, and copied: nothing of stats_A / stats_B
 * is read after the call returns.
 * *plan == NULL creates a plan object; a non-NULL *plan is re-planned in place and its device
 * buffers are reused (they only grow), so that steady-state calls allocate nothing.
 * Synchronises the stream (the sizes n', d', h' are needed on the host).
 * Errors: EINVAL; ERANGE if an exponent group is too long for int32 accumulation or a weight
 * s^k would not fit 62 bits; ENOMEM; EHIP. */
int imunpack_plan(const int32_t *A, int64_t n, int64_t d, int64_t lda,
                  const int32_t *B, int64_t h, int64_t ldb,
                  int b, int strategy_A, int strategy_B,
                  const imunpack_stats_t *stats_A, const imunpack_stats_t *stats_B,
                  imunpack_plan_t **plan, imunpack_stream_t stream);

/* Sizes of the unpacked problem (host outputs; any may be NULL): n', d', h' of Sec. 4.2 and the
 * number of distinct diagonal entries of S_uu (the GEMM groups of Alg. 3). */
int imunpack_plan_dims(const imunpack_plan_t *plan, int64_t *n_u, int64_t *d_u, int64_t *h_u,
                       int32_t *n_groups);

/* The plan in the order the paper's algorithms produce it (host buffers sized from
 * imunpack_plan_dims; any may be NULL).  Pi_A column R is s^rowA_exp[R] at row rowA_src[R]; Pi_B
 * likewise; S_uu[c,c] = s^col_exp[c]; col_src[c] is the original column that unpacked column c
 * descends from; col_parent[c] is the column that column c was appended for (the one whose
 * floor(. / s) it took and whose copy the partner received: Alg. 2 lines 4-7, Alg. 4 lines 11-14),
 * -1 for the d original columns.  ops (3 * (n' - n + h' - h + d' - d) int32, that count also written
 * to *n_ops) lists every split in the order the paper's algorithms make them, as triples
 * (0 = first / 1 = second Unpack call of Sec. 4 "Combining everything", 0 = row split / 1 = column
 * split, index of the split row or column at that moment).
 * Synchronises the stream used by imunpack_plan. */
int imunpack_plan_export(imunpack_plan_t *plan,
                         int32_t *rowA_src, int32_t *rowA_exp,                   /* n' */
                         int32_t *rowB_src, int32_t *rowB_exp,                   /* h' */
                         int32_t *col_src, int32_t *col_exp, int32_t *col_parent, /* d' */
                         int32_t *ops, int64_t *n_ops);

int imunpack_plan_destroy(imunpack_plan_t *plan);

/* ---- weights that stay resident (Sec. 4.2: weights are unpacked once, when they are loaded) -----
 * The unpacking of the second operand, Unpack(B_e, A_u, S_u, b, strategy_B), depends on the first operand
 * only through the column slots of A's unpacking (which columns B_e repeats, and their exponents).
 * keep != 0 is the caller's promise that from now on B, its statistics and its OB list are the same in
 * every imunpack_plan on this plan object: a plan call then compares, on the device, the column slots of
 * A's unpacking with those of the call before and, if they are the same, takes the second operand's
 * unpacking (for UnpackBoth: without running Alg. 4 on it again) and the layouts of B's rows and of the
 * columns over as they stand (the result is the same plan either way; if they differ, the host may wait a
 * second time); the first
 * imunpack_unpack after such a plan call writes only the A store if it is given the B_eu buffer that the
 * unpack before wrote (same address, same digit format): B_eu and its row norms are already what they
 * would become.  Otherwise, and in the first call after keep was set, B is unpacked as usual.
 * imunpack_plan_weights_reused tells which of the two the last plan call did.  keep == 0 (the default)
 * ends the promise.  Errors: EINVAL (null plan). */
int imunpack_plan_keep_weights(imunpack_plan_t *plan, int keep);
int imunpack_plan_weights_reused(const imunpack_plan_t *plan);

/* ---- digit storage format of the unpacked operands ---------------------------------------------
 * Sec. 4.2 ("arbitrarily low" bit widths): for b <= 4 every digit lies in [-7, 7] and is exactly
 * representable in the 6-bit floating-point format e2m3 (1 sign, 2 exponent, 3 mantissa bits), which the
 * matrix cores multiply at twice the int8 rate and which takes three quarters of the bytes.  The
 * products and their sums are integers below 2^24 in binary32 accumulators, hence exact (the call
 * checks the bound, as it does for int32); results are bit-identical to the int8 path.
 * IMUNPACK_DIGITS_INT8 (default): one int8 per digit.  IMUNPACK_DIGITS_FP6: 96 bytes per 128 columns; a
 * group of 64 columns takes 48 bytes: the 32 columns of each half form a 192-bit string (column j at
 * bits 6j .. 6j+5), stored as the first 16 bytes of both strings followed by the last 8 bytes of both
 * (those two in the other order in physical rows whose index has bit 4 set).  Physical rows 2i and 2i + 1 share their bytes: row 2i
 * holds the 96 bytes of both for every even group of 128 columns, row 2i + 1 for every odd one (zeros behind
 * a last group without a partner, unless it is the only one).  The request stays with the plan object
 * across re-planning and is in effect whenever the plan's b <= 4 (a plan with b > 4 keeps int8);
 * imunpack_plan_digits returns the format in effect.  Call after imunpack_plan and before
 * imunpack_unpacked_bytes / imunpack_unpack: the format changes the sizes and the row pitches.
 * Errors: EINVAL (no valid plan, unknown format, FP6 on a plan with b > 4). */
enum { IMUNPACK_DIGITS_INT8 = 0, IMUNPACK_DIGITS_FP6 = 1 };
int imunpack_plan_set_digits(imunpack_plan_t *plan, int format);
int imunpack_plan_digits(const imunpack_plan_t *plan);

/* ---- (4) digit scatter (Eq. (mod); Alg. 1 l.4-5, Alg. 2 l.4-6, Alg. 4 l.7-8, 11-13) -----------
 * Writes the unpacked operands as int8 in the plan's *physical* layout: rows grouped by source row (all
 * digit levels of a row of A inside one 64-row chunk of a GEMM tile, of a row of B inside one tile),
 * both padded to tile multiples; physical rows 2i and 2i + 1 share their bytes: row 2i holds the columns 128 k .. 128 k + 63 of both (64
 * of row 2i, 64 of row 2i + 1, and so on), row 2i + 1 the others.  B_eu is stored in full, its columns grouped by diagonal entry of S_uu
 * in whole k-tiles of 128.  Of A_ue only the columns of A_u are stored, each once ("A store"): where
 * column unpacking of the partner repeats a column (Alg. 2 line 6 / Alg. 4 line 13) the GEMM reads the
 * stored one again, so the copies cost neither memory nor traffic.
 * imunpack_unpacked_bytes gives the buffer sizes and the workspace an un-fused GEMM needs.
 * A, B: the int32 operands the plan was made from.  A_ue, B_eu: device, caller-allocated.
 * imunpack_unpack does not wait for the device: the accumulator bounds that select the GEMM path
 * reach the host later, and imunpack_gemm / imunpack_plan_fusable wait for them.  A plan may be unpacked
 * again, into the same or other buffers, also by the replays of a graph and beside an imunpack_gemm on other
 * buffers: what the plan itself holds for the GEMM is written once or again with the same bytes. */
int imunpack_unpacked_bytes(const imunpack_plan_t *plan, size_t *bytes_A, size_t *bytes_B,
                            size_t *bytes_workspace);
/* The shape of the two buffers (host output, six values): physical rows, stored columns and bytes from
 * one row to the next, of the A store and then of B_eu.  bytes_A = rows * pitch.  The bytes of a row
 * behind its stored columns (six-bit digits: behind those of an even number of groups of 128) are neither written nor read. */
int imunpack_plan_layout(const imunpack_plan_t *plan, int64_t *shape);
int imunpack_unpack(imunpack_plan_t *plan, const int32_t *A, int64_t lda,
                    const int32_t *B, int64_t ldb, int8_t *A_ue, int8_t *B_eu,
                    imunpack_stream_t stream);

/* Test aid: re-orders the physical operands into the paper's order, dense n' x d' and h' x d'. */
int imunpack_unpack_canonical(imunpack_plan_t *plan, const int8_t *A_ue, const int8_t *B_eu,
                              int8_t *A_canon, int8_t *B_canon, imunpack_stream_t stream);

/* ---- (5) int8 MFMA GEMM (Alg. 3) ---------------------------------------------------------------
 * Runs C_g = A_ue[:, I_g] B_eu[:, I_g]^T for every group g of equal diagonal entry with int32
 * accumulation on v_mfma_i32_*_i8 and combines the groups by shifts (six-bit digits: binary32
 * accumulation of integers below 2^24 on v_mfma_f32_32x32x64_f8f6f4, the bound below is 2^24 then).
 * fuse != 0: one launch; the recombination (6) and the dequantisation run in the epilogue and
 *   C_int (n x h int64, device, may be NULL) and/or C_fp (n x h fp32, device, may be NULL) are
 *   written directly (columns that UnpackBoth appended to B for a few heavy hitters each are not multiplied as columns: their digits,
 *   which the plan holds too, meet a transposed copy of A's columns that the plan keeps).  This needs the shifted sum of all groups to fit int32 for this plan's
 *   operands (bound measured by imunpack_unpack); if it does not, the call falls back to the
 *   un-fused path when workspace != NULL and returns ERANGE otherwise.  Products whose tiles are cut along the
 *   contraction meet in a buffer of 64 MiB that the first of them allocates (without it, and under stream
 *   capture, the tiles stay whole) and that stays with the plan object; calls that share it are ordered,
 *   whatever streams they are on.
 * fuse == 0: writes the unpacked product C_u = A_ue S_uu B_eu^T as int64 into workspace
 *   (imunpack_unpacked_bytes) for imunpack_recombine; C_int / C_fp are ignored.
 * ldc: row stride of C_int and C_fp in elements (>= h).  scale_A, scale_B: the RTN steps. */
int imunpack_gemm(imunpack_plan_t *plan, const int8_t *A_ue, const int8_t *B_eu,
                  void *workspace, int64_t *C_int, float *C_fp, int64_t ldc,
                  float scale_A, float scale_B, int fuse, imunpack_stream_t stream);

/* ---- the whole path over a strided batch of products (Sec. 1 "Notations": the GEMMs of a Transformer) -
 * C_i = step_A,i * step_B,i * (RTN(A_i / step_A,i) RTN(B_i / step_B,i)^T), i = 0 .. batch-1, the integer
 * product evaluated exactly with b-bit digits (Sec. 4), as fp32.  Every item is a GEMM of its own: its own
 * percentile steps alpha_p / (0.5 beta) (Eq. (quantized_A)), its own unpack plan.  A_i: n x d at
 * A + i * sa_b, element (r, c) at offset r * sa_r + c * sa_c (so transposed operands are views, nothing is
 * copied); B_i: h x d likewise; C_i: n x h row-major at C + i * sc_b with row stride ldc.  All device, fp32.
 * *ctx == NULL creates a context; passing it again reuses its buffers (Q_A, Q_B, statistics, the unpacked
 * operands, a plan: they only grow), so steady-state calls allocate nothing.  The library owns the context;
 * release it with imunpack_batch_destroy.  The steps never leave the device.  The items share every launch (up to
 * 1024 at a time, fewer if they are large or device memory runs short) and the host waits twice per such group: for the sizes of the
 * unpacked problems and at the end; items that write where another one reads or writes (C_i = A_(i+1), sc_b = 0)
 * go one after the other in the order of i.  Synchronises the stream before returning.
 * Errors: EINVAL; ERANGE if any operand held a NaN or Inf or a quotient beyond 32 bits (the outputs of
 * that item are then undefined); ENOMEM; EHIP.
 * For b <= 4 the digits are stored as six-bit floating-point codes (imunpack_plan_set_digits); the
 * results are the same bits either way. */
int imunpack_gemm_batched(const float *A, int64_t sa_b, int64_t sa_r, int64_t sa_c,
                          const float *B, int64_t sb_b, int64_t sb_r, int64_t sb_c,
                          int64_t batch, int64_t n, int64_t d, int64_t h,
                          double p, float beta_A, float beta_B, int b, int strategy_A, int strategy_B,
                          float *C, int64_t sc_b, int64_t ldc, imunpack_batch_t **ctx,
                          imunpack_stream_t stream);
int imunpack_batch_destroy(imunpack_batch_t *ctx);

/* ---- (6) recombination and dequantisation (Sec. 4 "Reconstructing A"; Eq. (quantized_gemm)) ---
 * C_int = Pi_A C_u Pi_B^T by shift-and-add in int64 from the workspace of an un-fused
 * imunpack_gemm, and C_fp = scale_A * scale_B * C_int (one rounding to fp32).  Either output may
 * be NULL. */
int imunpack_recombine(const imunpack_plan_t *plan, const void *workspace,
                       float scale_A, float scale_B, int64_t *C_int, float *C_fp, int64_t ldc,
                       imunpack_stream_t stream);

/* ================================================================================================
 * Around the products of a Transformer: norm, optimiser's step, loss over a vocabulary
 * ================================================================================================
 * Types of arrays that come in more than one. */
enum { IMUNPACK_F32 = 0, IMUNPACK_BF16 = 1 };

/* ---- root-mean-square norm ----------------------------------------------------------------------
 * For each of `rows` rows of d elements:  h = x + residual (residual may be NULL: h = x),
 *     rstd = 1 / sqrt(mean_j h_j^2 + eps),   y_j = h_j rstd weight_j.
 * x, residual, y, h: device, of type dtype (IMUNPACK_F32 or IMUNPACK_BF16), unit stride within a row, ld* elements from row to
 * row (at least d; no alignment is asked for beyond that of an element).  weight: device, d elements of
 * weight_dtype.  h (may be NULL) is the residual stream that goes on, rstd (fp32, may be NULL) is for the backward pass.  y or h may be x or residual.
 * Statistics and products are binary32; y is computed from h before h is rounded to dtype.
 * rows == 0 is allowed.  Errors: EINVAL (null pointers, d outside [1, 2^24], a pitch < d, eps < 0 or NaN, unknown types). */
int imunpack_rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *weight,
                     int64_t rows, int64_t d, int dtype, int weight_dtype, float eps,
                     void *y, int64_t ldy, void *h, int64_t ldh, float *rstd, imunpack_stream_t stream);

/* The same norm with its output as integers that are In-Bound for bit width b (Sec. 4: |q| <= 2^(b-1) - 1, so as an operand of
 * imunpack_plan they are never split), in 8 bits with a step per row:
 *     scale = max_j |y_j| / (2^(b-1) - 1),   q_j = rint(y_j / scale)        (binary32 division, half to even)
 * scale: device, one fp32 per row (below 2^-126 rounded up where its few bits would put a q_j beyond b bits); 1 for a row of zeros; NaN for a row that holds a NaN or an infinity (its q are 0).
 * values (device, dtype, may be NULL): q_j * scale, for callers that go on in dtype.  Other arguments and errors as above
 * (also EINVAL for b outside [2,8]). */
int imunpack_rmsnorm_quantize(const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *weight,
                              int64_t rows, int64_t d, int dtype, int weight_dtype, float eps, int b,
                              int8_t *q, int64_t ldq, float *scale, void *values, int64_t ldv, void *h, int64_t ldh,
                              imunpack_stream_t stream);

/* Gradients of imunpack_rmsnorm for gy, the gradient of y, and gh, that of h (NULL: none; the residual stream brings one).  The
 * pass forms h = x + residual again from the same x and residual (in fp32, where h was not rounded, x = h without a residual
 * does as well and is one array less to read):
 *     gx_j = gh_j + rstd (gy_j w_j - h_j rstd^2 mean_k(gy_k w_k h_k))      (x and residual share it)
 *     gweight_j = sum over rows of gy_j h_j rstd
 * gweight: device, weight_dtype, may be NULL (then no workspace is needed).  The sums over rows are taken in a fixed order:
 * equal inputs give equal bits.  gx may be gy or gh.  workspace: device, 16-byte aligned, of the size that
 * imunpack_rmsnorm_backward_workspace gives (0 for few rows: NULL will do).  Errors: EINVAL as above; ESMALL. */
int imunpack_rmsnorm_backward_workspace(int64_t rows, int64_t d, int dtype, size_t *bytes);
int imunpack_rmsnorm_backward(const void *gy, int64_t ldgy, const void *x, int64_t ldx, const void *residual, int64_t ldres,
                              const void *gh, int64_t ldgh, const void *weight, const float *rstd, int64_t rows, int64_t d, int dtype, int weight_dtype,
                              void *gx, int64_t ldgx, void *gweight, void *workspace, size_t workspace_bytes,
                              imunpack_stream_t stream);

/* ---- AdamW over many tensors ---------------------------------------------------------------------
 * One step, t = step >= 1, for each of `count` tensors of numel[k] elements (numel[k] == 0 is skipped):
 *     m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *     p = (1 - lr weight_decay) p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * The arrays of pointers and numel are host memory and are not read after the call returns; what they point to is device memory,
 * contiguous.  params: fp32.  grads: grad_dtype.  copies (NULL, or one bfloat16 tensor each): receive p rounded.
 * state_bits 32: exp_avg[k] = m and exp_avg_sq[k] = v, fp32; m_scales and v_scales are not read.
 * state_bits 8: exp_avg[k] holds m and exp_avg_sq[k] the square root of v, as 8-bit floating-point codes (e4m3) times a scale (fp32)
 * for every IMUNPACK_ADAMW_BLOCK elements, m_scales[k] and v_scales[k]; codes go over whole blocks
 * (ceil(numel / block) * block bytes, what lies behind the tensor's end zero).  Codes are rounded up or down at random, with the
 * probability that leaves the means of m and of the root unchanged, by a hash of seed, step, k and the element: the same call gives the same bits.  v,
 * the root's square, is thereby about 5 % too large under gradients that keep their size, and the root scatters by some 16 %.  A root that is not zero keeps at
 * least the smallest code, 2^-18 of the largest of its block.  All zeros is the state before the first step.
 * NaN and infinity in a gradient go into the element (32 bits) or the whole block (8 bits).
 * Errors: EINVAL (null pointers, lr, eps or weight_decay negative or not finite, a beta outside [0, 1), step < 1, unknown
 * types). */
#define IMUNPACK_ADAMW_BLOCK 256
int imunpack_adamw(int64_t count, float *const *params, const void *const *grads, void *const *exp_avg,
                   void *const *exp_avg_sq, float *const *m_scales, float *const *v_scales, void *const *copies,
                   const int64_t *numel, int grad_dtype, int state_bits, double lr, double beta1, double beta2,
                   double eps, double weight_decay, int64_t step, uint32_t seed, imunpack_stream_t stream);

/* ---- softmax cross entropy over a vocabulary -------------------------------------------------------
 * With logits l = x W^T (x: rows x d, W: vocab x d, never kept as a whole) and target (device int64, one per row):
 *     loss_t = log sum_v exp l[t, v] - l[t, target_t]
 * and, for the gradient g_t of loss_t,  gx = G W,  gW = G^T x  with  G[t, v] = (softmax(l)[t, v] - [v = target_t]) g_t.
 * Rows whose target is ignore_index take no part, whatever x holds there: loss 0, gradient 0.  A target outside [0, vocab) makes the
 * row's loss (and a sum or mean) NaN and adds nothing to the gradients.
 * x, W, gx, gW: device, of type dtype, unit stride within a row, ld* elements from row to row (at least d).
 * bfloat16: products of bfloat16 operands, exponentials and G rounded to bfloat16, sums in fp32.
 * fp32: operands and G are sums of two binary16 numbers each, under a power of two.  Losses are within what fp32 sums of fp32 products give,
 * whatever the sizes of the rows of x and W.  Softmax minus one-hot is held to 2^-22 of itself or 2^-38.  gx and gW are within what fp32 sums give with
 * those, but add over rows that need one scale: gx[t] is besides off by up to 2^-38 |g_t| max |W| sum_v |softmax - one-hot|, gW[v] by up to
 * 2^-38 max_t(|g_t| max_k |x[t, k]|) sum_t |softmax - one-hot|.
 * Infinity or NaN in a row of x or in its gradient g_t: that row's loss and gx, and gW (both types); in W: every row.
 * reduction: IMUNPACK_NONE: loss has one fp32 per row; SUM, MEAN (over the rows that take part; 0 if there are none): one fp32.
 * loss (device) may be NULL if gradients are asked for, gx and gW (device) may each be NULL.  The gradients are made in the same call,
 * with the logits in memory for some rows at a time: they are those for grad, the gradient of loss (device, as many values; NULL: 1, not
 * with NONE).  imunpack_xent_rescale multiplies gradients that were made for 1 with *grad, in place, and leaves them alone if that is 1 (bfloat16: rounded
 * once more, unless by a power of two).
 * workspace: device, 16-byte aligned, of the size that imunpack_xent_workspace gives: x and W in the forms the products read and, for
 * gradients, G of a piece of the rows (2 GiB at most, unless 256 rows take more) and partial sums; for the loss alone up to 2 GiB of these.
 * All sums are taken in a fixed order: equal inputs give equal bits.  rows == 0 is allowed.
 * Errors: EINVAL (null pointers, rows or vocab above 2^22, d above 2^20, a pitch < d, unknown types); ESMALL; EHIP. */
enum { IMUNPACK_NONE = 0, IMUNPACK_SUM = 1, IMUNPACK_MEAN = 2 };
int imunpack_xent_workspace(const void *w, int64_t ldw, int64_t rows, int64_t d, int64_t vocab, int dtype, int want_grad,
                            size_t *bytes);
int imunpack_xent(const void *x, int64_t ldx, const void *w, int64_t ldw, const int64_t *target, int64_t rows, int64_t d,
                  int64_t vocab, int dtype, int64_t ignore_index, int reduction, float *loss, const float *grad,
                  void *gx, int64_t ldgx, void *gw, int64_t ldgw, void *workspace, size_t workspace_bytes,
                  imunpack_stream_t stream);
int imunpack_xent_rescale(const float *grad, void *gx, int64_t nx, void *gw, int64_t nw, int dtype, imunpack_stream_t stream);

/* ---- tensors in 8-bit floating point, a power of two for every block of 128 ------------------------
 * A tensor x of `rows` rows of `cols` elements is held as codes of one of the formats below and, for each row and each 128 consecutive
 * columns (a block; the last one may be shorter), a byte that stands for 2^(byte - 127):
 *     e = the smallest whole number >= -127 with max |x| over the block <= top 2^e   (0 for a block of zeros),   byte = e + 127,
 *     code = x 2^-e, rounded to nearest with ties to even,                       value = code 2^e.
 * top is 448 (E4M3: four exponent bits, three of fraction, no infinity) or 57344 (E5M2).  A value is within 2^-4 (E4M3) or 2^-3 (E5M2) of x relative to x, or
 * within 2^-10 2^e (2^-17 2^e); what rounds to 2^128 is infinite where it becomes fp32 or bfloat16 again.  Infinities and NaN do not count for max |x|; they become NaN codes (E5M2: infinity stays).
 * "Square" blocks are 128 rows x 128 columns: their byte stands in each of their rows.
 * codes: device, row r at codes + r ldc, ldc bytes at least 128 ceil(cols / 128): the codes behind a row's end, up to a whole block, are
 * zeros (the calls that write codes see to that, the product counts on it).  scales: device, the byte of row r and block j at
 * scales + r lds + j, lds at least ceil(cols / 128); a row may be read up to a whole 16 bytes.  Both bases 16-byte aligned, both pitches multiples of 16.
 * No output of the calls below may overlap an input.  All sums are taken in a fixed order: equal inputs give equal bits. */
enum { IMUNPACK_E4M3 = 0, IMUNPACK_E5M2 = 1 };
#define IMUNPACK_BLOCK8 128

/* x (device, dtype, unit stride within a row, ldx elements from row to row) in 8 bits: as it lies (codes, scales; both NULL: not), and turned
 * (turned, turned_scales; NULL: not): the tensor x^T of `cols` rows of `rows` elements, whose blocks run along x's columns.  square: square
 * blocks; turned then holds the same values.  rows == 0 is allowed.
 * Errors: EINVAL (null pointers, rows outside [0, 2^31], with turned 2^24, cols outside [1, 2^24], pitches or alignments as above, unknown types); EHIP. */
int imunpack_block8_quantize(const void *x, int64_t ldx, int64_t rows, int64_t cols, int dtype, int format, int square,
                             void *codes, int64_t ldc, void *scales, int64_t lds,
                             void *turned, int64_t ldt, void *turned_scales, int64_t ldts, imunpack_stream_t stream);

/* The same of a tensor that is in 8 bits already (rows x cols, any blocks): its values, turned, in blocks along its columns.  A value of e4m3 or e5m2
 * under another power of two is the same value, unless it falls below that block's smallest codes and is rounded to those.  (From 2^129 on, which no call here writes, values count as infinite.) */
int imunpack_block8_turn(const void *codes, int64_t ldc, const void *scales, int64_t lds, int64_t rows, int64_t cols, int format,
                         void *turned, int64_t ldt, void *turned_scales, int64_t ldts, imunpack_stream_t stream);

/* Up to four tensors by one launch, with the results of the two calls above for each: `imunpack_block8_quantize` where x_scales is NULL, otherwise
 * `imunpack_block8_turn` of the codes x with these scales (dtype is not looked at then, codes and square are 0).  All arguments are checked before anything is launched.
 * Errors: EINVAL (count outside [1, 4], and as above for each tensor); EHIP. */
#define IMUNPACK_BLOCK8_MANY 4
typedef struct imunpack_block8_job {
    const void *x;
    int64_t ldx;
    const void *x_scales;
    int64_t ldxs;
    int64_t rows, cols;
    int dtype, square;
    void *codes;
    int64_t ldc;
    void *scales;
    int64_t lds;
    void *turned;
    int64_t ldt;
    void *turned_scales;
    int64_t ldts;
} imunpack_block8_job;
int imunpack_block8_many(int count, const imunpack_block8_job *jobs, int format, imunpack_stream_t stream);

/* out (device, dtype, ldo elements from row to row) = the values of a tensor in 8 bits (bfloat16 holds them exactly, but for magnitudes from 2^128 on or below
 * 2^-133).  Errors as above. */
int imunpack_block8_values(const void *codes, int64_t ldc, const void *scales, int64_t lds, int64_t rows, int64_t cols, int format,
                           void *out, int64_t ldo, int dtype, imunpack_stream_t stream);

/* out = A B^T (+ bias, fp32, one per column; NULL: none) for A: m x k and B: n x k in 8 bits, out: device, dtype, row stride ldo >= n elements.
 * fp32 results: products exact, or within 2^-126, and sums in fp32.  (Codes times their power of two are taken as bfloat16 numbers; where they are none, below 2^-133 or from 2^128 on, and it counts, the
 * 32 to 128 rows and columns around such a block take another way, several times as long.)
 * bfloat16 results: the matrix instruction takes codes and bytes as they are, at twice the rate.  It adds eight products at a time and cuts each of them below 2^-13 of
 * the largest's power of two before sums in fp32: a result is off by up to 2^-10 of the sum of its products' magnitudes, by 2^-16 of its size for random operands,
 * and then rounded to bfloat16.  Up to 16 rows of A both kinds may take other kernels with the same bounds.
 * A byte of 255, which no call here writes, makes the results it takes part in undefined.
 * workspace: device, 16-byte aligned, of the size that imunpack_block8_gemm_workspace gives (0: NULL will do).
 * Errors: EINVAL (null pointers, k outside [1, 2^24], m or n outside [0, 2^24], more than 2^23 tiles of the kernel that takes it, layouts as above, pitches above 2^24, unknown
 * types); ESMALL; EHIP. */
int imunpack_block8_gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, size_t *bytes);
int imunpack_block8_gemm(const void *a, int64_t lda, const void *a_scales, int64_t ldsa, int a_format,
                         const void *b, int64_t ldb, const void *b_scales, int64_t ldsb, int b_format,
                         int64_t m, int64_t n, int64_t k, const float *bias, void *out, int64_t ldo, int dtype,
                         void *workspace, size_t workspace_bytes, imunpack_stream_t stream);

/* ---- activation functions that keep their input in 8 bits -------------------------------------------
 * y = f(u), f = GELU: u Phi(u) (the normal distribution's), or SiLU: u / (1 + exp(-u)); gated: u has 2 cols columns and y = f(u[:, :cols]) u[:, cols:].
 * u, y: device, dtype, ld* elements from row to row.  y_codes, y_scales (NULL: not): y in 8 bits (E4M3, blocks along the rows), the operand of the
 * next product; y (may then be NULL) receives those values.  kept, kept_scales (NULL: not, for serving): u in 8 bits (E4M3); gated: its first cols columns,
 * and kept2, kept2_scales the others, pitches alike.
 * imunpack_act8_backward: with v the values that were kept,  gu = g f'(v);  gated:  gu = (g f'(v1) v2, g f(v1)), 2 cols columns.
 * f is within (16 + u^2) 2^-24 (GELU) or 2^-20 (SiLU) of itself, or 2^-120, before it is rounded to dtype or codes.
 * rows == 0 is allowed.  Errors: EINVAL (null pointers, sizes as for imunpack_block8_quantize, pitches, alignments, unknown types or functions); EHIP. */
enum { IMUNPACK_GELU = 0, IMUNPACK_SILU = 1 };
int imunpack_act8(const void *u, int64_t ldu, int64_t rows, int64_t cols, int dtype, int act, int gated, void *y, int64_t ldy,
                  void *y_codes, int64_t ldyc, void *y_scales, int64_t ldys, void *kept, void *kept2, int64_t ldk,
                  void *kept_scales, void *kept2_scales, int64_t ldks, imunpack_stream_t stream);
int imunpack_act8_backward(const void *g, int64_t ldg, int64_t rows, int64_t cols, int dtype, int act, int gated,
                           const void *kept, const void *kept2, int64_t ldk, const void *kept_scales, const void *kept2_scales, int64_t ldks,
                           void *gu, int64_t ldgu, imunpack_stream_t stream);

/* out (device fp32, dense) = the sums of the columns of x (device, dtype, unit stride within a row, ldx elements from row to row), in fp32, in an order that depends on the sizes
 * alone: the gradient of a bias.  rows == 0 gives zeros.  workspace: device, 16-byte aligned, of the size that imunpack_column_sums_workspace gives (0: NULL will do).
 * Errors: EINVAL (null pointers, rows outside [0, 2^31], cols outside [1, 2^24], a pitch < cols, unknown types); ESMALL; EHIP. */
int imunpack_column_sums_workspace(int64_t rows, int64_t cols, int dtype, size_t *bytes);
int imunpack_column_sums(const void *x, int64_t ldx, int64_t rows, int64_t cols, int dtype, float *out, void *workspace, size_t workspace_bytes, imunpack_stream_t stream);

/* ---- log probabilities of given tokens, entropy, top alternatives ------------------------------------
 * For each of `rows` rows l of `vocab` logits (device, dtype, unit stride within a row, ldl elements from row to row):
 *     lse = log sum_v exp l_v,   logp_j = l_[token_j] - lse for `count` tokens (device int64, row r's at tokens + r count),
 *     entropy = lse - sum_v p_v l_v  with  p = exp(l - lse),
 *     top_index, top_logp: the `top` largest logits' places (int64), largest first, of equals the lowest place first, and l - lse there.
 * A logit of -infinity has probability 0 and adds nothing to the entropy; NaN counts as -infinity for the order.
 * A row of nothing but -infinity: lse, logp and top_logp -infinity, entropy 0, places 0, 1, ...  +infinity or NaN in a row: its numbers are NaN.
 * A token that is ignore_index: logp 0, no gradient; another one outside [0, vocab): logp NaN, no gradient.
 * logp (rows x count), lse, entropy, top_logp (rows x top): device fp32, dense; lse and entropy may be NULL, logp with count == 0, the last two with top == 0.
 * stats (device fp32, two for each row, may be NULL): the row's maximum m and log sum_v exp(l_v - m), for the backward pass.
 * imunpack_logprobs_backward: with g_logp (rows x count), g_entropy, g_top (rows x top, for top_index's tokens) the gradients (fp32; each may be NULL):
 *     gl_v = sum_j g_j ([v = token_j] - p_v) - g_entropy p_v (l_v - lse + entropy)
 * over both kinds of tokens (0 for p_v times anything where l_v is -infinity); gl: device, dtype, ldg elements from row to row, 0 for a row of nothing but
 * -infinity.  gl may be l, with the same pitch.  stats and entropy are those of the forward call (entropy may be NULL without g_entropy).
 * workspace: device, 16-byte aligned, of the size that imunpack_logprobs_workspace gives (0: NULL will do).  Statistics in fp32, equal inputs give equal bits.
 * rows == 0 is allowed.  Errors: EINVAL (null pointers, rows outside [0, 2^31 - 1], vocab outside [1, 2^30], count outside [0, 1024], top outside [0, min(64, vocab)], a pitch < vocab,
 * unknown types); ESMALL; EHIP. */
#define IMUNPACK_LOGPROBS_TOP 64
int imunpack_logprobs_workspace(int64_t rows, int64_t vocab, int64_t count, int64_t top, int dtype, size_t *bytes);
int imunpack_logprobs(const void *logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int64_t *tokens, int64_t count, int64_t ignore_index, int64_t top,
                      float *logp, float *lse, float *stats, float *entropy, float *top_logp, int64_t *top_index, void *workspace, size_t workspace_bytes,
                      imunpack_stream_t stream);
int imunpack_logprobs_backward(const void *logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int64_t *tokens, int64_t count, int64_t ignore_index, int64_t top,
                               const int64_t *top_index, const float *stats, const float *entropy, const float *g_logp, const float *g_entropy, const float *g_top,
                               void *gl, int64_t ldg, imunpack_stream_t stream);

/* ---- diagnostics ------------------------------------------------------------------------------- */
/* Per-kernel device time of the last call of each stage on this plan is not kept; callers time
 * with events.  These two describe errors. */
const char *imunpack_strerror(int code);
int imunpack_last_hip_error(void);

/* Which GEMM path the plan's last imunpack_unpack selected: 1 = single fused launch is exact,
 * 0 = the shifted group sum may exceed int32 and the un-fused path is required.  Waits for that
 * unpack to finish on the device. */
int imunpack_plan_fusable(imunpack_plan_t *plan);

/* The two numbers that decision rests on, as the plan's last imunpack_unpack measured them:
 * bound[0] = max over the rows R of A_ue of sum_c s^e(c) |A_ue[R, c]|, bound[1] the same for B_eu,
 * e(c) the exponent of column c's diagonal entry of S_uu (Alg. 3).  Every entry of the other operand
 * is at most s - 1 in magnitude, so |sum_c s^e(c) a_c b_c| <= (s - 1) * min(bound[0], bound[1]), and
 * the fused launch is exact when that stays below 2^31.  Values of 2^44 and more are reported
 * saturated (at least 2^44).  bound: host, two elements.  Waits like imunpack_plan_fusable. */
int imunpack_plan_bounds(imunpack_plan_t *plan, uint64_t *bound);

/* Measured matrix-core peak (benchmark reporting only, not part of the method): launches
 * `workgroups` workgroups of 4 waves that each issue 8 * iters register-resident
 * v_mfma_i32_32x32x32_i8 with no memory traffic, and writes the number of integer operations
 * (2 per multiply-add) the launch performs to *ops.  The caller times the stream. */
int imunpack_diag_mfma_peak(int workgroups, int iters, int64_t *ops, imunpack_stream_t stream);

/* Measured HBM rate (benchmark reporting only): copies `bytes` (a multiple of 1 MiB, at most 65535 MiB)
 * from src to dst (device, 16-byte aligned, not overlapping) in the access pattern of the quantize pass,
 * with non-temporal loads and stores.  The caller times the stream; the traffic is 2 * bytes. */
int imunpack_diag_copy(const void *src, void *dst, int64_t bytes, imunpack_stream_t stream);

/* How the plan's last fused imunpack_gemm was launched (tests and benchmark reporting only): 0 = in tiles of
 * 64 x 64 unpacked rows, 1 = of 256 x 256 or half tiles, 2 to 4 = of 256 x 256, those of the last round cut into that many parts
 * along the contraction.  Errors: EINVAL (null plan).
 * imunpack_diag_gemm_halves: 1 if it was in tiles of 128 x 256, two workgroups to a CU, else 0. */
int imunpack_diag_gemm_parts(const imunpack_plan_t *plan);
int imunpack_diag_gemm_halves(const imunpack_plan_t *plan);

/* How many of the d' columns the fused imunpack_gemm of this plan does not multiply as columns (tests and benchmark reporting
 * only): columns that UnpackBoth appended to B for a few heavy hitters each, whose digits it takes one by one
 * (B_eu holds them like any other).  Errors: EINVAL (no valid plan). */
int imunpack_diag_list_columns(const imunpack_plan_t *plan);

/* Which kernel imunpack_block8_gemm takes for these sizes (tests and benchmark reporting only; nothing is launched): *tile = 1, 2 or 4 for tiles of 64, 128 or 256 squared, 0 for the kernel of up to 16
 * rows; *parts: into how many parts the contraction is cut.  Errors: EINVAL as for imunpack_block8_gemm_workspace. */
int imunpack_diag_block8_cut(int64_t m, int64_t n, int64_t k, int dtype, int *tile, int *parts);

/* Shader clock under the GEMM's own load (benchmark reporting only).  While `ticks` (device, two
 * elements, owned by the caller) is set, every fused imunpack_gemm launch of this process has its
 * first workgroup write ticks[0] = shader clock cycles and ticks[1] = ticks of the constant 100 MHz
 * clock that its loop over K took; ticks[0] / ticks[1] * 100 is the clock in MHz the matrix cores ran
 * at, which the power limit holds below the 2400 MHz the published peak assumes.  NULL switches the
 * probe off (the default).  Not thread safe; set it while no GEMM is in flight. */
int imunpack_diag_clock_probe(uint64_t *ticks);

#ifdef __cplusplus
}
#endif
#endif /* IMUNPACK_H */
