/*
 * mpq.h - C ABI of the MI355X (gfx950) multipoint quantization library.
 *
 * Multipoint quantization (Liu, Ye, Zhou, Liu, "Post-training Quantization
 * with Multiple Points: Mixed Precision without Mixed Precision") replaces
 * each output channel's weight vector w (length d) of a linear or conv layer
 * by a sum  sum_{i<n} a_i * q_i  of n low-bit integer vectors q_i with fp32
 * scales a_i (Sec. 3.2, Eq. (4)).
 *
 * Conventions shared by every entry point
 *  - Array arguments are DEVICE pointers (hipMalloc memory or ROCm torch
 *    tensors) unless the comment says HOST.  Arrays are dense, row-major.
 *  - The caller owns every buffer.  The library keeps no pointer after the
 *    stream work of a call has completed.  Outputs must not alias inputs.
 *  - Calls enqueue work on `stream` (a hipStream_t; NULL = default stream)
 *    and return without waiting for it.  Argument checks are synchronous and
 *    happen before anything is enqueued; on an error nothing is enqueued.
 *  - Results are deterministic: identical inputs give bitwise identical
 *    outputs.  Calls on distinct streams may run concurrently.
 *  - Every call returns an MPQ_* status; mpq_last_error() describes the
 *    last failure of the calling thread.  No C++ exception crosses the ABI.
 *  - Inputs must be finite (but for the microscaled calls, mpq_mx_*).
 *  - A layer with so many channels or weights that its launch would have 2^32
 *    threads is refused with MPQ_ERR_HIP (fits: 64 threads or more a channel;
 *    reconstruction: 2^36 weights; integer scales: 2^32 of them; of the
 *    microscaled calls only a product, of one matrix or by experts, of 2^37
 *    outputs and more).
 *
 * Codes and scales (readings of the paper, shared with the test oracle)
 *  - bits b in [2, 8]; codes are the integers [-M, M] with M = 2^(b-1) - 1,
 *    i.e. the symmetric set of Eq. (1) with its 2M+1 points, B = 0 and the
 *    step K * eps_b folded into the scale.  -2^(b-1) is never produced.
 *  - Rounding to the nearest code (Eq. (2)) breaks exact half-way ties to
 *    the even integer.
 */
#ifndef MPQ_H
#define MPQ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MPQ_OK 0
#define MPQ_ERR_INVALID_ARG (-1) /* a null pointer, a size or value out of range */
#define MPQ_ERR_SHAPE (-2)       /* d (with n_grid) too large for one workgroup's LDS */
#define MPQ_ERR_HIP (-3)         /* a HIP runtime call failed; see mpq_last_error() */
#define MPQ_ERR_NOMEM (-4)       /* device scratch allocation failed (or exceeded the
                                    MPQ_WORKSPACE_LIMIT environment variable: a cap in
                                    bytes on each scratch allocation, checked before
                                    any HIP call; unset means no cap) */

#define MPQ_MAX_BITS 8
#define MPQ_MAX_POINTS 64
#define MPQ_MAX_GRID 4096
#define MPQ_MAX_ERR_DIM 16777216   /* c_out and n of mpq_output_error */
#define MPQ_MAX_ERR_D 4194272      /* d of mpq_output_error (128 rows of the residual below 2 GiB) */
#define MPQ_MAX_INT_DIM 131072     /* d of mpq_integer_forward */

/*
 * mpq_fit_layer - greedy multipoint fit of every channel of a layer
 * (Sec. 3.2, Eq. (6)-(10), Algorithm 1, with the stopping rule of
 * Algorithm 2 / Eq. (12)).
 *
 * For each channel k (row W[k], length d), independently:
 *   r = w; n = 0
 *   loop:
 *     stop if n == max_points, or ||r||^2 == 0,
 *       or (n >= 1 and ||r||^2 <= tol * ||w||^2)
 *     candidate scales a_g = fl32(fl32(max_j |r_j|) * c_g / M), g = 1..G
 *     (products and quotient in fp64; Algorithm 1 sets the search grid up
 *     afresh from the residual at every step)
 *     a* = argmin_g || r - a_g * clip(round(r / a_g), -M, M) ||^2
 *          (Eq. (9); exactly equal errors: the smallest g; a candidate that
 *          rounds to 0 in fp32 is skipped, and if all do the fit stops)
 *     q* = clip(round(r / a*), -M, M)      (Eq. (10), fp64 quotient)
 *     r  = r - a* q*  (fp64)               (Eq. (7)); n += 1
 *   The stopping rule reads Algorithm 2's output-error threshold for an
 *   isotropic calibration distribution (E[x x^T] = I gives
 *   E (r . x)^2 = ||r||^2), relative to ||w||^2.  A nonzero channel always
 *   gets at least one point; an all-zero channel gets none.
 *
 * Arguments
 *   W          [c_out][d] fp32 weights (input).
 *   c_out, d   c_out >= 0 (0: nothing to do), d >= 1.
 *   bits       2..8.
 *   max_points 1..MPQ_MAX_POINTS: the per-channel cap on n.
 *   grid_host  HOST array of n_grid multipliers c_g, strictly ascending,
 *              each in (0, 1]; NULL selects c_g = g / n_grid (g = 1..n_grid,
 *              rounded to fp32).  Read before the call returns.
 *   n_grid     1..MPQ_MAX_GRID: number of candidate scales G.
 *   tol        relative stopping tolerance, finite and >= 0.
 *   codes      [c_out][max_points][d] int8 (output).  Rows at or after a
 *              channel's count are zero.
 *   scales     [c_out][max_points] fp32 (output), zero after the count.
 *   counts     [c_out] int32 (output): the number of points n of each channel.
 *   err_opt    NULL or [c_out][max_points] fp32 (output): ||r||^2 after
 *              each point (fp64 sum rounded to fp32), zero after the count.
 *   stream     hipStream_t or NULL.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_SHAPE (see mpq_fit_max_dim),
 *         MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int mpq_fit_layer(const float *W, int64_t c_out, int64_t d, int bits, int max_points,
                  const float *grid_host, int n_grid, float tol, int8_t *codes,
                  float *scales, int32_t *counts, float *err_opt, void *stream);

/*
 * How mpq_fit_layer evaluates Eq. (9): for d <= 32768 it counts, per element
 * and code level k, the candidates whose boundary (k + 1/2) a_g lies below
 * |r_j|, accumulates exact integer histograms, and gets every candidate's
 * error from ||r||^2 - 2 a A(g) + a^2 B(g) in fp64 (A, B: suffix sums), in
 * O(d M + G) per step; candidates whose error bound overlaps the minimum are
 * re-evaluated directly in fp64.  Longer channels use the dense search of
 * mpq_fit_layer_dense.
 *
 * mpq_fit_layer_dense - mpq_fit_layer with the dense candidate search:
 * every (element, candidate) pair is evaluated in fp32 on the residual
 * staged in LDS, with fp64 sums of 16-element blocks, in O(d G) per step.
 * Same arguments, outputs and errors as mpq_fit_layer; the two agree except
 * where the top-2 candidate errors lie within fp32 rounding of each other.
 */
int mpq_fit_layer_dense(const float *W, int64_t c_out, int64_t d, int bits, int max_points,
                        const float *grid_host, int n_grid, float tol, int8_t *codes,
                        float *scales, int32_t *counts, float *err_opt, void *stream);

/*
 * mpq_fit_max_dim - largest channel length d that mpq_fit_layer accepts for
 * n_grid candidates on the current device: the larger of 32768 (the
 * histogram search keeps a channel's residual in the registers of one
 * workgroup) and the dense search's limit (the residual staged in the LDS of
 * one workgroup).  Returns a negative MPQ_* status on failure.
 */
int64_t mpq_fit_max_dim(int n_grid);

/*
 * mpq_output_error - output error of the quantized layer on a calibration
 * batch (Sec. 3.3, Eq. (12)):
 *   err[k] = (1/n) sum_t ( (w_k - w~_k) . x_t )^2,
 *   ref[k] = (1/n) sum_t ( w_k . x_t )^2          (if ref_opt != NULL)
 * where w~_k = sum_{i<counts[k]} scales[k][i] * codes[k][i] and x_t is
 * column t of X.  The difference w_k - w~_k is formed in fp64 and rounded
 * to fp32; each fp32 product is summed on the 16-bit matrix cores, with fp32
 * accumulation, from four products of fp16 pieces of the scaled operands
 * (d >= 128, c_out >= 256, or 384 where d n > 3 2^20, and rows of X whose root
 * mean squares are at least 2^-10 of the power of two at or below X's largest
 * magnitude: three pieces of w - w~, exact to 2^-39 of its largest, and two of
 * X, within 2^-23), or else from six products of exact three-piece bf16 splits;
 * the sum over the batch is fp64.
 *
 * Arguments
 *   W, codes, scales, counts   as produced for mpq_fit_layer (inputs);
 *                              counts[k] in [0, max_points].
 *   c_out, d, max_points       as for mpq_fit_layer.
 *   X          [d][n] fp32 calibration inputs (input), n >= 1.
 *   c_out and n are at most MPQ_MAX_ERR_DIM, d at most MPQ_MAX_ERR_D.
 *   err        [c_out] fp32 (output).
 *   ref_opt    NULL or [c_out] fp32 (output).
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int mpq_output_error(const float *W, const int8_t *codes, const float *scales,
                     const int32_t *counts, int64_t c_out, int64_t d, int max_points,
                     const float *X, int64_t n, float *err, float *ref_opt, void *stream);

/*
 * mpq_output_error_noalloc - mpq_output_error for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, kernels and results
 * (bitwise those of mpq_output_error on the same inputs); the call
 * allocates nothing.  Its workspace (the residual rows in tiles, row
 * partials and per-K-range outputs; a little more behind it holds the rows'
 * and X's ranges) is a fixed array of MPQ_NOALLOC_BYTES
 * per device, held by the library from the moment its code loads on that
 * device until the process ends.  A call whose workspace would exceed it
 * (about 4 ceil(c_out / 128) 128 ceil(d / 32) 32 bytes for the residual,
 * doubled with ref_opt, plus 8 c_out ceil(n / 128) and, for long d,
 * 4 c_out n per K range) returns MPQ_ERR_SHAPE before anything is enqueued.
 * Every call on one device shares that device's array and leaves its
 * contents behind: calls that overlap on one device (on different streams,
 * or from different threads before the first finishes) race and must be
 * ordered by the caller.  Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_SHAPE,
 * MPQ_ERR_HIP.
 */
#define MPQ_NOALLOC_BYTES (64 << 20)
int mpq_output_error_noalloc(const float *W, const int8_t *codes, const float *scales,
                             const int32_t *counts, int64_t c_out, int64_t d, int max_points,
                             const float *X, int64_t n, float *err, float *ref_opt, void *stream);

/*
 * mpq_reconstruct - the quantized weights of Eq. (4):
 *   W_hat[k][j] = fl32( sum_{i<counts[k]} scales[k][i] * codes[k][i][j] ),
 * summed in fp64 in point order.
 *   codes [c_out][max_points][d] int8, scales [c_out][max_points] fp32,
 *   counts [c_out] int32 in [0, max_points] (inputs); W_hat [c_out][d] fp32
 *   (output).
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_reconstruct(const int8_t *codes, const float *scales, const int32_t *counts,
                    int64_t c_out, int64_t d, int max_points, float *W_hat, void *stream);

/*
 * Batched calls: one call covers the layers of a network.  Each layer is
 * described by an mpq_layer (a HOST array of them is passed; the pointers in
 * it are DEVICE pointers); every call reads only the fields it names.  The
 * result is the same as calling the single-layer entry point on each layer
 * in order, on the same stream.  Layers whose channel lengths select the
 * same kernel share one launch, so a whole network costs a handful of
 * launches.  Arguments are checked for every layer before anything is
 * enqueued.
 */
typedef struct mpq_layer {
    const float *W;       /* [c_out][d] fp32 weights                               */
    int64_t c_out, d;
    int8_t *codes;        /* [c_out][max_points][d]                                */
    float *scales;        /* [c_out][max_points]                                   */
    int32_t *counts;      /* [c_out]                                               */
    float *fit_err;       /* mpq_fit_layers: NULL or [c_out][max_points] (err_opt) */
    const float *X;       /* mpq_output_error_layers: [d][n] calibration inputs    */
    int64_t n;            /* mpq_output_error_layers: columns of X                 */
    float *out_err;       /* mpq_output_error_layers: [c_out]                      */
    float *out_ref;       /* mpq_output_error_layers: NULL or [c_out]              */
    float *W_hat;         /* mpq_reconstruct_layers: [c_out][d]                    */
    float *fit_xerr;      /* mpq_fit_layers_calib: [c_out][max_points]             */
    float *offsets;       /* NULL, or [c_out]: asymmetric codes (mpq_fit_options.asym):
                             written by the fit, read by mpq_output_error_layers and
                             mpq_reconstruct_layers (w~ = offset + sum a q)      */
} mpq_layer;

/* mpq_fit_layer on every layer (reads W, c_out, d, codes, scales, counts,
 * fit_err).  All layers share bits, max_points, the grid and tol. */
int mpq_fit_layers(const mpq_layer *layers, int n_layers, int bits, int max_points,
                   const float *grid_host, int n_grid, float tol, void *stream);

/* mpq_output_error on every layer (reads W, c_out, d, codes, scales, counts,
 * X, n, out_err, out_ref). */
int mpq_output_error_layers(const mpq_layer *layers, int n_layers, int max_points, void *stream);

/* mpq_reconstruct on every layer (reads c_out, d, codes, scales, counts,
 * W_hat). */
int mpq_reconstruct_layers(const mpq_layer *layers, int n_layers, int max_points, void *stream);

/*
 * mpq_quantize_layers - the whole path for a network in one call: the fit of
 * every layer (mpq_fit_layers), then, for each layer with out_err != NULL,
 * its output error (Eq. (12), as mpq_output_error_layers; X, n, out_err and
 * out_ref are read) and, for each layer with W_hat != NULL, its quantized
 * weights (Eq. (4), as mpq_reconstruct_layers).  The outputs are bitwise
 * those of the three batched calls made in that order on the same stream.
 * The fit launches run side by side (as in mpq_fit_layers), with the upload
 * of the output error's descriptor tables beside them; a fit launch of at
 * least 2e6 weights other than the longest one is followed on its stream by
 * its layers' reconstruction; every fit also writes its layers' rows of the
 * output error's residual D (bitwise what the output error would form from
 * the stored points).  Then the
 * output errors of all layers run as one batch while the remaining layers
 * are reconstructed beside them.  The streams are the caller's and
 * library-owned ones joined back to it.
 * The fit is symmetric: the layers' offsets fields are ignored.
 * Arguments as for mpq_fit_layers; every layer is checked before anything is
 * enqueued.
 */
int mpq_quantize_layers(const mpq_layer *layers, int n_layers, int bits, int max_points,
                        const float *grid_host, int n_grid, float tol, void *stream);

/*
 * mpq_fit_layer_calib - the greedy fit of mpq_fit_layer with Algorithm 2's
 * stopping rule on a calibration batch (Sec. 3.3, Eq. (12)) instead of the
 * isotropic one.  For each channel k, after each point n >= 1:
 *   e_n = (1/n_cols) sum_t ( (w_k - w~_k,n) . x_t )^2     (x_t: column t of X)
 * is computed as mpq_output_error does (fp64 difference rounded to fp32,
 * fp32 products from 16-bit pieces, fp64 sum over the batch), and the channel stops once
 *   e_n <= thr,  thr = eps * (1/n_cols) sum_t (w_k . x_t)^2   (relative != 0)
 *                thr = eps                                  (relative == 0),
 * or at max_points, or when its residual is zero.  The points themselves
 * are Algorithm 1's, which does not see X: a channel's points are the first
 * ones mpq_fit_layer would choose with tol = 0.  A nonzero channel gets at
 * least one point.
 *
 * The fit runs one step at a time: step s takes point s + 1 of every channel
 * still going, then scores those channels' output error on the batch (only
 * theirs), so the work follows the points each channel actually takes.
 *
 * Arguments as for mpq_fit_layer (tol replaced by eps and relative), plus
 *   X          [d][n] fp32 calibration inputs (input), 1 <= n <= MPQ_MAX_ERR_DIM.
 *   eps        threshold, finite and >= 0 (relative or absolute).
 *   relative   nonzero: thr relative to the output error of w itself.
 *   xerr       [c_out][max_points] fp32 (output): e_n after each point n,
 *              zero after the count.
 *   c_out <= MPQ_MAX_ERR_DIM; d within the histogram search (d <= 32768,
 *   else MPQ_ERR_SHAPE).
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_SHAPE, MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int mpq_fit_layer_calib(const float *W, int64_t c_out, int64_t d, int bits, int max_points,
                        const float *grid_host, int n_grid, const float *X, int64_t n, float eps,
                        int relative, int8_t *codes, float *scales, int32_t *counts, float *err_opt,
                        float *xerr, void *stream);

/* mpq_fit_layer_calib on every layer (reads W, c_out, d, codes, scales,
 * counts, fit_err, X, n, fit_xerr).  Each step's fits run side by side and
 * its output errors run as one batch over all layers. */
int mpq_fit_layers_calib(const mpq_layer *layers, int n_layers, int bits, int max_points,
                         const float *grid_host, int n_grid, float eps, int relative, void *stream);

/*
 * mpq_fit_layers_ex - mpq_fit_layers with options (opt == NULL: exactly
 * mpq_fit_layers).
 *   refit     nonzero: once a point's codes q are fixed (Eq. (10) at the
 *             scale Eq. (9) chose), its scale becomes the least-squares
 *             scale for them, fl32(<r, q> / <q, q>) (fp64 sums), and the
 *             residual of Eq. (7) uses that scale.  A variant of Algorithm 1
 *             (which keeps the searched scale).
 *   calib     nonzero: the stopping rule of mpq_fit_layers_calib with eps and
 *             relative (reads X, n and fit_xerr of every layer; tol unused).
 *   clip_grid 0, or the number Gc of clipping factors of Eq. (13) (the paper
 *             uses 20, K in [0.05 : 0.05 : 1] * max|w|): point 1 of each
 *             channel is the naive quantization, at the code step
 *             fl32(fl32(max|w|) * fl32(j / Gc) / M), j = 1..Gc, whose output
 *             error on the layer's X is smallest (ties: the smallest j); the
 *             points after it follow Algorithm 1 with the stopping rule.
 *             Reads X and n of every layer; c_out * Gc <= MPQ_MAX_ERR_DIM.
 *             Cannot be combined with refit.
 *   asym      nonzero: asymmetric per-channel codes (Eq. (1) with B != 0): the
 *             offset beta = fl32((max_j w_j + min_j w_j) / 2) is written to the
 *             layer's offsets [c_out] (must not be NULL), the points fit
 *             w - beta, and w~ = beta + sum a q.  The stopping rules still
 *             compare with w's own error (||w||^2, or w's output energy).
 *             With either stopping rule and refit; not with clip_grid or
 *             paper_eta.  The batched output error and reconstruction add the
 *             offsets of layers whose offsets are not NULL.
 *   paper_eta 0, or eta > 0: the candidate scales of each step are the
 *             paper's own grid (Eq. (11), Def. 1): a = g * gamma,
 *             g = 1 .. floor(2 M ||r|| / gamma), gamma = min(Delta_r / M, eta),
 *             Delta_r half the smallest positive difference of the |r_j|
 *             (none: gamma = eta); the paper uses eta = 2^-10.  The grid is
 *             searched exactly without enumerating it; the chosen scale is
 *             stored as fl32(g * gamma), and the point's codes and residual
 *             use that value.  grid_host and n_grid are ignored.  Only with
 *             the isotropic stopping rule (not with refit, calib,
 *             clip_grid, asym or gate); d <= 32768 (else MPQ_ERR_SHAPE;
 *             channels past 8192 keep their sorted magnitudes in a stream-
 *             ordered scratch of about 8 (2 d) bytes for each of up to 1024
 *             channels in flight).
 *   gate      nonzero: Algorithm 2's naive first point (Sec. 3.3).  Each
 *             channel is first quantized naively, a_N = fl32(fl32(max|w|) / M)
 *             (the candidate c = 1), q = [w / a_N]_Q; if that point already
 *             meets the threshold of the stopping rule (isotropic:
 *             ||w - a_N q||^2 <= tol ||w||^2; calib: its output error
 *             e <= thr), it is the channel's only point; otherwise it is
 *             discarded and Algorithm 1 runs from w (max_points bounds
 *             Algorithm 1 only).  Without it point 1 is always Algorithm 1's.
 *             Not with clip_grid or paper_eta; with calib not with asym.
 * refit, calib and clip_grid need the histogram search for every layer
 * (d <= 32768; else MPQ_ERR_SHAPE).  Errors as for mpq_fit_layers /
 * mpq_fit_layers_calib.
 */
typedef struct mpq_fit_options {
    int refit;
    int calib;
    float eps;
    int relative;
    int clip_grid;
    float paper_eta;
    int asym;
    int gate;
} mpq_fit_options;
int mpq_fit_layers_ex(const mpq_layer *layers, int n_layers, int bits, int max_points,
                      const float *grid_host, int n_grid, float tol, const mpq_fit_options *opt,
                      void *stream);

/*
 * Deployment arithmetic (Sec. 3.4).
 *
 * mpq_integer_scales - the integer scales of Eq. (14):
 *   A[k][i] = nearest integer to 2^p * scales[k][i] (ties to even; 2^p a is
 *   exact in fp64) for i < counts[k], 0 after the count.  A value beyond
 *   the 32-bit range is clamped to +-(2^31 - 1); if n_clamped_opt is not
 *   NULL, the number of clamped values is added to it (a DEVICE uint64 the
 *   caller zeroes).
 *   scales [c_out][max_points] fp32, counts [c_out] int32 in [0, max_points]
 *   (inputs); A [c_out][max_points] int32 (output); 0 <= p <= 62.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_integer_scales(const float *scales, const int32_t *counts, int64_t c_out, int max_points, int p,
                       int32_t *A, unsigned long long *n_clamped_opt, void *stream);

/*
 * mpq_integer_forward - a multipoint layer's integer dot products on a batch
 * of integer activations (Eq. (15), Steps 1-3).  For channel k and column t:
 *   Step 1  z_i = q_{k,i} . x_t   for i < counts[k], in 32-bit accumulators
 *           (int8 MFMA; exact for codes in [-127, 127], as the fit writes
 *           them, any int8 activations and d <= MPQ_MAX_INT_DIM)
 *   Step 2  s = sum_{i < counts[k]} A[k][i] * z_i, in 64 bits
 *   Step 3  Y[k][t] = s >> p, an arithmetic right shift (floor(s / 2^p))
 * Y is exact while |s| < 2^63 (e.g. |A| < 2^31 and counts[k] * d * 128 * 128
 * < 2^32).  Codes past a channel's count, and their A, are not read.
 *
 * Arguments
 *   codes    [c_out][max_points][d] int8 (the fit's codes), A [c_out][max_points]
 *            int32 (mpq_integer_scales), counts [c_out] int32 in [0, max_points].
 *   X        [n][d] int8: column t of the batch is the contiguous row X[t]
 *            (signed activation integers; the batch is stored transposed
 *            with respect to mpq_output_error's fp32 X).
 *   Y        [c_out][n] int64 (output).
 *   c_out, n >= 0; 1 <= d <= MPQ_MAX_INT_DIM; codes and X each below 2^31
 *   bytes; 0 <= p <= 62.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_integer_forward(const int8_t *codes, const int32_t *A, const int32_t *counts, int64_t c_out,
                        int64_t d, int max_points, const int8_t *X, int64_t n, int p, int64_t *Y,
                        void *stream);

/* mpq_integer_forward on a list of layers (HOST array; DEVICE pointers),
 * with one launch per 32 layers.  All layers share max_points and p. */
typedef struct mpq_int_layer {
    const int8_t *codes;    /* [c_out][max_points][d] */
    const int32_t *A;       /* [c_out][max_points]    */
    const int32_t *counts;  /* [c_out]                */
    int64_t c_out, d;
    const int8_t *X;        /* [n][d]                 */
    int64_t n;
    int64_t *Y;             /* [c_out][n]             */
} mpq_int_layer;
int mpq_integer_forward_layers(const mpq_int_layer *layers, int n_layers, int max_points, int p,
                               void *stream);

/*
 * Microscaled formats: what a quantized language model is served from.
 *
 * A block of MPQ_MX_BLOCK = 32 consecutive elements of a row shares the power
 * of two 2^(s - 127), s one byte; the element with code c stands for
 * value(c) * 2^(s - 127).
 *   MPQ_MX_FP4  E2M1: 1 sign bit, 2 exponent bits (bias 1), 1 mantissa bit:
 *               0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; two codes a
 *               byte, the even element in the low half.
 *   MPQ_MX_FP8  E4M3: 1 sign bit, 4 exponent bits (bias 7), 3 mantissa bits,
 *               largest 448 (the codes 0x7f and 0xff are no numbers and are
 *               not produced).
 * Quantization of a block with largest magnitude a: s = floor(log2 a) + 127 -
 * (2 for fp4, 8 for fp8), at least 0; each x / 2^(s - 127) is rounded to the
 * nearest element, ties to the even mantissa, magnitudes past the largest
 * element to it.  a = 0: s = 0.  A block that holds an infinity or a NaN has
 * s = 255 and codes 0, and stands for NaN throughout; other blocks are not
 * affected (these calls alone take inputs that are not finite).
 *
 * A dtype argument is MPQ_F32, MPQ_F16 or MPQ_BF16.  Strides (ld, *_stride)
 * are in elements; the innermost dimension is contiguous; matrices of a dtype
 * need only be aligned to their element.  Code arrays are 16-byte aligned,
 * fp4 rows' scale arrays and caches' scale arrays 4-byte aligned.  A value
 * past f16's range is rounded to f16 as the hardware does (to infinity).
 *
 * Rows of an output do not overlap: where it has several rows, their stride is
 * at least their length.
 *
 * fp4 rows: a row of d elements is held as D = ceil(d / 128) 128 elements,
 * zeros past d: codes [rows][D / 2], scales [rows][D / 32].
 */
#define MPQ_F32 0
#define MPQ_F16 1
#define MPQ_BF16 2
#define MPQ_MX_FP4 0
#define MPQ_MX_FP8 1
#define MPQ_MX_BLOCK 32
#define MPQ_MX_ROW 128
#define MPQ_MX_MAX_D 4194304        /* d of fp4 rows */
#define MPQ_MX_MAX_N 1048576        /* tokens of a product */
#define MPQ_MX_MAX_HEAD_DIM 256
#define MPQ_MX_MAX_PAGE 65536
#define MPQ_MX_MAX_TOKENS 536870912 /* tokens of one sequence: columns of the page table times page_size */
#define MPQ_MX_MAX_EXPERTS 1024
#define MPQ_MX_MAX_CHOICES 64       /* experts of one token */
#define MPQ_MX_MAX_ROWS 67108864    /* rows of a product by experts, of all tokens' choices together */

/*
 * mpq_mx_quantize - rows to fp4 blocks.
 *   X      [rows][ld] of dtype, the first d of each row (input); ld >= d.
 *   codes  [rows][D / 2], scales [rows][D / 32] (outputs).
 *   rows >= 0, 1 <= d <= MPQ_MX_MAX_D, rows * D at most 2^42.
 * mpq_mx_dequantize - the values that they stand for, rounded to dtype (exact
 * in fp32 and bf16).  Y [rows][ld] of dtype (output).
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_mx_quantize(const void *X, int dtype, int64_t rows, int64_t d, int64_t ld, uint8_t *codes,
                    uint8_t *scales, void *stream);
int mpq_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, void *Y, int dtype,
                      int64_t ld, void *stream);

/*
 * mpq_mx_product - Y = X W^T + b of two matrices of fp4 rows, on the 4-bit
 * matrix cores: products of elements and block scales are exact, sums fp32, Y
 * rounded once.
 *   x_codes, x_scales  [n] rows of d (inputs): the tokens.
 *   w_codes, w_scales  [c_out] rows of d (inputs): the weights.
 *   bias_opt           NULL or [c_out] fp32 (input), added in fp32.
 *   Y                  [n][ld] of dtype (output), ld >= c_out.
 *   0 <= n <= MPQ_MX_MAX_N, c_out >= 0.
 *
 * mpq_mx_linear - Y = Q(X) W^T + b: the tokens X [n][x_ld] of x_dtype are
 * quantized as mpq_mx_quantize does (bitwise the result of the two calls).
 *   workspace_opt      NULL, or a DEVICE buffer (16-byte aligned) of at least
 *                      mpq_mx_linear_workspace(n, c_out, d) bytes, which the call
 *                      overwrites; it may be reused by the next call on the
 *                      same stream.  NULL: stream-ordered scratch of the
 *                      library (MPQ_WORKSPACE_LIMIT applies).  With a
 *                      workspace the call allocates nothing and can be captured.
 * mpq_mx_linear_workspace returns the size (>= 0), or a negative status.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int mpq_mx_product(const uint8_t *x_codes, const uint8_t *x_scales, int64_t n, const uint8_t *w_codes,
                   const uint8_t *w_scales, int64_t c_out, int64_t d, const float *bias_opt, void *Y, int dtype,
                   int64_t ld, void *stream);
int64_t mpq_mx_linear_workspace(int64_t n, int64_t c_out, int64_t d);
int mpq_mx_linear(const void *X, int x_dtype, int64_t n, int64_t x_ld, const uint8_t *w_codes,
                  const uint8_t *w_scales, int64_t c_out, int64_t d, const float *bias_opt, void *Y, int dtype,
                  int64_t ld, void *workspace_opt, int64_t workspace_bytes, void *stream);

/*
 * A paged cache of keys and values, quantized in blocks along each head's
 * dimensions.  With nb = ceil(head_dim / 32) and R the bytes of 32 nb codes
 * (16 nb for fp4, 32 nb for fp8; dimensions past head_dim are zeros):
 *   k_codes, v_codes    [n_pages][kv_heads][page_size][R]
 *   k_scales, v_scales  [n_pages][kv_heads][nb][page_size]
 * The caller owns the arrays (DEVICE pointers in a HOST struct, read before
 * the call returns) and the pages.  Slot p * page_size + i is place i of
 * page p.
 *   n_pages >= 1; page_size a multiple of 16, at most MPQ_MX_MAX_PAGE; 1 <= head_dim <=
 *   MPQ_MX_MAX_HEAD_DIM; kv_heads >= 1; n_pages * page_size < 2^40.
 */
typedef struct mpq_mx_cache {
    uint8_t *k_codes, *v_codes;
    uint8_t *k_scales, *v_scales;
    int64_t n_pages;
    int32_t page_size, kv_heads, head_dim;
    int32_t format; /* MPQ_MX_FP4 or MPQ_MX_FP8 */
} mpq_mx_cache;

/*
 * mpq_mx_cache_write - quantizes the keys and values of n tokens into their
 * slots.  mpq_mx_cache_read - the values held at n slots, rounded to dtype.
 *   K, V    [n][kv_heads][head_dim] of dtype, with the strides of tokens and
 *           heads (inputs of the write, outputs of the read).
 *   slots   [n] int64 (DEVICE, input).  The write skips a token whose slot
 *           is outside [0, n_pages * page_size); the read gives zeros there.
 *           The slots of one write are distinct.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_mx_cache_write(const mpq_mx_cache *cache, const void *K, int64_t k_stride, int64_t k_head_stride,
                       const void *V, int64_t v_stride, int64_t v_head_stride, int dtype, int64_t n,
                       const int64_t *slots, void *stream);
int mpq_mx_cache_read(const mpq_mx_cache *cache, void *K, int64_t k_stride, int64_t k_head_stride, void *V,
                      int64_t v_stride, int64_t v_head_stride, int dtype, int64_t n, const int64_t *slots,
                      void *stream);

/*
 * mpq_mx_attend - attention of one new token of each sequence over its
 * cached tokens:
 *   O[b][h] = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale Q[b][h] . k_j),
 * j over the tokens [max(0, len - window), len) of sequence b (window = 0:
 * all), k_j and v_j the held values of cache head h / (q_heads / kv_heads).
 * Token j is place j % page_size of page page_table[b][j / page_size].
 *   Q, O        [batch][q_heads][head_dim] of dtype, with the strides of
 *               sequences and heads (input, output).
 *   q_heads     a multiple of kv_heads.
 *   page_table  [batch][table_ld] int32 (DEVICE), its first max_pages columns
 *               used; entries past a sequence's last page are not read as
 *               pages.  A token whose entry is outside [0, n_pages) takes no
 *               part.
 *   lengths     [batch] int32 (DEVICE): len, the new token included when its key
 *               was written; taken as at most max_pages * page_size (which is at
 *               most MPQ_MX_MAX_TOKENS), a negative one as 0.
 *   scale       finite.
 *   lse_opt     NULL or [batch][q_heads] fp32 (output): log sum_j p_j.
 * A sequence without tokens has O = 0 and lse = -infinity.  What the cache
 * holds outside the tokens named, NaN included, has no influence.  Sums and
 * softmax statistics are fp32; p_j enters the matrix cores as two or three
 * bf16 pieces (relative error 2^-16 for 16-bit dtypes, 2^-24 for fp32).  Held
 * values enter them as bf16: exactly, but for fp8 blocks with a scale byte
 * below 3 (nothing in them reaches 2^-116), whose values are rounded to
 * multiples of 2^-133.
 *   workspace_opt, workspace_bytes  as for mpq_mx_linear, of at least
 *               mpq_mx_attend_workspace(cache, batch, q_heads, max_pages)
 *               bytes (enough for any window).
 * Where a sequence is cut into pieces follows from batch, max_pages, window
 * and the heads, and so do the last bits of its results; they do not depend on
 * the other sequences' contents.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int64_t mpq_mx_attend_workspace(const mpq_mx_cache *cache, int64_t batch, int64_t q_heads, int64_t max_pages);
int mpq_mx_attend(const mpq_mx_cache *cache, const void *Q, int64_t q_stride, int64_t q_head_stride, int dtype,
                  int64_t batch, int64_t q_heads, const int32_t *page_table, int64_t table_ld, int64_t max_pages,
                  const int32_t *lengths, int64_t window, float scale, void *O, int64_t o_stride,
                  int64_t o_head_stride, float *lse_opt, void *workspace_opt, int64_t workspace_bytes, void *stream);

/*
 * What a serving step does around the products, the cache and attention: pages
 * and slots of its new tokens (mpq_mx_plan), norms and rotation of its heads
 * (mpq_mx_rotate, mpq_mx_cache_append), and a layer of experts (mpq_mx_route,
 * mpq_mx_experts, mpq_mx_combine).  None waits for the device or reads device
 * memory on the host.  An output of these calls overlaps no other array of the
 * call, unless said otherwise.
 *
 * mpq_mx_plan - the new tokens of `batch` sequences, `fresh[b]` behind the
 * `cached[b]` that sequence b has in the cache (both [batch] int32; negative
 * ones count as 0).  The tokens lie sequence after sequence, those of b from
 * row starts[b] on, as they do in the step's other tensors.
 *   page_table  [batch][table_ld] int32, max_pages columns used (in and out): the
 *               entries of a sequence's ceil(cached / page_size) held pages are
 *               read (only that of a page which new tokens continue), those
 *               of its new pages are written, others are left as they are.
 *   free_pages  [n_free] int32: pages not in use, of which the first *taken
 *               (int32) are already given away.  New pages are the next ones, in
 *               the order of the sequences; -1 where none is left.
 *   taken_out   int32 (output): *taken and the new pages, those without a
 *               free page included, so it exceeds n_free if some are missing;
 *               taken for the next step (pages given back are the caller's to put
 *               into another list).
 *   slots       [max_tokens] int64 (output): page * page_size + place; -1 for a
 *               token without a page (none free, past max_pages, or a table entry
 *               below 0) and for rows past the last token.  Cache calls skip it.
 *   positions   [max_tokens] int32 (output): the token's place in its sequence;
 *               0 for rows past the last token.
 *   starts      [batch + 1] int32, lengths [batch] int32 (outputs): lengths[b] =
 *               cached[b] + fresh[b], as mpq_mx_attend takes it.  A place or
 *               length past 2^31 - 1 is given as that.
 * Tokens past max_tokens in all are taken as not there: starts, lengths and
 * pages count the first max_tokens alone.
 *   batch in [0, 65535]; page_size as a cache's; max_pages * page_size and
 *   max_tokens at most MPQ_MX_MAX_TOKENS.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_mx_plan(const int32_t *cached, const int32_t *fresh, int64_t batch, int32_t *page_table, int64_t table_ld,
                int64_t max_pages, const int32_t *free_pages, int64_t n_free, const int32_t *taken, int64_t page_size,
                int64_t max_tokens, int64_t *slots, int32_t *positions, int32_t *starts, int32_t *lengths,
                int32_t *taken_out, void *stream);

/*
 * mpq_mx_rotate - norm and rotation of the heads of queries and keys.  Of a
 * head x, in fp32 (fp64 where dtype is MPQ_F32), rounded once at the end:
 *   with a weight w  x <- x / sqrt(mean x^2 + eps) w (in fp32, heads larger than
 *                    about 1e19 overflow);
 *   then the pairs (a, b) of its first rot elements, i = 0 .. rot / 2 - 1,
 *   become (a cos t - b sin t, b cos t + a sin t), t = position * freqs[i]; a
 *   and b are elements i and i + rot / 2, or 2 i and 2 i + 1 (interleaved).
 *   The angle is found in fp64, less its whole turns.
 *   Q, QO [n][q_heads][head_dim], K, KO [n][kv_heads][head_dim] of dtype, with
 *               the strides of tokens and heads.  QO may be Q and KO may be K, with
 *               the same strides.
 *   positions   [n] int32; may be NULL if rot = 0.
 *   freqs       [rot / 2] fp64 (DEVICE), radians per position.
 *   q_weight_opt, k_weight_opt  [head_dim] fp32, or NULL: no norm of the
 *               queries, of the keys.
 *   eps         finite and > 0 (looked at with a weight only).
 *   0 <= n < 2^31, 1 <= head_dim <= MPQ_MX_MAX_HEAD_DIM, rot even, at most
 *   head_dim.
 *
 * mpq_mx_cache_append - the same for queries Q to QO, while keys, so turned,
 * and values V are quantized into the cache at `slots` ([n] int64, as in
 * mpq_mx_cache_write).  The keys are not rounded in between: they are computed in
 * fp64, and the rounding to their blocks' elements is the only one.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_mx_rotate(const void *Q, int64_t q_stride, int64_t q_head_stride, const void *K, int64_t k_stride,
                  int64_t k_head_stride, int dtype, int64_t n, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                  const int32_t *positions, const double *freqs, int64_t rot, int interleaved, const float *q_weight_opt,
                  const float *k_weight_opt, float eps, void *QO, int64_t qo_stride, int64_t qo_head_stride, void *KO,
                  int64_t ko_stride, int64_t ko_head_stride, void *stream);
int mpq_mx_cache_append(const mpq_mx_cache *cache, const void *Q, int64_t q_stride, int64_t q_head_stride, const void *K,
                        int64_t k_stride, int64_t k_head_stride, const void *V, int64_t v_stride, int64_t v_head_stride,
                        int dtype, int64_t n, int64_t q_heads, const int32_t *positions, const int64_t *slots,
                        const double *freqs, int64_t rot, int interleaved, const float *q_weight_opt,
                        const float *k_weight_opt, float eps, void *QO, int64_t qo_stride, int64_t qo_head_stride,
                        void *stream);

/*
 * mpq_mx_route - the k largest of each token's expert logits, and the choices
 * sorted by expert.
 *   logits      [n][ld] of dtype, the first `experts` of each row (input).
 *   chosen      [n][k] int32 (output): the experts, by falling logit; equal ones
 *               by rising index (-0 equals 0; NaN counts as -infinity).
 *   weights     [n][k] fp32 (output): the softmax of the logits over all experts,
 *               or, with renorm = 1, over the chosen ones.  Among infinite
 *               logits the weight is shared; with every logit -infinity all are 0.
 *   order       [n * k] int32 (output): choice t * k + j of token t at the places
 *               of expert chosen[t][j], the experts one after the other, an
 *               expert's choices by rising token.
 *   place       [n][k] int32 (output): the inverse: order[place[t][j]] = t k + j.
 *   offsets     [experts + 1] int32 (output): expert e has the places
 *               offsets[e] .. offsets[e + 1] - 1.
 *   0 <= n <= MPQ_MX_MAX_N, 1 <= experts <= MPQ_MX_MAX_EXPERTS, 1 <= k <=
 *   min(experts, MPQ_MX_MAX_CHOICES).
 *   workspace_opt, workspace_bytes  as for mpq_mx_linear, of at least
 *               mpq_mx_route_workspace(n, experts, k) bytes, which do for
 *               fewer tokens too.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int64_t mpq_mx_route_workspace(int64_t n, int64_t experts, int64_t k);
int mpq_mx_route(const void *logits, int dtype, int64_t n, int64_t experts, int64_t ld, int64_t k, int renorm,
                 int32_t *chosen, float *weights, int32_t *order, int32_t *place, int32_t *offsets, void *workspace_opt,
                 int64_t workspace_bytes, void *stream);

/*
 * mpq_mx_experts - rows grouped by expert times their expert's weights:
 *   Y[p] = Q(X[order[p] / k]) W_e^T + b_e,  offsets[e] <= p < offsets[e + 1],
 * Q the quantization of mpq_mx_quantize, products and sums as in mpq_mx_product.
 *   X           [n][x_ld] of x_dtype, the first d of each row (input).
 *   w_codes, w_scales  [experts][c_out] fp4 rows of d (inputs).
 *   offsets     [experts + 1] int32 (DEVICE), ascending in [0, m]; one that is
 *               not is taken as the nearest that is, from the first on.
 *   order_opt   [m] int32 as mpq_mx_route gives it, with its k; or NULL: row p
 *               of X itself (then m = n and k = 1).  An entry that names no row of X
 *               stands for a row of zeros.
 *   bias_opt    NULL or [experts][c_out] fp32, added in fp32.
 *   Y           [m][ld] of dtype (output), ld >= c_out.  Rows of no group (before
 *               offsets[0], from offsets[experts] on) are left as they were.
 *   0 <= n <= MPQ_MX_MAX_N, 0 <= m <= MPQ_MX_MAX_ROWS; with D as above, (n + 1) D
 *   below 2^32 and experts * c_out * D at most 2^42.
 *   workspace_opt, workspace_bytes  as for mpq_mx_linear, of at least
 *               mpq_mx_experts_workspace(n, m, experts, c_out, d) bytes, which do
 *               for smaller n and m too.
 * How the work is cut follows from n, m, experts, c_out and d, and so do the last
 * bits of a row; they do not depend on the other rows or on the groups' sizes.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_NOMEM, MPQ_ERR_HIP.
 */
int64_t mpq_mx_experts_workspace(int64_t n, int64_t m, int64_t experts, int64_t c_out, int64_t d);
int mpq_mx_experts(const void *X, int x_dtype, int64_t n, int64_t x_ld, const uint8_t *w_codes, const uint8_t *w_scales,
                   int64_t experts, int64_t c_out, int64_t d, const int32_t *offsets, const int32_t *order_opt, int64_t m,
                   int64_t k, const float *bias_opt, void *Y, int dtype, int64_t ld, void *workspace_opt,
                   int64_t workspace_bytes, void *stream);

/*
 * mpq_mx_combine - every token's weighted sum of its experts' rows:
 *   Z[t] = residual[t] + sum_j weights[t][j] Y[place[t][j]],
 * in fp32 in the order of j, rounded once.
 *   Y           [m][y_ld] of y_dtype, the first c of each row (input).
 *   place       [n][k] int32, weights [n][k] fp32 (inputs).  A place outside
 *               [0, m) takes no part.
 *   residual_opt NULL or [n][residual_ld] of y_dtype (input).
 *   Z           [n][ld] of dtype (output); may be the residual, with the same
 *               type and stride.
 *   0 <= n <= MPQ_MX_MAX_N, 0 <= m <= MPQ_MX_MAX_ROWS, 0 <= c <= MPQ_MX_MAX_D,
 *   0 <= k <= MPQ_MX_MAX_CHOICES.
 * Errors: MPQ_ERR_INVALID_ARG, MPQ_ERR_HIP.
 */
int mpq_mx_combine(const void *Y, int y_dtype, int64_t m, int64_t c, int64_t y_ld, const int32_t *place,
                   const float *weights, int64_t n, int64_t k, const void *residual_opt, int64_t residual_ld, void *Z,
                   int dtype, int64_t ld, void *stream);

/*
 * Per-launch timing (instrumentation, not part of the method).  While it is
 * enabled, every kernel launch of the library is bracketed by two HIP events
 * recorded on the stream the kernel runs on (a call may run independent
 * launches on library-owned streams, joined back to the caller's stream).
 *
 * mpq_timing_enable(on): drops the records collected so far and turns the
 *   recording on (on != 0) or off.  Returns MPQ_OK.
 * mpq_timing_only(name): while the recording is on, record only the
 *   launches of the kernel of this name (a HOST string of up to 63 bytes, as
 *   mpq_timing_read reports it), so that timing one kernel adds no events
 *   around the others; NULL or "" records every launch again.  Returns MPQ_OK,
 *   or MPQ_ERR_INVALID_ARG for a longer name.
 * mpq_timing_read(out, cap): waits for the recorded events, writes up to cap
 *   records (HOST array) in launch order and returns the number of records
 *   (which may exceed cap), or MPQ_ERR_INVALID_ARG.  ms is -1 for a record
 *   whose events could not be read.
 * mpq_fit_kernel_of(d, bits, n_grid, default_grid, name, cap): writes to the
 *   HOST buffer name (cap bytes) the kernel name under which mpq_fit_layer
 *   records the fit of channels of length d (default_grid: grid_host ==
 *   NULL).  Returns an MPQ_* status.
 */
typedef struct mpq_kernel_time {
    char name[64];
    float ms;
} mpq_kernel_time;

int mpq_timing_enable(int on);
int mpq_timing_only(const char *name);
int mpq_timing_read(mpq_kernel_time *out, int cap);
int mpq_fit_kernel_of(int64_t d, int bits, int n_grid, int default_grid, char *name, int cap);

/* Text of the calling thread's last failure ("" if none).  The pointer stays
 * valid until the thread's next failing call. */
const char *mpq_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* MPQ_H */
