/*
 * turbomuon.h - C ABI of the MI355X (gfx950) Turbo-Muon orthogonalizer.
 *
 * The library approximates the polar factor of gradient matrices with the
 * pre-conditioned Newton-Schulz iteration of arXiv 2512.04632:
 *
 *   Algorithm 2 (Turbo-Muon): A0 = Gram of X0; AOL vector
 *     s_i = 1 / sqrt(sum_j |A0_ij|)                       (eq. (aol), Sec. 4.1)
 *   X1 = X0 scaled by s, A1 = diag(s) A0 diag(s) (no second product), then for
 *   k = 1..t:  A_k = Gram(X_k) (k >= 2), B_k = b_k A_k + c_k A_k^2,
 *              X_{k+1} = a_k X_k + X_k B_k                (Algorithm 1, eq. (ns_quintic))
 *   Algorithm 1 (Muon) instead scales by 1 / ||X0||_F (precond FROBENIUS); the
 *   Schatten-4 variant of the paper's appendix on other pre-conditionings scales
 *   by (sum_i sigma_i^4)^(-1/4) = ||A0||_F^(-1/2), again from the first Gram.
 *
 * Orientation.  For an m x n input with m <= n (square included) the Gram is
 * the m x m matrix X X^T and the AOL vector scales rows; for m > n it is the
 * n x n matrix X^T X and scales columns.  The Gram is always min(m, n) square
 * (Sec. 4.1 keeps the extra memory at O(min(m, n))).  The output keeps the
 * input's layout.
 *
 * Arithmetic.  bf16 entry points store X, A and B in bfloat16 (round to
 * nearest even) and accumulate every product in fp32 on the matrix cores; the
 * AOL row sums are taken from the fp32 Gram accumulators.  Where the long side
 * is much the longer (max(m, n) - min(m, n) at least 1280 to 2560 by min(m, n),
 * which is at least 256; 4096 for iters = 2 below 1536), two iterations share one Gram
 * and one update, with fp16 A, B between them (about half the error of one by
 * one; calls whose coefficients could leave fp16's range, and precond NONE, run
 * one by one).  f32 entry points store in fp32 and accumulate in fp32; matrices
 * with min(m, n) >= 64 are multiplied as two fp16 planes, scaled row by row, the
 * others (and the calls named above) in fp32.  The planes hold an entry to 2^-22
 * of itself, or to 2^-49 of its row's largest (between iterations, of sigma_max)
 * where that is more: rows of any size whose squares fp32 holds (1e-18 and more)
 * keep their accuracy, entries and columns from about 2^-20 of the others.  In either form a row far below the others is
 * worked on at a larger size under FROBENIUS and SCHATTEN4 and scaled back;
 * behind AOL, which levels the rows, rows keep their accuracy from about 1e-14 of
 * the others.  Results are deterministic (no float atomics) and do not depend on
 * what else is in the call.
 *
 * Small matrices.  A bf16 call with iters >= 1 whose every matrix has
 * min(m, n) <= 128 and fits, zero padded to multiples of 32, in one compute
 * unit's 160 KB of LDS (min(m, n) = 64: max(m, n) <= 1088; 128: <= 320) runs
 * as a single launch, one workgroup per matrix, with no workspace.  Its
 * results are bit for bit those of the tiled kernels that other calls use
 * (the same products in the same order, the same roundings); setting
 * TM_DISABLE_FUSED in the environment sends such calls to the tiled kernels.
 *
 * Streams and memory.  All work is enqueued on `stream` (a hipStream_t passed
 * as void*, NULL = the legacy default stream) without host synchronisation;
 * results are valid once the stream has passed the call.  Matrix pointers are
 * device pointers owned by the caller.  The library owns a workspace per
 * (device, stream), grown on first use with hipMalloc and kept until
 * tm_release_workspaces() or process exit; growing it synchronises `stream`.
 * Where that much memory is not to be had, the call tries the layout with the
 * least padding (the same results) and, in fp32, the fp32 products.
 * Calls on different streams may run concurrently; calls that overlap on the
 * same stream are ordered by the stream.  The cache is keyed by the stream
 * handle: synchronise a stream before destroying it, since a stream created
 * later may receive the same handle and reuse that workspace.
 *
 * Graph capture.  A call on a stream whose workspace is already large enough
 * (an earlier call of the same or larger shapes and the same type on that
 * stream, whatever its iters, coeffs and precond; calls of the single-launch
 * kernel need no workspace and reserve none) allocates nothing and synchronises
 * nothing, so it can be captured into a HIP graph; the captured kernels keep
 * that workspace's address.  A call under capture
 * whose workspace is too small returns TM_ERR_UNSUPPORTED (nothing can be
 * allocated during capture).  A workspace once used under capture is never
 * freed or reused in place by a larger call: a later, larger eager call on the
 * same stream handle (torch hands out pooled stream handles, so another stream
 * object may share it) gets a new workspace and the captured one stays valid
 * until tm_release_workspaces(), which must not be called while such a graph
 * is in use.  Graphs captured on one stream share its workspace: do not replay
 * them concurrently (on different streams) with each other or with eager calls
 * on that stream.  tm_orthogonalize_noalloc needs no workspace at all.
 *
 * Errors.  Arguments are validated before anything is enqueued; an invalid
 * call returns a negative status and leaves memory untouched.  Failures of the
 * HIP runtime return TM_ERR_HIP.  tm_last_error() gives a thread-local message
 * for the last failure.  Input values are not checked: NaN/Inf propagate.
 */
#ifndef TURBOMUON_H
#define TURBOMUON_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int tm_status;

#define TM_OK               0
#define TM_ERR_INVALID_ARG  (-1) /* null pointer, size or iteration count out of range, unknown precond */
#define TM_ERR_UNSUPPORTED  (-2) /* pointer not element aligned, no gfx950 device, launch too large */
#define TM_ERR_NO_MEMORY    (-3) /* workspace allocation failed */
#define TM_ERR_HIP          (-4) /* a HIP runtime call or kernel launch failed */

/* Pre-conditioning of the first iteration. */
#define TM_PRECOND_NONE       0  /* X1 = X0 */
#define TM_PRECOND_FROBENIUS  1  /* X1 = X0 / ||X0||_F: Algorithm 1 (Muon); zero stays zero */
#define TM_PRECOND_AOL        2  /* X1 = AOL(X0), eq. (aol): Algorithm 2 (Turbo-Muon) */
#define TM_PRECOND_SCHATTEN4  3  /* X1 = X0 / ||X0||_S4 with ||X0||_S4 = ||A0||_F^(1/2) from the
                                    first Gram (appendix on other pre-conditionings) */

/* Limits checked by every entry point. */
#define TM_MAX_DIM    65536      /* m, n <= TM_MAX_DIM */
#define TM_MAX_ITERS  64         /* 0 <= iters <= TM_MAX_ITERS */

/*
 * tm_orthogonalize - Algorithm 2 (precond AOL) or Algorithm 1 (FROBENIUS/NONE)
 * on `batch` bf16 matrices, in place.
 *
 *   X       device pointer, `batch` row-major m x n bfloat16 matrices stored
 *           back to back (matrix b starts at X + b*m*n); aligned to the
 *           element size (16-byte alignment and n % 8 == 0 enable vector loads).
 *           Overwritten with the result X_{iters+1}.
 *   m, n    1 <= m, n <= TM_MAX_DIM.
 *   batch   >= 0; 0 is a no-op returning TM_OK.
 *   iters   number t of (Gram, polynomial, update) triples, 0..TM_MAX_ITERS.
 *           iters = 0 returns the pre-conditioned X1.  Turbo-Muon's default
 *           is 4 (Sec. 2), Muon's 5.
 *   coeffs  host array of iters*3 floats (a_k, b_k, c_k) in iteration order,
 *           read during the call only; NULL selects the constant triple
 *           (3.4445, -4.7750, 2.0315) for every iteration.
 *   precond TM_PRECOND_*.
 *   stream  hipStream_t as void*.
 */
tm_status tm_orthogonalize(void* X, int64_t m, int64_t n, int64_t batch, int iters,
                           const float* coeffs, int precond, void* stream);

/* Same contract with fp32 storage (products as stated under Arithmetic). */
tm_status tm_orthogonalize_f32(float* X, int64_t m, int64_t n, int64_t batch, int iters,
                               const float* coeffs, int precond, void* stream);

/*
 * tm_orthogonalize_grouped - `count` independent bf16 matrices of arbitrary
 * shapes, processed together: every phase of the iteration (Gram, AOL
 * vector, polynomial, update) is one launch over the tiles of all matrices.
 *
 *   X       host array of `count` device pointers (element aligned, pairwise
 *           non-overlapping); matrix g is row-major m[g] x n[g].
 *   m, n    host arrays of `count` sizes, each in 1..TM_MAX_DIM.
 *   count   >= 0; 0 is a no-op.
 *   other arguments as tm_orthogonalize; the same coefficients and
 *   pre-conditioning apply to every matrix.  The host arrays are read during
 *   the call only.
 */
tm_status tm_orthogonalize_grouped(void* const* X, const int64_t* m, const int64_t* n,
                                   int64_t count, int iters, const float* coeffs,
                                   int precond, void* stream);

/* Grouped variant with fp32 storage. */
tm_status tm_orthogonalize_grouped_f32(float* const* X, const int64_t* m, const int64_t* n,
                                       int64_t count, int iters, const float* coeffs,
                                       int precond, void* stream);

/*
 * tm_muon_step_grouped - one optimizer step over `count` fp32 parameter
 * matrices: Muon's step with its orthogonalization done by this library (the
 * paper uses Turbo-Muon as a drop-in replacement of Muon's orthogonalization;
 * its steepest-descent appendix writes the update as -eta PolarFactor(G S)).
 * Per matrix g (rows m[g], columns n[g], row-major):
 *
 *   M <- momentum M + G
 *   U  = G + momentum M   if nesterov, else U = M      (rounded to bf16)
 *   O  = the bf16 orthogonalization of U (tm_orthogonalize_grouped semantics:
 *        iters, coeffs, precond as there)
 *   W <- W (1 - lr weight_decay) - lr scale O,
 *        scale = sqrt(max(1, m[g] / n[g])) if shape_scale, else 1
 *
 *   W, G, M  host arrays of `count` device pointers to fp32 matrices (4-byte
 *            aligned; W and M updated in place, G read only; no two of all
 *            these matrices may overlap).
 *   m, n     host arrays of sizes, each in 1..TM_MAX_DIM.
 * U lives in a second library-owned buffer per (device, stream), grown like
 * the workspace.  Errors as tm_orthogonalize_grouped.
 */
tm_status tm_muon_step_grouped(float* const* W, const float* const* G, float* const* M,
                               const int64_t* m, const int64_t* n, int64_t count, float lr,
                               float momentum, int nesterov, float weight_decay, int shape_scale,
                               int iters, const float* coeffs, int precond, void* stream);

/*
 * tm_schedule_tail - fewer iterations from a coefficient schedule designed for
 * more (appendix on the tuning of Newton-Schulz coefficients: a schedule
 * computed for a fixed number of iterations runs fewer by keeping its last
 * rows).
 *
 *   schedule  host array of rows*3 floats (a_k, b_k, c_k) in iteration order.
 *   rows      rows of the schedule, 1..TM_MAX_ITERS.
 *   iters     iterations to run, 0..rows.
 * Returns schedule + 3*(rows - iters): the last `iters` rows, to pass as the
 * `coeffs` of a call with that many iterations.  Reads no element and
 * allocates nothing; NULL (detail in tm_last_error) for a NULL schedule or
 * rows / iters out of range.
 */
const float* tm_schedule_tail(const float* schedule, int rows, int iters);

/*
 * tm_orthogonalize_noalloc - tm_orthogonalize for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same arguments, kernels and launch plan as
 * tm_orthogonalize (results are bitwise equal to it), but the workspace is a
 * static device array of TM_NOALLOC_SCRATCH_BYTES per GPU, placed with the
 * library's code object and held until the process ends, instead of the
 * per-stream cache.  The call allocates nothing, frees nothing and
 * synchronises nothing; the timing hooks do not apply to it.
 *
 *   Limit   the call's workspace (tm_workspace_bytes over `batch` copies of
 *           the shape m x n, dtype_bytes 2) must fit in
 *           TM_NOALLOC_SCRATCH_BYTES: e.g. one 2048 x 2048 matrix (48 MiB),
 *           one 1024 x 4096 (24 MiB) or a batch of 4 of 768 x 3072 (54 MiB);
 *           a larger call returns TM_ERR_UNSUPPORTED before anything is
 *           enqueued.
 *   Sharing every call on one GPU uses that GPU's one array: calls that
 *           overlap in time on a GPU (other streams or host threads) race and
 *           must be serialised by the caller.  The array keeps the last call's
 *           contents; nothing in it needs to start at zero.
 */
#define TM_NOALLOC_SCRATCH_BYTES 67108864   /* 64 MiB */
tm_status tm_orthogonalize_noalloc(void* X, int64_t m, int64_t n, int64_t batch, int iters,
                                   const float* coeffs, int precond, void* stream);

/* ------------------------------------------------------------------ operators
 * What a training step needs around the optimizer: layer norm and
 * root-mean-square norm, the routing of rows to experts, rows on their way to
 * the experts' order and back, products of ragged groups of rows with one
 * matrix per expert (whose weight gradients are the matrices that
 * tm_muon_step_grouped takes), the log probabilities of given tokens and the
 * clipped policy loss, with their gradients.  Matrices are row-major with a stride between rows (in
 * elements, at least the width); pointers are aligned to their element only,
 * though 16-byte alignment and strides are faster.  `dtype` is the type of the
 * activations; parameters, statistics and sums are fp32.  Streams, errors,
 * graph capture and timing are as stated above; the calls marked (W) keep
 * partial sums in a workspace of their own per (device, stream), which grows
 * and is captured like the orthogonalizer's.  Every result is the same on
 * every run (no float atomics); the order of a sum, and so the last bits, may
 * differ with the sizes, strides and alignment of a call (fp32 expert products:
 * and with the values of the rows and columns next to it).  NaN and Inf
 * propagate, but never out of rows that take no part.
 */
#define TM_DTYPE_BF16 0
#define TM_DTYPE_F32  1
#define TM_MAX_ROWS    1073741824  /* rows of an operator */
#define TM_MAX_EXPERTS 8192
#define TM_MAX_VOCAB   1073741824
#define TM_MAX_TOP     64          /* experts of a row, alternatives of a token */

/*
 * tm_layer_norm - per row of d elements
 *   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),
 *   y = (x - mean) rstd weight + bias.
 *   weight, bias  d floats each, or NULL (ones, zeros).
 *   mean, rstd    rows floats, written.
 *   y may be x (same stride).  rows 0..TM_MAX_ROWS, d 1..TM_MAX_DIM.
 */
tm_status tm_layer_norm(const void* x, int64_t ldx, const float* weight, const float* bias, void* y,
                        int64_t ldy, float* mean, float* rstd, int64_t rows, int64_t d, float eps,
                        int dtype, void* stream);

/*
 * tm_layer_norm_backward (W) - with h = (x - mean) rstd and g = dy weight
 *   dx = rstd (g - sum g / d - h sum(g h) / d),
 *   dweight = sum over rows of dy h,  dbias = sum over rows of dy.
 *   dweight, dbias  d floats each, written in full (zeros for no rows), or
 *                   NULL where not wanted.
 *   dx may be dy or x (same stride).
 */
tm_status tm_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                 const float* weight, const float* mean, const float* rstd, void* dx,
                                 int64_t lddx, float* dweight, float* dbias, int64_t rows, int64_t d,
                                 int dtype, void* stream);

/*
 * tm_rms_norm - per row of d elements
 *   s = x + residual (rounded to the type), or x without a residual,
 *   rstd = 1 / sqrt(sum s^2 / d + eps),  y = s rstd weight.
 *   residual  rows x d, or NULL.
 *   weight    d floats, or NULL (ones).
 *   sum       rows x d: s, written where there is a residual, else ignored.
 *   rstd      rows floats, written.
 *   sum and y may be x or the residual (same stride), not each other.  Squares
 *   are summed in fp32: a row with values of 1e19 and more gives zeros.
 */
tm_status tm_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight,
                      void* sum, int64_t lds, void* y, int64_t ldy, float* rstd, int64_t rows, int64_t d,
                      float eps, int dtype, void* stream);

/*
 * tm_rms_norm_backward (W) - with h = s rstd and g = dy weight
 *   ds = rstd (g - h sum(g h) / d) + dsum,  dweight = sum over rows of dy h.
 *   s        what was normalised: tm_rms_norm's sum, or its x.
 *   dsum     rows x d, the gradient that reaches s by another way, or NULL.
 *   ds       gradient of x and, the same, of the residual.
 *   dweight  d floats, written in full (zeros for no rows), or NULL.
 *   ds may be dy, s or dsum (same stride).
 */
tm_status tm_rms_norm_backward(const void* dy, int64_t lddy, const void* s, int64_t lds, const float* weight,
                               const float* rstd, const void* dsum, int64_t lddsum, void* ds, int64_t ldds,
                               float* dweight, int64_t rows, int64_t d, int dtype, void* stream);

/*
 * tm_expert_route (W, more than 64 rows) - the `top` experts of each row, by its scores l.  With
 * p = softmax(l) over the experts and N rows that take part:
 *   chosen   rows x top: the experts of the `top` largest l, largest first; of equal
 *            ones the lowest index; NaN counts as -inf.
 *   weights  rows x top: scale p of the chosen, over the sum of the row's chosen p
 *            if `renormalize`.
 *   slots    rows x top: where each choice stands in the experts' order (by expert,
 *            then by row), without gaps from 0.
 *   ends     `experts` entries: the choices of the experts up to and with each one, as
 *            tm_expert_matmul takes them.
 *   balance  one float: experts sum_e (c_e / (top N)) (sum over rows of p_e / N), c_e
 *            the choices of expert e: 1 where all are alike, 0 if N = 0.
 *   active   one byte per row, or NULL: rows of 0 take no part; they are not read,
 *            their choices and slots are -1, their weights 0.
 *   experts 1..TM_MAX_EXPERTS, top 1..min(experts, TM_MAX_TOP), rows top at most
 *   TM_MAX_ROWS.  A row of nothing but -inf, or with inf or NaN, has weights of NaN, and so is
 *   the balance; its choices are experts all the same.
 */
tm_status tm_expert_route(const void* logits, int64_t ld, const uint8_t* active, int renormalize, float scale,
                          int32_t* chosen, float* weights, int32_t* slots, int32_t* ends, float* balance,
                          int64_t rows, int64_t experts, int64_t top, int dtype, void* stream);

/*
 * tm_expert_route_backward - gradient by the logits from those of the weights
 * (dweights, rows x top) and of the balance (dbalance, a device float); NULL: zero.
 *   chosen, ends  tm_expert_route's; renormalize, scale as there.  A row whose first
 *                 choice is negative takes no part, its gradient is zero; other
 *                 choices that are no experts are left out.
 *   dlogits may be the logits.
 */
tm_status tm_expert_route_backward(const void* logits, int64_t ld, const int32_t* chosen, const int32_t* ends,
                                   const float* dweights, const float* dbalance, int renormalize, float scale,
                                   void* dlogits, int64_t ldd, int64_t rows, int64_t experts, int64_t top,
                                   int dtype, void* stream);

/*
 * tm_expert_gather - out[slots[i, j], :] = x[i, :].
 *   x      rows x d;  out  count x d, of the same type.
 *   slots  rows x top.  A slot that is negative, or not below *used, is none.  No two
 *          may be the same: their row would hold parts of both.
 *   used   device int32: rows of `out` that are filled (tm_expert_route's last entry of
 *          ends), or NULL: all.  Rows from there on come out as zeros; one below it
 *          that no slot names is left as it was.
 * Whatever slots and *used hold, nothing outside the matrices is read or written.
 * out overlaps nothing that is read.
 */
tm_status tm_expert_gather(const void* x, int64_t ldx, const int32_t* slots, const int32_t* used, void* out,
                           int64_t ldo, int64_t count, int64_t rows, int64_t top, int64_t d, int dtype,
                           void* stream);

/*
 * tm_expert_combine - out[i, :] = residual[i, :] + sum_j weights[i, j] y[slots[i, j], :],
 * summed in fp32 in the order of j, the residual last, and rounded once.
 *   y         count x d;  out  rows x d.
 *   weights   rows x top, or NULL: ones (what the gradient of tm_expert_gather is).
 *   residual  rows x d, or NULL.
 *   used      device int32: rows of y that are filled, or NULL: all.
 *   Slots that are negative or not below *used are left out (nor below count, whatever
 *   *used holds); the same one may be named twice.  out may be the residual (same
 *   stride), and overlaps nothing else.
 */
tm_status tm_expert_combine(const void* y, int64_t ldy, const int32_t* slots, const int32_t* used,
                            const float* weights, const void* residual, int64_t ldr, void* out, int64_t ldo,
                            int64_t count, int64_t rows, int64_t top, int64_t d, int dtype, void* stream);

/*
 * tm_expert_combine_backward - dy[slots[i, j], :] = weights[i, j] dout[i, :],
 * dweights[i, j] = sum over the columns of dout[i, :] y[slots[i, j], :].
 *   slots, used  as in tm_expert_gather, for dy;  a choice without a slot has a
 *                gradient of zero.
 *   dweights     rows x top, or NULL: y is not read then, and may be NULL.
 *   dy may be y (same stride).
 */
tm_status tm_expert_combine_backward(const void* dout, int64_t lddout, const void* y, int64_t ldy,
                                     const int32_t* slots, const int32_t* used, const float* weights, void* dy,
                                     int64_t lddy, float* dweights, int64_t count, int64_t rows, int64_t top,
                                     int64_t d, int dtype, void* stream);

/*
 * tm_expert_matmul (W) - y[i, :] = x[i, :] W[e], e the expert of row i.
 *   x     rows x k;  y  rows x n, of the same type.
 *   w     matrix e starts at w + e stride_w: k x n with row stride ldw, or
 *         n x k where `transposed` (y = x W^T: with the forward pass's w and dy
 *         for x this is the gradient of the rows).
 *   ends  device array of `experts` int32, not decreasing: expert e owns rows
 *         ends[e - 1] .. ends[e] - 1 (from 0 for e = 0).  Experts may own no
 *         row.  Rows after the last expert's come out as zeros.  Read on the
 *         stream: no host synchronisation.  Whatever it holds, nothing outside
 *         the matrices is read or written.
 *   k, n  1..TM_MAX_DIM;  experts 1..TM_MAX_EXPERTS.
 * y overlaps nothing that is read.  Sums are fp32.  fp32 products of many rows
 * are formed of three bf16 parts of each operand on the matrix cores and are as
 * exact as a sum of fp32 products; tiles with values that three parts do not hold
 * exactly (NaN, Inf, values that round past the largest bf16, values below about
 * 2^-110) or with results that are not finite take fp32 products, at less than
 * half the speed.
 * Workspace: a call whose summed index is cut into slices keeps a result in fp32
 * (rows x n) of each: calls of few tiles, up to 64 slices, and fp32 calls of few
 * tiles or up to 64 rows an expert, ceil(k / 2816) at least.  That is at most 100 MB
 * or a twentieth of the matrices.
 */
tm_status tm_expert_matmul(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t stride_w,
                           const int32_t* ends, void* y, int64_t ldy, int64_t rows, int64_t experts,
                           int64_t k, int64_t n, int transposed, int dtype, void* stream);

/*
 * tm_expert_wgrad (W) - dw[e] = x_e^T dy_e over the rows of each expert (k x n;
 * zeros for an expert without rows).
 *   x, dy      rows x k and rows x n of type `dtype`.
 *   dw         matrix e starts at dw + e stride_dw, row stride lddw; of type
 *              `out_dtype`: fp32, or bf16 where the rows are.
 * Sums as in tm_expert_matmul.  Workspace: calls of few tiles keep a matrix in
 * fp32 (k x n) for every chunk of 256 rows or more that an expert's are cut into.
 */
tm_status tm_expert_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* ends,
                          void* dw, int64_t lddw, int64_t stride_dw, int64_t rows, int64_t experts,
                          int64_t k, int64_t n, int dtype, int out_dtype, void* stream);

/*
 * tm_token_logp (W, rows that are cut: up to 128 of more than 200 KB, and any of
 * more than 512 KB) - over rows of logits l with target y, at temperature tau, with
 * m = max_v l_v and s = sum_v exp((l_v - m) / tau):
 *   logp     log p_y = (l_y - m) / tau - log s,
 *   entropy  -sum_v p_v log p_v,
 *   stats    m and s, two floats per row (what the gradient is taken from),
 *   top_logp, top_ids  rows x top: the largest log probabilities and their places,
 *            largest first; of equal logits the lowest place.  -inf and NaN are no
 *            alternatives: where there are fewer than `top`, -inf and -1.
 *   targets  int64 per row.  A negative target takes its row out: zeros, places of -1,
 *            its logits are not read; one of vocab or more makes its logp NaN.
 *   top      0..min(vocab, TM_MAX_TOP); with 0 top_logp and top_ids may be NULL.
 * A row of nothing but -inf, or with inf or NaN, gives NaN.
 */
tm_status tm_token_logp(const void* logits, int64_t ld, const int64_t* targets, float temperature, float* logp,
                        float* entropy, float* stats, int64_t top, float* top_logp, int64_t* top_ids,
                        int64_t rows, int64_t vocab, int dtype, void* stream);

/*
 * tm_token_logp_backward - with p from stats, g = dlogp and h = dentropy per row (NULL:
 * zeros)
 *   dlogits_v = (g ([v = y] - p_v) - h p_v (log p_v + entropy)) / tau.
 *   stats, entropy  tm_token_logp's on the same logits, targets and temperature.
 * Rows without a target, or with g = h = 0, are not read, their gradient is zero.
 * dlogits may be the logits.
 */
tm_status tm_token_logp_backward(const void* logits, int64_t ld, const int64_t* targets, const float* stats,
                                 const float* entropy, const float* dlogp, const float* dentropy,
                                 float temperature, void* dlogits, int64_t ld_dlogits, int64_t rows,
                                 int64_t vocab, int dtype, void* stream);

/*
 * tm_policy_loss (W) - clipped policy loss with a KL term over rows of logits
 * l with target y, at temperature tau:
 *   lse = log sum_v exp(l_v / tau),  logp = l_y / tau - lse,
 *   r = exp(logp - old_logp),  q = exp(ref_logp - logp),
 *   loss = sum over rows of weight (-min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *                                   + kl (q - log q - 1)),
 *   slope = d loss / d logp,  dlogits_v = slope ([v = y] - exp(l_v / tau - lse)) / tau.
 *   logits      rows x vocab.
 *   targets     int64 per row.  A negative target takes its row out, as weight
 *               0 does; a target of vocab or more makes its row's results NaN.
 *   old_logp, advantages, weights  fp32 per row; the weights hold the mask and
 *               whatever the loss is divided by.
 *   ref_logp    fp32 per row, or NULL: no KL term.
 *   loss        one float.
 *   logp        fp32 per row, written; lse, slope likewise, or NULL.
 *   dlogits     rows x vocab of the logits' type (it may be the logits), or
 *               NULL: the value alone.
 * Rows that take no part: logp, lse, slope and their gradient are zero, their
 * logits are not read.  A row of nothing but -inf gives NaN.  loss and logp have
 * the same bits with and without dlogits.
 */
tm_status tm_policy_loss(const void* logits, int64_t ld, const int64_t* targets, const float* old_logp,
                         const float* advantages, const float* weights, const float* ref_logp,
                         float clip_low, float clip_high, float kl, float temperature, float* loss,
                         float* logp, float* lse, float* slope, void* dlogits, int64_t ld_dlogits,
                         int64_t rows, int64_t vocab, int dtype, void* stream);

/*
 * tm_policy_loss_backward - dlogits from the lse and slope of an earlier
 * tm_policy_loss on the same logits, targets and temperature, times *grad (a
 * device float, NULL for 1).  Rows of slope 0 are not read, their gradient is
 * zero.  dlogits may be the logits.  The probabilities are taken from lse, whose
 * rounding (2^-24 of it) they carry: with logits of large size, such as a row of
 * nothing but the lowest value, tm_policy_loss's dlogits are the exact ones.
 */
tm_status tm_policy_loss_backward(const void* logits, int64_t ld, const int64_t* targets,
                                  const float* lse, const float* slope, const float* grad,
                                  float temperature, void* dlogits, int64_t ld_dlogits, int64_t rows,
                                  int64_t vocab, int dtype, void* stream);

/* Bytes of workspace a call with these shapes needs (0 on invalid shapes).
 * dtype_bytes is 2 (bf16) or 4 (fp32).  An upper bound: a bf16 call that the
 * fused small-matrix kernel serves uses none. */
uint64_t tm_workspace_bytes(const int64_t* m, const int64_t* n, int64_t count,
                            int dtype_bytes);

/* Free every cached workspace.  Synchronises the device first; must not be
 * called while another thread is inside a tm_* call. */
tm_status tm_release_workspaces(void);

/* Kernel phases, as counted by the timing hooks below. */
#define TM_PHASE_TRANSPOSE_IN  0  /* tall input: W = X^T */
#define TM_PHASE_FROB          1  /* partial sums of squares of X0 (Algorithm 1, first line) or of A0 (Schatten-4) */
#define TM_PHASE_GRAM          2  /* A = X X^T, upper tiles (+ AOL row sums at iteration 1) */
#define TM_PHASE_AOL_VECTOR    3  /* s_i = 1/sqrt(row sum) (Algorithm 2, second line) */
#define TM_PHASE_POLY          4  /* B = b A + c A^2 */
#define TM_PHASE_UPDATE        5  /* X <- a X + B X */
#define TM_PHASE_APPLY_SCALE   6  /* iters = 0: X1 = diag(s) X0 */
#define TM_PHASE_COPY_OUT      7  /* iters = 1: result copied into the caller's buffer */
#define TM_PHASE_LOAD_IN       8  /* X (or X^T) copied into the zero-padded workspace; fp32: row maxima,
                                    then the fp16 planes */
#define TM_PHASE_SCALE_A       9  /* tiled kernels: A1 = diag(s) A0 diag(s) (X1 is never stored: the first
                                    polynomial keeps B~ diag(s) and the update reads X0) */
#define TM_PHASE_OPT_MOMENTUM 10  /* optimizer step: momentum and the bf16 matrix to orthogonalize */
#define TM_PHASE_OPT_APPLY    11  /* optimizer step: parameter update */
#define TM_PHASE_FUSED        12  /* bf16 calls of small matrices: every iteration in one launch */
#define TM_PHASE_LAYER_NORM   13  /* from here on: one record per call, all of its launches */
#define TM_PHASE_LAYER_NORM_BACKWARD  14
#define TM_PHASE_EXPERT_MATMUL        15
#define TM_PHASE_EXPERT_WGRAD         16
#define TM_PHASE_POLICY_LOSS          17
#define TM_PHASE_POLICY_LOSS_BACKWARD 18
#define TM_PHASE_RMS_NORM             19
#define TM_PHASE_RMS_NORM_BACKWARD    20
#define TM_PHASE_EXPERT_ROUTE         21
#define TM_PHASE_EXPERT_ROUTE_BACKWARD   22
#define TM_PHASE_EXPERT_GATHER        23
#define TM_PHASE_EXPERT_COMBINE       24
#define TM_PHASE_EXPERT_COMBINE_BACKWARD 25
#define TM_PHASE_TOKEN_LOGP           26
#define TM_PHASE_TOKEN_LOGP_BACKWARD  27
#define TM_NUM_PHASES         28

/* Timing hooks (a profiling aid for benchmarks).  While enabled, every kernel
 * launch of later calls is bracketed by a pair of HIP events recorded on the
 * call's stream.  tm_timing_read synchronises the recorded events and returns
 * the summed event time (ms) and launch count of one phase since the last
 * reset; tm_timing_reset drops the records.  Not thread-safe with concurrent
 * tm_* calls on other threads. */
tm_status tm_timing_enable(int enable);
tm_status tm_timing_read(int phase, double* total_ms, int64_t* launches);
tm_status tm_timing_reset(void);

/* Static description of a status code. */
const char* tm_status_string(tm_status s);

/* Thread-local detail of the last failure in this thread ("" if none). */
const char* tm_last_error(void);

/* Library version, "major.minor.patch". */
const char* tm_version(void);

#ifdef __cplusplus
}
#endif

#endif /* TURBOMUON_H */
