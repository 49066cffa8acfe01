/*
 * sparseinfer.h -- C ABI of the MI355X (gfx950) SparseInfer decode path.
 *
 * SparseInfer (arXiv 2411.12692) predicts which rows of a ReLU-fied gated MLP
 * produce a zero activation by comparing sign bits only (Section IV-A), then
 * runs the MLP of Eq. (1) over the remaining rows (Section IV-B).  This
 * library implements that per-token path with hand-written HIP kernels.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Tensors are DEVICE pointers allocated by the caller (the library never
 *   allocates or frees), row-major, 16-byte aligned.  fp16 tensors are passed
 *   as uint16_t bit patterns (IEEE binary16).
 * - Shapes: d = model dimension, k = hidden (d_ff) dimension, b = tokens in
 *   the decode batch.  Supported: 1 <= k <= 2^24, 128 <= d <= 8192 with
 *   d % 128 == 0, 1 <= b <= 8.
 * - Work is enqueued asynchronously on `stream` (a hipStream_t; NULL means
 *   the default stream).  Calls return after enqueueing.
 * - Errors: arguments are validated on the host before anything is enqueued;
 *   on any error nothing is launched, outputs are untouched, the status code
 *   says which check failed and si_last_error() (thread-local) says why.
 *   A failed launch returns SI_ERR_HIP.  Faults inside kernels surface at the
 *   caller's next synchronisation, as for any HIP kernel.
 * - Workspace: entry points that take `workspace` need a caller-owned device
 *   buffer of at least si_workspace_bytes(k, d, b) bytes that is ZERO-FILLED
 *   before its first use.  The library keeps it consistent from one call to
 *   the next (it resets its own counters), so it must not be modified by the
 *   caller afterwards, and one workspace must not be used by two calls that
 *   can run at the same time (e.g. on two streams).
 * - Co-residency: where si_single_launch(k, d, b) is 1, a call is one kernel
 *   of one block per compute unit whose blocks hand each other data while it
 *   runs, so every block must be resident at once.  The call needs every
 *   compute unit of the device to itself: a kernel running concurrently on
 *   another stream, or a CU mask that hides compute units, can keep a block
 *   from starting.  Every wait inside the kernel is bounded (on the order of
 *   a millisecond); a wait that gives up lets the call finish with wrong
 *   results and sets a sticky error word in the workspace.  From then on the
 *   single-launch calls on that workspace compute nothing and fill y with NaN
 *   until si_workspace_check() has reported the error (SI_ERR_TIMEOUT) and
 *   reset the workspace.
 */
#ifndef SPARSEINFER_H
#define SPARSEINFER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SI_OK = 0,
  SI_ERR_NULL = 1,      /* a required pointer is NULL                      */
  SI_ERR_SHAPE = 2,     /* k, d or b outside the supported range           */
  SI_ERR_ALIGN = 3,     /* a pointer is not 16-byte aligned                */
  SI_ERR_ALPHA = 4,     /* alpha is NaN or negative                        */
  SI_ERR_WORKSPACE = 5, /* workspace smaller than si_workspace_bytes()     */
  SI_ERR_HIP = 6,       /* the HIP runtime reported an error               */
  SI_ERR_FLAGS = 7,     /* unknown bits in `flags`                         */
  SI_ERR_ARG = 8,       /* another argument out of range (eps, overlapping
                           buffers)                                        */
  SI_ERR_TIMEOUT = 9,   /* a bounded wait inside a kernel gave up (blocks of
                           a single-launch call were not all resident)     */
  SI_ERR_LIST = 10      /* a caller's active_idx held a row outside [0, k) */
} si_status;

/* Flags of si_sparse_mlp / si_predict_sparse_mlp. */
#define SI_NO_AS 1u /* ignore actual sparsity (Section IV-B 3): read the W_up
                       and W_down^T rows of every predicted-active row even
                       where h1 or h3 is zero.  Results are identical; only
                       the work differs.  Used for the paper's +-AS ablation. */
#define SI_NO_SPECULATION 2u /* read W_up / W_down^T rows strictly after the
                       values that decide whether they are needed.  By default
                       the single-kernel path requests them with the W_gate
                       row for rows that are likely active: with one token,
                       the rows Eq. (2) would keep at alpha = 1 (N_neg <=
                       d/2; rows kept only because alpha > 1 wait for their
                       gate value); with 2-4 tokens, rows d/16 inside that;
                       with 5-8 tokens, every kept row.  Results are
                       identical; only the work may differ. */

/* Human-readable reason of the last non-SI_OK status on this thread. */
const char* si_last_error(void);

/* Library version string. */
const char* si_version(void);

/*
 * Size in bytes of the packed sign buffer of one W_gate (Section IV-B 1):
 * one bit per element, rows padded to a multiple of 64.  Equals k*d/8 when
 * k % 64 == 0.  Returns 0 for unsupported shapes.
 */
size_t si_signs_bytes(int k, int d);

/*
 * Pack the sign bits (MSBs) of W_gate, once at model load (Section IV-B 1).
 *   w_gate : [k][d] fp16, read.
 *   signs  : si_signs_bytes(k, d) bytes, written.  The layout is private to
 *            the library (rows interleaved for coalesced per-row counting);
 *            si_signs_to_canonical() exports it.
 */
si_status si_pack_signs(const uint16_t* w_gate, int k, int d, uint32_t* signs, void* stream);

/*
 * Export packed signs in the canonical layout of Section IV-B 1) (each row's
 * sign bits packed 32 to a word, in element order): out[i][w] (k rows of
 * d/32 uint32, written) has bit j set iff W_gate[i][32*w + j] has its sign
 * bit set.  signs: si_signs_bytes(k, d) bytes from si_pack_signs, read.
 * For tests and inspection; the decode path never calls it.
 */
si_status si_signs_to_canonical(const uint32_t* signs, int k, int d, uint32_t* out, void* stream);

/*
 * W_down^T, once at model load (Section IV-B 4): the paper's W_down is
 * [d][k]; the down-projection kernel skips whole rows of the [k][d]
 * transpose.   w_down: [d][k] fp16, read.  w_down_t: [k][d] fp16, written.
 * The two buffers must not overlap.
 */
si_status si_transpose_down(const uint16_t* w_down, int d, int k, uint16_t* w_down_t, void* stream);

/*
 * Integer form of Eq. (2).  A row is sparse iff alpha * N_pos < N_neg with
 * N_pos = d - N_neg; this returns T = the smallest N_neg in [0, d] for which
 * the row is sparse (d + 1 if none, e.g. alpha = +inf), so a row is kept
 * iff N_neg < T.  alpha is taken as its exact float32 value; ties
 * (alpha * N_pos == N_neg) are kept.  Returns -1 for NaN or negative alpha
 * or unsupported d.  Host-only; needs no GPU.
 */
int32_t si_alpha_threshold(float alpha, int d);

/* Bytes of workspace needed by si_predict / si_sparse_mlp /
 * si_predict_sparse_mlp for these shapes (0 for unsupported shapes): the
 * scratch of the prediction's outputs handed between blocks (Section IV-B
 * 2)), of the h3 values handed from the gate/up step to the down-projection
 * (Eq. (1), steps 3 and 4; Section IV-B 3), 4)), and the call counter and
 * error bits.  Host-only. */
size_t si_workspace_bytes(int k, int d, int b);

/*
 * Errors found inside kernels, which no call can return when it is made
 * (calls only enqueue work).  Waits for `stream` (NULL: the default
 * stream), then reads the workspace's sticky error word:
 *   SI_OK          : no error since the workspace was zero-filled or last
 *                    checked;
 *   SI_ERR_TIMEOUT : a bounded wait gave up (see "Co-residency" above); the
 *                    results of that call and of the single-launch calls on
 *                    this workspace since then are wrong (y is NaN);
 *   SI_ERR_LIST    : a caller's active_idx held a row outside [0, k) (the
 *                    entry was skipped).
 * On an error the whole workspace (workspace_bytes bytes) is zero-filled,
 * which restores it to its first-use state, and later calls compute again.
 * Not for use during stream capture (it synchronizes).  SI_ERR_NULL /
 * SI_ERR_ALIGN for a bad pointer, SI_ERR_HIP if the synchronization or a
 * copy fails.
 */
si_status si_workspace_check(void* workspace, size_t workspace_bytes, void* stream);

/*
 * Host-only: the status that si_workspace_check() returns for the value
 * `bits` of the sticky error word (bit 0: a wait gave up, bit 2: a list row
 * outside [0, k); a wait that gave up takes precedence).  Unknown bits give
 * SI_ERR_ARG.  Needs no GPU.
 */
si_status si_device_error_status(uint32_t bits);

/*
 * Diagnostic read-back, for tests: the per-row values h3_i,t of Eq. (1)
 * step 3 (h3 = ReLU(W_gate,i . x_t) * (W_up,i . x_t); ReLU(W_fc1,i . x_t)
 * for the non-gated MLP; with the INT8 scales applied) that the last MLP
 * call made with this workspace computed.
 *   mask : [k] uint8, the rows that call kept (nonzero = kept), read.
 *   h3   : [k][b] float32, written: the call's value for each kept row, 0 for
 *          the other rows, NaN for a kept row for which the call left no
 *          value of its own (a row it dropped).
 *   b    : the batch of that call.
 * The MLP call must be the last call made with the workspace (a later
 * si_predict replaces what it left).  Enqueued on `stream`.
 */
si_status si_read_h3(const void* workspace, size_t workspace_bytes, int k, int d, int b, const uint8_t* mask,
                     float* h3, void* stream);

/*
 * Diagnostic, outside the path: read `bytes` bytes of device memory at `buf`
 * (16-byte aligned, bytes a positive multiple of 16) once, with 16-byte
 * non-temporal loads from a grid of 8 blocks of 256 threads per compute unit.
 * The time it takes gives the streaming-read bandwidth the device achieves,
 * which the benchmark reports beside the HBM peak.  `sink` ([1] uint32) is
 * written only if the XOR of the data equals one fixed constant (so that the
 * loads cannot be dropped).  Enqueued on `stream`.
 */
si_status si_read_bandwidth_probe(const void* buf, size_t bytes, uint32_t* sink, void* stream);

/*
 * Predict the rows of W_gate whose ReLU output will be zero (Section IV-A).
 * For every token t and row i: N_neg = popcount(sign(W_gate,i) XOR
 * sign(x_t)) over the d elements, and the row is sparse for that token iff
 * alpha * (d - N_neg) < N_neg (Eq. (2)).  A row is kept (predicted active)
 * when at least one token keeps it.
 *   signs      : from si_pack_signs(), read.
 *   x          : [b][d] fp16, read.
 *   alpha      : conservativeness, >= 0 (+inf keeps every row).
 *   mask       : [k] uint8, written; 1 = kept, 0 = predicted sparse.
 *   active_idx : [k] int32, written: the kept rows in ascending order in
 *                entries 0 .. n-1 (later entries untouched).  May be NULL.
 *   n_active   : [1] int32, written with n.  May be NULL.
 *   workspace  : see the conventions above.
 */
si_status si_predict(const uint32_t* signs, int k, int d, const uint16_t* x, int b, float alpha,
                     uint8_t* mask, int32_t* active_idx, int32_t* n_active,
                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gated MLP of Eq. (1) over the kept rows (Section IV-B 3)-4)), fp32
 * accumulation.  For every kept row i and token t:
 *   g = W_gate,i . x_t ;  h1 = max(g, 0) ;  u = W_up,i . x_t (read only when
 *   some token has h1 > 0) ;  h3 = h1 * u ;  y_t += h3 * W_down^T[i, :]
 *   (row read only when some token has h3 != 0).
 *   w_gate, w_up : [k][d] fp16; w_down_t : [k][d] fp16 (si_transpose_down).
 *   x            : [b][d] fp16.
 *   mask         : [k] uint8 (nonzero = kept); used only when active_idx is
 *                  NULL, in which case the kept list is built from it.
 *   active_idx, n_active : kept rows in ascending order and their count, as
 *                  written by si_predict (device memory).  Either both or
 *                  neither may be NULL.  Each row at most once: a row listed
 *                  more than once is added to y, and counted, once per entry.
 *   y            : [b][d] float, overwritten.
 *   flags        : 0, SI_NO_AS, SI_NO_SPECULATION or both.
 *   counters     : [3] int32 or NULL: rows whose W_gate, W_up and W_down^T
 *                  rows were read (n_gate, n_up, n_down; rows requested
 *                  speculatively count as read).
 */
si_status si_sparse_mlp(const uint16_t* w_gate, const uint16_t* w_up, const uint16_t* w_down_t,
                        int k, int d, const uint16_t* x, int b, const uint8_t* mask,
                        const int32_t* active_idx, const int32_t* n_active, float* y,
                        void* workspace, size_t workspace_bytes, uint32_t flags, int32_t* counters,
                        void* stream);

/*
 * 1 if si_predict, si_sparse_mlp and si_predict_sparse_mlp (and their
 * non-gated forms), the steps of Section IV-B for one layer, run as a
 * single kernel launch for these shapes on the
 * current device: at most 256 rows of W_gate per compute unit (k <= 65536 on
 * a 256-CU MI355X) and one block with 96-160 KB of LDS resident on every
 * compute unit; 0 if they take the multi-launch path (same results) or the
 * shapes are invalid.  (si_sparse_mlp over an active_idx is a single launch up
 * to 256 rows per compute unit also where d makes the answer 0 a few rows
 * earlier.)  Host-only query.
 */
int si_single_launch(int k, int d, int b);

/*
 * The whole per-token MLP path in one call: si_predict followed by
 * si_sparse_mlp, with the same arguments and outputs (mask, active_idx,
 * n_active and counters may each be NULL).  This is the decode hot path.
 */
si_status si_predict_sparse_mlp(const uint32_t* signs, const uint16_t* w_gate, const uint16_t* w_up,
                                const uint16_t* w_down_t, int k, int d, const uint16_t* x, int b,
                                float alpha, uint8_t* mask, int32_t* active_idx, int32_t* n_active,
                                float* y, void* workspace, size_t workspace_bytes, uint32_t flags,
                                int32_t* counters, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * si_predict_sparse_mlp without a workspace argument.  Its scratch is one
 * array of 8 MiB per device inside the library (a file-scope device array,
 * held on every device the library runs on until the process ends); the
 * call allocates and frees nothing.  Arguments, outputs and errors as
 * si_predict_sparse_mlp without workspace / workspace_bytes; shapes whose
 * workspace (si_workspace_bytes(k, d, b)) exceeds 8 MiB return
 * SI_ERR_WORKSPACE (every k <= 65536 fits, at any d and b).
 * Every call on one device shares that device's array: calls that can
 * overlap on one device (two streams, two host threads) race and must not
 * be made.  Nothing needs clearing between calls: the array starts
 * zero-filled, and a call reads only words it wrote itself or that carry its
 * own call tag, whatever shapes earlier calls had.  After a bounded wait has
 * given up (see "Co-residency") the later single-launch calls of this entry
 * point on that device fill y with NaN until the process ends.
 */
si_status si_predict_sparse_mlp_noalloc(const uint32_t* signs, const uint16_t* w_gate, const uint16_t* w_up,
                                        const uint16_t* w_down_t, int k, int d, const uint16_t* x, int b,
                                        float alpha, uint8_t* mask, int32_t* active_idx, int32_t* n_active,
                                        float* y, uint32_t flags, int32_t* counters, void* stream);

/*
 * Non-gated ReLU MLP: the MLP block of models without step 2 of Section III
 * (no W_up; e.g. OPT and Falcon after ReLUfication):
 *   MLP(X) = ReLU(X W_fc1) W_down^T.
 * For every kept row i and token t: g = W_fc1,i . x_t ; h = max(g, 0) ;
 * y_t += h * W_down^T[i, :] (row read only when some token has h != 0).
 * Arguments, outputs, flags and errors as si_sparse_mlp, with w_fc1 [k][d]
 * fp16 in place of w_gate and no w_up; counters[1] (n_up) is always 0.
 * The predictor runs on the signs of W_fc1 (si_pack_signs(w_fc1)).
 */
si_status si_sparse_relu_mlp(const uint16_t* w_fc1, const uint16_t* w_down_t, int k, int d, const uint16_t* x,
                             int b, const uint8_t* mask, const int32_t* active_idx, const int32_t* n_active,
                             float* y, void* workspace, size_t workspace_bytes, uint32_t flags, int32_t* counters,
                             void* stream);

/*
 * The whole per-token path of the non-gated ReLU MLP: si_predict on the
 * signs of W_fc1 followed by si_sparse_relu_mlp, with the arguments and
 * outputs of si_predict_sparse_mlp (no w_up).
 */
si_status si_predict_sparse_relu_mlp(const uint32_t* signs, const uint16_t* w_fc1, const uint16_t* w_down_t, int k,
                                     int d, const uint16_t* x, int b, float alpha, uint8_t* mask,
                                     int32_t* active_idx, int32_t* n_active, float* y, void* workspace,
                                     size_t workspace_bytes, uint32_t flags, int32_t* counters, void* stream);

/*
 * The MLP half of a decoder layer in one launch, with the path's neighbours
 * fused: the RMSNorm that produces the MLP input (whose sign words the
 * predictor needs, Section IV-B 1) and the residual add after the
 * down-projection.  Per token t:
 *   x_t = fp16( h_t / sqrt(mean_j(h_t,j^2) + eps) * norm_w )  (in the kernel)
 *   y_t = h_t + MLP(x_t)   with MLP as in si_predict_sparse_mlp (gated), or
 *                          si_predict_sparse_relu_mlp when w_up is NULL.
 *   h      : [b][d] float32, the residual stream, read.
 *   norm_w : [d] float32, the RMSNorm weight, read.
 *   eps    : finite, >= 0.
 *   y      : [b][d] float32, overwritten; must not overlap h.
 * Other arguments, outputs and errors as si_predict_sparse_mlp.  Runs only
 * where the single-launch path applies (si_single_launch(k, d, b) == 1);
 * other shapes return SI_ERR_SHAPE.
 */
si_status si_rmsnorm_predict_sparse_mlp(const float* h, const float* norm_w, float eps, const uint32_t* signs,
                                        const uint16_t* w_gate, const uint16_t* w_up, const uint16_t* w_down_t,
                                        int k, int d, int b, float alpha, uint8_t* mask, int32_t* active_idx,
                                        int32_t* n_active, float* y, void* workspace, size_t workspace_bytes,
                                        uint32_t flags, int32_t* counters, void* stream);

/*
 * INT8 weights.  The predictor reads only the sign bit of each weight, so it
 * applies to INT8 weights unchanged (Section IV-A, robustness to the
 * quantization scheme): the MSB of a two's-complement INT8 value is its
 * sign (0 for zero).  The paper names INT8 without a scheme; these entry
 * points use symmetric INT8 with one float32 scale per output channel, each
 * weight standing for scale * q:
 *   W_gate, W_up : [k][d] int8, scales [k] (one per row);
 *   W_down       : [d][k] int8 (the paper's layout), scales [d] (one per row,
 *                  i.e. per column of y); the kernels take its transpose
 *                  W_down^T [k][d] int8 (si_transpose_down_i8) and the
 *                  same [d] scales.
 */

/*
 * Symmetric per-row quantization, once at load: for each of `rows` rows of
 * n fp16 values, scale = max_j |w_j| / 127 and q_j = rint(w_j / scale)
 * (ties to even, clamped to [-127, 127]), computed in float32 with
 * correctly rounded division; a row of zeros gets scale 0 and q = 0.
 *   w     : [rows][n] fp16, read.       q : [rows][n] int8, written.
 *   scale : [rows] float32, written.    1 <= rows, n <= 2^24 (n need not be
 *   a multiple of anything; only the base pointers must be aligned).
 */
si_status si_quantize_rows_i8(const uint16_t* w, int rows, int n, int8_t* q, float* scale, void* stream);

/*
 * Pack the sign bits (MSBs) of INT8 W_gate (or W_fc1), once at load.
 * w_gate : [k][d] int8, read.  signs : si_signs_bytes(k, d) bytes, written,
 * in the same private layout as si_pack_signs (si_signs_to_canonical
 * exports it); si_predict accepts them as they are.
 */
si_status si_pack_signs_i8(const int8_t* w_gate, int k, int d, uint32_t* signs, void* stream);

/*
 * INT8 W_down [d][k] -> W_down^T [k][d], once at load (the buffers must not
 * overlap).
 */
si_status si_transpose_down_i8(const int8_t* w_down, int d, int k, int8_t* w_down_t, void* stream);

/*
 * Eq. (1) over the rows kept by a caller's mask with INT8 weights (the INT8
 * form of si_sparse_mlp / si_sparse_relu_mlp in mask mode).  For every kept
 * row i and token t:
 *   g = s_gate[i] * (q_gate,i . x_t) ; h1 = max(g, 0) ;
 *   u = s_up[i] * (q_up,i . x_t)  (read only when some token has h1 > 0) ;
 *   h3 = h1 * u ;  y_t[j] += s_down[j] * sum_i h3_i * q_downT[i][j]
 *   (rows read only when some token has h3 != 0).
 * w_up == NULL (s_up ignored) runs the non-gated ReLU MLP (h3 = h1).
 *   mask    : [k] uint8, nonzero = kept (required).
 *   y       : [b][d] float32, overwritten.
 * Flags, counters, workspace and errors as si_sparse_mlp.  Runs where the
 * single-launch path applies (si_single_launch(k, d, b) == 1); other shapes
 * return SI_ERR_SHAPE.
 */
si_status si_sparse_mlp_i8(const int8_t* w_gate, const float* s_gate, const int8_t* w_up, const float* s_up,
                           const int8_t* w_down_t, const float* s_down, int k, int d, const uint16_t* x, int b,
                           const uint8_t* mask, float* y, void* workspace, size_t workspace_bytes, uint32_t flags,
                           int32_t* counters, void* stream);

/*
 * The whole per-token path with INT8 weights: si_predict on the signs of
 * the INT8 W_gate (si_pack_signs_i8) followed by si_sparse_mlp_i8 over the
 * predicted rows, in one launch, with the arguments and outputs of
 * si_predict_sparse_mlp (mask, active_idx, n_active and counters may each be
 * NULL; w_up == NULL: the non-gated ReLU MLP).  Runs where the
 * single-launch path applies; other shapes return SI_ERR_SHAPE.
 */
si_status si_predict_sparse_mlp_i8(const uint32_t* signs, const int8_t* w_gate, const float* s_gate,
                                   const int8_t* w_up, const float* s_up, const int8_t* w_down_t,
                                   const float* s_down, int k, int d, const uint16_t* x, int b, float alpha,
                                   uint8_t* mask, int32_t* active_idx, int32_t* n_active, float* y,
                                   void* workspace, size_t workspace_bytes, uint32_t flags, int32_t* counters,
                                   void* stream);

/*
 * MXFP4 weights: 4-bit floating point with a scale for every 32 values.  A row
 * of n values is stored as np = 128 ceil(n / 128) of them (zeros behind the
 * n-th):
 *   codes  : [rows][np / 2] uint8, two 4-bit codes a byte, value 2 j in the low
 *            half of byte j.  A code is a sign bit (8) and one of
 *            0, 0.5, 1, 1.5, 2, 3, 4, 6 (0 .. 7).
 *   scales : [rows][np / 32] uint8, X + 127 for a scale of 2^X; 255 is NaN.
 * A value is its code times the scale of its 32.
 */

/* Element types of the calls that take more than one. */
typedef enum { SI_F16 = 0, SI_BF16 = 1, SI_F32 = 2 } si_dtype;

/* Bytes of the codes and of the scales of `rows` rows of n values (0 for
 * rows outside [0, 2^24] or n outside [1, 2^24]).  Host-only. */
size_t si_mxfp4_codes_bytes(int rows, int n);
size_t si_mxfp4_scales_bytes(int rows, int n);

/*
 * Rows to MXFP4: weights once at load, activations in front of a product with
 * _a4.  For each 32 values v of a row (the last ones padded with zeros), with m
 * the largest |v|:
 *   X = floor(log2 m) - 2, at least -127; the code of v is the nearest to
 *   v / 2^X, ties to the even code, 6 where |v| / 2^X > 6, with v's sign (that
 *   of zeros too).
 * m = 0 gives the scale byte 0; a block with an infinity or a NaN the byte 255
 * and codes of signs alone, so that it reads back as NaN.
 *   w     : rows of n values of type w_dtype, ldw elements from row to row
 *           (n to 2^32 where rows > 1), at any address that fits an element.
 *   q, scale : written, si_mxfp4_codes_bytes / si_mxfp4_scales_bytes.
 *   rows  : 0 to 2^24 (0 does nothing); n: 1 to 2^24, any length.
 */
si_status si_quantize_rows_mxfp4(const void* w, int w_dtype, size_t ldw, int rows, int n, uint8_t* q, uint8_t* scale,
                                 void* stream);

/* MXFP4 rows as values: w [rows][n] of type w_dtype (rounded to nearest even
 * where the type cannot hold a value; exact in bf16 and float32 down to
 * 2^-126, and in fp16 for rows quantized from fp16). */
si_status si_dequantize_rows_mxfp4(const uint8_t* q, const uint8_t* scale, int rows, int n, void* w, int w_dtype,
                                   void* stream);

/*
 * Packed signs of MXFP4 W_gate (or W_fc1) codes [k][d / 2], once at load, in
 * the layout of si_pack_signs: si_predict accepts them as they are.  They are
 * the signs of the values that were quantized.
 */
si_status si_pack_signs_mxfp4(const uint8_t* q_gate, int k, int d, uint32_t* signs, void* stream);

/*
 * Products with MXFP4 weights, for prompts and for tokens whose rows are not
 * predicted, float32 accumulation on the matrix cores:
 *   si_linear_mxfp4       : y[t][i] = sum_j x[t][j] W[i][j]
 *   si_gated_linear_mxfp4 : h[t][i] = max(sum_j x[t][j] W_gate[i][j], 0) *
 *                           (sum_j x[t][j] W_up[i][j]), Eq. (1) steps 1-3 over
 *                           every row; q_up = s_up = NULL: the non-gated
 *                           max(sum_j x[t][j] W_fc1[i][j], 0).
 *   x  : m rows of n values, fp16 or bf16 (x_dtype), ldx elements from row to
 *        row (n to 2^21 where m > 1), at any address that fits an element.
 *        With fp16 activations the weights take part as their fp16 values (the
 *        values themselves for weights quantized from fp16; beyond fp16's range
 *        infinities, and multiples of 2^-24 below its normal numbers); with bf16
 *        as they are.
 *   q, scale : W's [rows] rows of n values in MXFP4.
 *   y (h)    : [m][rows] of type y_dtype, written.
 *   m 0 to 2^24 (0 does nothing), rows 1 to 2^24, n 1 to 2^20; SI_ERR_SHAPE too
 *   where a launch would exceed 2^32 threads.
 *   workspace: si_linear_mxfp4_workspace_bytes() bytes of scratch (may be NULL
 *        where that is 0); nothing is kept in it from one call to the next, and
 *        two calls that can run at the same time need one each.
 * The _a4 forms take the activations in MXFP4 as well (xq, x_scale from
 * si_quantize_rows_mxfp4): products of 4-bit values with both scales, on the
 * matrix cores' own 4-bit instructions.
 * The sums' order depends on the shapes alone: the same call gives the same bits.
 */
si_status si_linear_mxfp4(const void* x, int x_dtype, size_t ldx, int m, int n, const uint8_t* q, const uint8_t* scale,
                          int rows, void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* stream);
si_status si_gated_linear_mxfp4(const void* x, int x_dtype, size_t ldx, int m, int n, const uint8_t* q_gate,
                                const uint8_t* s_gate, const uint8_t* q_up, const uint8_t* s_up, int rows, void* h,
                                int h_dtype, void* workspace, size_t workspace_bytes, void* stream);
si_status si_linear_mxfp4_a4(const uint8_t* xq, const uint8_t* x_scale, int m, int n, const uint8_t* q,
                             const uint8_t* scale, int rows, void* y, int y_dtype, void* workspace,
                             size_t workspace_bytes, void* stream);
si_status si_gated_linear_mxfp4_a4(const uint8_t* xq, const uint8_t* x_scale, int m, int n, const uint8_t* q_gate,
                                   const uint8_t* s_gate, const uint8_t* q_up, const uint8_t* s_up, int rows, void* h,
                                   int h_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace of the four products (`gated` nonzero: with W_up; x NULL:
 * the _a4 forms).  Of x only the alignment counts, with ldx: activations that
 * cannot be read in 16-byte pieces are copied into the workspace.  0 for
 * unsupported shapes and where none is needed.  Host-only. */
size_t si_linear_mxfp4_workspace_bytes(const void* x, size_t ldx, int m, int rows, int n, int gated);

/*
 * Diagnostic, host-only: which kernel a product of these sizes takes (`a4`
 * nonzero: one of the _a4 forms; `gated` as above).  -1: the one for a few tokens
 * and rows; 0 and up: the place of its tile in the library's list for that kind of
 * activations, smallest first; -2: a shape that the product refuses, or m = 0.
 */
int si_linear_mxfp4_tile(int a4, int m, int rows, int n, int gated);

/* Bytes of the workspace of the two calls below (0 for unsupported shapes): a
 * si_workspace_bytes() workspace, under the same rules (zero-filled before its
 * first use, one call at a time), which fp16, INT8 and MXFP4 calls may share;
 * si_read_h3 and si_workspace_check accept it. */
size_t si_mxfp4_workspace_bytes(int k, int d, int b);

/*
 * The MXFP4 forms of si_sparse_mlp (mask mode) and si_predict_sparse_mlp, with
 * their arguments, flags, counters and outputs, for every supported shape:
 *   q_gate, s_gate, q_up, s_up : W_gate, W_up [k] rows of d values in MXFP4
 *        (q_up = s_up = NULL: the non-gated ReLU MLP);
 *   q_down_t, s_down_t : W_down^T, [k] rows of d values in MXFP4 (transposed
 *        first, then quantized: a scale covers 32 columns of y).
 * Two launches, which do not need the device to themselves; y is the same bits
 * in every run.  x and y must not overlap.  A kept row whose gate value is NaN
 * makes y NaN.
 */
si_status si_sparse_mlp_mxfp4(const uint8_t* q_gate, const uint8_t* s_gate, const uint8_t* q_up, const uint8_t* s_up,
                              const uint8_t* q_down_t, const uint8_t* s_down_t, int k, int d, const uint16_t* x, int b,
                              const uint8_t* mask, float* y, void* workspace, size_t workspace_bytes, uint32_t flags,
                              int32_t* counters, void* stream);
si_status si_predict_sparse_mlp_mxfp4(const uint32_t* signs, const uint8_t* q_gate, const uint8_t* s_gate,
                                      const uint8_t* q_up, const uint8_t* s_up, const uint8_t* q_down_t,
                                      const uint8_t* s_down_t, int k, int d, const uint16_t* x, int b, float alpha,
                                      uint8_t* mask, int32_t* active_idx, int32_t* n_active, float* y, void* workspace,
                                      size_t workspace_bytes, uint32_t flags, int32_t* counters, void* stream);

/*
 * What stands between the products of two blocks, in one pass over each token:
 *   P  = RMSNorm(branch) * post_w, or branch itself where post_w is NULL
 *   h' = h + scale * gate * P       (gate NULL: 1; branch NULL: h' = h)
 *   x  = RMSNorm(h') * pre_w        (of h' before it is rounded to h_out's type)
 * with RMSNorm(v) = v / sqrt(mean(v^2) + eps), in float32.
 *   h, h_out : tokens rows of d values of type h_dtype, ldh and ldo elements
 *        from row to row; h_out is written and may be h itself, or NULL.
 *   branch   : rows of type branch_dtype, ldb; NULL (with post_w, gate and h_out
 *        NULL): only x is formed.
 *   post_w, pre_w : [d] float32; pre_w and x both given or both NULL.
 *   gate     : [ceil(tokens / rows_per_gate)][d] float32: token t is multiplied
 *        with row t / rows_per_gate (rows_per_gate = tokens: one gate for all).
 *   x        : rows of type x_dtype, ldx, written.
 *   tokens 0 to 2^23 - 1 (0 does nothing), d 1 to 16384, strides d to 2^32
 *   where tokens > 1, addresses that fit an element.  At least one of h_out and x.
 *   Outputs must not overlap anything else (columns of one matrix do not).
 */
si_status si_norm_residual(const void* h, int h_dtype, size_t ldh, const void* branch, int branch_dtype, size_t ldb,
                           const float* post_w, const float* gate, int rows_per_gate, float scale, void* h_out,
                           size_t ldo, const float* pre_w, void* x, int x_dtype, size_t ldx, int tokens, int d,
                           float eps, void* stream);

/*
 * The dense MLP outside decode: products over every row of fp16 or bf16 weights
 * (`dtype`, the type of x and W and of their gradients), float32 accumulation on
 * the matrix cores, with their gradients.
 *   si_linear       : y[t][i] = sum_j x[t][j] W[i][j]
 *   si_gated_linear : h[t][i] = max(g, 0) * u with g = sum_j x[t][j] W_gate[i][j] and
 *                     u = sum_j x[t][j] W_up[i][j], Eq. (1) steps 1-3 over every row
 *                     in one launch; w_up NULL: the non-gated max(g, 0).
 *   x   : m rows of n values, ldx elements from row to row (n to 2^21 where m > 1),
 *         at any address that fits an element.
 *   w   : [rows][n], at any address that fits an element; with w_transposed nonzero
 *         W^T, [n][rows] (what si_transpose_down makes of W_down: y = h W_down^T).
 *   y, h: [m][rows] of type y_dtype / h_dtype, written.
 *   g, u: both or neither: the two sums themselves, [m][rows] in float32, for the
 *         backward pass.  With w_up only.
 *   m 0 to 2^24 (0 does nothing), rows and n 1 to 2^20; m times rows, m times n and
 *         rows times n below 2^35, and few enough blocks for one launch (else
 *         SI_ERR_SHAPE).
 *   workspace: the ..._workspace_bytes() of the call: scratch for split sums and for
 *         copies of operands that cannot be read in 16-byte pieces (rows of a multiple
 *         of 8 values that start on 16 bytes can).  Nothing is kept in it from one call
 *         to the next; two calls that can run at the same time need one each.
 * The sums' order depends on the shapes and addresses' alignment alone: the same call
 * gives the same bits.
 */
si_status si_linear(const void* x, int dtype, size_t ldx, int m, int n, const void* w, int rows, int w_transposed,
                    void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* stream);
si_status si_gated_linear(const void* x, int dtype, size_t ldx, int m, int n, const void* w_gate, const void* w_up,
                          int rows, void* h, int h_dtype, float* g, float* u, void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * Their gradients, for a loss whose derivatives with respect to y (h) are dy (dh):
 *   si_linear_backward       : dx = dy W,  dw = dy^T x (in w's layout)
 *   si_gated_linear_backward : dg = dh u where g > 0, else 0;  du = dh max(g, 0);
 *                              dx = dg W_gate + du W_up,  dw_gate = dg^T x,
 *                              dw_up = du^T x
 *   si_mlp_backward          : of the whole MLP, y = h W_down^T with W_down [d][k]: dh =
 *                              dy W_down (float32, not stored), dw_down = dy^T h, and the
 *                              gradients of si_gated_linear for n = d and rows = k
 *   dy  : m rows of type dtype or float32, lddy elements from row to row; dh of any
 *         type.  dy (as an operand of the products), dg and du are rounded to dtype.
 *   g, u: as si_gated_linear kept them (g_dtype SI_F32).  w_up NULL: u NULL, and g is its
 *         output h, [m][rows] of type g_dtype (si_mlp_backward: g NULL); where that was
 *         rounded to 0 the gradient is 0.
 *   h   : [m][k] of type dtype, si_gated_linear's output.
 *   g, u and h on 16 bytes.
 *   dx, dw, dw_gate, dw_up, dw_down: [m][n] and the weights' shapes, of type dtype,
 *         written; each may be NULL (all of them with m = 0 alone).  With m = 0 the
 *         weights' gradients are zeros.
 *   workspace: ..._workspace_bytes() of the call; want_dx, want_dw (of either of w_gate
 *         and w_up) and want_dw_down say which of the gradients are not NULL.
 */
si_status si_linear_backward(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int n,
                             const void* w, int rows, int w_transposed, void* dx, void* dw, void* workspace,
                             size_t workspace_bytes, void* stream);
si_status si_gated_linear_backward(const void* dh, int dh_dtype, size_t lddh, const void* g, int g_dtype, const float* u,
                                   const void* x, int dtype, size_t ldx, int m, int n, const void* w_gate,
                                   const void* w_up, int rows, void* dx, void* dw_gate, void* dw_up, void* workspace,
                                   size_t workspace_bytes, void* stream);
si_status si_mlp_backward(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int d,
                          const void* w_gate, const void* w_up, const void* w_down, int k, const void* h, const float* g,
                          const float* u, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Bytes of workspace of the five calls above (0 for unsupported shapes and where none
 * is needed).  Of the operands only alignment, and of w_up the presence, counts.
 * Host-only. */
size_t si_linear_workspace_bytes(const void* x, size_t ldx, int m, int n, const void* w, int rows, int w_transposed);
size_t si_gated_linear_workspace_bytes(const void* x, size_t ldx, int m, int n, const void* w_gate, const void* w_up,
                                       int rows);
size_t si_linear_backward_workspace_bytes(const void* dy, int dy_dtype, size_t lddy, const void* x, size_t ldx, int m,
                                          int n, const void* w, int rows, int w_transposed, int want_dx, int want_dw);
size_t si_gated_linear_backward_workspace_bytes(const void* x, size_t ldx, int m, int n, const void* w_gate,
                                                const void* w_up, int rows, int want_dx, int want_dw);
size_t si_mlp_backward_workspace_bytes(const void* dy, int dy_dtype, size_t lddy, const void* x, size_t ldx, int m, int d,
                                       const void* w_gate, const void* w_up, const void* w_down, int k, int want_dx,
                                       int want_dw, int want_dw_down);

/*
 * Diagnostic, host-only: which kernel a dense product of these sizes takes.  kind 0:
 * si_linear (1: with W^T) or si_gated_linear; 2: the gradient with respect to x (3: with
 * W^T); 4: with respect to W (5: with W^T); 6: the FP8 products.  gated nonzero: with
 * W_up.  (si_mlp_backward: dh 1 and dw_down 5, of rows k and n d, the rest 2 and 4.)  100: the one for a few tokens; 0 and up: the place of its tile in the library's
 * list, smallest first; -2: sizes that the product refuses, or m = 0.
 */
int si_dense_tile(int kind, int m, int rows, int n, int gated);

/*
 * FP8 weights: e4m3 values (sign, 4 bits of exponent, 3 of fraction; largest 448, no
 * infinities) with float32 scales.  A row of n values is stored as n rounded up to
 * 16 codes (zeros behind the n-th); a value is its code times its scale:
 *   tokens  : a scale for each 128 values of a row, [rows][ceil(n / 128)];
 *   weights : one for each 128 x 128 block, [ceil(rows / 128)][ceil(n / 128)].
 */

/* Bytes of the codes, and of the scales of tokens and of weights (0 for rows outside
 * [0, 2^24] or n outside [1, 2^24]).  Host-only. */
size_t si_fp8_codes_bytes(int rows, int n);
size_t si_fp8_scales_bytes(int rows, int n);
size_t si_fp8_block_scales_bytes(int rows, int n);

/*
 * Rows (tokens) and blocks (weights, once at load) to FP8.  With m the largest |v| of
 * a block: scale = m * (1 / 448), the code of v is the e4m3 value nearest to v / scale,
 * ties to the even code; 1 / 448, the product and the quotient are each rounded to
 * float32.  A scale of 0 (m = 0, or so small that the product is 0) has codes 0; a block with an infinity or
 * a NaN the scale NaN and codes 0, so that it reads back as NaN.
 *   x (w) : rows of n values of type x_dtype, ldx elements from row to row (n to 2^32
 *           where rows > 1), at any address that fits an element.
 *   rows 0 to 2^24 (0 does nothing), n 1 to 2^24.
 */
si_status si_quantize_rows_fp8(const void* x, int x_dtype, size_t ldx, int rows, int n, uint8_t* q, float* scale,
                               void* stream);
si_status si_quantize_blocks_fp8(const void* w, int w_dtype, size_t ldw, int rows, int n, uint8_t* q, float* scale,
                                 void* stream);

/* FP8 rows as values: w [rows][n] of type w_dtype; rows_per_scale 1 (tokens) or 128
 * (weights). */
si_status si_dequantize_fp8(const uint8_t* q, const float* scale, int rows_per_scale, int rows, int n, void* w, int w_dtype,
                            void* stream);

/*
 * si_linear and si_gated_linear with FP8 weights (q, scale from si_quantize_blocks_fp8,
 * or a checkpoint's of that form) and FP8 tokens (xq, x_scale from
 * si_quantize_rows_fp8): the products of 128 codes are summed in float32 on the matrix
 * cores, then multiplied with both scales and added in float32.
 *   y (h) : [m][rows] of type y_dtype, written.  Sizes as si_linear.
 *   workspace: si_linear_fp8_workspace_bytes() bytes (gated nonzero: with q_up).
 */
si_status si_linear_fp8(const uint8_t* xq, const float* x_scale, int m, int n, const uint8_t* q, const float* scale,
                        int rows, void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* stream);
si_status si_gated_linear_fp8(const uint8_t* xq, const float* x_scale, int m, int n, const uint8_t* q_gate,
                              const float* s_gate, const uint8_t* q_up, const float* s_up, int rows, void* h, int h_dtype,
                              void* workspace, size_t workspace_bytes, void* stream);
size_t si_linear_fp8_workspace_bytes(int m, int rows, int n, int gated);

/*
 * LayerNorm (center nonzero) and RMSNorm (0) with their gradients, in float32:
 *   c = x - mean(x), or x;  r = 1 / sqrt(mean(c^2) + eps);  y = c r w + b
 *   with n = c r and e = dy w:  dx = r (e - mean(e) - n mean(e n))  (mean(e) with
 *   center alone),  dw = sum over tokens of dy n,  db = sum over tokens of dy.
 *   x, dy   : tokens rows of d values of type dtype, ldx and lddy elements from row to
 *             row (to 2^32 where tokens > 1).     y, dx : [tokens][d] of that type.
 *   w, b    : [d] of type w_dtype, as dw and db; b may be NULL.
 *   mean, rstd : [tokens] float32, the means and r of the rows, written by the forward
 *             pass where given (mean with center alone), read by the backward pass.
 *   dx, dw, db : written; each may be NULL (all of them with tokens = 0 alone).  With
 *             tokens = 0 dw and db are zeros.
 *   tokens 0 to 2^23 - 1, d 1 to 16384, addresses that fit an element.
 *   workspace: si_layer_norm_backward_workspace_bytes(), where dw or db is given.
 * The gradients' sums are taken in an order that depends on the sizes alone.
 */
si_status si_layer_norm(const void* x, int dtype, size_t ldx, const void* w, const void* b, int w_dtype, int center,
                        float eps, void* y, float* mean, float* rstd, int tokens, int d, void* stream);
si_status si_layer_norm_backward(const void* dy, size_t lddy, const void* x, int dtype, size_t ldx, const void* w,
                                 int w_dtype, int center, const float* mean, const float* rstd, void* dx, void* dw, void* db,
                                 int tokens, int d, void* workspace, size_t workspace_bytes, void* stream);
size_t si_layer_norm_backward_workspace_bytes(int tokens, int d);

#ifdef __cplusplus
}
#endif

#endif /* SPARSEINFER_H */
