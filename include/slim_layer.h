/*
 * libslim -- the rest of a language model's layer around the sliced attention,
 * on one NVIDIA GB300 (sm_103a):
 *
 *   slim_qk_norm_*     the root-mean-square norm of queries and keys per head
 *                      and their rotation by position, in one pass from a
 *                      projection's rows to the [B, H, L, d] that slim_fwd takes
 *   slim_gated_scan_*  a gated linear recurrence per channel, the sibling of the
 *                      attention's prefix state that forgets, with the same
 *                      carries in and out of a segment
 *   slim_gated_ff_*    the gated feed-forward's two projections, activation and
 *                      product in one kernel, and its gradients
 *
 * The conventions of slim.h hold: device pointers, every buffer owned by the
 * caller, arguments validated before anything is enqueued, all work on
 * `stream`, no synchronisation; host arrays are read during the call.
 * Workspaces are 256-byte aligned.  Results do not depend on the order in which
 * blocks run: two calls on the same inputs agree bit for bit.
 *
 * The gated feed-forward has device-side waits (its tile kernels'), and so has the
 * recurrence where it has a workspace; they are bounded and reported like those of
 * the vocabulary loss: the next slim_gated_ff_* or slim_gated_scan_* call on the same
 * workspace returns SLIM_ERR_TIMEOUT, and slim_check_device_error reads the failure
 * by blocking.  The other entry points have none.
 */
#ifndef SLIM_LAYER_H_
#define SLIM_LAYER_H_

#include "slim_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element strides of a [B, H, L, d] tensor whose last dimension is contiguous. */
typedef struct {
  long long b, h, l;
} slim_strides;

/*
 * Queries and keys of a layer, per token and head:
 *     y = scale * x / sqrt(mean(x^2) + eps) * weight
 * and then the first `rotary` features of y turned in pairs by the angle
 * position * inv_freq[p], (a, b) -> (a cos - b sin, a sin + b cos): pair p is
 * the features (p, p + rotary/2), or (2p, 2p + 1) with `interleaved`.
 *   q [B, Hq, L, d], k [B, Hk, L, d] dtype, with the given strides (null:
 *   contiguous), aligned to their element size; slices of a projection's rows
 *   are read where they are, in pieces of up to 16 bytes where pointers and strides
 *   allow it.  Hk = 0: no keys (k, k_out and k_weight are not read).
 *   q_weight, k_weight  [d] fp32, or null (1).
 *   positions  [B, L] ptype, any value, aligned to its own size; null: l.
 *   inv_freq   HOST array of rotary/2 finite numbers, radians per position.
 *              Angles are kept as 64-bit fractions of a turn: far positions lose
 *              nothing but the frequencies' own 53 bits.
 *   q_out, k_out  as q and k, no two elements in one place.  They may be q and k
 *              themselves, with the same strides.
 * Sums and turns are fp32, y is rounded once.  A row of zeros stays zero; a row
 * whose squares pass fp32's range is normalised all the same; a row that holds a
 * NaN becomes NaN; of a row that holds an infinity, that feature and the other of its
 * pair become NaN and the rest zero (its gradient is NaN); no other row changes.
 * 0 <= B, L and B L < 2^31 - 16; Hq >= 1; Hq, Hk <= 4096; 1 <= d <= 256; rotary even,
 * 0 <= rotary <= d; 0 < eps <= 1e38; B L (Hq + Hk) <= 2^40; strides in [0, 2^40],
 * offsets below 2^60.  B L = 0 enqueues nothing.
 */
slim_status slim_qk_norm_fwd(const void* q, const slim_strides* q_strides, const void* k,
                             const slim_strides* k_strides, const float* q_weight,
                             const float* k_weight, const void* positions, slim_index ptype,
                             const double* inv_freq, int rotary, int interleaved, int B, int Hq,
                             int Hk, int L, int d, slim_dtype dtype, float eps, float scale,
                             void* q_out, const slim_strides* q_out_strides, void* k_out,
                             const slim_strides* k_out_strides, void* stream);

/*
 * The gradients of <dq_out, q_out> + <dk_out, k_out> with respect to q, k and
 * the weights.  q, k and what follows as in the forward; nothing is kept from
 * it: the norms are computed again.
 *   dq_out, dk_out  as q and k, with strides of their own.
 *   dq, dk          written, with strides of their own; they may be dq_out and
 *                   dk_out themselves, with the same strides.
 *   dq_weight, dk_weight  [d] fp32, written; null: not wanted.  Sums are fp32,
 *                   by blocks and then over blocks in order.  B L = 0 zeroes them.
 *   workspace of slim_qk_norm_bwd_workspace_size() bytes.
 */
slim_status slim_qk_norm_bwd_workspace_size(int B, int Hq, int Hk, int L, int d, size_t* bytes);
slim_status slim_qk_norm_bwd(const void* q, const slim_strides* q_strides, const void* k,
                             const slim_strides* k_strides, const float* q_weight,
                             const float* k_weight, const void* positions, slim_index ptype,
                             const double* inv_freq, int rotary, int interleaved, int B, int Hq,
                             int Hk, int L, int d, slim_dtype dtype, float eps, float scale,
                             const void* dq_out, const slim_strides* dq_out_strides,
                             const void* dk_out, const slim_strides* dk_out_strides, void* dq,
                             const slim_strides* dq_strides, void* dk,
                             const slim_strides* dk_strides, float* dq_weight, float* dk_weight,
                             void* workspace, size_t workspace_bytes, void* stream);

/* How a gate g and an input x make a step h_t = a_t h_(t-1) + u_t. */
typedef enum {
  SLIM_GATE_VALUE = 0,  /* a = g,          u = x */
  SLIM_GATE_LOG = 1,    /* a = exp(g),     u = x */
  SLIM_GATE_SIGMOID = 2 /* a = sigmoid(g), u = (1 - a) x = sigmoid(-g) x */
} slim_gate;

/* Steps between the states that a forward keeps for its backward. */
#define SLIM_SCAN_CHUNK 64

/*
 * h_t = a_t h_(t-1) + u_t for every channel of every sequence, from h_0.
 *   gate, x  [B, L, D] dtype: element (b, t, c) at ((b L + t) pitch + c), aligned
 *            to their element size; pitch > D reads a slice of a projection's
 *            rows, pitch 0 one row for all.
 *   h0       [B, D] fp32, or null (zero): a segment starts from the last state of
 *            the one before.
 *   h        [B, L, D] dtype, written.
 *   last     [B, D] fp32, written (the state after the last step), or null; it may
 *            be h0 itself.
 *   kept     [B, ceil(L / SLIM_SCAN_CHUNK), D] fp32, written (the state before each
 *            chunk), or null: what slim_gated_scan_bwd reads.
 * States and sums are fp32, h is rounded once.  A gate near 1, which a state meets many
 * times over, is rounded once: LOG gates within 2^-3 of zero (bf16 2^-6), and the larger
 * of sigmoid(g) and sigmoid(-g).  The others are off by up to 2^-21 of themselves (bf16:
 * and by 1.25 |g| 2^-24), and below 2^-126 they are zero.  A gate of zero (VALUE 0, LOG
 * or SIGMOID -inf) starts anew: nothing before it reaches h, finite or not.  A state that
 * is not finite stays in its channel until such a gate, or until the gates' product since
 * sinks below fp32's range.  Gates are finite, and LOG gates' exponentials, but for those
 * infinities.  Beyond 1 they may grow a state past fp32's range; so may the product of up
 * to 128 of them alone: a state that is not zero is then not finite until such a gate
 * (backward, a gradient before them), one of zero stays zero.
 * Nothing written overlaps anything else but as said.
 *   workspace of slim_gated_scan_workspace_size() bytes, for either direction; where
 *   that is 0 (short sequences, few of them) it is not used and may be null.
 * 0 <= B, 0 <= L <= 2^30, 1 <= D <= 2^30, B D <= 2^32, B L D <= 2^40,
 * D <= pitch (0 <= pitch for inputs) <= 2^40, offsets below 2^60.  With B L = 0 the
 * state is passed on.
 */
slim_status slim_gated_scan_workspace_size(int B, int L, int D, slim_dtype dtype, size_t* bytes);
slim_status slim_gated_scan_fwd(const void* gate, long long gate_pitch, const void* x,
                                long long x_pitch, const float* h0, int B, int L, int D,
                                slim_dtype dtype, slim_gate kind, void* h, float* last, float* kept,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradients of <dh, h> + <dlast, last> with respect to gate, x and h0.
 *   kept     from the forward on the same gate, x and h0; the states inside a chunk
 *            are computed again from it, in fp32.
 *   dh       [B, L, D] dtype;  dlast [B, D] fp32, or null (zero).
 *   dgate, dx  [B, L, D] dtype with pitches of their own, written; they may be gate
 *            and x themselves, with the same pitches.
 *   dh0      [B, D] fp32, written, or null; it may be dlast itself.
 * Where a step starts anew its LOG or SIGMOID gate has gradient 0.
 */
slim_status slim_gated_scan_bwd(const void* gate, long long gate_pitch, const void* x,
                                long long x_pitch, const float* kept, const void* dh,
                                const float* dlast, int B, int L, int D, slim_dtype dtype,
                                slim_gate kind, void* dgate, long long dgate_pitch, void* dx,
                                long long dx_pitch, float* dh0, void* workspace,
                                size_t workspace_bytes, void* stream);

/*
 * Diagnostic: slim_gated_scan_fwd of one sequence (fp32, LOG, rows one behind the other)
 * whose tiles look back through the workspace, but whose first tile nobody runs.  The wait
 * for its state gives up after its limit (about a second), the kernel ends, and the failure
 * is reported as above.  h holds nothing of use.  Sizes that need no waits are refused.
 */
slim_status slim_diag_gated_scan_wait(const float* gate, const float* x, int L, int D, float* h,
                                      void* workspace, size_t workspace_bytes, void* stream);

/* The activation of a gate. */
typedef enum {
  SLIM_ACT_SILU = 0,      /* g sigmoid(g) */
  SLIM_ACT_GELU = 1,      /* g Phi(g), Phi the normal distribution's */
  SLIM_ACT_GELU_TANH = 2, /* g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2 */
  SLIM_ACT_RELU = 3,      /* max(g, 0) */
  SLIM_ACT_SIGMOID = 4    /* sigmoid(g) */
} slim_act;

/*
 * h = act(x w_gate^T) * (x w_up^T), elementwise: what the last projection of a
 * gated feed-forward reads.
 *   x  [N, D] dtype;  w [2F, D] dtype: w_gate the first F rows, w_up the others;
 *   h  [N, F] dtype, written.  16-byte aligned.
 *   kept  written, or null: both projections, x w^T, [N, 2 F'] fp32, F' being F
 *         rounded up to 16 (columns past F hold anything), 32-byte aligned; only
 *         where slim_gated_ff_kept_size says more than 0 (fp32, from 9 rows on):
 *         there the backward reads them sooner than it computes them again.
 * Without kept, neither projection is written.  bf16 operands are multiplied exactly and summed
 * in fp32; fp32 operands are split into three bf16 pieces (24 bits) and multiplied
 * piece by piece, six products each, smallest first, on the tensor cores (up to 8
 * rows, where that is quicker: fp32 FMA in either type).  h is rounded once.
 * Values are finite: an infinity in a row of x, or of w, makes what it enters
 * infinite or NaN.  Nothing written overlaps anything else, in either direction.
 * 0 <= N < 2^31 - 512, 1 <= D <= 2^30, 1 <= F <= 2^29, N F <= 2^45, N D and 2 F D
 * <= 2^40.  N = 0 enqueues nothing.
 *   workspace of slim_gated_ff_workspace_size(..., backward = 0) bytes; where that is
 *   0 (a few rows) it may be null.
 */
slim_status slim_gated_ff_workspace_size(long long N, int D, int F, slim_dtype dtype, int backward,
                                         size_t* bytes);
slim_status slim_gated_ff_kept_size(long long N, int D, int F, slim_dtype dtype, size_t* bytes);
slim_status slim_gated_ff_fwd(const void* x, const void* w, long long N, int D, int F,
                              slim_dtype dtype, slim_act act, void* h, float* kept,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradients of <dh, h> with respect to x and w.
 *   dh  [N, F] dtype;  dx [N, D] dtype, dw [2F, D] dtype, written.  16-byte aligned.
 *   kept  from the forward on the same x and w, or null.
 * With g and u the projections, from kept or computed again here,
 *     dz = [dh u act'(g), dh act(g)],   dx = dz w,   dw = dz^T x.
 * dz is rounded once for the products: to bf16 for bf16 problems (by up to 2^-8 of
 * itself, as the gradients themselves are), to three bf16 pieces for fp32
 * ones; the workspace holds it (2 N F elements of 2 or 6 bytes).  Sums are fp32, and
 * long ones are joined from parts; dx and dw are rounded once.  N = 0 zeroes dw.
 */
slim_status slim_gated_ff_bwd(const void* x, const void* w, const void* dh, long long N, int D,
                              int F, slim_dtype dtype, slim_act act, const float* kept, void* dx,
                              void* dw, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SLIM_LAYER_H_ */
