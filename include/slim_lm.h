/*
 * libslim -- the two ends of a language model around the attention stack, and
 * the guard of its training step, on one NVIDIA GB300 (sm_103a):
 *
 *   slim_embed_*       embedding lookup with scaling, and its gradient
 *   slim_vocab_loss_*  softmax cross entropy over a vocabulary, evaluated in
 *                      pieces of the vocabulary without keeping the logits,
 *                      and its gradients
 *   slim_clip_grads    the global norm of many gradients, and their clipping
 *
 * The conventions of slim.h hold: device pointers, contiguous row-major
 * tensors, every buffer owned by the caller, arguments validated before
 * anything is enqueued, all work on `stream`, no synchronisation.  Tensors are
 * 16-byte aligned unless their line below says otherwise; workspaces are
 * 256-byte aligned.  Results do not depend on the order in which blocks run:
 * two calls on the same inputs agree bit for bit.
 *
 * The vocabulary loss has device-side waits (its tile kernels'); they are bounded
 * and reported like those of slim_fwd: the next slim_vocab_loss_* call on the same
 * workspace returns SLIM_ERR_TIMEOUT, and slim_check_device_error reads the
 * failure by blocking.  The other entry points have none.
 */
#ifndef SLIM_LM_H_
#define SLIM_LM_H_

#include "slim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of token ids and targets. */
typedef enum { SLIM_I32 = 0, SLIM_I64 = 1 } slim_index;

/*
 * out_i = scale * table[ids_i], computed in fp32 and rounded to nearest even.
 *   ids    [N] itype, aligned to its own size.  An id outside [0, V) marks
 *          padding: its row of out is zero.
 *   table  [V, D] dtype;  out [N, D] dtype.
 * 0 <= N < 2^31, 1 <= D <= 2^30, V >= 1, N D and V D <= 2^42.  N = 0 enqueues
 * nothing.
 */
slim_status slim_embed_fwd(const void* ids, slim_index itype, const void* table, long long N,
                           int D, int V, slim_dtype dtype, float scale, void* out, void* stream);

/*
 * The gradient with respect to the table:
 *     dtable_v = scale * sum over {i : ids_i = v} of dout_i.
 * The tokens are sorted by id (stably), and each row's sum is taken in fp32
 * over its tokens in order of position, in fixed groups: no atomics, the same
 * bits from call to call.  Rounded once, at the end.
 *   dout    [N, D] dtype;  dtable [V, D] dtype.
 *   accumulate = 0: dtable is written, rows without a token as zero.
 *   accumulate = 1: the gradient is added to dtable (in fp32, rounded once);
 *           rows without a token are not touched.  A table that is also the
 *           output projection gets its second gradient this way.
 *   workspace of slim_embed_bwd_workspace_size() bytes.
 */
slim_status slim_embed_bwd_workspace_size(long long N, int D, int V, slim_dtype dtype,
                                          size_t* bytes);
slim_status slim_embed_bwd(const void* ids, slim_index itype, const void* dout, long long N, int D,
                           int V, slim_dtype dtype, float scale, int accumulate, void* dtable,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * Softmax cross entropy of the rows of x against a vocabulary w:
 *     z_iv   = sum_d x_id w_vd
 *     lse_i  = log sum_v exp(z_iv)
 *     loss_i = lse_i - z_i,target(i)
 * The logits z live in tiles on the chip; what is kept is O(N).
 *   x       [N, D] dtype;  w [V, D] dtype;  targets [N] itype, aligned to its
 *           own size.  A row whose target is ignore_index has loss 0 (its lse
 *           is written all the same).  Any other target outside [0, V) is an
 *           error of the caller's data and makes the row's loss NaN.
 *   loss    [N] fp32, written.  Computed as log1p of the other words' weight
 *           against the target's, so that a small loss keeps its digits.
 *   lse     [N] fp32, written; slim_vocab_loss_bwd reads it.
 *   total   [2] fp32, written: the sum of the losses, and the number of rows
 *           that are not ignored (their quotient is the mean loss).
 * bf16 operands are multiplied exactly and summed in fp32.  fp32 operands are
 * split into three bf16 pieces (24 bits) and multiplied piece by piece, six
 * products each, smallest first, on the tensor cores.
 * Values that count are finite: an infinity in w, or in a row that is not ignored,
 * makes the logits it enters infinite or NaN (among the fp32 pieces, 0 x inf).  A
 * word is masked through a constant feature of the type's lowest value.
 * 0 <= N < 2^31 - 512, 1 <= D <= 2^30, 1 <= V <= 2^30, N V <= 2^50, N D and V D
 * <= 2^40.  N = 0 only zeroes `total`.
 *
 * slim_vocab_loss_workspace_size: workspace bytes of the forward (backward =
 * 0, piece is not read) or of the backward with this piece.
 */
slim_status slim_vocab_loss_workspace_size(long long N, int D, int V, slim_dtype dtype, int piece,
                                           int backward, size_t* bytes);
slim_status slim_vocab_loss_fwd(const void* x, const void* w, const void* targets,
                                slim_index itype, long long N, int D, int V, slim_dtype dtype,
                                long long ignore_index, float* loss, float* lse, float* total,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradients of sum_i c_i loss_i with respect to x and w:
 *     g_iv = c_i (exp(z_iv - lse_i) - [v = target(i)]),  c_i = dloss_i / count
 *     dx = g w  [N, D] dtype,   dw = g^T x  [V, D] dtype
 * in pieces of `piece` words (rounded up to a multiple of 256): a piece's
 * logits are computed again and its g is held only until both products have
 * read it, so memory grows with N * piece and not with N * V (2 bytes an element for
 * bf16 problems, 6 for fp32 ones).
 *   lse          [N] fp32 from the forward on the same x, w and targets.
 *   dloss        fp32: [N] with dloss_stride 1, or [1] for every row with
 *                dloss_stride 0.
 *   count        [1] fp32 or null (1): for the mean loss, the forward's
 *                total[1].  Where it is 0 there is no row to divide among and
 *                the gradients are zero.
 * An ignored row passes nothing on: its dx is zero, and its x, whatever it
 * holds, does not reach dw.  A row whose target is out of range passes NaN.
 * g is rounded once for the products: to bf16 for bf16 problems (2^-9
 * relative, like the rounding of the gradients themselves), to three bf16
 * pieces for fp32 ones.  Sums are fp32, and long ones are joined from parts (the
 * tensor cores cut bits off a long sum); dx and dw are rounded once.
 */
slim_status slim_vocab_loss_bwd(const void* x, const void* w, const void* targets,
                                slim_index itype, const float* lse, const float* dloss,
                                int dloss_stride, const float* count, long long N, int D, int V,
                                slim_dtype dtype, int piece, long long ignore_index, void* dx,
                                void* dw, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The global 2-norm of n gradients and their clipping by it:
 *     norm = sqrt(sum over all tensors and elements of g^2)
 *     out  = min(1, max_norm / norm) * g, rounded to nearest even.
 * src, dst, numel and dtypes are HOST arrays of length n, read during the
 * call: tensor t has numel[t] >= 0 elements of type dtypes[t] at src[t], and
 * its clipped form goes to dst[t], in the same type.  Tensors are aligned to
 * their element size.  dst[t] = src[t] clips in place; otherwise no two
 * tensors may overlap.  An empty tensor's pointers may be null.
 *   norm      [1] fp32, written.  The squares are summed over the whole range
 *             of the types: neither 1e30 nor 1e-30 is lost.
 *   max_norm  > 0; infinity only measures and copies.
 * When the norm written is not finite (an infinity or NaN among the gradients,
 * or finite ones whose norm passes fp32's range) the gradients are passed on
 * unscaled: the caller reads the norm and skips the step.
 *   workspace of slim_clip_workspace_size(n) bytes.
 */
slim_status slim_clip_workspace_size(int n, size_t* bytes);
slim_status slim_clip_grads(const void* const* src, void* const* dst, const long long* numel,
                            const slim_dtype* dtypes, int n, float max_norm, float* norm,
                            void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SLIM_LM_H_ */
