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
 * 0 <= N < 2^31, D >= 1, V >= 1.  N = 0 enqueues nothing.
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
 * When the norm is not finite (an infinity or NaN among the gradients) the
 * gradients are passed on unscaled: the caller reads the norm and skips the
 * step.
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
