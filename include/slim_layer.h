/*
 * libslim -- the rest of a language model's layer around the sliced attention,
 * on one NVIDIA GB300 (sm_103a):
 *
 *   slim_qk_norm_*     the root-mean-square norm of queries and keys per head
 *                      and their rotation by position, in one pass from a
 *                      projection's rows to the [B, H, L, d] that slim_fwd takes
 *
 * The conventions of slim.h hold: device pointers, every buffer owned by the
 * caller, arguments validated before anything is enqueued, all work on
 * `stream`, no synchronisation; host arrays are read during the call.
 * Workspaces are 256-byte aligned.  Results do not depend on the order in which
 * blocks run: two calls on the same inputs agree bit for bit.
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
 *   are read where they are, in 4-element pieces where pointers and strides
 *   allow it.  Hk = 0: no keys (k, k_out and k_weight are not read).
 *   q_weight, k_weight  [d] fp32, or null (1).
 *   positions  [B, L] ptype, any value, aligned to its own size; null: l.
 *   inv_freq   HOST array of rotary/2 finite numbers, radians per position.
 *              Angles are kept as 64-bit fractions of a turn: far positions lose
 *              nothing but the frequencies' own 53 bits.
 *   q_out, k_out  as q and k, no two elements in one place.  They may be q and k
 *              themselves, with the same strides.
 * Sums and turns are fp32, y is rounded once.  A row of zeros stays zero; a row
 * whose squares pass fp32's range is normalised all the same; a row that holds
 * an infinity or NaN becomes NaN, and no other.
 * 0 <= B, L and B L < 2^31; Hq >= 1; Hq, Hk <= 4096; 1 <= d <= 256; rotary even,
 * 0 <= rotary <= d; eps > 0 and finite; B L (Hq + Hk) <= 2^40; strides in [0, 2^40],
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

#ifdef __cplusplus
}
#endif

#endif /* SLIM_LAYER_H_ */
