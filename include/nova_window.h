/*
 * libnova_attn - causal attention with a sliding window and sinks, and with shared key/value heads (C ABI): the forward and the
 * backward of training, and the form for one new token per sequence over a cache.
 *
 * The attention of nova_attn.h with another mask.  Query i keeps key j if
 *
 *     j <= i  and  (i - j < window  or  j < sinks):
 *
 * the last `window` keys, itself among them, and the first `sinks` keys of the sequence.  window >= 1; window >= T is the
 * whole causal triangle; sinks >= 0.  Tiles of which nothing is kept are not visited.  Every query keeps itself, so no row is
 * empty.
 *
 * Q, O, dO, dQ have H heads, K, V, dK, dV have H_kv, a divisor of H: query head h reads key/value head h / (H / H_kv), whose
 * gradient is the sum over the H / H_kv query heads that share it, in a fixed order.  H_kv = H is the attention of nova_attn.h.
 *
 * Conventions are those of nova_attn.h: device pointers, caller owns every buffer, work is only enqueued on `stream`, nothing is
 * allocated or synchronised, calls may be captured (after one call on the device), status codes are the NOVA_ATTN_* values and
 * nova_attn_poll_device_status applies.  bf16 tensors are addressed as (b, h, t, d) through strides as in the strided calls
 * there, with the same requirements; D is 64 or 128; scale is finite and > 0.  An element of Q, K, V or dO that is not finite
 * makes undefined, besides what it belongs in, the other results that come from its 128-row tile: those of every 128 queries (256 in
 * the backward) or keys of which one meets one of that tile under the mask.  So tokens that pad a sequence have to be finite.  In
 * the single-token form it reaches what keeps it and nothing else.
 *
 * Errors (checked on the host before any launch): NOVA_ATTN_ERR_NULL, NOVA_ATTN_ERR_SHAPE (sizes, strides, window < 1, sinks < 0,
 * H not a multiple of H_kv), NOVA_ATTN_ERR_UNSUPPORTED (D, or the device is not sm_100), NOVA_ATTN_ERR_ALIGNMENT,
 * NOVA_ATTN_ERR_SCALE, NOVA_ATTN_ERR_WORKSPACE, NOVA_ATTN_ERR_CUDA.
 */
#ifndef NOVA_WINDOW_H_
#define NOVA_WINDOW_H_

#include <stddef.h>

#include "nova_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Forward.
 *   Q, K, V : in,  bf16
 *   O       : out, bf16
 *   O_rest  : out, bf16 with the strides of O, or NULL: what the rounding took from O (O + O_rest is the sum before it was rounded,
 *             to 16 bits), for nova_window_bwd_preprocess.  A call with O_rest whose rows keep at most 64 keys (window + sinks, or T)
 *             takes more exact weights, so that its O and a call's without O_rest may differ by a rounding
 *   LSE     : out, fp32 [B,H,T] contiguous, natural-log log-sum-exp of the kept scaled scores
 */
int nova_window_fwd(const void* Q, const void* K, const void* V, void* O, void* O_rest, float* LSE, int B, int H, int H_kv,
                    int T, int D, int window, int sinks, const nova_attn_strides* q_strides,
                    const nova_attn_strides* k_strides, const nova_attn_strides* v_strides,
                    const nova_attn_strides* o_strides, float scale, void* stream);

/*
 * Delta = rowsum(dO * (O + O_rest)), fp32 [B,H,T].  O_rest may be NULL: then Delta carries the rounding of the stored O, which
 * reaches dQ and dK: the shorter the window, the more (where a row keeps a few keys, it is the largest part of their error).
 * The price of O_rest is its traffic, 2 bytes an element in the forward and here.
 */
int nova_window_bwd_preprocess(const void* O, const void* O_rest, const void* dO, float* Delta, int B, int H, int T, int D,
                               const nova_attn_strides* o_strides, const nova_attn_strides* do_strides, void* stream);

/* Bytes of workspace of nova_window_bwd; 0 for arguments that it would reject. */
size_t nova_window_bwd_workspace_bytes(int B, int H, int H_kv, int T, int D, int window, int sinks);

/*
 * Backward, in the two kernels of nova_attn_bwd_deterministic: every sum in a fixed order, bitwise reproducible.
 *   Q, K, V, dO : in,  bf16
 *   LSE, Delta  : in,  fp32 [B,H,T] of nova_window_fwd and nova_window_bwd_preprocess
 *   dQ, dK, dV  : out, bf16
 *   workspace   : at least nova_window_bwd_workspace_bytes bytes, 16-byte aligned; whatever it holds on entry does not matter.
 *                 Calls whose GPU work overlaps need one each.
 */
int nova_window_bwd(const void* Q, const void* K, const void* V, const void* dO, const float* LSE, const float* Delta, void* dQ,
                    void* dK, void* dV, int B, int H, int H_kv, int T, int D, int window, int sinks,
                    const nova_attn_strides* q_strides, const nova_attn_strides* k_strides,
                    const nova_attn_strides* v_strides, const nova_attn_strides* do_strides,
                    const nova_attn_strides* dq_strides, const nova_attn_strides* dk_strides,
                    const nova_attn_strides* dv_strides, float scale, void* workspace, size_t workspace_bytes, void* stream);

/*
 * One new token per sequence, for serving: the row i = lengths[b] - 1 of the attention above over a cache of T_max tokens, of
 * which the first lengths[b] are the sequence, the new token among them.
 *   Q       : in,  bf16 [B,H,1,D]
 *   K, V    : in,  bf16 [B,H_kv,T_max,D]; what is not kept is not read
 *   lengths : in,  int32 [B] on the device, from 0 to T_max (what is outside counts as the nearer end).  A sequence of length
 *             0 has no row: O = 0, LSE = -inf
 *   O       : out, bf16 [B,H,1,D]
 *   LSE     : out, fp32 [B,H]
 * A cache that keeps no more than sinks + window tokens, each new one in the place of the oldest behind the sinks, is read with
 * T_max = sinks + window and lengths[b] = min(tokens so far, T_max): the order of keys does not matter once they carry their
 * positions, and all that is there is kept.
 * The workspace (nova_window_decode_workspace_bytes bytes, 16-byte aligned; NULL if that is 0) as in the backward.  The order of
 * the sums follows from the shape alone: the same bits in every run.
 */
size_t nova_window_decode_workspace_bytes(int B, int H, int H_kv, int T_max, int D, int window, int sinks);
int nova_window_decode(const void* Q, const void* K, const void* V, const int* lengths, void* O, float* LSE, int B, int H,
                       int H_kv, int T_max, int D, int window, int sinks, const nova_attn_strides* q_strides,
                       const nova_attn_strides* k_strides, const nova_attn_strides* v_strides,
                       const nova_attn_strides* o_strides, float scale, void* workspace, size_t workspace_bytes,
                       void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NOVA_WINDOW_H_ */
