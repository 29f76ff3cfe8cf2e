/*
 * libnova_attn - rotary positions of queries and keys (C ABI), forward and backward.
 *
 * What stands in front of the attention of nova_attn.h and nova_window.h in a model with rotary positions: of every
 * head the first `rotary` dimensions are turned in pairs, each pair by the angle that the token's position has at that
 * pair's frequency.  The paper's model (GPT-2) learns its positions and has no counterpart.
 *
 *   a = positions[b, t] * inv_freq[i]                                    i < rotary / 2
 *   forward   y0 = amplitude * (x0 cos a - x1 sin a)     backward   dx0 = amplitude * (dy0 cos a + dy1 sin a)
 *             y1 = amplitude * (x1 cos a + x0 sin a)                dx1 = amplitude * (dy1 cos a - dy0 sin a)
 *
 * The pair i is (i, i + rotary/2), or (2i, 2i+1) if `interleaved` is not 0.  The dimensions from `rotary` on are copied.
 * Angles are products in 64 bits, brought to one turn before they are rounded to 32, so that a far position (2^31 - 1 is the
 * last) is as exact as a near one; sums are in 32 bits and rounded once.
 *
 * Conventions are those of nova_attn.h: device pointers, caller owns every buffer, work is only enqueued on `stream`,
 * nothing is allocated or synchronised, calls may be captured, status codes are the NOVA_ATTN_* values.
 */
#ifndef NOVA_ROPE_H_
#define NOVA_ROPE_H_

#include "nova_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Q, Q_out  bf16, elements (b, h, t, d) with b < B, h < H, t < T, d < D at base + b*batch + h*head + t*token + d (in / out)
 * K, K_out  the same with H_kv heads (which may be fewer, query heads sharing them); NULL, NULL: Q alone, H_kv is ignored
 * inv_freq  fp32 [rotary / 2], radians per position                         (in)
 * positions int32, token (b, t) at positions[b * position_stride + t]: T for a tensor [B, T], 0 for one row that all sequences
 *           share.  NULL: 0 .. T-1, position_stride is ignored.  Any value, negative ones too.        (in)
 *
 * A single token per sequence (T = 1) with its position is the form for serving; a slice of a fused projection output [B, T,
 * H + 2 H_kv, D] is turned where it lies: Q_out may be Q and K_out may be K, if their strides are the same; else outputs overlap
 * neither inputs nor each other.
 *
 * Requirements: D a multiple of 8 up to 1024, rotary even, 2 <= rotary <= D, B * T <= 2^30, H + H_kv <= 2^24, position_stride >= 0;
 * strides as in the strided calls of nova_attn.h (multiples of 8, token >= D, head and batch >= 8, below 2^39); tensors 16-byte
 * aligned, inv_freq and positions 4-byte; amplitude finite.  Errors (checked on the host before any launch):
 * NOVA_ATTN_ERR_NULL, NOVA_ATTN_ERR_SHAPE (sizes, rotary, strides), NOVA_ATTN_ERR_ALIGNMENT, NOVA_ATTN_ERR_SCALE (amplitude),
 * NOVA_ATTN_ERR_UNSUPPORTED (device is not sm_100), NOVA_ATTN_ERR_CUDA.
 */
int nova_rope_fwd(const void* Q, const void* K, void* Q_out, void* K_out, const float* inv_freq, const int* positions,
                  int B, int H, int H_kv, int T, int D, int rotary, int interleaved, float amplitude,
                  long long position_stride, const nova_attn_strides* q_strides, const nova_attn_strides* k_strides,
                  const nova_attn_strides* q_out_strides, const nova_attn_strides* k_out_strides, void* stream);

/* The gradients: dQ and dK of Q and K from dQ_out and dK_out of Q_out and K_out.  Arguments, checks and errors as above. */
int nova_rope_bwd(const void* dQ_out, const void* dK_out, void* dQ, void* dK, const float* inv_freq, const int* positions,
                  int B, int H, int H_kv, int T, int D, int rotary, int interleaved, float amplitude,
                  long long position_stride, const nova_attn_strides* dq_out_strides,
                  const nova_attn_strides* dk_out_strides, const nova_attn_strides* dq_strides,
                  const nova_attn_strides* dk_strides, void* stream);

/*
 * The frequencies of a model, on the host (no GPU): inv_freq[i] = base^(-2i / rotary) for i < rotary / 2, scaled for a context
 * `factor` times as long as the `original` positions that the model was trained on:
 *   NOVA_ROPE_PLAIN   not at all (factor and original are ignored)
 *   NOVA_ROPE_LINEAR  all divided by factor (positions interpolated)
 *   NOVA_ROPE_BASE    base * factor^(rotary / (rotary - 2)) in the place of base: the fastest stays, the slowest is divided by
 *                     factor
 *   NOVA_ROPE_BANDS   by how often a frequency turns in the original context, n = original * inv_freq / 2 pi: from `high` turns
 *                     on it stays, up to `low` turns it is divided by factor, between the two
 *                     inv_freq * (r + (1 - r) / factor) with r = (n - low) / (high - low)
 *   NOVA_ROPE_YARN    the same with r linear in the pair's number i between those at which n is high and low, rounded down and
 *                     up and kept within 0 and rotary - 1 (Peng et al., "YaRN", 2023); where every frequency turns `high` times
 *                     all stay, where none turns more than `low` times all are divided; amplitude = 0.1 ln(factor) + 1
 * Writes rotary / 2 numbers to inv_freq and the amplitude (1 but for YARN) to *amplitude, both on the host.  Returns
 * NOVA_ATTN_OK, NOVA_ATTN_ERR_NULL, or NOVA_ATTN_ERR_SHAPE: rotary odd or < 2 (< 4 for BASE), base <= 1, an unknown kind; where the
 * kind uses them factor < 1, original < 1, low <= 0 or high <= low; anything not finite.
 */
#define NOVA_ROPE_PLAIN 0
#define NOVA_ROPE_LINEAR 1
#define NOVA_ROPE_BASE 2
#define NOVA_ROPE_BANDS 3
#define NOVA_ROPE_YARN 4
int nova_rope_frequencies(float* inv_freq, float* amplitude, int rotary, double base, int kind, double factor,
                          long long original, double low, double high);

#ifdef __cplusplus
}
#endif
#endif /* NOVA_ROPE_H_ */
