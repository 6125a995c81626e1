/*
 * head_rope.h -- C ABI of what lies between a layer's projections and its attention (gfx950): norms of
 * queries and keys for each head, rotation by positions of one to four axes, and the layout that the
 * attention entry points of tile_attn.h, block_attn.h and cache4_attn.h take, in one pass; and the gradients.
 *
 * A row is the d values of one head of one token, x. Rows of q and k become
 *   TA_NORM_NONE   n = x
 *   TA_NORM_RMS    n = x * r * w,              r = (mean(x^2) + eps)^-1/2
 *   TA_NORM_LAYER  n = (x - mean(x)) * r * w + b,  r = (mean((x - mean(x))^2) + eps)^-1/2
 * with weights (and biases) of d values for q and for k, and then pairs (i, j) of their values are turned by
 * the angle a = position * frequency:
 *   y_i = n_i cos(a) - n_j sin(a),    y_j = n_j cos(a) + n_i sin(a).
 * Rows of v are carried over as they are. Everything between the bf16 input and the bf16 result is fp32, but for
 * the angles: a product in fp64, as a number of turns, whose fraction alone goes on. (A row's squares are summed in
 * fp32: with a norm, magnitudes up to 2^60.)
 *
 * Axes: values 0 .. dims[0] - 1 of a head belong to axis 0 (time, say), the next dims[1] to axis 1, and so on;
 * dims are even, their sum R is at most d, and values from R on are not turned. Pair p (of R / 2, those of axis 0
 * first) has frequency freqs[p] and turns with its axis' position. Which values it joins:
 *   TA_ROPE_INTERLEAVED  2 p and 2 p + 1
 *   TA_ROPE_HALVES       j and dims[a] / 2 + j of its axis' values, p being the j-th pair of the axis
 *   TA_ROPE_SPLIT        p and R / 2 + p
 *   TA_ROPE_NONE         no rotation: axes, dims, freqs and positions are not looked at
 *
 * Conventions as in block_attn.h: bf16 tensors, 16-byte aligned, on the current device; argument errors are found
 * before any HIP call; nothing is allocated and nothing kept; every call may be captured; the same call gives the
 * same bits; workspaces are the caller's. fp32 weights, biases and their gradients are 16-byte aligned, freqs
 * 8-byte, positions and lens 4-byte.
 */
#ifndef HEAD_ROPE_H
#define HEAD_ROPE_H

#include <stddef.h>
#include <stdint.h>

#include "tile_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TA_ROPE_AXES 4

typedef enum { TA_NORM_NONE = 0, TA_NORM_RMS = 1, TA_NORM_LAYER = 2 } ta_norm;
typedef enum { TA_ROPE_NONE = 0, TA_ROPE_INTERLEAVED = 1, TA_ROPE_HALVES = 2, TA_ROPE_SPLIT = 3 } ta_rope_layout;

/*
 * The rows of a tensor as a projection leaves them: value e of head h of token s of sequence b stands at
 * data[b * batch + s * token + h * head + e]. Strides are counted in values, multiples of 8, not negative; 0 is
 * allowed for what is read (one row for many), not for what is written.
 */
typedef struct {
  const void* data;
  int64_t batch, token, head;
} ta_rows;

/*
 * B sequences of S tokens, H heads of q, Hkv of k and of v, d (64, 96 or 128) values a head. B * S and S * d stay
 * below 2^31, H + 2 * Hkv below 2^16.
 * q_weight, k_weight, q_bias, k_bias: DEVICE fp32 [d], or NULL for ones and zeros (weights only with a norm,
 * biases only with TA_NORM_LAYER). eps: at least the smallest normal fp32 number.
 * freqs: DEVICE fp64 [R / 2], radians per position. positions: DEVICE int32 [S][axes], those of sequence b from
 * positions + b * positions_batch on (0: the same in every sequence).
 * lens: DEVICE int32 [B] or NULL for S. Tokens from lens[b] on are padding: whatever they hold, their results and
 * gradients are zeros, and weights and biases get nothing from them.
 */
typedef struct {
  int B, S, H, Hkv, d;
  int norm;
  float eps;
  const float* q_weight;
  const float* k_weight;
  const float* q_bias;
  const float* k_bias;
  int layout;
  int axes;
  int dims[TA_ROPE_AXES];
  const double* freqs;
  const int32_t* positions;
  int64_t positions_batch;
  const int32_t* lens;
} head_rope_spec;

/*
 * q_out: bf16 [B, H, S, d]; k_out, v_out: bf16 [B, Hkv, S, d]. Of q, k and v any may be left out (the ta_rows
 * NULL, and its output NULL), but not all. Inputs may lie in one tensor (a projection of everything); outputs
 * overlap no input and not each other.
 */
int head_rope_fwd(const head_rope_spec* spec, const ta_rows* q, const ta_rows* k, const ta_rows* v, void* q_out,
                  void* k_out, void* v_out, void* stream);

/*
 * Gradients for the same spec and inputs. dq_out: bf16 [B, H, S, d], dk_out, dv_out: bf16 [B, Hkv, S, d], the
 * gradients of head_rope_fwd's results. dq, dk, dv receive those of q, k and v, with strides of their own: rows
 * may interleave with the other two's in one tensor (heads behind heads of the same tokens, with the same batch
 * and token strides) but share no value. q and k are the forward's inputs (only looked at with a norm; v is
 * not asked for). What was left out of the forward is NULL throughout.
 * dq_weight, dk_weight, dq_bias, dk_bias: fp32 [d], summed over all tokens and heads, or NULL where not wanted (biases
 * only with TA_NORM_LAYER, weights only with a norm). A sum's terms are added in an order that the sizes alone set, each
 * through fewer than 512 additions in fp32, however many rows there are.
 */
int head_rope_bwd_workspace(const head_rope_spec* spec, size_t* bytes);
int head_rope_bwd(const head_rope_spec* spec, const ta_rows* q, const ta_rows* k, const void* dq_out,
                  const void* dk_out, const void* dv_out, const ta_rows* dq, const ta_rows* dk, const ta_rows* dv,
                  float* dq_weight, float* dk_weight, float* dq_bias, float* dk_bias, void* workspace,
                  size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* HEAD_ROPE_H */
