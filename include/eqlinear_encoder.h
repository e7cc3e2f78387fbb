/* eqlinear_encoder.h -- operators of image and video encoders around the
 * equivariant layers: rotary positions with several axes, attention with a
 * sliding window and first tokens that stay visible (training, whole sequences and single
 * tokens over a cache), and group norm with an activation, channels last.
 * Same library, dtypes, status codes and rules as eqlinear.h: device pointers,
 * the caller's stream, every argument checked before any launch, no allocation,
 * no synchronisation, outputs overwritten, bitwise reproducible (no atomics,
 * fixed orders of summation).  Sizes of 0 in B, L, Lq or S are no-ops.  An
 * address plus its strides must lie inside memory that the caller owns; strides
 * are counted in elements, and an output's keep its elements apart.  What is written
 * (outputs, statistics, workspace) overlaps nothing else of the call; outputs with
 * strides may lie between one another's elements where their strides agree. */
#ifndef EQLINEAR_ENCODER_H
#define EQLINEAR_ENCODER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions with several axes ----------------------------------
 * x [B, L, heads, dh, T] (channel, group element; the last two contiguous), y
 * alike.  The first n = sum(sections) channel pairs of every head turn:
 *   phi = positions[b, l, axis(c)] * freqs[c],  c < n
 *   y_lo = x_lo cos phi - x_hi sin phi,  y_hi = x_hi cos phi + x_lo sin phi
 * with (lo, hi) = (c, c + n), or (2c, 2c + 1) where interleaved; sections[a] pairs
 * belong to axis a.  Channels from 2n on are copied.  All group elements of
 * a channel turn alike, so the map commutes with the group action.  inverse:
 * -phi, which is also the gradient.  The angle is formed in 64 bits, products
 * in fp32, one rounding.  y == x with equal strides turns in place; any other
 * overlap is refused.  Elements need only their own alignment (16-byte aligned
 * bases and strides run faster).  1 <= axes <= 4, 2n <= dh, dh * T <= 1024,
 * T <= 16, n <= 2048 (EQL_ERR_UNSUPPORTED above). */
typedef struct {
  int64_t B, L;
  int32_t heads, dh, T, axes;
  int32_t sections[4];
  int32_t float_positions; /* positions are int32, or float where 1 */
  int32_t interleaved, inverse, dtype;
  int64_t x_stride[3], y_stride[3]; /* sequence, token, head */
  int64_t pos_stride[2];            /* sequence, token; the axes are contiguous */
} eqlinear_rotary_shape;

int eqlinear_rotary(const eqlinear_rotary_shape* shape, const void* x, const void* positions, const float* freqs,
                    void* y, void* stream);

/* ---- windowed attention ---------------------------------------------------
 * q, o [B, Lq, heads, head_dim], k, v [B, Lk, kv_heads, head_dim]; heads is a
 * multiple of kv_heads, query head h reads key/value head h / (heads / kv_heads).
 * Sequence b holds lengths[b] keys (NULL: Lk; values outside 0 .. Lk are taken as the
 * nearer end), and its query i stands at position p = starts[b] + i (NULL: Lk - Lq).
 * Query p sees key j iff p < lengths[b], j < lengths[b], j <= p + right and
 * (j >= p - left or j < sinks); left or right = -1 is no limit.
 *   o = sum_j softmax_j(scale * <q, k_j>) v_j over the keys seen, 0 where there are none.
 * Keys, values and gradients that a query does not see have no effect on it,
 * infinities and NaN among them.  Scores, softmax and sums in fp32, a probability
 * (and its gradient) rounded once to the dtype as the operand of the next product.
 * head_dim <= 128 and a multiple of 16 bytes; kv_heads * Lk <= 2^27 - 2^14, heads * Lq
 * <= 2^25 - 2^14; 65 token strides and, of queries, all head strides within 2 GiB
 * (EQL_ERR_UNSUPPORTED); strides of whole 16-byte words (EQL_ERR_ALIGNMENT).
 * lse (fp32 [B, kv_heads, Lq, heads / kv_heads], logarithm to base 2, +inf for
 * a query that sees nothing) may be NULL; the backward reads it. */
typedef struct {
  int64_t B, Lq, Lk;
  int64_t left, right, sinks;
  int32_t heads, kv_heads, head_dim, dtype;
  float scale;
  int32_t reserved; /* 0 */
  /* sequence, token, head */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
  int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3]; /* backward */
} eqlinear_window_shape;

size_t eqlinear_window_attention_workspace_bytes(const eqlinear_window_shape* shape);
int eqlinear_window_attention(const eqlinear_window_shape* shape, const void* q, const void* k, const void* v,
                              const int32_t* lengths, const int32_t* starts, void* o, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream);

/* Gradients of the above: o and lse as the forward wrote them.  dk, dv sum over
 * the query heads that share a head.  delta = <do, o> is taken from the
 * rounded o, or summed anew for 16-bit rows that see few keys. */
size_t eqlinear_window_attention_backward_workspace_bytes(const eqlinear_window_shape* shape);
int eqlinear_window_attention_backward(const eqlinear_window_shape* shape, const void* q, const void* k, const void* v,
                                       const int32_t* lengths, const int32_t* starts, const void* o, const float* lse,
                                       const void* d_o, void* dq, void* dk, void* dv, void* workspace,
                                       size_t workspace_bytes, void* stream);

/* ---- group norm with an activation, channels last ---------------------------
 * x, y [B, S, C, T] contiguous, weight, bias [C], one dtype.  Mean and variance
 * (mean squared deviation) over the S positions, the C / groups channels of a
 * group and T:  y = act((x - mean) / sqrt(var + eps) * weight[c] + bias[c]).
 * stats (fp32 [B, groups, 2], 8-byte aligned: mean, 1 / sqrt(var + eps)) may be NULL; the backward
 * reads it.  Sums in fp32, one rounding.  C is a multiple of groups, T <= 16, C <= 65536,
 * groups <= 1024, B <= 2^20, S <= 2^30, 2^46 elements (EQL_ERR_UNSUPPORTED above). */
enum { EQL_ACT_NONE = 0, EQL_ACT_RELU = 1, EQL_ACT_SILU = 2, EQL_ACT_GELU = 3 /* by erf */ };

size_t eqlinear_group_norm_act_workspace_bytes(int64_t B, int64_t S, int T, int C, int groups, int dtype);
int eqlinear_group_norm_act(const void* x, const void* weight, const void* bias, void* y, float* stats,
                            void* workspace, size_t workspace_bytes, int64_t B, int64_t S, int T, int C, int groups,
                            float eps, int act, int dtype, void* stream);
size_t eqlinear_group_norm_act_backward_workspace_bytes(int64_t B, int64_t S, int T, int C, int groups, int dtype);
int eqlinear_group_norm_act_backward(const void* x, const void* weight, const void* bias, const float* stats,
                                     const void* dy, void* dx, void* dw, void* db, void* workspace,
                                     size_t workspace_bytes, int64_t B, int64_t S, int T, int C, int groups, int act,
                                     int dtype, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* EQLINEAR_ENCODER_H */
