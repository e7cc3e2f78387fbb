/* eqlinear_recurrent.h -- operators of recurrent encoder blocks: a short causal
 * convolution along the tokens, the selective state space scan (training, whole
 * sequences and single tokens with a state that is kept), and the norms before and
 * after a block's branch with its gate, residual scale and sum.
 * Same library, dtypes, status codes and rules as eqlinear.h: device pointers,
 * the caller's stream, every argument checked before any launch, no allocation,
 * no synchronisation, outputs overwritten, bitwise reproducible (no atomics,
 * fixed orders of summation).  Features are [B, L, C, T] (sequence, token, channel,
 * group element); parameters per channel are shared over T, so every map commutes with the
 * group action.  Sizes of 0 in B and L are no-ops but for the states, which pass, and the
 * gradients of parameters, which are 0.  Strides are counted in elements, the [C, T] of a
 * token are contiguous, and an address plus its strides must lie inside memory that the caller
 * owns.  What is written overlaps nothing else of the call, but for a state that
 * is updated in place.  lengths (int32 [B], or NULL): tokens of each sequence that hold
 * data, values outside 0 .. L taken as the nearer end; what lies behind them is never used,
 * and outputs and gradients there are 0. */
#ifndef EQLINEAR_RECURRENT_H
#define EQLINEAR_RECURRENT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- selective state space scan --------------------------------------------
 * x, delta, z, y [B, L, C, T]; b, c [B, L, groups, N], the N of a token contiguous; channel ch reads
 * group ch / (C / groups); A [C, N], D and delta_bias [C] fp32 (D, z and delta_bias may be
 * NULL).  For every sequence, channel and group element, from h = state_in (fp32 [B, C, T, N], NULL: 0) on:
 *   d = delta_l + delta_bias, through softplus where asked for
 *   h[n] = exp(d A[n]) h[n] + d b_l[n] x_l
 *   y_l = (sum_n c_l[n] h[n] + D x_l) * silu(z_l)
 * state_out (fp32 [B, C, T, N], may be state_in or NULL) is h after the last token.  States,
 * sums and exponents in fp32, one rounding of y.  states (fp32, _states_bytes, or NULL) keeps
 * what the backward starts its runs of tokens from: 4 NP / 8 bytes for each element of x, NP the states rounded up to 4, 8, 16,
 * 32 or 64 (8 bytes at 16 states, 32 at 64; NP bytes up to 4 states), and the columns of a group, C / groups * T, rounded up to a
 * multiple of 1024 / NP: many narrow groups multiply it, and the workspaces.  1 <= N <= 64, T <= 16,
 * C * T <= 65536, groups <= C, B <= 2^20, L <= 2^30, 2^46 elements a tensor (EQL_ERR_UNSUPPORTED above).
 * Elements need only their own alignment; 16-byte aligned addresses and strides run faster.  Infinities and NaN inside a
 * sequence do to y and the states what they do in the formulas; a gradient that is infinite there may come as NaN. */
typedef struct {
  int64_t B, L;
  int32_t C, T, N, groups;
  int32_t softplus, dtype;
  int64_t x_stride[2], delta_stride[2], z_stride[2]; /* sequence, token; y and the gradients are dense */
  int64_t b_stride[3], c_stride[3];                  /* sequence, token, group */
} eqlinear_scan_shape;

size_t eqlinear_selective_scan_workspace_bytes(const eqlinear_scan_shape* shape);
size_t eqlinear_selective_scan_states_bytes(const eqlinear_scan_shape* shape);
int eqlinear_selective_scan(const eqlinear_scan_shape* shape, const void* x, const void* delta, const float* A,
                            const void* b, const void* c, const float* D, const void* z, const float* delta_bias,
                            const int32_t* lengths, const float* state_in, void* y, float* state_out, float* states,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of the above from dy (dense) and d_state_out (NULL: 0), with states as the forward wrote
 * them: dx, ddelta, dz [B, L, C, T], db, dc [B, L, groups, N], dA [C, N], dD, ddelta_bias [C] fp32 (NULL where not
 * wanted: dD, dz, ddelta_bias and d_state_in), d_state_in fp32 [B, C, T, N]. */
size_t eqlinear_selective_scan_backward_workspace_bytes(const eqlinear_scan_shape* shape);
int eqlinear_selective_scan_backward(const eqlinear_scan_shape* shape, const void* x, const void* delta, const float* A,
                                     const void* b, const void* c, const float* D, const void* z,
                                     const float* delta_bias, const int32_t* lengths, const float* states,
                                     const void* dy, const float* d_state_out, void* dx, void* ddelta, float* dA,
                                     void* db, void* dc, float* dD, void* dz, float* ddelta_bias, float* d_state_in,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* ---- short causal convolution ----------------------------------------------
 * x [B, L, C, T], weight [C, W], bias [C] (or NULL), one dtype; y dense:
 *   y_l = act(bias + sum_w weight[w] x_{l - W + 1 + w}),  act EQL_ACT_NONE or EQL_ACT_SILU (eqlinear_encoder.h)
 * state_in [B, W - 1, C, T] holds the W - 1 tokens before the first (NULL: zeros), state_out (may be state_in, or
 * NULL) receives the last ones.  Sums in fp32, one rounding.  1 <= W <= 8, T <= 16, C * T <= 65536,
 * B <= 2^20, L <= 2^30, 2^46 elements (EQL_ERR_UNSUPPORTED above).  Alignment as above. */
typedef struct {
  int64_t B, L;
  int32_t C, T, W;
  int32_t act, dtype;
  int32_t reserved;    /* 0 */
  int64_t x_stride[2]; /* sequence, token */
} eqlinear_conv_shape;

int eqlinear_causal_conv(const eqlinear_conv_shape* shape, const void* x, const void* weight, const void* bias,
                         const int32_t* lengths, const void* state_in, void* y, void* state_out, void* stream);

/* Gradients from dy (dense) and d_state_out (NULL: 0); dbias and d_state_in may be NULL. */
size_t eqlinear_causal_conv_backward_workspace_bytes(const eqlinear_conv_shape* shape);
int eqlinear_causal_conv_backward(const eqlinear_conv_shape* shape, const void* x, const void* weight, const void* bias,
                                  const int32_t* lengths, const void* state_in, const void* dy,
                                  const void* d_state_out, void* dx, void* dweight, void* dbias, void* d_state_in,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* ---- residual sum between two norms ------------------------------------------
 * x, branch, r, h [B, L, C, T] dense, one dtype with the parameters:
 *   v = norm(branch) * post_weight[c] + post_bias[c], or branch where post_weight is NULL
 *   r = x + scale[c] * gate[b, c] * v   (scale, gate NULL: 1)
 *   h = norm(r) * weight[c] + bias[c]   (weight NULL: h is not formed)
 * norm over the C * T elements of a token: (v - mean) / sqrt(mean squared deviation + eps) for
 * EQL_NORM_LAYER, v / sqrt(mean square + eps) for EQL_NORM_RMS.  bias, post_bias may be NULL (0).  branch NULL: r is x and is
 * not written (r NULL), no scale, gate or post norm.  h is formed from r before its rounding.  Sums in
 * fp32.  C * T <= 8192, T <= 16, B * L <= 2^36 (EQL_ERR_UNSUPPORTED above).  Addresses need their element's
 * alignment; 16-byte aligned ones with C * T a whole number of 16-byte words run faster. */
enum { EQL_NORM_LAYER = 0, EQL_NORM_RMS = 1 };
typedef struct {
  int64_t B, L;
  int32_t C, T;
  int32_t kind, dtype;
  float eps;
  int32_t reserved; /* 0 */
} eqlinear_residual_shape;

int eqlinear_residual_norm(const eqlinear_residual_shape* shape, const void* x, const void* branch, const void* weight,
                           const void* bias, const void* scale, const void* gate, const void* post_weight,
                           const void* post_bias, void* r, void* h, void* stream);

/* Gradients from dr and dh (each may be NULL: 0; dh only with weight).  dx, dbranch [B, L, C, T], dweight .. dpost_bias
 * [C], dgate [B, C]; a gradient may be NULL where it is not wanted, and is 0 where there are no tokens.  r is formed again
 * from x and branch. */
size_t eqlinear_residual_norm_backward_workspace_bytes(const eqlinear_residual_shape* shape);
int eqlinear_residual_norm_backward(const eqlinear_residual_shape* shape, const void* x, const void* branch,
                                    const void* weight, const void* scale, const void* gate, const void* post_weight,
                                    const void* post_bias, const void* dr, const void* dh, void* dx, void* dbranch,
                                    void* dweight, void* dbias, void* dscale, void* dgate, void* dpost_weight,
                                    void* dpost_bias, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* EQLINEAR_RECURRENT_H */
