/*
 * gdn_block.h -- C ABI of what stands around the recurrence in a block and at the end of a
 * training step: the gated linear map (the gated half of a feed-forward block), the short
 * causal convolution in front of the recurrence, both with their gradient and their form for
 * decoding batches, and the norm and clipping of all gradients.  Same library, same
 * conventions (device pointers on the current HIP device, 16-byte aligned and
 * contiguous unless said otherwise; asynchronous on `stream`; arguments checked
 * on the host, nothing enqueued on an error; values not checked) and the same
 * status codes as gdn.h.  is_bf16 = 1: the tensors called E below hold bf16, 0: fp32.
 * No call here allocates device memory, all may be captured, and their results are
 * deterministic.  Calls that run at once need a workspace each.
 */
#ifndef GDN_BLOCK_H
#define GDN_BLOCK_H

#include <stdint.h>

#include "gdn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations. */
enum {
    GDN_ACT_NONE = 0,     /* z */
    GDN_ACT_SILU = 1,     /* z / (1 + e^-z) */
    GDN_ACT_GELU = 2,     /* z Phi(z), the normal distribution's */
    GDN_ACT_GELU_TANH = 3 /* z / (1 + e^-2k), k = sqrt(2/pi) (z + 0.044715 z^3): gelu's tanh form */
};

/*
 * The gated linear map of M rows of C channels to F hidden units,
 *
 *   h = act(x Wg^T) o (x Wu^T)
 *
 *   x [M][C], w_gate, w_up [F][C], h [M][F]   E; those whose rows are no whole multiples of 16 bytes, here and in
 *      the gradient, aligned to an element only
 *
 * with fp32 sums; h is rounded once.  M, C, F >= 1, C < 2^21, F < 2^20, and M F, M C and F C so that a launch holds their
 * tiles (M F and M C below 2^35, F C below 2^37) and, where rows of x are no whole multiples of 16 bytes, their copies
 * ((M + 2 F) C below 2^35).  h overlaps nothing else.  In fp32, products are formed from three bf16 parts of each
 * operand, each to within 2^-21 of itself (mostly 2^-24), so that all but the shortest sums are as exact as in fp32
 * arithmetic: an infinity may give NaN where that would keep it (in its own row of h, or hidden unit), and of values
 * below 2^-110 the last bits may be lost.
 * `ws`: caller-owned device buffer, 256-byte aligned, of at least
 * gdn_gated_linear_workspace_bytes(..., 0) bytes.  That may be 0 (and ws NULL; it is for most sizes, and for arguments that
 * the call refuses); room is needed where rows of x are not whole multiples of 16 bytes, or few and long.
 */
size_t gdn_gated_linear_workspace_bytes(int M, int C, int F, int is_bf16, int backward);

int gdn_gated_linear_forward(const void *x, const void *w_gate, const void *w_up, void *h, int M, int C, int F,
                             int act, int is_bf16, void *ws, size_t ws_bytes, void *stream);

/*
 * Its gradient: from dh = dL/dh [M][F],
 *
 *   dx [M][C], dw_gate, dw_up [F][C]   E
 *
 * Nothing of the forward call is needed but its inputs: both projections are formed again.  Sums are fp32.
 * The gradients of the two projections are operands of the products behind them and are rounded to E
 * for those, as the results are.  An infinity or NaN makes NaN of what depends on it, and an infinity may also where
 * fp32 arithmetic would keep it.  Outputs overlap nothing else.
 * ws as above, of gdn_gated_linear_workspace_bytes(..., 1) bytes (2 M F of E and a little; 0 for arguments that the call refuses).
 */
int gdn_gated_linear_backward(const void *x, const void *w_gate, const void *w_up, const void *dh, void *dx,
                              void *dw_gate, void *dw_up, int M, int C, int F, int act, int is_bf16, void *ws,
                              size_t ws_bytes, void *stream);

/*
 * The short causal convolution, a channel each: with xe = [state; x], the W - 1 inputs before the first
 * token and the T tokens of a sequence,
 *
 *   y_t = act(bias + sum_i w[c][i] xe_{t+i}),   state_out = xe_T .. xe_{T+W-2}
 *
 *   x  [B][T][C] E, x_batch and x_token elements apart from sequence to sequence and from token to token
 *      (0 and more; aligned to an element)
 *   w  [C][W] fp32, bias [C] fp32 or NULL (zero), 2 <= W <= 4
 *   state_in, state_out [B][W-1][C] E, or NULL: zeros before the first token; not wanted
 *   y  [B][T][C] E
 *
 * Sums are fp32.  state_out may be state_in; outputs overlap nothing else.  B, T, C >= 1, T < 2^30, B T C / 8 < 2^33, and
 * for T = 1 B C / 8 < 2^32 - 2^8 (a launch's threads; C counts up to a multiple of 8 in both).
 */
int gdn_short_conv_forward(const void *x, int64_t x_batch, int64_t x_token, const float *w, const float *bias,
                           const void *state_in, void *y, void *state_out, int B, int T, int C, int W, int act,
                           int is_bf16, void *stream);

/*
 * Its gradient, from dy = dL/dy [B][T][C] E and dstate_out = dL/d(state_out) [B][W-1][C] E (NULL: zero):
 *
 *   dx [B][T][C] E, dx_batch and dx_token elements apart (its sequences one behind the other, or all sequences of a
 *      token before the next token, so that no two of its elements are the same)
 *   dw [C][W], dbias [C] fp32 (dbias may be NULL), dstate_in [B][W-1][C] E, or NULL
 *
 * The sums over tokens are fp32, in a fixed order.  Outputs overlap nothing.  B (C / 256 + 1) (T / 128 + 1) < 2^23,
 * (W + 1) C / 64 < 2^22.  ws: as above, at least gdn_short_conv_workspace_bytes(...) bytes (0 for arguments that the call refuses).
 */
size_t gdn_short_conv_workspace_bytes(int B, int T, int C, int W);

int gdn_short_conv_backward(const void *x, int64_t x_batch, int64_t x_token, const float *w, const float *bias,
                            const void *state_in, const void *dy, const void *dstate_out, void *dx, int64_t dx_batch,
                            int64_t dx_token, float *dw, float *dbias, void *dstate_in, int B, int T, int C, int W,
                            int act, int is_bf16, void *ws, size_t ws_bytes, void *stream);

/*
 * The same for N sequences with up to L new tokens each, their last W - 1 inputs kept in a pool of P slots
 * (state_in, state_out [P][W-1][C] E; usually the same buffer): x [N][L][C] as above, y [N][L][C].
 * slots and lengths are those of gdn_step_forward, and so is what happens to rows, slots and tokens that
 * they leave out or that are refused: padding, slots past the pool or named before (NaN in y, no
 * state written), and the time that looking for an earlier owner takes.  N, L, P, C >= 1, N C / 512 < 2^24.
 */
int gdn_short_conv_step(const void *x, int64_t x_row, int64_t x_token, const float *w, const float *bias,
                        const void *state_in, const int *slots, const int *lengths, void *y, void *state_out, int N,
                        int L, int P, int C, int W, int act, int is_bf16, void *stream);

/*
 * The norm over all elements of `count` tensors (host arrays of device pointers, of element counts and of
 * whether a tensor holds bf16; otherwise fp32),
 *
 *   norm = sqrt(sum x^2)   fp32, from fp64 squares and sums: nothing overflows but the result itself
 *
 * Tensors are aligned to an element and may be empty; one that is given twice counts twice.
 * ws: as above, at least gdn_grad_workspace_bytes(count) bytes.
 */
size_t gdn_grad_workspace_bytes(int count);

int gdn_grad_norm(const void *const *tensors, const int64_t *sizes, const int *is_bf16, int count, float *norm, void *ws,
                  size_t ws_bytes, void *stream);

/*
 * Clipping: out = min(1, max_norm / (norm + eps)) x for all tensors, rounded once.  out[i] is tensors[i] itself (where
 * nothing is then written if the factor is 1) or overlaps no tensor and no other out.  norm_in NULL: the
 * norm is formed as above; otherwise it is that fp32 value (a norm joined over several processes, say).
 * norm, or NULL, takes the norm that was used.  A norm that is NaN makes all NaN; an infinite one zeros, and NaN of
 * infinities.  max_norm and eps >= 0; with an infinite max_norm, or a norm of 0, nothing changes.
 */
int gdn_grad_clip(const void *const *tensors, void *const *out, const int64_t *sizes, const int *is_bf16, int count,
                  const float *norm_in, float *norm, float max_norm, float eps, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GDN_BLOCK_H */
