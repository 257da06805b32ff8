/*
 * gdn_ops.h -- C ABI of the operators around the gated delta-rule forward of
 * gdn.h: the recurrent step of a decoding batch, the gradient of the token-wise
 * chunk forward, and the norms, gate and scaled residual between two blocks with
 * their gradient.  Same library, same
 * conventions (device pointers on the current HIP device, 16-byte aligned and
 * contiguous unless said otherwise; asynchronous on `stream`; arguments checked
 * on the host, nothing enqueued on an error; values not checked) and the same
 * status codes.  is_bf16 = 1: the tensors called E below hold bf16, 0: fp32.
 * No call here allocates device memory.
 */
#ifndef GDN_OPS_H
#define GDN_OPS_H

#include "gdn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Recurrent step: N sequences, each with up to L new tokens, against recurrent
 * states kept in a pool of P slots.  For row n with slot s = slots[n], head h,
 * its key head g = h / (H / Hk) and t = 0 .. lengths[n] - 1:
 *
 *   u   = beta (v - alpha S^T k)        (S = the state H = S^T of gdn.h, [Dk][Dv])
 *   S   = alpha S + k u^T
 *   o_t = S^T q
 *
 * with fp32 arithmetic throughout.
 *
 *   q, k       [N][L][Hk][Dk]     E     Hk divides H: consecutive H / Hk heads share a key head
 *   v, out     [N][L][H][Dv]      E
 *   alpha, beta [N][L][H]         fp32
 *   state_in, state_out [P][H][Dk][Dv] fp32 (state_in == state_out, in place, is the usual call)
 *   slots      [N] int32 (4-byte aligned) or NULL: row n uses slot n (then N <= P)
 *   lengths    [N] int32 (4-byte aligned) or NULL: L tokens in every row; values are
 *              clamped to 0 .. L
 *
 * Only the slots named are read and written; out rows at and past a row's
 * length, and slots no row names, are left as they were.  A row of length 0
 * takes its state over unchanged.  A negative slot marks padding: nothing of
 * that row is written.  A slot >= P, or one that an earlier row names already,
 * is refused on the device: the row's out (up to its length) becomes NaN and
 * no state is written for it; the first row that names a slot has it.  Finding
 * that row takes time that grows with N^2: with slots in place of NULL, 4096 rows of 16 heads of 128
 * take no longer, 16384 rows 11.3 in place of 6.8 ms; one head of 64: 1024 rows no
 * longer, 4096 rows 29 in place of 21 us, 65536 rows 1.4 in place of 0.43 ms.
 * N, L, P, Hk, H >= 1, N H < 2^24; Dk, Dv in {64, 128}.  The call needs no workspace and may
 * be captured.
 */
int gdn_step_forward(const void *q, const void *k, const void *v, const float *alpha, const float *beta,
                     const float *state_in, const int *slots, const int *lengths, void *out,
                     float *state_out, int N, int L, int P, int Hk, int H, int Dk, int Dv, int is_bf16,
                     void *stream);

/*
 * Gradient of gdn_chunk_forward: from dout = dL/d(out) and dstate_out =
 * dL/d(state_out) (NULL: zero), with the inputs of the forward call,
 *
 *   dq, dk [B][T][H][Dk], dv [B][T][H][Dv]   E
 *   dalpha, dbeta [B][T][H]                  fp32
 *   dstate_in [B][H][Dk][Dv]                 fp32, or NULL to drop it
 *
 * dout is E [B][T][H][Dv], dstate_out fp32 [B][H][Dk][Dv]; the other inputs, the
 * sizes and chunk are those of gdn_chunk_forward.  Nothing of the forward call is
 * needed but its inputs: states and pseudo-values are formed again.  All
 * gradients are those of the recurrence itself: alpha and beta of 0 have theirs
 * too (alpha below 1.2e-38 acts as that value, as in the forward).  Sums, states
 * and their gradients are fp32, and on the bf16 path too the operands of products
 * that are not inputs keep fp32's mantissa.  Results are deterministic.  A NaN
 * or an infinity, given or where a sum leaves fp32's range, may make any gradient
 * of its batch and head NaN, also those of earlier tokens and where fp32
 * arithmetic would keep the infinity; other heads' are as without it.
 *
 * B H <= 65535, and B H chunks < 2^23.  Outputs may not overlap inputs or each other,
 * except dstate_in == dstate_out.
 * `ws`: caller-owned device buffer, 256-byte aligned, of at least
 * gdn_chunk_backward_workspace_bytes(...) bytes (0 for arguments that the call
 * refuses; 338 KB a chunk and head at Dk = Dv = 128).  Calls that run at once need
 * one each.
 */
size_t gdn_chunk_backward_workspace_bytes(int B, int H, int T, int Dk, int Dv, int chunk, int is_bf16);

int gdn_chunk_backward(const void *q, const void *k, const void *v, const float *alpha, const float *beta,
                       const float *state_in, const void *dout, const float *dstate_out, void *dq,
                       void *dk, void *dv, float *dalpha, float *dbeta, float *dstate_in, int B, int H,
                       int T, int Dk, int Dv, int chunk, int is_bf16, void *ws, size_t ws_bytes,
                       void *stream);

/*
 * The border between two blocks, for R rows (tokens) of C channels: the norm
 * behind a block's output y, its gate, the residual stream x scaled, and the
 * norm in front of the next block:
 *
 *   n = w_post o y / sqrt(mean(y^2) + eps)
 *   r = res_scale x + gate[row / gate_tokens] o n
 *   u = w_pre o r / sqrt(mean(r^2) + eps)
 *
 *   x, y, r, u  [R][C] E        gate [R / gate_tokens][C] E or NULL (all ones)
 *   w_post, w_pre [C] fp32      1 <= C <= 8192, any value; gate_tokens divides R
 *
 * u is formed from r before its rounding.  Sums and norms are fp32 (a row whose
 * squares sum to 2^128 or more has an infinite norm).  r may be x
 * or y itself and u may be y (whole buffers); outputs overlap nothing else.
 */
int gdn_block_norm_forward(const void *x, const void *y, const void *gate, const float *w_post,
                           const float *w_pre, void *r, void *u, int R, int C, int gate_tokens,
                           float res_scale, float eps, int is_bf16, void *stream);

/*
 * Its gradient: from du = dL/du and dr = dL/dr (NULL: zero; what reaches r
 * otherwise than through u),
 *
 *   dx [R][C] E, dy [R][C] E, dgate [R / gate_tokens][C] E (NULL if and only if
 *   gate is), dw_post, dw_pre [C] fp32.
 *
 * r and the norms are formed again from x and y.  The sums over rows run in a
 * fixed order in fp32 (results are deterministic); dgate is rounded once, at
 * its end.  dx may be dr or du and dy may be y or the other of them (whole
 * buffers); outputs overlap nothing else.  `ws`: caller-owned device buffer, 256-byte
 * aligned, of at least gdn_block_norm_workspace_bytes(...) bytes (0 for
 * arguments that the call refuses); calls that run at once need one each.
 */
size_t gdn_block_norm_workspace_bytes(int R, int C, int gate_tokens);

int gdn_block_norm_backward(const void *x, const void *y, const void *gate, const float *w_post,
                            const float *w_pre, const void *du, const void *dr, void *dx, void *dy,
                            void *dgate, float *dw_post, float *dw_pre, int R, int C, int gate_tokens,
                            float res_scale, float eps, int is_bf16, void *ws, size_t ws_bytes,
                            void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GDN_OPS_H */
