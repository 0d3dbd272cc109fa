/*
 * def_train.h -- operators of a language model's training step around def_step, on one B200 (sm_100a).
 *
 * def_step (def.h) consumes fp32 gradient rows; these calls are parts of the forward and backward passes that produce
 * them, with activations kept between the two in 8 bits, and of what is done with them before the step:
 *
 *   def_norm_*        root-mean-square norms before and after a block, fused with the block's gate and residual scale
 *   def_checkpoint_*  8-bit activation checkpoints, and the weight gradient taken straight from one
 *   def_gated_*       the gated activation, its checkpoints, and its backward pass from them
 *   def_logprob_*     log probabilities of given tokens with entropy and top alternatives, and their gradient
 *   def_recurrence_*  a gated linear recurrence over the tokens of packed sequences, with states kept between calls
 *   def_feed_forward* the gated feed-forward block, activation and checkpoints in the products' own kernels
 *   def_orthogonalize orthogonalised weight gradients (Newton-Schulz products), of one or of all workers' rows
 *
 * Conventions (beyond those of def.h)
 *   - Activations are rows [T, C]: T tokens, C consecutive elements of type `dtype` (DEF_DTYPE_*), row stride ld >= C
 *     in ELEMENTS.  Parameters, statistics and parameter gradients are fp32.  Any T >= 0 (0 is a no-op unless a call
 *     says otherwise; below 2^31 for weight gradients and log probabilities); offsets are 64-bit, and widths (C, F, O, I, V) are
 *     at most 2^30.
 *   - Arithmetic and sums are fp32 (the weight gradient: exact products, fp32 sums), rounded once when an output is
 *     stored.  Sums over tokens are taken in a fixed order: repeated calls give identical bits.
 *   - Rows whose base and stride are multiples of 16 bytes (and whose width is one of 8) run on 128-bit accesses; others on
 *     the aligned words around them, at a third to two thirds of that speed.
 *   - There is no context; calls may come from any host threads at the same time.  Work is enqueued on `cuda_stream` (a cudaStream_t, NULL = legacy default stream) of the
 *     current device; nothing is allocated or synchronised.  A workspace is device memory, 16-byte aligned, that the
 *     call may overwrite; calls that overlap on the GPU need one each.
 *   - Outputs must overlap no other argument (DEF_ERR_ALIAS) except where a call allows it.  Column halves of one
 *     buffer (same row stride) do not overlap.
 *   - Errors as in def.h: DEF_ERR_ARG, _NULL, _ALIGN, _ALIAS, _DEVICE, _CUDA; nothing is launched then.
 */
#ifndef DEF_TRAIN_B200_H
#define DEF_TRAIN_B200_H

#include <stdint.h>

#include "def.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { DEF_DTYPE_F32 = 0, DEF_DTYPE_BF16 = 1, DEF_DTYPE_F16 = 2 };

#define DEF_CHECKPOINT_GROUP 32   /* columns of a row that share one exponent            */
#define DEF_NORM_MAX_C 16384      /* widest row of def_norm_*                            */
#define DEF_LOGPROB_MAX_TOP 32    /* most alternatives def_logprob_* returns             */
#define DEF_ORTHOGONALIZE_MAX_STEPS 32

/*
 * The 8-bit checkpoint of X [T, C] (the OCP microscaling layout for 8-bit integers): each run of 32 consecutive
 * columns of a row (the last may be shorter) shares a power-of-two step,
 *     k = max(floor(log2 max|x|) - 6, -126),   e = k + 127,   q = clamp(round-to-nearest-even(x 2^-k), -127, 127),
 * and stands for x^ = q 2^(e - 127): |x^ - x| <= 2^(k-1), except that magnitudes above 127.5 steps are held as 127.
 * A group that holds an infinity or a NaN has e = 255 and q = 0 and reads back as NaN; an all-zero group has e = 1.
 * q: [T, ldq] int8, e: [T, lde] uint8, rows padded to the strides below (padding is neither read as data nor written):
 *     ldq = 16 ceil(C / 16),  lde = 4 ceil(ceil(C / 32) / 4).
 * Bases: q 16-byte, e 4-byte aligned.  x^ is exact in bf16 and fp32; in fp16 it is rounded where it leaves fp16's range.
 */
int def_checkpoint_layout(int64_t C, int64_t *ldq_out, int64_t *lde_out);

/* q, e <- checkpoint of x [T, C]. */
int def_checkpoint_pack(int32_t dtype, int64_t T, int64_t C, const void *x, int64_t ldx, int8_t *q, uint8_t *e,
                        void *cuda_stream);

/* out [T, C] <- the values the checkpoint stands for, rounded to `dtype`. */
int def_checkpoint_unpack(int32_t dtype, int64_t T, int64_t C, const int8_t *q, const uint8_t *e, void *out,
                          int64_t ldout, void *cuda_stream);

/*
 * The weight gradient of a linear layer Y = X W^T whose input was kept as a checkpoint:
 *     dw[o, i]  (+)=  sum_t dy[t, o] x^[t, i]        o < O, i < I
 * dy [T, O] of type dtype, dw [O, I] fp32 with row stride I (4-byte aligned: a layer's slice of one of def_step's
 * gradient rows).  accumulate != 0 adds to dw, 0 overwrites it (T = 0 then writes zeros).  With an fp16 dy, x^ is taken
 * in fp16.  Products are exact; they are summed in fp32.
 * The workspace holds partial products where tokens are split over CTAs, and a 16-byte aligned copy of dy in 16-bit
 * pieces where dy is fp32 or its rows are not multiples of 16 bytes; the second call says how much is needed for the
 * same arguments (at most 68 MiB + 8 O I + 6 T (O + 7) bytes).
 */
int def_checkpoint_weight_grad(int32_t dtype, int64_t T, int64_t O, int64_t I, const void *dy, int64_t lddy,
                               const int8_t *q, const uint8_t *e, float *dw, int32_t accumulate, void *workspace,
                               int64_t workspace_bytes, void *cuda_stream);
int def_checkpoint_weight_grad_workspace(int32_t dtype, int64_t T, int64_t O, int64_t I, const void *dy, int64_t lddy,
                                         int64_t *bytes_out);

/*
 * Gated activation h = silu(g) u, silu(g) = g / (1 + exp(-g)), on [T, F] rows; g and u may be column halves of one
 * projection's output.  gate_q/gate_e and up_q/up_e: checkpoints of g and u for def_gated_backward; each pair both
 * NULL or both given.
 */
int def_gated_forward(int32_t dtype, int64_t T, int64_t F, const void *gate, int64_t ldg, const void *up, int64_t ldu,
                      void *h, int64_t ldh, int8_t *gate_q, uint8_t *gate_e, int8_t *up_q, uint8_t *up_e,
                      void *cuda_stream);

/*
 * Its backward pass from the checkpoints (g^, u^), s = 1 / (1 + exp(-g^)):
 *     dgate = dh u^ s (1 + g^ (1 - s)),   dup = dh g^ s,   h^ = g^ s u^
 * h^, the recomputed product (the next layer's input), is written as values (h_out [T, F] of type dtype) and / or as a
 * checkpoint of those values (h_q, h_e); NULL skips either.
 */
int def_gated_backward(int32_t dtype, int64_t T, int64_t F, const void *dh, int64_t lddh, const int8_t *gate_q,
                       const uint8_t *gate_e, const int8_t *up_q, const uint8_t *up_e, void *dgate, int64_t lddg,
                       void *dup, int64_t lddu, void *h_out, int64_t ldh, int8_t *h_q, uint8_t *h_e, void *cuda_stream);

/*
 * The norms on both sides of a residual connection, in one pass over the rows:
 *     rstd_post = rsqrt(mean(b^2) + eps)
 *     h'        = res_scale h + gate[group] (b rstd_post w_post)
 *     rstd_pre  = rsqrt(mean(h'^2) + eps)
 *     n         = h' rstd_pre w_pre
 * h [T, C]: the residual stream; b [T, C]: the block's output; n: the next block's input.  gate [groups, C]: T must be
 * a multiple of groups, row t uses gate row t / (T / groups) (one row for all tokens, or one for each of equally long
 * sequences); gate NULL means 1.  n is formed from h' before it is rounded.  h_out may be h itself (same stride).
 * b NULL: there is no block yet: n = norm(h) only; w_post, gate, h_out, rstd_post and b_q, b_e must then be NULL.
 * The q / e pairs, each both NULL or both given: checkpoints of b, of h' and of n as stored.
 * C <= DEF_NORM_MAX_C.
 */
int def_norm_forward(int32_t dtype, int64_t T, int64_t C, const void *h, int64_t ldh, const void *b, int64_t ldb,
                     const float *w_post, const float *gate, int64_t groups, const float *w_pre, float res_scale,
                     float eps, void *h_out, int64_t ldho, void *n_out, int64_t ldn, float *rstd_post, float *rstd_pre,
                     int8_t *b_q, uint8_t *b_e, int8_t *h_q, uint8_t *h_e, int8_t *n_q, uint8_t *n_e,
                     void *cuda_stream);

/*
 * Its backward pass.  dn, dh_in [T, C]: gradients of n and of h' (dh_in NULL: zero).  h (that is, h') and b are given
 * as stored (pointer and stride, q and e NULL) or as checkpoints (pointer NULL).  With x = h' rstd_pre, y = b rstd_post,
 * a = dn w_pre:
 *     D  = dh_in + rstd_pre (a - x mean(a x))                 dh = res_scale D
 *     c  = D gate w_post,  db = rstd_post (c - y mean(c y))
 *     dw_pre = sum_t dn x,   S[g] = sum_{t in group g} D y,   dgate[g] = w_post S[g],   dw_post = sum_g gate[g] S[g]
 * dw_pre, dw_post [C] and dgate [groups, C] are fp32; accumulate != 0 adds to them.  dgate is NULL if and only if gate
 * is.  res_scale is a constant.  dh may be dh_in itself (same stride).
 * b absent (no pointer, no checkpoint): the backward pass of n = norm(h); w_post, gate, rstd_post, db, dw_post, dgate
 * must be NULL.  T = 0 writes zeros to the parameter gradients unless accumulate is set.
 * groups is below 2^31.  The workspace holds partial sums; the second call says how much is needed.
 */
int def_norm_backward(int32_t dtype, int64_t T, int64_t C, const void *dn, int64_t lddn, const void *dh_in,
                      int64_t lddhi, const void *h, int64_t ldh, const int8_t *h_q, const uint8_t *h_e, const void *b,
                      int64_t ldb, const int8_t *b_q, const uint8_t *b_e, const float *w_post, const float *gate,
                      int64_t groups, const float *w_pre, float res_scale, const float *rstd_post,
                      const float *rstd_pre, void *dh, int64_t lddh, void *db, int64_t lddb, float *dw_post,
                      float *dgate, float *dw_pre, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                      void *cuda_stream);
int def_norm_backward_workspace(int64_t T, int64_t C, int64_t groups, int64_t *bytes_out);

/*
 * Log probabilities from logits x [T, V], in one pass, p = softmax(x):
 *     m = max_j x_j,   l = log sum_j exp(x_j - m),   logp = (x_y - m) - l,   entropy = -sum_j p_j log p_j,
 *     top_ids [T, top], top_logp [T, top]: the `top` largest logits, largest first, ties by lowest index, and their
 *     log probabilities.
 * lse [T, 2] holds (m, l): the log of the row's sum in two parts, so that log probabilities near 0 keep their digits
 * where the logits are large.  0 <= top <= min(V, DEF_LOGPROB_MAX_TOP); top_ids and top_logp are NULL if and only if top = 0.
 * targets y [T] int64.  y < 0: the token is ignored (logp 0, and no gradient through logp).  y >= V: logp is NaN.
 * Logits at or below -1e30 (-infinity, and the lowest values of bf16 and fp32) are masked: in a row with others, p = 0 and
 * they add nothing to the entropy.  A row that is masked throughout: lse is (-infinity, 0), logp (0 <= y < V) and top_logp
 * are -infinity, the entropy is 0.  A NaN or +infinity makes l, logp (y >= 0), entropy and top_logp NaN; a NaN
 * ranks with -infinity among the alternatives.
 */
int def_logprob_forward(int32_t dtype, int64_t T, int64_t V, const void *logits, int64_t ldx, const int64_t *targets,
                        float *logp, float *entropy, float *lse, int32_t top, int64_t *top_ids, float *top_logp,
                        void *cuda_stream);

/*
 * The gradient of logits from those of logp, entropy and top_logp (dlogp, dentropy [T], dtop_logp [T, top]; each may be
 * NULL, with top = 0 where dtop_logp is), with lse and entropy of the forward call:
 *     dx_j = -p_j [ G + dentropy (log p_j + H) ] + dlogp [j = y] + sum_i dtop_i [j = id_i],   G = dlogp + sum_i dtop_i
 * (dlogp counts as 0 where y < 0).  A row that is masked throughout gets 0.
 * y >= V: the row's gradient is NaN where dlogp is given.  Every top id must be in [0, V) (others are skipped).
 * dlogits may be logits itself (same stride).
 */
int def_logprob_backward(int32_t dtype, int64_t T, int64_t V, const void *logits, int64_t ldx, const int64_t *targets,
                         const float *lse, const float *entropy, const float *dlogp, const float *dentropy,
                         int32_t top, const int64_t *top_ids, const float *dtop_logp, void *dlogits, int64_t lddx,
                         void *cuda_stream);

/*
 * Gated linear recurrence over the tokens of packed sequences, channel by channel:
 *     c_t = 1 / (1 + exp(g_t)),  a_t = 1 - c_t,     h_t = a_t h_{t-1} + c_t x_t,     y_t = h_t
 * x, gate (the logits g), y: [T, C], T <= 2^30.  Sequence s holds rows [offsets[s], offsets[s + 1]) (offsets: sequences + 1
 * numbers in device memory, 8-byte aligned, not decreasing; sequences may be empty), or, with offsets NULL, the s-th of
 * `sequences` equally long runs (T must be a multiple).  Rows of no sequence are not written, and what they hold does not matter.  Offsets that
 * decrease or leave [0, T] do no harm outside the arguments, but what is computed then is not specified.
 * h0, h_last [sequences, C] fp32: the state before a sequence's first token (NULL: 0) and behind its last one (NULL: not
 * written; a sequence without tokens hands on its h0; h_last is other memory than h0).  y may be x itself (same stride) where no
 * backward pass will need x.
 * One token of each sequence: T = sequences, offsets NULL, h_last of one call is the next one's h0.
 * The state is fp32.  What is handed on, from run to run of 8 or 16 steps and in h_last, is free of the rounding of 1 - c, so that memories
 * of many tokens (c of 2^-17 and less) do not drift by up to 2^-25 of the state a step.  An infinity or a NaN stays within its sequence
 * and channel.
 * The workspace holds maps of parts of long narrow calls; def_recurrence_workspace says how much is needed (at most
 * 4096 C bytes; the same forward and backward).
 */
int def_recurrence_forward(int32_t dtype, int64_t T, int64_t C, int64_t sequences, const int64_t *offsets, const void *x,
                           int64_t ldx, const void *gate, int64_t ldg, const float *h0, void *y, int64_t ldy, float *h_last,
                           void *workspace, int64_t workspace_bytes, void *cuda_stream);
int def_recurrence_workspace(int32_t dtype, int64_t T, int64_t C, int64_t *bytes_out);

/*
 * Its backward pass, from y as stored by the forward call.  With h_{t-1} = y_{t-1} (h0 or 0 before the first token):
 *     lambda_t = dy_t + a_{t+1} lambda_{t+1}   (the last token: dy_t + dh_last, dh_last NULL: 0)
 *     dx_t = c_t lambda_t,   dgate_t = lambda_t a_t c_t (h_{t-1} - x_t),   dh0 = a_1 lambda_1 of the first token
 * dh0 [sequences, C] may be NULL; without tokens it is dh_last.  dx and dgate overlap no input.
 */
int def_recurrence_backward(int32_t dtype, int64_t T, int64_t C, int64_t sequences, const int64_t *offsets, const void *dy,
                            int64_t lddy, const float *dh_last, const void *x, int64_t ldx, const void *gate, int64_t ldg,
                            const void *y, int64_t ldy, const float *h0, void *dx, int64_t lddx, void *dgate, int64_t lddg,
                            float *dh0, void *workspace, int64_t workspace_bytes, void *cuda_stream);

/*
 * Gated feed-forward block, one kernel per product, with the activation in the first one's epilogue:
 *     [g | u] = x w_in^T,   h = silu(g) u,   out = h w_down^T
 * x [T, C], h [T, F], out [T, O]; w_in [2F, C]: the gate's F rows, then those of u, and w_down [O, F], both contiguous, of
 * type dtype.  g and u stay in fp32; h is rounded to dtype once, and the second product takes it so.  w_down and out NULL:
 * h only.  gate_q/gate_e, up_q/up_e: checkpoints of g and u (of the fp32 values) for the backward pass; all NULL or all given.
 * 16-bit types: exact products, summed in fp32 by the matrix unit, which truncates: of sums of one sign at most 3 10^-5 is lost (fp16;
 * bf16: 3 10^-4), however many terms, less than a tenth of the rounding of the result.  fp32: operands in three bf16 pieces of 8 bits, the
 * six products of pieces that reach 2^-24 (an infinity may give NaN).  T <= 2^30, F <= 2^29.
 * The workspace holds partial products where k is cut over CTAs, the pieces of fp32 operands, and aligned copies of operands
 * whose rows are not multiples of 16 bytes or do not start on them; the second call says how much is needed for the same
 * arguments: at most, with r(n) = n + 7 and P = 3 for fp32, 1 else, 20 MiB + 2 P (T r(C) + 2F r(C) + T r(F) + O r(F)) bytes.
 */
int def_feed_forward(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *x, int64_t ldx, const void *w_in,
                     const void *w_down, void *h, int64_t ldh, void *out, int64_t ldout, int8_t *gate_q, uint8_t *gate_e,
                     int8_t *up_q, uint8_t *up_e, void *workspace, int64_t workspace_bytes, void *cuda_stream);
int def_feed_forward_workspace(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *x, int64_t ldx,
                               const void *w_in, const void *w_down, const void *h, int64_t ldh, int64_t *bytes_out);

/*
 * Its backward pass from the checkpoints (g^, u^), s = 1 / (1 + exp(-g^)):
 *     dh = dout w_down,   dgate = dh u^ s (1 + g^ (1 - s)),   dup = dh g^ s,   dx = [dgate | dup] w_in,   h^ = g^ s u^
 * dout [T, O]; dboth [T, 2F]: dgate in its first F columns, dup in the others; dx [T, C] (w_in and dx NULL: not computed).
 * dh stays in fp32; dboth is rounded to dtype once, and the product for dx takes it so.  h^ is written as values (h_out
 * [T, F]) and / or as a checkpoint of those values (h_q, h_e); NULL skips either.  The weights' gradients are
 * def_checkpoint_weight_grad of dboth with the checkpoint of x, and of dout with that of h^.
 * The workspace is as above, for dout, w_down, dboth and w_in.
 */
int def_feed_forward_backward(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *dout, int64_t lddout,
                              const void *w_in, const void *w_down, const int8_t *gate_q, const uint8_t *gate_e,
                              const int8_t *up_q, const uint8_t *up_e, void *dboth, int64_t lddb, void *dx, int64_t lddx,
                              void *h_out, int64_t ldh, int8_t *h_q, uint8_t *h_e, void *workspace,
                              int64_t workspace_bytes, void *cuda_stream);
int def_feed_forward_backward_workspace(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *dout,
                                        int64_t lddout, const void *w_in, const void *w_down, const void *dboth, int64_t lddb,
                                        int64_t *bytes_out);

/*
 * Orthogonalises updates: for each matrix x [rows, cols] of the batch, with X = x / (|x|_F + eps) (transposed if tall) and the
 * steps' coefficients (a, b, c) in turn,
 *     A = X X^T,   X <- (a I + b A + c A A) X,        out = scale X
 * which takes each singular value s to s (a + b s^2 + c s^4) and leaves the singular vectors.  coeffs: 3 * steps numbers in HOST
 * memory, read before the call returns, each within 8 of 0 (within 64 where the polynomials keep singular values that start in
 * [0, 1] below 4 and a + b s^2 + c s^4 below 16, as far as can be told from the coefficients); 1 <= steps <= DEF_ORTHOGONALIZE_MAX_STEPS.
 * Matrix i of x starts at element i * stride_x and has rows of ldx; out likewise.  So one call serves a weight in all W rows of
 * def_step's gradients (stride d), at any 4-byte address, and in place: out may be x itself (same strides).
 * rows, cols and batch are at most 2^16; batch = 0 is a no-op.
 * The norm is summed in 64 bits.  X, A and B are held in 22 bits (two fp16 pieces each), products are exact and summed in
 * fp32.  Singular values have to stay below 4 and the entries of B below 16 (larger ones give infinities and NaN), as they do
 * for polynomials that converge on [0, 1]; the 22 bits are relative to 1, so a matrix whose norm is far below eps loses
 * digits.  A matrix of zeros gives zeros; a NaN or an infinity makes its whole matrix NaN, and no other.
 * The workspace is at most batch (16 (m + 8) (n + m + 16) + 8192) bytes, m <= n the sides; the second call says how much.
 */
int def_orthogonalize(int32_t dtype, int64_t batch, int64_t rows, int64_t cols, const void *x, int64_t ldx,
                      int64_t stride_x, void *out, int64_t ldo, int64_t stride_o, const float *coeffs, int32_t steps,
                      float eps, float scale, void *workspace, int64_t workspace_bytes, void *cuda_stream);
int def_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols, int64_t *bytes_out);

#ifdef __cplusplus
}
#endif
#endif /* DEF_TRAIN_B200_H */
