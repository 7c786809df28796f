/*
 * t2i_ops.h -- kernel-level entry points of the denoising step.
 *
 * The same kernels t2i_dit_step launches, exposed one by one so that each can
 * be checked against its definition in isolation, and operators of transformer
 * blocks that the models above do not have: an 8-bit linear layer, a gated
 * feed-forward with its gradients, query / key norm with rotation and its
 * gradients, the residual's addition with an RMS norm and its gradients, a linear
 * layer with a low-rank adapter per row and their gradients, an AdamW step.
 * Conventions are those of
 * t2i_dit.h: device pointers are caller-owned HIP memory, `stream` is a
 * hipStream_t as void*, launches are asynchronous, arguments are validated
 * before any launch, errors come back as t2i_status (text in
 * t2i_ops_last_error(), per host thread).
 */
#ifndef T2I_OPS_H
#define T2I_OPS_H

#include <stdint.h>
#include "t2i_dit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogues of the linear layer y = A W^T + b. */
typedef enum {
  T2I_EPI_STORE = 0,       /* out = y */
  T2I_EPI_GELU = 1,        /* out = GELU_tanh(y) */
  T2I_EPI_SILU = 2,        /* out = SiLU(y) */
  T2I_EPI_RESID = 3,       /* resid += y  (fp32), resid_copy = bf16(resid) */
  T2I_EPI_RESID_GATED = 4  /* resid += gate (.) y, gate a [N] fp32 vector */
} t2i_epilogue;

/*
 * Linear layer (DiT projections, Sec. 4's model `forward`): y = A W^T + b,
 * A [M, K] with row stride lda, W [N, K] with row stride ldw, b [N].
 *   dtype T2I_BF16: A, W, b bf16, MFMA with fp32 accumulation, K % 64 == 0,
 *                   lda, ldw % 8 == 0.  `out` is bf16.  A and W that start
 *                   at a multiple of 16 bytes are loaded straight into LDS,
 *                   others through registers: same results, more time.
 *   dtype T2I_F32 : A, W, b, out fp32.
 * For T2I_EPI_RESID*: `resid` is fp32 [M, N] (stride ldr) updated in place,
 * `resid_copy` (bf16 [M, N], stride ldr, or NULL) receives its new value;
 * `out` is unused.  `gate` is fp32 [N] (T2I_EPI_RESID_GATED only).
 */
t2i_status t2i_op_linear(int32_t dtype, int32_t epilogue, int32_t M, int32_t N,
                         int32_t K, const void* A, int32_t lda, const void* W,
                         int32_t ldw, const void* bias, void* out, int32_t ldo,
                         float* resid, int32_t ldr, void* resid_copy,
                         const float* gate, void* stream);

/*
 * Multi-head attention softmax(Q K^T / sqrt(d)) V over packed variable-length
 * sequences (the DiT's self- and cross-attention, Sec. 4's model `forward`;
 * joint text+image attention of the Sec. 8.1 model family): query sequence s
 * holds rows q_start[s] .. q_start[s]+q_len[s]-1 of Q and attends to rows
 * k_start[s] .. +k_len[s]-1 of K and V and, when k2_start/k2_len are given
 * (both or neither), also to rows k2_start[s] .. +k2_len[s]-1 -- the joint
 * attention's text keys and image keys, wherever each stream's rows sit.
 * Host arrays of n_seq <= T2I_MAX_SEQ entries; k_len + k2_len >= 1.  Head h of
 * a row occupies columns h*d .. h*d+d-1.  Q, K, O are dtype (bf16 or fp32)
 * with row strides ldq, ldk, ldo (multiples of 8).
 *   fp32: V is row-major like K, row stride ldv.
 *   bf16: V is given transposed, V^T [heads*head_dim][ldv] (the key index is
 *         contiguous), the layout the fused qkv projection writes; every key
 *         segment must start at a multiple of 8 and end within ldv.  The
 *         kernel addresses K and V^T with 32-bit byte offsets:
 *         2*heads*head_dim*ldv and 2*(last key row + 64)*ldk must stay below
 *         2^31, else T2I_ERR_SHAPE.
 */
t2i_status t2i_op_attention(int32_t dtype, int32_t heads, int32_t head_dim,
                            int32_t n_seq, const int32_t* q_start,
                            const int32_t* q_len, const int32_t* k_start,
                            const int32_t* k_len, const int32_t* k2_start,
                            const int32_t* k2_len, const void* q, int32_t ldq,
                            const void* k, int32_t ldk, const void* v,
                            int32_t ldv, void* o, int32_t ldo, void* stream);

/*
 * Cross-attention of image queries to their request's text (Sec. 4's model
 * `forward`, the DiT block's attention to the caption): the operation of
 * t2i_op_attention with one key segment per sequence, bf16 only (else
 * T2I_ERR_INVALID_ARG), run by the kernels the model uses for it where it
 * does not fuse it into the query projection (t2i_op_linear_cross_attention)
 * -- texts of at most 128 keys (k_len 1..128) by the two-tile kernel that
 * keeps them in LDS across query tiles, longer texts by the pipelined one.
 * Arguments, layouts (V given transposed) and limits are those of
 * t2i_op_attention.
 */
t2i_status t2i_op_cross_attention(int32_t dtype, int32_t heads, int32_t head_dim,
                                  int32_t n_seq, const int32_t* q_start,
                                  const int32_t* q_len, const int32_t* k_start,
                                  const int32_t* k_len, const void* q, int32_t ldq,
                                  const void* k, int32_t ldk, const void* v,
                                  int32_t ldv, void* o, int32_t ldo, void* stream);

/*
 * The DiT block's cross-attention together with its query projection (Sec. 4's
 * model `forward`): q = A W^T + b for the query rows, then the operation of
 * t2i_op_cross_attention with those queries, bf16 only.  The queries are
 * kept multiplied by log2(e)/sqrt(head_dim) (rounded once to bf16, as the
 * model's projection writes them), so the softmax takes base-2 exponentials
 * of the scores directly.
 *   A [M, K] (row stride lda) with M = the largest q_start[s] + q_len[s];
 *   W [heads*head_dim, K] (row stride ldw), bias [heads*head_dim];
 *   K % 64 == 0, lda, ldw >= K and multiples of 8; text of 1 .. 128 keys per
 *   sequence (k_len), key starts % 8 == 0; K/V layouts (V given transposed),
 *   ldk, ldv, ldo and the 2^31-byte limits as for t2i_op_attention.
 * fused = 0: the projection writes the queries to q_buf [M, ldq] (caller-
 *   owned, ldq >= heads*head_dim, % 8 == 0), then the cross-attention kernel
 *   reads them: two launches.
 * fused = 1: one kernel; the queries never leave the chip (q_buf unused, may
 *   be NULL).  Needs head_dim 72, K % 192 == 0, sequences contiguous from
 *   row 0 whose lengths are multiples of 256, 16-byte aligned A, W, K, V and o,
 *   8-byte aligned bias, else T2I_ERR_SHAPE.  Both settings give the
 *   same bits; the model takes the fused one from 2048 rows wherever it
 *   applies.
 */
t2i_status t2i_op_linear_cross_attention(int32_t fused, int32_t heads, int32_t head_dim,
                                         int32_t n_seq, const int32_t* q_start,
                                         const int32_t* q_len, const int32_t* k_start,
                                         const int32_t* k_len, int32_t K, const void* A,
                                         int32_t lda, const void* W, int32_t ldw,
                                         const void* bias, const void* k, int32_t ldk,
                                         const void* v, int32_t ldv, void* q_buf,
                                         int32_t ldq, void* o, int32_t ldo, void* stream);

/*
 * LayerNorm (no affine, biased variance) fused with adaLN modulation:
 * out = (x - mean) / sqrt(var + eps) * (1 + scale) + shift per row of
 * x [rows, D] fp32; shift, scale fp32 [D]; out dtype (bf16 or fp32) [rows, D].
 * D % 4 == 0, D <= 3072; x and shift 16-byte aligned, out 8-byte (bf16) or
 * 16-byte (fp32) aligned.
 */
t2i_status t2i_op_ln_modulate(int32_t dtype, int32_t rows, int32_t D,
                              const float* x, const float* shift,
                              const float* scale, float eps, void* out,
                              void* stream);

/*
 * LoRA weight update merged on the device before sampling (the paper's
 * weight-update adapters, Sec. 2.2 / Sec. 3, which modify base-model weights
 * before inference): W <- W + alpha * B A for one linear layer, in place.
 *   W [n_out, n_in] with row stride ldw, A [rank, n_in] (row stride n_in),
 *   B [n_out, rank] (row stride rank), all of dtype (bf16 or fp32);
 *   1 <= rank <= 128.  The product is accumulated in fp32 over rank, added to
 *   W in fp32 and rounded once to W's dtype (round-to-nearest-even).
 * W is caller-owned memory (e.g. a tensor bound to a t2i_dit handle: merge
 * between calls, not during one).
 */
t2i_status t2i_op_lora_merge(int32_t dtype, int32_t n_out, int32_t n_in, int32_t rank,
                             float alpha, void* W, int32_t ldw, const void* A,
                             const void* B, void* stream);

/*
 * The LoRA merge of t2i_op_lora_merge for n weights of one shape (an adapter
 * applied to every layer of one kind: n_out, n_in, rank, ldw shared), weight
 * i at W[i] with its own A[i], B[i] -- host arrays of n device pointers.
 * Results are those of n t2i_op_lora_merge calls, bitwise; one launch per 64
 * weights instead of one each.  The weights must not overlap.
 */
t2i_status t2i_op_lora_merge_batch(int32_t dtype, int32_t n, int32_t n_out, int32_t n_in,
                                   int32_t rank, float alpha, void* const* W, int32_t ldw,
                                   const void* const* A, const void* const* B, void* stream);

/*
 * Rows quantised to 8 bits with one scale each, the input of the 8-bit linear
 * layer (activations per token, weights per output channel):
 *   scale[r] = max(max_k |x[r, k]| / 127, 2^-126), rounded once to fp32;
 *   q[r, k]  = x[r, k] / scale[r] to the nearest whole number, ties to even
 *              (of the exact quotient; -127 .. 127).
 * A row that holds a NaN or an infinity gets scale NaN and q = 0.
 *   x [rows, K] of dtype (bf16 or fp32), row stride ldx >= K, any alignment of
 *   its type; q [rows, ldq] with ldq % 16 == 0, ldq >= K rounded up to a
 *   multiple of 128, 16-byte aligned: columns K .. that multiple are written
 *   as zeros, columns behind it are left alone; scale [rows] fp32.  Fewer than
 *   2^26 - 4 rows (K > 2048: 2^24 - 4).
 */
t2i_status t2i_op_quant_rows(int32_t dtype, int32_t rows, int32_t K, const void* x, int32_t ldx,
                             int8_t* q, int32_t ldq, float* scale, void* stream);

/*
 * Linear layer in 8-bit integers with a scale for every row of A (token) and
 * every row of W (output channel), with the epilogues of t2i_op_linear:
 *   y[m, n] = a_scale[m] * w_scale[n] * sum_k A[m, k] W[n, k] + bias[n].
 * The sum is exact (32-bit integers, K <= 131071); it is rounded once to fp32,
 * the rest is fp32 (a_scale times the sum first).
 *   A [M, K], W [N, K] int8, 16-byte aligned, row strides lda, ldw multiples of
 *   16, at least K rounded up to a multiple of 128 and below 8 MiB: both are read
 *   up to that multiple, and one of the two must hold zeros behind K
 *   (t2i_op_quant_rows writes them).  dtype is the type of bias [N] (or NULL: none)
 *   and out; the remaining arguments are those of t2i_op_linear.  Fewer than 2^23
 *   pieces of 64 x 64 outputs.
 */
t2i_status t2i_op_linear_i8(int32_t dtype, int32_t epilogue, int32_t M, int32_t N, int32_t K,
                            const int8_t* A, int32_t lda, const float* a_scale, const int8_t* W,
                            int32_t ldw, const float* w_scale, const void* bias, void* out,
                            int32_t ldo, float* resid, int32_t ldr, void* resid_copy,
                            const float* gate, void* stream);

/*
 * Gated feed-forward, first half (both projections, the activation and the
 * product in one kernel; t2i_op_linear is the second half):
 *   g = A Wg^T + bg,  u = A Wu^T + bu,  out = act(g) (.) u,
 * act T2I_EPI_GELU (tanh form) or T2I_EPI_SILU.
 *   A [M, K] (stride lda), Wg and Wu [F, K] (common stride ldw; the halves of
 *   one [2F, K] matrix: Wu = Wg + F ldw), bg and bu [F] (both or neither),
 *   out [M, F] (stride ldo), all of dtype; sums, activation and product in
 *   fp32, one rounding.
 *   pre [M, 2F] fp32 (stride ldp) or NULL: receives g | u, which
 *   t2i_op_gated_linear_backward reads (fp32 for bf16 operands too: rounded to
 *   bf16 they would add a quarter to the gradients' error).
 *   bf16: F, K and the strides % 8 == 0 (ldp % 4), every pointer 16-byte
 *   aligned.  fp32: any sizes, strides and alignment (A, Wg and Wu in whole 16-byte
 *   rows are some percent faster, same results).  Rows of A, Wg and Wu less than 8
 *   MiB apart, fewer than 2^23 pieces of 64 x 64 values in g | u (backward: dA, dWg |
 *   dWu as well).
 * No output may overlap an input.
 */
t2i_status t2i_op_gated_linear(int32_t dtype, int32_t act, int32_t M, int32_t F, int32_t K,
                               const void* A, int32_t lda, const void* Wg, const void* Wu,
                               int32_t ldw, const void* bg, const void* bu, void* out,
                               int32_t ldo, float* pre, int32_t ldp, void* stream);

/*
 * Gradients of t2i_op_gated_linear: with dout [M, F] (stride ldd) the gradient
 * of out and pre the forward pass's,
 *   dg = dout (.) u (.) act'(g),  du = dout (.) act(g),
 *   dA = dg Wg + du Wu [M, K],  dWg = dg^T A,  dWu = du^T A [F, K],
 *   dbg, dbu = column sums of dg, du [F],
 * all of dtype.  dg and du are rounded to dtype once, for the products (the
 * bias sums take them unrounded); products and sums are fp32.  dA (stride
 * ldda), dWg, dWu (common stride lddw) may each be NULL: not computed; dbg and
 * dbu both or neither.  Sizes, strides and alignment as in the forward pass
 * (F below 2^20).
 * ws: device workspace of ws_bytes >= t2i_op_gated_linear_backward_ws_bytes,
 * 256-byte aligned, used by this call until it has finished on the stream;
 * the result does not depend on what it holds.  No output may overlap an
 * input.  Every sum has a fixed order.
 */
size_t t2i_op_gated_linear_backward_ws_bytes(int32_t dtype, int32_t M, int32_t F, int32_t K);
t2i_status t2i_op_gated_linear_backward(int32_t dtype, int32_t act, int32_t M, int32_t F, int32_t K,
                                        const void* A, int32_t lda, const void* Wg, const void* Wu,
                                        int32_t ldw, const float* pre, int32_t ldp, const void* dout,
                                        int32_t ldd, void* dA, int32_t ldda, void* dWg, void* dWu,
                                        int32_t lddw, void* dbg, void* dbu, void* ws,
                                        size_t ws_bytes, void* stream);

/* Which elements of a head make up the rotated pairs. */
typedef enum {
  T2I_ROPE_PAIRS = 0,   /* (2j, 2j + 1), as the joint-attention model's */
  T2I_ROPE_HALVES = 1   /* (j, j + head_dim / 2); head_dim % 16 == 0 */
} t2i_rope_pairing;

/*
 * RMS norm of every head of the queries and keys, then the position rotation,
 * in one pass (before t2i_op_attention):
 *   n = x / sqrt(mean(x^2) + eps) * w,
 *   pair j of the head turned by (cos, sin) = table[p][j]:
 *   (a, b) -> (a cos - b sin, a sin + b cos).
 *   q [rows, heads_q * head_dim] (stride ldq), k [rows, heads_k * head_dim]
 *   (stride ldk; the columns of one fused projection, or buffers of their
 *   own), wq, wk [head_dim] or NULL (ones), outputs q_out, k_out alike, all of
 *   dtype; the arithmetic is fp32, one rounding (squares past fp32 make a head's
 *   outputs 0; with eps 0 a head of zeros gives NaN).  heads_q or heads_k may be 0
 *   (its pointers are then unused); rows * (heads_q + heads_k) < 2^31, and head_dim
 *   times that < 2^34.
 *   table fp32 [n_pos][head_dim / 2][2] of (cos, sin), or NULL: no rotation
 *   (one, two or more position axes: the table's rows say which pair turns by
 *   which angle).  Row r turns by table row pos[r] (device, [rows]), or r when
 *   pos is NULL (then n_pos >= rows).  pos[r] < 0: row r is not turned (text
 *   rows of joint attention); pos[r] >= n_pos: row r's outputs are NaN.
 *   head_dim % 8 == 0, 8 .. 256, strides % 8 == 0, every pointer 16-byte
 *   aligned (pos: 4).
 * In place (q_out == q, ldqo == ldq; the same for k) is allowed, any other
 * overlap of an output with an input is not.  Keep the inputs if the backward
 * pass is to follow.
 */
t2i_status t2i_op_qk_norm_rope(int32_t dtype, int32_t rows, int32_t heads_q, int32_t heads_k,
                               int32_t head_dim, const void* q, int32_t ldq, const void* k,
                               int32_t ldk, const void* wq, const void* wk, float eps,
                               int32_t pairing, const float* table, int32_t n_pos,
                               const int32_t* pos, void* q_out, int32_t ldqo, void* k_out,
                               int32_t ldko, void* stream);

/*
 * Gradients of t2i_op_qk_norm_rope: dq, dk the gradients of q_out, k_out; q, k
 * and the other arguments the forward pass's inputs; dq_in, dk_in receive the
 * gradients of q, k, dwq, dwk [head_dim] (or NULL) those of the weights, summed
 * over rows and heads in a fixed order, all of dtype (a row with pos[r] >= n_pos
 * makes its own gradients and dwq, dwk NaN).  dq_in may be dq itself
 * (same stride), dk_in dk.  ws as in t2i_op_gated_linear_backward (may be NULL
 * when dwq and dwk are).
 */
size_t t2i_op_qk_norm_rope_backward_ws_bytes(int32_t rows, int32_t heads_q, int32_t heads_k,
                                             int32_t head_dim);
t2i_status t2i_op_qk_norm_rope_backward(int32_t dtype, int32_t rows, int32_t heads_q,
                                        int32_t heads_k, int32_t head_dim, const void* dq,
                                        int32_t lddq, const void* dk, int32_t lddk, const void* q,
                                        int32_t ldq, const void* k, int32_t ldk, const void* wq,
                                        const void* wk, float eps, int32_t pairing,
                                        const float* table, int32_t n_pos, const int32_t* pos,
                                        void* dq_in, int32_t lddqi, void* dk_in, int32_t lddki,
                                        void* dwq, void* dwk, void* ws, size_t ws_bytes,
                                        void* stream);

/*
 * The residual's addition and an RMS norm in one pass:
 *   h = resid + x,  r = 1 / sqrt(mean_k(h^2) + eps),  y = h r w,
 * h rounded once to resid's type, which the norm takes then; statistics and
 * products in fp32, y rounded once.
 *   x [rows, K] (stride ldx), w [K] or NULL (ones), y [rows, K] (stride ldy) of
 *   dtype; resid, h [rows, K] (strides ldr, ldh) of resid_dtype: dtype, or
 *   T2I_F32 beside bf16 operands (a residual stream in fp32).  resid NULL: the
 *   norm of x (h unused, resid_dtype must be dtype).  Any alignment and strides
 *   of their types, K <= 2^20; fewer than 2^26 - 4 rows (K > 2048: 2^22).
 *   h may be resid itself (same stride), y may be x; no other overlap of an
 *   output with an input or another output.
 * A row's results do not depend on the rows beside it.  Squares past fp32 make a
 * row's y 0 (an infinity or a NaN in h: NaN); with eps 0 a row of zeros gives NaN, and
 * one whose squares are all below fp32 infinities or NaN.
 */
t2i_status t2i_op_add_rms_norm(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K,
                               const void* x, int32_t ldx, const void* resid, int32_t ldr,
                               const void* w, float eps, void* h, int32_t ldh, void* y,
                               int32_t ldy, void* stream);

/*
 * The same with y in 8 bits and a scale for every row, the input of
 * t2i_op_linear_i8: with t = h w (exact) and T = max_k |t|,
 *   scale = T r / 127 (fp32),
 *   q[k] = 127 t[k] / T to the nearest whole number, ties to even, of the exact
 *          quotient (-127 .. 127; zeros for T = 0): the norm's factor r is in
 *          both and leaves it alone,
 * so that q scale stands for y.  q [rows, ldq] as in t2i_op_quant_rows (16-byte
 * aligned, ldq % 16 == 0, columns K .. K rounded up to 128 written as zeros).  A row
 * whose h or products h w are not finite in fp32 gets scale NaN and q = 0.
 */
t2i_status t2i_op_add_rms_norm_i8(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K,
                                  const void* x, int32_t ldx, const void* resid, int32_t ldr,
                                  const void* w, float eps, void* h, int32_t ldh, int8_t* q,
                                  int32_t ldq, float* scale, void* stream);

/*
 * Gradients of t2i_op_add_rms_norm: dy [rows, K] (stride lddy) of dtype the
 * gradient of y, h (stride ldh; without a residual x) and dh (stride lddh, or
 * NULL: none), of resid_dtype, the sum and its gradient from elsewhere.  With
 * n = h r, d = dy w:
 *   dsum = dh + r (d - n mean_k(d n)), the gradient of x and of resid alike:
 *   dx [rows, K] (stride lddx) of dtype, dresid (stride lddr) of resid_dtype, or
 *   NULL where one type serves both;
 *   dw [K] of dtype (or NULL) = sum over rows of dy n, in a fixed order.
 * Sizes and alignment as forward.  dx may lie over dy or (of its type) dh,
 * dresid over dh, same stride, if K <= 16384; no other overlap.  ws as in
 * t2i_op_gated_linear_backward (NULL without dw, or where it takes no bytes).
 */
size_t t2i_op_add_rms_norm_backward_ws_bytes(int32_t rows, int32_t K);
t2i_status t2i_op_add_rms_norm_backward(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K,
                                        const void* dy, int32_t lddy, const void* h, int32_t ldh,
                                        const void* w, float eps, const void* dh, int32_t lddh,
                                        void* dx, int32_t lddx, void* dresid, int32_t lddr,
                                        void* dw, void* ws, size_t ws_bytes, void* stream);

/*
 * A linear layer shared by the rows of many requests, each with a low-rank adapter of
 * its own or none (t2i_op_lora_merge changes W for everybody instead):
 *   t[m] = s_i A_i x[m],  y[m] = W x[m] + bias + B_i t[m],  i = index[m],
 * then the epilogues of t2i_op_linear.
 *   x [M, K] (stride ldx), w [N, K] (stride ldw), bias [N] or NULL, a
 *   [n][rank][K] and b [n][N][rank] (contiguous; adapters of smaller rank: zeros),
 *   out [M, N] (stride ldo), all of dtype; scale fp32 [n]
 *   or NULL (ones); index (device, [M]) or NULL: every row takes adapter 0.  A row
 *   whose index is not in 0 .. n - 1 takes no adapter.  The rest as t2i_op_linear.
 *   Products and sums in fp32, one rounding; bf16 operands meet all of t's bits, and an
 *   infinity among them makes infinities and NaN as in fp32 (of t and the gradients' u
 *   from 2^-86).  t fp32 receives rank columns and zeros up to rank rounded up to 32
 *   (ldt at least that, % 8 == 0, 16-byte aligned): scratch memory, or kept for
 *   t2i_op_adapter_linear_backward.
 *   bf16: N, K, ldx, ldw % 8 == 0, x, w, a 16-byte aligned.  fp32: any sizes, strides
 *   and alignment.  1 <= rank <= 128, n <= 32767, n max(N, K) times
 *   rank rounded up to 8 below 2^32; M <= 2^24,
 *   fewer than 2^23 pieces of 64 x 64 outputs; rows of x and w less than 8 MiB apart.
 * Any order of the index; rows of one adapter next to each other are faster.  For t,
 * rows whose neighbours (16 or 32 of them) take more than three adapters are brought
 * together within 4096 rows, but not with more than 512 adapters or rows of x 512 KiB
 * and more apart (4096 x 4096 x 4096, rank 16, scattered over 512 adapters 382 us, over
 * 520 460).  Nothing
 * of another row's adapter enters a row's sums, not even as zeros.  No output may
 * overlap an input or another output.
 */
t2i_status t2i_op_adapter_linear(int32_t dtype, int32_t epilogue, int32_t M, int32_t N, int32_t K,
                                 const void* x, int32_t ldx, const void* w, int32_t ldw,
                                 const void* bias, int32_t n, int32_t rank, const void* a,
                                 const void* b, const float* scale, const int32_t* index, float* t,
                                 int32_t ldt, void* out, int32_t ldo, float* resid, int32_t ldr,
                                 void* resid_copy, const float* gate, void* stream);

/*
 * Gradients of t2i_op_adapter_linear (T2I_EPI_STORE) for adapters trained beside a frozen
 * layer: with dy [M, N] (stride lddy) the gradient of y and t the forward pass's,
 *   u[m] = s_i B_i^T dy[m],
 *   dx[m] = W^T dy[m] + A_i^T u[m]   [M, K] (stride lddx),
 *   da_i = sum over the rows of adapter i of u[m] x[m]^T   [n][rank][K],
 *   db_i = sum of dy[m] t[m]^T   [n][N][rank],
 * all of dtype; zeros for an adapter that no row takes.  Products and sums are fp32 or
 * more, in a fixed order.  dx, da, db may each be NULL:
 * not computed.  Sizes and alignment as forward (dy as x); b 16-byte aligned; the
 * slices of the sums must fit a launch (T2I_ERR_SHAPE).  ws as in
 * t2i_op_gated_linear_backward.  No output may overlap an input.
 */
size_t t2i_op_adapter_linear_backward_ws_bytes(int32_t dtype, int32_t M, int32_t N, int32_t K,
                                               int32_t n, int32_t rank);
t2i_status t2i_op_adapter_linear_backward(int32_t dtype, int32_t M, int32_t N, int32_t K,
                                          const void* dy, int32_t lddy, const void* x, int32_t ldx,
                                          const void* w, int32_t ldw, int32_t n, int32_t rank,
                                          const void* a, const void* b, const float* scale,
                                          const int32_t* index, const float* t, int32_t ldt,
                                          void* dx, int32_t lddx, void* da, void* db, void* ws,
                                          size_t ws_bytes, void* stream);

/*
 * One AdamW step over n tensors (64 a launch).  For tensor i of numel[i] elements, with
 * g' = grad_scale g:
 *   m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
 *   p -= lr (m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps) + weight_decay p),
 * in place, fp32 arithmetic.
 *   params[i] of param_dtype, grads[i] of grad_dtype (T2I_F32 or T2I_BF16 each),
 *   moments exp_avg[i], exp_avg_sq[i] fp32; masters[i] fp32 for bf16 params, which
 *   then receive the rounded masters (NULL for fp32 ones).  Host arrays of device
 *   pointers to contiguous elements at any alignment of their type; read during the
 *   call.  numel[i] 0 .. 2^33 (0: its pointers are not used).
 *   step counts from 1.  lr_device, step_device (then lr, step are not used) and
 *   grad_scale (NULL: 1) are device scalars that the kernel reads: a captured call
 *   follows them from replay to replay.
 * No tensor that is written may overlap another tensor.
 */
t2i_status t2i_op_adamw_step(int32_t param_dtype, int32_t grad_dtype, int32_t n,
                             const int64_t* numel, void* const* params, const void* const* grads,
                             float* const* exp_avg, float* const* exp_avg_sq,
                             float* const* masters, double lr, double beta1, double beta2,
                             double eps, double weight_decay, int64_t step,
                             const float* lr_device, const int32_t* step_device,
                             const float* grad_scale, void* stream);

/*
 * Memory-counter calibration (not part of the denoising step): reads `bytes`
 * of src (device, 16-byte aligned; a multiple of 1024 below 2 GiB) exactly
 * once through the direct HBM -> LDS load path that the GEMM and attention
 * kernels use, and writes 1024 floats of no meaning to sink (device).  A
 * profiler's fetched-bytes counter read on this launch gives the factor that
 * turns the counter into bytes for kernels loading this way.
 */
t2i_status t2i_op_dma_read(const void* src, size_t bytes, float* sink, void* stream);

const char* t2i_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* T2I_OPS_H */
