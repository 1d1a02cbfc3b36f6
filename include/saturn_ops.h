/* saturn_ops.h -- kernel-level C ABI of libsaturn.so.
 *
 * Each call enqueues one kernel of the fine-tuning step (the step that the
 * Saturn paper, arXiv 2309.01226, schedules for every model-selection task;
 * Sec. 3.1, Table 3) on `stream` (a hipStream_t, NULL = null stream) and
 * returns without waiting.  All tensor pointers are device pointers owned by
 * the caller; matrices are row-major with the given leading dimension (in
 * elements).  bf16 means IEEE bfloat16 storage (uint16).  The calls exist so
 * that every kernel can be checked and timed on its own; the model calls in
 * saturn.h use the same kernels.  Errors: SAT_EINVAL for bad sizes or null
 * pointers, SAT_EHIP when the launch fails.  Status codes as in saturn.h.
 */
#ifndef SATURN_OPS_H
#define SATURN_OPS_H

#include <stdint.h>

#include "saturn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Dense contraction C[m, n] = sum_k A(m, k) B(n, k) (bf16 operands, fp32
 * accumulation), the forward, input-gradient and weight-gradient products of
 * every linear layer.  Layout 0: A(m, k) = A[m*lda + k], B(n, k) = B[n*ldb + k];
 * layout 1: A(m, k) = A[k*lda + m], B(n, k) = B[k*ldb + n].
 * Epilogue 0: fp32 out = C + bias.  1: fp32 out = resid + C + bias (resid may
 * equal out).  2: bf16 out = C + bias, and, when out2 != NULL, bf16
 * out2[m, n - gelu_col0] = GELU(C + bias) for n >= gelu_col0.  3: bf16 out =
 * C * GELU'(aux[m, n]).  bias (fp32, may be NULL) applies to columns
 * n >= bias_col0 as bias[n - bias_col0].  gelu_erf: 0 tanh form, 1 erf form.
 * splitk_ws (fp32 device scratch of splitk_ws_elems elements, may be NULL):
 * with it, an epilogue-0/1 product on layout-0 operands that has fewer than
 * 256 output tiles of 256 x 256 and K >= 1024 runs split-K: K slices of at
 * least 512 write fp32 partials there, then one reduction adds them in slice
 * order with bias and residual (unless smaller tiles that fill the chip unsplit
 * are estimated faster).  Such a product with more than 256 tiles
 * whose last round of 256 tiles would run mostly empty instead runs its
 * first rows (whole rounds) unsplit and only the remaining rows split-K,
 * when that is estimated faster.  Results then differ from the unsplit
 * product by summation order only.  The scratch is used only when it holds
 * slices * (split rows) * N elements; the call makes no allocation.  No other
 * product touches it. */
typedef struct {
  const void* A;
  const void* B;
  int32_t M, N, K;
  int64_t lda, ldb;
  int32_t a_layout, b_layout, epilogue;
  void* out;
  int64_t ldo;
  const float* bias;
  int32_t bias_col0;
  const float* resid;
  int64_t ldr;
  void* out2;
  int64_t ldo2;
  int32_t gelu_col0;
  const void* aux;
  int64_t ldaux;
  int32_t gelu_erf;
  float* splitk_ws;
  int64_t splitk_ws_elems;
} sat_gemm_desc;
sat_status sat_op_gemm(const sat_gemm_desc* d, void* stream);
/* The same, and an epilogue-0/1 product with a layout-1 operand and K >= 1024 may
 * use splitk_ws too, in slices of at least 512.  Calls that may overlap
 * (different streams, or different host threads) need a splitk_ws each. */
sat_status sat_op_gemm_splitk(const sat_gemm_desc* d, void* stream);

/* sat_op_gemm for callers that cannot allocate device memory: code under HIP
 * graph capture, tight serving loops and harnesses that forbid hipMalloc.
 * Same descriptor and result as sat_op_gemm given a workspace large enough
 * for the product's split-K plan, except that d->splitk_ws must be NULL and
 * d->splitk_ws_elems 0: the split-K partials go to a scratch array of
 * SAT_GEMM_NOALLOC_WS_ELEMS fp32 elements (32 MiB) that the library holds on
 * every device it runs on until the process ends.  The call allocates
 * nothing.  A product whose split-K partials would exceed the scratch is
 * rejected with SAT_EINVAL before any launch, except one that would split
 * only the rows of its last round: that runs unsplit, with the result of
 * sat_op_gemm without a workspace.  All calls on one device share
 * that device's scratch: calls whose products split K and that may overlap
 * (different streams, or different host threads) race and must be ordered
 * by the caller. */
#define SAT_GEMM_NOALLOC_WS_ELEMS (8L * 1024 * 1024)
sat_status sat_op_gemm_noalloc(const sat_gemm_desc* d, void* stream);

/* LayerNorm forward over `rows` rows of length d: x fp32 (row r at
 * x + r*row_stride*ldx), y bf16 [rows, ldy], mean / rstd fp32 [rows]. */
sat_status sat_op_layernorm_fwd(const float* x, int64_t ldx, int64_t row_stride, const float* g,
                                const float* b, void* y, int64_t ldy, float* mean, float* rstd,
                                int32_t rows, int32_t d, float eps, void* stream);
/* LayerNorm backward: dres[r] += dx[r] (fp32, same row addressing as x);
 * dg, db fp32 [d] (overwritten).  work: fp32 scratch of 2*n_part*d floats,
 * n_part = min(rows, 1024). */
sat_status sat_op_layernorm_bwd(const float* dy, int64_t lddy, const float* x, int64_t ldx,
                                int64_t row_stride, const float* g, const float* mean,
                                const float* rstd, float* dres, int64_t ldres, float* dg,
                                float* db, float* work, int32_t rows, int32_t d, void* stream);

/* Flash-style attention forward.  q, k, v, o: bf16, element (b, h, s, j) at
 * ptr[(b*S + s)*ld + h*dh + j].  lse: fp32 [B, H, S] natural-log
 * log-sum-exp of the scaled scores.  scale multiplies q.k.  dh is one of 16,
 * 32, 64, 80, 128, 256; for 64, 80 and 256, q, k, v must be 16-byte aligned
 * with ld % 8 == 0, o 8-byte aligned with ldo % 4 == 0 and scale > 0
 * (SAT_EINVAL otherwise). */
sat_status sat_op_attention_fwd(const void* q, const void* k, const void* v, int64_t ldq,
                                int64_t ldk, int64_t ldv, void* o, int64_t ldo, float* lse,
                                int32_t B, int32_t H, int32_t S, int32_t dh, int32_t causal,
                                float scale, void* stream);
/* Attention backward from dO (bf16, addressed like o), the forward's o and
 * lse; writes dq, dk, dv (bf16, addressed like q, k, v).  delta: fp32
 * [B, H, S] scratch.  Head dims and alignment as for the forward; for 64, 80
 * and 256, o and dout must also be 16-byte aligned with ld % 8 == 0 and dq,
 * dk, dv 8-byte aligned with ld % 4 == 0. */
sat_status sat_op_attention_bwd(const void* q, const void* k, const void* v, int64_t ldq,
                                int64_t ldk, int64_t ldv, const void* o, int64_t ldo,
                                const float* lse, const void* dout, int64_t lddo, float* delta,
                                void* dq, void* dk, void* dv, int64_t lddq, int64_t lddk,
                                int64_t lddv, int32_t B, int32_t H, int32_t S, int32_t dh,
                                int32_t causal, float scale, void* stream);

/* Attention inside packed sequences, forward and backward: rows of several
 * sequences follow each other in one buffer without padding between them.
 *   rows     cu: device int32 [n_seq + 1], not decreasing; rows cu[s] ..
 *            cu[s + 1] - 1 of every row array are sequence s (a length may be
 *            0).  T rows per array, 0 <= T <= 2^29, (T / 64 + 2 n_seq + 16) H below
 *            2^24.  Rows outside all sequences are
 *            not read and keep what they hold in every output.  cu is read on the
 *            device only, so a captured call takes the lengths of the
 *            replay; values outside [0, T] are taken as the nearer of the two.  A cu that decreases
 *            touches no row outside its values either, but leaves undefined what its sequences
 *            write.
 *   heads    H query heads, Hkv K / V heads, Hkv a divisor of H; query head h
 *            reads K / V head h / (H / Hkv).  dh: a multiple of 8 up to 256
 *            (32, 64, 80, 96, 128 and 256 have kernels of their width, others run
 *            in the next wider one).  Element (row t, head h, dim j) at ptr[t * ld + h * dh + j].
 *   mask     query i and key j of one sequence: j <= i when causal, and |i - j| <
 *            window when window > 0 (0: none).  Every query sees itself.
 *   values   o = softmax(scale q k^T) v as bf16, lse [H, T] fp32 the natural-log
 *            log-sum-exp; gradients of q, k, v as bf16, dk and dv summed in fp32 over
 *            the query heads that share them.  Products take p and dS rounded to
 *            bf16.  delta = rowsum(dout o) of the backward is the fp32 sum of p dP for dk and dv
 *            of up to 128 dims, and for dq there where a block of 64 or 128 queries sees keys of no more
 *            than two blocks of 64; elsewhere it is formed from the bf16 o.  A row of a sequence that holds NaN
 *            or infinities may spoil other rows of that sequence, none of another.
 *            The same inputs give the same bits on every call.
 * q, k, v, o and dout are 16-byte aligned with leading dimensions that are
 * multiples of 8 and below 2^22, dq, dk, dv 8-byte aligned with multiples of 4;
 * scale > 0.  Outputs overlap no input and no other output.  The backward reads the
 * forward's o and lse.  ws: fp32 scratch of ws_elems elements, 16-byte aligned.  The
 * forward uses it where few blocks of queries meet many keys, whose work is then split and joined,
 * and may have none (NULL); the backward needs at least H T (rounded up to 4) and
 * splits with more.  The _ws calls say how much each takes at most for the same sizes and
 * mask; results with and without differ by the order of the fp32 sums and by the running
 * maximum under which p is rounded, and keep the same bounds.  Calls that may overlap need a
 * ws each.  The forward reads nothing else from dout on.
 * Errors: SAT_EINVAL for null pointers (T > 0), sizes, alignment, or a ws that is too small. */
typedef struct {
  const void* q;
  const void* k;
  const void* v;
  int64_t ldq, ldk, ldv;
  void* o;
  int64_t ldo;
  float* lse;
  const int32_t* cu;
  int32_t n_seq, T, H, Hkv, dh, causal, window;
  float scale;
  const void* dout;
  int64_t lddo;
  void* dq;
  void* dk;
  void* dv;
  int64_t lddq, lddk, lddv;
  float* ws;
  int64_t ws_elems;
} sat_attn_packed_desc;
sat_status sat_op_attention_packed_fwd(const sat_attn_packed_desc* d, void* stream);
sat_status sat_op_attention_packed_bwd(const sat_attn_packed_desc* d, void* stream);
/* fp32 elements of ws for these sizes (n_seq, T, H, Hkv, dh, causal and window are read). */
sat_status sat_op_attention_packed_fwd_ws(const sat_attn_packed_desc* d, int64_t* elems);
sat_status sat_op_attention_packed_bwd_ws(const sat_attn_packed_desc* d, int64_t* elems);

/* Rotary on interleaved pairs of the first rd dims of every q and k head, in
 * place; qk bf16 [B*S, ld] with q at column 0 and k at column H*dh.
 * inverse = 1 applies the transpose rotation (backward).  ld and dh even, qk
 * 4-byte aligned (SAT_EINVAL otherwise). */
sat_status sat_op_rotary(void* qk, int64_t ld, int32_t B, int32_t S, int32_t H, int32_t dh,
                         int32_t rd, int32_t inverse, void* stream);

/* Rotary positions with one to four axes (for instance time, height, width) on
 * rows x [T, ldx] of H heads of dh dims, head h at column h * dh, written to y [T, ldy].
 * pos: int32 [T, ldp], one position per row and axis, any sign.  Axis a turns
 * pairs[a] >= 0 consecutive pairs, half = sum of pairs <= dh / 2 and <= 128 of
 * them in all, the first 2 half dims of every head: pair i is dims (2 i, 2 i + 1)
 * when interleaved, else (i, i + half).  Its angle is pos * base^(-i / half), or,
 * with own_freqs, pos * base^(-j / pairs[a]) with j its place among its axis' pairs; angles are
 * formed in 64 bits, cos and sin rounded to fp32.  inverse = 1 applies the
 * transpose (backward).  y == x (with ldy == ldx): in place, the other dims stay; else
 * the heads' other dims are copied, and y must not overlap x.  Columns behind
 * the heads are not touched.  f32: x and y are fp32, else bf16.  dh even, H dh^2 below
 * 2^32, T below 2^24, x and y aligned to their elements (16-byte aligned rows are fastest).
 * Errors: SAT_EINVAL for null pointers (T > 0), sizes and alignment. */
sat_status sat_op_rotary_axes(const void* x, int64_t ldx, void* y, int64_t ldy, int32_t f32,
                              const int32_t* pos, int64_t ldp, int32_t n_axes,
                              const int32_t* pairs, int32_t T, int32_t H, int32_t dh, double base,
                              int32_t interleaved, int32_t own_freqs, int32_t inverse,
                              void* stream);

/* Dropout of x [rows, ldx] to y [rows, ldy]: y = x up where an element is kept, else 0 (also of infinities
 * and NaN).  The generator is Philox4x32-10 with the key `seed` (low word, high word) and the counter
 * (column / 8, row, low and high word of *step); column 8 q + e takes the low (e even) or high half of
 * word e / 2 and is dropped when that is below t = round(65536 p); up = 65536 / (65536 - t).
 * Nothing is stored: the backward is the same call on the gradient.  step: device int64 [1], read by
 * the kernel, so that a captured call draws anew when the caller's own work moves it on; NULL: 0.
 * Calls with the same seed, step and place drop the same elements: give each place in a model a seed
 * of its own.  y == x (with ldy == ldx): in place; else y must not overlap x.  f32: x and y are fp32, else
 * bf16.  cols up to 2^18, rows ceil(cols / 8) below 2^31; x and y aligned to their elements.  Columns
 * behind `cols` are not touched.  Errors: SAT_EINVAL for null pointers, sizes, alignment and p outside [0, 1]. */
sat_status sat_op_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int32_t f32,
                          int32_t rows, int32_t cols, double p, uint64_t seed, const int64_t* step,
                          void* stream);

/* The boundary of two sublayers, over T rows of 1 <= d <= 8192 columns, forward and backward:
 *   u = N_post(f)                     the norm of the branch's rows (f bf16), or f itself
 *   y = alpha x + beta gate m u       the residual stream, fp32 when stream_f32, else bf16
 *   h = N_pre(y)                      bf16, from y as it is stored: what the next sublayer reads
 * pre, post: 0 none (pre: no h), 1 LayerNorm, 2 RMS norm (x / sqrt(mean x^2 + eps)), with gains g_*
 * (NULL: 1) and shifts b_* (NULL: 0), fp32 [d].  gate: fp32 [d], NULL: 1.  m: dropout with the numbers of
 * sat_op_dropout for the same p, seed, step, row and column (p 0: none); a dropped element adds
 * nothing, whatever f holds.  stats: fp32 [4, T], mean and 1 / sqrt(var + eps) of the branch's norm, then of
 * the next one's (a norm that is not there leaves its two rows as they are; an RMS norm's mean is 0);
 * may be NULL without norms.  y may be x (with ldy == ldx); no other output overlaps an input.
 * Backward, from dy (the gradient that reaches y along the stream, in its type; NULL: 0) and dh (bf16, with
 * pre): dx = alpha t and df of t = dy + N_pre'(dh), and, where not NULL, fp32 [d] (written): dg_*, db_* and
 * dgate, summed over the rows in fp32 in an order that depends on T, d and whether all rows are 16-byte aligned
 * alone.  It reads y (with pre), f (with post or dgate), stats, gains, post's shift, gate and the dropout's arguments;
 * dx may be dy (with lddx == lddy).  ws: fp32 scratch, as much as the _ws call says (T, d and which sums are wanted are
 * read); calls that may overlap need one each.  A row that holds NaN or infinities spoils its own rows of the outputs and the sums.
 * Arrays are aligned to their elements (16-byte aligned rows are fastest).
 * Errors: SAT_EINVAL for null pointers, sizes, alignment, constants, and a ws that is too small. */
typedef struct {
  const void* x;
  int64_t ldx;
  const void* f;
  int64_t ldf;
  void* y;
  int64_t ldy;
  void* h;
  int64_t ldh;
  float* stats;
  const float* g_pre;
  const float* b_pre;
  const float* g_post;
  const float* b_post;
  const float* gate;
  int32_t T, d, stream_f32, pre, post;
  float alpha, beta, eps;
  double p;
  uint64_t seed;
  const int64_t* step;
  const void* dy;
  int64_t lddy;
  const void* dh;
  int64_t lddh;
  void* dx;
  int64_t lddx;
  void* df;
  int64_t lddf;
  float* dg_pre;
  float* db_pre;
  float* dg_post;
  float* db_post;
  float* dgate;
  float* ws;
  int64_t ws_elems;
} sat_residual_norm_desc;
sat_status sat_op_residual_norm_fwd(const sat_residual_norm_desc* d, void* stream);
sat_status sat_op_residual_norm_bwd(const sat_residual_norm_desc* d, void* stream);
/* fp32 elements of ws for these sizes and sums. */
sat_status sat_op_residual_norm_bwd_ws(const sat_residual_norm_desc* d, int64_t* elems);

/* Softmax cross-entropy forward + backward over fp32 logits z [N, ldz]:
 * row_loss fp32 [N] (0 for label -1), dz bf16 [N, lddz] = (softmax - onehot)
 * * inv_n (0 rows for label -1), where inv_n = 1 / (number of labels != -1). */
sat_status sat_op_cross_entropy(const float* z, int64_t ldz, const int32_t* labels, int32_t N,
                                int32_t V, float* row_loss, void* dz, int64_t lddz, float* inv_n,
                                void* stream);

/* Softmax cross entropy of a linear head z = x w^T + bias over the whole vocabulary, and its gradients,
 * without keeping the logits.
 *   x [N, ldx] bf16, w [V, ldw] bf16, rows of d; bias fp32 [V] or NULL (-inf takes an entry out).  labels
 *   int32 [N]: a row whose label is outside [0, V) (-1: ignore) takes no part and costs no product; its
 *   loss and lse are 0, its dx is 0.
 *   row_loss, lse fp32 [N]; inv_n fp32 [1] = 1 / (rows that take part), 1 without any.
 *   Gradients of sum_t c_t row_loss_t, c = row_weight [N] or, when that is NULL, inv_n for every row: dx
 *   [N, lddx] bf16, dw [V, lddw] and db [V], fp32 when grad_f32, else bf16, each NULL when not wanted.  With
 *   accumulate (fp32 only) dw and db add to what is there.  Without any, rows are only scored.
 * N up to 2^25, d a multiple of 8 up to 2^16, V up to 2^20.  Logits, statistics and sums are fp32; the two products of the
 * gradients take dz = row_weight (softmax - onehot) rounded to bf16 (where a chunk of the tokens has at most 256 rows,
 * in two parts) and are multiplied by inv_n afterwards where there is no row_weight.  The softmax in dz comes from z - m
 * (m: the maximum of up to 128 entries) rounded to 2^-11.5 of its exponential, 2^-9.5 where that is below 2^-32; the
 * label's entry is apart from that.  db sums dz before its
 * rounding.  Whole gradients of thousands of rows are off, in bf16, by 0.0018 of their norm where rounding alone makes
 * 0.0017 (0.0022 with row_weight), fp32 dw by 0.0007 (0.0014).  A row whose entries are all -inf has loss 0, lse -inf and no gradient; one that holds NaN
 * or infinities spoils its own outputs and the gradients of w and bias.  The same inputs give the same bits.
 * x and w 16-byte aligned with leading dimensions that are multiples of 8 and below 2^21, dx and dw with
 * 16-byte aligned rows.  Outputs overlap no input and no other output.  ws: scratch, 256-byte aligned, of as many
 * bytes as the _ws call says (N, V, d, which gradients, grad_f32 are read): a copy of x and 16 bytes a row; for gradients
 * at most 1 GiB for a chunk of the tokens and a tenth of that for its statistics, 128 MiB of partial products (256 where
 * dx and dw are small and formed together), 512 V bytes, and, with bf16 gradients of several chunks, their fp32 sums; for
 * rows that are only scored a chunk's statistics, 8 bytes for 64 entries of a row, at most 1 GiB.  Calls that may
 * overlap need one each.
 * Errors: SAT_EINVAL for null pointers, sizes, alignment, and a ws that is too small. */
typedef struct {
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  const int32_t* labels;
  const float* bias;
  const float* row_weight;
  float* row_loss;
  float* lse;
  float* inv_n;
  void* dx;
  int64_t lddx;
  void* dw;
  int64_t lddw;
  void* db;
  int32_t N, V, d, grad_f32, accumulate, reserved;
  void* ws;
  int64_t ws_bytes;
} sat_linear_xent_desc;
sat_status sat_op_linear_xent(const sat_linear_xent_desc* d, void* stream);
sat_status sat_op_linear_xent_ws(const sat_linear_xent_desc* d, int64_t* bytes);

/* Fused AdamW over n fp32 values (torch semantics, decoupled decay) at step t
 * (t >= 1); refreshes the bf16 shadow when shadow != NULL. */
sat_status sat_op_adamw(float* p, const float* g, float* m, float* v, void* shadow, int64_t n,
                        double lr, double beta1, double beta2, double eps, double wd, int64_t t,
                        void* stream);

/* The same step over `count` tensors in few launches, moments in 32 or in 8 bits
 * (state_bits).  The table t is host memory, read during the call only.  Each
 * entry: 0 <= n <= 2^35 fp32 values p, their gradient g (bf16 when grad_bf16, else fp32), moments m
 * and v, the tensor's weight decay, a bf16 shadow that is refreshed (may be
 * NULL); no array that is written overlaps another of the table.
 *   32 bits: m, v fp32 [n]; with an fp32 gradient every value is bitwise that of
 *            sat_op_adamw.
 *   8 bits:  m, v uint8 [n], m_exp, v_exp uint8 [ceil(n / 256)], all zero before the
 *            first step.  The 256 elements of a block share the factor 2^(exp - 127).  m is a sign
 *            (bit 7) and a 7-bit, the root of v an 8-bit magnitude c, (1 + f / F) 2^(e - 15)
 *            with c = F e + f, F = 8 for m and 16 for the root, and 0 for c = 0.  The update takes m
 *            and v as they were formed in fp32; what is kept is rounded up or down at random
 *            with the mean right, by a hash of (seed, t, place in the table, element): the
 *            same call gives the same bits, and each step of a run should have its own
 *            seed or t.  A root over 0 is kept as no less than the least code, 2^-15 of its
 *            block's largest at most; an m under that is kept as 0.  The root and the division
 *            of the update are the hardware's approximations (1 ulp each), and a v below 2^-126
 *            counts as 0.  A gradient that is not finite spoils p and the moments of its block.
 * Arrays are aligned to their elements (16 bytes for all is fastest).  Step t >= 1,
 * as constants: a captured call repeats the same lr and t.
 * Errors: SAT_EINVAL for null pointers, sizes, state_bits and constants. */
typedef struct {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* m_exp;
  uint8_t* v_exp;
  void* shadow;
  int64_t n;
  double weight_decay;
} sat_adamw_tensor;
sat_status sat_op_adamw_multi(const sat_adamw_tensor* t, int32_t count, int32_t state_bits,
                              int32_t grad_bf16, double lr, double beta1, double beta2,
                              double eps, int64_t step, uint64_t seed, void* stream);
/* The values that 8-bit moments stand for, m and v of every tensor to m_out[k] and
 * v_out[k] (host arrays of device pointers to n values), fp32 (exact, but for a v
 * below 2^-126) or, with out_bf16, bf16 (m exact, v rounded once): to store 32-bit moments, or to look at them.  Of the
 * table, m, v, m_exp, v_exp and n are read.  No output overlaps another or what is read.
 * Errors: SAT_EINVAL for null pointers, sizes, alignment, and outputs that overlap; SAT_ENOMEM. */
sat_status sat_op_adamw_multi_state(const sat_adamw_tensor* t, int32_t count,
                                    void* const* m_out, void* const* v_out, int32_t out_bf16,
                                    void* stream);

/* Token embedding forward h[t] = wte[tok[t]] (+ wpe[t % S]) and its
 * deterministic backward dwte[v] = sum over t with tok[t] == v of dh[t] in
 * increasing t, written for every v < V (zero rows for absent tokens; a token
 * outside [0, V) adds to no row of the backward).  Past
 * 16384 positions the sum is formed per chunk of 16384 positions, in order,
 * and the chunks' sums are added in order.
 * work: int32 scratch of min(T, 16384) entries.  Backward limit: V < 65536
 * (SAT_EINVAL otherwise). */
sat_status sat_op_embed_fwd(const int32_t* tok, const float* wte, const float* wpe, float* h,
                            int32_t T, int32_t S, int32_t d, int32_t V, void* stream);
sat_status sat_op_embed_bwd(const int32_t* tok, const float* dh, float* dwte, int32_t T,
                            int32_t d, int32_t V, int32_t* work, void* stream);

/* Column sum out[c] = sum_r X[r, c] of an fp32 [rows, ldx] matrix,
 * deterministic; work: fp32 scratch of min(rows, 256) * cols floats. */
sat_status sat_op_colsum(const float* X, int64_t ldx, int32_t rows, int32_t cols, float* out,
                         float* work, void* stream);

/* Transpose of a bf16 matrix: dst[c * ldd + r] = src[r * lds + c] for
 * r < rows, c < cols.  rows, cols, lds and ldd are multiples of 8 with
 * lds >= cols, ldd >= rows; both pointers device memory, 16-byte aligned
 * (SAT_EINVAL otherwise).  The runtime keeps transposed bf16 copies of the
 * weights for the input-gradient products dX = dY W (each a product over the
 * contiguous index of both operands). */
sat_status sat_op_transpose_bf16(const void* src, int64_t lds, void* dst, int64_t ldd,
                                 int32_t rows, int32_t cols, void* stream);

/* ---- the ResNet workload's own kernels (Table 3: the ResNet fine-tuned on
 * ImageNet-shaped images).  Activations are NHWC: [N, H, W, C] is the
 * row-major matrix [N * H * W, C]; Ho = (H + 2 pad - k) / stride + 1.
 *
 * im2col: col [N * Ho * Wo, k * k * C] bf16, col[(n Ho + i) Wo + j,
 * (a k + b) C + c] = x[n, i stride - pad + a, j stride - pad + b, c] (zero
 * outside the image), from x bf16; C a positive multiple of 8.  The operand of
 * a k x k convolution computed as one GEMM against the weight [Cout, k k C]. */
sat_status sat_op_im2col(const void* x, void* col, int32_t N, int32_t H, int32_t W, int32_t C,
                         int32_t k, int32_t stride, int32_t pad, void* stream);
/* The same matrix transposed: colT [k * k * C, N * Ho * Wo] bf16 with row
 * stride ldt (>= N Ho Wo, a multiple of 8), a K-contiguous operand for a
 * convolution's weight-gradient product (the ResNet step itself gathers that operand, or
 * reads the matrix of sat_op_im2col as it lies).  N Ho Wo % 8 == 0, C % 8 == 0, x and
 * colT 16-byte aligned (SAT_EINVAL otherwise). */
sat_status sat_op_im2col_t(const void* x, void* colT, int64_t ldt, int32_t N, int32_t H, int32_t W,
                           int32_t C, int32_t k, int32_t stride, int32_t pad, void* stream);
/* col2im, the transpose of im2col: dx [N, H, W, C] fp32 = (accumulate: dx +)
 * the sum over the taps that read each input element of dcol [N * Ho * Wo,
 * k * k * C] fp32, in tap order; C a positive multiple of 4. */
sat_status sat_op_col2im(const float* dcol, float* dx, int32_t N, int32_t H, int32_t W, int32_t C,
                         int32_t k, int32_t stride, int32_t pad, int32_t accumulate, void* stream);
/* Batch norm in training mode over x [P, C] fp32 (statistics of the P rows,
 * biased variance): mean, rstd = 1 / sqrt(var + eps) [C]; y = (x - mean) rstd
 * g + b, with ReLU when relu, as bf16 (y, may be NULL) and fp32 (yf, may be
 * NULL, not both).  part: fp32 scratch of 2 * 1024 * C.  C % 4 == 0; every
 * fp32 array 16-byte aligned, y 8-byte aligned (SAT_EINVAL otherwise). */
sat_status sat_op_batchnorm_fwd(const float* x, int64_t P, int32_t C, const float* g,
                                const float* b, float eps, int32_t relu, float* part, float* mean,
                                float* rstd, void* y, float* yf, void* stream);
/* Its backward from dy [P, C] fp32, through a ReLU when mask_kind is 1 (dy
 * where the bf16 mask > 0) or 2 (fp32 mask > 0): dg = sum g' xhat, db = sum
 * g' (written), dx = rstd g (g' - db / P - xhat dg / P) as bf16.  Alignment as
 * for the forward (an fp32 mask 16-byte, a bf16 mask and dx 8-byte). */
sat_status sat_op_batchnorm_bwd(const float* dy, int32_t mask_kind, const void* mask,
                                const float* x, const float* mean, const float* rstd,
                                const float* g, int64_t P, int32_t C, float* part, float* dg,
                                float* db, void* dx, void* stream);
/* 3 x 3 max pool, stride 2, padding 1: y fp32, yb bf16 and the winning tap
 * arg (row-major index 0..8, the first maximum) [N, Ho, Wo, C]; the backward
 * routes dy to the winning taps: dx [N, H, W, C] fp32. */
sat_status sat_op_maxpool_fwd(const float* x, int32_t N, int32_t H, int32_t W, int32_t C, float* y,
                              void* yb, uint8_t* arg, void* stream);
sat_status sat_op_maxpool_bwd(const float* dy, const uint8_t* arg, int32_t N, int32_t H, int32_t W,
                              int32_t C, float* dx, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SATURN_OPS_H */
