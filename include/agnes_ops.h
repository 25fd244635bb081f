/*
 * agnes_ops.h -- C ABI of the operators that a model trained on prepared
 * hyperbatches needs next to them: learned node embeddings (lookup and
 * gradient), distillation from a teacher's top logits (loss and gradient),
 * feature rows in microscaled 4-bit floating point (quantisation, and their
 * product with 4-bit weights), and for deeper models rows in 8 bits (their
 * product with 8-bit weights and its gradients, nonlinearities that keep their
 * input in 8 bits) and the norms around a residual block.  They need no ctx.  The paper (arXiv
 * 2601.01473) has no counterpart; the student it trains is the user's model.
 *
 * Conventions, beside those of agnes.h: all work of a call is enqueued on
 * cuda_stream, nothing is allocated and nothing waited for; arrays are device
 * memory of one GPU, and the call runs on that GPU.  No output may overlap
 * an input or another output unless an entry says so.  A call with nothing to
 * compute (no rows) returns AGNES_OK.  On failure agnes_last_error(NULL) gives
 * a message.  Every call can be captured into a CUDA graph.
 *
 * Element types are AGNES_F32, AGNES_F16 or AGNES_BF16, each argument's own;
 * arithmetic is in fp32 and each output value is rounded once, to nearest even.
 * Strides are in elements (bytes for 4-bit and 8-bit rows) and may exceed the row's
 * length; a row's elements are adjacent.
 *
 * status: an optional int32 (4-byte aligned) in device memory.  What a kernel finds wrong with
 * its data is ORed into it (AGNES_OP_*): the caller clears it, and reads it when
 * it next waits for the stream.
 */
#ifndef AGNES_OPS_H
#define AGNES_OPS_H

#include "agnes.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AGNES_BF16 2 /* agnes_dtype of the operators: bfloat16 */

#define AGNES_OP_BAD_INDEX 1 /* an id or index at or past the end of its range */
#define AGNES_OP_TIMEOUT 2   /* a kernel's bounded wait ran out: its output is undefined */

/* out[t] = scale * table[ids[t]] for n tokens (for example the nodes of a
 * minibatch).  A negative id selects no row: zeros.  So does an id >= rows,
 * which also sets AGNES_OP_BAD_INDEX.
 *  table   rows x dim of table_dtype, table_stride apart; 0 <= rows < 2^31,
 *          1 <= dim <= 2^22.
 *  ids     n ids of ids_bits (32 or 64) bits; 0 <= n < 2^31.
 *  out     n x dim of out_dtype, out_stride apart.
 * Errors: EINVAL, ERANGE (a size above these limits, or n * dim above 2^40),
 * ECUDA. */
agnes_status agnes_embedding_lookup(const void* table, int32_t table_dtype, int64_t rows,
                                    int64_t table_stride, int64_t dim, const void* ids,
                                    int32_t ids_bits, int64_t n, float scale, void* out,
                                    int32_t out_dtype, int64_t out_stride, int32_t* status,
                                    void* cuda_stream);

/* The gradient of agnes_embedding_lookup to the table, from the gradients of
 * its n output rows: d[v] = scale * sum_{t: ids[t] = v} grad[t].  Tokens are
 * sorted by id (stably) and each row's tokens summed in fp32 in an order that
 * depends on n and the ids only: the result is the same, bit by bit, each time.
 * Negative ids have no gradient, nor have ids >= rows, which also set
 * AGNES_OP_BAD_INDEX.
 *  grad    n x dim of grad_dtype, grad_stride apart.
 *  out     dense: rows x dim of out_dtype, contiguous; every row is written
 *          (zeros where no token selects it).
 *  workspace  at least agnes_embedding_grad_workspace bytes, 256-byte aligned;
 *          its contents are not kept.
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_embedding_grad(const void* grad, int32_t grad_dtype, int64_t grad_stride,
                                  const void* ids, int32_t ids_bits, int64_t n, int64_t rows,
                                  int64_t dim, float scale, void* out, int32_t out_dtype,
                                  void* workspace, int64_t workspace_bytes, int32_t* status,
                                  void* cuda_stream);

/* The same gradient, of the selected rows only, for tables too large for a
 * dense one: with c distinct ids in [0, rows),
 *  out_ids   n int32: the c ids in ascending order, then -1;
 *  out       n x dim of out_dtype, contiguous: their rows of d, then zeros;
 *  count     one int32: c.
 * The sizes do not depend on the data, so a training step needs no read-back.
 * Arguments and errors as agnes_embedding_grad. */
agnes_status agnes_embedding_grad_rows(const void* grad, int32_t grad_dtype, int64_t grad_stride,
                                       const void* ids, int32_t ids_bits, int64_t n, int64_t rows,
                                       int64_t dim, float scale, int32_t* out_ids, void* out,
                                       int32_t out_dtype, int32_t* count, void* workspace,
                                       int64_t workspace_bytes, int32_t* status,
                                       void* cuda_stream);

/* Bytes of workspace that both take for n tokens of dim values. */
agnes_status agnes_embedding_grad_workspace(int64_t n, int64_t dim, int64_t* bytes);

/* The loss of a student's logits against a teacher's top logits, row by row:
 * with p = softmax(teacher / T) over the row's entries, q = softmax(logits / T)
 * over all classes,
 *   loss = T^2 sum_k p_k (ln p_k - ln q[index_k]).
 * An entry with a negative index is absent; so is one with an index >= classes,
 * which also sets AGNES_OP_BAD_INDEX.  Entries of a row that name the same class
 * each count.  A row without an entry (or with teacher logits of -inf only), and
 * one whose logits are all -inf, has loss 0 and gradient 0.  A logit of -inf has
 * q = 0: the loss is +inf where p is not 0 there.  Where a logit or a present
 * teacher logit is NaN or +inf, the row's loss and gradient are NaN.
 * A label is the entry (label, 0) with top = 1 and T = 1: its loss is the cross
 * entropy, and label -1 is ignored.
 *  logits   rows x classes of logits_dtype, logits_stride apart;
 *           1 <= classes <= AGNES_DISTILL_MAX_CLASSES.
 *  teacher  rows x top of teacher_dtype, contiguous; 0 <= top <=
 *           AGNES_DISTILL_MAX_TOP.
 *  index    rows x top of index_bits (32 or 64) bits, contiguous.
 *  temperature  T > 0.
 *  loss     rows floats.
 *  stats    rows x 2 floats, 8-byte aligned: each row's largest logit and its
 *           sum of exp((x - largest) / T), for agnes_distill_grad.
 * Errors: EINVAL, ERANGE, ECUDA. */
#define AGNES_DISTILL_MAX_TOP 512
#define AGNES_DISTILL_MAX_CLASSES (1 << 30)
agnes_status agnes_distill_loss(const void* logits, int32_t logits_dtype, int64_t logits_stride,
                                int64_t rows, int64_t classes, const void* teacher,
                                int32_t teacher_dtype, const void* index, int32_t index_bits,
                                int64_t top, float temperature, float* loss, float* stats,
                                int32_t* status, void* cuda_stream);

/* Its gradient to the logits, with the loss of row r weighted by
 * w_r = weight_scale * weight[r] (weight NULL: weight_scale):
 *   out[r][v] = w_r T (q_v sum_k p_k - sum_{k: index_k = v} p_k).
 *  stats    as agnes_distill_loss left it for the same arguments.
 *  out      rows x classes of out_dtype, out_stride apart.  It may be the logits
 *           themselves (the same address, type and stride).
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_distill_grad(const void* logits, int32_t logits_dtype, int64_t logits_stride,
                                int64_t rows, int64_t classes, const void* teacher,
                                int32_t teacher_dtype, const void* index, int32_t index_bits,
                                int64_t top, float temperature, const float* stats,
                                const float* weight, float weight_scale, void* out,
                                int32_t out_dtype, int64_t out_stride, int32_t* status,
                                void* cuda_stream);

/* Both in one call, for a training step that knows its rows' weights.  Rows of
 * up to 1.6 MB (8 CTAs' shared memory) are kept there and read from memory once;
 * short ones (up to 512 classes, 8192 where rows are many) are read twice, the
 * second time from L2 as far as it holds them.  Arguments, in-place use and
 * errors as above. */
agnes_status agnes_distill_loss_grad(const void* logits, int32_t logits_dtype,
                                     int64_t logits_stride, int64_t rows, int64_t classes,
                                     const void* teacher, int32_t teacher_dtype, const void* index,
                                     int32_t index_bits, int64_t top, float temperature,
                                     const float* weight, float weight_scale, float* loss,
                                     void* out, int32_t out_dtype, int64_t out_stride,
                                     int32_t* status, void* cuda_stream);

/* Rows in microscaled 4-bit floating point (OCP MX, MXFP4).  Blocks of 32
 * values share a scale 2^(byte - 127), byte - 127 = floor(log2(largest magnitude))
 * - 2 and at least -127; each value is a 4-bit code, sign and magnitude of 0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 (codes 0 to 7, the sign in bit 3) times the scale.  A row of
 * dim values is mx4_row_bytes(dim) bytes: with b = ceil(dim / 32), 16 b bytes of
 * codes (the even value in a byte's low half; codes past dim are 0), b scale
 * bytes, and zeros up to a multiple of 16 bytes.  Rows are 16-byte aligned, a
 * multiple of 16 bytes apart.  So a matrix of them can be loaded as a graph's
 * features (row_bytes / 2 "fp16" values a row): they are gathered byte for byte. */
agnes_status agnes_mx4_row_bytes(int64_t dim, int64_t* bytes);

/* Rounds rows of dim values of dtype (stride apart) to 4-bit rows (out_stride
 * bytes apart): each value to the nearest magnitude, ties to the even code, above
 * 6 scales to 6.  A block with an infinity or NaN gets scale byte 255 and codes
 * 0: it stands for NaN.  Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_mx4_quantize(const void* x, int32_t dtype, int64_t stride, int64_t rows,
                                int64_t dim, void* out, int64_t out_stride, void* cuda_stream);

/* The values that 4-bit rows (stride bytes apart) stand for, rounded to dtype.
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_mx4_dequantize(const void* x, int64_t stride, int64_t rows, int64_t dim,
                                  void* out, int32_t dtype, int64_t out_stride,
                                  void* cuda_stream);

/* out[r][j] = sum_i x[r][i] w[j][i] (+ bias[j]): rows of 4-bit values times 4-bit
 * weights, for example a model's first layer over gathered rows.  Products are
 * exact and summed in fp32 on the tensor cores (tcgen05, block-scaled).
 *  x      rows 4-bit rows of dim values, x_stride bytes apart.
 *  w      width 4-bit rows of dim values, w_stride bytes apart.
 *  bias   width floats, or NULL.
 *  out    rows x width of out_dtype, out_stride apart.
 *  status AGNES_OP_TIMEOUT where a wait inside the kernel ran out.
 * 0 <= rows, 0 <= width < 2^31 - 255; 1 <= dim <= 2^26.
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_mx4_linear(const void* x, int64_t x_stride, int64_t rows, const void* w,
                              int64_t w_stride, int64_t width, int64_t dim, const float* bias,
                              void* out, int32_t out_dtype, int64_t out_stride, int32_t* status,
                              void* cuda_stream);

/* Rows in 8 bits, for features and for activations that are kept for a backward
 * pass.  A row of dim values is int8_row_bytes(dim) bytes: dim whole numbers q
 * from -127 to 127, zeros, and in the last four bytes of a multiple of 16 a scale
 * s (fp32); it stands for q s.  s may be any fp32 number; agnes_int8_quantize writes
 * bfloat16 ones (eight significant bits), for which a value has 15 bits and the gradients
 * below take it whole, where of rows that came another way they take its leading 16 bits.
 * Rows are 16-byte aligned, a multiple of 16 bytes apart.  So a matrix of them can be
 * loaded as a graph's features (row_bytes / 2 "fp16" values a row): they are gathered
 * byte for byte.  1 <= dim <= 2^17, 0 <= rows < 2^31 - 255. */
#define AGNES_INT8_ROWS 3 /* an output's type: 8-bit rows, its stride in bytes */
agnes_status agnes_int8_row_bytes(int64_t dim, int64_t* bytes);

/* Rounds rows of dim values of dtype (stride apart) to 8-bit rows (out_stride
 * bytes apart): s is the row's largest magnitude / 127 in fp32, rounded up to
 * eight significant bits (a bfloat16 value), and q = round(x (1 / s)), the inverse
 * and the product in fp32, to nearest even.  A row whose largest magnitude is
 * below 2^-100 is zeros with scale 0; one with an infinity or NaN gets scale NaN
 * and zeros: it stands for NaN.  Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_int8_quantize(const void* x, int32_t dtype, int64_t stride, int64_t rows,
                                 int64_t dim, void* out, int64_t out_stride, void* cuda_stream);

/* The values that 8-bit rows (stride bytes apart) stand for, rounded to dtype.  As
 * s is rounded up, 127 s may lie past the type's largest number where the row did
 * not: such a value becomes that number.  Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_int8_dequantize(const void* x, int64_t stride, int64_t rows, int64_t dim,
                                   void* out, int32_t dtype, int64_t out_stride,
                                   void* cuda_stream);

/* out[r][j] = sum_i x[r][i] w[j][i] (+ bias[j]): 8-bit rows times 8-bit weights,
 * with a scale for each row of x (a token) and each row of w (a channel):
 * s_x[r] s_w[j] times the sum of the whole numbers' products, which is exact up to
 * 2^24 and in fp32 beyond.
 *  x      rows 8-bit rows of dim values, x_stride bytes apart.
 *  w      width 8-bit rows of dim values, w_stride bytes apart.
 *  bias   width floats, or NULL.
 *  out    rows x width of out_dtype, out_stride apart.
 *  workspace  at least agnes_int8_linear_workspace bytes, 256-byte aligned (NULL
 *         where that is 0); its contents are not kept.
 *  status AGNES_OP_TIMEOUT where a wait inside the kernel ran out.
 * 0 <= rows, 0 <= width < 2^29 (here and in the gradients).
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_int8_linear(const void* x, int64_t x_stride, int64_t rows, const void* w,
                               int64_t w_stride, int64_t width, int64_t dim, const float* bias,
                               void* out, int32_t out_dtype, int64_t out_stride, void* workspace,
                               int64_t workspace_bytes, int32_t* status, void* cuda_stream);
agnes_status agnes_int8_linear_workspace(int64_t rows, int64_t width, int64_t dim, int64_t* bytes);

/* The gradient of agnes_int8_linear to the weights, from the rows that the layer
 * keeps in 8 bits, and to the bias:
 *   out[j][i] = sum_r grad[r][j] x[r][i],  dbias[j] = sum_r grad[r][j].
 * Products are exact to 2^-21 (2^-16 where a scale has more than eight bits), sums are in
 * fp32 over an order that depends on the sizes only: the result is the same, bit by bit,
 * each time.
 *  grad   rows x width of grad_dtype, grad_stride apart.
 *  out    width x dim of out_dtype, out_stride apart (zeros where rows is 0).
 *  dbias  width floats, or NULL.
 *  workspace  at least agnes_int8_linear_grad_weight_workspace bytes, 256-byte
 *         aligned; its contents are not kept.  `direct` of that entry: 1 where grad is
 *         bfloat16, 16-byte aligned and its rows a multiple of 16 bytes apart, so that it
 *         is read as it is; else 0.
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_int8_linear_grad_weight(const void* grad, int32_t grad_dtype,
                                           int64_t grad_stride, int64_t rows, int64_t width,
                                           const void* x, int64_t x_stride, int64_t dim, void* out,
                                           int32_t out_dtype, int64_t out_stride, float* dbias,
                                           void* workspace, int64_t workspace_bytes,
                                           int32_t* status, void* cuda_stream);
agnes_status agnes_int8_linear_grad_weight_workspace(int64_t rows, int64_t width, int64_t dim,
                                                     int32_t grad_dtype, int32_t direct,
                                                     int64_t* bytes);

/* The gradient of agnes_int8_linear to its input: out[r][i] = sum_j grad[r][j] w[j][i].
 * As in the gradient to the weights, what an infinity or NaN of grad or a row that
 * stands for NaN enters is not finite (NaN, or an infinity), and nothing else is.
 *  out    rows x dim of out_dtype, out_stride apart.
 *  workspace  at least agnes_int8_linear_grad_input_workspace bytes, 256-byte
 *         aligned; its contents are not kept.  `direct` as above.
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_int8_linear_grad_input(const void* grad, int32_t grad_dtype,
                                          int64_t grad_stride, int64_t rows, int64_t width,
                                          const void* w, int64_t w_stride, int64_t dim, void* out,
                                          int32_t out_dtype, int64_t out_stride, void* workspace,
                                          int64_t workspace_bytes, int32_t* status,
                                          void* cuda_stream);
agnes_status agnes_int8_linear_grad_input_workspace(int64_t rows, int64_t width, int64_t dim,
                                                    int32_t grad_dtype, int32_t direct,
                                                    int64_t* bytes);

/* A nonlinearity, gated or not, that keeps its input in 8 bits for its backward
 * pass: out = f(x), or f(x[:, :dim]) x[:, dim:] where gated (x has 2 dim columns
 * then).  f is relu, silu (v / (1 + exp -v)) or gelu (v Phi(v)).
 *  x      rows x dim (2 dim) of dtype, stride apart.
 *  out    rows x dim of the same type, out_stride apart; or, with out_dtype
 *         AGNES_INT8_ROWS, 8-bit rows out_stride bytes apart, for a layer that
 *         takes them.
 *  kept   8-bit rows of x, kept_stride bytes apart; where gated the two halves are
 *         rows of their own side by side (2 int8_row_bytes(dim) bytes).  NULL: not
 *         kept (serving).
 * Errors: EINVAL, ERANGE, ECUDA. */
#define AGNES_F_RELU 0
#define AGNES_F_SILU 1
#define AGNES_F_GELU 2
agnes_status agnes_activation(const void* x, int32_t dtype, int64_t stride, int64_t rows,
                              int64_t dim, int32_t f, int32_t gated, void* out, int32_t out_dtype,
                              int64_t out_stride, void* kept, int64_t kept_stride,
                              void* cuda_stream);

/* Its gradient to x at the kept values k: grad f'(k), or where gated grad f'(k_1) k_2
 * and grad f(k_1) side by side.  relu' is 0 at 0.  A kept row that stands for NaN
 * has a gradient of NaN.
 *  grad   rows x dim of grad_dtype, grad_stride apart.
 *  out    rows x dim (2 dim) of out_dtype, out_stride apart.
 * Errors: EINVAL, ERANGE, ECUDA. */
agnes_status agnes_activation_grad(const void* grad, int32_t grad_dtype, int64_t grad_stride,
                                   const void* kept, int64_t kept_stride, int64_t rows, int64_t dim,
                                   int32_t f, int32_t gated, void* out, int32_t out_dtype,
                                   int64_t out_stride, void* cuda_stream);

/* The step between two blocks of a residual network.  With N(v) = v / sqrt(mean v^2
 * + eps) (AGNES_NORM_RMS) or (v - mean v) / sqrt(var v + eps) (AGNES_NORM_LAYER) of
 * a row,
 *   u    = N(branch) after + after_bias, or branch where after is NULL
 *   sum  = x + scale gate u, rounded to x's type
 *   next = N(sum) before + before_bias, of the rounded sum.
 * branch NULL: next of x itself, and no sum.  before NULL: no next.
 *  x, sum        rows x dim of x_dtype: branch's type, or fp32.
 *  branch, next  rows x dim of branch_dtype (next_dtype the same, or AGNES_INT8_ROWS:
 *                8-bit rows, next_stride bytes apart).
 *  gate          none, dim floats for all rows (AGNES_GATE_COLUMNS), or rows x dim
 *                of branch_dtype, gate_stride apart (AGNES_GATE_ROWS).
 *  after, after_bias, before, before_bias  dim floats each; a bias needs its norm.
 *  sum may be x itself (the same address and stride).
 * 0 <= rows < 2^31 - 2047, 1 <= dim <= 8192.  Errors: EINVAL, ERANGE, ECUDA. */
#define AGNES_NORM_RMS 0
#define AGNES_NORM_LAYER 1
#define AGNES_GATE_NONE 0
#define AGNES_GATE_COLUMNS 1
#define AGNES_GATE_ROWS 2
agnes_status agnes_residual_norm(const void* x, int32_t x_dtype, int64_t x_stride,
                                 const void* branch, int32_t branch_dtype, int64_t branch_stride,
                                 int64_t rows, int64_t dim, const void* gate, int32_t gate_kind,
                                 int64_t gate_stride, float scale, const float* after,
                                 const float* after_bias, const float* before,
                                 const float* before_bias, int32_t kind, float eps, void* sum,
                                 int64_t sum_stride, void* next, int32_t next_dtype,
                                 int64_t next_stride, void* cuda_stream);

/* Its gradients, from those of next (d_next, branch's type) and of sum (d_sum, x's
 * type; NULL: none), and from sum as the forward pass rounded it (x where branch is
 * NULL).
 *  dx        rows x dim of x_dtype;  dbranch  rows x dim of branch_dtype.
 *  dgate     dim floats or rows x dim of branch_dtype, as the gate is.
 *  dafter, dafter_bias, dbefore, dbefore_bias  dim floats each, or NULL: not computed.
 * The sums over rows are in fp32, in an order that depends on the sizes and the device
 * only.
 *  workspace  at least agnes_residual_norm_grad_workspace bytes, 256-byte aligned; its
 *         contents are not kept.
 * Other arguments, limits and errors as agnes_residual_norm. */
agnes_status agnes_residual_norm_grad(
    const void* d_next, int64_t d_next_stride, const void* d_sum, int64_t d_sum_stride,
    const void* sum, int32_t x_dtype, int64_t sum_stride, const void* branch, int32_t branch_dtype,
    int64_t branch_stride, int64_t rows, int64_t dim, const void* gate, int32_t gate_kind,
    int64_t gate_stride, float scale, const float* after, const float* after_bias,
    const float* before, int32_t kind, float eps, void* dx, int64_t dx_stride, void* dbranch,
    int64_t dbranch_stride, void* dgate, int64_t dgate_stride, float* dafter, float* dafter_bias,
    float* dbefore, float* dbefore_bias, void* workspace, int64_t workspace_bytes,
    void* cuda_stream);
agnes_status agnes_residual_norm_grad_workspace(int64_t rows, int64_t dim, int64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif
