/*
 * agnes_ops.h -- C ABI of the operators that a model trained on prepared
 * hyperbatches needs next to them: learned node embeddings (lookup and
 * gradient), distillation from a teacher's top logits (loss and gradient), and
 * feature rows in microscaled 4-bit floating point (quantisation, and their
 * product with 4-bit weights).  They need no ctx.  The paper (arXiv
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
 * Strides are in elements (bytes for 4-bit rows) and may exceed the row's
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

#ifdef __cplusplus
}
#endif
#endif
