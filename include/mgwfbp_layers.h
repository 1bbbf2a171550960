/*
 * mgwfbp_layers.h -- C ABI of the operators that make the per-layer gradients which mgwfbp.h merges, reduces and applies:
 *                    embedding lookup and its gradient, activation checkpoints in 8 bits with what the backward
 *                    pass makes of them, root-mean-square norm, a gated linear recurrence and the last layer's loss, each with its
 *                    way back.  For MI355X (gfx950); a shared object of its own, libmgwfbp_layers.so.
 *
 * The operators need no context: a call is described by its arguments, runs on the current device and on `hip_stream`
 * (a hipStream_t passed as void*; NULL is the default stream), returns without waiting, allocates nothing, keeps nothing
 * and may be captured into a HIP graph.  What they write (a tensor of the type of the context's gradients) is what
 * mgwfbp_pack and its fused forms read.  Functions return MGWFBP_OK (0) or a negative mgwfbp_status; nothing throws.
 *
 * Matrices are row-major; `stride` is the distance of two rows in elements (>= the row's length; any value for a
 * single row), pointers need the alignment of an element only, unless said otherwise.  Element types are
 * mgwfbp_dtype; all sums are binary32 and are rounded once, to nearest even.  Their order follows from the sizes
 * and ids alone, so that the same call gives the same bits.  Buffers that a call writes must not overlap any other, unless said
 * otherwise.  (Matrices whose rows are equally far apart may lie beside each other in the same rows.  norm, recur, their ways back and distill
 * refuse calls whose outputs overlap something, their workspace included; the ranges of matrices with rows at different distances have to be apart there.)
 * Where an output may be an input, it is so as a whole: the same address, size of an element and stride.
 * Sizes of zero are accepted.  Errors: MGWFBP_EINVAL (null or misaligned pointer, unknown type, a size out of range or
 * a workspace too small, a launch of 2^32 lanes or more: nothing has been enqueued), MGWFBP_EHIP (a launch failed; earlier launches of the same call
 * may have been enqueued).
 * Workspaces are device memory of at least as many bytes as the *_workspace function says for the same sizes, aligned to
 * 256 bytes; they carry nothing from one call to the next, and one that is used on several streams needs their calls
 * to be in order.
 */
#ifndef MGWFBP_LAYERS_H
#define MGWFBP_LAYERS_H

#include <stdint.h>

#include "mgwfbp.h" /* mgwfbp_status, mgwfbp_dtype */

#ifdef __cplusplus
extern "C" {
#endif

typedef enum mgwfbp_id_type { MGWFBP_I32 = 0, MGWFBP_I64 = 1 } mgwfbp_id_type;

#define MGWFBP_MAX_TABLES 4
typedef struct mgwfbp_table {
    const void* d_rows;  /* [n_rows][dim], elements of the call's table type                        */
    const void* d_ids;   /* [n_tokens] row numbers; one outside 0..n_rows-1 stands for no row        */
    int64_t n_rows;
    int64_t row_stride;
    float scale;
    int32_t id_type;     /* mgwfbp_id_type                                                          */
} mgwfbp_table;

/* Embedding lookup: out[t,:] = sum over the tables k = 0..n_tables-1, in order, of scale_k * rows_k[ids_k[t], :]
 * (e.g. word, position and token type in one pass).
 *   tables  host [n_tables], 1 <= n_tables <= MGWFBP_MAX_TABLES
 *   n_tokens 0..2^26, dim 0..2^23 */
int mgwfbp_embed(const mgwfbp_table* tables, int32_t n_tables, int32_t table_dtype, int64_t n_tokens, int64_t dim,
                 void* d_out, int64_t out_stride, int32_t out_dtype, void* hip_stream);

/* Gradient of one table of a lookup: grad[r,:] = scale * sum over the tokens t with ids[t] = r of dy[t,:].
 * Rows without tokens become zeros.  accumulate != 0 adds to what is there instead (a table that is also the output
 * layer's weight; rows without tokens stay untouched).
 *   padding_row  a row that gets no gradient from its tokens; -1 for none
 *   n_rows < 2^31-1; n_tokens, dim as above */
int mgwfbp_embed_grad_workspace(int64_t n_tokens, int64_t n_rows, int64_t dim, uint64_t* bytes_out);
int mgwfbp_embed_grad(const void* d_ids, int32_t id_type, int64_t n_tokens, const void* d_dy, int64_t dy_stride,
                      int32_t dy_dtype, float scale, int64_t padding_row, int32_t accumulate, void* d_grad, int64_t n_rows,
                      int64_t dim, int64_t grad_stride, int32_t grad_dtype, void* d_workspace, uint64_t workspace_bytes,
                      void* hip_stream);

typedef enum mgwfbp_act_kind {  /* the function f between two layers                                  */
    MGWFBP_IDENTITY = 0,        /* x                                                                  */
    MGWFBP_GELU = 1,            /* x Phi(x), Phi the normal distribution                              */
    MGWFBP_GELU_TANH = 2,       /* x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2                    */
    MGWFBP_SILU = 3             /* x / (1 + exp(-x))                                                  */
} mgwfbp_act_kind;
/* Of an infinity they give what the formulas do: f(+inf) = +inf, f(-inf) = -inf * 0 = NaN (identity: -inf);
 * the slope is NaN there (identity: 1).  Of every finite number both are finite. */

/* Activation checkpoints in 8 bits.  A checkpoint of x [n_tokens][n_channels] is
 *   q      int8 [n_tokens][ld]    whole numbers -127..127
 *   scale  float [n_groups][ld]   one for each channel and group of MGWFBP_ACT_GROUP consecutive tokens
 * and stands for x^[t,c] = q[t,c] * scale[t / MGWFBP_ACT_GROUP, c].  ld is a multiple of 16 and >= n_channels, q and
 * scale are aligned to 16 bytes.  mgwfbp_act_dims gives the smallest ld and the number of groups.  A checkpoint's own columns are
 * those up to the next multiple of 16 of n_channels; the ones behind them are neither read nor written, so that several checkpoints may lie
 * side by side in one memory.
 *   n_tokens 0..2^26 (mgwfbp_act_linear_grad: 2^23), n_channels 0..2^23 */
#define MGWFBP_ACT_GROUP 128
int mgwfbp_act_dims(int64_t n_tokens, int64_t n_channels, int64_t* ld_out, int64_t* n_groups_out);

/* Makes a checkpoint of x and, where d_y is not NULL, y = f(x) in the same pass (y of x's type; f sees x itself).
 *   scale = max(largest |x| of the group, 2^-100) * (1/127);  q = x * (1/scale), rounded to nearest even
 * A group with an infinity or NaN gets q = 0 and scale = NaN, so that what the backward pass makes of it is NaN and
 * the overflow is noticed.  Channels from n_channels to the next multiple of 16 become zeros; columns behind them, where ld
 * is larger, are left as they are. */
int mgwfbp_act_store(const void* d_x, int64_t x_stride, int32_t dtype, int64_t n_tokens, int64_t n_channels, int32_t kind,
                     int8_t* d_q, float* d_scale, int64_t ld, void* d_y, int64_t y_stride, void* hip_stream);

/* Back through f: dx = dy * f'(x^), and f's output once more, y = f(x^), from the checkpoint of its input.  Either
 * output may be left out: d_dy and d_dx are NULL together, d_y by itself.  With MGWFBP_IDENTITY, y is x^ itself.
 * dy, dx and y are of one type. */
int mgwfbp_act_backward(const int8_t* d_q, const float* d_scale, int64_t ld, int64_t n_tokens, int64_t n_channels, int32_t kind,
                        const void* d_dy, int64_t dy_stride, void* d_dx, int64_t dx_stride, void* d_y, int64_t y_stride,
                        int32_t dtype, void* hip_stream);

/* Weight and bias gradient of a linear layer, out[t,o] = sum over c of w[o,c] * x[t,c] + b[o], from the gradient dy of its
 * output [n_tokens][n_outputs] and the checkpoint of its input:
 *   dw[o,c] = sum over t of dy[t,o] * x^[t,c];  db[o] = sum over t of dy[t,o]        (d_db NULL: left out)
 * accumulate != 0 adds to what is in dw and db.  The products are exact; the sums binary32.  A group's sum is one of
 * dy * q, to which the scale is applied: dy stays below 2^114, so that 128 products of up to 127 stay finite.
 *   n_tokens 0..2^23, n_outputs 0..2^23; ceil(n_outputs/128) * ceil(n_channels/128) <= 2^22 */
int mgwfbp_act_linear_grad_workspace(int64_t n_tokens, int64_t n_channels, int64_t n_outputs, uint64_t* bytes_out);
int mgwfbp_act_linear_grad(const int8_t* d_q, const float* d_scale, int64_t ld, int64_t n_tokens, int64_t n_channels,
                           const void* d_dy, int64_t dy_stride, int32_t dy_dtype, int64_t n_outputs, int32_t accumulate,
                           void* d_dw, int64_t dw_stride, void* d_db, int32_t grad_dtype, void* d_workspace,
                           uint64_t workspace_bytes, void* hip_stream);

/* Root-mean-square norm between two layers, with the residual's addition:
 *   h = x + residual, rounded to the stream's type (without a residual h is x itself)
 *   rstd[t] = 1 / sqrt(mean over c of h[t,c]^2 + eps);  n = h * rstd;  y = n * weight          (d_weight NULL: 1)
 * The mean is a binary64 sum, rstd is rounded to binary32 once, n and y are binary32 products, y rounded to x's type.
 * x and y are of one type, residual and h of the same or of MGWFBP_F32.  d_h and d_y may each be d_residual or d_x (but not an x of which n is
 * kept).  d_residual and d_h are NULL together (stream_dtype is dtype then).  eps 2^-100..2^100.
 * Where d_q is not NULL, n is kept for mgwfbp_norm_backward as a checkpoint (above) of q and scale, with rstd [n_tokens]; and
 * linear_scale, as large as scale, is scale * weight: q and linear_scale are a checkpoint of n * weight, of y before its rounding, for
 * mgwfbp_act_linear_grad.  d_rstd, d_q, d_scale and d_linear_scale are NULL together.
 *   n_tokens 0..2^26, n_channels 0..2^23 (a row takes 16 to 1024 lanes) */
int mgwfbp_norm(const void* d_x, int64_t x_stride, int32_t dtype, const void* d_residual, int64_t residual_stride, int32_t stream_dtype,
                int64_t n_tokens, int64_t n_channels, const void* d_weight, int32_t weight_dtype, double eps, void* d_h, int64_t h_stride,
                void* d_y, int64_t y_stride, float* d_rstd, int8_t* d_q, float* d_scale, float* d_linear_scale, int64_t ld, void* hip_stream);

/* Its way back: with n^ = q * scale and g = dy * weight,
 *   dh = dresidual + rstd * (g - n^ * mean over c of g n^)     (d_dresidual, what flows into h by itself, NULL: 0)
 *   dw[c] = sum over t of dy[t,c] * n^[t,c]                    (d_dw NULL: left out; accumulate != 0 adds to what is there)
 * dh is the gradient of x and of residual alike; d_dx, where not NULL, gets it in dy's type, too.  dresidual and dh are of the stream's
 * type; d_dh and d_dx may each be d_dresidual or d_dy.  The workspace is needed for dw, and above 8192 channels. */
int mgwfbp_norm_backward_workspace(int64_t n_tokens, int64_t n_channels, uint64_t* bytes_out);
int mgwfbp_norm_backward(const int8_t* d_q, const float* d_scale, int64_t ld, const float* d_rstd, int64_t n_tokens, int64_t n_channels,
                         const void* d_weight, int32_t weight_dtype, const void* d_dy, int64_t dy_stride, int32_t dtype, const void* d_dresidual,
                         int64_t dresidual_stride, void* d_dh, int64_t dh_stride, int32_t stream_dtype, void* d_dx, int64_t dx_stride, int32_t accumulate,
                         void* d_dw, int32_t grad_dtype, void* d_workspace, uint64_t workspace_bytes, void* hip_stream);

/* Sequences in the rows of a matrix.  d_offsets NULL: n_sequences of n_tokens / n_sequences tokens each.  Otherwise sequence s has the
 * rows offsets[s]..offsets[s+1]-1; offsets, [n_sequences + 1] on the device, begin with 0, do not decrease and end at n_tokens or
 * before; rows behind the last sequence are neither read nor written.  (Offsets are kept within 0..n_tokens, whatever they are.) */
typedef struct mgwfbp_sequences {
    int64_t n_sequences;  /* 0..2^26 */
    int64_t n_tokens;     /* of all, 0..2^26 */
    const void* d_offsets;
    int32_t offset_type;  /* mgwfbp_id_type */
} mgwfbp_sequences;

typedef enum mgwfbp_recur_kind { /* c(a), the factor of x */
    MGWFBP_RECUR_FREE = 0,       /* 1                     */
    MGWFBP_RECUR_CONVEX = 1,     /* 1 - a                 */
    MGWFBP_RECUR_UNIT = 2        /* sqrt(1 - a^2)         */
} mgwfbp_recur_kind;

/* Gated linear recurrence, for every sequence and channel by itself:
 *   a = 1 / (1 + exp(-gate));  h[t] = a[t] * h[t-1] + c(a[t]) * x[t];  y = h
 * gate, x and y are of one type, h is binary32.  first [n_sequences][n_channels] is h before each sequence's first token (NULL: 0), last, as
 * large, gets h behind its last one (NULL: left out; of a sequence without tokens: first).  d_last may be d_first where sequences are of
 * one length: a step of an answer is a call with one token for each sequence.  d_y may be d_gate or d_x.
 * states (NULL: left out) gets what the way back needs, h before every MGWFBP_RECUR_BLOCK-th token, of each sequence where they are of one
 * length, of all rows where there are offsets: mgwfbp_recur_states rows of n_channels. */
#define MGWFBP_RECUR_BLOCK 128
int mgwfbp_recur_states(const mgwfbp_sequences* sequences, int64_t* rows_out);
int mgwfbp_recur_workspace(const mgwfbp_sequences* sequences, int64_t n_channels, int32_t dtype, uint64_t* bytes_out);
int mgwfbp_recur(const mgwfbp_sequences* sequences, int64_t n_channels, int32_t kind, int32_t dtype, const void* d_gate, int64_t gate_stride,
                 const void* d_x, int64_t x_stride, const float* d_first, void* d_y, int64_t y_stride, float* d_last, float* d_states,
                 void* d_workspace, uint64_t workspace_bytes, void* hip_stream);

/* Its way back: with D[t] = dy[t] + a[t+1] * D[t+1] within a sequence, dlast (NULL: 0) behind its last token,
 *   dx = c(a) * D;  dgate = D * dh/dgate;  dfirst = a D at a sequence's first token (NULL: left out; of a sequence without tokens: dlast)
 * from the same gate, x and first and the states that mgwfbp_recur has kept.  d_dgate and d_dx may each be d_gate, d_x or d_dy.  The workspace is as large as mgwfbp_recur's. */
int mgwfbp_recur_backward(const mgwfbp_sequences* sequences, int64_t n_channels, int32_t kind, int32_t dtype, const void* d_gate, int64_t gate_stride,
                          const void* d_x, int64_t x_stride, const float* d_first, const float* d_states, const void* d_dy, int64_t dy_stride,
                          const float* d_dlast, void* d_dgate, int64_t dgate_stride, void* d_dx, int64_t dx_stride, float* d_dfirst,
                          void* d_workspace, uint64_t workspace_bytes, void* hip_stream);

/* Loss of a row of logits z against a label and against a teacher that is known by its top logits, and its gradient:
 *   p_j = exp(s_j / tau) / sum over the row's entries
 *   loss[t] = w * (label_weight * (-log softmax(z)[label]) + teacher_weight * tau^2 * sum over j of p_j * (log p_j - log softmax(z / tau)[id_j]))
 *   dz[t,:] = its gradient, of z's type                        (d_dz NULL: left out; it may be d_z)
 * labels [n_tokens] (NULL: none; one outside 0..n_vocabulary-1: none), ids and teacher [n_tokens][n_top] with a stride each: an id outside
 * 0..n_vocabulary-1 or a logit of -inf is no entry, the same id twice counts twice.  w = row_weight[t] (NULL: 1).  A row whose w is 0, or
 * that has neither label nor entry (or a weight of 0 for what it has), is not looked at: its loss is 0 and its gradient zeros.  Otherwise an
 * infinity of +inf or a NaN in the row makes both NaN; -inf is a place that is masked out.
 * The divergence is a difference of binary32 numbers of some log n_vocabulary, off by 1e-7 of them and so the loss by that times tau^2.  Where entries cover the
 * vocabulary, it nears 0 as tau grows (a loss of 6 is off by 1e-6 of itself at tau = 4, 2e-4 at 64, 6 % at 1024), and the gradient's error grows as 2e-8 tau of itself.
 *   n_vocabulary 1..2^23, n_top 0..MGWFBP_MAX_TOP, temperature 2^-20..2^20, weights finite */
#define MGWFBP_MAX_TOP 1024
int mgwfbp_distill_workspace(int64_t n_tokens, int64_t n_vocabulary, int32_t n_top, uint64_t* bytes_out);
int mgwfbp_distill(const void* d_z, int64_t z_stride, int32_t dtype, int64_t n_tokens, int64_t n_vocabulary, const void* d_labels, int32_t label_type,
                   const void* d_ids, int64_t ids_stride, int32_t id_type, const void* d_teacher, int64_t teacher_stride, int32_t teacher_dtype, int32_t n_top,
                   float temperature, float label_weight, float teacher_weight, const float* d_row_weight, float* d_loss, void* d_dz, int64_t dz_stride,
                   void* d_workspace, uint64_t workspace_bytes, void* hip_stream);

int mgwfbp_layers_last_hip_error(void); /* hipError_t of the last failed HIP call of these operators on this thread, 0 if none */

#ifdef __cplusplus
}
#endif
#endif /* MGWFBP_LAYERS_H */
