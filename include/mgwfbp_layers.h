/*
 * mgwfbp_layers.h -- C ABI of the operators that make the per-layer gradients which mgwfbp.h merges, reduces and applies:
 *                    embedding lookup and its gradient, and activation checkpoints in 8 bits with what the backward
 *                    pass makes of them.  For MI355X (gfx950); a shared object of its own, libmgwfbp_layers.so.
 *
 * The operators need no context: a call is described by its arguments, runs on the current device and on `hip_stream`
 * (a hipStream_t passed as void*; NULL is the default stream), returns without waiting, allocates nothing, keeps nothing
 * and may be captured into a HIP graph.  What they write (a tensor of the type of the context's gradients) is what
 * mgwfbp_pack and its fused forms read.  Functions return MGWFBP_OK (0) or a negative mgwfbp_status; nothing throws.
 *
 * Matrices are row-major; `stride` is the distance of two rows in elements (>= the row's length; any value for a
 * single row), pointers need the alignment of an element only, unless said otherwise.  Element types are
 * mgwfbp_dtype; all sums are binary32 and are rounded once, to nearest even.  Their order follows from the sizes
 * and ids alone, so that the same call gives the same bits.  Buffers that a call writes must not overlap any other.
 * Sizes of zero are accepted.  Errors: MGWFBP_EINVAL (null or misaligned pointer, unknown type, a size out of range or
 * a workspace too small: nothing has been enqueued), MGWFBP_EHIP (a launch failed; earlier launches of the same call
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

int mgwfbp_layers_last_hip_error(void); /* hipError_t of the last failed HIP call of these operators on this thread, 0 if none */

#ifdef __cplusplus
}
#endif
#endif /* MGWFBP_LAYERS_H */
