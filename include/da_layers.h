/*
 * da_layers.h -- C ABI of libdaspmm.so, second part: the layers that stand between the aggregations of a model of
 * node features, forward and backward: group norm with an activation, a gated feed-forward block, and the loss of a
 * distillation from a teacher's best classes.
 *
 * The conventions are those of da_spmm.h: pointers are device pointers unless a comment says "host"; calls enqueue
 * on `stream`, allocate nothing and do not synchronise (they can be captured in a graph); every function returns a
 * da_status and never throws; da_spmm_last_error() has the text of the last failure.  Workspaces are device scratch
 * of the caller, 16-byte aligned, free for reuse once the stream has passed the call.  Outputs overlap neither
 * inputs nor each other.  Where nothing else is said, sums are taken in an order that follows from the sizes alone:
 * results are the same from run to run.
 *
 * Types: float32 and bfloat16.  bfloat16 arrays are read as they are and computed with in float32; every output is
 * rounded once, to nearest even.
 */
#ifndef DA_LAYERS_H
#define DA_LAYERS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { DA_F32 = 0, DA_BF16 = 1 };

/* z;  max(z, 0);  z / (1 + exp(-z));  z (1 + erf(z / sqrt 2)) / 2;  1 / (1 + exp(-z)).  NaN stays NaN; the
 * derivative of max(z, 0) at 0 is 0. */
enum { DA_ACT_NONE = 0, DA_ACT_RELU = 1, DA_ACT_SILU = 2, DA_ACT_GELU = 3, DA_ACT_SIGMOID = 4, DA_NUM_ACTS = 5 };

/*
 * Group norm with an activation, channels last:  y = act(w (x - mean) / sqrt(var + eps) + b), mean and variance
 * (divided by n) over the n numbers that a sample has in a group of channels / groups neighbouring channels.
 *
 *   x         rows x channels, row-major, ldx >= channels; y and dx are dense
 *   samples   equal ones of `length` rows each (rows == samples * length, offsets NULL: one graph is one sample,
 *             and with length 1 every node is), or ragged ones: sample s is rows offsets[s] .. offsets[s+1] - 1,
 *             int32[samples + 1], offsets[0] == 0, non-decreasing, offsets[samples] == rows (a batch of graphs;
 *             empty samples are fine).  `length` is not looked at then.  Offsets that break this leave rows of y
 *             unwritten or give wrong numbers, but touch no other memory.
 *   w, b      channels numbers of param_dtype; NULL for 1 and 0
 *   stats     float32, written by the forward call and read by the backward call on the same shape (mean and
 *             1 / sqrt(var + eps) of every sample and group where the kernels do not take them again);
 *             da_group_norm_sizes says how many numbers, possibly none.  NULL forward where no gradient is needed
 *             and the sizes are computed with train == 0.
 *   dw, db    channels numbers of param_dtype, overwritten; either may be NULL
 *
 * Limits: rows, samples < 2^31, channels <= 2^20, groups <= 65535 (DA_ERR_UNSUPPORTED beyond).
 */
int da_group_norm_sizes(int dtype, int64_t rows, int64_t samples, int ragged, int64_t channels, int64_t groups, int train,
                        size_t *stats_floats, size_t *forward_bytes, size_t *backward_bytes /* host, out */);
int da_group_norm(int dtype, int64_t rows, int64_t samples, const int32_t *offsets, int64_t channels, int64_t groups,
                  const void *x, int64_t ldx, const void *w, const void *b, int param_dtype, float eps, int act, void *y,
                  float *stats, void *workspace, size_t workspace_bytes, void *stream);
int da_group_norm_backward(int dtype, int64_t rows, int64_t samples, const int32_t *offsets, int64_t channels,
                           int64_t groups, const void *x, int64_t ldx, const void *dy, int64_t ldy, const void *w,
                           const void *b, int param_dtype, float eps, int act, const float *stats, void *dx, void *dw,
                           void *db, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Distillation from a teacher's best classes.  A row has `classes` logits z of the student and `best` entries of the
 * teacher: a class and its logit t.  An entry whose class is outside 0 .. classes-1 (-1, say) is missing.
 *
 *   p = softmax(t / temperature) over the row's entries,  q = softmax(z / temperature) over all classes
 *   loss[r] = temperature^2 sum_k p_k (log p_k - log q[class_k])
 *   dz[r,j] = dloss[r] temperature (q_j - sum of p_k over the entries k of class j)
 *
 * A row without entries, or all of whose entries are -inf, has loss 0 and gradient 0.  An entry with p_k = 0 (a logit of
 * -inf beside others) adds nothing.  An entry of NaN makes its row's loss NaN, and the gradient of its entries' classes.
 * Several entries of one class count as they stand.
 *
 *   z         rows x classes of dtype, ldz >= classes; dz dense
 *   index     rows x best, int32 or (index64 != 0) int64, dense
 *   top       rows x best of top_dtype, dense
 *   stats     float32[rows x 2], written by the forward call (a row's largest logit and 1 / the sum of exp((z - largest) /
 *             temperature)) and read backward; may be NULL where no gradient is needed
 *   loss, dloss   float32[rows]; dloss_stride 0 takes dloss[0] for every row
 * Without classes every entry is missing.  Limits: rows < 2^31, classes < 2^31 - 2^16, best <= 1024.
 */
int da_distill_workspace(int64_t rows, int64_t classes, size_t *bytes /* host, out */);
int da_distill(int dtype, int64_t rows, int64_t classes, int64_t best, const void *z, int64_t ldz, const void *index,
               int index64, const void *top, int top_dtype, float temperature, float *loss, float *stats, void *workspace,
               size_t workspace_bytes, void *stream);
int da_distill_backward(int dtype, int64_t rows, int64_t classes, int64_t best, const void *z, int64_t ldz,
                        const void *index, int index64, const void *top, int top_dtype, float temperature,
                        const float *stats, const float *dloss, int64_t dloss_stride, void *dz, void *stream);

/*
 * Gated feed-forward block on the matrix cores:
 *
 *   u = x . w_gate,  v = x . w_up,  a = act(u) v,  y = a . w_down
 *   da = dy . w_down^T,  du = da v act'(u),  dv = da act(u),  dx = du . w_gate^T + dv . w_up^T,
 *   dw_gate = x^T . du,  dw_up = x^T . dv,  dw_down = a^T . dy
 *
 *   x         rows x d, ldx >= d;  w_gate, w_up  d x h;  w_down  h x dout;  y, dy  rows x dout (ldy >= dout), all of dtype,
 *             row-major, dense where no leading dimension is given
 *   u, v      float32, rows x h: written forward where not NULL (a backward pass is to follow), read backward.  They stay in
 *             32 bits for bfloat16, too: rounded, they would add as much to the error of dx as everything else together.
 *   a         rows x h of dtype: scratch of the forward call, which leaves act(u) v there where u and v are not NULL; read
 *             backward.  With bfloat16 a, du and dv are rounded, since they are operands of the matrix cores (up to 8
 *             rows are multiplied by the vector units forward, with an a of 32 bits).
 *   dx, dw_*  dense; any of them may be NULL and is then not computed
 *
 * Sums are held in 32 bits.  float32 is multiplied as it is (fp32 matrix cores).  All sizes up to 2^30, and fewer than
 * 2^23 tiles of 128 x 128 of a result, 2^24 where smaller ones are taken (DA_ERR_UNSUPPORTED beyond).
 */
int da_gated_workspace(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout, size_t *forward_bytes,
                       size_t *backward_bytes /* host, out */);
int da_gated(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout, const void *x, int64_t ldx, const void *w_gate,
             const void *w_up, const void *w_down, int act, void *y, float *u, float *v, void *a, void *workspace,
             size_t workspace_bytes, void *stream);
int da_gated_backward(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout, const void *x, int64_t ldx, const void *dy,
                      int64_t ldy, const void *w_gate, const void *w_up, const void *w_down, int act, const float *u,
                      const float *v, const void *a, void *dx, void *dw_gate, void *dw_up, void *dw_down, void *workspace,
                      size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DA_LAYERS_H */
