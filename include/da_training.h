/*
 * da_training.h -- C ABI of libdaspmm.so, third part: what a training step of a model of node features has beside its
 * layers: root-mean-square norm with the residual's addition (serving: with a result in 8 bits), the cross entropy of a
 * linear layer over many classes, and the orthogonalised update of a weight.
 *
 * The conventions and types are those of da_layers.h: device pointers unless a comment says "host"; calls enqueue on
 * `stream`, allocate nothing and do not synchronise; every function returns a da_status and never throws;
 * workspaces are 16-byte aligned device scratch, free for reuse once the stream has passed the call; outputs overlap
 * neither inputs nor each other.  Sums are taken in an order that follows from the sizes alone.
 */
#ifndef DA_TRAINING_H
#define DA_TRAINING_H

#include <stddef.h>
#include <stdint.h>

#include "da_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Root-mean-square norm of rows:  s = x + residual,  y = w s / sqrt(mean(s^2) + eps).
 *
 *   x, residual   rows x channels of dtype, row-major, ldx, ldr >= channels; residual NULL: s is x
 *   sum       s, dense, written where there is a residual.  It is rounded to dtype, and the rounded s is normalised.
 *   w         channels numbers of param_dtype; NULL for 1
 *   y         dense
 *   q, scale  da_rms_norm_e4m3: y = q scale with q in e4m3 (OCP: up to 448, no infinities), dense, one byte a number,
 *             and scale[row] = max |y| / 448 of the row (float32; q is y where that is 0)
 *   backward: s as above (ld lds), dy the gradient of y, dsum that of s; either may be NULL for 0.  dx is that of x and of the
 *             residual alike; dw channels numbers of param_dtype.  dx or dw may be NULL.
 * Limits: rows < 2^31, channels <= 2^20.
 */
int da_rms_norm_workspace(int dtype, int64_t rows, int64_t channels, size_t *backward_bytes /* host, out */);
int da_rms_norm(int dtype, int64_t rows, int64_t channels, const void *x, int64_t ldx, const void *residual, int64_t ldr,
                const void *w, int param_dtype, float eps, void *sum, void *y, void *stream);
int da_rms_norm_e4m3(int dtype, int64_t rows, int64_t channels, const void *x, int64_t ldx, const void *residual, int64_t ldr,
                     const void *w, int param_dtype, float eps, void *sum, void *q, float *scale, void *stream);
int da_rms_norm_backward(int dtype, int64_t rows, int64_t channels, const void *s, int64_t lds, const void *dy, int64_t ldy,
                         const void *dsum, int64_t ldd, const void *w, int param_dtype, float eps, void *dx, void *dw,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Cross entropy of a linear layer, by pieces of the classes, without keeping logits:
 *
 *   z = x . w + b,  loss[r] = log sum_j exp z[r,j] - z[r, target[r]]
 *   dz[r,j] = g[r] (exp(z[r,j]) / sum exp - (j == target[r])),  dx = dz . w^T,  dw = x^T . dz,  db = sum of dz over the rows
 *
 * A row whose target is outside 0 .. classes-1 (-1, say) has none: its loss and its row of dx are 0, and it takes no
 * part in anything else, whatever its x holds.
 *
 *   x         rows x d, ldx >= d;  w  d x classes, dense;  both of dtype
 *   b         classes numbers of param_dtype; NULL for 0
 *   target    rows, int32 or (target64 != 0) int64
 *   loss      float32[rows] (DA_LOSS_ROWS), or one number: the sum over the rows, or that over the number of rows with a
 *             target (DA_LOSS_MEAN; 0 where there is none)
 *   stats     written by the forward call and read by the backward call on the same arguments (which rows have a target,
 *             their log sum exp, the magnitudes of x and w), 16-byte aligned; da_linear_cross_entropy_sizes says how many bytes
 *   dloss     float32, like loss; dloss_stride (DA_LOSS_ROWS) 0 takes dloss[0] for every row
 *   dx, dw, db   dense, of the types of x, w and b; any of them may be NULL and is then not computed
 *
 * The backward call computes the logits again, a piece of the classes at a time: workspaces hold x and w packed and dz of a
 * piece, up to 512 MB or 1024 classes (for few rows: all logits and dz, in 32 bits).  Sums are held in 32 bits.
 *
 * Products are of 32-bit numbers for both types up to 128 classes of up to 256 inner positions (with many of both: up to 64
 * classes), and up to 64 rows (bfloat16: 32).  Beyond that operands are packed for the 16-bit matrix cores:
 *   bfloat16   dz has the 11 bits of fp16 for dx and dw; x and w are exact
 *   float32    is multiplied as pairs of fp16, 22 bits of a number
 * Small numbers have fewer bits: those of a row of x are off by up to 2^-35 of the row's largest (float32), those of dz by 2^-40
 * of the row's factor, those of w by 2^-40 of the largest of all (bfloat16: of its line).  Loss and dx of a row do not depend on
 * other rows; to dw a row adds with an error of up to 2^-37 of the largest product of any row's largest x and its factor.
 *
 * Limits: rows <= 2^26, d, classes <= 2^22, and fewer than 2^23 tiles of 256 x 256 of any of the products' results
 * (DA_ERR_UNSUPPORTED beyond).
 */
enum { DA_LOSS_ROWS = 0, DA_LOSS_SUM = 1, DA_LOSS_MEAN = 2 };
int da_linear_cross_entropy_sizes(int dtype, int64_t rows, int64_t d, int64_t classes, size_t *stats_bytes, size_t *forward_bytes,
                                  size_t *backward_bytes /* host, out */);
int da_linear_cross_entropy(int dtype, int64_t rows, int64_t d, int64_t classes, const void *x, int64_t ldx, const void *w,
                            const void *b, int param_dtype, const void *target, int target64, int reduction, float *loss,
                            void *stats, void *workspace, size_t workspace_bytes, void *stream);
int da_linear_cross_entropy_backward(int dtype, int64_t rows, int64_t d, int64_t classes, const void *x, int64_t ldx,
                                     const void *w, const void *b, int param_dtype, int reduction, const void *stats,
                                     const float *dloss, int64_t dloss_stride, void *dx, void *dw, void *db, void *workspace,
                                     size_t workspace_bytes, void *stream);

/*
 * Orthogonalised updates: `batch` matrices g of rows x cols towards the nearest matrix with orthonormal rows or columns
 * (the shorter ones), by `steps` steps of an odd polynomial of the singular values:
 *
 *   X = g / (|g| + eps)  (Frobenius norm),   then for each step's (a, b, c):   A = X X^T,  X <- a X + (b A + c A^2) X
 *
 * (for rows > cols of the transposed matrix).  Products are of pairs of 16-bit halves with 22 bits for both types; sums are held in 32
 * bits, the norm's in 64.  bfloat16 is rounded to once, at the end.
 *
 *   g         of dtype; neighbouring columns, rows ldg, matrices `stride` numbers apart
 *   coefficients   host, 3 steps numbers.  Those with which singular values could grow beyond 128 or b x + c x^2 beyond 2^12
 *             are refused (DA_ERR_INVALID_ARG).
 *   out       dense, of dtype
 * Limits: rows, cols <= 2^17, batch <= 65535 and batch times tiles of 64 x 64 < 2^30 (DA_ERR_UNSUPPORTED beyond), 0 <= steps <= 64.
 */
int da_orthogonalise_workspace(int dtype, int64_t batch, int64_t rows, int64_t cols, int steps, size_t *bytes /* host, out */);
int da_orthogonalise(int dtype, int64_t batch, int64_t rows, int64_t cols, const void *g, int64_t ldg, int64_t stride, int steps,
                     const float *coefficients, float eps, void *out, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DA_TRAINING_H */
