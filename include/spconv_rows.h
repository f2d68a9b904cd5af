/* spconv_rows.h - operators on feature rows (one row per active site) of the
 * MI355X (gfx950) sparse-convolution library: what a block between two
 * convolutions does with the [n][C] features they leave behind.
 *
 *   layer norm   every row normalised, and its gradients;
 *   dropout      elements dropped by a counter-based generator, added to a
 *                residual; no mask is stored;
 *   route        every row's k largest logits, their softmax weights, and the
 *                (row, slot) pairs grouped by expert;
 *   grouped      products of ragged groups of rows, each group with its own
 *                weights, and their gradients;
 *   combine      the weighted sum of a row's expert outputs, and its gradients;
 *   rms norm     the residual added, every row divided by its root mean square,
 *                its output in the rows' type or in 8 bits, and its gradients;
 *   linear       dense products with bias, activation and residual, of rows in
 *                bf16, fp32 or 8 bits, and their gradients;
 *   route scores routing by sigmoid or softmax scores with a bias for balance,
 *                in groups of experts, and its gradient;
 *   8-bit rows   rows kept in 8 bits (a checkpoint of activations), as values
 *                again, and as operands of the gradients above.
 *
 * Conventions shared by every entry point (statuses and dtypes are those of
 * spconv.h)
 * ---------------------------------------
 * Memory.  Pointers are device pointers owned by the caller: contiguous,
 *          row-major, aligned to their element (no wider alignment is needed,
 *          so rows of any width and views at any element offset can be passed).
 *          Outputs are fully overwritten and must not overlap inputs, except
 *          where stated.  A pointer to no elements may be NULL.  Nothing is
 *          allocated; workspaces are the caller's, 16-byte aligned, need no
 *          initialisation and may be reused as soon as the call's work is done.
 * Sizes.   Row counts are in [0, 2^31), widths in [1, 2^31).  Element offsets
 *          are 64-bit.  A call with no rows is valid (weight gradients are then
 *          zero).
 * Streams. `stream` is a hipStream_t passed as void*.  All work is enqueued on
 *          it; no call waits for the device, and every call can be captured
 *          into a HIP graph.
 * Results. Sums, statistics and weights are held in fp32 and rounded once to
 *          the output's type (round to nearest even).  No atomics decide an
 *          order of summation: repeated calls give bit-identical results.
 * 8 bits.  Rows in 8 bits are e4m3 values q [n][C] (4 bits of exponent, 3 of
 *          mantissa, no infinity) and an fp32 scale a row; they stand for
 *          q * scale.  Written with top the row's largest magnitude, at least
 *          2^-100: scale = top / 448, q = v * (448 / top) rounded to nearest
 *          even.  A row with an infinity or NaN gets scale NaN and q = 0: it
 *          stands for NaN.  Where an argument's dtype can be SPCONV_E4M3, its
 *          scale is the pointer beside it, NULL for the other dtypes.
 * Indices. offsets, rows and pos are read on the device.  Entries out of range
 *          are never followed (each entry point says what they count as).
 * Errors.  EINVAL for a bad dtype, size, flag, NULL, misaligned or too small
 *          argument, or for more rows than one launch holds (2^32 threads: beyond
 *          100 GB of features; layer norm adds up dgamma and dbeta of at most
 *          16,776,960 columns), found on the host before any work is enqueued;
 *          EHIP.
 */
#ifndef SPCONV_ROWS_H
#define SPCONV_ROWS_H

#include "spconv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Experts and slots a routing can have. */
#define SPCONV_ROUTE_MAX_EXPERTS 1024
#define SPCONV_ROUTE_MAX_SLOTS 16
/* Groups of experts. */
#define SPCONV_ROUTE_MAX_GROUPS 64

/* Rows in 8 bits (a dtype where an entry point says so). */
#define SPCONV_E4M3 2

/* Scores of a routing. */
#define SPCONV_SCORE_SIGMOID 0
#define SPCONV_SCORE_SOFTMAX 1

/* Activations: z; max(z, 0); z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2;
 * z / (1 + exp(-z)).  Before they are rounded to the result's type, values are
 * within 8 units (2^-24) of |z|, those of the last one in fp32 also within 16 of
 * their own size down to z = -80; slopes within 32 + 2 |z| units of 1. */
#define SPCONV_ACT_NONE 0
#define SPCONV_ACT_RELU 1
#define SPCONV_ACT_GELU 2
#define SPCONV_ACT_SILU 3

/* Layer norm of every row:
 *   mean = sum x / C, rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),
 *   y = (x - mean) * rstd * gamma + beta.
 *   dt          dtype of x and y
 *   gamma, beta fp32 [C] or NULL (1 and 0)
 *   eps         >= 0 and finite
 *   mean, rstd  fp32 [n] for the gradient, or NULL (both or neither)
 * The variance is summed from the differences to the mean. */
int spconv_layer_norm_forward(int dt, const void* x, const float* gamma, const float* beta,
                              float eps, void* y, float* mean, float* rstd, int64_t n, int C,
                              void* stream);

/* Workspace bytes of spconv_layer_norm_backward with dgamma and dbeta. */
int spconv_layer_norm_backward_workspace(int64_t n, int C, size_t* bytes);

/* Gradients of the layer norm.  With z = (x - mean) * rstd and h = dy * gamma:
 *   dx     = rstd * (h - sum h / C - z * sum (h z) / C)
 *   dgamma = sum over rows of dy * z,  dbeta = sum over rows of dy   (fp32 [C])
 * dx has dtype dt.  dgamma and dbeta are given both or neither; without them
 * no workspace is needed (NULL, 0). */
int spconv_layer_norm_backward(int dt, const void* dy, const void* x, const float* mean,
                               const float* rstd, const float* gamma, void* dx, float* dgamma,
                               float* dbeta, int64_t n, int C, void* workspace,
                               size_t workspace_bytes, void* stream);

/* Dropout of `count` < 2^34 elements in flat order:
 *   y[i] = residual[i] + (u(i) >= round(p * 2^32) ? x[i] / (1 - p) : 0)
 * where u(i) is word i % 4 of Philox4x32 with 7 rounds (Salmon, Moraes, Dror
 * and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) for the
 * counter (i / 4, offset + *step), each 64 bits wide, low word first, under the
 * 64-bit key `seed`.  An element dropped contributes exactly zero, whatever it
 * holds.
 *   p         0 <= p < 1; 1 / (1 - p) is rounded to fp32
 *   residual  dtype dt, or NULL (= 0)
 *   step      one uint64 in device memory added to offset, or NULL (= 0): a
 *             captured graph that counts it up drops other elements each replay
 *   y         may be x or residual itself (in place) */
int spconv_dropout_forward(int dt, const void* x, const void* residual, double p, uint64_t seed,
                           uint64_t offset, const uint64_t* step, void* y, int64_t count,
                           void* stream);

/* Gradient of the dropout with respect to x: the forward's elements of dy,
 * times 1 / (1 - p), from the same p, seed, offset and *step.  (The gradient of
 * the residual is dy.)  dx may be dy itself. */
int spconv_dropout_backward(int dt, const void* dy, double p, uint64_t seed, uint64_t offset,
                            const uint64_t* step, void* dx, int64_t count, void* stream);

/* Workspace bytes of spconv_route_forward. */
int spconv_route_workspace(int64_t n, int E, int k, size_t* bytes);

/* Routing: every row is sent to the experts of its k largest logits.
 *   logits   dtype dt, [n][E]; 1 <= E <= SPCONV_ROUTE_MAX_EXPERTS
 *   k        1 <= k <= min(E, SPCONV_ROUTE_MAX_SLOTS); n * k < 2^31
 *   experts  int32 [n][k]: largest logit first, of equal ones the lowest
 *            expert.  A logit of -infinity is never chosen: a row with fewer
 *            than k others has -1 in its last slots.  NaN ranks above every
 *            number.
 *   weights  fp32 [n][k]: normalize = 1: the softmax of the chosen logits;
 *            normalize = 0: the chosen entries of the softmax of the whole
 *            row.  0 where no expert is chosen; NaN (or +infinity) in a row's
 *            logits makes its weights NaN as exp and / do.
 *   offsets  int32 [E+1]: expert e's pairs are the positions offsets[e] up to
 *            offsets[e+1]; offsets[0] = 0, offsets[E] = pairs chosen in all
 *   rows     int32 [n*k]: the row of every position, ascending within an
 *            expert; -1 from position offsets[E] on
 *   pos      int32 [n][k]: the position of every (row, slot), -1 for none */
int spconv_route_forward(int dt, const void* logits, int64_t n, int E, int k, int normalize,
                         int32_t* experts, float* weights, int32_t* offsets, int32_t* rows,
                         int32_t* pos, void* workspace, size_t workspace_bytes, void* stream);

/* Gradient of the routing's weights with respect to the logits (the choice
 * itself has none).  With D = sum over slots of weights * dweights:
 *   normalize = 1: dlogits = weight * (dweight - D) on the chosen experts
 *   normalize = 0: dlogits = p * ([chosen] dweight - D), p the row's softmax
 * and 0 elsewhere.  dweights of slots without an expert are not read into
 * anything.  logits (dtype dt) are read with normalize = 0 only and may be NULL
 * with 1; dlogits has dtype dt, [n][E]. */
int spconv_route_backward(int dt, const float* dweights, const void* logits,
                          const int32_t* experts, const float* weights, int64_t n, int E, int k,
                          int normalize, void* dlogits, void* stream);

/* Products of ragged groups: position j of group e (offsets[e] <= j <
 * offsets[e+1]) has
 *   y[j] = act(x[rows[j]] W[e] + bias[e]),  act(z) = relu && z < 0 ? 0 : z
 *   in_dt    dtype of x and w
 *   x        [n_x][C_in]
 *   w        [E][C_in][C_out]
 *   offsets  int32 [E+1], ascending within [0, m]; values outside are moved
 *            into that range, and one below those before it counts as the largest
 *            of them: a descending pair is an empty group, and no position has two
 *   rows     int32 [m] or NULL (position j reads row j); an entry outside
 *            [0, n_x) reads a row of zeros
 *   bias     fp32 [E][C_out] or NULL
 *   y        dtype out_dt, [m][C_out]; positions from offsets[E] on are zero
 * 1 <= E <= 65535, C_in and C_out up to 2^23; offsets[0] must be 0.  Non-finite values reach the
 * positions whose rows or group hold them, and no others. */
int spconv_grouped_forward(int in_dt, const void* x, int64_t n_x, const void* w,
                           const int32_t* offsets, const int32_t* rows, const float* bias,
                           int relu, int out_dt, void* y, int64_t m, int E, int C_in, int C_out,
                           void* stream);

/* Gradient of the grouped products with respect to the rows they read, per
 * position:  dx[j] = keep(dy[j] W[e]^T).
 *   dt    dtype of dy [m][C_out] and w [E][C_in][C_out]
 *   mask  dtype out_dt, [m][C_in], or NULL: an element of dx whose mask is <= 0
 *         is 0 (the gradient of the ReLU the layer's input came out of)
 *   dx    dtype out_dt, [m][C_in]; positions from offsets[E] on are zero
 * For gathered rows, spconv_combine_forward without weights sums the positions
 * of each row. */
int spconv_grouped_backward_data(int dt, const void* dy, const void* w, const int32_t* offsets,
                                 const void* mask, int out_dt, void* dx, int64_t m, int E,
                                 int C_in, int C_out, void* stream);

/* Workspace bytes of spconv_grouped_backward_weight. */
int spconv_grouped_backward_weight_workspace(int dt, int64_t m, int E, int C_in, int C_out,
                                             size_t* bytes);

/* Gradients of the groups' weights and biases:
 *   dw[e] = sum over the group's positions j of x[rows[j]]^T dy[j]
 *   db[e] = sum over the group's positions j of dy[j]
 *   dt      dtype of x [n_x][C_in] and dy [m][C_out]
 *   dw      fp32 [E][C_in][C_out];  db fp32 [E][C_out] or NULL
 * A group without positions gets zeros.  Large groups are summed in chunks of a
 * size fixed by the arguments, the chunks in ascending order. */
int spconv_grouped_backward_weight(int dt, const void* x, int64_t n_x, const void* dy,
                                   const int32_t* offsets, const int32_t* rows, float* dw,
                                   float* db, int64_t m, int E, int C_in, int C_out,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* Weighted sum of the positions of every row:
 *   out[i] = residual[i] + sum over slots s of weights[i][s] * y[pos[i][s]]
 *   dt        dtype of y [m][C], residual and out [n][C]
 *   pos       int32 [n][k]; an entry outside [0, m) adds nothing
 *   weights   fp32 [n][k] or NULL (= 1)
 *   residual  or NULL (= 0); may be out itself
 * 1 <= k <= SPCONV_ROUTE_MAX_SLOTS.  Slots are added in order. */
int spconv_combine_forward(int dt, const void* y, int64_t m, const int32_t* pos,
                           const float* weights, const void* residual, void* out, int64_t n,
                           int k, int C, void* stream);

/* Gradients of the weighted sum:
 *   dy[pos[i][s]] = weights[i][s] * dout[i],  dweights[i][s] = <dout[i], y[pos[i][s]]>
 *   count     one int32 in device memory: positions from *count on, which no
 *             pos may refer to, are set to zero (a routing's offsets[E]);
 *             NULL: all m positions are referred to
 *   dweights  fp32 [n][k] or NULL (y may then be NULL); 0 where pos is outside
 *             [0, m)
 * Every position below *count must be referred to by exactly one pos, as a
 * routing's are. */
int spconv_combine_backward(int dt, const void* dout, const void* y, const int32_t* pos,
                            const float* weights, const int32_t* count, void* dy,
                            float* dweights, int64_t m, int64_t n, int k, int C, void* stream);

/* Root-mean-square norm with the residual's addition:
 *   h = x + residual rounded to dt (x itself without a residual),
 *   rstd = 1 / sqrt(sum h^2 / C + eps),  y = h * rstd * gamma.
 *   dt        dtype of x, residual and h
 *   residual  or NULL
 *   gamma     fp32 [C] or NULL (1)
 *   eps       >= 0 and finite (sum h^2 is in fp32: |h| below 1e19 / sqrt(C))
 *   h         [n][C], or NULL if it is not wanted (NULL without a residual); may
 *             be x or residual itself
 *   out_dt    dt, or SPCONV_E4M3: y is then in 8 bits, packed from fp32, y_scale
 *             its scales
 *   rstd      fp32 [n] for the gradient, or NULL */
int spconv_rms_norm_forward(int dt, const void* x, const void* residual, const float* gamma,
                            float eps, void* h, int out_dt, void* y, float* y_scale, float* rstd,
                            int64_t n, int C, void* stream);

/* Workspace bytes of spconv_rms_norm_backward with dgamma. */
int spconv_rms_norm_backward_workspace(int64_t n, int C, size_t* bytes);

/* Gradients of the norm.  With z = h * rstd and g = dy * gamma:
 *   dx     = rstd * (g - z * sum (g z) / C) + dh     (the residual's is the same)
 *   dgamma = sum over rows of dy * z                  (fp32 [C])
 *   h_dt   dt, or SPCONV_E4M3: h was kept in 8 bits
 *   dh     what reaches h past the norm, dtype dt, or NULL (0)
 * dgamma may be NULL; without it no workspace is needed (NULL, 0).  An output in
 * 8 bits has the gradient of the values it was rounded from. */
int spconv_rms_norm_backward(int dt, const void* dy, int h_dt, const void* h, const float* h_scale,
                             const float* rstd, const float* gamma, const void* dh, void* dx,
                             float* dgamma, int64_t n, int C, void* workspace,
                             size_t workspace_bytes, void* stream);

/* Rows x [n][C] of dtype dt in 8 bits. */
int spconv_pack_rows(int dt, const void* x, void* q, float* scale, int64_t n, int C, void* stream);

/* y = act(q * scale), [n][C] of dtype out_dt. */
int spconv_unpack_rows(const void* q, const float* scale, int act, int out_dt, void* y, int64_t n,
                       int C, void* stream);

/* Gradient of an activation: dz = dy * act'(pre), with pre [n][C] the
 * activation's input, of dtype pre_dt = dt or SPCONV_E4M3.  The ReLU's slope at 0
 * is 0.  dz may be dy itself. */
int spconv_activation_backward(int dt, const void* dy, int pre_dt, const void* pre,
                               const float* pre_scale, int act, void* dz, int64_t n, int C,
                               void* stream);

/* Dense products:  z = x w + bias,  y = act(z) + residual.
 *   in_dt     dtype of x [n][C_in]; that of w [C_in][C_out] too, bf16 for rows in
 *             8 bits
 *   bias      fp32 [C_out] or NULL
 *   residual  dtype out_dt, [n][C_out], or NULL; may be y itself
 *   y, z      dtype out_dt, [n][C_out]; z NULL if it is not wanted (the gradient
 *             of an activation takes it); y is computed from the unrounded z
 * C_in and C_out up to 2^23, C_in * C_out < 2^31. */
int spconv_linear_forward(int in_dt, const void* x, const float* x_scale, const void* w,
                          const float* bias, int act, const void* residual, int out_dt, void* y,
                          void* z, int64_t n, int C_in, int C_out, void* stream);

/* Gradient of the product with respect to its input, through the activation that
 * the input came out of:  dx = (dy w^T) * act'(pre).
 *   dt      dtype of dy [n][C_out] and w
 *   act     that activation; SPCONV_ACT_NONE: dx = dy w^T, pre NULL
 *   pre     [n][C_in], its input, of dtype pre_dt = out_dt or SPCONV_E4M3
 *   dx      dtype out_dt, [n][C_in] */
int spconv_linear_backward_data(int dt, const void* dy, const void* w, int act, int pre_dt,
                                const void* pre, const float* pre_scale, int out_dt, void* dx,
                                int64_t n, int C_in, int C_out, void* stream);

/* Workspace bytes of spconv_linear_backward_weight. */
int spconv_linear_backward_weight_workspace(int x_dt, int64_t n, int C_in, int C_out,
                                            size_t* bytes);

/* Gradients of the weights and the bias:  dw = x^T dy,  db = sum over rows of dy.
 *   x_dt  dtype of x [n][C_in]; that of dy [n][C_out] too, bf16 for rows in 8 bits
 *   dw    fp32 [C_in][C_out];  db fp32 [C_out] or NULL
 * Many rows are summed in chunks of a size fixed by the arguments, the chunks in
 * ascending order.  The factor x_scale * dy of rows in 8 bits is rounded to fp32. */
int spconv_linear_backward_weight(int x_dt, const void* x, const float* x_scale, const void* dy,
                                  float* dw, float* db, int64_t n, int C_in, int C_out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* Routing by scores s = sigmoid(logit) or the softmax of the row's logits:
 *   bias        fp32 [E] or NULL (0): added to the scores for the choice alone
 *   groups      the experts are so many groups of E / groups adjacent ones, at
 *               most SPCONV_ROUTE_MAX_GROUPS; a group is worth the sum of its two
 *               largest biased scores (its one's), and the top_groups worth most,
 *               of equal ones the lowest, stay
 *   k           1 <= k <= min(SPCONV_ROUTE_MAX_SLOTS, top_groups * E / groups)
 *   experts     int32 [n][k]: of the groups that stay, the largest biased score
 *               first, of equal ones the lowest expert.  Scores are compared as
 *               64-bit arithmetic has them.  An expert whose logit or biased
 *               score is -infinity is never chosen (-1 in the slots left over);
 *               NaN ranks above every number.
 *   weights     fp32 [n][k]: the chosen scores without the bias; normalize = 1:
 *               divided by their sum, the scores 64-bit numbers here too (0 where
 *               the sum is 0); times scale (> 0 and finite).  0 where no expert is
 *               chosen.
 *   offsets, rows, pos and the workspace (spconv_route_workspace) as for
 *               spconv_route_forward */
int spconv_route_scores_forward(int dt, const void* logits, const float* bias, int64_t n, int E,
                                int k, int score, int groups, int top_groups, int normalize,
                                float scale, int32_t* experts, float* weights, int32_t* offsets,
                                int32_t* rows, int32_t* pos, void* workspace,
                                size_t workspace_bytes, void* stream);

/* Gradient of those weights with respect to the logits (the choice itself has
 * none), dlogits [n][E] of dtype dt.  experts are a forward's: an expert at most
 * once a row.  dweights of slots without an expert are not read into anything.
 * logits may be NULL for softmax scores with normalize = 1. */
int spconv_route_scores_backward(int dt, const float* dweights, const void* logits,
                                 const int32_t* experts, const float* weights, int64_t n, int E,
                                 int k, int score, int normalize, float scale, void* dlogits,
                                 void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPCONV_ROWS_H */
