/*
 * mp_layers.h -- C ABI of the operators around the aggregation: what a sparse
 * expert layer over node features needs next to message passing (mp.h) and
 * its typed products.  Part of libmp.so.
 *
 *   mp_group_norm       group norm with an activation over the nodes of each
 *                       graph of a batch (channels last), and its gradients
 *   mp_dropout          dropout from a counter-based generator; no mask is
 *                       stored, the gradient draws it again
 *   mp_route            softmax router: k experts a row, per-expert counts,
 *                       balance and z losses, and its gradient
 *   mp_mx_*             microscaled 4-bit floating point: quantisation, and
 *                       the product of row segments with 4-bit weights
 *
 * The dispatch between them is mp.h's: mp_coo_to_csr of (row, expert) pairs
 * sorts rows by expert and its rowptr is the segments of the products;
 * mp_message_gather copies the rows; mp_spmm with the router's weights adds
 * the experts' results up.
 *
 * Conventions are mp.h's: device arrays owned by the caller, host argument
 * checks before anything is enqueued, no allocation, no floating-point
 * atomics, every call asynchronous on `stream` and deterministic.  Sums,
 * statistics and normalisers are held in fp32; a bf16 output is rounded to
 * nearest even once.
 */
#ifndef MP_LAYERS_H_
#define MP_LAYERS_H_

#include "mp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * Group norm with an activation, over segments of consecutive rows.
 * Segment s holds rows ptr[s] <= r < ptr[s+1] (the graphs of a batch; ptr as
 * for mp_readout_multi), group g the channels g * F/G <= c < (g+1) * F/G.
 *   mean[s, g], var[s, g]  over the segment's rows and the group's channels
 *                          (population variance);  rstd = 1/sqrt(var + eps)
 *   xhat = (x - mean) * rstd,  z = xhat * gamma[c] + beta[c],  out = act(z)
 * The variance is taken about the mean (no difference of large squares).  An
 * empty segment has mean = rstd = 0.
 * ------------------------------------------------------------------------- */

typedef enum mp_act {
    MP_ACT_NONE = 0,
    MP_ACT_RELU = 1, /* max(z, 0), derivative 0 at z = 0 */
    MP_ACT_SILU = 2, /* z / (1 + exp(-z)) */
    MP_ACT_GELU = 3  /* z * (1 + erf(z / sqrt 2)) / 2 */
} mp_act;

/* Workspace bytes of mp_group_norm (backward = 0) or mp_group_norm_backward
 * (backward = 1) for N rows, S segments, F channels of x_dtype and G groups. */
int mp_group_norm_workspace(int64_t N, int64_t S, int64_t F, int64_t G, int x_dtype,
                            int backward, size_t* bytes);

/* Forward.
 *   ptr          [S+1] of ptr_itype: ptr[0] = 0, non-decreasing, ptr[S] = N
 *                (offsets outside [0, N] are taken as the nearest in it).
 *   x            [N, F] of x_dtype, row r at element r * ldx (ldx >= F).
 *   gamma, beta  [F] fp32 or NULL (1 and 0).
 *   eps          added to the variance, >= 0 and finite.
 *   out          [N, F] contiguous, of out_dtype; must not overlap x.
 *   mean, rstd   [S, G] fp32, written (the gradient takes them).
 * Sizes: 0 <= N, 1 <= S, both <= INT32_MAX, 1 <= F <= 65536, 1 <= G <= F and
 * F % G = 0. */
int mp_group_norm(const void* ptr, int ptr_itype, const void* x, int x_dtype, int64_t N,
                  int64_t S, int64_t F, int64_t ldx, int64_t G, const float* gamma,
                  const float* beta, float eps, int act, void* out, int out_dtype, float* mean,
                  float* rstd, void* ws, size_t ws_bytes, void* stream);

/* Gradients given dout = dL/dout [N, F] of x_dtype (contiguous) and the
 * forward's mean and rstd; ptr, x, gamma, beta and act as in the forward.
 *   da = dout * act'(z)
 *   dx[r, c]  = rstd * (gamma da - mean(gamma da) - xhat mean(gamma da xhat)),
 *               the means over the segment's rows and the group's channels
 *   dgamma[c] = sum over all rows of da * xhat,  dbeta[c] = sum of da
 *   dx           [N, F] contiguous of dx_dtype, or NULL; must not overlap x
 *                or dout.
 *   dgamma, dbeta  [F] fp32, both or neither; not all three outputs NULL. */
int mp_group_norm_backward(const void* ptr, int ptr_itype, const void* x, int x_dtype,
                           const void* dout, int64_t N, int64_t S, int64_t F, int64_t ldx,
                           int64_t G, const float* gamma, const float* beta, const float* mean,
                           const float* rstd, int act, void* dx, int dx_dtype, float* dgamma,
                           float* dbeta, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Dropout from a counter-based generator.  Element f of row r has the number
 * e = id(r) * F + f (or, with whole_rows, e = id(r) for the whole row), where
 * id(r) = ids[r], or r without ids.  Its random word is the (e % 8)-th 16-bit
 * word of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random
 * numbers: as easy as 1, 2, 3", 2011) with key (seed low, seed high) and
 * counter (e / 8 low, e / 8 high, t low, t high), t = offset + *step.
 * With limit = round(65536 p) the element stays iff word >= limit, multiplied
 * by 65536 / (65536 - limit): the expectation is kept exactly, at a
 * probability that is a multiple of 2^-16.  A dropped element is +0 whatever
 * it held (infinities and NaN included).
 * The mask is a function of (seed, offset, step, id, f) alone: the gradient
 * with respect to x is the same call on the output's gradient without a
 * residual, and with ids the edges of a CSR and of its transpose (ids = the
 * COO numbers of either order) are dropped alike.
 *   x         [N, F] of dtype, row r at element r * ldx.
 *   residual  [N, F] of dtype, row stride ldr, added to what stays, or NULL.
 *   ids       [N] int32, >= 0, or NULL.
 *   p         in [0, 1] (1 drops everything).
 *   step      [1] int64 on the device, or NULL (0): read when the call runs,
 *             so that a captured graph draws anew on each replay.
 *   out       [N, F] of dtype, row stride ldo; may be x or residual itself
 *             (same address and stride), must not overlap them otherwise.
 * Sizes: 0 <= N <= INT32_MAX, 1 <= F <= 65536, strides >= F.
 * ------------------------------------------------------------------------- */
int mp_dropout(const void* x, int dtype, int64_t N, int64_t F, int64_t ldx,
               const void* residual, int64_t ldr, const int32_t* ids, int whole_rows, double p,
               uint64_t seed, uint64_t offset, const int64_t* step, void* out, int64_t ldo,
               void* stream);

/* ---------------------------------------------------------------------------
 * Softmax router with per-expert counts, a balance loss and a z loss.  A row
 * takes part iff its mask is nonzero (no mask: every row) and it has a logit
 * above -inf; an expert whose logit is -inf is never chosen.  Of a row that
 * takes part:
 *   idx[r, j]    the expert of the j-th largest logit (equal logits: the
 *                lower number first), or -1 where fewer than j+1 are above
 *                -inf
 *   weight[r, j] exp(logit) over the sum of exp of the row's chosen logits
 *                (renorm = 1) or of all its logits (renorm = 0); 0 where
 *                idx is -1
 * All rows that take part, R of them, give
 *   counts[e]    how often expert e was chosen; counts[E] = R
 *   loss[0]      E * sum_e (counts[e] / sum of counts) * P_e, P_e = the mean
 *                softmax probability of expert e (the balance loss: 1 where
 *                all experts are chosen alike)
 *   loss[1]      the mean of logsumexp(row)^2 (the z loss)
 * both 0 if R = 0.  Other rows have idx -1, weight 0, and whatever they hold
 * (NaN included) reaches no output.  NaN in a row that takes part makes its
 * weights and the losses NaN (idx stays in range).
 *   logits  [N, E] of dtype, row stride ldl;  mask [N] bytes or NULL.
 * Sizes: 0 <= N <= INT32_MAX, 1 <= E <= 1024, 1 <= k <= min(E, 64),
 * N * k <= INT32_MAX (the counts).
 * ------------------------------------------------------------------------- */

/* Workspace bytes of mp_route (partial sums of the losses). */
int mp_route_workspace(int64_t N, int64_t E, size_t* bytes);

int mp_route(const void* logits, int dtype, int64_t N, int64_t E, int64_t ldl, int64_t k,
             const uint8_t* mask, int renorm, int32_t* idx, float* weight, int32_t* counts,
             float* loss, void* ws, size_t ws_bytes, void* stream);

/* dL/dlogits, given dweight = dL/dweight [N, k] fp32 (or NULL: 0) and dloss =
 * dL/dloss [2] fp32 on the device (or NULL: 0), with the forward's idx,
 * weight and counts (the choice itself and the counts have no gradient):
 *   dlogits  [N, E] contiguous of dtype, written in full (0 for rows that take
 *            no part); must not overlap logits. */
int mp_route_backward(const void* logits, int dtype, int64_t N, int64_t E, int64_t ldl,
                      int64_t k, const uint8_t* mask, int renorm, const int32_t* idx,
                      const float* weight, const int32_t* counts, const float* dweight,
                      const float* dloss, void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MP_LAYERS_H_ */
