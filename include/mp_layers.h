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

/* ---------------------------------------------------------------------------
 * Microscaled 4-bit floating point (OCP Microscaling Formats, 2023: MXFP4).
 * A row of K values is cut into blocks of 32, KB = ceil(K / 32) of them.  A
 * block has one scale byte s (E8M0: 2^(s - 127); 255: every value is NaN)
 * and 32 four-bit codes (E2M1: sign, and 0, 0.5, 1, 1.5, 2, 3, 4 or 6).
 * Layout of a table of N rows: codes [N, KB * 16] bytes, element i of a row in
 * byte i / 2, the lower nibble first; scales [N, KB] bytes.  The places past
 * K of a last block hold code 0.
 * Quantisation: the scale of a block is 2^(floor(log2 max|x|) - 2), no less
 * than 2^-127 (a block of zeros has s = 0); values are divided by it, rounded
 * to nearest with ties to the even code, and saturate at 6.  A block that
 * holds an infinity or NaN gets s = 255.
 * ------------------------------------------------------------------------- */

/* x [N, K] of dtype, row stride ldx -> codes and scales (both or neither), and
 * the values that they stand for, [N, K] contiguous of dtype, or NULL (for
 * training with quantised values; exact in either type).  0 <= N <=
 * INT32_MAX, 1 <= K <= 65536.  codes 16-byte aligned. */
int mp_mx_quantize(const void* x, int dtype, int64_t N, int64_t K, int64_t ldx, uint8_t* codes,
                   uint8_t* scales, void* values, void* stream);

/* The values that codes and scales stand for: out [N, K] contiguous of dtype. */
int mp_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K,
                     void* out, int dtype, void* stream);

/* Workspace bytes of mp_mx_segment_matmul (the rows' codes and scales, and all
 * scales in the order in which they are read). */
int mp_mx_segment_matmul_workspace(int64_t T, int64_t N, int64_t K, int64_t Fo, size_t* bytes);

/* out[r, o] = sum over k of q(x)[r, k] * W[t][o, k] for the rows r of segment t:
 * mp_segment_matmul for serving, on 4-bit matrix cores, with W quantised
 * along its input channels ([Fo, K] a type: transposed against mp.h) and
 * the rows of x quantised (as mp_mx_quantize does) on the way.
 *   seg     [T+1] of seg_itype on the DEVICE (the rowptr of a dispatch):
 *           seg[0] = 0, non-decreasing, seg[T] = N (offsets outside [0, N]
 *           are taken as the nearest in it; rows of no segment are not written).
 *   x       [N, K] of x_dtype, row stride ldx.
 *   w_codes [T, Fo, KB * 16], w_scales [T, Fo, KB].
 *   out     [N, Fo] contiguous of out_dtype, from fp32 sums.
 * Sizes: 0 <= N <= INT32_MAX, 1 <= T <= 4096, 1 <= K, Fo <= 65536, and where K > 128 or
 * Fo > 256 also (N / 128 + min(T, N)) * ceil(Fo / 256) <= 2^24 - 8 (the tiles of a
 * launch); w_codes and ws 16-byte aligned. */
int mp_mx_segment_matmul(const void* seg, int seg_itype, int64_t T, const void* x, int x_dtype,
                         int64_t N, int64_t K, int64_t ldx, const uint8_t* w_codes,
                         const uint8_t* w_scales, int64_t Fo, void* out, int out_dtype, void* ws,
                         size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MP_LAYERS_H_ */
