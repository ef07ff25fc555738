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
 *   mp_embed            embedding rows by id, and the table's gradient
 *   mp_rms_norm         root-mean-square norm with the residual's addition, in
 *                       the rows' type or in 8 bits, and its gradients
 *   mp_expert_mlp       the chosen experts of few rows in one call
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

/* ---------------------------------------------------------------------------
 * Embedding rows by id, times a scale:
 *   out[r] = scale * table[ids[r]]
 * An id outside [0, V), or equal to padding (-1: there is none), is padding:
 * its row is 0 and reaches no gradient.
 *   ids     [N] of ids_itype.
 *   table   [V, F] of dtype, row v at element v * ldt (ldt >= F).
 *   out     [N, F] contiguous of out_dtype; must not overlap the table.
 * Sizes: 0 <= N <= INT32_MAX, 1 <= V < INT32_MAX, 1 <= F <= 65536.
 * ------------------------------------------------------------------------- */
int mp_embed(const void* ids, int ids_itype, int64_t N, const void* table, int dtype, int64_t V,
             int64_t F, int64_t ldt, int64_t padding, float scale, void* out, int out_dtype,
             void* stream);

/* Workspace bytes of mp_embed_backward. */
int mp_embed_backward_workspace(int64_t N, int64_t V, int64_t F, size_t* bytes);

/* dL/dtable given dout = dL/dout [N, F] of dtype, row stride ldd:
 *   dtable[v] = scale * sum over the rows r of id v of dout[r]
 * summed in fp32 in an order that ids and sizes alone set, over rows sorted by id:
 * runs of an id's rows in their order, and what several runs and workgroups have of
 * it joined after that.
 *   dtable  [V, F] contiguous of dtable_dtype, written in full (0 for an id of
 *           no row); must not overlap dout.  All of it is NaN if the sort gave
 *           up (MP_ERR_SORT, as for mp_coo_to_csr).
 *   ws      16-byte aligned. */
int mp_embed_backward(const void* ids, int ids_itype, int64_t N, const void* dout, int dtype,
                      int64_t V, int64_t F, int64_t ldd, int64_t padding, float scale,
                      void* dtable, int dtable_dtype, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Root-mean-square norm of every row, after the residual's addition:
 *   total = x + residual, rounded to dtype (x itself without a residual)
 *   rstd  = 1 / sqrt(mean over the row of total^2 + eps)
 *   out   = total * rstd * weight[c]
 * The norm is that of total as it is stored, from which the gradient starts.
 *   x         [N, F] of dtype, row stride ldx.
 *   residual  [N, F] of dtype, row stride ldr, or NULL.
 *   weight    [F] fp32 or NULL (1).
 *   eps       at least the smallest normal fp32, at most 1e30.
 *   total     [N, F] contiguous of dtype, or NULL; may be x or residual itself
 *             (same address, rows contiguous), must not overlap them otherwise.
 *   out       [N, F] contiguous of out_dtype; must not overlap x, residual or
 *             total.
 *   rstd      [N] fp32 or NULL (the gradient takes it).
 * Sizes: 0 <= N <= INT32_MAX, 1 <= F <= 65536.
 * ------------------------------------------------------------------------- */
int mp_rms_norm(const void* x, int dtype, int64_t N, int64_t F, int64_t ldx, const void* residual,
                int64_t ldr, const float* weight, float eps, void* total, void* out, int out_dtype,
                float* rstd, void* stream);

/* The same with out in microscaled 8-bit floating point (MXFP8 of the OCP
 * Microscaling Formats, 2023, with E4M3 values): KB = ceil(F / 32) blocks of 32
 * values of a row, each with a scale byte s (E8M0: 2^(s - 127); 255: every value
 * is NaN).
 *   codes   [N, KB * 32] bytes, 0 past F, 16-byte aligned;  scales [N, KB] bytes.
 *   values  [N, F] contiguous of dtype: what they stand for (exact in either
 *           type but for bf16 values below 2^-126), or NULL.
 * The scale of a block is 2^(floor(log2 max|out|) - 8), no less than 2^-127 (a
 * block of zeros has s = 0); values are divided by it, rounded to nearest even,
 * and saturate at 448.  A block that holds an infinity or NaN gets s = 255. */
int mp_rms_norm_mx8(const void* x, int dtype, int64_t N, int64_t F, int64_t ldx,
                    const void* residual, int64_t ldr, const float* weight, float eps, void* total,
                    uint8_t* codes, uint8_t* scales, void* values, float* rstd, void* stream);

/* The values that 8-bit codes and scales of that layout stand for: out [N, K]
 * contiguous of dtype; codes 16-byte aligned. */
int mp_mx8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t N, int64_t K,
                      void* out, int dtype, void* stream);

/* Workspace bytes of mp_rms_norm_backward (partial sums of dweight). */
int mp_rms_norm_backward_workspace(int64_t N, int64_t F, int dtype, size_t* bytes);

/* Gradients given dout = dL/dout [N, F] of dtype (contiguous), the forward's total
 * (row stride ldt; x where there was no residual) and rstd:
 *   xhat = total * rstd,  g = dout * weight
 *   dx         = rstd * (g - xhat * mean over the row of g * xhat) + dtotal
 *   dweight[c] = sum over the rows of dout * xhat
 *   dtotal   [N, F] contiguous of dtype: the gradient that reaches total by
 *            itself, or NULL (0).
 *   dx       [N, F] contiguous of dx_dtype, the gradient of x and of residual, or
 *            NULL; must not overlap the inputs.
 *   dweight  [F] fp32 or NULL; not both outputs NULL.
 *   ws       16-byte aligned; none is needed without dweight. */
int mp_rms_norm_backward(const void* total, int dtype, int64_t N, int64_t F, int64_t ldt,
                         const void* dout, const float* rstd, const float* weight,
                         const void* dtotal, void* dx, int dx_dtype, float* dweight, void* ws,
                         size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * The experts of few rows: for serving, all that follows the router, in two
 * launches and without sorting the rows or waiting for the host.
 *   z = w1[e] x,  h = act(z), or with `gated` act(z[0 .. H-1]) * z[H .. 2H-1]
 *   out[r] = residual[r] + sum over the choices j of row r, e = idx[r, j], of
 *            weight[r, j] * w2[e] h
 * A choice with idx outside [0, E) adds nothing; an expert chosen twice by a row
 * counts with both weights.  Weights of experts that no row chose are not read.
 *   x          [N, K] of x_dtype, row stride ldx; or, with x_scales, 8-bit codes
 *              [N, KB * 32] and scales [N, KB] as mp_rms_norm_mx8 writes them
 *              (KB = ceil(K / 32); x_dtype and ldx are not looked at; codes
 *              past K are 0).
 *   idx        [N, k] int32, weight [N, k] fp32: mp_route's.
 *   w1, w2     [E, (1 + gated) H, K] and [E, Fo, H] bf16; or, with w1_scales and
 *              w2_scales (both or neither), 4-bit codes and scales as
 *              mp_mx_quantize writes them for tables of these shapes, 16-byte
 *              aligned (values past the largest fp32 are infinite).
 *   residual   [N, Fo] of out_dtype, row stride ldr, or NULL.
 *   out        [N, Fo] contiguous of out_dtype; may be residual itself (ldr = Fo),
 *              must not overlap the inputs otherwise.
 * An infinite weight makes the sums that it reaches infinite or NaN.
 * Products are exact, of fp32 rows and of h (fp32) too, and sums are in fp32: with the
 * same operands a bf16 out is the fp32 one rounded once (after the residual).
 * Values of rows and weights, and parts of h, are rounded to steps of 2^-133 (bf16's
 * least).
 * Sizes: 0 <= N <= 64, 1 <= k <= E <= 1024, N * k <= 1024, 1 <= K, H, Fo <= 65536.
 * ws 16-byte aligned; calls that may overlap need one each.
 * ------------------------------------------------------------------------- */
int mp_expert_mlp_workspace(int64_t N, int64_t k, int64_t E, int64_t H, int64_t Fo, int out_dtype,
                            size_t* bytes);

int mp_expert_mlp(const void* x, int x_dtype, const uint8_t* x_scales, int64_t N, int64_t K,
                  int64_t ldx, const int32_t* idx, const float* weight, int64_t k, int64_t E,
                  int64_t H, int64_t Fo, const void* w1, const uint8_t* w1_scales, const void* w2,
                  const uint8_t* w2_scales, int act, int gated, const void* residual, int64_t ldr,
                  void* out, int out_dtype, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MP_LAYERS_H_ */
