/*
 * nmfmu_routed.h -- the way of rows to the products over ragged ranges (nmfmu_ragged.h) and back: the norm in front of
 * them, which rows go to which group, and products in 8 bits.
 *
 *     norm              H = X + R,  Y = H w / sqrt(mean H^2 + eps), also in 8 bits;  its gradients
 *     routing           a row's k groups by its logits, gates, the groups' offsets, places among the sorted rows, and
 *                       how unequal the groups are (balance);  its gradient
 *     rows              to their places, back as a gated sum, and the gradients of that
 *     8 bits            blocks of entries rounded to codes with a scale;  grouped product of such rows and matrices
 *
 * Conventions, where they differ from nmfmu_ragged.h or add to it
 *   - `type`: NMF_F32, NMF_BF16 or NMF_F16 for all matrices of a call that are not said to be something else.  Sums, norms,
 *     softmaxes, gates and scales are floats; results are rounded once when they are written.
 *   - Codes are e4m3 (one sign, four exponent, three fraction bits; largest 448, no infinities), one byte each.  A block of
 *     codes stands for code * scale.  Rows have a scale for each 128 columns: float, rows x ceil(m / 128).  Matrices have one
 *     for each 128 x 128: ceil(m / 128) x ceil(n / 128) for an m x n matrix, in the layout that the matrix has.
 *     scale = max(largest magnitude / 448, 2^-126), rounded to a float, and codes are the nearest ones to entry * 448 / largest magnitude
 *     (to entry * 2^126 under the smallest scale), the even one of two: not to entry / scale, which differs by the scale's rounding.  A
 *     block with an entry that is not finite has the scale NaN and codes 0.
 *   - place: device, int32[rows x k]: where choice j of row r lies among the sorted rows, at [r k + j]; places are distinct.
 *     A place outside [0, sorted rows) stands for no choice (nmf_route writes -1).  Sorted rows that no place names are not
 *     written.
 *   - Malformed offsets, places and choices give meaningless results but no access out of range.
 *   - Rows stand alone, but in `balance` and in the gradient of the norm's weight, which are sums over all rows: what is in one row
 *     reaches no other one's results.  (The order in which nmf_grouped_product8 sums, and so a row's last bits, goes by the sizes of the
 *     call and by where the row lies.)
 *   - Results may not overlap operands, except where said.  Streams, capture, work and limits as in nmfmu_ragged.h; the scratch
 *     of a call is nmf_routed_work_bytes(...) bytes, with less it takes a slower plan (nmf_route one workgroup for all rows, which is
 *     for few of them).  Results are the same bits in every call
 *     with the same scratch.
 */
#ifndef NMFMU_ROUTED_H
#define NMFMU_ROUTED_H

#include "nmfmu_ragged.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { NMF_E4M3 = 3 };            /* type of nmf_spread_rows alone: codes and their scales */

#define NMF_NORM_MAX_M 32768      /* most columns of the norm */
#define NMF_ROUTE_MAX_GROUPS 1024
#define NMF_ROUTE_MAX_K 16        /* most choices of a row */

/*
 * H = X + R (rounded to `type`), s = 1 / sqrt(mean over columns of H^2 + eps), Y = H s w.  Without R (null): H = X.  (Squares are
 * added up in floats: s is 0 where they pass 2^128, and loses bits where they lie below 2^-126 and eps does too; with eps 0 it is
 * infinite for a row of zeros.)
 *   H       rows x m, or null; it may be X or R itself (the same pointer and leading dimension)
 *   weight  m entries, or null for 1
 *   Y       rows x m, or null;  Y8, scale: the floats that Y is rounded from, in codes, or both null;  one of them
 *           at least.  A code whose quotient is within 2^-22 of itself of the middle between two may be the farther one.
 *   rstd    float[rows]: s, or null
 */
int nmf_rms_norm(int32_t type, const void *X, int64_t ldx, const void *R, int64_t ldr, const void *weight, int64_t rows, int64_t m,
                 float eps, void *H, int64_t ldh, void *Y, int64_t ldy, void *Y8, int64_t ldy8, float *scale, int64_t lds,
                 float *rstd, void *stream);

/*
 * With z = dY w and h = H s:  dX = s (z - h mean(z h)) + dH, the gradient of X and of R;  dweight = sum over rows of dY h.
 *   H, rstd  as nmf_rms_norm left them (X if it had no R)
 *   dH       rows x m: the gradient that reaches H on other ways, or null;  dX may be dH or dY itself
 *   weight   m entries, or null for 1;  dweight: m entries, or null
 */
int nmf_rms_norm_gradient(int32_t type, const void *H, int64_t ldh, const float *rstd, const void *weight, const void *dY,
                          int64_t ldy, const void *dH, int64_t lddh, int64_t rows, int64_t m, void *dX, int64_t ldx, void *dweight,
                          void *work, size_t work_bytes, void *stream);

/*
 * `count` matrices of rows x m (matrix i at X + i * stride) to codes and scales, blocks of `block` (1 or 128) x 128.
 *   X8     matrix i at X8 + i * stride8;  scale: at scale + i * stride_s, ceil(rows / block) x ceil(m / 128), lds from row to row
 */
int nmf_round_blocks(int32_t type, const void *X, int64_t ldx, int64_t stride, int32_t count, int64_t rows, int64_t m, int32_t block,
                     void *X8, int64_t ldx8, int64_t stride8, float *scale, int64_t lds, int64_t stride_s, void *stream);

/*
 * Y_g = X_g B_g for the rows of each group g, X and B in codes: the sum over blocks of 128 of the contraction of the blocks'
 * scales times the product of their codes.
 *   X8, xscale  rows x m and its scales, ldxs from row to row
 *   B8, bscale  group g at B8 + g * stride_b and bscale + g * stride_bs: m x n, or n x m if `transposed`; stride 0: one for all
 *   Y           rows x n of `type`;  rows outside all groups are not written
 * The gradient dX_g = dY_g B_g^T of rounded dY is the same call with B in its other form; that of B is nmf_grouped_gradient of the
 * rows before they were rounded.  Rows of codes that begin and end on 16-byte borders are fastest (others are copied, or slower).
 * Results in float32 keep all bits of the products of codes.  Those in 16 bits leave out, of eight neighbouring products, what is below
 * 2^-13 of the largest one: 1.4e-5 of the results' root mean square, which is more than the last place of f16 where a result cancels to a
 * few hundredths of that.  The scales of two blocks are multiplied first, as floats: their product should be a normal one.
 */
int nmf_grouped_product8(int32_t type, const void *X8, int64_t ldx, const float *xscale, int64_t ldxs, const int64_t *offsets,
                         int32_t groups, int64_t rows, const void *B8, int64_t ldb, int64_t stride_b, const float *bscale, int64_t ldbs,
                         int64_t stride_bs, int32_t transposed, int64_t m, int64_t n, void *Y, int64_t ldy, void *work, size_t work_bytes,
                         void *stream);

/*
 * The groups of the k largest logits of each row, in falling order, the lower group first of equals.  Logits of -infinity and
 * NaN are never chosen.  p is the softmax of a row's logits (NaN where they hold a NaN or +infinity).
 *   logits   rows x groups;  k <= groups
 *   choice   int32[rows x k], gate float[rows x k]: p of the choice, divided by the sum over the row's choices if `normalise`;
 *            -1 and 0 behind a row's last choice
 *   offsets  int64[groups + 1]: where each group's rows begin among the sorted rows; offsets[groups] = C of all choices
 *   place    int32[rows x k]: a group's rows are in the order of their rows
 *   balance  float[1]: groups * sum over g of (count_g / C) (sum over rows of c_r p_rg / C), c_r the choices of row r: 1 where
 *            all groups are equal.  Rows without a choice take no part; 0 if no row has one.
 */
int nmf_route(int32_t type, const void *logits, int64_t ldl, int64_t rows, int32_t groups, int32_t k, int32_t normalise,
              int32_t *choice, float *gate, int64_t *offsets, int32_t *place, float *balance, void *work, size_t work_bytes,
              void *stream);

/*
 * Gradient of the logits from those of the gates and of balance (the counts are taken as constants).
 *   choice, offsets  as nmf_route left them
 *   dgate            float[rows x k], or null;  dbalance: float[1], or null.  dgate behind a row's last choice is not used.
 *   dlogits          rows x groups: zeros for a row without a choice
 */
int nmf_route_gradient(int32_t type, const void *logits, int64_t ldl, int64_t rows, int32_t groups, int32_t k, int32_t normalise,
                       const int32_t *choice, const int64_t *offsets, const float *dgate, const float *dbalance, void *dlogits,
                       int64_t lddl, void *stream);

/*
 * Y[place[r k + j]] = X[r]: each row to its places among `sorted` rows.  NMF_E4M3: X and Y hold codes, and xscale (rows x
 * ceil(m / 128)) goes to yscale the same way; else both are null.
 */
int nmf_spread_rows(int32_t type, const void *X, int64_t ldx, int64_t rows, int32_t k, const int32_t *place, int64_t m, void *Y, int64_t ldy,
                    int64_t sorted, const float *xscale, int64_t ldxs, float *yscale, int64_t ldys, void *stream);

/*
 * Y[r] = sum over j of gate[r k + j] X[place[r k + j]], in the order of j; gate null: 1 (then it is the gradient of
 * nmf_spread_rows).  X has `sorted` rows.  Gates of no choice are not used.
 */
int nmf_collect_rows(int32_t type, const void *X, int64_t ldx, int64_t sorted, int64_t rows, int32_t k, const int32_t *place,
                     const float *gate, int64_t m, void *Y, int64_t ldy, void *stream);

/*
 * Gradients of nmf_collect_rows:  dX[place[r k + j]] = gate[r k + j] dY[r];  dgate[r k + j] = <dY[r], X[place[r k + j]]>, 0 for no choice.
 *   X, dgate  both or neither (null)
 */
int nmf_collect_gradient(int32_t type, const void *dY, int64_t ldy, int64_t rows, int32_t k, const int32_t *place, const float *gate,
                         int64_t m, void *dX, int64_t lddx, int64_t sorted, const void *X, int64_t ldx, float *dgate, void *stream);

/*
 * Scratch of the fastest plan, in bytes (0: none needed, or invalid sizes).  kind: 0 nmf_route (m: groups), 1
 * nmf_rms_norm_gradient with dweight, 2 nmf_grouped_product8 (parts: groups; kind 2 alone takes n and parts, and, added to
 * it as in nmf_ragged_work_bytes, NMF_ODD_X and NMF_ODD_B, also for leading dimensions of 2^22 and more, NMF_ONE_B, and how B lies:
 * NMF_B_M_X_N, or NMF_B_N_X_M for `transposed`; with neither there is enough for both).
 */
enum { NMF_B_M_X_N = 256, NMF_B_N_X_M = 512 };
size_t nmf_routed_work_bytes(int kind, int64_t rows, int64_t m, int64_t n, int32_t parts);

#ifdef __cplusplus
}
#endif
#endif /* NMFMU_ROUTED_H */
