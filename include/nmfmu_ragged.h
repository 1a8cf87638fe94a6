/*
 * nmfmu_ragged.h -- products over ragged ranges of rows: matrices of many groups, and the factor pairs of
 * many runs at work beside one matrix.
 *
 * A run of nmfmu.h leaves a pair W (m x k), H (k x n); an ensemble leaves many, of different ranks.  These
 * entry points use such pairs, and full matrices, on rows that belong to different ones of them, and give
 * the gradients that refine them:
 *
 *     grouped product      Y_g  = X_g B_g                        rows of group g, its own matrix
 *                          dX_g = dY_g B_g^T                     (the same call, B in its other form)
 *     grouped gradient     dB_g = X_g^T dY_g
 *     low-rank product     Y    = X A + s_r (X W_r) H_r          r: the run of the row's segment, or none
 *                          dX   = dY A^T + s_r (dY H_r^T) W_r^T  (the same call, W and H exchanged)
 *     low-rank gradient    dW_r = X^T V,  dH_r = U^T dY          U = s_r X W_r and V = s_r dY H_r^T as saved
 *
 * Conventions, where they differ from nmfmu.h or add to it
 *   - `type` says what X, Y, A, B, W, H and their gradients hold: NMF_F32, NMF_BF16 or NMF_F16.  Products
 *     are summed in fp32 and rounded once when they are written; U and V are floats.  Floats meet the fp32
 *     matrix instruction; halves and bf16 are exact operands of theirs; where U meets them in the product it goes as two
 *     pieces (bf16: 16 bits of it and more; f16: 22 bits of what is above 2^-17 of the row's largest entry, and no entry is
 *     off by more than 2^-39 of the largest), in the gradients U and V go as three (all 24 bits).
 *   - Matrices are row-major; `ld...` is the distance of two rows in entries, at least the row's length.
 *     Base pointers are aligned to an entry.  Operands whose rows do not begin and end on 16-byte borders are
 *     copied into rows that do, once per call and in its scratch, where the product is long enough, or take
 *     slower kernels.
 *   - offsets: device, int64[groups + 1] (segments + 1), non-decreasing; range g is rows offsets[g] to
 *     offsets[g + 1] - 1, which may be none.  It is read by the kernels, not by the host.  Values are held
 *     inside [0, rows] where they are used: malformed offsets, runs or koff give a meaningless result but no
 *     access out of range.
 *   - Rows stand alone: what is not finite in one row, group or run reaches no other one's results.
 *   - Results may not overlap operands.  All calls are asynchronous on `stream`, allocate nothing, and
 *     share nothing: they may be made on several streams at once and captured into graphs.  All memory lies
 *     on the current device, which is the stream's.
 *   - work: device scratch of the call alone, 16-byte aligned, nmf_ragged_work_bytes(...) bytes for the
 *     plan that is fastest; with less (also NULL, 0) the call uses a plan that fits (nmf_lowrank_product with
 *     long segments then adds their adapters by plain sums, much slower).  It must stay valid until the work
 *     is done.  nmf_lowrank_product asks for the result in floats, 4 rows n bytes, for each part that its
 *     contraction is cut into, and one of them where segments have fewer than 24 rows on average, whose
 *     adapters are added to it; else for 4 rows kmax bytes, kmax in whole 32s.
 *   - Sizes below 2^31; more tiles, rows or runs than one launch has room for (2^23 workgroups, 65535 runs in
 *     nmf_lowrank_gradient) give NMF_EUNSUPPORTED.  rows == 0 is a successful no-op (gradients are then zeros).
 */
#ifndef NMFMU_RAGGED_H
#define NMFMU_RAGGED_H

#include "nmfmu.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { NMF_F32 = 0, NMF_BF16 = 1, NMF_F16 = 2 };

#define NMF_LOWRANK_MAX_K 256     /* largest rank of a run in the low-rank entry points */

/*
 * Y_g = X_g B_g for the rows of each group g.
 *   X  rows x m;  Y  rows x n;  rows outside all groups are not written
 *   B  group g at B + g * stride_b entries: m x n, or n x m if `transposed` (Y_g = X_g B_g^T); stride_b 0:
 *      one matrix for all
 */
int nmf_grouped_product(int32_t type, const void *X, int64_t ldx, const int64_t *offsets, int32_t groups,
                        int64_t rows, const void *B, int64_t ldb, int64_t stride_b, int32_t transposed,
                        int64_t m, int64_t n, void *Y, int64_t ldy, void *work, size_t work_bytes, void *stream);

/*
 * G_g = X_g^T dY_g (m x n at G + g * stride_g) for each group g; zeros for a group without rows.
 *   X  rows x m;  dY  rows x n.  The gradient of a `transposed` B is the call with X and dY exchanged.
 */
int nmf_grouped_gradient(int32_t type, const void *X, int64_t ldx, const void *dY, int64_t ldy,
                         const int64_t *offsets, int32_t groups, int64_t rows, int64_t m, int64_t n,
                         void *G, int64_t ldg, int64_t stride_g, void *work, size_t work_bytes, void *stream);

/*
 * Y = X A + s_r (X W_r) H_r, r = run[s] for the rows of segment s.
 *   A       m x n, or n x m if `transposed` (X A^T in its place)
 *   offsets, run   device, int64[segments + 1] and int32[segments]; rows of no segment, and of a segment
 *           whose run is outside [0, runs), get X A alone
 *   Wt, H   device, ktotal x m and ktotal x n, contiguous: the transposed W_r one below the other, and the
 *           H_r; run r is rows koff[r] to koff[r + 1] - 1 (koff: device, int32[runs + 1]) of both, at most
 *           kmax of them
 *   scale   device, float[runs], or NULL for 1
 *   U       device, float[rows x kmax], written: s_r X W_r in the first k_r columns of the rows that have a
 *           run; what else it holds is unspecified
 */
int nmf_lowrank_product(int32_t type, const void *X, int64_t ldx, int64_t rows, const void *A, int64_t lda,
                        int32_t transposed, int64_t m, int64_t n, const int64_t *offsets, const int32_t *run,
                        int32_t segments, const void *Wt, const void *H, const int32_t *koff, int32_t runs,
                        int32_t kmax, int64_t ktotal, const float *scale, float *U, void *Y, int64_t ldy,
                        void *work, size_t work_bytes, void *stream);

/*
 * Gradients of the factors of all runs, each summed over the rows of its segments in their order.
 *   X, dY   rows x m and rows x n
 *   U       s_r X W_r, as nmf_lowrank_product leaves it;  V  s_r dY H_r^T, as its call for dX leaves it
 *   dWt, dH ktotal x m and ktotal x n: zeros for a run without rows
 */
int nmf_lowrank_gradient(int32_t type, const void *X, int64_t ldx, const void *dY, int64_t ldy, int64_t rows,
                         int64_t m, int64_t n, const int64_t *offsets, const int32_t *run, int32_t segments,
                         const int32_t *koff, int32_t runs, int32_t kmax, int64_t ktotal, const float *U,
                         const float *V, void *dWt, void *dH, void *work, size_t work_bytes, void *stream);

/*
 * Scratch of the fastest plan, in bytes (0: none needed, or invalid sizes).  kind: 0 grouped product,
 * 1 grouped gradient, 2 low-rank product, 3 low-rank gradient; parts: groups or segments; runs, kmax,
 * ktotal: kinds 2 and 3 only.
 * To kinds 0 to 2 is added which operands lie off 16-byte borders, by their base pointer, leading dimension
 * or stride (their widths are seen from the sizes), so that there is room for copies of them:
 * NMF_ODD_X, NMF_ODD_B (B or A; dY for kind 1) and NMF_ODD_FACTORS (Wt or H); and to kind 0 NMF_ONE_B where
 * one matrix serves all groups (stride_b 0), of which there is one copy then.
 */
enum { NMF_ODD_X = 16, NMF_ODD_B = 32, NMF_ODD_FACTORS = 64, NMF_ONE_B = 128 };
size_t nmf_ragged_work_bytes(int kind, int32_t type, int64_t rows, int64_t m, int64_t n, int32_t parts,
                             int32_t runs, int32_t kmax, int64_t ktotal);

#ifdef __cplusplus
}
#endif
#endif /* NMFMU_RAGGED_H */
