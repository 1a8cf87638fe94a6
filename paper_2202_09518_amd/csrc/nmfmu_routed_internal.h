// Launchers of the norm, of routing, of the rows' way to their groups and back, and of products in 8 bits.
// Not part of the public ABI (that is include/nmfmu_routed.h).
#pragma once

#include "nmfmu_ragged_internal.h"
#include "nmfmu_routed.h"

namespace nmfmu {
namespace routed {

using ragged::bf16_t;
using ragged::f16_t;

constexpr int64_t blocks_of(int64_t n) { return (n + 127) / 128; }      // of 128

struct Norm {
    const void *x, *r, *w;      // r, w: or null
    int64_t ldx, ldr, rows, m;
    float eps;
    void *h, *y, *y8;           // or null
    int64_t ldh, ldy, ldy8, lds;
    float *scale, *rstd;
};
template <class T> hipError_t launch_norm(const Norm &a, hipStream_t st);

struct NormGradient {
    const void *h, *w, *dy, *dh;      // w, dh: or null
    const float *rstd;
    int64_t ldh, ldy, lddh, ldx, rows, m;
    void *dx, *dw;                    // dw: or null
    int parts;                        // workgroups, each with the sums of its rows in part
    float *part;                      // parts x m; null where parts is 1
};
template <class T> hipError_t launch_norm_gradient(const NormGradient &a, hipStream_t st);
int norm_parts(int64_t rows, int64_t m);      // workgroups of the fastest plan

struct Round {
    const void *x;
    int64_t ldx, stride, rows, m;
    int count, block;
    void *x8;
    int64_t ldx8, stride8;
    float *scale;
    int64_t lds, stride_s;
};
template <class T> hipError_t launch_round(const Round &a, hipStream_t st);

struct Spread {
    const void *x;
    int64_t ldx, rows, m, ldy, sorted;      // ldx, ldy and m in bytes
    int k;
    const int32_t *place;
    void *y;
    const float *xs;                        // scales of rows of codes, or null
    int64_t ldxs, ldys, ms;
    float *ys;
};
hipError_t launch_spread(const Spread &a, hipStream_t st);

struct Collect {
    const void *x;
    int64_t ldx, sorted, rows, m, ldy;
    int k;
    const int32_t *place;
    const float *gate;                      // or null
    void *y;
};
template <class T> hipError_t launch_collect(const Collect &a, hipStream_t st);

struct CollectGradient {
    const void *dy, *x;                     // x, dgate: both or neither
    int64_t ldy, rows, m, lddx, sorted, ldx;
    int k;
    const int32_t *place;
    const float *gate;
    void *dx;
    float *dgate;
};
template <class T> hipError_t launch_collect_gradient(const CollectGradient &a, hipStream_t st);

struct Route {
    const void *logits;
    int64_t ldl, rows;
    int groups, k, normalise;
    int32_t *choice;
    float *gate;
    int64_t *offsets;
    int32_t *place;
    float *balance;
    // plan: null for one workgroup
    int each;                               // rows of a block, at most kRouteRows
    int64_t blocks;
    int32_t *count;                         // blocks x groups: choices of each group in a block, then those in the blocks before
    float *share;                           // blocks x groups: sums of c_r p_rg
    int64_t *total;                         // groups
    double *mass;                           // groups
};
constexpr int kRouteRows = 64;
int route_each(int64_t rows, int groups);      // rows of a block
template <class T> hipError_t launch_route(const Route &a, hipStream_t st);

struct RouteGradient {
    const void *logits;
    int64_t ldl, rows, lddl;
    int groups, k, normalise;
    const int32_t *choice;
    const int64_t *offsets;
    const float *dgate, *dbalance;          // or null
    void *dlogits;
};
template <class T> hipError_t launch_route_gradient(const RouteGradient &a, hipStream_t st);

// Operands by columns, rows of ld codes from column c0 of m x n on: bytes from their first code to the array's end; whether a stage of 128 k
// from k0 on, up to k1, is loaded in chunks as they lie, of `count` columns of a tile; and where such a chunk begins.
constexpr int64_t kFarRows = 1 << 22;      // distances inside a stage go into 32 bits below this
constexpr int64_t column_bytes(int64_t m, int64_t n, int64_t ld, int64_t c0) { return (m - 1) * ld + n - c0; }
constexpr bool whole_stage(int64_t ld, int64_t k0, int64_t k1, int count, int64_t bytes)
{
    return ld < kFarRows && k1 - k0 >= 128 && (k0 + 127) * ld + (count + 15) / 16 * 16 <= bytes;
}
constexpr unsigned column_chunk(int k, int chunk, int64_t ld) { return (unsigned)k * (unsigned)ld + chunk * 16; }

struct Product8 {
    const void *x;
    int64_t ldx;
    const float *xs;
    int64_t ldxs;
    const int64_t *offsets;
    int32_t groups;
    int64_t rows, m, n;
    const void *b;
    int64_t ldb, stride_b;
    const float *bs;
    int64_t ldbs, stride_bs;
    int32_t transposed, type;
    void *y;
    int64_t ldy;
    // plan
    bool dma;                               // operands whose rows begin and end on 16-byte borders
    int shape, splits;                      // shapes as for the products of other types (256 x 256: with dma, not for float results)
    int64_t k_split;                        // of the contraction, whole blocks
    float *part;                            // splits x rows x (n rounded up to 4), where there are several
    bool vec;                               // rows of y begin on 16-byte borders
};
// `count` matrices of codes with rows of ldo, a multiple of 16, zero behind their ends.
hipError_t launch_whole_rows(const void *src, int64_t ld, int64_t stride, int64_t rows, int64_t cols, int64_t count, void *dst, int64_t ldo, hipStream_t st);
hipError_t launch_product8(const Product8 &p, hipStream_t st);

}  // namespace routed
}  // namespace nmfmu
