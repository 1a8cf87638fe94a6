// C ABI of the norm, routing, the rows' way to their groups and products in 8 bits: argument checks and plans.
// Public contract: include/nmfmu_routed.h.
#include "nmfmu_routed.h"
#include "nmfmu_test.h"
#include "nmfmu_internal.h"
#include "nmfmu_routed_internal.h"

#include <algorithm>

using namespace nmfmu;
using namespace nmfmu::routed;
using namespace nmfmu::ragged;

namespace {

constexpr int64_t kMost = ((int64_t)1 << 31) - 1;
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 23) - 1;
constexpr int kComputeUnits = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int bytes_of(int32_t type) { return type == NMF_F32 ? 4 : 2; }
bool aligned(const void *p, int to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool size_ok(int64_t n) { return n > 0 && n <= kMost; }
bool rows_ok(int64_t n) { return n >= 0 && n <= kMost; }

int check_type(int32_t type) { return type >= NMF_F32 && type <= NMF_F16 ? NMF_OK : set_error(NMF_EINVAL, "unknown type"); }
int check_work(const void *work, size_t bytes)
{
    if (bytes && !work) return set_error(NMF_EINVAL, "work is null but work_bytes is not 0");
    if (!aligned(work, 16)) return set_error(NMF_EINVAL, "work must be 16-byte aligned");
    return NMF_OK;
}
int bad(const char *what) { return set_error(NMF_EINVAL, what); }

const char *const kSizes = "sizes must be positive and below 2^31", *const kNull = "null pointer", *const kMisaligned = "misaligned pointer",
                  *const kShort = "leading dimension below the row's length";

int launched(hipError_t e) { return e == hipSuccess ? NMF_OK : set_error(NMF_EHIP, hipGetErrorString(e)); }
template <class P>
int launched(int32_t type, const P &p, void *stream, hipError_t (*f)(const P &, hipStream_t), hipError_t (*b)(const P &, hipStream_t),
             hipError_t (*h)(const P &, hipStream_t))
{
    return launched((type == NMF_F32 ? f : type == NMF_BF16 ? b : h)(p, static_cast<hipStream_t>(stream)));
}

// ---- plans ---------------------------------------------------------------------------------

// Rows that one workgroup takes at once are its alone rather than two or three launches': 24 rows of 64 groups 7.2 us and 11.2, but 40 of
// 512, three turns of it, 18.3 and 13.1.
bool route_alone(int64_t rows, int64_t groups) { return rows <= route_each(1, (int)groups); }

size_t route_bytes(int64_t blocks, int64_t groups)
{
    const int64_t each = ceil_div(blocks * groups, 4) * 4;
    return (size_t)(each * 8 + groups * 16);
}

size_t norm_bytes(int64_t parts, int64_t m) { return parts > 1 ? (size_t)(parts * m * 4) : 0; }

struct Plan {
    int shape, splits;
};

// Time of `tiles` tiles of a shape: those of the busiest compute unit, by their size and by what share of the large tile's rate
// they reach.  us, bf16 results: 8192 x 4096 x 4096 takes 131 in tiles of 256 x 256, 190 in 128 x 128, 230 in 64 x 128, 270 to 300 in
// 64 x 64; 1024 x 4096 x 4096 49, 32.1, 31.9, 39.3; 2000 x 2048 x 2048 28, 19.0, 18.7, 23.2; 4096 rows in 8 groups, 4096 x 2048, 52, 68, 75, 77.
// (Float results and codes that pass registers go by the same shares, which were not measured for them.)
double tile_time(int shape, int64_t tiles)
{
    const double rate = shape == k256x256 ? 1.0 : shape == k128x128 ? 0.7 : shape == k64x128 ? 0.5 : 0.45;
    return (double)ceil_div(tiles, kComputeUnits) * kTileRows[shape] * kTileCols[shape] / rate;
}

// Tile shape and parts of the contraction.  Groups end inside a tile, half a tile each on average.  large: the 256 x 256 tile can be had.
Plan product_plan(int64_t rows, int64_t groups, int64_t m, int64_t n, bool large)
{
    groups = std::max<int64_t>(1, std::min(groups, rows));
    const int64_t avg = ceil_div(rows, groups);
    auto tiles = [&](int shape) {
        const int64_t up = groups > 1 ? ceil_div(rows, kTileRows[shape]) + groups / 2 : ceil_div(rows, kTileRows[shape]);
        return up * ceil_div(n, kTileCols[shape]);
    };
    Plan p;
    if (avg <= 32) p.shape = k32x128;
    else if (avg <= 64) p.shape = k64x128;
    else {
        p.shape = large ? k256x256 : k128x128;
        for (int shape : {k128x128, k64x128, k64x64})
            if (tile_time(shape, tiles(shape)) < tile_time(p.shape, tiles(p.shape))) p.shape = shape;
    }
    const int64_t want = kComputeUnits / std::max<int64_t>(tiles(p.shape), 1), have = m / (4 * 128);
    const int64_t s = p.shape == k256x256 ? 1 : std::min<int64_t>(std::min(want, have), kMaxSplits);
    p.splits = s < 2 ? 1 : (int)s;
    return p;
}
size_t product_part(int64_t rows, int64_t n, int splits) { return splits > 1 ? (size_t)splits * rows * up4(n) * 4 : 0; }

// Codes whose rows do not begin and end on 16-byte borders pass registers on their way to LDS, which takes 2 to 3.5 times as long;
// where the product is long enough they are copied once per call into rows that do, if the scratch has room.
// (us, bf16 results: 6000 x 4095 x 2047 in 4 groups 239, transposed 141, through registers, 94 and 89 with copies; 2245 rows in 22 groups of
// 6197 x 5568 425 and 217, 8192 in 64 of 4095 x 4096 605 and 305, where only the rows are copied.  Float results take longer either way and
// go by the same rate.)
constexpr int64_t kFar = kFarRows;      // straight to LDS, distances inside a tile go into 32 bits: 256 rows below this, copied ones too
int64_t whole(int64_t cols) { return ceil_div(cols, 16) * 16; }
struct Codes {
    const void *p;
    int64_t ld, stride, rows, cols, count;
    bool bad() const { return !aligned(p, 16) || (ld | (count > 1 ? stride : 0) | cols) % 16 != 0 || ld >= kFar; }
    size_t bytes() const { return (size_t)count * rows * whole(cols); }
};
bool worth_copies(size_t bytes, double flops) { return 5e-6 + 2.0 * bytes / 4.5e12 < flops / 0.9e15; }

// Bytes of the copies of a product, of the operands that need them, with scratch enough; 0 if it makes none.
size_t copies_of(int64_t rows, int64_t m, int64_t n, int64_t count, bool transposed, bool odd_x, bool odd_b)
{
    const int64_t wide_x = whole(m), wide_b = whole(transposed ? m : n);
    if ((odd_x && wide_x >= kFar) || (odd_b && wide_b >= kFar)) return 0;
    const __int128 bytes = (odd_x ? (__int128)rows * wide_x : 0) + (odd_b ? (__int128)count * (transposed ? n : m) * wide_b : 0);
    return bytes < ((__int128)1 << 62) && worth_copies((size_t)bytes, 2.0 * rows * m * n) ? (size_t)bytes : 0;
}

// What a product does: its tiles, whether its codes go straight to LDS, and the bytes of copies that it makes for that.
struct Route8 {
    Plan tiles;
    bool straight;
    size_t copies;
};
Route8 route_of(int32_t type, const Codes &x, const Codes &b, int64_t ldxs, int64_t groups, bool transposed, int64_t m, int64_t n, size_t work_bytes)
{
    const bool near = ldxs < (1 << 20);
    Route8 r;
    r.copies = near ? copies_of(x.rows, m, n, b.count, transposed, x.bad(), b.bad()) : 0;
    if (r.copies > work_bytes) r.copies = 0;
    r.straight = near && ((!x.bad() && !b.bad()) || r.copies);
    r.tiles = product_plan(x.rows, groups, m, n, r.straight && type != NMF_F32);
    while (r.tiles.splits > 1 && product_part(x.rows, n, r.tiles.splits) > work_bytes - r.copies) --r.tiles.splits;
    return r;
}

// A matrix of entries of e bytes: rows x cols, ld from row to row.
int check_matrix(const void *p, int64_t ld, int64_t rows, int64_t cols, int e)
{
    if (rows && !p) return bad(kNull);
    if (!aligned(p, e)) return bad(kMisaligned);
    if (ld < cols) return bad(kShort);
    return NMF_OK;
}

}  // namespace

extern "C" {

int nmf_rms_norm(int32_t type, const void *X, int64_t ldx, const void *R, int64_t ldr, const void *weight, int64_t rows, int64_t m,
                 float eps, void *H, int64_t ldh, void *Y, int64_t ldy, void *Y8, int64_t ldy8, float *scale, int64_t lds,
                 float *rstd, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !size_ok(m)) return bad(kSizes);
    if (m > NMF_NORM_MAX_M) return set_error(NMF_EUNSUPPORTED, "more columns than NMF_NORM_MAX_M");
    if (!(eps >= 0.f)) return bad("eps must not be negative");
    const int e = bytes_of(type);
    if ((rc = check_matrix(X, ldx, rows, m, e))) return rc;
    if (R && (rc = check_matrix(R, ldr, rows, m, e))) return rc;
    if (H && (rc = check_matrix(H, ldh, rows, m, e))) return rc;
    if (Y && (rc = check_matrix(Y, ldy, rows, m, e))) return rc;
    if ((Y8 == nullptr) != (scale == nullptr)) return bad("Y8 and scale: both or neither");
    if (Y8 && ((rc = check_matrix(Y8, ldy8, rows, m, 1)) || (rc = check_matrix(scale, lds, rows, blocks_of(m), 4)))) return rc;
    if (rows && !Y && !Y8) return bad("neither Y nor Y8");
    if (!aligned(weight, e) || !aligned(rstd, 4)) return bad(kMisaligned);
    if ((H && H == X && ldh != ldx) || (H && H == R && ldh != ldr)) return bad("H in the place of an operand must have its leading dimension");
    if (rows == 0) return NMF_OK;
    Norm a = {};
    a.x = X; a.r = R; a.w = weight; a.ldx = ldx; a.ldr = ldr; a.rows = rows; a.m = m; a.eps = eps;
    a.h = H; a.y = Y; a.y8 = Y8; a.ldh = ldh; a.ldy = ldy; a.ldy8 = ldy8; a.lds = lds; a.scale = scale; a.rstd = rstd;
    return launched(type, a, stream, launch_norm<float>, launch_norm<bf16_t>, launch_norm<f16_t>);
}

int nmf_rms_norm_gradient(int32_t type, const void *H, int64_t ldh, const float *rstd, const void *weight, const void *dY,
                          int64_t ldy, const void *dH, int64_t lddh, int64_t rows, int64_t m, void *dX, int64_t ldx, void *dweight,
                          void *work, size_t work_bytes, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !size_ok(m)) return bad(kSizes);
    if (m > NMF_NORM_MAX_M) return set_error(NMF_EUNSUPPORTED, "more columns than NMF_NORM_MAX_M");
    if ((rc = check_work(work, work_bytes))) return rc;
    const int e = bytes_of(type);
    if ((rc = check_matrix(H, ldh, rows, m, e)) || (rc = check_matrix(dY, ldy, rows, m, e)) || (rc = check_matrix(dX, ldx, rows, m, e))) return rc;
    if (dH && (rc = check_matrix(dH, lddh, rows, m, e))) return rc;
    if (rows && !rstd) return bad(kNull);
    if (!aligned(weight, e) || !aligned(dweight, e) || !aligned(rstd, 4)) return bad(kMisaligned);
    if ((dX && dX == dH && ldx != lddh) || (dX && dX == dY && ldx != ldy)) return bad("dX in the place of an operand must have its leading dimension");
    if (rows == 0 && !dweight) return NMF_OK;
    NormGradient a = {};
    a.h = H; a.w = weight; a.dy = dY; a.dh = dH; a.rstd = rstd; a.ldh = ldh; a.ldy = ldy; a.lddh = lddh; a.ldx = ldx; a.rows = rows; a.m = m;
    a.dx = dX; a.dw = dweight;
    a.parts = norm_parts(rows, m);
    if (norm_bytes(a.parts, m) > work_bytes) a.parts = (int)std::max<int64_t>(1, (int64_t)(work_bytes / ((size_t)m * 4)));
    a.part = a.parts > 1 ? static_cast<float *>(work) : nullptr;
    return launched(type, a, stream, launch_norm_gradient<float>, launch_norm_gradient<bf16_t>, launch_norm_gradient<f16_t>);
}

int nmf_round_blocks(int32_t type, const void *X, int64_t ldx, int64_t stride, int32_t count, int64_t rows, int64_t m, int32_t block,
                     void *X8, int64_t ldx8, int64_t stride8, float *scale, int64_t lds, int64_t stride_s, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !size_ok(m) || count < 1) return bad(kSizes);
    if (block != 1 && block != 128) return bad("block must be 1 or 128");
    const int64_t lines = ceil_div(rows, block), M = blocks_of(m);
    if ((rc = check_matrix(X, ldx, rows, m, bytes_of(type))) || (rc = check_matrix(X8, ldx8, rows, m, 1)) || (rc = check_matrix(scale, lds, lines, M, 4)))
        return rc;
    if (rows == 0) return NMF_OK;
    if (count > 1 && (stride < 0 || stride8 < (rows - 1) * ldx8 + m || stride_s < (lines - 1) * lds + M)) return bad("results that overlap");
    if ((__int128)count * rows * M > ((__int128)1 << 62)) return set_error(NMF_EUNSUPPORTED, "too many blocks");
    Round a = {};
    a.x = X; a.ldx = ldx; a.stride = stride; a.rows = rows; a.m = m; a.count = count; a.block = block;
    a.x8 = X8; a.ldx8 = ldx8; a.stride8 = stride8; a.scale = scale; a.lds = lds; a.stride_s = stride_s;
    return launched(type, a, stream, launch_round<float>, launch_round<bf16_t>, launch_round<f16_t>);
}

int nmf_grouped_product8(int32_t type, const void *X8, int64_t ldx, const float *xscale, int64_t ldxs, const int64_t *offsets,
                         int32_t groups, int64_t rows, const void *B8, int64_t ldb, int64_t stride_b, const float *bscale, int64_t ldbs,
                         int64_t stride_bs, int32_t transposed, int64_t m, int64_t n, void *Y, int64_t ldy, void *work, size_t work_bytes,
                         void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !size_ok(m) || !size_ok(n) || groups < 1) return bad(kSizes);
    if ((rc = check_work(work, work_bytes))) return rc;
    const int e = bytes_of(type);
    const int64_t b_rows = transposed ? n : m, b_cols = transposed ? m : n;
    if ((rc = check_matrix(X8, ldx, rows, m, 1)) || (rc = check_matrix(xscale, ldxs, rows, blocks_of(m), 4)) ||
        (rc = check_matrix(B8, ldb, b_rows, b_cols, 1)) || (rc = check_matrix(bscale, ldbs, blocks_of(b_rows), blocks_of(b_cols), 4)) ||
        (rc = check_matrix(Y, ldy, rows, n, e)))
        return rc;
    if (!offsets) return bad(kNull);
    if (!aligned(offsets, 8)) return bad(kMisaligned);
    if (stride_b < 0 || stride_bs < 0) return bad("negative stride");
    if (rows == 0) return NMF_OK;
    Codes x = {X8, ldx, 0, rows, m, 1}, b = {B8, ldb, stride_b, b_rows, b_cols, stride_b ? groups : 1};
    const Route8 route = route_of(type, x, b, ldxs, groups, transposed != 0, m, n, work_bytes);
    const Plan plan = route.tiles;
    char *scratch = static_cast<char *>(work);
    const int64_t grid = (ceil_div(rows, kTileRows[plan.shape]) + groups) * ceil_div(n, kTileCols[plan.shape]) * plan.splits;
    if (std::max(grid, plan.splits > 1 ? rows * ceil_div(n, 1024) : 0) > kMostWorkgroups) return set_error(NMF_EUNSUPPORTED, "more tiles than one launch can have");
    if (route.copies)
        for (Codes *c : {&x, &b}) {
            if (!c->bad()) continue;
            if ((rc = launched(launch_whole_rows(c->p, c->ld, c->stride, c->rows, c->cols, c->count, scratch, whole(c->cols), static_cast<hipStream_t>(stream))))) return rc;
            c->p = scratch;
            c->ld = whole(c->cols);
            c->stride = c->count > 1 ? c->ld * c->rows : 0;
            scratch += c->bytes();
        }
    Product8 p = {};
    p.x = x.p; p.ldx = x.ld; p.xs = xscale; p.ldxs = ldxs; p.offsets = offsets; p.groups = groups; p.rows = rows; p.m = m; p.n = n;
    p.b = b.p; p.ldb = b.ld; p.stride_b = b.stride; p.bs = bscale; p.ldbs = ldbs; p.stride_bs = stride_bs; p.transposed = transposed != 0;
    p.type = type; p.y = Y; p.ldy = ldy;
    p.dma = route.straight;
    p.shape = plan.shape;
    p.splits = plan.splits;
    p.part = reinterpret_cast<float *>(scratch);
    p.k_split = ceil_div(blocks_of(m), p.splits);
    p.vec = aligned(Y, 16) && ldy * e % 16 == 0;
    return launched(launch_product8(p, static_cast<hipStream_t>(stream)));
}

int nmf_route(int32_t type, const void *logits, int64_t ldl, int64_t rows, int32_t groups, int32_t k, int32_t normalise,
              int32_t *choice, float *gate, int64_t *offsets, int32_t *place, float *balance, void *work, size_t work_bytes,
              void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || groups < 1 || k < 1 || k > groups || rows * k > kMost) return bad("sizes must be positive and below 2^31, and k at most groups");
    if (groups > NMF_ROUTE_MAX_GROUPS || k > NMF_ROUTE_MAX_K) return set_error(NMF_EUNSUPPORTED, "more groups or choices than the limits");
    if ((rc = check_work(work, work_bytes))) return rc;
    if ((rc = check_matrix(logits, ldl, rows, groups, bytes_of(type)))) return rc;
    if (!offsets || !balance || (rows && (!choice || !gate || !place))) return bad(kNull);
    if (!aligned(choice, 4) || !aligned(gate, 4) || !aligned(place, 4) || !aligned(balance, 4) || !aligned(offsets, 8)) return bad(kMisaligned);
    Route a = {};
    a.logits = logits; a.ldl = ldl; a.rows = rows; a.groups = groups; a.k = k; a.normalise = normalise != 0;
    a.choice = choice; a.gate = gate; a.offsets = offsets; a.place = place; a.balance = balance;
    a.each = route_each(rows, groups);
    a.blocks = ceil_div(rows, a.each);
    if (a.blocks > kMostWorkgroups) return set_error(NMF_EUNSUPPORTED, "more rows than one launch can have");
    if (!route_alone(rows, groups) && route_bytes(a.blocks, groups) <= work_bytes) {
        const int64_t each = ceil_div(a.blocks * groups, 4) * 4;
        a.total = static_cast<int64_t *>(work);
        a.mass = reinterpret_cast<double *>(a.total + groups);
        a.count = reinterpret_cast<int32_t *>(a.mass + groups);
        a.share = reinterpret_cast<float *>(a.count + each);
    }
    return launched(type, a, stream, launch_route<float>, launch_route<bf16_t>, launch_route<f16_t>);
}

int nmf_route_gradient(int32_t type, const void *logits, int64_t ldl, int64_t rows, int32_t groups, int32_t k, int32_t normalise,
                       const int32_t *choice, const int64_t *offsets, const float *dgate, const float *dbalance, void *dlogits,
                       int64_t lddl, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || groups < 1 || k < 1 || k > groups || rows * k > kMost) return bad("sizes must be positive and below 2^31, and k at most groups");
    if (groups > NMF_ROUTE_MAX_GROUPS || k > NMF_ROUTE_MAX_K) return set_error(NMF_EUNSUPPORTED, "more groups or choices than the limits");
    const int e = bytes_of(type);
    if ((rc = check_matrix(logits, ldl, rows, groups, e)) || (rc = check_matrix(dlogits, lddl, rows, groups, e))) return rc;
    if (!offsets || (rows && !choice)) return bad(kNull);
    if (!aligned(choice, 4) || !aligned(dgate, 4) || !aligned(dbalance, 4) || !aligned(offsets, 8)) return bad(kMisaligned);
    if (rows == 0) return NMF_OK;
    RouteGradient a = {};
    a.logits = logits; a.ldl = ldl; a.rows = rows; a.lddl = lddl; a.groups = groups; a.k = k; a.normalise = normalise != 0;
    a.choice = choice; a.offsets = offsets; a.dgate = dgate; a.dbalance = dbalance; a.dlogits = dlogits;
    return launched(type, a, stream, launch_route_gradient<float>, launch_route_gradient<bf16_t>, launch_route_gradient<f16_t>);
}

int nmf_spread_rows(int32_t type, const void *X, int64_t ldx, int64_t rows, int32_t k, const int32_t *place, int64_t m, void *Y, int64_t ldy,
                    int64_t sorted, const float *xscale, int64_t ldxs, float *yscale, int64_t ldys, void *stream)
{
    int rc = type == NMF_E4M3 ? NMF_OK : check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !rows_ok(sorted) || !size_ok(m) || k < 1 || rows * k > kMost) return bad(kSizes);
    const int e = type == NMF_E4M3 ? 1 : bytes_of(type);
    if ((rc = check_matrix(X, ldx, rows, m, e)) || (rc = check_matrix(Y, ldy, sorted, m, e))) return rc;
    if (rows && !place) return bad(kNull);
    if (!aligned(place, 4)) return bad(kMisaligned);
    if (type == NMF_E4M3) {
        if ((rc = check_matrix(xscale, ldxs, rows, blocks_of(m), 4)) || (rc = check_matrix(yscale, ldys, sorted, blocks_of(m), 4))) return rc;
    } else if (xscale || yscale) {
        return bad("scales are those of codes");
    }
    if (rows == 0 || sorted == 0) return NMF_OK;
    Spread a = {};
    a.x = X; a.ldx = ldx * e; a.rows = rows; a.m = m * e; a.ldy = ldy * e; a.sorted = sorted; a.k = k; a.place = place; a.y = Y;
    if (type == NMF_E4M3) { a.xs = xscale; a.ldxs = ldxs; a.ys = yscale; a.ldys = ldys; a.ms = blocks_of(m); }
    return launched(launch_spread(a, static_cast<hipStream_t>(stream)));
}

int nmf_collect_rows(int32_t type, const void *X, int64_t ldx, int64_t sorted, int64_t rows, int32_t k, const int32_t *place,
                     const float *gate, int64_t m, void *Y, int64_t ldy, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !rows_ok(sorted) || !size_ok(m) || k < 1 || rows * k > kMost) return bad(kSizes);
    const int e = bytes_of(type);
    if ((rc = check_matrix(X, ldx, sorted, m, e)) || (rc = check_matrix(Y, ldy, rows, m, e))) return rc;
    if (rows && !place) return bad(kNull);
    if (!aligned(place, 4) || !aligned(gate, 4)) return bad(kMisaligned);
    if (rows == 0) return NMF_OK;
    Collect a = {};
    a.x = X; a.ldx = ldx; a.sorted = sorted; a.rows = rows; a.m = m; a.ldy = ldy; a.k = k; a.place = place; a.gate = gate; a.y = Y;
    return launched(type, a, stream, launch_collect<float>, launch_collect<bf16_t>, launch_collect<f16_t>);
}

int nmf_collect_gradient(int32_t type, const void *dY, int64_t ldy, int64_t rows, int32_t k, const int32_t *place, const float *gate,
                         int64_t m, void *dX, int64_t lddx, int64_t sorted, const void *X, int64_t ldx, float *dgate, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!rows_ok(rows) || !rows_ok(sorted) || !size_ok(m) || k < 1 || rows * k > kMost) return bad(kSizes);
    const int e = bytes_of(type);
    if ((rc = check_matrix(dY, ldy, rows, m, e)) || (rc = check_matrix(dX, lddx, sorted, m, e))) return rc;
    if (dgate && (rc = check_matrix(X, ldx, sorted, m, e))) return rc;
    if (!dgate && X) return bad("X and dgate: both or neither");
    if (rows && !place) return bad(kNull);
    if (!aligned(place, 4) || !aligned(gate, 4) || !aligned(dgate, 4)) return bad(kMisaligned);
    if (rows == 0) return NMF_OK;
    CollectGradient a = {};
    a.dy = dY; a.x = X; a.ldy = ldy; a.rows = rows; a.m = m; a.lddx = lddx; a.sorted = sorted; a.ldx = ldx; a.k = k; a.place = place;
    a.gate = gate; a.dx = dX; a.dgate = dgate;
    return launched(type, a, stream, launch_collect_gradient<float>, launch_collect_gradient<bf16_t>, launch_collect_gradient<f16_t>);
}

int nmfmu_product8_route(int32_t type, const void *X8, int64_t ldx, int64_t ldxs, int32_t groups, int64_t rows, const void *B8, int64_t ldb,
                         int64_t stride_b, int32_t transposed, int64_t m, int64_t n, size_t work_bytes, int64_t *route)
{
    const Codes x = {X8, ldx, 0, rows, m, 1}, b = {B8, ldb, stride_b, transposed ? n : m, transposed ? m : n, stride_b ? groups : 1};
    const Route8 r = route_of(type, x, b, ldxs, groups, transposed != 0, m, n, work_bytes);
    route[0] = r.straight;
    route[1] = (int64_t)r.copies;
    route[2] = r.copies && x.bad() ? whole(x.cols) : ldx;
    route[3] = r.copies && b.bad() ? whole(b.cols) : ldb;
    route[4] = kTileRows[r.tiles.shape];
    route[5] = kTileCols[r.tiles.shape];
    route[6] = r.tiles.splits > 1 ? (int64_t)product_part(rows, n, r.tiles.splits) : 0;
    return NMF_OK;
}

int nmfmu_column_reads(int64_t m, int64_t n, int64_t ld, int64_t c0, int32_t columns, int64_t k1, int64_t *reads)
{
    const int64_t bytes = column_bytes(m, n, ld, c0);
    const int count = (int)std::min<int64_t>(n - c0, columns);
    reads[0] = reads[1] = 0;
    for (int64_t k0 = 0; k0 < k1; k0 += 128) {
        if (!whole_stage(ld, k0, k1, count, bytes)) continue;
        ++reads[0];
        for (int k = 0; k < 128; ++k)
            for (int chunk = 0; chunk * 16 < count; ++chunk) reads[1] = std::max(reads[1], k0 * ld + column_chunk(k, chunk, ld) + 16);
    }
    return NMF_OK;
}

size_t nmf_routed_work_bytes(int kind, int64_t rows, int64_t m, int64_t n, int32_t parts)
{
    const int odd = kind & (NMF_ODD_X | NMF_ODD_B | NMF_ONE_B | NMF_B_M_X_N | NMF_B_N_X_M);
    kind &= ~odd;
    if (!size_ok(rows) || !size_ok(m)) return 0;
    if (kind == 0) return m <= NMF_ROUTE_MAX_GROUPS && !route_alone(rows, m) ? route_bytes(ceil_div(rows, route_each(rows, (int)m)), m) : 0;
    if (kind == 1) return m <= NMF_NORM_MAX_M ? norm_bytes(norm_parts(rows, m), m) : 0;
    if (kind != 2 || !size_ok(n) || parts < 1) return 0;
    const int64_t count = odd & NMF_ONE_B ? 1 : parts;
    size_t most = 0;
    for (bool transposed : {false, true}) {
        if ((odd & (NMF_B_M_X_N | NMF_B_N_X_M)) && !(odd & (transposed ? NMF_B_N_X_M : NMF_B_M_X_N))) continue;
        const bool odd_x = m % 16 || (odd & NMF_ODD_X), odd_b = (transposed ? m : n) % 16 || (odd & NMF_ODD_B);
        const size_t copies = copies_of(rows, m, n, count, transposed, odd_x, odd_b);
        size_t joined = product_part(rows, n, product_plan(rows, parts, m, n, false).splits);
        if (copies || !(odd_x || odd_b)) joined = std::max(joined, product_part(rows, n, product_plan(rows, parts, m, n, true).splits));
        most = std::max(most, copies + joined);
    }
    return most;
}

}  // extern "C"
