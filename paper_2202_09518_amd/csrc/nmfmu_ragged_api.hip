// C ABI of the products over ragged ranges of rows: argument checks and plans.
// Public contract: include/nmfmu_ragged.h.
#include "nmfmu_ragged.h"
#include "nmfmu_internal.h"
#include "nmfmu_ragged_internal.h"

#include <algorithm>

using namespace nmfmu;
using namespace nmfmu::ragged;

namespace {

constexpr int64_t kMost = ((int64_t)1 << 31) - 1;
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 23) - 1;      // of up to 512: a launch has fewer than 2^32 threads
constexpr int kComputeUnits = 256;

int bytes_of(int32_t type) { return type == NMF_F32 ? 4 : 2; }
int stage_of(int32_t type) { return 128 / bytes_of(type); }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void *p, int to) { return ((uintptr_t)p & (to - 1)) == 0; }

struct Plan {
    int shape, splits;
};

// Parts of a contraction of k for `tiles` workgroups, so that there are about `workgroups`, each at least four stages long.
int splits_for(int64_t tiles, int64_t workgroups, int64_t k, int stage)
{
    const int64_t want = workgroups / std::max<int64_t>(tiles, 1), have = k / (4 * stage);
    const int64_t s = std::min<int64_t>(std::min(want, have), kMaxSplits);
    return s < 2 ? 1 : (int)s;
}

// ---- operands whose rows do not begin and end on 16 bytes ----------------------------------
// The tiles bring 16 bytes at a time straight to LDS; other operands pass registers, which takes 1.5 to 6 times as long
// (8192 x 4095 x 4097 bf16: 517 us, 641 with B by columns, its gradient 1430; aligned 243, 223, 211).  Where the product is
// long enough they are copied once per call into rows that do.
int64_t whole(int64_t cols, int e) { return (cols * e + 15) / 16 * 16 / e; }
size_t copy_bytes(int64_t lines, int64_t cols, int e) { return (size_t)lines * whole(cols, e) * e; }

// Copies of `bytes` are worth their time: launches and their bytes twice, against what the product loses without them, about as
// long as it takes at a middling rate.  2048 x 1023 x 2049 bf16: 31 us, without 42; 1237 rows of 515 x 389 in 9 groups f32,
// where they are not: 33 with, 25 without.
bool worth_copies(int e, size_t bytes, double flops)
{
    return 5e-6 + 2.0 * bytes / 4.5e12 < 1.2 * flops / (e == 4 ? 0.8e14 : 0.5e15);
}

// Scratch that they can take: of widths that do not fill 16 bytes, and of operands that `odd` says lie off their borders.
size_t copies_of(int32_t type, size_t bytes, double flops) { return bytes && worth_copies(bytes_of(type), bytes, flops) ? bytes : 0; }
bool ragged_rows(int64_t cols, int e) { return cols * e % 16 != 0; }
size_t product_copies(int32_t type, int64_t rows, int64_t count, int64_t m, int64_t n, int64_t ktotal, int odd)
{
    const int e = bytes_of(type);
    const bool bad_m = ragged_rows(m, e), bad_n = ragged_rows(n, e);
    size_t b = 0;
    if (bad_m || (odd & NMF_ODD_X)) b += copy_bytes(rows, m, e);
    if (bad_m || bad_n || (odd & NMF_ODD_B)) b += std::max(copy_bytes(count * m, n, e), copy_bytes(count * n, m, e));
    if (bad_m || (odd & NMF_ODD_FACTORS)) b += copy_bytes(ktotal, m, e);
    if (bad_n || (odd & NMF_ODD_FACTORS)) b += copy_bytes(ktotal, n, e);
    return copies_of(type, b, 2.0 * rows * m * n);
}
size_t gradient_copies(int32_t type, int64_t rows, int64_t m, int64_t n, int odd)
{
    const int e = bytes_of(type);
    size_t b = 0;
    if (ragged_rows(m, e) || (odd & NMF_ODD_X)) b += copy_bytes(rows, m, e);
    if (ragged_rows(n, e) || (odd & NMF_ODD_B)) b += copy_bytes(rows, n, e);
    return copies_of(type, b, 2.0 * rows * m * n);
}

// Time of `tiles` tiles of a shape: those of the busiest compute unit, by their size and by what share of the large tile's
// rate they reach.  us, bf16 unless said otherwise: 8192 x 4096 x 4096 takes 207 in tiles of 256 x 256; 2000 x 4096 x 2048
// 56 in 128 x 128 and 63 in 64 x 64; 2048 x 1024 x 2048 19.0 and 21.5; 1000 x 2048 x 1024, only 64 tiles of 128 x 128, 28.9
// and 14.6.  Float products hide a small tile's reads: 4096 x 4096 x 2048 with its gradients 1252 and 1439, 1999 rows of
// 720 x 1000 with theirs 119 and 85; 2048 x 4095 x 4097, 272 tiles of 256 x 256 and so twice the time of 256, 1002.
// Several groups of unequal lengths: the longest one's tiles take twice the others' at least.
double tile_time(int shape, bool floats, int64_t tiles, bool unequal)
{
    static const double rate[2][3] = {{1.0, 0.72, 0.5}, {0.93, 0.85, 0.74}};      // 256 x 256, 128 x 128, 64 x 64
    return (double)std::max<int64_t>(ceil_div(tiles, kComputeUnits), unequal ? 2 : 1) * kTileRows[shape] * kTileCols[shape] /
           rate[floats][std::min(shape, 2)];
}
template <class F> int fastest(bool floats, bool unequal, F tiles)
{
    int best = k256x256;
    for (int shape : {k128x128, k64x64})
        if (tile_time(shape, floats, tiles(shape), unequal) < tile_time(best, floats, tiles(best), unequal)) best = shape;
    return best;
}

// Time of a product in s parts, us: its stages, which take what their products do and the latency that a tile does not hide (more where
// rows pass registers), and the launch that joins the parts, by its workgroups and the parts' bytes written and read.  With adapters the
// join takes their factors too, and U's tiles run beside the parts, partly hidden; one part has two launches more, which form and pack U.
// Measured, one part and several: 8192 x 64 columns from 6000 rows f32 181 and 67 (8), from 16384 rows 188 and 169 (3); 64 groups, 8192 rows
// of 4096 x 64 f32 271 and 85 (4), bf16 22.0 and 27.6 (3); 8192 x 64 from 8192 rows bf16 39.7 and 33.5 (3); 1024 x 128 from 4096 rows bf16 8.6
// and 14.1 (3); 512 x 256 from 4096 rows f32 15.9 and 25.4 (3); 515 x 389 in 9 groups of 1237 rows f32 29.6 and 24.6 (4), bf16 13.5 and 14.6 (2).
// Adapters, ranks to 16 in long segments: 300 rows of 1024 x 512 bf16 21.2 and 12.9 (4), 2500 of 512 x 128 18.7 and 17.2 (2), 4096 of them 17.4 and
// 22.6 (2); f32 34.9 and 28.4 (4), 35.3 and 45.7 (4); ranks to 48, 2048 x 192 from 7000 rows f32 129 and 165 (2), from 3000 bf16 33.5 and 32.0 (2).
double parts_time(int shape, bool floats, int64_t tiles, int64_t stages, int s, int64_t rows, int64_t n, bool registers, int64_t segments, int kmax)
{
    const double product = floats ? 1.08e-4 : 1.3e-5;
    const double stage = tile_time(shape, floats, tiles * s, false) * product + (floats ? 0.1 : 0.2) + (registers ? 0.8 : 0.0);
    const double all = ceil_div(stages, s) * stage;
    if (s == 1) return all + (segments ? (floats ? 4.0 : 9.0) : 0.0);
    const double workgroups = (double)rows * ceil_div(n, 256);
    const double join = 3.0 + workgroups / 1100.0 + (double)s * rows * n * 8 / 4.5e6;
    if (!segments) return all + join;
    const double u_tiles = (double)(ceil_div(rows, kShrinkRows) + std::min(segments, rows)) * ceil_div(kmax, kShrinkCols);
    return all + join + 3e-5 * workgroups * kmax + 0.6 * u_tiles / kComputeUnits * stages * tile_time(k64x64, floats, 1, false) * product;
}

// Tile shape and parts of a product of `rows` rows in `groups` ranges.  Few rows take tiles of 64 or 32 rows, others the
// fastest; but up to 256 rows of a large matrix, which each row of tiles reads again, take the 128 x 128 rather than the
// 64 x 64 (160 x 8192 x 4096: 49 and 56 us).
// Parts (us): 500 x 4096 x 1000 (128 tiles of 64 x 64) 24.1 with one, 19.9 with two, 19.8 with four; 130 x 4096 x 1024
// (48) 25.8, 13.5 with four, 12.3 with eight; 1000 x 2048 x 1024 (256) 14.6 and 20.6 with two.  48 rows and their
// adapters (32 tiles) 17.7 with eight, 20.1 with four, 23.4 with sixteen.  None where the parts cost more than they save.
Plan product_plan(int32_t type, int64_t rows, int64_t groups, int64_t m, int64_t n, int64_t segments = 0, int kmax = 0)
{
    const int64_t count = groups;
    groups = std::max<int64_t>(1, std::min(groups, rows));
    const int64_t avg = ceil_div(rows, groups);
    auto tiles = [&](int shape) { return groups * ceil_div(avg, kTileRows[shape]) * ceil_div(n, kTileCols[shape]); };
    const bool floats = type == NMF_F32;
    Plan p;
    if (avg <= 32) p.shape = k32x128;
    else if (avg <= 64) p.shape = k64x128;
    else p.shape = fastest(floats, false, tiles);
    if (p.shape == k64x64 && avg <= 256 && groups * m * n * bytes_of(type) > (32 << 20)) p.shape = k128x128;
    const int64_t workgroups = p.shape != k64x64 ? kComputeUnits : (floats ? 800 : 400);
    const int stage = stage_of(type);
    p.splits = p.shape == k256x256 ? 1 : splits_for(tiles(p.shape), workgroups, m, stage);
    const bool registers = ragged_rows(m | n, bytes_of(type)) && product_copies(type, rows, count, m, n, 0, 0) == 0;
    auto time = [&](int s) { return parts_time(p.shape, floats, tiles(p.shape), ceil_div(m, stage), s, rows, n, registers, segments, kmax); };
    if (p.splits > 1 && time(1) <= time(p.splits)) p.splits = 1;
    return p;
}

// The same for a gradient, m x n for each group.  Parts of it cost their size again, written and read: only where there are few.
Plan gradient_plan(int32_t type, int64_t rows, int64_t groups, int64_t m, int64_t n)
{
    auto tiles = [&](int shape) { return groups * ceil_div(m, kTileRows[shape]) * ceil_div(n, kTileCols[shape]); };
    Plan p;
    p.shape = fastest(type == NMF_F32, groups > 1, tiles);
    p.splits = p.shape == k64x64 ? splits_for(tiles(p.shape), kComputeUnits, ceil_div(rows, groups) / 2, stage_of(type)) : 1;
    return p;
}

int shrink_plan(int32_t type, int64_t rows, int64_t segments, int64_t m, int kmax)
{
    const int64_t tiles = (ceil_div(rows, kShrinkRows) + std::min(segments, rows)) * ceil_div(kmax, kShrinkCols);
    return splits_for(tiles, rows > 4096 ? 2 * kComputeUnits : kComputeUnits, m, stage_of(type));
}

// A tile runs its segments' adapters one after the other, 2.5 us for each 32 factors; where segments are short, the launch that joins
// parts adds the adapters row by row, for the price of the product's floats written and read once (26 us for a tile of 256 x 256).
// The host knows the average alone: one segment of 16000 rows (448 us; 4096 x 4096 bf16, ranks to 64) beside 400 of one row (94) takes 2580.
bool joined_plan(int64_t rows, int64_t n, int64_t segments, int splits)
{
    return splits > 1 || (rows < 24 * segments && rows * ceil_div(n, 256) <= kMostWorkgroups);
}

// Blocks of rows to a workgroup, and chunks of so many: about four workgroups for each compute unit, at least four blocks each.
// A run of one chunk writes its gradients itself; runs with b > chunk blocks have b / chunk chunks, rounded up, which is at most
// b * 2 / (chunk + 1): so many parts there can be, however many runs there are.
struct FactorPlan {
    int chunk, chunks, slots;
};
FactorPlan factor_plan(int32_t type, int64_t rows, int64_t segments, int64_t runs, int64_t m, int64_t n, int kmax)
{
    const int64_t tiles = ceil_div(kmax, factor_tile(kmax)) * (ceil_div(m, 128) + ceil_div(n, 128));
    const int64_t blocks = ceil_div(rows, factor_rows(bytes_of(type), type == NMF_F16)) + std::min(segments, rows);
    const int64_t chunk = std::max<int64_t>(4, ceil_div(blocks, std::max<int64_t>(1, 4 * kComputeUnits / tiles)));
    if (blocks <= chunk) return FactorPlan{(int)chunk, (int)runs, 0};
    const int64_t chunks = ceil_div(blocks, chunk) + runs;
    return FactorPlan{(int)chunk, (int)chunks, (int)std::min(chunks, 2 * blocks / (chunk + 1))};
}

size_t product_part(int64_t rows, int64_t n, int splits) { return (size_t)splits * rows * up4(n) * 4; }
size_t shrink_part(int64_t rows, int kmax, int splits) { return splits > 1 ? (size_t)splits * up4(rows * kmax) * 4 : 0; }
size_t pack_part(int64_t rows, int kmax) { return (size_t)rows * (4 * ceil_div(kmax, 32) * 32) + (size_t)up4(rows) * 4; }
size_t gradient_part(int64_t groups, int64_t m, int64_t n, int splits) { return splits > 1 ? (size_t)splits * groups * m * up4(n) * 4 : 0; }
size_t factor_part(int kmax, int64_t m, int64_t n, int slots)
{
    return (size_t)slots * ceil_div(kmax, factor_tile(kmax)) * factor_tile(kmax) * (up4(m) + up4(n)) * 4;
}

size_t pieces_part(int32_t type, int64_t rows, int kmax)
{
    return type == NMF_F32 ? 0 : (size_t)rows * 2 * kFactorPieces * ceil_div(kmax, factor_tile(kmax)) * factor_tile(kmax) * 2;
}

// Splits that a scratch of `have` bytes can hold.
template <class F> int fit(int splits, size_t have, F bytes)
{
    while (splits > 1 && bytes(splits) > have) --splits;
    return splits;
}

struct Scratch {
    char *at;
    size_t left;
    void *take(size_t bytes)
    {
        bytes = (bytes + 15) / 16 * 16;
        if (bytes > left) return nullptr;
        void *p = at;
        at += bytes;
        left -= bytes;
        return p;
    }
};

struct Matrix {
    const void *p;
    int64_t ld, stride, rows, cols, count;
    bool bad(int e) const { return ((uintptr_t)p | (uint64_t)(ld * e) | (uint64_t)(count > 1 ? stride * e : 0) | (uint64_t)(cols * e)) & 15; }
    size_t bytes(int e) const { return copy_bytes(count * rows, cols, e); }
};

// Copies those of `n` matrices that need it, if that is worth it and fits; returns whether all are whole now.
int align_all(int32_t type, Matrix *const *all, int n, double flops, Scratch *s, hipStream_t st, bool *done)
{
    const int e = bytes_of(type);
    size_t bytes = 0;
    for (int i = 0; i < n; ++i)
        if (all[i]->bad(e)) bytes += all[i]->bytes(e);
    *done = false;
    if (!bytes || bytes > s->left || !worth_copies(e, bytes, flops)) return NMF_OK;
    for (int i = 0; i < n; ++i) {
        Matrix &m = *all[i];
        if (!m.bad(e)) continue;
        Align a = {m.p, m.ld, m.count > 1 ? m.stride : 0, m.rows, m.cols, m.count, s->take(m.bytes(e)), whole(m.cols, e)};
        const hipError_t rc = type == NMF_F32 ? launch_align<float>(a, st) : type == NMF_BF16 ? launch_align<bf16_t>(a, st) : launch_align<f16_t>(a, st);
        if (rc != hipSuccess) return set_error(NMF_EHIP, hipGetErrorString(rc));
        m.p = a.dst;
        m.ld = a.ldo;
        if (m.count > 1) m.stride = a.ldo * m.rows;
    }
    *done = true;
    return NMF_OK;
}
bool sizes_ok(int64_t rows, int64_t m, int64_t n) { return rows >= 0 && m > 0 && n > 0 && rows <= kMost && m <= kMost && n <= kMost; }

template <class P> int launched(int32_t type, const P &p, void *stream, hipError_t (*f)(const P &, hipStream_t),
                                hipError_t (*b)(const P &, hipStream_t), hipError_t (*h)(const P &, hipStream_t))
{
    const hipError_t e = (type == NMF_F32 ? f : type == NMF_BF16 ? b : h)(p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? NMF_OK : set_error(NMF_EHIP, hipGetErrorString(e));
}

int check_type(int32_t type) { return type >= NMF_F32 && type <= NMF_F16 ? NMF_OK : set_error(NMF_EINVAL, "unknown type"); }

int check_work(const void *work, size_t bytes)
{
    if (bytes && !work) return set_error(NMF_EINVAL, "work is null but work_bytes is not 0");
    if (!aligned(work, 16)) return set_error(NMF_EINVAL, "work must be 16-byte aligned");
    return NMF_OK;
}

int check_grid(int64_t workgroups)
{
    return workgroups <= kMostWorkgroups ? NMF_OK : set_error(NMF_EUNSUPPORTED, "more tiles than one launch can have");
}

int64_t product_grid(const Product &p)
{
    return (ceil_div(p.rows, kTileRows[p.shape]) + (p.offsets ? p.groups : 0)) * ceil_div(p.n, kTileCols[p.shape]) * p.splits;
}

}  // namespace

extern "C" {

int nmf_grouped_product(int32_t type, const void *X, int64_t ldx, const int64_t *offsets, int32_t groups, int64_t rows, const void *B,
                        int64_t ldb, int64_t stride_b, int32_t transposed, int64_t m, int64_t n, void *Y, int64_t ldy, void *work,
                        size_t work_bytes, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!sizes_ok(rows, m, n) || groups < 1) return set_error(NMF_EINVAL, "sizes must be positive and below 2^31");
    if ((rc = check_work(work, work_bytes))) return rc;
    if (!offsets || !B || (rows && (!X || !Y))) return set_error(NMF_EINVAL, "null pointer");
    const int e = bytes_of(type);
    if (!aligned(X, e) || !aligned(B, e) || !aligned(Y, e) || !aligned(offsets, 8)) return set_error(NMF_EINVAL, "misaligned pointer");
    if (ldx < m || ldy < n || ldb < (transposed ? m : n) || stride_b < 0) return set_error(NMF_EINVAL, "leading dimension below the row's length");
    if (rows == 0) return NMF_OK;
    const Plan plan = product_plan(type, rows, groups, m, n);
    Product p = {};
    p.x = X; p.ldx = ldx; p.offsets = offsets; p.groups = groups; p.rows = rows; p.m = m; p.n = n;
    p.b = B; p.ldb = ldb; p.stride_b = stride_b; p.transposed = transposed != 0; p.y = Y; p.ldy = ldy;
    p.shape = plan.shape;
    p.shrink_splits = 1;
    p.vec = aligned(Y, 16) && ldy * e % 16 == 0;
    Scratch scratch = {static_cast<char *>(work), work_bytes};
    p.splits = fit(plan.splits, work_bytes, [&](int s) { return product_part(rows, n, s); });
    if (p.splits > 1) p.part = static_cast<float *>(scratch.take(product_part(rows, n, p.splits)));
    p.joined = p.splits > 1;
    p.k_split = ceil_div(ceil_div(m, stage_of(type)), p.splits) * stage_of(type);
    if ((rc = check_grid(std::max(product_grid(p), p.joined ? rows * ceil_div(n, 256) : 0)))) return rc;
    Matrix x = {X, ldx, 0, rows, m, 1}, b = {B, ldb, stride_b, transposed ? n : m, transposed ? m : n, stride_b ? groups : 1};
    Matrix *const operands[] = {&x, &b};
    if ((rc = align_all(type, operands, 2, 2.0 * rows * m * n, &scratch, static_cast<hipStream_t>(stream), &p.padded))) return rc;
    p.x = x.p; p.ldx = x.ld;
    p.b = b.p; p.ldb = b.ld; p.stride_b = b.count > 1 ? b.stride : 0;
    return launched(type, p, stream, launch_product<float>, launch_product<bf16_t>, launch_product<f16_t>);
}

int nmf_grouped_gradient(int32_t type, const void *X, int64_t ldx, const void *dY, int64_t ldy, const int64_t *offsets, int32_t groups,
                         int64_t rows, int64_t m, int64_t n, void *G, int64_t ldg, int64_t stride_g, void *work, size_t work_bytes,
                         void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!sizes_ok(rows, m, n) || groups < 1) return set_error(NMF_EINVAL, "sizes must be positive and below 2^31");
    if ((rc = check_work(work, work_bytes))) return rc;
    if (!offsets || !G || (rows && (!X || !dY))) return set_error(NMF_EINVAL, "null pointer");
    const int e = bytes_of(type);
    if (!aligned(X, e) || !aligned(dY, e) || !aligned(G, e) || !aligned(offsets, 8)) return set_error(NMF_EINVAL, "misaligned pointer");
    if (ldx < m || ldy < n || ldg < n || (groups > 1 && stride_g < (m - 1) * ldg + n)) return set_error(NMF_EINVAL, "leading dimension below the row's length, or results that overlap");
    const Plan plan = gradient_plan(type, rows, groups, m, n);
    Gradient p = {};
    p.x = X; p.dy = dY; p.ldx = ldx; p.ldy = ldy; p.offsets = offsets; p.groups = groups; p.rows = rows; p.m = m; p.n = n;
    p.g = G; p.ldg = ldg; p.stride_g = stride_g;
    p.shape = plan.shape;
    p.splits = fit(plan.splits, work_bytes, [&](int s) { return gradient_part(groups, m, n, s); });
    p.part = static_cast<float *>(work);
    p.vec = aligned(G, 16) && ldg * e % 16 == 0 && stride_g * e % 16 == 0;
    if ((rc = check_grid((ceil_div(m, kTileRows[p.shape]) * ceil_div(n, kTileCols[p.shape]) * p.splits + 8) * groups))) return rc;
    if (rows) {
        Scratch scratch = {static_cast<char *>(work), work_bytes};
        if (p.splits > 1) scratch.take(gradient_part(groups, m, n, p.splits));
        Matrix x = {X, ldx, 0, rows, m, 1}, y = {dY, ldy, 0, rows, n, 1};
        Matrix *const operands[] = {&x, &y};
        if ((rc = align_all(type, operands, 2, 2.0 * rows * m * n, &scratch, static_cast<hipStream_t>(stream), &p.padded))) return rc;
        p.x = x.p; p.ldx = x.ld;
        p.dy = y.p; p.ldy = y.ld;
    }
    return launched(type, p, stream, launch_gradient<float>, launch_gradient<bf16_t>, launch_gradient<f16_t>);
}

int nmf_lowrank_product(int32_t type, const void *X, int64_t ldx, int64_t rows, const void *A, int64_t lda, int32_t transposed, int64_t m,
                        int64_t n, const int64_t *offsets, const int32_t *run, int32_t segments, const void *Wt, const void *H,
                        const int32_t *koff, int32_t runs, int32_t kmax, int64_t ktotal, const float *scale, float *U, void *Y, int64_t ldy,
                        void *work, size_t work_bytes, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!sizes_ok(rows, m, n) || segments < 0 || runs < 1 || kmax < 1 || ktotal < 1 || ktotal > kMost)
        return set_error(NMF_EINVAL, "sizes must be positive and below 2^31");
    if (kmax > NMF_LOWRANK_MAX_K) return set_error(NMF_EUNSUPPORTED, "kmax exceeds NMF_LOWRANK_MAX_K");
    if ((rc = check_work(work, work_bytes))) return rc;
    if (!A || (rows && (!X || !Y)) || (segments && (!offsets || !run || !Wt || !H || !koff || (rows && !U))))
        return set_error(NMF_EINVAL, "null pointer");
    const int e = bytes_of(type);
    if (!aligned(X, e) || !aligned(A, e) || !aligned(Y, e) || !aligned(Wt, e) || !aligned(H, e) || !aligned(offsets, 8) || !aligned(run, 4) ||
        !aligned(koff, 4) || !aligned(scale, 4) || !aligned(U, 4))
        return set_error(NMF_EINVAL, "misaligned pointer");
    if (ldx < m || ldy < n || lda < (transposed ? m : n)) return set_error(NMF_EINVAL, "leading dimension below the row's length");
    if (rows == 0) return NMF_OK;
    const Plan plan = product_plan(type, rows, 1, m, n, segments, kmax);
    Product p = {};
    p.x = X; p.ldx = ldx; p.groups = 1; p.rows = rows; p.m = m; p.n = n;
    p.b = A; p.ldb = lda; p.transposed = transposed != 0; p.y = Y; p.ldy = ldy;
    p.ad = Adapters{offsets, run, segments, koff, runs, kmax, ktotal, Wt, H, m, n, scale, U};
    p.shape = plan.shape;
    p.shrink_splits = 1;
    const int stage = stage_of(type);
    Scratch scratch = {static_cast<char *>(work), work_bytes};
    p.joined = joined_plan(rows, n, segments, plan.splits) && product_part(rows, n, 1) <= work_bytes;
    p.splits = p.joined ? fit(plan.splits, work_bytes, [&](int s) { return product_part(rows, n, s); }) : 1;
    if (p.joined && p.splits == 1 && !segments) p.joined = false;
    if (p.joined) {
        p.part = static_cast<float *>(scratch.take(product_part(rows, n, p.splits)));
    } else if (segments && pack_part(rows, kmax) <= work_bytes) {
        p.pack = scratch.take(pack_part(rows, kmax));
        p.row_scale = reinterpret_cast<float *>(static_cast<char *>(p.pack) + pack_part(rows, kmax)) - up4(rows);
    }
    p.k_split = ceil_div(ceil_div(m, stage), p.splits) * stage;
    if (segments) {
        // parts of u are added up by the launch that joins y or that packs u
        if (p.joined || p.pack)
            p.shrink_splits = fit(shrink_plan(type, rows, segments, m, kmax), scratch.left, [&](int s) { return shrink_part(rows, kmax, s); });
        p.shrink_k = ceil_div(ceil_div(m, stage), p.shrink_splits) * stage;
        if (p.shrink_splits > 1) p.upart = static_cast<float *>(scratch.take(shrink_part(rows, kmax, p.shrink_splits)));
    }
    p.vec = aligned(Y, 16) && ldy * e % 16 == 0;
    const int64_t shrink = segments ? (ceil_div(rows, kShrinkRows) + segments) * ceil_div(kmax, kShrinkCols) * p.shrink_splits : 0;
    if ((rc = check_grid(std::max(product_grid(p) + shrink, p.joined ? rows * ceil_div(n, 256) : ceil_div(rows, 16))))) return rc;
    Matrix x = {X, ldx, 0, rows, m, 1}, b = {A, lda, 0, transposed ? n : m, transposed ? m : n, 1};
    Matrix w = {Wt, m, 0, ktotal, m, 1}, h = {H, n, 0, ktotal, n, 1};
    Matrix *const operands[] = {&x, &b, &w, &h};
    if ((rc = align_all(type, operands, segments ? 4 : 2, 2.0 * rows * m * n, &scratch, static_cast<hipStream_t>(stream), &p.padded))) return rc;
    p.x = x.p; p.ldx = x.ld;
    p.b = b.p; p.ldb = b.ld;
    p.ad.down = w.p; p.ad.ld_down = w.ld;
    p.ad.up = h.p; p.ad.ld_up = h.ld;
    return launched(type, p, stream, launch_product<float>, launch_product<bf16_t>, launch_product<f16_t>);
}

int nmf_lowrank_gradient(int32_t type, const void *X, int64_t ldx, const void *dY, int64_t ldy, int64_t rows, int64_t m, int64_t n,
                         const int64_t *offsets, const int32_t *run, int32_t segments, const int32_t *koff, int32_t runs, int32_t kmax,
                         int64_t ktotal, const float *U, const float *V, void *dWt, void *dH, void *work, size_t work_bytes, void *stream)
{
    int rc = check_type(type);
    if (rc) return rc;
    if (!sizes_ok(rows, m, n) || segments < 0 || runs < 1 || kmax < 1 || ktotal < 1 || ktotal > kMost)
        return set_error(NMF_EINVAL, "sizes must be positive and below 2^31");
    if (kmax > NMF_LOWRANK_MAX_K) return set_error(NMF_EUNSUPPORTED, "kmax exceeds NMF_LOWRANK_MAX_K");
    if ((rc = check_work(work, work_bytes))) return rc;
    if (!koff || !dWt || !dH || (segments && (!offsets || !run)) || (segments && rows && (!X || !dY || !U || !V)))
        return set_error(NMF_EINVAL, "null pointer");
    const int e = bytes_of(type);
    if (!aligned(X, e) || !aligned(dY, e) || !aligned(dWt, e) || !aligned(dH, e) || !aligned(offsets, 8) || !aligned(run, 4) ||
        !aligned(koff, 4) || !aligned(U, 4) || !aligned(V, 4))
        return set_error(NMF_EINVAL, "misaligned pointer");
    if (ldx < m || ldy < n) return set_error(NMF_EINVAL, "leading dimension below the row's length");
    if (rows == 0) segments = 0;
    FactorGradient p = {};
    p.x = X; p.dy = dY; p.ldx = ldx; p.ldy = ldy; p.rows = rows; p.m = m; p.n = n;
    p.ad = Adapters{offsets, run, segments, koff, runs, kmax, ktotal, nullptr, nullptr, 0, 0, nullptr, nullptr};
    p.u = U; p.v = V; p.ddown = dWt; p.dup = dH;
    const FactorPlan plan = factor_plan(type, rows, segments, runs, m, n, kmax);
    p.chunk = plan.chunk;
    p.chunks = plan.chunks;
    p.slots = plan.slots;
    Scratch scratch = {static_cast<char *>(work), work_bytes};
    if (p.slots && !(p.part = static_cast<float *>(scratch.take(factor_part(kmax, m, n, p.slots))))) {      // each run in one chunk
        p.chunk = 1 << 30;
        p.chunks = runs;
        p.slots = 0;
    }
    if (type != NMF_F32 && segments) p.pieces = scratch.take(pieces_part(type, rows, kmax));
    if (p.chunks > 65535 || ceil_div(up4(m) + up4(n), 1024) > 65535 || (rc = check_grid(std::max((int64_t)runs * kmax, ceil_div(rows, 16)))))
        return set_error(NMF_EUNSUPPORTED, "more runs or columns than one launch can have");
    return launched(type, p, stream, launch_factor_gradient<float>, launch_factor_gradient<bf16_t>, launch_factor_gradient<f16_t>);
}

size_t nmf_ragged_work_bytes(int kind, int32_t type, int64_t rows, int64_t m, int64_t n, int32_t parts, int32_t runs, int32_t kmax,
                             int64_t ktotal)
{
    const int odd = kind & (NMF_ODD_X | NMF_ODD_B | NMF_ODD_FACTORS | NMF_ONE_B);
    if (type < NMF_F32 || type > NMF_F16 || !sizes_ok(rows, m, n) || rows == 0) return 0;
    switch (kind - odd) {
    case 0: {
        if (parts < 1) return 0;
        const int splits = product_plan(type, rows, parts, m, n).splits;
        return (splits > 1 ? product_part(rows, n, splits) : 0) + product_copies(type, rows, odd & NMF_ONE_B ? 1 : parts, m, n, 0, odd);
    }
    case 1:
        return parts < 1 ? 0 : gradient_part(parts, m, n, gradient_plan(type, rows, parts, m, n).splits) + gradient_copies(type, rows, m, n, odd);
    case 2: {
        if (parts < 0 || kmax < 1 || kmax > NMF_LOWRANK_MAX_K || ktotal < 0 || ktotal > kMost) return 0;
        const int splits = product_plan(type, rows, 1, m, n, parts, kmax).splits;
        const size_t copies = product_copies(type, rows, 1, m, n, ktotal, odd);
        if (parts == 0) return (splits > 1 ? product_part(rows, n, splits) : 0) + copies;
        return (joined_plan(rows, n, parts, splits) ? product_part(rows, n, splits) : pack_part(rows, kmax)) +
               shrink_part(rows, kmax, shrink_plan(type, rows, parts, m, kmax)) + copies;
    }
    case 3:
        if (parts < 1 || runs < 1 || kmax < 1 || kmax > NMF_LOWRANK_MAX_K || ktotal < 1 || ktotal > kMost) return 0;
        return factor_part(kmax, m, n, factor_plan(type, rows, parts, runs, m, n, kmax).slots) + pieces_part(type, rows, kmax);
    }
    return 0;
}

}  // extern "C"
