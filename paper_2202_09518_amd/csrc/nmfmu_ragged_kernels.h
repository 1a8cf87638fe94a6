// Kernels and launches of the products over ragged ranges of rows, for one type T; included by one source per type.
#pragma once

#include "nmfmu_ragged_internal.h"
#include "nmfmu_ragged_device.h"

#include <type_traits>

namespace nmfmu {
namespace ragged {

// ---- float factors on the halves' matrix cores -------------------------------------
// x = hi + lo + last, N = 3 bf16, is all 24 bits of a float (each piece takes 8 of them; below 2^-110 the last ones are lost),
// N = 2 all 11 bits of a half.  What is left of x once its piece is taken; nothing of what is not finite.
__device__ __forceinline__ float after_piece(float x)
{
    const float piece = Type<bf16_t>::load(Type<bf16_t>::round(x));
    return __builtin_isfinite(piece) ? x - piece : 0.f;
}
template <int N> __device__ __forceinline__ void cut_chunk(float (&x)[8], u32x4 (&pieces)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) pieces[n][i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = after_piece(x[i]);
    }
}
__device__ __forceinline__ void floats_of(u32x4 v, float (&x)[8])      // of halves
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Type<f16_t>::load(f16_t{(unsigned short)(v[i >> 1] >> (16 * (i & 1)))});
}

template <class T> struct Cut {                      // the type that float factors are multiplied in
    using E = bf16_t;
    static constexpr int kPieces = kFactorPieces;           // of a float operand
};
template <> struct Cut<float> {
    using E = float;
    static constexpr int kPieces = 1;
};
template <class T> constexpr bool two_piece_matrix() { return false; }
template <> constexpr bool two_piece_matrix<f16_t>() { return true; }      // its 11 bits are two bf16
template <class T> constexpr int block_rows() { return factor_rows(sizeof(T), two_piece_matrix<T>()); }

// Entries [k, k + N) of a row of `width` floats, zero from kend on.
template <int N> __device__ __forceinline__ void floats_at(const float *row, int k, int kend, int width, float (&x)[N])
{
    if (k + N <= width) {
        __builtin_memcpy(x, row + k, sizeof(x));
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = k + i < kend ? x[i] : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = k + i < kend ? row[k + i] : 0.f;
    }
}

// The product of the first pieces d with that of the others, which is left out where d is not finite: a second piece of an
// infinity, or of what meets one, would turn it into a NaN.
template <bool BOTH> __device__ __forceinline__ float both_pieces(float d, float low)
{
    return BOTH && __builtin_isfinite(d) ? d + low : d;
}

struct Run {
    int ko, k;        // its rows of the factors
};
__device__ __forceinline__ Run run_of(const Adapters &a, int segment)
{
    Run r = {0, 0};
    const int id = a.run[segment];
    if (id < 0 || id >= a.runs) return r;
    const int64_t lo = a.koff[id], hi = a.koff[id + 1];
    if (lo < 0 || hi <= lo || lo >= a.ktotal) return r;
    int64_t k = (hi < a.ktotal ? hi : a.ktotal) - lo;
    if (k > a.kmax) k = a.kmax;
    r.ko = (int)lo;
    r.k = (int)k;
    return r;
}

template <class T> __device__ __forceinline__ Operand operand(const void *base, int64_t entry, int64_t ld, int64_t count, int64_t last)
{
    constexpr int E = sizeof(T);
    return Operand{(const char *)base + entry * E, ld * E, count, last * E};
}

// ---- adapters in a tile's accumulators --------------------------------------------
// u as an operand of the matrix instructions: rows of `planes` x kp entries, kp = kmax in whole 32s, zero behind a run's
// rank and in rows without a run.  Floats: as they are.  Halves and bf16: u = hi + lo in two planes; the products with hi and
// with lo both run over H's rows.  bf16: 16 bits of u and more, 2^-8 of what an output's last place shows.  A half has too
// small a range for u, so f16 rows are scaled by a power of two that brings their largest entry to [2^14, 2^15), the top of the
// range: halves end at 2^-24, so lo is off by up to 2^-25 there, and an entry keeps 22 bits down to 2^-17 of the largest and 16
// down to 2^-23, as where W's columns and H's rows are scaled against each other; sums of 256 products stay below 2^39.
// row_scale undoes it.
// One row per 16 lanes; adds up the parts of u on the way.
template <class T> __global__ __launch_bounds__(256) void pack_kernel(Product a)
{
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int l = threadIdx.x & 15, kp = (a.ad.kmax + 31) / 32 * 32;
    if (row >= a.rows) return;
    Run run = {0, 0};
    const int s = range_at(a.ad.offsets, a.ad.segments, row);
    if (s < a.ad.segments && a.ad.offsets[s] <= row) run = run_of(a.ad, s);
    constexpr int N = kMaxRank / 16;
    float u[N];
    float most = 0.f;
#pragma unroll
    for (int t = 0; t < N; ++t) {
        const int k = 16 * t + l;
        u[t] = 0.f;
        if (k < run.k) {
            if (a.shrink_splits == 1) {
                u[t] = a.ad.u[row * a.ad.kmax + k];
            } else {
                for (int p = 0; p < a.shrink_splits; ++p) u[t] += a.upart[(p * a.rows + row) * a.ad.kmax + k];
                a.ad.u[row * a.ad.kmax + k] = u[t];
            }
        }
        most = __builtin_fmaxf(most, __builtin_fabsf(u[t]));
    }
    float up = 1.f;
    if constexpr (sizeof(T) == 2 && !std::is_same<T, bf16_t>::value) {
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d));
        const int e = half_exponent(__float_as_uint(most)) - 14;      // -126 to 114
        up = power_of_two(-e);
        if (l == 0) a.row_scale[row] = power_of_two(e);
    }
    T *out = (T *)a.pack + row * ((int64_t)kp * (4 / (int)sizeof(T)));
#pragma unroll
    for (int t = 0; t < N; ++t) {
        const int k = 16 * t + l;
        if (k >= kp) break;
        const float x = u[t] * up;
        const T hi = Type<T>::round(x);
        out[k] = hi;
        if constexpr (sizeof(T) == 2) out[kp + k] = Type<T>::round(__builtin_isfinite(Type<T>::load(hi)) ? x - Type<T>::load(hi) : 0.f);
    }
}

template <class T> __device__ __forceinline__ bool all_finite(u32x4 v)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            bad |= (v[i] & 0x7f800000u) == 0x7f800000u;
        } else {
            constexpr unsigned e = std::is_same<T, bf16_t>::value ? 0x7f80u : 0x7c00u;
            bad |= (v[i] & e) == e || (v[i] & e << 16) == e << 16;
        }
    }
    return !bad;
}

// acc += u H_r by plain sums, in the rows of their segments alone: for factors H that are not finite, which would reach other
// rows through the zeros of a matrix product, and for calls without scratch (packed false: all factors).  Slow.
// Takes groups of `group` factors that have such an entry in the tile's columns.
template <class C>
__device__ __forceinline__ void add_plainly(const Product &a, int64_t r0, int64_t r1, int64_t c0, bool packed, int group, typename C::Acc &acc)
{
    using T = typename C::T;
    for (int s = first_range(a.ad.offsets, a.ad.segments, r0); s < a.ad.segments; ++s) {
        int64_t lo, hi;
        range_of(a.ad.offsets, s, a.rows, lo, hi);
        if (lo >= r1) break;
        const Run run = run_of(a.ad, s);
        if (hi <= lo || hi <= r0) continue;
        bool use = !packed;
        for (int k = 0; k < run.k; ++k) {
            const T *h = (const T *)a.ad.up + (int64_t)(run.ko + k) * a.ad.ld_up;
            if (packed && k % group == 0) {
                bool bad = false;
                for (int64_t q = threadIdx.x; q < (int64_t)group * C::BN; q += C::THREADS) {
                    const int64_t kk = k + q / C::BN, col = c0 + q % C::BN;
                    if (kk < run.k && col < a.n) bad |= !__builtin_isfinite(Type<T>::load(h[q / C::BN * a.ad.ld_up + col]));
                }
                use = __syncthreads_or(bad);
            }
            if (!use) continue;
            float u[C::TM];
            bool in[C::TM];
#pragma unroll
            for (int i = 0; i < C::TM; ++i) {
                const int64_t row = r0 + C::row_of(i);
                in[i] = row >= lo && row < hi && row < r1;
                u[i] = in[i] ? a.ad.u[row * a.ad.kmax + k] : 0.f;
                if constexpr (std::is_same<T, f16_t>::value)
                    if (packed && in[i]) u[i] /= a.row_scale[row];
            }
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int64_t col = c0 + C::col_of(j) + v;
                    const float x = Type<T>::load(h[col < a.n ? col : a.n - 1]);
#pragma unroll
                    for (int i = 0; i < C::TM; ++i) acc[i][j][v] = in[i] ? __builtin_fmaf(u[i], x, acc[i][j][v]) : acc[i][j][v];
                }
        }
    }
}

// For floats a call with registers of its own (the training step of 4096 rows 1222 -> 1176 us); in 16 bits the same costs the
// tile more than it gives (prompts 434 -> 478 us).
template <class C>
__device__ __noinline__ void add_plainly_called(const Product &a, int64_t r0, int64_t r1, int64_t c0, bool packed, int group, typename C::Acc &acc)
{
    add_plainly<C>(a, r0, r1, c0, packed, group, acc);
}
template <class C>
__device__ __forceinline__ void add_rest(const Product &a, int64_t r0, int64_t r1, int64_t c0, bool packed, int group, typename C::Acc &acc)
{
    if constexpr (sizeof(typename C::T) == 2) {
        add_plainly<C>(a, r0, r1, c0, packed, group, acc);
    } else {
        typename C::Acc copy;
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) copy[i][j] = acc[i][j];
        add_plainly_called<C>(a, r0, r1, c0, packed, group, copy);
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) acc[i][j] = copy[i][j];
    }
}

// acc (cleared) += s_r x W_r H_r from the packed u, segment by segment, a stage of factors at a time, while the next one is
// on its way: the tile's product with H_r, in which the rows of other segments are zeros.  H is looked at first; what has
// entries that are not finite is left out.  (A row of u that is not finite is a row of the result.)  Returns whether
// something was.
template <class C, class X>
__device__ __forceinline__ bool add_packed(const Product &a, int64_t r0, int64_t r1, int64_t c0, char *lds, typename C::Acc &acc)
{
    using T = typename C::T;
    const int kp = (a.ad.kmax + 31) / 32 * 32;
    const int64_t row_n = kp * (4 / (int)sizeof(T));
    bool left_out = false;
    typename X::ReadP rp;
    typename X::ReadQ rq;
    rp.open(X::wave_row());
    rq.open(X::wave_col());
    typename X::LoadP lp;
    typename X::LoadQ lq;
    int s = first_range(a.ad.offsets, a.ad.segments, r0) - 1, k = 0;
    Run run = {0, 0};
    // the next stage: of the run at hand, or of the next segment that has one
    auto advance = [&]() {
        k += X::SK;
        while (k >= run.k) {
            if (++s >= a.ad.segments) return false;
            int64_t lo, hi;
            range_of(a.ad.offsets, s, a.rows, lo, hi);
            if (lo >= r1) return false;
            run = run_of(a.ad, s);
            k = 0;
            if (hi <= lo || hi <= r0) run.k = 0;
            if (run.k == 0) continue;
            Operand P = operand<T>(a.pack, r0 * row_n, row_n, (hi < r1 ? hi : r1) - r0, (a.rows - r0) * row_n);
            P.first = (int)((lo > r0 ? lo : r0) - r0);
            P.plane = kp * (int)sizeof(T);
            lp.open(P);
            lq.open(operand<T>(a.ad.up, run.ko * a.ad.ld_up + c0, a.ad.ld_up, a.n - c0, (a.ad.ktotal - 1 - run.ko) * a.ad.ld_up + a.n - c0));
        }
        return true;
    };
    auto bring = [&](char *stage) {
        lp.fetch(k, run.k, stage);
        lq.fetch(k, run.k, stage + X::kLdsP);
        if constexpr (!X::DMA) {
            lp.put(stage);
            lq.put(stage + X::kLdsP);
        }
    };
    bool more = advance();
    if (more) bring(lds);
    for (int n = 0; more; ++n) {
        const char *stage = lds + (n & 1) * X::kLdsStage;
        [[maybe_unused]] const int left = run.k - k;
        more = advance();
        if (more) {
            bring(lds + (~n & 1) * X::kLdsStage);
            wait_loads<X::DMA ? X::LoadP::kJobs + X::LoadQ::kJobs : 0>();
        } else {
            wait_loads<0>();
        }
        bool bad = false;
#pragma unroll
        for (int j = 0; j < X::LoadQ::kJobs; ++j)      // a thread looks at the chunks that it brought
            bad |= !all_finite<T>(*reinterpret_cast<const u32x4 *>(stage + X::kLdsP + (threadIdx.x + j * X::THREADS) * 16));
        bad = __syncthreads_or(bad);
        left_out |= bad;
        if (!bad) {
            // floats: a matrix step without factors is left out, it takes long
            if (sizeof(T) == 4 && left <= X::SK / 2) X::first_step(stage, rp, rq, acc);
            else X::step(stage, rp, rq, acc, [](int) {});
        }
        meet();
    }
    return left_out;
}

// Accumulators of f16 tiles out of the rows' scales.
template <class C> __device__ __forceinline__ void unscale(const Product &a, int64_t r0, int64_t r1, typename C::Acc &acc)
{
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        const int64_t row = r0 + C::row_of(i);
        const float up = a.row_scale[row < r1 ? row : r0];
#pragma unroll
        for (int j = 0; j < C::TN; ++j) acc[i][j] *= up;
    }
}

// u (or a part of it) for one tile of a segment's rows: s_r x W_r.  Bound by reading x: 16384 rows of 4096 bf16 take 25 to 29 us
// (5.4 to 4.6 TB/s), 8192 rows 16.7; 64 x 64 tiles because ranks are small, four stages of them because memory is far.
template <class C> __device__ __forceinline__ void shrink_tile(const Product &a, int id, char *lds)
{
    using T = typename C::T;
    const int ct = (a.ad.kmax + C::BN - 1) / C::BN;
    const int split = id % a.shrink_splits;
    id /= a.shrink_splits;
    Found f;
    Ranges ranges;
    ranges.open(a.ad.offsets, a.ad.segments, a.rows, C::BM);
    if (!ranges.find(id / ct, f)) return;
    const Run run = run_of(a.ad, f.g);
    const int c0 = id % ct * C::BN;
    if (c0 >= run.k) return;
    const Operand P = operand<T>(a.x, f.r0 * a.ldx, a.ldx, f.r1 - f.r0, (a.rows - 1 - f.r0) * a.ldx + a.m);
    const Operand Q = operand<T>(a.ad.down, (run.ko + c0) * a.ad.ld_down, a.ad.ld_down, run.k - c0, (a.ad.ktotal - 1 - run.ko - c0) * a.ad.ld_down + a.m);
    const int64_t k0 = split * a.shrink_k, k1 = k0 + a.shrink_k < a.m ? k0 + a.shrink_k : a.m;
    typename C::Acc acc;
    C::clear(acc);
    C::multiply(P, Q, k0, k1, lds, acc);
    float *out = a.ad.u;
    if (a.shrink_splits > 1) out = a.upart + (int64_t)split * a.rows * a.ad.kmax;
    const float scale = a.ad.scale ? a.ad.scale[a.ad.run[f.g]] : 1.f;
    C::store(acc, out + f.r0 * a.ad.kmax + c0, a.ad.kmax, f.r1 - f.r0, run.k - c0, false, lds, scale);
}

template <class S> __global__ __launch_bounds__(S::THREADS) void shrink_kernel(Product a)
{
    __shared__ __align__(1024) char lds[S::kLds];
    shrink_tile<S>(a, blockIdx.x, lds);
}

// Y, or parts of it over the contraction.  The first `shrink` workgroups form parts of u instead.  Long products are bound by
// their loads and by power: 8192 x 4096 x 4096 bf16 208 us (1325 TFLOP/s), 16384 rows with adapters up to rank 64 406 to 419 us
// (1310 to 1355), float32 in tiles of 256 x 256 144 TFLOP/s.  Few rows are bound by reading b: 512 rows over 64 groups of
// 4096 x 2048 f16 150 to 171 us (6.5 to 5.7 TB/s).
template <class C, class S, bool ADAPTERS> __global__ __launch_bounds__(C::THREADS) void product_kernel(Product a, int shrink)
{
    using T = typename C::T;
    constexpr bool both = ADAPTERS && S::THREADS == C::THREADS;      // else shrink is 0
    __shared__ __align__(1024) char lds[both && S::kLds > C::kLds ? S::kLds : C::kLds];
    if constexpr (both) {
        if ((int)blockIdx.x < shrink) {
            shrink_tile<S>(a, blockIdx.x, lds);
            return;
        }
    }
    Ranges ranges;
    const int rt = a.offsets ? ranges.open(a.offsets, a.groups, a.rows, C::BM) : (int)((a.rows + C::BM - 1) / C::BM);
    const int ct = (int)((a.n + C::BN - 1) / C::BN);
    const int each = rt * ct, total = each * a.splits, mine = blockIdx.x - shrink;
    if (mine >= total) return;
    int id = by_die(mine, total);
    const int split = id / each;
    id -= split * each;
    // four row tiles side by side share what they read of B
    const int block = id / (4 * ct), in = id - block * 4 * ct, high = rt - 4 * block < 4 ? rt - 4 * block : 4;
    const int r = 4 * block + in % high;
    const int64_t c0 = (int64_t)(in / high) * C::BN;
    Found f = {0, (int64_t)r * C::BM, 0};
    if (a.offsets) {
        if (!ranges.find(r, f)) return;
    } else {
        f.r1 = f.r0 + C::BM < a.rows ? f.r0 + C::BM : a.rows;
    }
    const Operand P = operand<T>(a.x, f.r0 * a.ldx, a.ldx, f.r1 - f.r0, (a.rows - 1 - f.r0) * a.ldx + a.m);
    const Operand Q = C::QRC ? operand<T>(a.b, f.g * a.stride_b + c0, a.ldb, a.n - c0, (a.m - 1) * a.ldb + a.n - c0)
                             : operand<T>(a.b, f.g * a.stride_b + c0 * a.ldb, a.ldb, a.n - c0, (a.n - 1 - c0) * a.ldb + a.m);
    const int64_t k0 = split * a.k_split, k1 = k0 + a.k_split < a.m ? k0 + a.k_split : a.m;
    typename C::Acc acc;
    C::clear(acc);
    if constexpr (ADAPTERS) {
        using X = Tile<T, C::BM, C::BN, C::WM, C::WN, 2, false, true, C::DMA, (sizeof(T) == 2 ? 2 : 1)>;
        if (!a.joined) {
            const bool packed = a.pack != nullptr;
            if (!packed || add_packed<C, X>(a, f.r0, f.r1, c0, lds, acc)) add_rest<C>(a, f.r0, f.r1, c0, packed, X::SK, acc);
            if constexpr (std::is_same<T, f16_t>::value)
                if (packed) unscale<C>(a, f.r0, f.r1, acc);
        }
    }
    C::multiply(P, Q, k0, k1, lds, acc);
    if (a.joined) {
        const int64_t n4 = up4(a.n);
        C::store(acc, a.part + ((int64_t)split * a.rows + f.r0) * n4 + c0, n4, f.r1 - f.r0, a.n - c0, true, lds);
        return;
    }
    C::store(acc, (T *)a.y + f.r0 * a.ldy + c0, a.ldy, f.r1 - f.r0, a.n - c0, a.vec, lds);
}

// Y of one row and 256 columns from the parts, and its adapter: wave w adds parts and factors w, w + 4, ..., and the four
// sums meet in order.  (A row a wave instead, four to a workgroup: 24 us against 21 for 48 rows, equal for 160.)
template <class T> __global__ __launch_bounds__(256) void join_product_kernel(Product a)
{
    const int ct = (int)((a.n + 255) / 256);
    const int64_t row = blockIdx.x / ct;
    const int c = blockIdx.x % ct, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    const int64_t col = (int64_t)c * 256 + lane * 4, n4 = up4(a.n), at = col < a.n ? col : 0;
    __shared__ float us[kMaxRank];
    __shared__ f32x4 sums[4][64];
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    {
        f32x4 t[kMaxSplits / 4];
#pragma unroll
        for (int i = 0; i < kMaxSplits / 4; ++i) {
            const int s = w + 4 * i;
            t[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (s < a.splits) t[i] = *reinterpret_cast<const f32x4 *>(a.part + ((int64_t)s * a.rows + row) * n4 + at);
        }
#pragma unroll
        for (int i = 0; i < kMaxSplits / 4; ++i) y += t[i];
    }
    if (a.offsets) {
        const int g = first_range(a.offsets, a.groups, row);
        if (g == a.groups || a.offsets[g] > row) return;
    }
    if (a.ad.segments) {
        Run run = {0, 0};
        const int s = first_range(a.ad.offsets, a.ad.segments, row);
        if (s < a.ad.segments && a.ad.offsets[s] <= row) run = run_of(a.ad, s);
        for (int k = threadIdx.x; k < run.k; k += 256) {
            float u = 0.f;
            if (a.shrink_splits > 1) {
                float t[kMaxSplits];
#pragma unroll
                for (int p = 0; p < kMaxSplits; ++p) t[p] = p < a.shrink_splits ? a.upart[(p * a.rows + row) * a.ad.kmax + k] : 0.f;
#pragma unroll
                for (int p = 0; p < kMaxSplits; ++p) u += t[p];
                if (c == 0) a.ad.u[row * a.ad.kmax + k] = u;
            } else {
                u = a.ad.u[row * a.ad.kmax + k];
            }
            us[k] = u;
        }
        __syncthreads();
        const T *h = (const T *)a.ad.up + run.ko * a.ad.ld_up;
        for (int k0 = w; k0 < run.k; k0 += 16) {
            float x[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = k0 + 4 * i < run.k ? k0 + 4 * i : run.k - 1;
                const T *line = h + k * a.ad.ld_up;
                if (col + 4 <= a.n) {
                    T four[4];
                    __builtin_memcpy(four, line + col, sizeof(four));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][e] = Type<T>::load(four[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][e] = Type<T>::load(line[col + e < a.n ? col + e : a.n - 1]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + 4 * i < run.k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __builtin_fmaf(us[k0 + 4 * i], x[i][e], y[e]);
        }
    }
    sums[w][lane] = y;
    __syncthreads();
    if (w || col >= a.n) return;
    y = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
    T *out = (T *)a.y + row * a.ldy + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < a.n) out[e] = Type<T>::round(y[e]);
}

// dB_g = X_g^T dY_g, or parts of it over the group's rows: both operands by columns, through the transposing reads.
// 8 groups of 8192 rows in all, 4096 x 2048, bf16: 139 us (992 TFLOP/s; one group of 8192 rows 203 us for 4096 x 4096, 1350).
template <class C> __global__ __launch_bounds__(C::THREADS) void gradient_kernel(Gradient a)
{
    using T = typename C::T;
    __shared__ __align__(1024) char lds[C::kLds];
    const int mt = (int)((a.m + C::BM - 1) / C::BM), nt = (int)((a.n + C::BN - 1) / C::BN);
    // Every die has its share of each group's tiles, the longest groups first: a tile takes as long as its group.
    const int tiles = mt * nt * a.splits, per = (tiles + 7) / 8, nth = blockIdx.x / 8;
    int id = blockIdx.x % 8 * per + nth % per;
    if (id >= tiles) return;
    const int g = nth_longest(a.offsets, a.groups, a.rows, nth / per);
    const int split = id % a.splits;
    id /= a.splits;
    const int block = id / (4 * nt), in = id - block * 4 * nt, high = mt - 4 * block < 4 ? mt - 4 * block : 4;
    const int64_t r0 = (int64_t)(4 * block + in % high) * C::BM, c0 = (int64_t)(in / high) * C::BN;
    int64_t lo, hi;
    range_of(a.offsets, g, a.rows, lo, hi);
    const int64_t len = hi - lo;
    const int64_t stages = (len + stage_k<T>() - 1) / stage_k<T>();
    const int64_t each = (stages + a.splits - 1) / a.splits * stage_k<T>();
    const int64_t k0 = split * each < len ? split * each : len, k1 = k0 + each < len ? k0 + each : len;
    const Operand P = operand<T>(a.x, lo * a.ldx + r0, a.ldx, a.m - r0, (a.rows - 1 - lo) * a.ldx + a.m - r0);
    const Operand Q = operand<T>(a.dy, lo * a.ldy + c0, a.ldy, a.n - c0, (a.rows - 1 - lo) * a.ldy + a.n - c0);
    typename C::Acc acc;
    C::clear(acc);
    if (k1 > k0) C::multiply(P, Q, k0, k1, lds, acc);
    if (a.splits > 1) {
        const int64_t n4 = up4(a.n);
        C::store(acc, a.part + (((int64_t)split * a.groups + g) * a.m + r0) * n4 + c0, n4, a.m - r0, a.n - c0, true, lds);
    } else {
        C::store(acc, (T *)a.g + g * a.stride_g + r0 * a.ldg + c0, a.ldg, a.m - r0, a.n - c0, a.vec, lds);
    }
}

// Sums of parts: line l of `lines` (n columns) to out + (l / m) * stride + (l % m) * ld.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(const float *part, int splits, int64_t lines, int64_t n, T *out, int64_t m,
                                                   int64_t stride, int64_t ld)
{
    const int64_t n4 = up4(n), per = n4 / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < lines * per; i += (int64_t)gridDim.x * 256) {
        const int64_t l = i / per, col = (i - l * per) * 4;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) y += *reinterpret_cast<const f32x4 *>(part + ((int64_t)s * lines + l) * n4 + col);
        T *o = out + l / m * stride + l % m * ld + col;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < n) o[e] = Type<T>::round(y[e]);
    }
}

// ---- gradients of the factors --------------------------------------------------------
// A run's rows, in blocks of `rows` within its segments, are dealt out in chunks of `chunk` blocks, so that a run with many
// rows takes many workgroups and one without rows a single one, which writes its zeros.
struct Chunks {
    int run, first, count;       // a run; its first chunk and how many it has
    int slot;                    // of the first one among the parts, which runs with several chunks have
};
// Of chunk `want`, or of run `want`.  Ranges that do not overlap give a.chunks chunks and a.slots parts at most; those that do
// can give any number, so blocks, counts and their sums are held to what the launch has, and chunks beyond do not exist.
constexpr int kMostBlocks = 1 << 28;      // rows / 32 and as many segments as rows, for the rows that a launch takes
template <bool BY_RUN = false> __device__ __forceinline__ bool find_chunk(const FactorGradient &a, int rows, int want, Chunks &f)
{
    const int lane = threadIdx.x & 63;
    int before = 0, slots = 0;
    for (int r0 = 0; r0 < a.ad.runs; r0 += 64) {
        int blocks = 0;
        for (int base = 0; base < a.ad.segments; base += 64) {
            int of = -1, nb = 0;
            if (base + lane < a.ad.segments) {
                int64_t lo, hi;
                range_of(a.ad.offsets, base + lane, a.rows, lo, hi);
                of = a.ad.run[base + lane];
                nb = (int)((hi - lo + rows - 1) / rows);
            }
            const int here = a.ad.segments - base < 64 ? a.ad.segments - base : 64;
            for (int i = 0; i < here; ++i)
                if (__builtin_amdgcn_readlane(of, i) == r0 + lane) blocks += __builtin_amdgcn_readlane(nb, i);
            if (blocks > kMostBlocks) blocks = kMostBlocks;      // (64 times what one segment can have fits)
        }
        int count = 0;
        if (r0 + lane < a.ad.runs) count = blocks <= a.chunk ? 1 : (blocks - 1) / a.chunk + 1;
        if (count > a.chunks) count = a.chunks;
        int sum = count, parts = count > 1 ? count : 0;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d), q = __shfl_up(parts, d);
            if (lane >= d) sum += o, parts += q;
        }
        const unsigned long long past = __ballot(BY_RUN ? r0 + lane == want : before + sum > want);
        if (past) {
            const int l = __builtin_ctzll(past);
            f.run = r0 + l;
            f.count = __builtin_amdgcn_readlane(count, l);
            f.first = before + __builtin_amdgcn_readlane(sum, l) - f.count;
            f.slot = slots + __builtin_amdgcn_readlane(parts, l) - f.count;
            if (f.count > a.chunks - f.first) f.count = a.chunks - f.first;
            if (f.count > 1 && f.count > a.slots - f.slot) f.count = a.slots - f.slot;
            return BY_RUN || want - f.first < f.count;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
        if (before > a.chunks) before = a.chunks;
        slots += __builtin_amdgcn_readlane(parts, 63);
        if (slots > a.slots) slots = a.slots;
    }
    return false;
}

// U and V (blockIdx.y) as the three bf16 pieces that the gradients' products take, once for all column tiles: rows x 3 planes x kp
// entries, kp = kmax in whole tiles, zero behind a run's rank and in rows without a run.  One row per 16 lanes.
__global__ __launch_bounds__(256) inline void pack_factors_kernel(FactorGradient a, int kp)
{
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    if (row >= a.rows) return;
    Run run = {0, 0};
    const int s = range_at(a.ad.offsets, a.ad.segments, row);
    if (s < a.ad.segments && a.ad.offsets[s] <= row) run = run_of(a.ad, s);
    const float *in = (blockIdx.y ? a.v : a.u) + row * a.ad.kmax;
    bf16_t *out = (bf16_t *)a.pieces + (blockIdx.y * a.rows + row) * (kFactorPieces * (int64_t)kp);
    for (int k = threadIdx.x & 15; k < kp; k += 16) {
        float x = k < run.k ? in[k] : 0.f;
#pragma unroll
        for (int n = 0; n < kFactorPieces; ++n, x = after_piece(x)) out[n * kp + k] = Type<bf16_t>::round(x);
    }
}

// BM factors of one run x 128 columns of m or of n, summed over a chunk of its rows, 64 (bf16) or 32 at a time.  (f16: X and dY are
// two pieces in LDS; 64 rows of them leave room for one workgroup on a compute unit, 32 for two or three.)
// Reads X and dY once for every BM factors; 8192 rows, 4096 + 4096 columns, ranks to 64: bf16 63 us (2.1 TB/s) on pieces (82 where each
// column tile cuts them itself), f16 90 (111), bound by the latency of its loads at two workgroups a compute unit; ranks to 16 44 and 63;
// 4096 rows of 4096 + 2048 floats, ranks to 16: 37 us (2.7 TB/s).
template <class T, int BM> __global__ __launch_bounds__(256) void factor_gradient_kernel(FactorGradient a)
{
    using E = typename Cut<T>::E;
    constexpr int BN = 128, SK = block_rows<T>();
    constexpr int N = Cut<T>::kPieces;
    constexpr bool two = two_piece_matrix<T>();
    constexpr int kP = SK * BM * (int)sizeof(E), kQ = SK * BN * (int)sizeof(E);
    constexpr int TM = BM / 16, TN = 2;
    constexpr int kAllP = kP * N, kStage = kAllP + kQ * (two ? 2 : 1);
    __shared__ __align__(1024) char lds[2 * kStage];

    const int mt = (int)((a.m + BN - 1) / BN);
    const bool down = (int)blockIdx.x < mt;                // dW: from v and X; dH: from u and dY
    const int64_t width = down ? a.m : a.n, c0 = (int64_t)(down ? blockIdx.x : blockIdx.x - mt) * BN;
    const char *src = (const char *)(down ? a.x : a.dy);
    const int64_t ld = down ? a.ldx : a.ldy;
    const float *fac = down ? a.v : a.u;
    const int kp = gridDim.y * BM;
    [[maybe_unused]] const bf16_t *pieces = a.pieces ? (const bf16_t *)a.pieces + (down ? a.rows * N * (int64_t)kp : 0) : nullptr;
    const int f0 = blockIdx.y * BM, z = blockIdx.z;
    Chunks mychunk;
    if (!find_chunk(a, SK, z, mychunk)) return;
    const int id = mychunk.run, from = (z - mychunk.first) * a.chunk;
    const int64_t klo = a.ad.koff[id], khi = a.ad.koff[id + 1];
    if (klo < 0 || khi <= klo || klo >= a.ad.ktotal) return;
    int64_t k = (khi < a.ad.ktotal ? khi : a.ad.ktotal) - klo;
    const int64_t mine = k - f0;                            // factors of this workgroup and behind it
    if (mine <= 0) return;
    if (k > a.ad.kmax) k = a.ad.kmax;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Reader<E, BM, true, 16> rp;
    Reader<E, BN, true, 16> rq;
    rp.open(0);
    rq.open(wave * 32);
    f32x4 acc[TM][TN], low[TM][TN];                        // products of the first pieces, and of the others
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = low[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    constexpr int EN = chunk_n<E>(), TE = chunk_n<T>();
    constexpr int pc = BM / EN, PJ = (SK * pc + 255) / 256, qc = BN / TE, QJ = SK * qc / 256;
    auto one_of = [](int q) { return SK * pc % 256 == 0 || q < SK * pc; };      // a thread's chunk of P exists

    // The run's rows in blocks of SK within its segments: a.chunk of them from `from` on.
    int base = -64, turn = -1;
    unsigned long long todo = 0;
    int64_t lo = 0, hi = 0, r = 0, shi = 0;
    auto advance = [&]() {
        for (;;) {
            r += SK;
            while (r >= shi) {
                while (!todo) {
                    base += 64;
                    if (base >= a.ad.segments) return false;
                    lo = hi = 0;
                    bool is = false;
                    if (base + lane < a.ad.segments) {
                        range_of(a.ad.offsets, base + lane, a.rows, lo, hi);
                        is = a.ad.run[base + lane] == id && hi > lo;
                    }
                    todo = __ballot(is);
                }
                const int l = __builtin_ctzll(todo);
                todo &= todo - 1;
                r = Ranges::lane_value(lo, l);
                shi = Ranges::lane_value(hi, l);
            }
            if (++turn >= from + a.chunk) return false;
            if (turn >= from) return true;
        }
    };
    u32x4 pv[PJ][N], qv[QJ];
    auto get = [&]() {
        const int64_t left = shi - r;
#pragma unroll
        for (int j = 0; j < QJ; ++j) {
            const int q = threadIdx.x + 256 * j, kr = q / qc, c = q % qc;
            qv[j] = u32x4{0, 0, 0, 0};
            if (kr < left && c0 + c * TE < width) {
                const int64_t e = (r + kr) * ld + c0 + c * TE;
                qv[j] = chunk_at<T>(src + e * (int64_t)sizeof(T), ((a.rows - 1) * ld + width - e) * (int64_t)sizeof(T));
            }
        }
#pragma unroll
        for (int j = 0; j < PJ; ++j) {
            const int q = threadIdx.x + 256 * j, kr = q / pc, c = q % pc;
            if (!one_of(q)) continue;
            if constexpr (N > 1) {
                if (pieces) {
                    const bf16_t *line = pieces + (r + (kr < left ? kr : 0)) * (N * (int64_t)kp) + f0 + c * EN;
#pragma unroll
                    for (int i = 0; i < N; ++i) pv[j][i] = kr < left ? *reinterpret_cast<const u32x4 *>(line + i * kp) : u32x4{0, 0, 0, 0};
                    continue;
                }
            }
            float x[EN];
            floats_at<EN>(fac + (r + (kr < left ? kr : 0)) * a.ad.kmax, f0 + c * EN, kr < left ? (int)k : 0, a.ad.kmax, x);
            if constexpr (N > 1) cut_chunk(x, pv[j]);
            else pv[j][0] = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
        }
    };
    auto put = [&](char *to) {
#pragma unroll
        for (int j = 0; j < PJ; ++j) {
            const int q = threadIdx.x + 256 * j, kr = q / pc, c = q % pc;
            if (!one_of(q)) continue;
            char *at = to + kr * (BM * (int)sizeof(E)) + ((c ^ rc_shift<E, BM>(kr)) << 4);
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4 *>(at + i * kP) = pv[j][i];
        }
#pragma unroll
        for (int j = 0; j < QJ; ++j) {
            const int q = threadIdx.x + 256 * j, kr = q / qc, c = q % qc;
            char *at = to + kAllP + kr * (BN * (int)sizeof(E)) + ((c ^ rc_shift<E, BN>(kr)) << 4);
            if constexpr (two) {
                float x[8];
                u32x4 two_of[2];
                floats_of(qv[j], x);
                cut_chunk(x, two_of);
                *reinterpret_cast<u32x4 *>(at) = two_of[0];
                *reinterpret_cast<u32x4 *>(at + kQ) = two_of[1];
            } else {
                *reinterpret_cast<u32x4 *>(at) = qv[j];
            }
        }
    };
    // the next block is on its way while one is multiplied
    bool more = advance();
    if (more) {
        get();
        put(lds);
    }
    for (int n = 0; more; ++n) {
        meet();
        more = advance();
        if (more) get();
        const char *lp = lds + (n & 1) * kStage, *lq = lp + kAllP;
#pragma unroll
        for (int kk = 0; kk < SK * (int)sizeof(E) / 64; ++kk) {
            u32x4 q[TN], ql[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                q[j] = rq.read(lq, j, kk);
                if constexpr (two) ql[j] = rq.read(lq + kQ, j, kk);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                // all products of pieces but a half's second with a float's last, below 2^-26 of the whole
                u32x4 p[N];
#pragma unroll
                for (int n = 0; n < N; ++n) p[n] = rp.read(lp + n * kP, i, kk);
                if constexpr (two) mac_row<E>(ql, p[1], low[i]);
                if constexpr (N > 1) mac_row<E>(q, p[N - 1], low[i]);
                mac_row<E>(q, p[0], acc[i]);
                if constexpr (two) mac_row<E>(ql, p[0], low[i]);
                if constexpr (N > 1) mac_row<E>(q, p[1], low[i]);
            }
        }
        if (more) put(lds + ((n + 1) & 1) * kStage);
    }
    const int64_t m4 = up4(a.m), n4 = up4(a.n);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = 16 * i + (lane & 15);
        if (row >= mine) continue;
        const bool real = f0 + row < k;                     // factors beyond kmax take no part: zero
        const int64_t line = klo + f0 + row;
        float *part = nullptr;
        if (mychunk.count > 1) part = a.part + ((int64_t)(mychunk.slot + z - mychunk.first) * gridDim.y * BM + f0 + row) * (m4 + n4) + (down ? 0 : m4);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t col = c0 + 32 * wave + 16 * j + 4 * (lane >> 4) + v;
                if (col >= width) continue;
                const float x = real ? both_pieces<(N > 1)>(acc[i][j][v], low[i][j][v]) : 0.f;
                if (part) part[col] = x;
                else ((T *)(down ? a.ddown : a.dup))[line * width + col] = Type<T>::round(x);
            }
    }
}

// The gradients of runs with several chunks: one factor of a run, 1024 columns of m and n side by side.
template <class T, int BM> __global__ __launch_bounds__(256) void join_factors_kernel(FactorGradient a, int padded)
{
    constexpr int SK = block_rows<T>();
    const int id = blockIdx.x / a.ad.kmax, k = blockIdx.x % a.ad.kmax;
    const int64_t lo = a.ad.koff[id], hi = a.ad.koff[id + 1];
    if (lo < 0 || lo + k >= hi || lo + k >= a.ad.ktotal) return;
    Chunks f;
    if (!find_chunk<true>(a, SK, id, f)) return;
    if (f.count < 2) return;
    const int64_t m4 = up4(a.m), n4 = up4(a.n), at = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
    if (at >= m4 + n4) return;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < f.count; ++c) y += *reinterpret_cast<const f32x4 *>(a.part + ((int64_t)(f.slot + c) * padded + k) * (m4 + n4) + at);
    const bool down = at < m4;
    const int64_t col = down ? at : at - m4, width = down ? a.m : a.n;
    T *out = (T *)(down ? a.ddown : a.dup) + (lo + k) * width + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < width) out[e] = Type<T>::round(y[e]);
}

// ---- launches --------------------------------------------------------------------------

// `count` matrices of rows x cols to rows of ldo entries (whole 16 bytes), zero behind their ends: operands whose rows do not
// begin and end on 16 bytes.
template <class T>
__global__ __launch_bounds__(256) void align_kernel(const char *src, int64_t ld, int64_t stride, int64_t rows, int64_t cols, int64_t count, char *dst,
                                                    int64_t ldo)
{
    constexpr int E = chunk_n<T>();
    const int64_t per = ldo / E, all = count * rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t line = i / per, c = (i - line * per) * E, g = line / rows, r = line - g * rows;
        const int64_t e = g * stride + r * ld + c;
        const int64_t end = (count - 1) * stride + (rows - 1) * ld + cols;
        *reinterpret_cast<u32x4 *>(dst + i * 16) = keep_first<T>(chunk_at<T>(src + e * (int64_t)sizeof(T), (end - e) * (int64_t)sizeof(T)), cols - c);
    }
}
template <class T> hipError_t launch_align(const Align &a, hipStream_t st)
{
    const int64_t chunks = a.count * a.rows * (a.ldo / chunk_n<T>()), blocks = (chunks + 255) / 256;
    hipLaunchKernelGGL((align_kernel<T>), dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st, (const char *)a.src, a.ld, a.stride,
                       a.rows, a.cols, a.count, (char *)a.dst, a.ldo);
    return hipGetLastError();
}

template <class T, bool QRC, bool DMA> void launch_shape(const Product &p, int shrink, hipStream_t st)
{
    using S = Tile<T, kShrinkRows, kShrinkCols, 2, 2, 4, false, false, DMA>;
    auto go = [&](auto tile) {
        using C = decltype(tile);
        const int64_t rt = (p.rows + C::BM - 1) / C::BM + (p.offsets ? p.groups : 0), ct = (p.n + C::BN - 1) / C::BN;
        const dim3 grid((unsigned)(rt * ct * p.splits + shrink));
        if (p.ad.segments) hipLaunchKernelGGL((product_kernel<C, S, true>), grid, dim3(C::THREADS), 0, st, p, shrink);
        else hipLaunchKernelGGL((product_kernel<C, S, false>), grid, dim3(C::THREADS), 0, st, p, shrink);
    };
    switch (p.shape) {
    case k256x256: go(Tile<T, 256, 256, 2, 4, 2, false, QRC, DMA>{}); break;
    case k128x128: go(Tile<T, 128, 128, 2, 2, 2, false, QRC, DMA>{}); break;
    case k64x64: go(Tile<T, 64, 64, 2, 2, 3, false, QRC, DMA>{}); break;
    case k64x128: go(Tile<T, 64, 128, 1, 4, 3, false, QRC, DMA>{}); break;
    default: go(Tile<T, 32, 128, 1, 4, 4, false, QRC, DMA>{}); break;
    }
}

inline bool by16(const void *p, int64_t a = 0, int64_t b = 0) { return (((uintptr_t)p | (uint64_t)a | (uint64_t)b) & 15) == 0; }

template <class T> hipError_t launch_product(const Product &p, hipStream_t st)
{
    constexpr int E = sizeof(T);
    const int64_t far = (int64_t)1 << 30;
    const bool whole_m = p.padded || p.m * E % 16 == 0, whole_n = p.padded || p.n * E % 16 == 0;       // rows fill their 16 bytes
    bool dma = whole_m && by16(p.x, p.ldx * E) && by16(p.b, p.ldb * E, p.stride_b * E) && p.ldx * E * 256 < far && p.ldb * E * 256 < far;
    if (p.transposed == 0) dma = dma && whole_n;
    if (p.ad.segments)
        dma = dma && whole_n && by16(p.ad.down, p.ad.ld_down * E) && by16(p.ad.up, p.ad.ld_up * E) && p.ad.ld_down * E * 256 < far &&
              p.ad.ld_up * E * 256 < far;
    using ShrinkDma = Tile<T, kShrinkRows, kShrinkCols, 2, 2, 4, false, false, true>;
    using Shrink = Tile<T, kShrinkRows, kShrinkCols, 2, 2, 4, false, false, false>;
    int shrink = 0;
    if (p.ad.segments) {
        const int64_t rt = (p.rows + kShrinkRows - 1) / kShrinkRows + p.ad.segments, ct = (p.ad.kmax + kShrinkCols - 1) / kShrinkCols;
        shrink = (int)(rt * ct * p.shrink_splits);
        // its tiles run in the product's launch where that has workgroups of their size and nothing waits for u there
        if (!p.joined || p.shape == k256x256) {
            if (dma) hipLaunchKernelGGL((shrink_kernel<ShrinkDma>), dim3(shrink), dim3(ShrinkDma::THREADS), 0, st, p);
            else hipLaunchKernelGGL((shrink_kernel<Shrink>), dim3(shrink), dim3(Shrink::THREADS), 0, st, p);
            shrink = 0;
            if (p.pack) hipLaunchKernelGGL((pack_kernel<T>), dim3((unsigned)((p.rows + 15) / 16)), dim3(256), 0, st, p);
        }
    }
    if (p.transposed) {
        if (dma) launch_shape<T, false, true>(p, shrink, st);
        else launch_shape<T, false, false>(p, shrink, st);
    } else {
        if (dma) launch_shape<T, true, true>(p, shrink, st);
        else launch_shape<T, true, false>(p, shrink, st);
    }
    if (p.joined) hipLaunchKernelGGL((join_product_kernel<T>), dim3((unsigned)((p.n + 255) / 256 * p.rows)), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <class T> void launch_join(const float *part, int splits, int64_t lines, int64_t n, T *out, int64_t m, int64_t stride, int64_t ld,
                                    hipStream_t st)
{
    const int64_t blocks = (lines * (up4(n) / 4) + 255) / 256;
    hipLaunchKernelGGL((join_kernel<T>), dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, part, splits, lines, n, out, m,
                       stride, ld);
}

template <class T> hipError_t launch_gradient(const Gradient &p, hipStream_t st)
{
    constexpr int E = sizeof(T);
    const int64_t far = (int64_t)1 << 30;
    const bool dma = by16(p.x, p.ldx * E) && by16(p.dy, p.ldy * E) && (p.padded || ((p.m | p.n) * E % 16 == 0)) && p.ldx * E * 64 < far &&
                     p.ldy * E * 64 < far;
    auto go = [&](auto tile) {
        using C = decltype(tile);
        const int64_t tiles = ((p.m + C::BM - 1) / C::BM * ((p.n + C::BN - 1) / C::BN) * p.splits + 7) / 8 * 8 * p.groups;
        hipLaunchKernelGGL((gradient_kernel<C>), dim3((unsigned)tiles), dim3(C::THREADS), 0, st, p);
    };
    auto any = [&](auto d) {
        constexpr bool DMA = d.value;
        switch (p.shape) {
        case k256x256: go(Tile<T, 256, 256, 2, 4, 2, true, true, DMA>{}); break;
        case k128x128: go(Tile<T, 128, 128, 2, 2, 2, true, true, DMA>{}); break;
        default: go(Tile<T, 64, 64, 2, 2, 3, true, true, DMA>{}); break;
        }
    };
    if (dma) any(std::true_type{});
    else any(std::false_type{});
    if (p.splits > 1)
        launch_join<T>(p.part, p.splits, (int64_t)p.groups * p.m, p.n, (T *)p.g, p.m, p.stride_g, p.ldg, st);
    return hipGetLastError();
}

template <class T> hipError_t launch_factor_gradient(const FactorGradient &p, hipStream_t st)
{
    const unsigned cols = (unsigned)((p.m + 127) / 128 + (p.n + 127) / 128);
    auto go = [&](auto bm) {
        constexpr int BM = bm.value;
        const unsigned kt = (unsigned)((p.ad.kmax + BM - 1) / BM);
        if (p.pieces) hipLaunchKernelGGL(pack_factors_kernel, dim3((unsigned)((p.rows + 15) / 16), 2), dim3(256), 0, st, p, (int)kt * BM);
        hipLaunchKernelGGL((factor_gradient_kernel<T, BM>), dim3(cols, kt, (unsigned)p.chunks), dim3(256), 0, st, p);
        if (p.slots)
            hipLaunchKernelGGL((join_factors_kernel<T, BM>), dim3((unsigned)(p.ad.runs * p.ad.kmax), (unsigned)((up4(p.m) + up4(p.n) + 1023) / 1024)),
                               dim3(256), 0, st, p, (int)kt * BM);
    };
    if (p.ad.kmax <= 32) go(std::integral_constant<int, 32>{});
    else go(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

}  // namespace ragged
}  // namespace nmfmu
