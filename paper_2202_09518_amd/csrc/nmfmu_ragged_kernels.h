// Kernels and launches of the products over ragged ranges of rows, for one type T; included by one source per type.
#pragma once

#include "nmfmu_ragged_internal.h"
#include "nmfmu_ragged_device.h"

namespace nmfmu {
namespace ragged {

// ---- float factors on the halves' matrix cores -------------------------------------
// u = hi + lo, two bf16: 16 to 17 bits of a float, which is 2^-8 of what an output in 16 bits can show.
template <bool LOW> __device__ __forceinline__ float piece(float x)
{
    const float hi = Type<bf16_t>::load(Type<bf16_t>::round(x));
    if (!LOW) return hi;
    const float lo = x - hi;
    return __builtin_isfinite(hi) ? lo : 0.f;
}
__device__ __forceinline__ void cut_chunk(const float (&x)[8], u32x4 &hi, u32x4 &lo)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
        lo[i] = cvt_pk_bf16(piece<true>(x[2 * i]), piece<true>(x[2 * i + 1]));
    }
}
__device__ __forceinline__ void floats_of(u32x4 v, float (&x)[8], f16_t)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Type<f16_t>::load(f16_t{(unsigned short)(v[i >> 1] >> (16 * (i & 1)))});
}
__device__ __forceinline__ void floats_of(u32x4 v, float (&x)[8], bf16_t)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Type<bf16_t>::load(bf16_t{(unsigned short)(v[i >> 1] >> (16 * (i & 1)))});
}

template <class T> struct Cut {                      // the type that float factors are multiplied in
    using E = bf16_t;
    static constexpr bool kBoth = sizeof(T) == 2;    // float operand in two pieces
};
template <> struct Cut<float> {
    using E = float;
    static constexpr bool kBoth = false;
};
template <class T> constexpr bool two_piece_matrix() { return false; }
template <> constexpr bool two_piece_matrix<f16_t>() { return true; }      // its 11 bits are two bf16

// Entries [k, k + N) of a row of floats that ends at kend; zero behind it.
template <int N> __device__ __forceinline__ void floats_at(const float *row, int k, int kend, float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = k + i < kend ? row[k + i] : 0.f;
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

// acc += u H_r for the rows of a tile, segment by segment, 32 factors at a time; u lies scaled in memory.
// A segment's product is formed on its own and added in its rows only: factors that are not finite reach no other
// request's rows.
template <class C>
__device__ __forceinline__ void add_adapters(const Product &a, int64_t r0, int64_t r1, int64_t c0, char *lds, typename C::Acc &acc)
{
    using T = typename C::T;
    using E = typename Cut<T>::E;
    constexpr int EN = chunk_n<E>();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    Reader<E, C::BM, false> rp;
    Reader<E, C::BN, true> rq;
    const int first = wave / C::WN * (C::BM / C::WM);
    rp.open(first);
    rq.open(wave % C::WN * (C::BN / C::WN));
    char *lq = lds + C::BM * kStageBytes;
    for (int s = first_range(a.ad.offsets, a.ad.segments, r0); s < a.ad.segments; ++s) {
        int64_t lo, hi;
        range_of(a.ad.offsets, s, a.rows, lo, hi);
        if (lo >= r1) break;
        const int from = (int)((lo > r0 ? lo : r0) - r0), to = (int)((hi < r1 ? hi : r1) - r0);
        const Run run = run_of(a.ad, s);
        if (run.k == 0 || to <= from) continue;
        for (int kc = 0; kc < run.k; kc += 32) {
            for (int q = threadIdx.x; q < C::BM * 32 / EN; q += C::THREADS) {
                const int row = q / (32 / EN), c = q % (32 / EN), swz = (row >> 1) & 7;
                const bool in = row >= from && row < to;
                const int64_t line = (r0 + (in ? row : from)) * a.ad.kmax;
                float x[EN];
                if (a.shrink_splits == 1) {
                    floats_at<EN>(a.ad.u + line, kc + c * EN, in ? run.k : 0, x);
                } else {
#pragma unroll
                    for (int e = 0; e < EN; ++e) x[e] = 0.f;
                    for (int s2 = 0; s2 < a.shrink_splits; ++s2) {
                        float y[EN];
                        floats_at<EN>(a.upart + s2 * a.rows * a.ad.kmax + line, kc + c * EN, in ? run.k : 0, y);
#pragma unroll
                        for (int e = 0; e < EN; ++e) x[e] += y[e];
                    }
                    if (c0 == 0 && in)
#pragma unroll
                        for (int e = 0; e < EN; ++e)
                            if (kc + c * EN + e < run.k) a.ad.u[line + kc + c * EN + e] = x[e];
                }
                char *at = lds + row * kStageBytes;
                if constexpr (sizeof(E) == 2) {
                    u32x4 h, l;
                    cut_chunk(x, h, l);
                    *reinterpret_cast<u32x4 *>(at + ((c ^ swz) << 4)) = h;
                    *reinterpret_cast<u32x4 *>(at + (((c + 4) ^ swz) << 4)) = l;
                } else {
                    *reinterpret_cast<f32x4 *>(at + ((c ^ swz) << 4)) = f32x4{x[0], x[1], x[2], x[3]};
                }
            }
            constexpr int TN = chunk_n<T>(), chunks = C::BN / TN;
            for (int q = threadIdx.x; q < 32 * chunks; q += C::THREADS) {
                const int k = q / chunks, c = q % chunks;
                u32x4 v = {0, 0, 0, 0};
                if (kc + k < run.k && c0 + c * TN < a.n) {
                    const int64_t e = (int64_t)(run.ko + kc + k) * a.n + c0 + c * TN;
                    v = chunk_at<T>((const char *)a.ad.up + e * (int64_t)sizeof(T), (a.ad.ktotal * a.n - e) * (int64_t)sizeof(T));
                }
                char *at = lq + k * (C::BN * (int)sizeof(E)) + ((c ^ rc_shift<E, C::BN>(k)) << 4);
                if constexpr (two_piece_matrix<T>()) {
                    float x[8];
                    u32x4 h, l;
                    floats_of(v, x, T{});
                    cut_chunk(x, h, l);
                    *reinterpret_cast<u32x4 *>(at) = h;
                    *reinterpret_cast<u32x4 *>(at + 32 * (C::BN * (int)sizeof(E))) = l;
                } else {
                    *reinterpret_cast<u32x4 *>(at) = v;
                }
            }
            meet();
            constexpr int KK = 32 / (2 * EN);         // matrix steps of 32 factors
#pragma unroll
            for (int i = 0; i < C::TM; ++i) {
                const int row = first + 32 * i + (lane & 31);
                const bool in = row >= from && row < to;
#pragma unroll
                for (int j = 0; j < C::TN; ++j) {
                    f32x16 d, low;                    // products of the first pieces, and of the others
#pragma unroll
                    for (int v = 0; v < 16; ++v) d[v] = low[v] = 0.f;
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
                        const u32x4 p = rp.read(lds, i, kk), q = rq.read(lq, j, kk);
                        if constexpr (Cut<T>::kBoth) {
                            if constexpr (two_piece_matrix<T>()) low = Type<E>::mac(rq.read(lq, j, kk + KK), p, low);
                            low = Type<E>::mac(q, rp.read(lds, i, kk + KK), low);
                        }
                        d = Type<E>::mac(q, p, d);
                    }
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[i][j][v] += in ? both_pieces<Cut<T>::kBoth>(d[v], low[v]) : 0.f;
                    __builtin_amdgcn_sched_barrier(0);      // one product's registers at a time
                }
            }
            meet();
        }
    }
}

template <class T> __device__ __forceinline__ Operand operand(const void *base, int64_t entry, int64_t ld, int64_t count, int64_t last)
{
    constexpr int E = sizeof(T);
    return Operand{(const char *)base + entry * E, ld * E, count, last * E};
}

// u (or a part of it) for one tile of a segment's rows: s_r x W_r.
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
    const Operand Q = operand<T>(a.ad.down, (run.ko + c0) * a.m, a.m, run.k - c0, (a.ad.ktotal - run.ko - c0) * a.m);
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

// Y, or parts of it over the contraction.  The first `shrink` workgroups form parts of u instead.
template <class C, class S, bool ADAPTERS> __global__ __launch_bounds__(C::THREADS) void product_kernel(Product a, int shrink)
{
    using T = typename C::T;
    constexpr bool both = ADAPTERS && S::THREADS == C::THREADS;
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
    C::multiply(P, Q, k0, k1, lds, acc);
    if (a.splits > 1) {
        const int64_t n4 = up4(a.n);
        C::store(acc, a.part + ((int64_t)split * a.rows + f.r0) * n4 + c0, n4, f.r1 - f.r0, a.n - c0, true, lds);
        return;
    }
    if constexpr (ADAPTERS) add_adapters<C>(a, f.r0, f.r1, c0, lds, acc);
    C::store(acc, (T *)a.y + f.r0 * a.ldy + c0, a.ldy, f.r1 - f.r0, a.n - c0, a.vec, lds);
}

// Y of one row and 1024 columns from the parts, in order, and its adapter.
template <class T> __global__ __launch_bounds__(256) void join_product_kernel(Product a)
{
    const int64_t row = blockIdx.y;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int64_t n4 = up4(a.n);
    __shared__ float us[kMaxRank];
    Run run = {0, 0};
    bool in = !a.offsets;
    if (a.offsets) {
        const int g = first_range(a.offsets, a.groups, row);
        if (g < a.groups) in = a.offsets[g] <= row;
        if (!in) return;
    }
    if (a.ad.segments) {
        const int s = first_range(a.ad.offsets, a.ad.segments, row);
        if (s < a.ad.segments && a.ad.offsets[s] <= row) run = run_of(a.ad, s);
        for (int k = threadIdx.x; k < run.k; k += 256) {
            float u;
            if (a.shrink_splits > 1) {
                u = 0.f;
                for (int s2 = 0; s2 < a.shrink_splits; ++s2) u += a.upart[((int64_t)s2 * a.rows + row) * a.ad.kmax + k];
                if (blockIdx.x == 0) a.ad.u[row * a.ad.kmax + k] = u;
            } else {
                u = a.ad.u[row * a.ad.kmax + k];
            }
            us[k] = u;
        }
        __syncthreads();
    }
    if (col >= a.n) return;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) y += *reinterpret_cast<const f32x4 *>(a.part + ((int64_t)s * a.rows + row) * n4 + col);
    const int have = a.n - col < 4 ? (int)(a.n - col) : 4;
    for (int k = 0; k < run.k; ++k) {
        const T *h = (const T *)a.ad.up + (int64_t)(run.ko + k) * a.n + col;
        const float u = us[k];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) y[e] = __builtin_fmaf(u, Type<T>::load(h[e]), y[e]);
    }
    T *out = (T *)a.y + row * a.ldy + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < have) out[e] = Type<T>::round(y[e]);
}

// dB_g = X_g^T dY_g, or parts of it over the group's rows.
template <class C> __global__ __launch_bounds__(C::THREADS) void gradient_kernel(Gradient a)
{
    using T = typename C::T;
    __shared__ __align__(1024) char lds[C::kLds];
    const int mt = (int)((a.m + C::BM - 1) / C::BM), nt = (int)((a.n + C::BN - 1) / C::BN);
    int id = by_die(blockIdx.x, gridDim.x);
    const int split = id % a.splits;
    id /= a.splits;
    const int g = id / (mt * nt);
    id -= g * mt * nt;
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

// Gradients of the factors of one run: BM of its factors x 128 columns of m or of n, summed over the rows of its segments,
// 64 (halves) or 32 (floats) rows at a time.
template <class T, int BM> __global__ __launch_bounds__(256) void factor_gradient_kernel(FactorGradient a)
{
    using E = typename Cut<T>::E;
    constexpr int BN = 128, SK = stage_k<E>();
    constexpr bool two = two_piece_matrix<T>(), both = Cut<T>::kBoth;
    constexpr int kP = SK * BM * (int)sizeof(E), kQ = SK * BN * (int)sizeof(E);
    constexpr int TM = BM / 32;
    __shared__ __align__(1024) char lds[kP * (both ? 2 : 1) + kQ * (two ? 2 : 1)];
    char *lp = lds, *lq = lds + kP * (both ? 2 : 1);

    const int mt = (int)((a.m + BN - 1) / BN);
    const bool down = (int)blockIdx.x < mt;                // dW: from v and X; dH: from u and dY
    const int64_t width = down ? a.m : a.n, c0 = (int64_t)(down ? blockIdx.x : blockIdx.x - mt) * BN;
    const char *src = (const char *)(down ? a.x : a.dy);
    const int64_t ld = down ? a.ldx : a.ldy;
    const float *fac = down ? a.v : a.u;
    const int kt = (a.ad.kmax + BM - 1) / BM;
    const int id = blockIdx.y / kt, f0 = blockIdx.y % kt * BM;
    const int split = blockIdx.z;
    const int64_t klo = a.ad.koff[id], khi = a.ad.koff[id + 1];
    if (klo < 0 || khi <= klo || klo >= a.ad.ktotal) return;
    int64_t k = (khi < a.ad.ktotal ? khi : a.ad.ktotal) - klo;
    const int64_t mine = k - f0;                            // factors of this workgroup and behind it
    if (mine <= 0) return;
    if (k > a.ad.kmax) k = a.ad.kmax;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Reader<E, BM, true> rp;
    Reader<E, BN, true> rq;
    rp.open(0);
    rq.open(wave * 32);
    f32x16 acc[TM], low[TM];                               // products of the first pieces, and of the others
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][v] = low[i][v] = 0.f;

    constexpr int EN = chunk_n<E>(), TE = chunk_n<T>();
    constexpr int pc = BM / EN, PJ = SK * pc / 256, qc = BN / TE, QJ = SK * qc / 256;
    int turn = 0;
    for (int base = 0; base < a.ad.segments; base += 64) {
        int64_t lo = 0, hi = 0;
        bool is = false;
        if (base + lane < a.ad.segments) {
            range_of(a.ad.offsets, base + lane, a.rows, lo, hi);
            is = a.ad.run[base + lane] == id && hi > lo;
        }
        unsigned long long todo = __ballot(is);
        while (todo) {
            const int l = __ffsll(todo) - 1;
            todo &= todo - 1;
            const int64_t slo = __shfl(lo, l), shi = __shfl(hi, l);
            for (int64_t r = slo; r < shi; r += SK) {
                if (turn++ % a.splits != split) continue;
                const int64_t left = shi - r;
                u32x4 ph[PJ], pl[PJ], qv[QJ];
#pragma unroll
                for (int j = 0; j < PJ; ++j) {
                    const int q = threadIdx.x + 256 * j, kr = q / pc, c = q % pc;
                    float x[EN];
                    floats_at<EN>(fac + (r + (kr < left ? kr : 0)) * a.ad.kmax, f0 + c * EN, kr < left ? (int)k : 0, x);
                    if constexpr (both) cut_chunk(x, ph[j], pl[j]);
                    else ph[j] = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
                }
#pragma unroll
                for (int j = 0; j < QJ; ++j) {
                    const int q = threadIdx.x + 256 * j, kr = q / qc, c = q % qc;
                    qv[j] = u32x4{0, 0, 0, 0};
                    if (kr < left && c0 + c * TE < width) {
                        const int64_t e = (r + kr) * ld + c0 + c * TE;
                        qv[j] = chunk_at<T>(src + e * (int64_t)sizeof(T), ((a.rows - 1) * ld + width - e) * (int64_t)sizeof(T));
                    }
                }
                meet();                 // the last stage has been read
#pragma unroll
                for (int j = 0; j < PJ; ++j) {
                    const int q = threadIdx.x + 256 * j, kr = q / pc, c = q % pc;
                    char *at = lp + kr * (BM * (int)sizeof(E)) + ((c ^ rc_shift<E, BM>(kr)) << 4);
                    *reinterpret_cast<u32x4 *>(at) = ph[j];
                    if constexpr (both) *reinterpret_cast<u32x4 *>(at + kP) = pl[j];
                }
#pragma unroll
                for (int j = 0; j < QJ; ++j) {
                    const int q = threadIdx.x + 256 * j, kr = q / qc, c = q % qc;
                    char *at = lq + kr * (BN * (int)sizeof(E)) + ((c ^ rc_shift<E, BN>(kr)) << 4);
                    if constexpr (two) {
                        float x[8];
                        u32x4 h, w;
                        floats_of(qv[j], x, T{});
                        cut_chunk(x, h, w);
                        *reinterpret_cast<u32x4 *>(at) = h;
                        *reinterpret_cast<u32x4 *>(at + kQ) = w;
                    } else {
                        *reinterpret_cast<u32x4 *>(at) = qv[j];
                    }
                }
                meet();
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    const u32x4 q = rq.read(lq, 0, kk);
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        const u32x4 p = rp.read(lp, i, kk);
                        if constexpr (both) {
                            if constexpr (two) low[i] = Type<E>::mac(rq.read(lq + kQ, 0, kk), p, low[i]);
                            low[i] = Type<E>::mac(q, rp.read(lp + kP, i, kk), low[i]);
                        }
                        acc[i] = Type<E>::mac(q, p, acc[i]);
                    }
                }
            }
        }
    }
    const int64_t m4 = up4(a.m), n4 = up4(a.n);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = 32 * i + (lane & 31);
        if (row >= mine) continue;
        const bool real = f0 + row < k;                     // factors beyond kmax take no part: zero
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int64_t col = c0 + 32 * wave + acc_row(v, lane >> 5);
            if (col >= width) continue;
            const float x = real ? both_pieces<both>(acc[i][v], low[i][v]) : 0.f;
            const int64_t line = klo + f0 + row;
            if (a.splits > 1) {
                float *o = down ? a.part + ((int64_t)split * a.ad.ktotal + line) * m4
                                : a.part + (int64_t)a.splits * a.ad.ktotal * m4 + ((int64_t)split * a.ad.ktotal + line) * n4;
                o[col] = x;
            } else {
                ((T *)(down ? a.ddown : a.dup))[line * width + col] = Type<T>::round(x);
            }
        }
    }
}

// ---- launches --------------------------------------------------------------------------

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
    case 0: go(Tile<T, 256, 256, 2, 4, 2, false, QRC, DMA>{}); break;
    case 1: go(Tile<T, 128, 128, 2, 2, 2, false, QRC, DMA>{}); break;
    case 2: go(Tile<T, 64, 128, 1, 4, 3, false, QRC, DMA>{}); break;
    default: go(Tile<T, 32, 128, 1, 4, 4, false, QRC, DMA>{}); break;
    }
}

inline bool by16(const void *p, int64_t a = 0, int64_t b = 0) { return (((uintptr_t)p | (uint64_t)a | (uint64_t)b) & 15) == 0; }

template <class T> hipError_t launch_product(const Product &p, hipStream_t st)
{
    constexpr int E = sizeof(T);
    const int64_t far = (int64_t)1 << 30;
    bool dma = by16(p.x, p.ldx * E, p.m * E) && by16(p.b, p.ldb * E, p.stride_b * E) && p.ldx * E * 256 < far && p.ldb * E * 256 < far;
    if (p.transposed == 0) dma = dma && p.n * E % 16 == 0;
    if (p.ad.segments) dma = dma && by16(p.ad.down);
    using ShrinkDma = Tile<T, kShrinkRows, kShrinkCols, 2, 2, 4, false, false, true>;
    using Shrink = Tile<T, kShrinkRows, kShrinkCols, 2, 2, 4, false, false, false>;
    int shrink = 0;
    if (p.ad.segments) {
        const int64_t rt = (p.rows + kShrinkRows - 1) / kShrinkRows + p.ad.segments, ct = (p.ad.kmax + kShrinkCols - 1) / kShrinkCols;
        shrink = (int)(rt * ct * p.shrink_splits);
        if (p.splits == 1) {
            if (dma) hipLaunchKernelGGL((shrink_kernel<ShrinkDma>), dim3(shrink), dim3(ShrinkDma::THREADS), 0, st, p);
            else hipLaunchKernelGGL((shrink_kernel<Shrink>), dim3(shrink), dim3(Shrink::THREADS), 0, st, p);
            shrink = 0;
        }
    }
    if (p.transposed) {
        if (dma) launch_shape<T, false, true>(p, shrink, st);
        else launch_shape<T, false, false>(p, shrink, st);
    } else {
        if (dma) launch_shape<T, true, true>(p, shrink, st);
        else launch_shape<T, true, false>(p, shrink, st);
    }
    if (p.splits > 1)
        hipLaunchKernelGGL((join_product_kernel<T>), dim3((unsigned)((p.n + 1023) / 1024), (unsigned)p.rows), dim3(256), 0, st, p);
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
    const bool dma = by16(p.x, p.ldx * E, p.m * E) && by16(p.dy, p.ldy * E, p.n * E) && p.ldx * E * 64 < far && p.ldy * E * 64 < far;
    auto go = [&](auto tile) {
        using C = decltype(tile);
        const int64_t tiles = (p.m + C::BM - 1) / C::BM * ((p.n + C::BN - 1) / C::BN) * p.groups * p.splits;
        hipLaunchKernelGGL((gradient_kernel<C>), dim3((unsigned)tiles), dim3(C::THREADS), 0, st, p);
    };
    if (p.shape == 0) {
        if (dma) go(Tile<T, 256, 256, 2, 4, 2, true, true, true>{});
        else go(Tile<T, 256, 256, 2, 4, 2, true, true, false>{});
    } else {
        if (dma) go(Tile<T, 128, 128, 2, 2, 2, true, true, true>{});
        else go(Tile<T, 128, 128, 2, 2, 2, true, true, false>{});
    }
    if (p.splits > 1)
        launch_join<T>(p.part, p.splits, (int64_t)p.groups * p.m, p.n, (T *)p.g, p.m, p.stride_g, p.ldg, st);
    return hipGetLastError();
}

template <class T> hipError_t launch_factor_gradient(const FactorGradient &p, hipStream_t st)
{
    const unsigned cols = (unsigned)((p.m + 127) / 128 + (p.n + 127) / 128);
    if (p.ad.kmax <= 32)
        hipLaunchKernelGGL((factor_gradient_kernel<T, 32>), dim3(cols, (unsigned)p.ad.runs, p.splits), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((factor_gradient_kernel<T, 64>), dim3(cols, (unsigned)(p.ad.runs * ((p.ad.kmax + 63) / 64)), p.splits), dim3(256), 0,
                           st, p);
    if (p.splits > 1) {
        launch_join<T>(p.part, p.splits, p.ad.ktotal, p.m, (T *)p.ddown, p.ad.ktotal, 0, p.m, st);
        launch_join<T>(p.part + (int64_t)p.splits * p.ad.ktotal * up4(p.m), p.splits, p.ad.ktotal, p.n, (T *)p.dup, p.ad.ktotal, 0, p.n, st);
    }
    return hipGetLastError();
}

}  // namespace ragged
}  // namespace nmfmu
