// Rows to their groups: choices, gates, the groups' offsets, places, balance; and the logits' gradient.
#include "nmfmu_routed_device.h"

#include <algorithm>
#include <type_traits>

namespace nmfmu {
namespace routed {

namespace {

constexpr int kThreads = 256;

// Logits as integers in the order that rows choose by: larger first, then the lower group.  0: never chosen.
__device__ __forceinline__ unsigned order_of(float x)
{
    const unsigned b = __float_as_uint(x);
    if (!(x > -__builtin_inff())) return 0;                  // -infinity and NaN
    if (x == 0.f) return 0x80000000u;                        // both zeros are equal
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// One row's logits, G of them, C neighbouring ones to each of W lanes.
template <class T, int W, int C> struct Logits {
    float x[C];
    int first;       // group of x[0]

    __device__ __forceinline__ void load(const T *row, int groups, bool is)
    {
        first = (int)(threadIdx.x % W) * C;
#pragma unroll
        for (int c = 0; c < C; ++c) x[c] = -__builtin_inff();
        if (!is) return;
        if (first + C <= groups) {
            T t[C];
            __builtin_memcpy(t, row + first, sizeof(t));
#pragma unroll
            for (int c = 0; c < C; ++c) x[c] = Type<T>::load(t[c]);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (first + c < groups) x[c] = Type<T>::load(row[first + c]);
        }
    }
    // x becomes exp(x - most); returns the sum over the row (NaN where the row holds a NaN or +infinity; rows of -infinity
    // alone are not asked).
    __device__ __forceinline__ float exponents()
    {
        float most = x[0];
#pragma unroll
        for (int c = 1; c < C; ++c) most = __builtin_fmaxf(most, x[c]);
#pragma unroll
        for (int d = 1; d < W; d <<= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d));
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[c] = expf(x[c] - most);
            sum += x[c];
        }
        return sum_of<W>(sum);
    }
};

// Choices of up to kRouteRows rows from `base` on: choice and gate to memory, which rows chose a group to `mask` (a bit for
// each row, zeroed before), c_r p_rg summed over the thread's rows to share[].
template <class T, int W, int C>
__device__ __forceinline__ void choose(const Route &a, int64_t base, unsigned long long *mask, float (&share)[C])
{
    constexpr int ROWS = kThreads / W;
    const int lane = threadIdx.x % W;
#pragma unroll
    for (int r = 0; r < kRouteRows / ROWS; ++r) {
        const int in = r * ROWS + threadIdx.x / W;
        const int64_t row = base + in;
        const bool is = row < a.rows;
        if (base + r * ROWS >= a.rows) break;
        Logits<T, W, C> l;
        l.load((const T *)a.logits + row * a.ldl, a.groups, is);
        unsigned key[C];
#pragma unroll
        for (int c = 0; c < C; ++c) key[c] = order_of(l.x[c]);
        const float sum = l.exponents();
        // the largest key of all that is left, and of equals the lowest group
        int mine = 0;
        float total = 0.f;
        constexpr int N = W < NMF_ROUTE_MAX_K ? NMF_ROUTE_MAX_K / W : 1;      // lane j % W keeps choice j
        float gate[N];
        int choice[N];
#pragma unroll
        for (int n = 0; n < N; ++n) gate[n] = 0.f, choice[n] = -1;
        for (int j = 0; j < a.k; ++j) {
            unsigned best = key[0];
            int at = 0;
#pragma unroll
            for (int c = 1; c < C; ++c)
                if (key[c] > best) best = key[c], at = c;
            int group = l.first + at;
#pragma unroll
            for (int d = 1; d < W; d <<= 1) {
                const unsigned o = (unsigned)__shfl_xor((int)best, d);
                const int g = __shfl_xor(group, d);
                if (o > best || (o == best && g < group)) best = o, group = g;
            }
            if (best == 0) break;
            float e = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (l.first + c == group) key[c] = 0, e = l.x[c];
            const float p = __shfl(e, group / C, W) / sum;
            total += p;
            ++mine;
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (j == lane + n * W) gate[n] = p, choice[n] = group;
        }
        if (is) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int j = lane + n * W, g = choice[n];
                if (j >= a.k) continue;
                a.choice[row * a.k + j] = g;
                a.gate[row * a.k + j] = g >= 0 && a.normalise ? gate[n] / total : gate[n];
                if (g >= 0) atomicOr(&mask[g], 1ull << in);
            }
            if (mine) {
#pragma unroll
                for (int c = 0; c < C; ++c) share[c] += (float)mine * (l.x[c] / sum);
            }
        }
    }
}

// share[] of a workgroup's threads, added in order, to out[groups].
template <int W, int C> __device__ __forceinline__ void add_share(const float (&share)[C], int groups, float *lds, float *out)
{
    constexpr int ROWS = kThreads / W;
#pragma unroll
    for (int c = 0; c < C; ++c) lds[threadIdx.x * C + c] = share[c];
    __syncthreads();
    for (int g = threadIdx.x; g < groups; g += kThreads) {
        float x = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) x += lds[(r * W + g / C) * C + g % C];
        out[g] = x;
    }
}

// Sums before each entry of `count` (up to 1024) to `before`, by the whole workgroup; returns the sum of all.
__device__ __forceinline__ int64_t sums_before(const int64_t *count, int n, int64_t *before, int64_t *meet)
{
    constexpr int E = NMF_ROUTE_MAX_GROUPS / kThreads;
    int64_t x[E], sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int at = threadIdx.x * E + e;
        x[e] = at < n ? count[at] : 0;
        sum += x[e];
    }
    int64_t up = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(up, d);
        if ((int)(threadIdx.x & 63) >= d) up += o;
    }
    if ((threadIdx.x & 63) == 63) meet[threadIdx.x / 64] = up;
    __syncthreads();
    int64_t base = up - sum, all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < (int)(threadIdx.x / 64)) base += meet[w];
        all += meet[w];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int at = threadIdx.x * E + e;
        if (at < n) before[at] = base;
        base += x[e];
    }
    __syncthreads();
    return all;
}

// groups * sum of count / C * mass / C, by the whole workgroup.
template <class M> __device__ __forceinline__ double balance_of(const int64_t *count, const M *mass, int groups, int64_t all, double *meet)
{
    double x = 0.;
    for (int g = threadIdx.x; g < groups; g += kThreads) x += (double)count[g] * (double)mass[g];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.;
    for (int w = 0; w < kThreads / 64; ++w) x += meet[w];
    return all ? x * groups / ((double)all * (double)all) : 0.;
}

}  // namespace

// All rows by one workgroup: for few rows, and for calls without scratch.  Places are first those within the group.
template <class T, int W, int C> __global__ __launch_bounds__(kThreads) void route_one_kernel(Route a)
{
    constexpr int G = W * C;
    __shared__ unsigned long long mask[G];
    __shared__ int64_t count[G], before[G], meet[kThreads / 64];
    __shared__ double mass[G], meet_d[kThreads / 64];
    __shared__ float lds[kThreads * C], part[G];
    for (int g = threadIdx.x; g < a.groups; g += kThreads) count[g] = 0, mass[g] = 0.;
    for (int64_t base = 0; base < a.rows; base += kRouteRows) {
        for (int g = threadIdx.x; g < a.groups; g += kThreads) mask[g] = 0;
        __syncthreads();
        float share[C];
#pragma unroll
        for (int c = 0; c < C; ++c) share[c] = 0.f;
        choose<T, W, C>(a, base, mask, share);
        __syncthreads();
        add_share<W, C>(share, a.groups, lds, part);
        const int64_t here = std::min<int64_t>(kRouteRows, a.rows - base) * a.k;
        for (int64_t i = threadIdx.x; i < here; i += kThreads) {
            const int g = a.choice[base * a.k + i];
            a.place[base * a.k + i] = g < 0 ? -1 : (int)(count[g] + __popcll(mask[g] & ((1ull << (i / a.k)) - 1)));
        }
        __syncthreads();
        for (int g = threadIdx.x; g < a.groups; g += kThreads) {
            count[g] += __popcll(mask[g]);
            mass[g] += part[g];
        }
    }
    __syncthreads();
    const int64_t all = sums_before(count, a.groups, before, meet);
    for (int64_t i = threadIdx.x; i < a.rows * a.k; i += kThreads) {
        const int g = a.choice[i];
        if (g >= 0) a.place[i] += (int)before[g];
    }
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.offsets[g] = before[g];
    const double b = balance_of(count, mass, a.groups, all, meet_d);
    if (threadIdx.x == 0) {
        a.offsets[a.groups] = all;
        a.balance[0] = (float)b;
    }
}

// Blocks of kRouteRows rows: choices, gates, places within the block's part of a group, counts and shares of the block.
template <class T, int W, int C> __global__ __launch_bounds__(kThreads) void route_rows_kernel(Route a)
{
    __shared__ unsigned long long mask[W * C];
    __shared__ float lds[kThreads * C];
    for (int g = threadIdx.x; g < a.groups; g += kThreads) mask[g] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kRouteRows;
    float share[C];
#pragma unroll
    for (int c = 0; c < C; ++c) share[c] = 0.f;
    choose<T, W, C>(a, base, mask, share);
    __syncthreads();
    add_share<W, C>(share, a.groups, lds, a.share + (int64_t)blockIdx.x * a.groups);
    const int64_t here = std::min<int64_t>(kRouteRows, a.rows - base) * a.k;
    for (int64_t i = threadIdx.x; i < here; i += kThreads) {
        const int g = a.choice[base * a.k + i];
        a.place[base * a.k + i] = g < 0 ? -1 : __popcll(mask[g] & ((1ull << (i / a.k)) - 1));
    }
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.count[(int64_t)blockIdx.x * a.groups + g] = __popcll(mask[g]);
}

// Counts of a group in all blocks to sums before each block: a group to each column of 16 threads' rows.
__global__ __launch_bounds__(kThreads) void route_sums_kernel(Route a)
{
    __shared__ int64_t sums[16][17];
    __shared__ double masses[16][17];
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4, g = blockIdx.x * 16 + c;
    const int64_t each = (a.blocks + 15) / 16, b0 = r * each, b1 = std::min<int64_t>(b0 + each, a.blocks);
    int64_t sum = 0;
    double mass = 0.;
    if (g < a.groups)
        for (int64_t b = b0; b < b1; ++b) {
            sum += a.count[b * a.groups + g];
            mass += (double)a.share[b * a.groups + g];
        }
    sums[r][c] = sum;
    masses[r][c] = mass;
    __syncthreads();
    if (g >= a.groups) return;
    int64_t before = 0, all = 0;
    mass = 0.;
    for (int i = 0; i < 16; ++i) {
        if (i < r) before += sums[i][c];
        all += sums[i][c];
        mass += masses[i][c];
    }
    for (int64_t b = b0; b < b1; ++b) {
        const int64_t at = b * a.groups + g;
        const int n = a.count[at];
        a.count[at] = (int)before;
        before += n;
    }
    if (r == 0) {
        a.total[g] = all;
        a.mass[g] = mass;
    }
}

__global__ __launch_bounds__(kThreads) void route_place_kernel(Route a)
{
    __shared__ int64_t before[NMF_ROUTE_MAX_GROUPS], meet[kThreads / 64];
    __shared__ double meet_d[kThreads / 64];
    const int64_t all = sums_before(a.total, a.groups, before, meet);
    const int64_t base = (int64_t)blockIdx.x * kRouteRows;
    const int64_t here = std::min<int64_t>(kRouteRows, a.rows - base) * a.k;
    for (int64_t i = threadIdx.x; i < here; i += kThreads) {
        const int g = a.choice[base * a.k + i];
        if (g >= 0) a.place[base * a.k + i] += (int)before[g] + a.count[(int64_t)blockIdx.x * a.groups + g];
    }
    if (blockIdx.x) return;
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.offsets[g] = before[g];
    const double b = balance_of(a.total, a.mass, a.groups, all, meet_d);
    if (threadIdx.x == 0) {
        a.offsets[a.groups] = all;
        a.balance[0] = (float)b;
    }
}

// f(lanes of a row, groups of a lane) for so many groups.
template <class F> void by_groups(int groups, F f)
{
    using std::integral_constant;
    if (groups <= 32) f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
    else if (groups <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (groups <= 128) f(integral_constant<int, 32>{}, integral_constant<int, 4>{});
    else if (groups <= 256) f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (groups <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <class T> hipError_t launch_route(const Route &a, hipStream_t st)
{
    by_groups(a.groups, [&](auto w, auto c) {
        constexpr int W = w.value, C = c.value;
        if (!a.count) {
            hipLaunchKernelGGL((route_one_kernel<T, W, C>), dim3(1), dim3(kThreads), 0, st, a);
            return;
        }
        hipLaunchKernelGGL((route_rows_kernel<T, W, C>), dim3((unsigned)a.blocks), dim3(kThreads), 0, st, a);
        hipLaunchKernelGGL(route_sums_kernel, dim3((unsigned)((a.groups + 15) / 16)), dim3(kThreads), 0, st, a);
        hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)a.blocks), dim3(kThreads), 0, st, a);
    });
    return hipGetLastError();
}

// ---- gradient of the logits ------------------------------------------------------------------
template <class T, int W, int C> __global__ __launch_bounds__(kThreads) void route_gradient_kernel(RouteGradient a)
{
    constexpr int ROWS = kThreads / W;
    const int first = (int)(threadIdx.x % W) * C;
    float q[C];                                   // d balance / d p_rg, but for c_r
    {
        const int64_t all = a.offsets[a.groups];
        const float up = a.dbalance && all > 0 ? a.dbalance[0] : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            q[c] = 0.f;
            if (a.dbalance && all > 0 && first + c < a.groups)
                q[c] = up * (float)((double)a.groups * (double)(a.offsets[first + c + 1] - a.offsets[first + c]) / ((double)all * (double)all));
        }
    }
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < a.rows; base += (int64_t)gridDim.x * ROWS) {
        const int64_t row = base + threadIdx.x / W;
        const bool is = row < a.rows;
        Logits<T, W, C> l;
        l.load((const T *)a.logits + row * a.ldl, a.groups, is);
        const float sum = l.exponents();
        float d[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            l.x[c] /= sum;                        // p
            d[c] = 0.f;
        }
        // the lane's own groups among the row's choices
        int mine = 0;
        float total = 0.f, dot = 0.f;             // sums over the choices of p and of p dgate
        for (int j = 0; j < a.k; ++j) {
            const int g = is ? a.choice[row * a.k + j] : -1;
            if (g < 0 || g >= a.groups) continue;
            ++mine;
            const float dg = a.dgate ? a.dgate[row * a.k + j] : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (first + c == g) {
                    total += l.x[c];
                    dot = __builtin_fmaf(l.x[c], dg, dot);
                    d[c] = 1.f;
                }
        }
        total = sum_of<W>(total);
        dot = sum_of<W>(dot);
        float mean = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) mean = __builtin_fmaf(l.x[c], q[c], mean);
        mean = sum_of<W>(mean);
        if (!is) continue;
        // p_i ([i chosen] dg_i - dot), or, normalised, p_i / total (dg_i - dot / total) of the chosen
        const float share = a.normalise ? 1.f / total : 1.f, less = a.normalise ? dot / total : dot;
        float out[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            out[c] = (float)mine * (q[c] - mean);
            if (!a.normalise) out[c] -= less;
            else if (d[c] != 0.f) out[c] -= less * share;
        }
        if (a.dgate)
            for (int j = 0; j < a.k; ++j) {
                const int g = a.choice[row * a.k + j];
                const float dg = a.dgate[row * a.k + j];
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (first + c == g) out[c] = __builtin_fmaf(dg, share, out[c]);
            }
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (first + c < a.groups) ((T *)a.dlogits)[row * a.lddl + first + c] = Type<T>::round(mine ? l.x[c] * out[c] : 0.f);
    }
}

template <class T> hipError_t launch_route_gradient(const RouteGradient &a, hipStream_t st)
{
    by_groups(a.groups, [&](auto w, auto c) {
        constexpr int W = w.value, C = c.value, rows = kThreads / W;
        hipLaunchKernelGGL((route_gradient_kernel<T, W, C>), dim3((unsigned)std::min<int64_t>((a.rows + rows - 1) / rows, 2048)), dim3(kThreads), 0, st, a);
    });
    return hipGetLastError();
}

#define NMFMU_ROUTE(T)                                            \
    template hipError_t launch_route<T>(const Route &, hipStream_t); \
    template hipError_t launch_route_gradient<T>(const RouteGradient &, hipStream_t);
NMFMU_ROUTE(float)
NMFMU_ROUTE(bf16_t)
NMFMU_ROUTE(f16_t)

}  // namespace routed
}  // namespace nmfmu
