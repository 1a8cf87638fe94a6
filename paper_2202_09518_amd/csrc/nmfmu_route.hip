// Rows to their groups: choices, gates, the groups' offsets, places, balance; and the logits' gradient.
#include "nmfmu_routed_device.h"

#include <algorithm>
#include <type_traits>

namespace nmfmu {
namespace routed {

namespace {

constexpr int kThreads = 1024;      // of a block of rows: a compute unit's worth, as choices follow each other and wait for lanes
constexpr int kFew = 256;           // of what comes behind

// Logits as integers in the order that rows choose by.  0: never chosen.
__device__ __forceinline__ unsigned order_of(float x)
{
    const unsigned b = __float_as_uint(x);
    if (!(x > -__builtin_inff())) return 0;                  // -infinity and NaN
    if (x == 0.f) return 0x80000000u;                        // both zeros are equal
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The largest key of all that is left in a row, and the lowest group that has it; 0 if nothing is left.  A lane's own groups are
// first, first + 1, ...  Keys of 16 bits take their group along in the lower half, the lower group above the higher: one maximum
// over the lanes finds both.
template <class T, int W, int C> struct Keys {
    static constexpr bool kBoth = sizeof(T) == 2;
    unsigned key[C];

    __device__ __forceinline__ void open(const float (&x)[C], int first)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            key[c] = order_of(x[c]);
            if (kBoth && key[c]) {
                unsigned top = key[c];      // of bf16 the upper half is all there is; of a half its own bits are taken the same way
                if (std::is_same<T, f16_t>::value) {
                    const unsigned h = (unsigned)__builtin_bit_cast(unsigned short, (_Float16)x[c]) << 16;
                    top = top == 0x80000000u ? top : (h & 0x80000000u ? ~h : h | 0x80000000u);
                }
                key[c] = (top & 0xffff0000u) | (unsigned)(0xffff - first - c);
            }
        }
    }
    __device__ __forceinline__ unsigned most(int first, int &group) const
    {
        unsigned best = key[0];
#pragma unroll
        for (int c = 1; c < C; ++c) best = key[c] > best ? key[c] : best;
        best = most_of<W>(best);
        if (kBoth) {
            group = 0xffff - (int)(best & 0xffff);
        } else {
            unsigned at = ~0u;
#pragma unroll
            for (int c = C - 1; c >= 0; --c) at = key[c] == best ? (unsigned)(first + c) : at;
            group = (int)least_of<W>(at);
        }
        return best;
    }
    // Whether a lane's group c is the one that was found; it is taken out.
    __device__ __forceinline__ bool take(int c, unsigned best, int group, int first)
    {
        const bool is = kBoth ? key[c] == best : first + c == group;
        key[c] = is ? 0 : key[c];
        return is;
    }
};

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
        most = most_of<W>(most);
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[c] = expf(x[c] - most);
            sum += x[c];
        }
        return sum_of<W>(sum);
    }
};

// Choices of up to `each` rows from `base` on: choice and gate to memory, choice to `picked` too, which rows chose a group to
// `mask` (a bit for each row, zeroed before), c_r p_rg summed over the thread's rows to share[].
template <class T, int W, int C>
__device__ __forceinline__ void choose(const Route &a, int64_t base, int each, unsigned long long *mask, int *picked, float (&share)[C])
{
    constexpr int ROWS = kThreads / W;
    const int lane = threadIdx.x % W;
    for (int r = 0; r * ROWS < each; ++r) {
        const int in = r * ROWS + threadIdx.x / W;
        const int64_t row = base + in;
        const bool is = row < a.rows && in < each;
        if (base + r * ROWS >= a.rows) break;
        Logits<T, W, C> l;
        l.load((const T *)a.logits + row * a.ldl, a.groups, is);
        Keys<T, W, C> keys;
        keys.open(l.x, l.first);
        const float one = 1.f / l.exponents();
        int mine = 0;
        float total = 0.f;
        constexpr int N = W < NMF_ROUTE_MAX_K ? NMF_ROUTE_MAX_K / W : 1;      // lane j % W keeps choice j
        float gate[N];
        int choice[N];
#pragma unroll
        for (int n = 0; n < N; ++n) gate[n] = 0.f, choice[n] = -1;
        for (int j = 0; j < a.k; ++j) {
            int group;
            const unsigned best = keys.most(l.first, group);
            if (best == 0) break;
            float e = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (keys.take(c, best, group, l.first)) e = l.x[c];
            const float p = __shfl(e, group / C, W) * one;
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
                picked[in * a.k + j] = g;
                a.gate[row * a.k + j] = g >= 0 && a.normalise ? gate[n] / total : gate[n];
                if (g >= 0) atomicOr(&mask[g], 1ull << in);
            }
            if (mine) {
#pragma unroll
                for (int c = 0; c < C; ++c) share[c] += (float)mine * (l.x[c] * one);
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
template <int THREADS> __device__ __forceinline__ int64_t sums_before(const int64_t *count, int n, int64_t *before, int64_t *meet)
{
    constexpr int E = NMF_ROUTE_MAX_GROUPS / THREADS;
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
    for (int w = 0; w < THREADS / 64; ++w) {
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
template <int THREADS> __device__ __forceinline__ double balance_of(const int64_t *count, const double *mass, int groups, int64_t all, double *meet)
{
    double x = 0.;
    for (int g = threadIdx.x; g < groups; g += THREADS) x += (double)count[g] * mass[g];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.;
    for (int w = 0; w < THREADS / 64; ++w) x += meet[w];
    return all ? x * groups / ((double)all * (double)all) : 0.;
}

}  // namespace

// Place of choice i of a block within the block's part of its group.
__device__ __forceinline__ int place_in(const unsigned long long *mask, int g, int row) { return __popcll(mask[g] & ((1ull << row) - 1)); }

// All rows by one workgroup: for few rows, and for calls without scratch.  With more than one block of rows, places are first those
// within the group.
template <class T, int W, int C> __global__ __launch_bounds__(kThreads) void route_one_kernel(Route a)
{
    constexpr int G = W * C;
    __shared__ unsigned long long mask[G];
    __shared__ int64_t count[G], before[G], meet[kThreads / 64];
    __shared__ double mass[G], meet_d[kThreads / 64];
    __shared__ float lds[kThreads * C], part[G];
    __shared__ int picked[kRouteRows * NMF_ROUTE_MAX_K];
    const bool several = a.rows > kRouteRows;
    for (int g = threadIdx.x; g < a.groups; g += kThreads) count[g] = 0, mass[g] = 0.;
    for (int64_t base = 0; base < a.rows; base += kRouteRows) {
        for (int g = threadIdx.x; g < a.groups; g += kThreads) mask[g] = 0;
        __syncthreads();
        float share[C];
#pragma unroll
        for (int c = 0; c < C; ++c) share[c] = 0.f;
        choose<T, W, C>(a, base, kRouteRows, mask, picked, share);
        add_share<W, C>(share, a.groups, lds, part);
        if (several) {
            const int here = (int)std::min<int64_t>(kRouteRows, a.rows - base) * a.k;
            for (int i = threadIdx.x; i < here; i += kThreads) {
                const int g = picked[i];
                a.place[base * a.k + i] = g < 0 ? -1 : (int)count[g] + place_in(mask, g, i / a.k);
            }
        }
        __syncthreads();
        for (int g = threadIdx.x; g < a.groups; g += kThreads) {
            count[g] += __popcll(mask[g]);
            mass[g] += part[g];
        }
    }
    __syncthreads();
    const int64_t all = sums_before<kThreads>(count, a.groups, before, meet);
    for (int64_t i = threadIdx.x; i < a.rows * a.k; i += kThreads) {
        const int g = several ? a.choice[i] : picked[i];
        if (!several) a.place[i] = g < 0 ? -1 : (int)before[g] + place_in(mask, g, (int)i / a.k);
        else if (g >= 0) a.place[i] += (int)before[g];
    }
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.offsets[g] = before[g];
    const double b = balance_of<kThreads>(count, mass, a.groups, all, meet_d);
    if (threadIdx.x == 0) {
        a.offsets[a.groups] = all;
        a.balance[0] = (float)b;
    }
}

// (16384 rows to 8 of 128 groups, bf16: 9.0 us for the choices, 4.0 for the sums of the blocks, 3.4 for the places; instructions
// bound the choices, 50 of them for each, and launches the rest.  24 rows of 64 floats to 4 groups, by one workgroup: 5.8 us.)
// Blocks of a.each rows: choices, gates, places within the block's part of a group, counts and shares of the block.
template <class T, int W, int C> __global__ __launch_bounds__(kThreads) void route_rows_kernel(Route a)
{
    __shared__ unsigned long long mask[W * C];
    __shared__ float lds[kThreads * C];
    __shared__ int picked[kRouteRows * NMF_ROUTE_MAX_K];
    for (int g = threadIdx.x; g < a.groups; g += kThreads) mask[g] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * a.each;
    float share[C];
#pragma unroll
    for (int c = 0; c < C; ++c) share[c] = 0.f;
    choose<T, W, C>(a, base, a.each, mask, picked, share);
    add_share<W, C>(share, a.groups, lds, a.share + (int64_t)blockIdx.x * a.groups);
    const int here = (int)std::min<int64_t>(a.each, a.rows - base) * a.k;
    for (int i = threadIdx.x; i < here; i += kThreads) {
        const int g = picked[i];
        a.place[base * a.k + i] = g < 0 ? -1 : place_in(mask, g, i / a.k);
    }
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.count[(int64_t)blockIdx.x * a.groups + g] = __popcll(mask[g]);
}

// Counts of a group in all blocks to the sums before each block: 16 groups to a workgroup, 64 runs of blocks to each.
__global__ __launch_bounds__(1024) void route_sums_kernel(Route a)
{
    constexpr int RUNS = 64;
    __shared__ int sums[RUNS][17];
    __shared__ double masses[RUNS][17];
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4, g = blockIdx.x * 16 + c;
    const int64_t each = (a.blocks + RUNS - 1) / RUNS, b0 = r * each, b1 = std::min<int64_t>(b0 + each, a.blocks);
    int sum = 0;
    double mass = 0.;
    if (g < a.groups)
#pragma unroll 4
        for (int64_t b = b0; b < b1; ++b) {
            sum += a.count[b * a.groups + g];
            mass += (double)a.share[b * a.groups + g];
        }
    sums[r][c] = sum;
    masses[r][c] = mass;
    __syncthreads();
    if (g >= a.groups) return;
    int before = 0;
    for (int i = 0; i < r; ++i) before += sums[i][c];
    if (r == RUNS - 1) {
        mass = 0.;
        for (int i = 0; i < RUNS; ++i) mass += masses[i][c];
        a.total[g] = before + sum;
        a.mass[g] = mass;
    }
#pragma unroll 4
    for (int64_t b = b0; b < b1; ++b) {
        const int64_t at = b * a.groups + g;
        const int n = a.count[at];
        a.count[at] = before;
        before += n;
    }
}

// 512 rows to 4 of 64 groups, 8 blocks: 11.0 us, 13.7 with the launch in between; 1024 of 256, 32 blocks, 19.1 and 15.5.
constexpr int kFewBlocks = 8;

// Places among all rows.  SUMS: of few blocks, whose counts each workgroup adds up itself instead of a launch in between.
template <bool SUMS> __global__ __launch_bounds__(kFew) void route_place_kernel(Route a)
{
    __shared__ int64_t before[NMF_ROUTE_MAX_GROUPS], meet[kFew / 64];
    __shared__ double meet_d[kFew / 64];
    __shared__ int64_t totals[SUMS ? NMF_ROUTE_MAX_GROUPS : 1];
    __shared__ double masses[SUMS ? NMF_ROUTE_MAX_GROUPS : 1];
    __shared__ int earlier[SUMS ? NMF_ROUTE_MAX_GROUPS : 1];
    constexpr int E = kRouteRows * NMF_ROUTE_MAX_K / kFew;      // choices of a thread
    const int64_t base = (int64_t)blockIdx.x * a.each;
    const int here = (int)std::min<int64_t>(a.each, a.rows - base) * a.k;
    int group[E], in[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = threadIdx.x + e * kFew;
        group[e] = i < here ? a.choice[base * a.k + i] : -1;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (group[e] >= 0) {
            in[e] = a.place[base * a.k + threadIdx.x + e * kFew];
            if (!SUMS) in[e] += a.count[(int64_t)blockIdx.x * a.groups + group[e]];
        }
    if constexpr (SUMS) {
        for (int g = threadIdx.x; g < a.groups; g += kFew) {
            int sum = 0, mine = 0;
            double mass = 0.;
#pragma unroll 8
            for (int b = 0; b < (int)a.blocks; ++b) {
                const int n = a.count[b * a.groups + g];
                if (blockIdx.x == 0) mass += (double)a.share[b * a.groups + g];
                sum += n;
                mine += b < (int)blockIdx.x ? n : 0;
            }
            totals[g] = sum;
            masses[g] = mass;
            earlier[g] = mine;
        }
        __syncthreads();
    }
    const int64_t *total = SUMS ? totals : a.total;
    const int64_t all = sums_before<kFew>(total, a.groups, before, meet);
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (group[e] >= 0) a.place[base * a.k + threadIdx.x + e * kFew] = in[e] + (int)before[group[e]] + (SUMS ? earlier[group[e]] : 0);
    if (blockIdx.x) return;
    for (int g = threadIdx.x; g < a.groups; g += kFew) a.offsets[g] = before[g];
    const double b = balance_of<kFew>(total, SUMS ? masses : a.mass, a.groups, all, meet_d);
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
    else if (groups <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (groups <= 256) f(integral_constant<int, 32>{}, integral_constant<int, 8>{});
    else if (groups <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

// As many rows to a block as a workgroup takes at once, more where that leaves a block to each compute unit: 174 rows of 292 groups in
// blocks of 16 rows 13.8 us, of 64 22; 4096 of 512 17.6 and 32.
int route_each(int64_t rows, int groups)
{
    int each = kRouteRows;
    by_groups(groups, [&](auto w, auto) {
        const int at_once = std::min(kRouteRows, kThreads / w.value);
        const int64_t turns = std::min<int64_t>((rows + 256 * at_once - 1) / (256 * at_once), kRouteRows / at_once);
        each = at_once * (int)std::max<int64_t>(turns, 1);
    });
    return each;
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
        if (a.blocks <= kFewBlocks) {
            hipLaunchKernelGGL((route_place_kernel<true>), dim3((unsigned)a.blocks), dim3(kFew), 0, st, a);
        } else {
            hipLaunchKernelGGL(route_sums_kernel, dim3((unsigned)((a.groups + 15) / 16)), dim3(1024), 0, st, a);
            hipLaunchKernelGGL((route_place_kernel<false>), dim3((unsigned)a.blocks), dim3(kFew), 0, st, a);
        }
    });
    return hipGetLastError();
}

// ---- gradient of the logits ------------------------------------------------------------------
// All from the logits again, as what the softmax was is not kept.  16384 x 128 bf16: 9.6 us (0.9 TB/s).  Instructions bound it, 780
// of the vector unit for a wave of four rows: eight compares of each lane for each choice, the opening, which each wave does in floats of
// 64 bits for its only turn, and the exponents, a sixth of them.
template <class T, int W, int C> __global__ __launch_bounds__(kFew) void route_gradient_kernel(RouteGradient a)
{
    constexpr int ROWS = kFew / W;
    const int first = (int)(threadIdx.x % W) * C;
    float q[C];                                   // d balance / d p_rg, but for c_r
    {
        const int64_t all = a.offsets[a.groups];
        const float up = a.dbalance && all > 0 ? a.dbalance[0] : 0.f;
        const double unit = all > 0 ? (double)a.groups / ((double)all * (double)all) : 0.;
#pragma unroll
        for (int c = 0; c < C; ++c)
            q[c] = a.dbalance && first + c < a.groups ? up * (float)(unit * (double)(a.offsets[first + c + 1] - a.offsets[first + c])) : 0.f;
    }
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < a.rows; base += (int64_t)gridDim.x * ROWS) {
        const int64_t row = base + threadIdx.x / W;
        const bool is = row < a.rows;
        Logits<T, W, C> l;
        l.load((const T *)a.logits + row * a.ldl, a.groups, is);
        // the lane's own groups among the row's choices, and their gates' gradients
        float d[C];
        unsigned own = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) d[c] = 0.f;
        int mine = 0;
        for (int j0 = 0; j0 < a.k; j0 += 4) {
            int g[4];
            float dg[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool there = is && j0 + j < a.k;
                g[j] = there ? a.choice[row * a.k + j0 + j] : -1;
                dg[j] = there && a.dgate ? a.dgate[row * a.k + j0 + j] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (g[j] < 0 || g[j] >= a.groups) continue;
                ++mine;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (first + c == g[j]) {
                        d[c] = dg[j];
                        own |= 1u << c;
                    }
            }
        }
        const float one = 1.f / l.exponents();
        float total = 0.f, dot = 0.f, mean = 0.f;      // sums of p and of p dgate over the choices, of p q over all groups
#pragma unroll
        for (int c = 0; c < C; ++c) {
            l.x[c] *= one;                        // p
            if (own >> c & 1) {
                total += l.x[c];
                dot = __builtin_fmaf(l.x[c], d[c], dot);
            }
            mean = __builtin_fmaf(l.x[c], q[c], mean);
        }
        dot = sum_of<W>(dot);
        mean = sum_of<W>(mean);
        if (a.normalise) total = sum_of<W>(total);
        if (!is) continue;
        // p_i ([i chosen] dg_i - dot), or, normalised, p_i / total (dg_i - dot / total) of the chosen
        const float share = a.normalise ? 1.f / total : 1.f, less = dot * share;
        T out[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const bool chosen = own >> c & 1;
            float x = chosen ? d[c] : 0.f;
            if (chosen || !a.normalise) x -= less;
            x = __builtin_fmaf((float)mine, q[c] - mean, x * share);
            out[c] = Type<T>::round(mine ? l.x[c] * x : 0.f);
        }
        T *to = (T *)a.dlogits + row * a.lddl + first;
        if (first + C <= a.groups) {
            __builtin_memcpy(to, out, sizeof(out));
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (first + c < a.groups) to[c] = out[c];
        }
    }
}

template <class T> hipError_t launch_route_gradient(const RouteGradient &a, hipStream_t st)
{
    by_groups(a.groups, [&](auto w, auto c) {
        constexpr int W = w.value, C = c.value, rows = kFew / W;
        hipLaunchKernelGGL((route_gradient_kernel<T, W, C>), dim3((unsigned)std::min<int64_t>((a.rows + rows - 1) / rows, 2048)), dim3(kFew), 0, st, a);
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
