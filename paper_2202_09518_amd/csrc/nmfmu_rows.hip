// The norm and its gradients, rounding to 8 bits, and the rows' way to their groups and back: all bound by memory.
#include "nmfmu_routed_device.h"

#include <algorithm>
#include <type_traits>

namespace nmfmu {
namespace routed {

namespace {

constexpr int64_t kMostBlocks = 1 << 20;      // workgroups of a launch: beyond, they take several turns
unsigned grid_of(int64_t blocks) { return (unsigned)std::min<int64_t>(std::max<int64_t>(blocks, 1), kMostBlocks); }

}  // namespace

// ---- norm ----------------------------------------------------------------------------------
// A row to W threads, C chunks of eight columns to each, read once and held in registers as they were; a workgroup keeps the
// weight's chunks for all its rows.  Threads without a row in the last turn go along to the barriers.  The squares are added as
// floats, eight at a time and then over lanes and waves in a fixed tree.
// Memory bounds it: 16384 x 4096 bf16 with the residual to H and 8 bits 96 us (4.9 TB/s; a large copy reads and writes 5.2), 8192 rows
// to H and Y 49 us (5.5); one row 3.2 us, its two trips to memory and the launch.
template <class T, int W, int C> __global__ __launch_bounds__(W < 256 ? 256 : W) void norm_kernel(Norm a)
{
    constexpr int ROWS = W < 256 ? 256 / W : 1;
    __shared__ float meet[2 * (W / 64)];
    const int lane = threadIdx.x % W;
    Eight<T> w[C];
    if (a.w) {
#pragma unroll
        for (int c = 0; c < C; ++c) w[c].load((const T *)a.w, (c * W + lane) * 8, a.m);
    }
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS, ++turn) {
        const int64_t row = first + threadIdx.x / W;
        const bool is = row < a.rows;
        Eight<T> h[C];
        if (is) {
#pragma unroll
            for (int c = 0; c < C; ++c) h[c].load((const T *)a.x + row * a.ldx, (c * W + lane) * 8, a.m);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) h[c].zero();
        }
        if (a.r && is) {
            Eight<T> r[C];
#pragma unroll
            for (int c = 0; c < C; ++c) r[c].load((const T *)a.r + row * a.ldr, (c * W + lane) * 8, a.m);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = h[c].at(i) + r[c].at(i);
                h[c].put(x);
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (a.h && is) h[c].store((T *)a.h + row * a.ldh, (c * W + lane) * 8, a.m);
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) part = __builtin_fmaf(h[c].at(i), h[c].at(i), part);
            sum += part;
        }
        sum = row_sum<W>(sum, meet, turn);
        const float s = 1.f / __builtin_sqrtf(sum / (float)a.m + a.eps);
        if (!is) continue;
        if (a.rstd && lane == 0) a.rstd[row] = s;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (c * W + lane) * 8;
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (a.w ? h[c].at(i) * w[c].at(i) : h[c].at(i)) * s;      // of 16-bit entries the product is exact
            if (a.y) {
                Eight<T> out;
                out.put(y);
                out.store((T *)a.y + row * a.ldy, col, a.m);
            }
            if (a.y8) {
                unsigned most = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const unsigned b = magnitude(y[i]);
                    most = most > b ? most : b;
                }
                const Scale z = scale_of(most_of<16>(most));
                store_codes((unsigned char *)a.y8 + row * a.ldy8, col, a.m, near_codes(y, z));
                if (lane % 16 == 0 && col < a.m) a.scale[row * a.lds + col / 128] = z.scale;
            }
        }
    }
}

// f(threads of a row, chunks of a thread) for rows of m entries.
template <class F> void by_width(int64_t m, F f)
{
    using std::integral_constant;
    if (m <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (m <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (m <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (m <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (m <= 8192) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (m <= 16384) f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

template <class T> hipError_t launch_norm(const Norm &a, hipStream_t st)
{
    by_width(a.m, [&](auto w, auto c) {
        constexpr int W = w.value, C = c.value, threads = W < 256 ? 256 : W, rows = threads / W;
        const int64_t blocks = (a.rows + rows - 1) / rows;
        hipLaunchKernelGGL((norm_kernel<T, W, C>), dim3((unsigned)std::min<int64_t>(blocks, 256 * 2048 / threads)), dim3(threads), 0, st, a);
    });
    return hipGetLastError();
}

// ---- gradients of the norm -------------------------------------------------------------------
// A thread has the same columns of all its rows, so it adds up the weight's gradient as it goes; the workgroups' sums meet in
// a second launch, in order.  Few rows are one workgroup's, which writes the weight's gradient itself.
// 8192 x 4096 bf16 with the residual's gradient: 50 us (5.4 TB/s) and 4.6 for the sums of 1024 workgroups.  Wider, both in turn: 8192 x
// 8192 130 us, 4096 x 16384 109; 2048 x 32768 232 (114 without the weight's gradient), as 1024 threads have 128 registers each, and
// beyond 16384 columns (8192 in float32, by a few) what they hold does not fit: memory takes the rest.  A wave for each narrow row leaves
// most of its lanes idle: 524288 x 128 396 us (1.4 TB/s).
template <class T, int W, int C, bool DW> __global__ __launch_bounds__(W < 256 ? 256 : W) void norm_gradient_kernel(NormGradient a)
{
    constexpr int ROWS = W < 256 ? 256 / W : 1;
    __shared__ float meet[2 * (W / 64)];
    const int lane = threadIdx.x % W;
    float dw[DW ? C : 1][8];
#pragma unroll
    for (int c = 0; c < (DW ? C : 1); ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS, ++turn) {
        const int64_t row = first + threadIdx.x / W;
        const bool is = row < a.rows;
        Eight<T> h[C], dy[C];
        float s = 0.f;
        if (is) {
            s = a.rstd[row];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                h[c].load((const T *)a.h + row * a.ldh, (c * W + lane) * 8, a.m);
                dy[c].load((const T *)a.dy + row * a.ldy, (c * W + lane) * 8, a.m);
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) h[c].zero(), dy[c].zero();
        }
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            Eight<T> w;
            if (a.w) w.load((const T *)a.w, (c * W + lane) * 8, a.m);
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = h[c].at(i) * s, z = a.w ? dy[c].at(i) * w.at(i) : dy[c].at(i);
                if (DW) dw[c][i] = __builtin_fmaf(dy[c].at(i), x, dw[c][i]);
                part = __builtin_fmaf(z, x, part);
            }
            sum += part;
        }
        const float mean = row_sum<W>(sum, meet, turn) / (float)a.m;
        if (!is) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (c * W + lane) * 8;
            Eight<T> w, d;
            if (a.w) w.load((const T *)a.w, col, a.m);
            if (a.dh) d.load((const T *)a.dh + row * a.lddh, col, a.m);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = a.w ? dy[c].at(i) * w.at(i) : dy[c].at(i);
                const float y = __builtin_fmaf(-(h[c].at(i) * s), mean, z);
                x[i] = a.dh ? __builtin_fmaf(s, y, d.at(i)) : s * y;
            }
            Eight<T> out;
            out.put(x);
            out.store((T *)a.dx + row * a.ldx, col, a.m);
        }
    }
    if constexpr (DW) {
        if constexpr (ROWS > 1) {
            __shared__ float other[ROWS - 1][C * W * 8];
            const int mine = threadIdx.x / W;
            if (mine) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) other[mine - 1][(c * 8 + i) * W + lane] = dw[c][i];
            }
            __syncthreads();
            if (mine) return;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int r = 0; r < ROWS - 1; ++r) dw[c][i] += other[r][(c * 8 + i) * W + lane];
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (c * W + lane) * 8;
            if (a.part) {
                Eight<float> out;
                out.put(dw[c]);
                out.store(a.part + (int64_t)blockIdx.x * a.m, col, a.m);
            } else {
                Eight<T> out;
                out.put(dw[c]);
                out.store((T *)a.dw, col, a.m);
            }
        }
    }
}

// 32 columns to a workgroup, every 32nd part to a thread of each column's; the 32 sums meet in order.
template <class T> __global__ __launch_bounds__(1024) void norm_weight_kernel(NormGradient a)
{
    __shared__ float sums[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + c;
    float x = 0.f;
    if (col < a.m)
#pragma unroll 8
        for (int p = r; p < a.parts; p += 32) x += a.part[(int64_t)p * a.m + col];
    sums[r][c] = x;
    __syncthreads();
    if (r || col >= a.m) return;
    x = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) x += sums[i][c];
    ((T *)a.dw)[col] = Type<T>::round(x);
}

// Four workgroups of 256 threads to a compute unit: 8192 x 4096 bf16, forward and backward, 104 us; with three 106, with two 115.  (The
// number for all widths, of which only that one was measured; of 4097 to 8192 columns the registers of two fit at once.)
constexpr int kNormThreads = 256 * 1024;
int norm_parts(int64_t rows, int64_t m)
{
    int parts = 1;
    by_width(m, [&](auto w, auto) {
        constexpr int W = w.value, threads = W < 256 ? 256 : W, each = threads / W;
        parts = (int)std::min<int64_t>(std::max<int64_t>((rows + each - 1) / each, 1), kNormThreads / threads);
        if (rows <= 4 * each) parts = 1;
    });
    return parts;
}

template <class T> hipError_t launch_norm_gradient(const NormGradient &a, hipStream_t st)
{
    by_width(a.m, [&](auto w, auto c) {
        constexpr int W = w.value, C = c.value, threads = W < 256 ? 256 : W, rows = threads / W;
        const int64_t blocks = std::max<int64_t>((a.rows + rows - 1) / rows, 1);
        if (a.dw) hipLaunchKernelGGL((norm_gradient_kernel<T, W, C, true>), dim3((unsigned)a.parts), dim3(threads), 0, st, a);
        else
            hipLaunchKernelGGL((norm_gradient_kernel<T, W, C, false>), dim3((unsigned)std::min<int64_t>(blocks, 256 * 2048 / threads)), dim3(threads), 0,
                               st, a);
    });
    if (a.dw && a.part) hipLaunchKernelGGL((norm_weight_kernel<T>), dim3((unsigned)((a.m + 31) / 32)), dim3(1024), 0, st, a);
    return hipGetLastError();
}

// ---- 8 bits ----------------------------------------------------------------------------------
// Blocks of a row: 16 lanes to each, 16 blocks to a workgroup, 2^shift of them side by side.  No index is divided: with divisions of
// 64 bits 3001 x 1433 floats took 8.7 us, without them 7.0 (2.8 TB/s; rows that begin anywhere).
template <class T> __global__ __launch_bounds__(256) void round_rows_kernel(Round a, int shift)
{
    const int64_t M = blocks_of(a.m);
    const int lane = threadIdx.x & 15, unit = threadIdx.x / 16, side = unit & ((1 << shift) - 1), up = unit >> shift;
    for (int64_t i = blockIdx.z; i < a.count; i += gridDim.z)
        for (int64_t row = ((int64_t)blockIdx.x << (4 - shift)) + up; row < a.rows; row += (int64_t)gridDim.x << (4 - shift))
            for (int64_t b = ((int64_t)blockIdx.y << shift) + side; b < M; b += (int64_t)gridDim.y << shift) {
                const int64_t col = b * 128 + lane * 8;
                Eight<T> v;
                v.load((const T *)a.x + i * a.stride + row * a.ldx, col, a.m);
                float x[8];
                unsigned most = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = v.at(e);
                    const unsigned g = magnitude(x[e]);
                    most = most > g ? most : g;
                }
                const Scale s = scale_of(most_of<16>(most));
                store_codes((unsigned char *)a.x8 + i * a.stride8 + row * a.ldx8, col, a.m, exact_codes<T>(x, s));
                if (lane == 0) a.scale[i * a.stride_s + row * a.lds + b] = s.scale;
            }
}

// Blocks of 128 x 128: a workgroup to each, eight rows of a chunk to a thread, so that the block is read once.
// 8 x 4096 x 2048 bf16: 34.5 us (5.8 TB/s).
template <class T> __global__ __launch_bounds__(256) void round_tiles_kernel(Round a)
{
    __shared__ unsigned meet[2][4];
    const int64_t M = blocks_of(a.m), R = blocks_of(a.rows), all = a.count * R * M;
    const int lane = threadIdx.x & 15, up = threadIdx.x / 16;
    int turn = 0;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x, ++turn) {
        const int64_t i = at / (R * M), in = at - i * R * M, r = in / M, b = in - r * M, col = b * 128 + lane * 8;
        const T *x = (const T *)a.x + i * a.stride;
        Eight<T> v[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const int64_t row = r * 128 + 16 * n + up;
            if (row < a.rows) v[n].load(x + row * a.ldx, col, a.m);
            else v[n].zero();
        }
        unsigned most = 0;
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned g = magnitude(v[n].at(e));
                most = most > g ? most : g;
            }
        most = most_of<64>(most);
        unsigned *m4 = meet[turn & 1];
        if ((threadIdx.x & 63) == 0) m4[threadIdx.x / 64] = most;
        __syncthreads();
#pragma unroll
        for (int n = 0; n < 4; ++n) most = most > m4[n] ? most : m4[n];
        const Scale s = scale_of(most);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const int64_t row = r * 128 + 16 * n + up;
            if (row >= a.rows) continue;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = v[n].at(e);
            store_codes((unsigned char *)a.x8 + i * a.stride8 + row * a.ldx8, col, a.m, exact_codes<T>(y, s));
        }
        if (threadIdx.x == 0) a.scale[i * a.stride_s + r * a.lds + b] = s.scale;
    }
}

template <class T> hipError_t launch_round(const Round &a, hipStream_t st)
{
    if (a.block == 1) {
        // as many blocks side by side as leave few lanes without one
        const int64_t M = blocks_of(a.m);
        int shift = 4;
        while (shift && ((((M - 1) >> shift) + 1) << shift) * 8 > M * 9) --shift;
        const int64_t y = std::min<int64_t>(((M - 1) >> shift) + 1, 64), z = std::min(a.count, 16);
        const int64_t x = std::min<int64_t>(((a.rows - 1) >> (4 - shift)) + 1, kMostBlocks / (y * z));
        hipLaunchKernelGGL((round_rows_kernel<T>), dim3((unsigned)x, (unsigned)y, (unsigned)z), dim3(256), 0, st, a, shift);
    } else {
        hipLaunchKernelGGL((round_tiles_kernel<T>), dim3(grid_of(a.count * blocks_of(a.rows) * blocks_of(a.m))), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

// ---- rows to their places and back -------------------------------------------------------------
// Rows of `chunks` chunks to 2^shift threads each, in parts of so many chunks.
struct Deal {
    int shift;
    int64_t parts, blocks;
};
inline Deal deal(int64_t rows, int64_t chunks)
{
    Deal d = {0, 1, 0};
    while (d.shift < 8 && (1 << d.shift) < chunks) ++d.shift;
    d.parts = (chunks + (1 << d.shift) - 1) >> d.shift;
    const int64_t each = 256 >> d.shift;
    d.blocks = (rows + each - 1) / each * d.parts;
    return d;
}
// The row and chunk of a thread in a workgroup's turn.
__device__ __forceinline__ void dealt(const Deal &d, int64_t block, int64_t &row, int64_t &chunk, int64_t &part)
{
    const int64_t rb = block / d.parts;
    part = block - rb * d.parts;
    row = rb * (256 >> d.shift) + (threadIdx.x >> d.shift);
    chunk = (part << d.shift) + (threadIdx.x & ((1 << d.shift) - 1));
}

// Each row is read once and written k times.  8192 x 4096 bf16 to 4 places: 50 us (6.3 TB/s, four fifths of it written).
__global__ __launch_bounds__(256) void spread_kernel(Spread a, Deal d)
{
    for (int64_t block = blockIdx.x; block < d.blocks; block += gridDim.x) {
        int64_t row, chunk, part;
        dealt(d, block, row, chunk, part);
        if (row >= a.rows) continue;
        const int64_t at = chunk * 16;
        u32x4 v = {0, 0, 0, 0};
        const char *x = (const char *)a.x + row * a.ldx + at;
        const int have = a.m - at >= 16 ? 16 : (int)(a.m - at);
        if (have == 16) {
            __builtin_memcpy(&v, x, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (i < have) v[i >> 2] |= (unsigned)(unsigned char)x[i] << (8 * (i & 3));
        }
        for (int j = 0; j < a.k; ++j) {
            const int64_t place = a.place[row * a.k + j];
            if (place < 0 || place >= a.sorted) continue;
            char *y = (char *)a.y + place * a.ldy + at;
            if (have == 16) {
                __builtin_memcpy(y, &v, 16);
            } else {
#pragma unroll
                for (int i = 0; i < 15; ++i)
                    if (i < have) y[i] = (char)(v[i >> 2] >> (8 * (i & 3)));
            }
            if (a.xs && part == 0)
                for (int64_t c = chunk; c < a.ms; c += 1 << d.shift) a.ys[place * a.ldys + c] = a.xs[row * a.ldxs + c];
        }
    }
}

hipError_t launch_spread(const Spread &a, hipStream_t st)
{
    const Deal d = deal(a.rows, (a.m + 15) / 16);
    hipLaunchKernelGGL(spread_kernel, dim3(grid_of(d.blocks)), dim3(256), 0, st, a, d);
    return hipGetLastError();
}

constexpr int kAtOnce = 4;      // choices whose rows are under way together

// The sum of a row's k rows, in the order of its choices, in floats.  8192 x 4096 bf16 from 4 places: 78 us (4.1 TB/s of rows anywhere).
template <class T> __global__ __launch_bounds__(256) void collect_kernel(Collect a, Deal d)
{
    for (int64_t block = blockIdx.x; block < d.blocks; block += gridDim.x) {
        int64_t row, chunk, part;
        dealt(d, block, row, chunk, part);
        const int64_t col = chunk * 8;
        if (row >= a.rows || col >= a.m) continue;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = 0.f;
        for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
            Eight<T> x[kAtOnce];
            float g[kAtOnce];
            bool is[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int64_t at = row * a.k + j0 + j;
                const int64_t place = j0 + j < a.k ? a.place[at] : -1;
                is[j] = place >= 0 && place < a.sorted;
                g[j] = is[j] && a.gate ? a.gate[at] : 1.f;
                if (is[j]) x[j].load((const T *)a.x + place * a.ldx, col, a.m);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (is[j])
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(g[j], x[j].at(i), y[i]);
        }
        Eight<T> out;
        out.put(y);
        out.store((T *)a.y + row * a.ldy, col, a.m);
    }
}

template <class T> hipError_t launch_collect(const Collect &a, hipStream_t st)
{
    const Deal d = deal(a.rows, (a.m + 7) / 8);
    hipLaunchKernelGGL((collect_kernel<T>), dim3(grid_of(d.blocks)), dim3(256), 0, st, a, d);
    return hipGetLastError();
}

// A row to W threads; its products with the rows of kAtOnce choices are summed over all columns, as its share goes to each of them.
// 8192 x 4096 bf16, 4 places: 103 us (5.6 TB/s).
template <class T, int W, bool DGATE> __global__ __launch_bounds__(256) void collect_gradient_kernel(CollectGradient a)
{
    constexpr int ROWS = 256 / W;
    __shared__ float meet[2 * (W / 64)];
    const int lane = threadIdx.x % W;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS) {
        const int64_t row = first + threadIdx.x / W;
        for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
            int64_t place[kAtOnce];
            float g[kAtOnce], dot[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const bool is = row < a.rows && j0 + j < a.k;
                place[j] = is ? a.place[row * a.k + j0 + j] : -1;
                if (place[j] >= a.sorted) place[j] = -1;
                g[j] = place[j] >= 0 && a.gate ? a.gate[row * a.k + j0 + j] : 1.f;
                dot[j] = 0.f;
            }
            if (row < a.rows)
                for (int64_t col = lane * 8; col < a.m; col += W * 8) {
                    Eight<T> dy;
                    dy.load((const T *)a.dy + row * a.ldy, col, a.m);
                    [[maybe_unused]] Eight<T> x[kAtOnce];
                    if constexpr (DGATE) {
#pragma unroll
                        for (int j = 0; j < kAtOnce; ++j)
                            if (place[j] >= 0) x[j].load((const T *)a.x + place[j] * a.ldx, col, a.m);
                    }
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) {
                        if (place[j] < 0) continue;
                        float d[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[i] = g[j] * dy.at(i);
                        Eight<T> out;
                        out.put(d);
                        out.store((T *)a.dx + place[j] * a.lddx, col, a.m);
                        if constexpr (DGATE) {
                            float part = 0.f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) part = __builtin_fmaf(dy.at(i), x[j].at(i), part);
                            dot[j] += part;
                        }
                    }
                }
            if constexpr (DGATE) {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const float sum = row_sum<W>(dot[j], meet, turn++);
                    if (lane == 0 && row < a.rows && j0 + j < a.k) a.dgate[row * a.k + j0 + j] = sum;
                }
            }
        }
    }
}

template <class T> hipError_t launch_collect_gradient(const CollectGradient &a, hipStream_t st)
{
    auto go = [&](auto w, auto dgate) {
        constexpr int W = w.value;
        const int64_t blocks = (a.rows + 256 / W - 1) / (256 / W);
        hipLaunchKernelGGL((collect_gradient_kernel<T, W, dgate.value>), dim3(grid_of(blocks)), dim3(256), 0, st, a);
    };
    using std::integral_constant;
    if (a.m <= 1024) {
        if (a.dgate) go(integral_constant<int, 64>{}, std::true_type{});
        else go(integral_constant<int, 64>{}, std::false_type{});
    } else {
        if (a.dgate) go(integral_constant<int, 256>{}, std::true_type{});
        else go(integral_constant<int, 256>{}, std::false_type{});
    }
    return hipGetLastError();
}

#define NMFMU_ROWS(T)                                                             \
    template hipError_t launch_norm<T>(const Norm &, hipStream_t);                \
    template hipError_t launch_norm_gradient<T>(const NormGradient &, hipStream_t); \
    template hipError_t launch_round<T>(const Round &, hipStream_t);              \
    template hipError_t launch_collect<T>(const Collect &, hipStream_t);          \
    template hipError_t launch_collect_gradient<T>(const CollectGradient &, hipStream_t);
NMFMU_ROWS(float)
NMFMU_ROWS(bf16_t)
NMFMU_ROWS(f16_t)

}  // namespace routed
}  // namespace nmfmu
