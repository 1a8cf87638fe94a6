// Device code of the norm, the rounding to 8 bits and the rows' way to their groups: eight entries of a row to a lane.
#pragma once

#include "nmfmu_ragged_device.h"
#include "nmfmu_routed_internal.h"

namespace nmfmu {
namespace routed {

using ragged::Type;

// Eight neighbouring entries as they lie in memory.
template <class T> struct Eight {
    static constexpr int N = sizeof(T) / 2;
    u32x4 v[N];

    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[i >> 2][i & 3]);
        else return Type<T>::load(T{(unsigned short)(v[0][i >> 1] >> (16 * (i & 1)))});
    }
    __device__ __forceinline__ void put(const float (&x)[8])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = __float_as_uint(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[0][i] = Type<T>::round2(x[2 * i], x[2 * i + 1]);
        }
    }
    // Entries [col, col + 8) of a row of m, zero behind its end.
    __device__ __forceinline__ void load(const T *row, int64_t col, int64_t m)
    {
        if (col + 8 <= m) {
            __builtin_memcpy(v, row + col, sizeof(v));
            return;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (col + i < m) {
                if constexpr (sizeof(T) == 4) {
                    v[i >> 2][i & 3] = __float_as_uint(row[col + i]);
                } else {
                    v[0][i >> 1] |= (unsigned)row[col + i].bits << (16 * (i & 1));
                }
            }
    }
    __device__ __forceinline__ void store(T *row, int64_t col, int64_t m) const
    {
        if (col + 8 <= m) {
            __builtin_memcpy(row + col, v, sizeof(v));
            return;
        }
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (col + i < m) {
                if constexpr (sizeof(T) == 4) row[col + i] = __uint_as_float(v[i >> 2][i & 3]);
                else row[col + i] = T{(unsigned short)(v[0][i >> 1] >> (16 * (i & 1)))};
            }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = u32x4{0, 0, 0, 0};
    }
};

// ---- 8 bits ------------------------------------------------------------------------------
// Magnitudes are compared by their bits, where infinities lie above all numbers and NaN above infinities.
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

struct Scale {
    float scale, up;              // scale: the largest magnitude / 448; up: 1 / scale
    float most, part, back;       // for exact_codes, where the magnitude is small 2^64 times it: the magnitude; 7 / 8 as many times; 512 / most
    bool finite;
};
__device__ __forceinline__ Scale scale_of(unsigned bits)
{
    Scale s;
    s.finite = bits < 0x7f800000u;
    const float most = __builtin_fmaxf(__uint_as_float(bits), 0x1.cp-118f);      // 448 2^-126
    // most / 448 and its inverse, each with its error taken back once
    constexpr float part = 1.f / 448.f;
    const float near = most * part, scale = __builtin_fmaf(__builtin_fmaf(-near, 448.f, most), part, near);
    const float inverse = __builtin_amdgcn_rcpf(scale);
    s.up = __builtin_fmaf(__builtin_fmaf(-scale, inverse, 1.f), inverse, inverse);
    const bool small = most < 0x1p-60f;
    s.most = small ? most * 0x1p64f : most;
    s.part = small ? 0.875f * 0x1p64f : 0.875f;
    s.back = s.up * (8.f / 7.f) * (small ? 0x1p-64f : 1.f);
    s.scale = s.finite ? scale : __builtin_nanf("");
    return s;
}
__device__ __forceinline__ ragged::u32x2 codes_of(const float (&q)[8], const Scale &s)
{
    ragged::u32x2 c = {0, 0};
    if (!s.finite) return c;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * n], q[4 * n + 1], 0, false);
        c[n] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * n + 2], q[4 * n + 3], w, true);
    }
    return c;
}
// Codes of eight floats, for the norm: the nearest ones to x 448 / largest but where that is within 2^-22 of itself of the middle between
// two.  (Scale, inverse and product are off by 2^-24 each; at most 448 (1 + 2^-22), which is 448.)  To look at quotients on borders again
// as exact_codes does costs the norm registers and its loads' overlap: 16384 x 4096 bf16 96 us and 98 to 101, 8192 x 8192 91 and 99.
__device__ __forceinline__ ragged::u32x2 near_codes(const float (&x)[8], const Scale &s)
{
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = x[i] * s.up;
    return codes_of(q, s);
}
// Codes of eight entries of T, the nearest ones to x 448 / largest: the error of the quotient by the inverse, from x 7 / 8 and most
// quotient / 512 so that nothing overflows, is taken back.  In small blocks both are 2^64 times that, as errors of 2^-48 of an entry
// would lie below 2^-149.  Of 16-bit entries the quotient lies on a border between two codes or 2^-16 away from it.  Of floats it
// can be nearer than its own last place, so there what is left of it sets that to odd, which no border has; it is looked at only
// where some quotient of the wave is within four last places of where borders are, multiples of 2^19 of them.
template <class T> __device__ __forceinline__ ragged::u32x2 exact_codes(const float (&x)[8], const Scale &s)
{
    float q[8];
    bool near = sizeof(T) == 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = x[i] * s.up;
        near |= ((__float_as_uint(q[i]) + 4) & 0x7ffff) <= 8;
    }
    if (sizeof(T) == 2 || __any(near)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float part = x[i] * s.part, rest = sizeof(T) == 4 ? __builtin_fmaf(x[i], s.part, -part) : 0.f;
            q[i] = __builtin_fmaf(__builtin_fmaf(q[i] * -0x1p-9f, s.most, part) + rest, s.back, q[i]);
            if (sizeof(T) == 4) {
                const float left = __builtin_fmaf(q[i] * -0x1p-9f, s.most, part) + rest;
                unsigned b = __float_as_uint(q[i]);
                if (left != 0.f) b = (b - ((b ^ __float_as_uint(left)) >> 31)) | 1u;
                q[i] = __uint_as_float(b);
            }
        }
    }
    return codes_of(q, s);
}
__device__ __forceinline__ void store_codes(unsigned char *row, int64_t col, int64_t m, ragged::u32x2 c)
{
    if (col + 8 <= m) {
        __builtin_memcpy(row + col, &c, 8);
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (col + i < m) row[col + i] = (unsigned char)(c[i >> 2] >> (8 * (i & 3)));
}

// f of W neighbouring lanes (a power of two), in all of them: partners are the other one of a pair, the other pair, then mirrored
// quads and halves of 16, which hold one value each by then, then the other 16 and 32 lanes.  f(a, b) is f(b, a), so all lanes end
// with the same bits.
template <int CONTROL> __device__ __forceinline__ unsigned moved(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, 0xf, 0xf, true); }
template <int W, class F> __device__ __forceinline__ unsigned over_lanes(unsigned x, F f)
{
    if constexpr (W >= 2) x = f(x, moved<0xb1>(x));       // quad_perm 1 0 3 2
    if constexpr (W >= 4) x = f(x, moved<0x4e>(x));       // quad_perm 2 3 0 1
    if constexpr (W >= 8) x = f(x, moved<0x141>(x));      // row_half_mirror
    if constexpr (W >= 16) x = f(x, moved<0x140>(x));     // row_mirror
    if constexpr (W >= 32) {
        const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = f(y[0], y[1]);
    }
    if constexpr (W >= 64) {
        const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = f(y[0], y[1]);
    }
    return x;
}
template <int W> __device__ __forceinline__ unsigned most_of(unsigned x)
{
    return over_lanes<W>(x, [](unsigned a, unsigned b) { return a > b ? a : b; });
}
template <int W> __device__ __forceinline__ unsigned least_of(unsigned x)
{
    return over_lanes<W>(x, [](unsigned a, unsigned b) { return a < b ? a : b; });
}
template <int W> __device__ __forceinline__ float most_of(float x)
{
    return __uint_as_float(over_lanes<W>(__float_as_uint(x), [](unsigned a, unsigned b) { return __float_as_uint(__builtin_fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int W> __device__ __forceinline__ float sum_of(float x)
{
    return __uint_as_float(over_lanes<W>(__float_as_uint(x), [](unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// Sum over the W threads of a row, W / 64 waves of which leave theirs in `meet` (two turns of it, so that one barrier does).
template <int W> __device__ __forceinline__ float row_sum(float x, float *meet, int turn)
{
    x = sum_of<(W < 64 ? W : 64)>(x);
    if constexpr (W > 64) {
        constexpr int N = W / 64;
        float *at = meet + (turn & 1) * N;
        if ((threadIdx.x & 63) == 0) at[threadIdx.x / 64] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) x += at[i];
    }
    return x;
}

}  // namespace routed
}  // namespace nmfmu
