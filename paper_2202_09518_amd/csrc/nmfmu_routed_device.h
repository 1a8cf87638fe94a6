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
    float scale, inverse;
    bool finite;
};
__device__ __forceinline__ Scale scale_of(unsigned most)
{
    Scale s;
    s.finite = most < 0x7f800000u;
    s.scale = __builtin_fmaxf(__uint_as_float(most) / 448.f, 0x1p-126f);
    s.inverse = 1.f / s.scale;
    if (!s.finite) s.scale = __builtin_nanf("");
    return s;
}
// Codes of eight entries: x / scale, to the last bit (the quotient's error is taken back once), rounded to nearest even.  No
// quotient is above 448 by more than 2^-23 of it, so none overflows.
__device__ __forceinline__ ragged::u32x2 codes_of(const float (&x)[8], const Scale &s)
{
    ragged::u32x2 c = {0, 0};
    if (!s.finite) return c;
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = x[i] * s.inverse;
        q[i] = __builtin_fmaf(__builtin_fmaf(-q[i], s.scale, x[i]), s.inverse, q[i]);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * n], q[4 * n + 1], 0, false);
        c[n] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * n + 2], q[4 * n + 3], w, true);
    }
    return c;
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

template <int W> __device__ __forceinline__ unsigned most_of(unsigned x)      // of W neighbouring lanes
{
#pragma unroll
    for (int d = 1; d < W; d <<= 1) {
        const unsigned o = (unsigned)__shfl_xor((int)x, d);
        x = x > o ? x : o;
    }
    return x;
}
template <int W> __device__ __forceinline__ float sum_of(float x)
{
#pragma unroll
    for (int d = 1; d < W; d <<= 1) x += __shfl_xor(x, d);
    return x;
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
