// Tiles of products over ragged ranges of rows: D (P x Q) += sum over k of p(k, row) q(k, column), for operands that keep
// k contiguous ("KC": rows of a matrix times rows of another) or their own index ("RC": columns), in bf16, f16 or fp32.
//
// A stage holds 128 bytes of k of KC operands (64 halves, 32 floats) and as many k of RC ones, in LDS as 16-byte chunks:
//   KC: [row][8 chunks of k], chunk c at place c ^ ((row >> 1) & 7);
//   RC: [k][chunks of columns], chunk c at place c ^ f(k).
// Both permutations keep the matrix instructions' reads free of bank conflicts: 16 lanes that a 16-byte read serves at
// once cover 16 rows, two rows fill the 256 bytes of all banks, so a place changes with every second row; the transposing
// 8-byte reads of an RC half operand serve 32 lanes on 8 values of k x 32 bytes, which f spreads over the banks; single
// floats of an RC operand are read on four k four apart, 64 bytes of each.
//
// Matrix instructions: v_mfma_f32_16x16x32 on halves, v_mfma_f32_16x16x4_f32 on floats (its k are taken in the order that
// a 16-byte read of a KC operand delivers them, on both operands alike).  On normal random bf16 the 16 x 16 form holds
// 2020 TFLOP/s in registers where the 32 x 32 form holds 1790: it moves half as much of the accumulators.  Q is the
// first operand, so a lane ends with four neighbouring columns of one row in its accumulators, which it stores together.
#pragma once

#include "nmfmu_device.h"
#include "nmfmu_ragged_internal.h"

#include <type_traits>
#include <utility>

namespace nmfmu {
namespace ragged {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

template <class T> struct Type;
template <> struct Type<bf16_t> {
    static constexpr int kBytes = 2;
    static constexpr int kParts = 1;      // matrix instructions of a step
    static __device__ __forceinline__ f32x4 mac(u32x4 q, u32x4 p, f32x4 c, int)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, p), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float load(bf16_t x) { return __uint_as_float((unsigned)x.bits << 16); }
    static __device__ __forceinline__ bf16_t round(float x)
    {
        return bf16_t{__builtin_bit_cast(unsigned short, (__bf16)x)};
    }
    static __device__ __forceinline__ unsigned round2(float x, float y) { return cvt_pk_bf16(x, y); }
};
template <> struct Type<f16_t> {
    static constexpr int kBytes = 2;
    static constexpr int kParts = 1;
    static __device__ __forceinline__ f32x4 mac(u32x4 q, u32x4 p, f32x4 c, int)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, q), __builtin_bit_cast(f16x8, p), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float load(f16_t x) { return (float)__builtin_bit_cast(_Float16, x.bits); }
    static __device__ __forceinline__ f16_t round(float x)
    {
        return f16_t{__builtin_bit_cast(unsigned short, (_Float16)x)};
    }
    static __device__ __forceinline__ unsigned round2(float x, float y)
    {
        return __builtin_bit_cast(unsigned, f16x2{(_Float16)x, (_Float16)y});
    }
};
template <> struct Type<float> {
    static constexpr int kBytes = 4;
    static constexpr int kParts = 4;
    static __device__ __forceinline__ f32x4 mac(u32x4 q, u32x4 p, f32x4 c, int part)
    {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[part]), __uint_as_float(p[part]), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float load(float x) { return x; }
    static __device__ __forceinline__ float round(float x) { return x; }
};

constexpr int kStageBytes = 128;      // bytes of k in a stage
constexpr unsigned kOutside = 0xfffffff0u;
constexpr int kBufferFlags = 0x00020000;

// c[i] += q[j] p for the columns' blocks j: parts outside, so that no instruction waits for the one before it.
template <class T, int N> __device__ __forceinline__ void mac_row(const u32x4 (&q)[N], u32x4 p, f32x4 (&c)[N])
{
#pragma unroll
    for (int part = 0; part < Type<T>::kParts; ++part)
#pragma unroll
        for (int j = 0; j < N; ++j) c[j] = Type<T>::mac(q[j], p, c[j], part);
}

// f(0), ..., f(N - 1) with constants.
template <class F, int... I> __device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void each(F &&f) { each_of(f, std::make_integer_sequence<int, N>{}); }
// How many of `jobs` jobs dealt out over `slots` slots are due by the end of slot n.
constexpr int jobs_due(int n, int jobs, int slots) { return n * jobs / slots + 1 < jobs ? n * jobs / slots + 1 : jobs; }

// k of a stage.
template <class T> constexpr int stage_k() { return kStageBytes / Type<T>::kBytes; }
// Entries of a chunk.
template <class T> constexpr int chunk_n() { return 16 / Type<T>::kBytes; }

// Place shift of the chunks of row k of an RC operand of R columns.
template <class T, int R> __device__ __forceinline__ int rc_shift(int k)
{
    constexpr int pitch = R * Type<T>::kBytes;                // bytes of a row
    if (Type<T>::kBytes == 4) return pitch >= 256 ? ((k >> 2) & 1) * 4 : 0;
    if (Type<T>::kBytes == 1) {                               // 32 lanes read 8 values of k twice, 16 apart, 16 bytes of each
        constexpr int a = pitch >= 256 ? 0 : (pitch == 128 ? 1 : 2);
        return (k & 7) >> a | ((k >> 4) & 1) << (3 - a);
    }
    constexpr int b = pitch >= 256 ? 0 : (pitch == 128 ? 1 : 2);      // bits of k that choose a part of the 256 bytes
    return 2 * (((k & 3) >> b) | ((k >> 3) & 1) << (2 - b));
}

// The same for row `row` of a KC operand.
__device__ __forceinline__ int kc_shift(int row) { return (row >> 1) & 7; }

// One operand of a tile as it lies in memory.
struct Operand {
    const char *base;        // its first entry: (row 0, k 0) of the tile
    int64_t ld;              // bytes from row to row (KC) or from k to k (RC)
    int64_t count;           // rows (KC) or columns (RC) of the tile that exist; may be 0 or less
    int64_t bytes;           // from base to the end of the array: nothing is read from there on
    int first = 0;           // KC: rows before this one are zero
    int64_t plane = 0;       // operands in two planes: bytes from the first to the second
};

// 16 bytes of which only those before `bytes` may be read; the others are zero.  (Loads on any border are as fast as they
// would be from the aligned words around them.)
template <class T> __device__ __forceinline__ u32x4 chunk_at(const char *at, int64_t bytes)
{
    u32x4 v = {0, 0, 0, 0};
    if (bytes >= 16) {
        __builtin_memcpy(&v, at, 16);
    } else if (Type<T>::kBytes == 4) {
        for (int i = 0; i < 3; ++i)
            if (4 * i + 4 <= bytes) __builtin_memcpy((char *)&v + 4 * i, at + 4 * i, 4);
    } else if (Type<T>::kBytes == 1) {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < bytes) v[i >> 2] |= (unsigned)(unsigned char)at[i] << (8 * (i & 3));
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (2 * i + 2 <= bytes) {
                unsigned short h;
                __builtin_memcpy(&h, at + 2 * i, 2);
                v[i >> 1] |= (unsigned)h << (16 * (i & 1));
            }
    }
    return v;
}

// Of a chunk's entries the first `keep`, zero for the others.
template <class T> __device__ __forceinline__ u32x4 keep_first(u32x4 v, int64_t keep)
{
    constexpr int E = chunk_n<T>();
    if (keep >= E) return v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (Type<T>::kBytes == 4) v[i] = i < keep ? v[i] : 0u;
        else if (Type<T>::kBytes == 1) v[i] &= keep >= 4 * i + 4 ? 0xffffffffu : (keep > 4 * i ? (1u << (8 * (int)(keep - 4 * i))) - 1u : 0u);
        else v[i] &= (2 * i < keep ? 0xffffu : 0u) | (2 * i + 1 < keep ? 0xffff0000u : 0u);
    }
    return v;
}

// Brings stages of an operand (R rows or columns) into LDS with THREADS threads.
// PLANES 2: half a stage is k of the first plane, the other half the same k of the second.
// DMA: base, ld and the extents are multiples of 16 bytes: the chunks go to LDS without passing registers; a chunk that is
// not there is asked for outside the descriptor's range, which delivers zeros.  Else: any alignment, through registers.
template <class T, int R, bool RC, int THREADS, bool DMA, int PLANES> struct Loader {
    static constexpr int kJobs = R * (kStageBytes / 16) / THREADS;            // chunks of a thread
    static constexpr int kRowChunks = RC ? R * Type<T>::kBytes / 16 : kStageBytes / 16;
    static constexpr int kRowStep = THREADS / kRowChunks;            // rows from job to job
    static_assert(R * (kStageBytes / 16) % THREADS == 0 && THREADS % kRowChunks == 0, "whole jobs");
    static_assert(RC || kRowStep % 16 == 0, "places repeat from job to job");

    const char *base;
    int64_t ld, bytes;
    int line, place;           // LDS line (row or k) of job 0, and place of its chunks
    int first, count;
    int64_t plane;
    unsigned off[kJobs];
    u32x4 reg[DMA ? 1 : kJobs];

    __device__ __forceinline__ int chunk(int j) const
    {
        return RC ? place ^ rc_shift<T, R>(line + j * kRowStep) : place ^ kc_shift(line);
    }
    // k of job j within its plane's part of a stage, and where its chunk lies from the stage's first k on.
    __device__ __forceinline__ int k_of(int j) const
    {
        return RC ? (line + j * kRowStep) % (stage_k<T>() / PLANES) : chunk(j) % (kStageBytes / 16 / PLANES) * chunk_n<T>();
    }
    __device__ __forceinline__ int64_t where(int j) const
    {
        const int row = line + j * kRowStep;
        if (RC) return k_of(j) * ld + chunk(j) * 16 + (PLANES == 2 && row >= stage_k<T>() / 2 ? plane : 0);
        return (int64_t)row * ld + k_of(j) * Type<T>::kBytes + (PLANES == 2 && chunk(j) >= kStageBytes / 32 ? plane : 0);
    }
    __device__ __forceinline__ bool there(int j) const
    {
        const int row = line + j * kRowStep;
        return RC ? chunk(j) * chunk_n<T>() < count : row >= first && row < count;
    }
    __device__ __forceinline__ void open(const Operand &o)
    {
        base = o.base;
        ld = o.ld;
        bytes = o.bytes;
        first = o.first;
        plane = o.plane;
        count = (int)(o.count < 0 ? 0 : (o.count > R ? R : o.count));
        const int tid = threadIdx.x;
        line = tid / kRowChunks;
        place = tid % kRowChunks;
        if (DMA)
#pragma unroll
            for (int j = 0; j < kJobs; ++j) off[j] = there(j) ? (unsigned)where(j) : kOutside;
    }
    // Chunk j of the stage at k0 (of K in all) to `lds`, or to a register.
    __device__ __forceinline__ void fetch_job(int j, int64_t k0, int64_t K, char *lds)
    {
        const int64_t left = K - k0;
        const char *at = base + (RC ? k0 * ld : k0 * Type<T>::kBytes);
        if (DMA) {
            // Written out, as the builtin makes the compiler wait for all loads before the next transposing read of LDS; the
            // load has no destination register, and wait_loads orders what it brings.
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
            typedef __attribute__((address_space(3))) char lds_char;
            const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_char *)(lds + j * THREADS * 16)) + wave * 1024;
            const u32x4 r = {(unsigned)__builtin_amdgcn_readfirstlane((int)(uintptr_t)at),
                             (unsigned)__builtin_amdgcn_readfirstlane((int)((uintptr_t)at >> 32)) & 0xffffu, 0x7fffffffu, (unsigned)kBufferFlags};
            unsigned o = off[j];
            if (left < stage_k<T>() / PLANES && k_of(j) >= left) o = kOutside;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(o), "s"(r) : "memory", "m0");
        } else {
            u32x4 v = {0, 0, 0, 0};
            if (there(j) && k_of(j) < left) {
                v = chunk_at<T>(at + where(j), bytes - (at - base) - where(j));
                v = keep_first<T>(v, RC ? count - chunk(j) * chunk_n<T>() : left - k_of(j));
            }
            reg[j] = v;
        }
    }
    // The same straight to LDS from a stage that begins at `at`, with `left` k from there on: fewer registers.
    __device__ __forceinline__ void bring(int j, const char *at, int left, char *lds) const
    {
        static_assert(DMA && PLANES == 1, "");
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        typedef __attribute__((address_space(3))) char lds_char;
        const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_char *)(lds + j * THREADS * 16)) + wave * 1024;
        const u32x4 r = {(unsigned)__builtin_amdgcn_readfirstlane((int)(uintptr_t)at),
                         (unsigned)__builtin_amdgcn_readfirstlane((int)((uintptr_t)at >> 32)) & 0xffffu, 0x7fffffffu, (unsigned)kBufferFlags};
        const unsigned o = (RC ? line >= left - j * kRowStep : k_of(j) >= left) ? kOutside : off[j];
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(o), "s"(r) : "memory", "m0");
    }
    __device__ __forceinline__ void fetch(int64_t k0, int64_t K, char *lds)
    {
#pragma unroll
        for (int j = 0; j < kJobs; ++j) fetch_job(j, k0, K, lds);
    }
    __device__ __forceinline__ void put(char *lds)
    {
#pragma unroll
        for (int j = 0; j < kJobs; ++j) *reinterpret_cast<u32x4 *>(lds + (threadIdx.x + j * THREADS) * 16) = reg[DMA ? 0 : j];
    }
};

// Reads operands of the matrix instruction from a stage: block of 16 rows or columns at first + t * STEP, matrix step kk.
template <class T, int R, bool RC, int STEP> struct Reader {
    int at[kStageBytes / 64];        // KC: by kk; RC: unused
    int lane, first;

    __device__ __forceinline__ void open(int first_)
    {
        lane = threadIdx.x & 63;
        first = first_;
        if (!RC) {
#pragma unroll
            for (int kk = 0; kk < kStageBytes / 64; ++kk) at[kk] = kc_at(kk);
        }
    }
    __device__ __forceinline__ int kc_at(int kk) const
    {
        const int row = first + (lane & 15);
        return row * kStageBytes + (((4 * kk + (lane >> 4)) ^ kc_shift(row)) << 4);
    }
    __device__ __forceinline__ u32x4 read(const char *lds, int t, int kk) const
    {
        if (!RC) return *reinterpret_cast<const u32x4 *>(lds + at[kk] + t * STEP * kStageBytes);
        constexpr int pitch = R * Type<T>::kBytes;
        u32x4 v;
        if constexpr (Type<T>::kBytes == 2) {
            // 16 lanes read 4 values of k x 16 columns, and each leaves with the 4 k of one column
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int i = lane & 15, k = 8 * (lane >> 4) + (i >> 2);
            const int col = first + t * STEP + 4 * (i & 3);
            const char *p = lds + (32 * kk + k) * pitch + (((col >> 3) ^ rc_shift<T, R>(k)) << 4) + (col & 7) * 2;
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
            const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * pitch)));
            v = u32x4{a[0], a[1], b[0], b[1]};
        } else if constexpr (Type<T>::kBytes == 1) {
            // 16 lanes read 8 values of k x 16 columns, and each leaves with the 8 k of one column
            typedef int i32x2 __attribute__((ext_vector_type(2)));
            typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
            const int i = lane & 15, k = 64 * kk + 16 * (lane >> 4) + (i >> 1), c = (first + t * STEP) >> 4;
            const char *p = lds + k * pitch + ((c ^ rc_shift<T, R>(k)) << 4) + (i & 1) * 8;      // (the shift of k + 8 is that of k)
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)p));
            const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(p + 8 * pitch)));
            v = u32x4{a[0], a[1], b[0], b[1]};
        } else {
            const int col = first + t * STEP + (lane & 15);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 16 * kk + 4 * (lane >> 4) + j;
                v[j] = *reinterpret_cast<const unsigned *>(lds + k * pitch + (((col >> 2) ^ rc_shift<T, R>(k)) << 4) + (col & 3) * 4);
            }
        }
        return v;
    }
};

template <int N> __device__ __forceinline__ void wait_loads()      // until at most N of a wave's loads are under way
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All waves' LDS reads and writes so far are done.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A tile of BM x BN by WM x WN waves.
template <class T_, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool PRC_, bool QRC_, bool DMA_, int PLANES_ = 1> struct Tile {
    using T = T_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = DMA_ ? STAGES_ : 2, THREADS = 64 * WM * WN;
    static constexpr bool PRC = PRC_, QRC = QRC_, DMA = DMA_;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;      // 16 x 16 blocks of a wave: every WM-th of the rows, neighbouring columns
    static constexpr int KK = kStageBytes / 64;                             // matrix steps of a stage
    static constexpr int PLANES = PLANES_, SK = stage_k<T>() / PLANES;      // k of a stage
    static constexpr int kLdsP = BM * kStageBytes, kLdsQ = BN * kStageBytes, kLdsStage = kLdsP + kLdsQ;
    static constexpr int kLds = STAGES * kLdsStage;
    using Acc = f32x4[TM][TN];
    using LoadP = Loader<T, BM, PRC, THREADS, DMA, PLANES>;
    using LoadQ = Loader<T, BN, QRC, THREADS, DMA, PLANES>;
    using ReadP = Reader<T, BM, PRC, 16 * WM>;
    using ReadQ = Reader<T, BN, QRC, 16>;

    static __device__ __forceinline__ void clear(Acc &acc)
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // First row and column of a wave; row and column of a lane's first entry in block (i, j), which has four columns.
    static __device__ __forceinline__ int wave_row() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64) / WN * 16; }
    static __device__ __forceinline__ int wave_col() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % WN * (BN / WN); }
    static __device__ __forceinline__ int row_of(int i) { return wave_row() + 16 * WM * i + (threadIdx.x & 15); }
    static __device__ __forceinline__ int col_of(int j) { return wave_col() + 16 * j + 4 * (threadIdx.x >> 4 & 3); }

    // One stage.  The operands of a matrix step are read while the one before runs; load(n) asks for chunk n of the next
    // stage, first of all (32 x 128 over 64 groups of 4096 x 2048: 165 us; spread over the products 242).
    template <class F>
    static __device__ __forceinline__ void step(const char *lds, const ReadP &rp, const ReadQ &rq, Acc &acc, F load)
    {
        constexpr int L = LoadP::kJobs + LoadQ::kJobs;
#pragma unroll
        for (int n = 0; n < L; ++n) load(n);
        constexpr int D = TM * TN < 32 ? 2 : 1;      // the large tile's registers hold one step's operands
        u32x4 p[D][TM], q[D][TN];
        auto get = [&](int kk) {
#pragma unroll
            for (int j = 0; j < TN; ++j) q[kk % D][j] = rq.read(lds + kLdsP, j, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i) p[kk % D][i] = rp.read(lds, i, kk);
        };
        get(0);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (D == 1 && kk) {
                __builtin_amdgcn_sched_barrier(0);
                get(kk);
            } else if (D == 2 && kk + 1 < KK) {
                get(kk + 1);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) mac_row<T>(q[kk % D], p[kk % D][i], acc[i]);
        }
    }

    // Stages of the large tile, two matrix steps each.  While the first step's products run, the second's operands are read;
    // then the stage's buffer is free, and the next stage has arrived.  While the second step's run, the next stage's first
    // operands are read, and the buffer is loaded again for the stage after it.  Reads and loads are dealt out between the
    // products: a load of all lanes keeps its unit busy for 16 cycles, and products wait behind what is issued before them.
    static constexpr bool kAhead = DMA && STAGES == 2 && TM * TN >= 32;
    static __device__ __forceinline__ void ahead(LoadP &lp, LoadQ &lq, const ReadP &rp, const ReadQ &rq, int64_t k0, int64_t k1, int steps, int64_t rows,
                                                 char *lds, Acc &acc)
    {
        static_assert(KK == 2, "two matrix steps");
        constexpr int L = LoadP::kJobs + LoadQ::kJobs;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            lp.fetch(k0 + s * SK, k1, lds + s * kLdsStage);
            lq.fetch(k0 + s * SK, k1, lds + s * kLdsStage + kLdsP);
        }
        wait_loads<L>();
        meet();
        auto run = [&](auto live) {
            constexpr int LIVE = live.value, N = LIVE * TN, R = LIVE + TN;
            u32x4 p[2][TM], q[2][TN];
            auto get = [&](auto n, auto kk, const char *stage) {      // operand n of a step
                if constexpr (n.value < TN) q[kk.value][n.value] = rq.read(stage + kLdsP, n.value, kk.value);
                else p[kk.value][n.value - TN] = rp.read(stage, n.value - TN, kk.value);
            };
            // products of step kk, and jobs between them
            auto products = [&](auto kk, auto jobs, auto job) {
                constexpr int parts = Type<T>::kParts, J = jobs.value, all = N * parts;
                each<all>([&](auto n) {
                    constexpr int i = n.value / (TN * parts), part = n.value / TN % parts, j = n.value % TN;
                    acc[i][j] = Type<T>::mac(q[kk.value][j], p[kk.value][i], acc[i][j], part);
                    constexpr int past = n.value ? jobs_due(n.value - 1, J, all - 4) : 0, due = jobs_due(n.value, J, all - 4);
                    if constexpr (due > past) {
                        __builtin_amdgcn_sched_barrier(0);
                        each<due - past>([&](auto t) { job(std::integral_constant<int, past + t.value>{}); });
                        __builtin_amdgcn_sched_barrier(0);
                    }
                });
            };
            using First = std::integral_constant<int, 0>;
            using Second = std::integral_constant<int, 1>;
            each<R>([&](auto n) { get(n, First{}, lds); });
            for (int s = 0; s < steps; ++s) {
                char *now = lds + (s & 1) * kLdsStage, *next = lds + (~s & 1) * kLdsStage;
                const int64_t k = k0 + (int64_t)(s + 2) * SK;
                products(First{}, std::integral_constant<int, R>{}, [&](auto n) { get(n, Second{}, now); });
                wait_loads<0>();
                meet();
                __builtin_amdgcn_sched_barrier(0);
                products(Second{}, std::integral_constant<int, R + L>{}, [&](auto n) {
                    // loads and reads in turn while there are both
                    constexpr int both = 2 * (R < L ? R : L), m = n.value;
                    constexpr bool reads = m < both ? m % 2 == 1 : R > L;
                    constexpr int nth = m < both ? m / 2 : m - both / 2;
                    if constexpr (reads) get(std::integral_constant<int, nth>{}, First{}, next);
                    else if constexpr (nth < LoadQ::kJobs) lq.fetch_job(nth, k, k1, now + kLdsP);
                    else lp.fetch_job(nth - LoadQ::kJobs, k, k1, now);
                });
            }
        };
        if (PRC || rows > BM / 2) run(std::integral_constant<int, TM>{});
        else run(std::integral_constant<int, TM / 2>{});      // the waves' rows lie in turn: half of each one's
        wait_loads<0>();
    }

    // The first matrix step of a stage alone.
    static __device__ __forceinline__ void first_step(const char *lds, const ReadP &rp, const ReadQ &rq, Acc &acc)
    {
        u32x4 p[TM], q[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) q[j] = rq.read(lds + kLdsP, j, 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) p[i] = rp.read(lds, i, 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) mac_row<T>(q, p[i], acc[i]);
    }

    // acc += the product over k in [k0, k1) of K.  Leaves LDS free for other use.
    static __device__ __forceinline__ void multiply(const Operand &P, const Operand &Q, int64_t k0, int64_t k1, char *lds, Acc &acc)
    {
        LoadP lp;
        LoadQ lq;
        lp.open(P);
        lq.open(Q);
        ReadP rp;
        ReadQ rq;
        rp.open(wave_row());
        rq.open(wave_col());
        const int steps = (int)((k1 - k0 + SK - 1) / SK);
        if constexpr (kAhead) {
            ahead(lp, lq, rp, rq, k0, k1, steps, P.count, lds, acc);
        } else if (DMA) {
            constexpr int L = LoadP::kJobs + LoadQ::kJobs;
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) {
                lp.fetch(k0 + (int64_t)s * SK, k1, lds + s * kLdsStage);
                lq.fetch(k0 + (int64_t)s * SK, k1, lds + s * kLdsStage + kLdsP);
            }
            int from = 0, to = STAGES - 1;
            for (int s = 0; s < steps; ++s) {
                wait_loads<(STAGES - 2) * L>();
                meet();
                const int64_t k = k0 + (int64_t)(s + STAGES - 1) * SK;
                step(lds + from * kLdsStage, rp, rq, acc, [&](int n) {
                    if (n < LoadQ::kJobs) lq.fetch_job(n, k, k1, lds + to * kLdsStage + kLdsP);
                    else lp.fetch_job(n - LoadQ::kJobs, k, k1, lds + to * kLdsStage);
                });
                from = from + 1 == STAGES ? 0 : from + 1;
                to = to + 1 == STAGES ? 0 : to + 1;
            }
            wait_loads<0>();
        } else if (steps > 0) {
            lp.fetch(k0, k1, nullptr);
            lq.fetch(k0, k1, nullptr);
            lp.put(lds);
            lq.put(lds + kLdsP);
            for (int s = 0; s < steps; ++s) {
                meet();
                const bool more = s + 1 < steps;
                if (more) {
                    lp.fetch(k0 + (int64_t)(s + 1) * SK, k1, nullptr);
                    lq.fetch(k0 + (int64_t)(s + 1) * SK, k1, nullptr);
                }
                step(lds + (s & 1) * kLdsStage, rp, rq, acc, [](int) {});
                if (more) {
                    lp.put(lds + ((s + 1) & 1) * kLdsStage);
                    lq.put(lds + ((s + 1) & 1) * kLdsStage + kLdsP);
                }
            }
        }
        meet();
    }

    // Entries (row, column) of the tile inside rows x cols to out (ld entries from row to row).  A lane's accumulators are
    // four columns at a time of one row; through LDS, two blocks' rows of a wave at a time, whole lines leave together.
    // vec: rows of out begin on 16-byte borders.  lds: as much as multiply had, free.
    template <class O>
    static __device__ __forceinline__ void store(const Acc &acc, O *out, int64_t ld, int64_t rows, int64_t cols, bool vec, char *lds,
                                                 float scale = 1.f)
    {
        constexpr int B = TM < 2 ? 1 : 2, H = 16 * B;           // blocks and rows at once
        constexpr int W = TN * 16, N = 16 / (int)sizeof(O), kPitch = W * (int)sizeof(O) + 16, kLanes = W / N, kAtOnce = 64 / kLanes;
        static_assert(H * kPitch * WM * WN <= kLds && H % kAtOnce == 0, "the waves' rows fit");
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
        char *mine = lds + wave * (H * kPitch);
        const int first = wave_row(), col = wave_col() + lane % kLanes * N, up = lane / kLanes;
        const int have = cols - col < N ? (int)(cols - col) : N;
#pragma unroll
        for (int i = 0; i < TM; i += B) {
            if (first + 16 * WM * i >= rows) break;
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const f32x4 x = acc[i + b][j] * scale;
                    char *to = mine + (16 * b + (lane & 15)) * kPitch + (16 * j + 4 * (lane >> 4)) * (int)sizeof(O);
                    if constexpr (sizeof(O) == 4) *reinterpret_cast<f32x4 *>(to) = x;
                    else *reinterpret_cast<u32x2 *>(to) = u32x2{Type<O>::round2(x[0], x[1]), Type<O>::round2(x[2], x[3])};
                }
            u32x4 w[H / kAtOnce];
#pragma unroll
            for (int r = 0; r < H / kAtOnce; ++r)
                w[r] = *reinterpret_cast<const u32x4 *>(mine + (up + r * kAtOnce) * kPitch + lane % kLanes * 16);
#pragma unroll
            for (int r = 0; r < H / kAtOnce; ++r) {
                const int in = up + r * kAtOnce, row = first + 16 * WM * (i + in / 16) + in % 16;
                if (row >= rows) continue;
                O *at = out + (int64_t)row * ld + col;
                if (have == N) {
                    if (vec) *reinterpret_cast<u32x4 *>(at) = w[r];
                    else __builtin_memcpy(at, &w[r], 16);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (e < have) {
                            if constexpr (sizeof(O) == 4) at[e] = __uint_as_float(w[r][e]);
                            else at[e] = O{(unsigned short)(w[r][e >> 1] >> (16 * (e & 1)))};
                        }
                }
            }
        }
    }
};

// ---- which rows a workgroup has ------------------------------------------------------

// Range g of offsets, held inside [0, rows] and in order, so that malformed offsets touch nothing outside.
__device__ __forceinline__ void range_of(const int64_t *offsets, int g, int64_t rows, int64_t &lo, int64_t &hi)
{
    lo = offsets[g];
    hi = offsets[g + 1];
    lo = lo < 0 ? 0 : (lo > rows ? rows : lo);
    hi = hi < lo ? lo : (hi > rows ? rows : hi);
}

// Row tiles of BM rows of all ranges, in order; every wave looks by itself, 64 ranges at a time.
struct Found {
    int g;              // range
    int64_t r0, r1;     // its rows [r0, r1)
};
struct Ranges {
    const int64_t *offsets;
    int groups, BM;
    int64_t rows, lo, hi;        // of the lane's range
    int count, sum, base;        // its tiles, and those up to and with it among the 64 from `base` on

    __device__ __forceinline__ void look(int base_)
    {
        const int lane = threadIdx.x & 63;
        base = base_;
        lo = hi = 0;
        if (base + lane < groups) range_of(offsets, base + lane, rows, lo, hi);
        count = (int)((hi - lo + BM - 1) / BM);
        sum = count;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
    }
    __device__ __forceinline__ int open(const int64_t *offsets_, int groups_, int64_t rows_, int BM_)      // returns how many tiles there are
    {
        offsets = offsets_;
        groups = groups_;
        rows = rows_;
        BM = BM_;
        int total = 0;
        for (int b = groups > 0 ? (groups - 1) / 64 * 64 : 0; b >= 0; b -= 64) {
            look(b);
            total += __builtin_amdgcn_readlane(sum, 63);
        }
        return total;
    }
    // Tile `want`, counted from the ranges looked at now (the first 64 after open).
    __device__ __forceinline__ bool find(int want, Found &f)
    {
        if (base != 0) look(0);
        for (;;) {
            const unsigned long long past = __ballot(sum > want);
            if (past) {
                const int l = __builtin_ctzll(past);
                f.g = base + l;
                const int before = __builtin_amdgcn_readlane(sum - count, l);
                const int64_t l0 = lane_value(lo, l), h0 = lane_value(hi, l);
                f.r0 = l0 + (int64_t)(want - before) * BM;
                f.r1 = h0 < f.r0 + BM ? h0 : f.r0 + BM;
                return f.r0 >= l0 && f.r0 < h0;        // (counts of malformed ranges can overflow)
            }
            want -= __builtin_amdgcn_readlane(sum, 63);
            if (base + 64 >= groups) return false;
            look(base + 64);
        }
    }
    static __device__ __forceinline__ int64_t lane_value(int64_t x, int l)
    {
        return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)x, l) |
                         (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32);
    }
};
// First range that ends behind row r (ranges in order), or `groups`.
__device__ __forceinline__ int first_range(const int64_t *offsets, int groups, int64_t r)
{
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < groups; base += 64) {
        const bool is = base + lane < groups && offsets[base + lane + 1] > r;
        const unsigned long long m = __ballot(is);
        if (m) return __builtin_amdgcn_readfirstlane(base + __ffsll(m) - 1);
    }
    return groups;
}

// The same for a lane's own row.
__device__ __forceinline__ int range_at(const int64_t *offsets, int groups, int64_t r)
{
    int lo = 0, hi = groups;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (offsets[mid + 1] > r) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}
// The range with `want` longer ones (or as long and before it), where there are up to 64; else range `want`.
__device__ __forceinline__ int nth_longest(const int64_t *offsets, int groups, int64_t rows, int want)
{
    if (groups > 64) return want;
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = 0;
    if (lane < groups) range_of(offsets, lane, rows, lo, hi);
    const int len = lane < groups ? (int)(hi - lo) : -1;
    int longer = 0;
    for (int i = 0; i < groups; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        longer += other > len || (other == len && i < lane);
    }
    const unsigned long long at = __ballot(lane < groups && longer == want);
    return __builtin_ctzll(at);
}

// Workgroups are dealt to the eight dies in turn, each with a cache of its own: a die gets neighbouring tiles.
__device__ __forceinline__ int by_die(int id, int total)
{
    const int each = total / 8, more = total % 8, die = id % 8, nth = id / 8;
    return die < more ? die * (each + 1) + nth : more * (each + 1) + (die - more) * each + nth;
}

}  // namespace ragged
}  // namespace nmfmu
