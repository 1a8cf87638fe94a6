// Tiles of products over ragged ranges of rows: D (P x Q) += sum over k of p(k, row) q(k, column), for operands that keep
// k contiguous ("KC": rows of a matrix times rows of another) or their own index ("RC": columns), in bf16, f16 or fp32.
//
// A stage holds 128 bytes of k of KC operands (64 halves, 32 floats) and as many k of RC ones, in LDS as 16-byte chunks:
//   KC: [row][8 chunks of k], chunk c at place c ^ ((row >> 1) & 7);
//   RC: [k][chunks of columns], chunk c at place c ^ f(k).
// Both permutations keep the matrix instructions' reads free of bank conflicts: 16 lanes that a 16-byte read serves at
// once cover 16 rows, two rows fill the 256 bytes of all banks, so a place changes with every second row; the transposing
// 8-byte reads of an RC half operand serve 32 lanes on 4 values of k x 64 bytes, which f spreads over the banks; single
// floats of an RC operand are read on two k four apart, 128 bytes of each.
//
// Matrix instructions: v_mfma_f32_32x32x16 on halves, v_mfma_f32_32x32x2_f32 on floats (its k are taken in the order that
// a 16-byte read of a KC operand delivers them, on both operands alike).  Q is the first operand, so a lane ends with four
// neighbouring columns of one row in its accumulators, which it stores together.
#pragma once

#include "nmfmu_device.h"
#include "nmfmu_ragged_internal.h"

#include <type_traits>

namespace nmfmu {
namespace ragged {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

template <class T> struct Type;
template <> struct Type<bf16_t> {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ f32x16 mac(u32x4 q, u32x4 p, f32x16 c) { return mfma_bf16(q, p, c); }
    static __device__ __forceinline__ float load(bf16_t x) { return __uint_as_float((unsigned)x.bits << 16); }
    static __device__ __forceinline__ bf16_t round(float x)
    {
        return bf16_t{__builtin_bit_cast(unsigned short, (__bf16)x)};
    }
    static __device__ __forceinline__ unsigned round2(float x, float y) { return cvt_pk_bf16(x, y); }
};
template <> struct Type<f16_t> {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ f32x16 mac(u32x4 q, u32x4 p, f32x16 c) { return mfma_f16(q, p, c); }
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
    static __device__ __forceinline__ f32x16 mac(u32x4 q, u32x4 p, f32x16 c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = mfma32(__uint_as_float(q[j]), __uint_as_float(p[j]), c);
        return c;
    }
    static __device__ __forceinline__ float load(float x) { return x; }
    static __device__ __forceinline__ float round(float x) { return x; }
};

constexpr int kStageBytes = 128;      // bytes of k in a stage, if not said otherwise
constexpr unsigned kOutside = 0xfffffff0u;
constexpr int kBufferFlags = 0x00020000;

// k of a stage.
template <class T, int SB = kStageBytes> constexpr int stage_k() { return SB / Type<T>::kBytes; }
// Entries of a chunk.
template <class T> constexpr int chunk_n() { return 16 / Type<T>::kBytes; }

// Place shift of the chunks of row k of an RC operand of R columns.
template <class T, int R> __device__ __forceinline__ int rc_shift(int k)
{
    constexpr int pitch = R * Type<T>::kBytes;                // bytes of a row
    if (Type<T>::kBytes == 4) return pitch >= 256 ? ((k >> 2) & 1) * 8 : 0;
    if (pitch >= 256) return (k & 3) * 4;
    if (pitch == 128) return ((k >> 1) & 1) * 4;
    return 0;
}

// The same for row `row` of a KC operand.
template <int SB> __device__ __forceinline__ int kc_shift(int row) { return SB == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }

// One operand of a tile as it lies in memory.
struct Operand {
    const char *base;        // its first entry: (row 0, k 0) of the tile
    int64_t ld;              // bytes from row to row (KC) or from k to k (RC)
    int64_t count;           // rows (KC) or columns (RC) of the tile that exist; may be 0 or less
    int64_t bytes;           // from base to the end of the array: nothing is read from there on
    int first = 0;           // KC: rows before this one are zero
    int64_t plane = 0;       // operands in two planes: bytes from the first to the second
};

// 16 bytes of which only those before `bytes` may be read; the others are zero.
template <class T> __device__ __forceinline__ u32x4 chunk_at(const char *at, int64_t bytes)
{
    u32x4 v = {0, 0, 0, 0};
    if (bytes >= 16) {
        __builtin_memcpy(&v, at, 16);
    } else if (Type<T>::kBytes == 4) {
        for (int i = 0; i < 3; ++i)
            if (4 * i + 4 <= bytes) __builtin_memcpy((char *)&v + 4 * i, at + 4 * i, 4);
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
        else v[i] &= (2 * i < keep ? 0xffffu : 0u) | (2 * i + 1 < keep ? 0xffff0000u : 0u);
    }
    return v;
}

// Brings stages of an operand (R rows or columns) into LDS with THREADS threads.
// PLANES 2: half a stage is k of the first plane, the other half the same k of the second.
// DMA: base, ld and the extents are multiples of 16 bytes: the chunks go to LDS without passing registers; a chunk that is
// not there is asked for outside the descriptor's range, which delivers zeros.  Else: any alignment, through registers.
template <class T, int R, bool RC, int THREADS, bool DMA, int SB, int PLANES> struct Loader {
    static constexpr int kJobs = R * (SB / 16) / THREADS;            // chunks of a thread
    static constexpr int kRowChunks = RC ? R * Type<T>::kBytes / 16 : SB / 16;
    static constexpr int kRowStep = THREADS / kRowChunks;            // rows from job to job
    static_assert(R * (SB / 16) % THREADS == 0 && THREADS % kRowChunks == 0, "whole jobs");
    static_assert(RC ? kRowStep % (Type<T>::kBytes == 4 ? 8 : 4) == 0 : kRowStep % 16 == 0, "places repeat from job to job");

    const char *base;
    int64_t ld, bytes;
    int line, chunk;           // LDS line (row or k) and chunk of job 0
    int first, count;
    int64_t plane;
    unsigned off[kJobs];
    u32x4 reg[DMA ? 1 : kJobs];

    // k of job j within its plane's part of a stage, and where its chunk lies from the stage's first k on.
    __device__ __forceinline__ int k_of(int j) const
    {
        return RC ? (line + j * kRowStep) % (stage_k<T, SB>() / PLANES) : chunk % (SB / 16 / PLANES) * chunk_n<T>();
    }
    __device__ __forceinline__ int64_t where(int j) const
    {
        const int row = line + j * kRowStep;
        if (RC) return k_of(j) * ld + chunk * 16 + (PLANES == 2 && row >= stage_k<T, SB>() / 2 ? plane : 0);
        return (int64_t)row * ld + k_of(j) * Type<T>::kBytes + (PLANES == 2 && chunk >= SB / 32 ? plane : 0);
    }
    __device__ __forceinline__ bool there(int j) const
    {
        const int row = line + j * kRowStep;
        return RC ? chunk * chunk_n<T>() < count : row >= first && row < count;
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
        const int place = tid % kRowChunks;
        chunk = RC ? place ^ rc_shift<T, R>(line) : place ^ kc_shift<SB>(line);
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
            const __amdgpu_buffer_rsrc_t r =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, 0x7fffffff, kBufferFlags);
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
            typedef __attribute__((address_space(3))) void lds_void;
            unsigned o = off[j];
            if (left < stage_k<T, SB>() / PLANES && k_of(j) >= left) o = kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(lds + j * THREADS * 16 + wave * 1024), 16, o, 0, 0, 0);
        } else {
            u32x4 v = {0, 0, 0, 0};
            if (there(j) && k_of(j) < left) {
                v = chunk_at<T>(at + where(j), bytes - (at - base) - where(j));
                v = keep_first<T>(v, RC ? count - chunk * chunk_n<T>() : left - k_of(j));
            }
            reg[j] = v;
        }
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

// Reads operands of the matrix instruction from a stage: block of 32 rows or columns at 32 * t + first, step kk of 4.
template <class T, int R, bool RC, int SB = kStageBytes> struct Reader {
    int at[SB / 32];        // KC: by kk; RC: unused
    int lane, first;

    __device__ __forceinline__ void open(int first_)
    {
        lane = threadIdx.x & 63;
        first = first_;
        if (!RC) {
            const int row = first + (lane & 31);
#pragma unroll
            for (int kk = 0; kk < SB / 32; ++kk) at[kk] = row * SB + (((2 * kk + (lane >> 5)) ^ kc_shift<SB>(row)) << 4);
        }
    }
    __device__ __forceinline__ u32x4 read(const char *lds, int t, int kk) const
    {
        if (!RC) return *reinterpret_cast<const u32x4 *>(lds + at[kk] + t * 32 * SB);
        constexpr int pitch = R * Type<T>::kBytes;
        u32x4 v;
        if (Type<T>::kBytes == 2) {
            // 16 lanes read 4 values of k x 16 columns, and each leaves with the 4 k of one column
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int i = lane & 15, k = 8 * (lane >> 5) + (i >> 2);
            const int col = first + 32 * t + 16 * ((lane >> 4) & 1) + 4 * (i & 3);
            const char *p = lds + (16 * kk + k) * pitch + (((col >> 3) ^ rc_shift<T, R>(k)) << 4) + (col & 7) * 2;
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
            const char *p4 = lds + (16 * kk + k + 4) * pitch + (((col >> 3) ^ rc_shift<T, R>(k + 4)) << 4) + (col & 7) * 2;
            const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p4));
            v = u32x4{a[0], a[1], b[0], b[1]};
        } else {
            const int col = first + 32 * t + (lane & 31);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 8 * kk + 4 * (lane >> 5) + j;
                v[j] = *reinterpret_cast<const unsigned *>(lds + k * pitch + (((col >> 2) ^ rc_shift<T, R>(k)) << 4) + (col & 3) * 4);
            }
        }
        return v;
    }
    // The same for a kk known at run time only (floats).
    __device__ __forceinline__ u32x4 read_at(const char *lds, int t, int kk) const
    {
        if (RC) return read(lds + kk * 8 * R * Type<T>::kBytes, t, 0);          // eight k further; their places repeat
        const int row = first + (lane & 31);
        return *reinterpret_cast<const u32x4 *>(lds + (row + 32 * t) * SB + (((2 * kk + (lane >> 5)) ^ kc_shift<SB>(row)) << 4));
    }
};

template <int N> __device__ __forceinline__ void wait_loads()      // until at most N of a wave's loads are under way
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All waves' LDS reads and writes so far are done.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A tile of BM x BN by WM x WN waves.
template <class T_, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool PRC_, bool QRC_, bool DMA_, int SB_ = kStageBytes, int PLANES_ = 1> struct Tile {
    using T = T_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = DMA_ ? STAGES_ : 2, THREADS = 64 * WM * WN;
    static constexpr bool PRC = PRC_, QRC = QRC_, DMA = DMA_;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;      // 32 x 32 tiles of a wave
    static constexpr int SB = SB_, PLANES = PLANES_, SK = stage_k<T, SB>() / PLANES;      // bytes of k in a stage; its k
    static constexpr int kLdsP = BM * SB, kLdsQ = BN * SB, kLdsStage = kLdsP + kLdsQ;
    static constexpr int kLds = STAGES * kLdsStage;
    using Acc = f32x16[TM][TN];
    using LoadP = Loader<T, BM, PRC, THREADS, DMA, SB, PLANES>;
    using LoadQ = Loader<T, BN, QRC, THREADS, DMA, SB, PLANES>;
    using ReadP = Reader<T, BM, PRC, SB>;
    using ReadQ = Reader<T, BN, QRC, SB>;

    static __device__ __forceinline__ void clear(Acc &acc)
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    }

    // One stage.  The operands of a matrix step are read while the one before runs; load(n) asks for chunk n of the next
    // stage.  A chunk of all lanes keeps the load unit busy for 16 cycles, so the large tile spreads them over its products,
    // one after every second (256 x 256, 8192 x 8192 x 4096, bf16: 443 us, all at the start 478; 448 after every fourth); a
    // tile with few products asks first (32 x 128 over 64 groups of 4096 x 2048: 165 us, spread 242).
    // KK: matrix steps of the stage; LIVE: blocks of 32 rows that take part.
    template <int KK = SB / 32, int LIVE = TM, class F>
    static __device__ __forceinline__ void step(const char *lds, const ReadP &rp, const ReadQ &rq, Acc &acc, F load)
    {
        constexpr int L = LoadP::kJobs + LoadQ::kJobs;
        constexpr bool spread = KK * LIVE * TN >= 4 * L;
        u32x4 p[2][TM], q[2][TN];
        auto get = [&](int kk) {
#pragma unroll
            for (int j = 0; j < TN; ++j) q[kk & 1][j] = rq.read(lds + kLdsP, j, kk);
#pragma unroll
            for (int i = 0; i < LIVE; ++i) p[kk & 1][i] = rp.read(lds, i, kk);
        };
        int done = 0;
        if (!spread)
#pragma unroll
            for (; done < L; ++done) load(done);
        if (LIVE == 0) return;
        get(0);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kk + 1 < KK) get(kk + 1);
#pragma unroll
            for (int i = 0; i < LIVE; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    acc[i][j] = Type<T>::mac(q[kk & 1][j], p[kk & 1][i], acc[i][j]);
                    if (spread && ((kk * LIVE + i) * TN + j) % 2 == 0 && done < L) {
                        __builtin_amdgcn_sched_barrier(0);
                        load(done++);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
        }
    }

    // The first kks matrix steps of a stage, one by one.
    static __device__ __forceinline__ void first_steps(const char *lds, const ReadP &rp, const ReadQ &rq, Acc &acc, int kks)
    {
#pragma unroll 1
        for (int kk = 0; kk < kks; ++kk) {
            u32x4 p[TM], q[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) q[j] = rq.read_at(lds + kLdsP, j, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i) p[i] = rp.read_at(lds, i, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = Type<T>::mac(q[j], p[i], acc[i][j]);
        }
    }

    // acc += the product over k in [k0, k1) of K.  Leaves LDS free for other use.
    static __device__ __forceinline__ void multiply(const Operand &P, const Operand &Q, int64_t k0, int64_t k1, char *lds, Acc &acc)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        LoadP lp;
        LoadQ lq;
        lp.open(P);
        lq.open(Q);
        ReadP rp;
        ReadQ rq;
        rp.open(wave / WN * (BM / WM));
        rq.open(wave % WN * (BN / WN));
        const int steps = (int)((k1 - k0 + SK - 1) / SK);
        if (DMA) {
            constexpr int L = LoadP::kJobs + LoadQ::kJobs;
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) {
                lp.fetch(k0 + (int64_t)s * SK, k1, lds + s * kLdsStage);
                lq.fetch(k0 + (int64_t)s * SK, k1, lds + s * kLdsStage + kLdsP);
            }
            int from = 0, to = STAGES - 1;
            auto run = [&](auto live) {
                for (int s = 0; s < steps; ++s) {
                    wait_loads<(STAGES - 2) * L>();
                    meet();
                    const int64_t k = k0 + (int64_t)(s + STAGES - 1) * SK;
                    step<SB / 32, live.value>(lds + from * kLdsStage, rp, rq, acc, [&](int n) {
                        if (n < LoadQ::kJobs) lq.fetch_job(n, k, k1, lds + to * kLdsStage + kLdsP);
                        else lp.fetch_job(n - LoadQ::kJobs, k, k1, lds + to * kLdsStage);
                    });
                    from = from + 1 == STAGES ? 0 : from + 1;
                    to = to + 1 == STAGES ? 0 : to + 1;
                }
            };
            // Waves whose rows are not there leave out their products: all of them, or half.
            const int have = (int)(P.count < BM ? P.count : BM) - wave / WN * (BM / WM);
            if (PRC || TM < 4 || have > TM * 16) run(std::integral_constant<int, TM>{});
            else if (have > 0) run(std::integral_constant<int, TM / 2>{});
            else run(std::integral_constant<int, 0>{});
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
    // four columns at a time of one row; through LDS, 32 rows of a wave at a time, whole lines leave together.
    // vec: rows of out begin on 16-byte borders.  lds: as much as multiply had, free.
    template <class O>
    static __device__ __forceinline__ void store(const Acc &acc, O *out, int64_t ld, int64_t rows, int64_t cols, bool vec, char *lds,
                                                 float scale = 1.f)
    {
        constexpr int W = TN * 32, N = 16 / (int)sizeof(O), kPitch = W * (int)sizeof(O) + 16, kLanes = W / N, kAtOnce = 64 / kLanes;
        static_assert(32 * kPitch * WM * WN <= kLds, "the waves' rows fit");
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
        char *mine = lds + wave * (32 * kPitch);
        const int first = wave / WN * (BM / WM), col = wave % WN * (BN / WN) + lane % kLanes * N, up = lane / kLanes;
        const int have = cols - col < N ? (int)(cols - col) : N;
        O *at = out + (int64_t)(first + up) * ld + col;
        const int64_t step = ld * kAtOnce;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if (first + 32 * i >= rows) break;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const f32x4 x = {acc[i][j][4 * v] * scale, acc[i][j][4 * v + 1] * scale, acc[i][j][4 * v + 2] * scale,
                                     acc[i][j][4 * v + 3] * scale};
                    char *to = mine + (lane & 31) * kPitch + (32 * j + 8 * v + 4 * (lane >> 5)) * (int)sizeof(O);
                    if constexpr (sizeof(O) == 4) *reinterpret_cast<f32x4 *>(to) = x;
                    else *reinterpret_cast<u32x2 *>(to) = u32x2{Type<O>::round2(x[0], x[1]), Type<O>::round2(x[2], x[3])};
                }
            u32x4 w[32 / kAtOnce];
#pragma unroll
            for (int r = 0; r < 32 / kAtOnce; ++r)
                w[r] = *reinterpret_cast<const u32x4 *>(mine + (up + r * kAtOnce) * kPitch + lane % kLanes * 16);
#pragma unroll
            for (int r = 0; r < 32 / kAtOnce; ++r, at += step) {
                if (first + 32 * i + up + r * kAtOnce >= rows) continue;
                if (vec && have == N) {
                    *reinterpret_cast<u32x4 *>(at) = w[r];
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
                return true;
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
