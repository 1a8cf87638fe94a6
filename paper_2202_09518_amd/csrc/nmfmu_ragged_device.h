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

constexpr int kStageBytes = 128;      // bytes of k in a stage
constexpr unsigned kOutside = 0xfffffff0u;
constexpr int kBufferFlags = 0x00020000;

// k of a stage.
template <class T> constexpr int stage_k() { return kStageBytes / Type<T>::kBytes; }
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

// One operand of a tile as it lies in memory.
struct Operand {
    const char *base;        // its first entry: (row 0, k 0) of the tile
    int64_t ld;              // bytes from row to row (KC) or from k to k (RC)
    int64_t count;           // rows (KC) or columns (RC) of the tile that exist; may be 0 or less
    int64_t bytes;           // from base to the end of the array: nothing is read from there on
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
// DMA: base, ld and the extents are multiples of 16 bytes: the chunks go to LDS without passing registers; a chunk that is
// not there is asked for outside the descriptor's range, which delivers zeros.  Else: any alignment, through registers.
template <class T, int R, bool RC, int THREADS, bool DMA> struct Loader {
    static constexpr int kBytesLds = R * kStageBytes;
    static constexpr int kJobs = R * 8 / THREADS;                    // chunks of a thread
    static constexpr int kRowChunks = RC ? R * Type<T>::kBytes / 16 : 8;
    static constexpr int kRowStep = THREADS / kRowChunks;            // rows from job to job
    static_assert(R * 8 % THREADS == 0 && THREADS % kRowChunks == 0, "whole jobs");
    static_assert(RC ? kRowStep % (Type<T>::kBytes == 4 ? 8 : 4) == 0 : kRowStep % 16 == 0, "places repeat from job to job");

    const char *base;
    int64_t ld, bytes;
    int line, chunk;           // LDS line (row or k) and source chunk of job 0
    int count;
    unsigned off[kJobs];
    u32x4 reg[DMA ? 1 : kJobs];

    __device__ __forceinline__ void open(const Operand &o)
    {
        base = o.base;
        ld = o.ld;
        bytes = o.bytes;
        count = (int)(o.count < 0 ? 0 : (o.count > R ? R : o.count));
        const int tid = threadIdx.x;
        line = tid / kRowChunks;
        const int place = tid % kRowChunks;
        chunk = RC ? place ^ rc_shift<T, R>(line) : place ^ ((line >> 1) & 7);
        if (DMA) {
#pragma unroll
            for (int j = 0; j < kJobs; ++j) {
                const int row = line + j * kRowStep;
                const bool there = RC ? chunk * chunk_n<T>() < count : row < count;
                off[j] = there ? (unsigned)(row * ld) + (unsigned)chunk * 16u : kOutside;
            }
        }
    }
    // The stage at k0 (of K in all) to `lds`, or to registers.
    __device__ __forceinline__ void fetch(int64_t k0, int64_t K, char *lds)
    {
        const int64_t left = K - k0;
        const char *at = base + (RC ? k0 * ld : k0 * Type<T>::kBytes);
        if (DMA) {
            const __amdgpu_buffer_rsrc_t r =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, 0x7fffffff, kBufferFlags);
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
            typedef __attribute__((address_space(3))) void lds_void;
#pragma unroll
            for (int j = 0; j < kJobs; ++j) {
                unsigned o = off[j];
                if (left < stage_k<T>()) {
                    const int64_t k = RC ? line + j * kRowStep : chunk * chunk_n<T>();
                    if (k >= left) o = kOutside;
                }
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(lds + j * THREADS * 16 + wave * 1024), 16, o, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kJobs; ++j) {
                const int row = line + j * kRowStep;
                u32x4 v = {0, 0, 0, 0};
                const int64_t where = (int64_t)row * ld + chunk * 16;
                const int64_t avail = bytes - (at - base) - where;
                if (RC) {
                    if (row < left && chunk * chunk_n<T>() < count) v = chunk_at<T>(at + where, avail);
                } else if (row < count && chunk * chunk_n<T>() < left) {
                    v = chunk_at<T>(at + where, avail);
                    v = keep_first<T>(v, left - chunk * chunk_n<T>());
                }
                reg[j] = v;
            }
        }
    }
    __device__ __forceinline__ void put(char *lds)
    {
#pragma unroll
        for (int j = 0; j < kJobs; ++j) *reinterpret_cast<u32x4 *>(lds + (threadIdx.x + j * THREADS) * 16) = reg[DMA ? 0 : j];
    }
};

// Reads operands of the matrix instruction from a stage: block of 32 rows or columns at 32 * t + first, step kk of 4.
template <class T, int R, bool RC> struct Reader {
    int at[4];              // KC: by kk; RC: unused
    int lane, first;

    __device__ __forceinline__ void open(int first_)
    {
        lane = threadIdx.x & 63;
        first = first_;
        if (!RC) {
            const int row = first + (lane & 31);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                at[kk] = row * kStageBytes + (((2 * kk + (lane >> 5)) ^ ((row >> 1) & 7)) << 4);
        }
    }
    __device__ __forceinline__ u32x4 read(const char *lds, int t, int kk) const
    {
        if (!RC) return *reinterpret_cast<const u32x4 *>(lds + at[kk] + t * 32 * kStageBytes);
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
};

template <int N> __device__ __forceinline__ void wait_loads()      // until at most N of a wave's loads are under way
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All waves' LDS reads and writes so far are done.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A tile of BM x BN by WM x WN waves.
template <class T_, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool PRC_, bool QRC_, bool DMA_> struct Tile {
    using T = T_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = DMA_ ? STAGES_ : 2, THREADS = 64 * WM * WN;
    static constexpr bool PRC = PRC_, QRC = QRC_, DMA = DMA_;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;      // 32 x 32 tiles of a wave
    static constexpr int kLdsP = BM * kStageBytes, kLdsQ = BN * kStageBytes, kLdsStage = kLdsP + kLdsQ;
    static constexpr int kLds = STAGES * kLdsStage;
    using Acc = f32x16[TM][TN];
    using LoadP = Loader<T, BM, PRC, THREADS, DMA>;
    using LoadQ = Loader<T, BN, QRC, THREADS, DMA>;

    static __device__ __forceinline__ void clear(Acc &acc)
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    }

    static __device__ __forceinline__ void step(const char *lds, const Reader<T, BM, PRC> &rp, const Reader<T, BN, QRC> &rq, Acc &acc)
    {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            u32x4 p[TM], q[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) p[i] = rp.read(lds, i, kk);
#pragma unroll
            for (int j = 0; j < TN; ++j) q[j] = rq.read(lds + kLdsP, j, kk);
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
        Reader<T, BM, PRC> rp;
        Reader<T, BN, QRC> rq;
        rp.open(wave / WN * (BM / WM));
        rq.open(wave % WN * (BN / WN));
        const int steps = (int)((k1 - k0 + stage_k<T>() - 1) / stage_k<T>());
        if (DMA) {
            constexpr int L = LoadP::kJobs + LoadQ::kJobs;
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) {
                lp.fetch(k0 + (int64_t)s * stage_k<T>(), k1, lds + s * kLdsStage);
                lq.fetch(k0 + (int64_t)s * stage_k<T>(), k1, lds + s * kLdsStage + kLdsP);
            }
            int from = 0, to = STAGES - 1;
            for (int s = 0; s < steps; ++s) {
                wait_loads<(STAGES - 2) * L>();
                meet();
                const int64_t k = k0 + (int64_t)(s + STAGES - 1) * stage_k<T>();
                lp.fetch(k, k1, lds + to * kLdsStage);
                lq.fetch(k, k1, lds + to * kLdsStage + kLdsP);
                step(lds + from * kLdsStage, rp, rq, acc);
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
                    lp.fetch(k0 + (int64_t)(s + 1) * stage_k<T>(), k1, nullptr);
                    lq.fetch(k0 + (int64_t)(s + 1) * stage_k<T>(), k1, nullptr);
                }
                step(lds + (s & 1) * kLdsStage, rp, rq, acc);
                if (more) {
                    lp.put(lds + ((s + 1) & 1) * kLdsStage);
                    lq.put(lds + ((s + 1) & 1) * kLdsStage + kLdsP);
                }
            }
        }
        meet();
    }

    // Entries (row, column) of the tile inside rows x cols to out (ld entries from row to row), four columns at a time;
    // vec: out + row * ld is a multiple of four entries' bytes for each row.
    template <class O>
    static __device__ __forceinline__ void store(const Acc &acc, O *out, int64_t ld, int64_t rows, int64_t cols, bool vec, float scale = 1.f)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
        const int r0 = wave / WN * (BM / WM) + (lane & 31), c0 = wave % WN * (BN / WN) + 4 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int row = r0 + 32 * i;
            if (row >= rows) continue;
            O *line = out + (int64_t)row * ld;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int col = c0 + 32 * j + 8 * v;
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * v + e] * scale;
                    if (vec && col + 4 <= cols) {
                        if constexpr (sizeof(O) == 4)
                            *reinterpret_cast<f32x4 *>(line + col) = f32x4{x[0], x[1], x[2], x[3]};
                        else
                            *reinterpret_cast<u32x2 *>(line + col) = u32x2{Type<O>::round2(x[0], x[1]), Type<O>::round2(x[2], x[3])};
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < cols) line[col + e] = Type<O>::round(x[e]);
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

// Row tiles of BM rows of all ranges, in order; every wave looks by itself, 64 ranges at a time.  Returns how many there are;
// where `want` is one of them, its range g and rows [r0, r1).
struct Found {
    int g;
    int64_t r0, r1;
};
__device__ __forceinline__ int count_tiles(const int64_t *offsets, int groups, int64_t rows, int BM)
{
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int base = 0; base < groups; base += 64) {
        int nt = 0;
        if (base + lane < groups) {
            int64_t lo, hi;
            range_of(offsets, base + lane, rows, lo, hi);
            nt = (int)((hi - lo + BM - 1) / BM);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) nt += __shfl_xor(nt, d);
        total += nt;
    }
    return __builtin_amdgcn_readfirstlane(total);
}
__device__ __forceinline__ bool find_tile(const int64_t *offsets, int groups, int64_t rows, int BM, int want, Found &f)
{
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < groups; base += 64) {
        int nt = 0;
        int64_t lo = 0, hi = 0;
        if (base + lane < groups) {
            range_of(offsets, base + lane, rows, lo, hi);
            nt = (int)((hi - lo + BM - 1) / BM);
        }
        int sum = nt;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        const unsigned long long past = __ballot(sum > want);
        if (past) {
            const int l = __ffsll(past) - 1;
            const int before = __shfl(sum - nt, l);
            const int64_t l0 = __shfl(lo, l), h0 = __shfl(hi, l);
            f.g = __builtin_amdgcn_readfirstlane(base + l);
            const int64_t r0 = l0 + (int64_t)(want - before) * BM;
            f.r0 = r0;
            f.r1 = h0 < r0 + BM ? h0 : r0 + BM;
            return true;
        }
        want -= __shfl(sum, 63);
    }
    return false;
}
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

// Workgroups are dealt to the eight dies in turn, each with a cache of its own: a die gets neighbouring tiles.
__device__ __forceinline__ int by_die(int id, int total)
{
    const int each = total / 8, more = total % 8, die = id % 8, nth = id / 8;
    return die < more ? die * (each + 1) + nth : more * (each + 1) + (die - more) * each + nth;
}

}  // namespace ragged
}  // namespace nmfmu
