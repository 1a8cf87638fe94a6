// Launchers of the products over ragged ranges of rows (grouped products, low-rank adapters), one set per type.
// Not part of the public ABI (that is include/nmfmu_ragged.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace nmfmu {
namespace ragged {

// Tile shapes of the product kernels (gradients: those of as many rows as columns).
enum Shape { k256x256, k128x128, k64x64, k64x128, k32x128 };
constexpr int kTileRows[] = {256, 128, 64, 64, 32}, kTileCols[] = {256, 128, 64, 128, 128};
constexpr int kShrinkRows = 64, kShrinkCols = 64;
constexpr int kMaxSplits = 16, kMaxRank = 256;
constexpr int kFactorPieces = 3;      // bf16 that hold a float

// Factor pairs of segments of rows.
struct Adapters {
    const int64_t *offsets;      // segments + 1
    const int32_t *run;          // segments
    int32_t segments;
    const int32_t *koff;         // runs + 1
    int32_t runs, kmax;
    int64_t ktotal;              // rows of down and up
    const void *down, *up;       // ktotal x m and ktotal x n
    int64_t ld_down, ld_up;
    const float *scale;          // runs, or null
    float *u;                    // rows x kmax
};

struct Product {
    const void *x;
    int64_t ldx;
    const int64_t *offsets;      // groups + 1, or null: one group of all rows
    int32_t groups;
    int64_t rows, m, n;
    const void *b;
    int64_t ldb, stride_b;
    int32_t transposed;
    void *y;
    int64_t ldy;
    Adapters ad;                 // ad.segments == 0: none
    // plan
    bool padded;                 // operands whose rows do not fill whole 16 bytes are copies that do, with zeros
    int shape, splits;
    bool joined;                 // y comes from parts (one at least), which a second launch joins; needs part
    int64_t k_split;             // k of a split, whole stages
    float *part;                 // splits x rows x (n rounded up to 4)
    int shrink_splits;           // parts of u
    int64_t shrink_k;
    float *upart;                // shrink_splits x rows x kmax, where there are several
    void *pack;                  // u as an operand, rows x 4 bytes x kmax in whole 32s, and for f16 a scale of each row;
    float *row_scale;            // null: none (slow)
    bool vec;                    // rows of y begin on 16-byte borders
};

struct Gradient {
    const void *x, *dy;
    int64_t ldx, ldy;
    const int64_t *offsets;
    int32_t groups;
    int64_t rows, m, n;
    void *g;
    int64_t ldg, stride_g;
    bool padded;                 // as for Product
    int shape, splits;
    float *part;                 // splits x groups x m x (n rounded up to 4)
    bool vec;
};

struct FactorGradient {
    const void *x, *dy;
    int64_t ldx, ldy, rows, m, n;
    Adapters ad;                 // its u, down, up and scale are not used
    const float *u, *v;          // rows x kmax
    void *ddown, *dup;           // ktotal x m, ktotal x n
    void *pieces;                // 16-bit types: u and v in pieces, 2 x rows x kFactorPieces x (kmax in whole tiles) bf16; null: cut where they are used
    int chunk, chunks;           // blocks of rows (factor_rows) to a workgroup, and how many such chunks there can be
    int slots;                   // chunks of runs with several: parts that a second launch joins
    float *part;                 // slots x (kmax in whole tiles) x (m rounded up to 4 + n rounded up to 4)
};

// Rows of a block, and factors of a tile.
constexpr int factor_rows(int bytes, bool f16) { return bytes == 4 || f16 ? 32 : 64; }
inline int factor_tile(int kmax) { return kmax <= 32 ? 32 : 64; }

// Types by their bits (float as it is).
struct bf16_t { unsigned short bits; };
struct f16_t { unsigned short bits; };

// A copy with rows of ldo entries, whole 16 bytes.
struct Align {
    const void *src;
    int64_t ld, stride, rows, cols, count;
    void *dst;
    int64_t ldo;
};
template <class T> hipError_t launch_align(const Align &a, hipStream_t st);
template <class T> hipError_t launch_product(const Product &p, hipStream_t st);
template <class T> hipError_t launch_gradient(const Gradient &p, hipStream_t st);
template <class T> hipError_t launch_factor_gradient(const FactorGradient &p, hipStream_t st);

__host__ __device__ inline int64_t up4(int64_t n) { return (n + 3) / 4 * 4; }

}  // namespace ragged
}  // namespace nmfmu
