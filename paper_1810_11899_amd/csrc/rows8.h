// Internal declarations of the 8-bit rows (rows8.hip) and the tile products
// (product.hip) shared by the entry points that use them.
#pragma once

#include "common.h"
#include "gcn_rows8.h"

namespace gcn {

constexpr int32_t kMostRows = 0x7FFFFE00;   // of an operand
constexpr int kRows8Block = 128;   // columns (and, for weights, rows) under one scale
inline int64_t blocks8(int64_t f) { return (f + kRows8Block - 1) / kRows8Block; }

// 16 bytes at any element's address: global memory needs no more alignment, and
// rows of an odd length would take eight loads or stores otherwise
__device__ __forceinline__ uint4 load16(const void *p) {
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
__device__ __forceinline__ void store16(void *p, uint4 v) { __builtin_memcpy(p, &v, 16); }

// ---------------------------------------------------------------- products
// C[M x N] = A B^T on the matrix cores, A [M x K] and B [N x K] in rows of kt
// 128-byte pieces (32 float32, 64 bfloat16 or 128 e4m3 values), 16-byte aligned, the
// columns past K zero in at least one of them and finite in the other.
// Operands stored along the other way (k-major; TN, NN) have kt pieces of 64
// (float32: 32) rows and rows of whole 16-byte chunks (M and N rounded up to 8,
// float32 to 4, elements are readable);
// the rows past K are zero in one operand and finite in the other.
enum TileType {
    TILE_BF16 = 0,       // bfloat16 operands
    TILE_FP8 = 1,        // e4m3 operands with scales, 8-bit matrix instructions
    TILE_FP8_EXACT = 2,  // the same, as bfloat16 products (exact), one float32 sum per 128 columns
    TILE_BF16_TN = 3,    // C = A^T B of bfloat16 operands stored K x M and K x N
    TILE_BF16_NN = 4,    // C = A B, A bfloat16 rows and B stored K x N
    TILE_F32 = 5,        // the three for float32 operands and products
    TILE_F32_TN = 6,
    TILE_F32_NN = 7
};
enum TileEpilogue {
    TILE_STORE = 0,    // C as bfloat16, bias, ReLU
    TILE_PARTIAL = 1,  // split s's sums to acc + s M N (float32), or added to what is there
    TILE_STATS = 2,    // per row and column tile: maximum and sum of exponentials
    TILE_GRAD = 3,     // softmax gradient rows, column sums
    TILE_STORE_F32 = 4, // C as float32, bias, ReLU
    TILE_STATS_STORE = 5   // TILE_STATS, and C as float32
};
struct TileProduct {
    const uint8_t *A, *B;
    int64_t lda, ldb;        // bytes
    int32_t M, N, kt;
    int32_t splits;          // TILE_PARTIAL only, else 1
    // scales of 8-bit operands: A's of row i, piece k at sa[i * ldsa + k]; B's
    // of row j, piece k at sb[(j / 128) * sb_n + k * sb_k]
    const uint8_t *sa, *sb;
    int64_t ldsa, sb_n, sb_k;
    // TILE_STORE, TILE_STORE_F32, TILE_STATS_STORE
    void *C;
    int64_t ldc;             // elements
    int relu;
    const float *bias;       // [N] or null (also TILE_STATS and TILE_GRAD)
    const float *scale;      // [1] or null: a factor of the sums (TILE_GRAD: of the column sums)
    // TILE_PARTIAL
    float *acc;
    int accumulate;
    // TILE_STATS, TILE_GRAD: column j of C is class class0 + j
    // of `classes`; a row whose label is none of them has no gradient
    const int32_t *labels;
    int32_t class0, classes;
    float *tile_max, *tile_sum;     // [tiles_n x M]
    float *label_logit;             // [M]
    const float *row_max, *log_sum; // [M]: a row's softmax is exp((x - row_max) - log_sum)
    uint16_t *G;                    // [g_rows x ldg] bfloat16, zeros past M and N
    int64_t ldg, g_rows;
    float *colpart;                 // [tiles_m x N]
};
// rows and columns of the tiles that this product runs on
struct TileShape {
    int32_t m, n;
};
TileShape tile_shape(TileType type, const TileProduct &p);
// rows of tiles (with TILE_GRAD they cover the rows of zeros behind the last one)
int32_t tile_rows(TileShape t, TileEpilogue epi, const TileProduct &p);
int tile_product(TileType type, TileEpilogue epi, const TileProduct &p, hipStream_t s);
// A B^T with TILE_PARTIAL, and A^T B with `epi` (TILE_PARTIAL, or TILE_STORE and
// with float32 TILE_STORE_F32), of bfloat16 or float32 operands; neither is empty, and
// neither reads what the other writes.  In one launch where both run on small tiles
int tile_products(bool f32, const TileProduct &nt, const TileProduct &tn, TileEpilogue epi, hipStream_t s);
// out (float32, or bfloat16 rows of ldo) = the sum of `splits` partials M x N, in
// order, times *scale, plus bias [N], through the ReLU, where given; out2 [N2] =
// the column sums of acc2 [rows2 x N2] in the same launch
int tile_reduce(int32_t splits, int32_t M, int32_t N, const float *acc, void *out, int out_bf16, int64_t ldo,
                hipStream_t s, int32_t rows2 = 0, int32_t N2 = 0, const float *acc2 = nullptr, float *out2 = nullptr,
                const float *scale = nullptr, const float *bias = nullptr, int relu = 0);
// how many parts to split `kt` pieces over, for a product with few tiles
int32_t tile_splits(int32_t M, int32_t N, int32_t kt, bool f32);

// ------------------------------------------------------------ 8-bit rows
int check_rows8(const gcn_rows8 *r, const char *who);
int rows8_pack(int32_t n, int32_t f, const void *X, int x_bf16, int64_t ldx, uint8_t *q, int64_t ldq,
               uint8_t *scale, int64_t lds, hipStream_t s);

}  // namespace gcn
