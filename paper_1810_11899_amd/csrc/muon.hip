// The orthogonalised update: Newton-Schulz products of up to kGroup matrices in
// common launches.
//
// An iteration on X [m x n] (m <= n; a matrix with more rows than columns is
// laid out transposed) is three products on the tile loops of tiles.h:
//     A = X X^T (rows against rows)    B = b A + c A A (A is symmetric: rows
//     against rows)    X' = a X + B X (X's rows as stored, k-major)
// Everything lies in known bounds: X's singular values in 0 .. 1.2025, A's
// eigenvalues in 0 .. 1.446, B's in -2.807 .. 0, and no element is larger than the
// largest of them.  So float16 holds each, scaled by a power of two, without a
// scale of its own:
//   GCN_F32   X, A and B are pairs, hi + lo of float16 (22 bits and the sign of lo),
//             and a product is the three part products that reach float32's
//             precision; half of what six bfloat16 part products take, which
//             values of any size would need.
//   GCN_BF16  products of the high parts alone; X keeps its low part, for a X.
//             A direction with a small singular value grows a-fold a step by a X
//             alone, and a rounding of X would grow with it: so it is not rounded.
// One power of two for a whole matrix leaves a floor: half a step of float16's smallest
// numbers, 2^-40 of |U| for an element of X, 2^-39 and 2^-38 for one of A and B.  A direction of
// the size s |U| carries it along as it grows, and is 2^-36 / s off at most (rows of unlike
// sizes, CPU model / float32 products: s = 1e-4, 8 steps 1.5e-7 / 1.3e-7, 1e-6, 13 steps 4.7e-6 /
// 6e-7, 1e-10, 20 steps 4.4e-2 / 3e-7).  Only many steps bring such directions up, and at
// the last few of them they are large enough: the steps ahead of the last kPairSteps, or
// kSingleSteps of GCN_BF16, are
//   WHOLE     float32 rows and products, on the same tiles (us, ten steps, pairs alone / so: 50 x 64
//             35 / 110, 602 x 128 137 / 164, 512 x 512 235 / 258, 1024 x 1024 442 / 544, 4096 x
//             4096 7740 / 15,050).
// The diagonals of A and B are the larger part of them (X's rows are nearly
// orthogonal after the first steps), and a rounding there moves a whole row alike.
// So they stay float32, in vectors e and d beside A' and B', which have zeros there:
//     A = e + A'     A A = e^2 + (e_i + e_j) A' + A' A'     X' = (a + d) X + B' X
// a apart from the products matters most where singular values are small: on B's
// diagonal it would be rounded to B's largest element.  Error against float64 (2-norm;
// float32 products throughout / pairs / pairs and diagonals; single products, the same):
//     50 x 64        1.1e-6  1.3e-6  7.0e-7    2.1e-3  8.7e-4
//     512 x 512      2.5e-6  1.6e-6  8.4e-7    1.5e-3  7.0e-4
//     17 x 900       1.6e-6  2.0e-6  1.4e-6    2.8e-3  9.0e-4
//     512 x 1024, 8 directions large
//                    2.0e-5  2.2e-5  2.1e-5 (a on the diagonal: 5.4e-5)    3.3e-4  5.8e-4
#include <algorithm>
#include <cmath>
#include <vector>

#include "gcn_muon.h"
#include "tiles.h"

namespace gcn {
namespace {

constexpr int kTB = 256;
// Matrices of a launch.  Which way of working and which tiles it takes goes by all of them: one with a short side takes
// the 256 x 256 tiles from a wide one (us, 4096 x 4096 and 602 x 128 in one call 4590, in two 3900 + 75; GCN_BF16 2150,
// 1750 + 85), while of like ones the launches are shared (602 x 128 and 50 x 64 75, 75 + 21).
constexpr int kGroup = 16;
constexpr int kMostParts = 1024;  // of a matrix's sum of squares
constexpr int kXBits = 15, kABits = 14, kBBits = 13;   // what X, A and B are scaled by
constexpr float kCoefA = 3.4445f, kCoefB = -4.7750f, kCoefC = 2.0315f;

constexpr float two_to(int k) {
    float v = 1.0f;
    for (int i = 0; i < (k < 0 ? -k : k); ++i) v = k < 0 ? v * 0.5f : v * 2.0f;
    return v;
}

// A matrix of the group.  X0 and X1 [mp x np], A and B [mp x mp] in the workspace:
// pairs in rows of 4 np bytes (32 high parts, 32 low ones, ..), or float16 rows,
// X's low parts in a second plane mp np elements on.
// (What a product needs first stands in its first 64 bytes.)
struct alignas(64) Job {
    uint8_t *X0, *X1, *A, *B;
    int32_t mp, np;
    int32_t rows, cols;
    int64_t ldw;             // of out too
    float step;              // lr * scale
    int32_t parts;
    float *W;                // updated, or null
    void *out;               // orthogonalise's result, or null
    const void *G;           // the gradient, or what is orthogonalised
    float *M;                // momentum, or null
    int64_t ldg, ldm;
    double *part;            // sums of squares
    float *e, *d;            // the diagonals of A and B
    int32_t slab;            // columns of X a workgroup where there are few rows, else 0
};
// A launch's arguments.  The chain of loads from its number to a block's operands is a
// good part of a small launch: the table of first blocks is one line, read
// whole.
struct alignas(64) Group {
    uint32_t first[kGroup];       // a launch's first block of each job, of no job 2^32 - 1
    uint32_t total, per_xcd, band;
    int32_t count;
    int full;                     // A and B: all of their tiles, not those on and below the diagonal alone
    float momentum, decay;
    int nesterov, grad_bf16, out_bf16;
    Job job[kGroup];
};
__device__ __forceinline__ int job_of(const Group &g, uint32_t block) {
    int j = 0;
#pragma unroll
    for (int k = 1; k < kGroup; ++k) j += block >= g.first[k];
    return j;
}

// Four consecutive columns of U from c of row r (zeros past the last), M updated on
// the way with UPDATE.
template <bool UPDATE>
__device__ __forceinline__ f32x4 four_of_u(const Group &g, const Job &J, int64_t r, int32_t c) {
    f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
    if (r >= J.rows || c >= J.cols) return u;
    const bool whole = c + 4 <= J.cols;
    if (g.grad_bf16) {
        const uint16_t *p = (const uint16_t *)J.G + r * J.ldg + c;
        if (whole) {
            uint2 w;
            __builtin_memcpy(&w, p, 8);
            u = f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                      __uint_as_float(w.y & 0xFFFF0000u)};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < J.cols) u[e] = __uint_as_float((uint32_t)p[e] << 16);
        }
    } else {
        const float *p = (const float *)J.G + r * J.ldg + c;
        if (whole) {
            u = __builtin_bit_cast(f32x4, load16(p));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < J.cols) u[e] = p[e];
        }
    }
    if (!J.M) return u;
    float *p = J.M + r * J.ldm + c;
    f32x4 m = {0.0f, 0.0f, 0.0f, 0.0f};
    if (whole) {
        m = __builtin_bit_cast(f32x4, load16(p));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < J.cols) m[e] = p[e];
    }
    if constexpr (UPDATE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = fmaf(g.momentum, m[e], u[e]);
        if (whole) {
            store16(p, __builtin_bit_cast(uint4, m));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < J.cols) p[e] = m[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = g.nesterov ? fmaf(g.momentum, m[e], u[e]) : m[e];
    return u;
}
__device__ __forceinline__ double squares(f32x4 u) {
    return ((double)u[0] * u[0] + (double)u[1] * u[1]) + ((double)u[2] * u[2] + (double)u[3] * u[3]);
}
// the factor that makes X0 of U: of a matrix of zeros 0
__device__ __forceinline__ double inverse_norm(double sum) { return sum > 0.0 ? (double)(1 << kXBits) / sqrt(sum) : 0.0; }

// M <- momentum M + G, and U's sum of squares in float64 (no overflow, and the norm
// of millions of elements to float32's last bit): a block's share of the
// elements, in order.
__global__ __launch_bounds__(kTB) void momentum_kernel(Group g) {
    __shared__ double red[kTB / 64];
    const int j = job_of(g, blockIdx.x);
    const Job &J = g.job[j];
    const uint32_t block = blockIdx.x - g.first[j], per_row = ((uint32_t)J.cols + 3) / 4;
    const uint32_t total = (uint32_t)J.rows * per_row, step = (uint32_t)J.parts * kTB;   // (sides up to 2^16: below 2^31)
    double sum = 0.0;
    for (uint32_t i = block * kTB + threadIdx.x; i < total; i += step)
        sum += squares(four_of_u<true>(g, J, i / per_row, 4 * (i % per_row)));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) J.part[block] = (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ uint16_t half_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ __forceinline__ float half_value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

// What operands are made of: float16, pairs, float32 (see above).
enum Kind { SINGLE = 0, PAIR = 1, WHOLE = 2 };
// The last steps, with pairs or GCN_BF16's operands.  Half of the rows a twentieth of what so many steps bring to one,
// how far they are off (model; pairs for the last 8 / 7 / 6 / 5 steps / float32 products): 20 x 3000 4.7e-6 / 1.4e-6 /
// 4.2e-7 / 1.8e-7 / 1.5e-7, 100 x 300 3.4e-6 / 1.0e-6 / 3.4e-7 / 2.0e-7 / 3.7e-7, 400 x 700 1.0e-5 / 3.0e-6 / 9.0e-7 /
// 3.6e-7 / 7.6e-7.  2^-36 3.4445^12 is a twentieth of what GCN_BF16 leaves, 2^-10.
constexpr int32_t kPairSteps = 6, kSingleSteps = 12;

// Four consecutive elements (column a multiple of 4) of an operand, and back.  `low`:
// bytes from the high parts to the low ones.  bytes: of a row.
template <int KIND>
__device__ __forceinline__ int64_t place(int64_t row, int64_t bytes, int64_t col) {
    return row * bytes + (KIND == PAIR ? pair_place(col) : (KIND == WHOLE ? 4 : 2) * col);
}
__device__ __forceinline__ f32x4 four_of(const uint8_t *p) {
    const uint2 h = *(const uint2 *)p;
    return f32x4{half_value(h.x & 0xFFFFu), half_value(h.x >> 16), half_value(h.y & 0xFFFFu), half_value(h.y >> 16)};
}
__device__ __forceinline__ uint2 four_halves(f32x4 v) {
    return make_uint2((uint32_t)half_bits(v[0]) | (uint32_t)half_bits(v[1]) << 16,
                      (uint32_t)half_bits(v[2]) | (uint32_t)half_bits(v[3]) << 16);
}
// the high parts at p, the low ones `low` bytes on (0: dropped)
__device__ __forceinline__ void store_parts(uint8_t *p, int64_t low, f32x4 v) {
    const uint2 h = four_halves(v);
    *(uint2 *)p = h;
    if (low) {
        const f32x4 hi = {half_value(h.x & 0xFFFFu), half_value(h.x >> 16), half_value(h.y & 0xFFFFu), half_value(h.y >> 16)};
        *(uint2 *)(p + low) = four_halves(v - hi);
    }
}
template <int KIND>
__device__ __forceinline__ void store_four(uint8_t *p, int64_t low, f32x4 v) {
    if constexpr (KIND == WHOLE) *(f32x4 *)p = v;
    else store_parts(p, low, v);
}
template <int KIND>
__device__ __forceinline__ int64_t row_bytes(int32_t cols) { return (int64_t)cols * (KIND == SINGLE ? 2 : 4); }

// X0 = U / |U|, 64 x 64 elements to a block, zeros past U's sides, through LDS
// where U is laid out transposed.
template <int KIND>
__global__ __launch_bounds__(kTB) void operand_kernel(Group g) {
    __shared__ float tile[64][65];
    __shared__ double red[kTB / 64];
    const int j = job_of(g, blockIdx.x);
    const Job &J = g.job[j];
    const uint32_t block = blockIdx.x - g.first[j], across = (uint32_t)((J.np + 63) / 64);
    const int64_t i0 = (int64_t)(block / across) * 64, j0 = (int64_t)(block % across) * 64;   // X's rows, columns
    const bool tall = J.rows > J.cols;
    const int64_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;   // U's
    const int tr = (int)(threadIdx.x >> 4), tc = 4 * (int)(threadIdx.x & 15);
    f32x4 u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = four_of_u<false>(g, J, r0 + 16 * k + tr, (int32_t)c0 + tc);
    double sum = 0.0;
    for (int i = threadIdx.x; i < J.parts; i += kTB) sum += J.part[i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = sum;
    __syncthreads();
    const double inv = inverse_norm((red[0] + red[1]) + (red[2] + red[3]));
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) u[k][e] = (float)((double)u[k][e] * inv);
    if (tall) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) tile[tc + e][16 * k + tr] = u[k][e];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) u[k][e] = tile[16 * k + tr][tc + e];
    }
    const int64_t bytes = row_bytes<KIND>(J.np), low = KIND == PAIR ? 64 : 2 * (int64_t)J.mp * J.np;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i0 + 16 * k + tr < J.mp && j0 + tc < J.np)
            store_four<KIND>(J.X0 + place<KIND>(i0 + 16 * k + tr, bytes, j0 + tc), low, u[k]);
}

// (TO_PAIR, TO_SINGLE: the next X of float32 products in the layout of the steps behind them)
enum Stage { GRAM = 0, POLY = 1, NEXT = 2, LAST = 3, TO_PAIR = 4, TO_SINGLE = 5 };

// What a product's epilogue reads beside four sums: A's or X's elements at their
// place, and A's diagonal at their row and columns or B's at their row.
struct Old {
    f32x4 v, cols;
    float row;
};
template <int KIND, int STAGE>
__device__ __forceinline__ f32x4 elements_at(const Job &J, const uint8_t *X, int row, int col) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (STAGE == GRAM) return v;
    const int32_t cols = STAGE == POLY ? J.mp : J.np;
    if (row < J.mp && col < cols) {
        const uint8_t *p = (STAGE == POLY ? J.A : X) + place<KIND>(row, row_bytes<KIND>(cols), col);
        if constexpr (KIND == WHOLE) return *(const f32x4 *)p;
        v = four_of(p);
        // (A of the single products is its high parts alone)
        if constexpr (KIND == PAIR) v += four_of(p + 64);
        else if (STAGE != POLY) v += four_of(p + 2 * (int64_t)J.mp * J.np);
    }
    return v;
}
template <int STAGE>
__device__ __forceinline__ float diagonal_at(const Job &J, int row) {
    if constexpr (STAGE == GRAM) return 0.0f;
    else return (STAGE == POLY ? J.e : J.d)[min(row, J.mp - 1)];
}
template <int STAGE>
__device__ __forceinline__ f32x4 diagonals_at(const Job &J, int col) {
    if constexpr (STAGE != POLY) return f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    else return *(const f32x4 *)(J.e + min(col, J.mp - 4));
}
template <int KIND, int STAGE>
__device__ __forceinline__ Old old_at(const Job &J, const uint8_t *X, int row, int col) {
    return Old{elements_at<KIND, STAGE>(J, X, row, col), diagonals_at<STAGE>(J, col), diagonal_at<STAGE>(J, row)};
}
// A's four elements at (row, col ..) from their sums, and B's from the sums of A' A';
// those of the diagonal go to *diagonal and leave zero
__device__ __forceinline__ f32x4 gram_of(f32x4 sum, int row, int col, float *diagonal) {
    f32x4 v = sum * two_to(kABits - 2 * kXBits);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (row == col + k) {
            *diagonal = sum[k] * two_to(-2 * kXBits);
            v[k] = 0.0f;
        }
    return v;
}
__device__ __forceinline__ f32x4 poly_of(f32x4 sum, f32x4 a, float e_row, f32x4 e_cols, int row, int col, float *diagonal) {
    f32x4 v = (sum * two_to(-kABits) + (e_cols + e_row) * a) * (kCoefC * two_to(kBBits - kABits)) +
              a * (kCoefB * two_to(kBBits - kABits));
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (row == col + k) {
            *diagonal = kCoefC * (sum[k] * two_to(-2 * kABits) + e_row * e_row) + kCoefB * e_row;
            v[k] = 0.0f;
        }
    return v;
}

// v of four consecutive columns of a row to four consecutive rows of a column: lane
// 4 q + k of a row of 16 gives element e to lane 4 q + e and takes element k of
// it.  In two exchanges, of single columns and of pairs.
__device__ __forceinline__ f32x4 turned(f32x4 v) {
    const bool odd = threadIdx.x & 1, up = threadIdx.x & 2;
    const float a = __shfl_xor(odd ? v[0] : v[1], 1), b = __shfl_xor(odd ? v[2] : v[3], 1);
    v = odd ? f32x4{a, v[1], b, v[3]} : f32x4{v[0], a, v[2], b};
    const float c = __shfl_xor(up ? v[0] : v[2], 2), d = __shfl_xor(up ? v[1] : v[3], 2);
    return up ? f32x4{c, d, v[2], v[3]} : f32x4{v[0], v[1], c, d};
}

// W <- decay W - step O, or out = O, for four consecutive columns of a row of O, a
// wavefront's 16 x 16 at a time.
__device__ __forceinline__ void apply(const Group &g, const Job &J, int row, int col, f32x4 o) {
    if (J.rows > J.cols) {   // O lies transposed
        o = turned(o);
        const int r = col + (row & 3);
        col = row & ~3;
        row = r;
    }
    if (row >= J.rows) return;
    const int64_t at = (int64_t)row * J.ldw + col;
    if (col + 4 <= J.cols) {
        if (J.W) {
            const f32x4 w = __builtin_bit_cast(f32x4, load16(J.W + at));
            store16(J.W + at, __builtin_bit_cast(uint4, g.decay * w - J.step * o));
        } else if (g.out_bf16) {
            const uint2 v = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
            __builtin_memcpy((uint16_t *)J.out + at, &v, 8);
        } else {
            store16((float *)J.out + at, __builtin_bit_cast(uint4, o));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (col + e >= J.cols) continue;
        if (J.W) J.W[at + e] = g.decay * J.W[at + e] - J.step * o[e];
        else if (g.out_bf16) ((uint16_t *)J.out)[at + e] = to_bf16(o[e]);
        else ((float *)J.out)[at + e] = o[e];
    }
}

// Four sums to what the product forms.  mirror: of a tile below the diagonal of A or
// B, whose other half they are too.
template <int KIND, int STAGE>
__device__ __forceinline__ void finish(const Group &g, const Job &J, uint8_t *next, int row, int col, bool mirror,
                                       const Old &old, f32x4 v) {
    constexpr int TO = STAGE == TO_PAIR ? PAIR : STAGE == TO_SINGLE ? SINGLE : KIND;
    const int32_t cols = STAGE <= POLY ? J.mp : J.np;
    const int64_t bytes = row_bytes<TO>(cols);
    // (A and B of the single products are their high parts alone)
    const int64_t low = TO == PAIR ? 64 : STAGE <= POLY ? 0 : 2 * (int64_t)J.mp * J.np;
    const bool in = row < J.mp && col < cols;
    if constexpr (STAGE <= POLY) {
        if (in) {
            if constexpr (STAGE == GRAM) v = gram_of(v, row, col, J.e + row);
            else v = poly_of(v, old.v, old.row, old.cols, row, col, J.d + row);
        }
        uint8_t *const to = STAGE == GRAM ? J.A : J.B;
        if (in) store_four<TO>(to + place<TO>(row, bytes, col), low, v);
        if (mirror) {   // (all lanes exchange; mp is a multiple of 32: a block of 16 x 16 is in or out)
            v = turned(v);
            if (in) store_four<TO>(to + place<TO>(col + (row & 3), bytes, row & ~3), low, v);
        }
    } else {
        if (!in) return;
        v = v * two_to(-kBBits) + old.v * (kCoefA + old.row);
        if constexpr (STAGE != LAST) store_four<TO>(next + place<TO>(row, bytes, col), low, v);
        else apply(g, J, row, col, v * two_to(-kXBits));
    }
}

template <int KIND, int STAGE>
constexpr int type_of() {
    if (KIND == WHOLE) return STAGE <= POLY ? TILE_F32 : TILE_F32_NN;
    return STAGE <= POLY ? (KIND == PAIR ? TILE_PAIR : TILE_F16) : (KIND == PAIR ? TILE_PAIR_NN : TILE_F16_NN);
}

// A tile of a product of one of the group's matrices.  odd: X is in X1.  The
// group's tiles are numbered matrix by matrix and dealt to the XCDs in eight
// runs, so that a matrix is read by as few L2s as can be; within a matrix in
// bands of `band` row tiles (A and B: tiles on and below the diagonal, row by row).
template <int KIND, int STAGE, int BM, int BN>
__device__ __forceinline__ void product_of(const Group &g, const Job &J, const uint8_t *X, uint32_t at, TileProduct &p,
                                           Coord &c) {
    constexpr int kUnit = KIND == SINGLE ? 64 : 32;   // columns of a piece
    p.M = J.mp;
    if constexpr (STAGE == GRAM) {
        p.A = p.B = X;
        p.lda = p.ldb = row_bytes<KIND>(J.np);
        p.N = J.mp;
        p.kt = J.np / kUnit;
    } else if constexpr (STAGE == POLY) {
        p.A = p.B = J.A;
        p.lda = p.ldb = row_bytes<KIND>(J.mp);
        p.N = J.mp;
        p.kt = J.mp / kUnit;
    } else {
        p.A = J.B;
        p.lda = row_bytes<KIND>(J.mp);
        p.B = X;
        p.ldb = row_bytes<KIND>(J.np);
        p.N = J.np;
        p.kt = J.mp / kUnit;
    }
    c.split = 0;
    if (STAGE <= POLY && !g.full) {
        // row t of the triangle starts at t (t + 1) / 2
        int t = (int)((sqrtf(8.0f * (float)at + 1.0f) - 1.0f) * 0.5f);
        while ((uint32_t)(t + 1) * (t + 2) / 2 <= at) ++t;
        while ((uint32_t)t * (t + 1) / 2 > at) --t;
        c.tm = t;
        c.tn = (int)(at - (uint32_t)t * (t + 1) / 2);
    } else {
        const uint32_t tiles_m = (uint32_t)(p.M + BM - 1) / BM, tiles_n = (uint32_t)(p.N + BN - 1) / BN;
        const uint32_t b = at / (g.band * tiles_n), q = at - b * g.band * tiles_n, h = min(g.band, tiles_m - b * g.band);
        c.tn = (int)(q / h);
        c.tm = (int)(b * g.band + (q - c.tn * h));
    }
    // (the same in every lane, and the copies take their bases in scalar registers)
    c.tm = __builtin_amdgcn_readfirstlane(c.tm);
    c.tn = __builtin_amdgcn_readfirstlane(c.tn);
}

// The block's tile, or the end of the block where it has none.
#define GCN_MUON_TILE(BM, BN)                                                     \
    const uint32_t L = (blockIdx.x & 7) * g.per_xcd + (blockIdx.x >> 3);       \
    if (L >= g.total) return;                                                  \
    const int job = job_of(g, L);                                              \
    const Job &J = g.job[job];                                                 \
    const uint8_t *const X = odd ? J.X1 : J.X0;                                \
    uint8_t *const next = odd ? J.X0 : J.X1;                                   \
    TileProduct p{};                                                           \
    Coord c;                                                                   \
    product_of<KIND, STAGE, BM, BN>(g, J, X, L - g.first[job], p, c);          \
    const bool mirror = STAGE <= POLY && !g.full && c.tm != c.tn

// KG groups of WM x WN wavefronts take a KG-th of the sum each, and share the tile's
// epilogue: a launch of fewer tiles than CUs has one wavefront a SIMD and group,
// which waits for its own copies, reads and products in turn.
template <int KIND, int STAGE, int BM, int BN, int WM, int WN, int KG>
__global__ __launch_bounds__(64 * WM *WN *KG) void muon_kernel(Group g, int odd) {
    constexpr int TYPE = type_of<KIND, STAGE>(), T = 64 * WM * WN;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16, kBlocks = FM * FN, kOwn = kBlocks < KG ? 1 : kBlocks / KG;
    constexpr int kLds = small_lds(TYPE, BM, BN);
    static_assert(KG == 1 || kBlocks * T * 16 <= kLds, "the groups' sums fit where the operands were");
    __shared__ __attribute__((aligned(16))) char lds[KG * kLds];
    GCN_MUON_TILE(BM, BN);
    const uint32_t tid = threadIdx.x % T;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / T), lane = tid & 63, wave = tid >> 6;
    const int r0 = c.tm * BM + wave / WN * (BM / WM) + (lane & 15), c0 = c.tn * BN + wave % WN * (BN / WN) + 4 * (lane >> 4);
    constexpr bool kAhead = kOwn <= 4;   // (a few registers)
    Old old[kAhead ? kOwn : 1];
    if constexpr (kAhead) {
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
            const int b = u * KG + group;
            old[u] = old_at<KIND, STAGE>(J, X, r0 + 16 * (b / FN), c0 + 16 * (b % FN));
        }
    }
    f32x4 acc[FM][FN];
    const int per = (p.kt + KG - 1) / KG, k0 = min(group * per, p.kt);
    small_loop<TYPE, BM, BN, WM, WN>(p, c, k0, min(per, p.kt - k0), lds + group * kLds, acc, tid, per);
    if constexpr (KG > 1) {
        f32x4 *const part = (f32x4 *)lds;   // [block][group][thread]
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) part[(b * KG + group) * T + tid] = acc[b / FN][b % FN];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
            const int b = u * KG + group;
            if (kBlocks < KG && b >= kBlocks) break;   // (more parts than blocks: a wavefront has none)
            f32x4 v = part[b * KG * T + tid];
#pragma unroll
            for (int q = 1; q < KG; ++q) v += part[(b * KG + q) * T + tid];
            finish<KIND, STAGE>(g, J, next, r0 + 16 * (b / FN), c0 + 16 * (b % FN), mirror,
                                kAhead ? old[kAhead ? u : 0] : old_at<KIND, STAGE>(J, X, r0 + 16 * (b / FN), c0 + 16 * (b % FN)), v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const Old o = kAhead ? old[kAhead ? i * FN + j : 0] : old_at<KIND, STAGE>(J, X, r0 + 16 * i, c0 + 16 * j);
                finish<KIND, STAGE>(g, J, next, r0 + 16 * i, c0 + 16 * j, mirror, o, acc[i][j]);
            }
    }
}
template <int KIND, int STAGE>
__global__ __launch_bounds__(kBigThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void muon_big_kernel(Group g, int odd) {
    constexpr int TYPE = type_of<KIND, STAGE>();
    __shared__ __attribute__((aligned(16))) char lds[big_lds(TYPE)];
    GCN_MUON_TILE(kBigT, kBigT);
    f32x4 acc[8][4];
    big_loop<TYPE>(p, c, 0, p.kt, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = c.tm * kBigT + (wave >> 2) * 128 + (lane & 15), c0 = c.tn * kBigT + (wave & 3) * 64 + 4 * (lane >> 4);
    f32x4 cols[4];
    float rows[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) cols[k] = diagonals_at<STAGE>(J, c0 + 16 * k);
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[i] = diagonal_at<STAGE>(J, r0 + 16 * i);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {   // (two rows' reads at a time)
        f32x4 old[2][4];
#pragma unroll
        for (int k = 0; k < 8; ++k) old[k / 4][k % 4] = elements_at<KIND, STAGE>(J, X, r0 + 16 * (i + k / 4), c0 + 16 * (k % 4));
#pragma unroll
        for (int k = 0; k < 8; ++k)
            finish<KIND, STAGE>(g, J, next, r0 + 16 * (i + k / 4), c0 + 16 * (k % 4), mirror,
                                Old{old[k / 4][k % 4], cols[k % 4], rows[i + k / 4]}, acc[i + k / 4][k % 4]);
    }
}

// ------------------------------------------------------------- small matrices
// A whole update of a matrix whose X and A fit in LDS as pairs, by one workgroup: no
// launches between the products.  X and A lie as pieces of 32 columns, a
// row's 128 bytes (high parts, low parts) beside the next row's, chunk c of row r at
// c ^ (r % 8), so that 16 rows' chunks are on different banks.  B takes A's place.
// A and B: a wavefront has one block of 16 TS x 16 TS.  a X + B X: a wavefront has
// 16 columns of X at a time, which no other reads, and writes them back in place.
// us, in launches of their own / here: 50 x 64 51 / 20, 64 x 560 62 / 55, 128 x 128
// 64 / 55, 128 x 160 65 / 62, sixteen of 128 x 128 75 / 58.
constexpr int kSmallLds = 160 << 10, kSmallThreads = 1024, kSmallSide = 128;
bool fits_lds(int64_t mp, int64_t np) { return mp <= kSmallSide && 4 * mp * (mp + np + 2) <= kSmallLds; }

struct Resident {
    char *base;
    int step;     // bytes from a piece of 32 columns to the next, 128 a row
    // of column c's high part in row r; its low part lies at the place of chunk + 4
    __device__ __forceinline__ char *at(int r, int c, int part) const {
        return base + c / 32 * step + r * 128 + (((c % 32 / 8 + 4 * part) ^ (r & 7)) * 16) + c % 8 * 2;
    }
    // 16 rows against a piece of 32 columns
    __device__ __forceinline__ Frag rows(int r0, int piece, int lane) const {
        const int fr = lane & 15, g = lane >> 4;
        const char *q = base + piece * step + (r0 + fr) * 128;
        return Frag{*(const uint4 *)(q + (g ^ (fr & 7)) * 16), *(const uint4 *)(q + ((g + 4) ^ (fr & 7)) * 16)};
    }
    // 16 columns from c0 against 32 rows
    __device__ __forceinline__ Frag columns(int piece, int c0, int lane) const {
        const int r = 32 * piece + 8 * (lane >> 4) + ((lane & 15) >> 2), c = c0 + 4 * (lane & 3);
        const uint2 a = km_read(at(r, c, 0)), b = km_read(at(r + 4, c, 0)), d = km_read(at(r, c, 1)), e = km_read(at(r + 4, c, 1));
        return Frag{make_uint4(a.x, a.y, b.x, b.y), make_uint4(d.x, d.y, e.x, e.y)};
    }
    __device__ __forceinline__ f32x4 four(int r, int c) const {
        return four_of((const uint8_t *)at(r, c, 0)) + four_of((const uint8_t *)at(r, c, 1));
    }
    __device__ __forceinline__ void put(int r, int c, f32x4 v) const {
        const uint2 h = four_halves(v);
        *(uint2 *)at(r, c, 0) = h;
        const f32x4 hi = {half_value(h.x & 0xFFFFu), half_value(h.x >> 16), half_value(h.y & 0xFFFFu), half_value(h.y >> 16)};
        *(uint2 *)at(r, c, 1) = four_halves(v - hi);
    }
    __device__ __forceinline__ void put_one(int r, int c, float v) const {
        const uint16_t h = half_bits(v);
        *(uint16_t *)at(r, c, 0) = h;
        *(uint16_t *)at(r, c, 1) = half_bits(v - half_value(h));
    }
};

// The wavefront's block of P P^T, P's rows against each other over `pieces`.
template <int TS>
__device__ __forceinline__ void block_of(const Resident &P, int pieces, int i0, int j0, int lane, f32x4 (&acc)[TS][TS]) {
#pragma unroll
    for (int i = 0; i < TS; ++i)
#pragma unroll
        for (int j = 0; j < TS; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int t = 0; t < pieces; ++t) {
        Frag b[TS];
#pragma unroll
        for (int j = 0; j < TS; ++j) b[j] = P.rows(j0 + 16 * j, t, lane);
#pragma unroll
        for (int i = 0; i < TS; ++i) {
            const Frag a = P.rows(i0 + 16 * i, t, lane);
#pragma unroll
            for (int j = 0; j < TS; ++j) mma<TILE_PAIR>(acc[i][j], a, b[j], 0, 0);
        }
    }
}
// The wavefront's block of an mp x mp matrix, if it has one: rows i0 .., columns j0 ...
template <int TS>
struct Block {
    int i0, j0;
    bool mine;
    __device__ __forceinline__ Block(int mp, int wave) {
        const int across = mp / (16 * TS);
        i0 = wave / across * 16 * TS;
        j0 = wave % across * 16 * TS;
        mine = wave < across * across;
    }
};
// A = X X^T; every wavefront calls it
template <int TS>
__device__ __forceinline__ void gram(const Resident &X, const Resident &A, float *e, int mp, int np, int lane, int wave) {
    const Block<TS> b(mp, wave);
    if (b.mine) {
        f32x4 acc[TS][TS];
        block_of<TS>(X, np / 32, b.i0, b.j0, lane, acc);
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int j = 0; j < TS; ++j) {
                const int row = b.i0 + 16 * i + (lane & 15), col = b.j0 + 16 * j + 4 * (lane >> 4);
                A.put(row, col, gram_of(acc[i][j], row, col, e + row));
            }
    }
    __syncthreads();
}
// B in A's place; every wavefront calls it
template <int TS>
__device__ __forceinline__ void poly(const Resident &A, const float *e, float *d, int mp, int lane, int wave) {
    const Block<TS> b(mp, wave);
    const int r0 = b.i0 + (lane & 15), c0 = b.j0 + 4 * (lane >> 4);
    f32x4 acc[TS][TS];
    if (b.mine) {
        block_of<TS>(A, mp / 32, b.i0, b.j0, lane, acc);
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int j = 0; j < TS; ++j) {
                const int row = r0 + 16 * i, col = c0 + 16 * j;
                acc[i][j] = poly_of(acc[i][j], A.four(row, col), e[row], *(const f32x4 *)(e + col), row, col, d + row);
            }
    }
    __syncthreads();   // A is read
    if (b.mine) {
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int j = 0; j < TS; ++j) A.put(r0 + 16 * i, c0 + 16 * j, acc[i][j]);
    }
    __syncthreads();
}
// X <- a X + B X in place, or, behind the last step, the update of W; column 0 of X
// here is column `first` of the matrix's.  Every wavefront calls it.
__device__ __forceinline__ void move_columns(const Group &g, const Job &J, const Resident &X, const Resident &B,
                                             const float *d, int mp, int np, int first, bool last, int lane, int wave) {
    for (int c0 = 16 * wave; c0 < np; c0 += 16 * (kSmallThreads / 64)) {
        f32x4 acc[kSmallSide / 16];
#pragma unroll
        for (int i = 0; i < kSmallSide / 16; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
        for (int t = 0; t < mp / 32; ++t) {
            const Frag x = X.columns(t, c0, lane);
#pragma unroll
            for (int i = 0; i < kSmallSide / 16; ++i)
                if (16 * i < mp) mma<TILE_PAIR>(acc[i], B.rows(16 * i, t, lane), x, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kSmallSide / 16; ++i) {
            if (16 * i >= mp) break;
            const int row = 16 * i + (lane & 15), col = c0 + 4 * (lane >> 4);
            const f32x4 v = acc[i] * two_to(-kBBits) + X.four(row, col) * (kCoefA + d[row]);
            if (last) apply(g, J, row, first + col, v * two_to(-kXBits));
            else X.put(row, col, v);
        }
    }
    __syncthreads();
}
// Zeros to X's pieces.
__device__ __forceinline__ void clear(const Resident &X, int mp, int np) {
    for (int i = threadIdx.x; i < mp * np / 4; i += kSmallThreads) *(uint4 *)(X.base + i * 16) = make_uint4(0u, 0u, 0u, 0u);
}
// four elements of U times inv to their places in X, whose column 0 is `first`
__device__ __forceinline__ void place_u(const Resident &X, const Job &J, int r, int c, int first, f32x4 u, double inv) {
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = (float)((double)u[e] * inv);
    if (J.rows > J.cols) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < J.cols) X.put_one(c + e, r - first, u[e]);
    } else {
        X.put(r, c - first, u);
    }
}

__global__ __launch_bounds__(kSmallThreads) void resident_kernel(Group g, int steps) {
    __shared__ __attribute__((aligned(16))) char lds[kSmallLds];
    const Job &J = g.job[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mp = J.mp, np = J.np;
    const Resident A{lds, 128 * mp}, X{lds + 4 * mp * mp, 128 * mp};
    float *const e = (float *)(lds + 4 * mp * (mp + np)), *const d = e + mp;
    // M and the norm, then X, each of a thread's own elements of U both times
    const uint32_t per_row = ((uint32_t)J.cols + 3) / 4, total = (uint32_t)J.rows * per_row;
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < total; i += kSmallThreads)
        sum += squares(four_of_u<true>(g, J, i / per_row, 4 * (i % per_row)));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    double *const red = (double *)lds;   // (A's place)
    if (lane == 0) red[wave] = sum;
    clear(X, mp, np);
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kSmallThreads / 64; ++w) sum += red[w];
    const double inv = inverse_norm(sum);
    for (uint32_t i = threadIdx.x; i < total; i += kSmallThreads) {
        const int r = (int)(i / per_row), c = 4 * (int)(i % per_row);
        place_u(X, J, r, c, 0, four_of_u<false>(g, J, r, c), inv);
    }
    __syncthreads();
    for (int k = 0; k < steps; ++k) {
        if (mp > 64) {
            gram<2>(X, A, e, mp, np, lane, wave);
            poly<2>(A, e, d, mp, lane, wave);
        } else {
            gram<1>(X, A, e, mp, np, lane, wave);
            poly<1>(A, e, d, mp, lane, wave);
        }
        move_columns(g, J, X, A, d, mp, np, 0, k + 1 == steps, lane, wave);
    }
}

// Few rows and many columns: a workgroup has J.slab of X's columns for one step.  It adds
// the workgroups' parts of A = X X^T from the step before, in order, forms B by
// itself, moves its columns, and leaves its part of the next A: one launch a step
// instead of three, and the sum over the columns in as many parts as there are
// workgroups.  Its columns go through memory as they lie in LDS.  Parts alternate
// between two places, since others may still read the old ones.  us, three launches a
// step / one: 64 x 700 89 / 56, 64 x 2000 111 / 65, 64 x 65,536 1245 / 191, 30 x 4000 135 / 53,
// 16 x 8000 201 / 63, 96 x 2000 115 / 105, 96 x 65,536 1222 / 576, but 128 x 1000 101 / 128, 128 x
// 8192 230 / 270: B and the part of A are formed by one CU each.
__global__ __launch_bounds__(kSmallThreads) void slab_kernel(Group g, int step, int steps) {
    __shared__ __attribute__((aligned(16))) char lds[kSmallLds];
    const int j = job_of(g, blockIdx.x);
    const Job &J = g.job[j];
    const int s = (int)(blockIdx.x - g.first[j]), slabs = (int)((j + 1 < g.count ? g.first[j + 1] : g.total) - g.first[j]);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mp = J.mp, np = J.slab;
    const int first = s * np;
    const Resident A{lds, 128 * mp}, X{lds + 4 * mp * mp, 128 * mp};
    float *const e = (float *)(lds + 4 * mp * (mp + np)), *const d = e + mp;
    uint4 *const image = (uint4 *)(J.X0 + (int64_t)s * 4 * mp * np);
    float *const parts = (float *)J.X1;   // [2][slabs][mp x mp]
    if (step < 0) {
        double sum = 0.0;
        for (int i = threadIdx.x; i < J.parts; i += kSmallThreads) sum += J.part[i];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        double *const red = (double *)lds;   // (A's place)
        if (lane == 0) red[wave] = sum;
        clear(X, mp, np);
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int w = 0; w < kSmallThreads / 64; ++w) sum += red[w];
        const double inv = inverse_norm(sum);
        const bool tall = J.rows > J.cols;
        const int r0 = tall ? first : 0, rows = tall ? min(np, J.rows - first) : J.rows;
        const int c0 = tall ? 0 : first, fours = tall ? (J.cols + 3) / 4 : (min(np, J.cols - first) + 3) / 4;
        for (int i = threadIdx.x; i < rows * fours; i += kSmallThreads) {
            const int r = r0 + i / fours, c = c0 + 4 * (i % fours);
            place_u(X, J, r, c, first, four_of_u<false>(g, J, r, c), inv);
        }
    } else {
        for (int i = threadIdx.x; i < mp * np / 4; i += kSmallThreads) *(uint4 *)(X.base + i * 16) = image[i];
        const f32x4 *const p = (const f32x4 *)(parts + (int64_t)(step & 1) * slabs * mp * mp);
        for (int i = threadIdx.x; i < mp * mp / 4; i += kSmallThreads) {
            f32x4 v = p[i];
#pragma unroll 8
            for (int w = 1; w < slabs; ++w) v += p[(int64_t)w * (mp * mp / 4) + i];
            const int row = 4 * i / mp, col = 4 * i % mp;
            A.put(row, col, gram_of(v, row, col, e + row));
        }
        __syncthreads();
        if (mp > 64) poly<2>(A, e, d, mp, lane, wave);
        else poly<1>(A, e, d, mp, lane, wave);
        const bool last = step + 1 == steps;
        move_columns(g, J, X, A, d, mp, np, first, last, lane, wave);
        if (last) return;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < mp * np / 4; i += kSmallThreads) image[i] = *(const uint4 *)(X.base + i * 16);
    float *const mine = parts + ((int64_t)((step + 1) & 1) * slabs + s) * mp * mp;
    auto leave = [&](auto ts) {
        constexpr int TS = decltype(ts)::value;
        const Block<TS> b(mp, wave);
        if (!b.mine) return;
        f32x4 acc[TS][TS];
        block_of<TS>(X, np / 32, b.i0, b.j0, lane, acc);
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int k = 0; k < TS; ++k)
                *(f32x4 *)(mine + (b.i0 + 16 * i + (lane & 15)) * mp + b.j0 + 16 * k + 4 * (lane >> 4)) = acc[i][k];
    };
    if (mp > 64) leave(std::integral_constant<int, 2>{});
    else leave(std::integral_constant<int, 1>{});
}

// B and a X + B X in one launch where A fits in LDS beside the columns of X: 32 rows and
// 64 columns of the next X to a workgroup, which forms its rows of B from A by itself.
// Up to twice the products, and A read once a workgroup, against a launch, five of
// which are 20 us.  For one round of a workgroup a CU (us, apart / so: 602 x 128 and 256 x
// 128, two each, 96 / 76, 128 x 300 89 / 68, 128 x 4096, 256 workgroups, 159 / 140, but six of
// 700 x 128, 264, 100 / 109, 128 x 8192 230 / 235).
constexpr int kStepRows = 32, kStepCols = 64, kStepThreads = 512, kMostSteps = 256;
__host__ __device__ __forceinline__ int64_t step_blocks(const Job &J) {
    return (int64_t)(J.mp / kStepRows) * ((J.np + kStepCols - 1) / kStepCols);
}
template <int STAGE>
__global__ __launch_bounds__(kStepThreads) void step_kernel(Group g, int odd) {
    constexpr int kSide = kSmallSide, kFours = kSide * kSide / 4 / kStepThreads, kXFours = kSide * kStepCols / 4 / kStepThreads;
    __shared__ __attribute__((aligned(16))) char lds[4 * kSide * (kSide + kStepCols) + 4 * kStepRows * kSide];
    __shared__ float d[kStepRows];
    const int j = job_of(g, blockIdx.x);
    const Job &J = g.job[j];
    const uint8_t *const from = odd ? J.X1 : J.X0;
    uint8_t *const next = odd ? J.X0 : J.X1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mp = J.mp, np = J.np;
    const int at = (int)(blockIdx.x - g.first[j]), down = mp / kStepRows;
    const int r0 = at % down * kStepRows, first = at / down * kStepCols, cols = min(kStepCols, np - first);
    const Resident A{lds, 128 * mp}, X{lds + 4 * mp * mp, 128 * mp}, B{lds + 4 * mp * (mp + kStepCols), 128 * kStepRows};
    f32x4 a[kFours], x[kXFours];
    const int per = mp / 4;   // chunks of 16 bytes of a row of A
#pragma unroll
    for (int u = 0; u < kFours; ++u) {
        const int i = u * kStepThreads + threadIdx.x;
        a[u] = *(const f32x4 *)(J.A + (int64_t)(i < mp * per ? i : 0) * 16);
    }
#pragma unroll
    for (int u = 0; u < kXFours; ++u) {
        const int i = u * kStepThreads + threadIdx.x, r = i / 16, c = i % 16;
        x[u] = *(const f32x4 *)(from + (r < mp && 4 * c < cols ? (int64_t)r * 4 * np + 4 * first + c * 16 : 0));
    }
    const int br = 16 * (wave & 1), bc = 16 * (wave >> 1);   // the wavefront's first block, of B and of X
    const int lr = br + (lane & 15), lc = bc + 4 * (lane >> 4);
    const float e_row = J.e[r0 + lr];
    const f32x4 e_cols[2] = {diagonals_at<POLY>(J, lc), diagonals_at<POLY>(J, lc + 64)};
#pragma unroll
    for (int u = 0; u < kFours; ++u) {
        const int i = u * kStepThreads + threadIdx.x, r = i / per, c = i - r * per;
        if (i < mp * per) *(f32x4 *)(A.base + c / 8 * A.step + r * 128 + ((c % 8) ^ (r & 7)) * 16) = a[u];
    }
#pragma unroll
    for (int u = 0; u < kXFours; ++u) {
        const int i = u * kStepThreads + threadIdx.x, r = i / 16, c = i % 16;
        if (r < mp && 4 * c < cols) *(f32x4 *)(X.base + c / 8 * X.step + r * 128 + ((c % 8) ^ (r & 7)) * 16) = x[u];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        const int pieces = bc + 64 * u < mp ? mp / 32 : 0;
#pragma unroll 1
        for (int t = 0; t < pieces; ++t) mma<TILE_PAIR>(v, A.rows(r0 + br, t, lane), A.rows(bc + 64 * u, t, lane), 0, 0);
        if (pieces) B.put(lr, lc + 64 * u, poly_of(v, A.four(r0 + lr, lc + 64 * u), e_row, e_cols[u], r0 + lr, lc + 64 * u, d + lr));
    }
    __syncthreads();
    if (bc >= cols) return;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int t = 0; t < mp / 32; ++t) mma<TILE_PAIR>(v, B.rows(br, t, lane), X.columns(t, bc, lane), 0, 0);
    v = v * two_to(-kBBits) + X.four(r0 + lr, lc) * (kCoefA + d[lr]);
    if constexpr (STAGE == NEXT) store_parts(next + place<PAIR>(r0 + lr, row_bytes<PAIR>(np), first + lc), 64, v);
    else apply(g, J, r0 + lr, first + lc, v * two_to(-kXBits));
}

// Whether a matrix takes pairs.  GCN_BF16 does so too for matrices with a short side,
// whose time is launches, not products.
constexpr int32_t kSingleSide = 128;
bool takes_pairs(int32_t rows, int32_t cols, int prec) {
    return prec == GCN_F32 || std::min(rows, cols) < kSingleSide;
}

bool aligned(const void *p, uintptr_t b) { return (uintptr_t)p % b == 0; }
int32_t up(int32_t x, int32_t to) { return (x + to - 1) / to * to; }

// Columns of a slab: the fewest of 128, 256 and 512 that make at most 16 of them (and fit in LDS).
constexpr int32_t kSlabSide = 96;
int32_t slab_of(int32_t mp, int32_t np) {
    int32_t c = 128;
    while (c < 512 && np > 16 * c && fits_lds(mp, 2 * c)) c *= 2;
    return c;
}

// The job's places in the workspace.
void plan_job(Job &J, bool pair, Arena &ar) {
    const int32_t unit = pair ? 32 : 64;
    J.mp = up(std::min(J.rows, J.cols), unit);
    J.np = up(std::max(J.rows, J.cols), unit);
    // (few rows: X0 takes whole slabs, X1 their parts of A, twice)
    J.slab = pair && J.mp <= kSlabSide ? slab_of(J.mp, J.np) : 0;
    const size_t slabs = J.slab ? (size_t)(J.np + J.slab - 1) / J.slab : 0;
    J.X0 = ar.take<uint8_t>(4 * (size_t)J.mp * std::max((size_t)J.np, slabs * J.slab));
    J.X1 = ar.take<uint8_t>(4 * (size_t)J.mp * std::max((size_t)J.np, 2 * slabs * J.mp));
    J.A = ar.take<uint8_t>(4 * (size_t)J.mp * J.mp);   // (of floats after many steps, whatever the precision)
    J.B = ar.take<uint8_t>(4 * (size_t)J.mp * J.mp);
    J.e = ar.take<float>((size_t)J.mp);
    J.d = ar.take<float>((size_t)J.mp);
    const int64_t total = (int64_t)J.rows * J.cols;
    J.parts = (int32_t)std::min<int64_t>(kMostParts, (total + 4 * kTB - 1) / (4 * kTB));
    J.part = ar.take<double>((size_t)J.parts);
}

// blocks(job) of each job to first[]; their sum
template <class F>
unsigned blocks_of(Group &g, F &&blocks) {
    uint64_t at = 0;
    for (int j = 0; j < g.count; ++j) {
        g.first[j] = (uint32_t)at;
        at += blocks(g.job[j]);
    }
    for (int j = g.count; j < kGroup; ++j) g.first[j] = 0xFFFFFFFFu;
    g.total = (uint32_t)at;
    return (unsigned)at;
}

int64_t tiles(int32_t m, int32_t n, int32_t tm, int32_t tn) {
    return (((int64_t)m + tm - 1) / tm) * (((int64_t)n + tn - 1) / tn);
}

template <int KIND, int STAGE>
int product(Group &g, int odd, hipStream_t s) {
    auto cols = [](const Job &J) { return STAGE <= POLY ? J.mp : J.np; };
    auto count = [&](const Job &J, int32_t tm, int32_t tn) {
        const int64_t t = (J.mp + tm - 1) / tm;
        return STAGE <= POLY && !g.full ? t * (t + 1) / 2 : t * ((cols(J) + tn - 1) / tn);
    };
    auto all = [&](int32_t tm, int32_t tn) {
        int64_t n = 0;
        for (int j = 0; j < g.count; ++j) n += count(g.job[j], tm, tn);
        return n;
    };
    double flops = 0.0;
    bool deep = true, long_k = false;
    for (int j = 0; j < g.count; ++j) {
        const Job &J = g.job[j];
        long_k = long_k || J.np >= 16 * (KIND == SINGLE ? 64 : 32);
        deep = deep && J.mp >= 256 && J.np < (1 << 22);   // (a large tile's row offsets within it: 32 bits)
        const double m = std::min(J.rows, J.cols), n = std::max(J.rows, J.cols);
        flops += STAGE == GRAM ? m * m * n : STAGE == POLY ? m * m * m : 2.0 * m * m * n;
    }
    ProfScope prof(K_MUON_PRODUCT, s, flops, 0.0);
    // Half of A's and B's tiles where all 32 x 32 ones would be more than a round (their
    // transposed stores cost about half a microsecond otherwise).
    g.full = 1;
    if (STAGE <= POLY && all(32, 32) > 256) g.full = 0;
    auto grid = [&](int32_t tm, int32_t tn) {
        const uint32_t total = blocks_of(g, [&](const Job &J) { return (uint64_t)count(J, tm, tn); });
        g.per_xcd = (total + 7) / 8;
        g.band = (uint32_t)std::max(1, std::min(8, (int)std::lround(std::sqrt((double)g.per_xcd))));
        return dim3(8 * g.per_xcd);
    };
#define GCN_MUON(BM, BN, WM, WN, KG)                                                                             \
    do {                                                                                                         \
        const dim3 b = grid(BM, BN);                                                                             \
        hipLaunchKernelGGL((muon_kernel<KIND, STAGE, BM, BN, WM, WN, KG>), b, dim3(64 * WM * WN * KG), 0, s, g, odd); \
    } while (0)
    // us a call of five steps, the two ways on either side of each border (taken with the diagonals still within A
    // and B, 1 to 2 % faster throughout).  Large tiles for a X + B X: 3000 x 3200 (156 of them) 2185 with 128 x 128
    // ones, 2121 with large; for A and B 3000 x 3200 (78) 2185 and 2850, 3400 x 3400 in GCN_BF16 (105) 1099 and 1386.
    if (KIND != WHOLE && deep && all(kBigT, kBigT) >= (STAGE <= POLY ? 120 : 150)) {
        const dim3 b = grid(kBigT, kBigT);
        if constexpr (KIND != WHOLE) hipLaunchKernelGGL((muon_big_kernel<KIND, STAGE>), b, dim3(kBigThreads), 0, s, g, odd);
    } else if constexpr (STAGE <= POLY) {
        // 32 x 32 tiles while they are few: a CU's own path to its L2 carries 64 bytes a cycle, and few tiles leave
        // most of the CUs, and their paths, idle (four of 602 x 128 and 256 x 128: 118 with 64 x 64 ones, 93 so; 700 x
        // 700, 253 of them, 176 and 148; 1024 x 1024, 528, 227 and 234).  64 x 64 in two parts a CU: 1500 x 1500
        // (300) 487 unsplit, 429 so; unsplit 2000 x 2500 (528) 850, 895 in 128 x 128 ones of two parts; those 2500 x
        // 2500 (820 or 210) 1267 and 1108.
        if (all(128, 128) > 256) GCN_MUON(128, 128, 2, 2, 1);
        else if (all(64, 64) > 640) GCN_MUON(128, 128, 2, 2, 2);
        else if (all(64, 64) > 512) GCN_MUON(64, 64, 4, 1, 1);
        else if (all(64, 64) > 256) GCN_MUON(64, 64, 4, 1, 2);
        else if (all(32, 32) > 400) GCN_MUON(64, 64, 4, 1, 4);
        else if (STAGE == GRAM && all(32, 32) <= 256 && long_k) GCN_MUON(32, 32, 1, 1, 8);
        else GCN_MUON(32, 32, 1, 1, 4);
    } else {
        // The smallest tiles that one round of a workgroup a CU holds: 512 x 512 and 1024 x 512, two each (416 of 32
        // rows, 208 of 64) 230 and 206; 1500 x 1500 (288 of 64, 144 of 128) 560 and 487; 1024 x 2048 (256 of 64, 128)
        // 287 and 321; 2000 x 2500 in GCN_BF16 (320 of 128) in two parts 508, unsplit 454.
        if (all(32, 128) <= 256) GCN_MUON(32, 128, 2, 2, 4);
        else if (all(64, 128) <= 256) GCN_MUON(64, 128, 2, 2, 2);
        else if (all(128, 128) <= 256) GCN_MUON(128, 128, 2, 2, 2);
        else GCN_MUON(128, 128, 2, 2, 1);
    }
#undef GCN_MUON
    GCN_LAUNCH_CHECK("muon_kernel");
    return GCN_OK;
}

// `ahead`: the first steps, in float32.
template <int KIND>
int run_group(Group &g, int32_t steps, int32_t ahead, hipStream_t s) {
    bool small = KIND == PAIR && ahead == 0, few = small, narrow = KIND == PAIR;
    double flops = 0.0;
    if constexpr (KIND == PAIR) {
        int64_t blocks = 0;
        int32_t most = 0;
        for (int j = 0; j < g.count; ++j) {
            const Job &J = g.job[j];
            small = small && fits_lds(J.mp, J.np);
            few = few && J.slab > 0;
            flops += (3.0 * J.np + J.mp) * J.mp * J.mp * steps;
            blocks += step_blocks(J);
            most = std::max(most, J.mp);
        }
        narrow = most <= kSmallSide && blocks <= kMostSteps;
        // (us, step_kernel / slab_kernel: 96 x 700 67 / 87, 96 x 2000, 96 workgroups of the former, 91 / 105, 96 x 3000,
        // 141, 111 / 109, 96 x 5000 155 / 119; 64 x 700 62 / 56, 64 x 2000 85 / 65)
        if (most > 64 && blocks <= kMostSteps / 2) few = false;
        if (small) {
            ProfScope prof(K_MUON_SMALL, s, flops, 0.0);
            hipLaunchKernelGGL(resident_kernel, dim3((unsigned)g.count), dim3(kSmallThreads), 0, s, g, (int)steps);
            GCN_LAUNCH_CHECK("resident_kernel");
            return GCN_OK;
        }
    }
    double bytes = 0.0;
    for (int j = 0; j < g.count; ++j) bytes += 12.0 * g.job[j].rows * g.job[j].cols;
    {
        ProfScope prof(K_MUON_PREP, s, 0.0, bytes);
        const dim3 b(blocks_of(g, [](const Job &J) { return (uint64_t)J.parts; }));
        hipLaunchKernelGGL(momentum_kernel, b, dim3(kTB), 0, s, g);
        GCN_LAUNCH_CHECK("momentum_kernel");
    }
    if (KIND == PAIR && few) {
        const dim3 b(blocks_of(g, [](const Job &J) { return (uint64_t)(J.np + J.slab - 1) / J.slab; }));
        for (int32_t k = -1; k < steps; ++k) {
            ProfScope prof(K_MUON_SMALL, s, flops / steps, 0.0);
            hipLaunchKernelGGL(slab_kernel, b, dim3(kSmallThreads), 0, s, g, (int)k, (int)steps);
            GCN_LAUNCH_CHECK("slab_kernel");
        }
        return GCN_OK;
    }
    {
        ProfScope prof(K_MUON_PREP, s, 0.0, bytes);
        const dim3 b = dim3(blocks_of(g, [](const Job &J) { return (uint64_t)tiles(J.mp, J.np, 64, 64); }));
        if (ahead) hipLaunchKernelGGL(operand_kernel<WHOLE>, b, dim3(kTB), 0, s, g);
        else hipLaunchKernelGGL(operand_kernel<KIND>, b, dim3(kTB), 0, s, g);
        GCN_LAUNCH_CHECK("operand_kernel");
    }
    int rc;
    for (int32_t k = 0; k < steps; ++k) {
        const int odd = k & 1;
        if (k < ahead) {
            if ((rc = product<WHOLE, GRAM>(g, odd, s)) || (rc = product<WHOLE, POLY>(g, odd, s))) return rc;
            constexpr int TO = KIND == PAIR ? TO_PAIR : TO_SINGLE;
            if ((rc = k + 1 < ahead ? product<WHOLE, NEXT>(g, odd, s) : product<WHOLE, TO>(g, odd, s))) return rc;
            continue;
        }
        if (KIND == PAIR && narrow) {
            if ((rc = product<KIND, GRAM>(g, odd, s))) return rc;
            ProfScope prof(K_MUON_PRODUCT, s, flops / steps, 0.0);
            const dim3 b(blocks_of(g, [](const Job &J) { return (uint64_t)step_blocks(J); }));
            if (k + 1 < steps) hipLaunchKernelGGL(step_kernel<NEXT>, b, dim3(kStepThreads), 0, s, g, odd);
            else hipLaunchKernelGGL(step_kernel<LAST>, b, dim3(kStepThreads), 0, s, g, odd);
            GCN_LAUNCH_CHECK("step_kernel");
            continue;
        }
        if ((rc = product<KIND, GRAM>(g, odd, s)) || (rc = product<KIND, POLY>(g, odd, s))) return rc;
        if ((rc = k + 1 < steps ? product<KIND, NEXT>(g, odd, s) : product<KIND, LAST>(g, odd, s))) return rc;
    }
    return GCN_OK;
}
int run_group(Group &g, int32_t steps, int prec, bool pairs, hipStream_t s) {
    if (g.count == 0) return GCN_OK;
    const int32_t ahead = std::max(0, steps - (prec == GCN_F32 ? kPairSteps : kSingleSteps));
    return pairs ? run_group<PAIR>(g, steps, ahead, s) : run_group<SINGLE>(g, steps, ahead, s);
}

constexpr int32_t kMostSide = 65536;   // (tile counts and row offsets of a launch within 32 bits)

int check_common(const char *who, int32_t steps, int prec) {
    GCN_REQUIRE(prec == GCN_F32 || prec == GCN_BF16, GCN_EINVAL, "%s: bad precision %d", who, prec);
    GCN_REQUIRE(steps >= 1 && steps <= 64, GCN_EINVAL, "%s: steps=%d is not within 1 .. 64", who, steps);
    return GCN_OK;
}
int check_sides(const char *who, int32_t rows, int32_t cols) {
    GCN_REQUIRE(rows >= 0 && cols >= 0, GCN_ESHAPE, "%s: matrix of %d x %d", who, rows, cols);
    GCN_REQUIRE(rows <= kMostSide && cols <= kMostSide, GCN_EUNSUPPORTED, "%s: matrix of %d x %d, sides beyond %d", who,
                rows, cols, kMostSide);
    return GCN_OK;
}

// Whether a matrix is one of a call's groups of pairs, or of singles.
bool of_group(const gcn_muon_matrix &m, int prec, bool pairs) {
    return m.rows > 0 && m.cols > 0 && takes_pairs(m.rows, m.cols, prec) == pairs;
}

// Elements [p, p + (rows - 1) ld + cols) of `size` bytes.
struct Span {
    uintptr_t begin, end;
    int64_t ld, cols, size;
    bool written;
};
bool clash(const Span &a, const Span &b) {   // a.begin <= b.begin
    if (b.begin >= a.end || !(a.written || b.written)) return false;
    // column ranges of one array's rows lie between each other
    const int64_t pitch = a.ld * a.size;
    if (pitch == b.ld * b.size && pitch > 0) {
        const int64_t off = (int64_t)((b.begin - a.begin) % (uintptr_t)pitch);
        if (off >= a.cols * a.size && off + b.cols * b.size <= pitch) return false;
    }
    return true;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" {

size_t gcn_orthogonalise_workspace_bytes(int32_t rows, int32_t cols, int prec) {
    if (rows < 0 || cols < 0 || std::max(rows, cols) > kMostSide || (prec != GCN_F32 && prec != GCN_BF16)) return 0;
    Job J{};
    J.rows = rows;
    J.cols = cols;
    Arena ar(nullptr, 0);
    plan_job(J, takes_pairs(rows, cols, prec), ar);
    return ar.used + 256;
}

int gcn_orthogonalise(const void *X, gcn_rows_type type, int32_t rows, int32_t cols, int32_t ldx, void *out,
                      int32_t ldo, int32_t steps, int prec, void *ws, size_t ws_bytes, void *stream) {
    const char *const who = "gcn_orthogonalise";
    int rc = check_common(who, steps, prec);
    if (rc || (rc = check_sides(who, rows, cols))) return rc;
    GCN_REQUIRE(type == GCN_ROWS_F32 || type == GCN_ROWS_BF16, GCN_EINVAL, "%s: bad element type %d", who, (int)type);
    GCN_REQUIRE(ldx >= cols && ldo >= cols, GCN_ESHAPE, "%s: ldx=%d ldo=%d < %d", who, ldx, ldo, cols);
    const int64_t el = type == GCN_ROWS_BF16 ? 2 : 4;
    const bool any = rows > 0 && cols > 0;
    GCN_REQUIRE(!any || (X && out && aligned(X, el) && aligned(out, el)), GCN_EINVAL, "%s: null or misaligned pointer", who);
    const size_t need = gcn_orthogonalise_workspace_bytes(rows, cols, prec);
    GCN_REQUIRE(ws && aligned(ws, 256) && ws_bytes >= need, GCN_EWORKSPACE,
                "%s: workspace %zu < %zu bytes, or not 256-byte aligned", who, ws_bytes, need);
    if (!any) return GCN_OK;
    const Span a{(uintptr_t)X, (uintptr_t)X + (uintptr_t)(((int64_t)(rows - 1) * ldx + cols) * el), ldx, cols, el, false};
    const Span b{(uintptr_t)out, (uintptr_t)out + (uintptr_t)(((int64_t)(rows - 1) * ldo + cols) * el), ldo, cols, el, true};
    GCN_REQUIRE((X == out && ldx == ldo) || !(a.begin <= b.begin ? clash(a, b) : clash(b, a)), GCN_EINVAL,
                "%s: out overlaps X and is not X", who);
    Group g{};
    Arena ar(ws, ws_bytes);
    Job &J = g.job[0];
    J.rows = rows;
    J.cols = cols;
    J.G = X;
    J.ldg = ldx;
    J.out = out;
    J.ldw = ldo;
    const bool pairs = takes_pairs(rows, cols, prec);
    plan_job(J, pairs, ar);
    g.count = 1;
    g.grad_bf16 = g.out_bf16 = type == GCN_ROWS_BF16;
    return run_group(g, steps, prec, pairs, (hipStream_t)stream);
}

size_t gcn_muon_workspace_bytes(int32_t count, const gcn_muon_matrix *mats, int prec) {
    if (count < 0 || (count > 0 && !mats) || (prec != GCN_F32 && prec != GCN_BF16)) return 0;
    for (int32_t i = 0; i < count; ++i)
        if (mats[i].rows < 0 || mats[i].cols < 0 || std::max(mats[i].rows, mats[i].cols) > kMostSide) return 0;
    // (groups run one behind the other in the same workspace)
    size_t most = 0;
    for (int pairs = 1; pairs >= 0; --pairs)
        for (int32_t i = 0; i < count;) {
            Arena ar(nullptr, 0);
            for (int k = 0; k < kGroup && i < count; ++i) {
                if (!of_group(mats[i], prec, pairs)) continue;
                Job J{};
                J.rows = mats[i].rows;
                J.cols = mats[i].cols;
                plan_job(J, pairs, ar);
                ++k;
            }
            most = std::max(most, ar.used);
        }
    return most + 256;
}

int gcn_muon_update(int32_t count, const gcn_muon_matrix *mats, gcn_rows_type grad_type, double lr, double momentum,
                    int nesterov, double weight_decay, int32_t steps, int prec, void *ws, size_t ws_bytes,
                    void *stream) {
    const char *const who = "gcn_muon_update";
    int rc = check_common(who, steps, prec);
    if (rc) return rc;
    GCN_REQUIRE(count >= 0 && (count == 0 || mats), GCN_EINVAL, "%s: null matrices or negative count", who);
    GCN_REQUIRE(grad_type == GCN_ROWS_F32 || grad_type == GCN_ROWS_BF16, GCN_EINVAL, "%s: bad element type %d", who,
                (int)grad_type);
    GCN_REQUIRE(std::isfinite(lr) && momentum >= 0.0 && momentum < 1.0 && std::isfinite(weight_decay), GCN_EINVAL,
                "%s: need a finite lr and weight decay and 0 <= momentum < 1", who);
    const int64_t el = grad_type == GCN_ROWS_BF16 ? 2 : 4;
    try {
        std::vector<Span> spans;
        spans.reserve(3 * (size_t)count);
        for (int32_t i = 0; i < count; ++i) {
            const gcn_muon_matrix &m = mats[i];
            if ((rc = check_sides(who, m.rows, m.cols))) return rc;
            GCN_REQUIRE(m.ldw >= m.cols && m.ldg >= m.cols && m.ldm >= m.cols, GCN_ESHAPE,
                        "%s: matrix %d: ldw=%d ldg=%d ldm=%d < %d", who, i, m.ldw, m.ldg, m.ldm, m.cols);
            GCN_REQUIRE(std::isfinite(m.scale), GCN_EINVAL, "%s: matrix %d: scale is not finite", who, i);
            if (m.rows == 0 || m.cols == 0) continue;
            GCN_REQUIRE(m.W && m.G && m.M && aligned(m.W, 4) && aligned(m.M, 4) && aligned(m.G, el), GCN_EINVAL,
                        "%s: matrix %d: null or misaligned pointer", who, i);
            auto span = [&](const void *p, int64_t ld, int64_t size, bool w) {
                spans.push_back(Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)(((m.rows - 1ll) * ld + m.cols) * size), ld,
                                     m.cols, size, w});
            };
            span(m.W, m.ldw, 4, true);
            span(m.M, m.ldm, 4, true);
            span(m.G, m.ldg, el, false);
        }
        std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.begin < b.begin; });
        for (size_t i = 0; i < spans.size(); ++i)
            for (size_t k = i + 1; k < spans.size() && spans[k].begin < spans[i].end; ++k)
                GCN_REQUIRE(!clash(spans[i], spans[k]), GCN_EINVAL, "%s: a W or M overlaps another matrix of the call", who);
    } catch (const std::bad_alloc &) {
        set_error("%s: out of host memory", who);
        return GCN_EINVAL;
    }
    const size_t need = gcn_muon_workspace_bytes(count, mats, prec);
    GCN_REQUIRE(ws && aligned(ws, 256) && ws_bytes >= need, GCN_EWORKSPACE,
                "%s: workspace %zu < %zu bytes, or not 256-byte aligned", who, ws_bytes, need);
    for (int pairs = 1; pairs >= 0; --pairs) for (int32_t i = 0; i < count;) {
        Group g{};
        Arena ar(ws, ws_bytes);
        for (; g.count < kGroup && i < count; ++i) {
            const gcn_muon_matrix &m = mats[i];
            if (!of_group(m, prec, pairs)) continue;
            Job &J = g.job[g.count++];
            J.rows = m.rows;
            J.cols = m.cols;
            J.W = m.W;
            J.G = m.G;
            J.M = m.M;
            J.ldw = m.ldw;
            J.ldg = m.ldg;
            J.ldm = m.ldm;
            J.step = (float)(lr * m.scale);
            plan_job(J, pairs, ar);
        }
        g.momentum = (float)momentum;
        g.decay = (float)(1.0 - lr * weight_decay);
        g.nesterov = nesterov != 0;
        g.grad_bf16 = grad_type == GCN_ROWS_BF16;
        if ((rc = run_group(g, steps, prec, pairs, (hipStream_t)stream))) return rc;
    }
    return GCN_OK;
}

}  // extern "C"
