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
// a X is added to the sums as its own term.  Put on B's diagonal it would be rounded
// there to B's largest element, which small singular values feel: 8 of 512 directions
// large, the error against float64 5.4e-5 instead of 2.2e-5 (float32 products
// throughout: 2.0e-5).
#include <algorithm>
#include <cmath>
#include <vector>

#include "gcn_muon.h"
#include "tiles.h"

namespace gcn {
namespace {

constexpr int kTB = 256;
constexpr int kGroup = 16;        // matrices of a launch
constexpr int kMostParts = 512;   // of a matrix's sum of squares
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
struct Job {
    float *W;                // updated, or null
    const void *G;           // the gradient, or what is orthogonalised
    float *M;                // momentum, or null
    void *out;               // orthogonalise's result, or null
    int64_t ldw, ldg, ldm;   // ldw: of out too
    int32_t rows, cols;
    int32_t m, n, mp, np;
    uint8_t *X0, *X1, *A, *B;
    double *part;            // sums of squares
    int32_t parts;
    float step;              // lr * scale
};
struct Group {
    Job job[kGroup];
    uint32_t first[kGroup + 1];   // a launch's blocks by job
    int32_t count;
    int32_t tile_m, tile_n;
    float momentum, decay;
    int nesterov, grad_bf16, out_bf16;
};
__device__ __forceinline__ int job_of(const Group &g) {
    int j = 0;
    while (j + 1 < g.count && blockIdx.x >= g.first[j + 1]) ++j;
    return j;
}

__device__ __forceinline__ float grad_at(const Group &g, const Job &J, int64_t r, int64_t c) {
    return g.grad_bf16 ? __uint_as_float((uint32_t)((const uint16_t *)J.G)[r * J.ldg + c] << 16)
                       : ((const float *)J.G)[r * J.ldg + c];
}
// U's element from the gradient and the updated momentum
__device__ __forceinline__ float update_of(const Group &g, float grad, float m) {
    return g.nesterov ? fmaf(g.momentum, m, grad) : m;
}

// M <- momentum M + G, and U's sum of squares in float64 (no overflow, and the norm
// of millions of elements to float32's last bit): a block's share of the
// elements, in order.
__global__ __launch_bounds__(kTB) void momentum_kernel(Group g) {
    __shared__ double red[kTB / 64];
    const Job &J = g.job[job_of(g)];
    const uint32_t block = blockIdx.x - g.first[job_of(g)];
    const int64_t total = (int64_t)J.rows * J.cols, step = (int64_t)J.parts * kTB;
    double sum = 0.0;
    for (int64_t i = (int64_t)block * kTB + threadIdx.x; i < total; i += step) {
        const int64_t r = i / J.cols, c = i - r * J.cols;
        float u = grad_at(g, J, r, c);
        if (J.M) {
            const float m = fmaf(g.momentum, J.M[r * J.ldm + c], u);
            J.M[r * J.ldm + c] = m;
            u = update_of(g, u, m);
        }
        sum += (double)u * u;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) J.part[block] = (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ uint16_t half_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ __forceinline__ float half_value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

// Four consecutive elements (column a multiple of 4) of an operand, and back.  `low`:
// bytes from the high parts to the low ones.  bytes: of a row.
template <bool PAIR>
__device__ __forceinline__ int64_t place(int64_t row, int64_t bytes, int64_t col) {
    return row * bytes + (PAIR ? pair_place(col) : 2 * col);
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
template <bool PAIR>
__device__ __forceinline__ int64_t row_bytes(int32_t cols) { return (int64_t)cols * (PAIR ? 4 : 2); }

// X0 = U / |U|, 64 x 64 elements to a block, zeros past U's sides, through LDS
// where U is laid out transposed.
template <bool PAIR>
__global__ __launch_bounds__(kTB) void operand_kernel(Group g) {
    __shared__ float tile[64][65];
    __shared__ double red[kTB / 64];
    const int j = job_of(g);
    const Job &J = g.job[j];
    const uint32_t block = blockIdx.x - g.first[j], across = (uint32_t)((J.np + 63) / 64);
    const int64_t i0 = (int64_t)(block / across) * 64, j0 = (int64_t)(block % across) * 64;   // X's rows, columns
    double sum = 0.0;
    for (int i = threadIdx.x; i < J.parts; i += kTB) sum += J.part[i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = sum;
    __syncthreads();
    sum = (red[0] + red[1]) + (red[2] + red[3]);
    const double inv = sum > 0.0 ? (double)(1 << kXBits) / sqrt(sum) : 0.0;
    const bool tall = J.rows > J.cols;
    const int64_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;   // U's
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int rl = 4 * k + (int)(threadIdx.x >> 6), cl = threadIdx.x & 63;
        const int64_t r = r0 + rl, c = c0 + cl;
        float u = 0.0f;
        if (r < J.rows && c < J.cols) {
            u = grad_at(g, J, r, c);
            if (J.M) u = update_of(g, u, J.M[r * J.ldm + c]);
        }
        (tall ? tile[cl][rl] : tile[rl][cl]) = (float)((double)u * inv);
    }
    __syncthreads();
    const int64_t bytes = row_bytes<PAIR>(J.np), low = PAIR ? 64 : 2 * (int64_t)J.mp * J.np;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = 16 * k + (int)(threadIdx.x >> 4), c = 4 * (int)(threadIdx.x & 15);
        if (i0 + i < J.mp && j0 + c < J.np)
            store_parts(J.X0 + place<PAIR>(i0 + i, bytes, j0 + c), low,
                        f32x4{tile[i][c], tile[i][c + 1], tile[i][c + 2], tile[i][c + 3]});
    }
}

enum Stage { GRAM = 0, POLY = 1, NEXT = 2, LAST = 3 };

// The sums of a product to what it forms.  acc[i][j]: row r0 + 16 i, columns c0 +
// 16 j .. + 3.
template <bool PAIR, int STAGE, int FM>
__device__ __forceinline__ void finish(const Job &J, const uint8_t *X, uint8_t *next, int r0, int c0, f32x4 (&acc)[FM][4]) {
    const int32_t cols = STAGE <= POLY ? J.mp : J.np;
    const int64_t bytes = row_bytes<PAIR>(cols);
    // (A and B of the single products are their high parts alone)
    const int64_t low = PAIR ? 64 : STAGE <= POLY ? 0 : 2 * (int64_t)J.mp * J.np;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = r0 + 16 * i, col = c0 + 16 * j;
            if (row >= J.mp || col >= cols) continue;
            const int64_t at = place<PAIR>(row, bytes, col);
            f32x4 v = acc[i][j];
            if constexpr (STAGE == GRAM) {
                v *= two_to(kABits - 2 * kXBits);
                store_parts(J.A + at, low, v);
            } else if constexpr (STAGE == POLY) {
                f32x4 a = four_of(J.A + at);
                if (low) a += four_of(J.A + at + low);
                v = v * (kCoefC * two_to(kBBits - 2 * kABits)) + a * (kCoefB * two_to(kBBits - kABits));
                store_parts(J.B + at, low, v);
            } else {
                const f32x4 x = four_of(X + at) + four_of(X + at + low);
                v = v * two_to(-kBBits) + x * kCoefA;
                if constexpr (STAGE == NEXT) {
                    store_parts(next + at, low, v);
                } else {
                    v *= two_to(-kXBits);
                    *(f32x4 *)((float *)next + (int64_t)row * J.np + col) = v;
                }
            }
        }
}

template <bool PAIR, int STAGE>
constexpr int type_of() {
    return STAGE <= POLY ? (PAIR ? TILE_PAIR : TILE_F16) : (PAIR ? TILE_PAIR_NN : TILE_F16_NN);
}

// A tile of a product of one of the group's matrices.  odd: X is in X1.
template <bool PAIR, int STAGE>
__device__ __forceinline__ bool product_of(const Group &g, int odd, const Job *&J, TileProduct &p, Coord &c, const uint8_t *&X,
                                           uint8_t *&next) {
    const int j = job_of(g);
    J = &g.job[j];
    X = odd ? J->X1 : J->X0;
    next = odd ? J->X0 : J->X1;
    constexpr int kUnit = PAIR ? 32 : 64;   // columns of a piece
    p.M = J->mp;
    if constexpr (STAGE == GRAM) {
        p.A = p.B = X;
        p.lda = p.ldb = row_bytes<PAIR>(J->np);
        p.N = J->mp;
        p.kt = J->np / kUnit;
    } else if constexpr (STAGE == POLY) {
        p.A = p.B = J->A;
        p.lda = p.ldb = row_bytes<PAIR>(J->mp);
        p.N = J->mp;
        p.kt = J->mp / kUnit;
    } else {
        p.A = J->B;
        p.lda = row_bytes<PAIR>(J->mp);
        p.B = X;
        p.ldb = row_bytes<PAIR>(J->np);
        p.N = J->np;
        p.kt = J->mp / kUnit;
    }
    Args a;
    a.tiles_m = (p.M + g.tile_m - 1) / g.tile_m;
    a.tiles_n = (p.N + g.tile_n - 1) / g.tile_n;
    a.band = 8;
    a.total = (uint32_t)a.tiles_m * a.tiles_n;
    a.per_xcd = (a.total + 7) / 8;
    return coord_of(a, blockIdx.x - g.first[j], c);
}

template <bool PAIR, int STAGE, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM *WN) void muon_kernel(Group g, int odd) {
    constexpr int TYPE = type_of<PAIR, STAGE>(), FM = BM / WM / 16;
    __shared__ __attribute__((aligned(16))) char lds[small_lds(TYPE, BM, BN)];
    const Job *J;
    TileProduct p{};
    Coord c;
    const uint8_t *X;
    uint8_t *next;
    if (!product_of<PAIR, STAGE>(g, odd, J, p, c, X, next)) return;
    f32x4 acc[FM][4];
    small_loop<TYPE, BM, BN, WM, WN>(p, c, 0, p.kt, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    finish<PAIR, STAGE, FM>(*J, X, next, c.tm * BM + wave / WN * (BM / WM) + (lane & 15),
                            c.tn * BN + wave % WN * (BN / WN) + 4 * (lane >> 4), acc);
}
template <bool PAIR, int STAGE>
__global__ __launch_bounds__(kBigThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void muon_big_kernel(Group g, int odd) {
    constexpr int TYPE = type_of<PAIR, STAGE>();
    __shared__ __attribute__((aligned(16))) char lds[big_lds(TYPE)];
    const Job *J;
    TileProduct p{};
    Coord c;
    const uint8_t *X;
    uint8_t *next;
    if (!product_of<PAIR, STAGE>(g, odd, J, p, c, X, next)) return;
    f32x4 acc[8][4];
    big_loop<TYPE>(p, c, 0, p.kt, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    finish<PAIR, STAGE, 8>(*J, X, next, c.tm * kBigT + (wave >> 2) * 128 + (lane & 15),
                           c.tn * kBigT + (wave & 3) * 64 + 4 * (lane >> 4), acc);
}

// W <- decay W - step O, or out = O, from O [m x n] (rows of np float32), through LDS
// where it lies transposed.
__global__ __launch_bounds__(kTB) void update_kernel(Group g, int odd) {
    __shared__ float tile[64][65];
    const int j = job_of(g);
    const Job &J = g.job[j];
    const uint32_t block = blockIdx.x - g.first[j], across = (uint32_t)((J.cols + 63) / 64);
    const int64_t r0 = (int64_t)(block / across) * 64, c0 = (int64_t)(block % across) * 64;
    const bool tall = J.rows > J.cols;
    const float *O = (const float *)(odd ? J.X0 : J.X1);
    if (tall) {
#pragma unroll 4
        for (int k = 0; k < 16; ++k) {
            const int i = 4 * k + (int)(threadIdx.x >> 6), c = threadIdx.x & 63;   // O's row c0 + i, column r0 + c
            if (c0 + i < J.cols && r0 + c < J.rows) tile[c][i] = O[(c0 + i) * J.np + r0 + c];
        }
        __syncthreads();
    }
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int rl = 4 * k + (int)(threadIdx.x >> 6), cl = threadIdx.x & 63;
        const int64_t r = r0 + rl, c = c0 + cl;
        if (r >= J.rows || c >= J.cols) continue;
        const float o = tall ? tile[rl][cl] : O[r * J.np + c];
        if (J.W) {
            float *w = J.W + r * J.ldw + c;
            *w = g.decay * *w - J.step * o;
        } else if (g.out_bf16) {
            ((uint16_t *)J.out)[r * J.ldw + c] = to_bf16(o);
        } else {
            ((float *)J.out)[r * J.ldw + c] = o;
        }
    }
}

// Whether a matrix takes pairs.  GCN_BF16 does so too for matrices with a short side: a
// single product's roundings average out over many singular values only (one row:
// 4e-3 off, 128 rows 1.7e-3), and their time is launches, not products.
constexpr int32_t kSingleSide = 128;
bool takes_pairs(int32_t rows, int32_t cols, int prec) {
    return prec == GCN_F32 || std::min(rows, cols) < kSingleSide;
}

bool aligned(const void *p, uintptr_t b) { return (uintptr_t)p % b == 0; }
int32_t up(int32_t x, int32_t to) { return (x + to - 1) / to * to; }

// The job's places in the workspace.
void plan_job(Job &J, bool pair, Arena &ar) {
    J.m = std::min(J.rows, J.cols);
    J.n = std::max(J.rows, J.cols);
    const int32_t unit = pair ? 32 : 64;
    J.mp = up(J.m, unit);
    J.np = up(J.n, unit);
    // (X1 also takes the result, four bytes an element)
    J.X0 = ar.take<uint8_t>(4 * (size_t)J.mp * J.np);
    J.X1 = ar.take<uint8_t>(4 * (size_t)J.mp * J.np);
    J.A = ar.take<uint8_t>((pair ? 4 : 2) * (size_t)J.mp * J.mp);
    J.B = ar.take<uint8_t>((pair ? 4 : 2) * (size_t)J.mp * J.mp);
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
    g.first[g.count] = (uint32_t)at;
    return (unsigned)at;
}

int64_t tiles(int32_t m, int32_t n, int32_t tm, int32_t tn) {
    return (((int64_t)m + tm - 1) / tm) * (((int64_t)n + tn - 1) / tn);
}

template <bool PAIR, int STAGE>
int product(Group &g, int odd, hipStream_t s) {
    auto cols = [](const Job &J) { return STAGE <= POLY ? J.mp : J.np; };
    int64_t big = 0, mid = 0;
    double flops = 0.0;
    bool deep = true;
    for (int j = 0; j < g.count; ++j) {
        const Job &J = g.job[j];
        big += tiles(J.mp, cols(J), kBigT, kBigT);
        mid += tiles(J.mp, cols(J), 128, 128);
        deep = deep && J.mp >= 256 && J.np < (1 << 22);   // (a large tile's row offsets within it: 32 bits)
        flops += 2.0 * J.m * J.m * (STAGE == POLY ? J.m : J.n);
    }
    ProfScope prof(K_MUON_PRODUCT, s, flops, 0.0);
    auto grid = [&](int32_t tm, int32_t tn) {
        g.tile_m = tm;
        g.tile_n = tn;
        return dim3(blocks_of(g, [&](const Job &J) { return (uint64_t)(tiles(J.mp, cols(J), tm, tn) + 7) / 8 * 8; }));
    };
    if (deep && big >= 160) {
        const dim3 b = grid(kBigT, kBigT);
        hipLaunchKernelGGL((muon_big_kernel<PAIR, STAGE>), b, dim3(kBigThreads), 0, s, g, odd);
    } else if (mid >= 256) {
        const dim3 b = grid(128, 128);
        hipLaunchKernelGGL((muon_kernel<PAIR, STAGE, 128, 128, 2, 2>), b, dim3(256), 0, s, g, odd);
    } else if constexpr (STAGE <= POLY) {
        const dim3 b = grid(64, 64);
        hipLaunchKernelGGL((muon_kernel<PAIR, STAGE, 64, 64, 4, 1>), b, dim3(256), 0, s, g, odd);
    } else {
        const dim3 b = grid(32, 128);
        hipLaunchKernelGGL((muon_kernel<PAIR, STAGE, 32, 128, 2, 2>), b, dim3(256), 0, s, g, odd);
    }
    GCN_LAUNCH_CHECK("muon_kernel");
    return GCN_OK;
}

template <bool PAIR>
int run_group(Group &g, int32_t steps, hipStream_t s) {
    {
        double bytes = 0.0;
        for (int j = 0; j < g.count; ++j) bytes += 12.0 * g.job[j].rows * g.job[j].cols;
        ProfScope prof(K_MUON_PREP, s, 0.0, bytes);
        dim3 b(blocks_of(g, [](const Job &J) { return (uint64_t)J.parts; }));
        hipLaunchKernelGGL(momentum_kernel, b, dim3(kTB), 0, s, g);
        GCN_LAUNCH_CHECK("momentum_kernel");
        b = dim3(blocks_of(g, [](const Job &J) { return (uint64_t)tiles(J.mp, J.np, 64, 64); }));
        hipLaunchKernelGGL(operand_kernel<PAIR>, b, dim3(kTB), 0, s, g);
        GCN_LAUNCH_CHECK("operand_kernel");
    }
    int rc;
    for (int32_t k = 0; k < steps; ++k) {
        const int odd = k & 1;
        if ((rc = product<PAIR, GRAM>(g, odd, s)) || (rc = product<PAIR, POLY>(g, odd, s))) return rc;
        if ((rc = k + 1 < steps ? product<PAIR, NEXT>(g, odd, s) : product<PAIR, LAST>(g, odd, s))) return rc;
    }
    double bytes = 0.0;
    for (int j = 0; j < g.count; ++j) bytes += 12.0 * g.job[j].rows * g.job[j].cols;
    ProfScope prof(K_MUON_UPDATE, s, 0.0, bytes);
    const dim3 b(blocks_of(g, [](const Job &J) { return (uint64_t)tiles(J.rows, J.cols, 64, 64); }));
    hipLaunchKernelGGL(update_kernel, b, dim3(kTB), 0, s, g, (int)((steps - 1) & 1));
    GCN_LAUNCH_CHECK("update_kernel");
    return GCN_OK;
}
int run_group(Group &g, int32_t steps, bool pairs, hipStream_t s) {
    if (g.count == 0) return GCN_OK;
    return pairs ? run_group<true>(g, steps, s) : run_group<false>(g, steps, s);
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
    return run_group(g, steps, pairs, (hipStream_t)stream);
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
        if ((rc = run_group(g, steps, pairs, (hipStream_t)stream))) return rc;
    }
    return GCN_OK;
}

}  // extern "C"
