// Products C = A B^T of bfloat16, 8-bit or float32 rows on the matrix cores, with
// the epilogues of the 8-bit layer products and of the many-class loss (the tile
// loops: tiles.h).
#include <algorithm>

#include "tiles.h"

namespace gcn {
namespace {

constexpr bool is_stats(int epi) { return epi == TILE_STATS || epi == TILE_STATS_STORE; }

// the column of row's label, maybe outside this product's; kNoLabel without one
constexpr int kNoLabel = -0x7FFFFFFF - 1;
__device__ __forceinline__ int label_of(const TileProduct &p, int row) {
    const int l = row < p.M ? p.labels[row] : -1;
    return l >= 0 && l < p.classes ? l - p.class0 : kNoLabel;
}

// bfloat16 rows out of a wavefront's 16 FM x 64 block, through its own part of
// LDS so that each store fills whole 128-byte lines (8 rows of 16 bytes a lane;
// straight from the registers a store is 16 pieces of 32 bytes, and 16,384 x
// 16,384 results of K = 1024 take 695 us instead of 605).  Chunk c of 16 bytes of
// row r lies at c ^ (r % 8).  `mine`: 16 FM rows of 128 bytes that no other
// wavefront touches; row0, col0: the block's origin.
template <int FM>
__device__ __forceinline__ void store_rows(const f32x4 (&v)[FM][4], char *mine, uint16_t *dst, int64_t ld, int row0,
                                           int col0, int64_t rows, int64_t cols) {
    const int lane = threadIdx.x & 63, fr = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *(uint2 *)(mine + (16 * i + fr) * 128 + (((2 * j + (g >> 1)) ^ (fr & 7)) * 16) + (g & 1) * 8) =
                make_uint2(pack_bf16x2(v[i][j][0], v[i][j][1]), pack_bf16x2(v[i][j][2], v[i][j][3]));
    asm volatile("" ::: "memory");   // (LDS accesses of one wavefront stay in order)
    const int lr = lane >> 3, col = col0 + 8 * (lane & 7);
    const bool vec = col + 8 <= cols;
#pragma unroll
    for (int q = 0; q < 2 * FM; ++q) {
        const int r = 8 * q + lr;
        const uint4 x = *(const uint4 *)(mine + r * 128 + (((lane & 7) ^ (r & 7)) * 16));
        if (row0 + r >= rows) continue;
        uint16_t *d = dst + (int64_t)(row0 + r) * ld + col;
        if (vec) {
            store16(d, x);
        } else {
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < cols) d[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
        }
    }
}

// ------------------------------------------------------------- epilogues
// What an epilogue reads besides the sums.  The small tiles of the loss load it
// ahead of their products (17 rows of 128 columns, 1009 classes: the call 33.8 ->
// 32.5 us); the others, whose registers it would take meanwhile, behind them (8000 x 512
// x 1024 11.9 instead of 12.2).
template <int FM, int FN>
struct Extras {
    float bias[FN][4];
    float scale;
    int lab[FM];
    float top[FM], log2_sum[FM];
};
constexpr float kLog2e = 1.44269504088896340736f;
template <int EPI, int BM, int BN, int WM, int WN, int FM, int FN>
__device__ __forceinline__ void load_extras(const TileProduct &p, const Coord &c, Extras<FM, FN> &x) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = c.tm * BM + wave / WN * (BM / WM) + (lane & 15);
    const int c0 = c.tn * BN + wave % WN * (BN / WN) + 4 * (lane >> 4);
    if constexpr (EPI != TILE_PARTIAL) {
        // (the logits' columns past the last class: minus infinity)
        const float past = is_stats(EPI) || EPI == TILE_GRAD ? -INFINITY : 0.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = c0 + 16 * j + e;
                x.bias[j][e] = col < p.N ? (p.bias ? p.bias[col] : 0.0f) : past;
            }
    }
    if constexpr (EPI != TILE_PARTIAL && !is_stats(EPI)) x.scale = p.scale ? p.scale[0] : 1.0f;
    if constexpr (is_stats(EPI) || EPI == TILE_GRAD) {
#pragma unroll
        for (int i = 0; i < FM; ++i) x.lab[i] = label_of(p, r0 + 16 * i);
    }
    if constexpr (EPI == TILE_GRAD) {
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const bool in = r0 + 16 * i < p.M;
            x.top[i] = in ? p.row_max[r0 + 16 * i] : 0.0f;
            x.log2_sum[i] = in ? p.log_sum[r0 + 16 * i] * kLog2e : 0.0f;
        }
    }
}

// acc[i][j]: row m0 + 16 i + lane % 16 of C, columns n0 + 16 j + 4 (lane / 16)
// .. + 3 of the wavefront's block; `scratch`: the idle operand LDS.
// float32 results, row by row: a wavefront's stores fill whole lines one after another
template <int FM, int FN>
__device__ __forceinline__ void store_f32(const f32x4 (&acc)[FM][FN], const TileProduct &p, int r0, int c0) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int row = r0 + 16 * i;
        if (row >= p.M) continue;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int col = c0 + 16 * j;
            float *d = (float *)p.C + (int64_t)row * p.ldc + col;
            if (col + 4 <= p.N) {
                store16(d, __builtin_bit_cast(uint4, acc[i][j]));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < p.N) d[e] = acc[i][j][e];
            }
        }
    }
}

template <int EPI, int BM, int BN, int WM, int WN, int FM, int FN>
__device__ __forceinline__ void finish(const Args &a, const Coord &c, const Extras<FM, FN> &x,
                                       f32x4 (&acc)[FM][FN], char *scratch) {
    const TileProduct &p = a.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / WN, wn = wave % WN;
    const int r0 = c.tm * BM + wm * (BM / WM) + (lane & 15);
    const int c0 = c.tn * BN + wn * (BN / WN) + 4 * (lane >> 4);
    static_assert(FN == 4, "a wavefront's block is 64 columns wide");
    if constexpr (EPI == TILE_STORE || EPI == TILE_STORE_F32) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = acc[i][j][e] * x.scale + x.bias[j][e];
                if (p.relu)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = acc[i][j][e] < 0.0f ? 0.0f : acc[i][j][e];   // (NaN stays)
            }
        if constexpr (EPI == TILE_STORE) {
            __syncthreads();   // the operands are read
            store_rows<FM>(acc, scratch + wave * FM * 2048, (uint16_t *)p.C, p.ldc, c.tm * BM + wm * (BM / WM),
                           c.tn * BN + wn * (BN / WN), p.M, p.N);
            return;
        }
        store_f32<FM, FN>(acc, p, r0, c0);
    } else if constexpr (EPI == TILE_PARTIAL) {
        float *base = p.acc + (int64_t)c.split * p.M * p.N;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int row = r0 + 16 * i, col = c0 + 16 * j;
                if (row >= p.M || col >= p.N) continue;
                float *d = base + (int64_t)row * p.N + col;
                if (col + 4 <= p.N) {
                    f32x4 v = acc[i][j];
                    if (p.accumulate) v += __builtin_bit_cast(f32x4, load16(d));
                    store16(d, __builtin_bit_cast(uint4, v));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e < p.N) d[e] = p.accumulate ? d[e] + acc[i][j][e] : acc[i][j][e];
                }
            }
    } else {
        // the logits
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] += x.bias[j][e];
        if constexpr (EPI == TILE_STATS_STORE) store_f32<FM, FN>(acc, p, r0, c0);
        const int w0 = c.tn * BN + wn * (BN / WN);   // the wavefront's first column
        if constexpr (is_stats(EPI)) {
            // a row's columns lie in 4 lanes of WN wavefronts: maximum and sum
            // over the lane's own, two exchanges, then LDS across wavefronts
            float2 *part = (float2 *)scratch;   // [WN][BM]
            __syncthreads();
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int row = r0 + 16 * i;
                float m = -INFINITY;
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
                m = fmaxf(m, __shfl_xor(m, 16));
                m = fmaxf(m, __shfl_xor(m, 32));
                const float base = m == -INFINITY ? 0.0f : m;   // no finite logit yet: the sum stays 0
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f((acc[i][j][e] - base) * kLog2e);
                s += __shfl_xor(s, 16);
                s += __shfl_xor(s, 32);
                if (lane < 16) part[wn * BM + row - c.tm * BM] = make_float2(m, s);
                const int lab = x.lab[i];
                if (__any(lab >= w0 && lab < w0 + BN / WN)) {   // (few wavefronts see one of their labels)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c0 + 16 * j + e == lab && lab < p.N) p.label_logit[row] = acc[i][j][e];
                }
            }
            __syncthreads();
            for (int r = threadIdx.x; r < BM; r += 64 * WM * WN) {
                const int row = c.tm * BM + r;
                if (row >= p.M) continue;
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < WN; ++w) m = fmaxf(m, part[w * BM + r].x);
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < WN; ++w) {
                    const float2 q = part[w * BM + r];
                    s += q.x == -INFINITY ? q.y : q.y * __expf(q.x - m);
                }
                p.tile_max[(int64_t)c.tn * p.M + row] = m;
                p.tile_sum[(int64_t)c.tn * p.M + row] = s;
            }
        } else {
            float cs[FN][4];
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) cs[j][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const float top = x.top[i], log2_sum = x.log2_sum[i];
                const int lab = x.lab[i];
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[i][j][e] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][e] - top, kLog2e, -log2_sum));
                if (__any(lab >= w0 && lab < w0 + BN / WN)) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c0 + 16 * j + e == lab) acc[i][j][e] -= 1.0f;
                }
                if (__any(lab == kNoLabel)) {   // no gradient, whatever its logits are
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = lab == kNoLabel ? 0.0f : acc[i][j][e];
                }
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) cs[j][e] += acc[i][j][e];
            }
            __syncthreads();   // the operands are read
            // (G's columns past the last class: 2^-infinity)
            store_rows<FM>(acc, scratch + wave * FM * 2048, p.G, p.ldg, c.tm * BM + wm * (BM / WM), w0, p.g_rows, p.ldg);
            // column sums: 16 lanes of a wavefront, then the WM wavefronts
            float *part = (float *)scratch;   // [WM][BN]
            __syncthreads();
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = cs[j][e];
#pragma unroll
                    for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
                    if ((lane & 15) == 0) part[wm * BN + c0 - c.tn * BN + 16 * j + e] = v;
                }
            __syncthreads();
            for (int k = threadIdx.x; k < BN; k += 64 * WM * WN) {
                const int col = c.tn * BN + k;
                if (col >= p.N || c.tm * BM >= p.M) continue;   // (a tile of the rows behind the last has no sums)
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < WM; ++w) v += part[w * BN + k];
                v *= x.scale;
                p.colpart[(int64_t)c.tm * p.N + col] = v;
            }
        }
    }
}

// ------------------------------------------------------------ small tiles
template <int TYPE, int EPI, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void small_tile(const Args &a, uint32_t block, char *lds) {
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    Coord c;
    if (!coord_of(a, block, c)) return;
    const TileProduct &p = a.p;
    const int kt0 = c.split * a.kt_per_split, nt = min(a.kt_per_split, p.kt - kt0);
    Extras<FM, FN> extras;
    constexpr bool kEarly = FM == 1 && (is_stats(EPI) || EPI == TILE_GRAD);
    if constexpr (kEarly) load_extras<EPI, BM, BN, WM, WN>(p, c, extras);
    f32x4 acc[FM][FN];
    small_loop<TYPE, BM, BN, WM, WN>(p, c, kt0, nt, lds, acc);
    if constexpr (!kEarly) load_extras<EPI, BM, BN, WM, WN>(p, c, extras);
    finish<EPI, BM, BN, WM, WN, FM, FN>(a, c, extras, acc, lds);
}
template <int TYPE, int EPI, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM *WN) void tile_kernel(Args a) {
    __shared__ __attribute__((aligned(16))) char lds[small_lds(TYPE, BM, BN)];
    small_tile<TYPE, EPI, BM, BN, WM, WN>(a, blockIdx.x, lds);
}
// two products in one launch, `first` workgroups (a multiple of 8) for the first:
// few tiles leave CUs idle, and a launch costs about 4 us (the whole loss, in two
// launches / one: 17 x 128, 1009 classes 32.5 / 28.6 us; 2000 x 256, 1009 classes 58 /
// 51)
template <int TYPE, int EPI, int TYPE2, int EPI2>
__global__ __launch_bounds__(256) void pair_kernel(Args a, Args b, uint32_t first) {
    constexpr int la = small_lds(TYPE, 128, 128), lb = small_lds(TYPE2, 128, 128);
    __shared__ __attribute__((aligned(16))) char lds[la > lb ? la : lb];
    if (blockIdx.x < first) small_tile<TYPE, EPI, 128, 128, 2, 2>(a, blockIdx.x, lds);
    else small_tile<TYPE2, EPI2, 128, 128, 2, 2>(b, blockIdx.x - first, lds);
}
// ------------------------------------------------------------ large tiles
template <int TYPE, int EPI>
__global__ __launch_bounds__(kBigThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void big_kernel(Args a) {
    __shared__ __attribute__((aligned(16))) char lds[big_lds(TYPE)];
    Coord c;
    if (!coord_of(a, blockIdx.x, c)) return;
    const TileProduct &p = a.p;
    const int kt0 = c.split * a.kt_per_split;
    f32x4 acc[8][4];
    big_loop<TYPE>(p, c, kt0, min(a.kt_per_split, p.kt - kt0), lds, acc);
    Extras<8, 4> extras;
    load_extras<EPI, kBigT, kBigT, 2, 4>(p, c, extras);
    finish<EPI, kBigT, kBigT, 2, 4, 8, 4>(a, c, extras, acc, lds);
}

// --------------------------------------------------------------- few rows
// Up to 16 FM rows: the weights are read once and there is little to multiply, so
// nothing goes through LDS on the way in.  A workgroup has 16 columns of C and
// all rows; its eight wavefronts take every eighth piece of K, fragments straight
// from memory to registers, and add their sums in wavefront order.  1 x 4096 x 4096:
// 7.2 us, 2.3 TB/s; the launch and a chain of four loads are most of it.
constexpr int kThinWaves = 8, kThin = 64;   // wavefronts; the most rows
template <int TYPE, int EPI, int FM>
__global__ __launch_bounds__(64 * kThinWaves) void thin_kernel(TileProduct p) {
    __shared__ f32x4 part[kThinWaves][FM][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const uint8_t *const b = p.B + (int64_t)min(n0 + fr, p.N - 1) * p.ldb + g * 16;
    const uint8_t *const sbp = p.sb + (int64_t)(n0 / kRows8Block) * p.sb_n;
    const uint8_t *a[FM], *sap[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t r = min(16 * i + fr, p.M - 1);
        a[i] = p.A + r * p.lda + g * 16;
        sap[i] = p.sa + r * p.ldsa;
    }
    f32x4 acc[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int t = wave; t < p.kt; t += kThinWaves) {   // (a second piece's loads in flight: no faster)
        const int64_t o = (int64_t)t * kPiece;
        const Frag fb = {*(const uint4 *)(b + o), *(const uint4 *)(b + o + 64)};
        const int sb = sbp[t * p.sb_k];
        bf16v8 wb[4];
        if constexpr (TYPE == TILE_FP8_EXACT) {
            wb[0] = widen8(fb.lo.x, fb.lo.y);
            wb[1] = widen8(fb.lo.z, fb.lo.w);
            wb[2] = widen8(fb.hi.x, fb.hi.y);
            wb[3] = widen8(fb.hi.z, fb.hi.w);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const Frag fa = {*(const uint4 *)(a[i] + o), *(const uint4 *)(a[i] + o + 64)};
            const int sa = sap[i][t];
            if constexpr (TYPE == TILE_FP8_EXACT) {
                const bf16v8 wa[4] = {widen8(fa.lo.x, fa.lo.y), widen8(fa.lo.z, fa.lo.w), widen8(fa.hi.x, fa.hi.y),
                                      widen8(fa.hi.z, fa.hi.w)};
                f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < 4; ++k) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[k], wa[k], z, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] += __builtin_amdgcn_ldexpf(z[e], sa + sb - 254);
            } else {
                mma<TYPE>(acc[i], fa, fb, sa, sb);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= FM) return;
    f32x4 v = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kThinWaves; ++w) v += part[w][wave][lane];
    const int row = 16 * wave + fr;
    if (row >= p.M) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int col = n0 + 4 * g + e;
        if (col >= p.N) break;
        float x = v[e] + (p.bias ? p.bias[col] : 0.0f);
        if (p.relu) x = x < 0.0f ? 0.0f : x;
        const int64_t at = (int64_t)row * p.ldc + col;
        if constexpr (EPI == TILE_STORE) ((uint16_t *)p.C)[at] = to_bf16(x);
        else ((float *)p.C)[at] = x;
    }
}

// The same of 4-bit rows: a wavefront takes every eighth piece of 256 columns.
template <int EPI, int FM>
__global__ __launch_bounds__(64 * kThinWaves) void thin4_kernel(TileProduct p) {
    __shared__ f32x4 part[kThinWaves][FM][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const uint8_t *const b = p.B + (int64_t)min(n0 + fr, p.N - 1) * p.ldb + g * 16;
    const uint8_t *const sbp = p.sb + (int64_t)(n0 / 64) * 512 + lane * 4;
    const int by = n0 % 64 / 16 * 8;
    const uint8_t *a[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) a[i] = p.A + (int64_t)min(16 * i + fr, p.M - 1) * p.lda + g * 16;
    f32x4 acc[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int t = wave; t < p.kt; t += kThinWaves) {
        const int64_t o = (int64_t)t * kPiece;
        const Frag fb = {*(const uint4 *)(b + o), *(const uint4 *)(b + o + 64)};
        const uint8_t *sbt = sbp + (int64_t)t * p.groups_b * 512, *sat = p.sa + (int64_t)t * p.groups_a * 512 + lane * 4;
        const int b4[2] = {*(const int *)sbt >> by, *(const int *)(sbt + 256) >> by};
        const int a4[2] = {*(const int *)sat, *(const int *)(sat + 256)};
        static_for<FM>([&](auto i) {
            const Frag fa = {*(const uint4 *)(a[i.value] + o), *(const uint4 *)(a[i.value] + o + 64)};
            mma4<i.value, 0>(acc[i.value], fa, fb, a4, b4);
        });
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= FM) return;
    f32x4 v = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kThinWaves; ++w) v += part[w][wave][lane];
    const int row = 16 * wave + fr;
    if (row >= p.M) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int col = n0 + 4 * g + e;
        if (col >= p.N) break;
        float x = v[e] + (p.bias ? p.bias[col] : 0.0f);
        if (p.relu) x = x < 0.0f ? 0.0f : x;   // (NaN stays)
        const int64_t at = (int64_t)row * p.ldc + col;
        if constexpr (EPI == TILE_STORE) ((uint16_t *)p.C)[at] = to_bf16(x);
        else ((float *)p.C)[at] = x;
    }
}

template <int V>
__device__ __forceinline__ auto load_bias(const float *b) {
    typedef float vec __attribute__((ext_vector_type(V)));
    vec v;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = b[e];
    return v;
}
// out = the sum of the partials in split order; the blocks past `main` sum the
// rows of a second small matrix (column sums) the same way.  V elements a
// thread, the partials' loads eight at a time.
template <int V, bool BF>
__global__ __launch_bounds__(256) void reduce_kernel(int32_t splits, int64_t count, int32_t N, const float *acc, void *out,
                                                     int64_t ldo, uint32_t main, int32_t rows2, int32_t N2,
                                                     const float *acc2, float *out2, const float *scale,
                                                     const float *bias, int relu) {
    typedef float vec __attribute__((ext_vector_type(V)));
    if (blockIdx.x >= main) {
        const int32_t k = (int32_t)(blockIdx.x - main) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
        if (k >= N2) return;
        float v = 0.0f;
        for (int32_t r = lane; r < rows2; r += 64) v += acc2[(int64_t)r * N2 + k];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
        if (lane == 0) out2[k] = v;
        return;
    }
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V; i < count; i += (int64_t)main * 256 * V) {
        vec v = *(const vec *)(acc + i);
        int32_t s = 1;
        for (; s + 8 <= splits; s += 8) {
            vec x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = *(const vec *)(acc + (int64_t)(s + u) * count + i);
#pragma unroll
            for (int u = 0; u < 8; ++u) v += x[u];
        }
        for (; s < splits; ++s) v += *(const vec *)(acc + (int64_t)s * count + i);
        if (scale) v *= scale[0];
        const int64_t at = i / N * ldo + i % N;
        if (bias) v += load_bias<V>(bias + i % N);
        if (relu)
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = v[e] < 0.0f ? 0.0f : v[e];   // (NaN stays)
        if constexpr (BF) {
#pragma unroll
            for (int e = 0; e < V; ++e) ((uint16_t *)out)[at + e] = to_bf16(v[e]);
        } else {
            *(vec *)((float *)out + at) = v;
        }
    }
}

template <int TYPE, int EPI>
void launch(TileShape t, const Args &a, unsigned grid, hipStream_t s) {
    if constexpr (TYPE == TILE_FP4) {
        if constexpr (EPI != TILE_PARTIAL) if (t.n == 16) {
            const dim3 g((unsigned)((a.p.N + 15ll) / 16)), b(64 * kThinWaves);
            if (a.p.M <= 16) hipLaunchKernelGGL((thin4_kernel<EPI, 1>), g, b, 0, s, a.p);
            else if (a.p.M <= 32) hipLaunchKernelGGL((thin4_kernel<EPI, 2>), g, b, 0, s, a.p);
            else hipLaunchKernelGGL((thin4_kernel<EPI, 4>), g, b, 0, s, a.p);
            return;
        }
        if (t.m == 64) {
            hipLaunchKernelGGL((tile_kernel<TYPE, EPI, 64, 64, 4, 1>), dim3(grid), dim3(256), 0, s, a);
            return;
        }
    }
    if constexpr (TYPE == TILE_FP8 || TYPE == TILE_FP8_EXACT) {
        if constexpr (EPI != TILE_PARTIAL) if (t.n == 16) {
            const dim3 g((unsigned)((a.p.N + 15) / 16)), b(64 * kThinWaves);
            if (a.p.M <= 16) hipLaunchKernelGGL((thin_kernel<TYPE, EPI, 1>), g, b, 0, s, a.p);
            else if (a.p.M <= 32) hipLaunchKernelGGL((thin_kernel<TYPE, EPI, 2>), g, b, 0, s, a.p);
            else hipLaunchKernelGGL((thin_kernel<TYPE, EPI, 4>), g, b, 0, s, a.p);
            return;
        }
        if constexpr (EPI == TILE_STORE_F32) if (t.m == 64 && t.n == 128) {
            hipLaunchKernelGGL((tile_kernel<TYPE, EPI, 64, 128, 2, 2>), dim3(grid), dim3(256), 0, s, a);
            return;
        }
        if (t.m == 64) {
            hipLaunchKernelGGL((tile_kernel<TYPE, EPI, 64, 64, 4, 1>), dim3(grid), dim3(256), 0, s, a);
            return;
        }
    }
    if constexpr (TYPE == TILE_BF16_NN || TYPE == TILE_F32_NN) {
        if (t.m == 32) {
            hipLaunchKernelGGL((tile_kernel<TYPE, EPI, 32, 128, 2, 2>), dim3(grid), dim3(256), 0, s, a);
            return;
        }
    }
    if constexpr (TYPE == TILE_F32_NN) {
        if (t.m == 64) {
            hipLaunchKernelGGL((tile_kernel<TYPE, EPI, 64, 128, 2, 2>), dim3(grid), dim3(256), 0, s, a);
            return;
        }
    }
    if constexpr (TYPE != TILE_FP8_EXACT && !is_f32(TYPE) && !(TYPE == TILE_FP8 && EPI == TILE_PARTIAL)) {
        if (t.m == kBigT) {
            hipLaunchKernelGGL((big_kernel<TYPE, EPI>), dim3(grid), dim3(kBigThreads), 0, s, a);
            return;
        }
    }
    if constexpr (!(is_fp8(TYPE) && EPI == TILE_PARTIAL) && TYPE != TILE_F32_NN)
        hipLaunchKernelGGL((tile_kernel<TYPE, EPI, 128, 128, 2, 2>), dim3(grid), dim3(256), 0, s, a);
}

int64_t tiles_of(int64_t M, int64_t N, int64_t t) { return ((M + t - 1) / t) * ((N + t - 1) / t); }

}  // namespace

TileShape tile_shape(TileType type, const TileProduct &p) {
    const int32_t splits = std::max(1, p.splits), per = (p.kt + splits - 1) / splits;
    if (type == TILE_FP4) {
        const int64_t t128 = tiles_of(p.M, p.N, 128);
        if (splits > 1) return t128 * splits >= 192 && per >= 16 ? TileShape{128, 128} : TileShape{64, 64};   // (split4)
        // (us, few rows / 64 x 64: 64 x 4096 x 4096 7.3 / 7.8, 32 rows 6.5 / 7.8; 64 x 512 x 1024 6.5 / 6.6)
        if (p.M <= kThin) return TileShape{kThin, 16};
        // us, 64 x 64 / 128 x 128 / 256 x 256, bfloat16 results (the first two 0.3 less since): 6205 x 512 x 602 6.6 / 7.0 /
        // 12.0, 8000 x 512 x 1024 7.4 / 7.7 / 13.5, 2000 x 2048 x 2048 11.2 / 10.5 / 19.7, 16,384 x 512 x 512 9.8 / 8.7 /
        // 11.9, 4000 x 4096 x 1024 23.4 / 19.3 / 18.2; float32 results 24.4 / 31 / 25, 8000 x 2048 x 2048 38 / 36 / 29 (as
        // chosen, 6205 x 512 x 602 7.9, 8000 x 512 x 1024 9.3, 2000 x 2048 x 2048 11.7, 16,384 x 512 x 512 11.3)
        if (tiles_of(p.M, p.N, kBigT) >= 160 && per >= 4 && std::max(p.lda, p.ldb) < (1 << 24)) return TileShape{kBigT, kBigT};
        return t128 < 256 ? TileShape{64, 64} : TileShape{128, 128};
    }
    if (splits > 1 && (type == TILE_FP8 || type == TILE_FP8_EXACT)) return TileShape{64, 64};   // (split8)
    const bool big = type != TILE_FP8_EXACT && !is_f32(type) && tiles_of(p.M, p.N, kBigT) * splits >= 160 && per >= 4 &&
                     (type != TILE_FP8 || per <= kBigPieces) && std::max(p.lda, p.ldb) < (1 << 24);
    // (The count of tiles alone: where the rows fill a part of one tile row only, the other
    // sizes are up to a sixth faster.  The bfloat16 loss with gradients, us, 256 / 128 / 32
    // rows a tile: 17 x 256, 65,536 classes 75 / 67 / 64, 131,072 classes 130 / 115 /
    // 106; 17 x 1024, 131,072 classes 338 / 313 / 323; 128 x 256, 131,072 classes 140 /
    // 127 / 159; but 256 x 256, 131,072 classes 160 / 187 / 222.)
    if (big) return TileShape{kBigT, kBigT};
    if (type == TILE_FP8 || type == TILE_FP8_EXACT) {
        // Few rows (us, few rows / 64 x 64, 4096 x 4096): 1 row 5.0 / 14.7, 16 7.4 /
        // 14.8, 32 10.3 / 14.8, 64 15.8 / 14.9, 128 27 / 15; float32 results 1 5.1 /
        // 20.9, 64 16.1 / 21.4, 128 28 / 22; 64 rows, 1024 x 512 4.3 / 5.0.
        if (p.M <= kThin) return TileShape{kThin, 16};
        // 64 x 64 tiles where 128 x 128 ones leave CUs without a block (us, 128 /
        // 64, 8-bit): 500 x 4096 x 4096 33 / 20, 2000 x 512 x 1024 11.2 / 6.8,
        // 8000 x 512 x 640 10.3 / 9.4, but 8000 x 1024 x 512 (504 blocks) 12.1 /
        // 13.8; float32 results 50 / 35, 16.4 / 9.0, 14.3 / 14.9 (6205 x 512 x
        // 640), 8000 x 2048 x 2048 88 / 118.
        // 64 x 128 tiles for float32 results widen fewer operands a product.  They take
        // the place of 64 x 64 ones past one and a half a CU (us, 64 x 64 / 64 x 128:
        // K = 1024 at 384 of them 14.8 / 16.5, at 400 18.6 / 16.3; K = 128 7.6 / 8.1
        // and 8.9 / 8.0; K = 4096 41.6 / 45 and 53 / 45) and of the second round of 128 x
        // 128 ones while they need three rounds themselves (128 x 128 / 64 x 128: K =
        // 1024 at 513 .. 768 24.5 / 20.8, 772 .. 1024 25.0 / 26.8; K = 4096 71 / 60-64 and
        // 72 / 80; K = 128 10.5 / 9.2 and 10.8 / 12.0).  Whole columns of tiles; where
        // the last one is at most half full they gain less and 64 x 64 ones would be the
        // fastest (38,400 x 64, K = 2048: 128 x 128 38, 64 x 128 32, 64 x 64 23).  bfloat16
        // results: 1000 x 4096 x 2048 (64 x 64 / 64 x 128) 18.7 / 21.8.
        const int64_t wide = ((int64_t)p.M + 63) / 64 * (((int64_t)p.N + 127) / 128);
        if (type == TILE_FP8_EXACT && splits == 1 && wide > 384 && wide <= 768) return TileShape{64, 128};
        if (tiles_of(p.M, p.N, 128) < 256) return TileShape{64, 64};
    }
    if ((type == TILE_BF16_NN || type == TILE_F32_NN) && tiles_of(p.M, p.N, 128) < 256) return TileShape{32, 128};
    // Three of these a CU instead of two 128 x 128 ones (the loss, 128 / 64 rows, us): 2000
    // x 64, 3000 classes without gradient 25.5 / 21.8, 2000 x 256, 10,007 classes 124 / 114,
    // with gradient 353 / 344; but 4096 x 512, 20,000 classes 2207 / 2227.
    if (type == TILE_F32_NN) return TileShape{64, 128};
    return TileShape{128, 128};
}

int32_t tile_splits(int32_t M, int32_t N, int32_t kt, bool f32) {
    if (f32)   // one round of two blocks a CU, four pieces or more each
        return (int32_t)std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(1, tiles_of(M, N, 128)), kt / 4, 64}));
    // large tiles: one round of the 256 CUs; small ones: two blocks a CU, as
    // long as a part has two pieces
    const int64_t tiles = std::max<int64_t>(1, tiles_of(M, N, kBigT));
    int64_t sp = std::max<int64_t>(1, 256 / tiles);
    if (sp > kt / 8) sp = std::min<int64_t>(512 / std::max<int64_t>(1, tiles_of(M, N, 128)), kt / 2);
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(sp, 64));
}

int32_t tile_rows(TileShape t, TileEpilogue epi, const TileProduct &p) {
    return (int32_t)(((epi == TILE_GRAD ? std::max<int64_t>(p.M, p.g_rows) : p.M) + t.m - 1) / t.m);
}

// a product's tiles and grid
static int tile_args(const TileShape &t, TileEpilogue epi, const TileProduct &p, Args &a, unsigned &grid) {
    if (std::max(p.M, p.N) > kMostRows) {   // (row numbers past the last tile's end stay within 32 bits)
        set_error("tile_product: %d x %d is too large", p.M, p.N);
        return GCN_EUNSUPPORTED;
    }
    a.p = p;
    a.tiles_m = tile_rows(t, epi, p);
    a.tiles_n = (int32_t)(((int64_t)p.N + t.n - 1) / t.n);
    const int32_t splits = std::max(1, p.splits);
    a.kt_per_split = (p.kt + splits - 1) / splits;
    a.band = 8;
    const int64_t total = (int64_t)splits * a.tiles_m * a.tiles_n;
    if (total > 0x7FFFF0) {   // (threads of a launch: 32 bits)
        set_error("tile_product: %d x %d is too large", p.M, p.N);
        return GCN_EUNSUPPORTED;
    }
    a.total = (uint32_t)total;
    a.per_xcd = (a.total + 7) / 8;
    grid = 8 * a.per_xcd;
    return GCN_OK;
}

int tile_products(bool f32, const TileProduct &nt, const TileProduct &tn, TileEpilogue epi, hipStream_t s) {
    const TileType tt = f32 ? TILE_F32 : TILE_BF16, ut = f32 ? TILE_F32_TN : TILE_BF16_TN;
    const TileShape t = tile_shape(tt, nt), u = tile_shape(ut, tn);
    int rc;
    if (t.m != 128 || u.m != 128) {
        if ((rc = tile_product(tt, TILE_PARTIAL, nt, s))) return rc;
        return tile_product(ut, epi, tn, s);
    }
    Args a, b;
    unsigned ga, gb;
    if ((rc = tile_args(t, TILE_PARTIAL, nt, a, ga)) || (rc = tile_args(u, epi, tn, b, gb))) return rc;
    // (the long sums first: the other's many short parts fill what their last round leaves)
#define GCN_PAIR(NT, TN, EPI) \
    hipLaunchKernelGGL((pair_kernel<TN, EPI, NT, TILE_PARTIAL>), dim3(ga + gb), dim3(256), 0, s, b, a, gb)
    if (f32 && epi == TILE_STORE_F32) GCN_PAIR(TILE_F32, TILE_F32_TN, TILE_STORE_F32);
    else if (f32) GCN_PAIR(TILE_F32, TILE_F32_TN, TILE_PARTIAL);
    else if (epi == TILE_STORE) GCN_PAIR(TILE_BF16, TILE_BF16_TN, TILE_STORE);
    else GCN_PAIR(TILE_BF16, TILE_BF16_TN, TILE_PARTIAL);
#undef GCN_PAIR
    GCN_LAUNCH_CHECK("pair_kernel");
    return GCN_OK;
}

int tile_product(TileType type, TileEpilogue epi, const TileProduct &p, hipStream_t s) {
    if (p.M <= 0 || p.N <= 0) return GCN_OK;
    const TileShape t = tile_shape(type, p);
    Args a;
    unsigned grid;
    if (const int rc = tile_args(t, epi, p, a, grid)) return rc;
    // (the pairs that the entry points use)
    if (type == TILE_BF16_NN && epi == TILE_STATS) launch<TILE_BF16_NN, TILE_STATS>(t, a, grid, s);
    else if (type == TILE_BF16_NN && epi == TILE_GRAD) launch<TILE_BF16_NN, TILE_GRAD>(t, a, grid, s);
    else if (type == TILE_F32_NN && epi == TILE_STATS) launch<TILE_F32_NN, TILE_STATS>(t, a, grid, s);
    else if (type == TILE_F32_NN && epi == TILE_STATS_STORE) launch<TILE_F32_NN, TILE_STATS_STORE>(t, a, grid, s);
    else if (type == TILE_F32_NN && epi == TILE_STORE_F32) launch<TILE_F32_NN, TILE_STORE_F32>(t, a, grid, s);
    else if (type == TILE_BF16 && epi == TILE_PARTIAL) launch<TILE_BF16, TILE_PARTIAL>(t, a, grid, s);
    else if (type == TILE_BF16_TN && epi == TILE_STORE) launch<TILE_BF16_TN, TILE_STORE>(t, a, grid, s);
    else if (type == TILE_BF16_TN && epi == TILE_PARTIAL) launch<TILE_BF16_TN, TILE_PARTIAL>(t, a, grid, s);
    else if (type == TILE_FP4 && epi == TILE_STORE) launch<TILE_FP4, TILE_STORE>(t, a, grid, s);
    else if (type == TILE_FP4 && epi == TILE_STORE_F32) launch<TILE_FP4, TILE_STORE_F32>(t, a, grid, s);
    else if (type == TILE_FP4 && epi == TILE_PARTIAL) launch<TILE_FP4, TILE_PARTIAL>(t, a, grid, s);
    else if (type == TILE_FP8 && epi == TILE_STORE) launch<TILE_FP8, TILE_STORE>(t, a, grid, s);
    else if (type == TILE_FP8 && epi == TILE_PARTIAL) launch<TILE_FP8, TILE_PARTIAL>(t, a, grid, s);
    else if (type == TILE_FP8_EXACT && epi == TILE_PARTIAL) launch<TILE_FP8_EXACT, TILE_PARTIAL>(t, a, grid, s);
    else if (type == TILE_FP8_EXACT && epi == TILE_STORE_F32) launch<TILE_FP8_EXACT, TILE_STORE_F32>(t, a, grid, s);
    else {
        set_error("tile_product: type %d with epilogue %d", (int)type, (int)epi);
        return GCN_EUNSUPPORTED;
    }
    GCN_LAUNCH_CHECK("tile_kernel");
    return GCN_OK;
}

int tile_reduce(int32_t splits, int32_t M, int32_t N, const float *acc, void *out, int out_bf16, int64_t ldo, hipStream_t s,
                int32_t rows2, int32_t N2, const float *acc2, float *out2, const float *scale,
                const float *bias, int relu) {
    const int64_t count = (int64_t)M * N;
    if (count == 0) return GCN_OK;
    const bool vec = N % 4 == 0 && ldo % 4 == 0 && (uintptr_t)out % 16 == 0;
    const uint32_t main = (uint32_t)std::min<int64_t>((count / (vec ? 4 : 1) + 255) / 256, 8192);
    const dim3 g(main + (uint32_t)((N2 + 3) / 4));
#define GCN_REDUCE(V, BF) \
    hipLaunchKernelGGL((reduce_kernel<V, BF>), g, dim3(256), 0, s, splits, count, N, acc, out, ldo, main, rows2, N2, acc2, out2, scale, bias, relu)
    if (vec) {
        if (out_bf16) GCN_REDUCE(4, true);
        else GCN_REDUCE(4, false);
    } else {
        if (out_bf16) GCN_REDUCE(1, true);
        else GCN_REDUCE(1, false);
    }
#undef GCN_REDUCE
    GCN_LAUNCH_CHECK("reduce_kernel");
    return GCN_OK;
}

}  // namespace gcn

using namespace gcn;

// Parts of a product's contraction: where 64 x 64 tiles leave half of the CUs
// without a block and there are pieces enough to pay for a second launch (us,
// unsplit / split: 500 x 4096 x 512 15.3 / 10.9, 500 x 2048 x 512 9.4 / 10.5, 1000 x
// 1024 x 512 7.9 / 10.6; float32 results 500 x 4096 x 512 21.6 / 12.9, 300 x 2048 x
// 256 12.5 / 10.2, 100 x 1024 x 256 8.4 / 10.4).
static int32_t split8(int32_t M, int32_t N, int32_t kt, bool bf) {
    const int64_t tiles = ((int64_t)M + 63) / 64 * (((int64_t)N + 63) / 64);
    if (M <= 64 || tiles > 128 || kt < (bf ? 24 : 16)) return 1;
    const int32_t sp = (int32_t)std::min<int64_t>(256 / tiles, kt / 4), per = (kt + sp - 1) / sp;
    return (kt + per - 1) / per;
}

extern "C" {

size_t gcn_rows8_product_workspace_bytes(int32_t n, int32_t K, int32_t N) {
    if (n < 0 || K <= 0 || N <= 0) return 0;
    // (either direction; float32 results are split earlier)
    size_t most = 0;
    for (int t = 0; t < 2; ++t) {
        const int32_t cols = t ? K : N, sp = split8(n, cols, (int32_t)blocks8(t ? N : K), false);
        if (sp > 1) most = std::max(most, (size_t)sp * n * cols);
    }
    return 256 + sizeof(float) * most;
}

int gcn_rows8_product(const gcn_rows8 *X8, const gcn_weights8 *W8, int transpose, const float *bias, int relu, void *Y,
                      gcn_rows_type type, int32_t ldy, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_rows8(X8, "gcn_rows8_product");
    if (rc) return rc;
    GCN_REQUIRE(W8, GCN_EINVAL, "gcn_rows8_product: null 8-bit weights");
    GCN_REQUIRE(W8->K > 0 && W8->N > 0, GCN_ESHAPE, "gcn_rows8_product: 8-bit weights of %d x %d", W8->K, W8->N);
    GCN_REQUIRE(type == GCN_ROWS_F32 || type == GCN_ROWS_BF16, GCN_EINVAL, "gcn_rows8_product: bad element type %d",
                (int)type);
    const int32_t K = transpose ? W8->N : W8->K, N = transpose ? W8->K : W8->N;   // contraction, columns of Y
    const uint8_t *w = transpose ? W8->q : W8->qT;
    const int32_t ldw = transpose ? W8->ldq : W8->ldqT;
    GCN_REQUIRE(X8->f == K, GCN_ESHAPE, "gcn_rows8_product: rows of %d columns against %d", X8->f, K);
    GCN_REQUIRE(w && W8->scale, GCN_EINVAL, "gcn_rows8_product: the weights' %s orientation is missing",
                transpose ? "q" : "qT");
    GCN_REQUIRE(ldw % 16 == 0 && ldw >= kRows8Block * blocks8(K) && (uintptr_t)w % 16 == 0, GCN_ESHAPE,
                "gcn_rows8_product: weight rows need 16-byte alignment and a stride (%d) that is a multiple of 16 of at "
                "least %lld", ldw, (long long)(kRows8Block * blocks8(K)));
    GCN_REQUIRE(W8->ldscale >= blocks8(W8->N), GCN_ESHAPE, "gcn_rows8_product: ldscale=%d < %lld", W8->ldscale,
                (long long)blocks8(W8->N));
    GCN_REQUIRE(ldy >= N, GCN_ESHAPE, "gcn_rows8_product: ldy=%d < %d", ldy, N);
    GCN_REQUIRE(X8->n == 0 || Y, GCN_EINVAL, "gcn_rows8_product: null Y");
    GCN_REQUIRE(X8->n == 0 || (uintptr_t)Y % (type == GCN_ROWS_BF16 ? 2 : 4) == 0, GCN_EINVAL,
                "gcn_rows8_product: misaligned Y");
    GCN_REQUIRE(ws && (uintptr_t)ws % 256 == 0 &&
                    ws_bytes >= gcn_rows8_product_workspace_bytes(X8->n, W8->K, W8->N), GCN_EWORKSPACE,
                "gcn_rows8_product: workspace %zu < %zu bytes, or not 256-byte aligned", ws_bytes,
                gcn_rows8_product_workspace_bytes(X8->n, W8->K, W8->N));
    if (X8->n == 0) return GCN_OK;
    TileProduct p{};
    p.A = X8->q;
    p.lda = X8->ldq;
    p.B = w;
    p.ldb = ldw;
    p.M = X8->n;
    p.N = N;
    p.kt = (int32_t)blocks8(K);
    p.splits = 1;
    p.sa = X8->scale;
    p.ldsa = X8->ldscale;
    p.sb = W8->scale;
    p.sb_n = transpose ? W8->ldscale : 1;
    p.sb_k = transpose ? 1 : W8->ldscale;
    p.C = Y;
    p.ldc = ldy;
    const bool bf = type == GCN_ROWS_BF16;
    p.relu = relu;
    p.bias = bias;
    hipStream_t s = (hipStream_t)stream;
    ProfScope prof(K_ROWS8_PRODUCT, s, 2.0 * p.M * N * K,
                   (double)p.M * K + (double)N * K + (double)p.M * N * (bf ? 2.0 : 4.0));
    p.splits = split8(p.M, p.N, p.kt, bf);
    if (p.splits > 1) {
        p.acc = (float *)ws;
        if ((rc = tile_product(bf ? TILE_FP8 : TILE_FP8_EXACT, TILE_PARTIAL, p, s))) return rc;
        return tile_reduce(p.splits, p.M, p.N, p.acc, Y, bf, ldy, s, 0, 0, nullptr, nullptr, nullptr, bias, relu);
    }
    return bf ? tile_product(TILE_FP8, TILE_STORE, p, s) : tile_product(TILE_FP8_EXACT, TILE_STORE_F32, p, s);
}

}  // extern "C"
