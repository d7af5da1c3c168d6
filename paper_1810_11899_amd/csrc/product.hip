// Products C = A B^T of bfloat16, 8-bit or float32 rows on the matrix cores, with
// the epilogues of the 8-bit layer products and of the many-class loss.
//
// Both operands come in rows of 128-byte pieces (32 float32, 64 bfloat16 or 128
// e4m3 values), so one tile loop serves all types: a piece of each tile row is
// copied from global memory straight into LDS (16 bytes a lane), and a lane's
// share of a fragment is the two 16-byte chunks g and g + 4 of a row (g = lane
// / 16): eight k-steps of v_mfma_f32_16x16x4_f32, two of
// v_mfma_f32_16x16x32_bf16, or the one of
// v_mfma_scale_f32_16x16x128_f8f6f4.  Which 16 of the 128 columns a chunk holds
// does not matter as long as both operands agree.  LDS rows are 128 bytes with
// their chunks XOR-swizzled by row, so that the 16 lanes of a fragment read
// spread over the banks.
//
// The instructions are issued with B's fragment first, which leaves a lane
// with four consecutive columns of one row of C.
#include <algorithm>
#include <type_traits>

#include "rows8.h"

namespace gcn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16v8 __attribute__((ext_vector_type(8)));

constexpr int kPiece = 128;   // bytes of a row in one stage

struct Args {
    TileProduct p;
    int32_t tiles_m, tiles_n, kt_per_split, band;
    uint32_t total, per_xcd;
};

// Workgroups go round-robin over the 8 XCDs (workgroup b runs on XCD b % 8);
// logical tiles are numbered XCD-major, and within that in bands of `band` row
// tiles, row tile fastest, so that the tiles running at once on an XCD share
// operand panels in its L2.
struct Coord {
    int split, tm, tn;
};
__device__ __forceinline__ bool coord_of(const Args &a, uint32_t block, Coord &c) {
    const uint32_t L = (block & 7) * a.per_xcd + (block >> 3);
    if (L >= a.total) return false;
    const uint32_t per_split = (uint32_t)a.tiles_m * a.tiles_n;
    c.split = (int)(L / per_split);
    const uint32_t r = L - c.split * per_split;
    const uint32_t in_band = (uint32_t)a.band * a.tiles_n;
    const uint32_t b = r / in_band, q = r - b * in_band;
    const uint32_t h = (uint32_t)min(a.band, a.tiles_m - (int)b * a.band);
    c.tn = (int)(q / h);
    c.tm = (int)b * a.band + (int)(q - c.tn * h);
    return true;
}

struct Frag {
    uint4 lo, hi;
};

constexpr bool is_fp8(int type) { return type == TILE_FP8 || type == TILE_FP8_EXACT; }
constexpr bool is_f32(int type) { return type == TILE_F32 || type == TILE_F32_TN || type == TILE_F32_NN; }
// which operands are stored along the other way
constexpr bool km_a(int type) { return type == TILE_BF16_TN || type == TILE_F32_TN; }
constexpr bool km_b(int type) { return km_a(type) || type == TILE_BF16_NN || type == TILE_F32_NN; }
constexpr bool is_stats(int epi) { return epi == TILE_STATS || epi == TILE_STATS_STORE; }

template <int TYPE>
__device__ __forceinline__ void mma(f32x4 &acc, const Frag &a, const Frag &b, int sa, int sb) {
    if constexpr (!is_fp8(TYPE)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16v8, b.lo),
                                                      __builtin_bit_cast(bf16v8, a.lo), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16v8, b.hi),
                                                      __builtin_bit_cast(bf16v8, a.hi), acc, 0, 0, 0);
    } else if constexpr (TYPE == TILE_FP8) {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, b),
                                                               __builtin_bit_cast(i32x8, a), acc, 0, 0, 0, sb, 0, sa);
    }
}

// Operands stored along the other way (KM: K x rows): a stage holds 64 k-rows
// of 128 elements, 16 chunks of 16 bytes each, chunk c of k-row k at place
// c ^ 4 (k % 4).  The gfx950 transposing LDS read gives a group of 16 lanes, whose
// lane j addresses 4 elements of k-row kb + j / 4 at 4 (j % 4), the elements of
// its own column at k-rows kb .. kb + 3; the swizzle keeps the four k-rows of a
// group on different banks.  km_place: lane's byte offset for the 16 columns
// from chunk c0 (c0 even) in group g's k-rows 8 g ..; a fragment is the four
// pieces of k-rows 8 g, 8 g + 4 and 32 further on.
typedef short v4i16 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ int km_place(int lane, int c0) {
    const int j = lane & 15, k = 8 * (lane >> 4) + (j >> 2);
    return k * 256 + (((c0 + ((j & 3) >> 1)) ^ (4 * (j >> 2))) * 16) + (j & 1) * 8;
}
__device__ __forceinline__ uint2 km_read(const char *p) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)p));
}
__device__ __forceinline__ Frag km_frag(const char *p) {
    const uint2 a = km_read(p), b = km_read(p + 4 * 256), c = km_read(p + 32 * 256), d = km_read(p + 36 * 256);
    return Frag{make_uint4(a.x, a.y, b.x, b.y), make_uint4(c.x, c.y, d.x, d.y)};
}

// The same of float32: a stage holds 32 k-rows of 128 elements, 32 chunks each,
// chunk c of k-row k at place c ^ 4 (k / 4 % 4), which keeps the k-rows 4 g + q that
// one read takes on different banks; an element at a time.
__device__ __forceinline__ Frag km_frag_f32(const char *tile, int lane, int col) {
    const int fr = lane & 15, g = lane >> 4;
    const char *p = tile + 4 * g * 512 + (((col + fr) / 4) ^ (4 * g)) * 16 + (fr & 3) * 4;
    Frag f;
    uint32_t *l = (uint32_t *)&f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        l[q] = *(const uint32_t *)(p + q * 512);
        l[q + 4] = *(const uint32_t *)(p + (q + 16) * 512);
    }
    return f;
}

// eight e4m3 values as bfloat16, exactly
typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16v8 widen8(uint32_t x, uint32_t y) {
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, (bf16v2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false));
    r.y = __builtin_bit_cast(uint32_t, (bf16v2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true));
    r.z = __builtin_bit_cast(uint32_t, (bf16v2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.0f, false));
    r.w = __builtin_bit_cast(uint32_t, (bf16v2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.0f, true));
    return __builtin_bit_cast(bf16v8, r);
}

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

// ---------------------------------------------------------------- copies
// 16 bytes a lane from base + off straight to LDS at dst + 16 lane (base, dst
// uniform).  In assembly because the compiler, which sees only that both touch
// LDS, puts a wait for every outstanding copy before each LDS read, and these
// kernels keep copies in flight over many of them.  The instruction has no
// register result that could be taken for written, its operands are read as it
// is issued, and the kernel waits by wait_copies and a barrier.
__device__ __forceinline__ void copy_to_lds(const uint8_t *base, uint32_t off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy_to_lds(const uint8_t *from, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(from) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// a barrier alone: the fence of __syncthreads would wait for every copy
__device__ __forceinline__ void turn() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// ------------------------------------------------------------ small tiles
// WM x WN wavefronts and two stages: while piece t is multiplied, the copies of
// the next are in flight, and one barrier a piece both publishes it and frees
// the stage of the piece before.  Two or more workgroups a CU hide what a copy
// takes beyond that (three and four stages, which leave room for fewer of
// them, were no faster at any of the sizes below).  Scales are staged for
// kScalePieces pieces at a time.
constexpr int kScalePieces = 64;
constexpr int small_lds(int type, int BM, int BN) {
    return 2 * (BM + BN) * kPiece + (is_fp8(type) ? kScalePieces * (BM + 1) : 0);
}
template <int TYPE, int EPI, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void small_tile(const Args &a, uint32_t block, char *lds) {
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16, T = 64 * WM * WN;
    constexpr int kStage = (BM + BN) * kPiece;
    constexpr int LA = BM * kPiece / 16 / T, LB = BN * kPiece / 16 / T;
    static_assert(LA * T * 16 == BM * kPiece && LB * T * 16 == BN * kPiece, "whole chunks per lane");
    static_assert(kRows8Block % BN == 0, "a tile's columns share a scale");
    constexpr bool SCALED = is_fp8(TYPE);
    Coord c;
    if (!coord_of(a, block, c)) return;
    const TileProduct &p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int m0 = c.tm * BM, n0 = c.tn * BN;
    const int kt0 = c.split * a.kt_per_split, nt = min(a.kt_per_split, p.kt - kt0);
    constexpr bool KA = km_a(TYPE), KB = km_b(TYPE);
    static_assert((!KA || BM == 128) && (!KB || BN == 128), "k-rows of 128 elements");
    constexpr int E = is_f32(TYPE) ? 4 : 2, V = 16 / E, CH = 128 / V;   // of k-major operands: bytes, elements a chunk, chunks a row
    const int64_t step_a = KA ? kPiece / E * p.lda : kPiece, step_b = KB ? kPiece / E * p.ldb : kPiece;
    // Copy u of a thread: tile row (u T + thread) / 8, stored chunk thread % 8,
    // which holds the row's chunk (thread % 8) ^ (row % 8); rows past the extent
    // are clamped (their products are dropped).  k-major: k-row (u T + thread) /
    // CH, its chunks clamped to the last whole one.
    const int lr = threadIdx.x >> 3, chunk = ((threadIdx.x & 7) ^ (lr & 7)) * 16;
    auto km_at = [&](int64_t ld, int x0, int extent, int u) {
        const int k = (u * T + threadIdx.x) / CH, ch = V * ((threadIdx.x % CH) ^ (4 * ((is_f32(TYPE) ? k >> 2 : k) & 3)));
        return k * ld + E * (int64_t)min(x0 + ch, ((extent + V - 1) & -V) - V);
    };
    const uint8_t *ga[LA], *gb[LB];
#pragma unroll
    for (int u = 0; u < LA; ++u)
        ga[u] = p.A + kt0 * step_a +
                (KA ? km_at(p.lda, m0, p.M, u) : (int64_t)min(m0 + u * (T / 8) + lr, p.M - 1) * p.lda + chunk);
#pragma unroll
    for (int u = 0; u < LB; ++u)
        gb[u] = p.B + kt0 * step_b +
                (KB ? km_at(p.ldb, n0, p.N, u) : (int64_t)min(n0 + u * (T / 8) + lr, p.N - 1) * p.ldb + chunk);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
    auto copy = [&](int t, int stage) {
        const uint32_t d = lds0 + stage * kStage;
#pragma unroll
        for (int u = 0; u < LA; ++u) copy_to_lds(ga[u] + t * step_a, d + u * T * 16);
#pragma unroll
        for (int u = 0; u < LB; ++u) copy_to_lds(gb[u] + t * step_b, d + BM * kPiece + u * T * 16);
    };
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Extras<FM, FN> extras;
    constexpr bool kEarly = FM == 1 && (is_stats(EPI) || EPI == TILE_GRAD);
    if constexpr (kEarly) load_extras<EPI, BM, BN, WM, WN>(p, c, extras);
    const int fr = lane & 15, g = lane >> 4;
    const int o0 = (g ^ (fr & 7)) * 16, o1 = ((g + 4) ^ (fr & 7)) * 16;   // (a fragment's rows start at multiples of 16)
    auto frag = [&](const char *tile, int row, bool km) {
        if (km) return is_f32(TYPE) ? km_frag_f32(tile, lane, row) : km_frag(tile + km_place(lane, row / 8));
        const char *q = tile + (row + fr) * kPiece;
        return Frag{*(const uint4 *)(q + o0), *(const uint4 *)(q + o1)};
    };
    uint8_t *const s8 = (uint8_t *)lds + 2 * kStage;   // [piece][BM rows], then [piece]
    auto scales = [&](int t) {
        const int w = min(kScalePieces, nt - t);
        for (int i = threadIdx.x; i < BM * w; i += T) {
            const int r = i / w, k = i - r * w;
            s8[k * BM + r] = p.sa[(int64_t)min(m0 + r, p.M - 1) * p.ldsa + kt0 + t + k];
        }
        for (int k = threadIdx.x; k < w; k += T)
            s8[kScalePieces * BM + k] = p.sb[(int64_t)(n0 / kRows8Block) * p.sb_n + (int64_t)(kt0 + t + k) * p.sb_k];
    };
    if constexpr (SCALED) {
        if (nt > 0) scales(0);
    }
    if (nt > 0) copy(0, 0);
    for (int t = 0; t < nt; ++t) {
        if constexpr (SCALED) {
            if (t % kScalePieces == 0 && t) {
                turn();   // every wavefront has read the old ones
                scales(t);
            }
            wait_reads();   // the scales' LDS writes, ahead of the barrier
        }
        wait_copies<0>();   // piece t has landed
        turn();
        // (every wavefront has used what it read of piece t - 1: its stage is free)
        if (t + 1 < nt) copy(t + 1, (t + 1) & 1);
        const char *ta = lds + (t & 1) * kStage, *tb = ta + BM * kPiece;
        int sa[FM], sb = 0;
        if constexpr (SCALED) {
            const int k = t % kScalePieces;
#pragma unroll
            for (int i = 0; i < FM; ++i) sa[i] = s8[k * BM + wm * (BM / WM) + 16 * i + fr];
            sb = s8[kScalePieces * BM + k];
        }
        Frag fb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[j] = frag(tb, wn * (BN / WN) + 16 * j, KB);
        if constexpr (TYPE == TILE_FP8_EXACT) {
            bf16v8 wb[FN][4];
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                wb[j][0] = widen8(fb[j].lo.x, fb[j].lo.y);
                wb[j][1] = widen8(fb[j].lo.z, fb[j].lo.w);
                wb[j][2] = widen8(fb[j].hi.x, fb[j].hi.y);
                wb[j][3] = widen8(fb[j].hi.z, fb[j].hi.w);
            }
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const Frag fa = frag(ta, wm * (BM / WM) + 16 * i, KA);
                const bf16v8 wa[4] = {widen8(fa.lo.x, fa.lo.y), widen8(fa.lo.z, fa.lo.w), widen8(fa.hi.x, fa.hi.y),
                                      widen8(fa.hi.z, fa.hi.w)};
                const int e = sa[i] + sb - 254;
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][k], wa[k], z, 0, 0, 0);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j][q] += __builtin_amdgcn_ldexpf(z[q], e);
                }
            }
        } else if constexpr (is_f32(TYPE)) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const Frag fa = frag(ta, wm * (BM / WM) + 16 * i, KA);
                // element q of the lo and hi chunks: k = 4 g + q, 16 + 4 g + q; the columns
                // innermost, so that a product does not wait for the sum before it
#pragma unroll
                for (int q = 0; q < 8; ++q)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            __builtin_bit_cast(f32x4, q < 4 ? fb[j].lo : fb[j].hi)[q & 3],
                            __builtin_bit_cast(f32x4, q < 4 ? fa.lo : fa.hi)[q & 3], acc[i][j], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const Frag fa = frag(ta, wm * (BM / WM) + 16 * i, KA);
#pragma unroll
                for (int j = 0; j < FN; ++j) mma<TYPE>(acc[i][j], fa, fb[j], TYPE == TILE_FP8 ? sa[i] : 0, sb);
            }
        }
        // what was read is used before the next barrier: the products stay above it
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                if constexpr (TYPE == TILE_FP8_EXACT) asm volatile("" : "+v"(acc[i][j]));
                else asm volatile("" : "+a"(acc[i][j]));   // (where the products leave them: pinned elsewhere they are moved there and back)
            }
    }
    __syncthreads();
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
// 256 x 256 tiles of 8 wavefronts (2 along M, 4 along N; 128 x 64 each), one
// workgroup a CU, two wavefronts a SIMD that take turns: while one multiplies a
// quarter of its tile, the other reads fragments and issues copies, and a
// barrier every quarter swaps them.  The wavefronts of the second row start one
// barrier late, which keeps the two halves apart for the whole loop.
//
// A piece of the tile is four regions of 128 rows: A's and B's rows that the
// first and the second quarter of every wavefront reads.  Quarters of piece t:
//   0: A-lo x B-lo (reads A-lo)      1: A-lo x B-hi (reads B-hi)
//   2: A-hi x B-hi (reads A-hi)      3: A-hi x B-lo (reads B-lo of t + 1)
// Two pieces are in LDS (128 KB); a region is refilled two quarters after it
// was read, with the rows of two pieces later, which are read six quarters
// after that: copies have about 3000 cycles to land, and no wait is ever for
// the newest ones.
//
// Order of events.  Call a stretch between barriers a turn: the first half of
// the wavefronts reads in quarter q at turn 2q and multiplies at 2q + 1, the
// second one a turn later.  Reads of quarter q have returned to their
// wavefront by the end of its multiplication, turn 2q + 2 at the latest, and
// copies over them go out in quarter q + 2, turn 2q + 4 at the earliest.  A
// wavefront waits for its own copies of what quarter q + 1 reads in quarter q,
// turn 2q + 1 at the latest; quarter q + 1 reads at turn 2q + 2 at the earliest.
//
// 16,384 x 4096 x 8192 of 8-bit operands: 450 us, 2.4 PFLOP/s; 16,384 x 1024 x
// 16,384 of bfloat16 ones: 410-425 us, 1300 TFLOP/s.  The chip's power bounds both
// (zeros instead of random operands: 505 -> 385 us).
constexpr int kBigT = 256, kBigThreads = 512;
constexpr int kRegion = 128 * kPiece, kBuffer = 4 * kRegion;
constexpr int kBigPieces = 120;                          // pieces whose scales fit in LDS
constexpr int kScaleA = kBigPieces * 64 * 4, kScaleB = kBigPieces * 2;

template <int TYPE, int I>
__device__ __forceinline__ void mma_big(f32x4 &acc, const Frag &a, const Frag &b, int sa, int sb) {
    if constexpr (TYPE == TILE_FP8)
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, b),
                                                               __builtin_bit_cast(i32x8, a), acc, 0, 0, 0, sb, I, sa);
    else
        mma<TYPE>(acc, a, b, 0, 0);
}

template <int TYPE, int EPI>
__global__ __launch_bounds__(kBigThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void big_kernel(Args a) {
    __shared__ __attribute__((aligned(16))) char lds[2 * kBuffer + (TYPE == TILE_FP8 ? kScaleA + kScaleB : 0)];
    Coord c;
    if (!coord_of(a, blockIdx.x, c)) return;
    const TileProduct &p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const int m0 = c.tm * kBigT, n0 = c.tn * kBigT;
    const int kt0 = c.split * a.kt_per_split;
    const int nt = min(a.kt_per_split, p.kt - kt0);

    // Copies: region row (8 u + wave) 8 + lane / 8, stored chunk lane % 8 with
    // the row's chunk (lane % 8) ^ (row % 8); rows past the extent are clamped.
    // k-major: k-row (8 u + wave) 4 + lane / 16, stored chunk lane % 16, which is one
    // of the 8 of A's first or second half's columns in the region, or of the 4
    // of B's four quarters'; chunks past the extent are clamped to the last.
    constexpr bool KA = km_a(TYPE), KB = km_b(TYPE);
    const int64_t step_a = KA ? 64 * p.lda : kPiece, step_b = KB ? 64 * p.ldb : kPiece;
    const uint8_t *const ba = p.A + (KA ? (int64_t)m0 * 2 : (int64_t)m0 * p.lda) + kt0 * step_a;
    const uint8_t *const bb = p.B + (KB ? (int64_t)n0 * 2 : (int64_t)n0 * p.ldb) + kt0 * step_b;
    uint32_t oa[2][2], ob[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int rr = (8 * u + wave) * 8 + (lane >> 3);
        const uint32_t ch = (uint32_t)(((lane & 7) ^ (rr & 7)) * 16);
        const int k = (8 * u + wave) * 4 + (lane >> 4), gc = (lane & 15) ^ (4 * (k & 3));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (KA)
                oa[h][u] = (uint32_t)k * (uint32_t)p.lda +
                           2 * (uint32_t)min((gc >> 3) * 128 + 64 * h + (gc & 7) * 8, ((p.M + 7) & ~7) - 8 - m0);
            else
                oa[h][u] = (uint32_t)min((rr >> 6) * 128 + (rr & 63) + 64 * h, p.M - 1 - m0) * (uint32_t)p.lda + ch;
            if constexpr (KB)
                ob[h][u] = (uint32_t)k * (uint32_t)p.ldb +
                           2 * (uint32_t)min((gc >> 2) * 64 + 32 * h + (gc & 3) * 8, ((p.N + 7) & ~7) - 8 - n0);
            else
                ob[h][u] = (uint32_t)min((rr >> 5) * 64 + (rr & 31) + 32 * h, p.N - 1 - n0) * (uint32_t)p.ldb + ch;
        }
    }
    // region 0, 1: A-lo, A-hi; 2, 3: B-lo, B-hi
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
    auto copy = [&](int region, int t) {
        const uint8_t *g = region < 2 ? ba + t * step_a : bb + t * step_b;
        const uint32_t d = lds0 + (t & 1) * kBuffer + region * kRegion;
#pragma unroll
        for (int u = 0; u < 2; ++u) copy_to_lds(g, region < 2 ? oa[region & 1][u] : ob[region & 1][u], d + u * 8192);
    };

    f32x4 acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int fr = lane & 15, g = lane >> 4;
    const int o0 = (g ^ (fr & 7)) * 16, o1 = ((g + 4) ^ (fr & 7)) * 16;
    const char *const la = lds + (wm * 64 + fr) * kPiece, *const lb = lds + 2 * kRegion + (wn * 32 + fr) * kPiece;
    const char *const ka[2] = {lds + km_place(lane, wm * 8), lds + km_place(lane, wm * 8 + 4)};
    const char *const kb = lds + 2 * kRegion + km_place(lane, wn * 4);
    auto read_a = [&](Frag (&f)[4], int t, int h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (KA) {
                f[i] = km_frag(ka[i >> 1] + (t & 1) * kBuffer + h * kRegion + (i & 1) * 32);
                continue;
            }
            const char *q = la + (t & 1) * kBuffer + h * kRegion + i * 16 * kPiece;
            f[i] = Frag{*(const uint4 *)(q + o0), *(const uint4 *)(q + o1)};
        }
    };
    auto read_b = [&](Frag (&f)[2], int t, int h) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (KB) {
                f[j] = km_frag(kb + (t & 1) * kBuffer + h * kRegion + j * 32);
                continue;
            }
            const char *q = lb + (t & 1) * kBuffer + h * kRegion + j * 16 * kPiece;
            f[j] = Frag{*(const uint4 *)(q + o0), *(const uint4 *)(q + o1)};
        }
    };
    // Scales: for a piece, 16 lanes' words of four row blocks' bytes (the
    // instruction picks one): [piece][wm][lo, hi][lane % 16]; B's by 128 columns.
    const uint32_t *const wsa = (const uint32_t *)(lds + 2 * kBuffer) + wm * 32 + fr;
    const uint8_t *const wsb = (const uint8_t *)lds + 2 * kBuffer + kScaleA + (wn >> 1);
    int sa[2] = {0, 0}, sb = 0;

    Frag fa[4], bl[2], bh[2], bn[2];
    auto quarter = [&](int h, int k, const Frag (&b)[2]) {   // rows half h, columns half k
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            mma_big<TYPE, 0>(acc[4 * h + 0][2 * k + j], fa[0], b[j], sa[h], sb);
            mma_big<TYPE, 1>(acc[4 * h + 1][2 * k + j], fa[1], b[j], sa[h], sb);
            mma_big<TYPE, 2>(acc[4 * h + 2][2 * k + j], fa[2], b[j], sa[h], sb);
            mma_big<TYPE, 3>(acc[4 * h + 3][2 * k + j], fa[3], b[j], sa[h], sb);
        }
        // (the sums are pinned here, or the compiler moves the products past the barriers)
        asm volatile("" : "+v"(acc[4 * h][2 * k]), "+v"(acc[4 * h + 1][2 * k]), "+v"(acc[4 * h + 2][2 * k]),
                     "+v"(acc[4 * h + 3][2 * k]), "+v"(acc[4 * h][2 * k + 1]), "+v"(acc[4 * h + 1][2 * k + 1]),
                     "+v"(acc[4 * h + 2][2 * k + 1]), "+v"(acc[4 * h + 3][2 * k + 1]));
        __builtin_amdgcn_s_setprio(0);
    };
    // waits until at most N loads are outstanding, N by the pieces left behind
    // this one (two or more, one, none): the loads issued after the awaited ones
    auto wait_for = [&](int left, auto n2, auto n1, auto n0) {
        if (left >= 2) wait_copies<decltype(n2)::value>();
        else if (left == 1) wait_copies<decltype(n1)::value>();
        else wait_copies<decltype(n0)::value>();
    };
    using std::integral_constant;
    auto piece = [&](int t) {
        const int left = nt - 1 - t;
        // quarter 0
        read_a(fa, t, 0);
        if constexpr (TYPE == TILE_FP8) {
            sa[0] = (int)wsa[t * 64];
            sa[1] = (int)wsa[t * 64 + 16];
            sb = wsb[t * 2];
        }
        if (left >= 1) copy(1, t + 1);
        wait_for(left, integral_constant<int, 10>{}, integral_constant<int, 10>{}, integral_constant<int, 2>{});
        turn();
        quarter(0, 0, bl);
        turn();
        // quarter 1
        read_b(bh, t, 1);
        if (left >= 2) copy(2, t + 2);
        wait_for(left, integral_constant<int, 10>{}, integral_constant<int, 8>{}, integral_constant<int, 0>{});
        turn();
        quarter(0, 1, bh);
        turn();
        // quarter 2
        read_a(fa, t, 1);
        if (left >= 2) copy(0, t + 2);
        wait_for(left, integral_constant<int, 10>{}, integral_constant<int, 6>{}, integral_constant<int, 0>{});
        turn();
        quarter(1, 1, bh);
        turn();
        // quarter 3 (behind the last piece the read is of a stale one, unused)
        read_b(bn, t + 1, 0);
        if (left >= 2) copy(3, t + 2);
        wait_for(left, integral_constant<int, 10>{}, integral_constant<int, 4>{}, integral_constant<int, 0>{});
        turn();
        wait_reads();   // bn's: its region is refilled in quarter 1, before bn is used
        quarter(1, 0, bl);
        turn();
        bl[0] = bn[0];
        bl[1] = bn[1];
    };
    if (nt > 0) {
        if constexpr (TYPE == TILE_FP8) {
            // (before any copy is in flight: these loads are waited for)
            uint8_t *s8 = (uint8_t *)lds + 2 * kBuffer;
            for (int i = threadIdx.x; i < kBigT * nt; i += kBigThreads) {
                const int r = i / nt, t = i - r * nt;   // row of the tile: wm 128 + lo/hi 64 + block 16 + lane
                s8[(t * 64 + (r >> 7) * 32 + ((r >> 6) & 1) * 16 + (r & 15)) * 4 + ((r >> 4) & 3)] =
                    p.sa[(int64_t)min(m0 + r, p.M - 1) * p.ldsa + kt0 + t];
            }
            for (int i = threadIdx.x; i < 2 * nt; i += kBigThreads)
                s8[kScaleA + i] = p.sb[(int64_t)(min(n0 + (i & 1) * 128, p.N - 1) / kRows8Block) * p.sb_n +
                                       (int64_t)(kt0 + (i >> 1)) * p.sb_k];
            __syncthreads();
        }
        copy(2, 0);
        copy(0, 0);
        copy(3, 0);
        copy(1, 0);
        if (nt > 1) {
            copy(2, 1);
            copy(0, 1);
            copy(3, 1);
            wait_copies<10>();
        } else {
            wait_copies<4>();
        }
        turn();
        read_b(bl, 0, 0);
        wait_reads();
        if (wm) turn();
        for (int t = 0; t < nt; ++t) piece(t);
        if (!wm) turn();
    }
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
