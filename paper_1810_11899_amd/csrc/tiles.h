// The tile loops of the products (product.hip, muon.hip): sums of A B^T of bfloat16,
// float16, 8-bit, 4-bit or float32 rows on the matrix cores, left in registers for
// the epilogue of the kernel around them.
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
#pragma once

#include <type_traits>

#include "rows8.h"

namespace gcn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16v8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16v8 __attribute__((ext_vector_type(8)));

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

// byte of column c's high part in a row of pairs: 32 high parts, then their 32
// low ones, 64 bytes on
__host__ __device__ __forceinline__ int64_t pair_place(int64_t c) { return c / 32 * 128 + c % 32 * 2; }

constexpr bool is_fp8(int type) { return type == TILE_FP8 || type == TILE_FP8_EXACT; }
constexpr bool is_f32(int type) { return type == TILE_F32 || type == TILE_F32_TN || type == TILE_F32_NN; }
// which operands are stored along the other way
constexpr bool km_a(int type) { return type == TILE_BF16_TN || type == TILE_F32_TN; }
constexpr bool km_b(int type) {
    return km_a(type) || type == TILE_BF16_NN || type == TILE_F32_NN || type == TILE_F16_NN || type == TILE_PAIR_NN;
}
constexpr bool is_f16(int type) { return type == TILE_F16 || type == TILE_F16_NN; }
constexpr bool is_pair(int type) { return type == TILE_PAIR || type == TILE_PAIR_NN; }

template <int TYPE>
__device__ __forceinline__ void mma(f32x4 &acc, const Frag &a, const Frag &b, int sa, int sb) {
    if constexpr (is_f16(TYPE)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16v8, b.lo), __builtin_bit_cast(f16v8, a.lo),
                                                     acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16v8, b.hi), __builtin_bit_cast(f16v8, a.hi),
                                                     acc, 0, 0, 0);
    } else if constexpr (is_pair(TYPE)) {
        // 32 columns: their high parts in the first chunks, their low parts in the
        // others; the product of the low parts is below the sum's last bit
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16v8, b.lo), __builtin_bit_cast(f16v8, a.hi),
                                                     acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16v8, b.hi), __builtin_bit_cast(f16v8, a.lo),
                                                     acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16v8, b.lo), __builtin_bit_cast(f16v8, a.lo),
                                                     acc, 0, 0, 0);
    } else if constexpr (!is_fp8(TYPE)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16v8, b.lo),
                                                      __builtin_bit_cast(bf16v8, a.lo), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16v8, b.hi),
                                                      __builtin_bit_cast(bf16v8, a.hi), acc, 0, 0, 0);
    } else if constexpr (TYPE == TILE_FP8) {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, b),
                                                               __builtin_bit_cast(i32x8, a), acc, 0, 0, 0, sb, 0, sa);
    }
}

// 4-bit operands: a chunk is one block of 32 values, which one lane of the
// instruction holds, so that the chunks g and g + 4 are two instructions' shares.
// sa, sb: words of the scales of four 16-row blocks for the first and the second
// half of the piece; the instruction picks byte I of A's and J of B's.
__device__ __forceinline__ i32x8 four_words(uint4 v) {
    return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
}
template <int I, int J>
__device__ __forceinline__ void mma4(f32x4 &acc, const Frag &a, const Frag &b, const int (&sa)[2], const int (&sb)[2]) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(four_words(b.lo), four_words(a.lo), acc, 4, 4, J, sb[0], I, sa[0]);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(four_words(b.hi), four_words(a.hi), acc, 4, 4, J, sb[1], I, sa[1]);
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
// f(0), f(1) .. f(N - 1) of compile-time numbers
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, I + 1>(f);
    }
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
    return 2 * (BM + BN) * kPiece + (is_fp8(type) ? kScalePieces * (BM + 1) : type == TILE_FP4 ? 16 * (BM + BN) : 0);
}
// `lds`: small_lds bytes; behind the loop they are free again.  `tid`: the thread's
// number among the loop's 64 WM WN, where a workgroup runs several of them side by
// side, with LDS of their own; then `turns` is the largest nt among them (they share
// their barriers).
template <int TYPE, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void small_loop(const TileProduct &p, const Coord &c, int kt0, int nt, char *lds,
                                           f32x4 (&acc)[BM / WM / 16][BN / WN / 16], uint32_t tid, int turns) {
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16, T = 64 * WM * WN;
    constexpr int kStage = (BM + BN) * kPiece;
    constexpr int LA = BM * kPiece / 16 / T, LB = BN * kPiece / 16 / T;
    static_assert(LA * T * 16 == BM * kPiece && LB * T * 16 == BN * kPiece, "whole chunks per lane");
    constexpr bool SCALED = is_fp8(TYPE);
    static_assert(!SCALED || kRows8Block % BN == 0, "a tile's columns share a scale");
    static_assert(TYPE != TILE_FP4 || (BM % 64 == 0 && BN % 64 == 0 && FN == 4), "scales come in groups of 64 rows");
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int m0 = c.tm * BM, n0 = c.tn * BN;
    constexpr bool KA = km_a(TYPE), KB = km_b(TYPE);
    static_assert((!KA || BM == 128) && (!KB || BN == 128), "k-rows of 128 elements");
    constexpr int E = is_f32(TYPE) ? 4 : 2, V = 16 / E, CH = 128 / V;   // of k-major operands: bytes, elements a chunk, chunks a row
    // (pairs along the columns: a stage holds 32 rows' high parts, then their low ones)
    const int64_t step_a = KA ? kPiece / E * p.lda : kPiece, step_b = KB ? kPiece / (is_pair(TYPE) ? 4 : E) * p.ldb : kPiece;
    // Copy u of a thread: tile row (u T + thread) / 8, stored chunk thread % 8,
    // which holds the row's chunk (thread % 8) ^ (row % 8); rows past the extent
    // are clamped (their products are dropped).  k-major: k-row (u T + thread) /
    // CH, its chunks clamped to the last whole one.
    const int lr = tid >> 3, chunk = ((tid & 7) ^ (lr & 7)) * 16;
    auto km_at = [&](int64_t ld, int x0, int extent, int u) {
        const int k = (u * T + tid) / CH, ch = V * ((tid % CH) ^ (4 * ((is_f32(TYPE) ? k >> 2 : k) & 3)));
        if constexpr (is_pair(TYPE)) return (k & 31) * ld + pair_place(min(x0 + ch, ((extent + 31) & -32) - 8)) + (k >> 5) * 64;
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
    // 4-bit operands: the piece's scales, 32 lanes a group of 64 rows, A's groups first
    const uint8_t *g4 = nullptr;
    int64_t step4 = 0;
    if constexpr (TYPE == TILE_FP4) {
        const int r = tid >> 5, nb = BM / 64;
        const bool of_a = r < nb;
        step4 = (int64_t)(of_a ? p.groups_a : p.groups_b) * 512;
        g4 = (of_a ? p.sa + (int64_t)min(m0 / 64 + r, p.groups_a - 1) * 512
                   : p.sb + (int64_t)min(n0 / 64 + r - nb, p.groups_b - 1) * 512) +
             kt0 * step4 + (tid & 31) * 16;
    }
    auto copy = [&](int t, int stage) {
        const uint32_t d = lds0 + stage * kStage;
#pragma unroll
        for (int u = 0; u < LA; ++u) copy_to_lds(ga[u] + t * step_a, d + u * T * 16);
#pragma unroll
        for (int u = 0; u < LB; ++u) copy_to_lds(gb[u] + t * step_b, d + BM * kPiece + u * T * 16);
        if constexpr (TYPE == TILE_FP4) {
            if (tid < (BM + BN) / 2) copy_to_lds(g4 + t * step4, lds0 + 2 * kStage + stage * 8 * (BM + BN));
        }
    };
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
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
        for (int i = tid; i < BM * w; i += T) {
            const int r = i / w, k = i - r * w;
            s8[k * BM + r] = p.sa[(int64_t)min(m0 + r, p.M - 1) * p.ldsa + kt0 + t + k];
        }
        for (int k = tid; k < w; k += T)
            s8[kScalePieces * BM + k] = p.sb[(int64_t)(n0 / kRows8Block) * p.sb_n + (int64_t)(kt0 + t + k) * p.sb_k];
    };
    if constexpr (SCALED) {
        if (nt > 0) scales(0);
    }
    // both stages at once: the second piece's copy would wait for the first's otherwise
    // (8-bit scales pass through registers behind the first copy).  The many-class loss, us,
    // one stage first / so: 17 x 128, 1009 classes 28.9 / 28.4, 5003 x 600, 50,021 classes
    // without gradient 369 / 365, 16,384 x 1024, 131,072 classes 15,750 / 15,620
    constexpr bool kBoth = !SCALED;
    if (nt > 0) copy(0, 0);
    if (kBoth && nt > 1) copy(1, 1);
    for (int t = 0; t < nt; ++t) {
        if constexpr (SCALED) {
            if (t % kScalePieces == 0 && t) {
                turn();   // every wavefront has read the old ones
                scales(t);
            }
            wait_reads();   // the scales' LDS writes, ahead of the barrier
        }
        // piece t has landed
        if (kBoth && t == 0 && nt > 1) {
            if (TYPE == TILE_FP4 && wave * 64 < (BM + BN) / 2) wait_copies<LA + LB + 1>();
            else wait_copies<LA + LB>();
        } else {
            wait_copies<0>();
        }
        turn();
        // (every wavefront has used what it read of piece t - 1: its stage is free)
        if ((t || !kBoth) && t + 1 < nt) copy(t + 1, (t + 1) & 1);
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
        if constexpr (TYPE == TILE_FP4) {
            const char *s4 = lds + 2 * kStage + (t & 1) * 8 * (BM + BN) + lane * 4;
            const char *qb = s4 + (BM / 64 + wn) * 512, *qa = s4 + wm * (BM / WM) / 64 * 512;
            const int b4[2] = {*(const int *)qb, *(const int *)(qb + 256)};
            const int by = wm * (BM / WM) % 64 / 16 * 8;   // (a wavefront with fewer rows than 64: its first block to byte 0)
            const int a4[2] = {*(const int *)qa >> by, *(const int *)(qa + 256) >> by};
            static_for<FM>([&](auto i) {
                const Frag fa = frag(ta, wm * (BM / WM) + 16 * i.value, false);
                static_for<FN>([&](auto j) { mma4<i.value, j.value>(acc[i.value][j.value], fa, fb[j.value], a4, b4); });
            });
        } else if constexpr (TYPE == TILE_FP8_EXACT) {
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
                // (where the products leave them: pinned elsewhere they are moved there and back)
                else asm volatile("" : "+a"(acc[i][j]));
            }
    }
    for (int t = nt; t < turns; ++t) turn();
    __syncthreads();
}
template <int TYPE, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void small_loop(const TileProduct &p, const Coord &c, int kt0, int nt, char *lds,
                                           f32x4 (&acc)[BM / WM / 16][BN / WN / 16]) {
    // (sums of its own: formed in the caller's array, they are cleared on a path of
    // their own where there is no piece; 6205 x 512 x 602 of 8-bit rows 12.5 / 12.2 us)
    f32x4 sum[BM / WM / 16][BN / WN / 16];
    small_loop<TYPE, BM, BN, WM, WN>(p, c, kt0, nt, lds, sum, threadIdx.x, nt);
#pragma unroll
    for (int i = 0; i < BM / WM / 16; ++i)
#pragma unroll
        for (int j = 0; j < BN / WN / 16; ++j) acc[i][j] = sum[i][j];
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
// 16,384 of bfloat16 ones: 410-425 us, 1300 TFLOP/s.  The chip's power is part of both
// (zeros instead of random operands, on two cards: 505 -> 385 us, 458 -> 408; of 4-bit
// operands 287 -> 254).
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

constexpr int kScales4 = 16 * 2 * kBigT / 2;   // of the 512 rows of a 4-bit piece, 8 a row
constexpr int big_lds(int type) {
    return 2 * kBuffer + (type == TILE_FP8 ? kScaleA + kScaleB : type == TILE_FP4 ? 2 * kScales4 : 0);
}
// `lds`: big_lds bytes.
template <int TYPE>
__device__ __forceinline__ void big_loop(const TileProduct &p, const Coord &c, int kt0, int nt, char *lds,
                                         f32x4 (&acc)[8][4]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const int m0 = c.tm * kBigT, n0 = c.tn * kBigT;

    // Copies: region row (8 u + wave) 8 + lane / 8, stored chunk lane % 8 with
    // the row's chunk (lane % 8) ^ (row % 8); rows past the extent are clamped.
    // k-major: k-row (8 u + wave) 4 + lane / 16, stored chunk lane % 16, which is one
    // of the 8 of A's first or second half's columns in the region, or of the 4
    // of B's four quarters'; chunks past the extent are clamped to the last.
    constexpr bool KA = km_a(TYPE), KB = km_b(TYPE);
    constexpr bool PB = TYPE == TILE_PAIR_NN;   // (a stage: 32 rows' high parts, then their low ones)
    const int64_t step_a = KA ? 64 * p.lda : kPiece, step_b = KB ? (PB ? 32 : 64) * p.ldb : kPiece;
    const uint8_t *const ba = p.A + (KA ? (int64_t)m0 * 2 : (int64_t)m0 * p.lda) + kt0 * step_a;
    const uint8_t *const bb = p.B + (KB ? (int64_t)n0 * (PB ? 4 : 2) : (int64_t)n0 * p.ldb) + kt0 * step_b;
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
            if constexpr (PB)
                ob[h][u] = (uint32_t)(k & 31) * (uint32_t)p.ldb + 64 * (uint32_t)(k >> 5) +
                           (uint32_t)pair_place(min((gc >> 2) * 64 + 32 * h + (gc & 3) * 8, ((p.N + 31) & ~31) - 8 - n0));
            else if constexpr (KB)
                ob[h][u] = (uint32_t)k * (uint32_t)p.ldb +
                           2 * (uint32_t)min((gc >> 2) * 64 + 32 * h + (gc & 3) * 8, ((p.N + 7) & ~7) - 8 - n0);
            else
                ob[h][u] = (uint32_t)min((rr >> 5) * 64 + (rr & 31) + 32 * h, p.N - 1 - n0) * (uint32_t)p.ldb + ch;
        }
    }
    const uint8_t *g4 = nullptr;
    int64_t step4 = 0;
    if constexpr (TYPE == TILE_FP4) {
        step4 = (int64_t)(wave < 4 ? p.groups_a : p.groups_b) * 512;
        g4 = (wave < 4 ? p.sa + (int64_t)min(m0 / 64 + wave, p.groups_a - 1) * 512
                       : p.sb + (int64_t)min(n0 / 64 + wave - 4, p.groups_b - 1) * 512) +
             kt0 * step4 + lane * 16;
    }
    // region 0, 1: A-lo, A-hi; 2, 3: B-lo, B-hi
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
    auto copy = [&](int region, int t) {
        const uint8_t *g = region < 2 ? ba + t * step_a : bb + t * step_b;
        const uint32_t d = lds0 + (t & 1) * kBuffer + region * kRegion;
#pragma unroll
        for (int u = 0; u < 2; ++u) copy_to_lds(g, region < 2 ? oa[region & 1][u] : ob[region & 1][u], d + u * 8192);
        if constexpr (TYPE == TILE_FP4) {
            // the piece's scales go with its first region, a group of 64 rows to half a wavefront
            if (region == 0 && lane < 32) copy_to_lds(g4 + t * step4, lds0 + 2 * kBuffer - wave * 512 + (t & 1) * kScales4);
        }
    };

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
    int a4[2][2] = {}, b4[2] = {};   // 4-bit operands: the scales of A's two halves and of B, by halves of the piece
    auto quarter = [&](auto hh, auto kk, const Frag (&b)[2]) {   // rows half h, columns half k
        constexpr int h = decltype(hh)::value, k = decltype(kk)::value;
        __builtin_amdgcn_s_setprio(1);
        if constexpr (TYPE == TILE_FP4) {
            static_for<2>([&](auto j) {
                static_for<4>([&](auto i) {
                    mma4<i.value, 2 * k + j.value>(acc[4 * h + i.value][2 * k + j.value], fa[i.value], b[j.value], a4[h], b4);
                });
            });
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                mma_big<TYPE, 0>(acc[4 * h + 0][2 * k + j], fa[0], b[j], sa[h], sb);
                mma_big<TYPE, 1>(acc[4 * h + 1][2 * k + j], fa[1], b[j], sa[h], sb);
                mma_big<TYPE, 2>(acc[4 * h + 2][2 * k + j], fa[2], b[j], sa[h], sb);
                mma_big<TYPE, 3>(acc[4 * h + 3][2 * k + j], fa[3], b[j], sa[h], sb);
            }
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
    constexpr int X = TYPE == TILE_FP4;   // (region 0 takes one copy more)
    auto piece = [&](int t) {
        const int left = nt - 1 - t;
        // quarter 0
        read_a(fa, t, 0);
        if constexpr (TYPE == TILE_FP8) {
            sa[0] = (int)wsa[t * 64];
            sa[1] = (int)wsa[t * 64 + 16];
            sb = wsb[t * 2];
        }
        if constexpr (TYPE == TILE_FP4) {
            const char *s4 = lds + 2 * kBuffer + (t & 1) * kScales4 + lane * 4;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                a4[0][q] = *(const int *)(s4 + (2 * wm) * 512 + q * 256);
                a4[1][q] = *(const int *)(s4 + (2 * wm + 1) * 512 + q * 256);
                b4[q] = *(const int *)(s4 + (4 + wn) * 512 + q * 256);
            }
        }
        if (left >= 1) copy(1, t + 1);
        wait_for(left, integral_constant<int, 10 + X>{}, integral_constant<int, 10 + X>{}, integral_constant<int, 2>{});
        turn();
        quarter(integral_constant<int, 0>{}, integral_constant<int, 0>{}, bl);
        turn();
        // quarter 1
        read_b(bh, t, 1);
        if (left >= 2) copy(2, t + 2);
        wait_for(left, integral_constant<int, 10 + X>{}, integral_constant<int, 8 + X>{}, integral_constant<int, 0>{});
        turn();
        quarter(integral_constant<int, 0>{}, integral_constant<int, 1>{}, bh);
        turn();
        // quarter 2
        read_a(fa, t, 1);
        if (left >= 2) copy(0, t + 2);
        wait_for(left, integral_constant<int, 10 + 2 * X>{}, integral_constant<int, 6 + X>{}, integral_constant<int, 0>{});
        turn();
        quarter(integral_constant<int, 1>{}, integral_constant<int, 1>{}, bh);
        turn();
        // quarter 3 (behind the last piece the read is of a stale one, unused)
        read_b(bn, t + 1, 0);
        if (left >= 2) copy(3, t + 2);
        wait_for(left, integral_constant<int, 10 + X>{}, integral_constant<int, 4>{}, integral_constant<int, 0>{});
        turn();
        wait_reads();   // bn's: its region is refilled in quarter 1, before bn is used
        quarter(integral_constant<int, 1>{}, integral_constant<int, 0>{}, bl);
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
            wait_copies<10 + X>();
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
}

}  // namespace
}  // namespace gcn
