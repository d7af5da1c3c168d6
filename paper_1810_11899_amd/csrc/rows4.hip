// Microscaled 4-bit rows: e2m1 values with one power-of-two scale for each block
// of 32 columns.
#include <algorithm>

#include "gcn_rows4.h"
#include "rows8.h"

namespace gcn {
namespace {

constexpr int kTB = 256;
constexpr int kTile = 128;      // rows and columns of a packing tile
constexpr int kNaNScale = 255;

int64_t pieces4(int64_t f) { return (f + 255) / 256; }
int64_t groups4(int64_t n) { return (n + 63) / 64; }

// The scale byte of a block from the bits of its largest magnitude a = m 2^k:
// exponent k - 2 where m <= 1.5 (6 = 1.5 * 2^2 is the largest e2m1 value), k - 1
// above, at least -126; 0 for a block of zeros; kNaNScale where a is not finite.
__device__ __forceinline__ int scale_byte(uint32_t a) {
    const int e = max((int)(a >> 23) - 129 + ((a & 0x7FFFFFu) > 0x400000u ? 1 : 0), -126);
    return a >= 0x7F800000u ? kNaNScale : a == 0u ? 127 : e + 127;
}
// where the scale byte of row i and block b lies
__device__ __forceinline__ int64_t scale_place(int64_t i, int64_t b, int64_t groups) {
    return ((b >> 3) * groups + (i >> 6)) * 512 + ((b >> 2) & 1) * 256 + (b & 3) * 64 + (i & 15) * 4 + ((i >> 4) & 3);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// eight values under the scale with byte s (1 .. 254), the first in the low bits:
// the hardware's rounding (nearest, ties to even); zeros under kNaNScale
__device__ __forceinline__ uint32_t held8(const float *x, int s) {
    const float scale = __uint_as_float((uint32_t)s << 23);
    uint32_t r = 0u;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
    return s == kNaNScale ? 0u : r;
}

// Eight consecutive elements from column c of a row as they lie in memory (zeros past
// f); their values.  Apart, so that all of a thread's loads are in flight before
// the first is used.
template <bool BF>
struct Raw {
    uint4 v[BF ? 1 : 2];
};
template <bool BF>
__device__ __forceinline__ Raw<BF> load_raw(const void *row, int64_t c, int32_t f) {
    Raw<BF> x;
    const int64_t left = f - c;
    if (left >= 8) {
        if constexpr (BF) {
            x.v[0] = load16((const uint16_t *)row + c);
        } else {
            x.v[0] = load16((const float *)row + c);
            x.v[1] = load16((const float *)row + c + 4);
        }
    } else {
        uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) w[i] = BF ? (uint32_t)((const uint16_t *)row)[c + i] : ((const uint32_t *)row)[c + i];
        if constexpr (BF) {
            x.v[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        } else {
            x.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
            x.v[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
    return x;
}
template <bool BF>
__device__ __forceinline__ void values_of(const Raw<BF> &r, float (&x)[8]) {
    if constexpr (BF) {
        const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
        const uint32_t w[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    }
}

struct PackArgs {
    int32_t n, f;
    const void *X, *mask;
    int64_t ldx, ldm;
    uint8_t *q, *scale;      // of the rows, or null
    int64_t ldq;
    uint8_t *qt, *scale_t;   // of the columns, or null
    int64_t ldqt;
    float *part;             // [row tiles x f] column sums, or null
    int32_t tiles_r, tiles_c;
};
// 128 x 128 of X to a workgroup, the tiles past X's last row and column up to whole
// pieces of 256 included (they hold zeros).  A thread's 8 values of 8 rows
// come from memory; 4 lanes hold a block of a row, which they pack at once.  The
// columns are packed from LDS, one thread a block of 32 rows, and written
// through LDS again, 64 bytes a row.
// Bound by memory: 65,536 x 1024 bfloat16 with a mask, both orientations, 91 us,
// 3.7 TB/s (loads waited for one row after another: 113).
constexpr int kPackT = 512;
template <bool BF, bool COLS>
__global__ __launch_bounds__(kPackT) void pack4_kernel(PackArgs a) {
    typedef typename std::conditional<BF, uint16_t, float>::type T;
    constexpr int kLd = kTile + (BF ? 8 : 4), kRows = kTile * 16 / kPackT;
    __shared__ __attribute__((aligned(16))) T tile[COLS ? kTile : 1][kLd];
    __shared__ uint4 turned[COLS ? kTile * 4 : 1];
    __shared__ float sums[COLS ? 4 : 1][kTile];
    const int64_t tiles = (int64_t)a.tiles_r * a.tiles_c, groups = (a.n + 63ll) / 64, groups_t = (a.f + 63ll) / 64;
    for (int64_t b = blockIdx.x; b < tiles; b += gridDim.x) {
        const int64_t tr = b / a.tiles_c, tc = b - tr * a.tiles_c;
        const int64_t r0 = tr * kTile, c0 = tc * kTile;
        const int cl = 8 * (int)(threadIdx.x & 15), rl0 = (int)(threadIdx.x >> 4);
        const int64_t c = c0 + cl;
        Raw<BF> raw[kRows], mask[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int64_t row = r0 + (kTile / kRows) * u + rl0;
            const int32_t f = row < a.n ? a.f : 0;
            raw[u] = load_raw<BF>((const T *)a.X + row * a.ldx, c, f);
            if (a.mask) mask[u] = load_raw<BF>((const T *)a.mask + row * a.ldm, c, f);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int rl = (kTile / kRows) * u + rl0;
            const int64_t row = r0 + rl;
            float x[8];
            values_of<BF>(raw[u], x);
            if (a.mask) {
                float m[8];
                values_of<BF>(mask[u], m);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = m[i] > 0.0f ? x[i] : 0.0f;
            }
            if (a.q) {
                uint32_t top = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, magnitude(x[i]));
                top = max(top, (uint32_t)__shfl_xor((int)top, 1));
                top = max(top, (uint32_t)__shfl_xor((int)top, 2));
                const int s = scale_byte(top);
                if (row < a.n && c < (((int64_t)a.f + 255) & ~255ll)) {
                    *(uint32_t *)(a.q + row * a.ldq + c / 2) = held8(x, s);
                    if ((threadIdx.x & 3) == 0) a.scale[scale_place(row, c >> 5, groups)] = (uint8_t)s;
                }
            }
            if constexpr (COLS) {
                if constexpr (BF) {   // (bfloat16 values, or zeros: nothing is rounded)
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xFFFF0000u);
                    *(uint4 *)&tile[rl][cl] = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
                    *(float4 *)&tile[rl][cl] = make_float4(x[0], x[1], x[2], x[3]);
                    *(float4 *)&tile[rl][cl + 4] = make_float4(x[4], x[5], x[6], x[7]);
                }
            }
        }
        if constexpr (COLS) {
            __syncthreads();
            const int col = threadIdx.x & (kTile - 1), blk = (int)threadIdx.x / kTile;   // of 32 rows
            const bool to_t = a.qt && r0 < (((int64_t)a.n + 255) & ~255ll);
            {
                float x[32];
                uint32_t top = 0u;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const T v = tile[32 * blk + i][col];
                    if constexpr (BF) x[i] = __uint_as_float((uint32_t)v << 16);
                    else x[i] = v;
                    top = max(top, magnitude(x[i]));
                    sum += x[i];
                }
                sums[blk][col] = sum;
                if (to_t) {
                    const int s = scale_byte(top);
                    turned[col * 4 + blk] = make_uint4(held8(x, s), held8(x + 8, s), held8(x + 16, s), held8(x + 24, s));
                    if (c0 + col < a.f) a.scale_t[scale_place(c0 + col, (r0 >> 5) + blk, groups_t)] = (uint8_t)s;
                }
            }
            __syncthreads();
            if (to_t) {
                const int64_t row = c0 + (threadIdx.x >> 2);
                if (row < a.f) *(uint4 *)(a.qt + row * a.ldqt + r0 / 2 + (threadIdx.x & 3) * 16) = turned[threadIdx.x];
            }
            if (a.part && threadIdx.x < kTile && c0 + threadIdx.x < a.f && r0 < a.n)
                a.part[tr * a.f + c0 + threadIdx.x] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) +
                                                      (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
            // (the next tile's rows are written behind a barrier that the last reads of this one's are ahead of)
        }
    }
}

// colsum = the column sums of part [rows x f], one wavefront a column
__global__ __launch_bounds__(kTB) void colsum4_kernel(int32_t rows, int32_t f, const float *part, float *out) {
    for (int64_t k = (int64_t)blockIdx.x * (kTB / 64) + (threadIdx.x >> 6); k < f; k += (int64_t)gridDim.x * (kTB / 64)) {
        float v = 0.0f;
        for (int32_t r = (int32_t)(threadIdx.x & 63); r < rows; r += 64) v += part[(int64_t)r * f + k];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
        if ((threadIdx.x & 63) == 0) out[k] = v;
    }
}

// eight columns to a thread
template <bool BF>
__global__ __launch_bounds__(kTB) void unpack4_kernel(int32_t n, int32_t f, const uint8_t *q, int64_t ldq,
                                                      const uint8_t *scale, void *X, int64_t ldx) {
    const uint32_t per_row = ((uint32_t)f + 7) / 8;
    const int64_t total = (int64_t)n * per_row, groups = (n + 63ll) / 64;
    for (int64_t i = (int64_t)blockIdx.x * kTB + threadIdx.x; i < total; i += (int64_t)gridDim.x * kTB) {
        const int64_t row = i / per_row, c = (i - row * per_row) * 8;
        const uint32_t v = *(const uint32_t *)(q + row * ldq + c / 2);   // (zeros past f)
        const uint32_t s = scale[scale_place(row, c >> 5, groups)];
        // 2^(s - 127): 2^-127 is a subnormal number, 255 a NaN
        const float m = __uint_as_float(s == kNaNScale ? 0x7FC00000u : s == 0u ? 0x400000u : s << 23);
        float x[8];
#define GCN_TWO(I)                                                                            \
    {                                                                                         \
        const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, I);                  \
        x[2 * I] = p[0] * m;                                                                  \
        x[2 * I + 1] = p[1] * m;                                                              \
    }
        GCN_TWO(0) GCN_TWO(1) GCN_TWO(2) GCN_TWO(3)
#undef GCN_TWO
        if (BF) {
            uint16_t *d = (uint16_t *)X + row * ldx + c;
            if (c + 8 <= f) {
                store16(d, make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                      pack_bf16x2(x[6], x[7])));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < f) d[e] = to_bf16(x[e]);
            }
        } else {
            float *d = (float *)X + row * ldx + c;
            if (c + 8 <= f) {
#pragma unroll
                for (int h = 0; h < 8; h += 4)
                    store16(d + h, make_uint4(__float_as_uint(x[h]), __float_as_uint(x[h + 1]), __float_as_uint(x[h + 2]),
                                              __float_as_uint(x[h + 3])));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < f) d[e] = x[e];
            }
        }
    }
}

bool aligned(const void *p, uintptr_t b) { return (uintptr_t)p % b == 0; }
uintptr_t el(gcn_rows_type t) { return t == GCN_ROWS_BF16 ? 2 : 4; }

int check_type(gcn_rows_type t, const char *who) {
    GCN_REQUIRE(t == GCN_ROWS_F32 || t == GCN_ROWS_BF16, GCN_EINVAL, "%s: bad element type %d", who, (int)t);
    return GCN_OK;
}

int check_rows4(const gcn_rows4 *r, const char *who) {
    GCN_REQUIRE(r, GCN_EINVAL, "%s: null 4-bit rows", who);
    GCN_REQUIRE(r->n >= 0 && r->f >= 0, GCN_ESHAPE, "%s: 4-bit rows of %d x %d", who, r->n, r->f);
    GCN_REQUIRE(r->n <= kMostRows && r->f <= kMostRows, GCN_EUNSUPPORTED, "%s: 4-bit rows of %d x %d", who, r->n, r->f);
    GCN_REQUIRE(r->ldq % 16 == 0 && r->ldq >= 128 * pieces4(r->f), GCN_ESHAPE,
                "%s: ldq=%d is not a multiple of 16 of at least %lld", who, r->ldq, (long long)(128 * pieces4(r->f)));
    GCN_REQUIRE(r->n == 0 || r->f == 0 || (r->q && r->scale), GCN_EINVAL, "%s: null 4-bit rows", who);
    GCN_REQUIRE(aligned(r->q, 16) && aligned(r->scale, 16), GCN_EINVAL, "%s: 4-bit rows must be 16-byte aligned", who);
    return GCN_OK;
}

// Parts of a product's sum, for products with few tiles and long sums (weight
// gradients): 128 x 128 tiles, two a CU and 16 pieces a part or more, where they fill the
// CUs, else 64 x 64 ones of 8 pieces.  Parts are written and read again, which
// costs about 3 us and 0.4 us a megabyte (us, in 1 / 2 / 4 / 8 / 16 parts, float32 results, the
// operands in the caches; 1024 x 512 x 65,536 is 36 where they are others every call;
// 64 x 64: 1024 x 512 x 8000 12.6 / 12.0 / 13.3, 512 x 256 x 8000 12.2 / 9.9 / 9.5 / 9.7,
// 256 x 256 x 32,000 38 / 22 / 14.5 / 11.7 / 11.5, 1024 x 1024 x 8192 13.3 / 16.4; 128 x 128:
// 1024 x 512 x 65,536 151 / 84 / 48 / 32 / 33, 1024 x 1024 x 65,536 156 / 85 / 52 / 45 / 61, 64 x 64
// 116 / 67 / 61 / 65; 256 x 256 tiles 363 / 192 / 105 / 63 / 44 and 364 / 193 / 107 / 66 / 54).
// Few rows take thin4_kernel unless it has few workgroups and a long sum.
int32_t split4(int32_t M, int32_t N, int32_t kt) {
    if (M <= 0 || N <= 0 || kt < 24 || (M <= 64 && N > 2048)) return 1;
    const int64_t t64 = ((M + 63ll) / 64) * ((N + 63ll) / 64), t128 = ((M + 127ll) / 128) * ((N + 127ll) / 128);
    int64_t sp = std::min<int64_t>(512 / t128, kt / 16);
    if (t128 * sp < 192) sp = std::min<int64_t>({(kt < 64 ? 256 : 512) / t64, kt / 8, 32});
    if (sp <= 1) return 1;
    const int32_t per = (int32_t)((kt + sp - 1) / sp);
    return (kt + per - 1) / per;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" {

size_t gcn_rows4_pack_workspace_bytes(int32_t n, int32_t f) {
    if (n < 0 || f < 0 || std::max(n, f) > kMostRows) return 0;
    return 256 + sizeof(float) * (size_t)((n + (int64_t)kTile - 1) / kTile) * (size_t)f;
}

int gcn_rows4_pack(const void *X, gcn_rows_type type, int32_t n, int32_t f, int32_t ldx, const void *mask,
                   int32_t ldmask, const gcn_rows4 *out, const gcn_rows4 *outT, float *colsum, void *ws,
                   size_t ws_bytes, void *stream) {
    const char *const who = "gcn_rows4_pack";
    int rc = check_type(type, who);
    if (rc) return rc;
    GCN_REQUIRE(n >= 0 && f >= 0, GCN_ESHAPE, "%s: n=%d f=%d", who, n, f);
    GCN_REQUIRE(n <= kMostRows && f <= kMostRows, GCN_EUNSUPPORTED, "%s: n=%d f=%d", who, n, f);
    GCN_REQUIRE(out || outT || colsum, GCN_EINVAL, "%s: no output", who);
    if (out) {
        if ((rc = check_rows4(out, who))) return rc;
        GCN_REQUIRE(out->n == n && out->f == f, GCN_ESHAPE, "%s: out is %d x %d, not %d x %d", who, out->n, out->f, n, f);
    }
    if (outT) {
        if ((rc = check_rows4(outT, who))) return rc;
        GCN_REQUIRE(outT->n == f && outT->f == n, GCN_ESHAPE, "%s: outT is %d x %d, not %d x %d", who, outT->n, outT->f, f, n);
    }
    GCN_REQUIRE(ldx >= f && (!mask || ldmask >= f), GCN_ESHAPE, "%s: ldx=%d ldmask=%d < f=%d", who, ldx, ldmask, f);
    GCN_REQUIRE(n == 0 || f == 0 || X, GCN_EINVAL, "%s: null X", who);
    GCN_REQUIRE(aligned(X, el(type)) && aligned(mask, el(type)) && aligned(colsum, 4), GCN_EINVAL,
                "%s: misaligned pointer", who);
    const size_t need = gcn_rows4_pack_workspace_bytes(n, f);
    GCN_REQUIRE(!colsum || (ws && aligned(ws, 256) && ws_bytes >= need), GCN_EWORKSPACE,
                "%s: workspace %zu < %zu bytes, or not 256-byte aligned", who, ws_bytes, need);
    hipStream_t s = (hipStream_t)stream;
    if (f == 0) return GCN_OK;
    if (n == 0) return colsum ? fill_zero(colsum, f, s) : GCN_OK;   // (rows of no columns hold nothing)
    const bool bf = type == GCN_ROWS_BF16, cols = outT || colsum;
    PackArgs a{};
    a.n = n;
    a.f = f;
    a.X = X;
    a.mask = mask;
    a.ldx = ldx;
    a.ldm = ldmask;
    if (out) {
        a.q = out->q;
        a.scale = out->scale;
        a.ldq = out->ldq;
    }
    if (outT) {
        a.qt = outT->q;
        a.scale_t = outT->scale;
        a.ldqt = outT->ldq;
    }
    a.part = colsum ? (float *)ws : nullptr;
    a.tiles_r = (int32_t)(outT ? 2 * pieces4(n) : (n + (int64_t)kTile - 1) / kTile);
    a.tiles_c = (int32_t)(out ? 2 * pieces4(f) : (f + (int64_t)kTile - 1) / kTile);
    {
        ProfScope prof(K_ROWS4_PACK, s, 0.0,
                       (double)n * f * ((bf ? 2.0 : 4.0) * (mask ? 2 : 1) + 0.53125 * ((out ? 1 : 0) + (outT ? 1 : 0))));
        const unsigned g = (unsigned)std::min<int64_t>((int64_t)a.tiles_r * a.tiles_c, 1 << 16);
#define GCN_PACK4(BF, COLS) hipLaunchKernelGGL((pack4_kernel<BF, COLS>), dim3(g), dim3(kPackT), 0, s, a)
        if (bf && cols) GCN_PACK4(true, true);
        else if (bf) GCN_PACK4(true, false);
        else if (cols) GCN_PACK4(false, true);
        else GCN_PACK4(false, false);
#undef GCN_PACK4
        GCN_LAUNCH_CHECK("pack4_kernel");
    }
    if (colsum) {
        const int32_t rows = (int32_t)((n + (int64_t)kTile - 1) / kTile);
        ProfScope prof(K_ROWS4_PACK, s, 0.0, 4.0 * rows * f);
        const dim3 b((unsigned)std::min<int64_t>((f + 3ll) / 4, 1 << 16));
        hipLaunchKernelGGL(colsum4_kernel, b, dim3(kTB), 0, s, rows, f, a.part, colsum);
        GCN_LAUNCH_CHECK("colsum4_kernel");
    }
    return GCN_OK;
}

int gcn_rows4_unpack(const gcn_rows4 *r, void *X, gcn_rows_type type, int32_t ldx, void *stream) {
    const char *const who = "gcn_rows4_unpack";
    int rc = check_rows4(r, who);
    if (rc) return rc;
    if ((rc = check_type(type, who))) return rc;
    GCN_REQUIRE(ldx >= r->f, GCN_ESHAPE, "%s: ldx=%d < f=%d", who, ldx, r->f);
    if (r->n == 0 || r->f == 0) return GCN_OK;
    GCN_REQUIRE(X && aligned(X, el(type)), GCN_EINVAL, "%s: null or misaligned pointer", who);
    hipStream_t s = (hipStream_t)stream;
    const bool bf = type == GCN_ROWS_BF16;
    ProfScope prof(K_ROWS4_PACK, s, 0.0, (double)r->n * r->f * (bf ? 2.53125 : 4.53125));
    const unsigned g = (unsigned)std::min<int64_t>(((int64_t)r->n * ((r->f + 7ll) / 8) + kTB - 1) / kTB, 16384);
    if (bf)
        hipLaunchKernelGGL(unpack4_kernel<true>, dim3(g), dim3(kTB), 0, s, r->n, r->f, r->q, (int64_t)r->ldq, r->scale, X,
                           (int64_t)ldx);
    else
        hipLaunchKernelGGL(unpack4_kernel<false>, dim3(g), dim3(kTB), 0, s, r->n, r->f, r->q, (int64_t)r->ldq, r->scale, X,
                           (int64_t)ldx);
    GCN_LAUNCH_CHECK("unpack4_kernel");
    return GCN_OK;
}

size_t gcn_rows4_product_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M < 0 || N < 0 || K < 0 || std::max({M, N, K}) > kMostRows) return 0;
    const int32_t sp = split4(M, N, (int32_t)pieces4(K));
    return 256 + (sp > 1 ? sizeof(float) * sp * (size_t)M * (size_t)N : 0);
}

int gcn_rows4_product(const gcn_rows4 *A, const gcn_rows4 *B, const float *bias, int relu, void *Y,
                      gcn_rows_type type, int32_t ldy, void *ws, size_t ws_bytes, void *stream) {
    const char *const who = "gcn_rows4_product";
    int rc;
    if ((rc = check_rows4(A, who)) || (rc = check_rows4(B, who)) || (rc = check_type(type, who))) return rc;
    GCN_REQUIRE(A->f == B->f, GCN_ESHAPE, "%s: rows of %d columns against %d", who, A->f, B->f);
    GCN_REQUIRE(ldy >= B->n, GCN_ESHAPE, "%s: ldy=%d < %d", who, ldy, B->n);
    const size_t need = gcn_rows4_product_workspace_bytes(A->n, B->n, A->f);
    GCN_REQUIRE(ws && aligned(ws, 256) && ws_bytes >= need, GCN_EWORKSPACE,
                "%s: workspace %zu < %zu bytes, or not 256-byte aligned", who, ws_bytes, need);
    if (A->n == 0 || B->n == 0) return GCN_OK;
    GCN_REQUIRE(Y && aligned(Y, el(type)) && aligned(bias, 4), GCN_EINVAL, "%s: null or misaligned pointer", who);
    TileProduct p{};
    p.A = A->q;
    p.lda = A->ldq;
    p.B = B->q;
    p.ldb = B->ldq;
    p.M = A->n;
    p.N = B->n;
    p.kt = (int32_t)pieces4(A->f);
    p.sa = A->scale;
    p.sb = B->scale;
    p.groups_a = (int32_t)groups4(A->n);
    p.groups_b = (int32_t)groups4(B->n);
    p.C = Y;
    p.ldc = ldy;
    p.bias = bias;
    p.relu = relu;
    const bool bf = type == GCN_ROWS_BF16;
    hipStream_t s = (hipStream_t)stream;
    ProfScope prof(K_ROWS4_PRODUCT, s, 2.0 * p.M * p.N * A->f,
                   ((double)p.M + p.N) * A->f * 0.53125 + (double)p.M * p.N * (bf ? 2.0 : 4.0));
    p.splits = split4(p.M, p.N, p.kt);
    if (p.splits > 1) {
        p.acc = (float *)ws;
        if ((rc = tile_product(TILE_FP4, TILE_PARTIAL, p, s))) return rc;
        return tile_reduce(p.splits, p.M, p.N, p.acc, Y, bf, ldy, s, 0, 0, nullptr, nullptr, nullptr, bias, relu);
    }
    return tile_product(TILE_FP4, bf ? TILE_STORE : TILE_STORE_F32, p, s);
}

}  // extern "C"
