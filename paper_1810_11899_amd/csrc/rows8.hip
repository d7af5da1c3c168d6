// 8-bit rows: e4m3 values with one power-of-two scale for each block of 128
// columns (weights: of 128 x 128), and the elementwise pass of the backward
// pass that reads them.
#include <algorithm>

#include "rows8.h"

namespace gcn {
namespace {

constexpr int kTB = 256;
constexpr int kBlk = kRows8Block;

// The scale exponent of a block from the bits of its largest finite magnitude
// a = m 2^k: k - 8 where m <= 1.75 (448 = 1.75 * 2^8 is the largest e4m3
// value), k - 7 above, within -126 .. 127; 0 for a block of zeros.
__device__ __forceinline__ int block_exponent(uint32_t a) {
    const int k = (int)(a >> 23) - 127;
    const int e = k - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return a == 0u ? 0 : max(e, -126);   // (a subnormal a has k = -127: the bound holds it)
}
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}
// 2^-e, e in -126 .. 120
__device__ __forceinline__ float inverse_scale(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }

// four values to four e4m3 bytes: the hardware's rounding (nearest even), and
// the two departures: no value but zero becomes zero, not finite becomes NaN
__device__ __forceinline__ uint32_t held4(const float (&x)[4], float inv) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, r, true);
    uint32_t q = (uint32_t)r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        if (u != 0u && (q & (0x7Fu << (8 * i))) == 0u) q |= 1u << (8 * i) | ((__float_as_uint(x[i]) >> 31) << (8 * i + 7));
        if (u >= 0x7F800000u) q = (q & ~(0xFFu << (8 * i))) | (0x7Fu << (8 * i));
    }
    return q;
}

// eight consecutive elements from column c of a row (zeros past f)
template <bool BF>
__device__ __forceinline__ void load8(const void *row, int c, int f, float (&x)[8]) {
    if (c + 8 <= f) {
        if (BF) {
            const uint4 v = load16((const uint16_t *)row + c);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const uint4 a = load16((const float *)row + c), b = load16((const float *)row + c + 4);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = c + i < f ? (BF ? __uint_as_float((uint32_t)((const uint16_t *)row)[c + i] << 16)
                                   : ((const float *)row)[c + i])
                             : 0.0f;
    }
}

// Packs the 16 lanes' 128 values (8 a lane) and writes them; every lane of the
// 16 calls it.  The largest magnitude by four exchanges between the lanes.
__device__ __forceinline__ void pack_block(const float (&x)[8], uint8_t *q, uint8_t *scale, bool write) {
    uint32_t a = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, finite_magnitude(x[i]));
#pragma unroll
    for (int d = 1; d < 16; d *= 2) a = max(a, (uint32_t)__shfl_xor((int)a, d));
    const int e = block_exponent(a);
    const float inv = inverse_scale(e);
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    if (write) {
        *(uint2 *)(q + 8 * (threadIdx.x & 15)) = make_uint2(held4(lo, inv), held4(hi, inv));
        if ((threadIdx.x & 15) == 0) *scale = (uint8_t)(e + 127);
    }
}

// One block of 128 columns to 16 lanes, the lanes of a wavefront along the row
// (whole lines both ways).  Bound by memory: 65,536 x 1024 bfloat16 48 us, 4.2 TB/s.
template <bool BF>
__global__ __launch_bounds__(kTB) void pack_kernel(int64_t blocks, int32_t per_row, int32_t f, const void *X,
                                                   int64_t ldx, uint8_t *q, int64_t ldq, uint8_t *scale,
                                                   int64_t lds) {
    const int64_t stride = (int64_t)gridDim.x * (kTB / 16);
    for (int64_t b = (int64_t)blockIdx.x * (kTB / 16) + threadIdx.x / 16; b < ((blocks + 3) & ~(int64_t)3); b += stride) {
        const bool in = b < blocks;    // (the 64 lanes of a wavefront stay together)
        const int64_t row = in ? b / per_row : 0;
        const int32_t bc = in ? (int32_t)(b - row * per_row) : 0;
        float x[8];
        load8<BF>((const char *)X + row * ldx * (BF ? 2 : 4), bc * kBlk + 8 * (int)(threadIdx.x & 15), f, x);
        pack_block(x, q + row * ldq + bc * kBlk, scale + row * lds + bc, in);
    }
}

// eight 8-bit values under one scale
__device__ __forceinline__ void values8(uint2 q, int e, float (&x)[8]) {
    const uint32_t w[2] = {q.x, q.y};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
        x[4 * h] = __builtin_amdgcn_ldexpf(lo[0], e);
        x[4 * h + 1] = __builtin_amdgcn_ldexpf(lo[1], e);
        x[4 * h + 2] = __builtin_amdgcn_ldexpf(hi[0], e);
        x[4 * h + 3] = __builtin_amdgcn_ldexpf(hi[1], e);
    }
}

// eight columns to a thread; rows n .. drows - 1 and columns past f (to the last
// whole eight, where ldx holds them) are written as zeros when PAD
template <bool BF, bool PAD>
__device__ __forceinline__ void unpack_rows(int64_t first, int64_t step, int32_t drows, int32_t n, int32_t f,
                                            const uint8_t *q, int64_t ldq, const uint8_t *scale, int64_t lds, void *X,
                                            int64_t ldx) {
    const uint32_t per_row = (uint32_t)(f + 7) / 8;
    const int64_t total = (int64_t)drows * per_row;
    for (int64_t i = first; i < total; i += step) {
        const int64_t row = i / per_row;
        const int32_t c = (int32_t)(i - row * per_row) * 8;
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (!PAD || row < n)   // (q's columns past f hold zeros)
            values8(*(const uint2 *)(q + row * ldq + c), (int)scale[row * lds + c / kBlk] - 127, x);
        if (BF) {
            uint16_t *d = (uint16_t *)X + row * ldx + c;
            if (PAD || c + 8 <= f) {
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
template <bool BF>
__global__ __launch_bounds__(kTB) void unpack_kernel(int32_t n, int32_t f, const uint8_t *q, int64_t ldq,
                                                     const uint8_t *scale, int64_t lds, void *X, int64_t ldx) {
    unpack_rows<BF, false>((int64_t)blockIdx.x * kTB + threadIdx.x, (int64_t)gridDim.x * kTB, n, n, f, q, ldq, scale,
                                lds, X, ldx);
}

// One 128 x 128 block of the weights to a workgroup: the largest magnitude in
// a first pass over it, the values to both orientations in a second (through
// LDS, so that both are written along their rows).
template <bool BF>
__global__ __launch_bounds__(kTB) void pack_weights_kernel(int32_t K, int32_t N, const void *W, int64_t ldw, uint8_t *q,
                                                           int64_t ldq, uint8_t *qT, int64_t ldqT, uint8_t *scale,
                                                           int64_t lds) {
    __shared__ uint8_t tile[kBlk][kBlk + 4];
    __shared__ uint32_t top[kTB / 64];
    const int k0 = blockIdx.y * kBlk, n0 = blockIdx.x * kBlk;
    auto at = [&](int k, int n) {
        if (k >= K || n >= N) return 0.0f;
        const int64_t i = (int64_t)k * ldw + n;
        return BF ? __uint_as_float((uint32_t)((const uint16_t *)W)[i] << 16) : ((const float *)W)[i];
    };
    uint32_t a = 0u;
    for (int i = threadIdx.x; i < kBlk * kBlk; i += kTB) a = max(a, finite_magnitude(at(k0 + i / kBlk, n0 + i % kBlk)));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) a = max(a, (uint32_t)__shfl_xor((int)a, d));
    if ((threadIdx.x & 63) == 0) top[threadIdx.x / 64] = a;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTB / 64; ++w) a = max(a, top[w]);
    const int e = block_exponent(a);
    const float inv = inverse_scale(e);
    if (threadIdx.x == 0) scale[blockIdx.y * lds + blockIdx.x] = (uint8_t)(e + 127);
    for (int i = threadIdx.x; i < kBlk * kBlk / 4; i += kTB) {
        const int k = i / (kBlk / 4), n = i % (kBlk / 4) * 4;
        const float x[4] = {at(k0 + k, n0 + n), at(k0 + k, n0 + n + 1), at(k0 + k, n0 + n + 2), at(k0 + k, n0 + n + 3)};
        const uint32_t v = held4(x, inv);
        *(uint32_t *)&tile[k][n] = v;
        if (q && k0 + k < K) *(uint32_t *)(q + (int64_t)(k0 + k) * ldq + n0 + n) = v;
    }
    if (!qT) return;
    __syncthreads();
    for (int i = threadIdx.x; i < kBlk * kBlk / 4; i += kTB) {
        const int n = i / (kBlk / 4), k = i % (kBlk / 4) * 4;
        if (n0 + n >= N) continue;
        *(uint32_t *)(qT + (int64_t)(n0 + n) * ldqT + k0 + k) =
            (uint32_t)tile[k][n] | (uint32_t)tile[k + 1][n] << 8 | (uint32_t)tile[k + 2][n] << 16 | (uint32_t)tile[k + 3][n] << 24;
    }
}

// The elementwise half of the backward pass: dZ = bf16(dY) where the mask byte
// is a positive e4m3 value (1 .. 0x7E), zero elsewhere, as bfloat16 rows; the
// column sums of a strip of rows; and, when wanted, dZ's 8-bit rows.  All three,
// and dW, are of the rounded dZ: db belongs to the dW beside it.  One
// block of 128 columns and a strip of rows to a workgroup, 16 lanes a row, so
// that one pass over dY and the mask serves all three.  The rows from n to nz
// are zeros.  The workgroups past the strips widen X8 to bfloat16 rows.  Bound by
// memory: 65,536 x 512 bfloat16 dY beside 65,536 x 1024 X8 67 us for 400 MB (part of
// it in the last-level cache), as long as the product behind it.
struct MaskArgs {
    int32_t n, nz, N, rows_per_strip, strips, blocks;   // blocks: of 128 columns
    const void *dY;
    int64_t lddy;
    const uint8_t *mask;
    int64_t ldm;
    uint16_t *dZ;
    int64_t lddz;
    float *part;
    uint8_t *q;
    int64_t ldq;
    uint8_t *scale;
    int64_t lds;
    // X8 [n x f] to X [nz x ldx]
    int32_t f;
    const uint8_t *xq;
    int64_t ldxq;
    const uint8_t *xscale;
    int64_t ldxs;
    uint16_t *X;
    int64_t ldx;
};
template <bool BF>
__global__ __launch_bounds__(kTB) void mask_kernel(MaskArgs a) {
    __shared__ float red[kTB / 16][kBlk];
    const int strip = (int)(blockIdx.x / a.blocks), cb = (int)(blockIdx.x % a.blocks);
    if (strip >= a.strips) {
        const int64_t b = (int64_t)blockIdx.x - (int64_t)a.strips * a.blocks;
        unpack_rows<true, true>(b * kTB + threadIdx.x, ((int64_t)gridDim.x - (int64_t)a.strips * a.blocks) * kTB, a.nz,
                                      a.n, a.f, a.xq, a.ldxq, a.xscale, a.ldxs, a.X, a.ldx);
        return;
    }
    const int32_t n = a.n, N = a.N;
    const void *const dY = a.dY;
    const int64_t lddy = a.lddy, ldm = a.ldm, lddz = a.lddz, ldq = a.ldq, lds = a.lds;
    const uint8_t *const mask = a.mask;
    uint16_t *const dZ = a.dZ;
    float *const part = a.part;
    uint8_t *const q = a.q, *const scale = a.scale;
    const int c = cb * kBlk + 8 * (int)(threadIdx.x & 15);
    const int64_t r0 = (int64_t)strip * a.rows_per_strip;
    const int64_t r1 = min(r0 + a.rows_per_strip, (int64_t)a.nz);
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    // (the strip's rows in steps of 16; the lanes past its end stay for the
    // exchanges of pack_block)
    for (int64_t b = r0; b < r1; b += kTB / 16) {
        const int64_t r = b + threadIdx.x / 16;
        const bool in = r < r1 && r < n;
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (in) {
            load8<BF>((const char *)dY + r * lddy * (BF ? 2 : 4), c, N, x);
            uint32_t m[2] = {0x01010101u, 0x01010101u};
            if (mask) {
                const uint8_t *mp = mask + r * ldm + c;
                if (c + 8 <= N) {
                    __builtin_memcpy(m, mp, 8);
                } else {
                    m[0] = m[1] = 0u;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i < N) m[i / 4] |= (uint32_t)mp[i] << (8 * (i & 3));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t byte = (m[i / 4] >> (8 * (i & 3))) & 0xFFu;
                const float v = BF ? x[i] : __uint_as_float((uint32_t)to_bf16(x[i]) << 16);
                x[i] = byte - 1u < 0x7Eu ? v : 0.0f;
                sum[i] += x[i];
            }
        }
        if (r < r1) {
            if (c < lddz)
                *(uint4 *)(dZ + r * lddz + c) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                           pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
        }
        if (q) pack_block(x, q + (in ? r : 0) * ldq + cb * kBlk, scale + (in ? r : 0) * lds + cb, in);
    }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) red[threadIdx.x / 16][8 * (threadIdx.x & 15) + i] = sum[i];
    __syncthreads();
    const int k = cb * kBlk + threadIdx.x;
    if (threadIdx.x < kBlk && k < N) {
        float t = 0.0f;
#pragma unroll
        for (int g = 0; g < kTB / 16; ++g) t += red[g][threadIdx.x];
        part[(int64_t)strip * N + k] = t;
    }
}

int check_type(gcn_rows_type t, const char *who) {
    GCN_REQUIRE(t == GCN_ROWS_F32 || t == GCN_ROWS_BF16, GCN_EINVAL, "%s: bad element type %d", who, (int)t);
    return GCN_OK;
}

bool aligned(const void *p, uintptr_t b) { return (uintptr_t)p % b == 0; }
uintptr_t el(gcn_rows_type t) { return t == GCN_ROWS_BF16 ? 2 : 4; }

unsigned grid_of(int64_t work, int64_t per_block, int64_t most) {
    return (unsigned)std::max<int64_t>(1, std::min(most, (work + per_block - 1) / per_block));
}

}  // namespace

int check_rows8(const gcn_rows8 *r, const char *who) {
    GCN_REQUIRE(r, GCN_EINVAL, "%s: null 8-bit rows", who);
    GCN_REQUIRE(r->n >= 0 && r->f > 0, GCN_ESHAPE, "%s: 8-bit rows of %d x %d", who, r->n, r->f);
    GCN_REQUIRE(r->ldq % 16 == 0 && r->ldq >= kBlk * blocks8(r->f), GCN_ESHAPE,
                "%s: ldq=%d is not a multiple of 16 of at least %lld", who, r->ldq, (long long)(kBlk * blocks8(r->f)));
    GCN_REQUIRE(r->ldscale >= blocks8(r->f), GCN_ESHAPE, "%s: ldscale=%d < %lld", who, r->ldscale,
                (long long)blocks8(r->f));
    GCN_REQUIRE(r->n == 0 || (r->q && r->scale), GCN_EINVAL, "%s: null 8-bit rows", who);
    GCN_REQUIRE(aligned(r->q, 16), GCN_EINVAL, "%s: 8-bit rows must be 16-byte aligned", who);
    return GCN_OK;
}

int rows8_pack(int32_t n, int32_t f, const void *X, int x_bf16, int64_t ldx, uint8_t *q, int64_t ldq,
               uint8_t *scale, int64_t lds, hipStream_t s) {
    if (n == 0) return GCN_OK;
    const int32_t per_row = (int32_t)blocks8(f);
    const int64_t blocks = (int64_t)n * per_row;
    ProfScope prof(K_ROWS8_PACK, s, 0.0, (double)n * f * (x_bf16 ? 3.0 : 5.0) + (double)blocks);
    const unsigned g = grid_of(blocks, kTB / 16, 16384);
    if (x_bf16)
        hipLaunchKernelGGL(pack_kernel<true>, dim3(g), dim3(kTB), 0, s, blocks, per_row, f, X, ldx, q, ldq, scale, lds);
    else
        hipLaunchKernelGGL(pack_kernel<false>, dim3(g), dim3(kTB), 0, s, blocks, per_row, f, X, ldx, q, ldq, scale, lds);
    GCN_LAUNCH_CHECK("pack_kernel");
    return GCN_OK;
}

}  // namespace gcn

using namespace gcn;

extern "C" {

int gcn_rows8_pack(const void *X, gcn_rows_type type, int32_t ldx, const gcn_rows8 *out, void *stream) {
    int rc = check_rows8(out, "gcn_rows8_pack");
    if (rc) return rc;
    if ((rc = check_type(type, "gcn_rows8_pack"))) return rc;
    GCN_REQUIRE(ldx >= out->f, GCN_ESHAPE, "gcn_rows8_pack: ldx=%d < f=%d", ldx, out->f);
    GCN_REQUIRE(out->n == 0 || (X && aligned(X, el(type))), GCN_EINVAL, "gcn_rows8_pack: null or misaligned pointer");
    return rows8_pack(out->n, out->f, X, type == GCN_ROWS_BF16, ldx, out->q, out->ldq, out->scale, out->ldscale,
                      (hipStream_t)stream);
}

int gcn_rows8_unpack(const gcn_rows8 *r, void *X, gcn_rows_type type, int32_t ldx, void *stream) {
    int rc = check_rows8(r, "gcn_rows8_unpack");
    if (rc) return rc;
    if ((rc = check_type(type, "gcn_rows8_unpack"))) return rc;
    GCN_REQUIRE(ldx >= r->f, GCN_ESHAPE, "gcn_rows8_unpack: ldx=%d < f=%d", ldx, r->f);
    GCN_REQUIRE(r->n == 0 || (X && aligned(X, el(type))), GCN_EINVAL, "gcn_rows8_unpack: null or misaligned pointer");
    if (r->n == 0) return GCN_OK;
    hipStream_t s = (hipStream_t)stream;
    const bool bf = type == GCN_ROWS_BF16;
    ProfScope prof(K_ROWS8_PACK, s, 0.0, (double)r->n * r->f * (bf ? 3.0 : 5.0));
    const unsigned g = grid_of((int64_t)r->n * ((r->f + 7) / 8), kTB, 16384);
    if (bf)
        hipLaunchKernelGGL(unpack_kernel<true>, dim3(g), dim3(kTB), 0, s, r->n, r->f, r->q, (int64_t)r->ldq, r->scale,
                           (int64_t)r->ldscale, X, (int64_t)ldx);
    else
        hipLaunchKernelGGL(unpack_kernel<false>, dim3(g), dim3(kTB), 0, s, r->n, r->f, r->q, (int64_t)r->ldq, r->scale,
                           (int64_t)r->ldscale, X, (int64_t)ldx);
    GCN_LAUNCH_CHECK("unpack_kernel");
    return GCN_OK;
}

int gcn_weights8_pack(const void *W, gcn_rows_type type, int32_t ldw, const gcn_weights8 *out, void *stream) {
    GCN_REQUIRE(out && W, GCN_EINVAL, "gcn_weights8_pack: null pointer");
    const int32_t K = out->K, N = out->N;
    GCN_REQUIRE(K > 0 && N > 0, GCN_ESHAPE, "gcn_weights8_pack: K=%d N=%d", K, N);
    int rc = check_type(type, "gcn_weights8_pack");
    if (rc) return rc;
    GCN_REQUIRE(aligned(W, el(type)), GCN_EINVAL, "gcn_weights8_pack: misaligned pointer");
    GCN_REQUIRE(ldw >= N, GCN_ESHAPE, "gcn_weights8_pack: ldw=%d < N=%d", ldw, N);
    GCN_REQUIRE((out->q || out->qT) && out->scale, GCN_EINVAL, "gcn_weights8_pack: null 8-bit weights");
    GCN_REQUIRE(!out->q || (out->ldq % 16 == 0 && out->ldq >= kBlk * blocks8(N) && aligned(out->q, 16)), GCN_ESHAPE,
                "gcn_weights8_pack: q needs 16-byte alignment and ldq=%d a multiple of 16 of at least %lld", out->ldq,
                (long long)(kBlk * blocks8(N)));
    GCN_REQUIRE(!out->qT || (out->ldqT % 16 == 0 && out->ldqT >= kBlk * blocks8(K) && aligned(out->qT, 16)), GCN_ESHAPE,
                "gcn_weights8_pack: qT needs 16-byte alignment and ldqT=%d a multiple of 16 of at least %lld",
                out->ldqT, (long long)(kBlk * blocks8(K)));
    GCN_REQUIRE(out->ldscale >= blocks8(N), GCN_ESHAPE, "gcn_weights8_pack: ldscale=%d < %lld", out->ldscale,
                (long long)blocks8(N));
    GCN_REQUIRE(blocks8(K) <= 65535, GCN_EUNSUPPORTED, "gcn_weights8_pack: K=%d", K);
    hipStream_t s = (hipStream_t)stream;
    ProfScope prof(K_ROWS8_PACK, s, 0.0,
                   (double)K * N * ((type == GCN_ROWS_BF16 ? 2.0 : 4.0) + (out->q ? 1 : 0) + (out->qT ? 1 : 0)));
    const dim3 g((unsigned)blocks8(N), (unsigned)blocks8(K));
    if (type == GCN_ROWS_BF16)
        hipLaunchKernelGGL(pack_weights_kernel<true>, g, dim3(kTB), 0, s, K, N, W, (int64_t)ldw, out->q,
                           (int64_t)out->ldq, out->qT, (int64_t)out->ldqT, out->scale, (int64_t)out->ldscale);
    else
        hipLaunchKernelGGL(pack_weights_kernel<false>, g, dim3(kTB), 0, s, K, N, W, (int64_t)ldw, out->q,
                           (int64_t)out->ldq, out->qT, (int64_t)out->ldqT, out->scale, (int64_t)out->ldscale);
    GCN_LAUNCH_CHECK("pack_weights_kernel");
    return GCN_OK;
}

namespace {
// Rows and columns of the operands in whole 64-row pieces and 16-byte chunks.
struct GradPlan {
    int32_t nz, Np, fp, splits, strip, strips;
    size_t total;
};
struct GradBuffers {
    uint16_t *dZ, *X;
    float *part, *acc;
};
GradPlan plan_grad(int32_t n, int32_t f, int32_t N, void *ws, size_t ws_bytes, GradBuffers &b) {
    GradPlan p{};
    p.nz = (n + 63) / 64 * 64;
    p.Np = (N + 7) / 8 * 8;
    p.fp = (f + 7) / 8 * 8;
    p.splits = tile_splits(f, N, p.nz / 64, false);
    // strips: about 2048 workgroups, at least 16 rows each
    const int64_t most = std::max<int64_t>(1, 2048 / blocks8(N));
    p.strip = (int32_t)std::max<int64_t>(16, ((p.nz + most - 1) / most + 15) / 16 * 16);
    p.strips = std::max(1, (int32_t)(((int64_t)p.nz + p.strip - 1) / p.strip));
    Arena ar(ws, ws_bytes);
    b.dZ = ar.take<uint16_t>((size_t)p.nz * p.Np);
    b.X = ar.take<uint16_t>((size_t)p.nz * p.fp);
    b.part = ar.take<float>((size_t)p.strips * N);
    b.acc = ar.take<float>((size_t)p.splits * f * N);
    p.total = ar.used + 256;
    return p;
}
}  // namespace

size_t gcn_rows8_weight_grad_workspace_bytes(int32_t n, int32_t f, int32_t N) {
    if (n < 0 || f <= 0 || N <= 0 || std::max({n, f, N}) > kMostRows) return 0;
    GradBuffers b;
    return plan_grad(n, f, N, nullptr, 0, b).total;
}

int gcn_rows8_weight_grad(const gcn_rows8 *X8, const uint8_t *mask, int32_t ldmask, const void *dY, gcn_rows_type type,
                          int32_t lddy, int32_t N, float *dW, int32_t lddw, float *db, const gcn_rows8 *dZ8, void *ws,
                          size_t ws_bytes, void *stream) {
    int rc = check_rows8(X8, "gcn_rows8_weight_grad");
    if (rc) return rc;
    if ((rc = check_type(type, "gcn_rows8_weight_grad"))) return rc;
    const int32_t n = X8->n, f = X8->f;
    GCN_REQUIRE(N > 0, GCN_ESHAPE, "gcn_rows8_weight_grad: N=%d", N);
    GCN_REQUIRE(lddy >= N && lddw >= N && (!mask || ldmask >= N), GCN_ESHAPE,
                "gcn_rows8_weight_grad: lddy=%d lddw=%d ldmask=%d < N=%d", lddy, lddw, ldmask, N);
    GCN_REQUIRE(dW && (n == 0 || (dY && aligned(dY, el(type)))) && aligned(dW, 4) && aligned(db, 4), GCN_EINVAL,
                "gcn_rows8_weight_grad: null or misaligned pointer");
    GCN_REQUIRE(n <= kMostRows && N <= kMostRows && f <= kMostRows, GCN_EUNSUPPORTED,
                "gcn_rows8_weight_grad: n=%d f=%d N=%d", n, f, N);
    if (dZ8) {
        if ((rc = check_rows8(dZ8, "gcn_rows8_weight_grad"))) return rc;
        GCN_REQUIRE(dZ8->n == n && dZ8->f == N, GCN_ESHAPE, "gcn_rows8_weight_grad: dZ8 is %d x %d, not %d x %d", dZ8->n,
                    dZ8->f, n, N);
    }
    GradBuffers b;
    const GradPlan p = plan_grad(n, f, N, ws, ws_bytes, b);
    GCN_REQUIRE(ws && aligned(ws, 256) && ws_bytes >= p.total, GCN_EWORKSPACE,
                "gcn_rows8_weight_grad: workspace %zu < %zu bytes, or not 256-byte aligned", ws_bytes, p.total);
    hipStream_t s = (hipStream_t)stream;
    if (n == 0) {
        if (lddw == N) rc = fill_zero(dW, (int64_t)f * N, s);
        if (rc) return rc;
        for (int32_t i = 0; lddw != N && i < f; ++i)
            if ((rc = fill_zero(dW + (int64_t)i * lddw, N, s))) return rc;
        return db ? fill_zero(db, N, s) : GCN_OK;
    }
    {
        const bool bf = type == GCN_ROWS_BF16;
        ProfScope prof(K_ROWS8_MASK, s, 0.0,
                       (double)n * N * ((bf ? 4.0 : 6.0) + (mask ? 1.0 : 0.0) + (dZ8 ? 1.0 : 0.0)) + 3.0 * n * f);
        const int32_t blocks = (int32_t)blocks8(N);
        const MaskArgs m{n, p.nz, N, p.strip, p.strips, blocks, dY, lddy, mask, ldmask, b.dZ, p.Np, db ? b.part : nullptr,
                         dZ8 ? dZ8->q : nullptr, dZ8 ? dZ8->ldq : 0, dZ8 ? dZ8->scale : nullptr, dZ8 ? dZ8->ldscale : 0,
                         f, X8->q, X8->ldq, X8->scale, X8->ldscale, b.X, p.fp};
        const dim3 g((unsigned)(p.strips * blocks) + grid_of((int64_t)p.nz * (p.fp / 8), kTB, 4096));
        if (bf) hipLaunchKernelGGL(mask_kernel<true>, g, dim3(kTB), 0, s, m);
        else hipLaunchKernelGGL(mask_kernel<false>, g, dim3(kTB), 0, s, m);
        GCN_LAUNCH_CHECK("mask_kernel");
    }
    ProfScope prof(K_ROWS8_WEIGHT_GRAD, s, 2.0 * n * f * N, 2.0 * n * f + 2.0 * n * N + 4.0 * f * N);
    TileProduct w{};
    w.A = (const uint8_t *)b.X;
    w.lda = 2 * (int64_t)p.fp;
    w.B = (const uint8_t *)b.dZ;
    w.ldb = 2 * (int64_t)p.Np;
    w.M = f;
    w.N = N;
    w.kt = p.nz / 64;
    w.splits = p.splits;
    w.acc = b.acc;
    if ((rc = tile_product(TILE_BF16_TN, TILE_PARTIAL, w, s))) return rc;
    return tile_reduce(p.splits, f, N, b.acc, dW, 0, lddw, s, p.strips, db ? N : 0, b.part, db);
}

}  // extern "C"
