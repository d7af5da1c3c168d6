// PREDICT and softmax cross entropy over many classes in pieces of the
// classes, without keeping the logits (gcn_classes.h).
//
//   pass 1, per piece: logits of the piece in the product's registers; per row
//     and column tile their maximum and the sum of exponentials relative to
//     it, joined into the row's running maximum and sum
//   loss: row_loss = max + log(sum) - label's logit
//   pass 2, per piece: the logits again, n_l G = softmax - onehot in the same
//     registers, written as bfloat16 rows; then n_l dHL += n_l G W_piece^T and
//     n_l dW_piece = HL^T n_l G.  1 / n_l is a factor of the float32 sums: in G it
//     would be rounded, and the same way in every row (17 rows: the gradients
//     0.0036 off in the 2-norm instead of 0.0018).
#include <algorithm>

#include "gcn_classes.h"
#include "rows8.h"

namespace gcn {
namespace {

constexpr int kTB = 256;
constexpr int kSmallRows = 32, kSmallTile = 128;   // rows and columns of the smallest tiles

__device__ __forceinline__ bool has_label(int32_t l, int32_t C) { return l >= 0 && l < C; }

// (m, s): a maximum and the sum of exponentials relative to it, joined with (q, u)
__device__ __forceinline__ void join(float &m, float &s, float q, float u) {
    const float b = fmaxf(m, q);
    s = (m == b ? s : s * __expf(m - b)) + (q == b ? u : u * __expf(q - b));
    m = b;
}

// dst [drows x ldd] = src [rows x cols] (lds), zero past rows and cols and in
// rows without a label
template <class T>
struct CopyRows {
    int32_t drows, rows, cols;
    const T *src;
    int64_t lds;
    T *dst;
    int64_t ldd;
    const int32_t *labels;   // null: every row counts
    int32_t C;
};
template <class T>
__device__ __forceinline__ void copy_rows(const CopyRows<T> &a, int64_t first, int64_t step) {
    constexpr int V = 16 / sizeof(T);   // elements of a store
    const bool wide = a.ldd % V == 0;
    const int64_t per = (a.ldd + V - 1) / V, total = a.drows * per;
    for (int64_t i = first; i < total; i += step) {
        const int64_t r = i / per;
        const int32_t c = (int32_t)(i - r * per) * V;
        const bool in = r < a.rows && (!a.labels || has_label(a.labels[r], a.C));
        const T *x = a.src + r * a.lds + c;
        T v[V];
        if (in && c + V <= a.cols) {
            *(uint4 *)v = load16(x);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = in && c + e < a.cols ? x[e] : (T)0;
        }
        T *d = a.dst + r * a.ldd + c;
        if (wide) {
            *(uint4 *)d = *(uint4 *)v;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < a.ldd) d[e] = v[e];
        }
    }
}
// Block 0: inv_count = 1 / max(1, rows with a label); the next `split` blocks the
// first copy, the others the second (which may be empty).
template <class T>
__global__ __launch_bounds__(kTB) void prep_kernel(int32_t n, float *inv_count, CopyRows<T> a, uint32_t split, CopyRows<T> b) {
    if (blockIdx.x == 0) {
        __shared__ int32_t part[kTB / 64];
        int32_t k = 0;
#pragma unroll 8
        for (int32_t i = threadIdx.x; i < n; i += kTB) k += has_label(a.labels[i], a.C);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) k += __shfl_xor(k, d);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = k;
        __syncthreads();
        if (threadIdx.x == 0) {
            int32_t t = 0;
            for (int w = 0; w < kTB / 64; ++w) t += part[w];
            inv_count[0] = (float)(1.0 / (double)max(t, 1));
        }
        return;
    }
    const uint32_t k = blockIdx.x - 1;
    if (k < split) copy_rows(a, (int64_t)k * kTB + threadIdx.x, (int64_t)split * kTB);
    else copy_rows(b, (int64_t)(k - split) * kTB + threadIdx.x, (int64_t)(gridDim.x - 1 - split) * kTB);
}
template <class T>
__global__ __launch_bounds__(kTB) void copy_rows_kernel(CopyRows<T> a) {
    copy_rows(a, (int64_t)blockIdx.x * kTB + threadIdx.x, (int64_t)gridDim.x * kTB);
}

// the tiles' maxima and sums of one piece joined into the running ones: 32 rows
// to a workgroup, eight threads a row, so that many loads are in flight
__global__ __launch_bounds__(kTB) void join_kernel(int32_t n, int32_t tiles, const float *tile_max,
                                                   const float *tile_sum, float *run_max, float *run_sum, int first) {
    __shared__ float sm[8][32], ss[8][32];
    const int lr = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int32_t i = blockIdx.x * 32 + lr;
    float m = -INFINITY, s = 0.0f;
    if (i < n) {
#pragma unroll 4
        for (int32_t t = part; t < tiles; t += 8) join(m, s, tile_max[(int64_t)t * n + i], tile_sum[(int64_t)t * n + i]);
    }
    sm[part][lr] = m;
    ss[part][lr] = s;
    __syncthreads();
    if (part != 0 || i >= n) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) join(m, s, sm[k][lr], ss[k][lr]);
    if (!first) join(m, s, run_max[i], run_sum[i]);
    run_max[i] = m;
    run_sum[i] = s;
}

// logits of one piece (float32 rows of ldx, a multiple of 4) joined into the
// running maximum and sum, a workgroup a row (and grid rows on, beyond 2^20)
__global__ __launch_bounds__(kTB) void stats_rows_kernel(int32_t n, int32_t P, const float *X, int64_t ldx, const int32_t *labels,
                                                         int32_t class0, int32_t C, float *run_max, float *run_sum,
                                                         float *label_logit, int first) {
    __shared__ float sm[kTB / 64], ss[kTB / 64];
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        __syncthreads();   // (the row before has been read)
        const float *x = X + row * ldx;
        float m = -INFINITY, s = 0.0f;
        for (int32_t c = 4 * (int32_t)threadIdx.x; c < P; c += 4 * kTB) {
            const float4 v = *(const float4 *)(x + c);
            float y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 1; e < 4; ++e)
                if (c + e >= P) y[e] = -INFINITY;
            const float b = fmaxf(m, fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])));
            if (b > m) {
                s *= expf(m - b);   // (0 of the empty sum: exp(-infinity))
                m = b;
            }
            const float base = m == -INFINITY ? 0.0f : m;   // no finite logit yet: the sum stays 0
#pragma unroll
            for (int e = 0; e < 4; ++e) s += expf(y[e] - base);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const float q = __shfl_xor(m, d), u = __shfl_xor(s, d);
            join(m, s, q, u);
        }
        if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m, ss[threadIdx.x >> 6] = s;
        __syncthreads();
        if (threadIdx.x != 0) continue;
        for (int w = 1; w < kTB / 64; ++w) join(m, s, sm[w], ss[w]);
        if (!first) join(m, s, run_max[row], run_sum[row]);
        run_max[row] = m;
        run_sum[row] = s;
        const int32_t l = labels[row];
        if (has_label(l, C) && l >= class0 && l - class0 < P) label_logit[row] = x[l - class0];
    }
}

// X <- G, and the column sums of strips of kStrip rows: a thread has a column
constexpr int kStrip = 32;
__global__ __launch_bounds__(kTB) void grad_rows_kernel(int32_t n, int32_t P, float *X, int64_t ldx,
                                                        const int32_t *labels, int32_t class0, int32_t C,
                                                        const float *lse, const float *inv_count, float *part) {
    __shared__ float z[kStrip];
    __shared__ int32_t lab[kStrip];
    const int32_t c = blockIdx.x * kTB + threadIdx.x, strips = (n + kStrip - 1) / kStrip;
    const float inv = inv_count[0];
    for (int32_t strip = blockIdx.y; strip < strips; strip += gridDim.y) {
        const int32_t r0 = strip * kStrip, rows = min(kStrip, n - r0);
        __syncthreads();
        if ((int32_t)threadIdx.x < rows) {
            const int32_t l = labels[r0 + threadIdx.x];
            z[threadIdx.x] = lse[r0 + threadIdx.x];
            lab[threadIdx.x] = has_label(l, C) ? l : -1;
        }
        __syncthreads();
        if (c >= P) continue;
        float sum = 0.0f;
        float *x = X + r0 * ldx + c;
        // (eight loads before the first store, behind which the next one would wait)
        for (int32_t r = 0; r < rows; r += 8, x += 8 * ldx) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = r + e < rows ? x[e * ldx] : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (r + e >= rows) break;
                const int32_t l = lab[r + e];
                const float g = l >= 0 ? (expf(v[e] - z[r + e]) - (class0 + c == l ? 1.0f : 0.0f)) * inv : 0.0f;
                x[e * ldx] = g;
                sum += g;
            }
        }
        part[(int64_t)strip * P + c] = sum;
    }
}

// lse, the rows' losses and their mean, by one workgroup in a fixed order.
// tiles > 0: the only piece's tiles are joined here (few rows and tiles).
__global__ __launch_bounds__(1024) void loss_kernel(int32_t n, int32_t C, const int32_t *__restrict__ labels,
                                                    int32_t tiles, const float *__restrict__ tile_max,
                                                    const float *__restrict__ tile_sum, const float *__restrict__ run_max,
                                                    const float *__restrict__ run_sum,
                                                    const float *__restrict__ label_logit, float *__restrict__ lse,
                                                    float *__restrict__ row_loss, const float *__restrict__ inv_count,
                                                    float *__restrict__ loss) {
    __shared__ double part[16];
    double t = 0.0;
#pragma unroll 4
    for (int32_t i = threadIdx.x; i < n; i += 1024) {
        float m, s;
        if (tiles > 0) {
            m = -INFINITY, s = 0.0f;
            for (int32_t k = 0; k < tiles; ++k) join(m, s, tile_max[(int64_t)k * n + i], tile_sum[(int64_t)k * n + i]);
        } else {
            m = run_max[i], s = run_sum[i];
        }
        const float z = m + logf(s);
        lse[i] = z;
        const bool has = has_label(labels[i], C);
        const float v = has ? z - label_logit[i] : 0.0f;
        if (row_loss) row_loss[i] = v;
        t += v;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) t += __shfl_xor(t, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        double a = 0.0;
        for (int w = 0; w < 16; ++w) a += part[w];
        loss[0] = (float)(a * (double)inv_count[0]);
    }
}

__global__ __launch_bounds__(kTB) void add_kernel(int32_t rows, int32_t cols, const float *x, float *y, int64_t ldy) {
    const int64_t total = (int64_t)rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * kTB + threadIdx.x; i < total; i += (int64_t)gridDim.x * kTB)
        y[i / cols * ldy + i % cols] += x[i];
}

__global__ __launch_bounds__(kTB) void zero_kernel(uint16_t *x, int64_t rows, int64_t cols, int64_t ld) {
    for (int64_t i = (int64_t)blockIdx.x * kTB + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * kTB)
        x[i / cols * ld + i % cols] = 0;
}

unsigned grid_of(int64_t work, int64_t most = 8192) {
    return (unsigned)std::max<int64_t>(1, std::min(most, (work + kTB - 1) / kTB));
}
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// How a call is cut and what of the workspace it uses.
struct Plan {
    int64_t fp, np;            // f and n in whole 64-column pieces (bfloat16)
    int32_t piece, pieces;     // classes per piece
    int32_t split_h, split_w;  // parts of the two gradient products (bfloat16)
    bool in_place;             // W_pred's own rows serve as operands
    size_t total;
};
struct Buffers {
    float *inv_count, *run_max, *run_sum, *label_logit, *lse, *tile_max, *tile_sum, *colpart, *acc, *part, *X, *tmp;
    uint16_t *H, *W, *G;
    float *Hz;
    void *gemm_ws;
    size_t gemm_bytes;
};

GemmProblem dw_f32(int32_t f, int32_t P, int32_t n) {
    GemmProblem w{};
    w.M = f;
    w.N = P;
    w.seg[0].K = n;
    return w;
}

// About 640 blocks: the library's rule for weight gradients fills four blocks a
// CU, whose partials here are as wide as the classes (2000 x 256, 10,007 classes,
// the call: 1 part 445 us, 2 384, 4 359, 6 407, 8 398, 16 461).
int32_t dw_split_f32(const GemmProblem &w) {
    const int64_t tiles = ((int64_t)w.M + 127) / 128 * (((int64_t)w.N + 127) / 128);
    return (int32_t)std::min<int64_t>(gemm_pick_split(1, &w, true), std::max<int64_t>(1, 640 / tiles));
}
GemmProblem dh_f32(int32_t n, int32_t f, int32_t P) {
    GemmProblem d{};
    d.M = n;
    d.N = f;
    d.seg[0].K = P;
    return d;
}

// The elements of a piece: bfloat16 G takes 2 bytes each, float32 logits 4.
constexpr int64_t kPieceElems = (int64_t)1 << 28, kPieceElemsF32 = (int64_t)1 << 26;

// W: the weights, or null in the workspace query, which counts on copying them.
Plan plan_of(int32_t n, int32_t f, int32_t C, bool bf, bool grad, const void *W, void *ws, size_t ws_bytes, Buffers &b) {
    Plan p{};
    Arena ar(ws, ws_bytes);
    const int64_t rows = std::max(n, 1);
    p.fp = up(f, 64);
    p.np = up(rows, 64);
    p.in_place = W && (uintptr_t)W % 16 == 0 && C % 8 == 0 && f % 64 == 0;
    int64_t piece = std::max<int64_t>(256, (bf ? kPieceElems / p.np : kPieceElemsF32 / rows) / 256 * 256);
    piece = std::min<int64_t>(piece, up(C, 256));
    p.pieces = (int32_t)((C + piece - 1) / piece);
    p.piece = (int32_t)std::min<int64_t>(piece, C);
    b = Buffers{};
    b.inv_count = ar.take<float>(1);
    b.run_max = ar.take<float>(rows);
    b.run_sum = ar.take<float>(rows);
    b.label_logit = ar.take<float>(rows);
    b.lse = ar.take<float>(rows);
    if (bf) {
        // (sized for the smallest tiles: a last, smaller piece may run on them)
        const int64_t tn = (p.piece + kSmallTile - 1) / kSmallTile;
        b.tile_max = ar.take<float>(tn * rows);
        b.tile_sum = ar.take<float>(tn * rows);
        b.H = ar.take<uint16_t>(p.np * p.fp);
        // (a piece of whole 64-column parts is read in place where W_pred's rows
        // are 16-byte aligned and f is whole: only a ragged last piece is copied)
        const int32_t last = C - (p.pieces - 1) * p.piece;
        const int64_t copied = std::max(p.in_place && p.piece % 64 == 0 ? 0 : p.piece, p.in_place && last % 64 == 0 ? 0 : last);
        b.W = copied ? ar.take<uint16_t>(p.fp * up(copied, 64)) : nullptr;
        if (grad) {
            const int64_t pp = up(p.piece, 64);
            b.G = ar.take<uint16_t>(p.np * pp);
            b.colpart = ar.take<float>((p.np + kSmallRows - 1) / kSmallRows * p.piece);
            p.split_h = tile_splits(n, f, (int32_t)(pp / 64));
            p.split_w = tile_splits(f, p.piece, (int32_t)(p.np / 64));
            b.acc = ar.take<float>((size_t)p.split_h * rows * f);
            if (p.split_w > 1) b.part = ar.take<float>((size_t)p.split_w * f * p.piece);
        }
    } else {
        b.Hz = ar.take<float>(rows * f);
        b.X = ar.take<float>(rows * up(p.piece, 4));
        if (grad) {
            // (a last, smaller piece may be split more than the others)
            const int32_t last = C - (p.pieces - 1) * p.piece;
            for (int32_t P : {p.piece, last}) {
                const GemmProblem w = dw_f32(f, P, n), h = dh_f32(n, f, P);
                b.gemm_bytes = std::max(b.gemm_bytes, gemm_workspace_bytes(1, &w, dw_split_f32(w)));
                b.gemm_bytes = std::max(b.gemm_bytes, gemm_workspace_bytes(1, &h, gemm_pick_split(1, &h, false)));
            }
            b.gemm_ws = b.gemm_bytes ? ar.take<char>(b.gemm_bytes) : nullptr;
            b.colpart = ar.take<float>((rows + kStrip - 1) / kStrip * p.piece);
            if (p.pieces > 1) b.tmp = ar.take<float>(rows * f);
        }
    }
    p.total = ar.used + 256;
    return p;
}

int loss_bf16(const Plan &p, const Buffers &b, const uint16_t *HL, int32_t n, int32_t f, int64_t ldhl, const uint16_t *W,
              const float *bias, int32_t C, const int32_t *labels, float *loss, float *row_loss, uint16_t *dHL,
              int64_t lddhl, uint16_t *dW, float *db, hipStream_t s) {
    int rc;
    // (a single copied piece of W_pred goes along)
    auto w_copy = [&](int32_t c0, int32_t P) {
        return CopyRows<uint16_t>{(int32_t)p.fp, f, P, W + c0, C, b.W, up(P, 64), nullptr, 0};
    };
    const bool copied = p.pieces == 1 && !(p.in_place && C % 64 == 0);
    {
        ProfScope prof(K_CLASS_PREP, s, 0.0, 4.0 * n * f);
        const CopyRows<uint16_t> h{(int32_t)p.np, n, f, HL, ldhl, b.H, p.fp, labels, C};
        const unsigned gh = grid_of(p.np * p.fp / 8, 4096), gw = copied ? grid_of(p.fp * up(C, 64) / 8, 4096) : 0;
        hipLaunchKernelGGL(prep_kernel<uint16_t>, dim3(1 + gh + gw), dim3(kTB), 0, s, n, b.inv_count, h, gh, w_copy(0, C));
        GCN_LAUNCH_CHECK("prep_kernel");
    }
    // the piece's columns of W_pred, rows of ldw elements: in place, or copied to
    // whole 64 x 64 pieces
    const uint16_t *Wp = nullptr;
    int64_t ldw = 0;
    auto weights = [&](int32_t c0, int32_t P) -> int {
        if (p.in_place && P % 64 == 0) {
            Wp = W + c0;
            ldw = C;
            return GCN_OK;
        }
        ldw = up(P, 64);
        Wp = b.W;
        if (copied) return GCN_OK;
        ProfScope prof(K_CLASS_PREP, s, 0.0, 4.0 * f * P);
        hipLaunchKernelGGL(copy_rows_kernel<uint16_t>, dim3(grid_of(p.fp * ldw / 8)), dim3(kTB), 0, s, w_copy(c0, P));
        GCN_LAUNCH_CHECK("copy_rows_kernel");
        return GCN_OK;
    };
    auto logits = [&](int32_t c0, int32_t P) {
        TileProduct t{};
        t.A = (const uint8_t *)b.H;
        t.lda = 2 * p.fp;
        t.B = (const uint8_t *)Wp;
        t.ldb = 2 * ldw;
        t.M = n;
        t.N = P;
        t.kt = (int32_t)(p.fp / 64);
        t.splits = 1;
        t.bias = bias ? bias + c0 : nullptr;
        t.labels = labels;
        t.class0 = c0;
        t.classes = C;
        return t;
    };
    int32_t tiles = 0;   // left to the loss's workgroup
    for (int32_t i = 0; i < p.pieces; ++i) {
        const int32_t c0 = i * p.piece, P = std::min(p.piece, C - c0);
        if ((rc = weights(c0, P))) return rc;
        TileProduct t = logits(c0, P);
        t.tile_max = b.tile_max;
        t.tile_sum = b.tile_sum;
        t.label_logit = b.label_logit;
        {
            ProfScope prof(K_CLASS_STATS, s, 2.0 * n * f * P, 2.0 * ((double)n + P) * f);
            if ((rc = tile_product(TILE_BF16_NN, TILE_STATS, t, s))) return rc;
        }
        const TileShape sh = tile_shape(TILE_BF16_NN, t);
        tiles = (P + sh.n - 1) / sh.n;
        // (up to 16 tiles of 1024 rows the loss's workgroup joins in no more time)
        if (p.pieces == 1 && n <= 1024 && tiles <= 16) break;
        ProfScope prof(K_CLASS_PREP, s, 0.0, 8.0 * n * tiles);
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)((n + 31) / 32)), dim3(kTB), 0, s, n, tiles,
                           b.tile_max, b.tile_sum, b.run_max, b.run_sum, i == 0);
        tiles = 0;
        GCN_LAUNCH_CHECK("join_kernel");
    }
    hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, s, n, C, labels, tiles, b.tile_max, b.tile_sum, b.run_max,
                       b.run_sum, b.label_logit, b.lse,
                       row_loss, b.inv_count, loss);
    GCN_LAUNCH_CHECK("loss_kernel");
    if (!dHL) return GCN_OK;
    for (int32_t i = 0; i < p.pieces; ++i) {
        const int32_t c0 = i * p.piece, P = std::min(p.piece, C - c0);
        const int64_t pp = up(P, 64);
        if ((rc = weights(c0, P))) return rc;
        TileProduct t = logits(c0, P);
        t.lse = b.lse;
        t.scale = b.inv_count;
        t.G = b.G;
        t.ldg = pp;
        t.g_rows = p.np;
        const int32_t row_tiles = tile_rows(tile_shape(TILE_BF16_NN, t), TILE_STATS, t);   // (those with real rows)
        t.colpart = row_tiles == 1 ? db + c0 : b.colpart;   // (one row of tiles: the sums themselves)
        {
            ProfScope prof(K_CLASS_GRAD, s, 2.0 * n * f * P, 2.0 * ((double)n + P) * f + 4.0 * n * P);
            if ((rc = tile_product(TILE_BF16_NN, TILE_GRAD, t, s))) return rc;
        }
        if (row_tiles > 1 && (rc = colsum_reduce_rows(row_tiles, P, b.colpart, db + c0, s))) return rc;
        ProfScope prof(K_CLASS_PRODUCT, s, 4.0 * n * f * P, 4.0 * n * P);
        TileProduct h{};
        h.A = (const uint8_t *)b.G;
        h.lda = 2 * pp;
        h.B = (const uint8_t *)Wp;
        h.ldb = 2 * ldw;
        h.M = n;
        h.N = f;
        h.kt = (int32_t)(pp / 64);
        h.splits = p.split_h;
        h.acc = b.acc;
        h.accumulate = i > 0;
        TileProduct w{};
        w.A = (const uint8_t *)b.H;
        w.lda = 2 * p.fp;
        w.B = (const uint8_t *)b.G;
        w.ldb = 2 * pp;
        w.M = f;
        w.N = P;
        w.kt = (int32_t)(p.np / 64);
        w.splits = p.split_w;
        if (p.split_w > 1) {
            w.acc = b.part;
        } else {
            w.C = dW + c0;
            w.ldc = C;
            w.scale = b.inv_count;
        }
        if ((rc = tile_products(h, w, p.split_w > 1 ? TILE_PARTIAL : TILE_STORE, s))) return rc;
        if (p.split_w > 1 &&
            (rc = tile_reduce(p.split_w, f, P, b.part, dW + c0, 1, C, s, 0, 0, nullptr, nullptr, b.inv_count)))
            return rc;
    }
    return tile_reduce(p.split_h, n, f, b.acc, dHL, 1, lddhl, s, 0, 0, nullptr, nullptr, b.inv_count);
}

int loss_f32(const Plan &p, const Buffers &b, const float *HL, int32_t n, int32_t f, int64_t ldhl, const float *W,
             const float *bias, int32_t C, const int32_t *labels, float *loss, float *row_loss, float *dHL, int64_t lddhl,
             float *dW, float *db, hipStream_t s) {
    int rc;
    const CopyRows<float> h{n, n, f, HL, ldhl, b.Hz, f, labels, C};
    const unsigned gh = grid_of((int64_t)n * f / 4, 4096);
    hipLaunchKernelGGL(prep_kernel<float>, dim3(1 + gh), dim3(kTB), 0, s, n, b.inv_count, h, gh, h);
    GCN_LAUNCH_CHECK("class_prep");
    auto logits = [&](int32_t c0, int32_t P) {
        GemmProblem g{};
        g.M = n;
        g.N = P;
        g.C = b.X;
        g.ldc = up(P, 4);
        g.bias = bias ? bias + c0 : nullptr;
        g.seg[0] = GemmSeg{b.Hz, f, W + c0, C, f};
        return gemm(L_NN, 1, &g, 0, 1, nullptr, 0, s);
    };
    for (int32_t i = 0; i < p.pieces; ++i) {
        const int32_t c0 = i * p.piece, P = std::min(p.piece, C - c0);
        if ((rc = logits(c0, P))) return rc;
        ProfScope prof(K_CLASS_STATS, s, 0.0, 4.0 * n * P);
        hipLaunchKernelGGL(stats_rows_kernel, dim3((unsigned)std::min(n, 1 << 20)), dim3(kTB), 0, s, n, P, b.X, up(P, 4), labels, c0, C,
                           b.run_max, b.run_sum, b.label_logit, i == 0);
        GCN_LAUNCH_CHECK("stats_rows_kernel");
    }
    hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, s, n, C, labels, 0, b.tile_max, b.tile_sum, b.run_max,
                       b.run_sum, b.label_logit, b.lse,
                       row_loss, b.inv_count, loss);
    GCN_LAUNCH_CHECK("loss_kernel");
    if (!dHL) return GCN_OK;
    for (int32_t i = 0; i < p.pieces; ++i) {
        const int32_t c0 = i * p.piece, P = std::min(p.piece, C - c0);
        const int64_t ldx = up(P, 4);
        // (a single piece's logits are still in place)
        if (p.pieces > 1 && (rc = logits(c0, P))) return rc;
        {
            ProfScope prof(K_CLASS_GRAD, s, 0.0, 8.0 * n * P);
            const dim3 g((unsigned)((P + kTB - 1) / kTB), (unsigned)std::min(65535, (n + kStrip - 1) / kStrip));
            hipLaunchKernelGGL(grad_rows_kernel, g, dim3(kTB), 0, s, n, P, b.X, ldx, labels, c0, C, b.lse, b.inv_count,
                               b.colpart);
            GCN_LAUNCH_CHECK("grad_rows_kernel");
        }
        if ((rc = colsum_reduce_rows((n + kStrip - 1) / kStrip, P, b.colpart, db + c0, s))) return rc;
        GemmProblem w = dw_f32(f, P, n);
        w.C = dW + c0;
        w.ldc = C;
        w.seg[0] = GemmSeg{b.Hz, f, b.X, ldx, n};
        if ((rc = gemm(L_TN, 1, &w, 0, dw_split_f32(w), b.gemm_ws, b.gemm_bytes, s))) return rc;
        GemmProblem d = dh_f32(n, f, P);
        d.C = i ? b.tmp : dHL;
        d.ldc = i ? f : lddhl;
        d.seg[0] = GemmSeg{b.X, ldx, W + c0, C, P};
        if ((rc = gemm(L_NT, 1, &d, 0, gemm_pick_split(1, &d, false), b.gemm_ws, b.gemm_bytes, s))) return rc;
        if (i) {
            hipLaunchKernelGGL(add_kernel, dim3(grid_of((int64_t)n * f)), dim3(kTB), 0, s, n, f, b.tmp, dHL, lddhl);
            GCN_LAUNCH_CHECK("add_kernel");
        }
    }
    return GCN_OK;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" {

size_t gcn_class_loss_workspace_bytes(int32_t n, int32_t f, int32_t C, gcn_rows_type type, int need_grad) {
    if (n < 0 || f <= 0 || C <= 0 || std::max({n, f, C}) > kMostRows) return 0;
    Buffers b;
    return plan_of(n, f, C, type == GCN_ROWS_BF16, need_grad != 0, nullptr, nullptr, 0, b).total;
}

int gcn_class_loss(const void *HL, int32_t n, int32_t f, int32_t ldhl, const void *W_pred, const float *b_pred,
                   int32_t C, const int32_t *labels, gcn_rows_type type, float *loss, float *row_loss, void *dHL,
                   int32_t lddhl, void *dW_pred, float *db_pred, void *ws, size_t ws_bytes, void *stream) {
    GCN_REQUIRE(n >= 0 && f > 0 && C > 0, GCN_ESHAPE, "gcn_class_loss: n=%d f=%d C=%d", n, f, C);
    GCN_REQUIRE(type == GCN_ROWS_F32 || type == GCN_ROWS_BF16, GCN_EINVAL, "gcn_class_loss: bad element type %d",
                (int)type);
    GCN_REQUIRE(n <= kMostRows && f <= kMostRows && C <= kMostRows, GCN_EUNSUPPORTED, "gcn_class_loss: n=%d f=%d C=%d", n, f, C);
    const bool grad = dW_pred != nullptr, bf = type == GCN_ROWS_BF16;
    GCN_REQUIRE((db_pred != nullptr) == grad && (dHL != nullptr || (grad && n == 0) || !grad) && (grad || !dHL), GCN_EINVAL,
                "gcn_class_loss: dHL, dW_pred and db_pred are given together or not at all");
    GCN_REQUIRE(ldhl >= f && (!grad || lddhl >= f), GCN_ESHAPE, "gcn_class_loss: ldhl=%d lddhl=%d < f=%d", ldhl, lddhl, f);
    GCN_REQUIRE(W_pred && loss, GCN_EINVAL, "gcn_class_loss: null pointer");
    GCN_REQUIRE(n == 0 || (HL && labels), GCN_EINVAL, "gcn_class_loss: null HL or labels");
    const uintptr_t el = bf ? 1 : 3;
    GCN_REQUIRE((((uintptr_t)HL | (uintptr_t)W_pred | (uintptr_t)dHL | (uintptr_t)dW_pred) & el) == 0, GCN_EINVAL,
                "gcn_class_loss: misaligned operand");
    Buffers b;
    const Plan p = plan_of(n, f, C, bf, grad, W_pred, ws, ws_bytes, b);
    GCN_REQUIRE(ws && ((uintptr_t)ws & 255) == 0 && ws_bytes >= p.total, GCN_EWORKSPACE,
                "gcn_class_loss: workspace %zu < %zu bytes, or not 256-byte aligned", ws_bytes, p.total);
    hipStream_t s = (hipStream_t)stream;
    if (n == 0) {
        int rc = fill_zero(loss, 1, s);
        if (!rc && grad) rc = fill_zero(db_pred, C, s);
        if (!rc && grad) {
            if (bf) {
                hipLaunchKernelGGL(zero_kernel, dim3(grid_of((int64_t)f * C)), dim3(kTB), 0, s, (uint16_t *)dW_pred,
                                   (int64_t)f, (int64_t)C, (int64_t)C);
                GCN_LAUNCH_CHECK("zero_kernel");
            } else {
                rc = fill_zero((float *)dW_pred, (int64_t)f * C, s);
            }
        }
        return rc;
    }
    if (bf)
        return loss_bf16(p, b, (const uint16_t *)HL, n, f, ldhl, (const uint16_t *)W_pred, b_pred, C, labels, loss,
                         row_loss, (uint16_t *)dHL, lddhl, (uint16_t *)dW_pred, db_pred, s);
    return loss_f32(p, b, (const float *)HL, n, f, ldhl, (const float *)W_pred, b_pred, C, labels, loss, row_loss,
                    (float *)dHL, lddhl, (float *)dW_pred, db_pred, s);
}

}  // extern "C"
