// PREDICT and softmax cross entropy over many classes in pieces of the
// classes, without keeping the logits (gcn_classes.h).
//
//   pass 1, per piece: logits of the piece in the product's registers; per row
//     and column tile their maximum and the sum of exponentials relative to
//     it, joined into the row's running maximum and sum
//   loss: row_loss = (max - label's logit) + log(sum).  max and log(sum) stay two
//     numbers, here and in G: where a row is sure of its label log(sum) is all of
//     its loss, and added to a max of 1000 it would be rounded to steps of 2^-14
//   pass 2, per piece: the logits again, n_l G = exp((x - max) - log(sum)) - onehot in the same
//     registers, written as bfloat16 rows; then n_l dHL += n_l G W_piece^T and
//     n_l dW_piece = HL^T n_l G.  1 / n_l is a factor of the float32 sums: in G it
//     would be rounded, and the same way in every row (17 rows: the gradients
//     0.0036 off in the 2-norm instead of 0.0018).
//
// float32 operands: pass 1 keeps the logits of a single piece where G will be,
// and pass 2 turns them into G (1 / n_l included, no rounding to fewer bits) by an
// elementwise pass; with several pieces it computes them again.  The products
// run at 87-113 TFLOP/s (peak 157) and are nine tenths of the time at 2000 x 256,
// 10,007 classes (349 us; 17 x 128, 1009 classes: 36 us of launches).  bfloat16:
// 16,384 x 1024, 131,072 classes 15.4 ms, four products of 1080-1330 TFLOP/s.
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

// X <- G (float32), and the column sums of strips of kStrip rows: a thread has a
// column.  Zeros in the columns past P and the rows past n, which the products read.
constexpr int kStrip = 32;
__global__ __launch_bounds__(kTB) void grad_rows_kernel(int32_t n, int32_t P, float *X, int64_t ldx,
                                                        const int32_t *labels, int32_t class0, int32_t C,
                                                        const float *row_max, const float *log_sum,
                                                        const float *inv_count, float *part) {
    __shared__ float top[kStrip], ls[kStrip];
    __shared__ int32_t lab[kStrip];
    const int64_t c = (int64_t)blockIdx.x * kTB + threadIdx.x;
    const int32_t strips = (n + kStrip - 1) / kStrip;
    const float inv = inv_count[0];
    for (int32_t strip = blockIdx.y; strip < strips; strip += gridDim.y) {
        const int64_t r0 = (int64_t)strip * kStrip;
        __syncthreads();
        if (threadIdx.x < kStrip) {
            const int64_t row = r0 + threadIdx.x;
            const int32_t l = row < n ? labels[row] : -1;
            top[threadIdx.x] = row < n ? row_max[row] : 0.0f;
            ls[threadIdx.x] = row < n ? log_sum[row] : 0.0f;
            lab[threadIdx.x] = has_label(l, C) ? l : -1;
        }
        __syncthreads();
        if (c >= ldx) continue;
        float sum = 0.0f;
        float *x = X + r0 * ldx + c;
        // (eight loads before the first store, behind which the next one would wait)
        for (int32_t r = 0; r < kStrip; r += 8, x += 8 * ldx) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = lab[r + e] >= 0 && c < P ? x[e * ldx] : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int32_t l = lab[r + e];
                const float g = l >= 0 && c < P ? (expf((v[e] - top[r + e]) - ls[r + e]) - (class0 + c == l ? 1.0f : 0.0f)) * inv : 0.0f;
                x[e * ldx] = g;
                sum += g;
            }
        }
        if (c < P) part[(int64_t)strip * P + c] = sum;
    }
}

// The sums' logarithms, the rows' losses and their mean, by one workgroup in a fixed
// order.  tiles > 0: the only piece's tiles are joined here (few rows and tiles).
__global__ __launch_bounds__(1024) void loss_kernel(int32_t n, int32_t C, const int32_t *__restrict__ labels,
                                                    int32_t tiles, const float *__restrict__ tile_max,
                                                    const float *__restrict__ tile_sum, float *__restrict__ run_max,
                                                    const float *__restrict__ run_sum,
                                                    const float *__restrict__ label_logit, float *__restrict__ log_sum,
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
            run_max[i] = m;
        } else {
            m = run_max[i], s = run_sum[i];
        }
        const float ls = logf(s);
        log_sum[i] = ls;
        const bool has = has_label(labels[i], C);
        const float v = has ? (m - label_logit[i]) + ls : 0.0f;
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

__global__ __launch_bounds__(kTB) void zero_kernel(uint16_t *x, int64_t rows, int64_t cols, int64_t ld) {
    for (int64_t i = (int64_t)blockIdx.x * kTB + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * kTB)
        x[i / cols * ld + i % cols] = 0;
}

unsigned grid_of(int64_t work, int64_t most = 8192) {
    return (unsigned)std::max<int64_t>(1, std::min(most, (work + kTB - 1) / kTB));
}
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// How a call is cut and what of the workspace it uses.  T: the elements' type.
struct Plan {
    int32_t unit;              // elements of a 128-byte piece
    int64_t fp, np;            // f and n in whole units
    int32_t piece, pieces;     // classes per piece
    int32_t split_h, split_w;  // parts of the two gradient products
    bool in_place;             // W_pred's own rows serve as operands
    size_t total;
};
template <class T>
struct Buffers {
    float *inv_count, *run_max, *run_sum, *label_logit, *log_sum, *tile_max, *tile_sum, *colpart, *acc, *part;
    T *H, *W, *G;              // (float32: G holds the logits first)
};

// The elements of a piece: 512 MB of bfloat16 gradient rows, or of float32 logits.
constexpr int64_t kPieceElems = (int64_t)1 << 28, kPieceElemsF32 = (int64_t)1 << 27;

// W: the weights, or null in the workspace query, which counts on copying them.
template <class T>
Plan plan_of(int32_t n, int32_t f, int32_t C, bool grad, const void *W, void *ws, size_t ws_bytes, Buffers<T> &b) {
    constexpr bool bf = sizeof(T) == 2;
    Plan p{};
    Arena ar(ws, ws_bytes);
    const int64_t rows = std::max(n, 1), u = 128 / sizeof(T);
    p.unit = (int32_t)u;
    p.fp = up(f, u);
    p.np = up(rows, u);
    p.in_place = W && (uintptr_t)W % 16 == 0 && C % (16 / sizeof(T)) == 0 && f % u == 0;
    int64_t piece = std::max<int64_t>(256, (bf ? kPieceElems : kPieceElemsF32) / p.np / 256 * 256);
    piece = std::min<int64_t>(piece, up(C, 256));
    p.pieces = (int32_t)((C + piece - 1) / piece);
    p.piece = (int32_t)std::min<int64_t>(piece, C);
    b = Buffers<T>{};
    b.inv_count = ar.take<float>(1);
    b.run_max = ar.take<float>(rows);
    b.run_sum = ar.take<float>(rows);
    b.label_logit = ar.take<float>(rows);
    b.log_sum = ar.take<float>(rows);
    // (sized for the smallest tiles: a last, smaller piece may run on them)
    const int64_t tn = (p.piece + kSmallTile - 1) / kSmallTile;
    b.tile_max = ar.take<float>(tn * rows);
    b.tile_sum = ar.take<float>(tn * rows);
    b.H = ar.take<T>(p.np * p.fp);
    // (a piece of whole units is read in place where W_pred's rows are 16-byte
    // aligned and f is whole: only a ragged last piece is copied)
    const int32_t last = C - (p.pieces - 1) * p.piece;
    const int64_t copied = std::max(p.in_place && p.piece % u == 0 ? 0 : p.piece, p.in_place && last % u == 0 ? 0 : last);
    b.W = copied ? ar.take<T>(p.fp * up(copied, u)) : nullptr;
    if (grad) {
        const int64_t pp = up(p.piece, u);
        b.G = ar.take<T>(p.np * pp);
        b.colpart = ar.take<float>((p.np + kSmallRows - 1) / kSmallRows * p.piece);
        p.split_h = tile_splits(n, f, (int32_t)(pp / u), !bf);
        // (float32: parts of about 64 pieces fill the last round of the other product, in
        // the same launch)
        if (!bf) p.split_h = (int32_t)std::max<int64_t>(p.split_h, std::min<int64_t>(64, pp / u / 64));
        p.split_w = tile_splits(f, p.piece, (int32_t)(p.np / u), !bf);
        b.acc = ar.take<float>((size_t)p.split_h * rows * f);
        if (p.split_w > 1) b.part = ar.take<float>((size_t)p.split_w * f * p.piece);
    }
    p.total = ar.used + 256;
    return p;
}

template <class T>
int class_loss(const Plan &p, const Buffers<T> &b, const T *HL, int32_t n, int32_t f, int64_t ldhl, const T *W,
               const float *bias, int32_t C, const int32_t *labels, float *loss, float *row_loss, T *dHL, int64_t lddhl,
               T *dW, float *db, hipStream_t s) {
    constexpr bool bf = sizeof(T) == 2;
    constexpr TileType kNN = bf ? TILE_BF16_NN : TILE_F32_NN;
    constexpr int64_t E = sizeof(T), U = 128 / E, V = 16 / E;
    int rc;
    // (a single copied piece of W_pred goes along)
    auto w_copy = [&](int32_t c0, int32_t P) {
        return CopyRows<T>{(int32_t)p.fp, f, P, W + c0, C, b.W, up(P, U), nullptr, 0};
    };
    const bool copied = p.pieces == 1 && !(p.in_place && C % U == 0);
    {
        ProfScope prof(K_CLASS_PREP, s, 0.0, 2.0 * E * n * f);
        const CopyRows<T> h{(int32_t)p.np, n, f, HL, ldhl, b.H, p.fp, labels, C};
        const unsigned gh = grid_of(p.np * p.fp / V, 4096), gw = copied ? grid_of(p.fp * up(C, U) / V, 4096) : 0;
        hipLaunchKernelGGL(prep_kernel<T>, dim3(1 + gh + gw), dim3(kTB), 0, s, n, b.inv_count, h, gh, w_copy(0, C));
        GCN_LAUNCH_CHECK("prep_kernel");
    }
    // the piece's columns of W_pred, rows of ldw elements: in place, or copied to
    // whole pieces
    const T *Wp = nullptr;
    int64_t ldw = 0;
    auto weights = [&](int32_t c0, int32_t P) -> int {
        if (p.in_place && P % U == 0) {
            Wp = W + c0;
            ldw = C;
            return GCN_OK;
        }
        ldw = up(P, U);
        Wp = b.W;
        if (copied) return GCN_OK;
        ProfScope prof(K_CLASS_PREP, s, 0.0, 2.0 * E * f * P);
        hipLaunchKernelGGL(copy_rows_kernel<T>, dim3(grid_of(p.fp * ldw / V)), dim3(kTB), 0, s, w_copy(c0, P));
        GCN_LAUNCH_CHECK("copy_rows_kernel");
        return GCN_OK;
    };
    auto logits = [&](int32_t c0, int32_t P) {
        TileProduct t{};
        t.A = (const uint8_t *)b.H;
        t.lda = E * p.fp;
        t.B = (const uint8_t *)Wp;
        t.ldb = E * ldw;
        t.M = n;
        t.N = P;
        t.kt = (int32_t)(p.fp / U);
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
        const bool keep = !bf && p.pieces == 1 && dHL;   // (float32 logits of a single piece stay where G will be)
        t.C = b.G;
        t.ldc = up(P, U);
        {
            ProfScope prof(K_CLASS_STATS, s, 2.0 * n * f * P, E * ((double)n + P) * f + (keep ? 4.0 * n * P : 0.0));
            if constexpr (bf) rc = tile_product(kNN, TILE_STATS, t, s);
            else rc = tile_product(kNN, keep ? TILE_STATS_STORE : TILE_STATS, t, s);
            if (rc) return rc;
        }
        const TileShape sh = tile_shape(kNN, t);
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
                       b.run_sum, b.label_logit, b.log_sum, row_loss, b.inv_count, loss);
    GCN_LAUNCH_CHECK("loss_kernel");
    if (!dHL) return GCN_OK;
    const float *const factor = bf ? b.inv_count : nullptr;   // (float32 G has it already)
    for (int32_t i = 0; i < p.pieces; ++i) {
        const int32_t c0 = i * p.piece, P = std::min(p.piece, C - c0);
        const int64_t pp = up(P, U);
        if ((rc = weights(c0, P))) return rc;
        TileProduct t = logits(c0, P);
        if constexpr (bf) {
            t.row_max = b.run_max;
            t.log_sum = b.log_sum;
            t.scale = b.inv_count;
            t.G = b.G;
            t.ldg = pp;
            t.g_rows = p.np;
            const int32_t row_tiles = tile_rows(tile_shape(kNN, t), TILE_STATS, t);   // (those with real rows)
            t.colpart = row_tiles == 1 ? db + c0 : b.colpart;   // (one row of tiles: the sums themselves)
            {
                ProfScope prof(K_CLASS_GRAD, s, 2.0 * n * f * P, E * ((double)n + P) * f + 4.0 * n * P);
                if ((rc = tile_product(kNN, TILE_GRAD, t, s))) return rc;
            }
            if (row_tiles > 1 && (rc = colsum_reduce_rows(row_tiles, P, b.colpart, db + c0, s))) return rc;
        } else {
            const int32_t strips = (n + kStrip - 1) / kStrip;
            {
                ProfScope prof(K_CLASS_GRAD, s, p.pieces > 1 ? 2.0 * n * f * P : 0.0, 8.0 * n * P);
                t.C = b.G;
                t.ldc = pp;
                if (p.pieces > 1 && (rc = tile_product(kNN, TILE_STORE_F32, t, s))) return rc;
                const dim3 g((unsigned)((pp + kTB - 1) / kTB), (unsigned)std::min(65535, strips));
                hipLaunchKernelGGL(grad_rows_kernel, g, dim3(kTB), 0, s, n, P, b.G, pp, labels, c0, C, b.run_max,
                                   b.log_sum, b.inv_count, strips == 1 ? db + c0 : b.colpart);
                GCN_LAUNCH_CHECK("grad_rows_kernel");
            }
            if (strips > 1 && (rc = colsum_reduce_rows(strips, P, b.colpart, db + c0, s))) return rc;
        }
        ProfScope prof(K_CLASS_PRODUCT, s, 4.0 * n * f * P, 4.0 * n * P);
        TileProduct h{};
        h.A = (const uint8_t *)b.G;
        h.lda = E * pp;
        h.B = (const uint8_t *)Wp;
        h.ldb = E * ldw;
        h.M = n;
        h.N = f;
        h.kt = (int32_t)(pp / U);
        h.splits = p.split_h;
        h.acc = b.acc;
        h.accumulate = i > 0;
        TileProduct w{};
        w.A = (const uint8_t *)b.H;
        w.lda = E * p.fp;
        w.B = (const uint8_t *)b.G;
        w.ldb = E * pp;
        w.M = f;
        w.N = P;
        w.kt = (int32_t)(p.np / U);
        w.splits = p.split_w;
        if (p.split_w > 1) {
            w.acc = b.part;
        } else {
            w.C = dW + c0;
            w.ldc = C;
            w.scale = factor;
        }
        if ((rc = tile_products(!bf, h, w, p.split_w > 1 ? TILE_PARTIAL : bf ? TILE_STORE : TILE_STORE_F32, s))) return rc;
        if (p.split_w > 1 &&
            (rc = tile_reduce(p.split_w, f, P, b.part, dW + c0, bf, C, s, 0, 0, nullptr, nullptr, factor)))
            return rc;
    }
    return tile_reduce(p.split_h, n, f, b.acc, dHL, bf, lddhl, s, 0, 0, nullptr, nullptr, factor);
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" {

size_t gcn_class_loss_workspace_bytes(int32_t n, int32_t f, int32_t C, gcn_rows_type type, int need_grad) {
    if (n < 0 || f <= 0 || C <= 0 || std::max({n, f, C}) > kMostRows) return 0;
    Buffers<uint16_t> b;
    Buffers<float> c;
    return type == GCN_ROWS_BF16 ? plan_of(n, f, C, need_grad != 0, nullptr, nullptr, 0, b).total
                                 : plan_of(n, f, C, need_grad != 0, nullptr, nullptr, 0, c).total;
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
    Buffers<uint16_t> b;
    Buffers<float> c;
    const Plan p = bf ? plan_of(n, f, C, grad, W_pred, ws, ws_bytes, b) : plan_of(n, f, C, grad, W_pred, ws, ws_bytes, c);
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
        return class_loss(p, b, (const uint16_t *)HL, n, f, ldhl, (const uint16_t *)W_pred, b_pred, C, labels, loss, row_loss,
                          (uint16_t *)dHL, lddhl, (uint16_t *)dW_pred, db_pred, s);
    return class_loss(p, c, (const float *)HL, n, f, ldhl, (const float *)W_pred, b_pred, C, labels, loss, row_loss,
                      (float *)dHL, lddhl, (float *)dW_pred, db_pred, s);
}

}  // extern "C"
