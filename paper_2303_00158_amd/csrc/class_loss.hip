// Softmax cross-entropy of the logits Z = A Wt^T + b of many classes, with its
// gradients, in pieces of the classes, without keeping Z:
//   lse_i = log sum_c exp z_ic,  row loss = lse_i - z_iy,
//   dZ = s (exp(z - lse) - onehot(y)),  dWt = dZ^T A,  db = sum_i dZ,  dA = dZ Wt.
//
// Bound by the matrix products: 2 b K C operations for the loss, 6 b K C with the
// gradients, and 2 b K C more where there is more than one piece, whose logits are then
// computed twice, once for the rows' sums and once for dZ.  Only one piece of
// Z and dZ exists at a time, so memory goes by b, not by b C.
#include "class_loss.h"
#include "gemm_engine.h"
#include "loss_dev.h"
#include "row_dev.h"

namespace gnn {

namespace {

using namespace closs;

constexpr int kThreads = 256;

unsigned grid_of(int64_t n) {
    return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, int64_t(kThreads)), 16384)));
}

// ---------------------------------------------------------------------------
// rows: labels and weights, operands in the products' type
// ---------------------------------------------------------------------------
struct RowState {
    int32_t *label;   // -1: the row takes no part
    float *weight;    // 0 then
    float *top, *sum; // of the pieces so far: largest logit, sum of exp(z - top)
    float *z_label;
    float *lse;
};

__global__ void __launch_bounds__(kThreads) class_rows_kernel(CeArgs a, RowState r) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= a.b) return;
    const int64_t y = a.labels[a.targets ? a.targets[i] : i];
    const float w = a.row_scale ? a.row_scale[i] : 1.f / static_cast<float>(a.b);
    const bool live = y >= 0 && y < a.c && w != 0.f;
    r.label[i] = live ? static_cast<int32_t>(y) : -1;
    r.weight[i] = live ? w : 0.f;
    r.top[i] = -INFINITY;
    r.sum[i] = 0.f;
    r.z_label[i] = 0.f;
}

// rows of K values to rows of ld, zeros behind them; rows that take no part (label < 0) are
// zeros: dWt multiplies them by 0, which a NaN there would survive.
template <class TI, class TO>
__global__ void __launch_bounds__(kThreads) class_pack_kernel(const TI *in, int64_t rows, int64_t K, int64_t ld, const int32_t *label,
                                                              TO *out) {
    const int64_t groups = ld / 4;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; t < rows * groups;
         t += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t r = t / groups, c = (t - r * groups) * 4;
        row::Vec<TI, 4> v;
        v.load_upto(in + r * K + c, label && label[r] < 0 ? 0 : K - c);
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = v.get(e);
        row::Vec<TO, 4> o;
        o.set(x);
        o.store(out + r * ld + c);
    }
}

gnn_status pack(const void *in, int idt, int64_t rows, int64_t K, int64_t ld, const int32_t *label, void *out, int odt, hipStream_t s) {
    const unsigned grid = grid_of(rows * (ld / 4));
    if (idt == GNN_BF16) {
        const uint16_t *x = static_cast<const uint16_t *>(in);
        if (odt == GNN_BF16) class_pack_kernel<<<grid, kThreads, 0, s>>>(x, rows, K, ld, label, static_cast<uint16_t *>(out));
        else class_pack_kernel<<<grid, kThreads, 0, s>>>(x, rows, K, ld, label, static_cast<float *>(out));
    } else {
        const float *x = static_cast<const float *>(in);
        if (odt == GNN_BF16) class_pack_kernel<<<grid, kThreads, 0, s>>>(x, rows, K, ld, label, static_cast<uint16_t *>(out));
        else class_pack_kernel<<<grid, kThreads, 0, s>>>(x, rows, K, ld, label, static_cast<float *>(out));
    }
    GNN_LAUNCHED("update_ce_pack");
    return GNN_OK;
}

// ---------------------------------------------------------------------------
// a piece of the logits
// ---------------------------------------------------------------------------
// T threads to a row: the piece's largest logit and its sum join the row's.
template <int T> __global__ void __launch_bounds__(kThreads) class_sums_kernel(const float *z, int64_t b, int64_t cols, int64_t ld, int64_t c0,
                                                                              const float *bias, RowState r) {
    constexpr int kRows = kThreads / T;
    __shared__ float sh[2][kThreads / 64];
    const int lane = threadIdx.x % T;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / T;
    if (i >= b) return;  // T = 256: the whole workgroup
    const float *zi = z + i * ld;
    float top = -INFINITY;
    for (int64_t c = lane; c < cols; c += T) top = fmaxf(top, zi[c] + (bias ? bias[c0 + c] : 0.f));
    top = loss::wave_max(top);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) sh[0][threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < T / 64; ++w) top = fmaxf(top, sh[0][w]);
    }
    const float old = r.top[i], now = fmaxf(old, top), from = now == -INFINITY ? 0.f : now;
    float sum = 0.f;
    for (int64_t c = lane; c < cols; c += T) sum += expf(zi[c] + (bias ? bias[c0 + c] : 0.f) - from);
    sum = loss::wave_sum(sum);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) sh[1][threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) sum += sh[1][w];
    }
    if (lane != 0) return;
    const float before = r.sum[i];
    r.sum[i] = (old == now || before == 0.f ? before : before * expf(old - from)) + sum;
    r.top[i] = now;
    const int64_t y = r.label[i] - c0;
    if (r.label[i] >= 0 && y >= 0 && y < cols) r.z_label[i] = zi[y] + (bias ? bias[c0 + y] : 0.f);
}

__global__ void __launch_bounds__(kThreads) class_loss_kernel(CeArgs a, RowState r, float *row_loss) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= a.b) return;
    const float lse = r.top[i] + logf(r.sum[i]);
    r.lse[i] = lse;
    row_loss[i] = r.label[i] < 0 ? 0.f : lse - r.z_label[i];
}

// The weighted sum of the rows' losses, in a fixed order.
__global__ void __launch_bounds__(1024) class_total_kernel(const float *row_loss, const float *weight, int64_t b, float *loss) {
    __shared__ float sh[16];
    float s = 0.f;
    for (int64_t i = threadIdx.x; i < b; i += 1024)
        if (weight[i] != 0.f) s += row_loss[i] * weight[i];
    s = loss::wave_sum(s);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) t += sh[w];
    *loss = t;
}

// dZ of a piece from its logits (in place where it is fp32), zeros in the columns up to ld,
// and the column sums of a part of the rows.
constexpr int kStripe = 256;  // columns of a workgroup: 64 threads of 4, times 4 rows
template <class T>
__global__ void __launch_bounds__(kThreads) class_dz_kernel(const float *z, int64_t ldz, T *dz, int64_t ld, int64_t b, int64_t cols, int64_t c0,
                                                            const float *bias, RowState r, float *part, int64_t parts) {
    __shared__ float sh[4][kStripe];
    const int64_t stripes = ceil_div(ld, int64_t(kStripe)), stripe = blockIdx.x % stripes, p = blockIdx.x / stripes;
    const int64_t per = ceil_div(b, parts), beg = min(b, p * per), end = min(b, beg + per);
    const int x = (threadIdx.x & 63) * 4, y = threadIdx.x >> 6;
    const int64_t c = stripe * kStripe + x;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < ld) {
        float bs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) bs[e] = bias && c + e < cols ? bias[c0 + c + e] : 0.f;
        for (int64_t i = beg + y; i < end; i += 4) {
            const float w = r.weight[i], lse = r.lse[i];
            const int64_t label = r.label[i] - c0;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (w != 0.f) {
                const float4 zz = *reinterpret_cast<const float4 *>(z + i * ldz + c);
                v[0] = zz.x;
                v[1] = zz.y;
                v[2] = zz.z;
                v[3] = zz.w;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = c + e < cols ? w * (expf(v[e] + bs[e] - lse) - (c + e == label ? 1.f : 0.f)) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += v[e];
            row::Vec<T, 4> o;
            o.set(v);
            o.store(dz + i * ld + c);
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) sh[y][x + e] = sum[e];
    __syncthreads();
    const int64_t col = stripe * kStripe + threadIdx.x;
    if (col >= cols) return;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) t += sh[k][threadIdx.x];
    part[p * cols + col] = t;
}

__global__ void __launch_bounds__(kThreads) class_db_kernel(const float *part, int64_t parts, int64_t cols, float *db) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (c >= cols) return;
    float t = 0.f;
#pragma unroll 8
    for (int64_t p = 0; p < parts; ++p) t += part[p * cols + c];
    db[c] = t;
}

// out = the partials in their order; rows of `ld` to rows of `cols`
template <class T>
__global__ void __launch_bounds__(kThreads) class_reduce_kernel(const float *part, int64_t nsplit, int64_t rows, int64_t cols, int64_t ld, T *out) {
    const int64_t groups = ld / 4;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; t < rows * groups;
         t += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t r = t / groups, c = (t - r * groups) * 4;
        const float4 v = gemm::sum_splits(part + r * ld + c, rows * ld, static_cast<int>(nsplit));
        const float x[4] = {v.x, v.y, v.z, v.w};
        row::Vec<T, 4> o;
        o.set(x);
        o.store_upto(out + r * cols + c, cols - c);
    }
}
gnn_status reduce(const float *part, int64_t nsplit, int64_t rows, int64_t cols, int64_t ld, void *out, int odt, hipStream_t s) {
    const unsigned grid = grid_of(rows * (ld / 4));
    if (odt == GNN_BF16) class_reduce_kernel<<<grid, kThreads, 0, s>>>(part, nsplit, rows, cols, ld, static_cast<uint16_t *>(out));
    else class_reduce_kernel<<<grid, kThreads, 0, s>>>(part, nsplit, rows, cols, ld, static_cast<float *>(out));
    GNN_LAUNCHED("update_ce_reduce");
    return GNN_OK;
}

// ---------------------------------------------------------------------------
// the call's buffers
// ---------------------------------------------------------------------------
constexpr int64_t kPiece = 1 << 27;  // logits of a piece, about
constexpr int64_t kPieceCols = 256;  // its columns: a multiple of these

int64_t row_of(int64_t n) { return (n + 7) / 8 * 8; }

struct Plan {
    bool bf;
    int64_t ldk, piece, pieces, parts;
    int64_t da_splits, dw_splits_of[2];  // of a full piece and of the last one
    size_t label, weight, top, sum, z_label, lse, row_loss, a, w, z, dz, db, dw_part, da_part, total;
    Plan(int64_t b, int64_t k, int64_t c, int gemm_dt, bool grads) {
        bf = gemm_dt == GNN_BF16;
        ldk = row_of(k);
        const int64_t all = static_cast<int64_t>(round_up(static_cast<size_t>(c), kPieceCols));
        piece = std::min(all, std::max<int64_t>(kPiece / std::max<int64_t>(b, 1) / kPieceCols * kPieceCols, kPieceCols));
        pieces = ceil_div(c, piece);
        const size_t es = bf ? 2 : 4;
        const int64_t width = std::min(piece, row_of(c));
        parts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(2048, ceil_div(width, int64_t(kStripe))), ceil_div(b, int64_t(16))));
        auto splits = [&](Kind kind, int64_t m, int64_t n, int64_t r) {
            return bf ? splits_bf16(kind, m, n, r, true) : splits_f32(kind, m, n, r, true);
        };
        Carver cv(nullptr);
        auto rows = [&]() { return cv.take(static_cast<size_t>(b) * 4); };
        label = rows();
        weight = rows();
        top = rows();
        sum = rows();
        z_label = rows();
        lse = rows();
        row_loss = rows();
        a = cv.take(static_cast<size_t>(b * ldk) * es);
        w = cv.take(static_cast<size_t>(width * ldk) * es);
        z = cv.take(static_cast<size_t>(b * width) * 4);
        dz = db = dw_part = da_part = 0;
        da_splits = dw_splits_of[0] = dw_splits_of[1] = 1;
        if (grads) {
            const int64_t last = row_of(c - (pieces - 1) * piece);
            da_splits = splits(kNT, b, k, width);
            dw_splits_of[0] = splits(kTT, width, k, b);
            dw_splits_of[1] = splits(kTT, last, k, b);
            dz = bf ? cv.take(static_cast<size_t>(b * width) * 2) : z;
            db = cv.take(static_cast<size_t>(parts * width) * 4);
            const int64_t dw = std::max(dw_splits_of[0] > 1 ? dw_splits_of[0] * width : 0, dw_splits_of[1] > 1 ? dw_splits_of[1] * last : 0);
            dw_part = cv.take(static_cast<size_t>(dw * ldk) * 4);
            da_part = cv.take(da_splits > 1 || pieces > 1 ? static_cast<size_t>(da_splits * b * ldk) * 4 : 0);
        }
        total = round_up(cv.off, 256);
    }
};

}  // namespace

size_t update_ce_ws_bytes(int64_t b, int64_t k, int64_t c, int gemm_dt, bool grads) { return Plan(b, k, c, gemm_dt, grads).total; }

gnn_status launch_update_ce(const CeArgs &a, void *ws, hipStream_t s) {
    const bool grads = a.d_a || a.dwt || a.db;
    const Plan pl(a.b, a.k, a.c, a.gemm_dt, grads);
    char *base = static_cast<char *>(ws);
    const int gdt = a.gemm_dt;
    const size_t es = dtype_size(gdt);
    auto f = [&](size_t at) { return reinterpret_cast<float *>(base + at); };
    const RowState r{reinterpret_cast<int32_t *>(base + pl.label), f(pl.weight), f(pl.top), f(pl.sum), f(pl.z_label), f(pl.lse)};
    float *row_loss = a.row_loss ? a.row_loss : f(pl.row_loss);
    if (a.b > 0) {
        class_rows_kernel<<<static_cast<unsigned>(ceil_div(a.b, int64_t(kThreads))), kThreads, 0, s>>>(a, r);
        GNN_LAUNCHED("update_ce_rows");
    }
    const void *A = a.a;
    int64_t lda = a.k;
    const bool rows16 = a.k * static_cast<int64_t>(es) % 16 == 0;
    if (a.b > 0 && (a.dwt || a.adt != gdt || !rows16 || !aligned(a.a, 16))) {
        GNN_TRY(pack(a.a, a.adt, a.b, a.k, pl.ldk, r.label, base + pl.a, gdt, s));
        A = base + pl.a;
        lda = pl.ldk;
    }
    const bool copy_w = a.wdt != gdt || !rows16 || !aligned(a.wt, 16);
    float *z = f(pl.z);
    // the weights' rows [c0, c0 + cols) as the products read them
    auto weights = [&](int64_t c0, int64_t cols, const void **w, int64_t *ldw) -> gnn_status {
        const char *from = static_cast<const char *>(a.wt) + c0 * a.k * static_cast<int64_t>(dtype_size(a.wdt));
        *w = from;
        *ldw = a.k;
        if (!copy_w) return GNN_OK;
        *w = base + pl.w;
        *ldw = pl.ldk;
        return pack(from, a.wdt, cols, a.k, pl.ldk, nullptr, base + pl.w, gdt, s);
    };
    auto product = [&](Kind kind, const Product &p) { return gdt == GNN_BF16 ? product_bf16(kind, p, s) : product_f32(kind, p, s); };
    auto logits = [&](const void *w, int64_t ldw, int64_t cols) {
        const int64_t K = std::min(lda, ldw), ld = row_of(cols);
        return product(kNN, Product{A, w, lda, ldw, a.b, cols, K, K, z, GNN_F32, ld, 1, 0, false});
    };
    if (a.b > 0) {
        for (int64_t q = 0; q < pl.pieces; ++q) {
            const int64_t c0 = q * pl.piece, cols = std::min(pl.piece, a.c - c0), ld = row_of(cols);
            const void *w;
            int64_t ldw;
            GNN_TRY(weights(c0, cols, &w, &ldw));
            GNN_TRY(logits(w, ldw, cols));
            if (cols <= 1024) class_sums_kernel<64><<<static_cast<unsigned>(ceil_div(a.b, int64_t(4))), kThreads, 0, s>>>(z, a.b, cols, ld, c0, a.bias, r);
            else class_sums_kernel<256><<<static_cast<unsigned>(a.b), kThreads, 0, s>>>(z, a.b, cols, ld, c0, a.bias, r);
            GNN_LAUNCHED("update_ce_sums");
        }
        class_loss_kernel<<<static_cast<unsigned>(ceil_div(a.b, int64_t(kThreads))), kThreads, 0, s>>>(a, r, row_loss);
        GNN_LAUNCHED("update_ce_loss");
    }
    class_total_kernel<<<1, 1024, 0, s>>>(row_loss, r.weight, a.b, a.loss_out);
    GNN_LAUNCHED("update_ce_total");
    if (!grads) return GNN_OK;
    void *dz = base + pl.dz;
    for (int64_t q = 0; q < pl.pieces; ++q) {
        const int64_t c0 = q * pl.piece, cols = std::min(pl.piece, a.c - c0), ld = row_of(cols);
        const void *w;
        int64_t ldw;
        if (pl.pieces > 1 || a.d_a) GNN_TRY(weights(c0, cols, &w, &ldw));
        if (a.b > 0) {
            if (pl.pieces > 1) GNN_TRY(logits(w, ldw, cols));
            const unsigned grid = static_cast<unsigned>(ceil_div(ld, int64_t(kStripe)) * pl.parts);
            float *part = a.db ? f(pl.db) : nullptr;
            if (pl.bf) class_dz_kernel<<<grid, kThreads, 0, s>>>(z, ld, static_cast<uint16_t *>(dz), ld, a.b, cols, c0, a.bias, r, part, pl.parts);
            else class_dz_kernel<<<grid, kThreads, 0, s>>>(z, ld, static_cast<float *>(dz), ld, a.b, cols, c0, a.bias, r, part, pl.parts);
            GNN_LAUNCHED("update_ce_dz");
        }
        if (a.db) {
            class_db_kernel<<<static_cast<unsigned>(ceil_div(cols, int64_t(kThreads))), kThreads, 0, s>>>(f(pl.db), a.b > 0 ? pl.parts : 0, cols, a.db + c0);
            GNN_LAUNCHED("update_ce_db");
        }
        if (a.dwt) {
            const int64_t n = q + 1 < pl.pieces ? pl.dw_splits_of[0] : pl.dw_splits_of[1];
            char *to = static_cast<char *>(a.dwt) + c0 * a.k * static_cast<int64_t>(dtype_size(a.dwdt));
            if (n == 1) {
                GNN_TRY(product(kTT, Product{dz, A, ld, lda, cols, a.k, a.b, a.b, to, a.dwdt, a.k, 1, 0, false}));
            } else {
                GNN_TRY(product(kTT, Product{dz, A, ld, lda, cols, a.k, a.b, a.b, base + pl.dw_part, GNN_F32, pl.ldk, n, cols * pl.ldk, false}));
                GNN_TRY(reduce(f(pl.dw_part), n, cols, a.k, pl.ldk, to, a.dwdt, s));
            }
        }
        if (a.d_a && a.b > 0) {
            const bool whole = pl.pieces == 1 && pl.da_splits == 1;
            GNN_TRY(product(kNT, Product{dz, w, ld, ldw, a.b, a.k, ld, cols, whole ? a.d_a : base + pl.da_part, whole ? a.gdt : static_cast<int>(GNN_F32),
                                         whole ? a.k : pl.ldk, pl.da_splits, a.b * pl.ldk, q > 0}));
        }
    }
    if (a.d_a && a.b > 0 && (pl.pieces > 1 || pl.da_splits > 1))
        GNN_TRY(reduce(f(pl.da_part), pl.da_splits, a.b, a.k, pl.ldk, a.d_a, a.gdt, s));
    return GNN_OK;
}

}  // namespace gnn
