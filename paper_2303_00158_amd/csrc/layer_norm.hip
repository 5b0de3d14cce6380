// Layer normalisation of activation rows, forward and backward.
//
// Both directions are bound by memory: one read of every input and one write
// of every output.  A row is held in registers from its load to its last use
// by as many threads as give each of them 8 elements (a part of a wavefront, up
// to 512 columns, and 256 threads, to 2,048), 16 (a wavefront, to 1,024, and
// 256, 512 and 1,024 threads, to 16,384), 32 or 64 (1,024, to 65,536), so the two passes of the
// statistics (the mean, then the squares of the distances from it) and the
// output's cost no second read.  Threads take 16 bytes at a time, neighbours
// next to each other; rows of any alignment are read so too (the hardware
// takes 16-byte accesses at the element's alignment), only a row's last
// few elements one by one.
//
// The backward takes the sums of dgamma and dbeta on the same read: a thread
// keeps its columns' sums over all rows that its workgroup walks, and the
// workgroups' partial rows are added by a second kernel in their order.  Rows
// above 16,384 columns, whose sums do not fit the registers beside the row,
// read x and g once more for them, column stripe by column stripe.
#include "row_dev.h"

namespace gnn {

namespace {

using namespace row;

constexpr int64_t kCus = 256;

// A thread's copies of gamma (or 1) or beta (or 0).  Up to 8 (16 in the
// backward) stay in registers over all rows; more come from the caches where
// they are used and leave the registers to the rows.
template <class S, bool KEEP> struct Weights {
    const float *p;
    int64_t f;
    float missing;
    Vec<float, S::VE> w[KEEP ? S::NV : 1];
    __device__ __forceinline__ Weights(const float *p_, int64_t f_, float missing_) : p(p_), f(f_), missing(missing_) {
        if constexpr (KEEP)
#pragma unroll
            for (int v = 0; v < S::NV; ++v) fetch(v, w[v]);
    }
    __device__ __forceinline__ void fetch(int v, Vec<float, S::VE> &r) const {
        if (p) {
            r.load_upto(p + S::col(v), f - S::col(v));
        } else {
#pragma unroll
            for (int e = 0; e < S::VE; ++e) r.w[e] = __float_as_uint(missing);
        }
    }
    __device__ __forceinline__ Vec<float, S::VE> operator()(int v) const {
        if constexpr (KEEP) return w[v];
        Vec<float, S::VE> r;
        fetch(v, r);
        return r;
    }
};

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <class S, class TX, class TY>
__global__ void __launch_bounds__(S::kThreads) layer_norm_fwd_kernel(const TX *x, const int64_t *m_dev, int64_t cap_m,
                                                                     int64_t f, const float *gamma, const float *beta,
                                                                     float eps, TY *y, float *mean, float *rstd) {
    __shared__ typename RowReduce<S>::Shared sh;
    RowReduce<S> over(sh);
    const int64_t M = live_rows(m_dev, cap_m);
    const float n = static_cast<float>(f);
    const Weights<S, S::E <= 8> ga(gamma, f, 1.f), be(beta, f, 0.f);
    // 64 elements a thread leave no registers for anything else: rows that
    // long are read again for each pass, from the caches
    constexpr bool kHold = S::E <= 32;
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * S::kRows; i0 < M; i0 += static_cast<int64_t>(gridDim.x) * S::kRows) {
        const int64_t i = i0 + S::row();
        const bool live = i < M;
        const TX *xi = x + (live ? i : i0) * f;
        Vec<TX, S::VE> r[kHold ? S::NV : 1];
        if constexpr (kHold)
#pragma unroll
            for (int v = 0; v < S::NV; ++v) r[v].load_upto(xi + S::col(v), f - S::col(v));
        float s[1] = {0.f};
#pragma unroll(kHold ? S::NV : 1)
        for (int v = 0; v < S::NV; ++v) {
            Vec<TX, S::VE> &o = r[kHold ? v : 0];
            if constexpr (!kHold) o.load_upto(xi + S::col(v), f - S::col(v));
#pragma unroll
            for (int e = 0; e < S::VE; ++e) s[0] += o.get(e);
        }
        over(Add{}, s);
        const float mu = s[0] / n;
        s[0] = 0.f;
#pragma unroll(kHold ? S::NV : 1)
        for (int v = 0; v < S::NV; ++v) {
            Vec<TX, S::VE> &o = r[kHold ? v : 0];
            if constexpr (!kHold) o.load_upto(xi + S::col(v), f - S::col(v));
#pragma unroll
            for (int e = 0; e < S::VE; ++e) {
                const float d = o.get(e) - mu;
                if (S::col(v) + e < f) s[0] = fmaf(d, d, s[0]);
            }
        }
        over(Add{}, s);
        const float q = 1.f / sqrtf(s[0] / n + eps);
        if (live) {
#pragma unroll(kHold ? S::NV : 1)
            for (int v = 0; v < S::NV; ++v) {
                const Vec<float, S::VE> wg = ga(v), wb = be(v);
                Vec<TX, S::VE> &in = r[kHold ? v : 0];
                if constexpr (!kHold) in.load_upto(xi + S::col(v), f - S::col(v));
                float o[S::VE];
#pragma unroll
                for (int e = 0; e < S::VE; ++e) o[e] = fmaf((in.get(e) - mu) * q, wg.get(e), wb.get(e));
                Vec<TY, S::VE> w;
                w.set(o);
                w.store_upto(y + i * f + S::col(v), f - S::col(v));
            }
            if (S::lane() == 0) {
                if (mean) mean[i] = mu;
                if (rstd) rstd[i] = q;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
struct BwdArgs {
    const void *g, *x;
    const int64_t *m_dev;
    int64_t cap_m, f;
    const float *gamma, *mean, *rstd;
    const void *d_res;
    void *d_x;
    float *part;  // row p: workgroup p's sums of g h (f of them), then of g; or null
};

// d_x of every row, and with SUMS the workgroup's column sums.
template <class S, class TG, class TX, bool SUMS>
__global__ void __launch_bounds__(S::kThreads) layer_norm_bwd_kernel(BwdArgs p) {
    __shared__ typename RowReduce<S>::Shared sh;
    RowReduce<S> over(sh);
    const int64_t M = live_rows(p.m_dev, p.cap_m), f = p.f;
    const TG *g = static_cast<const TG *>(p.g), *d_res = static_cast<const TG *>(p.d_res);
    const TX *x = static_cast<const TX *>(p.x);
    TG *d_x = static_cast<TG *>(p.d_x);
    const float n = static_cast<float>(f);
    constexpr int E = SUMS ? S::E : 1;
    float sa[E], sb[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sa[e] = sb[e] = 0.f;
    const Weights<S, S::E <= 16 && S::T <= 512> ga(p.gamma, f, 1.f);
    // Both operands of a row stay in registers up to 32 words a thread (else
    // the second pass reads them again, from the caches), and the residual's
    // gradient is loaded with them where there is room
    constexpr bool kHold = S::E * (sizeof(TG) + sizeof(TX)) / 4 <= 32, kEarly = S::T <= 512;
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * S::kRows; i0 < M; i0 += static_cast<int64_t>(gridDim.x) * S::kRows) {
        const int64_t i = i0 + S::row();
        const bool live = i < M;
        const int64_t at = (live ? i : i0) * f;
        Vec<TG, S::VE> vg[kHold ? S::NV : 1], vd[kEarly ? S::NV : 1];
        Vec<TX, S::VE> vx[kHold ? S::NV : 1];
        if constexpr (kHold)
#pragma unroll
            for (int v = 0; v < S::NV; ++v) {
                vg[v].load_upto(g + at + S::col(v), f - S::col(v));
                vx[v].load_upto(x + at + S::col(v), f - S::col(v));
            }
        if constexpr (kEarly)
            if (d_res)
#pragma unroll
                for (int v = 0; v < S::NV; ++v) vd[v].load_upto(d_res + at + S::col(v), f - S::col(v));
        const float mu = p.mean[live ? i : i0], r = p.rstd[live ? i : i0];
        float s[2] = {0.f, 0.f};
#pragma unroll(kHold ? S::NV : 1)
        for (int v = 0; v < S::NV; ++v) {
            const Vec<float, S::VE> wg = ga(v);
            Vec<TG, S::VE> &og = vg[kHold ? v : 0];
            Vec<TX, S::VE> &ox = vx[kHold ? v : 0];
            if constexpr (!kHold) {
                og.load_upto(g + at + S::col(v), f - S::col(v));
                ox.load_upto(x + at + S::col(v), f - S::col(v));
            }
#pragma unroll
            for (int e = 0; e < S::VE; ++e) {
                // Past the row's end g is 0, and so are q and its product with the
                // finite d: the row's sum takes its factor r behind (d r there is
                // -mu r, which can be infinite in a finite row, and 0 times it NaN).
                const float ge = og.get(e), d = ox.get(e) - mu, q = ge * wg.get(e);
                s[0] += q;
                s[1] = fmaf(q, d, s[1]);
                if constexpr (SUMS) {
                    if (live) {
                        sa[v * S::VE + e] = fmaf(ge, d * r, sa[v * S::VE + e]);
                        sb[v * S::VE + e] += ge;
                    }
                }
            }
        }
        if (!d_x) continue;
        over(Add{}, s);
        const float m0 = s[0] / n, m1 = s[1] * r / n;
        if (!live) continue;
#pragma unroll(kHold ? S::NV : 1)
        for (int v = 0; v < S::NV; ++v) {
            const Vec<float, S::VE> wg = ga(v);
            Vec<TG, S::VE> &og = vg[kHold ? v : 0], &od = vd[kEarly ? v : 0];
            Vec<TX, S::VE> &ox = vx[kHold ? v : 0];
            if constexpr (!kHold) {
                og.load_upto(g + at + S::col(v), f - S::col(v));
                ox.load_upto(x + at + S::col(v), f - S::col(v));
            }
            if constexpr (!kEarly)
                if (d_res) od.load_upto(d_res + at + S::col(v), f - S::col(v));
            float o[S::VE];
#pragma unroll
            for (int e = 0; e < S::VE; ++e) {
                const float h = (ox.get(e) - mu) * r, q = og.get(e) * wg.get(e);
                o[e] = r * (q - m0 - h * m1);
                if (d_res) o[e] += od.get(e);
            }
            Vec<TG, S::VE> w;
            w.set(o);
            w.store_upto(d_x + at + S::col(v), f - S::col(v));
        }
    }
    if constexpr (SUMS) {
        // the rows that the workgroup held at a time, added in their order
        float *pa = p.part + static_cast<int64_t>(blockIdx.x) * 2 * f;
        if constexpr (S::kRows > 1) {
            __shared__ float cols[2][S::kRows][S::T * S::E];
#pragma unroll
            for (int v = 0; v < S::NV; ++v)
#pragma unroll
                for (int e = 0; e < S::VE; ++e) {
                    cols[0][S::row()][S::col(v) + e] = sa[v * S::VE + e];
                    cols[1][S::row()][S::col(v) + e] = sb[v * S::VE + e];
                }
            __syncthreads();
            for (int64_t j = threadIdx.x; j < 2 * f; j += S::kThreads) {
                const int which = j >= f, c = static_cast<int>(j - which * f);
                float t = 0.f;
#pragma unroll
                for (int k = 0; k < S::kRows; ++k) t += cols[which][k][c];
                pa[j] = t;
            }
        } else {
#pragma unroll
            for (int v = 0; v < S::NV; ++v) {
                Vec<float, S::VE> w;
                w.set(sa + v * S::VE);
                w.store_upto(pa + S::col(v), f - S::col(v));
                w.set(sb + v * S::VE);
                w.store_upto(pa + f + S::col(v), f - S::col(v));
            }
        }
    }
}

// Column sums alone, for rows whose sums do not fit the registers beside the
// row: workgroup (stripe, p) adds columns [1024 stripe, + 1024) over the p-th
// part of the rows.
constexpr int kStripe = 1024;
template <class TG, class TX> __global__ void __launch_bounds__(256) layer_norm_columns_kernel(BwdArgs p, int64_t parts) {
    const int64_t M = live_rows(p.m_dev, p.cap_m), f = p.f;
    const int64_t stripes = ceil_div(f, kStripe), stripe = blockIdx.x % stripes, q = blockIdx.x / stripes;
    const int64_t per = ceil_div(M, parts), beg = min(M, q * per), end = min(M, beg + per);
    const int64_t c = stripe * kStripe + threadIdx.x * 4;
    if (c >= f) return;
    const TG *g = static_cast<const TG *>(p.g) + c;
    const TX *x = static_cast<const TX *>(p.x) + c;
    float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t i = beg; i < end; ++i) {
        const float mu = p.mean[i], r = p.rstd[i];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < f) {
                const float v = Elem<TG>::load(g, i * f + e);
                a[e] = fmaf(v, (Elem<TX>::load(x, i * f + e) - mu) * r, a[e]);
                b[e] += v;
            }
    }
    float *pa = p.part + q * 2 * f + c;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < f) {
            pa[e] = a[e];
            pa[f + e] = b[e];
        }
}

// dgamma and dbeta from the partial rows, in a fixed order: a workgroup takes 32
// columns, each of its 32 groups every 32nd partial (eight loads in flight), and
// adds the groups.  `rows` is how many rows one partial takes at a time;
// workgroups that had none left no partial.
constexpr int kReduceThreads = 1024;
__global__ void __launch_bounds__(kReduceThreads) layer_norm_reduce_kernel(const float *part, int64_t parts, int64_t rows,
                                                                           const int64_t *m_dev, int64_t cap_m,
                                                                           int64_t f, float *dgamma, float *dbeta) {
    __shared__ float sh[32][33];
    const int c = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int64_t j = static_cast<int64_t>(blockIdx.x) * 32 + c;
    const int64_t n = min(parts, ceil_div(live_rows(m_dev, cap_m), rows));
    float s = 0.f;
    if (j < 2 * f)
        for (int64_t q = grp; q < n; q += 8 * 32) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = part[min(q + 32 * k, n - 1) * 2 * f + j];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += q + 32 * k < n ? v[k] : 0.f;
        }
    sh[grp][c] = s;
    __syncthreads();
    // column `grp` of the 32, its groups' sums in a wavefront's half
    s = sh[c][grp];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor(s, o, 32);
    const int64_t k = static_cast<int64_t>(blockIdx.x) * 32 + grp;
    if (c != 0 || k >= 2 * f) return;
    float *out = k < f ? dgamma : dbeta;
    if (out) out[k < f ? k : k - f] = s;
}

template <class F> void with_types(int a, int b, F &&go) {
    if (a == GNN_BF16 && b == GNN_BF16) go(uint16_t{}, uint16_t{});
    else if (a == GNN_BF16) go(uint16_t{}, float{});
    else if (b == GNN_BF16) go(float{}, uint16_t{});
    else go(float{}, float{});
}

// The shape for rows of f columns; fp32 rows are read in vectors of 4.
template <int VE, class F> void with_shape(int64_t f, F &&go) {
    if (f <= 32) go(Shape<4, 8, VE>{});
    else if (f <= 64) go(Shape<8, 8, VE>{});
    else if (f <= 128) go(Shape<16, 8, VE>{});
    else if (f <= 256) go(Shape<32, 8, VE>{});
    else if (f <= 512) go(Shape<64, 8, VE>{});
    else if (f <= 1024) go(Shape<64, 16, VE>{});
    else if (f <= 2048) go(Shape<256, 8, VE>{});
    else if (f <= 4096) go(Shape<256, 16, VE>{});
    else if (f <= 8192) go(Shape<512, 16, VE>{});
    else if (f <= 16384) go(Shape<1024, 16, VE>{});
    else if (f <= 32768) go(Shape<1024, 32, VE>{});
    else go(Shape<1024, 64, VE>{});
}

// Rows that one workgroup of the backward takes at a time.
int64_t rows_at_a_time(int64_t f) {
    int64_t n = 1;
    with_shape<8>(f, [&](auto shape) { n = decltype(shape)::kRows; });
    return n;
}

// Workgroups that walk the rows.  Threads of 8 elements fit eight workgroups of
// 256 to a CU: a grid of one round keeps their weights loaded.  Longer rows
// take more registers and fewer workgroups fit, so their grid is of many
// short rounds (32,768 x 8,192 bf16: 278 us with four workgroups to a CU, of
// which three are resident).
constexpr int64_t kFullGrid = 8 * kCus, kLongGrid = 32 * kCus;
constexpr int64_t kSumsMax = 16384;  // columns whose sums stay in registers
// Workgroups that keep sums: two to a CU fill the memory pipeline; each costs
// a partial row.
constexpr int64_t kParts = 2 * kCus;

struct BwdPlan {
    int64_t parts, rows;  // partial rows, and rows that each takes at a time
};
BwdPlan plan_bwd(int64_t f, int64_t cap_m) {
    BwdPlan p{};
    p.rows = f <= kSumsMax ? rows_at_a_time(f) : 1;
    p.parts = std::max<int64_t>(1, std::min<int64_t>(f <= kSumsMax ? kParts : 64, ceil_div(cap_m, p.rows)));
    return p;
}

}  // namespace

gnn_status launch_layer_norm_fwd(const void *x, int xdt, const int64_t *m_dev, int64_t cap_m, int64_t f,
                                 const float *gamma, const float *beta, float eps, void *y, int ydt, float *mean,
                                 float *rstd, hipStream_t s) {
    if (cap_m == 0) return GNN_OK;
    with_types(xdt, ydt, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        with_shape<sizeof(TX) + sizeof(TY) == 8 ? 4 : 8>(f, [&](auto shape) {
            using S = decltype(shape);
            const int64_t grid = std::min<int64_t>(ceil_div(cap_m, S::kRows), S::E <= 8 ? kFullGrid : kLongGrid);
            layer_norm_fwd_kernel<S, TX, TY><<<static_cast<unsigned>(grid), S::kThreads, 0, s>>>(
                static_cast<const TX *>(x), m_dev, cap_m, f, gamma, beta, eps, static_cast<TY *>(y), mean, rstd);
        });
    });
    GNN_LAUNCHED("layer_norm_fwd");
    return GNN_OK;
}

size_t layer_norm_bwd_ws_bytes(int64_t f, int64_t cap_m) {
    return round_up(static_cast<size_t>(plan_bwd(f, cap_m).parts * 2 * f * 4), 256);
}

gnn_status launch_layer_norm_bwd(const void *g, int gdt, const void *x, int xdt, const int64_t *m_dev, int64_t cap_m,
                                 int64_t f, const float *gamma, const float *mean, const float *rstd,
                                 const void *d_res, void *d_x, float *dgamma, float *dbeta, void *ws, hipStream_t s) {
    const BwdArgs p{g, x, m_dev, cap_m, f, gamma, mean, rstd, d_res, d_x, static_cast<float *>(ws)};
    const BwdPlan plan = plan_bwd(f, cap_m);
    const bool dw = dgamma || dbeta, fused = dw && f <= kSumsMax;
    with_types(gdt, xdt, [&](auto tg, auto tx) {
        using TG = decltype(tg);
        using TX = decltype(tx);
        // the columns' sums first: d_x may be g itself
        if (dw && !fused && cap_m > 0)
            layer_norm_columns_kernel<TG, TX><<<static_cast<unsigned>(ceil_div(f, kStripe) * plan.parts), 256, 0, s>>>(
                p, plan.parts);
        if (cap_m > 0 && (fused || d_x))
            with_shape<sizeof(TG) + sizeof(TX) == 8 ? 4 : 8>(f, [&](auto shape) {
                using S = decltype(shape);
                const int64_t grid = std::min<int64_t>(ceil_div(cap_m, S::kRows), kLongGrid);
                if constexpr (S::T * S::E <= kSumsMax) {
                    if (fused) {
                        layer_norm_bwd_kernel<S, TG, TX, true><<<static_cast<unsigned>(plan.parts), S::kThreads, 0, s>>>(p);
                        return;
                    }
                }
                layer_norm_bwd_kernel<S, TG, TX, false><<<static_cast<unsigned>(grid), S::kThreads, 0, s>>>(p);
            });
    });
    GNN_LAUNCHED("layer_norm_bwd");
    if (dw) {
        layer_norm_reduce_kernel<<<static_cast<unsigned>(ceil_div(2 * f, 32)), kReduceThreads, 0, s>>>(
            p.part, plan.parts, fused ? plan.rows : 1, m_dev, cap_m, f, dgamma, dbeta);
        GNN_LAUNCHED("layer_norm_reduce");
    }
    return GNN_OK;
}

}  // namespace gnn
