// Layer normalisation of activation rows, forward and backward.
#include "internal.h"
#include "loss_dev.h"

namespace gnn {

namespace {

constexpr int kThreads = 256;

// Sum of v over the workgroup, in every thread, in a fixed order.
__device__ __forceinline__ float block_sum(float v, float *sh) {
    v = loss::wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) t += sh[w];
    return t;
}

__device__ __forceinline__ int64_t live_rows(const int64_t *m_dev, int64_t cap_m) {
    return m_dev ? max(min(*m_dev, cap_m), int64_t(0)) : cap_m;
}

// One workgroup per row.
template <class TX, class TY>
__global__ void __launch_bounds__(kThreads) layer_norm_fwd_kernel(const TX *x, const int64_t *m_dev, int64_t cap_m,
                                                                  int64_t f, const float *gamma, const float *beta,
                                                                  float eps, TY *y, float *mean, float *rstd) {
    __shared__ float sh[kThreads / 64];
    const int64_t i = blockIdx.x;
    if (i >= live_rows(m_dev, cap_m)) return;
    float s = 0.f;
    for (int64_t j = threadIdx.x; j < f; j += kThreads) s += Elem<TX>::load(x, i * f + j);
    const float mu = block_sum(s, sh) / static_cast<float>(f);
    float q = 0.f;
    for (int64_t j = threadIdx.x; j < f; j += kThreads) {
        const float d = Elem<TX>::load(x, i * f + j) - mu;
        q += d * d;
    }
    const float r = 1.f / sqrtf(block_sum(q, sh) / static_cast<float>(f) + eps);
    for (int64_t j = threadIdx.x; j < f; j += kThreads) {
        const float h = (Elem<TX>::load(x, i * f + j) - mu) * r;
        Elem<TY>::store(y, i * f + j, h * (gamma ? gamma[j] : 1.f) + (beta ? beta[j] : 0.f));
    }
    if (threadIdx.x == 0) {
        if (mean) mean[i] = mu;
        if (rstd) rstd[i] = r;
    }
}

template <class TG, class TX>
__global__ void __launch_bounds__(kThreads) layer_norm_dx_kernel(const TG *g, const TX *x, const int64_t *m_dev,
                                                                 int64_t cap_m, int64_t f, const float *gamma,
                                                                 const float *mean, const float *rstd,
                                                                 const TG *d_res, TG *d_x) {
    __shared__ float sh[kThreads / 64];
    const int64_t i = blockIdx.x;
    if (i >= live_rows(m_dev, cap_m)) return;
    const float mu = mean[i], r = rstd[i];
    float s = 0.f, t = 0.f;
    for (int64_t j = threadIdx.x; j < f; j += kThreads) {
        const float q = Elem<TG>::load(g, i * f + j) * (gamma ? gamma[j] : 1.f);
        s += q;
        t += q * ((Elem<TX>::load(x, i * f + j) - mu) * r);
    }
    s = block_sum(s, sh) / static_cast<float>(f);
    t = block_sum(t, sh) / static_cast<float>(f);
    for (int64_t j = threadIdx.x; j < f; j += kThreads) {
        const float q = Elem<TG>::load(g, i * f + j) * (gamma ? gamma[j] : 1.f);
        const float h = (Elem<TX>::load(x, i * f + j) - mu) * r;
        Elem<TG>::store(d_x, i * f + j, r * (q - s - h * t) + (d_res ? Elem<TG>::load(d_res, i * f + j) : 0.f));
    }
}

// Row group p's sums: part[p][0][j] of g h, part[p][1][j] of g.
constexpr int64_t kGroups = 256;

template <class TG, class TX>
__global__ void __launch_bounds__(kThreads) layer_norm_dw_kernel(const TG *g, const TX *x, const int64_t *m_dev,
                                                                 int64_t cap_m, int64_t f, const float *mean,
                                                                 const float *rstd, float *part) {
    const int64_t M = live_rows(m_dev, cap_m), p = blockIdx.x, per = ceil_div(M, kGroups);
    const int64_t beg = min(M, p * per), end = min(M, beg + per);
    for (int64_t j = threadIdx.x; j < f; j += kThreads) {
        float a = 0.f, b = 0.f;
        for (int64_t i = beg; i < end; ++i) {
            const float v = Elem<TG>::load(g, i * f + j);
            a += v * ((Elem<TX>::load(x, i * f + j) - mean[i]) * rstd[i]);
            b += v;
        }
        part[p * 2 * f + j] = a;
        part[(p * 2 + 1) * f + j] = b;
    }
}

__global__ void __launch_bounds__(kThreads) layer_norm_dw_reduce_kernel(const float *part, int64_t f, float *dgamma,
                                                                        float *dbeta) {
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (j >= 2 * f) return;
    float *out = j < f ? dgamma : dbeta;
    if (!out) return;
    float s = 0.f;
    for (int64_t p = 0; p < kGroups; ++p) s += part[p * 2 * f + j];
    out[j < f ? j : j - f] = s;
}

template <class F> void with_types(int a, int b, F &&go) {
    if (a == GNN_BF16 && b == GNN_BF16) go(uint16_t{}, uint16_t{});
    else if (a == GNN_BF16) go(uint16_t{}, float{});
    else if (b == GNN_BF16) go(float{}, uint16_t{});
    else go(float{}, float{});
}

}  // namespace

gnn_status launch_layer_norm_fwd(const void *x, int xdt, const int64_t *m_dev, int64_t cap_m, int64_t f,
                                 const float *gamma, const float *beta, float eps, void *y, int ydt, float *mean,
                                 float *rstd, hipStream_t s) {
    if (cap_m == 0) return GNN_OK;
    with_types(xdt, ydt, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        layer_norm_fwd_kernel<TX, TY><<<static_cast<unsigned>(cap_m), kThreads, 0, s>>>(
            static_cast<const TX *>(x), m_dev, cap_m, f, gamma, beta, eps, static_cast<TY *>(y), mean, rstd);
    });
    GNN_LAUNCHED("layer_norm_fwd");
    return GNN_OK;
}

size_t layer_norm_bwd_ws_bytes(int64_t f, int64_t) { return round_up(static_cast<size_t>(kGroups * 2 * f * 4), 256); }

gnn_status launch_layer_norm_bwd(const void *g, int gdt, const void *x, int xdt, const int64_t *m_dev, int64_t cap_m,
                                 int64_t f, const float *gamma, const float *mean, const float *rstd,
                                 const void *d_res, void *d_x, float *dgamma, float *dbeta, void *ws, hipStream_t s) {
    float *part = static_cast<float *>(ws);
    const bool dw = dgamma || dbeta;
    with_types(gdt, xdt, [&](auto tg, auto tx) {
        using TG = decltype(tg);
        using TX = decltype(tx);
        const TG *gp = static_cast<const TG *>(g);
        const TX *xp = static_cast<const TX *>(x);
        // the weights' sums first: d_x may be g itself
        if (dw)
            layer_norm_dw_kernel<TG, TX><<<static_cast<unsigned>(kGroups), kThreads, 0, s>>>(gp, xp, m_dev, cap_m, f,
                                                                                          mean, rstd, part);
        if (d_x && cap_m > 0)
            layer_norm_dx_kernel<TG, TX><<<static_cast<unsigned>(cap_m), kThreads, 0, s>>>(
                gp, xp, m_dev, cap_m, f, gamma, mean, rstd, static_cast<const TG *>(d_res), static_cast<TG *>(d_x));
    });
    GNN_LAUNCHED("layer_norm_bwd");
    if (dw) {
        layer_norm_dw_reduce_kernel<<<static_cast<unsigned>(ceil_div(2 * f, kThreads)), kThreads, 0, s>>>(part, f,
                                                                                                         dgamma, dbeta);
        GNN_LAUNCHED("layer_norm_dw_reduce");
    }
    return GNN_OK;
}

}  // namespace gnn
