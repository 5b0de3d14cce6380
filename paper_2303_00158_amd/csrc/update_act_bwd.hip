// Gradients of the update with an activation: dZ = g act'(Z), then the
// update's own products (gemm_bwd.hip) on dZ.
#include "act_dev.h"

namespace gnn {

namespace {

constexpr int kThreads = 256;

template <int ACT, class TG, class TZ>
__global__ void __launch_bounds__(kThreads) act_slope_kernel(const TG *g, const TZ *z, const int64_t *m_dev,
                                                             int64_t cap_m, int64_t n_out, float *dz) {
    const int64_t n = (m_dev ? max(min(*m_dev, cap_m), int64_t(0)) : cap_m) * n_out;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads) {
        float v = Elem<TG>::load(g, i);
        if constexpr (ACT != GNN_ACT_NONE) v *= act::slope<ACT>(Elem<TZ>::load(z, i));
        dz[i] = v;
    }
}

// out (n values, or the counted rows of row length ld) = bf16(in)
__global__ void __launch_bounds__(kThreads) act_narrow_kernel(const float *in, const int64_t *m_dev, int64_t rows,
                                                              int64_t ld, uint16_t *out) {
    const int64_t n = (m_dev ? max(min(*m_dev, rows), int64_t(0)) : rows) * ld;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads)
        out[i] = f32_to_bf16(in[i]);
}

// w[k][n] = wt[n][k]
__global__ void __launch_bounds__(kThreads) act_unshadow_kernel(const uint16_t *wt, int64_t K, int64_t n_out, float *w) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < K * n_out;
         i += static_cast<int64_t>(gridDim.x) * kThreads)
        w[i] = bf16_to_f32(wt[(i % n_out) * K + i / n_out]);
}

unsigned grid_of(int64_t n) {
    return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, kThreads), 8192)));
}

struct Layout {
    size_t dz, w, dw, d_a, gemm, total;
};
Layout layout(int64_t K, int64_t n_out, int64_t cap_m, int gdt, int dwdt, int gemm_dt, bool shadow) {
    Carver c(nullptr);
    Layout l{};
    l.dz = c.take(static_cast<size_t>(cap_m * n_out * 4));
    l.w = c.take(shadow ? static_cast<size_t>(K * n_out * 4) : 0);
    l.dw = c.take(dwdt == GNN_BF16 ? static_cast<size_t>(K * n_out * 4) : 0);
    l.d_a = c.take(gdt == GNN_BF16 ? static_cast<size_t>(cap_m * K * 4) : 0);
    l.gemm = c.take(update_bwd_ws_bytes(K, n_out, cap_m, gemm_dt));
    l.total = round_up(c.off, 256);
    return l;
}

}  // namespace

size_t act_bwd_ws_bytes(int, int64_t k_each, bool two, int64_t n_out, int64_t cap_m, int gdt, int dwdt, int gemm_dt,
                        bool shadow) {
    return layout(two ? 2 * k_each : k_each, n_out, cap_m, gdt, dwdt, gemm_dt, shadow).total;
}

gnn_status launch_act_bwd(const ActBwd &a, void *ws, hipStream_t s) {
    const int64_t K = a.K();
    const Layout l = layout(K, a.n_out, a.cap_m, a.gdt, a.dwdt, a.gemm_dt, a.wt != nullptr);
    char *base = static_cast<char *>(ws);
    float *dz = reinterpret_cast<float *>(base + l.dz);
    if (a.cap_m > 0) {
        const unsigned grid = grid_of(a.cap_m * a.n_out);
        act::with(a.act, [&](auto code) {
            constexpr int ACT = decltype(code)::value;
            auto go = [&](auto tg, auto tz) {
                using TG = decltype(tg);
                using TZ = decltype(tz);
                act_slope_kernel<ACT, TG, TZ><<<grid, kThreads, 0, s>>>(
                    static_cast<const TG *>(a.g), static_cast<const TZ *>(a.z), a.m_dev, a.cap_m, a.n_out, dz);
            };
            if (a.gdt == GNN_BF16) {
                if (a.zdt == GNN_BF16) go(uint16_t{}, uint16_t{});
                else go(uint16_t{}, float{});
            } else {
                if (a.zdt == GNN_BF16) go(float{}, uint16_t{});
                else go(float{}, float{});
            }
        });
        GNN_LAUNCHED("act_slope");
    }
    const float *w = a.w;
    if (a.d_a && a.wt) {
        float *wf = reinterpret_cast<float *>(base + l.w);
        act_unshadow_kernel<<<grid_of(K * a.n_out), kThreads, 0, s>>>(a.wt, K, a.n_out, wf);
        GNN_LAUNCHED("act_unshadow");
        w = wf;
    }
    float *dw = a.dwdt == GNN_BF16 ? reinterpret_cast<float *>(base + l.dw) : static_cast<float *>(a.dw);
    float *d_a = !a.d_a ? nullptr : a.gdt == GNN_BF16 ? reinterpret_cast<float *>(base + l.d_a) : static_cast<float *>(a.d_a);
    GNN_TRY(launch_update_bwd(a.a_self, a.a_nbr, a.adt, a.k_each, a.m_dev, a.cap_m, w, dz, a.n_out, a.gemm_dt, dw, a.db,
                              d_a, base + l.gemm, nullptr, nullptr, nullptr, 0.f, s));
    if (a.dwdt == GNN_BF16) {
        act_narrow_kernel<<<grid_of(K * a.n_out), kThreads, 0, s>>>(dw, nullptr, K, a.n_out,
                                                                    static_cast<uint16_t *>(a.dw));
        GNN_LAUNCHED("act_narrow");
    }
    if (a.d_a && a.gdt == GNN_BF16 && a.cap_m > 0) {
        act_narrow_kernel<<<grid_of(a.cap_m * K), kThreads, 0, s>>>(d_a, a.m_dev, a.cap_m, K,
                                                                    static_cast<uint16_t *>(a.d_a));
        GNN_LAUNCHED("act_narrow");
    }
    return GNN_OK;
}

}  // namespace gnn
