// The loss of a student's logits against a teacher's top logits, with its
// gradient in the same launch.
#include "internal.h"
#include "loss_dev.h"

namespace gnn {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float *sh) {
    v = loss::wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
    for (int w = 0; w < kThreads / 64; ++w) t += sh[w];
    return t;
}

__device__ __forceinline__ float block_max(float v, float *sh) {
    v = loss::wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = -INFINITY;
    for (int w = 0; w < kThreads / 64; ++w) t = fmaxf(t, sh[w]);
    return t;
}

// One workgroup per row; the row's loss goes to row_loss (the workspace when
// the caller wants none).
template <class TL, class TT, class TG>
__global__ void __launch_bounds__(kThreads) distill_kernel(DistillArgs a, float *row_loss) {
    __shared__ float sh[kThreads / 64];
    __shared__ float prob[GNN_MAX_TOP];
    __shared__ int32_t cls[GNN_MAX_TOP];
    __shared__ float zt[GNN_MAX_TOP];
    const int64_t i = blockIdx.x, c = a.c;
    const int tid = threadIdx.x, k = static_cast<int>(a.k);
    const TL *z = static_cast<const TL *>(a.logits) + i * c;
    TG *g = a.g_out ? static_cast<TG *>(a.g_out) + i * c : nullptr;
    const float scale = a.row_scale ? a.row_scale[i] : 1.f / static_cast<float>(a.b);
    if (scale == 0.f) {
        if (g)
            for (int64_t j = tid; j < c; j += kThreads) Elem<TG>::store(g, j, 0.f);
        if (tid == 0) row_loss[i] = 0.f;
        return;
    }
    const float inv_t = 1.f / a.temperature;
    // the teacher's distribution over the present entries
    float tmax = -INFINITY;
    if (a.alpha > 0.f) {
        for (int e = tid; e < k; e += kThreads) {
            const int64_t id = a.t_idx[i * k + e];
            const float v = Elem<TT>::load(static_cast<const TT *>(a.t_val), i * k + e);
            const bool in = id >= 0 && id < c && v != -INFINITY;
            cls[e] = in ? static_cast<int32_t>(id) : -1;
            prob[e] = v;
            if (in) {
                tmax = fmaxf(tmax, v);
                zt[e] = Elem<TL>::load(z, id);
            }
        }
    }
    tmax = block_max(tmax, sh);
    float ts = 0.f;
    if (a.alpha > 0.f)
        for (int e = tid; e < k; e += kThreads) {
            prob[e] = cls[e] >= 0 ? expf((prob[e] - tmax) * inv_t) : 0.f;
            ts += prob[e];
        }
    ts = block_sum(ts, sh);
    const bool soft = ts != 0.f;  // a NaN counts as present
    int64_t y = -1;
    if (a.labels && a.alpha < 1.f) y = a.labels[a.targets ? a.targets[i] : i];
    const bool hard = y >= 0 && y < c;
    const float zy = hard ? Elem<TL>::load(z, y) : 0.f;
    // the student's sums, at the temperature and at 1
    float mx = -INFINITY;
    for (int64_t j = tid; j < c; j += kThreads) mx = fmaxf(mx, Elem<TL>::load(z, j));
    mx = block_max(mx, sh);
    float st = 0.f, s1 = 0.f;
    for (int64_t j = tid; j < c; j += kThreads) {
        const float d = Elem<TL>::load(z, j) - mx;
        st += expf(d * inv_t);
        s1 += expf(d);
    }
    st = block_sum(st, sh);
    s1 = block_sum(s1, sh);
    float l = 0.f;
    if (soft) {
        const float logts = logf(ts), logst = logf(st);
        for (int e = tid; e < k; e += kThreads) {
            const float p = prob[e] / ts;
            const float logp = (Elem<TT>::load(static_cast<const TT *>(a.t_val), i * k + e) - tmax) * inv_t - logts;
            if (cls[e] >= 0 && p != 0.f) l += p * (logp - ((zt[e] - mx) * inv_t - logst));
            prob[e] = p;
        }
    }
    l = block_sum(l, sh) * a.alpha * a.temperature * a.temperature;
    if (hard) l += (1.f - a.alpha) * (logf(s1) - (zy - mx));
    if (tid == 0) row_loss[i] = l;
    if (!g) return;
    const float ct = soft ? scale * a.alpha * a.temperature : 0.f, c1 = hard ? scale * (1.f - a.alpha) : 0.f;
    auto grad = [&](float v, int64_t j) {
        const float d = v - mx;
        float x = 0.f;
        if (soft) x += ct * (expf(d * inv_t) / st);
        if (hard) x += c1 * (expf(d) / s1 - (j == y ? 1.f : 0.f));
        return x;
    };
    for (int64_t j = tid; j < c; j += kThreads) Elem<TG>::store(g, j, grad(Elem<TL>::load(z, j), j));
    if (!soft) return;
    __syncthreads();
    // each listed class again, by its first entry: less its entries' shares
    for (int e = tid; e < k; e += kThreads) {
        const int32_t id = cls[e];
        if (id < 0) continue;
        bool first = true;
        float p = 0.f;
        for (int o = 0; o < k; ++o)
            if (cls[o] == id) {
                first = first && o >= e;
                p += prob[o];
            }
        if (first) Elem<TG>::store(g, id, grad(zt[e], id) - ct * p);
    }
}

// loss = sum over the rows of scale x row loss, by one workgroup.
__global__ void __launch_bounds__(kThreads) distill_loss_kernel(const float *row_loss, const float *row_scale,
                                                                int64_t b, float *loss) {
    __shared__ float sh[kThreads / 64];
    float s = 0.f;
    for (int64_t i = threadIdx.x; i < b; i += kThreads) s += row_scale ? row_scale[i] * row_loss[i] : row_loss[i];
    s = block_sum(s, sh);
    if (threadIdx.x == 0) *loss = row_scale || b == 0 ? s : s / static_cast<float>(b);
}

}  // namespace

size_t distill_ws_bytes(int64_t b, int64_t, int64_t) { return round_up(static_cast<size_t>(b > 0 ? b : 1) * 4, 256); }

gnn_status launch_distill(const DistillArgs &a, void *ws, hipStream_t s) {
    float *row_loss = a.row_loss ? a.row_loss : static_cast<float *>(ws);
    if (a.b > 0) {
        const unsigned grid = static_cast<unsigned>(a.b);
        auto go = [&](auto tl, auto tt, auto tg) {
            distill_kernel<decltype(tl), decltype(tt), decltype(tg)><<<grid, kThreads, 0, s>>>(a, row_loss);
        };
        auto by_grad = [&](auto tl, auto tt) {
            if (a.gdt == GNN_BF16) go(tl, tt, uint16_t{});
            else go(tl, tt, float{});
        };
        auto by_teacher = [&](auto tl) {
            if (a.tdt == GNN_BF16) by_grad(tl, uint16_t{});
            else by_grad(tl, float{});
        };
        if (a.ldt == GNN_BF16) by_teacher(uint16_t{});
        else by_teacher(float{});
        GNN_LAUNCHED("distill_topk");
    }
    distill_loss_kernel<<<1, kThreads, 0, s>>>(row_loss, a.row_scale, a.b, a.loss_out);
    GNN_LAUNCHED("distill_topk_loss");
    return GNN_OK;
}

}  // namespace gnn
