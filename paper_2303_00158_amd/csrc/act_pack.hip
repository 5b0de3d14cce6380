// Copies of bf16 operands in the form the tiles' kernels read (act_pack.h).
#include "act_pack.h"

namespace gnn {
namespace pack {

namespace {

constexpr int kThreads = 256;

// out[r][c] = bf16([x0 || x1][r][c]) for c < K, 0 for K <= c < ld; eight values a
// thread.  Rows at or past the count are left alone.
template <class T>
__global__ void __launch_bounds__(kThreads) pack_rows_kernel(const T *x0, const T *x1, int64_t k_each, int64_t K,
                                                             const int64_t *m_dev, int64_t rows, int64_t ld,
                                                             uint16_t *out) {
    const int64_t M = m_dev ? min(*m_dev, rows) : rows, groups = ld / 8;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; t < M * groups;
         t += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t r = t / groups, c = (t - r * groups) * 8;
        uint16_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool hi = x1 && c + e >= k_each;
            v[e] = c + e < K ? f32_to_bf16(Elem<T>::load(hi ? x1 : x0, r * k_each + c + e - (hi ? k_each : 0))) : uint16_t(0);
        }
        uint4 o;
        o.x = v[0] | (static_cast<uint32_t>(v[1]) << 16);
        o.y = v[2] | (static_cast<uint32_t>(v[3]) << 16);
        o.z = v[4] | (static_cast<uint32_t>(v[5]) << 16);
        o.w = v[6] | (static_cast<uint32_t>(v[7]) << 16);
        *reinterpret_cast<uint4 *>(out + r * ld + c) = o;
    }
}

// out[n][k] = bf16(w[k][n]) for k < K, 0 for K <= k < ld: 64 x 64 squares through
// LDS, so that both sides go by rows.
__global__ void __launch_bounds__(kThreads) pack_transpose_kernel(const float *w, int64_t K, int64_t n_out, int64_t ld,
                                                                  uint16_t *out) {
    __shared__ uint16_t sq[64][66];
    const int64_t squares = ceil_div(n_out, int64_t(64));
    const int64_t k0 = blockIdx.x / squares * 64, n0 = blockIdx.x % squares * 64;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t k = k0 + y + 4 * i, n = n0 + x;
        sq[y + 4 * i][x] = k < K && n < n_out ? f32_to_bf16(w[k * n_out + n]) : uint16_t(0);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t n = n0 + y + 4 * i, k = k0 + x;
        if (n < n_out && k < ld) out[n * ld + k] = sq[x][y + 4 * i];
    }
}

unsigned grid_of(int64_t n) {
    return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, kThreads), 16384)));
}

}  // namespace

gnn_status prepare(const ActArgs &a, int64_t chunk, bool weights, void *ws, Operands *o, hipStream_t s) {
    const int64_t K = a.K(), ld = row8(K);
    const Layout l(a.cap_m, K, a.n_out);
    char *base = static_cast<char *>(ws);
    *o = Operands{static_cast<const uint16_t *>(a.a_self), static_cast<const uint16_t *>(a.a_nbr), a.k_each, K, a.k_each,
                  a.wt, K};
    if (copies_a(a, chunk)) {
        uint16_t *out = reinterpret_cast<uint16_t *>(base + l.a);
        const unsigned grid = grid_of(a.cap_m * (ld / 8));
        if (a.adt == GNN_BF16)
            pack_rows_kernel<uint16_t><<<grid, kThreads, 0, s>>>(static_cast<const uint16_t *>(a.a_self),
                                                                 static_cast<const uint16_t *>(a.a_nbr), a.k_each, K,
                                                                 a.m_dev, a.cap_m, ld, out);
        else
            pack_rows_kernel<float><<<grid, kThreads, 0, s>>>(static_cast<const float *>(a.a_self),
                                                              static_cast<const float *>(a.a_nbr), a.k_each, K, a.m_dev,
                                                              a.cap_m, ld, out);
        GNN_LAUNCHED("act_pack_rows");
        o->a0 = out;
        o->a1 = nullptr;
        o->k_each = o->K = o->lda = ld;
    }
    if (!weights || !copies_w(a)) return GNN_OK;
    if (!a.wt) {
        uint16_t *out = reinterpret_cast<uint16_t *>(base + l.w);
        pack_transpose_kernel<<<static_cast<unsigned>(ceil_div(ld, int64_t(64)) * ceil_div(a.n_out, int64_t(64))), kThreads,
                                0, s>>>(a.w, K, a.n_out, ld, out);
        GNN_LAUNCHED("act_pack_w");
        o->wt = out;
        o->ldw = ld;
    } else {
        uint16_t *out = reinterpret_cast<uint16_t *>(base + l.w);
        pack_rows_kernel<uint16_t><<<grid_of(a.n_out * (ld / 8)), kThreads, 0, s>>>(a.wt, nullptr, K, K, nullptr, a.n_out,
                                                                                  ld, out);
        GNN_LAUNCHED("act_pack_wt");
        o->wt = out;
        o->ldw = ld;
    }
    return GNN_OK;
}

}  // namespace pack
}  // namespace gnn
