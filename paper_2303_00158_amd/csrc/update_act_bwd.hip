// Gradients of the update with an activation:
//   dZ = g act'(Z),  dW = A^T dZ,  db = column sums of dZ,  dA = dZ W^T.
//
// bf16 products: one pass over g and Z writes dZ as bf16 and takes db's partial
// sums from the unrounded values on the way; both products then read dZ through
// the tiles of gemm_tile_dev.h.  dW reduces over the rows: both operands run down
// their matrices (T layout), and where the gradient has too few tiles to fill the
// chip the rows are split, each split writing an fp32 partial that a last
// kernel adds in order.  dA reduces over the columns: dZ is an N operand and the
// shadow W^T, whose rows are the reduction, a T operand, so that the weights are
// read as the forward keeps them.  (Without the shadow, W is rounded to bf16 rows
// in the workspace, an N operand.)
// fp32 products, and small ones, take the update's own kernels (gemm_bwd.hip) on an
// fp32 dZ.
#include "act_pack.h"
#include "gemm_tile_dev.h"

namespace gnn {

namespace {

constexpr int kThreads = 256;

unsigned grid_of(int64_t n) {
    return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, kThreads), 8192)));
}

__device__ __forceinline__ int64_t count(const int64_t *m_dev, int64_t cap_m) {
    return m_dev ? max(min(*m_dev, cap_m), int64_t(0)) : cap_m;
}

// go(tag of g's type, tag of z's type)
template <class F> void with_types(int gdt, int zdt, F &&go) {
    if (gdt == GNN_BF16) {
        if (zdt == GNN_BF16) go(uint16_t{}, uint16_t{});
        else go(uint16_t{}, float{});
    } else {
        if (zdt == GNN_BF16) go(float{}, uint16_t{});
        else go(float{}, float{});
    }
}

// ---------------------------------------------------------------------------
// on the general engine
// ---------------------------------------------------------------------------
template <int ACT, class TG, class TZ>
__global__ void __launch_bounds__(kThreads) act_slope_kernel(const TG *g, const TZ *z, const int64_t *m_dev,
                                                             int64_t cap_m, int64_t n_out, float *dz) {
    const int64_t n = count(m_dev, cap_m) * n_out;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads) {
        float v = Elem<TG>::load(g, i);
        if constexpr (ACT != GNN_ACT_NONE) v *= act::slope<ACT>(Elem<TZ>::load(z, i));
        dz[i] = v;
    }
}

// out (the counted rows of row length ld) = bf16(in)
__global__ void __launch_bounds__(kThreads) act_narrow_kernel(const float *in, const int64_t *m_dev, int64_t rows,
                                                              int64_t ld, uint16_t *out) {
    const int64_t n = count(m_dev, rows) * ld;
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

struct EngineLayout {
    size_t dz, w, dw, d_a, gemm, total;
    EngineLayout(int64_t K, int64_t n_out, int64_t cap_m, int gdt, int dwdt, int gemm_dt, bool shadow) {
        Carver c(nullptr);
        dz = c.take(static_cast<size_t>(cap_m * n_out * 4));
        w = c.take(shadow ? static_cast<size_t>(K * n_out * 4) : 0);
        dw = c.take(dwdt == GNN_BF16 ? static_cast<size_t>(K * n_out * 4) : 0);
        d_a = c.take(gdt == GNN_BF16 ? static_cast<size_t>(cap_m * K * 4) : 0);
        gemm = c.take(update_bwd_ws_bytes(K, n_out, cap_m, gemm_dt));
        total = round_up(c.off, 256);
    }
};

gnn_status launch_engine(const ActBwd &a, void *ws, hipStream_t s) {
    const int64_t K = a.K();
    const EngineLayout l(K, a.n_out, a.cap_m, a.gdt, a.dwdt, a.gemm_dt, a.wt != nullptr);
    char *base = static_cast<char *>(ws);
    float *dz = reinterpret_cast<float *>(base + l.dz);
    if (a.cap_m > 0) {
        const unsigned grid = grid_of(a.cap_m * a.n_out);
        act::with(a.act, [&](auto code) {
            constexpr int ACT = decltype(code)::value;
            with_types(a.gdt, a.zdt, [&](auto tg, auto tz) {
                using TG = decltype(tg);
                using TZ = decltype(tz);
                act_slope_kernel<ACT, TG, TZ><<<grid, kThreads, 0, s>>>(
                    static_cast<const TG *>(a.g), static_cast<const TZ *>(a.z), a.m_dev, a.cap_m, a.n_out, dz);
            });
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

// ---------------------------------------------------------------------------
// on the tiles: dZ and db's partial sums
// ---------------------------------------------------------------------------
constexpr int kStripe = 256;  // columns of a workgroup: 32 threads of 8, times 8 rows at a time

struct DzArgs {
    const void *g, *z;
    const int64_t *m_dev;
    int64_t cap_m, n_out;
    uint16_t *dz;        // row length ld, 0 past n_out
    int64_t ld;
    float *part;         // parts x n_out, or null (db is not wanted)
    int64_t parts;
    bool vec;            // g's and z's rows and pointers allow eight elements at a time
};

template <class T> __device__ __forceinline__ void get8(const T *p, int64_t room, bool vec, float (&v)[8]) {
    if (vec) {
        const float4 a = load4(p, 0), b = load4(p, 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < room ? Elem<T>::load(p, e) : 0.f;
    }
}

template <int ACT, class TG, class TZ>
__global__ void __launch_bounds__(kThreads) act_dz_kernel(DzArgs p) {
    __shared__ float sh[8][kStripe];
    const int64_t M = count(p.m_dev, p.cap_m);
    const int64_t stripes = ceil_div(p.ld, int64_t(kStripe)), stripe = blockIdx.x % stripes, part = blockIdx.x / stripes;
    const int64_t per = ceil_div(ceil_div(M, p.parts), int64_t(8)) * 8;
    const int64_t beg = min(M, part * per), end = min(M, beg + per);
    const int y = threadIdx.x >> 5, x = (threadIdx.x & 31) * 8;
    const int64_t c = stripe * kStripe + x, room = p.n_out - c;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < p.ld) {
        const TG *g = static_cast<const TG *>(p.g) + c;
        const TZ *z = static_cast<const TZ *>(p.z) + c;
        const bool vec = p.vec && room >= 8;
#pragma unroll 4
        for (int64_t i = beg + y; i < end; i += 8) {
            float v[8];
            get8(g + i * p.n_out, room, vec, v);
            if constexpr (ACT != GNN_ACT_NONE) {
                float zz[8];
                get8(z + i * p.n_out, room, vec, zz);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= act::slope<ACT>(zz[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
            uint4 o;
            o.x = wide::pack_bf16(v[0], v[1]);
            o.y = wide::pack_bf16(v[2], v[3]);
            o.z = wide::pack_bf16(v[4], v[5]);
            o.w = wide::pack_bf16(v[6], v[7]);
            *reinterpret_cast<uint4 *>(p.dz + i * p.ld + c) = o;
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sh[y][x + e] = sum[e];
    __syncthreads();
    const int64_t col = stripe * kStripe + threadIdx.x;
    if (col >= p.n_out) return;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) t += sh[k][threadIdx.x];
    p.part[part * p.n_out + col] = t;
}

// ---------------------------------------------------------------------------
// on the tiles: the products
// ---------------------------------------------------------------------------

// dW: output tiles of K x n_out, in each half of [a0 || a1] apart; split s of the
// rows writes to out + s * split_stride.
struct DwArgs {
    const uint16_t *a0, *a1;
    int64_t k_each, lda;
    const uint16_t *dz;
    int64_t ldz;
    const int64_t *m_dev;
    int64_t cap_m, n_out;
    void *out;
    int64_t ld, split_stride, nsplit;
    bool vec;
};

template <class C, class T> __global__ void __launch_bounds__(C::kThreads, C::PER_CU) act_dw_kernel(DwArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    const int64_t M = count(p.m_dev, p.cap_m);
    const int64_t half_tiles = ceil_div(p.k_each, int64_t(C::BM)), tm = p.a1 ? 2 * half_tiles : half_tiles;
    const int64_t tn = ceil_div(p.n_out, int64_t(C::BN));
    const int64_t item = wide::xcd_item(blockIdx.x, tm * tn * p.nsplit);
    if (item < 0) return;
    const int64_t split = item / (tm * tn);
    int64_t m, n;
    tile::tile_of(item % (tm * tn), tm, tn, &m, &n);
    const bool hi = m >= half_tiles;
    const int64_t k0 = (hi ? m - half_tiles : m) * C::BM, col0 = n * C::BN;
    const int64_t per = ceil_div(ceil_div(M, p.nsplit), int64_t(tile::kBK)) * tile::kBK;
    const int64_t beg = min(M, split * per), rows = min(M, beg + per) - beg;
    const tile::Operand oa{(hi ? p.a1 : p.a0) + beg * p.lda + k0, nullptr, p.lda, 0, p.lda - k0, rows};
    const tile::Operand ob{p.dz + beg * p.ldz + col0, nullptr, p.ldz, 0, p.ldz - col0, rows};
    tile::Acc<C> acc;
    acc.clear();
    const tile::Ring ring{{st0, st1}};
    if (rows > 0)
        tile::Product<C, true, true>(oa, ob).run(acc, ring, static_cast<int>(ceil_div(rows, int64_t(tile::kBK))));
    const int wave = threadIdx.x >> 6;
    T *out = static_cast<T *>(p.out) + split * p.split_stride + (hi ? p.k_each * p.ld : 0);
    const tile::Epilogue ep{nullptr, nullptr, nullptr, out, p.ld, p.vec};
    tile::finish<C, GNN_ACT_NONE, T>(acc, ep, k0 + (wave >> 1) * 16 * C::MI, col0 + (wave & 1) * 16 * C::NI, p.k_each);
}

// dA: rows of dZ against W^T, whose rows are the reduction (TB), or against bf16
// rows of W.
struct DaArgs {
    const uint16_t *dz;
    int64_t ldz;
    const int64_t *m_dev;
    int64_t cap_m, n_out, K;
    const uint16_t *w;
    int64_t ldw;
    void *out;
    bool vec;
};

template <class C, class T, bool TB>
__global__ void __launch_bounds__(C::kThreads, C::PER_CU) act_da_kernel(DaArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    const int64_t M = count(p.m_dev, p.cap_m);
    const int64_t tm = ceil_div(M, int64_t(C::BM)), tn = ceil_div(p.K, int64_t(C::BN));
    const int64_t t = wide::xcd_item(blockIdx.x, tm * tn);
    if (t < 0) return;
    int64_t m, n;
    tile::tile_of(t, tm, tn, &m, &n);
    const int64_t row0 = m * C::BM, col0 = n * C::BN;
    const tile::Operand oa{p.dz + row0 * p.ldz, nullptr, p.ldz, p.ldz, M - row0, p.ldz};
    const tile::Operand ob = TB ? tile::Operand{p.w + col0, nullptr, p.ldw, 0, p.ldw - col0, p.n_out}
                                : tile::Operand{p.w + col0 * p.ldw, nullptr, p.ldw, p.ldw, p.K - col0, p.ldw};
    tile::Acc<C> acc;
    acc.clear();
    const tile::Ring ring{{st0, st1}};
    tile::Product<C, false, TB>(oa, ob).run(acc, ring, static_cast<int>(ceil_div(p.ldz, int64_t(tile::kBK))));
    const int wave = threadIdx.x >> 6;
    const tile::Epilogue ep{nullptr, nullptr, nullptr, p.out, p.K, p.vec};
    tile::finish<C, GNN_ACT_NONE, T>(acc, ep, row0 + (wave >> 1) * 16 * C::MI, col0 + (wave & 1) * 16 * C::NI, M);
}

// wb[k][n] = bf16(w[k][n]) for n < n_out, 0 to ld; eight a thread.
__global__ void __launch_bounds__(kThreads) act_w_rows_kernel(const float *w, int64_t K, int64_t n_out, int64_t ld,
                                                              uint16_t *wb) {
    const int64_t groups = ld / 8;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; t < K * groups;
         t += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t k = t / groups, n = (t - k * groups) * 8;
        float v[8];
        get8(w + k * n_out + n, n_out - n, false, v);
        uint4 o;
        o.x = wide::pack_bf16(v[0], v[1]);
        o.y = wide::pack_bf16(v[2], v[3]);
        o.z = wide::pack_bf16(v[4], v[5]);
        o.w = wide::pack_bf16(v[6], v[7]);
        *reinterpret_cast<uint4 *>(wb + k * ld + n) = o;
    }
}

// dW = the splits' partials in their order (when there are any); db = the row
// parts' sums, in a fixed order: a workgroup takes 32 columns, each of its 8 groups
// every eighth part.
template <class T>
__global__ void __launch_bounds__(kThreads) act_reduce_kernel(const float *part, int64_t nsplit, int64_t K, int64_t n_out,
                                                              int64_t ld, T *dw, unsigned db_blocks, const float *db_part,
                                                              int64_t parts, float *db) {
    if (blockIdx.x < db_blocks) {
        __shared__ float sh[8][32];
        const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
        const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + x;
        float t = 0.f;
        if (c < n_out)
#pragma unroll 4
            for (int64_t q = y; q < parts; q += 8) t += db_part[q * n_out + c];
        sh[y][x] = t;
        __syncthreads();
        if (y != 0 || c >= n_out) return;
        t = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += sh[k][x];
        db[c] = t;
        return;
    }
    const int64_t groups = ld / 4;
    for (int64_t t = static_cast<int64_t>(blockIdx.x - db_blocks) * kThreads + threadIdx.x; t < K * groups;
         t += static_cast<int64_t>(gridDim.x - db_blocks) * kThreads) {
        const int64_t k = t / groups, n = (t - k * groups) * 4;
        const float *p = part + k * ld + n;
        tile::f32x4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int64_t q = 0; q < nsplit; ++q) {
            const float4 v = *reinterpret_cast<const float4 *>(p + q * K * ld);
            s[0] += v.x;
            s[1] += v.y;
            s[2] += v.z;
            s[3] += v.w;
        }
        tile::put4(dw + k * n_out + n, static_cast<int>(min(n_out - n, int64_t(4))), n_out % 4 == 0 && aligned_dev(dw, 4 * sizeof(T)), s);
    }
}

struct Plan {
    bool mid;            // dW in 128 x 128 tiles, else 256 x 256
    int64_t nsplit, parts, ldz, ldw, ld_part;
    size_t pack, dz, wb, db_part, part, total;
    Plan(int64_t k_each, bool two, int64_t n_out, int64_t cap_m, bool shadow) {
        const int64_t K = two ? 2 * k_each : k_each, halves = two ? 2 : 1;
        ldz = pack::row8(n_out);
        // dW: large tiles where they fill half the chip or the rows are long
        // enough to split; each split at least 512 rows, one round of the CUs
        auto tiles = [&](int64_t edge) { return halves * ceil_div(k_each, edge) * ceil_div(n_out, edge); };
        mid = tiles(256) < 64;
        const int64_t t = tiles(mid ? 128 : 256), slots = mid ? 512 : 256;
        nsplit = std::max<int64_t>(1, std::min<int64_t>(slots / t, ceil_div(cap_m, int64_t(512))));
        // dZ: about four workgroups to a CU, at least 32 rows each
        const int64_t stripes = ceil_div(ldz, int64_t(kStripe));
        parts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(2048, stripes), ceil_div(cap_m, int64_t(32))));
        ldw = ldz;
        ld_part = (n_out + 3) / 4 * 4;
        Carver c(nullptr);
        pack = c.take(pack::Layout(cap_m, K, n_out).total);
        dz = c.take(static_cast<size_t>(cap_m * ldz * 2));
        wb = c.take(shadow ? 0 : static_cast<size_t>(K * ldw * 2));
        db_part = c.take(static_cast<size_t>(parts * n_out * 4));
        part = c.take(nsplit > 1 ? static_cast<size_t>(nsplit * K * ld_part * 4) : 0);
        total = round_up(c.off, 256);
    }
};

template <class C> gnn_status launch_dw(const DwArgs &p, int odt, hipStream_t s) {
    const int64_t tiles = (p.a1 ? 2 : 1) * ceil_div(p.k_each, int64_t(C::BM)) * ceil_div(p.n_out, int64_t(C::BN));
    const unsigned grid = static_cast<unsigned>(round_up(tiles * p.nsplit, wide::kXcds));
    if (odt == GNN_BF16) act_dw_kernel<C, uint16_t><<<grid, C::kThreads, 0, s>>>(p);
    else act_dw_kernel<C, float><<<grid, C::kThreads, 0, s>>>(p);
    GNN_LAUNCHED("update_bwd_act_dw");
    return GNN_OK;
}

template <class C> gnn_status launch_da(const DaArgs &p, int odt, bool shadow, hipStream_t s) {
    const int64_t tiles = ceil_div(p.cap_m, int64_t(C::BM)) * ceil_div(p.K, int64_t(C::BN)), grid64 = round_up(tiles, wide::kXcds);
    GNN_CHECK(grid64 <= kMaxGrid / C::kThreads, GNN_ESIZE, "update_bwd_act: cap_m exceeds the grid limit");
    const unsigned grid = static_cast<unsigned>(grid64);
    if (odt == GNN_BF16) {
        if (shadow) act_da_kernel<C, uint16_t, true><<<grid, C::kThreads, 0, s>>>(p);
        else act_da_kernel<C, uint16_t, false><<<grid, C::kThreads, 0, s>>>(p);
    } else {
        if (shadow) act_da_kernel<C, float, true><<<grid, C::kThreads, 0, s>>>(p);
        else act_da_kernel<C, float, false><<<grid, C::kThreads, 0, s>>>(p);
    }
    GNN_LAUNCHED("update_bwd_act_da");
    return GNN_OK;
}

gnn_status launch_tiles(const ActBwd &a, void *ws, hipStream_t s) {
    const int64_t K = a.K();
    const Plan pl(a.k_each, a.a_nbr != nullptr, a.n_out, a.cap_m, a.wt != nullptr);
    char *base = static_cast<char *>(ws);
    pack::Operands o;
    GNN_TRY(pack::prepare(a, 8, a.d_a && a.wt, base + pl.pack, &o, s));
    DzArgs z{};
    z.g = a.g;
    z.z = a.z;
    z.m_dev = a.m_dev;
    z.cap_m = a.cap_m;
    z.n_out = a.n_out;
    z.dz = reinterpret_cast<uint16_t *>(base + pl.dz);
    z.ld = pl.ldz;
    z.part = a.db ? reinterpret_cast<float *>(base + pl.db_part) : nullptr;
    z.parts = pl.parts;
    z.vec = a.n_out % 4 == 0 && aligned(a.g, 4 * dtype_size(a.gdt)) && aligned(a.z, 4 * dtype_size(a.zdt));
    const unsigned dz_grid = static_cast<unsigned>(ceil_div(pl.ldz, int64_t(kStripe)) * pl.parts);
    act::with(a.act, [&](auto code) {
        with_types(a.gdt, a.zdt, [&](auto tg, auto tz) {
            act_dz_kernel<decltype(code)::value, decltype(tg), decltype(tz)><<<dz_grid, kThreads, 0, s>>>(z);
        });
    });
    GNN_LAUNCHED("update_bwd_act_dz");
    // dW, straight into its own type unless the rows are split
    const bool split = pl.nsplit > 1;
    DwArgs w{};
    w.a0 = o.a0;
    w.a1 = o.a1;
    w.k_each = o.a1 ? o.k_each : K;
    w.lda = o.lda;
    w.dz = z.dz;
    w.ldz = pl.ldz;
    w.m_dev = a.m_dev;
    w.cap_m = a.cap_m;
    w.n_out = a.n_out;
    w.nsplit = pl.nsplit;
    float *part = reinterpret_cast<float *>(base + pl.part);
    w.out = split ? part : a.dw;
    w.ld = split ? pl.ld_part : a.n_out;
    w.split_stride = split ? K * pl.ld_part : 0;
    w.vec = split || (a.n_out % 4 == 0 && aligned(a.dw, 4 * dtype_size(a.dwdt)));
    const int wdt = split ? static_cast<int>(GNN_F32) : a.dwdt;
    if (pl.mid) GNN_TRY(launch_dw<tile::Mid>(w, wdt, s));
    else GNN_TRY(launch_dw<tile::Big>(w, wdt, s));
    if (split || a.db) {
        const unsigned db_blocks = a.db ? static_cast<unsigned>(ceil_div(a.n_out, int64_t(32))) : 0;
        const unsigned dw_blocks = split ? static_cast<unsigned>(std::min<int64_t>(ceil_div(K * (pl.ld_part / 4), int64_t(kThreads)), 4096)) : 0;
        if (a.dwdt == GNN_BF16)
            act_reduce_kernel<uint16_t><<<db_blocks + dw_blocks, kThreads, 0, s>>>(
                part, pl.nsplit, K, a.n_out, pl.ld_part, static_cast<uint16_t *>(a.dw), db_blocks, z.part, pl.parts, a.db);
        else
            act_reduce_kernel<float><<<db_blocks + dw_blocks, kThreads, 0, s>>>(
                part, pl.nsplit, K, a.n_out, pl.ld_part, static_cast<float *>(a.dw), db_blocks, z.part, pl.parts, a.db);
        GNN_LAUNCHED("update_bwd_act_reduce");
    }
    if (!a.d_a) return GNN_OK;
    DaArgs d{};
    d.dz = z.dz;
    d.ldz = pl.ldz;
    d.m_dev = a.m_dev;
    d.cap_m = a.cap_m;
    d.n_out = a.n_out;
    d.K = K;
    d.w = o.wt;
    d.ldw = o.ldw;
    if (!a.wt) {
        uint16_t *wb = reinterpret_cast<uint16_t *>(base + pl.wb);
        act_w_rows_kernel<<<grid_of(K * (pl.ldw / 8)), kThreads, 0, s>>>(a.w, K, a.n_out, pl.ldw, wb);
        GNN_LAUNCHED("update_bwd_act_w");
        d.w = wb;
        d.ldw = pl.ldw;
    }
    d.out = a.d_a;
    d.vec = K % 4 == 0 && aligned(a.d_a, 4 * dtype_size(a.gdt));
    switch (tile::pick(a.cap_m, K)) {
        case tile::kBig:
        case tile::kBig7: return launch_da<tile::Big>(d, a.gdt, a.wt != nullptr, s);
        case tile::kMid: return launch_da<tile::Mid>(d, a.gdt, a.wt != nullptr, s);
        default: return launch_da<tile::Small>(d, a.gdt, a.wt != nullptr, s);
    }
}

}  // namespace

size_t act_bwd_ws_bytes(int, int64_t k_each, bool two, int64_t n_out, int64_t cap_m, int gdt, int dwdt, int gemm_dt,
                        bool shadow) {
    const int64_t K = two ? 2 * k_each : k_each;
    if (pack::small(cap_m, K, n_out, gemm_dt)) return EngineLayout(K, n_out, cap_m, gdt, dwdt, gemm_dt, shadow).total;
    return Plan(k_each, two, n_out, cap_m, shadow).total;
}

gnn_status launch_act_bwd(const ActBwd &a, void *ws, hipStream_t s) {
    if (pack::small(a.cap_m, a.K(), a.n_out, a.gemm_dt)) return launch_engine(a, ws, s);
    return launch_tiles(a, ws, s);
}

}  // namespace gnn
