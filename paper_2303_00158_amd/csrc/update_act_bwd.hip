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
// dZ is an operand of bf16 products, so it is rounded before them: with A or W^T
// exact in bf16, dW and dA are then off by 0.0023 in the root mean square (8,192 x 4,096 x
// 4,096), where the rounding of a bf16 output alone is 0.0017.
// fp32 products take the update's own kernels (gemm_bwd.hip) on an fp32 dZ.
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

struct EngineLayout {
    size_t dz, gemm, total;
    EngineLayout(int64_t K, int64_t n_out, int64_t cap_m) {
        Carver c(nullptr);
        dz = c.take(static_cast<size_t>(cap_m * n_out * 4));
        gemm = c.take(update_bwd_ws_bytes(K, n_out, cap_m, GNN_F32));
        total = round_up(c.off, 256);
    }
};

// fp32 products: every operand but A and Z is fp32.
gnn_status launch_engine(const ActBwd &a, void *ws, hipStream_t s) {
    const EngineLayout l(a.K(), a.n_out, a.cap_m);
    char *base = static_cast<char *>(ws);
    float *dz = reinterpret_cast<float *>(base + l.dz);
    const float *g = static_cast<const float *>(a.g);
    if (a.cap_m > 0 && a.act != GNN_ACT_NONE) {
        const unsigned grid = grid_of(a.cap_m * a.n_out);
        act::with(a.act, [&](auto code) {
            constexpr int ACT = decltype(code)::value;
            if (a.zdt == GNN_BF16)
                act_slope_kernel<ACT, float, uint16_t><<<grid, kThreads, 0, s>>>(g, static_cast<const uint16_t *>(a.z), a.m_dev,
                                                                                 a.cap_m, a.n_out, dz);
            else
                act_slope_kernel<ACT, float, float><<<grid, kThreads, 0, s>>>(g, static_cast<const float *>(a.z), a.m_dev,
                                                                              a.cap_m, a.n_out, dz);
        });
        GNN_LAUNCHED("act_slope");
        g = dz;
    }
    return launch_update_bwd(a.a_self, a.a_nbr, a.adt, a.k_each, a.m_dev, a.cap_m, a.w, g, a.n_out, GNN_F32,
                             static_cast<float *>(a.dw), a.db, static_cast<float *>(a.d_a), base + l.gemm, nullptr, nullptr,
                             nullptr, 0.f, s);
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
};

template <class T> __device__ __forceinline__ void get8(const T *p, int64_t room, float (&v)[8]) {
    if (room >= 8) {
        row::Vec<T, 8> x;
        x.load(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x.get(e);
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
#pragma unroll 4
        for (int64_t i = beg + y; i < end; i += 8) {
            float v[8];
            get8(g + i * p.n_out, room, v);
            if constexpr (ACT != GNN_ACT_NONE) {
                float zz[8];
                get8(z + i * p.n_out, room, zz);
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
    const tile::Epilogue ep{nullptr, nullptr, nullptr, out, p.ld};
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
    int64_t ld, split_stride, nsplit;
};

template <class C, class T, bool TB>
__global__ void __launch_bounds__(C::kThreads, C::PER_CU) act_da_kernel(DaArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    const int64_t M = count(p.m_dev, p.cap_m);
    const int64_t tm = ceil_div(M, int64_t(C::BM)), tn = ceil_div(p.K, int64_t(C::BN));
    const int64_t item = wide::xcd_item(blockIdx.x, tm * tn * p.nsplit);
    if (item < 0) return;
    const int64_t split = item / (tm * tn);
    int64_t m, n, beg, end;
    tile::tile_of(item - split * (tm * tn), tm, tn, &m, &n);
    tile::split_of(p.ldz, p.nsplit, split, &beg, &end);
    const int64_t row0 = m * C::BM, col0 = n * C::BN, red = end - beg;
    const tile::Operand oa{p.dz + row0 * p.ldz + beg, nullptr, p.ldz, 0, M - row0, red};
    const tile::Operand ob = TB ? tile::Operand{p.w + beg * p.ldw + col0, nullptr, p.ldw, 0, p.ldw - col0, min(end, p.n_out) - beg}
                                : tile::Operand{p.w + col0 * p.ldw + beg, nullptr, p.ldw, 0, p.K - col0, red};
    tile::Acc<C> acc;
    acc.clear();
    const tile::Ring ring{{st0, st1}};
    if (red > 0)
        tile::Product<C, false, TB>(oa, ob).run(acc, ring, static_cast<int>(ceil_div(red, int64_t(tile::kBK))));
    const int wave = threadIdx.x >> 6;
    const tile::Epilogue ep{nullptr, nullptr, nullptr, static_cast<T *>(p.out) + split * p.split_stride, p.ld};
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
        get8(w + k * n_out + n, n_out - n, v);
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
struct ReduceArgs {
    const float *part;   // nsplit partials of `rows` x ld; of them the rows counted by m_dev are summed
    int64_t nsplit, rows, cols, ld;
    const int64_t *m_dev;
    void *out;
    const float *db_part;
    int64_t parts, n_out;
    float *db;
    unsigned db_blocks;
};
template <class T> __global__ void __launch_bounds__(kThreads) act_reduce_kernel(ReduceArgs a) {
    const float *db_part = a.db_part;
    const int64_t n_out = a.n_out, parts = a.parts;
    if (blockIdx.x < a.db_blocks) {
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
        a.db[c] = t;
        return;
    }
    const int64_t groups = a.ld / 4, rows = count(a.m_dev, a.rows);
    for (int64_t t = static_cast<int64_t>(blockIdx.x - a.db_blocks) * kThreads + threadIdx.x; t < rows * groups;
         t += static_cast<int64_t>(gridDim.x - a.db_blocks) * kThreads) {
        const int64_t r = t / groups, c = (t - r * groups) * 4;
        const float *p = a.part + r * a.ld + c;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int64_t q = 0; q < a.nsplit; ++q) {
            const float4 v = *reinterpret_cast<const float4 *>(p + q * a.rows * a.ld);
            s[0] += v.x;
            s[1] += v.y;
            s[2] += v.z;
            s[3] += v.w;
        }
        T *out = static_cast<T *>(a.out) + r * a.cols + c;
        if (a.cols - c >= 4) {
            row::Vec<T, 4> v;
            v.set(s);
            v.store(out);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < a.cols - c) Elem<T>::store(out, e, s[e]);
        }
    }
}

gnn_status launch_reduce(const ReduceArgs &a, int odt, bool sums, hipStream_t s) {
    const unsigned blocks = sums ? static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(a.rows * (a.ld / 4), int64_t(kThreads)), 4096))) : 0;
    if (odt == GNN_BF16) act_reduce_kernel<uint16_t><<<a.db_blocks + blocks, kThreads, 0, s>>>(a);
    else act_reduce_kernel<float><<<a.db_blocks + blocks, kThreads, 0, s>>>(a);
    GNN_LAUNCHED("update_bwd_act_reduce");
    return GNN_OK;
}

struct Plan {
    bool mid;            // dW in 128 x 128 tiles, else 256 x 256
    int64_t nsplit, parts, ldz, ldw, ld_part, ld_a;
    tile::Choice da;
    size_t pack, dz, wb, db_part, part, a_part, total;
    Plan(int64_t k_each, bool two, int64_t n_out, int64_t cap_m, bool shadow) {
        const int64_t K = two ? 2 * k_each : k_each, halves = two ? 2 : 1;
        ldz = pack::row8(n_out);
        da = tile::choose(cap_m, K, ldz);
        ld_a = (K + 3) / 4 * 4;
        // dW: the tile size and the split of the rows that take the least time, as
        // tile::choose has it, with at least four chunks a split; 128 x 128 tiles read
        // twice as many T fragments a multiplication and are slower than their
        // pace there, and the partials come back from the last-level cache.  With dZ,
        // us in 256 x 256 and in 128 x 128 tiles: 8,192 x 1,024 x 1,024 54 and 44, 26,624 x
        // 1,024 x 1,024 99 and 108, 8,192 x 2,048 x 2,048 91 and 96, 4,096 x 2,048 x 4,096 92
        // and 80, 16,384 x 256 x 256 43 and 29.
        const int64_t chunks = std::max<int64_t>(ceil_div(cap_m, int64_t(tile::kBK)), 1);
        double least = -1;
        auto look = [&](auto cfg, bool is_mid, const tile::Pace &pace) {
            using C = decltype(cfg);
            const int64_t t = halves * ceil_div(k_each, int64_t(C::BM)) * ceil_div(n_out, int64_t(C::BN));
            for (int64_t n = 1; n == 1 || (n * t <= 256 * C::PER_CU && n * 4 <= chunks); n *= 2) {
                const double us = tile::cost<C>(t, chunks, n, pace) + (n > 1 ? 4 + static_cast<double>(n) * K * n_out * 8 / 8e6 : 0);
                if (least < 0 || us < least) {
                    least = us;
                    mid = is_mid;
                    nsplit = n;
                }
            }
        };
        look(tile::Big{}, false, tile::kBigPace);
        look(tile::Mid{}, true, tile::Pace{0.62, 0.8, 4});
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
        a_part = c.take(da.nsplit > 1 ? static_cast<size_t>(da.nsplit * cap_m * ld_a * 4) : 0);
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
    const int64_t tiles = ceil_div(p.cap_m, int64_t(C::BM)) * ceil_div(p.K, int64_t(C::BN));
    const int64_t grid64 = round_up(tiles * p.nsplit, wide::kXcds);
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
    const int wdt = split ? static_cast<int>(GNN_F32) : a.dwdt;
    if (pl.mid) GNN_TRY(launch_dw<tile::Mid>(w, wdt, s));
    else GNN_TRY(launch_dw<tile::Big>(w, wdt, s));
    if (split || a.db) {
        ReduceArgs r{part, pl.nsplit, K, a.n_out, pl.ld_part, nullptr, a.dw, z.part, pl.parts, a.n_out, a.db, 0};
        r.db_blocks = a.db ? static_cast<unsigned>(ceil_div(a.n_out, int64_t(32))) : 0;
        GNN_TRY(launch_reduce(r, a.dwdt, split, s));
    }
    if (!a.d_a || a.cap_m == 0) return GNN_OK;
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
    float *a_part = reinterpret_cast<float *>(base + pl.a_part);
    const bool a_split = pl.da.nsplit > 1;
    d.out = a_split ? static_cast<void *>(a_part) : a.d_a;
    d.ld = a_split ? pl.ld_a : K;
    d.nsplit = pl.da.nsplit;
    d.split_stride = a_split ? a.cap_m * pl.ld_a : 0;
    const int adt = a_split ? static_cast<int>(GNN_F32) : a.gdt;
    switch (pl.da.pick) {
        case tile::kBig: GNN_TRY(launch_da<tile::Big>(d, adt, a.wt != nullptr, s)); break;
        case tile::kBig7: GNN_TRY(launch_da<tile::Big7>(d, adt, a.wt != nullptr, s)); break;
        case tile::kMid: GNN_TRY(launch_da<tile::Mid>(d, adt, a.wt != nullptr, s)); break;
        default: GNN_TRY(launch_da<tile::Small>(d, adt, a.wt != nullptr, s));
    }
    if (!a_split) return GNN_OK;
    return launch_reduce(ReduceArgs{a_part, pl.da.nsplit, a.cap_m, K, pl.ld_a, a.m_dev, a.d_a, nullptr, 0, 0, nullptr, 0}, a.gdt,
                         true, s);
}

}  // namespace

size_t act_bwd_ws_bytes(int, int64_t k_each, bool two, int64_t n_out, int64_t cap_m, int, int, int gemm_dt, bool shadow) {
    if (gemm_dt != GNN_BF16) return EngineLayout(two ? 2 * k_each : k_each, n_out, cap_m).total;
    return Plan(k_each, two, n_out, cap_m, shadow).total;
}

gnn_status launch_act_bwd(const ActBwd &a, void *ws, hipStream_t s) {
    return a.gemm_dt == GNN_BF16 ? launch_tiles(a, ws, s) : launch_engine(a, ws, s);
}

}  // namespace gnn
