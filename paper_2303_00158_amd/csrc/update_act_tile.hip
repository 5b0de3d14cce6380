// The update with an activation and a residual on the tiles of
// gemm_tile_dev.h, and the layout of bf16 operands that they read.
#include "act_pack.h"
#include "gemm_tile_dev.h"
#include "update_act_few.h"

namespace gnn {

namespace {

struct TileArgs {
    const uint16_t *a0, *a1;  // A = [a0 || a1], rows of k_each bf16 values each
    int64_t k_each, K, lda;
    const int64_t *m_dev;
    int64_t cap_m;
    const uint16_t *wt;       // W^T, n_out rows of K values, ldw apart
    int64_t ldw;
    tile::Epilogue ep;
    float *part;              // partial tiles of a split reduction, or null
    int64_t nsplit, part_ld;
};

// Tile of this workgroup and its split of the reduction; false: none.
template <class C> struct Place {
    int64_t M, row0, col0, beg, end, split;
    __device__ __forceinline__ bool find(const TileArgs &p) {
        M = p.m_dev ? max(min(*p.m_dev, p.cap_m), int64_t(0)) : p.cap_m;
        const int64_t tm = ceil_div(M, int64_t(C::BM)), tn = ceil_div(p.ep.ld, int64_t(C::BN));
        const int64_t t = wide::xcd_item(blockIdx.x, tm * tn * p.nsplit);
        if (t < 0) return false;
        split = t / (tm * tn);
        int64_t m, n;
        tile::tile_of(t - split * (tm * tn), tm, tn, &m, &n);
        row0 = m * C::BM;
        col0 = n * C::BN;
        tile::split_of(p.K, p.nsplit, split, &beg, &end);
        return true;
    }
};

template <class C> __device__ __forceinline__ void tile_product(const TileArgs &p, const Place<C> &at, const tile::Ring &ring, tile::Acc<C> &acc) {
    // a split's part of [a0 || a1] starts in one half and may end in the other
    const bool hi = p.a1 && at.beg >= p.k_each;
    const int64_t off = at.row0 * p.lda + (hi ? at.beg - p.k_each : at.beg);
    const tile::Operand oa{(hi ? p.a1 : p.a0) + off, p.a1 && !hi ? p.a1 + at.row0 * p.lda : nullptr, p.lda,
                           p.a1 && !hi ? p.k_each - at.beg : at.end - at.beg, at.M - at.row0, at.end - at.beg};
    const tile::Operand ob{p.wt + at.col0 * p.ldw + at.beg, nullptr, p.ldw, 0, p.ep.ld - at.col0, at.end - at.beg};
    acc.clear();
    if (at.end > at.beg)
        tile::Product<C, false, false>(oa, ob).run(acc, ring, static_cast<int>(ceil_div(at.end - at.beg, int64_t(tile::kBK))));
}

template <class C, int ACT, class T>
__global__ void __launch_bounds__(C::kThreads, C::PER_CU) act_tile_kernel(TileArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    Place<C> at;
    if (!at.find(p)) return;
    tile::Acc<C> acc;
    tile_product<C>(p, at, tile::Ring{{st0, st1}}, acc);
    const int wave = threadIdx.x >> 6;
    tile::finish<C, ACT, T>(acc, p.ep, at.row0 + (wave >> 1) * 16 * C::MI, at.col0 + (wave & 1) * 16 * C::NI, at.M);
}

// The same for a split's partial tile.
template <class C> __global__ void __launch_bounds__(C::kThreads, C::PER_CU) act_tile_part_kernel(TileArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    Place<C> at;
    if (!at.find(p)) return;
    tile::Acc<C> acc;
    tile_product<C>(p, at, tile::Ring{{st0, st1}}, acc);
    const int wave = threadIdx.x >> 6;
    const tile::Epilogue ep{nullptr, nullptr, nullptr, p.part + at.split * p.cap_m * p.part_ld, p.part_ld};
    tile::finish<C, GNN_ACT_NONE, float>(acc, ep, at.row0 + (wave >> 1) * 16 * C::MI, at.col0 + (wave & 1) * 16 * C::NI, at.M);
}

template <class C> gnn_status launch_tiles(const ActFwd &a, const TileArgs &p, hipStream_t s) {
    const int64_t tiles = ceil_div(p.cap_m, int64_t(C::BM)) * ceil_div(p.ep.ld, int64_t(C::BN));
    const int64_t grid = round_up(tiles * p.nsplit, wide::kXcds);
    GNN_CHECK(grid <= kMaxGrid / C::kThreads, GNN_ESIZE, "update_fwd_act: cap_m exceeds the grid limit");
    if (p.nsplit > 1) {
        act_tile_part_kernel<C><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
        GNN_LAUNCHED("update_fwd_act_part");
        return launch_act_finish(a, p.part, p.nsplit, p.part_ld, s);
    }
    act::with(a.act, [&](auto code) {
        constexpr int ACT = decltype(code)::value;
        if (a.odt == GNN_BF16) act_tile_kernel<C, ACT, uint16_t><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
        else act_tile_kernel<C, ACT, float><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
    });
    GNN_LAUNCHED("update_fwd_act");
    return GNN_OK;
}

struct Plan {
    tile::Choice choice;
    int64_t part_ld;
    size_t pack, part, total;
    Plan(int64_t cap_m, int64_t K, int64_t n_out) : choice(tile::choose(cap_m, n_out, K)), part_ld((n_out + 3) / 4 * 4) {
        Carver c(nullptr);
        pack = c.take(pack::Layout(cap_m, K, n_out).total);
        part = c.take(choice.nsplit > 1 ? static_cast<size_t>(choice.nsplit * cap_m * part_ld * 4) : 0);
        total = round_up(c.off, 256);
    }
};

}  // namespace

size_t act_fwd_ws_bytes(int, int64_t k_each, bool two, int64_t n_out, int64_t cap_m, int gemm_dt, bool shadow) {
    const int64_t K = two ? 2 * k_each : k_each;
    if (act_few(cap_m, K, gemm_dt, shadow)) return 0;
    // whether operands are copied goes by their addresses too
    const size_t engine = pack::small(cap_m, K, n_out, gemm_dt, true) ? act_engine_ws_bytes(K, n_out, cap_m, gemm_dt) : 0;
    return pack::small(cap_m, K, n_out, gemm_dt, false) ? engine : std::max(engine, Plan(cap_m, K, n_out).total);
}

gnn_status launch_act_fwd(const ActFwd &a, void *ws, hipStream_t s) {
    if (a.cap_m == 0) return GNN_OK;
    const int64_t K = a.K();
    if (act_few(a.cap_m, K, a.gemm_dt, a.wt != nullptr)) return launch_act_few(a, s);
    if (pack::small(a.cap_m, K, a.n_out, a.gemm_dt, pack::copies_a(a, tile::kBK) || pack::copies_w(a)))
        return launch_act_engine(a, ws, s);
    const Plan pl(a.cap_m, K, a.n_out);
    pack::Operands o;
    GNN_TRY(pack::prepare(a, tile::kBK, true, static_cast<char *>(ws) + pl.pack, &o, s));
    TileArgs p{};
    p.a0 = o.a0;
    p.a1 = o.a1;
    p.k_each = o.k_each;
    p.K = o.K;
    p.lda = o.lda;
    p.m_dev = a.m_dev;
    p.cap_m = a.cap_m;
    p.wt = o.wt;
    p.ldw = o.ldw;
    p.ep = tile::Epilogue{a.bias, a.residual, a.z, a.out, a.n_out};
    p.part = reinterpret_cast<float *>(static_cast<char *>(ws) + pl.part);
    p.nsplit = pl.choice.nsplit;
    p.part_ld = pl.part_ld;
    switch (pl.choice.pick) {
        case tile::kBig: return launch_tiles<tile::Big>(a, p, s);
        case tile::kBig7: return launch_tiles<tile::Big7>(a, p, s);
        case tile::kMid: return launch_tiles<tile::Mid>(a, p, s);
        default: return launch_tiles<tile::Small>(a, p, s);
    }
}

}  // namespace gnn
