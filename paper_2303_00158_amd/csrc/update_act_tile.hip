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
};

template <class C, int ACT, class T>
__global__ void __launch_bounds__(C::kThreads, C::PER_CU) act_tile_kernel(TileArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    const int64_t M = p.m_dev ? min(*p.m_dev, p.cap_m) : p.cap_m;
    const int64_t tm = ceil_div(M, int64_t(C::BM)), tn = ceil_div(p.ep.ld, int64_t(C::BN));
    const int64_t t = wide::xcd_item(blockIdx.x, tm * tn);
    if (t < 0) return;
    int64_t m, n;
    tile::tile_of(t, tm, tn, &m, &n);
    const int64_t row0 = m * C::BM, col0 = n * C::BN;
    const tile::Operand oa{p.a0 + row0 * p.lda, p.a1 ? p.a1 + row0 * p.lda : nullptr, p.lda, p.k_each, M - row0, p.K};
    const tile::Operand ob{p.wt + col0 * p.ldw, nullptr, p.ldw, p.K, p.ep.ld - col0, p.K};
    tile::Acc<C> acc;
    acc.clear();
    const tile::Ring ring{{st0, st1}};
    tile::Product<C, false, false>(oa, ob).run(acc, ring, static_cast<int>(ceil_div(p.K, int64_t(tile::kBK))));
    const int wave = threadIdx.x >> 6;
    tile::finish<C, ACT, T>(acc, p.ep, row0 + (wave >> 1) * 16 * C::MI, col0 + (wave & 1) * 16 * C::NI, M);
}

template <class C> gnn_status launch_tiles(const ActFwd &a, const TileArgs &p, hipStream_t s) {
    const int64_t tiles = ceil_div(p.cap_m, int64_t(C::BM)) * ceil_div(p.ep.ld, int64_t(C::BN));
    const int64_t grid = round_up(tiles, wide::kXcds);
    GNN_CHECK(grid <= kMaxGrid / C::kThreads, GNN_ESIZE, "update_fwd_act: cap_m exceeds the grid limit");
    act::with(a.act, [&](auto code) {
        constexpr int ACT = decltype(code)::value;
        if (a.odt == GNN_BF16) act_tile_kernel<C, ACT, uint16_t><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
        else act_tile_kernel<C, ACT, float><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
    });
    GNN_LAUNCHED("update_fwd_act");
    return GNN_OK;
}

}  // namespace

size_t act_fwd_ws_bytes(int, int64_t k_each, bool two, int64_t n_out, int64_t cap_m, int gemm_dt, bool shadow) {
    if (act_few(cap_m, gemm_dt, shadow) || pack::small(cap_m, two ? 2 * k_each : k_each, n_out, gemm_dt)) return 0;
    return pack::Layout(cap_m, two ? 2 * k_each : k_each, n_out).total;
}

gnn_status launch_act_fwd(const ActFwd &a, void *ws, hipStream_t s) {
    if (a.cap_m == 0) return GNN_OK;
    const int64_t K = a.K();
    if (act_few(a.cap_m, a.gemm_dt, a.wt != nullptr)) return launch_act_few(a, s);
    if (pack::small(a.cap_m, K, a.n_out, a.gemm_dt)) return launch_act_engine(a, s);
    pack::Operands o;
    GNN_TRY(pack::prepare(a, tile::kBK, true, ws, &o, s));
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
    const size_t osz = dtype_size(a.odt);
    p.ep = tile::Epilogue{a.bias, a.residual, a.z, a.out, a.n_out,
                          a.n_out % 4 == 0 && aligned(a.residual, 4 * osz) && aligned(a.z, 4 * osz) && aligned(a.out, 4 * osz)};
    switch (tile::pick(a.cap_m, a.n_out)) {
        case tile::kBig: return launch_tiles<tile::Big>(a, p, s);
        case tile::kBig7: return launch_tiles<tile::Big7>(a, p, s);
        case tile::kMid: return launch_tiles<tile::Mid>(a, p, s);
        default: return launch_tiles<tile::Small>(a, p, s);
    }
}

}  // namespace gnn
