// bf16 products of the loss over many classes, on the tiles of gemm_tile_dev.h.
#include "class_loss.h"
#include "gemm_tile_dev.h"

namespace gnn {
namespace closs {

namespace {

template <class C, bool TX, bool TY, class T>
__global__ void __launch_bounds__(C::kThreads, C::PER_CU) class_product_kernel(Product p) {
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    const int64_t tm = ceil_div(p.M, int64_t(C::BM)), tn = ceil_div(p.N, int64_t(C::BN));
    const int64_t item = wide::xcd_item(blockIdx.x, tm * tn * p.nsplit);
    if (item < 0) return;
    const int64_t split = item / (tm * tn);
    int64_t m, n, beg, end;
    tile::tile_of(item - split * (tm * tn), tm, tn, &m, &n);
    tile::split_of(p.R, p.nsplit, split, &beg, &end);
    const int64_t row0 = m * C::BM, col0 = n * C::BN, red = end - beg;
    const uint16_t *x = static_cast<const uint16_t *>(p.x), *y = static_cast<const uint16_t *>(p.y);
    const tile::Operand ox = TX ? tile::Operand{x + beg * p.ldx + row0, nullptr, p.ldx, 0, p.ldx - row0, red}
                                : tile::Operand{x + row0 * p.ldx + beg, nullptr, p.ldx, 0, p.M - row0, red};
    const tile::Operand oy = TY ? tile::Operand{y + beg * p.ldy + col0, nullptr, p.ldy, 0, p.ldy - col0, min(end, p.Ry) - beg}
                                : tile::Operand{y + col0 * p.ldy + beg, nullptr, p.ldy, 0, p.N - col0, red};
    tile::Acc<C> acc;
    acc.clear();
    const tile::Ring ring{{st0, st1}};
    if (red > 0) tile::Product<C, TX, TY>(ox, oy).run(acc, ring, static_cast<int>(ceil_div(red, int64_t(tile::kBK))));
    const int wave = threadIdx.x >> 6;
    T *out = static_cast<T *>(p.out) + split * p.split_stride;
    // (rows are `ld` long in memory and the output's N columns are all stored up to there)
    const tile::Epilogue ep{nullptr, p.add ? out : nullptr, nullptr, out, p.ld};
    tile::finish<C, GNN_ACT_NONE, T>(acc, ep, row0 + (wave >> 1) * 16 * C::MI, col0 + (wave & 1) * 16 * C::NI, p.M);
}

tile::Choice choice(Kind kind, int64_t M, int64_t N, int64_t R, bool may_split) {
    if (kind != kTT) return tile::choose(M, N, R, may_split ? 16 : 1);
    // T fragments take twice the reads: 128 x 128 tiles are slower than their pace, and smaller ones are not worth it
    tile::Choice best{tile::kMid, 1};
    double least = -1;
    const int64_t chunks = std::max<int64_t>(ceil_div(R, int64_t(tile::kBK)), 1);
    auto look = [&](auto cfg, tile::Pick pick, const tile::Pace &pace) {
        using C = decltype(cfg);
        const int64_t t = ceil_div(M, int64_t(C::BM)) * ceil_div(N, int64_t(C::BN));
        for (int64_t n = 1; n == 1 || (may_split && n <= 64 && n * t <= 256 * C::PER_CU && n * 4 <= chunks); n *= 2) {
            const double us = tile::cost<C>(t, chunks, n, pace) + (n > 1 ? 4 + static_cast<double>(n) * M * N * 8 / 8e6 : 0);
            if (least < 0 || us < least) {
                least = us;
                best = tile::Choice{pick, n};
            }
        }
    };
    look(tile::Big{}, tile::kBig, tile::kBigPace);
    look(tile::Mid{}, tile::kMid, tile::Pace{0.62, 0.8, 4});
    return best;
}

template <class C, bool TX, bool TY> gnn_status launch(const Product &p, hipStream_t s) {
    const int64_t tiles = ceil_div(p.M, int64_t(C::BM)) * ceil_div(p.N, int64_t(C::BN));
    const int64_t grid = static_cast<int64_t>(round_up(tiles * p.nsplit, wide::kXcds));
    GNN_CHECK(grid <= kMaxGrid / C::kThreads, GNN_ESIZE, "update_ce: sizes exceed the grid limit");
    if (p.odt == GNN_BF16) class_product_kernel<C, TX, TY, uint16_t><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
    else class_product_kernel<C, TX, TY, float><<<static_cast<unsigned>(grid), C::kThreads, 0, s>>>(p);
    GNN_LAUNCHED("update_ce_product");
    return GNN_OK;
}

}  // namespace

int64_t splits_bf16(Kind kind, int64_t M, int64_t N, int64_t R, bool may_split) { return choice(kind, M, N, R, may_split).nsplit; }

gnn_status product_bf16(Kind kind, const Product &p, hipStream_t s) {
    const tile::Pick pick = choice(kind, p.M, p.N, p.R, p.nsplit > 1).pick;
    if (kind == kTT) return pick == tile::kBig ? launch<tile::Big, true, true>(p, s) : launch<tile::Mid, true, true>(p, s);
    auto go = [&](auto ty) -> gnn_status {
        constexpr bool TY = decltype(ty)::value;
        switch (pick) {
            case tile::kBig: return launch<tile::Big, false, TY>(p, s);
            case tile::kBig7: return launch<tile::Big7, false, TY>(p, s);
            case tile::kMid: return launch<tile::Mid, false, TY>(p, s);
            default: return launch<tile::Small, false, TY>(p, s);
        }
    };
    return kind == kNT ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace closs
}  // namespace gnn
