// fp32 products of the loss over many classes, on the general engine.
#include "class_loss.h"
#include "gemm_engine.h"

namespace gnn {
namespace closs {

namespace {

using namespace gemm;

template <int TILE, bool T> struct Source {
    using type = SrcRows<false, TILE, float, true, depth<TILE>()>;
    __device__ static type make(const void *p, int64_t ld, int64_t out, int64_t, int64_t r_cols, int64_t at) {
        return type{static_cast<const float *>(p), nullptr, ld, ld, out, r_cols, at, {}};
    }
};
template <int TILE> struct Source<TILE, true> {
    using type = SrcCols<false, TILE, float, true, depth<TILE>()>;
    __device__ static type make(const void *p, int64_t ld, int64_t, int64_t r_end, int64_t, int64_t at) {
        return type{static_cast<const float *>(p), nullptr, ld, ld, ld, r_end, at, {}};
    }
};

template <int TILE, bool TX, bool TY> __global__ void __launch_bounds__(gemm::kThreads) class_engine_kernel(Product p, TileMap map) {
    constexpr int D = depth<TILE>();
    __shared__ __attribute__((aligned(16))) char lds[lds_bytes<TILE, TILE>()];
    int64_t tx, ty;
    map.tile_of(blockIdx.x, &tx, &ty);
    const int64_t row0 = tx * TILE, col0 = ty * TILE;
    if (tx >= map.mt) return;
    int64_t beg, end;
    split_range<Cfg<false>::BK>(p.R, gridDim.z, blockIdx.z, &beg, &end);
    end = min(end, p.Ry);
    auto sx = Source<TILE, TX>::make(p.x, p.ldx, p.M, end, p.ldx, row0);
    auto sy = Source<TILE, TY>::make(p.y, p.ldy, p.N, end, p.ldy, col0);
    Acc<TILE, TILE> acc;
    run_tile<false, D>(acc, sx, sy, beg, end, lds, [](const auto &, int, int64_t, bool) {});
    const int64_t gc = col0 + TileOut<TILE, TILE>::col(), M = p.M, N = p.N, ld = p.ld;
    float *out = static_cast<float *>(p.out) + blockIdx.z * p.split_stride;
    const bool add = p.add;
    const float factor = p.factor ? *p.factor : 1.f;
    emit_tile(acc, lds, [&](int, int r, int, float4 v) {
        const int64_t gr = row0 + r;
        if (gr >= M || gc >= N) return;
        v = make_float4(v.x * factor, v.y * factor, v.z * factor, v.w * factor);
        if (add) {
            const float4 o = load4_clamped<false>(out, gr * ld, gc, N);
            v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
        }
        store4_masked<false>(out, gr * ld, gc, N, v);
    });
}

}  // namespace

int64_t splits_f32(Kind, int64_t M, int64_t N, int64_t R, bool may_split) {
    const int tile = pick_tile(M, N);
    const int64_t tiles = ceil_div(M, tile) * ceil_div(N, tile), chunks = ceil_div(R, int64_t(Cfg<false>::BK));
    if (!may_split || tiles >= 128 || chunks < 16) return 1;
    return std::min<int64_t>({chunks / 8, ceil_div(256, tiles), 16});
}

gnn_status product_f32(Kind kind, const Product &p, hipStream_t s) {
    const int tile = pick_tile(p.M, p.N);
    const TileMap map{ceil_div(p.M, tile), ceil_div(p.N, tile)};
    GNN_CHECK(map.blocks() <= kMaxGrid / gemm::kThreads, GNN_ESIZE, "update_ce: sizes exceed the grid limit");
    const dim3 grid(static_cast<unsigned>(map.blocks()), 1, static_cast<unsigned>(p.nsplit));
    auto go = [&](auto tx, auto ty) {
        constexpr bool TX = decltype(tx)::value, TY = decltype(ty)::value;
        if (tile == 128) class_engine_kernel<128, TX, TY><<<grid, gemm::kThreads, 0, s>>>(p, map);
        else class_engine_kernel<64, TX, TY><<<grid, gemm::kThreads, 0, s>>>(p, map);
    };
    if (kind == kNN) go(std::false_type{}, std::false_type{});
    else if (kind == kTT) go(std::true_type{}, std::true_type{});
    else go(std::false_type{}, std::true_type{});
    GNN_LAUNCHED("update_ce_product");
    return GNN_OK;
}

}  // namespace closs
}  // namespace gnn
