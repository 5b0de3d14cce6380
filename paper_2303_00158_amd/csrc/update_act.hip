// The update with an activation and a residual in its epilogue:
//   Z = [A_self || A_nbr] W + b,  out = act(Z) + residual
// on the matrix-core engine of gemm_engine.h.
#include "act_pack.h"
#include "act_dev.h"
#include "gemm_engine.h"

namespace gnn {

namespace {

using namespace gemm;

// One epilogue's operands.
struct Epilogue {
    const float *bias;
    const void *residual;
    void *z, *out;
    int64_t n_out;
    bool bf16;  // the type of residual, z and out
    bool vec;   // rows and pointers allow four elements at a time
};

template <class TO> __device__ __forceinline__ void put4(TO *p, int64_t at, int64_t room, bool vec, float4 v) {
    if (vec) {
        store4(p, at, v);
        return;
    }
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < room) Elem<TO>::store(p, at + e, x[e]);
}
template <class TO> __device__ __forceinline__ float4 get4(const TO *p, int64_t at, int64_t room, bool vec) {
    if (vec) return load4(p, at);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < room) x[e] = Elem<TO>::load(p, at + e);
    return make_float4(x[0], x[1], x[2], x[3]);
}

// Columns c .. c + 3 (those below n_out) of row r: z + bias stored, activated,
// the residual added.
template <int ACT, class TO> __device__ __forceinline__ void finish4(const Epilogue &p, int64_t r, int64_t c, float4 v) {
    const int64_t room = p.n_out - c, at = r * p.n_out + c;
    if (room <= 0) return;
    if (p.bias) {
        const float4 b = get4(p.bias + c, 0, room, false);
        v = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
    }
    if (p.z) put4(static_cast<TO *>(p.z), at, room, p.vec, v);
    v = make_float4(act::apply<ACT>(v.x), act::apply<ACT>(v.y), act::apply<ACT>(v.z), act::apply<ACT>(v.w));
    if (p.residual) {
        const float4 d = get4(static_cast<const TO *>(p.residual), at, room, p.vec);
        v = make_float4(v.x + d.x, v.y + d.y, v.z + d.z, v.w + d.w);
    }
    put4(static_cast<TO *>(p.out), at, room, p.vec, v);
}

// The W operand: fp32 W (K x n_out) transposed on the way, or the bf16
// shadow W^T.
template <bool BF16, int TILE, bool V, bool WT, int D> struct WOf {
    using type = SrcCols<BF16, TILE, float, V, D>;
    __device__ static type make(const void *w, int64_t, int64_t n_out, int64_t r_end, int64_t col0) {
        return type{static_cast<const float *>(w), nullptr, n_out, n_out, n_out, r_end, col0, {}};
    }
};
template <int TILE, bool V, int D> struct WOf<true, TILE, V, true, D> {
    using type = SrcRows<true, TILE, uint16_t, V, D>;
    __device__ static type make(const void *wt, int64_t K, int64_t n_out, int64_t, int64_t col0) {
        return type{static_cast<const uint16_t *>(wt), nullptr, K, K, n_out, K, col0, {}};
    }
};

template <bool BF16, int TILE, class TA, bool V, bool WT, int ACT>
__global__ void __launch_bounds__(kThreads) act_engine_kernel(const TA *__restrict__ a_self, const TA *__restrict__ a_nbr,
                                                              int64_t k_each, int64_t K, const int64_t *m_dev, int64_t cap_m,
                                                              const void *__restrict__ w, const float *__restrict__ bias,
                                                              const void *residual, void *z, void *out, int64_t n_out,
                                                              int out_bf16, int vec, float *__restrict__ part, TileMap map) {
    // (arguments one by one: a struct of them, used in the epilogue's lambdas, went
    // through scratch memory and made every access a flat one, 10% of 8,192 x 4,096 x
    // 4,096 in fp32)
    constexpr int D = depth<TILE>();
    __shared__ __attribute__((aligned(16))) char lds[lds_bytes<TILE, TILE>()];
    int64_t tx, ty;
    map.tile_of(blockIdx.x, &tx, &ty);
    const int64_t M = m_dev ? min(*m_dev, cap_m) : cap_m;
    const int64_t row0 = tx * TILE, col0 = ty * TILE;
    if (tx >= map.mt || row0 >= M) return;
    SrcRows<BF16, TILE, TA, V, D> sp{a_self, a_nbr, k_each, k_each, M, K, row0, {}};
    int64_t r_beg, r_end;
    split_range<Cfg<BF16>::BK>(K, gridDim.z, blockIdx.z, &r_beg, &r_end);
    auto sq = WOf<BF16, TILE, V, WT, D>::make(w, K, n_out, r_end, col0);
    Acc<TILE, TILE> acc;
    run_tile<BF16, D>(acc, sp, sq, r_beg, r_end, lds, [](const auto &, int, int64_t, bool) {});
    const int64_t gc = col0 + TileOut<TILE, TILE>::col();
    if (gridDim.z > 1) {
        const int64_t ld = part_ld(n_out);
        float *pp = part + blockIdx.z * cap_m * ld;
        emit_tile(acc, lds, [&](int, int r, int, float4 v) {
            const int64_t gr = row0 + r;
            if (gr < M && gc < ld) *reinterpret_cast<float4 *>(pp + gr * ld + gc) = v;
        });
        return;
    }
    const bool bf = out_bf16;
    emit_tile(acc, lds, [&](int, int r, int, float4 v) {
        const int64_t gr = row0 + r;
        if (gr >= M) return;
        const Epilogue ep{bias, residual, z, out, n_out, bf, vec != 0};
        if (bf) finish4<ACT, uint16_t>(ep, gr, gc, v);
        else finish4<ACT, float>(ep, gr, gc, v);
    });
}

// Four columns of a row from the partials.
template <int ACT, class TO>
__global__ void __launch_bounds__(kThreads) act_finish_kernel(const float *part, int64_t nsplit, int64_t ld,
                                                              const int64_t *m_dev, int64_t cap_m, Epilogue ep) {
    const int64_t M = m_dev ? max(min(*m_dev, cap_m), int64_t(0)) : cap_m, groups = ld / 4;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; t < M * groups;
         t += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t r = t / groups, c = (t - r * groups) * 4;
        finish4<ACT, TO>(ep, r, c, sum_splits(part + r * ld + c, cap_m * ld, static_cast<int>(nsplit)));
    }
}

Epilogue epilogue_of(const ActFwd &a) {
    const size_t osz = dtype_size(a.odt);
    return Epilogue{a.bias, a.residual, a.z, a.out, a.n_out, a.odt == GNN_BF16,
                    a.n_out % 4 == 0 && aligned(a.residual, 4 * osz) && aligned(a.z, 4 * osz) && aligned(a.out, 4 * osz)};
}

// Few tiles of a long reduction are split, eight chunks a split at least (fp32,
// 880 x 512 x 100: 28 tiles of 16 chunks).
int engine_splits(int64_t K, int64_t n_out, int64_t cap_m, bool bf) {
    const int tile = pick_tile(cap_m, n_out);
    const int64_t tiles = ceil_div(std::max<int64_t>(cap_m, 1), tile) * ceil_div(n_out, tile), chunks = ceil_div(K, bk_of(bf));
    if (tiles >= 128 || chunks < 16) return 1;
    return static_cast<int>(std::min<int64_t>({chunks / 8, ceil_div(256, tiles), 16}));
}

}  // namespace

size_t act_engine_ws_bytes(int64_t K, int64_t n_out, int64_t cap_m, int gemm_dt) {
    const int n = engine_splits(K, n_out, cap_m, gemm_dt == GNN_BF16);
    return n > 1 ? round_up(static_cast<size_t>(n * cap_m * part_ld(n_out) * 4), 256) : 0;
}

gnn_status launch_act_finish(const ActFwd &a, const float *part, int64_t nsplit, int64_t ld, hipStream_t s) {
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(a.cap_m * (ld / 4), int64_t(kThreads)), 8192));
    act::with(a.act, [&](auto code) {
        constexpr int ACT = decltype(code)::value;
        if (a.odt == GNN_BF16)
            act_finish_kernel<ACT, uint16_t><<<grid, kThreads, 0, s>>>(part, nsplit, ld, a.m_dev, a.cap_m, epilogue_of(a));
        else
            act_finish_kernel<ACT, float><<<grid, kThreads, 0, s>>>(part, nsplit, ld, a.m_dev, a.cap_m, epilogue_of(a));
    });
    GNN_LAUNCHED("update_fwd_act_finish");
    return GNN_OK;
}

gnn_status launch_act_engine(const ActFwd &a, void *ws, hipStream_t s) {
    const bool bf = a.gemm_dt == GNN_BF16, wt = bf && a.wt;
    const size_t asz = dtype_size(a.adt);
    const int64_t K = a.K();
    const void *w = wt ? static_cast<const void *>(a.wt) : a.w;
    const Epilogue ep = epilogue_of(a);
    float *part = static_cast<float *>(ws);
    const int tile = pick_tile(a.cap_m, a.n_out), nsplit = engine_splits(K, a.n_out, a.cap_m, bf);
    const TileMap map{ceil_div(a.cap_m, tile), ceil_div(a.n_out, tile)};
    GNN_CHECK(map.blocks() <= kMaxGrid / kThreads, GNN_ESIZE, "update_fwd_act: cap_m exceeds the grid limit");
    const bool vec = a.k_each % 4 == 0 && aligned(a.a_self, 4 * asz) && aligned(a.a_nbr, 4 * asz) &&
                     (wt ? aligned(a.wt, 8) : a.n_out % 4 == 0 && aligned(a.w, 16));
    const dim3 grid(static_cast<unsigned>(map.blocks()), 1, static_cast<unsigned>(nsplit));
    act::with(a.act, [&](auto code) {
        constexpr int ACT = decltype(code)::value;
        auto go = [&](auto bf16, auto t, auto ta, auto v, auto shadow) {
            using TA = decltype(ta);
            act_engine_kernel<decltype(bf16)::value, decltype(t)::value, TA, decltype(v)::value, decltype(shadow)::value, ACT>
                <<<grid, kThreads, 0, s>>>(static_cast<const TA *>(a.a_self), static_cast<const TA *>(a.a_nbr), a.k_each, K,
                                           a.m_dev, a.cap_m, w, ep.bias, ep.residual, ep.z, ep.out, ep.n_out, ep.bf16, ep.vec,
                                           part, map);
        };
        using std::bool_constant;
        using std::integral_constant;
        auto by_tile = [&](auto bf16, auto ta, auto v, auto shadow) {
            if (tile == 128) go(bf16, integral_constant<int, 128>{}, ta, v, shadow);
            else go(bf16, integral_constant<int, 64>{}, ta, v, shadow);
        };
        auto by_vec = [&](auto bf16, auto ta, auto shadow) {
            if (vec) by_tile(bf16, ta, bool_constant<true>{}, shadow);
            else by_tile(bf16, ta, bool_constant<false>{}, shadow);
        };
        auto by_type = [&](auto bf16, auto shadow) {
            if (a.adt == GNN_BF16) by_vec(bf16, uint16_t{}, shadow);
            else by_vec(bf16, float{}, shadow);
        };
        if (wt) by_type(bool_constant<true>{}, bool_constant<true>{});
        else if (bf) by_type(bool_constant<true>{}, bool_constant<false>{});
        else by_type(bool_constant<false>{}, bool_constant<false>{});
    });
    GNN_LAUNCHED("update_fwd_act");
    return nsplit > 1 ? launch_act_finish(a, part, nsplit, part_ld(a.n_out), s) : GNN_OK;
}

}  // namespace gnn
