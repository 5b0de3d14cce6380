// The update with an activation and a residual for few rows (a serving program's
// single answers) against the bf16 shadow W^T.
//
// Bound by the weights' bytes: each is read once, straight into the registers of
// the wavefront that multiplies it (no LDS, no barrier in the loop).  A workgroup
// takes 16 columns; its wavefronts deal the reduction in runs of 64 (a whole
// 128-byte line of a row of W^T) among themselves and add their sums in LDS, in
// their order, before the epilogue.  The columns are the first operand of
// v_mfma_f32_16x16x32_bf16 and the rows, 16 at a time, the second, so a lane ends
// with four columns of one row.  Which eight reduction elements a lane holds is free
// as long as both operands agree: lane group g holds elements 16 g .. + 15 of a
// run, eight for each of its two MFMAs.
#include "act_dev.h"
#include "gemm_wide_dev.h"
#include "update_act_few.h"

namespace gnn {

namespace {

using wide::bf16x8;
using wide::f32x4;

struct FewArgs {
    ActFwd a;
    int64_t K;
};

struct Bits8 {
    uint16_t v[8];
};

// Eight bf16 values at p, of which `room` belong to the row; the others are 0.
__device__ __forceinline__ bf16x8 load8(const uint16_t *p, int64_t room) {
    struct __attribute__((packed, aligned(2))) Chunk {
        uint32_t w[4];
    };
    if (room >= 8) return __builtin_bit_cast(bf16x8, *reinterpret_cast<const Chunk *>(p));
    Bits8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b.v[e] = e < room ? p[e] : uint16_t(0);
    return __builtin_bit_cast(bf16x8, b);
}
__device__ __forceinline__ bf16x8 load8(const float *p, int64_t room) {
    Bits8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b.v[e] = e < room ? f32_to_bf16(p[e]) : uint16_t(0);
    return __builtin_bit_cast(bf16x8, b);
}

// Eight elements of a row of [x0 || x1] from k on, 0 past K.
template <class TA>
__device__ __forceinline__ bf16x8 load_row(const TA *x0, const TA *x1, int64_t k_each, int64_t K, int64_t row, int64_t k) {
    if (!x1) return load8(x0 + row * K + min(k, K - 1), K - k);
    if (k + 8 <= k_each) return load8(x0 + row * k_each + k, 8);
    if (k >= k_each) return load8(x1 + row * k_each + min(k - k_each, k_each - 1), K - k);
    Bits8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool hi = k + e >= k_each;
        const TA *p = (hi ? x1 : x0) + row * k_each + (hi ? k + e - k_each : k + e);
        if constexpr (sizeof(TA) == 2) b.v[e] = k + e < K ? *p : uint16_t(0);
        else b.v[e] = k + e < K ? f32_to_bf16(*p) : uint16_t(0);
    }
    return __builtin_bit_cast(bf16x8, b);
}

template <class T> __device__ __forceinline__ void finish_one(const ActFwd &a, int64_t r, int64_t c, float v) {
    const int64_t at = r * a.n_out + c;
    if (a.bias) v += a.bias[c];
    if (a.z) Elem<T>::store(static_cast<T *>(a.z), at, v);
    if (a.act == GNN_ACT_RELU) v = act::apply<GNN_ACT_RELU>(v);
    else if (a.act == GNN_ACT_GELU) v = act::apply<GNN_ACT_GELU>(v);
    else if (a.act == GNN_ACT_GELU_TANH) v = act::apply<GNN_ACT_GELU_TANH>(v);
    else if (a.act == GNN_ACT_SILU) v = act::apply<GNN_ACT_SILU>(v);
    if (a.residual) v += Elem<T>::load(static_cast<const T *>(a.residual), at);
    Elem<T>::store(static_cast<T *>(a.out), at, v);
}

// MT blocks of 16 rows, NW wavefronts.
template <int MT, int NW, class TA>
__global__ void __launch_bounds__(NW * 64) act_few_kernel(FewArgs p) {
    __shared__ float sums[NW][MT * 16][17];  // a row's 16 columns, 17 apart against bank conflicts
    const ActFwd &a = p.a;
    const int64_t M = a.m_dev ? max(min(*a.m_dev, a.cap_m), int64_t(0)) : a.cap_m, K = p.K;
    if (M == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = lane & 15, g = lane >> 4;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16, n = min(n0 + x, a.n_out - 1);
    const uint16_t *w = a.wt + n * K;
    const TA *x0 = static_cast<const TA *>(a.a_self), *x1 = static_cast<const TA *>(a.a_nbr);
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // whole runs of all the wavefronts first, without a bound in the loop
    constexpr int64_t kRun = 64;
    constexpr int kAhead = MT == 1 ? 4 : MT == 2 && NW <= 4 ? 2 : 1;  // runs whose loads are in flight together
    auto runs = [&](int64_t k0, auto ahead, auto whole) {
        constexpr int N = decltype(ahead)::value;
        bf16x8 wf[N][2], xf[N][2][MT];
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = k0 + u * NW * kRun + g * 16 + h * 8;
                if constexpr (decltype(whole)::value) wf[u][h] = load8(w + k, 8);
                else wf[u][h] = load8(w + min(k, K - 1), K - k);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    // rows past the count give columns of the product that are not kept
                    const int64_t r = min(static_cast<int64_t>(t * 16 + x), M - 1);
                    xf[u][h][t] = load_row(x0, x1, a.k_each, K, r, k);
                }
            }
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[u][h], xf[u][h][t], acc[t], 0, 0, 0);
    };
    int64_t k = wave * kRun;
    for (; k + (kAhead - 1) * NW * kRun + kRun <= K; k += kAhead * NW * kRun)
        runs(k, std::integral_constant<int, kAhead>{}, std::true_type{});
    for (; k < K; k += NW * kRun) runs(k, std::integral_constant<int, 1>{}, std::false_type{});
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[wave][t * 16 + x][g * 4 + q] = acc[t][q];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += NW * 64) {
        const int r = i >> 4, c = i & 15;
        if (r >= M || n0 + c >= a.n_out) continue;
        float v = 0.f;
#pragma unroll
        for (int s = 0; s < NW; ++s) v += sums[s][r][c];
        if (a.odt == GNN_BF16) finish_one<uint16_t>(a, r, n0 + c, v);
        else finish_one<float>(a, r, n0 + c, v);
    }
}

}  // namespace

gnn_status launch_act_few(const ActFwd &a, hipStream_t s) {
    const FewArgs p{a, a.K()};
    const int64_t blocks = ceil_div(a.n_out, int64_t(16));
    auto go = [&](auto mt, auto nw, auto ta) {
        act_few_kernel<decltype(mt)::value, decltype(nw)::value, decltype(ta)>
            <<<static_cast<unsigned>(blocks), decltype(nw)::value * 64, 0, s>>>(p);
    };
    // sixteen wavefronts share a column block where there are few blocks (each
    // CU then draws more of the memory) and the reduction is long enough
    const bool wide_group = blocks < 512 && p.K >= 2048;
    auto by_type = [&](auto mt, auto nw) {
        if (a.adt == GNN_BF16) go(mt, nw, uint16_t{});
        else go(mt, nw, float{});
    };
    auto by_waves = [&](auto mt) {
        if (wide_group) by_type(mt, std::integral_constant<int, 16>{});
        else by_type(mt, std::integral_constant<int, 4>{});
    };
    if (a.cap_m <= 16) by_waves(std::integral_constant<int, 1>{});
    else if (a.cap_m <= 32) by_waves(std::integral_constant<int, 2>{});
    else by_type(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});  // K <= 1,024
    GNN_LAUNCHED("update_fwd_act_few");
    return GNN_OK;
}

}  // namespace gnn
