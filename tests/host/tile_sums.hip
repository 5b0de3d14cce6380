// A product on the tiles whose sums go straight to memory, for
// tests/test_tile_sums.py, which reads what the compiler makes of it.
#include "gemm_tile_dev.h"

using namespace gnn;

extern "C" __global__ void __launch_bounds__(256) tile_sums(tile::Operand a, tile::Operand b, int chunks, tile::f32x4 *out) {
    using C = tile::Small;
    __shared__ __attribute__((aligned(16))) uint16_t st0[C::kStageElems], st1[C::kStageElems];
    tile::Acc<C> acc;
    acc.clear();
    tile::Product<C, false, false>(a, b).run(acc, tile::Ring{{st0, st1}}, chunks);
    for (int i = 0; i < C::MI; ++i)
        for (int j = 0; j < C::NI; ++j) out[(threadIdx.x * C::MI + i) * C::NI + j] = acc.v[i][j];
}
