// The update with an activation for few rows (update_act_few.hip).
#pragma once

#include "internal.h"

namespace gnn {

// Whether the kernel takes the call: bf16 products on the shadow, of up to 32
// rows, 64 where the reduction is short.  With GELU and a residual, us here and on
// the tiles (theirs with one row more than the limit, which costs them nothing): 64
// x 1,024 x 1,024 9.8 and 12.4, 32 x 2,048 x 512 9.3 and 12.7, 16 x 4,096 x 4,096 10.8 and
// 13.7.  Of a reduction of 4,096 both take the same at 24 rows, and at 32 the tiles
// are ahead by 1.2 us (32 x 4,096 x 4,096 14.9 and 13.7, x 512 13.9 and 12.7).
inline bool act_few(int64_t cap_m, int64_t K, int gemm_dt, bool shadow) {
    return cap_m <= (K <= 1024 ? 64 : 32) && gemm_dt == GNN_BF16 && shadow;
}
gnn_status launch_act_few(const ActFwd &a, hipStream_t s);

}  // namespace gnn
