// The update with an activation for few rows (update_act_few.hip).
#pragma once

#include "internal.h"

namespace gnn {

// Whether the kernel takes the call: bf16 products on the shadow, of up to 32
// rows, 64 where the reduction is short (with GELU and a residual, us here and on the
// tiles: 32 x 4,096 x 4,096 14.9 and 17, 33 rows 21.5 and 17; 64 x 1,024 x 1,024
// 9.8 and 12.4).
inline bool act_few(int64_t cap_m, int64_t K, int gemm_dt, bool shadow) {
    return cap_m <= (K <= 1024 ? 64 : 32) && gemm_dt == GNN_BF16 && shadow;
}
gnn_status launch_act_few(const ActFwd &a, hipStream_t s);

}  // namespace gnn
