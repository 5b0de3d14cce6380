// The update with an activation for few rows (update_act_few.hip).
#pragma once

#include "internal.h"

namespace gnn {

constexpr int64_t kFewRows = 64;
// Whether the kernel takes the call: bf16 products on the shadow.
inline bool act_few(int64_t cap_m, int gemm_dt, bool shadow) {
    return cap_m <= kFewRows && gemm_dt == GNN_BF16 && shadow;
}
gnn_status launch_act_few(const ActFwd &a, hipStream_t s);

}  // namespace gnn
