/* The host-side validation of layer norm, the update with an activation and
 * the distillation loss with bad and good arguments, and their workspace sizes
 * over the whole range of sizes, under AddressSanitizer and
 * UndefinedBehaviorSanitizer.  Nothing here reaches the GPU. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "gnn.h"

#define EXPECT(call, want)                                                                  \
    do {                                                                                    \
        gnn_status st_ = (call);                                                            \
        if (st_ != (want)) {                                                                \
            fprintf(stderr, "line %d: %s returned %d, expected %d (%s)\n", __LINE__, #call, \
                    (int)st_, (int)(want), gnn_last_error());                               \
            return 1;                                                                       \
        }                                                                                   \
    } while (0)

int main(void) {
    char *fake = (char *)(uintptr_t)(1u << 24);
    int64_t *ids = (int64_t *)fake;
    float *f = (float *)fake;
    size_t nb = 0;
    const int64_t sizes[] = {0, 1, 3, 64, 65, 1000, 26624, 1 << 20, 2147483647}, dims[] = {1, 7, 8, 64, 1001, 4096, GNN_MAX_DIM};
    for (size_t i = 0; i < sizeof sizes / sizeof *sizes; ++i)
        for (size_t j = 0; j < sizeof dims / sizeof *dims; ++j) {
            EXPECT(gnn_layer_norm_bwd_workspace_size(dims[j], sizes[i], &nb), GNN_OK);
            for (size_t k = 0; k < sizeof dims / sizeof *dims; ++k)
                for (int t = 0; t < 8; ++t) {
                    const gnn_dtype gemm = t & 1 ? GNN_BF16 : GNN_F32;
                    EXPECT(gnn_update_fwd_act_workspace_size(GNN_BF16, dims[j], t >> 1 & 1, dims[k], sizes[i], gemm, t >> 2, &nb),
                           GNN_OK);
                    EXPECT(gnn_update_bwd_act_workspace_size(GNN_F32, dims[j], t >> 1 & 1, dims[k], sizes[i], GNN_F32, GNN_F32,
                                                             gemm, t >> 2, &nb),
                           GNN_OK);
                }
        }
    for (int64_t c = 1; c <= GNN_MAX_CLASSES; c = c * 3 + 1)
        for (int64_t b = 0; b <= 100000; b = b * 5 + 1) EXPECT(gnn_distill_topk_workspace_size(b, c, 1 + c % GNN_MAX_TOP, &nb), GNN_OK);

    EXPECT(gnn_layer_norm_bwd_workspace_size(0, 4, &nb), GNN_EINVAL);
    EXPECT(gnn_layer_norm_bwd_workspace_size(4, 4, NULL), GNN_EINVAL);
    EXPECT(gnn_layer_norm_bwd_workspace_size(4, INT64_MAX, &nb), GNN_EINVAL);
    EXPECT(gnn_layer_norm_fwd(NULL, GNN_F32, NULL, 4, 8, f, f, 1e-5f, fake, GNN_F32, NULL, NULL, NULL), GNN_EINVAL);
    EXPECT(gnn_layer_norm_fwd(fake, 77, NULL, 4, 8, f, f, 1e-5f, fake, GNN_F32, NULL, NULL, NULL), GNN_EUNSUPPORTED);
    EXPECT(gnn_layer_norm_fwd(fake, GNN_F32, NULL, 4, 8, f, f, NAN, fake, GNN_F32, NULL, NULL, NULL), GNN_EINVAL);
    EXPECT(gnn_layer_norm_fwd(fake, GNN_F32, NULL, 4, 8, f, f, 1e-5f, fake, GNN_BF16, NULL, NULL, NULL), GNN_EINVAL);
    EXPECT(gnn_layer_norm_bwd(fake, GNN_F32, fake + 256, GNN_F32, NULL, 4, 8, f, f, f, NULL, NULL, NULL, NULL, NULL, 0, NULL),
           GNN_EINVAL);
    EXPECT(gnn_layer_norm_bwd(fake, GNN_F32, fake + 256, GNN_F32, NULL, 4, 8, f, f, f, NULL, fake, f, f, fake, 16, NULL),
           GNN_ESIZE);

    EXPECT(gnn_update_fwd_act_workspace_size(GNN_BF16, 8, 0, 8, 8, GNN_BF16, 1, NULL), GNN_EINVAL);
    EXPECT(gnn_update_fwd_act_workspace_size(-5, 8, 0, 8, 8, GNN_BF16, 1, &nb), GNN_EUNSUPPORTED);
    EXPECT(gnn_update_fwd_act_workspace_size(GNN_BF16, INT64_MAX, 1, 8, 8, GNN_BF16, 1, &nb), GNN_EINVAL);
    EXPECT(gnn_update_fwd_act(fake, NULL, GNN_F32, 8, NULL, 4, f, NULL, NULL, 8, INT32_MIN, NULL, NULL, GNN_F32, fake + 4096,
                              GNN_F32, NULL, 0, NULL),
           GNN_EINVAL);
    EXPECT(gnn_update_fwd_act(fake, NULL, GNN_BF16, 4096, NULL, 4096, f, NULL, NULL, 4096, GNN_ACT_GELU, NULL, NULL, GNN_BF16,
                              fake + 4096, GNN_F32, fake, 256, NULL),
           GNN_ESIZE);
    EXPECT(gnn_update_bwd_act(fake, NULL, GNN_BF16, 64, NULL, 100, f, NULL, NULL, GNN_BF16, fake, GNN_BF16, 64, GNN_ACT_SILU,
                              GNN_BF16, fake, GNN_F32, f, NULL, fake, 1 << 30, NULL),
           GNN_EINVAL); /* no z */
    EXPECT(gnn_update_bwd_act(fake, NULL, GNN_BF16, 64, NULL, 100, f, NULL, fake, GNN_BF16, fake, GNN_BF16, 64, GNN_ACT_SILU,
                              GNN_BF16, fake, GNN_F32, f, NULL, fake, 1, NULL),
           GNN_ESIZE);

    EXPECT(gnn_distill_topk_workspace_size(-1, 8, 2, &nb), GNN_EINVAL);
    EXPECT(gnn_distill_topk_workspace_size(4, GNN_MAX_CLASSES + 1, 2, &nb), GNN_EINVAL);
    EXPECT(gnn_distill_topk(fake, GNN_F32, 4, 8, fake, GNN_F32, ids, 2, INFINITY, 1.f, NULL, NULL, NULL, NULL, GNN_F32, NULL, f,
                            fake, 1 << 20, NULL),
           GNN_EINVAL);
    EXPECT(gnn_distill_topk(fake, GNN_F32, 4, 8, fake, GNN_F32, ids, 2, 1.f, NAN, NULL, NULL, NULL, NULL, GNN_F32, NULL, f, fake,
                            1 << 20, NULL),
           GNN_EINVAL);
    EXPECT(gnn_distill_topk(fake, GNN_F32, 4, 8, fake, GNN_F32, ids, 2, 1.f, 1.f, NULL, NULL, NULL, fake, GNN_BF16, NULL, f, fake,
                            1 << 20, NULL),
           GNN_EINVAL);
    printf("abi layers driver: ok\n");
    return 0;
}
