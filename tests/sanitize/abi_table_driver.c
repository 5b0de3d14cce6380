/* The host-side validation of the embedding table, the loss over many classes
 * and AdamW with bad and good arguments, and their workspace sizes over the
 * whole range of sizes, under AddressSanitizer and
 * UndefinedBehaviorSanitizer.  Nothing here reaches the GPU. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

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
    const int64_t sizes[] = {0, 1, 3, 64, 65, 1000, 8192, 8193, 26624, 1 << 20, 8388607}, dims[] = {1, 7, 8, 64, 1001, 4096, GNN_MAX_DIM};
    for (size_t i = 0; i < sizeof sizes / sizeof *sizes; ++i)
        for (size_t j = 0; j < sizeof dims / sizeof *dims; ++j) {
            for (int64_t rows = 1; rows < INT32_MAX; rows = rows * 7 + 1)
                EXPECT(gnn_embed_bwd_workspace_size(sizes[i], rows, dims[j], &nb), GNN_OK);
            for (int64_t c = 1; c <= GNN_MAX_CLASSES; c = c * 3 + 1)
                for (int t = 0; t < 4; ++t)
                    EXPECT(gnn_update_ce_workspace_size(sizes[i], dims[j], c, t & 1 ? GNN_BF16 : GNN_F32, t >> 1, &nb), GNN_OK);
        }
    EXPECT(gnn_embed_bwd_workspace_size(INT32_MAX, INT32_MAX, GNN_MAX_DIM, &nb), GNN_OK);

    EXPECT(gnn_embed_bwd_workspace_size(-1, 10, 8, &nb), GNN_EINVAL);
    EXPECT(gnn_embed_bwd_workspace_size(4, INT64_MAX, 8, &nb), GNN_EINVAL);
    EXPECT(gnn_embed_fwd(fake, GNN_F32, 10, 8, INT64_MIN, ids, NULL, 4, 1.f, fake + 4096, GNN_F32, NULL), GNN_EINVAL);
    EXPECT(gnn_embed_fwd(fake, INT32_MIN, 10, 8, 8, ids, NULL, 4, 1.f, fake + 4096, GNN_F32, NULL), GNN_EUNSUPPORTED);
    EXPECT(gnn_embed_fwd(fake, GNN_F32, 10, 8, 8, ids, NULL, 4, NAN, fake + 4096, GNN_F32, NULL), GNN_EINVAL);
    EXPECT(gnn_embed_fwd(NULL, GNN_F32, 10, 8, 8, NULL, NULL, 0, 1.f, NULL, GNN_F32, NULL), GNN_OK); /* no ids */
    EXPECT(gnn_embed_bwd(fake, GNN_F32, ids, NULL, 4, 8, 1.f, 10, 0, fake + 4096, GNN_F32, fake, 8, NULL), GNN_ESIZE);
    EXPECT(gnn_embed_bwd(fake, GNN_F32, ids, NULL, 4, 8, 1.f, 10, 1, fake + 4096, GNN_F32, NULL, 0, NULL), GNN_EINVAL);
    EXPECT(gnn_embed_bwd(NULL, GNN_F32, NULL, NULL, 0, 8, 1.f, 10, 1, fake, GNN_F32, NULL, 0, NULL), GNN_OK); /* nothing to add */

    EXPECT(gnn_update_ce_workspace_size(8, 8, 8, GNN_F16, 1, &nb), GNN_EUNSUPPORTED);
    EXPECT(gnn_update_ce_workspace_size(INT64_MAX, 8, 8, GNN_F32, 1, &nb), GNN_EINVAL);
    EXPECT(gnn_update_ce(fake, GNN_F32, 4, 8, fake + 1024, GNN_F32, f, 10, ids, ids, f, GNN_F32, f, f, fake + 2048, GNN_F32, fake + 4096,
                         GNN_F32, f, fake, 0, NULL),
           GNN_ESIZE);
    EXPECT(gnn_update_ce(fake, GNN_F32, 4, 8, fake + 1024, GNN_F32, f, 10, NULL, ids, f, GNN_F32, f, f, NULL, GNN_F32, NULL, GNN_F32, NULL,
                         fake, SIZE_MAX, NULL),
           GNN_EINVAL);
    EXPECT(gnn_update_ce(fake, GNN_F32, 4, INT64_MAX, fake + 1024, GNN_F32, f, 10, ids, ids, f, GNN_F32, f, f, NULL, GNN_F32, NULL, GNN_F32,
                         NULL, fake, SIZE_MAX, NULL),
           GNN_EINVAL);

    gnn_adamw_tensor t[100];
    memset(t, 0, sizeof t);
    EXPECT(gnn_adamw(t, 100, GNN_F8E4M3, 1e-3, 0.9, 0.999, 1e-8, 1, NULL, NULL, UINT64_MAX, NULL), GNN_OK); /* all empty */
    EXPECT(gnn_adamw(NULL, 0, GNN_F32, 1e-3, 0.9, 0.999, 1e-8, INT64_MAX, NULL, NULL, 0, NULL), GNN_OK);
    EXPECT(gnn_adamw(NULL, 1, GNN_F32, 1e-3, 0.9, 0.999, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EINVAL);
    EXPECT(gnn_adamw(t, INT64_MAX, GNN_F32, 1e-3, 0.9, 0.999, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EINVAL);
    EXPECT(gnn_adamw(t, 1, GNN_F16, 1e-3, 0.9, 0.999, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EUNSUPPORTED);
    EXPECT(gnn_adamw(t, 1, GNN_F32, NAN, 0.9, 0.999, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EINVAL);
    EXPECT(gnn_adamw(t, 1, GNN_F32, 1e-3, 0.9, 1.0, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EINVAL);
    t[99].n = INT64_MAX;
    EXPECT(gnn_adamw(t, 100, GNN_F32, 1e-3, 0.9, 0.999, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EINVAL);
    t[99].n = 5;
    EXPECT(gnn_adamw(t, 100, GNN_F32, 1e-3, 0.9, 0.999, 1e-8, 1, NULL, NULL, 0, NULL), GNN_EINVAL);
    printf("abi table driver: ok\n");
    return 0;
}
