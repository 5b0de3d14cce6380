// bf16 operands as the tiles' kernels read them (act_pack.hip): 16-byte
// aligned rows of a multiple of eight values.  Operands that lie so are used where
// they are; others (fp32 activations, weights without a shadow, odd row lengths,
// halves that are no whole number of chunks, misaligned pointers) are copied to the
// workspace first, which always has room for both.
#pragma once

#include "internal.h"

namespace gnn {

size_t act_engine_ws_bytes(int64_t K, int64_t n_out, int64_t cap_m, int gemm_dt);
gnn_status launch_act_engine(const ActFwd &a, void *ws, hipStream_t s);

// The epilogue of a split reduction: out = act(sum of the partials, in order, +
// bias) + residual for the counted rows.  Partial q's row r starts at
// part + (q cap_m + r) ld, ld a multiple of 4.
gnn_status launch_act_finish(const ActFwd &a, const float *part, int64_t nsplit, int64_t ld, hipStream_t s);

namespace pack {

// fp32 products, and small ones, stay with the general engine, which reads any
// operand as it lies.  Small is below 2^25 where the tiles could do so as well (all of
// these take 12.5 to 13.5 us either way; 512 x 1,024 x 512 13 on the tiles, 16 on
// the engine), and below 2^28 where they would copy operands first, which is 6 us of
// launches (1,000 x 100 x 1,000: 19 us and 13; 20,000 x 100 x 47: 20 and 13; 2,000 x 602 x
// 256: 19.5 and 22).
inline bool small(int64_t cap_m, int64_t K, int64_t n_out, int gemm_dt, bool copied) {
    return gemm_dt != GNN_BF16 || static_cast<double>(cap_m) * static_cast<double>(K) * static_cast<double>(n_out) <
                                      static_cast<double>(copied ? 1 << 28 : 1 << 25);
}

inline int64_t row8(int64_t n) { return (n + 7) / 8 * 8; }

struct Layout {
    size_t a = 0, w = 0, total = 0;
    Layout(int64_t cap_m, int64_t K, int64_t n_out) {
        Carver c(nullptr);
        a = c.take(static_cast<size_t>(cap_m * row8(K) * 2));
        w = c.take(static_cast<size_t>(row8(n_out) * row8(K) * 2));
        total = round_up(c.off, 256);
    }
};

struct Operands {
    const uint16_t *a0, *a1;   // A = [a0 || a1] (a1 null: A = a0), lda values a row each
    int64_t k_each, K, lda;    // K: row8 of the operator's K where A was copied
    const uint16_t *wt;        // W^T: n_out rows, ldw values apart
    int64_t ldw;
};

// Whether the tiles must have A (W) copied.
inline bool copies_a(const ActArgs &a, int64_t chunk) {
    return a.adt != GNN_BF16 || a.K() % 8 != 0 || (a.a_nbr && a.k_each % chunk != 0) || !aligned(a.a_self, 16) ||
           !aligned(a.a_nbr, 16);
}
inline bool copies_w(const ActArgs &a) { return !a.wt || a.K() % 8 != 0 || !aligned(a.wt, 16); }

// The operands of a (a1's halves of a whole number of `chunk` values), copied on s
// where they must be.  weights: wt is wanted.
gnn_status prepare(const ActArgs &a, int64_t chunk, bool weights, void *ws, Operands *o, hipStream_t s);

}  // namespace pack
}  // namespace gnn
