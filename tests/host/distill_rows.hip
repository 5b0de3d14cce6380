// The rows of the distillation loss that are held in registers: for every class
// count on stdin ("type c k", type 0 fp32 and 1 bf16), over all places of a row in
// its 128-byte line, whether the chosen shape's threads take each class exactly
// once.  A line each: "T E heads", heads the number of places at which some class
// is missed or taken twice (T = 0: no shape holds the row).  Host code only.
#include <cstdio>
#include <vector>

#include "distill_rows.h"

using namespace gnn;

namespace {

template <class S, class TL> int bad_places(int c) {
    using Span = distill::Span<S, TL>;
    int bad = 0;
    std::vector<int> change(c + 1);
    for (int head = 0; head < Span::kLine; ++head) {
        std::fill(change.begin(), change.end(), 0);
        const int whole = Span::whole(c, head);
        auto take = [&](int v) {
            for (int lane = 0; lane < S::T; ++lane) {
                const int at = Span::place(head, v, lane), lo = std::max(at, 0), hi = std::min(at + S::VE, c);
                if (lo < hi) ++change[lo], --change[hi];
            }
        };
        for (int v = 0; v < S::NV; ++v)
            if (v < whole) take(v);
        take(whole);  // the row's end
        int times = 0;
        bool good = true;
        for (int j = 0; j < c; ++j) good &= (times += change[j]) == 1;
        bad += !good;
    }
    return bad;
}

template <class TL> void look(int c, int k) {
    int t = 0, e = 0, bad = 0;
    distill::with_shape<TL>(c, k, [&](auto shape) {
        using S = decltype(shape);
        t = S::T;
        e = S::E;
        bad = bad_places<S, TL>(c);
    });
    std::printf("%d %d %d\n", t, e, bad);
}

}  // namespace

int main() {
    int type, c, k;
    while (std::scanf("%d %d %d", &type, &c, &k) == 3) {
        if (type) look<uint16_t>(c, k);
        else look<float>(c, k);
    }
    return 0;
}
