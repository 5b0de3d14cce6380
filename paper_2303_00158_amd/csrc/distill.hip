// The loss of a student's logits against a teacher's top logits, with its
// gradient in the same launch.
//
// Bound by memory: one read of the logits and one write of the gradient (the
// teacher's entries are a few hundred bytes a row).  With m the row's maximum
// and e_j = exp((z_j - m) / T), s = sum e, everything else follows from m and
// s: log softmax(z / T)_j = (z_j - m) / T - log s, and the gradient's dense part
// is a constant times e_j.  So a row is held in registers from its load to the
// store of its gradient (by a part of a wavefront up to a workgroup of 1,024
// threads with 128 bf16 elements each), and a thread that has stored a vector
// loads the same vector of its next row into those registers: memory works
// through the exponentials of the gradient, and only the maximum and the sums
// wait for a whole row.  With labels at a temperature other than 1 there are
// two exponentials per element and sum (TWO), else one.
//
// What is subtracted for the teacher's classes and the label is put right
// after the dense part: each listed class is written once more, by the thread
// of its first entry, less the weights of all entries of that class in their
// order (no atomics).
//
// Few rows of many classes, and rows that no workgroup's registers hold, are
// split over workgroups: one launch takes each part's maximum and sums (and
// keeps the listed classes' logits, which a gradient in place of the logits
// may overwrite), the next joins them and writes each part's gradient.
#include "row_dev.h"

namespace gnn {

namespace {

using namespace row;

constexpr int64_t kCus = 256;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// What a row's terms are, and the entries of its teacher and label.
// Entry k is the label's.  Weights are what the gradient subtracts.
struct Entries {
    float *w, *z;     // weight (first the teacher's value); the class's logit
    int32_t *cls;     // class, or -1; padded with -1 to a multiple of 4
};
__host__ __device__ inline int entries_padded(int64_t k) { return static_cast<int>((k + 1 + 3) / 4 * 4); }
__device__ __forceinline__ Entries entries_at(float *lds, int slot, int kp) {
    float *p = lds + static_cast<int64_t>(slot) * 3 * kp;
    return Entries{p, p + kp, reinterpret_cast<int32_t *>(p + 2 * kp)};
}

__device__ __forceinline__ float teacher_value(const DistillArgs &a, int64_t at) {
    return a.tdt == GNN_BF16 ? bf16_to_f32(static_cast<const uint16_t *>(a.t_val)[at])
                             : static_cast<const float *>(a.t_val)[at];
}

// Row i's class of entry e (-1: absent) and, for a present teacher's entry, its
// value.
__device__ __forceinline__ int32_t entry_of(const DistillArgs &a, int64_t i, int e, float *value) {
    *value = -INFINITY;
    if (e < a.k) {
        if (!(a.alpha > 0.f)) return -1;
        const int64_t id = a.t_idx[i * a.k + e];
        const float v = teacher_value(a, i * a.k + e);
        if (id < 0 || id >= a.c || v == -INFINITY) return -1;
        *value = v;
        return static_cast<int32_t>(id);
    }
    if (e > a.k || !a.labels || !(a.alpha < 1.f)) return -1;
    const int64_t y = a.labels[a.targets ? a.targets[i] : i];
    return y < 0 || y >= a.c ? -1 : static_cast<int32_t>(y);
}

// The constants of a row whose maximum and sums are known.
struct RowTerms {
    float m, ka, kb;   // maximum; exponent factors of the two families
    float ca, cb;      // what multiplies each family's exponentials in the gradient
    bool any;          // a term is present
    template <bool TWO> __device__ __forceinline__ float dense(float z) const {
        const float d = z - m;
        float g = ca * exp2_of(d * ka);
        if constexpr (TWO) g = fmaf(cb, exp2_of(d * kb), g);
        return g;
    }
};

// Entry e's part of the row's loss, and its weight in the gradient.
//   soft: alpha T^2 p (log p - log q);  label: (1 - alpha) (log s - (z - m)).
struct LossTerms {
    float alpha, temp, inv_t, scale;
    float tmax, ts, log_ts;  // the teacher's maximum, sum and its logarithm
    float m, log_sa, log_sb; // the student's maximum and the sums' logarithms (at T and at 1)
    __device__ __forceinline__ float teacher(float value, float z, float *w) const {
        const float d = (value - tmax) * inv_t, p = exp2_of(d * kLog2e) / ts;
        *w = scale * alpha * temp * p;
        return p != 0.f ? alpha * temp * temp * p * ((d - log_ts) - ((z - m) * inv_t - log_sa)) : 0.f;
    }
    __device__ __forceinline__ float label(float z, float *w) const {
        *w = scale * (1.f - alpha);
        return (1.f - alpha) * (log_sb - (z - m));
    }
};

// Exponent factors: family A is the temperature's wherever the teacher counts.
__device__ __forceinline__ float factor_a(const DistillArgs &a) { return a.alpha > 0.f ? kLog2e / a.temperature : kLog2e; }

__device__ __forceinline__ float row_scale_of(const DistillArgs &a, int64_t i) {
    return a.row_scale ? a.row_scale[i] : 1.f / static_cast<float>(a.b);
}

// Write each listed class of [lo, hi) again: its dense part less its weights.
template <bool TWO, class TG>
__device__ __forceinline__ void put_entries(const Entries &en, const RowTerms &t, int kp, int first, int step, TG *g,
                                            int64_t lo, int64_t hi) {
    for (int e = first; e < kp; e += step) {
        const int32_t id = en.cls[e];
        if (id < 0 || id < lo || id >= hi) continue;
        bool mine = true;
        float w = 0.f;
        for (int o = 0; o < kp; o += 4) {
            const int4 c = *reinterpret_cast<const int4 *>(en.cls + o);
            const int32_t cc[4] = {c.x, c.y, c.z, c.w};
            if (cc[0] != id && cc[1] != id && cc[2] != id && cc[3] != id) continue;
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (cc[x] == id) {
                    mine = mine && o + x >= e;
                    w += en.w[o + x];
                }
        }
        if (mine) Elem<TG>::store(g, id, t.dense<TWO>(en.z[e]) - w);
    }
}

// ---------------------------------------------------------------------------
// rows in registers
// ---------------------------------------------------------------------------

// A thread's share of a row of c elements: the vectors that are whole in all of
// the row's threads (`full` of them, at most NV, the same in every thread), and
// the one after them, of which the row's end leaves some threads a part or
// nothing.  One uniform count in place of every vector's bounds keeps those out
// of the registers: with bounds, 1,024 threads x 128 elements spilled 154.
template <class S, class TL> struct RowRegs {
    Vec<TL, S::VE> r[S::NV], tail;
    int full, rest;  // rest: elements of `tail` that belong to the row (of this thread)
    static constexpr int64_t kMost = static_cast<int64_t>(S::T) * (S::E + S::VE) - 1;  // longest row
    __device__ __forceinline__ explicit RowRegs(int64_t c) {
        full = static_cast<int>(c / (S::T * S::VE));
        rest = static_cast<int>(c) - (full * S::T + S::lane()) * S::VE;
    }
    __device__ __forceinline__ static uint32_t off() { return static_cast<uint32_t>(S::lane()) * S::VE; }
    template <class F> __device__ __forceinline__ void each(F &&go) {
#pragma unroll
        for (int v = 0; v < S::NV; ++v)
            if (v < full) go(r[v]);
        go(tail);
    }
    __device__ __forceinline__ void load(const TL *row, int v) { r[v].load(row + v * (S::T * S::VE) + off()); }
    __device__ __forceinline__ void load_tail(const TL *row) {
        tail.load_upto(row + full * (S::T * S::VE) + off(), rest, -INFINITY);
    }
    __device__ __forceinline__ void load(const TL *row) {
#pragma unroll
        for (int v = 0; v < S::NV; ++v)
            if (v < full) load(row, v);
        load_tail(row);
    }
};

// Workgroups to a CU that the registers are to leave room for.
template <class S> constexpr int waves_wanted() { return S::T >= 512 ? 4 : 1; }

template <class S, class TL, class TG, bool TWO>
__global__ void __launch_bounds__(S::kThreads, waves_wanted<S>()) distill_rows_kernel(DistillArgs a, float *row_loss) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    __shared__ typename RowReduce<S>::Shared sh;
    RowReduce<S> over(sh);
    const int kp = entries_padded(a.k), lane = S::lane();
    const int64_t c = a.c, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const TL *logits = static_cast<const TL *>(a.logits);
    TG *grad = static_cast<TG *>(a.g_out);
    int64_t i = static_cast<int64_t>(blockIdx.x) * S::kRows + S::row();
    if (i >= a.b) return;  // threads of whole rows; above 64 a workgroup has one
    RowRegs<S, TL> r(c);
    float scale = row_scale_of(a, i);
    if (scale != 0.f) r.load(logits + i * c);
    for (int turn = 0; i < a.b; i += step, turn ^= 1) {
        const int64_t next = i + step;
        const float next_scale = next < a.b ? row_scale_of(a, next) : 0.f;
        RowTerms t{0.f, factor_a(a), kLog2e, 0.f, 0.f, false};
        // two sets of entries in turn: a row's are read until its last store
        const Entries en = entries_at(lds, S::row() * 2 + turn, kp);
        float loss = 0.f;
        if (scale != 0.f) {
            float mx[2] = {-INFINITY, -INFINITY};
            for (int e = lane; e < kp; e += S::T) {
                float value;
                const int32_t id = entry_of(a, i, e, &value);
                en.cls[e] = id;
                en.w[e] = value;
                if (id >= 0) en.z[e] = Elem<TL>::load(logits, i * c + id);
                mx[1] = fmaxf(mx[1], value);
            }
            r.each([&](Vec<TL, S::VE> &x) {
#pragma unroll
                for (int e = 0; e < S::VE; ++e) mx[0] = fmaxf(mx[0], x.get(e));
                x.pin();
            });
            over(Max{}, mx);
            if constexpr (S::T <= 64) row_sync<S>();
            t.m = mx[0];
            float s[3] = {0.f, 0.f, 0.f};
            r.each([&](Vec<TL, S::VE> &x) {
#pragma unroll
                for (int e = 0; e < S::VE; ++e) {
                    const float d = x.get(e) - t.m;
                    s[0] += exp2_of(d * t.ka);
                    if constexpr (TWO) s[1] += exp2_of(d * t.kb);
                }
                x.pin();
            });
            const float inv_t = 1.f / a.temperature;
            for (int e = lane; e < kp; e += S::T)
                if (en.cls[e] >= 0 && e < a.k) s[2] += exp2_of((en.w[e] - mx[1]) * inv_t * kLog2e);
            over(Add{}, s);
            const float s1 = TWO ? s[1] : s[0];
            const LossTerms lt{a.alpha, a.temperature, inv_t, scale, mx[1], s[2], logf(s[2]), t.m, logf(s[0]), logf(s1)};
            const bool soft = s[2] != 0.f, hard = en.cls[a.k] >= 0;
            float l[1] = {0.f};
            for (int e = lane; e < kp; e += S::T) {
                float w = 0.f;
                if (en.cls[e] >= 0) l[0] += e < a.k ? lt.teacher(en.w[e], en.z[e], &w) : lt.label(en.z[e], &w);
                en.w[e] = w;
            }
            over(Add{}, l);
            loss = l[0];
            t.any = soft || hard;
            const float cs = soft ? scale * a.alpha * a.temperature : 0.f, ch = hard ? scale * (1.f - a.alpha) : 0.f;
            t.ca = TWO ? cs / s[0] : (cs + ch) / s[0];
            t.cb = ch / s1;
        }
        if (lane == 0) row_loss[i] = loss;
        // the gradient, vector by vector, and the next row into its registers
        const TL *ahead = logits + next * c;
        TG *g = grad + i * c;
        auto dense = [&](const Vec<TL, S::VE> &x) {
            float o[S::VE];
#pragma unroll
            for (int e = 0; e < S::VE; ++e) o[e] = t.any ? t.dense<TWO>(x.get(e)) : 0.f;
            Vec<TG, S::VE> w;
            w.set(o);
            return w;
        };
#pragma unroll
        for (int v = 0; v < S::NV; ++v)
            if (v < r.full) {
                if (grad) dense(r.r[v]).store(g + v * (S::T * S::VE) + r.off());
                if (next_scale != 0.f) r.load(ahead, v);
            }
        if (grad) dense(r.tail).store_upto(g + r.full * (S::T * S::VE) + r.off(), r.rest);
        if (next_scale != 0.f) r.load_tail(ahead);
        if (grad) {
            row_sync<S>();
            if (t.any) put_entries<TWO>(en, t, kp, lane, S::T, g, 0, c);
        }
        scale = next_scale;
    }
}

// ---------------------------------------------------------------------------
// rows split over workgroups
// ---------------------------------------------------------------------------
constexpr int kSplitThreads = 256;
using SplitShape = Shape<kSplitThreads, 8, 8>;

struct SplitPlan {
    int64_t parts, len;  // parts of a row, and their columns (a multiple of 2,048)
};

struct SplitState {
    float *stats;   // b x parts x 3: maximum, sum at T, sum at 1
    float *z;       // b x kp: the entries' logits
};

template <class TL, bool TWO>
__global__ void __launch_bounds__(kSplitThreads) distill_part_kernel(DistillArgs a, SplitPlan p, SplitState st) {
    using S = SplitShape;
    __shared__ typename RowReduce<S>::Shared sh;
    RowReduce<S> over(sh);
    const int64_t i = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    if (row_scale_of(a, i) == 0.f) return;
    const TL *z = static_cast<const TL *>(a.logits) + i * a.c;
    const int64_t lo = part * p.len, hi = min(a.c, lo + p.len);
    const int kp = entries_padded(a.k);
    if (part == 0)
        for (int e = threadIdx.x; e < kp; e += kSplitThreads) {
            float value;
            const int32_t id = entry_of(a, i, e, &value);
            if (id >= 0) st.z[i * kp + e] = Elem<TL>::load(z, id);
        }
    const float ka = factor_a(a), kb = kLog2e;
    // each thread's own running maximum; sums move to a new one as it comes
    float m = -INFINITY, sa = 0.f, sb = 0.f;
    for (int64_t c0 = lo; c0 < hi; c0 += kSplitThreads * S::VE) {
        Vec<TL, S::VE> r;
        const int64_t c = c0 + S::col(0);
        r.load_upto(z + c, hi - c, -INFINITY);
        float top = r.get(0);
#pragma unroll
        for (int e = 1; e < S::VE; ++e) top = fmaxf(top, r.get(e));
        if (top > m) {
            sa *= exp2_of((m - top) * ka);
            if constexpr (TWO) sb *= exp2_of((m - top) * kb);
            m = top;
        }
        // nothing but -infinity so far (or a NaN, which the sums keep)
        const float at = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int e = 0; e < S::VE; ++e) {
            const float d = r.get(e) - at;
            sa += exp2_of(d * ka);
            if constexpr (TWO) sb += exp2_of(d * kb);
        }
    }
    float top[1] = {m};
    over(Max{}, top);
    const float at = top[0] == -INFINITY ? 0.f : top[0], own = m == -INFINITY ? at : m;
    float s[2] = {sa * exp2_of((own - at) * ka), TWO ? sb * exp2_of((own - at) * kb) : 0.f};
    over(Add{}, s);
    if (threadIdx.x == 0) {
        float *o = st.stats + (i * p.parts + part) * 3;
        o[0] = top[0];
        o[1] = s[0];
        o[2] = s[1];
    }
}

template <class TL, class TG, bool TWO>
__global__ void __launch_bounds__(kSplitThreads) distill_join_kernel(DistillArgs a, SplitPlan p, SplitState st,
                                                                     float *row_loss) {
    using S = SplitShape;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    __shared__ typename RowReduce<S>::Shared sh;
    RowReduce<S> over(sh);
    const int64_t i = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const int64_t lo = part * p.len, hi = min(a.c, lo + p.len);
    const TL *z = static_cast<const TL *>(a.logits) + i * a.c;
    TG *g = a.g_out ? static_cast<TG *>(a.g_out) + i * a.c : nullptr;
    const int kp = entries_padded(a.k);
    const float scale = row_scale_of(a, i);
    RowTerms t{0.f, factor_a(a), kLog2e, 0.f, 0.f, false};
    const Entries en = entries_at(lds, 0, kp);
    float loss = 0.f;
    if (scale != 0.f) {
        // join the parts
        const float *q = st.stats + i * p.parts * 3;
        float mx[2] = {-INFINITY, -INFINITY};
        for (int64_t e = threadIdx.x; e < p.parts; e += kSplitThreads) mx[0] = fmaxf(mx[0], q[e * 3]);
        for (int e = threadIdx.x; e < kp; e += kSplitThreads) {
            float value;
            const int32_t id = entry_of(a, i, e, &value);
            en.cls[e] = id;
            en.w[e] = value;
            if (id >= 0) en.z[e] = st.z[i * kp + e];
            mx[1] = fmaxf(mx[1], value);
        }
        over(Max{}, mx);
        t.m = mx[0];
        const float inv_t = 1.f / a.temperature;
        float s[3] = {0.f, 0.f, 0.f};
        for (int64_t e = threadIdx.x; e < p.parts; e += kSplitThreads) {
            const float d = q[e * 3] == -INFINITY && t.m != -INFINITY ? -INFINITY : q[e * 3] - t.m;
            s[0] += q[e * 3 + 1] * exp2_of(d * t.ka);
            if constexpr (TWO) s[1] += q[e * 3 + 2] * exp2_of(d * t.kb);
        }
        for (int e = threadIdx.x; e < kp; e += kSplitThreads)
            if (en.cls[e] >= 0 && e < a.k) s[2] += exp2_of((en.w[e] - mx[1]) * inv_t * kLog2e);
        over(Add{}, s);
        const float s1 = TWO ? s[1] : s[0];
        const LossTerms lt{a.alpha, a.temperature, inv_t, scale, mx[1], s[2], logf(s[2]), t.m, logf(s[0]), logf(s1)};
        const bool soft = s[2] != 0.f, hard = en.cls[a.k] >= 0;
        row_sync<S>();
        float l[1] = {0.f};
        for (int e = threadIdx.x; e < kp; e += kSplitThreads) {
            float w = 0.f;
            if (en.cls[e] >= 0) l[0] += e < a.k ? lt.teacher(en.w[e], en.z[e], &w) : lt.label(en.z[e], &w);
            en.w[e] = w;
        }
        over(Add{}, l);
        loss = l[0];
        t.any = soft || hard;
        const float cs = soft ? scale * a.alpha * a.temperature : 0.f, ch = hard ? scale * (1.f - a.alpha) : 0.f;
        t.ca = TWO ? cs / s[0] : (cs + ch) / s[0];
        t.cb = ch / s1;
    }
    if (part == 0 && threadIdx.x == 0) row_loss[i] = loss;
    if (!g) return;
    for (int64_t c0 = lo; c0 < hi; c0 += kSplitThreads * S::VE) {
        const int64_t c = c0 + S::col(0);
        float o[S::VE];
#pragma unroll
        for (int e = 0; e < S::VE; ++e) o[e] = 0.f;
        if (t.any) {
            Vec<TL, S::VE> r;
            r.load_upto(z + c, hi - c);
#pragma unroll
            for (int e = 0; e < S::VE; ++e) o[e] = t.dense<TWO>(r.get(e));
        }
        Vec<TG, S::VE> w;
        w.set(o);
        w.store_upto(g + c, hi - c);
    }
    row_sync<S>();
    if (t.any) put_entries<TWO>(en, t, kp, threadIdx.x, kSplitThreads, g, lo, hi);
}

// loss = sum over the rows of scale x row loss, by one workgroup.
constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads) distill_loss_kernel(const float *row_loss, const float *row_scale,
                                                                    int64_t b, float *loss) {
    using S = Shape<kLossThreads, 8, 8>;
    __shared__ RowReduce<S>::Shared sh;
    RowReduce<S> over(sh);
    float s[1] = {0.f};
    for (int64_t i = threadIdx.x; i < b; i += kLossThreads) {
        const float l = row_loss[i], w = row_scale ? row_scale[i] : 1.f;
        s[0] += w != 0.f ? w * l : 0.f;
    }
    over(Add{}, s);
    if (threadIdx.x == 0) *loss = row_scale || b == 0 ? s[0] : s[0] / static_cast<float>(b);
}

// The shape of a row of c classes in registers: at most 68 words a thread.
template <class S, class F> bool if_fits(int64_t c, F &&go) {
    if (c > RowRegs<S, float>::kMost) return false;
    go(S{});
    return true;
}
template <int VE, bool BF16, class F> bool with_shape(int64_t c, F &&go) {
    return if_fits<Shape<16, 8, VE>>(c, go) || if_fits<Shape<64, 8, VE>>(c, go) || if_fits<Shape<64, 16, VE>>(c, go) ||
           if_fits<Shape<256, 16, VE>>(c, go) || if_fits<Shape<256, 32, VE>>(c, go) ||
           if_fits<Shape<256, 64, VE>>(c, go) || if_fits<Shape<512, 64, VE>>(c, go) ||
           if_fits<Shape<1024, 64, VE>>(c, go) || (BF16 && if_fits<Shape<1024, BF16 ? 128 : 64, VE>>(c, go));
}

// Classes of a row in registers, fp32 (with a gradient of either type) and bf16.
constexpr int64_t kRowsMax[2] = {RowRegs<Shape<1024, 64, 4>, float>::kMost, RowRegs<Shape<1024, 128, 8>, uint16_t>::kMost};

// Rows are split when they do not fit, and where so few of 8,192 classes and
// more come that most CUs would have none.
SplitPlan plan_split(int64_t b, int64_t c, int ldt) {
    SplitPlan p{1, c};
    const bool fits = c <= kRowsMax[ldt == GNN_BF16];
    if (fits && (c < 8192 || b >= kCus / 2)) return p;
    const int64_t unit = kSplitThreads * SplitShape::VE;
    const int64_t want = std::max<int64_t>(ceil_div(2 * kCus, std::max<int64_t>(b, 1)), fits ? 1 : 4);
    const int64_t units = ceil_div(c, unit);
    p.len = ceil_div(units, std::min(want, units)) * unit;
    p.parts = ceil_div(c, p.len);
    return p;
}

}  // namespace

size_t distill_ws_bytes(int64_t b, int64_t c, int64_t k) {
    // either type's plan: the row losses, the parts' sums, the entries' logits
    int64_t parts = 0;
    for (int dt : {GNN_F32, GNN_BF16}) {
        const SplitPlan p = plan_split(b, c, dt);
        if (p.parts > 1) parts = std::max(parts, p.parts);
    }
    size_t bytes = round_up(static_cast<size_t>(std::max<int64_t>(b, 1)) * 4, 256);
    if (parts) bytes += round_up(static_cast<size_t>(b * parts * 12), 256) + round_up(static_cast<size_t>(b * entries_padded(k) * 4), 256);
    return bytes;
}

gnn_status launch_distill(const DistillArgs &a, void *ws, hipStream_t s) {
    char *base = static_cast<char *>(ws);
    const size_t rows_bytes = round_up(static_cast<size_t>(std::max<int64_t>(a.b, 1)) * 4, 256);
    float *row_loss = a.row_loss ? a.row_loss : reinterpret_cast<float *>(base);
    if (a.b > 0) {
        const SplitPlan p = plan_split(a.b, a.c, a.ldt);
        const int entry_bytes = entries_padded(a.k) * 12;
        const bool two = a.labels && a.alpha > 0.f && a.alpha < 1.f && a.temperature != 1.f;
        auto go = [&](auto tl, auto tg, auto t2) {
            using TL = decltype(tl);
            using TG = decltype(tg);
            constexpr bool TWO = decltype(t2)::value;
            if (p.parts > 1) {
                SplitState st{};
                st.stats = reinterpret_cast<float *>(base + rows_bytes);
                st.z = reinterpret_cast<float *>(base + rows_bytes + round_up(static_cast<size_t>(a.b * p.parts * 12), 256));
                const unsigned grid = static_cast<unsigned>(a.b * p.parts);
                distill_part_kernel<TL, TWO><<<grid, kSplitThreads, 0, s>>>(a, p, st);
                distill_join_kernel<TL, TG, TWO><<<grid, kSplitThreads, entry_bytes, s>>>(a, p, st, row_loss);
                return;
            }
            with_shape<sizeof(TL) == 4 ? 4 : 8, sizeof(TL) == 2>(a.c, [&](auto shape) {
                using S = decltype(shape);
                // one round of the CUs with what fits on each: workgroups walk
                // their rows and load each ahead
                const int64_t grid = std::min<int64_t>(ceil_div(a.b, S::kRows), kCus * (S::T >= 256 ? 1024 / S::T : 8));
                distill_rows_kernel<S, TL, TG, TWO>
                    <<<static_cast<unsigned>(grid), S::kThreads, 2 * S::kRows * entry_bytes, s>>>(a, row_loss);
            });
        };
        auto by_two = [&](auto tl, auto tg) {
            if (two) go(tl, tg, std::true_type{});
            else go(tl, tg, std::false_type{});
        };
        if (a.ldt == GNN_BF16) {
            if (a.gdt == GNN_BF16) by_two(uint16_t{}, uint16_t{});
            else by_two(uint16_t{}, float{});
        } else {
            if (a.gdt == GNN_BF16) by_two(float{}, uint16_t{});
            else by_two(float{}, float{});
        }
        GNN_LAUNCHED("distill_topk");
    }
    distill_loss_kernel<<<1, kLossThreads, 0, s>>>(row_loss, a.row_scale, a.b, a.loss_out);
    GNN_LAUNCHED("distill_topk_loss");
    return GNN_OK;
}

}  // namespace gnn
