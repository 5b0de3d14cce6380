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
#include "distill_rows.h"

namespace gnn {

namespace {

using namespace row;
using namespace distill;

constexpr int64_t kCus = 256;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// What a row's terms are, and the entries of its teacher and label.
// Entry k is the label's.  Weights are what the gradient subtracts.
struct Entries {
    float *w, *z;     // weight (first the teacher's value); the class's logit
    int32_t *cls;     // class, or -1; padded with -1 to a multiple of 4
};
__device__ __forceinline__ Entries entries_at(float *lds, int slot, int kp) {
    float *p = lds + static_cast<int64_t>(slot) * 3 * kp;
    return Entries{p, p + kp, reinterpret_cast<int32_t *>(p + 2 * kp)};
}

// Entry e of row i as it lies in memory: nothing is looked at here, so that the
// loads are still on their way when a row ahead asks for them.
struct RawEntry {
    int64_t id;
    uint32_t bits;
    __device__ __forceinline__ void load(const DistillArgs &a, int64_t i, int e) {
        id = -1;
        bits = 0;
        if (e < a.k) {
            if (!(a.alpha > 0.f)) return;
            const int64_t at = i * a.k + e;
            id = a.t_idx[at];
            if (a.tdt == GNN_BF16) bits = static_cast<const uint16_t *>(a.t_val)[at];
            else bits = static_cast<const uint32_t *>(a.t_val)[at];
        } else if (e == a.k && a.labels && a.alpha < 1.f) {
            id = a.labels[a.targets ? a.targets[i] : i];
        }
    }
};

// One entry of a row: class (-1: absent), teacher's value (-infinity for the
// label's and absent ones), the class's logit.
struct Entry {
    int32_t cls;
    float value, z;
    __device__ __forceinline__ void take(const DistillArgs &a, const RawEntry &r, int e) {
        value = a.tdt == GNN_BF16 ? __uint_as_float(r.bits << 16) : __uint_as_float(r.bits);
        const bool teacher = e < a.k, in = r.id >= 0 && r.id < a.c && !(teacher && value == -INFINITY);
        cls = in ? static_cast<int32_t>(r.id) : -1;
        if (!in || !teacher) value = -INFINITY;
        z = 0.f;
    }
    __device__ __forceinline__ void load(const DistillArgs &a, int64_t i, int e) {
        RawEntry r;
        r.load(a, i, e);
        take(a, r, e);
    }
};

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
// A first look over the list, without branches, tells whether a class stands
// there more than once; only then are its weights added up.
template <bool TWO, class TG>
__device__ __forceinline__ void put_entries(const Entries &en, const RowTerms &t, int kp, int first, int step, TG *g,
                                            int64_t lo, int64_t hi) {
    for (int e = first; e < kp; e += step) {
        const int32_t id = en.cls[e];
        if (id < 0 || id < lo || id >= hi) continue;
        int earlier = 0, times = 0;
#pragma unroll 4
        for (int o = 0; o < kp; o += 4) {
            const int4 c = *reinterpret_cast<const int4 *>(en.cls + o);
            const int n = (c.x == id) + (c.y == id) + (c.z == id) + (c.w == id);
            times += n;
            earlier |= (c.x == id && o < e) | (c.y == id && o + 1 < e) | (c.z == id && o + 2 < e) | (c.w == id && o + 3 < e);
        }
        if (earlier) continue;
        float w = en.w[e];
        if (times > 1)
            for (int o = e + 1; o < kp; ++o)
                if (en.cls[o] == id) w += en.w[o];
        Elem<TG>::store(g, id, t.dense<TWO>(en.z[e]) - w);
    }
}

// ---------------------------------------------------------------------------
// rows in registers
// ---------------------------------------------------------------------------

// A thread's running maximum and the sums relative to it.
template <bool TWO> struct Online {
    float m = -INFINITY, sa = 0.f, sb = 0.f;
    // nothing but -infinity so far: distances are from 0 (a NaN is kept by the sums)
    __device__ __forceinline__ float from() const { return m == -INFINITY ? 0.f : m; }
    template <class V, int VE> __device__ __forceinline__ void add(const V &x, float ka, float kb) {
        float top = x.get(0);
#pragma unroll
        for (int e = 1; e < VE; ++e) top = fmaxf(top, x.get(e));
        if (top > m) {
            sa *= exp2_of((m - top) * ka);
            if constexpr (TWO) sb *= exp2_of((m - top) * kb);
            m = top;
        }
        const float at = from();
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float d = x.get(e) - at;
            sa += exp2_of(d * ka);
            if constexpr (TWO) sb += exp2_of(d * kb);
        }
    }
    // the sums relative to `top`, which is at least m
    __device__ __forceinline__ void to(float top, float ka, float kb) {
        const float d = m == top ? 0.f : m - top;
        sa *= exp2_of(d * ka);
        if constexpr (TWO) sb *= exp2_of(d * kb);
    }
};

// Maxima and sums over a row's threads with one meeting: a wavefront's in
// registers, then each wavefront joins all of theirs from LDS by itself.
// tm, ts: the teacher's.
template <class S> struct Meeting {
    static constexpr int kWaves = S::T > 64 ? S::T / 64 : 1;
    typedef float Shared[2][5][kWaves];
    static constexpr int kIn = S::T < 64 ? S::T : 64;
    template <int W, class Op> __device__ __forceinline__ static float fold(Op op, float v) {
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
        return v;
    }
    // each thread's own: `on`, and its entries' largest value; sum(tm) is its
    // entries' sum relative to tm
    template <bool TWO, class F>
    __device__ __forceinline__ static void inside(Online<TWO> &on, float &tm, float &ts, float ka, float kb, F &&sum) {
        const float top = fold<kIn>(Max{}, on.m);
        tm = fold<kIn>(Max{}, tm);
        on.to(top, ka, kb);
        on.m = top;
        on.sa = fold<kIn>(Add{}, on.sa);
        if constexpr (TWO) on.sb = fold<kIn>(Add{}, on.sb);
        ts = fold<kIn>(Add{}, sum(tm));
    }
    template <bool TWO> __device__ __forceinline__ static void put(Shared &sh, int turn, const Online<TWO> &on, float tm, float ts) {
        if constexpr (kWaves > 1)
            if ((threadIdx.x & 63) == 0) {
                const int w = threadIdx.x >> 6;
                sh[turn][0][w] = on.m;
                sh[turn][1][w] = on.sa;
                if constexpr (TWO) sh[turn][2][w] = on.sb;
                sh[turn][3][w] = tm;
                sh[turn][4][w] = ts;
            }
    }
    template <bool TWO>
    __device__ __forceinline__ static void join(const Shared &sh, int turn, Online<TWO> &on, float &tm, float &ts, float kt,
                                                float ka, float kb) {
        if constexpr (kWaves > 1) {
            const int w = threadIdx.x % kWaves;
            on.m = sh[turn][0][w];
            on.sa = sh[turn][1][w];
            if constexpr (TWO) on.sb = sh[turn][2][w];
            tm = sh[turn][3][w];
            ts = sh[turn][4][w];
            const float top = fold<kWaves>(Max{}, on.m), t_top = fold<kWaves>(Max{}, tm);
            on.to(top, ka, kb);
            on.m = top;
            on.sa = fold<kWaves>(Add{}, on.sa);
            if constexpr (TWO) on.sb = fold<kWaves>(Add{}, on.sb);
            ts = fold<kWaves>(Add{}, ts * exp2_of(tm == t_top ? 0.f : (tm - t_top) * kt));
            tm = t_top;
        }
    }
};

// Wavefronts to a SIMD that the registers are to leave room for.
template <class S> constexpr int waves_wanted() { return S::T >= 512 ? 4 : 1; }
// Vectors between a load and its use: a vector of 1,024 threads takes a CU's
// share of the memory 1.6 us, in and out.
constexpr int kLag = 2;
// A row passes one meeting of its threads, after which its constants are known;
// what is left of the row before (its listed classes' second store, its loss) is
// done after the same meeting, which orders it behind that row's dense stores.
template <class S, class TL, class TG, bool TWO>
__global__ void __launch_bounds__(S::kThreads, waves_wanted<S>()) distill_rows_kernel(DistillArgs a, float *row_loss) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    typedef Meeting<S> Meet;
    __shared__ typename Meet::Shared sh;
    __shared__ float sh_loss[2][Meet::kWaves];
    typedef Vec<TL, S::VE> V;
    const int kp = entries_padded(a.k), lane = S::lane();
    const int64_t c = a.c, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const TL *logits = static_cast<const TL *>(a.logits);
    TG *grad = static_cast<TG *>(a.g_out);
    const float ka = factor_a(a), kb = kLog2e, inv_t = 1.f / a.temperature, kt = inv_t * kLog2e;
    int64_t i = static_cast<int64_t>(blockIdx.x) * S::kRows + S::row();
    if (i >= a.b) return;  // threads of whole rows; above 64 a workgroup has one
    V r[S::NV], tail;
    Span<S, TL> span(logits + i * c, c);
    Online<TWO> on;
    // the first entry of each thread is fetched a row ahead
    Entry mine{-1, -INFINITY, 0.f};
    float scale = row_scale_of(a, i);
    if (scale != 0.f) {
        const TL *z = logits + i * c;
#pragma unroll
        for (int v = 0; v < S::NV; ++v)
            if (v < span.full) span.load(r[v], z, v);
        span.load_tail(tail, z);
        if (lane < kp) mine.load(a, i, lane);
        if (mine.cls >= 0) mine.z = Elem<TL>::load(z, mine.cls);
#pragma unroll
        for (int v = 0; v < S::NV; ++v)
            if (v < span.full) {
                span.trim(r[v], v);
                on.template add<V, S::VE>(r[v], ka, kb);
            }
        span.trim_tail(tail);
        on.template add<V, S::VE>(tail, ka, kb);
    }
    // the row before: its constants, its entries' set and where its gradient is
    RowTerms tp{0.f, ka, kb, 0.f, 0.f, false};
    int set = 0, turn = 0;
    int64_t before = -1;
    auto finish_before = [&]() {
        if (before < 0) return;
        const Entries en = entries_at(lds, S::row() * kSets + (set + kSets - 1) % kSets, kp);
        if (grad && tp.any) put_entries<TWO>(en, tp, kp, lane, S::T, grad + before * c, 0, c);
        if (lane == 0) {
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < Meet::kWaves; ++w) l += sh_loss[turn ^ 1][w];
            if constexpr (Meet::kWaves > 1) row_loss[before] = l;
        }
    };
    for (; i < a.b; i += step) {
        const int64_t next = i + step;
        const float next_scale = next < a.b ? row_scale_of(a, next) : 0.f;
        RawEntry coming{-1, 0};
        if (next_scale != 0.f && lane < kp) coming.load(a, next, lane);
        const Entries en = entries_at(lds, S::row() * kSets + set, kp);
        float tm = -INFINITY, ts = 0.f;
        if (scale != 0.f) {
            for (int e = lane; e < kp; e += S::T) {
                Entry x = mine;
                if (e >= S::T) {
                    x.load(a, i, e);
                    if (x.cls >= 0) x.z = Elem<TL>::load(logits, i * c + x.cls);
                }
                en.cls[e] = x.cls;
                en.w[e] = x.value;
                en.z[e] = x.z;
                tm = fmaxf(tm, x.value);
            }
            Meet::template inside<TWO>(on, tm, ts, ka, kb, [&](float top) {
                float x = 0.f;
                for (int e = lane; e < kp; e += S::T)
                    if (en.cls[e] >= 0 && e < a.k) x += exp2_of((en.w[e] - top) * kt);
                return x;
            });
            Meet::template put<TWO>(sh, turn, on, tm, ts);
        }
        row_sync<S>();
        finish_before();
        RowTerms t{0.f, ka, kb, 0.f, 0.f, false};
        float l = 0.f;
        if (scale != 0.f) {
            Meet::template join<TWO>(sh, turn, on, tm, ts, kt, ka, kb);
            t.m = on.m;
            const float s1 = TWO ? on.sb : on.sa;
            const LossTerms lt{a.alpha, a.temperature, inv_t, scale, tm, ts, logf(ts), t.m, logf(on.sa), logf(s1)};
            const bool soft = ts != 0.f, hard = en.cls[a.k] >= 0;
            for (int e = lane; e < kp; e += S::T) {
                float w = 0.f;
                if (en.cls[e] >= 0) l += e < a.k ? lt.teacher(en.w[e], en.z[e], &w) : lt.label(en.z[e], &w);
                en.w[e] = w;
            }
            l = Meet::template fold<Meet::kIn>(Add{}, l);
            t.any = soft || hard;
            const float cs = soft ? scale * a.alpha * a.temperature : 0.f, ch = hard ? scale * (1.f - a.alpha) : 0.f;
            t.ca = TWO ? cs / on.sa : (cs + ch) / on.sa;
            t.cb = ch / s1;
        }
        if constexpr (Meet::kWaves > 1) {
            if ((threadIdx.x & 63) == 0) sh_loss[turn][threadIdx.x >> 6] = l;
        } else {
            if (lane == 0) row_loss[i] = l;
        }
        const TL *below = logits + next * c;
        Entry ahead;
        ahead.take(a, coming, lane);
        if (ahead.cls >= 0) ahead.z = Elem<TL>::load(below, ahead.cls);
        // the gradient, vector by vector; the next row into its registers, and
        // its maximum and sums kLag vectors behind
        TG *g = grad + i * c;
        auto dense = [&](const V &x) {
            float o[S::VE];
#pragma unroll
            for (int e = 0; e < S::VE; ++e) o[e] = t.any ? t.dense<TWO>(x.get(e)) : 0.f;
            Vec<TG, S::VE> w;
            w.set(o);
            return w;
        };
        on = Online<TWO>{};
        auto take = [&](V &x) {
            on.template add<V, S::VE>(x, ka, kb);
            x.pin();
        };
        const Span<S, TL> to(below, c);
        const int to_full = next_scale != 0.f ? to.full : 0;
        if (grad) span.store_tail(dense(tail), g);
#pragma unroll
        for (int v = 0; v < S::NV; ++v) {
            if (grad && v < span.full) span.store(dense(r[v]), g, v);
            if (v < to_full) {
                to.load(r[v], below, v);
                if (v >= kLag) {
                    to.trim(r[v >= kLag ? v - kLag : 0], v - kLag);
                    take(r[v >= kLag ? v - kLag : 0]);
                }
            }
        }
        if (next_scale != 0.f) {
            to.load_tail(tail, below);
#pragma unroll
            for (int v = 0; v < S::NV; ++v)
                if (v < to_full && v >= to_full - kLag) {
                    to.trim(r[v], v);
                    take(r[v]);
                }
            to.trim_tail(tail);
            take(tail);
        }
        before = i;
        tp = t;
        span = to;
        mine = ahead;
        scale = next_scale;
        set = (set + 1) % kSets;
        turn ^= 1;
    }
    row_sync<S>();
    finish_before();
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
            Entry x;
            x.load(a, i, e);
            if (x.cls >= 0) st.z[i * kp + e] = Elem<TL>::load(z, x.cls);
        }
    const float ka = factor_a(a), kb = kLog2e;
    Online<TWO> on;
    for (int64_t c0 = lo; c0 < hi; c0 += kSplitThreads * S::VE) {
        Vec<TL, S::VE> r;
        const int64_t c = c0 + S::col(0);
        r.load_upto(z + c, hi - c, -INFINITY);
        on.template add<Vec<TL, S::VE>, S::VE>(r, ka, kb);
    }
    float top[1] = {on.m};
    over(Max{}, top);
    on.to(top[0], ka, kb);
    float s[2] = {on.sa, on.sb};
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
            Entry x;
            x.load(a, i, e);
            en.cls[e] = x.cls;
            en.w[e] = x.value;
            if (x.cls >= 0) en.z[e] = st.z[i * kp + e];
            mx[1] = fmaxf(mx[1], x.value);
        }
        over(Max{}, mx);
        t.m = mx[0];
        const float inv_t = 1.f / a.temperature;
        float s[3] = {0.f, 0.f, 0.f};
        for (int64_t e = threadIdx.x; e < p.parts; e += kSplitThreads) {
            const float d = q[e * 3] == t.m ? 0.f : q[e * 3] - t.m;
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

// Rows are split when they do not fit, and where so few long ones come that most
// CUs would have none (bf16, 64 entries, us whole and split: 1 x 20,000 12.7 and 15.1,
// 100 x 20,000 17 and 19; 1 x 65,536 18 and 15.5, 64 rows of it 23 and 19, 127 rows 25 and
// 24; 127 x 100,003 30 either way).
SplitPlan plan_split(int64_t b, int64_t c, int64_t k, int ldt) {
    SplitPlan p{1, c};
    const auto none = [](auto) {};
    const bool fits = ldt == GNN_BF16 ? with_shape<uint16_t>(c, k, none) : with_shape<float>(c, k, none);
    if (fits && (c < 32768 || b >= kCus / 2)) return p;
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
        const SplitPlan p = plan_split(b, c, k, dt);
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
        const SplitPlan p = plan_split(a.b, a.c, a.k, a.ldt);
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
            with_shape<TL>(a.c, a.k, [&](auto shape) {
                using S = decltype(shape);
                // one round of the CUs with what fits on each: workgroups walk
                // their rows and load each ahead
                const int64_t grid = std::min<int64_t>(ceil_div(a.b, S::kRows), kCus * (S::T >= 256 ? 1024 / S::T : 8));
                distill_rows_kernel<S, TL, TG, TWO>
                    <<<static_cast<unsigned>(grid), S::kThreads, kSets * S::kRows * entry_bytes, s>>>(a, row_loss);
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
