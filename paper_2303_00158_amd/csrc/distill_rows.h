// Which shape holds a row of the distillation loss in registers, and where a
// thread's vectors of such a row lie (distill.hip).
#pragma once

#include "row_dev.h"

namespace gnn {
namespace distill {

using row::Shape;
using row::Vec;

// Entries of a row's list, the label's behind the teacher's, in whole vectors.
__host__ __device__ inline int entries_padded(int64_t k) { return static_cast<int>((k + 1 + 3) / 4 * 4); }

// Sets of entries: a row's are read until after the next row's meeting, when a
// thread may be at the row after that.
constexpr int kSets = 3;

// A thread's share of a row of c elements, in vectors that lie in whole 128-byte
// lines whatever the row's own address (off them a row of 100,003 bf16 classes
// took 18% longer than one of 100,000).  `full` vectors hold elements in all of
// the row's threads (at most NV, the same in every thread) but for the first
// line's; the one after them is the row's end, of which some threads have a
// part or nothing.  One uniform count in place of every vector's bounds keeps
// those out of the registers: with bounds, 1,024 threads x 128 elements spilled
// 154.  Where a thread's vector reaches over the row's start or end, the row's
// first or last VE elements are loaded in its place, and those that are other
// threads' are masked when it is used (trim): nothing waits for the load.
template <class S, class TL> struct Span {
    int c, head, full, rest;  // head: elements from the line to the row; rest: from the tail's place to the row's end
    static constexpr int kLine = 128 / sizeof(TL);
    // the longest row: with kLine - 1 elements before it, `full` is at most NV
    static constexpr int64_t kMost = static_cast<int64_t>(S::T) * (S::E + S::VE) - kLine;
    static constexpr int kStep = S::T * S::VE;
    // whole vectors of a row, and where vector v of a thread starts in it
    __host__ __device__ __forceinline__ static int whole(int c, int head) { return (c + head) / kStep; }
    __host__ __device__ __forceinline__ static int place(int head, int v, int lane) {
        return (v * S::T + lane) * S::VE - head;
    }
    __device__ __forceinline__ Span(const TL *row, int64_t c_) {
        c = static_cast<int>(c_);
        head = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 127) / sizeof(TL));
        full = whole(c, head);
        rest = c - place(head, full, S::lane());
    }
    __device__ __forceinline__ static uint32_t off() { return static_cast<uint32_t>(S::lane()) * S::VE; }
    __device__ __forceinline__ int skip() const { return -place(head, 0, S::lane()); }  // of the first vector, before the row
    __device__ __forceinline__ bool first(int v) const { return v == 0 && skip() > 0; }
    template <class T> __device__ __forceinline__ T *at(T *row, int v) const { return row - head + v * kStep + off(); }
    // a whole vector (v < full)
    __device__ __forceinline__ void load(Vec<TL, S::VE> &x, const TL *row, int v) const {
        x.load(first(v) ? row : at(row, v));
    }
    __device__ __forceinline__ void trim(Vec<TL, S::VE> &x, int v) const {
        if (first(v)) x.keep(0, S::VE - skip());
    }
    template <class T> __device__ __forceinline__ void store(const Vec<T, S::VE> &x, T *row, int v) const {
        if (first(v)) x.store_some(row, 0, S::VE - skip());
        else x.store(at(row, v));
    }
    // the row's end; rows of less than one whole vector a thread are taken
    // element by element
    __device__ __forceinline__ void load_tail(Vec<TL, S::VE> &x, const TL *row) const {
        if (full == 0) x.load_some(at(row, 0), max(skip(), 0), rest, -INFINITY);
        else x.load(rest >= S::VE ? at(row, full) : row + c - S::VE);
    }
    __device__ __forceinline__ void trim_tail(Vec<TL, S::VE> &x) const {
        if (full != 0 && rest < S::VE) x.keep(S::VE - max(rest, 0), S::VE);
    }
    template <class T> __device__ __forceinline__ void store_tail(const Vec<T, S::VE> &x, T *row) const {
        if (full == 0) x.store_some(at(row, 0), max(skip(), 0), rest);
        else if (rest >= S::VE) x.store(at(row, full));
        else if (rest > 0) x.store_some(row + c - S::VE, S::VE - rest, S::VE);
    }
};

// go with the shape of a row of c classes in registers, at most 68 words a
// thread; false where none holds it.  A bf16 row may start twice as many elements
// into its line as an fp32 one, so the longest row goes by the logits' type.
// Long lists take a workgroup to a row: the sets of all its rows' entries lie in
// LDS (64 KB hold 112 entries of 16 rows, 454 of four).
template <class S, class TL, class F> bool if_fits(int64_t c, int64_t k, F &&go) {
    if (c > Span<S, TL>::kMost || kSets * S::kRows * entries_padded(k) * 12 > (64 << 10)) return false;
    go(S{});
    return true;
}
template <class TL, class F> bool with_shape(int64_t c, int64_t k, F &&go) {
    constexpr bool BF16 = sizeof(TL) == 2;
    constexpr int VE = BF16 ? 8 : 4;
    return if_fits<Shape<16, 8, VE>, TL>(c, k, go) || if_fits<Shape<64, 8, VE>, TL>(c, k, go) ||
           if_fits<Shape<64, 16, VE>, TL>(c, k, go) || if_fits<Shape<64, 32, VE>, TL>(c, k, go) ||
           if_fits<Shape<64, 64, VE>, TL>(c, k, go) || if_fits<Shape<256, 32, VE>, TL>(c, k, go) ||
           if_fits<Shape<256, 64, VE>, TL>(c, k, go) || if_fits<Shape<512, 64, VE>, TL>(c, k, go) ||
           if_fits<Shape<1024, 64, VE>, TL>(c, k, go) ||
           (BF16 && if_fits<Shape<1024, BF16 ? 128 : 64, VE>, TL>(c, k, go));
}

}  // namespace distill
}  // namespace gnn
