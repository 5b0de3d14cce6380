// Building blocks of the operators that hold a whole row in registers
// (layer_norm.hip, distill.hip).
#pragma once

#include "internal.h"

namespace gnn {
namespace row {

__device__ __forceinline__ int64_t live_rows(const int64_t *m_dev, int64_t cap_m) {
    return m_dev ? max(min(*m_dev, cap_m), int64_t(0)) : cap_m;
}

// ---------------------------------------------------------------------------
// VE consecutive elements as they lie in memory
// ---------------------------------------------------------------------------
template <class T, int VE> struct Vec {
    static constexpr int kWords = VE * static_cast<int>(sizeof(T)) / 4;
    uint32_t w[kWords];
    // accesses of 16 (8) bytes that ask for no more than the element's alignment
    static constexpr int kAt = kWords < 4 ? kWords : 4;
    struct __attribute__((packed, aligned(sizeof(T)))) Chunk {
        uint32_t w[kAt];
    };
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int q = 0; q < kWords / kAt; ++q) {
            const Chunk v = reinterpret_cast<const Chunk *>(p)[q];
#pragma unroll
            for (int e = 0; e < kAt; ++e) w[kAt * q + e] = v.w[e];
        }
    }
    __device__ __forceinline__ void store(T *p) const {
#pragma unroll
        for (int q = 0; q < kWords / kAt; ++q) {
            Chunk v;
#pragma unroll
            for (int e = 0; e < kAt; ++e) v.w[e] = w[kAt * q + e];
            reinterpret_cast<Chunk *>(p)[q] = v;
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float((e & 1) ? (w[e / 2] & 0xffff0000u) : (w[e / 2] << 16));
    }
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
            else w[i] = static_cast<uint32_t>(f32_to_bf16(x[2 * i])) | (static_cast<uint32_t>(f32_to_bf16(x[2 * i + 1])) << 16);
        }
    }
    // Keep the words as they are from here on: without it the compiler carries
    // the unpacked elements from one pass over a row to the next, which takes
    // twice the registers.
    __device__ __forceinline__ void pin() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    }
    // -infinity everywhere but in elements [lo, hi)
    __device__ __forceinline__ void keep(int lo, int hi) {
        constexpr int kPer = 4 / static_cast<int>(sizeof(T));
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80u, kMask = sizeof(T) == 4 ? 0xffffffffu : 0xffffu;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const int at = (e % kPer) * 16;
            if (e < lo || e >= hi) w[e / kPer] = (w[e / kPer] & ~(kMask << at)) | (kNone << at);
        }
    }
    // elements [lo, hi) of p; the rest are `fill`, or are not written
    __device__ __forceinline__ void load_some(const T *p, int lo, int hi, float fill) {
        float x[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = e >= lo && e < hi ? Elem<T>::load(p, e) : fill;
        set(x);
    }
    __device__ __forceinline__ void store_some(T *p, int lo, int hi) const {
#pragma unroll
        for (int e = 0; e < VE; ++e)
            if (e >= lo && e < hi) Elem<T>::store(p, e, get(e));
    }
    __device__ __forceinline__ void load_upto(const T *p, int64_t n, float fill = 0.f) {
        if (n >= VE) load(p);
        else load_some(p, 0, static_cast<int>(max(n, int64_t(0))), fill);
    }
    __device__ __forceinline__ void store_upto(T *p, int64_t n) const {
        if (n >= VE) store(p);
        else store_some(p, 0, static_cast<int>(max(n, int64_t(0))));
    }
};

// T threads to a row, E elements to a thread, in vectors of VE.
template <int T_, int E_, int VE_> struct Shape {
    static constexpr int T = T_, E = E_, VE = VE_, NV = E / VE;
    static constexpr int kThreads = T > 256 ? T : 256;
    static constexpr int kRows = kThreads / T;  // rows of a workgroup at a time
    __device__ __forceinline__ static int lane() { return static_cast<int>(threadIdx.x) % T; }
    // one value in a wavefront's scalar registers where a row is a wavefront's
    __device__ __forceinline__ static int row() {
        if constexpr (kRows == 1) return 0;
        const int r = static_cast<int>(threadIdx.x) / T;
        return T == 64 ? __builtin_amdgcn_readfirstlane(r) : r;
    }
    __device__ __forceinline__ static int64_t col(int v) { return (static_cast<int64_t>(v) * T + lane()) * VE; }
};

// Sums (or maxima) of N values over a row's threads, in all of them.  More than
// a wavefront meets in LDS, where two buffers in turn make one barrier enough.
struct Add {
    static constexpr float kNone = 0.f;
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    static constexpr float kNone = -INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
template <class S> struct RowReduce {
    static constexpr int kWaves = S::T > 64 ? S::T / 64 : 1, kMost = 3;
    typedef float Shared[2][kMost][kWaves];
    Shared &sh;
    int turn = 0;
    __device__ __forceinline__ explicit RowReduce(Shared &s) : sh(s) {}
    template <class Op, int N> __device__ __forceinline__ void operator()(Op op, float (&v)[N]) {
        static_assert(N <= kMost, "buffers hold kMost values");
#pragma unroll
        for (int o = (S::T < 64 ? S::T : 64) / 2; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] = op(v[n], __shfl_xor(v[n], o, 64));
        if constexpr (kWaves > 1) {
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int n = 0; n < N; ++n) sh[turn][n][wave] = v[n];
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float t = Op::kNone;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) t = op(t, sh[turn][n][w]);
                v[n] = t;
            }
            turn ^= 1;
        }
    }
};

// What a row's threads wrote to LDS (and to memory) before is seen by all of
// them after.
template <class S> __device__ __forceinline__ void row_sync() {
    if constexpr (S::T > 64) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

}  // namespace row
}  // namespace gnn
