// Matrix products of bf16 operands on the matrix cores (update_act.hip,
// update_act_bwd.hip): C = P Q, rows of P and columns of Q reduced over r,
// with fp32 accumulation, in output tiles of 256 x 256 down to 64 x 64.
//
// Four wavefronts (2 x 2) share a tile.  The reduction runs in chunks of 64: both
// operands' chunks are copied from memory straight into LDS (buffer loads with
// the LDS bit) into one of two stages, while the matrix cores work on the other,
// and a wavefront reads the fragments of the next half chunk from LDS into a
// second set of registers while it multiplies this one's.  So a chunk has one
// wait, for copies made a chunk ago, and one barrier.  A wavefront's part of the
// tile is as large as its registers hold (128 x 128 of a 256 x 256 tile: 256
// accumulators, two sets of 64 fragment registers), since what a chunk reads
// from LDS goes by its edges and what it multiplies by its area: per chunk, 128
// KB of fragments and 64 KB of copies pass the LDS (128 bytes a cycle: 1,536
// cycles) under 2,048 cycles of v_mfma_f32_16x16x32_bf16; eight wavefronts of
// 128 x 64 would read 192 KB.  Chunks are 64 deep for the copies' sake: a row's
// part of a chunk is a whole 128-byte line (with chunks of 32, four stages of
// them, every line came from the L2 twice: 8,192^3 took 1,000 us; now 818).
//
// Operand layouts, in memory and in LDS:
//  * N: rows of P (columns of Q) run along the reduction in memory.  LDS holds
//    128-byte rows whose eight 16-byte granules are XOR-swizzled by the row's low
//    three bits, so that fragment reads (16 rows of one granule) have no bank
//    conflicts.
//  * T: the reduction runs down the rows of a row-major matrix.  LDS holds the
//    chunk's 64 rows; fragments are read by the transposing ds_read_b64_tr_b16,
//    and 16-byte units are XOR-swizzled so that the 16 rows one such read
//    touches lie in distinct banks.
// Buffer descriptors bound every copy: what lies past the operand reads as
// zero, rows of the reduction as well as rows of the output.
#pragma once

#include "act_dev.h"
#include "gemm_wide_dev.h"
#include "row_dev.h"

namespace gnn {
namespace tile {

using wide::bf16x8;
using wide::f32x4;
using wide::i16x4;
using wide::i16x8;
using wide::lds_i16x4;
using wide::lds_void;

constexpr int kBK = 64;
constexpr int kOob = 0x7ffffff0;  // a byte offset past any operand

// MI x NI MFMA tiles of 16 x 16 a wavefront, 2 x 2 wavefronts, PER_CU workgroups
// to a CU.
template <int MI_, int NI_, int PER_CU_> struct Cfg {
    static constexpr int MI = MI_, NI = NI_, PER_CU = PER_CU_;
    static constexpr int BM = 32 * MI, BN = 32 * NI, kThreads = 256;
    static constexpr int CA = BM / 32, CB = BN / 32;  // copies of 1 KB a wavefront and chunk, of P and of Q
    static constexpr int kStageElems = (BM + BN) * kBK;
};

using Big = Cfg<8, 8, 1>;    // 256 x 256
using Big7 = Cfg<7, 8, 1>;   // 224 x 256
using Mid = Cfg<4, 4, 2>;    // 128 x 128
using Small = Cfg<2, 2, 4>;  // 64 x 64

// The tile size for an output of rows x cols over a reduction of `red`, and how many
// ways the reduction is split: the choice that takes the least time by the rounds
// of tiles that the CUs work through.  Measured: a chunk of a tile takes `busy` us of
// a CU that has all it holds (8,192^3: 1.34 PFLOP/s in 256 x 256 tiles, 1.12 in 128 x
// 128, 0.72 in 64 x 64), but no less than `lone` (250 x 16,384 x 256: 289, 158 and 121
// us); a tile takes `ends` us beside its chunks, for its first copies and its
// epilogue, which in large tiles nothing overlaps (14,591 x 512 x 1,024 with a residual:
// 39 us in 256 x 256 tiles, 35 in 128 x 128).  A split (fp32 partial tiles,
// added in order by another kernel) costs their bytes, out and in, and a launch;
// each has at least four chunks, and there are at most `splits`.  4,096 x 1,024 x 2,048: 43 us in 256 x 256 tiles, 24 in
// 128 x 128, 35 in 64 x 64; 8,192 x 4,096 x 4,096: 221, 266 and 410.
enum Pick { kBig, kBig7, kMid, kSmall };
struct Choice {
    Pick pick;
    int64_t nsplit;
};
struct Pace {
    double busy, lone, ends;
};
constexpr Pace kBigPace{1.6, 1.13, 20}, kBig7Pace{1.42, 1.02, 18}, kMidPace{0.48, 0.7, 4}, kSmallPace{0.19, 0.5, 1};
// us of `tiles` tiles of `chunks` chunks, split n ways
template <class C> inline double cost(int64_t tiles, int64_t chunks, int64_t n, const Pace &p) {
    constexpr int64_t round = 256 * C::PER_CU;
    const double each = static_cast<double>(ceil_div(chunks, n));
    const int64_t last = ceil_div(n * tiles % round, int64_t(256));  // tiles a CU holds in the last round
    double t = static_cast<double>(n * tiles / round * C::PER_CU) * (each * p.busy + p.ends);
    if (last) t += each * std::max(p.lone, p.busy * last) + p.ends * last;
    return t;
}
inline Choice choose(int64_t rows, int64_t cols, int64_t red, int64_t splits = 16) {
    Choice best{kSmall, 1};
    double least = -1;
    auto look = [&](auto cfg, Pick pick, const Pace &p) {
        using C = decltype(cfg);
        const int64_t chunks = std::max<int64_t>(ceil_div(red, int64_t(kBK)), 1);
        const int64_t tiles = ceil_div(rows, int64_t(C::BM)) * ceil_div(cols, int64_t(C::BN)), round = 256 * C::PER_CU;
        for (int64_t n = 1; n <= splits && (n == 1 || (n * tiles <= round && n * 4 <= chunks)); n *= 2) {
            const double t = cost<C>(tiles, chunks, n, p) + (n > 1 ? 4 + static_cast<double>(n) * rows * cols * 8 / 4e6 : 0);
            if (least < 0 || t < least) {
                least = t;
                best = Choice{pick, n};
            }
        }
    };
    look(Big{}, kBig, kBigPace);
    look(Big7{}, kBig7, kBig7Pace);
    look(Mid{}, kMid, kMidPace);
    look(Small{}, kSmall, kSmallPace);
    return best;
}
// Reduction elements [*beg, *end) of split `split`, whole chunks.
__device__ __forceinline__ void split_of(int64_t red, int64_t nsplit, int64_t split, int64_t *beg, int64_t *end) {
    const int64_t per = ceil_div(ceil_div(red, nsplit), int64_t(kBK)) * kBK;
    *beg = min(red, split * per);
    *end = min(red, *beg + per);
}

// --- one operand's copies --------------------------------------------------
// T layout: place of 16-byte unit u in reduction row k of a W-wide chunk
template <int W> __device__ __forceinline__ int t_unit(int k, int u) {
    return u ^ ((((k & 3) | ((k >> 1) & 12)) << 1) & (W / 8 - 1));
}
template <int W> __device__ __forceinline__ int t_idx(int k, int c) {
    return k * W + (t_unit<W>(k, c >> 3) << 3) + (c & 7);
}

// N layout: `rows` output rows of `red` reduction elements (a multiple of 8)
// from x0, or the first `half` of them (a multiple of 64) from x0 and the others
// from x1.  T layout: `red` reduction rows, from whose ends x0's column is `rows` values
// away, a multiple of 8 (a copy of 16 bytes that reaches past the bound is all 0).
struct Operand {
    const uint16_t *x0, *x1;
    int64_t ld, half, rows, red;
};

template <int W, int COPIES, bool T> struct Copier {
    __amdgpu_buffer_rsrc_t r0, r1;
    const uint16_t *x0;
    int64_t ld, left;  // T: bytes from x0 to the operand's end
    int half, red;     // N
    int off[COPIES], k8;
    __device__ static __amdgpu_buffer_rsrc_t desc(const uint16_t *p, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p), 0,
                                                 static_cast<int>(min(max(bytes, int64_t(0)), int64_t(kOob))), 0x00020000);
    }
    __device__ __forceinline__ explicit Copier(const Operand &o) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        x0 = o.x0;
        ld = o.ld;
        if constexpr (T) {
            left = o.red > 0 ? ((o.red - 1) * o.ld + o.rows) * 2 : 0;
            constexpr int kRows = 512 / W;  // reduction rows of one copy
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int k = (wave + 4 * i) * kRows + lane * 8 / W, u = (lane * 8 % W) / 8;
                off[i] = static_cast<int>((k * o.ld + t_unit<W>(k, u) * 8) * 2);
            }
        } else {
            red = static_cast<int>(o.red);
            half = o.x1 ? static_cast<int>(o.half) : red;
            const int64_t rows = min(o.rows, int64_t(W));
            auto bytes = [&](int64_t cols) { return rows > 0 ? ((rows - 1) * o.ld + cols) * 2 : 0; };
            r0 = desc(o.x0, bytes(half));
            r1 = desc(o.x1 ? o.x1 : o.x0, bytes(o.red - half));
            k8 = ((lane & 7) ^ (lane >> 3)) * 8;
#pragma unroll
            for (int i = 0; i < COPIES; ++i)
                off[i] = static_cast<int>((((wave + 4 * i) * 8 + (lane >> 3)) * o.ld + k8) * 2);
        }
    }
    // copy i of chunk c into `dst` (this operand's part of a stage)
    __device__ __forceinline__ void copy(int c, uint16_t *dst, int i) const {
#if defined(__HIP_DEVICE_COMPILE__)  // the LDS-bit buffer load exists for the device pass only
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if constexpr (T) {
            const int64_t at = static_cast<int64_t>(c) * kBK * ld;
            const __amdgpu_buffer_rsrc_t r = desc(x0 + at, left - at * 2);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(dst + (wave + 4 * i) * 512), 16, off[i], 0, 0, 0);
        } else {
            const int k0 = c * kBK;
            const bool hi = k0 >= half;
            const __amdgpu_buffer_rsrc_t r = hi ? r1 : r0;
            const int base = (hi ? k0 - half : k0) * 2;
            const bool in = k0 + k8 < red;  // past the last column lies the next row
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(dst + (wave + 4 * i) * 512), 16,
                                                     in ? off[i] : kOob, base, 0, 0);
        }
#endif
    }
};

// A fragment of 16 output rows (columns) from r0 in half `sub` of a chunk: lane l
// holds row r0 + l % 16, reduction elements 32 sub + 8 (l / 16) .. + 7.
template <int W, bool T> __device__ __forceinline__ bf16x8 frag(const uint16_t *S, int r0, int sub) {
    const int lane = threadIdx.x & 63;
    if constexpr (T) {
        const int k = (lane >> 4) * 8 + ((lane >> 2) & 3), c = r0 + 4 * (lane & 3);
        const uint16_t *s = S + sub * 32 * W;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(s + t_idx<W>(k, c)));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(s + t_idx<W>(k + 4, c)));
        const i16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, v);
    } else {
        const int g = (sub * 4 + (lane >> 4)) ^ (lane & 7);
        return *reinterpret_cast<const bf16x8 *>(S + (r0 + (lane & 15)) * kBK + g * 8);
    }
}

// --- the product of one tile ------------------------------------------------
// Q's fragment is the instruction's first operand, so a lane holds four
// consecutive columns of one row: v[i][j][q] is row 16 i + lane % 16, column
// 16 j + 4 (lane / 16) + q of the wavefront's part, and the epilogue needs no LDS.
template <class C> struct Acc {
    f32x4 v[C::MI][C::NI];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < C::MI; ++i)
#pragma unroll
            for (int j = 0; j < C::NI; ++j) v[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};
// acc += the product of two fragments, in place in the accumulation registers.
// Written out, because the compiler's own choice of form for 256 accumulators
// moved them between registers in every pass (532 moves beside 256 of these).
// The wait states that it would otherwise see to: settle() covers the first use of the
// sums; and the two that the instruction needs behind a move into one of its
// operands are free of charge as long as there is none, which is the case where
// fragments come from LDS reads (they have a wait of their own) and the sums stay in
// place: tests/test_tile_code.py holds the built code to it.  (Two wait states with
// every instruction cost 4% of the loop.)
__device__ __forceinline__ void mma(f32x4 &acc, const bf16x8 &x, const bf16x8 &y) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(x), "v"(y));
}
// Each sum passes through a statement of no instructions behind the wait, so that
// what reads it cannot be moved in front (tests/test_tile_sums.py).
template <class C> __device__ __forceinline__ void settle(Acc<C> &acc) {
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
        for (int j = 0; j < C::NI; ++j) asm volatile("" : "+a"(acc.v[i][j]));
}

template <class C> struct Frags {
    bf16x8 a[C::MI], b[C::NI];
};

// The stages are separate LDS arrays, so that the compiler sees that reads of one
// do not wait for copies into the other.
struct Ring {
    uint16_t *st[2];
};

template <class C, bool TA, bool TB> struct Product {
    Copier<C::BM, C::CA, TA> a;
    Copier<C::BN, C::CB, TB> b;
    __device__ __forceinline__ Product(const Operand &oa, const Operand &ob) : a(oa), b(ob) {}

    static constexpr int kCopies = C::CA + C::CB, kFrags = C::MI + C::NI, kMma = C::MI * C::NI;
    __device__ __forceinline__ void copy(int c, uint16_t *stage, int n) const {
        if (n < C::CA) a.copy(c, stage, n);
        else b.copy(c, stage + C::BM * kBK, n - C::CA);
    }
    // fragment n of half `sub` of a chunk: the columns' first, then the rows'
    __device__ __forceinline__ static void read(Frags<C> &f, const uint16_t *stage, int sub, int n) {
        const int wave = threadIdx.x >> 6;
        if (n < C::NI) f.b[n] = frag<C::BN, TB>(stage + C::BM * kBK, ((wave & 1) * C::NI + n) * 16, sub);
        else f.a[n - C::NI] = frag<C::BM, TA>(stage, ((wave >> 1) * C::MI + n - C::NI) * 16, sub);
    }
    // MFMAs [from, to) of a half chunk
    __device__ __forceinline__ static void multiply(Acc<C> &acc, const Frags<C> &f, int from, int to) {
#pragma unroll
        for (int m = from; m < to; ++m) mma(acc.v[m / C::NI][m % C::NI], f.b[m % C::NI], f.a[m / C::NI]);
    }

    // Chunk c, which lies in stage AT.  Its first half: the second half's
    // fragments are read among its MFMAs, and the scheduling barriers keep them
    // there.  Its second half: own copies of chunk c + 1 have landed and own reads
    // of chunk c are here, then everyone's; chunk c + 1's first fragments are
    // read, and stage AT takes chunk c + 2.
    template <int AT> __device__ __forceinline__ void step(Acc<C> &acc, Frags<C> (&f)[2], const Ring &ring, int c) const {
#pragma unroll
        for (int s = 0; s < kFrags; ++s) {
            read(f[1], ring.st[AT], 1, s);
            __builtin_amdgcn_sched_barrier(0);
            multiply(acc, f[0], s * kMma / kFrags, (s + 1) * kMma / kFrags);
            __builtin_amdgcn_sched_barrier(0);
        }
        wide::chunk_barrier<wide::waitcnt(0, 0)>();
        constexpr int kSlots = kFrags + kCopies;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            // copies stand evenly among the reads
            const int n = s * kCopies / kSlots;
            if ((s + 1) * kCopies / kSlots > n) copy(c + 2, ring.st[AT], n);
            else read(f[0], ring.st[AT ^ 1], 0, s - n);
            __builtin_amdgcn_sched_barrier(0);
            multiply(acc, f[1], s * kMma / kSlots, (s + 1) * kMma / kSlots);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // acc += the product over `chunks` chunks.  Copies past the last chunk are
    // of zeros; an odd count multiplies one chunk of them (with the last chunk
    // in code of its own, the compiler moved accumulators about).  MOVES: what follows
    // may make the compiler move accumulators on the loop's way out, in front
    // of settle()'s wait (an epilogue with branches did), so the loop's end waits
    // itself: 18 states of some 5,400 cycles.
    template <bool MOVES = false> __device__ __forceinline__ void run(Acc<C> &acc, const Ring &ring, int chunks) const {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < kCopies; ++n) copy(s, ring.st[s], n);
        Frags<C> f[2];
        wide::chunk_barrier<wide::waitcnt(kCopies, 15)>();
#pragma unroll
        for (int n = 0; n < kFrags; ++n) read(f[0], ring.st[0], 0, n);
        for (int c = 0; c < chunks; c += 2) {
            step<0>(acc, f, ring, c);
            step<1>(acc, f, ring, c + 1);
            if constexpr (MOVES) asm volatile("s_nop 15\n\ts_nop 1" ::: "memory");
        }
        wide::chunk_barrier<wide::waitcnt(0, 0)>();  // the stages are drained
        settle(acc);
    }
};

// --- the tile's place ---------------------------------------------------------
// Tiles are dealt to the XCDs in contiguous ranges (wide::xcd_item), in an order
// that takes kGroup row tiles down before it moves a column on: the 32 tiles that
// an XCD's CUs work on at a time then share 4 row blocks and 8 column blocks
// in its L2, in place of one and 32.
constexpr int64_t kGroup = 4;
__device__ __forceinline__ void tile_of(int64_t t, int64_t tm, int64_t tn, int64_t *m, int64_t *n) {
    const int64_t per = kGroup * tn, g = t / per, in = t - g * per, height = min(kGroup, tm - g * kGroup);
    *m = g * kGroup + in % height;
    *n = in / height;
}

// --- the epilogue ---------------------------------------------------------------
// out = act(acc + bias) + residual for rows below M, and acc + bias to z; rows of
// `ld` elements, which the output has columns.
struct Epilogue {
    const float *bias;
    const void *residual;
    void *z, *out;
    int64_t ld;
};

// Eight elements of a row, `room` of them inside it.
template <class T> __device__ __forceinline__ void put8(T *p, int64_t room, const float (&x)[8]) {
    if (room >= 8) {
        row::Vec<T, 8> v;
#pragma unroll
        for (int e = 0; e < (sizeof(T) == 2 ? 4 : 8); ++e) {
            if constexpr (sizeof(T) == 2) v.w[e] = wide::pack_bf16(x[2 * e], x[2 * e + 1]);
            else v.w[e] = __float_as_uint(x[e]);
        }
        v.store(p);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < room) Elem<T>::store(p, e, x[e]);
    }
}

// The epilogue of a wavefront's part of the tile, whose origin in the output is
// (row0, col0).  Of two neighbouring MFMA tiles' columns a lane holds four each;
// exchanging one half with the lane 16 away gives every lane eight consecutive ones
// of one of the two, so that an instruction moves 16 bytes a lane and 64 a row
// of bf16 (with four columns a lane, 8 and 32).  The residual is asked
// for whole before the first row is finished, in the fragments' registers (26,624 x 1,536
// x 1,024: 141 us, with one row ahead 147), an fp32 one two rows ahead.
template <class C, int ACT, class T>
__device__ __forceinline__ void finish(const Acc<C> &acc, const Epilogue &p, int64_t row0, int64_t col0, int64_t M) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    constexpr int kPairs = C::NI / 2;
    const int64_t r0 = row0 + (lane & 15), c0 = col0 + (g & 1) * 16 + (g >> 1) * 8;
    const T *res = static_cast<const T *>(p.residual);
    T *z = static_cast<T *>(p.z), *out = static_cast<T *>(p.out);
    float bias[kPairs][8];
#pragma unroll
    for (int j = 0; j < kPairs; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[j][e] = p.bias && c0 + 32 * j + e < p.ld ? p.bias[c0 + 32 * j + e] : 0.f;
    constexpr int kAhead = sizeof(T) == 2 ? C::MI : 2;
    row::Vec<T, 8> ahead[kAhead][kPairs];
    auto fetch = [&](int i) {
        const int64_t r = r0 + 16 * i;
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
            if (res && r < M && c0 + 32 * j + 8 <= p.ld) ahead[i % kAhead][j].load(res + r * p.ld + c0 + 32 * j);
    };
#pragma unroll
    for (int i = 0; i < kAhead && i < C::MI; ++i) fetch(i);
#pragma unroll
    for (int i = 0; i < C::MI; ++i) {
        const int64_t r = r0 + 16 * i;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            float x[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc.v[i][2 * j][q]),
                                                                  __float_as_uint(acc.v[i][2 * j + 1][q]), false, false);
                x[q] = __uint_as_float(two[0]);
                x[q + 4] = __uint_as_float(two[1]);
            }
            const int64_t c = c0 + 32 * j, at = r * p.ld + c, room = p.ld - c;
            if (r >= M || room <= 0) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += bias[j][e];
            if (z) put8(z + at, room, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = act::apply<ACT>(x[e]);
            if (res) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (room >= 8) x[e] += ahead[i % kAhead][j].get(e);
                    else if (e < room) x[e] += Elem<T>::load(res, at + e);
                }
            }
            put8(out + at, room, x);
        }
        if (i + kAhead < C::MI) fetch(i + kAhead);
    }
}

}  // namespace tile
}  // namespace gnn
