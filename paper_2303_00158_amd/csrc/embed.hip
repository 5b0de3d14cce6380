// Lookup of rows of a trained table, scaled, and the table's gradient.
//
// The lookup is bound by memory: each named row once in (rows that repeat come
// from the caches) and each output row once out.
//
// The gradient sums the rows of g that name the same table row.  Their
// positions are sorted by id (a stable radix sort, so every sum has the order of
// its positions), cut into tiles of equal length, and each tile's runs of equal ids are
// summed in registers; a run inside one tile goes straight to the table.  Of a run
// that crosses tiles each tile leaves a partial row, which the next launch adds in order: a
// frequent id costs no more than as many rare ones, and there are no
// floating-point atomics.  Where the gradient is not added to what the table
// holds, rows that no id names are written with zeros in the same launch.
#include <type_traits>

#include "internal.h"
#include "row_dev.h"

namespace gnn {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
struct LookupArgs {
    const void *table;
    int64_t rows, dim, stride;
    const int64_t *ids, *n_dev;
    int64_t cap;
    float scale;
    void *out;
    int64_t passes;  // vectors of a row, in steps of the lanes that share it
};

// LANES lanes to a row, VE elements a lane; a wavefront takes 64 / LANES rows side by side,
// UNITS such (or passes of a row) in flight: four where there are many, else two, so that twice
// the wavefronts wait for memory (26,624 rows of 256 fp32 values 11.3 us with two, 12.6 with
// four, 14.7 with eight; 131,072 of 4,096 bf16 310, 302 and 316).
constexpr int64_t kFewUnits = 1 << 17;
template <class TI, class TO, int VE, int LANES,
    int UNITS> __global__ void __launch_bounds__(kThreads) embed_fwd_kernel(LookupArgs a) {
    constexpr int kRows = 64 / LANES;
    const int64_t n = row::live_rows(a.n_dev, a.cap);
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t units = ceil_div(n, int64_t(kRows)) * a.passes;
    const int64_t waves = static_cast<int64_t>(gridDim.x) * kWaves,
        wave = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const TI *table = static_cast<const TI *>(a.table);
    TO *out = static_cast<TO *>(a.out);
    for (int64_t u0 = wave * UNITS; u0 < units; u0 += waves * UNITS) {
        int64_t r[UNITS], c[UNITS], id[UNITS];
        row::Vec<TI, VE> x[UNITS];
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
            const int64_t u = u0 + k, block = u / a.passes;
            r[k] = block * kRows + slot;
            c[k] = ((u - block * a.passes) * LANES + lane) * VE;
            id[k] = u < units && r[k] < n ? a.ids[r[k]] : -1;
        }
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
            const bool there = id[k] >= 0 && id[k] < a.rows;
            x[k].load_upto(table + (there ? id[k] : 0) * a.stride + c[k], there ? a.dim - c[k] : 0);
        }
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
            if (u0 + k >= units || r[k] >= n || c[k] >= a.dim) continue;
            float y[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) y[e] = id[k] >= 0 && id[k] < a.rows ? x[k].get(e) * a.scale : 0.f;
            row::Vec<TO, VE> o;
            o.set(y);
            o.store_upto(out + r[k] * a.dim + c[k], a.dim - c[k]);
        }
    }
}

// go(tag) with the lanes to a row of `vectors` vectors
template <class F> void with_lanes(int64_t vectors, F &&go) {
    if (vectors > 32) go(std::integral_constant<int, 64>{});
    else if (vectors > 16) go(std::integral_constant<int, 32>{});
    else if (vectors > 8) go(std::integral_constant<int, 16>{});
    else if (vectors > 4) go(std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 4>{});
}
// go(tag of the input's type, tag of the output's, elements of a 16-byte vector of the wider)
template <class F> void with_types(int idt, int odt, F &&go) {
    constexpr std::integral_constant<int, 8> eight{};
    constexpr std::integral_constant<int, 4> four{};
    if (idt == GNN_BF16) {
        if (odt == GNN_BF16) go(uint16_t{}, uint16_t{}, eight);
        else go(uint16_t{}, float{}, four);
    } else {
        if (odt == GNN_BF16) go(float{}, uint16_t{}, four);
        else go(float{}, float{}, four);
    }
}

// ---------------------------------------------------------------------------
// the gradient: positions sorted by id
// ---------------------------------------------------------------------------
// Keys are ids; what names no row, and positions at or past the count, get the
// key `rows` and come last.  A stable radix sort, least digit first.  Up to kSortTile
// positions one workgroup does all of it in LDS (8,192 positions of 32,000 rows: 36 us in
// four launches, 20 in this one).  More take two launches a digit: one counts each
// tile's digits, the next moves the tile's pairs behind all smaller digits and behind
// the same digit in earlier tiles, adding up the tiles' counts by itself.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortKeys = 8, kSortTile = kSortThreads * kSortKeys;  // of the one workgroup
constexpr int kMoveKeys = 2, kMoveTile = kSortThreads * kMoveKeys;  // of a tile among others

struct SortArgs {
    const int64_t *ids, *n_dev;
    int64_t cap, rows;
    uint32_t *key[2], *pos[2];
    uint32_t *counts;  // tiles x bins
    uint32_t *totals;  // bins
    int64_t tiles;
    int passes;
};
// Up to so many tiles each adds up the others' counts by itself (128 KB to 2 MB out of
// the L2, a few us); above, what that reads grows with the square of the tiles, and a launch
// of its own makes the counts of earlier tiles.
constexpr int64_t kDirectTiles = 256;

// Digits of BITS bits, and the counts of a tile's wavefronts.
template <int BITS> struct Digits {
    static constexpr int kBins = 1 << BITS;
    typedef uint32_t WaveBins[kSortWaves][kBins];
    __device__ __forceinline__ static uint32_t of(uint32_t key, int pass) { return (key >> (BITS * pass)) & (kBins - 1); }

    // own[k] = how many of the wavefront's earlier elements (of smaller k, or in a lower lane)
    // have the digit of its element k; bins[wave] = the wavefront's counts.
    template <int KEYS>
    __device__ __forceinline__ static void rank(const uint32_t (&digit)[KEYS], const bool (&in)[KEYS], int rounds,
                                                WaveBins &bins,
                                                uint32_t (&own)[KEYS]) {
        const int wave = threadIdx.x >> 6;
        for (int i = threadIdx.x; i < kSortWaves * kBins; i += kSortThreads) (&bins[0][0])[i] = 0;
        __syncthreads();
        volatile uint32_t *mine = bins[wave];
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            if (k >= rounds) break;
            // lanes whose digit has the same bits, in two halves: a bit costs the lane four instructions
            const uint64_t there = __ballot(in[k]);
            uint32_t lo = static_cast<uint32_t>(there), hi = static_cast<uint32_t>(there >> 32);
#pragma unroll
            for (int b = 0; b < BITS; ++b) {
                const uint32_t bit = static_cast<uint32_t>(static_cast<int32_t>(digit[k] << (31 - b)) >> 31);  // all ones, or none
                const uint64_t set = __ballot(bit != 0);
                lo &= ~(static_cast<uint32_t>(set) ^ bit);
                hi &= ~(static_cast<uint32_t>(set >> 32) ^ bit);
            }
            const uint32_t below = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
            const uint32_t before = in[k] ? mine[digit[k]] : 0;
            own[k] = before + below;
            __builtin_amdgcn_wave_barrier();
            if (in[k] && below == 0) mine[digit[k]] = before + __popc(lo) + __popc(hi);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
    }

    // bins[w][d] becomes the place of wavefront w's first element of digit d, where all
    // smaller digits take `total` places of theirs and digit d starts `earlier` places on.
    // total and earlier: of the digits that threads 0 .. kSortThreads hold, kEach each.
    static constexpr int kEach = kBins > kSortThreads ? kBins / kSortThreads : 1;
    __device__ __forceinline__ static void place(WaveBins &bins, const uint32_t (&total)[kEach],
                                                 const uint32_t (&earlier)[kEach],
                                                 uint32_t *sh) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        uint32_t mine = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) mine += total[e];
        uint32_t sum = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = __shfl_up(sum, o, 64);
            if (lane >= o) sum += y;
        }
        if (lane == 63) sh[wave] = sum;
        __syncthreads();
        uint32_t at = sum - mine;
        for (int w = 0; w < wave; ++w) at += sh[w];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int d = threadIdx.x * kEach + e;
            if (d < kBins) {
                uint32_t to = at + earlier[e], c[kSortWaves];
#pragma unroll
                for (int w = 0; w < kSortWaves; ++w) c[w] = bins[w][d];
#pragma unroll
                for (int w = 0; w < kSortWaves; ++w) {
                    bins[w][d] = to;
                    to += c[w];
                }
            }
            at += total[e];
        }
        __syncthreads();
    }
};

__device__ __forceinline__ uint32_t key_of(const SortArgs &a, int64_t i, int64_t n) {
    if (i >= n) return static_cast<uint32_t>(a.rows);
    const int64_t id = a.ids[i];
    return static_cast<uint32_t>(id >= 0 && id < a.rows ? id : a.rows);
}
// Element k of this thread: a wavefront's elements are consecutive, 64 to a round.
__device__ __forceinline__ int64_t sort_at(int64_t tile, int rounds, int k) {
    return tile * (kSortThreads * rounds) + (threadIdx.x >> 6) * (64 * rounds) + k * 64 + (threadIdx.x & 63);
}

template <int BITS> __global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(SortArgs a) {
    using D = Digits<BITS>;
    __shared__ typename D::WaveBins bins;
    __shared__ uint32_t keys[kSortTile], places[kSortTile], sh[kSortWaves];
    const int64_t n = row::live_rows(a.n_dev, a.cap);
    const int rounds = static_cast<int>(ceil_div(a.cap, int64_t(kSortThreads)));
    uint32_t x[kSortKeys], p[kSortKeys], digit[kSortKeys], own[kSortKeys];
    bool in[kSortKeys];
#pragma unroll
    for (int k = 0; k < kSortKeys; ++k) {
        const int64_t i = sort_at(0, rounds, k);
        in[k] = k < rounds && i < a.cap;
        x[k] = in[k] ? key_of(a, i, n) : 0;
        p[k] = static_cast<uint32_t>(i);
    }
    for (int pass = 0; pass < a.passes; ++pass) {
#pragma unroll
        for (int k = 0; k < kSortKeys; ++k) digit[k] = D::of(x[k], pass);
        D::rank(digit, in, rounds, bins, own);
        uint32_t total[1] = {0}, none[1] = {0};
        if (threadIdx.x < D::kBins)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) total[0] += bins[w][threadIdx.x];
        D::place(bins, total, none, sh);
        const bool last = pass + 1 == a.passes;
        uint32_t *key_to = last ? a.key[0] : keys, *pos_to = last ? a.pos[0] : places;
#pragma unroll
        for (int k = 0; k < kSortKeys; ++k)
            if (in[k]) {
                const uint32_t to = bins[threadIdx.x >> 6][digit[k]] + own[k];
                key_to[to] = x[k];
                pos_to[to] = p[k];
            }
        if (last) return;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSortKeys; ++k)
            if (in[k]) {
                x[k] = keys[sort_at(0, rounds, k)];
                p[k] = places[sort_at(0, rounds, k)];
            }
    }
}

template <int BITS> __global__ void __launch_bounds__(kSortThreads) embed_count_kernel(SortArgs a, int pass) {
    using D = Digits<BITS>;
    __shared__ uint32_t bins[D::kBins];
    const int64_t n = row::live_rows(a.n_dev, a.cap), tile = blockIdx.x;
    uint32_t x[kMoveKeys];
#pragma unroll
    for (int k = 0; k < kMoveKeys; ++k) {
        const int64_t i = sort_at(tile, kMoveKeys, k);
        x[k] = i >= a.cap ? 0 : pass == 0 ? key_of(a, i, n) : a.key[pass & 1][i];
    }
    for (int d = threadIdx.x; d < D::kBins; d += kSortThreads) bins[d] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kMoveKeys; ++k) {
        const int64_t i = sort_at(tile, kMoveKeys, k);
        if (i >= a.cap) continue;
        if (pass == 0) {
            a.key[0][i] = x[k];
            a.pos[0][i] = static_cast<uint32_t>(i);
        }
        atomicAdd(&bins[D::of(x[k], pass)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < D::kBins; d += kSortThreads) a.counts[tile * D::kBins + d] = bins[d];
}

// counts[t][d] becomes the sum over the tiles before t, totals[d] the sum over all: 32 digits
// of a workgroup, the tiles in 32 ranges.
template <int BITS> __global__ void __launch_bounds__(kSortThreads) embed_scan_kernel(SortArgs a) {
    constexpr int kBins = Digits<BITS>::kBins;
    __shared__ uint32_t sh[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, d = blockIdx.x * 32 + x;
    const int64_t per = ceil_div(a.tiles, int64_t(32)), beg = min(a.tiles, y * per), end = min(a.tiles, beg + per);
    uint32_t sum = 0;
#pragma unroll 8
    for (int64_t t = beg; t < end; ++t) sum += a.counts[t * kBins + d];
    sh[y][x] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int q = 0; q < y; ++q) before += sh[q][x];
    if (y == 31) a.totals[d] = before + sum;
#pragma unroll 8
    for (int64_t t = beg; t < end; ++t) {
        const uint32_t c = a.counts[t * kBins + d];
        a.counts[t * kBins + d] = before;
        before += c;
    }
}

template <int BITS> __global__ void __launch_bounds__(kSortThreads) embed_move_kernel(SortArgs a, int pass) {
    using D = Digits<BITS>;
    __shared__ typename D::WaveBins bins;
    __shared__ uint32_t sh[kSortWaves], sums[2][kSortThreads];
    const int64_t tile = blockIdx.x;
    const uint32_t *key = a.key[pass & 1], *pos = a.pos[pass & 1];
    uint32_t x[kMoveKeys], p[kMoveKeys], digit[kMoveKeys], own[kMoveKeys];
    bool in[kMoveKeys];
#pragma unroll
    for (int k = 0; k < kMoveKeys; ++k) {
        const int64_t i = sort_at(tile, kMoveKeys, k);
        in[k] = i < a.cap;
        x[k] = in[k] ? key[i] : 0;
        p[k] = in[k] ? pos[i] : 0;
        digit[k] = D::of(x[k], pass);
    }
    // a digit's places: in all tiles, and in earlier ones
    uint32_t total[D::kEach], earlier[D::kEach];
    auto add_up = [&](int d, int64_t first, int64_t step, uint32_t &all, uint32_t &before) {
        all = before = 0;
        if (a.tiles > kDirectTiles) {
            if (first == 0) {
                all = a.totals[d];
                before = a.counts[tile * D::kBins + d];
            }
            return;
        }
#pragma unroll 8
        for (int64_t t = first; t < a.tiles; t += step) {
            const uint32_t c = a.counts[t * D::kBins + d];
            all += c;
            before += t < tile ? c : 0;
        }
    };
    if constexpr (D::kBins >= kSortThreads) {
#pragma unroll
        for (int e = 0; e < D::kEach; ++e) add_up(threadIdx.x * D::kEach + e, 0, 1, total[e], earlier[e]);
    } else {
        constexpr int kParts = kSortThreads / D::kBins;
        const int d = threadIdx.x % D::kBins;
        add_up(d, threadIdx.x / D::kBins, kParts, sums[0][threadIdx.x], sums[1][threadIdx.x]);
        __syncthreads();
        total[0] = earlier[0] = 0;
        if (threadIdx.x < D::kBins)
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                total[0] += sums[0][q * D::kBins + d];
                earlier[0] += sums[1][q * D::kBins + d];
            }
    }
    D::rank(digit, in, kMoveKeys, bins, own);
    D::place(bins, total, earlier, sh);
    uint32_t *key_to = a.key[(pass & 1) ^ 1], *pos_to = a.pos[(pass & 1) ^ 1];
#pragma unroll
    for (int k = 0; k < kMoveKeys; ++k) {
        if (!in[k]) continue;
        const uint32_t to = bins[threadIdx.x >> 6][digit[k]] + own[k];
        key_to[to] = x[k];
        pos_to[to] = p[k];
    }
}

int key_bits(int64_t rows) {
    int bits = 1;
    while (rows >> bits) ++bits;
    return bits;
}

// go(tag of a digit's width, 5 to 11), at least `bits`
template <class F> gnn_status with_bits(int64_t bits, F &&go) {
    if (bits <= 5) return go(std::integral_constant<int, 5>{});
    if (bits == 6) return go(std::integral_constant<int, 6>{});
    if (bits == 7) return go(std::integral_constant<int, 7>{});
    if (bits == 8) return go(std::integral_constant<int, 8>{});
    if (bits == 9) return go(std::integral_constant<int, 9>{});
    if (bits == 10) return go(std::integral_constant<int, 10>{});
    return go(std::integral_constant<int, 11>{});
}

// Sorts; which of key and pos hold the result goes to *where.
gnn_status sort_ids(SortArgs a, int *where, hipStream_t s) {
    const int bits = key_bits(a.rows);
    *where = 0;
    if (a.cap <= kSortTile) {
        // digits of up to 9 bits: the counts of wider ones would not fit beside the positions
        a.passes = static_cast<int>(ceil_div(bits, 9));
        return with_bits(ceil_div(bits, a.passes), [&](auto width) -> gnn_status {
            constexpr int BITS = decltype(width)::value;
            if constexpr (BITS <= 9) embed_sort_kernel<BITS><<<1, kSortThreads, 0, s>>>(a);
            GNN_LAUNCHED("embed_sort");
            return GNN_OK;
        });
    }
    // digits of up to 11 bits, whose counts fill 128 KB of LDS: few launches first
    a.passes = static_cast<int>(ceil_div(bits, 11));
    *where = a.passes & 1;
    return with_bits(std::max<int64_t>(8, ceil_div(bits, a.passes)), [&](auto width) -> gnn_status {
        constexpr int BITS = decltype(width)::value;
        if constexpr (BITS >= 8)
            for (int pass = 0; pass < a.passes; ++pass) {
                embed_count_kernel<BITS><<<static_cast<unsigned>(a.tiles), kSortThreads, 0, s>>>(a, pass);
                GNN_LAUNCHED("embed_count");
                if (a.tiles > kDirectTiles) {
                    embed_scan_kernel<BITS><<<Digits<BITS>::kBins / 32, kSortThreads, 0, s>>>(a);
                    GNN_LAUNCHED("embed_scan");
                }
                embed_move_kernel<BITS><<<static_cast<unsigned>(a.tiles), kSortThreads, 0, s>>>(a, pass);
                GNN_LAUNCHED("embed_move");
            }
        return GNN_OK;
    });
}

// ---------------------------------------------------------------------------
// the gradient: sums of runs
// ---------------------------------------------------------------------------
struct SumArgs {
    const void *g;
    const uint32_t *key, *pos;  // sorted
    int64_t cap, rows, dim;
    float scale;
    int add;
    void *d_table;
    float *first, *last;        // tiles x dim: the sums of a tile's run that began before it, and of the one that goes on behind it
    int64_t tile, tiles;        // positions of a tile; tiles
    int64_t passes;             // column blocks
    int64_t sum_blocks;         // workgroups that sum; the others write zeros
    int64_t zero_rows;          // table rows of one of those
};

template <class T, int VE> __device__ __forceinline__ void put_row(const SumArgs &a, uint32_t row, int64_t c,
                                                                   float (&sum)[VE]) {
    T *to = static_cast<T *>(a.d_table) + static_cast<int64_t>(row) * a.dim + c;
    const int64_t room = a.dim - c;
    float y[VE];
    row::Vec<T, VE> v;
    if (a.add) v.load_upto(to, room);
#pragma unroll
    for (int e = 0; e < VE; ++e) y[e] = a.add ? fmaf(sum[e], a.scale, v.get(e)) : sum[e] * a.scale;
    v.set(y);
    v.store_upto(to, room);
}
template <int VE> __device__ __forceinline__ void put_part(float *to, int64_t room, const float (&sum)[VE]) {
    row::Vec<float, VE> v;
    v.set(sum);
    v.store_upto(to, room);
}

// The first position whose key is at least k, among [lo, hi), by LANES neighbouring
// lanes that ask for the same: each looks at one place, so 262,144 positions take a
// wavefront three loads behind each other and not eighteen.
template <int LANES> __device__ __forceinline__ int64_t lower(const uint32_t *key, int64_t lo, int64_t hi, uint32_t k) {
    const int lane = threadIdx.x & (LANES - 1), shift = (threadIdx.x & 63) & ~(LANES - 1);
    while (lo < hi) {
        const int64_t step = ceil_div(hi - lo, int64_t(LANES)), p = lo + lane * step;
        uint64_t below = __ballot(p < hi && key[p] < k) >> shift;
        if constexpr (LANES < 64) below &= (1ull << LANES) - 1;
        const int n = __popcll(below);  // the first n places are below k
        if (n == 0) return lo;
        hi = min(hi, lo + n * step);
        lo += (n - 1) * step + 1;
    }
    return lo;
}

// Rows [v0, v1) that no id names: zeros.  The positions that name these rows are marked off.
template <class T> __device__ __forceinline__ void zero_rows(const SumArgs &a, int64_t blk) {
    __shared__ uint8_t named[kThreads];
    __shared__ int64_t ends[2];
    const int64_t v0 = blk * a.zero_rows, v1 = min(a.rows, v0 + a.zero_rows);
    named[threadIdx.x] = 0;
    const int wave = threadIdx.x >> 6;
    if (wave < 2) {
        const int64_t p = lower<64>(a.key, 0, a.cap, static_cast<uint32_t>(wave == 0 ? v0 : v1));
        if ((threadIdx.x & 63) == 0) ends[wave] = p;
    }
    __syncthreads();
    constexpr int VE = 16 / sizeof(T);
    row::Vec<T, VE> zero;
#pragma unroll
    for (int i = 0; i < row::Vec<T, VE>::kWords; ++i) zero.w[i] = 0;
    if (ends[0] == ends[1]) {
        // no position names any of them: one stretch (113,538 rows of 1,024 fp32 values and three
        // positions: row by row 101 us, 91 so, in stretches of 24 KB)
        T *to = static_cast<T *>(a.d_table) + v0 * a.dim;
        const int64_t n = (v1 - v0) * a.dim;
#pragma unroll 4
        for (int64_t e = threadIdx.x * VE; e < n; e += kThreads * VE) zero.store_upto(to + e, n - e);
        return;
    }
    for (int64_t p = ends[0] + threadIdx.x; p < ends[1]; p += kThreads) named[a.key[p] - v0] = 1;
    __syncthreads();
    // a row to as many threads as it has vectors, several rows side by side
    const int64_t vectors = ceil_div(a.dim, int64_t(VE));
    const int64_t span = vectors >= kThreads ? kThreads : vectors, side = kThreads / span;
    const int64_t slot = threadIdx.x / span, lane = threadIdx.x - slot * span;
    if (slot >= side) return;
    for (int64_t v = v0 + slot; v < v1; v += side) {
        if (named[v - v0]) continue;
        T *to = static_cast<T *>(a.d_table) + v * a.dim;
        for (int64_t c = lane * VE; c < a.dim; c += span * VE) zero.store_upto(to + c, a.dim - c);
    }
}

// A tile's keys and positions are read at once, one to a lane, and handed around, so that
// what the rows of g wait for is one load and not two behind each other, and kAhead rows are
// in flight (tiles of 32 with four rows in flight and every key read where it is used: 8,192
// x 1,024 in 36 us).
constexpr int kAhead = 8;
template <class TG, class T, int VE, int LANES> __global__ void __launch_bounds__(kThreads) embed_sum_kernel(SumArgs a) {
    if (blockIdx.x >= a.sum_blocks) {
        zero_rows<T>(a, blockIdx.x - a.sum_blocks);
        return;
    }
    constexpr int kSlots = 64 / LANES, kStep = LANES < kAhead ? kAhead : LANES;  // positions read at once
    constexpr int kOwn = kStep / LANES;                                          // of these a lane's
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t t = unit / a.passes * kSlots + slot;
    if (t >= a.tiles) return;
    const int64_t c = ((unit % a.passes) * LANES + lane) * VE, room = a.dim - c;
    const int64_t beg = t * a.tile, end = min(a.cap, beg + a.tile);
    const TG *g = static_cast<const TG *>(a.g);
    const uint32_t none = static_cast<uint32_t>(a.rows);
    const uint32_t before = beg > 0 ? a.key[beg - 1] : none, after = end < a.cap ? a.key[end] : none;
    uint32_t run = a.key[beg];
    if (run >= none) return;
    bool began = before != run;  // the run begins in this tile
    float sum[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) sum[e] = 0.f;
    for (int64_t p0 = beg; p0 < end; p0 += kStep) {
        uint32_t keys[kOwn], places[kOwn];
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            const int64_t p = p0 + o * LANES + lane;
            keys[o] = p < end ? a.key[p] : none;
            places[o] = p < end ? a.pos[p] : 0;
        }
        const int here = static_cast<int>(min(end - p0, int64_t(kStep)));
#pragma unroll 1
        for (int q0 = 0; q0 < here; q0 += kAhead) {
            uint32_t k[kAhead];
            row::Vec<TG, VE> x[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                uint32_t i;
                if constexpr (LANES == 64) {
                    k[q] = __builtin_amdgcn_readlane(keys[0], q0 + q);
                    i = __builtin_amdgcn_readlane(places[0], q0 + q);
                } else if constexpr (kOwn == 1) {
                    k[q] = __shfl(keys[0], q0 + q, LANES);
                    i = __shfl(places[0], q0 + q, LANES);
                } else {
                    k[q] = __shfl(keys[q / LANES], q % LANES, LANES);
                    i = __shfl(places[q / LANES], q % LANES, LANES);
                }
                if (k[q] < none) x[q].load_upto(g + static_cast<int64_t>(i) * a.dim + c, room);
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                if (k[q] != run && run < none && q0 + q < here) {
                    if (began) put_row<T, VE>(a, run, c, sum);
                    else put_part(a.first + t * a.dim + c, room, sum);
                    began = true;
                    run = k[q];
#pragma unroll
                    for (int e = 0; e < VE; ++e) sum[e] = 0.f;
                }
                if (k[q] < none) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) sum[e] += x[q].get(e);
                }
            }
        }
    }
    if (run >= none) return;
    // the tile's last run: over, or one that goes on
    if (!began) put_part(a.first + t * a.dim + c, room, sum);
    else if (after == run) put_part(a.last + t * a.dim + c, room, sum);
    else put_row<T, VE>(a, run, c, sum);
}

// Runs that cross tiles.  Groups of kGroup tiles that one run spans, from before them to
// their end, are summed first, in the place of their first tile's sum: a run of
// n tiles takes its first tile's wavefront n / kGroup + 2 kGroup loads and not n (262,144
// positions, the most frequent id 15,000 times, 2,048 wide: 254 us so, 32 this way).  Few
// tiles are joined without (kFewTiles): the launch would cost what it saves.
constexpr int64_t kGroup = 16, kFewTiles = 2048;
__device__ __forceinline__ bool group_spanned(const SumArgs &a, int64_t u, uint32_t *run) {
    const int64_t beg = u * a.tile, end = beg + kGroup * a.tile;
    if (u == 0 || end > a.cap) return false;
    *run = a.key[beg];
    return *run < static_cast<uint32_t>(a.rows) && a.key[beg - 1] == *run && a.key[end - 1] == *run;
}
template <int VE> __device__ __forceinline__ void add_parts(const SumArgs &a, int64_t c, int64_t from, int64_t to,
                                                            int64_t step, float (&sum)[VE]) {
#pragma unroll 8
    for (int64_t u = from; u < to; u += step) {
        row::Vec<float, VE> x;
        x.load_upto(a.first + u * a.dim + c, a.dim - c);
#pragma unroll
        for (int e = 0; e < VE; ++e) sum[e] += x.get(e);
    }
}
template <int VE, int LANES> __global__ void __launch_bounds__(kThreads) embed_group_kernel(SumArgs a) {
    constexpr int kSlots = 64 / LANES;
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t u = (unit / a.passes * kSlots + slot) * kGroup, c = ((unit % a.passes) * LANES + lane) * VE;
    uint32_t run;
    if (u + kGroup > a.tiles || !group_spanned(a, u, &run)) return;
    float sum[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) sum[e] = 0.f;
    add_parts<VE>(a, c, u, u + kGroup, 1, sum);
    put_part(a.first + u * a.dim + c, a.dim - c, sum);
}

// Of a run that begins in tile t, the sum that t left and those of the tiles (groups) behind it.
template <class T, int VE, int LANES> __global__ void __launch_bounds__(kThreads) embed_join_kernel(SumArgs a) {
    constexpr int kSlots = 64 / LANES;
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t t = unit / a.passes * kSlots + slot;
    if (t + 1 >= a.tiles) return;
    const int64_t c = ((unit % a.passes) * LANES + lane) * VE, room = a.dim - c;
    const int64_t beg = t * a.tile, next = beg + a.tile;
    const uint32_t run = a.key[next], end_key = a.key[next - 1], beg_key = a.key[beg], before = t > 0
        ? a.key[beg - 1] : ~0u;
    if (run >= static_cast<uint32_t>(a.rows) || end_key != run) return;
    if (beg_key == run && before == run) return;  // it began earlier
    const int64_t over = lower<LANES>(a.key, next, a.cap, run + 1);
    const int64_t tiles = ceil_div(over, a.tile), head = a.tiles > kFewTiles ? min(tiles, ceil_div(t + 1,
            kGroup) * kGroup) : tiles;
    const int64_t whole = max(head, over / (a.tile * kGroup) * kGroup);  // groups up to there are spanned
    row::Vec<float, VE> x;
    x.load_upto(a.last + t * a.dim + c, room);
    float sum[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) sum[e] = x.get(e);
    add_parts<VE>(a, c, t + 1, head, 1, sum);
    add_parts<VE>(a, c, head, whole, kGroup, sum);
    add_parts<VE>(a, c, whole, tiles, 1, sum);
    put_row<T, VE>(a, run, c, sum);
}

struct Plan {
    int64_t sort_tiles, tile, tiles;
    size_t key[2], pos[2], counts, totals, first, last, total;
    Plan(int64_t cap, int64_t rows, int64_t dim) {
        sort_tiles = std::max<int64_t>(1, ceil_div(cap, int64_t(kMoveTile)));
        // positions of a tile: enough wavefronts for the chip (of 512 columns), up to 64, where the
        // partial rows are a sixteenth of what is read
        tile = 8;
        while (tile < 64 && cap * ceil_div(dim, int64_t(512)) / (2 * tile) >= 4096) tile *= 2;
        tiles = ceil_div(cap, tile);
        const int bits = key_bits(rows);
        const int64_t bins = int64_t(1) << std::max<int64_t>(8, ceil_div(bits, ceil_div(bits, 11)));
        Carver c(nullptr);
        for (int i = 0; i < 2; ++i) {
            key[i] = c.take(static_cast<size_t>(cap) * 4);
            pos[i] = c.take(static_cast<size_t>(cap) * 4);
        }
        counts = c.take(static_cast<size_t>(bins * sort_tiles) * 4);
        totals = c.take(static_cast<size_t>(bins) * 4);
        first = c.take(static_cast<size_t>(tiles * dim) * 4);
        last = c.take(static_cast<size_t>(tiles * dim) * 4);
        total = round_up(c.off, 256);
    }
};

}  // namespace

gnn_status launch_embed_fwd(const void *table, int tdt, int64_t rows, int64_t dim, int64_t stride, const int64_t *ids,
                            const int64_t *n_dev, int64_t cap, float scale, void *out, int odt, hipStream_t s) {
    if (cap == 0) return GNN_OK;
    LookupArgs a{table, rows, dim, stride, ids, n_dev, cap, scale, out, 0};
    with_types(tdt, odt, [&](auto ti, auto to, auto ve) {
        constexpr int VE = decltype(ve)::value;
        const int64_t vectors = ceil_div(dim, int64_t(VE));
        with_lanes(vectors, [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            a.passes = ceil_div(vectors, int64_t(LANES));
            const int64_t units = ceil_div(cap, int64_t(64 / LANES)) * a.passes;
            auto go = [&](auto at_once) {
                constexpr int UNITS = decltype(at_once)::value;
                const unsigned grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(units,
                        int64_t(UNITS * kWaves)), 1 << 20));
                embed_fwd_kernel<decltype(ti), decltype(to), VE, LANES, UNITS><<<grid, kThreads, 0, s>>>(a);
            };
            if (units <= kFewUnits) go(std::integral_constant<int, 2>{});
            else go(std::integral_constant<int, 4>{});
        });
    });
    GNN_LAUNCHED("embed_fwd");
    return GNN_OK;
}

size_t embed_bwd_ws_bytes(int64_t cap, int64_t rows, int64_t dim) { return Plan(cap, rows, dim).total; }

gnn_status launch_embed_bwd(const void *g, int gdt, const int64_t *ids, const int64_t *n_dev, int64_t cap, int64_t dim,
                            float scale, int64_t rows, bool add, void *d_table, int ddt, void *ws, hipStream_t s) {
    const Plan pl(cap, rows, dim);
    // (without ids there may be no workspace)
    auto at = [&](size_t off) -> void * { return cap > 0 ? static_cast<char *>(ws) + off : nullptr; };
    SortArgs o{};
    o.ids = ids;
    o.n_dev = n_dev;
    o.cap = cap;
    o.rows = rows;
    for (int i = 0; i < 2; ++i) {
        o.key[i] = static_cast<uint32_t *>(at(pl.key[i]));
        o.pos[i] = static_cast<uint32_t *>(at(pl.pos[i]));
    }
    o.counts = static_cast<uint32_t *>(at(pl.counts));
    o.totals = static_cast<uint32_t *>(at(pl.totals));
    o.tiles = pl.sort_tiles;
    SumArgs a{};
    a.g = g;
    a.cap = cap;
    a.rows = rows;
    a.dim = dim;
    a.scale = scale;
    a.add = add;
    a.d_table = d_table;
    a.first = static_cast<float *>(at(pl.first));
    a.last = static_cast<float *>(at(pl.last));
    a.tile = pl.tile;
    a.tiles = pl.tiles;
    // a workgroup of zeros: 24 KB where most stretches have no named row (113,538 x 1,024 in fp32
    // for three ids 91 us, with 64 or 160 KB 103), else 64 (262,144 ids of 131,072 x 2,048 401 us, with 24 KB 409)
    const int64_t stretch = cap < rows / 8 ? 24 << 10 : 64 << 10;
    a.zero_rows = std::max<int64_t>(1, std::min<int64_t>(kThreads,
                                                         stretch / (dim * static_cast<int64_t>(dtype_size(ddt)))));
    const int64_t zero_blocks = add ? 0 : ceil_div(rows, a.zero_rows);
    gnn_status st = GNN_OK;
    with_types(gdt, ddt, [&](auto tg, auto td, auto ve) {
        constexpr int VE = decltype(ve)::value;
        using TG = decltype(tg);
        using T = decltype(td);
        const int64_t vectors = ceil_div(dim, int64_t(VE));
        with_lanes(vectors, [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            a.passes = ceil_div(vectors, int64_t(LANES));
            const int64_t units = ceil_div(a.tiles, int64_t(64 / LANES)) * a.passes;
            a.sum_blocks = ceil_div(units, int64_t(kWaves));
            const int64_t grid = a.sum_blocks + zero_blocks;
            if (grid > kMaxGrid / kThreads) {
                st = fail(GNN_ESIZE, "embed_bwd: sizes exceed the grid limit");
                return;
            }
            if (grid == 0) return;
            if (cap > 0) {
                int where = 0;
                st = sort_ids(o, &where, s);
                if (st != GNN_OK) return;
                a.key = o.key[where];
                a.pos = o.pos[where];
            }
            embed_sum_kernel<TG, T, VE, LANES><<<static_cast<unsigned>(grid), kThreads, 0, s>>>(a);
            st = launch_status("embed_sum");
            if (st != GNN_OK || a.tiles < 2) return;
            if (a.tiles > kFewTiles) {
                const int64_t groups = ceil_div(ceil_div(a.tiles / kGroup, int64_t(64 / LANES)) * a.passes,
                                                int64_t(kWaves));
                embed_group_kernel<VE, LANES><<<static_cast<unsigned>(groups), kThreads, 0, s>>>(a);
                st = launch_status("embed_group");
                if (st != GNN_OK) return;
            }
            embed_join_kernel<T, VE, LANES><<<static_cast<unsigned>(a.sum_blocks), kThreads, 0, s>>>(a);
            st = launch_status("embed_join");
        });
    });
    return st;
}

}  // namespace gnn
