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

// LANES lanes to a row, VE elements a lane; a wavefront takes 64 / LANES rows
// side by side, kUnits of them (or of a row's passes) in flight.
constexpr int kUnits = 4;
template <class TI, class TO, int VE, int LANES> __global__ void __launch_bounds__(kThreads) embed_fwd_kernel(LookupArgs a) {
    constexpr int kRows = 64 / LANES;
    const int64_t n = row::live_rows(a.n_dev, a.cap);
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t units = ceil_div(n, int64_t(kRows)) * a.passes;
    const int64_t waves = static_cast<int64_t>(gridDim.x) * kWaves, wave = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const TI *table = static_cast<const TI *>(a.table);
    TO *out = static_cast<TO *>(a.out);
    for (int64_t u0 = wave * kUnits; u0 < units; u0 += waves * kUnits) {
        int64_t r[kUnits], c[kUnits], id[kUnits];
        row::Vec<TI, VE> x[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int64_t u = u0 + k, block = u / a.passes;
            r[k] = block * kRows + slot;
            c[k] = ((u - block * a.passes) * LANES + lane) * VE;
            id[k] = u < units && r[k] < n ? a.ids[r[k]] : -1;
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const bool there = id[k] >= 0 && id[k] < a.rows;
            x[k].load_upto(table + (there ? id[k] : 0) * a.stride + c[k], there ? a.dim - c[k] : 0);
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
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
// key `rows` and come last.  Eight bits a pass, least first: a launch counts each
// tile's digits, the next moves the tile's pairs behind the places of all
// smaller digits, and of the same digit in earlier tiles.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortKeys = 8;
constexpr int kSortTile = kSortThreads * kSortKeys;
constexpr int kBits = 8, kBins = 1 << kBits;

struct SortArgs {
    const int64_t *ids, *n_dev;
    int64_t cap, rows;
    uint32_t *key[2], *pos[2];
    uint32_t *counts;  // kBins x tiles
    int64_t tiles;
    int passes;
};

__device__ __forceinline__ uint32_t key_of(const SortArgs &a, int64_t i, int64_t n) {
    if (i >= n) return static_cast<uint32_t>(a.rows);
    const int64_t id = a.ids[i];
    return static_cast<uint32_t>(id >= 0 && id < a.rows ? id : a.rows);
}
// Element k of this thread's: a wavefront's elements are consecutive, 64 to a round.
__device__ __forceinline__ int64_t sort_at(int64_t tile, int k) {
    return tile * kSortTile + (threadIdx.x >> 6) * (64 * kSortKeys) + k * 64 + (threadIdx.x & 63);
}

__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(SortArgs a, int pass) {
    __shared__ uint32_t bins[kBins];
    const int64_t n = row::live_rows(a.n_dev, a.cap), tile = blockIdx.x;
    if (threadIdx.x < kBins) bins[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortKeys; ++k) {
        const int64_t i = sort_at(tile, k);
        if (i >= a.cap) continue;
        uint32_t x;
        if (pass == 0) {
            x = key_of(a, i, n);
            a.key[0][i] = x;
            a.pos[0][i] = static_cast<uint32_t>(i);
        } else {
            x = a.key[pass & 1][i];
        }
        atomicAdd(&bins[(x >> (kBits * pass)) & (kBins - 1)], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kBins) a.counts[threadIdx.x * a.tiles + tile] = bins[threadIdx.x];
}

// Exclusive sums of one value of each of the first kBins threads.
__device__ __forceinline__ uint32_t scan_bins(uint32_t x, uint32_t *sh) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(sum, o, 64);
        if (lane >= o) sum += y;
    }
    if (threadIdx.x < kBins && lane == 63) sh[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < kBins / 64; ++w)
        if (w < wave) before += sh[w];
    return before + sum - x;
}

// Places of this thread's keys among their tile's equal digits, in the order of their
// elements: a wavefront counts its own rounds in `mine`, and start[wave][digit]
// becomes the place of the wavefront's first one.
struct Ranks {
    uint32_t own[kSortKeys];
};
typedef uint32_t WaveBins[kSortWaves][kBins];
__device__ __forceinline__ void rank_digits(const uint32_t (&digit)[kSortKeys], const bool (&in)[kSortKeys], WaveBins &bins, Ranks &r) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < kSortWaves * kBins; i += kSortThreads) bins[i / kBins][i % kBins] = 0;
    __syncthreads();
    volatile uint32_t *mine = bins[wave];
#pragma unroll
    for (int k = 0; k < kSortKeys; ++k) {
        uint64_t same = __ballot(in[k]);
#pragma unroll
        for (int b = 0; b < kBits; ++b) {
            const uint64_t set = __ballot((digit[k] >> b) & 1);
            same &= (digit[k] >> b) & 1 ? set : ~set;
        }
        const uint64_t below = same & ((1ull << lane) - 1);
        const uint32_t before = in[k] ? mine[digit[k]] : 0;
        r.own[k] = before + __popcll(below);
        __builtin_amdgcn_wave_barrier();
        if (in[k] && below == 0) mine[digit[k]] = before + __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
}

__global__ void __launch_bounds__(kSortThreads) embed_move_kernel(SortArgs a, int pass) {
    __shared__ WaveBins bins;
    __shared__ uint32_t sh[kBins / 64];
    const int64_t tile = blockIdx.x;
    const uint32_t *key = a.key[pass & 1], *pos = a.pos[pass & 1];
    uint32_t x[kSortKeys], p[kSortKeys], digit[kSortKeys];
    bool in[kSortKeys];
#pragma unroll
    for (int k = 0; k < kSortKeys; ++k) {
        const int64_t i = sort_at(tile, k);
        in[k] = i < a.cap;
        x[k] = in[k] ? key[i] : 0;
        p[k] = in[k] ? pos[i] : 0;
        digit[k] = (x[k] >> (kBits * pass)) & (kBins - 1);
    }
    Ranks r;
    rank_digits(digit, in, bins, r);
    // a digit's first place: all smaller digits, and this one in earlier tiles
    uint32_t total = 0, earlier = 0;
    if (threadIdx.x < kBins)
        for (int64_t t = 0; t < a.tiles; ++t) {
            const uint32_t c = a.counts[threadIdx.x * a.tiles + t];
            total += c;
            if (t < tile) earlier += c;
        }
    const uint32_t smaller = scan_bins(total, sh);
    if (threadIdx.x < kBins) {
        uint32_t at = smaller + earlier;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = bins[w][threadIdx.x];
            bins[w][threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
    uint32_t *key_to = a.key[(pass & 1) ^ 1], *pos_to = a.pos[(pass & 1) ^ 1];
#pragma unroll
    for (int k = 0; k < kSortKeys; ++k) {
        if (!in[k]) continue;
        const uint32_t to = bins[threadIdx.x >> 6][digit[k]] + r.own[k];
        key_to[to] = x[k];
        pos_to[to] = p[k];
    }
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

template <class T, int VE> __device__ __forceinline__ void put_row(const SumArgs &a, uint32_t row, int64_t c, float (&sum)[VE]) {
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

// The first position whose key is at least k, among [lo, hi).
__device__ __forceinline__ int64_t lower(const uint32_t *key, int64_t lo, int64_t hi, uint32_t k) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (key[mid] < k) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Rows [v0, v1) that no id names: zeros.  A lane looks for one row, the
// workgroup writes them.
template <class T> __device__ __forceinline__ void zero_rows(const SumArgs &a, int64_t blk) {
    __shared__ uint8_t named[kThreads];
    const int64_t v0 = blk * a.zero_rows, v1 = min(a.rows, v0 + a.zero_rows);
    if (v0 + threadIdx.x < v1) {
        const uint32_t v = static_cast<uint32_t>(v0 + threadIdx.x);
        const int64_t p = lower(a.key, 0, a.cap, v);
        named[threadIdx.x] = p < a.cap && a.key[p] == v;
    }
    __syncthreads();
    constexpr int VE = 16 / sizeof(T);
    row::Vec<T, VE> zero;
#pragma unroll
    for (int i = 0; i < row::Vec<T, VE>::kWords; ++i) zero.w[i] = 0;
    for (int64_t v = v0; v < v1; ++v) {
        if (named[v - v0]) continue;
        T *to = static_cast<T *>(a.d_table) + v * a.dim;
        for (int64_t c = threadIdx.x * VE; c < a.dim; c += kThreads * VE) zero.store_upto(to + c, a.dim - c);
    }
}

constexpr int kAhead = 4;  // rows of g in flight
template <class TG, class T, int VE, int LANES> __global__ void __launch_bounds__(kThreads) embed_sum_kernel(SumArgs a) {
    if (blockIdx.x >= a.sum_blocks) {
        zero_rows<T>(a, blockIdx.x - a.sum_blocks);
        return;
    }
    constexpr int kSlots = 64 / LANES;
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t t = unit / a.passes * kSlots + slot;
    if (t >= a.tiles) return;
    const int64_t c = ((unit % a.passes) * LANES + lane) * VE, room = a.dim - c;
    const int64_t beg = t * a.tile, end = min(a.cap, beg + a.tile);
    const TG *g = static_cast<const TG *>(a.g);
    const uint32_t none = static_cast<uint32_t>(a.rows);
    uint32_t run = a.key[beg];
    if (run >= none) return;
    bool began = beg == 0 || a.key[beg - 1] != run;  // the run begins in this tile
    float sum[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) sum[e] = 0.f;
    for (int64_t p0 = beg; p0 < end; p0 += kAhead) {
        uint32_t k[kAhead];
        row::Vec<TG, VE> x[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            k[q] = p0 + q < end ? a.key[p0 + q] : none;
            if (k[q] < none) x[q].load_upto(g + static_cast<int64_t>(a.pos[p0 + q]) * a.dim + c, room);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            if (k[q] != run) {
                if (run < none && p0 + q < end) {
                    if (began) put_row<T, VE>(a, run, c, sum);
                    else put_part(a.first + t * a.dim + c, room, sum);
                    began = true;
                    run = k[q];
#pragma unroll
                    for (int e = 0; e < VE; ++e) sum[e] = 0.f;
                }
            }
            if (k[q] < none) {
#pragma unroll
                for (int e = 0; e < VE; ++e) sum[e] += x[q].get(e);
            }
        }
    }
    if (run >= none) return;
    // the tile's last run: over, or one that goes on
    if (!began) put_part(a.first + t * a.dim + c, room, sum);
    else if (end < a.cap && a.key[end] == run) put_part(a.last + t * a.dim + c, room, sum);
    else put_row<T, VE>(a, run, c, sum);
}

// The runs that cross tiles: of a run that begins in tile t, the sum that t left and those
// of the tiles behind it, in order.
template <class T, int VE, int LANES> __global__ void __launch_bounds__(kThreads) embed_join_kernel(SumArgs a) {
    constexpr int kSlots = 64 / LANES;
    const int lane = threadIdx.x & (LANES - 1), slot = (threadIdx.x & 63) / LANES;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t t = unit / a.passes * kSlots + slot;
    if (t + 1 >= a.tiles) return;
    const int64_t c = ((unit % a.passes) * LANES + lane) * VE, room = a.dim - c;
    const int64_t beg = t * a.tile, next = beg + a.tile;
    const uint32_t run = a.key[next];
    if (run >= static_cast<uint32_t>(a.rows) || a.key[next - 1] != run) return;
    if (t > 0 && a.key[beg] == run && a.key[beg - 1] == run) return;  // it began earlier
    const int64_t over = lower(a.key, next, a.cap, run + 1);
    row::Vec<float, VE> x;
    x.load_upto(a.last + t * a.dim + c, room);
    float sum[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) sum[e] = x.get(e);
#pragma unroll 4
    for (int64_t u = t + 1; u * a.tile < over; ++u) {
        x.load_upto(a.first + u * a.dim + c, room);
#pragma unroll
        for (int e = 0; e < VE; ++e) sum[e] += x.get(e);
    }
    put_row<T, VE>(a, run, c, sum);
}

int sort_passes(int64_t rows) {
    int bits = 1;
    while (rows >> bits) ++bits;
    return static_cast<int>(ceil_div(bits, kBits));
}

struct Plan {
    int64_t sort_tiles, tile, tiles;
    size_t key[2], pos[2], counts, first, last, total;
    Plan(int64_t cap, int64_t dim) {
        sort_tiles = std::max<int64_t>(1, ceil_div(cap, int64_t(kSortTile)));
        tile = 32;
        tiles = ceil_div(cap, tile);
        Carver c(nullptr);
        for (int i = 0; i < 2; ++i) {
            key[i] = c.take(static_cast<size_t>(cap) * 4);
            pos[i] = c.take(static_cast<size_t>(cap) * 4);
        }
        counts = c.take(static_cast<size_t>(kBins * sort_tiles) * 4);
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
            const unsigned grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(units, int64_t(kUnits * kWaves)), 1 << 20));
            embed_fwd_kernel<decltype(ti), decltype(to), VE, LANES><<<grid, kThreads, 0, s>>>(a);
        });
    });
    GNN_LAUNCHED("embed_fwd");
    return GNN_OK;
}

size_t embed_bwd_ws_bytes(int64_t cap, int64_t, int64_t dim) { return Plan(cap, dim).total; }

gnn_status launch_embed_bwd(const void *g, int gdt, const int64_t *ids, const int64_t *n_dev, int64_t cap, int64_t dim,
                            float scale, int64_t rows, bool add, void *d_table, int ddt, void *ws, hipStream_t s) {
    const Plan pl(cap, dim);
    char *base = static_cast<char *>(ws);
    SortArgs o{};
    o.ids = ids;
    o.n_dev = n_dev;
    o.cap = cap;
    o.rows = rows;
    for (int i = 0; i < 2; ++i) {
        o.key[i] = reinterpret_cast<uint32_t *>(base + pl.key[i]);
        o.pos[i] = reinterpret_cast<uint32_t *>(base + pl.pos[i]);
    }
    o.counts = reinterpret_cast<uint32_t *>(base + pl.counts);
    o.tiles = pl.sort_tiles;
    o.passes = sort_passes(rows);
    if (cap > 0)
        for (int pass = 0; pass < o.passes; ++pass) {
            embed_count_kernel<<<static_cast<unsigned>(o.tiles), kSortThreads, 0, s>>>(o, pass);
            GNN_LAUNCHED("embed_count");
            embed_move_kernel<<<static_cast<unsigned>(o.tiles), kSortThreads, 0, s>>>(o, pass);
            GNN_LAUNCHED("embed_move");
        }
    SumArgs a{};
    a.g = g;
    a.key = o.key[o.passes & 1];
    a.pos = o.pos[o.passes & 1];
    a.cap = cap;
    a.rows = rows;
    a.dim = dim;
    a.scale = scale;
    a.add = add;
    a.d_table = d_table;
    a.first = reinterpret_cast<float *>(base + pl.first);
    a.last = reinterpret_cast<float *>(base + pl.last);
    a.tile = pl.tile;
    a.tiles = pl.tiles;
    // a workgroup of zeros: about 64 KB
    a.zero_rows = std::max<int64_t>(1, std::min<int64_t>(kThreads, (64 << 10) / (dim * static_cast<int64_t>(dtype_size(ddt)))));
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
            embed_sum_kernel<TG, T, VE, LANES><<<static_cast<unsigned>(grid), kThreads, 0, s>>>(a);
            st = launch_status("embed_sum");
            if (st != GNN_OK || a.tiles < 2) return;
            embed_join_kernel<T, VE, LANES><<<static_cast<unsigned>(a.sum_blocks), kThreads, 0, s>>>(a);
            st = launch_status("embed_join");
        });
    });
    return st;
}

}  // namespace gnn
