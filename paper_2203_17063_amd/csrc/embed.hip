// Token embedding: scaled rows of a table, and the table's gradient summed
// over tokens sorted by row.
//
// The lookup reads one row per token and writes one: bound by memory.
//
// The gradient G_p[v] = scale * sum of dY[t] over worker p's tokens t of row
// v has to read every token's row of dY and to write every row of G.  The
// rows of dY that belong together lie anywhere, and a few tokens of a
// language make up much of a text, so neither a workgroup per row of G (the
// commonest token's would run alone) nor atomic additions (their order, and
// so the result, would change) will do.  Instead the tokens are sorted by
// (worker, row), stably, and the sorted order is cut into tiles of equal
// length:
//  - a run of equal tokens no longer than a tile is added by the tile that it
//    begins in, to its end, and written at once; a longer one is added in
//    every tile that it touches, and each leaves its sum in the work buffer
//    (at most two a tile);
//  - a second launch adds the pieces of every longer run, in tile order (few:
//    a run of a text's 131,072 tokens is longer than 64 only for its
//    commonest hundred or two);
//  - rows of G without tokens, by flags that the sort has left, are zeroed by
//    further workgroups of the first launch, behind those that add (128,000
//    rows of 4,096: 0.62 ms, 0.68 ms dealt out among them), past the caches
//    where G exceeds the last of them (29,436 rows of 2,378 fp32: 48 us, through
//    them 60 us; 32,003 rows of 2,048, which it holds: 47 us past them, 33 us
//    through them), but not where most of a much larger G is zeros (136,669
//    rows of 2,378: 246 us past them, 225 us through them; equal near 0.6 GB).
// Every element of G is written once, by one thread, in a fixed order.
//
// The sort is by counting, digit by digit from the lowest: up to
// kSmallSort tokens per worker in one launch, a workgroup per worker with
// tokens and positions in LDS; beyond, three launches per digit of up to 9
// bits (counts of each tile, their running sums, the moves).
#include <algorithm>

#include "lm_common.h"

namespace ecc {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int64_t kSmallSort = 16 * kSortThreads;  // tokens of a worker that one workgroup sorts
constexpr int kPosBits = 14;                       // bits of such a token's position
static_assert(kSmallSort == int64_t(1) << kPosBits, "positions of a sort in LDS");
constexpr int kSmallBits = 5;
constexpr int kSmallBins = 1 << kSmallBits;
constexpr int kTileThreads = 1024;                 // the launches of a longer sort
constexpr int kTileItems = 2;
constexpr int kScanThreads = 256;
constexpr int kSortTile = kTileThreads * kTileItems;
constexpr int kBigBits = 9;
constexpr int kBigBins = 1 << kBigBits;

__device__ __forceinline__ int64_t load_id(const void *ids, int id64, int64_t t) {
    return id64 ? reinterpret_cast<const int64_t *>(ids)[t]
                : (int64_t) reinterpret_cast<const int32_t *>(ids)[t];
}

// The row of a token within the table, V for one outside it.
__device__ __forceinline__ uint32_t local_row(int64_t id, int64_t row0, int64_t V) {
    // (the difference of two int64 may pass int64: compared as unsigned)
    const uint64_t r = (uint64_t)id - (uint64_t)row0;
    return id >= row0 && r < (uint64_t)V ? (uint32_t)r : (uint32_t)V;
}

// Lanes of the wave whose digit (rb bits) is this lane's.
__device__ __forceinline__ uint64_t digit_peers(uint32_t d, int rb) {
    uint64_t peers = ~0ull;
    for (int b = 0; b < rb; ++b) {
        const bool bit = (d >> b) & 1u;
        const uint64_t set = __ballot(bit);
        peers &= bit ? set : ~set;
    }
    return peers;
}

// One digit of this lane's element: its place among the wave's elements of
// that digit so far, counted in hist (a row of bins for the wave).
__device__ __forceinline__ uint32_t count_digit(uint32_t d, int rb, uint32_t *hist, int lane) {
    const uint64_t peers = digit_peers(d, rb);
    const int leader = __ffsll((unsigned long long)peers) - 1;
    uint32_t old = 0;
    if (lane == leader) old = atomicAdd(&hist[d], (uint32_t)__popcll(peers));
    old = __shfl(old, leader, 64);
    return old + (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
}

// Exclusive running sums over `bins` (<= NT) values, one per thread; `sums`
// holds NT / 64 + 1 words of LDS.
template <int NT>
__device__ __forceinline__ uint32_t bins_scan(uint32_t v, uint32_t *sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t run = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(run, o, 64);
        if (lane >= o) run += up;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    uint32_t base = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) base += w < wave ? sums[w] : 0u;
    return base + run - v;
}

// A worker's n <= 1024 * ITEMS tokens sorted in LDS, ITEMS consecutive ones per
// thread, by digits of 5 bits: every thread counts its digits in counters
// of its own, whose running sums in the order (digit, thread) are the places
// of its tokens.  The one CU's LDS bounds it: rows and positions travel in one
// word where that holds them (PACK: tables below 2^18 rows).
template <int ITEMS, bool PACK>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(int64_t worker0, int64_t n,
                                                             int64_t V, int64_t row0,
                                                             const void *ids, int id64,
                                                             int passes,
                                                             uint32_t *__restrict__ keys_out,
                                                             int32_t *__restrict__ order_out,
                                                             uint8_t *touched) {
    // the counters, and in turn the tokens on their way to their places
    constexpr int kTokens = kSortThreads * ITEMS;
    // (four words more after every thread's share of the counters, one after
    // that of the tokens, against bank conflicts)
    constexpr int kCountBytes = kSmallBins * kSortThreads * 2 + kSortThreads * 16;
    constexpr int kTokenBytes = kTokens * 6 + kSortThreads * 8;
    __shared__ uint4 s_mem[(kCountBytes > kTokenBytes ? kCountBytes : kTokenBytes) / 16];
    __shared__ uint32_t s_sums[kSortWaves + 1];
    uint16_t *s_count = reinterpret_cast<uint16_t *>(s_mem);
    uint32_t *s_key = reinterpret_cast<uint32_t *>(s_mem);
    uint16_t *s_pos = reinterpret_cast<uint16_t *>(s_key + kTokens + kSortThreads);
    auto key_at = [](uint32_t i) { return i + i / ITEMS; };
    auto pos_at = [](uint32_t i) { return i + i / ITEMS * 2; };
    const int tid = threadIdx.x;
    const int64_t worker = worker0 + blockIdx.x, first = worker * n;
    constexpr int rb = kSmallBits, bins = kSmallBins;
    constexpr uint32_t mask = bins - 1;
    auto count_at = [&](uint32_t digit) {
        const uint32_t i = digit * kSortThreads + tid;
        return s_count + i + 8 * (i >> rb);
    };
    // (cleared before the barriers that lie ahead of the flags set below)
    uint8_t *const flags = touched + worker * V;
    const int64_t whole = min((int64_t)(-(uintptr_t)flags & 15), V);  // before 16-byte accesses
    const int64_t quads16 = (V - whole) / 16, behind = whole + 16 * quads16;
    if (tid < whole) flags[tid] = 0;
    for (int64_t i = tid; i < quads16; i += kSortThreads)
        reinterpret_cast<uint4 *>(flags + whole)[i] = make_uint4(0, 0, 0, 0);
    if (tid < V - behind) flags[behind + tid] = 0;
    constexpr int LOW = PACK ? kPosBits : 0;
    uint32_t key[ITEMS], place[ITEMS];
    uint16_t pos[PACK ? 1 : ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int at = tid * ITEMS + i;
        // past the end: the highest value of the digits sorted, which stays
        // behind the tokens that were ahead of it
        key[i] = at < n ? local_row(load_id(ids, id64, first + at), row0, V) : ~0u;
        if constexpr (PACK) key[i] = key[i] << kPosBits | (uint32_t)at;
        else pos[i] = (uint16_t)at;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = LOW + pass * rb;
        for (int i = tid; i < (bins + 8) * kSortThreads / 8; i += kSortThreads)
            s_mem[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            uint16_t *c = count_at((key[i] >> shift) & mask);
            place[i] = *c;
            *c = (uint16_t)(place[i] + 1);
        }
        __syncthreads();
        // this thread's `bins` consecutive counters to running sums (a total
        // of at most 16,384)
        uint4 *quads = s_mem + tid * (bins / 8 + 1);
        auto pair = [](uint32_t c) { return (c & 0xffffu) + (c >> 16); };
        uint32_t total = 0;
#pragma unroll
        for (int i = 0; i < bins / 8; ++i) {
            const uint4 c = quads[i];
            total += pair(c.x) + pair(c.y) + pair(c.z) + pair(c.w);
        }
        uint32_t run = bins_scan<kSortThreads>(total, s_sums);
        auto sums = [&](uint32_t c) {
            const uint32_t low = c & 0xffffu, both = run | (run + low) << 16;
            run += low + (c >> 16);
            return both;
        };
#pragma unroll
        for (int i = 0; i < bins / 8; ++i) {
            uint4 c = quads[i];
            c.x = sums(c.x);
            c.y = sums(c.y);
            c.z = sums(c.z);
            c.w = sums(c.w);
            quads[i] = c;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            place[i] += *count_at((key[i] >> shift) & mask);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            s_key[key_at(place[i])] = key[i];
            if constexpr (!PACK) s_pos[pos_at(place[i])] = pos[i];
        }
        __syncthreads();
        if (pass + 1 < passes) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                key[i] = s_key[key_at(tid * ITEMS + i)];
                if constexpr (!PACK) pos[i] = s_pos[pos_at(tid * ITEMS + i)];
            }
            __syncthreads();
        }
    }
    const uint32_t key0 = (uint32_t)worker * (uint32_t)(V + 1);
    for (int i = tid; i < n; i += kSortThreads) {
        const uint32_t row = s_key[key_at(i)] >> LOW;
        const int32_t t = (int32_t)(first + (PACK ? s_key[key_at(i)] & ((1u << kPosBits) - 1)
                                                  : s_pos[pos_at(i)]));
        keys_out[first + i] = key0 + row;
        order_out[first + i] = row < (uint32_t)V ? t : ~t;
        if (row < (uint32_t)V) flags[row] = 1;
    }
}

// The elements of one digit pass of a longer sort: (worker, row) and position
// from the tokens (keys == NULL), or as the pass before left them.
struct SortIn {
    const uint32_t *keys;
    const int32_t *order;
    const void *ids;
    int64_t N, n, V, row0;
    int id64;
};
__device__ __forceinline__ uint32_t sort_key(const SortIn &in, int64_t t) {
    if (in.keys) return in.keys[t];
    const uint32_t worker = (uint32_t)(t / in.n);
    return worker * (uint32_t)(in.V + 1) + local_row(load_id(in.ids, in.id64, t), in.row0, in.V);
}

// counts[d][tile]: elements of digit d in each tile.
// The first pass also clears the `rows` flags of rows with tokens.
__global__ __launch_bounds__(kTileThreads) void k_sort_count(SortIn in, int shift, int rb,
                                                             uint32_t *__restrict__ counts,
                                                             uint8_t *touched, int64_t rows) {
    __shared__ uint32_t s_hist[kBigBins];
    if (touched)
        for (int64_t i = (int64_t)blockIdx.x * kTileThreads + threadIdx.x; i < rows;
             i += (int64_t)gridDim.x * kTileThreads)
            touched[i] = 0;
    const uint32_t mask = (1u << rb) - 1u;
    for (int i = threadIdx.x; i < kBigBins; i += kTileThreads) s_hist[i] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kSortTile + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t t = base + i * kTileThreads;
        if (t < in.N) atomicAdd(&s_hist[(sort_key(in, t) >> shift) & mask], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < (1 << rb); d += kTileThreads)
        counts[(int64_t)d * gridDim.x + blockIdx.x] = s_hist[d];
}

// Running sums of digit d's counts over the tiles (workgroup d); totals[d].
__global__ __launch_bounds__(kScanThreads) void k_sort_scan(int64_t tiles,
                                                            uint32_t *__restrict__ counts,
                                                            uint32_t *__restrict__ totals) {
    __shared__ uint32_t s_sums[kScanThreads / 64 + 1];
    __shared__ uint32_t s_total;
    uint32_t *row = counts + (int64_t)blockIdx.x * tiles;
    uint32_t run = 0;
    for (int64_t at = 0; at < tiles; at += kScanThreads) {
        const int64_t i = at + threadIdx.x;
        const uint32_t v = i < tiles ? row[i] : 0u;
        const uint32_t before = bins_scan<kScanThreads>(v, s_sums);
        if (i < tiles) row[i] = run + before;
        if (threadIdx.x == kScanThreads - 1) s_total = before + v;
        __syncthreads();
        run += s_total;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = run;
}

__global__ __launch_bounds__(kTileThreads) void k_sort_move(SortIn in, int shift, int rb,
                                                            const uint32_t *__restrict__ counts,
                                                            const uint32_t *__restrict__ totals,
                                                            uint32_t *__restrict__ keys_out,
                                                            int32_t *__restrict__ order_out,
                                                            uint8_t *touched) {
    constexpr int kWaves = kTileThreads / 64;
    __shared__ uint32_t s_hist[kWaves][kBigBins];
    __shared__ uint32_t s_base[kBigBins];
    __shared__ uint32_t s_sums[kWaves + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t mask = (1u << rb) - 1u;
    const int bins = 1 << rb;
    for (int i = tid; i < kWaves * kBigBins; i += kTileThreads) (&s_hist[0][0])[i] = 0;
    // the first place of each digit: those of the lower digits, then those of
    // this digit in the tiles before
    uint32_t low = 0;
    for (int d0 = 0; d0 < bins; d0 += kTileThreads) {
        const int d = d0 + tid;
        const uint32_t v = d < bins ? totals[d] : 0u;
        const uint32_t before = bins_scan<kTileThreads>(v, s_sums);
        if (d < bins) s_base[d] = low + before + counts[(int64_t)d * gridDim.x + blockIdx.x];
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) low += s_sums[w];
    }
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortTile + wave * 64 * kTileItems + lane;
    uint32_t key[kTileItems], place[kTileItems];
    int32_t pos[kTileItems];
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t t = first + i * 64;
        const bool live = t < in.N;
        key[i] = live ? sort_key(in, t) : ~0u;
        pos[i] = !live ? 0 : in.keys ? in.order[t] : (int32_t)t;
    }
#pragma unroll
    for (int i = 0; i < kTileItems; ++i)
        place[i] = count_digit((key[i] >> shift) & mask, rb, s_hist[wave], lane);
    __syncthreads();
    for (int d = tid; d < bins; d += kTileThreads) {
        uint32_t run = s_base[d];
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = s_hist[w][d];
            s_hist[w][d] = run;
            run += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        // (elements past the end come last in their digit: their places are
        // not used)
        if (first + i * 64 < in.N) {
            const uint32_t to = place[i] + s_hist[wave][(key[i] >> shift) & mask];
            keys_out[to] = key[i];
            bool held = true;
            if (touched) {  // the last pass
                const uint32_t per = (uint32_t)(in.V + 1), worker = key[i] / per,
                               row = key[i] % per;
                held = row < (uint32_t)in.V;
                if (held) touched[(int64_t)worker * in.V + row] = 1;
            }
            order_out[to] = held ? pos[i] : ~pos[i];
        }
    }
}

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
constexpr int kEmbedThreads = 256;

// 131,072 tokens' rows of 4,096 from fp32 to bf16: 339 us for 3.2 GB through
// the L2s (1.6 GB from and to memory: a text's rows repeat, and come from the
// caches); one chunk of a row per wave, four as fast, half a chunk 508 us.
template <typename T, typename O, typename A, int VEC>
__global__ __launch_bounds__(kEmbedThreads) void k_embed_lookup(
    int64_t n, int64_t V, int64_t D, int64_t row0, const void *ids, int id64,
    const T *__restrict__ table, int64_t ld_table, A scale, O *__restrict__ out, int64_t ld_out,
    int log2_lanes, int64_t chunks) {
    const int lanes = 1 << log2_lanes;
    const int64_t unit =
        ((int64_t)blockIdx.x * kEmbedThreads + threadIdx.x) >> log2_lanes;
    const int64_t t = unit / chunks;
    if (t >= n) return;
    const int64_t col = ((unit % chunks) * lanes + (threadIdx.x & (lanes - 1))) * VEC;
    const uint32_t row = local_row(load_id(ids, id64, t), row0, V);
    if (col >= D) return;
    A v[VEC];
    if (row < V) {
        Raw<T, VEC> in;
        in.load_upto(table + (int64_t)row * ld_table + col, D - col);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = in.template get<A>(i) * scale;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (A)0;
    }
    Raw<O, VEC> r;
    r.set_all(v);
    r.template store_upto<true>(out + t * ld_out + col, D - col);
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
template <typename Y, typename G, typename A>
struct EmbedGradArgs {
    int64_t N, V, D;              // tokens of all workers, rows and columns of the table
    int64_t rows;                 // P * V
    const uint32_t *keys;         // [N] worker * (V + 1) + row, sorted
    const int32_t *order;         // [N] the token t, whose row of dy it is; ~t outside the table
    const Y *dy;
    int64_t ld_dy;
    A scale;
    G *grad;
    int64_t ld_grad, stride;      // a row's and a worker's distance
    A *pieces;                    // [tiles][2][D]: sums of a tile's first and last run
    int64_t tiles;
    int32_t tile;                 // tokens of a tile
    int32_t accumulate;
    int32_t log2_lanes;           // lanes that hold a chunk of a row
    int64_t chunks;               // chunks of a row
    const uint8_t *touched;       // [rows] rows with tokens; NULL: none has any
    int64_t sum_blocks;           // workgroups that add; the others zero
    int32_t zero_rows;            // rows a zeroing workgroup looks after
    int32_t stream;               // zeros pass the caches by
    int32_t flat;                 // the rows of all workers follow each other
};

template <typename Y, typename G, typename A, int VEC>
__device__ __forceinline__ void embed_write(const EmbedGradArgs<Y, G, A> &a, uint32_t key,
                                            int64_t col, const A (&sum)[VEC]) {
    const int64_t worker = key / (uint32_t)(a.V + 1), row = key % (uint32_t)(a.V + 1);
    G *g = a.grad + worker * a.stride + row * a.ld_grad + col;
    A v[VEC];
    if (a.accumulate) {
        Raw<G, VEC> old;
        old.load_upto(g, a.D - col);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = old.template get<A>(i) + a.scale * sum[i];
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = a.scale * sum[i];
    }
    Raw<G, VEC> r;
    r.set_all(v);
    r.store_upto(g, a.D - col);
}

// Zeros in the rows that no token names, workgroup `block`'s share of them.
// Where all rows follow each other (a.flat), that is kZeroBytes of memory in
// 16-byte accesses at 16-byte boundaries wherever the rows begin, or element by
// element where some of the rows there have tokens; otherwise zero_rows rows,
// which the threads write side by side.
constexpr int kZeroBytes = 16384;

template <bool STREAM, typename Y, typename G, typename A>
__device__ __forceinline__ void embed_zero(const EmbedGradArgs<Y, G, A> &a, int64_t block) {
    constexpr int W = kVec<G>;
    Raw<G, W> zero;
#pragma unroll
    for (int i = 0; i < Raw<G, W>::kWords; ++i) zero.w[i] = 0;
    if (a.flat) {
        constexpr int U = kZeroBytes / 16 / kEmbedThreads;
        const int64_t e0 = block * (kZeroBytes / (int)sizeof(G));
        const uint32_t count =
            (uint32_t)min((int64_t)(kZeroBytes / (int)sizeof(G)), a.rows * a.D - e0);
        const int64_t row0 = e0 / a.D;
        const uint32_t D = (uint32_t)a.D, in0 = (uint32_t)(e0 - row0 * a.D);
        G *const g = a.grad + e0;
        // the rows of the workgroup's share: none with tokens, or all?
        const uint32_t n = (in0 + count - 1) / D + 1, lane = threadIdx.x & 63;
        bool none = a.touched == nullptr;
        if (!none && n <= 64) {
            const uint64_t with = __ballot(lane < n && a.touched[row0 + (lane < n ? lane : 0)]);
            if ((uint32_t)__popcll(with) == n) return;
            none = with == 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t at = (u * kEmbedThreads + threadIdx.x) * W;  // from e0 on
            if (none && at + W <= count) {
                zero.template store<STREAM>(g + at);
                continue;
            }
            for (uint32_t i = at; i < at + W && i < count; ++i)
                if (none || !a.touched[row0 + (in0 + i) / D]) store_elem<A>(g + i, (A)0);
        }
        return;
    }
    // as many neighbouring threads to a row as it has accesses, or all
    int lg = 0;
    while (lg < 8 && ((int64_t)W << lg) < a.D) ++lg;
    static_assert(kEmbedThreads == 256, "up to all threads to a row");
    const int64_t r1 = min((block + 1) * a.zero_rows, a.rows);
    for (int64_t r = block * a.zero_rows + (threadIdx.x >> lg); r < r1; r += kEmbedThreads >> lg) {
        if (a.touched && a.touched[r]) continue;
        const int64_t worker = a.rows == a.V ? 0 : (int64_t)((uint32_t)r / (uint32_t)a.V);
        G *g = a.grad + worker * a.stride + (r - worker * a.V) * a.ld_grad;
        for (int64_t col = (threadIdx.x & ((1 << lg) - 1)) * W; col < a.D; col += (int64_t)W << lg)
            zero.template store_upto<STREAM>(g + col, a.D - col);
    }
}

// The run of equal keys around a position, counted up to a limit (lanes of a
// group alike): how many positions just below `at` (down to lo), or from `at`
// on (below hi), hold `key`.
__device__ __forceinline__ int run_below(const uint32_t *keys, int64_t at, int64_t lo,
                                         uint32_t key) {
    int64_t l = lo, h = at;
    while (l < h) {
        const int64_t mid = (l + h) >> 1;
        if (keys[mid] < key) l = mid + 1;
        else h = mid;
    }
    return (int)(at - l);
}
__device__ __forceinline__ int run_from(const uint32_t *keys, int64_t at, int64_t hi,
                                        uint32_t key) {
    int64_t l = at, h = hi;
    while (l < h) {
        const int64_t mid = (l + h) >> 1;
        if (keys[mid] > key) h = mid;
        else l = mid + 1;
    }
    return (int)(l - at);
}
__device__ __forceinline__ int leading(uint64_t mask) {  // ones from bit 0 on
    return ~mask ? __ffsll((unsigned long long)~mask) - 1 : 64;
}

// A tile's share of the work: tokens t0 + i for begin <= i < end, of which the
// first run is a piece of a longer one (head), or the last (rest).
struct TileWork {
    int64_t t0;
    int begin, end, count;
    bool head, rest;
};

template <typename Y, typename G, typename A, bool WHOLE_WAVE>
__global__ __launch_bounds__(kEmbedThreads) void k_embed_sum(EmbedGradArgs<Y, G, A> a) {
    constexpr int VEC = kVec<Y>, U = 8;
    if ((int64_t)blockIdx.x >= a.sum_blocks) {
        if (a.stream) embed_zero<true>(a, (int64_t)blockIdx.x - a.sum_blocks);
        else embed_zero<false>(a, (int64_t)blockIdx.x - a.sum_blocks);
        return;
    }
    int64_t unit = ((int64_t)blockIdx.x * kEmbedThreads + threadIdx.x) >> a.log2_lanes;
    if constexpr (WHOLE_WAVE) unit = (int64_t)wave_uniform((uint64_t)unit);
    const int64_t tile = unit / a.chunks;
    if (tile >= a.tiles) return;
    const int lanes = 1 << a.log2_lanes, lane = threadIdx.x & 63;
    const int64_t col = ((unit % a.chunks) * lanes + (threadIdx.x & (lanes - 1))) * VEC;
    const bool live = col < a.D;
    TileWork w;
    w.t0 = tile * a.tile;
    w.count = (int)min((int64_t)a.tile, a.N - w.t0);
    const int64_t t1 = w.t0 + w.count;
    // the tokens of the tile and of the one after it, a lane each (WHOLE_WAVE)
    uint32_t key = 0, key2 = 0;
    int32_t order = 0, order2 = 0;
    uint64_t ends = 0;
    {
        int below, head, tail, beyond;  // of the first run: before, within; of the last: within, after
        if constexpr (WHOLE_WAVE) {
            const bool in = lane < w.count, in2 = lane < a.tile && t1 + lane < a.N;
            const bool in0 = lane < a.tile && w.t0 - 1 - lane >= 0;
            const uint32_t key0 = in0 ? a.keys[w.t0 - 1 - lane] : ~0u;
            key = in ? a.keys[w.t0 + lane] : ~0u;
            key2 = in2 ? a.keys[t1 + lane] : ~0u;
            order = in ? a.order[w.t0 + lane] : -1;
            order2 = in2 ? a.order[t1 + lane] : -1;
            const uint32_t first = __builtin_amdgcn_readlane(key, 0);
            const uint32_t last = __builtin_amdgcn_readlane(key, w.count - 1);
            const uint32_t next = __shfl(key, (lane + 1) & 63, 64);
            below = leading(__ballot(in0 && key0 == first));
            head = leading(__ballot(in && key == first));
            tail = w.count - leading(__ballot(in && key != last));
            beyond = leading(__ballot(in2 && key2 == last));
            ends = __ballot(in && (lane == w.count - 1 || next != key));
        } else {
            const uint32_t first = a.keys[w.t0], last = a.keys[t1 - 1];
            below = run_below(a.keys, w.t0, max(w.t0 - a.tile, (int64_t)0), first);
            head = run_from(a.keys, w.t0, t1, first);
            tail = run_below(a.keys, t1, w.t0, last);
            beyond = run_from(a.keys, t1, min(t1 + a.tile, a.N), last);
        }
        const bool one_run = head == w.count;
        const bool began = below > 0;
        const bool head_long = began && below + head + (one_run ? beyond : 0) > a.tile;
        // a run that began in an earlier tile: its piece, or that tile's alone
        w.head = head_long;
        w.begin = began && !head_long ? head : 0;
        w.rest = beyond > 0 && (one_run && began ? head_long : tail + beyond > a.tile);
        w.end = w.count + (w.rest ? 0 : beyond);
        if (one_run && began && !head_long) return;
    }
    auto order_of = [&](int i) -> int32_t {
        if constexpr (WHOLE_WAVE) {
            const int32_t x = __builtin_amdgcn_readlane(order, i < w.count ? i : 0);
            const int32_t y = __builtin_amdgcn_readlane(order2, i < w.count ? 0 : i - w.count);
            return i < w.count ? x : y;
        } else {
            return a.order[w.t0 + i];
        }
    };
    auto ends_at = [&](int i) -> bool {
        if (i == w.end - 1) return true;
        if constexpr (WHOLE_WAVE) return i < w.count - 1 && (ends >> i & 1);
        else return a.keys[w.t0 + i] != a.keys[w.t0 + i + 1];
    };
    A acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = (A)0;
    bool head = w.head;
    for (int j = w.begin; j < w.end; j += U) {
        int32_t row[U];
        Raw<Y, VEC> y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = j + u < w.end ? order_of(j + u) : -1;
            if (live && row[u] >= 0)
                y[u].template load_upto<true>(a.dy + row[u] * a.ld_dy + col, a.D - col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u < w.end && row[u] >= 0) {
                if (live)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] += y[u].template get<A>(i);
                if (ends_at(j + u)) {
                    if (live) {
                        const bool rest = w.rest && j + u == w.end - 1;
                        if (head || rest) {
                            Raw<A, VEC> r;
                            r.set_all(acc);
                            r.store_upto(a.pieces + (2 * tile + (head ? 0 : 1)) * a.D + col,
                                         a.D - col);
                        } else {
                            embed_write<Y, G, A, VEC>(a, a.keys[w.t0 + j + u], col, acc);
                        }
                    }
                    head = false;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] = (A)0;
                }
            } else if (j + u < w.end && ends_at(j + u)) {
                head = false;  // a run of tokens outside the table
            }
        }
    }
}

// Runs longer than a tile: the piece that the run's first tile left, then
// those of the tiles it goes on in, in order.  The waves of a workgroup look
// for such runs in a tile each; a wave adds a short one's pieces by itself, and
// all take sections of a long one's, whose sums are added in order.
constexpr int kJoinThreads = 512;
constexpr int kJoinTiles = kJoinThreads / 64;

template <typename Y, typename G, typename A>
__global__ __launch_bounds__(kJoinThreads) void k_embed_join(EmbedGradArgs<Y, G, A> a) {
    constexpr int W = kVec<A>, NW = kJoinThreads / 64, U = 8;
    __shared__ A s_part[NW][64 * W];
    __shared__ int64_t s_more[kJoinTiles];  // tiles that the run goes on in, 0: no such run
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = ((int64_t)blockIdx.y * 64 + lane) * W;
    const bool live = col < a.D;
    // pieces lo .. hi - 1 of the run that begins in `tile`: its last run's,
    // then the first runs' of the tiles after it
    auto add_pieces = [&](int64_t tile, int64_t lo, int64_t hi, A(&acc)[W]) {
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] = (A)0;
        for (int64_t s = lo; s < hi; s += U) {
            Raw<A, W> r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t piece = s + u == 0 ? 2 * tile + 1 : 2 * (tile + s + u);
                if (live && s + u < hi) r[u].load_upto(a.pieces + piece * a.D + col, a.D - col);
                else
#pragma unroll
                    for (int i = 0; i < Raw<A, W>::kWords; ++i) r[u].w[i] = 0;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < W; ++i) acc[i] += r[u].template get<A>(i);
        }
    };
    {
        const int64_t tile = (int64_t)blockIdx.x * kJoinTiles + wave;
        const int64_t t0 = tile * a.tile, t1 = t0 + a.tile;
        int64_t more = 0;
        if (tile < a.tiles && t1 < a.N) {
            const uint32_t last = a.keys[t1 - 1];
            const bool in = lane < a.tile;
            const uint32_t key = in ? a.keys[t0 + lane] : ~0u;
            const bool in2 = in && t1 + lane < a.N;
            const uint32_t key2 = in2 ? a.keys[t1 + lane] : ~0u;
            const bool began = t0 > 0 && a.keys[t0 - 1] == last;
            const int tail = a.tile - leading(__ballot(in && key != last));
            const int beyond = leading(__ballot(in2 && key2 == last));
            if (!began && beyond > 0 && tail + beyond > a.tile && a.order[t1] >= 0) {
                for (;;) {
                    const int64_t at = (tile + 1 + more + lane) * a.tile;
                    const int run = leading(__ballot(at < a.N &&
                                                     a.keys[at < a.N ? at : a.N - 1] == last));
                    more += run;
                    if (run < 64) break;
                }
            }
        }
        // a wave alone adds a few pieces, all together a longer run's
        const bool alone = more > 0 && more < U;
        if (lane == 0) s_more[wave] = alone ? 0 : more;
        if (alone) {
            A acc[W];
            add_pieces(tile, 0, more + 1, acc);
            if (live) embed_write<Y, G, A, W>(a, a.keys[t1], col, acc);
        }
    }
    __syncthreads();
    for (int q = 0; q < kJoinTiles; ++q) {
        const int64_t more = s_more[q];
        if (more == 0) continue;
        const int64_t tile = (int64_t)blockIdx.x * kJoinTiles + q;
        A acc[W];
        add_pieces(tile, (more + 1) * wave / NW, (more + 1) * (wave + 1) / NW, acc);
#pragma unroll
        for (int i = 0; i < W; ++i) s_part[wave][lane * W + i] = acc[i];
        __syncthreads();
        if (wave == 0 && live) {
            for (int w = 1; w < NW; ++w)
#pragma unroll
                for (int i = 0; i < W; ++i) acc[i] += s_part[w][lane * W + i];
            embed_write<Y, G, A, W>(a, a.keys[(tile + 1) * a.tile], col, acc);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
constexpr int64_t kCacheBytes = 256 << 20;       // the device's last cache
constexpr int64_t kManyZeros = 640 << 20;        // surely zeros: through the caches again
constexpr int64_t kMaxDim = int64_t(1) << 22;  // columns of a gradient

inline int64_t round16(int64_t bytes) { return (bytes + 15) & ~int64_t(15); }

inline int key_bits(int64_t values) {
    int bits = 1;
    while ((int64_t(1) << bits) < values) ++bits;
    return bits;
}

// Where an index keeps what: the sorted keys, their tokens, a flag for every
// row of every worker that has tokens; then, for a longer sort, a second copy
// of keys and tokens, the counts and the totals.
struct IndexLayout {
    int64_t N = 0, tiles = 0, order = 0, touched = 0, keys2 = 0, order2 = 0, counts = 0,
            totals = 0, bytes = 0;
};
inline bool index_layout(int64_t P, int64_t n, int64_t V, IndexLayout *l) {
    const int64_t lim = (int64_t(1) << 31) - 1;
    if (P < 1 || n < 0 || V < 1 || V >= lim || (n > 0 && P > lim / n) || P * n >= lim ||
        P > lim / (V + 1) || P * (V + 1) >= lim)
        return false;
    l->N = P * n;
    const int64_t part = round16(4 * l->N);
    l->order = part;
    l->touched = 2 * part;
    l->bytes = l->touched + round16(P * V);
    if (n > kSmallSort) {
        l->tiles = (l->N + kSortTile - 1) / kSortTile;
        l->keys2 = l->bytes;
        l->order2 = l->keys2 + part;
        l->counts = l->order2 + part;
        l->totals = l->counts + round16(4 * kBigBins * l->tiles);
        l->bytes = l->totals + 4 * kBigBins;
    }
    l->bytes = std::max<int64_t>(l->bytes, 16);
    return true;
}

// The tiles of a gradient's sum: as many units of work (a tile's chunk of
// columns) as fill the device, but no fewer tokens than keep the pieces'
// traffic low and no more than are summed in one order.
struct GradShape {
    int log2_lanes;
    int64_t chunks;
    int32_t tile;
    int64_t tiles;
};
inline GradShape grad_shape(int64_t N, int64_t D, int vec) {
    GradShape s;
    const int64_t vecs = (D + vec - 1) / vec;
    s.log2_lanes = 0;
    while ((1 << s.log2_lanes) < vecs && s.log2_lanes < 6) ++s.log2_lanes;
    s.chunks = (vecs + (1 << s.log2_lanes) - 1) >> s.log2_lanes;
    s.tile = 8;
    while (s.tile < 64 && (N / (2 * s.tile)) * (s.chunks << s.log2_lanes) >= 64 * 32768) s.tile *= 2;
    s.tiles = (N + s.tile - 1) / s.tile;
    return s;
}

}  // namespace ecc

using namespace ecc;

extern "C" {

ecc_status_t ecc_embed_lookup(int64_t n, int64_t V, int64_t D, int64_t row0, const void *d_ids,
                              int32_t id_type, const void *d_table, int32_t table_type,
                              int64_t ld_table, double scale, void *d_out, int32_t out_type,
                              int64_t ld_out, void *hip_stream) {
    clear_error();
    ECC_ARG(n >= 0 && V >= 1 && D >= 1, "n must be >= 0, V and D >= 1");
    ECC_ARG(id_type == ECC_I32 || id_type == ECC_I64, "id_type must be ECC_I32 or ECC_I64");
    ECC_ARG(known_type(table_type) && known_type(out_type), "unknown element type");
    ECC_ARG(ld_table >= D && ld_out >= D, "a leading dimension is below D");
    if (n == 0) return ECC_OK;
    ECC_ARG(d_ids && d_table && d_out, "NULL pointer");
    const int64_t ib = id_type == ECC_I64 ? 8 : 4, tb = type_size(table_type),
                  ob = type_size(out_type);
    ECC_ARG((uintptr_t)d_ids % ib == 0 && (uintptr_t)d_table % tb == 0 &&
                (uintptr_t)d_out % ob == 0,
            "an array is not aligned to its elements");
    if (V >= (int64_t(1) << 32) - 1 || D >= (int64_t(1) << 40) || n >= (int64_t(1) << 32) ||
        ld_table >= (int64_t(1) << 40) || ld_out >= (int64_t(1) << 40)) {
        set_error("a size is too large");
        return ECC_ERR_RANGE;
    }
    const int vec = (int)(16 / std::min(tb, ob));
    const int64_t vecs = (D + vec - 1) / vec;
    int log2_lanes = 0;
    while ((1 << log2_lanes) < vecs && log2_lanes < 6) ++log2_lanes;
    const int64_t chunks = (vecs + (1 << log2_lanes) - 1) >> log2_lanes;
    const int64_t per_block = kEmbedThreads >> log2_lanes;
    const int64_t most = 0x7fffff * per_block / chunks;  // tokens of one launch
    if (most == 0) {
        set_error("D is too large for one launch");
        return ECC_ERR_RANGE;
    }
    const Span out = span_of(d_out, n, ld_out, D, ob);
    ECC_ARG(!spans_meet(out, span_of(d_table, V, ld_table, D, tb)) &&
                !spans_meet(out, span_of(d_ids, n * ib)),
            "the output overlaps an input");
    for (int64_t t0 = 0; t0 < n; t0 += most) {
        const int64_t m = std::min(most, n - t0);
        const dim3 grid((unsigned)((m * chunks + per_block - 1) / per_block));
        with_type(table_type, [&](auto t) {
            with_type(out_type, [&](auto o) {
                using T = decltype(t);
                using O = decltype(o);
                using A = Wider<T, O>;
                constexpr int VEC = kVec<T> > kVec<O> ? kVec<T> : kVec<O>;
                hipLaunchKernelGGL((k_embed_lookup<T, O, A, VEC>), grid, dim3(kEmbedThreads), 0,
                                   (hipStream_t)hip_stream, m, V, D, row0,
                                   (const char *)d_ids + t0 * ib, id_type == ECC_I64,
                                   (const T *)d_table, ld_table, (A)scale,
                                   (O *)d_out + t0 * ld_out, ld_out, log2_lanes, chunks);
            });
        });
    }
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

int64_t ecc_embed_index_size(int32_t P, int64_t n, int64_t V) {
    IndexLayout l;
    return index_layout(P, n, V, &l) ? l.bytes : -1;
}

ecc_status_t ecc_embed_index(int32_t P, int64_t n, int64_t V, int64_t row0, const void *d_ids,
                             int32_t id_type, void *d_index, void *hip_stream) {
    clear_error();
    ECC_ARG(P >= 1 && n >= 0 && V >= 1, "P and V must be >= 1, n >= 0");
    ECC_ARG(id_type == ECC_I32 || id_type == ECC_I64, "id_type must be ECC_I32 or ECC_I64");
    IndexLayout l;
    if (!index_layout(P, n, V, &l)) {
        set_error("P * n and P * (V + 1) must be below 2^31 - 1");
        return ECC_ERR_RANGE;
    }
    if (n == 0) return ECC_OK;
    ECC_ARG(d_ids && d_index, "NULL pointer");
    ECC_ARG((uintptr_t)d_index % 16 == 0, "d_index must be 16-byte aligned");
    const int64_t ib = id_type == ECC_I64 ? 8 : 4;
    ECC_ARG((uintptr_t)d_ids % ib == 0, "d_ids is not aligned to its elements");
    ECC_ARG(!spans_meet(span_of(d_ids, l.N * ib), span_of(d_index, l.bytes)),
            "d_ids and d_index overlap");
    hipStream_t s = (hipStream_t)hip_stream;
    char *base = (char *)d_index;
    uint32_t *keys = (uint32_t *)base;
    int32_t *order = (int32_t *)(base + l.order);
    uint8_t *touched = (uint8_t *)(base + l.touched);
    const int id64 = id_type == ECC_I64;
    if (n <= kSmallSort) {
        const int passes = (key_bits(V + 1) + kSmallBits - 1) / kSmallBits;
        const bool pack = key_bits(V + 1) + kPosBits <= 32;
        // (a launch has fewer than 2^32 threads)
        constexpr int64_t kMost = (int64_t(1) << 31) / kSortThreads;
        for (int64_t worker0 = 0; worker0 < P; worker0 += kMost) {
            const dim3 grid((unsigned)std::min(kMost, P - worker0)), block(kSortThreads);
            auto sort = [&](auto items) {
                constexpr int ITEMS = decltype(items)::value;
                if (pack)
                    hipLaunchKernelGGL((k_embed_sort<ITEMS, true>), grid, block, 0, s, worker0, n,
                                       V, row0, d_ids, id64, passes, keys, order, touched);
                else
                    hipLaunchKernelGGL((k_embed_sort<ITEMS, false>), grid, block, 0, s, worker0, n,
                                       V, row0, d_ids, id64, passes, keys, order, touched);
            };
            if (n <= kSortThreads) sort(std::integral_constant<int, 1>{});
            else if (n <= 2 * kSortThreads) sort(std::integral_constant<int, 2>{});
            else if (n <= 4 * kSortThreads) sort(std::integral_constant<int, 4>{});
            else if (n <= 8 * kSortThreads) sort(std::integral_constant<int, 8>{});
            else sort(std::integral_constant<int, 16>{});
        }
        ECC_LAUNCH_CHECK();
        return ECC_OK;
    }
    const int bits = key_bits((int64_t)P * (V + 1)), passes = (bits + kBigBits - 1) / kBigBits,
              rb = (bits + passes - 1) / passes;
    uint32_t *keys2 = (uint32_t *)(base + l.keys2);
    int32_t *order2 = (int32_t *)(base + l.order2);
    uint32_t *counts = (uint32_t *)(base + l.counts), *totals = (uint32_t *)(base + l.totals);
    SortIn in{nullptr, nullptr, d_ids, l.N, n, V, row0, id64};
    for (int pass = 0; pass < passes; ++pass) {
        const bool to_first = (passes - 1 - pass) % 2 == 0;  // the last pass: the index itself
        uint32_t *k_out = to_first ? keys : keys2;
        int32_t *o_out = to_first ? order : order2;
        hipLaunchKernelGGL(k_sort_count, dim3((unsigned)l.tiles), dim3(kTileThreads), 0, s, in,
                           pass * rb, rb, counts, pass == 0 ? touched : nullptr, (int64_t)P * V);
        ECC_LAUNCH_CHECK();
        hipLaunchKernelGGL(k_sort_scan, dim3(1u << rb), dim3(kScanThreads), 0, s, l.tiles, counts,
                           totals);
        ECC_LAUNCH_CHECK();
        hipLaunchKernelGGL(k_sort_move, dim3((unsigned)l.tiles), dim3(kTileThreads), 0, s, in,
                           pass * rb, rb, counts, totals, k_out, o_out,
                           pass + 1 == passes ? touched : nullptr);
        ECC_LAUNCH_CHECK();
        in.keys = k_out;
        in.order = o_out;
    }
    return ECC_OK;
}

int64_t ecc_embed_work_size(int32_t P, int64_t n, int64_t D, int32_t dy_type, int32_t grad_type) {
    if (P < 1 || n < 0 || D < 1 || D > kMaxDim || !known_type(dy_type) ||
        !known_type(grad_type) || (n > 0 && P >= (int64_t(1) << 31) / n))
        return -1;
    const GradShape g = grad_shape(P * n, D, (int)(16 / type_size(dy_type)));
    const int64_t acc = dy_type == ECC_F64 || grad_type == ECC_F64 ? 8 : 4;
    return std::max<int64_t>(16, round16(2 * g.tiles * D * acc));
}

ecc_status_t ecc_embed_grad(int32_t P, int64_t n, int64_t V, int64_t D, const void *d_index,
                            const void *d_dy, int32_t dy_type, int64_t ld_dy, double scale,
                            void *d_grad, int32_t grad_type, int64_t ld_grad,
                            int64_t worker_stride, int32_t accumulate, void *d_work,
                            void *hip_stream) {
    clear_error();
    ECC_ARG(P >= 1 && n >= 0 && V >= 1 && D >= 1, "P, V and D must be >= 1, n >= 0");
    ECC_ARG(known_type(dy_type) && known_type(grad_type), "unknown element type");
    ECC_ARG(accumulate == 0 || accumulate == 1, "accumulate must be 0 or 1");
    IndexLayout l;
    if (!index_layout(P, n, V, &l) || D > kMaxDim || ld_dy >= (int64_t(1) << 40) ||
        ld_grad >= (int64_t(1) << 40) || worker_stride >= (int64_t(1) << 50) ||
        worker_stride < 0) {
        set_error("P * n and P * (V + 1) must be below 2^31 - 1, D at most 2^22");
        return ECC_ERR_RANGE;
    }
    ECC_ARG(ld_dy >= D && ld_grad >= D, "a leading dimension is below D");
    const int64_t per_worker = row_extent(V, ld_grad, D);
    ECC_ARG(P == 1 || worker_stride >= per_worker, "workers' gradients overlap");
    ECC_ARG(d_grad, "NULL pointer");
    ECC_ARG(n == 0 || (d_index && d_dy && d_work), "NULL pointer");
    const int64_t yb = type_size(dy_type), gb = type_size(grad_type);
    ECC_ARG((uintptr_t)d_grad % gb == 0 && (n == 0 || (uintptr_t)d_dy % yb == 0),
            "an array is not aligned to its elements");
    if (n > 0) {
        ECC_ARG((uintptr_t)d_work % 16 == 0 && (uintptr_t)d_index % 16 == 0,
                "d_work and d_index must be 16-byte aligned");
        // (workers' gradients that do not follow each other row by row are
        // compared as a whole)
        const Span grad = P == 1 || worker_stride == V * ld_grad
                              ? span_of(d_grad, P * V, ld_grad, D, gb)
                              : span_of(d_grad, row_extent(P, worker_stride, per_worker) * gb);
        const Span dy = span_of(d_dy, l.N, ld_dy, D, yb), index = span_of(d_index, l.bytes),
                   work = span_of(d_work, ecc_embed_work_size(P, n, D, dy_type, grad_type));
        ECC_ARG(!spans_meet(grad, dy) && !spans_meet(grad, index) && !spans_meet(grad, work) &&
                    !spans_meet(work, dy) && !spans_meet(work, index),
                "the gradient, the work buffer and the inputs must not overlap");
    }
    if (n == 0 && accumulate) return ECC_OK;
    const GradShape g = grad_shape(l.N, D, (int)(16 / yb));
    const int64_t per_block = kEmbedThreads >> g.log2_lanes;
    const int64_t sum_blocks = (g.tiles * g.chunks + per_block - 1) / per_block;
    const int64_t rows = (int64_t)P * V;
    const int64_t zero_rows = std::max(kZeroBytes / (D * gb), (rows >> 22) + 1);
    // Zeros as rows or flat, where the rows follow each other.  Rows of 16 KiB up
    // to 24 that begin at 16-byte boundaries are written as rows: a gradient of
    // 64,000 rows of 17 KiB with 64,000 and 16,000 tokens 348 and 231 us, flat
    // 370 and 245; of 128,000 rows of 16 KiB 590 and 596, of 64,000 of 20 KiB 405
    // and 418, but with few tokens 213 and 194.  From 24 KiB on the last share
    // of a row is small, and flat is faster where the gradient exceeds the last
    // cache (64,000 rows of 24 KiB with 64,000, 16,000 and 100 tokens 480, 319
    // and 231 us, as rows 493, 346 and 283; of 28 KiB 562, 376 and 266, as rows
    // 568, 402 and 331), slower by 1 us where it does not (4,000 rows of 28 KiB 40
    // and 39 us).  A gradient of more shares than one launch takes beside the
    // sums is written as rows.
    const int64_t flat_from = rows * D * gb > kCacheBytes ? 3 * kZeroBytes / 2 : 2 * kZeroBytes;
    const bool flat = ld_grad == D && (P == 1 || worker_stride == V * D) &&
                      (uintptr_t)d_grad % 16 == 0 &&
                      (D * gb < kZeroBytes || D * gb >= flat_from || D * gb % 16 != 0) &&
                      rows * D * gb / kZeroBytes < int64_t(1) << 22;
    const int64_t zero_blocks = accumulate ? 0
                                : flat     ? (rows * D * gb + kZeroBytes - 1) / kZeroBytes
                                           : (rows + zero_rows - 1) / zero_rows;
    if (sum_blocks + zero_blocks > 0x7fffff) {
        set_error("P * n * D or P * V is too large for one launch");
        return ECC_ERR_RANGE;
    }
    hipStream_t s = (hipStream_t)hip_stream;
    with_type(dy_type, [&](auto y) {
        with_type(grad_type, [&](auto gr) {
            using Y = decltype(y);
            using G = decltype(gr);
            using A = Wider<Y, G>;
            EmbedGradArgs<Y, G, A> a{};
            a.N = l.N;
            a.V = V;
            a.D = D;
            a.rows = rows;
            a.keys = (const uint32_t *)d_index;
            a.order = (const int32_t *)((const char *)d_index + l.order);
            a.dy = (const Y *)d_dy;
            a.ld_dy = ld_dy;
            a.scale = (A)scale;
            a.grad = (G *)d_grad;
            a.ld_grad = ld_grad;
            a.stride = worker_stride;
            a.pieces = (A *)d_work;
            a.tiles = g.tiles;
            a.tile = g.tile;
            a.accumulate = accumulate;
            a.log2_lanes = g.log2_lanes;
            a.chunks = g.chunks;
            a.sum_blocks = sum_blocks;
            a.touched = n > 0 ? (const uint8_t *)d_index + l.touched : nullptr;
            a.zero_rows = (int32_t)zero_rows;
            a.stream = rows * D * gb > kCacheBytes && (rows - l.N) * D * gb < kManyZeros;
            a.flat = flat;
            const dim3 grid((unsigned)(sum_blocks + zero_blocks));
            if (g.log2_lanes == 6)
                hipLaunchKernelGGL((k_embed_sum<Y, G, A, true>), grid, dim3(kEmbedThreads), 0, s,
                                   a);
            else
                hipLaunchKernelGGL((k_embed_sum<Y, G, A, false>), grid, dim3(kEmbedThreads), 0, s,
                                   a);
            if (g.tiles > 1) {
                constexpr int W = kVec<A>;
                hipLaunchKernelGGL((k_embed_join<Y, G, A>),
                                   dim3((unsigned)((g.tiles + kJoinTiles - 1) / kJoinTiles),
                                        (unsigned)((D + 64 * W - 1) / (64 * W))),
                                   dim3(kJoinThreads), 0, s, a);
            }
        });
    });
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
