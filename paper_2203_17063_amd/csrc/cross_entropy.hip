// Cross entropy straight from hidden states, loss and gradients:
//   z = s h E^T,  loss_r = w_r (log sum exp z_r - z_r[y_r]),
//   dz = s w_r (softmax z_r - [j = y_r]),  dh = dz E,  dE_p = dz_p^T h_p.
// The logits exist for one piece of rows at a time.  Rows that count (weight
// not 0, label in the vocabulary) are packed first, so that the others cost
// nothing.  Per piece:
//   1. z as fp32, with every row's maximum and sum of exponentials per 64
//      columns formed from the sums in registers (alone where only the loss is
//      wanted: z is not stored then);
//   2. a wave per row joins them: loss, maximum, 1 / sum (vocabularies of up to
//      32 times 64 join them in the next launch);
//   3. softmax - [label] as bf16 (as the pieces of gemm.h where a gradient is
//      fp32), in both orders;
//   4. dh, scattered to the rows' places, and dE, added up over pieces in fp32.
// What is rounded to bf16 for gradients that are bf16 themselves is softmax -
// [label], one rounding of the terms beside the one of the result: weights and
// the scale are factors of dh's rows afterwards.  For dE they are rounded with
// the term, unless a worker's weights are all alike and one factor does: a
// label's term is near the weight in most rows of a model that learns, and
// would be off by one and the same half step everywhere (0.0037 of dE).
//
// Up to 64 rows in all take kernels of their own, which need no transposed table,
// and a packed one only where tiles form the logits sooner all the same
// (few_by_tiles): the table's two passes are most of such a call.  61 rows, D 96,
// V 1,003, fp32: 20 us against 47 us, in three launches instead of seven (four for
// V above 2,048);
// 8 rows, D 4,096, V 128,000, bf16: 0.93 ms against 1.28 ms; 64 workers' rows, D
// 256, V 32,000, bf16: 0.29 ms against 0.92 ms.
#include "pack.h"

namespace ecc {
namespace {

// Bytes of logits and their gradients at a time, unless 256 rows take more: of V
// 4,194,304 in fp32 those are 16 GiB, and 1,024 rows of D 64 with their gradients
// take 77 ms, by pieces of 64 rows, which would fit, 204 ms.
constexpr int64_t kPieceBytes = int64_t(5) << 30;

struct Rows {
    int32_t *map;      // packed row -> position, -1: none
    int32_t *label;
    float *weight;
    float *factor;     // weight * scale: of dh's row
    float *inside;     // of its terms in dE
    int32_t *live;     // packed rows that hold anything (a multiple of 64)
    int2 *ranges;      // of every worker
    int32_t *counts;   // rows per worker, rounded up
    float *outside;    // of every worker's dE
};

struct Positions {
    const int32_t *labels;
    const float *weight;  // NULL: 1
    int64_t n;
    int32_t V;
    __device__ __forceinline__ bool counts(int64_t i) const {
        const int32_t y = labels[i];
        return y >= 0 && y < V && (!weight || weight[i] != 0.0f);
    }
};

constexpr int kMapThreads = 1024;
constexpr int kMapRows = 8;  // positions of a thread at a time

__device__ __forceinline__ int wave_scan(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(v, d, 64);
        if (lane >= d) v += u;
    }
    return v;
}

// Rows that count per worker, rounded up to 64: a workgroup each.
__global__ __launch_bounds__(kMapThreads) void k_ce_count(Positions q, Rows rows) {
    __shared__ int s_sum[kMapThreads / 64];
    int sum = 0;
    const int64_t base = blockIdx.x * q.n;
    for (int64_t i = threadIdx.x; i < q.n; i += kMapThreads) sum += q.counts(base + i);
    sum = wave_scan(sum);
    if ((threadIdx.x & 63) == 63) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        int all = 0;
        for (int w = 0; w < kMapThreads / 64; ++w) all += s_sum[w];
        rows.counts[blockIdx.x] = (all + 63) & ~63;
    }
}

// A thread's positions from i on: labels and weights, and which count.
struct Taken {
    int32_t y[kMapRows];
    float w[kMapRows];
    uint32_t held;
    __device__ __forceinline__ void load(const Positions &q, int64_t base, int64_t i) {
#pragma unroll
        for (int e = 0; e < kMapRows; ++e) {
            y[e] = i + e < q.n ? q.labels[base + i + e] : -1;
            w[e] = q.weight && i + e < q.n ? q.weight[base + i + e] : 1.0f;
        }
        held = 0;
#pragma unroll
        for (int e = 0; e < kMapRows; ++e)
            if (y[e] >= 0 && y[e] < q.V && w[e] != 0.0f) held |= 1u << e;
    }
};

// Every worker's rows in order, each worker's from a multiple of 64 on: a
// workgroup per worker, which first adds up the counts of those before it, and
// looks whether its weights are all alike.
__global__ __launch_bounds__(kMapThreads) void k_ce_map(Positions q, Rows rows, int32_t P,
                                                        int64_t capacity, float scale,
                                                        float *loss) {
    constexpr int kWaves = kMapThreads / 64;
    __shared__ int s_sum[kWaves];
    __shared__ float s_least[kWaves], s_most[kWaves];
    __shared__ int s_odd;   // a weight that is NaN
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int32_t p = blockIdx.x;
    const int64_t base = p * q.n, step = kMapThreads * kMapRows;
    if (threadIdx.x == 0) s_odd = 0;
    int before = 0;
    for (int32_t i = threadIdx.x; i < p; i += kMapThreads) before += rows.counts[i];
    before = wave_scan(before);
    if (lane == 63) s_sum[wave] = before;
    Taken t;
    float least = __builtin_inff(), most = -__builtin_inff();
    bool odd = false;
    for (int64_t i = threadIdx.x * kMapRows; i < q.n; i += step) {
        t.load(q, base, i);
#pragma unroll
        for (int e = 0; e < kMapRows; ++e)
            if (t.held >> e & 1) {
                least = fminf(least, t.w[e]);
                most = fmaxf(most, t.w[e]);
                odd = odd || t.w[e] != t.w[e];
            }
    }
    for (int d = 32; d; d >>= 1) {
        least = fminf(least, __shfl_xor(least, d, 64));
        most = fmaxf(most, __shfl_xor(most, d, 64));
    }
    if (lane == 0) s_least[wave] = least, s_most[wave] = most;
    __syncthreads();
    if (odd) s_odd = 1;
    before = 0;
    for (int w = 0; w < kWaves; ++w) {
        before += s_sum[w];
        least = fminf(least, s_least[w]);
        most = fmaxf(most, s_most[w]);
    }
    __syncthreads();
    // weights that are all alike become a factor of the whole sum
    const bool alike = least == most && !s_odd;
    int at = before;
    for (int64_t i0 = 0; i0 < q.n; i0 += step) {
        const int64_t i = i0 + threadIdx.x * kMapRows;
        // (of up to one step, the positions are those at hand)
        if (q.n > step) t.load(q, base, i);
        else if (i >= q.n) t.held = 0;
        const int mine = __popc(t.held), upto = wave_scan(mine);
        if (lane == 63) s_sum[wave] = upto;
        __syncthreads();
        int row = at + upto - mine;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) row += s_sum[w];
            at += s_sum[w];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kMapRows; ++e) {
            const int64_t from = base + i + e;
            if (t.held >> e & 1) {
                const float factor = t.w[e] * scale;
                rows.map[row] = (int32_t)from;
                rows.label[row] = t.y[e];
                rows.weight[row] = t.w[e];
                rows.factor[row] = factor;
                rows.inside[row] = alike ? 1.0f : factor;
                ++row;
            } else if (i + e < q.n) {
                loss[from] = 0.0f;
            }
        }
    }
    const int end = (at + 63) & ~63;
    const bool last = p == P - 1;
    if (threadIdx.x == 0) {
        rows.ranges[p] = make_int2(before, end);
        rows.outside[p] = alike ? least * scale : 1.0f;
        if (last) *rows.live = end;
    }
    for (int64_t r = at + threadIdx.x; r < (last ? capacity : end); r += kMapThreads) {
        rows.map[r] = -1;
        rows.label[r] = -1;
        rows.weight[r] = rows.factor[r] = 0.0f;
        rows.inside[r] = 1.0f;
    }
}

// Zeros for the rows of dh that do not count: positions first .. + count - 1,
// a wave's.
struct Unread {
    Positions q;
    int64_t N, D;
    void *dh;        // NULL: none
    int64_t ld;
    int32_t type;
    __device__ __forceinline__ void zero(int64_t first, int count) const {
        for (int64_t i = first; i < min(N, first + count); ++i) {
            if (q.counts(i)) continue;
            for (int64_t d = threadIdx.x & 63; d < D; d += 64) {
                if (type == ECC_F32) ((float *)dh)[i * ld + d] = 0.0f;
                else ((bf16_t *)dh)[i * ld + d].bits = 0;
            }
        }
    }
};
constexpr int kUnread = 16;  // positions of a wave

// Logits and what the softmax needs of them, per row and 64 columns.
struct LogitsOut {
    static constexpr bool kPair = false;
    float *z;          // NULL: not kept
    int64_t ld;
    float scale;
    float2 *stats;     // [row][tiles]: maximum, sum
    int32_t tiles;
    const int32_t *label;
    float *picked;     // the label's logit

    template <int MI, int NI>
    __device__ __forceinline__ void finish(const GemmTile &t, const GemmArgs &g,
                                           f32x4 (&acc)[MI][NI]) const {
        const bool first = (threadIdx.x & 63) < 16;
        const int32_t n0 = t.n - (threadIdx.x >> 4 & 3) * 4;
        const bool whole = n0 + 16 * NI <= g.N;   // no column is behind the last
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int32_t m = t.m + 16 * i;
            const bool row = m < g.M;
            const int32_t y = row ? label[m] : -1;
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] *= scale;
            if (z)
                turn<NI>(t.lds, acc[i], [&](int r, int col, f32x4 v) {
                    const int32_t to = (t.m & ~15) + 16 * i + r;
                    if (to < g.M && (whole || n0 + col < ld))
                        *reinterpret_cast<f32x4 *>(z + to * ld + n0 + col) = v;
                });
            if (y >= n0 && y < n0 + 16 * NI) {
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (t.n + 16 * j + e == y) picked[m] = acc[i][j][e];
            }
            float most = -__builtin_inff(), sum = 0.0f;
            if (whole) {
                sums_of<NI, true>(acc[i], t.n, g.N, most, sum);
            } else {
                sums_of<NI, false>(acc[i], t.n, g.N, most, sum);
            }
            if (first && row && t.tile_n < tiles)
                stats[(int64_t)m * tiles + t.tile_n] = make_float2(most, sum);
        }
    }
    // 64 columns of a row, one per lane.
    __device__ __forceinline__ void row(int32_t m, int32_t tile, int32_t N, int32_t y,
                                        float v) const {
        const int32_t n = tile * 64 + (threadIdx.x & 63);
        const bool in = n < N;
        if (in && n == y) picked[m] = v;
        if (z) z[m * ld + n] = in ? v : 0.0f;
        const float most = wave_all(in ? v : -__builtin_inff(), OpMax());
        const float from = most == -__builtin_inff() ? 0.0f : most;
        const float sum = wave_all(in ? exp_short(v - from) : 0.0f, OpSum());
        if ((threadIdx.x & 63) == 0) stats[(int64_t)m * tiles + tile] = make_float2(most, sum);
    }
    template <int NI, bool WHOLE>
    __device__ static __forceinline__ void sums_of(const f32x4 (&v)[NI], int32_t n, int32_t N,
                                                   float &most, float &sum) {
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (WHOLE || n + 16 * j + e < N) most = fmaxf(most, v[j][e]);
        most = fmaxf(most, __shfl_xor(most, 16, 64));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        const float from = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (WHOLE || n + 16 * j + e < N) sum += exp_short(v[j][e] - from);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
    }
};

// The same from the parts of a product that is split along D: a wave per row
// and 64 columns.
__global__ __launch_bounds__(256) void k_ce_logits(LogitsOut out, const float *parts,
                                                   int32_t splits, int32_t M, int32_t N,
                                                   const int32_t *live, int32_t first) {
    const int64_t wave = blockIdx.x * (int64_t)4 + (threadIdx.x >> 6);
    const int32_t m = (int32_t)(wave / out.tiles), tile = (int32_t)(wave % out.tiles);
    if (m >= M || m + first >= *live) return;
    const int32_t lane = threadIdx.x & 63, n = tile * 64 + lane;
    const int64_t ld4 = (N + 3) & ~3;
    float v = 0.0f;
    if (n < N) {
        const float *p = parts + m * ld4 + n;
        v = *p;
        for (int32_t s = 1; s < splits; ++s) v += p[s * (int64_t)M * ld4];
        v *= out.scale;
    }
    out.row(m, tile, N, out.label[m], v);
}

struct RowTerms {
    float *most, *soft;  // softmax = exp(z - most) soft
};

// A row's maximum and sum from its tiles', by `lanes` neighbouring lanes.
__device__ __forceinline__ void join_tiles(const float2 *s, int32_t tiles, int lane, int lanes,
                                           float &most, float &sum) {
    most = -__builtin_inff();
    for (int32_t i = lane; i < tiles; i += lanes) most = fmaxf(most, s[i].x);
    for (int d = lanes / 2; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
    if (most == -__builtin_inff()) most = 0.0f;
    sum = 0.0f;
    for (int32_t i = lane; i < tiles; i += lanes) {
        const float2 v = s[i];
        // (a tile of NaN has a sum of NaN, and so has the row)
        sum += v.y * (v.x == -__builtin_inff() ? 1.0f : expf(v.x - most));
    }
    for (int d = lanes / 2; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
}

struct RowArgs {
    int32_t first, M, tiles;
    const float2 *stats;
    const float *picked;
    Rows rows;
    float *loss;
    RowTerms out;
    Unread unread;
};

// A wave per packed row: the loss, and the terms of its gradient.  Then waves
// for the positions that do not count.
__global__ __launch_bounds__(256) void k_ce_rows(RowArgs a) {
    const int64_t wave = blockIdx.x * (int64_t)4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (wave >= a.M) {
        a.unread.zero((wave - a.M) * kUnread, kUnread);
        return;
    }
    const int32_t m = (int32_t)wave;
    if (a.first + m >= *a.rows.live) return;
    const int32_t to = a.rows.map[a.first + m];
    if (to < 0) return;
    float most, sum;
    join_tiles(a.stats + (int64_t)m * a.tiles, a.tiles, lane, 64, most, sum);
    if (lane == 0) {
        a.loss[to] = a.rows.weight[a.first + m] * ((most - a.picked[m]) + logf(sum));
        if (a.out.most) {
            a.out.most[m] = most;
            a.out.soft[m] = 1.0f / sum;
        }
    }
}

struct DzArgs {
    const float *z;
    int64_t ld;               // of z and of dz, a multiple of 64
    int32_t V;
    RowArgs r;
    bf16_t *dz, *dzt;
    int64_t plane, plane_t, ld_t;
    int32_t pieces, pieces_t;
    int32_t col_blocks, blocks;
};
constexpr int32_t kFewTiles = 32;

// softmax - [label] in both orders, blocks of 64 x 64.  Bound by memory: 4 bytes
// read and 2 written for each order and piece.  FEW: the blocks join the tiles
// of their rows by themselves, and zero the positions that do not count.  Rows of
// fp32 take exponentials within 2 ulp, so that small probabilities keep their digits.
template <typename T, bool FEW>
__global__ __launch_bounds__(256) void k_ce_dz(DzArgs a) {
    __shared__ PackTile s;
    __shared__ float s_most[kTile], s_soft[kTile];
    const RowArgs &q = a.r;
    if (FEW && (int32_t)blockIdx.x >= a.blocks) {
        q.unread.zero((((int64_t)blockIdx.x - a.blocks) * 4 + (threadIdx.x >> 6)) * kUnread,
                      kUnread);
        return;
    }
    const int32_t row0 = (int32_t)(blockIdx.x / a.col_blocks) * kTile;
    const int32_t col0 = (int32_t)(blockIdx.x % a.col_blocks) * kTile;
    if (row0 + q.first >= *q.rows.live) return;
    const int c8 = (threadIdx.x & 7) * 8, r = threadIdx.x >> 3;
    Raw<float, 8> x[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
        x[p].load(a.z + (int64_t)(row0 + p * 32 + r) * a.ld + col0 + c8);
    if constexpr (FEW) {
        const int i = threadIdx.x >> 2;
        const int32_t to = q.rows.map[q.first + row0 + i];
        float most = 0.0f, sum = 1.0f;
        if (to >= 0) join_tiles(q.stats + (int64_t)(row0 + i) * q.tiles, q.tiles, threadIdx.x & 3, 4,
                                most, sum);
        if ((threadIdx.x & 3) == 0) {
            s_most[i] = most;
            s_soft[i] = 1.0f / sum;
            if (to >= 0 && col0 == 0)
                q.loss[to] = q.rows.weight[q.first + row0 + i] *
                             ((most - q.picked[row0 + i]) + logf(sum));
        }
        __syncthreads();
    }
    float mine[2][8], by[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int32_t m = row0 + p * 32 + r;
        const int32_t y = q.rows.label[q.first + m];
        const float most = FEW ? s_most[p * 32 + r] : q.out.most[m];
        const float soft = FEW ? s_soft[p * 32 + r] : q.out.soft[m];
        by[p] = q.rows.inside[q.first + m];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t j = col0 + c8 + e;
            float v = exp_of<T>(x[p].get<float>(e) - most) * soft;
            if (j == y) v -= 1.0f;
            mine[p][e] = y >= 0 && j < a.V ? v : 0.0f;
        }
    }
    write_block(s, mine, by, row0, col0, a.V, a.dz, a.ld, a.plane, a.pieces, a.dzt, a.ld_t,
                a.plane_t, a.pieces_t);
}

// ---------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------

// Up to kFewRows rows of all workers, which stay where they are (those that do not count have label -1), and
// nothing is packed: the table is read once for the logits and once for dh, by
// kernels that are bound by that and by their latency (1 row, D 3,268, V 49,125,
// bf16: 92 us for 321 MB of logits' operands; gradients 233 us for 642 MB).
struct FewArgs {
    const void *h, *table;
    int64_t ld_h, ld_table;
    Positions q;         // n: of all workers
    int32_t of_worker;
    int64_t D;
    LogitsOut out;
    Rows rows;
    float *loss;
    float scale;
};

// What k_ce_map leaves, by a wave, a row per lane.
__device__ __forceinline__ void few_rows(const FewArgs &a) {
    const int32_t r = threadIdx.x & 63, n = (int32_t)a.q.n, first = r - r % a.of_worker;
    const bool held = r < n && a.q.counts(r);
    const float w = held ? (a.q.weight ? a.q.weight[r] : 1.0f) : 0.0f;
    // (its worker's rows)
    float least = held ? w : __builtin_inff(), most = held ? w : -__builtin_inff();
    bool odd = w != w;
    if (a.of_worker == n) {
        least = -wave_all(-least, OpMax());
        most = wave_all(most, OpMax());
        odd = __any(odd);
    } else {
        const float low = least, high = most;
        const uint64_t all_odd = __ballot(odd);
        for (int32_t i = 0; i < a.of_worker; ++i) {
            least = fminf(least, __shfl(low, first + i, 64));
            most = fmaxf(most, __shfl(high, first + i, 64));
            odd = odd || (all_odd >> (first + i & 63) & 1);
        }
    }
    const bool alike = least == most && !odd;
    const float factor = w * a.scale;
    a.rows.map[r] = held ? r : -1;
    a.rows.label[r] = held ? a.q.labels[r] : -1;
    a.rows.weight[r] = w;
    a.rows.factor[r] = factor;
    a.rows.inside[r] = alike ? 1.0f : factor;
    if (r < n && !held) a.loss[r] = 0.0f;
    if (r < n && r == first) a.rows.outside[r / a.of_worker] = alike ? least * a.scale : 1.0f;
    if (r == 0) *a.rows.live = kTile;
}

__global__ __launch_bounds__(64) void k_ce_few_rows(FewArgs a) { few_rows(a); }

// Logits of 64 columns: four waves for 16 of them each, by two (fp32, which is
// bound by its splitting: four) that share the elements along D in turn and add
// up in LDS; then a wave per row.
template <typename T>
constexpr int kFewThreads = std::is_same_v<T, float> ? 1024 : 512;
template <typename T, int MB>
__global__ __launch_bounds__(kFewThreads<T>) void k_ce_few(FewArgs a) {
    using S = FewStep<T>;
    // (fp32 takes more registers: it is split where it is loaded)
    constexpr int kParts = kFewThreads<T> / 256;
    constexpr int kAhead = S::kPieces == 3 ? 4 / MB : MB == 4 ? 2 : 4;
    __shared__ f32x4 s_acc[kParts][4][MB][64];
    __shared__ __attribute__((aligned(16))) float s_z[16 * MB][68];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    const int32_t n = (int32_t)a.q.n, V = a.q.V, v0 = blockIdx.x * 64;
    if (blockIdx.x == 0 && wave == kFewThreads<T> / 64 - 1) few_rows(a);
    const int cols = wave & 3, part = wave >> 2;
    const T *row = (const T *)a.table + min(v0 + cols * 16 + c, V - 1) * a.ld_table;
    const T *mine[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) mine[i] = (const T *)a.h + min(i * 16 + c, n - 1) * a.ld_h;
    f32x4 acc[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i] = f32x4{0, 0, 0, 0};
    for (int64_t k = part * S::kStep; k < a.D; k += kParts * kAhead * S::kStep) {
        S w[kAhead], x[kAhead][MB];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            const int64_t at = k + s * kParts * S::kStep + q * S::kLane;
            w[s].load(row, at, a.D);
#pragma unroll
            for (int i = 0; i < MB; ++i) x[s][i].load(mine[i], at, a.D);
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            bf16x8 fw[S::kFrags][S::kPieces];
            w[s].frags(fw);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                bf16x8 fx[S::kFrags][S::kPieces];
                x[s][i].frags(fx);
#pragma unroll
                for (int j = 0; j < S::kFrags; ++j)
                    products<S::kPieces, S::kPieces>([&](int px, int pw) {
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[j][pw], fx[j][px],
                                                                         acc[i], 0, 0, 0);
                    });
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) s_acc[part][cols][i][lane] = acc[i];
    __syncthreads();
    for (int t = wave; t < 4 * MB; t += kFewThreads<T> / 64) {
        const int i = t >> 2;
        f32x4 z = s_acc[0][t & 3][i][lane];
#pragma unroll
        for (int p = 1; p < kParts; ++p) z += s_acc[p][t & 3][i][lane];
        *reinterpret_cast<f32x4 *>(&s_z[i * 16 + c][(t & 3) * 16 + q * 4]) = z * a.scale;
    }
    __syncthreads();
    for (int32_t r = wave; r < n; r += kFewThreads<T> / 64)
        a.out.row(r, blockIdx.x, V, a.q.labels[r], s_z[r][lane]);
}

// (four of the table's gradient)
template <typename T>
__device__ __forceinline__ void add_quad(T *to, f32x4 v, int64_t left, bool add) {
    Raw<T, 4> x;
    if (add) {
        x.load_upto(to, left);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += x.template get<float>(e);
    }
    const float y[4] = {v[0], v[1], v[2], v[3]};
    x.set_all(y);
    x.store_upto(to, left);
}

// Workgroups of the gradients, about: what the CUs' LDS holds at a time.
constexpr int few_blocks(int np, int pt) { return np == 3 ? 256 : pt == 3 ? 512 : 1024; }
struct FewGrad {
    const void *h, *table;
    int64_t ld_h, ld_table;
    int32_t n, of_worker, V;   // rows of all workers, of one
    int64_t D;
    const float *z;
    int64_t ld_z;
    RowArgs r;
    float *dh;            // [splits][64][ld_dh], NULL: none
    int64_t ld_dh;
    void *dtable;         // NULL: none
    int64_t ld_dtable, worker_stride;
    int32_t type, add;
    int32_t blocks_d, per;   // blocks along D; tiles of 64 columns of a split
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kFewPitch = 72;   // of a row of 64 in LDS: 16-byte accesses

// Where a block's element lies in LDS, turned round: the four threads that write
// a row's elements reach different banks (39 rows, D 3,473, V 43,897, fp32: the
// call takes 1.00 ms, and 1.19 ms where they meet in one).
__device__ __forceinline__ int turned(int col, int row) {
    return col * kFewPitch + (row ^ (col & 48));
}
// A piece of N neighbouring columns of a row.
template <int N>
__device__ __forceinline__ void put_columns(uint16_t *s, int col, int row, const float (&v)[N],
                                            int which, bool split) {
    Raw<bf16_t, N> x;
    set_piece(x, v, which, split);
    uint16_t *to = s + turned(col, row);
#pragma unroll
    for (int e = 0; e < N; ++e) to[e * kFewPitch] = (uint16_t)(x.w[e / 2] >> (e & 1) * 16);
}

// Gradients, 64 elements along D for a split of the vocabulary's tiles: the
// tile's softmax - [label] (FEW: of rows whose tiles are joined here) and the
// table's elements lie in LDS in the orders that the two products want, dh's
// sums stay in registers.  The next tile is under way meanwhile.  dE is formed
// once for each worker (WORKERS: several), of all rows with the others' masked.
// fp32's pieces fill a CU's LDS with one workgroup, which then has 16 waves (8:
// 1.01 ms for the case above; bf16 with pieces of dE, 4 waves: 182 us, 8: 217 us
// for 32 rows, D 2,048, V 32,000).
template <typename T>
constexpr int kFewWaves = std::is_same_v<T, float> ? 16 : 4;
template <typename T, int PT, bool FEW, bool WORKERS>
__global__ __launch_bounds__((64 * kFewWaves<T>), 4) void k_ce_few_grad(FewGrad a) {
    constexpr int W = kFewWaves<T>, CN = kTile / W, N = CN < 8 ? CN : 8, J = 16 / W;
    constexpr int NP = std::is_same_v<T, float> ? 3 : 1, kSize = kTile * kFewPitch;
    __shared__ __attribute__((aligned(16))) uint16_t s_dz[NP][kSize], s_dzt[PT][kSize],
        s_h[NP][kSize], s_e[NP][kSize];
    const RowArgs &q = a.r;
    // a thread's columns of a row of a tile; a wave's rows and columns of sums
    const int r = threadIdx.x / W, c0 = threadIdx.x % W * CN;
    const int lane = threadIdx.x & 63, c = lane & 15, k8 = lane >> 4;
    const int wave = threadIdx.x >> 6 & 3, j0 = (threadIdx.x >> 8) * J;
    // (an XCD's blocks are neighbours: rows' ends share lines of its L2)
    const int32_t b = xcd_block(blockIdx.x, gridDim.x);
    const int64_t d0 = (int64_t)(b % a.blocks_d) * kTile, left = a.D - d0 - c0;
    const int32_t split = b / a.blocks_d;
    const int32_t t0 = split * a.per, t1 = min(q.tiles, t0 + a.per);
    const int32_t y = q.rows.label[r];
    const bool held = y >= 0;
    const float inside = q.rows.inside[r];
    float most = 0.0f, soft = 0.0f;
    if constexpr (FEW) {
        float sum = 1.0f;
        if (held) join_tiles(q.stats + (int64_t)r * q.tiles, q.tiles, threadIdx.x % W, W, most, sum);
        soft = 1.0f / sum;
        if (held && b == 0 && c0 == 0)
            q.loss[r] = q.rows.weight[r] * ((most - q.picked[r]) + logf(sum));
    } else if (held) {
        most = q.out.most[r];
        soft = q.out.soft[r];
    }
    const uint64_t live = __ballot(q.rows.label[lane] >= 0);
    const int32_t workers = WORKERS ? a.n / a.of_worker : 1;
    const float outside = q.rows.outside[WORKERS ? min(lane, workers - 1) : 0];
    if (a.dtable) {
        Raw<T, N> x[CN / N];
#pragma unroll
        for (int i = 0; i < CN / N; ++i) {
            x[i].load_upto((const T *)a.h + (held ? r * a.ld_h + d0 + c0 + i * N : 0),
                           held ? left - i * N : 0);
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = x[i].template get<float>(e);
            for (int p = 0; p < NP; ++p)
                put_columns(s_h[p], c0 + i * N, r, v, p, NP > 1);
        }
    }
    Raw<float, N> z[CN / N];
    Raw<T, N> w[CN / N];
    auto fetch = [&](int32_t t) {
        const int64_t v = (int64_t)t * kTile + r;
#pragma unroll
        for (int i = 0; i < CN / N; ++i) {
            z[i].load_upto(a.z + (held ? r * a.ld_z + t * kTile + c0 + i * N : 0), held ? N : 0);
            const bool in = a.dh && v < a.V;
            w[i].load_upto((const T *)a.table + (in ? v * a.ld_table + d0 + c0 + i * N : 0),
                           in ? left - i * N : 0);
        }
    };
    auto frag = [&](const uint16_t *s, int row, int kk) {
        return *reinterpret_cast<const bf16x8 *>(s + row * kFewPitch + kk * 32 + k8 * 8);
    };
    auto frag_t = [&](const uint16_t *s, int col, int kk) {
        return *reinterpret_cast<const bf16x8 *>(s + turned(col, kk * 32 + k8 * 8));
    };
    f32x4 dh[J];
#pragma unroll
    for (int j = 0; j < J; ++j) dh[j] = f32x4{0, 0, 0, 0};
    fetch(t0);
    for (int32_t t = t0; t < t1; ++t) {
#pragma unroll
        for (int i = 0; i < CN / N; ++i) {
            float v[N], u[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int32_t j = t * kTile + c0 + i * N + e;
                float p = exp_of<T>(z[i].template get<float>(e) - most) * soft;
                if (j == y) p -= 1.0f;
                v[e] = held && j < a.V ? p : 0.0f;
                u[e] = v[e] * inside;
            }
            const int at = c0 + i * N;
            for (int p = 0; p < NP; ++p) {
                Raw<bf16_t, N> x;
                set_piece(x, v, p, NP > 1);
                *reinterpret_cast<Raw<bf16_t, N> *>(s_dz[p] + r * kFewPitch + at) = x;
            }
            if (a.dtable)
                for (int p = 0; p < PT; ++p)
                    put_columns(s_dzt[p], at, r, u, p, PT > 1);
            if (a.dh) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = w[i].template get<float>(e);
                for (int p = 0; p < NP; ++p)
                    put_columns(s_e[p], at, r, v, p, NP > 1);
            }
        }
        if (t + 1 < t1) fetch(t + 1);
        __syncthreads();
        if (a.dh && wave * 16 < a.n) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int j = 0; j < J; ++j)
                    products<NP, NP>([&](int pz, int pw) {
                        dh[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            frag_t(s_e[pw], (j0 + j) * 16 + c, kk), frag(s_dz[pz], wave * 16 + c, kk),
                            dh[j], 0, 0, 0);
                    });
        }
        for (int32_t p = 0; a.dtable && p < workers; ++p) {
            const int32_t lo = WORKERS ? p * a.of_worker : 0, hi = lo + a.of_worker;
            if (a.add && !(live >> lo & (~uint64_t(0) >> (64 - a.of_worker)))) continue;
            f32x4 de[J];
#pragma unroll
            for (int j = 0; j < J; ++j) de[j] = f32x4{0, 0, 0, 0};
            for (int kk = lo / 32; kk * 32 < hi; ++kk) {
                // one worker's rows, of both operands: another's may be NaN
                u32x4 keep;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int32_t row = kk * 32 + k8 * 8 + 2 * e;
                    keep[e] = (row >= lo && row < hi ? 0xffffu : 0u) |
                              (row + 1 >= lo && row + 1 < hi ? 0xffff0000u : 0u);
                }
                auto kept = [&](bf16x8 v) {
                    if (!WORKERS) return v;
                    return __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, v) & keep);
                };
                bf16x8 dz[PT];
#pragma unroll
                for (int i = 0; i < PT; ++i) dz[i] = kept(frag_t(s_dzt[i], wave * 16 + c, kk));
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    bf16x8 h[NP];
#pragma unroll
                    for (int i = 0; i < NP; ++i)
                        h[i] = kept(frag_t(s_h[i], (j0 + j) * 16 + c, kk));
                    products<PT, NP>([&](int pz, int ph) {
                        de[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[ph], dz[pz], de[j], 0, 0,
                                                                       0);
                    });
                }
            }
            const float by = WORKERS ? __shfl(outside, p, 64) : outside;
            const int32_t v = t * kTile + wave * 16 + c;
            const int64_t at = p * a.worker_stride + v * a.ld_dtable;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int64_t d = d0 + (j0 + j) * 16 + k8 * 4;
                if (v >= a.V || d >= a.D) continue;
                if (a.type == ECC_F32)
                    add_quad((float *)a.dtable + at + d, de[j] * by, a.D - d, a.add);
                else
                    add_quad((bf16_t *)a.dtable + at + d, de[j] * by, a.D - d, a.add);
            }
        }
        __syncthreads();
    }
    if (!a.dh) return;
#pragma unroll
    for (int j = 0; j < J; ++j)
        *reinterpret_cast<f32x4 *>(a.dh + ((int64_t)split * kTile + wave * 16 + c) * a.ld_dh + d0 +
                                   (j0 + j) * 16 + k8 * 4) = dh[j];
}

// dh from its splits: 16 threads per four elements, each of every sixteenth
// split, and then of their sums in order; zeros for the rows that do not count.
template <typename T>
__global__ __launch_bounds__(256) void k_ce_few_join(const float *parts, int64_t ld, int32_t splits,
                                                     Rows rows, int64_t D, T *dh, int64_t ld_dh) {
    __shared__ f32x4 s_sum[16][16];
    const int64_t r = blockIdx.y, d = (blockIdx.x * (int64_t)16 + (threadIdx.x & 15)) * 4;
    const int part = threadIdx.x >> 4;
    f32x4 sum = {0, 0, 0, 0};
    if (rows.map[r] >= 0 && d < D)
        for (int32_t s = part; s < splits; s += 16)
            sum += *reinterpret_cast<const f32x4 *>(parts + ((int64_t)s * kTile + r) * ld + d);
    s_sum[part][threadIdx.x & 15] = sum;
    __syncthreads();
    if (part || d >= D) return;
    for (int p = 1; p < min(16, splits); ++p) sum += s_sum[p][threadIdx.x];
    sum *= rows.factor[r];
    const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    Raw<T, 4> x;
    x.set_all(v);
    x.store_upto(dh + r * ld_dh + d, D - d);
}

// ---------------------------------------------------------------------------
// sizes and work memory
// ---------------------------------------------------------------------------

struct Plan {
    int64_t N, n_pad, rows, R, pieces_of_rows;
    int64_t Dp, Vp;
    int32_t tiles;
    int np;                      // pieces of the operands
    int pz, pzt;                 // of dz for dh, for dE
    bool pack_table;
    bool few;                    // up to kFewRows rows in all
    bool tiles_z, pack_h;        // few rows: logits by tiles, of packed rows
    int32_t blocks_d, splits, per;
    GemmShape shape_z, shape_h, shape_e;
    // offsets into the work buffer
    int64_t map, label, weight, factor, inside, live, ranges, counts, outside, table, table_t, h, h_t,
        z, dz, dzt, stats, picked, terms, sums, parts[2], parts_z, bytes;
};

// Do few rows' logits take gemm.h's tiles?  By the times that both take, in us:
// k_ce_few takes so much per round of 256 workgroups and element of D for its
// one, two or four blocks of 16 rows, which it reads again for every 64 columns
// (twice as much for rows of bf16 that do not begin at 4 bytes); tiles read the
// table at 5 bytes a ns, once they are under way, but pack it first if its rows
// are fp32 or no multiple of 64.  The loss alone, bf16: 64 rows, D 4,096, V
// 128,000: 590 us and 223 us; 1 row, D 1,024, V 1,000: 13 us and 20 us; 32 rows, D
// 2,001, V 5,003: 65 us and 30 us; 64 rows, D 3,268, V 49,125: 194 us and 237 us.
// fp32, 64 rows: D 4,096, V 1,000: 155 us and 40 us; D 2,048, V 32,000: 171 us and
// 283 us.
bool few_by_tiles(const ecc_cross_entropy_t *a) {
    const bool f32 = a->type == ECC_F32;
    static constexpr double kTimes[2][3] = {{0.0075, 0.0115, 0.0165}, {0.013, 0.022, 0.036}};
    const int64_t N = a->P * a->n;
    const double each = kTimes[f32][N <= 16 ? 0 : N <= 32 ? 1 : 2];
    const double odd = f32 || a->D % 2 == 0 ? 1.0 : 2.0;
    const double few = 8.0 + (double)((a->V + 64 * 256 - 1) / (64 * 256)) * a->D * each * odd;
    const double table = (double)a->V * a->D * 1e-6;
    const double tiles = f32 || a->D % 64 ? 24.0 + table * (f32 ? 3.6 : 1.4) : 19.0 + table * 0.4;
    return tiles < few;
}

Plan make_plan(const ecc_cross_entropy_t *a, bool gradient) {
    Plan p{};
    p.N = a->P * a->n;
    p.n_pad = pad64(a->n);
    p.few = p.N <= kFewRows;
    p.rows = p.few ? kFewRows : a->P * p.n_pad;
    p.Dp = pad64(a->D);
    p.Vp = pad64(a->V);
    p.tiles = (int32_t)(p.Vp / 64);
    const bool f32 = a->type == ECC_F32;
    p.np = f32 ? 3 : 1;
    p.pz = f32 ? 3 : 1;
    p.pzt = a->grad_type == ECC_F32 ? 3 : 1;
    p.pack_table = !as_it_lies(a->d_table, a->ld_table, a->D, a->type);
    const int64_t row = p.np * 2 * p.Dp * (gradient ? 2 : 1) + p.tiles * 8 + 16 +
                        (gradient ? 4 * p.Vp + 2 * p.pz * p.Vp + 2 * p.pzt * p.Vp : 0);
    p.R = std::max<int64_t>(256, kPieceBytes / row & ~int64_t(255));
    p.R = std::max<int64_t>(64, std::min(p.R, p.rows));
    p.pieces_of_rows = (p.rows + p.R - 1) / p.R;
    // (pieces of equal length)
    if (p.pieces_of_rows > 1)
        p.R = (p.rows / p.pieces_of_rows + 255 + (p.rows % p.pieces_of_rows > 0)) & ~int64_t(255);
    p.pieces_of_rows = (p.rows + p.R - 1) / p.R;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) & ~int64_t(255);
        return here;
    };
    p.map = take(4 * p.rows);
    p.label = take(4 * p.rows);
    p.weight = take(4 * p.rows);
    p.factor = take(4 * p.rows);
    p.inside = take(4 * p.rows);
    p.live = take(4);
    p.ranges = take(8 * (int64_t)a->P);
    p.counts = take(4 * (int64_t)a->P);
    p.outside = take(4 * (int64_t)a->P);
    if (p.few) {
        p.tiles_z = few_by_tiles(a);
        if (p.tiles_z) {
            p.pack_h = !as_it_lies(a->d_h, a->ld_h, a->D, a->type);
            p.h = take(p.pack_h ? p.np * 2 * p.R * p.Dp : 0);
            p.table = take(p.pack_table ? p.np * 2 * p.Vp * p.Dp : 0);
            p.shape_z = gemm_shape(p.N, a->V, p.Dp / kGemmK * (p.np == 3 ? 6 : 1), 1, true);
            p.parts_z = take(split_bytes(p.N, a->V, p.shape_z.splits, 1));
        }
        p.stats = take(8 * p.R * p.tiles);
        p.picked = take(4 * p.R);
        if (gradient) {
            p.z = take(4 * p.R * p.Vp);
            p.terms = take(8 * p.R);
            p.blocks_d = (int32_t)(p.Dp / kTile);
            p.splits = std::min(p.tiles, std::max(1, few_blocks(p.np, p.pzt) / p.blocks_d));
            p.per = (p.tiles + p.splits - 1) / p.splits;
            p.splits = (p.tiles + p.per - 1) / p.per;
            p.parts[0] = take(4 * p.splits * p.R * p.Dp);
        }
        p.bytes = at;
        return p;
    }
    p.table = take(p.pack_table ? p.np * 2 * p.Vp * p.Dp : 0);
    p.h = take(p.np * 2 * p.R * p.Dp);
    p.stats = take(8 * p.R * p.tiles);
    p.picked = take(4 * p.R);
    p.shape_z = gemm_shape(p.R, a->V, p.Dp / kGemmK * (p.np == 3 ? 6 : 1), 1, true);
    p.parts_z = take(split_bytes(p.R, a->V, p.shape_z.splits, 1));
    if (gradient) {
        p.table_t = take(p.np * 2 * a->D * p.Vp);
        p.h_t = take(p.np * 2 * a->D * p.R);
        p.z = take(4 * p.R * p.Vp);
        p.dz = take(2 * p.pz * p.R * p.Vp);
        p.dzt = take(2 * p.pzt * a->V * p.R);
        p.terms = take(8 * p.R);
        p.sums = take(p.pieces_of_rows > 1 && a->grad_type != ECC_F32 ? 4 * a->P * a->V * a->D : 0);
        p.shape_h = gemm_shape(p.R, a->D, p.Vp / kGemmK * (p.np == 3 ? 6 : 1), 1, true);
        // (a worker's rows in a piece)
        p.shape_e = gemm_shape(a->V, a->D,
                               std::min(p.n_pad, p.R) / kGemmK * (p.np == 3 ? 6 : p.pzt), a->P,
                               true);
        p.parts[0] = take(split_bytes(p.R, a->D, p.shape_h.splits, 1));
        p.parts[1] = take(split_bytes(a->V, a->D, p.shape_e.splits, a->P));
    }
    p.bytes = std::max<int64_t>(at, 16);
    return p;
}

ecc_status_t check(const ecc_cross_entropy_t *a) {
    ECC_ARG(a, "NULL description");
    ECC_ARG(a->n >= 0 && a->V >= 1 && a->D >= 1 && a->P >= 1, "a size is out of range");
    ECC_ARG(a->type == ECC_F32 || a->type == ECC_BF16, "the operands must be fp32 or bf16");
    ECC_ARG(a->grad_type == ECC_F32 || a->grad_type == a->type,
            "the table's gradient must be fp32 or of the operands' type");
    ECC_ARG(a->scale == a->scale && __builtin_fabs(a->scale) <= 3e38, "the scale must be finite");
    ECC_ARG(a->ld_h >= a->D && a->ld_table >= a->D, "a leading dimension is below D");
    // (rows: grids of fewer than 2^32 threads, k_ce_rows' being the largest)
    if (a->V > ECC_CROSS_ENTROPY_MAX_VOCAB || a->D > ECC_CROSS_ENTROPY_MAX_DIM ||
        a->n > ECC_CROSS_ENTROPY_MAX_ROWS ||
        (__int128)a->P * pad64(a->n) > ECC_CROSS_ENTROPY_MAX_ROWS ||
        a->ld_h >= (int64_t(1) << 40) || a->ld_table >= (int64_t(1) << 40) ||
        !gemm_in_range(a->V, a->D, a->P)) {
        set_error("the sizes are beyond what the library supports");
        return ECC_ERR_RANGE;
    }
    const int64_t size = type_size(a->type);
    if (a->n == 0) return ECC_OK;
    ECC_ARG(a->d_h && a->d_table && a->d_labels, "NULL pointer");
    ECC_ARG((uintptr_t)a->d_h % size == 0 && (uintptr_t)a->d_table % size == 0 &&
                (uintptr_t)a->d_labels % 4 == 0 && (uintptr_t)a->d_weight % 4 == 0,
            "an array is not aligned");
    return ECC_OK;
}

// The logits' product, in one go or in parts along D.
void launch_logits(GemmArgs g, const Plan &p, char *w, const LogitsOut &out, const int32_t *live,
                   hipStream_t s) {
    if (p.shape_z.splits == 1) {
        launch_gemm(g, out, s);
        return;
    }
    float *parts = (float *)(w + p.parts_z);
    g.splits = p.shape_z.splits;
    launch_tiles({Product{g, parts_alone(parts)}, {}}, 1, {p.shape_z, {}}, s);
    const int64_t waves = (int64_t)g.M * p.tiles;
    hipLaunchKernelGGL(k_ce_logits, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, out, parts,
                       g.splits, g.M, g.N, live, g.m_lo);
}

template <typename T>
void launch_few(const FewArgs &f, const Plan &p, char *w, const FewGrad &g, bool gradient, void *dh,
                int64_t ld_dh, hipStream_t s) {
    const int32_t tiles = p.tiles, splits = p.splits;
    if (p.tiles_z) {
        hipLaunchKernelGGL(k_ce_few_rows, dim3(1), dim3(64), 0, s, f);
        GemmArgs z{};
        z.a = GemmOperand{(const bf16_t *)f.h, f.ld_h, 0};
        z.b = GemmOperand{(const bf16_t *)f.table, f.ld_table, 0};
        Packing packing;
        auto pack = [&](const void *src, int64_t ld, int64_t rows, int64_t to) {
            PackArgs k{};
            k.src = src;
            k.ld = ld;
            k.cols = f.D;
            k.n = k.total = rows;
            k.rows_packed = k.n_pad = pad64(rows);
            k.pieces = p.np;
            k.rows = (bf16_t *)(w + to);
            k.ld_rows = p.Dp;
            k.plane_rows = k.rows_packed * p.Dp;
            packing.add(k);
            return GemmOperand{k.rows, p.Dp, k.plane_rows};
        };
        if (p.pack_h) z.a = pack(f.h, f.ld_h, g.n, p.h);
        if (p.pack_table) z.b = pack(f.table, f.ld_table, g.V, p.table);
        packing.launch(std::is_same_v<T, float> ? ECC_F32 : ECC_BF16, s);
        z.M = g.n;
        z.N = g.V;
        z.K = (int32_t)p.Dp;
        z.batches = 1;
        set_products(z, p.np, p.np);
        launch_logits(z, p, w, f.out, f.rows.live, s);
    } else {
        auto logits = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(kFewThreads<T>), 0, s, f);
        };
        if (g.n <= 16) logits(k_ce_few<T, 1>);
        else if (g.n <= 32) logits(k_ce_few<T, 2>);
        else logits(k_ce_few<T, 4>);
    }
    const bool few = gradient && tiles <= kFewTiles;
    if (!few) hipLaunchKernelGGL(k_ce_rows, dim3(kTile / 4), dim3(256), 0, s, g.r);
    if (!gradient) return;
    auto gradients = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(g.blocks_d * splits)), dim3(waves * 64), 0,
                           s, g);
    };
    auto of_pieces = [&](auto pieces) {
        constexpr int PT = decltype(pieces)::value;
        auto of = [&](auto workers) {
            constexpr bool WORKERS = decltype(workers)::value;
            if (few) gradients(k_ce_few_grad<T, PT, true, WORKERS>, kFewWaves<T>);
            else gradients(k_ce_few_grad<T, PT, false, WORKERS>, kFewWaves<T>);
        };
        if (g.of_worker < g.n) of(std::true_type{});
        else of(std::false_type{});
    };
    if constexpr (std::is_same_v<T, float>) of_pieces(std::integral_constant<int, 3>{});
    else if (g.type == ECC_F32) of_pieces(std::integral_constant<int, 3>{});
    else of_pieces(std::integral_constant<int, 1>{});
    if (!dh) return;
    hipLaunchKernelGGL(k_ce_few_join<T>, dim3((unsigned)((g.D + 63) / 64), (unsigned)g.n), dim3(256),
                       0, s, g.dh, g.ld_dh, splits, g.r.rows, g.D, (T *)dh, ld_dh);
}

// The gradient of a table without rows to learn from.
template <typename T>
__global__ __launch_bounds__(256) void k_ce_zero(int64_t rows, int64_t V, int64_t D, T *g,
                                                 int64_t ld, int64_t stride) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        T *to = g + r / V * stride + r % V * ld;
        for (int64_t d = threadIdx.x; d < D; d += 256) store_elem<float>(to + d, 0.0f);
    }
}

}  // namespace
}  // namespace ecc

using namespace ecc;

extern "C" {

int64_t ecc_cross_entropy_work_size(const ecc_cross_entropy_t *a, int32_t gradient) {
    if (check(a) != ECC_OK) return -1;
    return make_plan(a, gradient != 0).bytes;
}

ecc_status_t ecc_cross_entropy(const ecc_cross_entropy_t *a, void *d_loss, void *d_dh,
                               int64_t ld_dh, void *d_dtable, int64_t ld_dtable,
                               int64_t worker_stride, int32_t accumulate, void *d_work,
                               void *hip_stream) {
    clear_error();
    const ecc_status_t st = check(a);
    if (st != ECC_OK) return st;
    const bool gradient = d_dh || d_dtable;
    const int64_t V = a->V, D = a->D, size = type_size(a->type), gsize = type_size(a->grad_type);
    const int32_t P = a->P;
    ECC_ARG(!d_dh || ld_dh >= D, "a leading dimension is below D");
    ECC_ARG(!d_dtable || ld_dtable >= D, "a leading dimension is below D");
    ECC_ARG(!d_dtable || P == 1 || worker_stride >= (V - 1) * ld_dtable + D,
            "workers' gradients overlap");
    ECC_ARG(accumulate == 0 || accumulate == 1, "accumulate must be 0 or 1");
    if (ld_dh >= (int64_t(1) << 40) || ld_dtable >= (int64_t(1) << 36) ||
        worker_stride >= (int64_t(1) << 56)) {
        set_error("a stride is too large");
        return ECC_ERR_RANGE;
    }
    ECC_ARG((uintptr_t)d_dh % size == 0 && (uintptr_t)d_dtable % gsize == 0 &&
                (uintptr_t)d_loss % 4 == 0 && (uintptr_t)d_work % 16 == 0,
            "an array is not aligned");
    hipStream_t s = (hipStream_t)hip_stream;
    if (a->n == 0) {
        if (d_dtable && !accumulate) {
            const int64_t rows = (int64_t)P * V;
            const dim3 grid((unsigned)std::min<int64_t>(rows, 4096));
            if (a->grad_type == ECC_F32)
                hipLaunchKernelGGL(k_ce_zero<float>, grid, dim3(256), 0, s, rows, V, D,
                                   (float *)d_dtable, ld_dtable, worker_stride);
            else
                hipLaunchKernelGGL(k_ce_zero<bf16_t>, grid, dim3(256), 0, s, rows, V, D,
                                   (bf16_t *)d_dtable, ld_dtable, worker_stride);
            ECC_LAUNCH_CHECK();
        }
        return ECC_OK;
    }
    const Plan p = make_plan(a, gradient);
    const int64_t N = p.N;
    ECC_ARG(d_loss && d_work, "NULL pointer");
    const Span in[4] = {span_of(a->d_h, N, a->ld_h, D, size),
                        span_of(a->d_table, V, a->ld_table, D, size),
                        span_of(a->d_labels, N * 4), span_of(a->d_weight, N * 4)};
    // (workers one behind the other are rows of one matrix)
    const Span out[4] = {
        span_of(d_loss, N * 4), span_of(d_dh, N, ld_dh, D, size),
        P == 1 ? span_of(d_dtable, V, ld_dtable, D, gsize)
               : span_of(d_dtable, P, worker_stride, (V - 1) * ld_dtable + D, gsize),
        span_of(d_work, p.bytes)};
    for (int o = 0; o < 4; ++o) {
        for (const Span &i : in) ECC_ARG(!spans_meet(out[o], i), "an output overlaps an input");
        for (int q = 0; q < o; ++q)
            ECC_ARG(!spans_meet(out[o], out[q]),
                    "two outputs, or an output and the work buffer, overlap");
    }
    char *w = (char *)d_work;
    const Rows rows{(int32_t *)(w + p.map), (int32_t *)(w + p.label), (float *)(w + p.weight),
                    (float *)(w + p.factor), (float *)(w + p.inside), (int32_t *)(w + p.live),
                    (int2 *)(w + p.ranges), (int32_t *)(w + p.counts), (float *)(w + p.outside)};
    const Positions q{a->d_labels, a->d_weight, a->n, (int32_t)V};
    if (p.few) {
        const LogitsOut logits{gradient ? (float *)(w + p.z) : nullptr, p.Vp, (float)a->scale,
                               (float2 *)(w + p.stats), p.tiles, a->d_labels, (float *)(w + p.picked)};
        const FewArgs f{a->d_h, a->d_table, a->ld_h, a->ld_table,
                        {a->d_labels, a->d_weight, N, (int32_t)V}, (int32_t)a->n, D, logits, rows,
                        (float *)d_loss, (float)a->scale};
        RowArgs row{};
        row.M = kTile;
        row.tiles = p.tiles;
        row.stats = logits.stats;
        row.picked = logits.picked;
        row.rows = rows;
        row.loss = (float *)d_loss;
        float *terms = gradient ? (float *)(w + p.terms) : nullptr;
        row.out = RowTerms{terms, gradient ? terms + kTile : nullptr};
        const FewGrad g{a->d_h, a->d_table, a->ld_h, a->ld_table, (int32_t)N, (int32_t)a->n,
                        (int32_t)V, D, logits.z, p.Vp, row,
                        d_dh ? (float *)(w + p.parts[0]) : nullptr, p.Dp, d_dtable, ld_dtable,
                        worker_stride, a->grad_type, accumulate, p.blocks_d, p.per};
        if (a->type == ECC_F32) launch_few<float>(f, p, w, g, gradient, d_dh, ld_dh, s);
        else launch_few<bf16_t>(f, p, w, g, gradient, d_dh, ld_dh, s);
        ECC_LAUNCH_CHECK();
        return ECC_OK;
    }
    if (P > 1)
        hipLaunchKernelGGL(k_ce_count, dim3((unsigned)P), dim3(kMapThreads), 0, s, q, rows);
    hipLaunchKernelGGL(k_ce_map, dim3((unsigned)P), dim3(kMapThreads), 0, s, q, rows, P, p.rows,
                       (float)a->scale, (float *)d_loss);
    Packing packing;
    if (p.pack_table || d_dh) {
        PackArgs k{};
        k.src = a->d_table;
        k.ld = a->ld_table;
        k.cols = D;
        k.rows_packed = k.n_pad = p.Vp;
        k.n = k.total = V;
        k.pieces = p.np;
        k.rows = p.pack_table ? (bf16_t *)(w + p.table) : nullptr;
        k.ld_rows = p.Dp;
        k.plane_rows = p.Vp * p.Dp;
        k.cols_out = d_dh ? (bf16_t *)(w + p.table_t) : nullptr;
        k.ld_cols = p.Vp;
        k.plane_cols = D * p.Vp;
        packing.add(k);
    }
    for (int64_t r0 = 0; r0 < p.rows; r0 += p.R) {
        const int64_t R = std::min(p.R, p.rows - r0);
        PackArgs k{};
        k.src = a->d_h;
        k.ld = a->ld_h;
        k.cols = D;
        k.rows_packed = R;
        k.row_map = rows.map + r0;
        k.live = rows.live;
        k.row0 = r0;
        k.pieces = p.np;
        k.rows = (bf16_t *)(w + p.h);
        k.ld_rows = p.Dp;
        k.plane_rows = R * p.Dp;
        k.cols_out = d_dtable ? (bf16_t *)(w + p.h_t) : nullptr;
        k.ld_cols = R;
        k.plane_cols = D * R;
        packing.add(k);
        packing.launch(a->type, s);
        packing = Packing{};
        GemmArgs g{};
        g.a = GemmOperand{k.rows, p.Dp, k.plane_rows};
        g.b = p.pack_table ? GemmOperand{(bf16_t *)(w + p.table), p.Dp, p.Vp * p.Dp}
                           : GemmOperand{(const bf16_t *)a->d_table, a->ld_table, 0};
        g.M = (int32_t)R;
        g.N = (int32_t)V;
        g.K = (int32_t)p.Dp;
        g.batches = 1;
        g.live = rows.live;
        g.m_lo = (int32_t)r0;
        set_products(g, p.np, p.np);
        const LogitsOut logits{gradient ? (float *)(w + p.z) : nullptr, p.Vp, (float)a->scale,
                               (float2 *)(w + p.stats), p.tiles, rows.label + r0,
                               (float *)(w + p.picked)};
        launch_logits(g, p, w, logits, rows.live, s);
        RowArgs row{};
        row.first = (int32_t)r0;
        row.M = (int32_t)R;
        row.tiles = p.tiles;
        row.stats = logits.stats;
        row.picked = logits.picked;
        row.rows = rows;
        row.loss = (float *)d_loss;
        // (positions that do not count: with the first piece)
        row.unread = Unread{q, d_dh && r0 == 0 ? N : 0, D, d_dh, ld_dh, a->type};
        const int64_t unread = (row.unread.N + kUnread - 1) / kUnread;
        const bool few = gradient && p.tiles <= kFewTiles;
        if (!few) {
            float *terms = gradient ? (float *)(w + p.terms) : nullptr;
            row.out = RowTerms{terms, gradient ? terms + R : nullptr};
            hipLaunchKernelGGL(k_ce_rows, dim3((unsigned)((R + unread + 3) / 4)), dim3(256), 0, s,
                               row);
        }
        if (!gradient) continue;
        DzArgs z{};
        z.z = logits.z;
        z.ld = p.Vp;
        z.V = (int32_t)V;
        z.r = row;
        z.dz = d_dh ? (bf16_t *)(w + p.dz) : nullptr;
        z.dzt = d_dtable ? (bf16_t *)(w + p.dzt) : nullptr;
        z.plane = R * p.Vp;
        z.ld_t = R;
        z.plane_t = V * R;
        z.pieces = p.pz;
        z.pieces_t = p.pzt;
        z.col_blocks = p.tiles;
        z.blocks = (int32_t)(R / kTile * p.tiles);
        const dim3 dz_grid((unsigned)(z.blocks + (few ? (unread + 3) / 4 : 0)));
        auto softmax = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dz_grid, dim3(256), 0, s, z);
        };
        if (a->type == ECC_F32) softmax(few ? k_ce_dz<float, true> : k_ce_dz<float, false>);
        else softmax(few ? k_ce_dz<bf16_t, true> : k_ce_dz<bf16_t, false>);
        Product products[2];
        GemmShape shapes[2];
        float *parts[2];
        int count = 0;
        if (d_dh) {
            GemmArgs d{};
            d.a = GemmOperand{z.dz, p.Vp, z.plane};
            d.b = GemmOperand{(bf16_t *)(w + p.table_t), p.Vp, D * p.Vp};
            d.M = (int32_t)R;
            d.N = (int32_t)D;
            d.K = (int32_t)p.Vp;
            d.batches = 1;
            d.live = rows.live;
            d.m_lo = (int32_t)r0;
            set_products(d, p.pz, p.np);
            MatrixOut out{};
            out.out = d_dh;
            out.ld = ld_dh;
            out.type = a->type;
            out.row_map = rows.map + r0;
            out.row_scale = rows.factor + r0;
            products[count] = Product{d, out};
            shapes[count] = p.shape_h;
            parts[count++] = (float *)(w + p.parts[0]);
        }
        if (d_dtable) {
            const bool first = r0 == 0, last = r0 + R >= p.rows;
            GemmArgs d{};
            d.a = GemmOperand{z.dzt, R, z.plane_t};
            d.b = GemmOperand{k.cols_out, R, k.plane_cols};
            d.M = (int32_t)V;
            d.N = (int32_t)D;
            d.batches = P;
            d.ranges = rows.ranges;
            d.k_lo = (int32_t)r0;
            d.k_hi = (int32_t)(r0 + R);
            set_products(d, p.pzt, p.np);
            MatrixOut out{};
            out.out = d_dtable;
            out.ld = ld_dtable;
            out.batch_stride = worker_stride;
            out.type = a->grad_type;
            out.scale = rows.outside;
            if (a->grad_type == ECC_F32 || p.pieces_of_rows == 1) {
                out.add = accumulate || !first;
                out.skip_empty = out.add;
            } else if (!last) {
                // pieces of a bf16 gradient are added up in fp32
                out.out = w + p.sums;
                out.ld = D;
                out.batch_stride = V * D;
                out.type = ECC_F32;
                out.add = out.skip_empty = !first;
            } else {
                out.sums = (const float *)(w + p.sums);
                out.add = accumulate;
            }
            products[count] = Product{d, out};
            shapes[count] = p.shape_e;
            parts[count++] = (float *)(w + p.parts[1]);
        }
        launch_products(products, count, shapes, parts, s);
    }
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
