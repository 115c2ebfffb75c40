// Cross entropy straight from hidden states, loss and gradients:
//   z = s h E^T,  loss_r = w_r (log sum exp z_r - z_r[y_r]),
//   dz = s w_r (softmax z_r - [j = y_r]),  dh = dz E,  dE_p = dz_p^T h_p.
// The logits exist for one piece of rows at a time.  Rows that count (weight
// not 0, label in the vocabulary) are packed first, so that the others cost
// nothing.  Per piece:
//   1. z as fp32, with every row's maximum and sum of exponentials per 64
//      columns formed from the sums in registers (alone where only the loss is
//      wanted: z is not stored then);
//   2. a wave per row joins them: loss, maximum, weight / sum;
//   3. dz as bf16 (the pieces of gemm.h where a gradient is fp32), in both
//      orders;
//   4. dh, scattered to the rows' places, and dE, added up over pieces in fp32.
// dz is rounded to bf16 for gradients that are bf16 themselves: one rounding of
// the terms beside the one of the result.
#include "gemm.h"
#include "pack.h"

namespace ecc {
namespace {

// Bytes of logits and their gradients at a time.
constexpr int64_t kPieceBytes = int64_t(5) << 30;

struct Rows {
    int32_t *map;      // packed row -> position, -1: none
    int32_t *label;
    float *weight;
    int32_t *live;     // packed rows that hold anything (a multiple of 64)
    int2 *ranges;      // of every worker
    int32_t *counts;   // rows per worker, rounded up
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

// Every worker's rows in order, each worker's from a multiple of 64 on: a
// workgroup per worker, which first adds up the counts of those before it.
__global__ __launch_bounds__(kMapThreads) void k_ce_map(Positions q, Rows rows, int32_t P,
                                                        int64_t capacity, float *loss) {
    __shared__ int s_sum[kMapThreads / 64 + 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int32_t p = blockIdx.x;
    int before = 0;
    for (int32_t i = threadIdx.x; i < p; i += kMapThreads) before += rows.counts[i];
    before = wave_scan(before);
    if (lane == 63) s_sum[wave] = before;
    __syncthreads();
    before = 0;
    for (int w = 0; w < kMapThreads / 64; ++w) before += s_sum[w];
    __syncthreads();
    int at = before;
    const int64_t base = p * q.n;
    for (int64_t i0 = 0; i0 < q.n; i0 += kMapThreads * kMapRows) {
        const int64_t i = i0 + threadIdx.x * kMapRows;
        uint32_t held = 0;
#pragma unroll
        for (int e = 0; e < kMapRows; ++e)
            if (i + e < q.n) {
                if (q.counts(base + i + e)) held |= 1u << e;
                else loss[base + i + e] = 0.0f;
            }
        const int mine = __popc(held), upto = wave_scan(mine);
        if (lane == 63) s_sum[wave] = upto;
        __syncthreads();
        int row = at + upto - mine;
        for (int w = 0; w < kMapThreads / 64; ++w) {
            if (w < wave) row += s_sum[w];
            at += s_sum[w];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kMapRows; ++e)
            if (held >> e & 1) {
                const int64_t from = base + i + e;
                rows.map[row] = (int32_t)from;
                rows.label[row] = q.labels[from];
                rows.weight[row] = q.weight ? q.weight[from] : 1.0f;
                ++row;
            }
    }
    const int end = (at + 63) & ~63;
    if (threadIdx.x == 0) rows.ranges[p] = make_int2(before, end);
    const bool last = p == P - 1;
    if (last && threadIdx.x == 0) *rows.live = end;
    for (int64_t r = at + threadIdx.x; r < (last ? capacity : end); r += kMapThreads) {
        rows.map[r] = -1;
        rows.label[r] = -1;
        rows.weight[r] = 0.0f;
    }
}

// Zeros for the rows of dh that do not count: a wave per position.
template <typename T>
__global__ __launch_bounds__(256) void k_ce_dead(Positions q, int64_t first, int64_t N, int64_t D,
                                                 T *dh, int64_t ld) {
    const int64_t i = first + blockIdx.x * (int64_t)4 + (threadIdx.x >> 6);
    if (i >= N || q.counts(i)) return;
    for (int64_t d = threadIdx.x & 63; d < D; d += 64) store_elem<float>(dh + i * ld + d, 0.0f);
}

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
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int32_t m = t.m + 16 * i;
            const bool row = m < g.M;
            const int32_t y = row ? label[m] : -1;
            float most = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int32_t n = t.n + 16 * j;
                acc[i][j] *= scale;
                if (z && row && n < ld) *reinterpret_cast<f32x4 *>(z + m * ld + n) = acc[i][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (n + e == y && y >= 0) picked[m] = acc[i][j][e];
                    if (n + e < g.N) most = fmaxf(most, acc[i][j][e]);
                }
            }
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float from = most == -__builtin_inff() ? 0.0f : most;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t.n + 16 * j + e < g.N) sum += expf(acc[i][j][e] - from);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (first && row && t.tile_n < tiles)
                stats[(int64_t)m * tiles + t.tile_n] = make_float2(most, sum);
        }
    }
};

struct RowTerms {
    float *most, *soft, *hard;  // dz = exp(z - most) soft - [label] hard
};

// A wave per packed row: the loss, and the terms of its gradient.
__global__ __launch_bounds__(256) void k_ce_rows(int32_t first, int32_t M, const int32_t *live,
                                                 const float2 *stats, int32_t tiles,
                                                 const float *picked, Rows rows, float scale,
                                                 float *loss, RowTerms out) {
    const int32_t m = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (m >= M || first + m >= *live) return;
    const int32_t to = rows.map[first + m];
    float most = 0.0f, soft = 0.0f, hard = 0.0f;
    if (to >= 0) {
        const float2 *s = stats + (int64_t)m * tiles;
        float top = -__builtin_inff();
        for (int32_t i = lane; i < tiles; i += 64) top = fmaxf(top, s[i].x);
        top = wave_all(top, OpMax());
        const float from = top == -__builtin_inff() ? 0.0f : top;
        float sum = 0.0f;
        for (int32_t i = lane; i < tiles; i += 64) {
            const float2 v = s[i];
            // (a tile of NaN has a sum of NaN, and so has the row)
            sum += v.y * (v.x == -__builtin_inff() ? 1.0f : expf(v.x - from));
        }
        sum = wave_all(sum, OpSum());
        const float w = rows.weight[first + m];
        most = from;
        hard = w * scale;
        soft = hard / sum;
        if (lane == 0) loss[to] = w * ((from - picked[m]) + logf(sum));
    }
    if (out.most && lane == 0) {
        out.most[m] = most;
        out.soft[m] = soft;
        out.hard[m] = hard;
    }
}

struct DzArgs {
    const float *z;
    int64_t ld;               // of z and of dz, a multiple of 64
    int32_t V, first;
    const int32_t *live, *label;
    RowTerms row;
    bf16_t *dz, *dzt;
    int64_t plane, plane_t, ld_t;
    int32_t pieces, pieces_t;
    int32_t col_blocks;
};

// dz in both orders, blocks of 64 x 64.  Bound by memory: 4 bytes read and 2
// written for each order and piece.
__global__ __launch_bounds__(256) void k_ce_dz(DzArgs a) {
    __shared__ PackTile s;
    const int64_t row0 = (int64_t)(blockIdx.x / a.col_blocks) * kTile;
    const int64_t col0 = (int64_t)(blockIdx.x % a.col_blocks) * kTile;
    if (row0 + a.first >= *a.live) return;
    const int c8 = (threadIdx.x & 7) * 8, r = threadIdx.x >> 3;
    float mine[2][8];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int64_t m = row0 + p * 32 + r;
        Raw<float, 8> x;
        x.load(a.z + m * a.ld + col0 + c8);
        const int32_t y = a.label[m];
        const float most = a.row.most[m], soft = a.row.soft[m], hard = a.row.hard[m];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t j = (int32_t)col0 + c8 + e;
            float v = expf(x.get<float>(e) - most) * soft;
            if (j == y) v -= hard;
            mine[p][e] = y >= 0 && j < a.V ? v : 0.0f;
        }
    }
    write_block(s, mine, row0, col0, a.V, a.dz, a.ld, a.plane, a.pieces, a.dzt, a.ld_t, a.plane_t,
                a.pieces_t);
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
    GemmShape shape_h, shape_e;
    // offsets into the work buffer
    int64_t map, label, weight, live, ranges, counts, table, table_t, h, h_t, z, dz, dzt, stats,
        picked, terms, sums, parts, bytes;
};

Plan make_plan(const ecc_cross_entropy_t *a, bool gradient) {
    Plan p{};
    p.N = a->P * a->n;
    p.n_pad = pad64(a->n);
    p.rows = a->P * p.n_pad;
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
    p.live = take(4);
    p.ranges = take(8 * (int64_t)a->P);
    p.counts = take(4 * (int64_t)a->P);
    p.table = take(p.pack_table ? p.np * 2 * p.Vp * p.Dp : 0);
    p.h = take(p.np * 2 * p.R * p.Dp);
    p.stats = take(8 * p.R * p.tiles);
    p.picked = take(4 * p.R);
    if (gradient) {
        p.table_t = take(p.np * 2 * a->D * p.Vp);
        p.h_t = take(p.np * 2 * a->D * p.R);
        p.z = take(4 * p.R * p.Vp);
        p.dz = take(2 * p.pz * p.R * p.Vp);
        p.dzt = take(2 * p.pzt * a->V * p.R);
        p.terms = take(12 * p.R);
        p.sums = take(p.pieces_of_rows > 1 && a->grad_type != ECC_F32 ? 4 * a->P * a->V * a->D : 0);
        p.shape_h = gemm_shape(p.R, a->D, p.Vp / kGemmK * (p.np == 3 ? 6 : 1), 1, true);
        // (a worker's rows in a piece)
        p.shape_e = gemm_shape(a->V, a->D,
                               std::min(p.n_pad, p.R) / kGemmK * (p.np == 3 ? 6 : p.pzt), a->P,
                               true);
        p.parts = take(std::max(split_bytes(p.R, a->D, p.shape_h.splits, 1),
                                split_bytes(a->V, a->D, p.shape_e.splits, a->P)));
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
    if (a->V > ECC_CROSS_ENTROPY_MAX_VOCAB || a->D > ECC_CROSS_ENTROPY_MAX_DIM ||
        a->n > (int64_t(1) << 31) || (__int128)a->P * pad64(a->n) >= (int64_t(1) << 31) - 1024 ||
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

template <typename T>
void zero_dead(const Positions &q, int64_t N, int64_t D, void *dh, int64_t ld, hipStream_t s) {
    const int64_t most = int64_t(1) << 25;
    for (int64_t i = 0; i < N; i += most)
        hipLaunchKernelGGL(k_ce_dead<T>, dim3((unsigned)((std::min(most, N - i) + 3) / 4)),
                           dim3(256), 0, s, q, i, std::min(N, i + most), D, (T *)dh, ld);
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
                    (int32_t *)(w + p.live), (int2 *)(w + p.ranges), (int32_t *)(w + p.counts)};
    const Positions q{a->d_labels, a->d_weight, a->n, (int32_t)V};
    if (P > 1)
        hipLaunchKernelGGL(k_ce_count, dim3((unsigned)P), dim3(kMapThreads), 0, s, q, rows);
    hipLaunchKernelGGL(k_ce_map, dim3((unsigned)P), dim3(kMapThreads), 0, s, q, rows, P, p.rows,
                       (float *)d_loss);
    if (d_dh) {
        if (a->type == ECC_F32) zero_dead<float>(q, N, D, d_dh, ld_dh, s);
        else zero_dead<bf16_t>(q, N, D, d_dh, ld_dh, s);
    }
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
        launch_pack(k, a->type, s);
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
        launch_pack(k, a->type, s);
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
        launch_gemm(g, logits, s);
        float *terms = gradient ? (float *)(w + p.terms) : nullptr;
        const RowTerms row{terms, gradient ? terms + R : nullptr,
                           gradient ? terms + 2 * R : nullptr};
        hipLaunchKernelGGL(k_ce_rows, dim3((unsigned)((R + 3) / 4)), dim3(256), 0, s, (int32_t)r0,
                           (int32_t)R, rows.live, logits.stats, p.tiles, logits.picked, rows,
                           (float)a->scale, (float *)d_loss, row);
        if (!gradient) continue;
        DzArgs z{};
        z.z = logits.z;
        z.ld = p.Vp;
        z.V = (int32_t)V;
        z.first = (int32_t)r0;
        z.live = rows.live;
        z.label = rows.label + r0;
        z.row = row;
        z.dz = d_dh ? (bf16_t *)(w + p.dz) : nullptr;
        z.dzt = d_dtable ? (bf16_t *)(w + p.dzt) : nullptr;
        z.plane = R * p.Vp;
        z.ld_t = R;
        z.plane_t = V * R;
        z.pieces = p.pz;
        z.pieces_t = p.pzt;
        z.col_blocks = p.tiles;
        hipLaunchKernelGGL(k_ce_dz, dim3((unsigned)(R / kTile * p.tiles)), dim3(256), 0, s, z);
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
            launch_product(d, out, p.shape_h, (float *)(w + p.parts), s);
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
            if (a->grad_type == ECC_F32 || p.pieces_of_rows == 1) {
                out.add = accumulate || !first;
                out.skip_empty = out.add;
            } else {
                out.sums = first ? nullptr : (const float *)(w + p.sums);
                out.to_sums = last ? nullptr : (float *)(w + p.sums);
                out.add = last && accumulate;
                out.skip_empty = !first && !last;
            }
            launch_product(d, out, p.shape_e, (float *)(w + p.parts), s);
        }
    }
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
