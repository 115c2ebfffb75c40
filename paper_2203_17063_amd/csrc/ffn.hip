// The gated feed-forward block up to its inner width, and its gradients:
//   g = x Wg^T,  u = x Wu^T,  y = act(g) u
//   dg = dy u act'(g),  du = dy act(g)
//   dx = dg Wg + du Wu,  dWg_p = dg_p^T x_p,  dWu_p = du_p^T x_p.
// Forward is one product kernel: a wave holds the same columns of g and u, so
// that y is formed from the sums in registers and rounded once.  Backward forms
// g and u again instead of keeping them (a third of its operations), and dg and
// du from them in registers; they are stored beside each other as one matrix
// [dg | du], so that dx is one product over both along k, and the weights'
// gradients one product with both stacked.  dg and du are rounded to bf16
// where the gradient is bf16 itself, and kept as three pieces (gemm.h) where
// it is fp32.
#include "pack.h"

namespace ecc {
namespace {

// act(g) and its derivative.  The error function is Abramowitz and Stegun's
// 7.1.26 (Hastings), within 1.5e-7 of it: half of 1 - erf(|x|) is a polynomial
// in 1 / (1 + p |x|) times exp(-x^2), at x = g / sqrt 2 the exponential that the
// derivative needs too.  For negative g that half is the factor itself, within
// 7.5e-8; the bound is an absolute one, so that small factors have fewer digits
// (off by 5e-5 of themselves at g = -3, 5e-4 at -4, 1.6e-3 at -5, 1e-2 at -8, where
// 1 + erf in fp32 has none left from -5.5 on).  Exponentials of fp32 rows within 2
// ulp, of bf16 rows the short ones: 8,192 rows, D 256, F 2,501: 40 us against 45 us.
template <int ACT, typename T>
__device__ __forceinline__ void activation(float g, float &a, float &da) {
    if constexpr (ACT == ECC_ACT_SILU) {
        const float q = recip_fast(1.0f + exp_of<T>(-g));
        a = g * q;
        da = q * (1.0f + g * (1.0f - q));
    } else {
        const float e = exp_of<T>(-0.5f * g * g);
        const float t = recip_fast(__builtin_fmaf(__builtin_fabsf(g), 0.3275911f * 0.70710678f, 1.0f));
        float h = __builtin_fmaf(t, 1.061405429f, -1.453152027f);
        h = __builtin_fmaf(t, h, 1.421413741f);
        h = __builtin_fmaf(t, h, -0.284496736f);
        h = __builtin_fmaf(t, h, 0.254829592f);
        h *= 0.5f * t * e;
        const float c = g < 0.0f ? h : 1.0f - h;
        a = g * c;
        da = c + g * e * 0.39894228f;
    }
}

template <typename T, int ACT>
struct FfnOut {
    static constexpr bool kPair = true;
    T *y;
    int64_t ld;
    template <int MI, int NI>
    __device__ __forceinline__ void finish(const GemmTile &t, const GemmArgs &g,
                                           f32x4 (&acc)[MI][NI]) const {
        const int32_t m0 = t.m & ~15, n0 = t.n - (threadIdx.x >> 4 & 3) * 4;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            f32x4 v[NI / 2];
#pragma unroll
            for (int j = 0; j < NI / 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, da;
                    activation<ACT, T>(acc[i][j][e], a, da);
                    v[j][e] = a * acc[i][j + NI / 2][e];
                }
            turn<NI / 2>(t.lds, v, [&](int row, int col, f32x4 u) {
                const int32_t m = m0 + 16 * i + row, n = n0 + col;
                if (m >= g.M || n >= g.N) return;
                const float w[4] = {u[0], u[1], u[2], u[3]};
                Raw<T, 4> x;
                x.set_all(w);
                x.store_upto(y + m * ld + n, g.N - n);
            });
        }
    }
};

template <typename T, int ACT>
struct FfnGradOut {
    static constexpr bool kPair = true;
    const T *dy;
    int64_t ld_dy;
    bf16_t *d;            // [piece][row][dg | du], each F_pad long
    int64_t F_pad, plane;
    int32_t pieces;
    template <int MI, int NI>
    __device__ __forceinline__ void finish(const GemmTile &t, const GemmArgs &g,
                                           f32x4 (&acc)[MI][NI]) const {
        const int32_t m0 = t.m & ~15, n0 = t.n - (threadIdx.x >> 4 & 3) * 4;
        const bool whole = m0 + 16 * MI <= g.M && n0 + 8 * NI <= g.N;
        // (the loads of some rows go together)
        constexpr int G = MI < 4 ? MI : 4;
#pragma unroll
        for (int i0 = 0; i0 < MI; i0 += G) {
            Raw<T, 4> x[G][NI / 2];
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int j = 0; j < NI / 2; ++j) {
                    const int32_t m = t.m + 16 * (i0 + i), n = t.n + 16 * j;
                    if (whole) x[i][j].load(dy + m * ld_dy + n);
                    else x[i][j].load_upto(dy + (m < g.M ? m * ld_dy + n : 0),
                                           m < g.M ? (int64_t)g.N - n : 0);
                }
#pragma unroll
            for (int i = 0; i < G; ++i) {
                f32x4 dg[NI / 2], du[NI / 2];
#pragma unroll
                for (int j = 0; j < NI / 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float a, da;
                        activation<ACT, T>(acc[i0 + i][j][e], a, da);
                        const float v = x[i][j].template get<float>(e);
                        // (columns behind the last are zeros: what was summed
                        // for them is the last one's again)
                        const bool in = whole || t.n + 16 * j + e < g.N;
                        dg[j][e] = in ? v * acc[i0 + i][j + NI / 2][e] * da : 0.0f;
                        du[j][e] = in ? v * a : 0.0f;
                    }
                auto put = [&](const f32x4 (&v)[NI / 2], int64_t at) {
                    turn<NI / 2>(t.lds, v, [&](int row, int col, f32x4 u) {
                        const int32_t m = m0 + 16 * (i0 + i) + row, n = n0 + col;
                        if (!whole && (m >= g.M || n >= F_pad)) return;
                        float w[4] = {u[0], u[1], u[2], u[3]};
                        store_pieces(d + m * 2 * F_pad + at + n, w);
                    });
                };
                put(dg, 0);
                put(du, F_pad);
            }
        }
    }
    // (a piece is what is left, rounded; then it is taken off)
    __device__ __forceinline__ void store_pieces(bf16_t *to, float (&v)[4]) const {
        Raw<bf16_t, 4> p;
        p.set_all(v);
        p.store(to);
        if (pieces == 1) return;
#pragma unroll
        for (int which = 1; which < 3; ++which) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] -= p.get<float>(e);
            p.set_all(v);
            p.store(to + which * plane);
        }
    }
};

// The same from the parts of two products that are split along D (few tiles, a
// long sum): a thread per four columns of a row.
struct FfnParts {
    const float *g, *u;
    int32_t splits, M, N;
};
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_ffn_join(FfnParts p, FfnOut<T, ACT> out, int64_t quads) {
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i >= quads) return;
    const int32_t per = (p.N + 3) / 4;
    const int64_t m = i / per;
    const int32_t n = (int32_t)(i - m * per) * 4;
    const f32x4 g = sum_of_parts(p.g, p.splits, p.M, p.N, m, n);
    const f32x4 u = sum_of_parts(p.u, p.splits, p.M, p.N, m, n);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, da;
        activation<ACT, T>(g[e], a, da);
        v[e] = a * u[e];
    }
    Raw<T, 4> x;
    x.set_all(v);
    x.store_upto(out.y + m * out.ld + n, p.N - n);
}
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_ffn_grad_join(FfnParts p, FfnGradOut<T, ACT> out,
                                                       int64_t quads) {
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i >= quads) return;
    const int32_t per = (int32_t)(out.F_pad / 4);
    const int64_t m = i / per;
    const int32_t n = (int32_t)(i - m * per) * 4;
    float dg[4] = {0, 0, 0, 0}, du[4] = {0, 0, 0, 0};
    if (n < p.N) {
        const f32x4 g = sum_of_parts(p.g, p.splits, p.M, p.N, m, n);
        const f32x4 u = sum_of_parts(p.u, p.splits, p.M, p.N, m, n);
        Raw<T, 4> x;
        x.load_upto(out.dy + m * out.ld_dy + n, (int64_t)p.N - n);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= p.N) continue;
            float a, da;
            activation<ACT, T>(g[e], a, da);
            const float v = x.template get<float>(e);
            dg[e] = v * u[e] * da;
            du[e] = v * a;
        }
    }
    bf16_t *to = out.d + m * 2 * out.F_pad + n;
    out.store_pieces(to, dg);
    out.store_pieces(to + out.F_pad, du);
}

// ---------------------------------------------------------------------------
// few rows (single tokens)
// ---------------------------------------------------------------------------

// Bound by the weights' bytes, which are read once, straight into the matrix
// cores' registers: a workgroup forms 16 columns of g and u for all rows, its
// eight waves share the elements along D in turn, kAhead loads of each wave
// under way at once, and add up in LDS in their order.  Operands need no
// alignment and fp32 is split where it is loaded, so that nothing is packed.
// 8 rows, D 4,096, F 12,288, bf16: 37 us (5.5 TB/s).
constexpr int kFewWaves = 8;

template <typename T, int ACT, int MB>
__global__ __launch_bounds__(64 * kFewWaves) void k_ffn_few(const T *x, int64_t ld_x,
                                                            const T *w_gate, int64_t ld_gate,
                                                            const T *w_up, int64_t ld_up, T *y,
                                                            int64_t ld_y, int32_t M, int32_t F,
                                                            int64_t D) {
    using S = FewStep<T>;
    constexpr int kAhead = MB == 4 ? 2 : 4;
    __shared__ f32x4 s_acc[kFewWaves][2][MB][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    const int32_t f0 = blockIdx.x * 16;
    const T *rows[2] = {w_gate + min(f0 + c, F - 1) * ld_gate, w_up + min(f0 + c, F - 1) * ld_up};
    const T *mine[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) mine[i] = x + min(i * 16 + c, M - 1) * ld_x;
    f32x4 acc[2][MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[0][i] = acc[1][i] = f32x4{0, 0, 0, 0};
    for (int64_t k = (int64_t)wave * S::kStep; k < D; k += kFewWaves * kAhead * S::kStep) {
        S w[kAhead][2], a[kAhead][MB];
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            const int64_t at = k + h * kFewWaves * S::kStep + q * S::kLane;
#pragma unroll
            for (int g = 0; g < 2; ++g) w[h][g].load(rows[g], at, D);
#pragma unroll
            for (int i = 0; i < MB; ++i) a[h][i].load(mine[i], at, D);
        }
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            bf16x8 fw[2][S::kFrags][S::kPieces];
#pragma unroll
            for (int g = 0; g < 2; ++g) w[h][g].frags(fw[g]);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                bf16x8 fa[S::kFrags][S::kPieces];
                a[h][i].frags(fa);
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int j = 0; j < S::kFrags; ++j) {
                        products<S::kPieces, S::kPieces>([&](int pw, int pa) {
                            acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                fw[g][j][pw], fa[j][pa], acc[g][i], 0, 0, 0);
                        });
                    }
            }
        }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < MB; ++i) s_acc[wave][g][i][lane] = acc[g][i];
    __syncthreads();
    // a lane's four columns of a row
    if (wave >= MB) return;
    f32x4 g = s_acc[0][0][wave][lane], u = s_acc[0][1][wave][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) {
        g += s_acc[w][0][wave][lane];
        u += s_acc[w][1][wave][lane];
    }
    const int32_t m = wave * 16 + c, n = f0 + q * 4;
    if (m >= M || n >= F) return;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float b, db;
        activation<ACT, T>(g[e], b, db);
        v[e] = b * u[e];
    }
    Raw<T, 4> out;
    out.set_all(v);
    out.store_upto(y + m * ld_y + n, F - n);
}

template <typename T, int ACT>
void launch_few(const ecc_ffn_t *a, void *d_y, int64_t ld_y, hipStream_t s) {
    const int32_t M = (int32_t)(a->P * a->n), F = (int32_t)a->F;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((F + 15) / 16)), dim3(64 * kFewWaves), 0, s,
                           (const T *)a->d_x, a->ld_x, (const T *)a->d_w_gate, a->ld_gate,
                           (const T *)a->d_w_up, a->ld_up, (T *)d_y, ld_y, M, F, a->D);
    };
    if (M <= 16) launch(k_ffn_few<T, ACT, 1>);
    else if (M <= 32) launch(k_ffn_few<T, ACT, 2>);
    else launch(k_ffn_few<T, ACT, 4>);
}

struct Plan {
    int64_t N, n_pad, rows, Dp, Fp;
    int np, pd;                   // pieces of the operands, of dg and du
    bool few;                     // forward by k_ffn_few
    bool pack_x, pack_gate, pack_up;
    GemmShape shape_f, shape_x, shape_w;
    int64_t parts_f[2];
    int64_t x, gate, up, x_t, w_t, d, d_t, parts[2], bytes;
};

// Do few rows go by k_ffn_few?  By the times that it and the tiles take, in us per
// MB of bf16 weights out of memory: one, two or four blocks of 16 rows, each read
// again for every 16 columns, of rows that begin at 4 bytes or not; and how long
// one workgroup takes for its share of D.  Tiles pack weights whose rows are no
// multiple of 64.  Rows are taken to lie one behind the other: the choice goes by
// the sizes alone, so that operands at another place or pitch give the same bits.
// D 4,096, F 12,288: 8 rows 39 us and 48 us, 64 rows 74 us and 50
// us; D 4,096, F 1,000: 8 rows 13 us and 17 us, 64 rows 25 us and 21 us; D 2,001, F
// 5,003: 8 rows 29 us and 35 us, 64 rows 64 us and 37 us; D 1,000, F 8,000: 64 rows
// 16 us and 30 us.  (Weights that the last cache holds come out in 34 us instead of
// 48, a loop over one layer's.)  fp32, 64 rows, D 4,096, F 4,096: 63 us and 138 us.
bool takes_few(const ecc_ffn_t *a) {
    const int64_t N = a->P * a->n;
    if (N > kFewRows) return false;
    if (a->type == ECC_F32) return true;
    static constexpr double kTimes[2][3] = {{0.165, 0.225, 0.325}, {0.57, 0.87, 1.38}};
    static constexpr double kLong[3] = {0.0013, 0.0021, 0.0039};
    const int rows = N <= 16 ? 0 : N <= 32 ? 1 : 2;
    const double mb = 4e-6 * (double)a->D * a->F;
    const double few = 9.0 + std::max(mb * kTimes[a->D % 2][rows], a->D * kLong[rows]);
    return few <= (a->D % 64 ? 12.0 + mb * 0.57 : std::max(17.0, 10.0 + mb * 0.19));
}

Plan make_plan(const ecc_ffn_t *a, bool gradient) {
    Plan p{};
    p.N = a->P * a->n;
    p.n_pad = pad64(a->n);
    p.rows = a->P * p.n_pad;
    p.Dp = pad64(a->D);
    p.Fp = pad64(a->F);
    p.np = a->type == ECC_F32 ? 3 : 1;
    p.pd = a->type == ECC_F32 || a->grad_type == ECC_F32 ? 3 : 1;
    p.few = !gradient && takes_few(a);
    if (p.few) {
        p.bytes = 16;
        return p;
    }
    p.pack_x = !as_it_lies(a->d_x, a->ld_x, a->D, a->type);
    p.pack_gate = !as_it_lies(a->d_w_gate, a->ld_gate, a->D, a->type);
    p.pack_up = !as_it_lies(a->d_w_up, a->ld_up, a->D, a->type);
    // (a pair of matrices has one pitch)
    if (p.pack_gate || p.pack_up || a->ld_gate != a->ld_up) p.pack_gate = p.pack_up = true;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) & ~int64_t(255);
        return here;
    };
    p.x = take(p.pack_x ? p.np * 2 * pad64(p.N) * p.Dp : 0);
    p.gate = take(p.pack_gate ? p.np * 2 * p.Fp * p.Dp : 0);
    p.up = take(p.pack_up ? p.np * 2 * p.Fp * p.Dp : 0);
    p.shape_f = gemm_shape(p.N, a->F, p.Dp / kGemmK * (p.np == 3 ? 6 : 1), 2, true);
    for (int64_t &at_f : p.parts_f) at_f = take(split_bytes(p.N, a->F, p.shape_f.splits, 1));
    if (gradient) {
        p.x_t = take(p.np * 2 * a->D * p.rows);
        p.w_t = take(p.np * 2 * a->D * 2 * p.Fp);
        p.d = take(p.pd * 2 * pad64(p.N) * 2 * p.Fp);
        p.d_t = take(p.pd * 2 * 2 * a->F * p.rows);
        p.shape_x = gemm_shape(p.N, a->D, 2 * p.Fp / kGemmK * (p.np == 3 ? 6 : 1), 1, true);
        p.shape_w = gemm_shape(2 * a->F, a->D, p.n_pad / kGemmK * (p.np == 3 ? 6 : p.pd), a->P, true);
        p.parts[0] = take(split_bytes(p.N, a->D, p.shape_x.splits, 1));
        p.parts[1] = take(split_bytes(2 * a->F, a->D, p.shape_w.splits, a->P));
    }
    p.bytes = std::max<int64_t>(at, 16);
    return p;
}

ecc_status_t check(const ecc_ffn_t *a) {
    ECC_ARG(a, "NULL description");
    ECC_ARG(a->n >= 0 && a->F >= 1 && a->D >= 1 && a->P >= 1, "a size is out of range");
    ECC_ARG(a->type == ECC_F32 || a->type == ECC_BF16, "the operands must be fp32 or bf16");
    ECC_ARG(a->grad_type == ECC_F32 || a->grad_type == a->type,
            "the weights' gradients must be fp32 or of the operands' type");
    ECC_ARG(a->act == ECC_ACT_SILU || a->act == ECC_ACT_GELU, "unknown activation");
    ECC_ARG(a->ld_x >= a->D && a->ld_gate >= a->D && a->ld_up >= a->D,
            "a leading dimension is below D");
    if (a->F > ECC_FFN_MAX_DIM || a->D > ECC_FFN_MAX_DIM || a->n > ECC_FFN_MAX_ROWS ||
        (__int128)a->P * pad64(a->n) > ECC_FFN_MAX_ROWS || a->ld_x >= (int64_t(1) << 40) ||
        a->ld_gate >= (int64_t(1) << 40) || a->ld_up >= (int64_t(1) << 40) ||
        !gemm_in_range(a->P * a->n, 2 * a->F, 1) || !gemm_in_range(a->P * a->n, a->D, 1) ||
        !gemm_in_range(2 * a->F, a->D, a->P)) {
        set_error("the sizes are beyond what the library supports");
        return ECC_ERR_RANGE;
    }
    if (a->n == 0) return ECC_OK;
    const int64_t size = type_size(a->type);
    ECC_ARG(a->d_x && a->d_w_gate && a->d_w_up, "NULL pointer");
    ECC_ARG((uintptr_t)a->d_x % size == 0 && (uintptr_t)a->d_w_gate % size == 0 &&
                (uintptr_t)a->d_w_up % size == 0,
            "an array is not aligned");
    return ECC_OK;
}

// The projections' operands, packed where they have to be.
GemmArgs projections(const ecc_ffn_t *a, const Plan &p, char *w, hipStream_t s) {
    PackArgs k{};
    k.cols = a->D;
    k.pieces = p.np;
    k.ld_rows = p.Dp;
    GemmArgs g{};
    g.a = GemmOperand{(const bf16_t *)a->d_x, a->ld_x, 0};
    g.b = GemmOperand{(const bf16_t *)a->d_w_gate, a->ld_gate, 0};
    g.b2 = (const bf16_t *)a->d_w_up;
    Packing packing;
    auto pack = [&](const void *src, int64_t ld, int64_t rows, int64_t to) {
        k.src = src;
        k.ld = ld;
        k.n = k.total = rows;
        k.rows_packed = k.n_pad = pad64(rows);
        k.rows = (bf16_t *)(w + to);
        k.plane_rows = k.rows_packed * p.Dp;
        packing.add(k);
        return GemmOperand{k.rows, p.Dp, k.plane_rows};
    };
    if (p.pack_x) g.a = pack(a->d_x, a->ld_x, p.N, p.x);
    if (p.pack_gate) {
        g.b = pack(a->d_w_gate, a->ld_gate, a->F, p.gate);
        g.b2 = pack(a->d_w_up, a->ld_up, a->F, p.up).p;
    }
    packing.launch(a->type, s);
    g.M = (int32_t)p.N;
    g.N = (int32_t)a->F;
    g.K = (int32_t)p.Dp;
    g.batches = 1;
    set_products(g, p.np, p.np);
    return g;
}

// Both projections into parts, where that is quicker.
bool split_projections(GemmArgs g, const Plan &p, char *w, FfnParts &parts, hipStream_t s) {
    if (p.shape_f.splits == 1) return false;
    float *to[2] = {(float *)(w + p.parts_f[0]), (float *)(w + p.parts_f[1])};
    g.splits = p.shape_f.splits;
    GemmArgs u = g;
    u.b.p = g.b2;
    launch_tiles({Product{g, parts_alone(to[0])}, Product{u, parts_alone(to[1])}}, 2,
                 {p.shape_f, p.shape_f}, s);
    parts = FfnParts{to[0], to[1], g.splits, g.M, g.N};
    return true;
}

template <typename F>
void with_kind(const ecc_ffn_t *a, F &&f) {
    auto act = [&](auto t) {
        if (a->act == ECC_ACT_SILU) f(t, std::integral_constant<int, ECC_ACT_SILU>{});
        else f(t, std::integral_constant<int, ECC_ACT_GELU>{});
    };
    if (a->type == ECC_F32) act(float{});
    else act(bf16_t{});
}

// Gradients of weights that no row reached.
template <typename T>
__global__ __launch_bounds__(256) void k_ffn_zero(int64_t rows, int64_t F, int64_t D, T *g,
                                                  int64_t stride) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        T *to = g + r / F * stride + r % F * D;
        for (int64_t d = threadIdx.x; d < D; d += 256) store_elem<float>(to + d, 0.0f);
    }
}

}  // namespace
}  // namespace ecc

using namespace ecc;

extern "C" {

int64_t ecc_ffn_work_size(const ecc_ffn_t *a, int32_t gradient) {
    if (check(a) != ECC_OK) return -1;
    return make_plan(a, gradient != 0).bytes;
}

ecc_status_t ecc_ffn_forward(const ecc_ffn_t *a, void *d_y, int64_t ld_y, void *d_work,
                             void *hip_stream) {
    clear_error();
    const ecc_status_t st = check(a);
    if (st != ECC_OK) return st;
    ECC_ARG(ld_y >= a->F, "a leading dimension is below F");
    if (ld_y >= (int64_t(1) << 40)) {
        set_error("a leading dimension is too large");
        return ECC_ERR_RANGE;
    }
    if (a->n == 0) return ECC_OK;
    const int64_t size = type_size(a->type);
    ECC_ARG(d_y && d_work, "NULL pointer");
    ECC_ARG((uintptr_t)d_y % size == 0 && (uintptr_t)d_work % 16 == 0, "an array is not aligned");
    const Plan p = make_plan(a, false);
    const Span in[3] = {span_of(a->d_x, p.N, a->ld_x, a->D, size),
                        span_of(a->d_w_gate, a->F, a->ld_gate, a->D, size),
                        span_of(a->d_w_up, a->F, a->ld_up, a->D, size)};
    const Span out[2] = {span_of(d_y, p.N, ld_y, a->F, size), span_of(d_work, p.bytes)};
    for (const Span &o : out)
        for (const Span &i : in) ECC_ARG(!spans_meet(o, i), "an output overlaps an input");
    ECC_ARG(!spans_meet(out[0], out[1]), "an output and the work buffer overlap");
    hipStream_t s = (hipStream_t)hip_stream;
    if (p.few) {
        with_kind(a, [&](auto t, auto act) {
            launch_few<decltype(t), decltype(act)::value>(a, d_y, ld_y, s);
        });
        ECC_LAUNCH_CHECK();
        return ECC_OK;
    }
    const GemmArgs g = projections(a, p, (char *)d_work, s);
    FfnParts parts{};
    const bool split = split_projections(g, p, (char *)d_work, parts, s);
    with_kind(a, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int ACT = decltype(act)::value;
        const FfnOut<T, ACT> out{(T *)d_y, ld_y};
        const int64_t quads = p.N * ((a->F + 3) / 4);
        if (split)
            hipLaunchKernelGGL((k_ffn_join<T, ACT>), dim3((unsigned)((quads + 255) / 256)),
                               dim3(256), 0, s, parts, out, quads);
        else launch_gemm(g, out, s);
    });
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

ecc_status_t ecc_ffn_grad(const ecc_ffn_t *a, const void *d_dy, int64_t ld_dy, void *d_dx,
                          int64_t ld_dx, void *d_dw_gate, void *d_dw_up, int64_t worker_stride,
                          int32_t accumulate, void *d_work, void *hip_stream) {
    clear_error();
    const ecc_status_t st = check(a);
    if (st != ECC_OK) return st;
    const int64_t D = a->D, F = a->F, size = type_size(a->type), gsize = type_size(a->grad_type);
    const int32_t P = a->P;
    ECC_ARG(ld_dy >= F, "a leading dimension is below F");
    ECC_ARG(!d_dx || ld_dx >= D, "a leading dimension is below D");
    ECC_ARG(!d_dw_gate == !d_dw_up, "the weights' gradients are formed together");
    ECC_ARG(!d_dw_gate || P == 1 || worker_stride >= F * D, "workers' gradients overlap");
    ECC_ARG(accumulate == 0 || accumulate == 1, "accumulate must be 0 or 1");
    if (ld_dy >= (int64_t(1) << 40) || ld_dx >= (int64_t(1) << 40) ||
        worker_stride >= (int64_t(1) << 56)) {
        set_error("a stride is too large");
        return ECC_ERR_RANGE;
    }
    ECC_ARG((uintptr_t)d_dy % size == 0 && (uintptr_t)d_dx % size == 0 &&
                (uintptr_t)d_dw_gate % gsize == 0 && (uintptr_t)d_dw_up % gsize == 0 &&
                (uintptr_t)d_work % 16 == 0,
            "an array is not aligned");
    hipStream_t s = (hipStream_t)hip_stream;
    const Span weights[2] = {
        P == 1 ? span_of(d_dw_gate, F * D * gsize) : span_of(d_dw_gate, P, worker_stride, F * D, gsize),
        P == 1 ? span_of(d_dw_up, F * D * gsize) : span_of(d_dw_up, P, worker_stride, F * D, gsize)};
    ECC_ARG(!spans_meet(weights[0], weights[1]), "two outputs overlap");
    if (a->n == 0) {
        if (d_dw_gate && !accumulate) {
            const int64_t rows = P * F;
            const dim3 grid((unsigned)std::min<int64_t>(rows, 4096));
            for (void *to : {d_dw_gate, d_dw_up}) {
                if (a->grad_type == ECC_F32)
                    hipLaunchKernelGGL(k_ffn_zero<float>, grid, dim3(256), 0, s, rows, F, D,
                                       (float *)to, worker_stride);
                else
                    hipLaunchKernelGGL(k_ffn_zero<bf16_t>, grid, dim3(256), 0, s, rows, F, D,
                                       (bf16_t *)to, worker_stride);
            }
            ECC_LAUNCH_CHECK();
        }
        return ECC_OK;
    }
    ECC_ARG(d_dy && d_work, "NULL pointer");
    const Plan p = make_plan(a, true);
    const Span in[4] = {span_of(a->d_x, p.N, a->ld_x, D, size),
                        span_of(a->d_w_gate, F, a->ld_gate, D, size),
                        span_of(a->d_w_up, F, a->ld_up, D, size),
                        span_of(d_dy, p.N, ld_dy, F, size)};
    const Span out[4] = {span_of(d_dx, p.N, ld_dx, D, size), weights[0], weights[1],
                         span_of(d_work, p.bytes)};
    for (int o = 0; o < 4; ++o) {
        for (const Span &i : in) ECC_ARG(!spans_meet(out[o], i), "an output overlaps an input");
        for (int q = 0; q < o; ++q)
            ECC_ARG(!spans_meet(out[o], out[q]),
                    "two outputs, or an output and the work buffer, overlap");
    }
    char *w = (char *)d_work;
    // dg and du
    const GemmArgs g = projections(a, p, w, s);
    bf16_t *d = (bf16_t *)(w + p.d);
    const int64_t plane = pad64(p.N) * 2 * p.Fp;
    FfnParts halves{};
    const bool split = split_projections(g, p, w, halves, s);
    with_kind(a, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int ACT = decltype(act)::value;
        const FfnGradOut<T, ACT> out{(const T *)d_dy, ld_dy, d, p.Fp, plane, p.pd};
        const int64_t quads = p.N * (p.Fp / 4);
        if (split)
            hipLaunchKernelGGL((k_ffn_grad_join<T, ACT>), dim3((unsigned)((quads + 255) / 256)),
                               dim3(256), 0, s, halves, out, quads);
        else launch_gemm(g, out, s);
    });
    // the other order of everything: [Wg | Wu] transposed, as long as [dg | du],
    // x and [dg | du] with workers padded to multiples of 64 rows
    Packing packing;
    Product products[2];
    GemmShape shapes[2];
    float *parts[2];
    int count = 0;
    if (d_dx) {
        PackArgs k{};
        k.cols = D;
        k.pieces = p.np;
        k.n = k.total = F;
        k.rows_packed = k.n_pad = p.Fp;
        k.ld_cols = 2 * p.Fp;
        k.plane_cols = D * 2 * p.Fp;
        for (int i = 0; i < 2; ++i) {
            k.src = i ? a->d_w_up : a->d_w_gate;
            k.ld = i ? a->ld_up : a->ld_gate;
            k.cols_out = (bf16_t *)(w + p.w_t) + i * p.Fp;
            packing.add(k);
        }
        GemmArgs x{};
        x.a = GemmOperand{d, 2 * p.Fp, plane};
        x.b = GemmOperand{(bf16_t *)(w + p.w_t), 2 * p.Fp, k.plane_cols};
        x.M = (int32_t)p.N;
        x.N = (int32_t)D;
        x.K = (int32_t)(2 * p.Fp);
        x.batches = 1;
        set_products(x, p.np, p.np);
        MatrixOut to{};
        to.out = d_dx;
        to.ld = ld_dx;
        to.type = a->type;
        products[count] = Product{x, to};
        shapes[count] = p.shape_x;
        parts[count++] = (float *)(w + p.parts[0]);
    }
    if (d_dw_gate) {
        PackArgs k{};
        k.n = a->n;
        k.n_pad = p.n_pad;
        k.total = p.N;
        k.rows_packed = k.ld_cols = p.rows;
        k.src = a->d_x;
        k.ld = a->ld_x;
        k.cols = D;
        k.pieces = p.np;
        k.cols_out = (bf16_t *)(w + p.x_t);
        k.plane_cols = D * p.rows;
        packing.add(k);
        k.ld = 2 * p.Fp;
        k.cols = F;
        k.pieces = 1;
        const int64_t plane_t = 2 * F * p.rows;
        Packing gradients;
        for (int which = 0; which < p.pd; ++which)
            for (int i = 0; i < 2; ++i) {
                k.src = d + which * plane + i * p.Fp;
                k.cols_out = (bf16_t *)(w + p.d_t) + which * plane_t + i * F * p.rows;
                gradients.add(k);
            }
        gradients.launch(ECC_BF16, s);
        GemmArgs x{};
        x.a = GemmOperand{(bf16_t *)(w + p.d_t), p.rows, plane_t};
        x.b = GemmOperand{(bf16_t *)(w + p.x_t), p.rows, D * p.rows};
        x.M = (int32_t)(2 * F);
        x.N = (int32_t)D;
        x.K = (int32_t)p.n_pad;
        x.batches = P;
        set_products(x, p.pd, p.np);
        MatrixOut to{};
        to.out = d_dw_gate;
        to.out2 = d_dw_up;
        to.second = (int32_t)F;
        to.ld = D;
        to.batch_stride = worker_stride;
        to.type = a->grad_type;
        to.add = accumulate;
        products[count] = Product{x, to};
        shapes[count] = p.shape_w;
        parts[count++] = (float *)(w + p.parts[1]);
    }
    packing.launch(a->type, s);
    launch_products(products, count, shapes, parts, s);
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
