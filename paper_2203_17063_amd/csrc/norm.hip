// The joint between two blocks of a residual network, forward and backward:
//   u = rms(f) (o + w_post),  x' = a x + b g u,  h = rms(x') (o + w_pre)
// (see libecc.h for what may be absent).  Bound by memory: forward reads x, f
// and the gate and writes x' and h; backward reads x', f, the gate and the
// gradients of x' and h and writes those of x, f and the gate.
//
// A workgroup holds a row in registers: it reads every operand of the row
// once and writes every result once, and the weights are read once per
// workgroup, which walks several rows.  The workgroup is as wide as makes a
// thread hold 16 elements of the row (backward 8, for its registers); of rows
// that 8, 16 or 32 lanes hold, a wave takes 8, 4 or 2 at a time.
//
// Forward has two sums per row, that of f^2 and then that of x'^2 (formed
// from the squares themselves: as a combination of sums over x and f they
// could cancel).  Backward takes one round for all of its sums.  With
//   q = 1/sqrt(mean x'^2 + eps),  k = 1/sqrt(mean f^2 + eps),
//   A = dh (o + w_pre),  C = b g (o + w_post) f:
//   dX = dx' + q A - c x',                 c = q^3 mean(A x')
//   df = k (C/f dX - f k^2 mean(C dX)),    sum C dX = sum C dx' + q sum C A - c sum C x'
// so sum x'^2, f^2, A x', C dx', C A and C x' are formed together, and no
// statistics are kept from the forward call.
//
// The sums over rows (gradients of the weights and of a shared gate) stay in
// registers while a workgroup walks its unit of consecutive rows; the units'
// sums go to the work buffer and a second launch adds them in order.  They are
// held in fp64 where the rows or the parameters' gradients are fp64.
#include <algorithm>

#include "lm_common.h"

namespace ecc {

constexpr int kNormCus = 256;

struct NormArgs {
    int64_t N, D;
    const void *x, *f, *gate, *w_post, *w_pre;
    int64_t ld_x, ld_f, ld_gate;
    int64_t gate_rows;  // rows that share a gate row; 0: a parameter
    int32_t w_type;
    double offset, res, branch, eps;
};

template <typename A>
__device__ __forceinline__ void store_param(void *p, int32_t type, int64_t i, A v, int accumulate) {
    if (type == ECC_F64) {
        double *q = reinterpret_cast<double *>(p) + i;
        *q = accumulate ? *q + (double)v : (double)v;
    } else if (type == ECC_F32) {
        float *q = reinterpret_cast<float *>(p) + i;
        *q = accumulate ? (float)((A)*q + v) : (float)v;
    } else {
        bf16_t *q = reinterpret_cast<bf16_t *>(p) + i;
        store_elem<A>(q, accumulate ? load_elem<A>(q) + v : v);
    }
}

__device__ __forceinline__ float fma_(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fma_(double a, double b, double c) { return __builtin_fma(a, b, c); }
__device__ __forceinline__ float rsqrt_(float v) { return 1.0f / __builtin_sqrtf(v); }
__device__ __forceinline__ double rsqrt_(double v) { return 1.0 / __builtin_sqrt(v); }

// The sum over the 16 lanes of a DPP row, and a lane's value in all lanes.
__device__ __forceinline__ float row_add(float v) {
    v += dpp_f32<kDppQuadXor1>(v);
    v += dpp_f32<kDppQuadXor2>(v);
    v += dpp_f32<kDppRowHalfMirror>(v);
    return v + dpp_f32<kDppRowMirror>(v);
}
__device__ __forceinline__ double row_add(double v) { return group_sum<16>(v); }
__device__ __forceinline__ float read_lane(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ double read_lane(double v, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                            __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// The sum over every N = 8, 16 or 32 neighbouring lanes, in all of them.
template <int N, typename A>
__device__ __forceinline__ A lanes_sum(A v) {
    if constexpr (std::is_same_v<A, float>) {
        v += dpp_f32<kDppQuadXor1>(v);
        v += dpp_f32<kDppQuadXor2>(v);
        v += dpp_f32<kDppRowHalfMirror>(v);
        if constexpr (N >= 16) v += dpp_f32<kDppRowMirror>(v);
        if constexpr (N >= 32) v += __shfl_xor(v, 16, 64);
        return v;
    } else {
        return group_sum<N>(v);
    }
}

// K sums over the workgroup's NT threads, in every thread.  s holds [2][NT /
// 64][K]; the two halves are used in turn, so that one barrier is enough:
// a half is written again only after every wave has passed the barrier of
// the other, and so has read this one.
// With LANES < 64 (NT = 64) the sums are those of every LANES neighbours.
template <int NT, int LANES, int K, typename A>
__device__ __forceinline__ void row_sums(A (&v)[K], A *s, int &half) {
    if constexpr (LANES < 64) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = lanes_sum<LANES>(v[k]);
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_all(v[k], OpSum{});
    if constexpr (NT > 64) {
        constexpr int NW = NT / 64;
        A *b = s + half * NW * K;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) b[(threadIdx.x >> 6) * K + k] = v[k];
        }
        lds_barrier();
        half ^= 1;
        if constexpr (K * NW <= 16) {
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = b[k];
#pragma unroll
            for (int w = 1; w < NW; ++w)
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] += b[w * K + k];
            return;
        }
        // every wave joins the waves' sums for itself: lane 16 r + w takes wave
        // w's sums r and r + 4, a row of 16 lanes adds them up
        const int lane = threadIdx.x & 63, w = lane & 15, r = lane >> 4;
        static_assert(NW <= 16 && K <= 8, "a lane for every wave, two sums in a lane");
        A lo = w < NW && r < K ? b[w * K + r] : (A)0, hi = (A)0;
        if constexpr (K > 4) hi = w < NW && r + 4 < K ? b[w * K + r + 4] : (A)0;
        lo = row_add(lo);
        if constexpr (K > 4) hi = row_add(hi);
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = read_lane(k < 4 ? lo : hi, 16 * (k & 3));
    }
}

template <typename T, int NT, int NV, int LANES>
__global__ __launch_bounds__(NT) void k_norm_forward(NormArgs a, void *x_out, int64_t ld_x_out,
                                                     void *h_out, int64_t ld_h) {
    using A = Acc<T>;
    constexpr int VEC = kVec<T>, E = NV * VEC;
    __shared__ A s_red[2 * (NT / 64)];
    int half = 0;
    // the rows of a pass, this thread's among them, its place in it
    constexpr int AT_ONCE = NT / LANES;
    const int sub = AT_ONCE == 1 ? 0 : threadIdx.x / LANES;
    const uint32_t tid = AT_ONCE == 1 ? threadIdx.x : threadIdx.x % LANES;
    const A res = (A)a.res, branch = (A)a.branch, eps = (A)a.eps, inv_d = (A)1 / (A)a.D;
    A wq[E], wp[E];  // branch scale, parameter gate and post-norm weight; pre-norm weight
    // (all their loads under way at once: 8,192 rows of 1,001 fp32 23.7 us,
    // element by element 34.7 us)
    auto load_weights = [&](auto type) {
        using W = decltype(type);
        const bool gate = a.gate && a.gate_rows == 0;
        Raw<W, VEC> post[NV], gates[NV], pre[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const uint32_t c = (v * NT + tid) * VEC;
            const int32_t n = (int32_t)a.D - (int32_t)c;
            if (a.w_post) post[v].load_upto(reinterpret_cast<const W *>(a.w_post) + c, n);
            if (gate) gates[v].load_upto(reinterpret_cast<const W *>(a.gate) + c, n);
            if (a.w_pre) pre[v].load_upto(reinterpret_cast<const W *>(a.w_pre) + c, n);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const bool in = (v * NT + tid) * VEC + i < a.D;
                A q = branch, p = (A)0;
                if (a.w_post) q *= (A)a.offset + post[v].template get<A>(i);
                if (gate) q *= gates[v].template get<A>(i);
                if (a.w_pre) p = (A)a.offset + pre[v].template get<A>(i);
                wq[v * VEC + i] = in ? q : branch;
                wp[v * VEC + i] = in ? p : (A)0;
            }
    };
    if constexpr (std::is_same_v<T, double>) {
        if (a.w_type == ECC_F64) load_weights(double{});
    }
    if (a.w_type == ECC_F32) load_weights(float{});
    if (a.w_type == ECC_BF16) load_weights(bf16_t{});
    for (int64_t first = (int64_t)blockIdx.x * AT_ONCE; first < a.N;
         first += (int64_t)gridDim.x * AT_ONCE) {
        // (lanes past the last row go along with it and write nothing)
        const bool live = AT_ONCE == 1 || first + sub < a.N;
        const int64_t row = live ? first + sub : a.N - 1;
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.ld_x;
        const T *f = reinterpret_cast<const T *>(a.f) + row * a.ld_f;
        const bool row_gate = a.gate && a.gate_rows > 0;
        const T *g = reinterpret_cast<const T *>(a.gate) +
                     (row_gate ? row / a.gate_rows * a.ld_gate : 0);
        Raw<T, VEC> rx[NV], rf[NV], rg[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const uint32_t c = (v * NT + tid) * VEC;
            rx[v].load_upto(x + c, (int32_t)a.D - (int32_t)c);
            if (a.f) rf[v].load_upto(f + c, (int32_t)a.D - (int32_t)c);
            if (row_gate) rg[v].load_upto(g + c, (int32_t)a.D - (int32_t)c);
        }
        A y[E];
        A k = (A)1;
        if (a.f && a.w_post) {
            A sum[1] = {(A)0};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const A t = rf[e / VEC].template get<A>(e % VEC);
                sum[0] = fma_(t, t, sum[0]);
            }
            row_sums<NT, LANES>(sum, s_red, half);
            k = rsqrt_(fma_(sum[0], inv_d, eps));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            y[e] = res * rx[e / VEC].template get<A>(e % VEC);
            if (a.f) {
                A u = k * rf[e / VEC].template get<A>(e % VEC) * wq[e];
                if (row_gate) u *= rg[e / VEC].template get<A>(e % VEC);
                y[e] += u;
            }
        }
        if (x_out) {
            T *o = reinterpret_cast<T *>(x_out) + row * ld_x_out;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const uint32_t c = (v * NT + tid) * VEC;
                A t[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) t[i] = y[v * VEC + i];
                Raw<T, VEC> r;
                r.set_all(t);
                if (live) r.store_upto(o + c, (int32_t)a.D - (int32_t)c);
            }
        }
        if (h_out) {
            A sum[1] = {(A)0};
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] = fma_(y[e], y[e], sum[0]);
            row_sums<NT, LANES>(sum, s_red, half);
            const A q = rsqrt_(fma_(sum[0], inv_d, eps));
            T *o = reinterpret_cast<T *>(h_out) + row * ld_h;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const uint32_t c = (v * NT + tid) * VEC;
                A t[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) t[i] = y[v * VEC + i] * q * wp[v * VEC + i];
                Raw<T, VEC> r;
                r.set_all(t);
                if (live) r.store_upto(o + c, (int32_t)a.D - (int32_t)c);
            }
        }
    }
}

// How the rows are shared out in backward.  A group is the rows of a worker
// that share a gate row (all of a worker's rows where the gate is no row
// gate).  Units are `rows` consecutive rows: several whole groups where a
// group is shorter (split = 0), a part of one otherwise.
struct NormUnits {
    int64_t n, group, rows, per_worker, per_group, total;
    int32_t split;
};
inline NormUnits norm_units(int64_t P, int64_t n, int64_t group, int64_t target) {
    NormUnits u{};
    u.n = n;
    u.group = std::max<int64_t>(1, std::min(group, n));
    const int64_t want = std::max<int64_t>(1, (P * n + target - 1) / target);
    if (want >= u.group) {
        u.rows = want / u.group * u.group;
        u.per_group = 1;
        u.per_worker = (n + u.rows - 1) / u.rows;
        u.split = 0;
    } else {
        u.per_group = (u.group + want - 1) / want;
        u.rows = (u.group + u.per_group - 1) / u.per_group;
        u.per_group = (u.group + u.rows - 1) / u.rows;
        u.per_worker = (n + u.group - 1) / u.group * u.per_group;
        u.split = 1;
    }
    u.total = P * u.per_worker;
    return u;
}

struct NormGradArgs {
    const void *dh, *dxo;
    int64_t ld_dh, ld_dxo;
    void *dx, *df, *dgate;
    int64_t ld_dx, ld_df, ld_dgate;
    void *pre, *post, *share;  // [units][D] sums of a unit: dw_pre, dw_post, dgate (or NULL)
    NormUnits u;
};

// Vectors (16 bytes) a thread of the backward kernel holds of an operand's row.
template <typename T>
constexpr int kBackwardVecs = std::is_same_v<T, bf16_t> ? 1 : 2;

// HOLD: the row's operands stay in registers between the sums and the results,
// and the weights lie in LDS, each where the thread that needs it has put it
// (in registers, 173 of them for a row of 4,096 bf16, one workgroup filled a
// CU: 129 us for 8,192 such rows, 95 us with two).  Otherwise (the longest
// rows) both are read again, and the sums over rows stay in the work buffer.
// S: the type of the sums over rows, fp64 where the parameters' gradients are
// (8,192 rows of 4,096 bf16: 120 us, with sums in fp32 97 us; 8,192 rows of
// 8,192: 193 and 172 us; 2,000 rows of 16,000, whose sums go through memory: 425
// and 210 us).
template <typename T, typename S, int NT, int NV, bool HOLD>
constexpr int kGradWaves = HOLD && NV > kBackwardVecs<T> ? 2
                           : NT == 64 || (HOLD && sizeof(S) == 8) ? 3 : 4;
template <typename T, typename S, int NT, int NV, bool HOLD, int LANES>
__global__ __launch_bounds__(NT, (kGradWaves<T, S, NT, NV, HOLD>)) void k_norm_grad(
    NormArgs a, NormGradArgs g) {
    using A = Acc<T>;
    constexpr int VEC = kVec<T>, KEEP = HOLD ? NV : 1;
    constexpr int Q = 16 / (int)sizeof(A), CH = VEC / Q;  // accumulators of 16 bytes
    typedef A quad __attribute__((ext_vector_type(Q)));
    extern __shared__ double s_weights[];  // [3][NV * CH][NT] quads
    __shared__ A s_red[2 * (NT / 64) * 6];
    int half = 0;
    // rows at a time (several only where no gate row is shared by a few)
    constexpr int AT_ONCE = NT / LANES;
    const int sub = AT_ONCE == 1 ? 0 : threadIdx.x / LANES;
    const uint32_t tid = AT_ONCE == 1 ? threadIdx.x : threadIdx.x % LANES;
    const A res = (A)a.res, branch = (A)a.branch, eps = (A)a.eps, inv_d = (A)1 / (A)a.D;
    const bool post = a.f && a.w_post, pre = a.w_pre != nullptr;
    const bool row_gate = a.f && a.gate && a.gate_rows > 0;
    const bool param_gate = a.f && a.gate && a.gate_rows == 0;
    // the unit's rows
    const NormUnits &u = g.u;
    const int64_t worker = blockIdx.x / u.per_worker, part = blockIdx.x % u.per_worker;
    int64_t r0, r1;
    if (u.split) {
        const int64_t group = part / u.per_group;
        r0 = group * u.group + part % u.per_group * u.rows;
        r1 = min(min(r0 + u.rows, (group + 1) * u.group), u.n);
    } else {
        r0 = part * u.rows;
        r1 = min(r0 + u.rows, u.n);
    }
    r0 += worker * u.n;
    r1 += worker * u.n;
    // quad c of vector v's columns of the post-norm weight (0), the pre-norm
    // weight (1) and b times a parameter gate (2)
    // (read as vectors: 2,000 rows of 16,000 bf16, that read them with each row, 204
    // us, element by element 266; 8,192 rows of 4,096, weights in LDS, 103 and 109)
    auto read_weights = [&](int which, int v, int c, A(&w)[Q]) {
        const uint32_t col = (v * NT + tid) * VEC + c * Q;
        const int32_t n = (int32_t)a.D - (int32_t)col;
        const bool there = which == 0 ? post : which == 1 ? pre : param_gate;
        const void *from = which == 0 ? a.w_post : which == 1 ? a.w_pre : a.gate;
        auto read = [&](auto type) {
            using W = decltype(type);
            Raw<W, Q> r;
            r.load_upto(reinterpret_cast<const W *>(from) + col, n);
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const A t = r.template get<A>(i);
                if (i < n) w[i] = which == 2 ? branch * t : (A)a.offset + t;
            }
        };
#pragma unroll
        for (int i = 0; i < Q; ++i) w[i] = which == 0 ? (A)1 : which == 1 ? (A)0 : branch;
        if (!there) return;
        if constexpr (std::is_same_v<T, double>) {
            if (a.w_type == ECC_F64) read(double{});
        }
        if (a.w_type == ECC_F32) read(float{});
        if (a.w_type == ECC_BF16) read(bf16_t{});
    };
    quad *const lds = reinterpret_cast<quad *>(s_weights) + threadIdx.x;
    auto weights = [&](int which, int v, int c, A(&w)[Q]) {
        if constexpr (HOLD) {
            const quad t = lds[((which * NV + v) * CH + c) * NT];
#pragma unroll
            for (int i = 0; i < Q; ++i) w[i] = t[i];
        } else {
            read_weights(which, v, c, w);
        }
    };
    if constexpr (HOLD) {
#pragma unroll
        for (int which = 0; which < 3; ++which)
#pragma unroll
            for (int vc = 0; vc < NV * CH; ++vc) {
                A w[Q];
                read_weights(which, vc / CH, vc % CH, w);
                quad t;
#pragma unroll
                for (int i = 0; i < Q; ++i) t[i] = w[i];
                lds[(which * NV * CH + vc) * NT] = t;
            }
    }
    struct Operands {
        Raw<T, VEC> x, f, gate, dh, dxo;
    };
    auto fetch = [&](int64_t row, int v, Operands &o) {
        const uint32_t c = (v * NT + tid) * VEC;
        const int32_t left = AT_ONCE == 1 || row < r1 ? (int32_t)a.D - (int32_t)c : 0;
#pragma unroll
        for (int i = 0; i < Raw<T, VEC>::kWords; ++i)
            o.x.w[i] = o.f.w[i] = o.gate.w[i] = o.dh.w[i] = o.dxo.w[i] = 0;
        if (pre) {
            o.x.load_upto(reinterpret_cast<const T *>(a.x) + row * a.ld_x + c, left);
            o.dh.load_upto(reinterpret_cast<const T *>(g.dh) + row * g.ld_dh + c, left);
        }
        if (g.dxo)
            o.dxo.load_upto(reinterpret_cast<const T *>(g.dxo) + row * g.ld_dxo + c, left);
        if (a.f) o.f.load_upto(reinterpret_cast<const T *>(a.f) + row * a.ld_f + c, left);
        if (row_gate)
            o.gate.load_upto(reinterpret_cast<const T *>(a.gate) + row / a.gate_rows * a.ld_gate + c,
                             left);
    };
    // the sums over rows, in registers for all of the thread's columns, or for
    // PER of them in turn (a vector's, unless fp64 sums make that too many
    // registers), kept in the work buffer from row to row (from the unit's or
    // the gate's first row on)
    const int64_t at = (int64_t)blockIdx.x * a.D;
    constexpr int PER = HOLD || std::is_same_v<S, A> ? VEC : Q, SUMS = HOLD ? NV * VEC : PER;
    S s_pre[SUMS], s_post[SUMS], s_gate[SUMS];
#pragma unroll
    for (int e = 0; e < SUMS; ++e) s_pre[e] = s_post[e] = s_gate[e] = (S)0;
    auto get = [&](const void *from, uint32_t c, bool first, S(&sum)[SUMS]) {
        Raw<S, SUMS> r;
        if (from && !first)
            r.load_upto(reinterpret_cast<const S *>(from) + at + c, (int32_t)a.D - (int32_t)c);
#pragma unroll
        for (int i = 0; i < SUMS; ++i) sum[i] = from && !first ? r.template get<S>(i) : (S)0;
    };
    auto put = [&](void *to, uint32_t c, const S *sum) {
        if (!to) return;
        S t[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) t[i] = sum[i];
        Raw<S, PER> r;
        r.set_all(t);
        r.store_upto(reinterpret_cast<S *>(to) + at + c, (int32_t)a.D - (int32_t)c);
    };
    constexpr int UNROLL = HOLD ? NV : 1;
    Operands op[KEEP];
    for (int64_t first = r0; first < r1; first += AT_ONCE) {
        const int64_t row = first + sub;
        const bool live = AT_ONCE == 1 || row < r1;
        if constexpr (HOLD)
#pragma unroll
            for (int v = 0; v < NV; ++v) fetch(row, v, op[v]);
        // sums of x^2, f^2, A x, C dx', C A, C x
        A s[6] = {(A)0, (A)0, (A)0, (A)0, (A)0, (A)0};
#pragma unroll UNROLL
        for (int v = 0; v < NV; ++v) {
            if constexpr (!HOLD) fetch(row, v, op[0]);
            const Operands &o = op[HOLD ? v : 0];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                A wq[Q], wp[Q], wg[Q];
                weights(0, v, c, wq);
                weights(1, v, c, wp);
                weights(2, v, c, wg);
#pragma unroll
                for (int j = 0; j < Q; ++j) {
                    const int i = c * Q + j;
                    const A x = o.x.template get<A>(i), f = o.f.template get<A>(i);
                    const A d = o.dxo.template get<A>(i);
                    const A ah = o.dh.template get<A>(i) * wp[j];
                    A b = wg[j] * wq[j] * f;
                    if (row_gate) b *= o.gate.template get<A>(i);
                    s[0] = fma_(x, x, s[0]);
                    s[1] = fma_(f, f, s[1]);
                    s[2] = fma_(ah, x, s[2]);
                    s[3] = fma_(b, d, s[3]);
                    s[4] = fma_(b, ah, s[4]);
                    s[5] = fma_(b, x, s[5]);
                }
                __builtin_amdgcn_sched_barrier(0);  // a quad's weights at a time
            }
        }
        row_sums<NT, LANES>(s, s_red, half);
        const A q = pre ? rsqrt_(fma_(s[0], inv_d, eps)) : (A)0;
        const A k = post ? rsqrt_(fma_(s[1], inv_d, eps)) : (A)1;
        // (the sums first: the cube of a norm factor alone may pass the type's range)
        const A c = s[2] * inv_d * q * q * q;
        const A m = post ? (s[3] + q * s[4] - c * s[5]) * inv_d * k * k : (A)0;
        const bool group_end = row_gate && !u.split &&
                               ((row + 1) % a.gate_rows == 0 || row + 1 == r1);
        const bool group_begin = row == r0 || (row_gate && !u.split && row % a.gate_rows == 0);
#pragma unroll UNROLL
        for (int v = 0; v < NV; ++v) {
            const uint32_t col = (v * NT + tid) * VEC;
            const int32_t left = live ? (int32_t)a.D - (int32_t)col : 0;
            if constexpr (!HOLD) fetch(row, v, op[0]);
            const Operands &o = op[HOLD ? v : 0];
            Raw<T, VEC> rdx, rdf, rdg;
#pragma unroll
            for (int cq = 0; cq < CH; ++cq) {
                A wq[Q], wp[Q], wg[Q], dx[Q], df[Q];
                S dg[Q];
                if (!HOLD && cq * Q % PER == 0) {
                    get(g.pre, col + cq * Q, row == r0, s_pre);
                    get(g.post, col + cq * Q, row == r0, s_post);
                    get(g.share, col + cq * Q, group_begin, s_gate);
                }
                weights(0, v, cq, wq);
                weights(1, v, cq, wp);
                weights(2, v, cq, wg);
#pragma unroll
                for (int j = 0; j < Q; ++j) {
                    const int i = cq * Q + j, e = HOLD ? v * VEC + i : i % PER;
                    const A x = o.x.template get<A>(i), f = o.f.template get<A>(i);
                    const A h = o.dh.template get<A>(i);
                    const A d = o.dxo.template get<A>(i) + q * (h * wp[j]) - c * x;
                    A gb = wg[j];  // b g
                    if (row_gate) gb *= o.gate.template get<A>(i);
                    const A du = gb * d;
                    dx[j] = res * d;
                    df[j] = k * (du * wq[j] - f * m);
                    s_pre[e] = fma_((S)h, (S)(x * q), s_pre[e]);
                    s_post[e] = fma_((S)du, (S)(f * k), s_post[e]);
                    s_gate[e] = fma_((S)(branch * d), (S)(f * k * wq[j]), s_gate[e]);
                    dg[j] = s_gate[e];
                    if (group_end) s_gate[e] = (S)0;
                }
                rdx.template set_some<Q>(cq * Q, dx);
                rdf.template set_some<Q>(cq * Q, df);
                rdg.template set_some<Q>(cq * Q, dg);
                if (!HOLD && (cq + 1) * Q % PER == 0) {
                    const uint32_t first_col = col + (cq + 1) * Q - PER;
                    put(g.pre, first_col, s_pre);
                    put(g.post, first_col, s_post);
                    put(g.share, first_col, s_gate);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (g.dx)
                rdx.store_upto(reinterpret_cast<T *>(g.dx) + row * g.ld_dx + col, left);
            if (g.df)
                rdf.store_upto(reinterpret_cast<T *>(g.df) + row * g.ld_df + col, left);
            if (g.dgate && group_end)
                rdg.store_upto(
                    reinterpret_cast<T *>(g.dgate) + row / a.gate_rows * g.ld_dgate + col, left);
        }
    }
    if constexpr (!HOLD) {
        // (a short last group has units without rows: their sums are zero)
        if (r0 >= r1)
            for (int i = 0; i < NV * VEC / PER; ++i) {
                const uint32_t c = (i * PER / VEC * NT + tid) * VEC + i * PER % VEC;
                put(g.pre, c, s_pre);
                put(g.post, c, s_post);
                put(g.share, c, s_gate);
            }
    }
    if constexpr (AT_ONCE > 1) {
        // the wave's rows together
#pragma unroll
        for (int e = 0; e < SUMS; ++e)
#pragma unroll
            for (int o = LANES; o < 64; o <<= 1) {
                s_pre[e] += __shfl_xor(s_pre[e], o, 64);
                s_post[e] += __shfl_xor(s_post[e], o, 64);
                s_gate[e] += __shfl_xor(s_gate[e], o, 64);
            }
        if (sub > 0) return;
    }
    if constexpr (HOLD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const uint32_t c = (v * NT + tid) * VEC;
            put(g.pre, c, s_pre + v * VEC);
            put(g.post, c, s_post + v * VEC);
            put(g.share, c, s_gate + v * VEC);
        }
    }
}

// Sums of consecutive units: result j (of `count`) adds units [j per, (j + 1)
// per) of up to three arrays of [units][D] sums.  A workgroup takes COLS
// columns of a result: 64, 16 where that would leave under 64 workgroups
// (28,651 rows of 85 fp64: 60.5 us with 64, 40.9 with 16).  Its groups of COLS
// lanes take every SLOTS-th unit each, and their sums are added in order.
struct NormJoin {
    const void *from[3];
    void *to[3];
    int64_t ld[3];        // elements from one result to the next
    int32_t type[3];
    int32_t accumulate;
    int64_t per, count, D;
};
constexpr int kNormJoinThreads = 1024;

template <typename A, int COLS>
__global__ __launch_bounds__(kNormJoinThreads) void k_norm_join(NormJoin a) {
    constexpr int SLOTS = kNormJoinThreads / COLS, U = 8;
    __shared__ A s_part[SLOTS][COLS];
    const int lane = threadIdx.x % COLS, slot = threadIdx.x / COLS;
    const int64_t cols = (a.D + COLS - 1) / COLS;
    const int64_t j = blockIdx.x / cols, c = blockIdx.x % cols * COLS + lane;
    const int z = blockIdx.y;
    const A *from = reinterpret_cast<const A *>(z == 0 ? a.from[0] : z == 1 ? a.from[1]
                                                                           : a.from[2]);
    void *to = z == 0 ? a.to[0] : z == 1 ? a.to[1] : a.to[2];
    const int64_t ld = z == 0 ? a.ld[0] : z == 1 ? a.ld[1] : a.ld[2];
    const int32_t type = z == 0 ? a.type[0] : z == 1 ? a.type[1] : a.type[2];
    if (!to) return;
    A sum = (A)0;
    for (int64_t i = slot; i < a.per; i += SLOTS * U) {
        A t[U];
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int64_t at = i + s * SLOTS;
            t[s] = at < a.per && c < a.D ? from[(j * a.per + at) * a.D + c] : (A)0;
        }
#pragma unroll
        for (int s = 0; s < U; ++s) sum += t[s];
    }
    s_part[slot][lane] = sum;
    __syncthreads();
    if (slot == 0 && c < a.D) {
        for (int w = 1; w < SLOTS; ++w) sum += s_part[w][lane];
        store_param<A>(to, type, j * ld + c, sum, a.accumulate);
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

// Calls f with the thread count and vectors per thread that hold a row: the
// narrowest workgroup whose threads hold up to FULL vectors each, beyond 1,024
// threads (WIDER) twice as many, or beyond 512 (DEEP); where `several` rows may
// share a wave, as few lanes as hold a row (308,420 rows of 106 bf16: 199 us
// backward, 348 us with a wave to a row).
template <int NT, int NV, int LANES = NT>
struct RowShape {
    static constexpr int nt = NT, nv = NV, lanes = LANES;
};
template <int FULL, bool WIDER, bool DEEP, typename F>
void with_row_shape(int64_t vecs, bool several, F &&f) {
    if (several && vecs <= 8) f(RowShape<64, 1, 8>{});
    else if (several && vecs <= 16) f(RowShape<64, 1, 16>{});
    else if (several && vecs <= 32) f(RowShape<64, 1, 32>{});
    else if (FULL > 1 && vecs <= 64 * (FULL / 2)) f(RowShape<64, (FULL > 1 ? FULL / 2 : 1)>{});
    else if (vecs <= 64 * FULL) f(RowShape<64, FULL>{});
    else if (vecs <= 128 * FULL) f(RowShape<128, FULL>{});
    else if (vecs <= 256 * FULL) f(RowShape<256, FULL>{});
    else if (vecs <= 512 * FULL) f(RowShape<512, FULL>{});
    else if (!WIDER || vecs <= 1024 * FULL) f(RowShape<DEEP ? 512 : 1024, DEEP ? 2 * FULL : FULL>{});
    else f(RowShape<1024, (WIDER ? 2 : 1) * FULL>{});
}
// Vectors (16 bytes) a thread holds of an operand's row.
template <typename T>
constexpr int kForwardVecs = std::is_same_v<T, bf16_t> ? 2 : 4;
static_assert(1024 * kForwardVecs<bf16_t> * kVec<bf16_t> == ECC_NORM_MAX_DIM &&
                  1024 * kForwardVecs<float> * kVec<float> == ECC_NORM_MAX_DIM &&
                  1024 * kForwardVecs<double> * kVec<double> == ECC_NORM_MAX_DIM / 2,
              "the widest workgroup holds the longest row");
// fp64 sums over narrower rows: too many registers for 1,024 threads, so 512
// hold twice as many vectors (8,192 rows of 8,192 bf16: 192 us, with 1,024
// threads and the sums in memory 747 us).
template <typename T, typename S>
constexpr bool kDeep = sizeof(S) == 8 && !std::is_same_v<T, double>;

inline int64_t backward_threads(int32_t type, int64_t D) {
    const int64_t vec = 16 / type_size(type), full = type == ECC_BF16 ? 1 : 2;
    const int64_t vecs = (D + vec - 1) / vec;
    int64_t nt = 64;
    while (nt < 1024 && vecs > nt * full) nt *= 2;
    return nt;
}
// A CU holds 1,024 threads of the backward kernel: one unit for each workgroup.
inline NormUnits units_of(const ecc_norm_t *a) {
    const int64_t target = kNormCus * 1024 / backward_threads(a->type, a->D);
    const int64_t group = a->d_f && a->d_gate && a->gate_rows > 0 ? a->gate_rows : a->n;
    return norm_units(a->P, a->n, group, target);
}

// eps in the rows' arithmetic: one that fp32 would round to zero is its least
// number, so that rows of zeros stay zeros.
inline double held_eps(const ecc_norm_t *a) {
    return a->type == ECC_F64 ? a->eps : std::max(a->eps, 0x1p-149);
}

static ecc_status_t check_norm(const ecc_norm_t *a) {
    ECC_ARG(a != nullptr, "the description is NULL");
    ECC_ARG(a->P >= 1 && a->n >= 0 && a->D >= 1, "P and D must be >= 1, n >= 0");
    ECC_ARG(known_type(a->type) && known_type(a->w_type), "unknown element type");
    ECC_ARG(a->eps > 0.0, "eps must be positive");
    ECC_ARG(a->gate_rows >= 0, "gate_rows must be >= 0");
    const int64_t most = a->type == ECC_F64 ? ECC_NORM_MAX_DIM / 2 : ECC_NORM_MAX_DIM;
    const int64_t lim = int64_t(1) << 40;
    if (a->D > most || a->n >= lim || (a->n > 0 && a->P >= lim / a->n) || a->ld_x >= lim ||
        a->ld_f >= lim || a->ld_gate >= lim) {
        set_error("D = %lld exceeds %lld, or another size is too large", (long long)a->D,
                  (long long)most);
        return ECC_ERR_RANGE;
    }
    ECC_ARG(a->w_type != ECC_F64 || a->type == ECC_F64,
            "fp64 weights go with fp64 rows only");
    // (the arrays of no rows may be NULL)
    ECC_ARG(a->n == 0 || a->d_f || (!a->d_gate && !a->d_w_post), "a gate or a post-norm weight without f");
    ECC_ARG(a->ld_x >= a->D && (!a->d_f || a->ld_f >= a->D), "a leading dimension is below D");
    const int64_t tb = type_size(a->type), wb = type_size(a->w_type);
    ECC_ARG(((uintptr_t)a->d_x | (uintptr_t)a->d_f) % tb == 0 &&
                ((uintptr_t)a->d_w_post | (uintptr_t)a->d_w_pre) % wb == 0,
            "an array is not aligned to its elements");
    if (a->d_gate) {
        ECC_ARG((uintptr_t)a->d_gate % (a->gate_rows ? tb : wb) == 0,
                "an array is not aligned to its elements");
        if (a->gate_rows) {
            ECC_ARG(a->ld_gate >= a->D, "a leading dimension is below D");
            ECC_ARG(a->P == 1 || a->n % a->gate_rows == 0,
                    "a gate row would be shared by two workers");
        }
    }
    return ECC_OK;
}

// Does an output meet the gate or a weight?
static bool meets_input(const ecc_norm_t *a, const Span &o) {
    const int64_t rows = a->P * a->n, tb = type_size(a->type), wb = type_size(a->w_type);
    const Span gate = a->gate_rows ? span_of(a->d_gate, (rows + a->gate_rows - 1) / a->gate_rows,
                                             a->ld_gate, a->D, tb)
                                   : span_of(a->d_gate, a->D * wb);
    return spans_meet(o, gate) || spans_meet(o, span_of(a->d_w_post, a->D * wb)) ||
           spans_meet(o, span_of(a->d_w_pre, a->D * wb));
}

}  // namespace ecc

using namespace ecc;

extern "C" {

ecc_status_t ecc_norm_forward(const ecc_norm_t *a, void *d_x_out, int64_t ld_x_out, void *d_h,
                              int64_t ld_h, void *hip_stream) {
    clear_error();
    const ecc_status_t st = check_norm(a);
    if (st != ECC_OK) return st;
    ECC_ARG(a->n == 0 || (d_h != nullptr) == (a->d_w_pre != nullptr), "d_h goes with d_w_pre");
    ECC_ARG(a->n == 0 || d_x_out || d_h, "no output");
    const int64_t lim = int64_t(1) << 40, tb = type_size(a->type), N = a->P * a->n;
    ECC_ARG((!d_x_out || ld_x_out >= a->D) && (!d_h || ld_h >= a->D),
            "a leading dimension is below D");
    if (ld_x_out >= lim || ld_h >= lim) {
        set_error("a leading dimension is too large");
        return ECC_ERR_RANGE;
    }
    if (N == 0) return ECC_OK;
    ECC_ARG(a->d_x, "NULL pointer");
    ECC_ARG(((uintptr_t)d_x_out | (uintptr_t)d_h) % tb == 0,
            "an array is not aligned to its elements");
    const Span x = span_of(a->d_x, N, a->ld_x, a->D, tb), f = span_of(a->d_f, N, a->ld_f, a->D, tb),
               xo = span_of(d_x_out, N, ld_x_out, a->D, tb), h = span_of(d_h, N, ld_h, a->D, tb);
    const bool xo_is_x = d_x_out == a->d_x && ld_x_out == a->ld_x;
    const bool h_is_f = d_h == a->d_f && ld_h == a->ld_f;
    const bool h_is_x = d_h == a->d_x && ld_h == a->ld_x;
    ECC_ARG((!spans_meet(xo, x) || xo_is_x) && !spans_meet(xo, f) &&
                (!spans_meet(h, f) || h_is_f) && (!spans_meet(h, x) || h_is_x) &&
                !spans_meet(xo, h) && !meets_input(a, xo) && !meets_input(a, h),
            "an output overlaps an input or the other output");
    NormArgs n{N,          a->D,      a->d_x,    a->d_f,       a->d_gate, a->d_w_post,
               a->d_w_pre, a->ld_x,   a->ld_f,   a->ld_gate,   a->gate_rows, a->w_type,
               a->w_offset, a->res_scale, a->branch_scale, held_eps(a)};
    with_type(a->type, [&](auto t) {
        using T = decltype(t);
        const int64_t vecs = (a->D + kVec<T> - 1) / kVec<T>;
        with_row_shape<kForwardVecs<T>, false, false>(vecs, true, [&](auto shape) {
            constexpr int NT = decltype(shape)::nt, NV = decltype(shape)::nv;
            constexpr int LANES = decltype(shape)::lanes;
            const int64_t grid = std::min<int64_t>((N + NT / LANES - 1) / (NT / LANES),
                                                   kNormCus * (2048 / NT));
            hipLaunchKernelGGL((k_norm_forward<T, NT, NV, LANES>), dim3((unsigned)grid), dim3(NT),
                               0, (hipStream_t)hip_stream, n, d_x_out, ld_x_out, d_h, ld_h);
        });
    });
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

int64_t ecc_norm_work_size(const ecc_norm_t *a) {
    if (check_norm(a) != ECC_OK) return -1;
    // (sums of 8 bytes: whether they are is a matter of the gradients' type)
    return std::max<int64_t>(16, 3 * units_of(a).total * a->D * 8);
}

ecc_status_t ecc_norm_grad(const ecc_norm_t *a, const ecc_norm_grad_t *g, void *d_work,
                           void *hip_stream) {
    clear_error();
    const ecc_status_t st = check_norm(a);
    if (st != ECC_OK) return st;
    ECC_ARG(g != nullptr, "the gradients' description is NULL");
    ECC_ARG(a->n == 0 || (g->d_dh != nullptr) == (a->d_w_pre != nullptr),
            "d_dh goes with d_w_pre");
    ECC_ARG(known_type(g->grad_type), "unknown element type");
    ECC_ARG(g->accumulate == 0 || g->accumulate == 1, "accumulate must be 0 or 1");
    ECC_ARG(a->n == 0 || g->d_dx || g->d_df || g->d_dgate || g->d_dw_post || g->d_dw_pre,
            "no output");
    ECC_ARG(a->n == 0 || (!g->d_df && !g->d_dgate && !g->d_dw_post) || a->d_f,
            "gradients of f without f");
    ECC_ARG(a->n == 0 || ((!g->d_dw_post || a->d_w_post) && (!g->d_dw_pre || a->d_w_pre) &&
                    (!g->d_dgate || a->d_gate)),
            "a gradient of an operand that is absent");
    const int64_t lim = int64_t(1) << 40, tb = type_size(a->type), N = a->P * a->n, D = a->D;
    const int64_t gb = type_size(g->grad_type);
    const bool row_gate = g->d_dgate && a->gate_rows > 0;
    ECC_ARG((!g->d_dh || g->ld_dh >= D) && (!g->d_dx_out || g->ld_dx_out >= D) &&
                (!g->d_dx || g->ld_dx >= D) && (!g->d_df || g->ld_df >= D) &&
                (!row_gate || g->ld_dgate >= D),
            "a leading dimension is below D");
    if (g->ld_dh >= lim || g->ld_dx_out >= lim || g->ld_dx >= lim || g->ld_df >= lim ||
        g->ld_dgate >= lim || g->worker_stride >= lim) {
        set_error("a leading dimension or the stride is too large");
        return ECC_ERR_RANGE;
    }
    const bool params = g->d_dw_post || g->d_dw_pre || (g->d_dgate && !row_gate);
    ECC_ARG(a->P == 1 || !params || g->worker_stride >= D, "workers' gradients overlap");
    ECC_ARG(N == 0 || d_work, "NULL pointer");
    ECC_ARG(N == 0 || (a->d_x || !a->d_w_pre), "NULL pointer");
    ECC_ARG((uintptr_t)d_work % 16 == 0, "d_work must be 16-byte aligned");
    ECC_ARG(((uintptr_t)g->d_dh | (uintptr_t)g->d_dx_out | (uintptr_t)g->d_dx |
             (uintptr_t)g->d_df | (row_gate ? (uintptr_t)g->d_dgate : 0)) % tb == 0 &&
                ((uintptr_t)g->d_dw_post | (uintptr_t)g->d_dw_pre |
                 (row_gate ? 0 : (uintptr_t)g->d_dgate)) % gb == 0,
            "an array is not aligned to its elements");
    // inputs and outputs, and which output may stand in for which input
    const int64_t gate_n = a->gate_rows ? (N + a->gate_rows - 1) / a->gate_rows : 0;
    auto rows = [&](const void *p, int64_t ld) { return span_of(p, N, ld, D, tb); };
    auto param = [&](const void *p) { return span_of(p, a->P, g->worker_stride, D, gb); };
    const Span in[4] = {rows(a->d_x, a->ld_x), rows(a->d_f, a->ld_f), rows(g->d_dh, g->ld_dh),
                        rows(g->d_dx_out, g->ld_dx_out)};
    const Span out[6] = {rows(g->d_dx, g->ld_dx),
                         rows(g->d_df, g->ld_df),
                         row_gate ? span_of(g->d_dgate, gate_n, g->ld_dgate, D, tb)
                                  : param(g->d_dgate),
                         param(g->d_dw_post),
                         param(g->d_dw_pre),
                         span_of(d_work, N ? ecc_norm_work_size(a) : 0)};
    const int64_t in_ld[4] = {a->ld_x, a->ld_f, g->ld_dh, g->ld_dx_out};
    const int64_t out_ld[2] = {g->ld_dx, g->ld_df};
    for (int o = 0; o < 6; ++o) {
        for (int i = 0; i < 4; ++i) {
            const bool stands_in = o < 2 && out[o].p == in[i].p && out_ld[o] == in_ld[i] &&
                                   (o == 0 ? i >= 2 : i == 1 || i == 2);
            ECC_ARG(stands_in || !spans_meet(out[o], in[i]), "an output overlaps an input");
        }
        ECC_ARG(!meets_input(a, out[o]), "an output overlaps an input");
        for (int q = 0; q < o; ++q)
            ECC_ARG(!spans_meet(out[o], out[q]),
                    "two outputs, or an output and the work buffer, overlap");
    }
    hipStream_t s = (hipStream_t)hip_stream;
    if (N == 0 && (!params || g->accumulate)) return ECC_OK;
    NormArgs n{N,          D,          a->d_x,    a->d_f,       a->d_gate, a->d_w_post,
               a->d_w_pre, a->ld_x,   a->ld_f,   a->ld_gate,   a->gate_rows, a->w_type,
               a->w_offset, a->res_scale, a->branch_scale, held_eps(a)};
    NormGradArgs ga{};
    ga.dh = g->d_dh;
    ga.dxo = g->d_dx_out;
    ga.ld_dh = g->ld_dh;
    ga.ld_dxo = g->ld_dx_out;
    ga.dx = g->d_dx;
    ga.df = g->d_df;
    ga.ld_dx = g->ld_dx;
    ga.ld_df = g->ld_df;
    ga.ld_dgate = g->ld_dgate;
    ga.u = units_of(a);
    if (ga.u.total >= (int64_t(1) << 32) / backward_threads(a->type, D)) {
        set_error("P = %d workers are too many for one launch", a->P);
        return ECC_ERR_RANGE;
    }
    auto run = [&](auto t, auto sum) {
        using T = decltype(t);
        using S = decltype(sum);
        S *work = (S *)d_work;
        const int64_t sums = ga.u.total * D;
        ga.pre = g->d_dw_pre ? work : nullptr;
        ga.post = g->d_dw_post ? work + sums : nullptr;
        const bool gate_sums = g->d_dgate && (!row_gate || ga.u.split);
        ga.share = gate_sums ? work + 2 * sums : nullptr;
        ga.dgate = row_gate && !ga.u.split ? g->d_dgate : nullptr;
        // (a shared gate row's sum is one wave's, row by row)
        const bool several = !(a->d_f && a->d_gate) || a->gate_rows <= 1;
        if (N > 0)
            with_row_shape<kBackwardVecs<T>, true, kDeep<T, S>>(
                (D + kVec<T> - 1) / kVec<T>, several, [&](auto shape) {
                constexpr int NT = decltype(shape)::nt, NV = decltype(shape)::nv;
                constexpr int LANES = decltype(shape)::lanes;
                constexpr bool HOLD = kDeep<T, S> ? NT < 1024
                                                  : NV <= kBackwardVecs<T> &&
                                                        !(std::is_same_v<T, double> && NT == 1024);
                constexpr size_t lds = HOLD ? 3 * sizeof(Acc<T>) * NV * kVec<T> * NT : 0;
                static_assert(lds <= 128 << 10, "the weights of a row in LDS");
                NormGradArgs args = ga;
                // (the longest rows' sums lie there even where a group ends
                // within its unit)
                if (!HOLD && g->d_dgate) args.share = work + 2 * sums;
                auto kernel = k_norm_grad<T, S, NT, NV, HOLD, LANES>;
                if constexpr (lds > (64 << 10))
                    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                              hipFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)lds);
                hipLaunchKernelGGL(kernel, dim3((unsigned)ga.u.total), dim3(NT), lds, s, n,
                                   args);
            });
        // (as many results at a time as a launch of fewer than 2^32 threads has)
        auto join = [&](NormJoin j, int arrays) {
            const int64_t results = j.count;
            const bool wide = (D + 63) / 64 * results >= 64;
            const int64_t blocks = wide ? (D + 63) / 64 : (D + 15) / 16;
            const int64_t most = (int64_t(1) << 31) / kNormJoinThreads / blocks;
            for (int64_t at = 0; at < results; at += most) {
                j.count = std::min(most, results - at);
                const dim3 grid((unsigned)(blocks * j.count), arrays), threads(kNormJoinThreads);
                if (wide) hipLaunchKernelGGL((k_norm_join<S, 64>), grid, threads, 0, s, j);
                else hipLaunchKernelGGL((k_norm_join<S, 16>), grid, threads, 0, s, j);
                for (int z = 0; z < arrays; ++z) {
                    j.from[z] = j.from[z] ? (const S *)j.from[z] + j.count * j.per * D : nullptr;
                    j.to[z] = j.to[z] ? (char *)j.to[z] + j.count * j.ld[z] * type_size(j.type[z])
                                      : nullptr;
                }
            }
        };
        if (params) {
            NormJoin j{};
            j.from[0] = ga.pre;
            j.from[1] = ga.post;
            j.from[2] = ga.share;
            j.to[0] = g->d_dw_pre;
            j.to[1] = g->d_dw_post;
            j.to[2] = row_gate ? nullptr : g->d_dgate;
            for (int z = 0; z < 3; ++z) {
                j.ld[z] = g->worker_stride;
                j.type[z] = g->grad_type;
            }
            j.accumulate = g->accumulate;
            j.per = ga.u.per_worker;
            j.count = a->P;
            j.D = D;
            join(j, 3);
        }
        if (row_gate && ga.u.split && N > 0) {
            NormJoin j{};
            j.from[0] = ga.share;
            j.to[0] = g->d_dgate;
            j.ld[0] = g->ld_dgate;
            j.type[0] = a->type;
            j.per = ga.u.per_group;
            j.count = gate_n;
            j.D = D;
            join(j, 1);
        }
    };
    with_type(a->type, [&](auto t) {
        if (params && g->grad_type == ECC_F64) run(t, double{});
        else run(t, Acc<decltype(t)>{});
    });
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
