// Distillation from a teacher's top logits: loss and logit gradients of N rows
// of V student logits (the formulas are in libecc.h).
//
// Bound by memory: a row's logits are read and its gradient is written, with
// one exponential per logit for the sum, one for the gradient, and as many
// more for hard labels at a temperature other than 1.  A row's gradient
// needs the sums over the whole row first, so a workgroup keeps the row in its
// registers in between, as memory holds it: up to 16 vectors of 16 bytes per
// thread.  Of a longer row the rest is read a second time.
//
// Each thread keeps a running maximum and the sums of exp((z - maximum) /
// tau) and exp(z - maximum) over its logits, rescaled when the maximum grows;
// lanes, waves and (where a row is split) workgroups join theirs in order.
// The K entries of the teacher take part twice: their logits are gathered
// for the loss before anything is written (the gradient may take the place of
// the logits), and their elements of the gradient are written again, with the
// teacher's share, after the whole row's.
//
// With few rows a row is split over workgroups: one launch leaves every
// part's maximum and sums and the entries' logits in the work buffer, a
// second joins them and writes the gradient.
#include <algorithm>

#include "lm_common.h"

namespace ecc {

constexpr int kTopMax = ECC_DISTILL_MAX_TOP;
constexpr int kSplitThreads = 256;
// Parts of split rows (24 rows of 200,001 fp32 logits: 20.1 us, 128,000 bf16
// logits of one row: 12.4 us; with at least 8,192 logits in a part and 512
// parts 21.1 and 14.1 us).
constexpr int64_t kPartMin = 2048;   // logits of a part at least
constexpr int64_t kPartRows = 1024;  // parts that are wanted in all
constexpr int64_t kRowsAlone = 512;  // rows that are not split

struct DistillArgs {
    int64_t V;
    int32_t K, top_type;
    const void *z;
    int64_t ld_z;
    const void *top;
    const int32_t *idx, *labels;
    const float *weight;
    double tau, kd, ce;
    void *loss;
    void *dz;
    int64_t ld_dz;
    // a split row: parts, logits of a part, and the work buffer's [N][parts]
    // maxima and sums and [N][K + 1] logits of the entries and the label
    int64_t parts, part;
    void *stats, *picked;
};

__device__ __forceinline__ float ln(float v) { return ::logf(v); }
__device__ __forceinline__ double ln(double v) { return ::log(v); }
template <typename A>
__device__ __forceinline__ A minus_inf() {
    return -(A)__builtin_inff();
}
__device__ __forceinline__ float fma_(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fma_(double a, double b, double c) { return __builtin_fma(a, b, c); }
__device__ __forceinline__ float magnitude(float v) { return __builtin_fabsf(v); }
__device__ __forceinline__ double magnitude(double v) { return __builtin_fabs(v); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;  // (the compiler's own maxima first quiet every operand)
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ double max3(double a, double b, double c) { return fmax(fmax(a, b), c); }

// Exponentials at one temperature.  fp32 works with powers of two (the
// hardware's): with c = log2(e) / tau an exponential is 2^(z c - r), its
// argument one multiply-add, for a reference r = fl(m c) that stands for the
// maximum m.  r is off by up to 2^-24 m c, which shifts a row's arguments alike
// and falls out of every quotient as long as it is small: up to |m c| = 2^20,
// where it stays below 2^-5.  Beyond, m is subtracted first (rows masked with
// a large finite value, temperatures near 0).  fp64 uses exp with c = 1 / tau,
// and a limit of 2^49.
template <typename A>
struct Temper {
    A c;
    __device__ __forceinline__ explicit Temper(double tau)
        : c(std::is_same_v<A, float> ? (A)(1.4426950408889634 / tau) : (A)(1.0 / tau)) {}
    static constexpr A kPlain = std::is_same_v<A, float> ? (A)0x1p20 : (A)0x1p49;
    __device__ __forceinline__ A power(A x) const {
        if constexpr (std::is_same_v<A, float>) return __builtin_amdgcn_exp2f(x);
        else return ::exp(x);
    }
    // does fl(m c) stand for m?
    __device__ __forceinline__ bool plain(A m) const { return magnitude(m * c) <= kPlain; }
    // how far m's reference lies above m c
    __device__ __forceinline__ A shift(A m) const { return plain(m) ? -fma_(m, c, -(m * c)) : (A)0; }
    // the exponent of z above m's, and exp of it
    __device__ __forceinline__ A above(A z, A m) const {
        return plain(m) ? fma_(z, c, -(m * c)) : (z - m) * c;
    }
    __device__ __forceinline__ A operator()(A z, A m) const { return power(above(z, m)); }
    // the factor that takes sums above m to sums above a higher one
    __device__ __forceinline__ A rescale(A m, A to) const {
        return power(plain(to) && plain(m) ? m * c - to * c
                                           : (m - to) * c + (shift(m) - shift(to)));
    }
    // the natural logarithm of exp(exponent)
    __device__ __forceinline__ A log_of(A exponent) const {
        return std::is_same_v<A, float> ? exponent * (A)0.6931471805599453 : exponent;
    }
};

// Which exponentials a row needs: at the temperature alone (no hard labels,
// or both at temperature 1), or at both; where the temperature is 2 or 4, that
// at temperature 1 is the other's square or fourth power, which costs no
// second exponential (16,384 rows of 131,072 bf16: 1.70 ms at temperature 2, 2.01
// at 3.5; of 32,000, which memory bounds, 0.38 ms both).
enum { kOneExp = 0, kTwoExps = 1, kSquare = 2, kFourth = 3 };
// exp(z - m), given e = exp((z - m) / tau)
template <int MODE, typename A>
__device__ __forceinline__ A power_of(A e) {
    if constexpr (MODE == kSquare) return e * e;
    else if constexpr (MODE == kFourth) return (e * e) * (e * e);
    else return e;
}

// Running maximum m and sums of exp((z - m) / tau) and exp(z - m).
template <typename A, int MODE>
struct Running {
    A m, s, s1;
    __device__ __forceinline__ void clear() {
        m = minus_inf<A>();
        s = s1 = (A)0;
    }
    // what z is compared with: a row (so far) of -infinity has no maximum
    static __device__ __forceinline__ A base(A m) { return m == minus_inf<A>() ? (A)0 : m; }
    __device__ __forceinline__ void raise(A to, const Temper<A> &at, const Temper<A> &one) {
        if (to > m) {
            const A f = at.rescale(m, to);
            s *= f;
            if constexpr (MODE == kTwoExps) s1 *= one.rescale(m, to);
            else if constexpr (MODE != kOneExp) s1 *= power_of<MODE>(f);
            m = to;
        }
    }
    __device__ __forceinline__ void add(A z, const Temper<A> &at, const Temper<A> &one) {
        const A e = at(z, base(m));
        s += e;
        if constexpr (MODE == kTwoExps) s1 += one(z, base(m));
        else if constexpr (MODE != kOneExp) s1 += power_of<MODE>(e);
    }
    // another's sums
    __device__ __forceinline__ void add(const Running &o, const Temper<A> &at,
                                        const Temper<A> &one) {
        raise(o.m, at, one);
        const A f = at.rescale(o.m, base(m));
        s += o.s * f;
        if constexpr (MODE == kTwoExps) s1 += o.s1 * one.rescale(o.m, base(m));
        else if constexpr (MODE != kOneExp) s1 += o.s1 * power_of<MODE>(f);
    }
    // the wave's 64, in every lane
    __device__ __forceinline__ void join_wave(const Temper<A> &at, const Temper<A> &one) {
        const A most = wave_all(m, OpMax{});
        const A f = at.rescale(m, base(most));
        s = wave_all(s * f, OpSum{});
        if constexpr (MODE == kTwoExps)
            s1 = wave_all(s1 * one.rescale(m, base(most)), OpSum{});
        else if constexpr (MODE != kOneExp) s1 = wave_all(s1 * power_of<MODE>(f), OpSum{});
        m = most;
    }
    // n <= 64 of them in memory, in every lane
    __device__ __forceinline__ void join(const A *from, int n, const Temper<A> &at,
                                         const Temper<A> &one) {
        const int lane = threadIdx.x & 63;
        m = lane < n ? from[3 * lane] : minus_inf<A>();
        s = lane < n ? from[3 * lane + 1] : (A)0;
        s1 = lane < n ? from[3 * lane + 2] : (A)0;
        join_wave(at, one);
    }
};

// G vectors of logits in registers into r: the first `live` of the thread's.
template <typename T, typename A, int MODE, int G>
__device__ __forceinline__ void add_vectors(Running<A, MODE> &r, const Raw<T, kVec<T>> *v,
                                            int32_t live, const Temper<A> &at,
                                            const Temper<A> &one) {
    A most = r.m;
#pragma unroll
    for (int g = 0; g < G; ++g)
        if (g < live)
#pragma unroll
            for (int i = 0; i < kVec<T>; i += 2)
                most = max3(most, v[g].template get<A>(i), v[g].template get<A>(i + 1));
    r.raise(most, at, one);
    const A m = Running<A, MODE>::base(r.m);
    if (at.plain(m) && one.plain(m)) {
        const A ref = -(m * at.c), ref1 = -(m * one.c);
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (g < live)
#pragma unroll
                for (int i = 0; i < kVec<T>; ++i) {
                    const A z = v[g].template get<A>(i);
                    const A e = at.power(fma_(z, at.c, ref));
                    r.s += e;
                    if constexpr (MODE == kTwoExps) r.s1 += one.power(fma_(z, one.c, ref1));
                    else if constexpr (MODE == kSquare) r.s1 = fma_(e, e, r.s1);
                    else if constexpr (MODE == kFourth) r.s1 = fma_(e * e, e * e, r.s1);
                }
    } else {
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (g < live)
#pragma unroll
                for (int i = 0; i < kVec<T>; ++i) r.add(v[g].template get<A>(i), at, one);
    }
}

// Vector j of a row.
template <typename T>
__device__ __forceinline__ T *vector_at(T *row, int32_t j) {
    return row + (int64_t)j * kVec<std::remove_const_t<T>>;
}

// How many of the vectors threadIdx.x + g NT, g = 0, 1, ..., lie below n.
__device__ __forceinline__ int32_t vectors(int32_t n, int nt) {
    return (n - (int32_t)threadIdx.x + nt - 1) / nt;
}

// The teacher's entries of a row in LDS, and what the row's labels ask for.
template <typename A>
struct Entries {
    A *p, *z, *label_z;
    int32_t *idx;  // -1 outside the vocabulary
    // in a workgroup's LDS of entries_bytes
    __device__ __forceinline__ Entries(double *lds, int K) {
        p = reinterpret_cast<A *>(lds);
        z = p + K;
        label_z = z + K;
        idx = reinterpret_cast<int32_t *>(label_z + 1);
    }
};
template <typename A>
constexpr size_t entries_bytes(int K) {
    return (2 * (size_t)K + 1) * sizeof(A) + (size_t)K * sizeof(int32_t);
}

// Reads a row's entries, in three steps so that what each waits for is under
// way long before: a thread's first entry and the label; the logits that they
// name, from the row itself or from where an earlier launch has put them; and
// all of it, with a thread's further entries, into LDS.
template <typename T, typename A>
struct EntryReads {
    int32_t i = -1;
    A p, z = (A)0, label_z = (A)0;
    __device__ __forceinline__ void names(const DistillArgs &a, int64_t row, int K) {
        p = minus_inf<A>();
        if ((int)threadIdx.x < K) {
            i = a.idx[row * a.K + threadIdx.x];
            p = load_typed<A>(a.top, a.top_type, row * a.K + threadIdx.x);
        }
        if (i < 0 || i >= a.V) {
            i = -1;
            p = minus_inf<A>();
        }
    }
    __device__ __forceinline__ void logits(const DistillArgs &a, int32_t label, const T *zr,
                                           const A *picked) {
        if (i >= 0) z = picked ? picked[threadIdx.x] : load_elem<A>(zr + i);
        if (threadIdx.x == 0 && label >= 0)
            label_z = picked ? picked[a.K] : load_elem<A>(zr + label);
    }
    __device__ __forceinline__ void keep(const DistillArgs &a, int64_t row, int K, const T *zr,
                                         const A *picked, const Entries<A> &e) const {
        if ((int)threadIdx.x < K) {
            e.idx[threadIdx.x] = i;
            e.p[threadIdx.x] = p;
            e.z[threadIdx.x] = z;
        }
        if (threadIdx.x == 0) *e.label_z = label_z;
        for (int k = threadIdx.x + blockDim.x; k < K; k += blockDim.x) {
            const int32_t n = a.idx[row * a.K + k];
            const bool held = n >= 0 && n < a.V;
            e.idx[k] = held ? n : -1;
            e.p[k] = held ? load_typed<A>(a.top, a.top_type, row * a.K + k) : minus_inf<A>();
            e.z[k] = !held ? (A)0 : picked ? picked[k] : load_elem<A>(zr + n);
        }
    }
};

// The elements of a row (or a part of one) as whole vectors and up to VEC - 1
// single ones behind them, one per thread.  The vectors start with the row,
// at whatever element that lies, so that a row's result does not depend on
// where it is (vectors at 16-byte boundaries would: of 16,384 rows of 50,003
// bf16 logits in 0.70 ms, against 0.81 ms).
template <typename T>
struct Pieces {
    int32_t full, edge;  // vectors; this thread's element, or -1
    __device__ __forceinline__ explicit Pieces(int64_t n) {
        full = (int32_t)(n / kVec<T>);
        edge = (int32_t)threadIdx.x < (int32_t)(n % kVec<T>)
                   ? full * kVec<T> + (int32_t)threadIdx.x
                   : -1;
    }
};

// The entries' logits to probabilities; false when there is none.  Every wave
// forms the sum for itself.  The workgroup has passed a barrier since
// read_entries, and passes one before p is read as a probability.
template <typename A>
__device__ __forceinline__ bool teacher(int K, const Temper<A> &at, const Entries<A> &e) {
    const int lane = threadIdx.x & 63;
    A most = minus_inf<A>();
    for (int k = lane; k < K; k += 64) most = OpMax{}(most, e.p[k]);
    most = wave_all(most, OpMax{});
    const bool some = most != minus_inf<A>();
    A sum = (A)0;
    for (int k = lane; k < K; k += 64) sum += some ? at(e.p[k], most) : (A)0;
    sum = wave_all(sum, OpSum{});
    __syncthreads();  // every wave has read the logits
    for (int k = threadIdx.x; k < K; k += blockDim.x)
        e.p[k] = some ? at(e.p[k], most) / sum : (A)0;
    return some;
}

// What a row's sums make of its weights: the gradient is e soft + e1 hard with
// e = exp((z - m) / tau), e1 = exp(z - m).
template <typename A, int MODE>
struct RowTerms {
    A m, soft, hard, s, s1;
    Temper<A> at, one;
    bool plain;
    A ref, ref1;
    __device__ __forceinline__ RowTerms(const Running<A, MODE> &r, A soft_, A hard_,
                                        const Temper<A> &at_, const Temper<A> &one_)
        : m(Running<A, MODE>::base(r.m)), soft(soft_), hard(hard_), s(r.s), s1(r.s1), at(at_),
          one(one_), plain(at_.plain(m) && one_.plain(m)), ref(-(m * at_.c)),
          ref1(-(m * one_.c)) {}
    __device__ __forceinline__ A weigh(A e, A e1) const {
        if constexpr (MODE == kOneExp) return e * (soft + hard);
        else if constexpr (MODE == kSquare) return e * fma_(e, hard, soft);
        else return fma_(e, soft, e1 * hard);
    }
    __device__ __forceinline__ A dense(A z) const {
        const A e = at(z, m);
        return weigh(e, MODE == kTwoExps ? one(z, m) : power_of<MODE>(e));
    }
    // log of the hard labels' q at z, given the logarithm of their sum
    __device__ __forceinline__ A log_hard(A z, A log_sum) const {
        if constexpr (MODE == kTwoExps) return one.log_of(one.above(z, m)) - log_sum;
        const A times = MODE == kSquare ? (A)2 : MODE == kFourth ? (A)4 : (A)1;
        return at.log_of(times * at.above(z, m)) - log_sum;
    }
    // a vector of logits to their gradients
    template <typename T>
    __device__ __forceinline__ void put(const Raw<T, kVec<T>> &v, T *to) const {
        A d[kVec<T>];
        if (plain) {
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) {
                const A z = v.template get<A>(i);
                const A e = at.power(fma_(z, at.c, ref));
                d[i] = weigh(e, MODE == kTwoExps ? one.power(fma_(z, one.c, ref1))
                                                 : power_of<MODE>(e));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) d[i] = dense(v.template get<A>(i));
        }
        Raw<T, kVec<T>> o;
        o.set_all(d);
        o.template store<true>(to);
    }
};

// The loss of a row, by the first wave.
template <typename A, int MODE>
__device__ __forceinline__ void write_loss(const DistillArgs &a, int64_t row, int K, int32_t label,
                                           A w, const RowTerms<A, MODE> &t, const Entries<A> &e) {
    if (threadIdx.x >= 64) return;
    const A log_s = ln(t.s);
    A kl = (A)0;
    for (int k = threadIdx.x; k < K; k += 64) {
        const A p = e.p[k];
        if (p > (A)0) kl += p * (ln(p) - (t.at.log_of(t.at.above(e.z[k], t.m)) - log_s));
        else if (p != p) kl += p;
    }
    kl = wave_all(kl, OpSum{});
    if (threadIdx.x == 0) {
        A loss = K > 0 ? (A)(a.kd * a.tau * a.tau) * kl : (A)0;
        if (label >= 0) {
            const A log_s1 = MODE == kOneExp ? log_s : ln(t.s1);
            loss -= (A)a.ce * t.log_hard(*e.label_z, log_s1);
        }
        reinterpret_cast<A *>(a.loss)[row] = w * loss;
    }
}

// The gradient's elements of the entries and the label within [lo, hi).
template <typename T, typename A, int MODE>
__device__ __forceinline__ void write_entries(const DistillArgs &a, int K, int32_t label, A w,
                                              int64_t lo, int64_t hi, T *dz,
                                              const RowTerms<A, MODE> &t, const Entries<A> &e) {
    const A soft = w * (A)(a.kd * a.tau), hard = w * (A)a.ce;
    bool named = false;  // the label is one of the entries
    for (int k0 = 0; k0 < K; k0 += blockDim.x) {
        const int k = k0 + threadIdx.x;
        const int32_t i = k < K ? e.idx[k] : -1;
        if (i < lo || i >= hi) continue;
        // entries that name the same logit add up, each writes the same sum
        A p = (A)0;
        for (int q = 0; q < K; ++q) p += e.idx[q] == i ? e.p[q] : (A)0;
        A v = t.dense(e.z[k]) - soft * p;
        if (i == label) v -= hard;
        store_elem<A>(dz + i, v);
    }
    if (label >= lo && label < hi && threadIdx.x < 64) {
        for (int k = threadIdx.x; k < K; k += 64) named = named || e.idx[k] == label;
        if (!__any(named) && threadIdx.x == 0)
            store_elem<A>(dz + label, t.dense(*e.label_z) - hard);
    }
}

template <typename T>
__device__ __forceinline__ void write_zeros(T *dz, const Pieces<T> &piece, int nt) {
    constexpr int VEC = kVec<T>;
    Raw<T, VEC> zero;
#pragma unroll
    for (int i = 0; i < Raw<T, VEC>::kWords; ++i) zero.w[i] = 0;
    for (int32_t j = threadIdx.x; j < piece.full; j += nt) zero.template store<true>(vector_at(dz, j));
    if (piece.edge >= 0) store_elem<Acc<T>>(dz + piece.edge, (Acc<T>)0);
}

// A whole row per workgroup.
template <typename T, int NT, int HELD, int WAVES, int MODE>
__global__ __launch_bounds__(NT, WAVES) void k_distill_row(DistillArgs a) {
    using A = Acc<T>;
    constexpr int VEC = kVec<T>, G = 4, NW = NT / 64;
    static_assert(HELD % G == 0, "whole groups of vectors");
    extern __shared__ double s_entries[];
    const Entries<A> e(s_entries, a.K);
    __shared__ A s_run[3 * NW];
    const int64_t row = blockIdx.x;
    const T *z = reinterpret_cast<const T *>(a.z) + row * a.ld_z;
    T *dz = a.dz ? reinterpret_cast<T *>(a.dz) + row * a.ld_dz : nullptr;
    const A w = a.weight ? (A)a.weight[row] : (A)1;
    const Pieces<T> piece(a.V);
    const int32_t full = piece.full;
    if (w == (A)0) {
        if (threadIdx.x == 0) reinterpret_cast<A *>(a.loss)[row] = (A)0;
        if (dz) write_zeros(dz, piece, NT);
        return;
    }
    const int K = a.kd != 0.0 ? a.K : 0;
    int32_t label = a.labels && a.ce != 0.0 ? a.labels[row] : -1;
    if (label >= a.V) label = -1;
    const Temper<A> at(a.tau), one(1.0);
    Running<A, MODE> r;
    r.clear();
    EntryReads<T, A> entry;
    entry.names(a, row, K);
    Raw<T, VEC> held[HELD];
#pragma unroll
    for (int v = 0; v < HELD; ++v) {
        const int32_t j = v * NT + (int32_t)threadIdx.x;
        if (j < full) held[v].template load<true>(vector_at(z, j));
    }
    const A edge = piece.edge >= 0 ? load_elem<A>(z + piece.edge) : (A)0;
    entry.logits(a, label, z, nullptr);
#pragma unroll
    for (int v = 0; v < HELD; v += G) {
        add_vectors<T, A, MODE, G>(r, held + v, vectors(full - v * NT, NT), at, one);
    }
    for (int32_t j0 = HELD * NT; j0 < full; j0 += G * NT) {
        Raw<T, VEC> more[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int32_t j = j0 + g * NT + (int32_t)threadIdx.x;
            if (j < full) more[g].load(vector_at(z, j));
        }
        add_vectors<T, A, MODE, G>(r, more, vectors(full - j0, NT), at, one);
    }
    if (piece.edge >= 0) {
        r.raise(edge, at, one);
        r.add(edge, at, one);
    }
    entry.keep(a, row, K, z, nullptr, e);
    r.join_wave(at, one);
    if constexpr (NW > 1) {
        if ((threadIdx.x & 63) == 0) {
            s_run[3 * (threadIdx.x >> 6)] = r.m;
            s_run[3 * (threadIdx.x >> 6) + 1] = r.s;
            s_run[3 * (threadIdx.x >> 6) + 2] = r.s1;
        }
    }
    __syncthreads();
    if constexpr (NW > 1) r.join(s_run, NW, at, one);
    const bool some = K > 0 && teacher(K, at, e);
    const A soft = some ? w * (A)(a.kd * a.tau) / r.s : (A)0;
    const A hard = label >= 0 ? w * (A)a.ce / (MODE == kOneExp ? r.s : r.s1) : (A)0;
    const RowTerms<A, MODE> t(r, soft, hard, at, one);
    if (dz) {
#pragma unroll
        for (int v = 0; v < HELD; ++v) {
            const int32_t j = v * NT + (int32_t)threadIdx.x;
            if (j < full) t.put(held[v], vector_at(dz, j));
        }
        for (int32_t j0 = HELD * NT; j0 < full; j0 += G * NT) {
            Raw<T, VEC> more[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int32_t j = j0 + g * NT + (int32_t)threadIdx.x;
                if (j < full) more[g].load(vector_at(z, j));
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int32_t j = j0 + g * NT + (int32_t)threadIdx.x;
                if (j < full) t.put(more[g], vector_at(dz, j));
            }
        }
        if (piece.edge >= 0) store_elem<A>(dz + piece.edge, t.dense(edge));
    }
    __syncthreads();  // the row is written and the probabilities stand
    write_loss<A, MODE>(a, row, some ? K : 0, label, w, t, e);
    if (dz) write_entries<T, A, MODE>(a, some ? K : 0, label, w, 0, a.V, dz, t, e);
}

// A part of a row: its maximum and sums; part 0 also gathers the entries'
// logits.
template <typename T, int MODE>
__global__ __launch_bounds__(kSplitThreads) void k_distill_part(DistillArgs a) {
    using A = Acc<T>;
    constexpr int VEC = kVec<T>, G = 4, NT = kSplitThreads, NW = NT / 64;
    __shared__ A s_run[3 * NW];
    const int64_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const T *z = reinterpret_cast<const T *>(a.z) + row * a.ld_z;
    if (a.weight && a.weight[row] == 0.0f) return;
    const int64_t lo = part * a.part, hi = min(lo + a.part, a.V);
    const Temper<A> at(a.tau), one(1.0);
    if (part == 0) {
        A *picked = reinterpret_cast<A *>(a.picked) + row * (a.K + 1);
        for (int k = threadIdx.x; k < a.K; k += NT) {
            const int32_t i = a.idx[row * a.K + k];
            picked[k] = i >= 0 && i < a.V ? load_elem<A>(z + i) : (A)0;
        }
        const int32_t label = a.labels ? a.labels[row] : -1;
        if (threadIdx.x == 0 && label >= 0 && label < a.V) picked[a.K] = load_elem<A>(z + label);
    }
    z += lo;
    const Pieces<T> piece(hi - lo);
    const int32_t full = piece.full;
    Running<A, MODE> r;
    r.clear();
    for (int32_t j0 = 0; j0 < full; j0 += G * NT) {
        Raw<T, VEC> more[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int32_t j = j0 + g * NT + (int32_t)threadIdx.x;
            if (j < full) more[g].load(vector_at(z, j));
        }
        add_vectors<T, A, MODE, G>(r, more, vectors(full - j0, NT), at, one);
    }
    if (piece.edge >= 0) {
        const A edge = load_elem<A>(z + piece.edge);
        r.raise(edge, at, one);
        r.add(edge, at, one);
    }
    r.join_wave(at, one);
    if ((threadIdx.x & 63) == 0) {
        s_run[3 * (threadIdx.x >> 6)] = r.m;
        s_run[3 * (threadIdx.x >> 6) + 1] = r.s;
        s_run[3 * (threadIdx.x >> 6) + 2] = r.s1;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        r.join(s_run, NW, at, one);
        if (threadIdx.x == 0) {
            A *to = reinterpret_cast<A *>(a.stats) + 3 * (row * a.parts + part);
            to[0] = r.m;
            to[1] = r.s;
            to[2] = r.s1;
        }
    }
}

// A part of a row's gradient (part 0: the loss too), from the parts' sums.
template <typename T, int MODE>
__global__ __launch_bounds__(kSplitThreads) void k_distill_parts(DistillArgs a) {
    using A = Acc<T>;
    constexpr int VEC = kVec<T>, G = 4, NT = kSplitThreads;
    extern __shared__ double s_entries[];
    const Entries<A> e(s_entries, a.K);
    const int64_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const T *z = reinterpret_cast<const T *>(a.z) + row * a.ld_z;
    T *dz = a.dz ? reinterpret_cast<T *>(a.dz) + row * a.ld_dz : nullptr;
    const int64_t lo = part * a.part, hi = min(lo + a.part, a.V);
    const Pieces<T> piece(hi - lo);
    const int32_t full = piece.full;
    const A w = a.weight ? (A)a.weight[row] : (A)1;
    if (w == (A)0) {
        if (threadIdx.x == 0 && part == 0) reinterpret_cast<A *>(a.loss)[row] = (A)0;
        if (dz) write_zeros(dz + lo, piece, NT);
        return;
    }
    const int K = a.kd != 0.0 ? a.K : 0;
    int32_t label = a.labels && a.ce != 0.0 ? a.labels[row] : -1;
    if (label >= a.V) label = -1;
    const Temper<A> at(a.tau), one(1.0);
    const A *picked = reinterpret_cast<const A *>(a.picked) + row * (a.K + 1);
    EntryReads<T, A> entry;
    entry.names(a, row, K);
    entry.logits(a, label, z, picked);
    entry.keep(a, row, K, z, picked, e);
    // the parts' sums, 64 at a time in order
    const A *from = reinterpret_cast<const A *>(a.stats) + 3 * row * a.parts;
    Running<A, MODE> r;
    r.clear();
    for (int64_t p = 0; p < a.parts; p += 64) {
        Running<A, MODE> q;
        q.join(from + 3 * p, (int)min((int64_t)64, a.parts - p), at, one);
        r.add(q, at, one);
    }
    __syncthreads();
    const bool some = K > 0 && teacher(K, at, e);
    const A soft = some ? w * (A)(a.kd * a.tau) / r.s : (A)0;
    const A hard = label >= 0 ? w * (A)a.ce / (MODE == kOneExp ? r.s : r.s1) : (A)0;
    const RowTerms<A, MODE> t(r, soft, hard, at, one);
    if (dz) {
        const T *zv = z + lo;
        T *dv = dz + lo;
        for (int32_t j0 = 0; j0 < full; j0 += G * NT) {
            Raw<T, VEC> more[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int32_t j = j0 + g * NT + (int32_t)threadIdx.x;
                if (j < full) more[g].load(vector_at(zv, j));
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int32_t j = j0 + g * NT + (int32_t)threadIdx.x;
                if (j < full) t.put(more[g], vector_at(dv, j));
            }
        }
        if (piece.edge >= 0)
            store_elem<A>(dz + lo + piece.edge, t.dense(load_elem<A>(z + lo + piece.edge)));
    }
    __syncthreads();
    if (part == 0) write_loss<A, MODE>(a, row, some ? K : 0, label, w, t, e);
    if (dz) write_entries<T, A, MODE>(a, some ? K : 0, label, w, lo, hi, dz, t, e);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

// Parts of a row: 1 where the rows alone occupy the device.
inline int64_t distill_parts(int64_t N, int64_t V) {
    if (N <= 0 || N >= kRowsAlone) return 1;
    return std::max<int64_t>(1, std::min((kPartRows + N - 1) / N, V / kPartMin));
}

static ecc_status_t check_distill(const ecc_distill_t *a) {
    ECC_ARG(a != nullptr, "the description is NULL");
    ECC_ARG(a->N >= 0 && a->V >= 1, "N must be >= 0, V >= 1");
    ECC_ARG(a->K >= 0 && a->K <= kTopMax, "K = %d must lie in [0, %d]", a->K, kTopMax);
    ECC_ARG(known_type(a->type) && known_type(a->top_type), "unknown element type");
    ECC_ARG(a->tau >= 1e-15 && a->tau <= 1e15, "tau must lie in [1e-15, 1e15]");
    const int64_t lim = (int64_t(1) << 31) - 1;
    if (a->N >= lim || a->V >= lim || a->ld_z >= (int64_t(1) << 40)) {
        set_error("N or V is too large");
        return ECC_ERR_RANGE;
    }
    ECC_ARG(a->ld_z >= a->V, "a leading dimension is below V");
    if (a->N == 0) return ECC_OK;
    ECC_ARG(a->d_z && (a->K == 0 || (a->d_top && a->d_idx)), "NULL pointer");
    ECC_ARG((uintptr_t)a->d_z % type_size(a->type) == 0 &&
                (uintptr_t)a->d_top % type_size(a->top_type) == 0 &&
                ((uintptr_t)a->d_idx | (uintptr_t)a->d_labels | (uintptr_t)a->d_weight) % 4 == 0,
            "an array is not aligned to its elements");
    return ECC_OK;
}

// Bytes of the work buffer's two parts.
inline int64_t stats_bytes(const ecc_distill_t *a, int64_t parts) {
    return (3 * a->N * parts * (a->type == ECC_F64 ? 8 : 4) + 15) & ~int64_t(15);
}
inline int64_t work_bytes(const ecc_distill_t *a) {
    const int64_t parts = distill_parts(a->N, a->V);
    if (parts == 1) return 16;
    return stats_bytes(a, parts) + a->N * (a->K + 1) * (a->type == ECC_F64 ? 8 : 4);
}

// The same from a later row on.
template <typename T>
DistillArgs rows_from(DistillArgs a, int64_t row) {
    a.z = (const T *)a.z + row * a.ld_z;
    if (a.dz) a.dz = (T *)a.dz + row * a.ld_dz;
    a.loss = (Acc<T> *)a.loss + row;
    if (a.K > 0) {
        a.top = (const char *)a.top + row * a.K * type_size(a.top_type);
        a.idx += row * a.K;
    }
    if (a.labels) a.labels += row;
    if (a.weight) a.weight += row;
    return a;
}

// Rows of their own workgroups: as many threads as hold a row in 16 vectors
// each, up to 1,024.  16 vectors leave 16 waves to a CU, four rows of 32,000
// bf16 logits at a time (16,384 rows, temperature 2 with hard labels: 0.43 ms,
// against 0.46 ms with 512 threads and 4 vectors; 131,072 logits: 1.77 ms,
// against 1.97 ms with 8 vectors, and the rest read twice in both; since
// then, with accesses past the caches, 0.38 and 1.68 ms, 5.4 and 5.0 TB/s).
// Rows of up to 4 vectors a thread fill the CU with more waves (100,000 rows of
// 1,000: 0.15 against 0.30 ms).  fp64, whose exponentials need registers,
// holds half as many in half as many threads.
template <typename T, int MODE>
void launch_distill(const DistillArgs &a, int64_t N, hipStream_t s) {
    const size_t lds = entries_bytes<Acc<T>>(a.K);
    if (a.parts > 1) {
        const dim3 grid((unsigned)(N * a.parts)), block(kSplitThreads);
        hipLaunchKernelGGL((k_distill_part<T, MODE>), grid, block, 0, s, a);
        hipLaunchKernelGGL((k_distill_parts<T, MODE>), grid, block, lds, s, a);
        return;
    }
    const int64_t vecs = a.V / kVec<T>;
    // (a launch has fewer than 2^32 threads)
    auto launch = [&](auto kernel, int threads) {
        const int64_t most = (int64_t(1) << 31) / threads;
        for (int64_t row = 0; row < N; row += most)
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(most, N - row)), dim3(threads), lds,
                               s, rows_from<T>(a, row));
    };
    constexpr bool f64 = std::is_same_v<T, double>;
    constexpr int H = f64 ? 8 : 16, W = f64 ? 2 : 4, MOST = f64 ? 512 : 1024;
    if (vecs <= 64 * 4) launch(k_distill_row<T, 64, 4, f64 ? 2 : 7, MODE>, 64);
    else if (vecs <= 64 * H) launch(k_distill_row<T, 64, H, W, MODE>, 64);
    else if (vecs <= 128 * H) launch(k_distill_row<T, 128, H, W, MODE>, 128);
    else if (vecs <= 256 * H) launch(k_distill_row<T, 256, H, W, MODE>, 256);
    else if (vecs <= 512 * H) launch(k_distill_row<T, 512, H, W, MODE>, 512);
    else launch(k_distill_row<T, MOST, H, W, MODE>, MOST);
}

}  // namespace ecc

using namespace ecc;

extern "C" {

int64_t ecc_distill_work_size(const ecc_distill_t *a) {
    if (check_distill(a) != ECC_OK) return -1;
    return work_bytes(a);
}

ecc_status_t ecc_distill(const ecc_distill_t *a, void *d_loss, void *d_dz, int64_t ld_dz,
                         void *d_work, void *hip_stream) {
    clear_error();
    const ecc_status_t st = check_distill(a);
    if (st != ECC_OK) return st;
    const int64_t N = a->N, tb = type_size(a->type), lb = a->type == ECC_F64 ? 8 : 4;
    ECC_ARG(!d_dz || ld_dz >= a->V, "a leading dimension is below V");
    if (ld_dz >= (int64_t(1) << 40)) {
        set_error("a leading dimension is too large");
        return ECC_ERR_RANGE;
    }
    if (N == 0) return ECC_OK;
    ECC_ARG(d_loss && d_work, "NULL pointer");
    ECC_ARG((uintptr_t)d_loss % lb == 0 && (uintptr_t)d_dz % tb == 0 &&
                (uintptr_t)d_work % 16 == 0,
            "an array is not aligned");
    const bool in_place = d_dz == a->d_z && ld_dz == a->ld_z;
    const Span out[3] = {span_of(d_dz, N, ld_dz, a->V, tb), span_of(d_loss, N * lb),
                         span_of(d_work, work_bytes(a))};
    const Span in[5] = {span_of(a->d_z, N, a->ld_z, a->V, tb),
                        span_of(a->d_top, N * a->K * type_size(a->top_type)),
                        span_of(a->d_idx, N * a->K * 4), span_of(a->d_labels, N * 4),
                        span_of(a->d_weight, N * 4)};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 5; ++i)
            ECC_ARG((o == 0 && i == 0 && in_place) || !spans_meet(out[o], in[i]),
                    "an output overlaps an input");
        for (int q = 0; q < o; ++q)
            ECC_ARG(!spans_meet(out[o], out[q]),
                    "two outputs, or an output and the work buffer, overlap");
    }
    DistillArgs d{};
    d.V = a->V;
    d.K = a->K;
    d.top_type = a->top_type;
    d.z = a->d_z;
    d.ld_z = a->ld_z;
    d.top = a->d_top;
    d.idx = a->d_idx;
    d.labels = a->d_labels;
    d.weight = a->d_weight;
    d.tau = a->tau;
    d.kd = a->kd_weight;
    d.ce = a->ce_weight;
    d.loss = d_loss;
    d.dz = d_dz;
    d.ld_dz = ld_dz;
    d.parts = distill_parts(N, a->V);
    // parts of whole vectors (of the narrowest type: 8 elements)
    d.part = ((a->V + d.parts - 1) / d.parts + 7) & ~int64_t(7);
    d.parts = (a->V + d.part - 1) / d.part;
    d.stats = d_work;
    d.picked = (char *)d_work + stats_bytes(a, distill_parts(N, a->V));
    const bool two = a->d_labels && a->ce_weight != 0.0 && a->tau != 1.0;
    with_type(a->type, [&](auto t) {
        using T = decltype(t);
        if (two && a->tau == 2.0) launch_distill<T, kSquare>(d, N, (hipStream_t)hip_stream);
        else if (two && a->tau == 4.0) launch_distill<T, kFourth>(d, N, (hipStream_t)hip_stream);
        else if (two) launch_distill<T, kTwoExps>(d, N, (hipStream_t)hip_stream);
        else launch_distill<T, kOneExp>(d, N, (hipStream_t)hip_stream);
    });
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
