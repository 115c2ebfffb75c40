// Distillation from a teacher's top logits: loss and logit gradients of N rows
// of V student logits (the formulas are in libecc.h).
//
// Bound by memory: a row's logits are read and its gradient is written, with
// one exponential per logit for the sum, one for the gradient, and as many
// more for hard labels at a temperature other than 1.  A row's gradient
// needs the sums over the whole row first, so a workgroup keeps the row in its
// registers in between, as memory holds it: NV vectors of 16 bytes per
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
constexpr int kHeld = 8;            // vectors of a row that a thread keeps
constexpr int kSplitThreads = 256;
constexpr int64_t kPartMin = 8192;  // logits of a part at least
constexpr int64_t kPartRows = 512;  // parts that are wanted in all

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

// exp(d / tau) for d <= 0: fp32 by the hardware's power of two with the
// factor log2(e) / tau, fp64 by the library function.
template <typename A>
struct Temper {
    A c;
    __device__ __forceinline__ explicit Temper(double tau)
        : c(std::is_same_v<A, float> ? (A)(1.4426950408889634 / tau) : (A)(1.0 / tau)) {}
    __device__ __forceinline__ A operator()(A d) const {
        if constexpr (std::is_same_v<A, float>) return __builtin_amdgcn_exp2f(d * c);
        else return ::exp(d * c);
    }
};
template <typename A>
__device__ __forceinline__ A minus_inf() {
    return -(A)__builtin_inff();
}
__device__ __forceinline__ float ln(float v) { return ::logf(v); }
__device__ __forceinline__ double ln(double v) { return ::log(v); }

// Which exponentials a row needs: at the temperature alone (no hard labels,
// or both at temperature 1), or at both.
enum { kOneExp = 0, kTwoExps = 1 };

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
            const A d = m - to;
            s *= at(d);
            if constexpr (MODE == kTwoExps) s1 *= one(d);
            m = to;
        }
    }
    __device__ __forceinline__ void add(A z, A ref, const Temper<A> &at, const Temper<A> &one) {
        s += at(z - ref);
        if constexpr (MODE == kTwoExps) s1 += one(z - ref);
    }
    // the wave's 64, in every lane
    __device__ __forceinline__ void join_wave(const Temper<A> &at, const Temper<A> &one) {
        const A most = wave_all(m, OpMax{}), d = m - base(most);
        s = wave_all(s * at(d), OpSum{});
        if constexpr (MODE == kTwoExps) s1 = wave_all(s1 * one(d), OpSum{});
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

// G vectors of logits in registers (live ones: below `live`) into r.
template <typename T, typename A, int MODE, int G>
__device__ __forceinline__ void add_vectors(Running<A, MODE> &r, const Raw<T, kVec<T>> *v,
                                            const bool (&live)[G], const Temper<A> &at,
                                            const Temper<A> &one) {
    A most = r.m;
#pragma unroll
    for (int g = 0; g < G; ++g)
        if (live[g])
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) most = OpMax{}(most, v[g].template get<A>(i));
    r.raise(most, at, one);
    const A ref = Running<A, MODE>::base(r.m);
#pragma unroll
    for (int g = 0; g < G; ++g)
        if (live[g])
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) r.add(v[g].template get<A>(i), ref, at, one);
}

// The teacher's entries of a row in LDS, and what the row's labels ask for.
template <typename A>
struct Entries {
    int32_t idx[kTopMax];  // -1 outside the vocabulary
    A p[kTopMax];
    A z[kTopMax];
    A label_z;
};

// Reads a row's entries; the logits that they name come from the row itself or
// from where an earlier launch has put them.
template <typename T, typename A>
__device__ __forceinline__ void read_entries(const DistillArgs &a, int64_t row, int K, int32_t label,
                                             const T *z, const A *picked, Entries<A> &e) {
    for (int k = threadIdx.x; k < K; k += blockDim.x) {
        const int32_t i = a.idx[row * a.K + k];
        const bool held = i >= 0 && i < a.V;
        e.idx[k] = held ? i : -1;
        e.p[k] = held ? load_typed<A>(a.top, a.top_type, row * a.K + k) : minus_inf<A>();
        e.z[k] = !held ? (A)0 : picked ? picked[k] : load_elem<A>(z + i);
    }
    if (threadIdx.x == 0 && label >= 0) e.label_z = picked ? picked[a.K] : load_elem<A>(z + label);
}

// The entries' logits to probabilities; false when there is none.  Every wave
// forms the sum for itself.  The workgroup has passed a barrier since
// read_entries, and passes one before p is read as a probability.
template <typename A>
__device__ __forceinline__ bool teacher(int K, const Temper<A> &at, Entries<A> &e) {
    const int lane = threadIdx.x & 63;
    A most = minus_inf<A>();
    for (int k = lane; k < K; k += 64) most = OpMax{}(most, e.p[k]);
    most = wave_all(most, OpMax{});
    const bool some = most != minus_inf<A>();
    A sum = (A)0;
    for (int k = lane; k < K; k += 64) sum += some ? at(e.p[k] - most) : (A)0;
    sum = wave_all(sum, OpSum{});
    __syncthreads();  // every wave has read the logits
    for (int k = threadIdx.x; k < K; k += blockDim.x)
        e.p[k] = some ? at(e.p[k] - most) / sum : (A)0;
    return some;
}

// What a row's sums make of its weights: the gradient is e A + e1 B with e =
// exp((z - m) / tau), e1 = exp(z - m).
template <typename A, int MODE>
struct RowTerms {
    A m, soft, hard, s, s1;
    Temper<A> at, one;
    __device__ __forceinline__ A dense(A z) const {
        const A d = z - m;
        if constexpr (MODE == kTwoExps) return at(d) * soft + one(d) * hard;
        else return at(d) * (soft + hard);
    }
};

// The loss of a row, by the first wave.
template <typename A, int MODE>
__device__ __forceinline__ void write_loss(const DistillArgs &a, int64_t row, int K, int32_t label,
                                           A w, const RowTerms<A, MODE> &t, const Entries<A> &e) {
    if (threadIdx.x >= 64) return;
    const A inv_tau = (A)(1.0 / a.tau), log_s = ln(t.s);
    A kl = (A)0;
    for (int k = threadIdx.x; k < K; k += 64) {
        const A p = e.p[k];
        if (p > (A)0) kl += p * (ln(p) - ((e.z[k] - t.m) * inv_tau - log_s));
        else if (p != p) kl += p;
    }
    kl = wave_all(kl, OpSum{});
    if (threadIdx.x == 0) {
        A loss = K > 0 ? (A)(a.kd * a.tau * a.tau) * kl : (A)0;
        if (label >= 0) {
            const A log_s1 = MODE == kTwoExps ? ln(t.s1) : log_s;
            loss += (A)a.ce * (log_s1 - (e.label_z - t.m));
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
            store_elem<A>(dz + label, t.dense(e.label_z) - hard);
    }
}

// A whole row per workgroup.
template <typename T, int NT, int MODE>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 4) void k_distill_row(DistillArgs a) {
    using A = Acc<T>;
    constexpr int VEC = kVec<T>, G = 4, NW = NT / 64;
    static_assert(kHeld % G == 0, "whole groups of vectors");
    __shared__ Entries<A> e;
    __shared__ A s_run[3 * NW];
    const int64_t row = blockIdx.x;
    const T *z = reinterpret_cast<const T *>(a.z) + row * a.ld_z;
    T *dz = a.dz ? reinterpret_cast<T *>(a.dz) + row * a.ld_dz : nullptr;
    const A w = a.weight ? (A)a.weight[row] : (A)1;
    const int64_t full = a.V / VEC, tail = full * VEC + threadIdx.x;  // whole vectors; the rest
    if (w == (A)0) {
        if (threadIdx.x == 0) reinterpret_cast<A *>(a.loss)[row] = (A)0;
        if (dz) {
            Raw<T, VEC> zero;
#pragma unroll
            for (int i = 0; i < Raw<T, VEC>::kWords; ++i) zero.w[i] = 0;
            for (int64_t j = threadIdx.x; j < full; j += NT) zero.store(dz + j * VEC);
            if (tail < a.V) store_elem<A>(dz + tail, (A)0);
        }
        return;
    }
    const int K = a.kd != 0.0 ? a.K : 0;
    int32_t label = a.labels && a.ce != 0.0 ? a.labels[row] : -1;
    if (label >= a.V) label = -1;
    const Temper<A> at(a.tau), one(1.0);
    Running<A, MODE> r;
    r.clear();
    Raw<T, VEC> held[kHeld];
#pragma unroll
    for (int v = 0; v < kHeld; ++v) {
        const int64_t j = (int64_t)v * NT + threadIdx.x;
        if (j < full) held[v].load(z + j * VEC);
    }
    read_entries<T, A>(a, row, K, label, z, nullptr, e);
    const A last = tail < a.V ? load_elem<A>(z + tail) : (A)0;
#pragma unroll
    for (int v = 0; v < kHeld; v += G) {
        bool live[G];
#pragma unroll
        for (int g = 0; g < G; ++g) live[g] = (int64_t)(v + g) * NT + threadIdx.x < full;
        add_vectors<T, A, MODE, G>(r, held + v, live, at, one);
    }
    for (int64_t j0 = (int64_t)kHeld * NT; j0 < full; j0 += G * NT) {
        Raw<T, VEC> more[G];
        bool live[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int64_t j = j0 + g * NT + threadIdx.x;
            live[g] = j < full;
            if (live[g]) more[g].load(z + j * VEC);
        }
        add_vectors<T, A, MODE, G>(r, more, live, at, one);
    }
    if (tail < a.V) {
        r.raise(OpMax{}(r.m, last), at, one);
        r.add(last, Running<A, MODE>::base(r.m), at, one);
    }
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
    const A hard = label >= 0 ? w * (A)a.ce / (MODE == kTwoExps ? r.s1 : r.s) : (A)0;
    const RowTerms<A, MODE> t{Running<A, MODE>::base(r.m), soft, hard, r.s, r.s1, at, one};
    if (dz) {
        auto put = [&](const Raw<T, VEC> &v, int64_t j) {
            A d[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) d[i] = t.dense(v.template get<A>(i));
            Raw<T, VEC> o;
            o.set_all(d);
            o.store(dz + j * VEC);
        };
#pragma unroll
        for (int v = 0; v < kHeld; ++v) {
            const int64_t j = (int64_t)v * NT + threadIdx.x;
            if (j < full) put(held[v], j);
        }
        for (int64_t j0 = (int64_t)kHeld * NT; j0 < full; j0 += G * NT) {
            Raw<T, VEC> more[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t j = j0 + g * NT + threadIdx.x;
                if (j < full) more[g].load(z + j * VEC);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t j = j0 + g * NT + threadIdx.x;
                if (j < full) put(more[g], j);
            }
        }
        if (tail < a.V) store_elem<A>(dz + tail, t.dense(last));
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
    const int64_t full = (hi - lo) / VEC, tail = full * VEC + threadIdx.x;
    Running<A, MODE> r;
    r.clear();
    for (int64_t j0 = 0; j0 < full; j0 += G * NT) {
        Raw<T, VEC> more[G];
        bool live[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int64_t j = j0 + g * NT + threadIdx.x;
            live[g] = j < full;
            if (live[g]) more[g].load(z + j * VEC);
        }
        add_vectors<T, A, MODE, G>(r, more, live, at, one);
    }
    if (tail < hi - lo) {
        const A last = load_elem<A>(z + tail);
        r.raise(OpMax{}(r.m, last), at, one);
        r.add(last, Running<A, MODE>::base(r.m), at, one);
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
    __shared__ Entries<A> e;
    const int64_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const T *z = reinterpret_cast<const T *>(a.z) + row * a.ld_z;
    T *dz = a.dz ? reinterpret_cast<T *>(a.dz) + row * a.ld_dz : nullptr;
    const int64_t lo = part * a.part, hi = min(lo + a.part, a.V);
    const int64_t full = (hi - lo) / VEC, tail = lo + full * VEC + threadIdx.x;
    const A w = a.weight ? (A)a.weight[row] : (A)1;
    if (w == (A)0) {
        if (threadIdx.x == 0 && part == 0) reinterpret_cast<A *>(a.loss)[row] = (A)0;
        if (dz) {
            Raw<T, VEC> zero;
#pragma unroll
            for (int i = 0; i < Raw<T, VEC>::kWords; ++i) zero.w[i] = 0;
            for (int64_t j = threadIdx.x; j < full; j += NT) zero.store(dz + lo + j * VEC);
            if (tail < hi) store_elem<A>(dz + tail, (A)0);
        }
        return;
    }
    const int K = a.kd != 0.0 ? a.K : 0;
    int32_t label = a.labels && a.ce != 0.0 ? a.labels[row] : -1;
    if (label >= a.V) label = -1;
    const Temper<A> at(a.tau), one(1.0);
    read_entries<T, A>(a, row, K, label, z,
                       reinterpret_cast<const A *>(a.picked) + row * (a.K + 1), e);
    // the parts' sums, 64 at a time in order
    const A *from = reinterpret_cast<const A *>(a.stats) + 3 * row * a.parts;
    Running<A, MODE> r;
    r.clear();
    for (int64_t p = 0; p < a.parts; p += 64) {
        Running<A, MODE> q;
        q.join(from + 3 * p, (int)min((int64_t)64, a.parts - p), at, one);
        if (q.m > r.m) {
            r.raise(q.m, at, one);
            r.s += q.s;
            r.s1 += q.s1;
        } else {
            const A d = q.m - Running<A, MODE>::base(r.m);
            r.s += q.s * at(d);
            if constexpr (MODE == kTwoExps) r.s1 += q.s1 * one(d);
        }
    }
    __syncthreads();
    const bool some = K > 0 && teacher(K, at, e);
    const A soft = some ? w * (A)(a.kd * a.tau) / r.s : (A)0;
    const A hard = label >= 0 ? w * (A)a.ce / (MODE == kTwoExps ? r.s1 : r.s) : (A)0;
    const RowTerms<A, MODE> t{Running<A, MODE>::base(r.m), soft, hard, r.s, r.s1, at, one};
    if (dz) {
        for (int64_t j0 = 0; j0 < full; j0 += G * NT) {
            Raw<T, VEC> more[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t j = j0 + g * NT + threadIdx.x;
                if (j < full) more[g].load(z + lo + j * VEC);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t j = j0 + g * NT + threadIdx.x;
                if (j < full) {
                    A d[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[i] = t.dense(more[g].template get<A>(i));
                    Raw<T, VEC> o;
                    o.set_all(d);
                    o.store(dz + lo + j * VEC);
                }
            }
        }
        if (tail < hi) store_elem<A>(dz + tail, t.dense(load_elem<A>(z + tail)));
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
    if (N <= 0) return 1;
    return std::max<int64_t>(1, std::min((kPartRows + N - 1) / N, V / kPartMin));
}

static ecc_status_t check_distill(const ecc_distill_t *a) {
    ECC_ARG(a != nullptr, "the description is NULL");
    ECC_ARG(a->N >= 0 && a->V >= 1, "N must be >= 0, V >= 1");
    ECC_ARG(a->K >= 0 && a->K <= kTopMax, "K = %d must lie in [0, %d]", a->K, kTopMax);
    ECC_ARG(known_type(a->type) && known_type(a->top_type), "unknown element type");
    ECC_ARG(a->tau > 0.0 && a->tau <= 1e30, "tau must be positive");
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

template <typename T, int MODE>
void launch_distill(const DistillArgs &a, int64_t N, hipStream_t s) {
    if (a.parts > 1) {
        const dim3 grid((unsigned)(N * a.parts)), block(kSplitThreads);
        hipLaunchKernelGGL((k_distill_part<T, MODE>), grid, block, 0, s, a);
        hipLaunchKernelGGL((k_distill_parts<T, MODE>), grid, block, 0, s, a);
        return;
    }
    const dim3 grid((unsigned)N);
    const int64_t vecs = a.V / kVec<T>;
    if (vecs <= 64 * kHeld)
        hipLaunchKernelGGL((k_distill_row<T, 64, MODE>), grid, dim3(64), 0, s, a);
    else if (vecs <= 256 * kHeld)
        hipLaunchKernelGGL((k_distill_row<T, 256, MODE>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((k_distill_row<T, 1024, MODE>), grid, dim3(1024), 0, s, a);
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
    const int64_t z_bytes = row_extent(N, a->ld_z, a->V) * tb,
                  dz_bytes = d_dz ? row_extent(N, ld_dz, a->V) * tb : 0, w_bytes = work_bytes(a);
    const bool in_place = d_dz == a->d_z && ld_dz == a->ld_z;
    struct Range {
        const void *p;
        int64_t n;
    };
    const Range out[3] = {{d_dz, dz_bytes}, {d_loss, N * lb}, {d_work, w_bytes}};
    const Range in[5] = {{a->d_z, z_bytes},
                         {a->d_top, N * a->K * type_size(a->top_type)},
                         {a->d_idx, N * a->K * 4},
                         {a->d_labels, a->d_labels ? N * 4 : 0},
                         {a->d_weight, a->d_weight ? N * 4 : 0}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 5; ++i)
            ECC_ARG((o == 0 && i == 0 && in_place) ||
                        !ranges_meet(out[o].p, out[o].n, in[i].p, in[i].n),
                    "an output overlaps an input");
        for (int q = 0; q < o; ++q)
            ECC_ARG(!ranges_meet(out[o].p, out[o].n, out[q].p, out[q].n),
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
        if (two) launch_distill<T, kTwoExps>(d, N, (hipStream_t)hip_stream);
        else launch_distill<T, kOneExp>(d, N, (hipStream_t)hip_stream);
    });
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // extern "C"
