// Global norms of the workers' gradients over many tensors, and gradients
// scaled to at most a norm, in place or into the contributions of a collective:
//   norm_p = sqrt(sum over tensors and elements of g^2)
//   out = g max_norm / norm_p where norm_p > max_norm, else g.
// Squares are added in fp64 whatever the gradients' type: the squares of fp32
// neither overflow nor vanish there, and 10^9 of them lose nothing.  Bound by
// memory: gradients are read once for the norm and once for the scaling, which
// writes them (nothing in place where the norm is within the limit).
//
// Both kernels share one cut of all tensors into chunks, a workgroup each.  Of
// few chunks the scaling adds the sums by itself, in their order (a few KiB from
// the L2), so that clipping is two launches; more are added in a launch between.
// Chunks are short and many, so that what runs at a time lies close together in
// memory, and all accesses go past the caches: 0.67e9 fp32 gradients take 0.38
// ms for the norm (7.0 TB/s) and 0.97 ms for the scaling (5.5 TB/s), against 0.51 and
// 1.08 ms in 2,048 long chunks, and 0.61 and 1.19 ms through the caches.  Up to kTableEntries tensors are
// described in the launch itself; more by small launches that write a table
// into the work buffer first, so that nothing is copied from the host and a
// captured call holds all that it needs.
#include <algorithm>
#include <new>
#include <vector>

#include "lm_common.h"

namespace ecc {
namespace {

constexpr int kThreads = 256;
constexpr int kTableEntries = 56;     // 3.1 KiB of a launch's 4 KiB of arguments
constexpr int64_t kChunkMin = 4096;   // elements
constexpr int64_t kChunks = 32768;    // of all workers, about
constexpr int64_t kFewChunks = 1024;  // of a worker, whose sums the scaling adds
constexpr int kAddThreads = 1024;     // in the launch that adds more of them

struct Entry {
    const void *g;
    void *out;
    int64_t n, stride, out_stride;
    int64_t first;        // its first chunk
    int32_t type, out_type;
};
struct Entries {
    Entry e[kTableEntries];
};

struct ClipArgs {
    int32_t count, P;
    int64_t chunk, chunks;      // elements; chunks of a worker
    const Entry *table;
    double *sums;               // [P][chunks]
    double *norms;
    double max_norm;
    int32_t zero;               // norms that are not finite: zeros
};

__global__ __launch_bounds__(64) void k_clip_table(Entries some, int32_t at, int32_t count,
                                                   Entry *table) {
    const int32_t i = threadIdx.x;
    if (i < count) table[at + i] = some.e[i];
}

// The tensor that a chunk belongs to: the last that begins at or before it.
template <class T>
__device__ __forceinline__ int32_t tensor_of(const T &entries, int32_t count, int64_t chunk) {
    int32_t lo = 0, hi = count - 1;
    while (lo < hi) {
        const int32_t mid = (lo + hi + 1) / 2;
        if (entries[mid].first <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Sum of a workgroup's values, in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double *s) {
    v = wave_all(v, OpSum());
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    double all = s[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) all += s[w];
    __syncthreads();
    return all;
}

// Calls f(first element, vectors that are whole) for a thread's vectors of V in
// groups of U, a workgroup's vectors side by side.
template <int V, int U, class F>
__device__ __forceinline__ void vectors_of(int64_t n, F &&f) {
    int64_t i = threadIdx.x * V;
    for (; i + (U - 1) * kThreads * V + V <= n; i += kThreads * V * U) f(i, std::true_type{});
    for (; i < n; i += kThreads * V * U) f(i, std::false_type{});
}
template <int V, int U, class T, class WHOLE>
__device__ __forceinline__ void load_group(Raw<T, V> (&x)[U], const T *g, int64_t i, int64_t n,
                                           WHOLE) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t at = i + u * kThreads * V;
        if constexpr (WHOLE::value) x[u].template load<true>(g + at);
        else x[u].template load_upto<true>(g + at, n - at);
    }
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T *g, int64_t n) {
    constexpr int V = kVec<T>, U = 4;
    double sum[2] = {0.0, 0.0};
    vectors_of<V, U>(n, [&](int64_t i, auto whole) {
        Raw<T, V> x[U];
        load_group(x, g, i, n, whole);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const double v = x[u].template get<double>(e);
                sum[e & 1] = __builtin_fma(v, v, sum[e & 1]);
            }
    });
    return sum[0] + sum[1];
}

template <class E>
__device__ __forceinline__ void norm_chunk(const E &entries, const ClipArgs &a, double *s) {
    const int32_t p = blockIdx.y;
    const int64_t chunk = blockIdx.x;
    const Entry t = entries[tensor_of(entries, a.count, chunk)];
    const int64_t at = (chunk - t.first) * a.chunk, n = min(a.chunk, t.n - at);
    const int64_t from = p * t.stride + at;
    double sum;
    if (t.type == ECC_F32) sum = chunk_squares((const float *)t.g + from, n);
    else if (t.type == ECC_BF16) sum = chunk_squares((const bf16_t *)t.g + from, n);
    else sum = chunk_squares((const double *)t.g + from, n);
    sum = block_sum<kThreads>(sum, s);
    if (threadIdx.x == 0) a.sums[p * a.chunks + chunk] = sum;
}

// A worker's norm from its chunks' sums.
template <int THREADS>
__device__ __forceinline__ double norm_of(const ClipArgs &a, int32_t p, double *s) {
    double sum = 0.0;
    const double *sums = a.sums + p * a.chunks;
    int64_t i = threadIdx.x;
    for (; i + 7 * THREADS < a.chunks; i += 8 * THREADS) {
        double v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sums[i + e * THREADS];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
    }
    for (; i < a.chunks; i += THREADS) sum += sums[i];
    return sqrt(block_sum<THREADS>(sum, s));
}

template <typename T, typename O>
__device__ __forceinline__ void scale_chunk(const T *g, O *out, int64_t n, double by, bool zero) {
    constexpr int V = kVec<T> > kVec<O> * 2 ? kVec<O> * 2 : kVec<T>, U = 4;
    vectors_of<V, U>(n, [&](int64_t i, auto whole) {
        Raw<T, V> x[U];
        load_group(x, g, i, n, whole);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = i + u * kThreads * V;
            Raw<O, V> y;
            double v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = zero ? 0.0 : x[u].template get<double>(e) * by;
            y.set_all(v);
            if constexpr (decltype(whole)::value) y.template store<true>(out + at);
            else y.template store_upto<true>(out + at, n - at);
        }
    });
}

template <class E>
__device__ __forceinline__ void clip_chunk(const E &entries, const ClipArgs &a, double *s) {
    const int32_t p = blockIdx.y;
    const int64_t chunk = blockIdx.x;
    double norm;
    if (a.chunks <= kFewChunks) {
        norm = norm_of<kThreads>(a, p, s);
        if (chunk == 0 && threadIdx.x == 0) a.norms[p] = norm;
    } else {
        norm = a.norms[p];
    }
    const bool finite = norm < __builtin_inf();
    const bool zero = !finite && a.zero;
    const double by = finite && norm > a.max_norm ? a.max_norm / norm : 1.0;
    const Entry t = entries[tensor_of(entries, a.count, chunk)];
    if (by == 1.0 && !zero && t.out == t.g) return;
    const int64_t at = (chunk - t.first) * a.chunk, n = min(a.chunk, t.n - at);
    const int64_t from = p * t.stride + at, to = p * t.out_stride + at;
    auto with_out = [&](auto *g) {
        if (t.out_type == ECC_F32) scale_chunk(g, (float *)t.out + to, n, by, zero);
        else if (t.out_type == ECC_BF16) scale_chunk(g, (bf16_t *)t.out + to, n, by, zero);
        else scale_chunk(g, (double *)t.out + to, n, by, zero);
    };
    if (t.type == ECC_F32) with_out((const float *)t.g + from);
    else if (t.type == ECC_BF16) with_out((const bf16_t *)t.g + from);
    else with_out((const double *)t.g + from);
}

__global__ __launch_bounds__(kThreads) void k_norm_few(Entries few, ClipArgs a) {
    __shared__ double s[kThreads / 64];
    norm_chunk(few.e, a, s);
}
__global__ __launch_bounds__(kThreads) void k_norm_many(ClipArgs a) {
    __shared__ double s[kThreads / 64];
    norm_chunk(a.table, a, s);
}
__global__ __launch_bounds__(kThreads) void k_clip_few(Entries few, ClipArgs a) {
    __shared__ double s[kThreads / 64];
    clip_chunk(few.e, a, s);
}
__global__ __launch_bounds__(kThreads) void k_clip_many(ClipArgs a) {
    __shared__ double s[kThreads / 64];
    clip_chunk(a.table, a, s);
}
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_only(ClipArgs a) {
    __shared__ double s[THREADS / 64];
    const double norm = norm_of<THREADS>(a, blockIdx.x, s);
    if (threadIdx.x == 0) a.norms[blockIdx.x] = norm;
}

// ---------------------------------------------------------------------------
// the cut and its checks
// ---------------------------------------------------------------------------

struct Cut {
    int64_t chunk = kChunkMin, chunks = 0;
    int64_t table_bytes(int32_t count) const {
        return count > kTableEntries ? (int64_t)sizeof(Entry) * count : 0;
    }
    int64_t bytes(int32_t P, int32_t count) const {
        return std::max<int64_t>(16, table_bytes(count) + 8 * P * chunks);
    }
};

Cut make_cut(int32_t P, int32_t count, const ecc_tensor_t *t) {
    Cut c;
    __int128 m = 0;
    for (int32_t i = 0; i < count; ++i) m += t[i].n;
    const __int128 want = (m * P + kChunks - 1) / kChunks;
    if (want > c.chunk) c.chunk = (int64_t)((want + 8191) / 8192 * 8192);
    for (int32_t i = 0; i < count; ++i) c.chunks += (t[i].n + c.chunk - 1) / c.chunk;
    return c;
}

ecc_status_t check(int32_t P, int32_t count, const ecc_tensor_t *t, bool outputs) {
    ECC_ARG(P >= 1 && count >= 0, "a size is out of range");
    ECC_ARG(t || count == 0, "NULL pointer");
    if (P > 65535 || count > (1 << 20)) {
        set_error("the sizes are beyond what the library supports");
        return ECC_ERR_RANGE;
    }
    __int128 m = 0;
    for (int32_t i = 0; i < count; ++i) {
        ECC_ARG(t[i].n >= 0, "tensor %d has a negative size", i);
        ECC_ARG(known_type(t[i].type), "tensor %d has an unknown type", i);
        ECC_ARG(t[i].n == 0 || t[i].d_grad, "tensor %d is NULL", i);
        ECC_ARG((uintptr_t)t[i].d_grad % type_size(t[i].type) == 0, "tensor %d is not aligned", i);
        ECC_ARG(P == 1 || t[i].stride >= t[i].n, "tensor %d: workers overlap", i);
        if (outputs && t[i].d_out) {
            ECC_ARG(known_type(t[i].out_type), "output %d has an unknown type", i);
            ECC_ARG((uintptr_t)t[i].d_out % type_size(t[i].out_type) == 0,
                    "output %d is not aligned", i);
            ECC_ARG(P == 1 || t[i].out_stride >= t[i].n, "output %d: workers overlap", i);
            if (t[i].out_stride >= (int64_t(1) << 56)) {
                set_error("a stride is too large");
                return ECC_ERR_RANGE;
            }
        }
        if (t[i].stride >= (int64_t(1) << 56)) {
            set_error("a stride is too large");
            return ECC_ERR_RANGE;
        }
        m += t[i].n;
    }
    if (m * P >= (int64_t(1) << 45)) {
        set_error("the sizes are beyond what the library supports");
        return ECC_ERR_RANGE;
    }
    return ECC_OK;
}

// Do outputs meet anything that is not their own gradient?  Spans are compared
// along their addresses, so that separate tensors cost a sort; rows of one
// pitch (parameters within the workers' contributions) by where they lie in it.
struct Held {
    Span s;
    int32_t tensor;
    bool out;
};

bool two_meet(const Held &a, const Held &b, const ecc_tensor_t *t) {
    if (!a.out && !b.out) return false;
    if (a.tensor == b.tensor && a.out != b.out && t[a.tensor].d_out == t[a.tensor].d_grad &&
        t[a.tensor].type == t[a.tensor].out_type && a.s.pitch == b.s.pitch)
        return false;
    return spans_meet(a.s, b.s);
}

bool outputs_meet(int32_t P, int32_t count, const ecc_tensor_t *t, const Span &work,
                  const Span &norms) {
    std::vector<Held> held;
    held.reserve(2 * (size_t)count + 2);
    auto rows = [&](const void *p, int64_t n, int64_t stride, int64_t size) {
        return P == 1 ? span_of(p, n * size) : span_of(p, P, stride, n, size);
    };
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].n == 0) continue;
        const bool own = !t[i].d_out || (t[i].d_out == t[i].d_grad && t[i].type == t[i].out_type &&
                                         (P == 1 || t[i].stride == t[i].out_stride));
        if (!own)
            held.push_back({rows(t[i].d_grad, t[i].n, t[i].stride, type_size(t[i].type)), i, false});
        held.push_back({own ? rows(t[i].d_grad, t[i].n, t[i].stride, type_size(t[i].type))
                            : rows(t[i].d_out, t[i].n, t[i].out_stride, type_size(t[i].out_type)),
                        i, true});
    }
    held.push_back({work, -1, true});
    held.push_back({norms, -2, true});
    // outputs that are rows of one pitch and lie apart within it are one block
    int64_t pitch = 0;
    bool one = P > 1;
    uintptr_t lo = ~uintptr_t(0), hi = 0;
    std::vector<std::pair<int64_t, int64_t>> within;
    for (const Held &h : held)
        if (h.out && h.tensor >= 0) {
            if (pitch == 0) pitch = h.s.pitch;
            one = one && h.s.pitch == pitch;
            lo = std::min(lo, (uintptr_t)h.s.p);
            hi = std::max(hi, (uintptr_t)h.s.p + (uintptr_t)h.s.bytes());
        }
    if (one && pitch > 0) {
        for (const Held &h : held)
            if (h.out && h.tensor >= 0) {
                const int64_t at = (int64_t)(((uintptr_t)h.s.p - lo) % (uintptr_t)pitch);
                within.push_back({at, at + h.s.width});
            }
        std::sort(within.begin(), within.end());
        for (size_t i = 0; i < within.size(); ++i) {
            const int64_t next = i + 1 < within.size() ? within[i + 1].first
                                                       : within[0].first + pitch;
            one = one && within[i].second <= next;
        }
        if (one) {
            std::vector<Held> rest;
            for (const Held &h : held)
                if (!h.out || h.tensor < 0) rest.push_back(h);
            const Span block = span_of((const void *)lo, (int64_t)(hi - lo));
            bool clear = true;
            for (const Held &h : rest) clear = clear && !spans_meet(h.s, block);
            if (clear) held.swap(rest);
        }
    }
    std::sort(held.begin(), held.end(),
              [](const Held &a, const Held &b) { return (uintptr_t)a.s.p < (uintptr_t)b.s.p; });
    std::vector<size_t> open;
    for (size_t i = 0; i < held.size(); ++i) {
        size_t kept = 0;
        for (size_t o : open)
            if ((uintptr_t)held[o].s.p + (uintptr_t)held[o].s.bytes() > (uintptr_t)held[i].s.p) {
                if (held[o].tensor >= 0 && held[i].tensor >= 0) {
                    if (two_meet(held[o], held[i], t)) return true;
                } else if ((held[o].out || held[i].out) && spans_meet(held[o].s, held[i].s)) {
                    return true;
                }
                open[kept++] = o;
            }
        open.resize(kept);
        open.push_back(i);
    }
    return false;
}

// Chunks of every tensor in the launch itself or the work buffer's table, then
// the sums of squares.
ecc_status_t run(int32_t P, int32_t count, const ecc_tensor_t *t, const Cut &cut, bool clip,
                 double max_norm, bool zero, double *d_norms, void *d_work, hipStream_t s) {
    ClipArgs a{};
    a.P = P;
    a.chunk = cut.chunk;
    a.chunks = cut.chunks;
    a.sums = (double *)((char *)d_work + cut.table_bytes(count));
    a.norms = d_norms;
    a.max_norm = max_norm;
    a.zero = zero;
    const bool many = count > kTableEntries;
    a.table = (const Entry *)d_work;
    Entries some{};
    int32_t held = 0, written = 0;
    int64_t first = 0;
    auto flush = [&] {
        if (held)
            hipLaunchKernelGGL(k_clip_table, dim3(1), dim3(64), 0, s, some, written, held,
                               (Entry *)d_work);
        written += held;
        held = 0;
    };
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].n == 0) continue;  // (a tensor without elements has no chunk)
        some.e[held++] = Entry{t[i].d_grad, t[i].d_out ? t[i].d_out : const_cast<void *>(t[i].d_grad),
                               t[i].n, t[i].stride, t[i].d_out ? t[i].out_stride : t[i].stride,
                               first, t[i].type, t[i].d_out ? t[i].out_type : t[i].type};
        first += (t[i].n + cut.chunk - 1) / cut.chunk;
        if (many && held == kTableEntries) flush();
    }
    if (many) flush();
    a.count = many ? written : held;
    const dim3 grid((unsigned)cut.chunks, (unsigned)P), block(kThreads);
    if (cut.chunks > 0) {
        if (many) hipLaunchKernelGGL(k_norm_many, grid, block, 0, s, a);
        else hipLaunchKernelGGL(k_norm_few, grid, block, 0, s, some, a);
    }
    // (few sums in the order in which the scaling adds them: the same norms)
    if (cut.chunks > kFewChunks)
        hipLaunchKernelGGL(k_norm_only<kAddThreads>, dim3((unsigned)P), dim3(kAddThreads), 0, s, a);
    else if (!clip || cut.chunks == 0)
        hipLaunchKernelGGL(k_norm_only<kThreads>, dim3((unsigned)P), block, 0, s, a);
    if (!clip || cut.chunks == 0) {
    } else if (many) hipLaunchKernelGGL(k_clip_many, grid, block, 0, s, a);
    else hipLaunchKernelGGL(k_clip_few, grid, block, 0, s, some, a);
    ECC_LAUNCH_CHECK();
    return ECC_OK;
}

}  // namespace
}  // namespace ecc

using namespace ecc;

extern "C" {

int64_t ecc_grad_norm_work_size(int32_t P, int32_t count, const ecc_tensor_t *h_tensors) {
    if (check(P, count, h_tensors, false) != ECC_OK) return -1;
    return make_cut(P, count, h_tensors).bytes(P, count);
}

ecc_status_t ecc_grad_norm(int32_t P, int32_t count, const ecc_tensor_t *h_tensors,
                           double *d_norms, void *d_work, void *hip_stream) {
    clear_error();
    const ecc_status_t st = check(P, count, h_tensors, false);
    if (st != ECC_OK) return st;
    ECC_ARG(d_norms && d_work, "NULL pointer");
    ECC_ARG((uintptr_t)d_norms % 8 == 0 && (uintptr_t)d_work % 16 == 0, "an array is not aligned");
    const Cut cut = make_cut(P, count, h_tensors);
    const Span norms = span_of(d_norms, 8 * (int64_t)P),
               work = span_of(d_work, cut.bytes(P, count));
    ECC_ARG(!spans_meet(norms, work), "an output and the work buffer overlap");
    for (int32_t i = 0; i < count; ++i) {
        const int64_t size = type_size(h_tensors[i].type);
        const Span g = P == 1 ? span_of(h_tensors[i].d_grad, h_tensors[i].n * size)
                              : span_of(h_tensors[i].d_grad, P, h_tensors[i].stride,
                                        h_tensors[i].n, size);
        ECC_ARG(!spans_meet(g, norms) && !spans_meet(g, work), "an output overlaps tensor %d", i);
    }
    return run(P, count, h_tensors, cut, false, 0.0, false, d_norms, d_work,
               (hipStream_t)hip_stream);
}

ecc_status_t ecc_clip_grads(int32_t P, int32_t count, const ecc_tensor_t *h_tensors,
                            double max_norm, int32_t nonfinite, double *d_norms, void *d_work,
                            void *hip_stream) {
    clear_error();
    const ecc_status_t st = check(P, count, h_tensors, true);
    if (st != ECC_OK) return st;
    ECC_ARG(max_norm >= 0.0, "max_norm must be >= 0");
    ECC_ARG(nonfinite == ECC_CLIP_KEEP || nonfinite == ECC_CLIP_ZERO, "nonfinite is unknown");
    ECC_ARG(d_norms && d_work, "NULL pointer");
    ECC_ARG((uintptr_t)d_norms % 8 == 0 && (uintptr_t)d_work % 16 == 0, "an array is not aligned");
    const Cut cut = make_cut(P, count, h_tensors);
    bool meet = true;
    try {
        meet = outputs_meet(P, count, h_tensors, span_of(d_work, cut.bytes(P, count)),
                            span_of(d_norms, 8 * (int64_t)P));
    } catch (const std::bad_alloc &) {
        set_error("out of host memory");
        return ECC_ERR_ALLOC;
    }
    ECC_ARG(!meet, "outputs overlap each other, another gradient, the norms or the work buffer");
    return run(P, count, h_tensors, cut, true, max_norm, nonfinite == ECC_CLIP_ZERO, d_norms,
               d_work, (hipStream_t)hip_stream);
}

}  // extern "C"
