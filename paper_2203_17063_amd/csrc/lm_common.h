// Shared by the language-model operators (embed.hip, norm.hip, distill.hip):
// element types, accesses of several elements at any element alignment, and
// the sums a wave or a workgroup forms.
//
// Sums are held in fp32 where the operands are fp32 or bf16 and in fp64 where
// one of them is fp64 (Acc below); a result is rounded once, when it is
// stored.  bf16 is rounded to nearest even (v_cvt_pk_bf16_f32), from fp64 by
// way of an fp32 that cannot change the outcome (on_the_way_to_bf16).
#pragma once

#include <algorithm>
#include <type_traits>

#include "ecc_common.h"

namespace ecc {

struct bf16_t {
    uint16_t bits;
};

template <typename T>
using Acc = std::conditional_t<std::is_same_v<T, double>, double, float>;
template <typename A, typename B>
using Wider = std::conditional_t<std::is_same_v<A, double> || std::is_same_v<B, double>, double,
                                 float>;

inline bool known_type(int32_t t) { return t == ECC_F64 || t == ECC_F32 || t == ECC_BF16; }

inline int64_t type_size(int32_t type) {
    switch (type) {
        case ECC_F64: return 8;
        case ECC_F32: return 4;
        case ECC_BF16: return 2;
        default: return 0;
    }
}

// Calls f with a value of the element type `type` names (checked before).
template <typename F>
inline void with_type(int32_t type, F &&f) {
    if (type == ECC_F64) f(double{});
    else if (type == ECC_F32) f(float{});
    else f(bf16_t{});
}

// Do the element ranges [a, a + na) and [b, b + nb) (in bytes) meet?
inline bool ranges_meet(const void *a, int64_t na, const void *b, int64_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Elements between the first and the end of the last row (up to 2^59, beyond
// any memory, so that their bytes fit 64 bits).
inline int64_t row_extent(int64_t rows, int64_t ld, int64_t cols) {
    const __int128 n = rows > 0 ? (__int128)(rows - 1) * ld + cols : 0;
    return (int64_t)std::min<__int128>(n, int64_t(1) << 59);
}

// Memory of a matrix, in bytes: rows of `width`, `pitch` from one to the next.
struct Span {
    const void *p = nullptr;
    int64_t rows = 0, pitch = 0, width = 0;
    int64_t bytes() const { return p ? row_extent(rows, pitch, width) : 0; }
};
inline Span span_of(const void *p, int64_t rows, int64_t ld, int64_t cols, int64_t size) {
    return Span{p, rows, ld * size, cols * size};
}
inline Span span_of(const void *p, int64_t bytes) { return Span{p, 1, bytes, bytes}; }

// Do two of them share a byte?  Rows of one pitch may lie beside each other in
// one buffer; matrices of different pitches are compared as a whole, gaps
// included.
inline bool spans_meet(const Span &a, const Span &b) {
    if (!ranges_meet(a.p, a.bytes(), b.p, b.bytes())) return false;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if ((a.rows == 1 && b.rows == 1) || (b.rows > 1 && b.pitch != pitch) || a.width > pitch ||
        b.width > pitch)
        return true;
    // row j of b begins d + (j - i) pitch after row i of a: between b's width
    // ahead of it and a's width behind for one of two differences only
    const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
    const int64_t below = d >= 0 ? d / pitch : -((-d + pitch - 1) / pitch), rest = d - below * pitch;
    auto there = [&](int64_t k) { return k > -a.rows && k < b.rows; };  // k = j - i
    return (there(-below) && rest < a.width) || (there(-below - 1) && rest - pitch > -b.width);
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two floats rounded to bf16, the first in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// An fp64 value as an fp32 that rounds to the same bf16: the value itself, or of
// its two fp32 neighbours the one whose last bit is set, which lies on the
// same side of every middle between two bf16 (to the nearest fp32, values
// close to such a middle would land on it and then go to the even bf16).
__device__ __forceinline__ float on_the_way_to_bf16(float v) { return v; }
__device__ __forceinline__ float on_the_way_to_bf16(double v) {
    const float f = (float)v;
    const double d = (double)f;
    if (d == v || v != v) return f;
    const uint32_t down = __builtin_fabs(d) > __builtin_fabs(v);  // f was rounded away from 0
    return __uint_as_float((__float_as_uint(f) - down) | 1u);
}

template <typename A, typename T>
__device__ __forceinline__ A load_elem(const T *p) {
    if constexpr (std::is_same_v<T, bf16_t>) return (A)bf16_value(p->bits);
    else return (A)*p;
}
template <typename A, typename T>
__device__ __forceinline__ void store_elem(T *p, A v) {
    if constexpr (std::is_same_v<T, bf16_t>) p->bits = (uint16_t)bf16_pair(on_the_way_to_bf16(v), 0.0f);
    else *p = (T)v;
}

// Element i of an array whose type is known at run time only.
template <typename A>
__device__ __forceinline__ A load_typed(const void *p, int32_t type, int64_t i) {
    if (type == ECC_F64) return (A) reinterpret_cast<const double *>(p)[i];
    if (type == ECC_F32) return (A) reinterpret_cast<const float *>(p)[i];
    return load_elem<A>(reinterpret_cast<const bf16_t *>(p) + i);
}

// W 32-bit words as memory holds them, at the alignment of one element
// (gfx950 takes 4-, 8- and 16-byte global accesses at any alignment).
template <int W, int ALIGN>
struct Words {
    typedef uint32_t t __attribute__((ext_vector_type(W), aligned(ALIGN)));
};

// N consecutive elements of T in registers, as memory holds them.
template <typename T, int N>
struct Raw {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    static_assert(kWords * 4 == N * (int)sizeof(T) && kWords >= 1, "whole words");
    uint32_t w[kWords];

    // all N elements
    template <bool STREAM = false>
    __device__ __forceinline__ void load(const T *p) {
        constexpr int Q = kWords >= 4 ? 4 : kWords;
        using V = typename Words<Q, sizeof(T)>::t;
#pragma unroll
        for (int i = 0; i < kWords; i += Q) {
            const V *src = reinterpret_cast<const V *>(p) + i / Q;
            V v;
            if constexpr (STREAM) v = __builtin_nontemporal_load(src);
            else v = *src;
#pragma unroll
            for (int j = 0; j < Q; ++j) w[i + j] = v[j];
        }
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(T *p) const {
        constexpr int Q = kWords >= 4 ? 4 : kWords;
        using V = typename Words<Q, sizeof(T)>::t;
#pragma unroll
        for (int i = 0; i < kWords; i += Q) {
            V v;
#pragma unroll
            for (int j = 0; j < Q; ++j) v[j] = w[i + j];
            V *dst = reinterpret_cast<V *>(p) + i / Q;
            if constexpr (STREAM) __builtin_nontemporal_store(v, dst);
            else *dst = v;
        }
    }
    // the first n elements (fewer than N), zeros for the others
    __device__ __forceinline__ void load_head(const T *p, int n) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) set_bits(i, p + i);
    }
    __device__ __forceinline__ void store_head(T *p, int n) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) get_bits(i, p + i);
    }
    // min(n, N) elements, none for n <= 0
    template <bool STREAM = false>
    __device__ __forceinline__ void load_upto(const T *p, int64_t n) {
        if (n >= N) load<STREAM>(p);
        else load_head(p, (int)n);
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store_upto(T *p, int64_t n) const {
        if (n >= N) store<STREAM>(p);
        else store_head(p, (int)n);
    }
    template <typename A>
    __device__ __forceinline__ A get(int i) const {
        if constexpr (std::is_same_v<T, bf16_t>)
            return (A)__uint_as_float((i & 1) ? (w[i / 2] & 0xffff0000u) : (w[i / 2] << 16));
        else if constexpr (std::is_same_v<T, float>) return (A)__uint_as_float(w[i]);
        else return (A)__hiloint2double((int)w[2 * i + 1], (int)w[2 * i]);
    }
    template <typename A>
    __device__ __forceinline__ void set_all(const A (&v)[N]) {
        set_some<N>(0, v);
    }
    // elements first .. first + M - 1
    template <int M, typename A>
    __device__ __forceinline__ void set_some(int first, const A (&v)[M]) {
        if constexpr (std::is_same_v<T, bf16_t>) {
#pragma unroll
            for (int i = 0; i < M; i += 2)
                w[(first + i) / 2] =
                    bf16_pair(on_the_way_to_bf16(v[i]), on_the_way_to_bf16(v[i + 1]));
        } else if constexpr (std::is_same_v<T, float>) {
#pragma unroll
            for (int i = 0; i < M; ++i) w[first + i] = __float_as_uint((float)v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < M; ++i) {
                w[2 * (first + i)] = (uint32_t)__double2loint((double)v[i]);
                w[2 * (first + i) + 1] = (uint32_t)__double2hiint((double)v[i]);
            }
        }
    }

private:
    __device__ __forceinline__ void set_bits(int i, const T *p) {
        if constexpr (std::is_same_v<T, bf16_t>)
            w[i / 2] |= (i & 1) ? (uint32_t)p->bits << 16 : (uint32_t)p->bits;
        else if constexpr (std::is_same_v<T, float>) w[i] = __float_as_uint(*p);
        else {
            w[2 * i] = (uint32_t)__double2loint(*p);
            w[2 * i + 1] = (uint32_t)__double2hiint(*p);
        }
    }
    __device__ __forceinline__ void get_bits(int i, T *p) const {
        if constexpr (std::is_same_v<T, bf16_t>)
            p->bits = (uint16_t)((i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
        else *p = get<T>(i);
    }
};

// Elements of one 16-byte access.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, false));
}

// Wave reductions in a fixed order; every lane has the result.
struct OpSum {
    template <typename A>
    __device__ __forceinline__ A operator()(A a, A b) const { return a + b; }
};
struct OpMax {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
    __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); }
};
template <typename A, typename OP>
__device__ __forceinline__ A wave_all(A v, OP op) {
    if constexpr (std::is_same_v<A, float>) {
        v = op(v, dpp_f32<kDppQuadXor1>(v));
        v = op(v, dpp_f32<kDppQuadXor2>(v));
        v = op(v, dpp_f32<kDppRowHalfMirror>(v));
        v = op(v, dpp_f32<kDppRowMirror>(v));
    } else {
        v = op(v, dpp_f64<kDppQuadXor1>(v));
        v = op(v, dpp_f64<kDppQuadXor2>(v));
        v = op(v, dpp_f64<kDppRowHalfMirror>(v));
        v = op(v, dpp_f64<kDppRowMirror>(v));
    }
    v = op(v, __shfl_xor(v, 16, 64));
    v = op(v, __shfl_xor(v, 32, 64));
    return v;
}

}  // namespace ecc
