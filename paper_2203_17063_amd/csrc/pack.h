// Operands of the products (gemm.h) out of the caller's matrices: bf16 planes
// whose rows are a multiple of 64 long, 16-byte aligned and padded with zeros,
// in the matrix's own order or transposed.
#pragma once

#include "gemm.h"

namespace ecc {

constexpr int64_t pad64(int64_t n) { return (n + 63) & ~int64_t(63); }

// An fp32 value as three bf16 that add up to it: each the nearest to what the
// ones before leave (8 + 8 + 8 bits and the signs hold all 24).  Values that
// would round to an infinity are cut off instead; infinities and NaN are their
// first piece's.  (Pieces below 2^-133 of values below 2^-117 are lost.)
__device__ __forceinline__ void split3(float v, float (&piece)[3]) {
    float hi = bf16_value(bf16_pair(v, 0.0f) & 0xffffu);
    const uint32_t bits = __float_as_uint(v);
    if (__builtin_isinf(hi)) hi = __uint_as_float(bits & 0xffff0000u);
    float rest = v - hi;
    if ((bits & 0x7f800000u) == 0x7f800000u) rest = 0.0f;  // infinity or NaN
    piece[0] = hi;
    piece[1] = bf16_value(bf16_pair(rest, 0.0f) & 0xffffu);
    piece[2] = rest - piece[1];
}

// Piece `which` of values v as bf16.
template <int N>
__device__ __forceinline__ void set_piece(Raw<bf16_t, N> &x, const float (&v)[N], int which,
                                          bool split) {
    float y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        float p[3] = {v[e], 0.0f, 0.0f};
        if (split) split3(v[e], p);
        y[e] = which == 0 ? p[0] : which == 1 ? p[1] : p[2];
    }
    x.set_all(y);
}

// Where packed rows come from: row_map (negative: zeros), or rows of workers
// padded from n to n_pad rows each.
struct PackArgs {
    const void *src;
    int64_t ld;
    int64_t cols;
    int64_t rows_packed;       // a multiple of 64
    int64_t n, n_pad, total;   // total: source rows
    const int32_t *row_map;
    const int32_t *live;       // row blocks from *live - row0 on are left alone
    int64_t row0;
    int32_t pieces;
    bf16_t *rows;              // [pieces][rows_packed][ld_rows] or NULL
    int64_t ld_rows;           // >= cols, a multiple of 64: zeros up to there
    bf16_t *cols_out;          // [pieces][cols][ld_cols] or NULL
    int64_t ld_cols;
    int64_t plane_rows, plane_cols;
    int32_t col_blocks;
};

constexpr int kTile = 64;  // rows and columns of a block

// A block of 64 x 64 values in LDS, as [column][row].
struct PackTile {
    float v[kTile][kTile + 1];
};

// Writes the block's pieces: `mine[p]` are this thread's 8 columns c8 .. + 7 of
// row p * 32 + r, times by[p] in the transposed order.  Loads and stores are of
// 16 bytes, eight to a row.
__device__ __forceinline__ void write_block(PackTile &s, const float (&mine)[2][8],
                                            const float (&by)[2], int64_t row0,
                                            int64_t col0, int64_t cols, bf16_t *rows,
                                            int64_t ld_rows, int64_t plane_rows, int pieces_rows,
                                            bf16_t *cols_out, int64_t ld_cols, int64_t plane_cols,
                                            int pieces_cols) {
    const int c8 = (threadIdx.x & 7) * 8, r = threadIdx.x >> 3;
    if (rows && col0 + c8 < ld_rows) {
        for (int which = 0; which < pieces_rows; ++which)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                Raw<bf16_t, 8> x;
                set_piece(x, mine[p], which, pieces_rows > 1);
                x.store(rows + which * plane_rows + (row0 + p * 32 + r) * ld_rows + col0 + c8);
            }
    }
    if (!cols_out) return;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) s.v[c8 + e][p * 32 + r] = mine[p][e] * by[p];
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int c = p * 32 + r;
        if (col0 + c >= cols) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s.v[c][c8 + e];
        for (int which = 0; which < pieces_cols; ++which) {
            Raw<bf16_t, 8> x;
            set_piece(x, v, which, pieces_cols > 1);
            x.store(cols_out + which * plane_cols + (col0 + c) * ld_cols + row0 + c8);
        }
    }
}

// A block of 64 x 64, columns first.  Bound by memory: each value is read once
// and written once per layout and piece.
template <typename T>
__device__ __forceinline__ void pack_block(const PackArgs &a, int64_t block) {
    __shared__ PackTile s;
    const int64_t row0 = block / a.col_blocks * kTile;
    const int64_t col0 = block % a.col_blocks * kTile;
    if (a.live && row0 + a.row0 >= *a.live) return;
    const int c8 = (threadIdx.x & 7) * 8, r = threadIdx.x >> 3;
    float mine[2][8];
    const float by[2] = {1.0f, 1.0f};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        int64_t row = row0 + p * 32 + r;
        if (a.row_map) row = a.row_map[row];
        else {
            const int64_t w = row / a.n_pad, i = row - w * a.n_pad;
            row = i < a.n ? w * a.n + i : -1;
            if (row >= a.total) row = -1;
        }
        Raw<T, 8> x;
        x.load_upto((const T *)a.src + (row < 0 ? 0 : row * a.ld) + (row < 0 ? 0 : col0 + c8),
                    row < 0 ? 0 : a.cols - col0 - c8);
#pragma unroll
        for (int e = 0; e < 8; ++e) mine[p][e] = x.template get<float>(e);
    }
    write_block(s, mine, by, row0, col0, a.cols, a.rows, a.ld_rows, a.plane_rows, a.pieces,
                a.cols_out, a.ld_cols, a.plane_cols, a.pieces);
}

// Up to eight matrices in one launch, one after another.
struct PackList {
    PackArgs a[8];
    int32_t count;
    int32_t first[8];   // their first blocks
    int32_t at;         // the launch's first block
};

template <typename T>
static __global__ __launch_bounds__(256) void k_pack(PackList l) {
    const int32_t block = (int32_t)blockIdx.x + l.at;
    int i = 0;
    for (int k = 1; k < l.count; ++k)
        if (block >= l.first[k]) i = k;
    pack_block<T>(l.a[i], block - l.first[i]);
}

// Matrices of one type to pack.
struct Packing {
    PackList l{};
    int64_t blocks = 0;
    void add(PackArgs a) {
        a.col_blocks = (int32_t)((a.cols + kTile - 1) / kTile);
        l.first[l.count] = (int32_t)blocks;
        l.a[l.count++] = a;
        blocks += a.rows_packed / kTile * a.col_blocks;
    }
    void launch(int32_t type, hipStream_t s) {
        // (a launch has fewer than 2^32 threads)
        constexpr int64_t kMost = int64_t(1) << 23;
        for (int64_t at = 0; at < blocks; at += kMost) {
            l.at = (int32_t)at;
            const dim3 grid((unsigned)std::min(kMost, blocks - at));
            if (type == ECC_F32) hipLaunchKernelGGL(k_pack<float>, grid, dim3(256), 0, s, l);
            else hipLaunchKernelGGL(k_pack<bf16_t>, grid, dim3(256), 0, s, l);
        }
    }
};

// Up to this many rows need nothing packed: operands go straight into the matrix
// cores' registers, at any alignment, fp32 split where it is loaded.
constexpr int kFewRows = 64;

// A lane's share of a step along k: 16 bf16, or 8 fp32.
template <typename T>
struct FewStep;
template <>
struct FewStep<bf16_t> {
    static constexpr int kStep = 64, kLane = 16, kFrags = 2, kPieces = 1;
    Raw<bf16_t, 8> raw[2];
    __device__ __forceinline__ void load(const bf16_t *row, int64_t k, int64_t D) {
#pragma unroll
        for (int j = 0; j < 2; ++j) raw[j].load_upto(row + k + j * 8, D - k - j * 8);
    }
    __device__ __forceinline__ void frags(bf16x8 (&f)[2][1]) const {
#pragma unroll
        for (int j = 0; j < 2; ++j) f[j][0] = __builtin_bit_cast(bf16x8, raw[j]);
    }
};
template <>
struct FewStep<float> {
    static constexpr int kStep = 32, kLane = 8, kFrags = 1, kPieces = 3;
    Raw<float, 8> raw;
    __device__ __forceinline__ void load(const float *row, int64_t k, int64_t D) {
        raw.load_upto(row + k, D - k);
    }
    __device__ __forceinline__ void frags(bf16x8 (&f)[1][3]) const {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = raw.get<float>(e);
#pragma unroll
        for (int which = 0; which < 3; ++which) {
            Raw<bf16_t, 8> x;
            set_piece(x, v, which, true);
            f[0][which] = __builtin_bit_cast(bf16x8, x);
        }
    }
};

// Can a product take a bf16 matrix as it lies?
inline bool as_it_lies(const void *p, int64_t ld, int64_t cols, int32_t type) {
    return type == ECC_BF16 && (uintptr_t)p % 16 == 0 && ld % 8 == 0 && cols % 64 == 0 &&
           ld < kGemmMaxLd;
}

}  // namespace ecc
