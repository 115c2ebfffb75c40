// Products of the language-model operators on the matrix cores:
//     C[m, n] = sum over k of A[m, k] B[n, k]
// for operands of bf16 whose rows are contiguous along k, sums in fp32.
//
// fp32 operands take the same path as three pieces of bf16 each (split3), laid
// out as planes: hi + mid + lo is the fp32 value (24 bits in 3 x 8), and the
// six products of pieces down to 2^-16 of the largest (mid mid, hi lo, lo hi,
// hi mid, mid hi, hi hi, in this order) leave out terms of 2^-24 of an
// element's product, below fp32's own rounding.  The loop over k just walks
// the planes one product after another.
//
// The kernel: a workgroup of eight waves holds a tile of BM x BN sums in
// registers, as 16 x 16 blocks.  Steps of 64 along k are brought into LDS by
// direct 16-byte loads; a row of a step is 128 bytes, its 16-byte chunks stored
// at chunk ^ (row & 7), so that no reads of a wave meet in a bank (counted: 0
// conflicts; the loads write LDS lane after lane, so the exchange is in the
// addresses that they read).  Rows behind the last one are read as the last row
// and not stored.  Workgroups go round the eight XCDs, each of which walks a
// contiguous part of the tiles in bands of four tile rows, so that its L2 serves
// the operands of neighbours.
//
// 256 x 256: the waves are two groups, the upper and the lower half of the tile,
// that take turns: while one reads a whole step from LDS into registers, the
// other keeps the matrix cores busy with the step that it has read, and issues
// loads.  A's steps have two buffers (a half is free once its group has read
// it), B's three, all 160 KiB of a CU, so that loads have three or four turns
// to arrive.  8,192^3: 1.26 PFLOP/s, 4,096 x 4,096 x 128,000: 1.37 (zeros, which
// draw less power: 1.56 and 1.66; without loads 2.10).  A plain double buffer
// of both made 1.11 and 1.14, two groups over it 1.21 and 1.20; products of
// 32 x 32 blocks 1.15 and 1.25; loads between the products 1.20 and 1.31.
//
// 128 x 128, four buffers of both, one meeting of the waves a step: for products
// whose large tiles would leave CUs idle.  2,048^2 x 16,384: 0.89 PFLOP/s (four
// waves 0.79).
#pragma once

#include "lm_common.h"

namespace ecc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kGemmK = 64;        // elements along k of one step
constexpr int kGemmGroup = 4;     // tile rows of a band
// Row pitch of an operand, below this: 32-bit offsets reach the rows of a tile.
constexpr int64_t kGemmMaxLd = int64_t(1) << 23;

// Rows of `ld` elements (a multiple of 8, 16-byte aligned), pieces `plane`
// elements apart.
struct GemmOperand {
    const bf16_t *p;
    int64_t ld, plane;
};

struct GemmArgs {
    GemmOperand a, b;
    const bf16_t *b2;      // the second matrix of pairs (Epi::kPair), like b
    int32_t M, N;          // rows of A and of B (of one of the pair)
    int32_t K;             // along k, a multiple of kGemmK: of every batch
    int32_t tiles_m, tiles_n, batches, splits;
    // Batches are ranges along k: [batch * K, + K), or those of the device
    // array ranges (begin, end), cut to [k_lo, k_hi) and counted from k_lo.
    const int2 *ranges;
    int32_t k_lo, k_hi;
    // Rows of A that hold anything, from m_lo on (device; NULL: all): tiles
    // behind them are left out.
    const int32_t *live;
    int32_t m_lo;
    int32_t nprod;         // products of pieces
    int64_t a_piece[6], b_piece[6];  // where each one's pieces begin
};

// The products of operands (set before) of `na` and `nb` pieces, small ones
// first.
inline void set_products(GemmArgs &g, int na, int nb) {
    static const uint8_t both[6][2] = {{1, 1}, {0, 2}, {2, 0}, {0, 1}, {1, 0}, {0, 0}};
    g.nprod = 0;
    for (auto &p : both) {
        if (p[0] >= na || p[1] >= nb) continue;
        g.a_piece[g.nprod] = p[0] * g.a.plane;
        g.b_piece[g.nprod++] = p[1] * g.b.plane;
    }
}

// The same for pieces in registers: f(piece of A, piece of B).
template <int NA, int NB, class F>
__device__ __forceinline__ void products(F &&f) {
    if constexpr (NA > 1 && NB > 1) f(1, 1);
    if constexpr (NB > 2) f(0, 2);
    if constexpr (NA > 2) f(2, 0);
    if constexpr (NB > 1) f(0, 1);
    if constexpr (NA > 1) f(1, 0);
    f(0, 0);
}

// Where a lane's sums lie: acc[i][j][e] is row m + 16 i, column n + 16 j + e
// of the tile's matrix (of pairs: acc[i][j] and acc[i][j + NI / 2] are the
// first's and the second's column n + 16 j + e).
struct GemmTile {
    int32_t m, n;
    int32_t batch, split;
    int32_t k;        // elements along k that the tile has summed
    int32_t tile_n;   // 64-column tile of the wave
    f32x4 *lds;       // 4 KiB of the wave's own
};

// Turns 16 rows of a wave's block round: quads of a column of lanes (v[j]: row
// lane & 15, columns 16 j + 4 (lane / 16)) become rows, f(row, column, quad) for
// NQ neighbouring rows of lanes after each other, so that 16 lanes (NQ = 4: 8
// for NQ = 2) reach a row's 16 NQ columns with one access.  Chunks are stored at
// chunk ^ row, free of conflicts.
template <int NQ, class F>
__device__ __forceinline__ void turn(f32x4 *lds, const f32x4 (&v)[NQ], F &&f) {
    constexpr int CH = NQ * 4;
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
#pragma unroll
    for (int j = 0; j < NQ; ++j) lds[c * CH + ((j * 4 + q) ^ (c & (CH - 1)))] = v[j];
    const int first = lane / CH, chunk = lane % CH;
#pragma unroll
    for (int it = 0; it < NQ; ++it) {
        const int row = it * (64 / CH) + first;
        f(row, chunk * 4, lds[row * CH + (chunk ^ (row & (CH - 1)))]);
    }
}

typedef __attribute__((address_space(3))) void lds_void;

// A value that all lanes share, in a scalar register.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Where the next step of an operand lies; products of pieces follow each other.
// Behind the last step nothing is read, so that loads need no condition.
struct GemmCursor {
    int prod, left, todo;   // steps left of this product, of all
    const bf16_t *next;
    __device__ __forceinline__ int bytes() const { return uniform(~((todo - 1) >> 31)); }
    __device__ __forceinline__ void step(int ksteps, int nprod, const bf16_t *base,
                                         const int64_t *piece) {
        next += kGemmK;
        --todo;
        if (--left == 0) {
            left = ksteps;
            prod = min(prod + 1, nprod - 1);
            next = base + piece[prod];
        }
    }
};
// 16 bytes a lane from base + offset into LDS, lane after lane; zeros where
// `bytes` from base on are none.
__device__ __forceinline__ void load_to_lds(const void *base, int bytes, uint32_t offset,
                                            uint16_t *to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00020000),
        (lds_void *)to, 16, (int)offset, 0, 0, 0);
}

// This wave's direct loads are in LDS; its reads of LDS are in registers.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4 << 14));
}
__device__ __forceinline__ void wait_reads() { __builtin_amdgcn_s_waitcnt(0xc07f); }
// Where all waves of a workgroup meet; nothing moves across.
__device__ __forceinline__ void phase_end() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Blocks go round the XCDs: each takes a contiguous share.
__device__ __forceinline__ int xcd_block(int block, int blocks) {
    const int per = (blocks + 7) >> 3, more = blocks - ((per - 1) << 3);
    const int xcd = block & 7, at = block >> 3;
    return xcd * per + at - max(0, xcd - more);
}

template <int BM, int BN, int WM, int WN, int STAGES, class Epi>
__device__ __forceinline__ void gemm_tile(const GemmArgs &g, const Epi &epi, int block,
                                          int blocks) {
    constexpr int NW = WM * WN;
    constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW;  // loads of 8 rows a wave
    static_assert(BN / WN == 64, "a wave's columns: 64, or 32 of each of a pair");
    // (separate arrays: the compiler tells the loads into one from the reads of
    // another by their names)
    constexpr int kA = BM * kGemmK, kB = BN * kGemmK;
    constexpr bool kThree = BM == 256, kFour = STAGES == 4;
    __shared__ __attribute__((aligned(1024))) uint16_t s_a0[kA], s_a1[kA], s_b0[kB], s_b1[kB],
        s_b2[kThree || kFour ? kB : 8], s_a2[kFour ? kA : 8], s_a3[kFour ? kA : 8],
        s_b3[kFour ? kB : 8];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;

    int t = xcd_block(block, blocks);  // (uniform: from scalars alone)
    const int tiles = g.tiles_m * g.tiles_n;
    const int part = t / tiles;
    t -= part * tiles;
    const int split = uniform(part % g.splits), batch = uniform(part / g.splits);
    const int band = kGemmGroup * g.tiles_n;
    const int first = t / band * kGemmGroup, in = t % band;
    const int rows = min(kGemmGroup, g.tiles_m - first);
    const int tm = uniform(first + in % rows), tn = uniform(in / rows);
    const int m0 = tm * BM, n0 = tn * (Epi::kPair ? BN / 2 : BN);
    if (g.live && m0 + g.m_lo >= uniform(*g.live)) return;

    // the range along k, in steps; this split's share of all products' steps
    int k0 = batch * g.K, k1 = k0 + g.K;
    if (g.ranges) {
        const int2 r = g.ranges[batch];
        k0 = uniform(max(r.x, g.k_lo) - g.k_lo);
        k1 = uniform(max(k0, min(r.y, g.k_hi) - g.k_lo));
    }
    const int ksteps = (k1 - k0) / kGemmK;
    const int all = ksteps * g.nprod;
    const int step = uniform((int)((int64_t)all * split / g.splits));
    const int end = uniform((int)((int64_t)all * (split + 1) / g.splits));

    uint32_t oa[LA], ob[LB];
    const int sub = lane >> 3, chunk = ((lane & 7) ^ sub) * 16;
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int r = min((wave * LA + i) * 8 + sub, g.M - 1 - m0);
        oa[i] = (uint32_t)(r * (int64_t)g.a.ld * 2 + chunk);
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        int r = (wave * LB + i) * 8 + sub;
        if constexpr (Epi::kPair) r = r / 64 * 32 + r % 32;
        r = min(r, g.N - 1 - n0);
        ob[i] = (uint32_t)(r * (int64_t)g.b.ld * 2 + chunk);
    }
    // where the next step lies; the products of pieces follow each other
    const bf16_t *a_base = g.a.p + (int64_t)m0 * g.a.ld + k0;
    const bf16_t *b_base = g.b.p + (int64_t)n0 * g.b.ld + k0;
    if constexpr (Epi::kPair) {
        static_assert(LB == 2 || LB == 4, "a wave loads rows of one of the pair");
        if (wave * LB / 4 & 1) b_base += g.b2 - g.b.p;
    }
    const int prod0 = uniform(ksteps ? step / ksteps : 0);
    GemmCursor at_a{prod0, (prod0 + 1) * ksteps - step, end - step, nullptr}, at_b = at_a;
    at_a.next = a_base + g.a_piece[prod0] + (ksteps - at_a.left) * kGemmK;
    at_b.next = b_base + g.b_piece[prod0] + (ksteps - at_b.left) * kGemmK;

    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    // bring this wave's rows of the next step of A or B into a buffer
    auto load_a = [&](uint16_t *to) {
#pragma unroll
        for (int i = 0; i < LA; ++i)
            load_to_lds(at_a.next, at_a.bytes(), oa[i], to + (wave * LA + i) * 8 * kGemmK);
        at_a.step(ksteps, g.nprod, a_base, g.a_piece);
    };
    auto load_b = [&](uint16_t *to) {
#pragma unroll
        for (int i = 0; i < LB; ++i)
            load_to_lds(at_b.next, at_b.bytes(), ob[i], to + (wave * LB + i) * 8 * kGemmK);
        at_b.step(ksteps, g.nprod, b_base, g.b_piece);
    };
    const int ra = wm * (BM / WM) + (lane & 15), rb = wn * (BN / WN) + (lane & 15);
    const int x = lane & 7, q = lane >> 4;
    struct Held {
        bf16x8 a[2][MI], b[2][NI];
    } f;
    auto read = [&](const uint16_t *sa, const uint16_t *sb) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int c = ((kk * 4 + q) ^ x) * 8;
#pragma unroll
            for (int j = 0; j < NI; ++j)
                f.b[kk][j] = *reinterpret_cast<const bf16x8 *>(sb + (rb + j * 16) * kGemmK + c);
#pragma unroll
            for (int i = 0; i < MI; ++i)
                f.a[kk][i] = *reinterpret_cast<const bf16x8 *>(sa + (ra + i * 16) * kGemmK + c);
        }
    };
    // (B first: a lane then holds four neighbouring columns)
    auto multiply = [&] {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int jj = 0; jj < NI; ++jj) {
                    const int j = i & 1 ? NI - 1 - jj : jj;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.b[kk][j], f.a[kk][i],
                                                                       acc[i][j], 0, 0, 0);
                }
    };
    const int steps = end - step;
    if (steps > 0) {
        if constexpr (BM == 256) {
            const bool late = wave >= 4;
            load_a(s_a0);
            load_b(s_b0);
            if (late) {
                load_b(s_b1);
                load_a(s_a1);
                load_b(s_b2);
            } else {
                load_a(s_a1);
                load_b(s_b1);
            }
            wait_loads<8>();
            phase_end();
            if (late) phase_end();
            auto turn = [&](uint16_t *a, uint16_t *b, uint16_t *b_two) {
                read(a, b);
                wait_reads();
                phase_end();
                load_a(a);
                if (late) load_b(b);
                else load_b(b_two);
                __builtin_amdgcn_s_setprio(1);
                multiply();
                __builtin_amdgcn_s_setprio(0);
                wait_loads<8>();
                phase_end();
            };
            for (int t = 0;;) {
                turn(s_a0, s_b0, s_b2);
                if (++t >= steps) break;
                turn(s_a1, s_b1, s_b0);
                if (++t >= steps) break;
                turn(s_a0, s_b2, s_b1);
                if (++t >= steps) break;
                turn(s_a1, s_b0, s_b2);
                if (++t >= steps) break;
                turn(s_a0, s_b1, s_b0);
                if (++t >= steps) break;
                turn(s_a1, s_b2, s_b1);
                if (++t >= steps) break;
            }
            wait_loads<0>();
            if (!late) phase_end();
        } else if constexpr (STAGES == 2) {
            // (two steps at most)
            load_a(s_a0);
            load_b(s_b0);
            load_a(s_a1);
            load_b(s_b1);
            wait_loads<LA + LB>();
            phase_end();
            read(s_a0, s_b0);
            multiply();
            wait_loads<0>();
            phase_end();
            if (steps > 1) {
                read(s_a1, s_b1);
                multiply();
            }
        } else {
            load_a(s_a0);
            load_b(s_b0);
            load_a(s_a1);
            load_b(s_b1);
            load_a(s_a2);
            load_b(s_b2);
            auto turn = [&](uint16_t *a, uint16_t *b, uint16_t *next_a, uint16_t *next_b) {
                wait_loads<2 * (LA + LB)>();
                phase_end();  // the step is in LDS, and the one before is read
                load_a(next_a);
                load_b(next_b);
                read(a, b);
                multiply();
                wait_reads();
            };
            for (int t = 0;;) {
                turn(s_a0, s_b0, s_a3, s_b3);
                if (++t >= steps) break;
                turn(s_a1, s_b1, s_a0, s_b0);
                if (++t >= steps) break;
                turn(s_a2, s_b2, s_a1, s_b1);
                if (++t >= steps) break;
                turn(s_a3, s_b3, s_a2, s_b2);
                if (++t >= steps) break;
            }
            wait_loads<0>();
        }
    }
    const int n_wave = n0 + wn * (Epi::kPair ? 32 : 64);
    __syncthreads();  // nobody reads LDS any more: 4 KiB of it are the wave's
    f32x4 *lds = reinterpret_cast<f32x4 *>(BM == 256 || wave < 4 ? s_a0 : s_a1) +
                 (BM == 256 ? wave : wave & 3) * 256;
    epi.finish(GemmTile{m0 + ra, n_wave + q * 4, batch, split, k1 - k0, n_wave / 64, lds}, g, acc);
}

template <int BM, int BN, int WM, int WN, int STAGES, class Epi>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm(GemmArgs g, Epi epi) {
    gemm_tile<BM, BN, WM, WN, STAGES>(g, epi, blockIdx.x, gridDim.x);
}

// Tiles of BM x BN (of pairs: BN / 2 columns): their number.
template <int BM, int BN, class Epi>
int64_t set_tiles(GemmArgs &g) {
    g.tiles_m = (g.M + BM - 1) / BM;
    const int cols = Epi::kPair ? BN / 2 : BN;
    g.tiles_n = (g.N + cols - 1) / cols;
    return (int64_t)g.tiles_m * g.tiles_n * g.batches * g.splits;
}
template <int BM, int BN, int WM, int WN, int STAGES, class Epi>
void launch_tile(GemmArgs g, const Epi &epi, hipStream_t s) {
    const int64_t grid = set_tiles<BM, BN, Epi>(g);
    if (grid > 0)
        hipLaunchKernelGGL((k_gemm<BM, BN, WM, WN, STAGES, Epi>), dim3((unsigned)grid),
                           dim3(64 * WM * WN), 0, s, g, epi);
}
template <class Epi>
void launch_large_tiles(const GemmArgs &g, const Epi &epi, hipStream_t s) {
    launch_tile<256, 256, 2, 4, 3>(g, epi, s);
}
template <class Epi>
void launch_small_tiles(const GemmArgs &g, const Epi &epi, hipStream_t s) {
    launch_tile<128, 128, 4, 2, 4>(g, epi, s);
}
template <class Epi>
void launch_short_tiles(const GemmArgs &g, const Epi &epi, hipStream_t s) {
    launch_tile<128, 128, 4, 2, 2>(g, epi, s);
}

// Tiles, and parts along k of a product whose tiles would leave CUs idle (the
// parts are joined by k_gemm_join): what takes the least by the times that a
// round of 256 tiles takes, in us: 1.5 a step and 8 before and after them for
// large tiles, 0.6 and 4 for small ones, and the join at 4 TB/s.  (M x N and
// `steps` of all products, per batch.)  4,136 x 1,001 of 516 steps: 7 parts of
// large tiles, 0.32 ms with their join (the call that holds it 593 us; 590 us by 3
// parts, 619 by 6, 687 by 2, 719 by 4, 994 in one; small tiles 835 us in one).
// Products of one or two steps take short tiles instead: small ones of 64 KiB of
// LDS, two to a CU, so that one's results are written while the other begins.
// 5,000 rows x 2 x 2,178 columns of two steps: 18 us against 25 us; gradients of
// 100,003 x 237 for each of 15 workers, of one: 329 us against 367 us.
struct GemmShape {
    bool large;
    int32_t splits;
    bool brief;
};
constexpr int kShortSteps = 2;
inline GemmShape gemm_shape(int64_t M, int64_t N, int64_t steps, int64_t batches, bool may_split) {
    GemmShape best{false, 1, steps <= kShortSteps};
    if (best.brief) return best;
    double least = 1e30;
    for (int large = 0; large < 2; ++large) {
        const int64_t tile = large ? 256 : 128;
        const int64_t tiles = ((M + tile - 1) / tile) * ((N + tile - 1) / tile) * batches;
        for (int64_t s = 1; s <= 32 && (s == 1 || (may_split && s * 4 <= steps)); ++s) {
            const double rounds = (double)((tiles * s + 255) / 256), part = (double)((steps + s - 1) / s);
            double us = rounds * (large ? 1.5 * part + 8.0 : 0.6 * part + 4.0);
            if (s > 1) us += 4.0 + (double)(s + 1) * batches * M * N * 4.0 / 4e6;
            if (us < least) least = us, best = GemmShape{large != 0, (int32_t)s, false};
        }
    }
    return best;
}
template <class Epi>
void launch_gemm(GemmArgs g, const Epi &epi, hipStream_t s) {
    g.splits = 1;
    const GemmShape shape = gemm_shape(g.M, (int64_t)g.N * (Epi::kPair ? 2 : 1),
                                       (int64_t)g.K / kGemmK * g.nprod, g.batches, false);
    if (shape.brief) launch_short_tiles(g, epi, s);
    else if (shape.large) launch_large_tiles(g, epi, s);
    else launch_small_tiles(g, epi, s);
}

inline int64_t split_bytes(int64_t M, int64_t N, int64_t splits, int64_t batches) {
    return splits > 1 ? splits * batches * M * ((N + 3) & ~int64_t(3)) * 4 : 0;
}
// (grids of fewer than 2^32 threads)
inline bool gemm_in_range(int64_t M, int64_t N, int64_t batches) {
    return (__int128)((M + 127) / 128) * ((N + 127) / 128) * batches < (int64_t(1) << 22);
}

// A plain matrix out of the sums: rows of out (from row `second` on those of
// out2), batches apart, rounded to `type` once, what was there or `sums`
// (fp32, dense) added before; or fp32 parts of a split product.
struct MatrixOut {
    static constexpr bool kPair = false;
    void *out, *out2;
    int64_t ld, batch_stride;
    int32_t type, second;
    int32_t add;              // to what out holds
    int32_t skip_empty;       // batches without a range along k are left alone
    const int32_t *row_map;   // out's row of each row; negative: none
    const float *row_scale;   // the sums' factor, of each row
    const float *scale;       // of each batch
    const float *sums;        // added before (dense)
    float *parts;

    __device__ __forceinline__ void put(const GemmArgs &g, int32_t batch, int32_t m, int32_t n,
                                        f32x4 v) const {
        if (m >= g.M || n >= g.N) return;
        int64_t r = m;
        if (row_map) {
            r = row_map[m];
            if (r < 0) return;
        }
        if (row_scale) v *= row_scale[m];
        if (scale) v *= scale[batch];
        const int w = min(4, g.N - n);
        if (sums) v += load4(sums + ((int64_t)batch * g.M + m) * g.N + n, w);
        char *base = (char *)out;
        if (second && r >= second) {
            base = (char *)out2;
            r -= second;
        }
        const int64_t at = batch * batch_stride + r * ld + n;
        if (type == ECC_F32) {
            float *p = (float *)base + at;
            if (add) v += load4(p, w);
            store4(p, v, w);
        } else {
            bf16_t *p = (bf16_t *)base + at;
            Raw<bf16_t, 4> x;
            if (add) {
                x.load_upto(p, w);
                for (int e = 0; e < 4; ++e) v[e] += x.get<float>(e);
            }
            const float y[4] = {v[0], v[1], v[2], v[3]};
            x.set_all(y);
            x.store_upto(p, w);
        }
    }
    __device__ static __forceinline__ f32x4 load4(const float *p, int w) {
        Raw<float, 4> x;
        x.load_upto(p, w);
        return f32x4{x.get<float>(0), x.get<float>(1), x.get<float>(2), x.get<float>(3)};
    }
    __device__ static __forceinline__ void store4(float *p, f32x4 v, int w) {
        Raw<float, 4> x;
        const float y[4] = {v[0], v[1], v[2], v[3]};
        x.set_all(y);
        x.store_upto(p, w);
    }
    template <int MI, int NI>
    __device__ __forceinline__ void finish(const GemmTile &t, const GemmArgs &g,
                                           f32x4 (&acc)[MI][NI]) const {
        if (parts) {
            const int64_t ld4 = (g.N + 3) & ~3;
            float *p = parts + (int64_t)(t.batch * g.splits + t.split) * g.M * ld4;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
                    if (t.m + 16 * i < g.M && t.n + 16 * j < g.N)
                        *reinterpret_cast<f32x4 *>(p + (t.m + 16 * i) * ld4 + t.n + 16 * j) =
                            acc[i][j];
            return;
        }
        if (skip_empty && t.k == 0) return;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
                put(g, t.batch, t.m + 16 * i, t.n + 16 * j, acc[i][j]);
    }
};

// The same for rows that are the output's own and not split, with what happens
// to each element settled beforehand (large tiles: asked element by element, a
// table gradient of 128,000 x 4,096 takes 3.5 to 3.9 ms per 4,096 rows).
enum { kWrite = 0, kAdd = 1, kFromSums = 2 };  // kFromSums: sums, and out with `add`
template <typename T, int MODE>
struct BlockOut {
    static constexpr bool kPair = false;
    MatrixOut o;
    template <int MI, int NI>
    __device__ __forceinline__ void finish(const GemmTile &t, const GemmArgs &g,
                                           f32x4 (&acc)[MI][NI]) const {
        if (o.skip_empty && t.k == 0) return;
        const float by = o.scale ? o.scale[t.batch] : 1.0f;
        const int32_t m0 = t.m & ~15, n0 = t.n - (threadIdx.x >> 4 & 3) * 4;
        const bool whole = m0 + 16 * MI <= g.M && n0 + 16 * NI <= g.N;
#pragma unroll
        for (int i = 0; i < MI; ++i)
            turn<NI>(t.lds, acc[i], [&](int row, int col, f32x4 v) {
                const int32_t m = m0 + 16 * i + row, n = n0 + col;
                if (whole) put<true>(t, g, m, n, v * by);
                else if (m < g.M && n < g.N) put<false>(t, g, m, n, v * by);
            });
    }
    template <bool WHOLE>
    __device__ __forceinline__ void put(const GemmTile &t, const GemmArgs &g, int32_t m, int32_t n,
                                        f32x4 v) const {
        const bool last = o.second && m >= o.second;
        T *to = (T *)(last ? o.out2 : o.out) + t.batch * o.batch_stride +
                (int64_t)(last ? m - o.second : m) * o.ld + n;
        const int32_t w = g.N - n;
        if (MODE == kFromSums) {
            const float *from = o.sums + ((int64_t)t.batch * g.M + m) * g.N + n;
            Raw<float, 4> sum;
            if (WHOLE) sum.load(from);
            else sum.load_upto(from, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += sum.template get<float>(e);
        }
        if (MODE == kAdd || (MODE == kFromSums && o.add)) {
            Raw<T, 4> old;
            if (WHOLE) old.load(to);
            else old.load_upto(to, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += old.template get<float>(e);
        }
        Raw<T, 4> x;
        const float y[4] = {v[0], v[1], v[2], v[3]};
        x.set_all(y);
        if (WHOLE) x.store(to);
        else x.store_upto(to, w);
    }
};

// Adds the parts of a split product in their order: one thread per four
// columns of a row.
__device__ __forceinline__ void join_parts(const GemmArgs &g, MatrixOut out, int64_t i) {
    const int32_t per_row = (g.N + 3) / 4;
    const int64_t row = i / per_row;
    const int32_t n = (int32_t)(i - row * per_row) * 4;
    const int32_t batch = (int32_t)(row / g.M), m = (int32_t)(row - (int64_t)batch * g.M);
    if (g.live && m + g.m_lo >= *g.live) return;
    if (out.skip_empty && g.ranges) {
        const int2 r = g.ranges[batch];
        if (min(r.y, g.k_hi) <= max(r.x, g.k_lo)) return;
    }
    const int64_t ld4 = (g.N + 3) & ~3;
    const float *p = out.parts + ((int64_t)batch * g.splits * g.M + m) * ld4 + n;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (int32_t s = 1; s < g.splits; ++s)
        v += *reinterpret_cast<const f32x4 *>(p + s * (int64_t)g.M * ld4);
    out.parts = nullptr;
    out.put(g, batch, m, n, v);
}

// A product into a plain matrix, and two of them in one launch: of few tiles
// each, that leave CUs to each other.
struct Product {
    GemmArgs g;
    MatrixOut out;
};
struct TwoProducts {
    Product p[2];
    int64_t first[2];   // blocks, or quads to join, of the first; of both
};
static __global__ __launch_bounds__(512) void k_gemm_two(TwoProducts t) {
    const int second = (int)blockIdx.x >= t.first[0];
    const Product &p = t.p[second];
    const int before = second ? (int)t.first[0] : 0;
    gemm_tile<128, 128, 4, 2, 4>(p.g, p.out, (int)blockIdx.x - before,
                              (int)(second ? t.first[1] : t.first[0]) - before);
}
static __global__ __launch_bounds__(256) void k_gemm_join(TwoProducts t) {
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i < t.first[0]) join_parts(t.p[0].g, t.p[0].out, i);
    else if (i < t.first[1]) join_parts(t.p[1].g, t.p[1].out, i - t.first[0]);
}

inline int64_t quads_to_join(const Product &p) {
    return p.g.splits > 1 ? (int64_t)p.g.batches * p.g.M * ((p.g.N + 3) / 4) : 0;
}

// A product of large or short tiles.
inline void launch_blocks(const Product &p, bool brief, hipStream_t s) {
    const MatrixOut &o = p.out;
    auto tiles = [&](const auto &epi) {
        if (brief) launch_short_tiles(p.g, epi, s);
        else launch_large_tiles(p.g, epi, s);
    };
    auto typed = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        if (o.type == ECC_F32) tiles(BlockOut<float, MODE>{o});
        else tiles(BlockOut<bf16_t, MODE>{o});
    };
    if (o.parts || o.row_map || o.row_scale) tiles(o);
    else if (o.sums) tiles(BlockOut<bf16_t, kFromSums>{o});
    else if (o.add) typed(std::integral_constant<int, kAdd>{});
    else typed(std::integral_constant<int, kWrite>{});
}

// Up to two products (count) of the given shapes, small ones in one launch.
inline void launch_tiles(const Product (&p)[2], int count, const GemmShape (&shape)[2],
                         hipStream_t s) {
    auto small = [&](int i) { return !shape[i].large && !shape[i].brief; };
    if (count == 2 && small(0) && small(1)) {
        TwoProducts t{};
        t.p[0] = p[0];
        t.p[1] = p[1];
        t.first[0] = set_tiles<128, 128, MatrixOut>(t.p[0].g);
        t.first[1] = t.first[0] + set_tiles<128, 128, MatrixOut>(t.p[1].g);
        hipLaunchKernelGGL(k_gemm_two, dim3((unsigned)t.first[1]), dim3(512), 0, s, t);
        return;
    }
    for (int i = 0; i < count; ++i)
        if (small(i)) launch_small_tiles(p[i].g, p[i].out, s);
        else launch_blocks(p[i], shape[i].brief, s);
}

// The same into their matrices; parts: work memory of split_bytes for each.
inline void launch_products(Product (&p)[2], int count, const GemmShape (&shape)[2],
                            float *const (&parts)[2], hipStream_t s) {
    TwoProducts t{};
    int64_t quads[2] = {0, 0};
    for (int i = 0; i < count; ++i) {
        p[i].g.splits = shape[i].splits;
        if (shape[i].splits > 1) p[i].out.parts = parts[i];
        quads[i] = quads_to_join(p[i]);
        t.p[i] = p[i];
    }
    launch_tiles(p, count, shape, s);
    t.first[0] = quads[0];
    t.first[1] = quads[0] + quads[1];
    if (t.first[1] > 0)
        hipLaunchKernelGGL(k_gemm_join, dim3((unsigned)((t.first[1] + 255) / 256)), dim3(256), 0, s,
                           t);
}

// The parts of a split product alone, [split][row][N rounded up to 4].
inline MatrixOut parts_alone(float *parts) {
    MatrixOut out{};
    out.parts = parts;
    return out;
}
// Four columns of a row of them, added in their order.
__device__ __forceinline__ f32x4 sum_of_parts(const float *parts, int32_t splits, int64_t M,
                                              int32_t N, int64_t m, int32_t n) {
    const int64_t ld4 = (N + 3) & ~3;
    const float *p = parts + m * ld4 + n;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (int32_t s = 1; s < splits; ++s)
        v += *reinterpret_cast<const f32x4 *>(p + s * M * ld4);
    return v;
}

}  // namespace ecc
