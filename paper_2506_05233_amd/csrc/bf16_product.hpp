// Products of two bf16 matrices on the matrix cores (gfx950): the tile that a workgroup
// computes, C[m][n] = sum_k A(m, k) B(n, k) in fp32, for operands that lie in memory either row by
// row along k or, transposed, row by row along m or n.
//
// A step is 64 of k.  Its two operand tiles go from memory straight to LDS in 16-byte pieces (no
// registers, no LDS store instructions), into one of two buffers while the other is multiplied,
// so a step needs one barrier.  Pieces are permuted inside their rows so that both the plain and
// the transposing LDS reads touch every bank evenly.  A wave holds its part of C in registers.
#pragma once

#include "mesa_mfma.hpp"

namespace mesa {

constexpr int kStepK = 64;

// A bf16 matrix in memory, or several planes of one, `plane` elements apart.
struct Matrix {
    const uint16_t* p;      // 16-byte aligned
    int64_t ld;             // elements between rows: a multiple of 8, below 2^22
    int64_t plane;
    int64_t rows;           // rows that may be read
    int64_t cols;           // elements of a row that may be read, a multiple of 8
};

// The three bf16 planes that an fp32 value is split into (8 bits each: their sum is the value) make
// six products of planes; the rest is below 2^-24 of the whole.  The smallest come first.
__device__ __forceinline__ int pair_plane_a(int pair) { return (0x012010 >> (4 * (5 - pair))) & 3; }
__device__ __forceinline__ int pair_plane_b(int pair) { return (0x210100 >> (4 * (5 - pair))) & 3; }

// Row swizzle of a tile of `Pieces` 16-byte pieces a row that is read transposed: the 32-byte pairs
// of eight rows that one read takes stand in different banks.
template <int Pieces>
__device__ __forceinline__ int transposed_swizzle(int row)
{
    return (2 * ((row & 3) | ((row >> 1) & 4))) & (Pieces - 2);
}

// One operand's tile: N rows of C (or columns), 64 of k.  Along: the matrix' rows run along k;
// otherwise they run along m or n and there is one for each k.
template <int N, int Threads, bool Along>
struct TileLoad {
    static constexpr int kPieces = N / 8;                     // 16-byte pieces of a row, when not Along
    static constexpr int kEach = N * kStepK / 8 / Threads;    // 16-byte pieces of the tile a thread
    static_assert(kEach >= 1 && N * kStepK / 8 % Threads == 0, "whole pieces a thread");
    const char* base;                                         // of the tile's first row or column
    uint32_t off[kEach];

    __device__ void init(const Matrix& m, int64_t first)
    {
        base = reinterpret_cast<const char*>(Along ? m.p + first * m.ld : m.p + first);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int q = j * Threads + int(threadIdx.x);
            if constexpr (Along) {
                const int row = q / 8, piece = (q % 8) ^ (row % 8);
                const int64_t r = min(int64_t(row), m.rows - 1 - first);      // rows past the end read the last
                off[j] = uint32_t(r * m.ld * 2 + piece * 16);
            } else {
                const int row = q / kPieces, piece = (q % kPieces) ^ transposed_swizzle<kPieces>(row);
                const int64_t c = min(int64_t(piece) * 8, m.cols - 8 - first);
                off[j] = uint32_t(row * m.ld * 2 + c * 2);
            }
        }
    }
    // The tile of k .. k + 63 of a plane to LDS.  Rows of k past the matrix' end read zeros.
    __device__ __forceinline__ void issue(const Matrix& m, int64_t k, int plane, const void* zeros, uint16_t* lds) const
    {
        const char* src = base + (int64_t(plane) * m.plane + (Along ? k : k * m.ld)) * 2;
        uint16_t* dst = lds + int(threadIdx.x) / kWave * (kWave * 8);
        if (Along || k + kStepK <= m.rows) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) load_lds16(src + off[j], dst + j * Threads * 8);
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int row = (j * Threads + int(threadIdx.x)) / kPieces;
                load_lds16(k + row < m.rows ? src + off[j] : static_cast<const char*>(zeros), dst + j * Threads * 8);
            }
        }
    }
    // The operand of 16 rows (or columns) from 16 i on, k = 32 s + 8 g .. + 7 in lane group g.
    __device__ static __forceinline__ bf16x8 operand(const uint16_t* tile, int i, int s, int g, int n)
    {
        if constexpr (Along) {
            return *reinterpret_cast<const bf16x8*>(tile + (16 * i + n) * kStepK + 8 * ((4 * s + g) ^ (n % 8)));
        } else {
#if defined(__HIP_DEVICE_COMPILE__)
            uint2 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = 32 * s + 8 * g + 4 * h + n / 4;
                const uint16_t* src = tile + row * N + 8 * ((2 * i + n % 4 / 2) ^ transposed_swizzle<kPieces>(row)) + 4 * (n % 2);
                half[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src)));
            }
            return __builtin_bit_cast(bf16x8, make_uint4(half[0].x, half[0].y, half[1].x, half[1].y));
#else
            return bf16x8{};
#endif
        }
    }
};

// M x N of C by WM x WN waves.
template <int M_, int N_, int WM_, int WN_>
struct TileShape {
    static constexpr int M = M_, N = N_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * kWave;
    static constexpr int MT = M / WM / 16, NT = N / WN / 16;      // 16 x 16 tiles a wave
    static constexpr int kBuffer = (M + N) * kStepK;              // bf16 elements of one step
    static constexpr int kLds = 2 * kBuffer;
};

template <class S, bool AlongA, bool AlongB>
struct Product {
    using LoadA = TileLoad<S::M, S::kThreads, AlongA>;
    using LoadB = TileLoad<S::N, S::kThreads, AlongB>;

    // One step: the next one's tiles are asked for, this one's are multiplied.  The two buffers are
    // marked as not overlapping: otherwise each LDS read would wait for every load under way.
    __device__ static __forceinline__ void step(const uint16_t* __restrict cur, uint16_t* __restrict next, bool more, const LoadA& la,
                                                const LoadB& lb, const Matrix& a, const Matrix& b, int64_t k, int pair, int pairs,
                                                const void* zeros, int wm, int wn, int g, int n, f32x4 (&acc)[S::MT][S::NT])
    {
        if (more) {
            la.issue(a, k, pairs == 1 ? 0 : pair_plane_a(pair), zeros, next);
            lb.issue(b, k, pairs == 1 ? 0 : pair_plane_b(pair), zeros, next + S::M * kStepK);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 x[S::MT], y[S::NT];
#pragma unroll
            for (int j = 0; j < S::NT; ++j) y[j] = LoadB::operand(cur + S::M * kStepK, wn * S::NT + j, s, g, n);
#pragma unroll
            for (int i = 0; i < S::MT; ++i) x[i] = LoadA::operand(cur, wm * S::MT + i, s, g, n);
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int j = 0; j < S::NT; ++j) acc[i][j] = mfma16(x[i], y[j], acc[i][j]);
        }
    }

    // acc[i][j], lane (g, n), element r: row m0 + (wm MT + i) 16 + 4 g + r, column n0 + (wn NT + j) 16 + n,
    // summed over k0 <= k < k1 (multiples of 64 but for k1, past which the matrices hold zeros) and over
    // the pairs of planes.  After it the LDS is free.
    __device__ static void run(const Matrix& a, int64_t m0, const Matrix& b, int64_t n0, int64_t k0, int64_t k1, int pairs,
                               const void* zeros, uint16_t* lds, f32x4 (&acc)[S::MT][S::NT])
    {
        const int lane = int(threadIdx.x) % kWave, g = lane / 16, n = lane % 16;
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave), wm = wave / S::WN, wn = wave % S::WN;
        LoadA la;
        LoadB lb;
        la.init(a, m0);
        lb.init(b, n0);
#pragma unroll
        for (int i = 0; i < S::MT; ++i)
#pragma unroll
            for (int j = 0; j < S::NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (k1 <= k0) return;
        int64_t k = k0;
        int pair = 0, at = 0;
        la.issue(a, k, pairs == 1 ? 0 : pair_plane_a(0), zeros, lds);
        lb.issue(b, k, pairs == 1 ? 0 : pair_plane_b(0), zeros, lds + S::M * kStepK);
        const int64_t steps = (k1 - k0 + kStepK - 1) / kStepK * pairs;
        for (int64_t i = 0; i < steps; ++i) {
            __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
            __syncthreads();
            k += kStepK;
            if (k >= k1) k = k0, ++pair;
            step(lds + at, lds + (S::kBuffer - at), i + 1 < steps, la, lb, a, b, k, pair, pairs, zeros, wm, wn, g, n, acc);
            at = S::kBuffer - at;
        }
        __syncthreads();
    }
};

// Tiles of C in an order that keeps the workgroups of one XCD, which run about 32 at a time, on a
// block of 8 by 4 tiles: the fewest rows and columns that they can share through their L2.
__device__ __forceinline__ void tile_of(int64_t tiles_m, int64_t tiles_n, int64_t& m, int64_t& n)
{
    constexpr int kGroup = 4;
    const int64_t id = xcd_major_block(int(blockIdx.x), int(gridDim.x));
    const int64_t group = id / (kGroup * tiles_m), in = id - group * (kGroup * tiles_m);
    const int64_t wide = min(int64_t(kGroup), tiles_n - group * kGroup);
    m = in / wide;
    n = group * kGroup + in % wide;
}

}  // namespace mesa
