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
// otherwise they run along m or n and there is one for each k.  Tail: of the latter, the last step
// may have fewer than 64 rows, and reads the last one in the place of the others (whose products
// the other operand's zeros have to take out).
template <int N, int Threads, bool Along, bool Tail>
struct TileLoad {
    static constexpr int kPieces = N / 8;                     // 16-byte pieces of a row, when not Along
    static constexpr int kEach = N * kStepK / 8 / Threads;    // 16-byte pieces of the tile a thread
    static constexpr int kReads = Along ? 1 : 2;              // LDS reads of an operand
    static_assert(kEach >= 1 && N * kStepK / 8 % Threads == 0, "whole pieces a thread");
    static_assert(!(Along && Tail), "rows along k are filled up with zeros");
    const char* base;                                         // of the tile's first row or column
    uint32_t off[kEach];
    uint32_t last[Tail ? kEach : 1];

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
                if constexpr (Tail) last[j] = uint32_t(min(int64_t(row), (m.rows - 1) % kStepK) * m.ld * 2 + c * 2);
            }
        }
    }
    // Where the tile of k .. k + 63 of a plane lies: one address for the workgroup, in scalar registers.
    __device__ __forceinline__ const char* source(const Matrix& m, int64_t k, int plane) const
    {
        const uint64_t at = uint64_t(base + (int64_t(plane) * m.plane + (Along ? k : k * m.ld)) * 2);
        return reinterpret_cast<const char*>(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(at)))) |
                                             uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(at >> 32)))) << 32);
    }
    // Its j-th piece of every thread to LDS.
    __device__ __forceinline__ void issue(const char* src, bool whole, int j, uint16_t* lds) const
    {
        uint16_t* dst = lds + __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave) * (kWave * 8);
        load_lds16(src + (Tail && !whole ? last[Tail ? j : 0] : off[j]), dst + j * Threads * 8);
    }
    __device__ __forceinline__ bool whole(const Matrix& m, int64_t k) const { return !Tail || k + kStepK <= m.rows; }
    // Where lane (g, n) of a wave whose rows (or columns) start at 16 i0 reads in a tile, in elements:
    // that of its i-th 16 rows and half s of the step differ from it in known bits.
    __device__ static __forceinline__ uint32_t lane_at(int i0, int g, int n)
    {
        if constexpr (Along) return uint32_t((16 * i0 + n) * kStepK + 8 * (g ^ (n % 8)));
        const int row = 8 * g + n / 4;
        return uint32_t((row * N + 8 * ((n % 4 / 2) ^ transposed_swizzle<kPieces>(row)) + 4 * (n % 2)) ^ (16 * (i0 % 8))) + 128u * uint32_t(i0 / 8);
    }
    // The operand of 16 rows (or columns), k = 32 s + 8 g .. + 7 in lane group g.
    __device__ static __forceinline__ bf16x8 operand(const uint16_t* tile, uint32_t at, int i, int s)
    {
        if constexpr (Along) {
            return *reinterpret_cast<const bf16x8*>(tile + (at ^ uint32_t(32 * s)) + 16 * i * kStepK);
        } else {
#if defined(__HIP_DEVICE_COMPILE__)
            const uint16_t* src = tile + (at ^ uint32_t(16 * i)) + 32 * s * N;
            uint2 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                half[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src + 4 * h * N)));
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
    static_assert((MT == 8 || 8 % MT == 0) && (NT == 8 || 8 % NT == 0), "a wave's tiles differ in the low three bits of their number");
};

template <class S, bool AlongA, bool AlongB, bool TailA = false>
struct Product {
    using LoadA = TileLoad<S::M, S::kThreads, AlongA, TailA>;
    using LoadB = TileLoad<S::N, S::kThreads, AlongB, false>;
    static constexpr int kLoads = LoadA::kEach + LoadB::kEach;

    struct Operands {
        bf16x8 x[S::MT], y[S::NT];
    };
    struct Where {
        uint32_t a, b;      // lane_at of the two tiles
    };
    // What is asked for next: step after step, pair after pair, and the last one again at the end
    // (so that the loop's loads hang on nothing; nobody reads those).
    struct Next {
        const Matrix &a, &b;
        int64_t k0, k1, k, left;
        int pair, pairs;
        const LoadA& la;
        const LoadB& lb;
        const char *from_a, *from_b;
        bool whole;
        __device__ __forceinline__ void look_up()
        {
            from_a = la.source(a, k, pairs == 1 ? 0 : pair_plane_a(pair));
            from_b = lb.source(b, k, pairs == 1 ? 0 : pair_plane_b(pair));
            whole = la.whole(a, k);
            const bool more = --left > 0, wrap = k + kStepK >= k1;
            if (more) pair += wrap ? 1 : 0, k = wrap ? k0 : k + kStepK;
        }
        __device__ __forceinline__ void issue(int j, uint16_t* tiles) const
        {
            if (j < LoadA::kEach)
                la.issue(from_a, whole, j, tiles);
            else
                lb.issue(from_b, true, j - LoadA::kEach, tiles + S::M * kStepK);
        }
    };

    // One half of a step's products, with what the scheduler would otherwise leave to the end spread
    // under them: the reads of the next half's operands, done before the last quarter of the products, which
    // covers their latency, and (Load) the loads of a later step's tiles.  The lane's places are made
    // opaque, so that those of the single reads are formed next to them, in one instruction each,
    // instead of being held in registers across the loop.
    template <bool Load>
    __device__ static __forceinline__ void half(const Operands& now, Operands& then, const uint16_t* tiles, int s, const Where& w, const Next& next,
                                                uint16_t* free, f32x4 (&acc)[S::MT][S::NT])
    {
        constexpr int kReads = S::NT + S::MT, kGroups = S::MT;
        constexpr int kReadGroups = kGroups * 3 / 4 > 0 ? kGroups * 3 / 4 : 1;
        constexpr int kReadEach = (kReads + kReadGroups - 1) / kReadGroups, kLoadEach = (kLoads + kGroups - 1) / kGroups;
        uint32_t a = w.a, b = w.b;
        asm volatile("" : "+v"(a), "+v"(b));
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
#pragma unroll
            for (int r = i * kReadEach; r < (i + 1) * kReadEach && r < kReads; ++r) {
                if (r < S::NT)
                    then.y[r] = LoadB::operand(tiles + S::M * kStepK, b, r, s);
                else
                    then.x[r - S::NT] = LoadA::operand(tiles, a, r - S::NT, s);
            }
            if constexpr (Load) {
#pragma unroll
                for (int j = i * kLoadEach; j < (i + 1) * kLoadEach && j < kLoads; ++j) next.issue(j, free);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < S::NT; ++j) acc[i][j] = mfma16(now.x[i], now.y[j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // The steps, two buffers in turn.  A step's second half of k is read under the products of its
    // first; then comes the barrier, after which the next step's tiles are there and this one's
    // are free; the next step's first half is read, and the step after it asked for, under the
    // products of the second.  The buffers are marked as not overlapping: otherwise each LDS read would
    // wait for every load under way.
    __device__ static __forceinline__ void steps(uint16_t* __restrict even, uint16_t* __restrict odd, Next& next, int64_t count, const Where& w,
                                                 f32x4 (&acc)[S::MT][S::NT])
    {
        Operands first, second;
        next.look_up();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) next.issue(j, even);
        __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
        __syncthreads();
        next.look_up();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) next.issue(j, odd);
#pragma unroll
        for (int j = 0; j < S::NT; ++j) first.y[j] = LoadB::operand(even + S::M * kStepK, w.b, j, 0);
#pragma unroll
        for (int i = 0; i < S::MT; ++i) first.x[i] = LoadA::operand(even, w.a, i, 0);
        for (int64_t i = 0;; i += 2) {
            half<false>(first, second, even, 1, w, next, nullptr, acc);
            next.look_up();
            __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
            __syncthreads();
            half<true>(second, first, odd, 0, w, next, even, acc);
            if (i + 1 >= count) break;
            half<false>(first, second, odd, 1, w, next, nullptr, acc);
            next.look_up();
            __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
            __syncthreads();
            half<true>(second, first, even, 0, w, next, odd, acc);
            if (i + 2 >= count) break;
        }
        __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
        __syncthreads();
    }

    // acc[i][j], lane (g, n), element r: row m0 + (wm MT + i) 16 + 4 g + r, column n0 + (wn NT + j) 16 + n,
    // summed over k0 <= k < k1 (multiples of 64 but for k1, past which B holds zeros) and over the pairs
    // of planes.  After it the LDS is free.
    __device__ static void run(const Matrix& a, int64_t m0, const Matrix& b, int64_t n0, int64_t k0, int64_t k1, int pairs, uint16_t* lds,
                               f32x4 (&acc)[S::MT][S::NT])
    {
        const int lane = int(threadIdx.x) % kWave;
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
        const Where w{LoadA::lane_at(wave / S::WN * S::MT, lane / 16, lane % 16), LoadB::lane_at(wave % S::WN * S::NT, lane / 16, lane % 16)};
        LoadA la;
        LoadB lb;
        la.init(a, m0);
        lb.init(b, n0);
#pragma unroll
        for (int i = 0; i < S::MT; ++i)
#pragma unroll
            for (int j = 0; j < S::NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (k1 <= k0) return;
        const int64_t count = (k1 - k0 + kStepK - 1) / kStepK * pairs;
        Next next{a, b, k0, k1, k0, count, 0, pairs, la, lb, nullptr, nullptr, true};
        steps(lds, lds + S::kBuffer, next, count, w, acc);
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
