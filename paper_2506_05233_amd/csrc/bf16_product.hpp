// Products of two bf16 matrices on the matrix cores (gfx950): the tile that a workgroup
// computes, C[m][n] = sum_k A(m, k) B(n, k) in fp32, for operands that lie in memory either row by
// row along k or, transposed, row by row along m or n.  Or of two fp32 matrices, each held as planes
// whose sum it is: three of bf16, six products of which are formed (the others are below 2^-24 of the
// whole), or two of fp16 (22 bits and a sign), three products (the fourth is below 2^-22, and 2^-24 as a
// rule); the latter of rows scaled by a power of two into fp16's range.
//
// A step is 64 of k (of planes: 32).  Its operand tiles go from memory straight to LDS in 16-byte
// pieces (no registers, no LDS store instructions), into one of two buffers while the other is
// multiplied, so a step needs one barrier.  Pieces are permuted inside their rows so that both the
// plain and the transposing LDS reads touch every bank evenly (no conflicts by the counters, but
// for transposed tiles of fewer than 128).  A wave holds its part of C in registers.
//
// What bounds it is the matrix cores' clock under load.  The products 16384 x 50257 x 2048 with
// their exponentials' sums take 2.70 ms, 1250 TFLOP/s, a library's product of the same size alone
// 2.60.  Reading a half step's operands just ahead of its products took 3.20: the reads' latency
// stood between them.
#pragma once

#include "mesa_mfma.hpp"

namespace mesa {

// A matrix of 16-bit values in memory, or planes of one, `plane` elements apart.
struct Matrix {
    const uint16_t* p;      // 16-byte aligned
    int64_t ld;             // elements between rows: a multiple of 8, below 2^22
    int64_t plane;
    int64_t rows;           // rows that may be read
    int64_t cols;           // elements of a row that may be read, a multiple of 8 (along k: of the step)
};

constexpr int step_k(int planes) { return planes == 1 ? 64 : 32; }

// Row swizzle of a tile of `Pieces` 16-byte pieces a row that is read transposed: the 32-byte pairs
// of eight rows that one read takes stand in different banks.
template <int Pieces>
__device__ __forceinline__ int transposed_swizzle(int row)
{
    return (2 * ((row & 3) | ((row >> 1) & 4))) & (Pieces - 2);
}
// and of one whose rows of k are read along: eight rows' pieces stand in different banks.
template <int K>
__device__ __forceinline__ int along_swizzle(int row)
{
    return K == 64 ? row % 8 : (row / 2) % 4;
}

// One operand's tile: N rows of C (or columns), one step of k, all planes.  Along: the matrix' rows
// run along k; otherwise they run along m or n and there is one for each k.  Tail: of the latter,
// the last step may have fewer rows, and reads the last one in the place of the others (whose
// products the other operand's zeros have to take out).
template <int N, int Threads, bool Along, bool Tail, int Planes>
struct TileLoad {
    static constexpr int K = step_k(Planes);
    static constexpr int kRow = Along ? K / 8 : N / 8;        // 16-byte pieces of a row in LDS
    static constexpr int kEach = N * K / 8 / Threads;         // pieces of a plane's tile a thread
    static constexpr int kLoads = kEach * Planes;
    static constexpr int kTile = N * K;                       // elements of a plane's tile
    static_assert(kEach >= 1 && N * K / 8 % Threads == 0, "whole pieces a thread");
    static_assert(!(Along && Tail), "rows along k are filled up with zeros");
    const char* base;                                         // of the tile's first row or column
    uint32_t off[kEach];
    uint32_t last[Tail ? kEach : 1];

    __device__ void init(const Matrix& m, int64_t first)
    {
        base = reinterpret_cast<const char*>(Along ? m.p + first * m.ld : m.p + first);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int q = j * Threads + int(threadIdx.x), row = q / kRow;
            if constexpr (Along) {
                const int piece = (q % kRow) ^ along_swizzle<K>(row);
                const int64_t r = min(int64_t(row), m.rows - 1 - first);      // rows past the end read the last
                off[j] = uint32_t(r * m.ld * 2 + piece * 16);
            } else {
                const int piece = (q % kRow) ^ transposed_swizzle<kRow>(row);
                const int64_t c = min(int64_t(piece) * 8, m.cols - 8 - first);
                off[j] = uint32_t(row * m.ld * 2 + c * 2);
                if constexpr (Tail) last[j] = uint32_t(min(int64_t(row), (m.rows - 1) % K) * m.ld * 2 + c * 2);
            }
        }
    }
    // Where the tile of k .. of a plane lies: one address for the workgroup, in scalar registers.
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
    __device__ __forceinline__ bool whole(const Matrix& m, int64_t k) const { return !Tail || k + K <= m.rows; }
    // Where lane (g, n) of a wave whose rows (or columns) start at 16 i0 reads in a tile, in elements:
    // that of its i-th 16 rows and, of 64 of k, half s differ from it in known bits.
    __device__ static __forceinline__ uint32_t lane_at(int i0, int g, int n)
    {
        if constexpr (Along) return uint32_t((16 * i0 + n) * K + 8 * (g ^ along_swizzle<K>(n)));
        const int row = 8 * g + n / 4;
        return uint32_t((row * N + 8 * ((n % 4 / 2) ^ transposed_swizzle<kRow>(row)) + 4 * (n % 2)) ^ (16 * (i0 % 8))) + 128u * uint32_t(i0 / 8);
    }
    // The operand of 16 rows (or columns), 32 of k (8 g .. + 7 of them in lane group g): half `part` of the
    // step, or its plane, of the tile that starts `tile` elements into a buffer.  One sum for the whole
    // index: through a chain of them the compiler no longer sees which buffer a transposing read is of.
    __device__ static __forceinline__ bf16x8 operand(const uint16_t* buffer, uint32_t tile, uint32_t at, int i, int part)
    {
        const uint32_t from = tile + uint32_t(Planes > 1 ? part * kTile : 0), s = Planes > 1 ? 0u : uint32_t(part);
        if constexpr (Along) {
            return *reinterpret_cast<const bf16x8*>(buffer + (from + uint32_t(16 * i * K) + (at ^ (32u * s))));
        } else {
#if defined(__HIP_DEVICE_COMPILE__)
            uint2 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t* src = buffer + (from + 32u * s * N + uint32_t(4 * h * N) + (at ^ uint32_t(16 * i)));
                half[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src)));
            }
            return __builtin_bit_cast(bf16x8, make_uint4(half[0].x, half[0].y, half[1].x, half[1].y));
#else
            return bf16x8{};
#endif
        }
    }
};

// Tiles of C in an order that keeps the workgroups of one XCD, which run about 32 at a time, on a
// block of 8 by 4 tiles: the fewest rows and columns that they can share through their L2.
// Fewer than 2^31 tiles.
__device__ __forceinline__ void tile_of(int tiles_m, int tiles_n, int& m, int& n)
{
    constexpr int kGroup = 4;
    const int id = xcd_major_block(int(blockIdx.x), tiles_m * tiles_n);
    const int group = id / (kGroup * tiles_m), in = id - group * (kGroup * tiles_m);
    const int wide = min(kGroup, tiles_n - group * kGroup);
    m = in / wide;
    n = group * kGroup + (in - m * wide);
}

// M x N of C by WM x WN waves, from bf16 (Planes 1), or fp32 in two fp16 planes or three bf16 ones.
template <int Planes_, int M_, int N_, int WM_, int WN_>
struct TileShape {
    static constexpr int Planes = Planes_, M = M_, N = N_, WM = WM_, WN = WN_;
    static constexpr int K = step_k(Planes);
    static constexpr int kThreads = WM * WN * kWave;
    static constexpr int MT = M / WM / 16, NT = N / WN / 16;      // 16 x 16 tiles a wave
    static constexpr int kBuffer = (M + N) * K * Planes;          // bf16 elements of one step
    static_assert((MT == 8 || 8 % MT == 0) && (NT == 8 || 8 % NT == 0), "a wave's tiles differ in the low three bits of their number");
};

template <class S, bool AlongA, bool AlongB, bool TailA = false>
struct Product {
    static constexpr int Planes = S::Planes, K = S::K;
    using LoadA = TileLoad<S::M, S::kThreads, AlongA, TailA, Planes>;
    using LoadB = TileLoad<S::N, S::kThreads, AlongB, false, Planes>;
    static constexpr int kLoads = LoadA::kLoads + LoadB::kLoads;
    static constexpr int kB = S::M * K * Planes;                  // where B's tiles start in a buffer

    struct Operands {
        bf16x8 x[S::MT], y[S::NT];
    };
    struct Where {
        uint32_t a, b;      // lane_at of the two tiles
    };

    // What is asked for next: step after step, and the last one again at the end (so that the loop's
    // loads hang on nothing; nobody reads those).
    struct Next {
        const Matrix &a, &b;
        int64_t k, left;
        const LoadA& la;
        const LoadB& lb;
        const char *from_a[Planes], *from_b[Planes];
        bool whole;
        __device__ __forceinline__ void look_up()
        {
#pragma unroll
            for (int p = 0; p < Planes; ++p) from_a[p] = la.source(a, k, p), from_b[p] = lb.source(b, k, p);
            whole = la.whole(a, k);
            if (--left > 0) k += K;
        }
        __device__ __forceinline__ void issue(int j, uint16_t* tiles) const
        {
            if (j < LoadA::kLoads) {
                const int p = j / LoadA::kEach;
                la.issue(from_a[p], whole, j % LoadA::kEach, tiles + p * LoadA::kTile);
            } else {
                const int i = j - LoadA::kLoads, p = i / LoadB::kEach;
                lb.issue(from_b[p], true, i % LoadB::kEach, tiles + kB + p * LoadB::kTile);
            }
        }
    };

    __device__ static __forceinline__ f32x4 matrix(const bf16x8& x, const bf16x8& y, const f32x4& c)
    {
        if constexpr (Planes == 2) {
            typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
        } else {
            return mfma16(x, y, c);
        }
    }

    __device__ static __forceinline__ void read_one(const uint16_t* tiles, int r, int part, uint32_t a, uint32_t b, Operands& o)
    {
        if (r < S::NT)
            o.y[r] = LoadB::operand(tiles, kB, b, r, part);
        else
            o.x[r - S::NT] = LoadA::operand(tiles, 0, a, r - S::NT, part);
    }

    // Products of P pairs of operands, with what the scheduler would otherwise leave to the end spread under
    // them: the reads of the operands after next, done before the last quarter of the products, which covers
    // their latency, and (Load) the loads of a later step's tiles.  The lane's places are made opaque, so
    // that those of the single reads are formed next to them, in one instruction each, instead of being
    // held in registers across the loop.
    template <bool Load, int P>
    __device__ static __forceinline__ void phase(const Operands* const (&px)[P], const Operands* const (&py)[P], Operands& then,
                                                 const uint16_t* tiles, int part, const Where& w, const Next& next, uint16_t* free,
                                                 f32x4 (&acc)[S::MT][S::NT])
    {
        constexpr int kReads = S::NT + S::MT, kGroups = S::MT * P;
        constexpr int kReadGroups = kGroups * 3 / 4 > 0 ? kGroups * 3 / 4 : 1;
        constexpr int kReadEach = (kReads + kReadGroups - 1) / kReadGroups, kLoadEach = (kLoads + kGroups - 1) / kGroups;
        uint32_t a = w.a, b = w.b;
        asm volatile("" : "+v"(a), "+v"(b));
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
#pragma unroll
            for (int r = q * kReadEach; r < (q + 1) * kReadEach && r < kReads; ++r) read_one(tiles, r, part, a, b, then);
            if constexpr (Load) {
#pragma unroll
                for (int j = q * kLoadEach; j < (q + 1) * kLoadEach && j < kLoads; ++j) next.issue(j, free);
            }
            __builtin_amdgcn_sched_barrier(0);
            const int p = q / S::MT, i = q % S::MT;
#pragma unroll
            for (int j = 0; j < S::NT; ++j) acc[i][j] = matrix(px[p]->x[i], py[p]->y[j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    __device__ static __forceinline__ void turn()
    {
        __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
        __syncthreads();
    }

    // A step.  Its operands are read a part (half of its k, or a plane) ahead of their products.  When the last
    // is read comes the barrier, after which the next step's tiles are there and this one's are free; the next
    // step's first part is read, and the step after it asked for, under this one's last products.
    __device__ static __forceinline__ void step(uint16_t* cur, uint16_t* other, Next& next, const Where& w, Operands& first, Operands& later,
                                                Operands& second, Operands& third, f32x4 (&acc)[S::MT][S::NT])
    {
        if constexpr (Planes == 1) {
            phase<false, 1>({&first}, {&first}, second, cur, 1, w, next, nullptr, acc);
            next.look_up();
            turn();
            phase<true, 1>({&second}, {&second}, later, other, 0, w, next, cur, acc);
        } else if constexpr (Planes == 2) {
            phase<false, 1>({&first}, {&first}, second, cur, 1, w, next, nullptr, acc);
            next.look_up();
            turn();
            phase<true, 2>({&first, &second}, {&second, &first}, later, other, 0, w, next, cur, acc);
        } else {
            phase<false, 1>({&first}, {&first}, second, cur, 1, w, next, nullptr, acc);
            phase<false, 3>({&first, &second, &second}, {&second, &first, &second}, third, cur, 2, w, next, nullptr, acc);
            next.look_up();
            turn();
            phase<true, 2>({&first, &third}, {&third, &first}, later, other, 0, w, next, cur, acc);
        }
    }

    // Tile (m, n) of C, summed over k0 <= k < k1 (k0 < k1, multiples of a step but for k1, past which B holds
    // zeros), two buffers in turn: acc[i][j], lane (g, n), element r is row m S::M + (wm MT + i) 16 + 4 g + r,
    // column n S::N + (wn NT + j) 16 + n.  `even` and `odd` are two LDS variables of kBuffer elements (of
    // parts of one, each LDS read would wait for every load under way), and free after it.
    // One workgroup a compute unit that went on from tile to tile with the next one's loads under way was
    // slower (11.45 ms for 11.31 of a training pass over 16384 rows): what the dispatcher balances is worth more.
    __device__ static __forceinline__ void run(const Matrix& a, const Matrix& b, int m, int n, int64_t k0, int64_t k1, uint16_t* even, uint16_t* odd,
                                               f32x4 (&acc)[S::MT][S::NT])
    {
        const int lane = int(threadIdx.x) % kWave;
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
        const Where w{LoadA::lane_at(wave / S::WN * S::MT, lane / 16, lane % 16), LoadB::lane_at(wave % S::WN * S::NT, lane / 16, lane % 16)};
        LoadA la;
        LoadB lb;
        la.init(a, int64_t(m) * S::M);
        lb.init(b, int64_t(n) * S::N);
#pragma unroll
        for (int i = 0; i < S::MT; ++i)
#pragma unroll
            for (int j = 0; j < S::NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int64_t count = (k1 - k0 + K - 1) / K;
        Next next{a, b, k0, count, la, lb, {}, {}, true};
        Operands first, later, second, third;
        next.look_up();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) next.issue(j, even);
        turn();
        next.look_up();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) next.issue(j, odd);
#pragma unroll
        for (int r = 0; r < S::NT + S::MT; ++r) read_one(even, r, 0, w.a, w.b, first);
        for (int64_t i = 0;; i += 2) {
            step(even, odd, next, w, first, later, second, third, acc);
            if (i + 1 >= count) break;
            step(odd, even, next, w, later, first, second, third, acc);
            if (i + 2 >= count) break;
        }
        turn();
    }
};

}  // namespace mesa
