// Softmax cross entropy over a vocabulary with a soft cap on the logits, and its gradient, without
// ever keeping the logits of all rows and the whole vocabulary:
//     z = h . E_v,  l = cap tanh(z / cap),  lse = log sum_v exp(l),  loss = lse - l_target
//     dz = dloss (exp(l - lse) - [v = target]) (1 - (l / cap)^2),  dh = sum_v dz E_v,  dE_v = sum_n dz h_n
//
// Three matrix products of 2 rows vocab width operations each, the logits' one twice, since they are formed again
// for the gradient: to keep them would take 3.3 GB for 16384 rows by 50257 and bf16, which is written and read again in
// about the time that the product takes.  All run on the matrix cores (bf16_product.hpp), and but for few rows
// those are what bounds them.  Forward, a workgroup leaves of its tile two numbers a row, the largest logit and the
// sum of exponentials to it, and a small launch joins them.  Backward, dz is formed a piece of the vocabulary
// at a time and multiplied from both sides while it lies in the last cache.
//
// Training passes over 16384 rows by 50257 of 2048 bf16 channels take 11.3 to 11.8 ms by the clock that the card holds, logits
// 2.74 (1231 TFLOP/s), dz 3.13, dh 2.99, the table's gradient 2.75 and the targets' rests 0.17; over 777 rows by 5003 of
// 768 fp32 ones 186 us.  One row by 50257 of 2048 takes 54 us, which reads its 206 MB at 4.4 TB/s, 256 rows 76.
//
// fp32 is multiplied as parts of 16 bits: the logits of more than 32 rows from two fp16 parts of rows scaled by a power of two (three
// products; the first version took three bf16 parts, six products: 80 us and 38 for 777 rows by 5003 of 768), the
// gradients from three bf16 parts, since a scale of its own for each row stands in the way of sums over rows.
#include <algorithm>
#include <type_traits>

#include "bf16_product.hpp"
#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"
#include "vocab.hpp"
#include "vocab_plan.hpp"

namespace mesa {
namespace {

using namespace vocab;

constexpr float kInf = __builtin_inff();

// Tiles of the three products: rows of the table or channels by rows of h or of the table.  Planes 1:
// bf16; of fp32, 2 (fp16) for the logits and 3 (bf16) for the gradients.  The wide ones fill the registers and most of
// the LDS of a compute unit with one workgroup and feed the matrix cores best; of the middle ones two fit, of the
// narrow ones three to five, whose starts and ends overlap: which is used is a question of how many there are (kCost).
// The thin one is for up to 32 rows, where the table is read once and bounds everything.
template <int Planes>
struct Shapes;
template <>
struct Shapes<1> {
    using Wide = TileShape<1, 256, 256, 2, 4>;
    using Middle = TileShape<1, 128, 128, 2, 2>;
    using Narrow = TileShape<1, 64, 64, 2, 2>;
    using Thin = TileShape<1, 64, 32, 4, 1>;
};
template <>
struct Shapes<2> {
    using Wide = TileShape<2, 128, 256, 2, 4>;
    using Middle = TileShape<2, 128, 128, 2, 2>;
    using Narrow = TileShape<2, 64, 64, 2, 2>;
    using Thin = TileShape<2, 64, 32, 4, 1>;      // by Stream
};
template <>
struct Shapes<3> {
    using Wide = TileShape<3, 128, 256, 2, 4>;
    using Middle = TileShape<3, 128, 128, 2, 4>;
    using Narrow = TileShape<3, 64, 64, 2, 2>;
};

// ------------------------------------------------------------------ operands as the products read them
constexpr int kPackThreads = 256;

struct PackArgs {
    const uint16_t* x;       // [rows] rows of width, stride apart
    int64_t rows, width, stride;
    Tokens targets;          // p null: every row counts; else rows whose target is none come out as zeros
    int64_t vocab;
    uint16_t* out;           // [out_rows, ld]
    int64_t out_rows, ld;
    int64_t again;           // from this row on the rows once more; 0: never
};

// The three parts of an fp32 value, whose sum it is: each the nearest bf16 to what the parts before
// leave, which are exact differences (the first cut off where the nearest would be an infinity).  The
// products of parts that are left out are below 2^-25 of the whole.  An infinity or a NaN stays in the
// first part alone.
__device__ __forceinline__ void three_parts(float x, uint32_t (&p)[3])
{
    const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
    p[0] = pack_bf16(x, 0.0f);
    if (finite && (p[0] & 0x7F80u) == 0x7F80u) p[0] = __float_as_uint(x) >> 16;
    const float a = finite ? x - __uint_as_float(p[0] << 16) : 0.0f;
    p[1] = pack_bf16(a, 0.0f);
    p[2] = pack_bf16(a - __uint_as_float(p[1] << 16), 0.0f);
}

// Eight consecutive values from an address that is aligned to an element only, which vector memory
// instructions take as well.
__device__ __forceinline__ void load8_unaligned(const float* p, float (&x)[8])
{
    typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
    const f32x4_any lo = reinterpret_cast<const f32x4_any*>(p)[0], hi = reinterpret_cast<const f32x4_any*>(p)[1];
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = lo[v], x[v + 4] = hi[v];
}
// bf16 rows as the products read them, eight consecutive channels a thread, out_rows x ld of them; what x
// does not hold is zero.  One or two matrices a launch.  A copy (16384 x 2048 in 23 us, 5.8 TB/s; rows of 1000, whose
// 16-byte pieces are unaligned, 32003 and 3997 of them, 146 MB, in 24).
__global__ void __launch_bounds__(kPackThreads) pack_copy_kernel(PackArgs one, PackArgs two, unsigned blocks_one)
{
    const bool first = blockIdx.x < blocks_one;
    const PackArgs& a = first ? one : two;
    const int64_t i = int64_t(blockIdx.x - (first ? 0 : blocks_one)) * kPackThreads + threadIdx.x;
    const int64_t per = a.ld / 8;
    if (i >= a.out_rows * per) return;
    // fewer than 2^32 threads a launch
    const uint32_t at = uint32_t(i), row32 = at / uint32_t(per);
    const int64_t to = row32, row = a.again > 0 && to >= a.again ? to - a.again : to, c = int64_t(at - row32 * uint32_t(per)) * 8;
    bool counts = row < a.rows;
    if (counts && a.targets.p != nullptr) {
        const int64_t t = token_at(a.targets, row);
        counts = t >= 0 && t < a.vocab;
    }
    uint32_t w[4] = {0, 0, 0, 0};
    if (counts) {
        const uint16_t* src = a.x + row * a.stride + c;
        if (c + 8 <= a.width) {
            typedef uint32_t words_any __attribute__((ext_vector_type(4), aligned(2)));
            const words_any u = *reinterpret_cast<const words_any*>(src);
#pragma unroll
            for (int v = 0; v < 4; ++v) w[v] = u[v];
        } else {
#pragma unroll
            for (int v = 0; v < 8; ++v)
                if (c + v < a.width) w[v / 2] |= uint32_t(src[v]) << (16 * (v % 2));
        }
    }
    *reinterpret_cast<uint4*>(a.out + to * a.ld + c) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Either may have no rows.
hipError_t pack_copy(const PackArgs& one, const PackArgs& two, hipStream_t stream)
{
    const int64_t b1 = ceil_div(one.out_rows * (one.ld / 8), kPackThreads), b2 = ceil_div(two.out_rows * (two.ld / 8), kPackThreads);
    if (b1 + b2 == 0) return hipSuccess;
    if (!grid_fits(b1 + b2, kPackThreads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(pack_copy_kernel, dim3(unsigned(b1 + b2)), dim3(kPackThreads), 0, stream, one, two, unsigned(b1));
    return hipGetLastError();
}

// fp32 rows in planes, a wave a row: two fp16 planes of x 2^-e, e the power of two that brings the row's
// largest magnitude into [2^14, 2^15): of 24 bits the first plane takes 11 and a sign, the second 11 of the 12 that
// are left, so an element down to 2^-16 of the largest is off by 2^-23 of itself at most, a smaller one (whose second
// part is subnormal) by 2^-39 of the largest.  And three bf16 planes, which need no scale and so serve sums along
// either way.
struct RowArgs {
    const float* x;          // [rows] rows of width, stride apart
    int64_t rows, width, stride;
    Tokens targets;          // as in PackArgs
    int64_t vocab;
    uint16_t* halves;        // two planes of [out_rows, ld], or null
    int32_t* exponent;       // of halves, [exponents]: e, and zeros, which whole tiles read
    int64_t exponents;
    uint16_t* parts;         // three planes, or null
    int64_t out_rows, ld;
    // a wave each; neither planes: nothing to do
    int64_t waves() const { return halves != nullptr ? exponents : parts != nullptr ? out_rows : 0; }
};

__device__ __forceinline__ void two_halves(float x, int e, uint32_t& hi, uint32_t& lo)
{
    const float y = __builtin_ldexpf(x, -e);
    const _Float16 h = _Float16(y);
    const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
    const _Float16 l = finite ? _Float16(y - float(h)) : _Float16(0.0f);
    hi = __builtin_bit_cast(uint16_t, h);
    lo = __builtin_bit_cast(uint16_t, l);
}

__global__ void __launch_bounds__(kPackThreads) pack_rows_kernel(RowArgs one, RowArgs two, unsigned blocks_one)
{
    constexpr int kRows = kPackThreads / kWave;
    const bool first = blockIdx.x < blocks_one;
    const RowArgs& a = first ? one : two;
    const int lane = int(threadIdx.x) % kWave;
    const int64_t row = int64_t(blockIdx.x - (first ? 0 : blocks_one)) * kRows + threadIdx.x / kWave;
    if (row >= a.out_rows) {
        if (lane == 0 && a.halves != nullptr && row < a.exponents) a.exponent[row] = 0;
        return;
    }
    bool counts = row < a.rows;
    if (counts && a.targets.p != nullptr) {
        const int64_t t = token_at(a.targets, row);
        counts = t >= 0 && t < a.vocab;
    }
    const float* src = a.x + row * a.stride;
    auto load = [&](int64_t c, float (&x)[8]) {
#pragma unroll
        for (int v = 0; v < 8; ++v) x[v] = 0.0f;
        if (!counts) return;
        if (c + 8 <= a.width) {
            load8_unaligned(src + c, x);
        } else {
#pragma unroll
            for (int v = 0; v < 8; ++v)
                if (c + v < a.width) x[v] = src[c + v];
        }
    };
    int e = 0;
    if (a.halves != nullptr) {
        uint32_t most = 0;       // bits of the largest finite magnitude
        for (int64_t c = int64_t(lane) * 8; c < a.width; c += kWave * 8) {
            float x[8];
            load(c, x);
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                const uint32_t u = abs_bits(x[v]);
                most = u < 0x7F800000u ? max(most, u) : most;
            }
        }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) most = max(most, uint32_t(__shfl_xor(int(most), d)));
        // ilogb of it (of a subnormal by its fraction); a row of zeros is not scaled
        e = most == 0 ? 0 : __builtin_amdgcn_frexp_expf(__uint_as_float(most)) - 1 - 14;
        if (lane == 0) a.exponent[row] = e;
    }
    const int64_t plane = a.out_rows * a.ld;
    for (int64_t c = int64_t(lane) * 8; c < a.ld; c += kWave * 8) {
        float x[8];
        load(c, x);
        uint32_t w[5][4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            uint32_t h0, l0, h1, l1;
            two_halves(x[2 * v], e, h0, l0);
            two_halves(x[2 * v + 1], e, h1, l1);
            w[0][v] = h0 | h1 << 16;
            w[1][v] = l0 | l1 << 16;
            if (a.parts != nullptr) {
                uint32_t p[3], q[3];
                three_parts(x[2 * v], p);
                three_parts(x[2 * v + 1], q);
#pragma unroll
                for (int k = 0; k < 3; ++k) w[2 + k][v] = p[k] | q[k] << 16;
            }
        }
        const int64_t to = row * a.ld + c;
        if (a.halves != nullptr)
#pragma unroll
            for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4*>(a.halves + k * plane + to) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
        if (a.parts != nullptr) {
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(a.parts + k * plane + to) = make_uint4(w[2 + k][0], w[2 + k][1], w[2 + k][2], w[2 + k][3]);
        }
    }
}

// Either may have no rows.
hipError_t pack_rows(const RowArgs& one, const RowArgs& two, hipStream_t stream)
{
    const int64_t b1 = ceil_div(one.waves(), kPackThreads / kWave), b2 = ceil_div(two.waves(), kPackThreads / kWave);
    if (b1 + b2 == 0) return hipSuccess;
    if (!grid_fits(b1 + b2, kPackThreads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(pack_rows_kernel, dim3(unsigned(b1 + b2)), dim3(kPackThreads), 0, stream, one, two, unsigned(b1));
    return hipGetLastError();
}

// ------------------------------------------------------------------ the logits
// tanh(x) and 1 - tanh(x)^2, each to fp32 accuracy relative to itself: with e = exp(-2 |x|) they are
// (1 - e) / (1 + e) and 4 e / (1 + e)^2; near 0, where 1 - e cancels, the series of tanh.
__device__ __forceinline__ float tanh_of(float x, float& slope)
{
    const float y = fabsf(x), e = __builtin_amdgcn_exp2f(-2.0f * kLog2e * y), q = __builtin_amdgcn_rcpf(1.0f + e);
    slope = 4.0f * e * q * q;
    const float s = x * x;
    const float series = y * fmaf(s, fmaf(s, fmaf(s, fmaf(s, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    return copysignf(y < 0.3f ? series : (1.0f - e) * q, x);
}

// The same for |x| <= kNear as x P(x^2), P of degree four: 2^-24.5 of itself by its coefficients (a
// fit that levels the largest relative error), 2^-22.7 as evaluated.  A third of the instructions of the
// general form, and none of the slow ones.  A soft cap is there to hold the few far logits, so waves
// whose logits are all near are the rule; the others evaluate both for 16 rows at a time.
constexpr float kNear = 0.5625f;
struct NearTanh {
    float c[5];      // for z in the place of x = z / cap
    float edge;      // largest |z|
    __device__ explicit NearTanh(float cap)
    {
        const float inv = cap > 0.0f ? 1.0f / cap : 0.0f, q = inv * inv;
        c[0] = 0.99999996002f * inv;
        c[1] = -0.33332697360f * inv * q;
        c[2] = 0.13316993368f * inv * q * q;
        c[3] = -0.05247611788f * inv * q * q * q;
        c[4] = 0.01610694871f * inv * q * q * q * q;
        edge = kNear * cap;
        // powers of a far cap that leave fp32's range, up or down, take the general form
        const float last = inv * q * q * q * q;
        if (!(last > 1e-30f && last < 1e30f)) edge = -1.0f;
    }
    __device__ __forceinline__ float operator()(float z) const
    {
        const float s = z * z;
        return z * fmaf(s, fmaf(s, fmaf(s, fmaf(s, c[4], c[3]), c[2]), c[1]), c[0]);
    }
};

// The form that an element's own magnitude asks for: what a row gets does not hang on its neighbours'.
__device__ __forceinline__ float any_tanh(const NearTanh& near, float z, float inv, float& slope)
{
    const float far = tanh_of(z * inv, slope), y = near(z);
    const bool is_near = fabsf(z) <= near.edge;
    slope = is_near ? fmaf(-y, y, 1.0f) : slope;
    return is_near ? y : far;
}

// Up to this cap exp(l) and sums of them stay far inside fp32's range, whatever l is.
constexpr float kPlainCap = 60.0f;
__device__ __forceinline__ bool plain_cap(float cap) { return cap > 0.0f && cap <= kPlainCap; }

// max over the four 16-lane rows: every lane receives that of its column position
__device__ __forceinline__ float row_pair_max(float v)
{
    const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s16[0]), __uint_as_float(s16[1]));
    const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
}
__device__ __forceinline__ int row_pair_min(int v)
{
    const auto s16 = __builtin_amdgcn_permlane16_swap(uint32_t(v), uint32_t(v), false, false);
    v = min(int(s16[0]), int(s16[1]));
    const auto s32 = __builtin_amdgcn_permlane32_swap(uint32_t(v), uint32_t(v), false, false);
    return min(int(s32[0]), int(s32[1]));
}

struct LogitsArgs {
    Matrix table, h;          // from the piece's first row of the table on
    const float* whole;       // of Stream: the table's rows in fp32, and h is three bf16 planes
    int64_t whole_stride;
    const int32_t* table_e;   // fp16 planes: the exponents that their rows were scaled by (readable up to whole tiles)
    const int32_t* h_e;
    int64_t width;
    int64_t first, vocab;     // the piece's first row; rows of the whole table
    int64_t piece;            // rows of the piece
    int64_t rows;
    int64_t tiles_m, tiles_n;
    Tokens targets;
    float cap;
    // forward: of each tile of the vocabulary, [tile][row]
    float2* part;             // largest logit, sum of exp(logit - that)
    float* best_z;            // largest product and the lowest v that has it, or null
    int32_t* best_v;
    int64_t tile0;            // the piece's first tile
    float* at;                // [rows]: the target's logit, of capped ones its tanh
    // gradient
    const float* lse;
    const float* dloss;
    float* rest;              // [rows], of bf16: what rounding takes off the target's dz
    uint16_t* dz;             // planes of [row][piece], dz_ld elements a row
    int64_t dz_ld, dz_plane, dz_rows;
    bool twice;               // of bf16: what its rounding takes off follows as rows dz_rows ...
};

// Products of scaled rows to those of the rows: column c0 + .. of the piece, row r0 + ... (of what lies past the
// piece or the rows no matter what.)
template <class S>
__device__ __forceinline__ void scale_back(f32x4 (&acc)[S::MT][S::NT], const LogitsArgs& a, int64_t c0, int64_t r0, int g, int n)
{
    int rows[S::NT];
#pragma unroll
    for (int j = 0; j < S::NT; ++j) rows[j] = a.h_e[r0 + 16 * j + n];
#pragma unroll
    for (int i = 0; i < S::MT; ++i) {
        const int4 e = *reinterpret_cast<const int4*>(a.table_e + c0 + 16 * i + 4 * g);
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
            acc[i][j] = f32x4{__builtin_ldexpf(acc[i][j][0], e.x + rows[j]), __builtin_ldexpf(acc[i][j][1], e.y + rows[j]),
                              __builtin_ldexpf(acc[i][j][2], e.z + rows[j]), __builtin_ldexpf(acc[i][j][3], e.w + rows[j])};
    }
}

// The fp32 product of the thin tile: few rows of h against a table that is read once, as it lies, which bounds it.  A wave
// holds 16 rows of the table; a lane (g, n) loads the pieces of 8 channels of row n that it multiplies itself, 128
// channels ahead, and parts them into three bf16 in registers (six products).  h's parts come through LDS, 128
// channels at a time; they are asked for before the table's, so that waiting for them leaves those under way, and so
// does the barrier, which waits for LDS only.  One row by 50257 of 2048 channels takes 119 us (412 MB, 3.5 TB/s), where
// a copy of the table in fp16 parts ahead of the tiled product took 318: three times the bytes.  (Few bf16 rows keep
// the tiled product: loads to registers like these took 53.4 us there for 52.6.)
struct Stream {
    static constexpr int K = 128, kRows = 32, kPieces = K / 8, kSteps = K / 32, kEach = kRows * kPieces / 256;
    static constexpr int kBuffer = 3 * kRows * K;
    typedef float floats_any __attribute__((ext_vector_type(4), aligned(4)));
    struct Piece {
        floats_any lo, hi;
    };
    __device__ static __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
    // h: three planes, zeros past the width up to a multiple of 64
    __device__ static __forceinline__ void run(const float* table, int64_t stride, int64_t rows, int64_t width, const Matrix& h, int64_t m0,
                                               uint16_t* even, uint16_t* odd, f32x4 (&acc)[1][2])
    {
        const int t = int(threadIdx.x), lane = t % kWave, g = lane / 16, n = lane % 16;
        const float* row = table + min(m0 + t / kWave * 16 + n, rows - 1) * stride + 8 * g;      // rows past the end read the last
        const int column = t % kPieces * 8;
        const uint16_t* from[kEach];
        int to[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = (j * 256 + t) / kPieces;
            from[j] = h.p + min(int64_t(r), h.rows - 1) * h.ld + column;
            to[j] = r * K + 8 * ((t % kPieces) ^ (r & 15));      // sixteen rows' pieces stand in different banks
        }
        // past the end the last piece, in whose place zeros are put
        auto load_h = [&](int64_t k, uint4 (&x)[3][kEach]) {
            const int64_t at = min(k, h.cols - 8 - column);
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int j = 0; j < kEach; ++j) x[p][j] = *reinterpret_cast<const uint4*>(from[j] + p * h.plane + at);
        };
        auto put = [&](int64_t k, const uint4 (&x)[3][kEach], uint16_t* lds) {
            const bool there = k + column < h.cols;
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    *reinterpret_cast<uint4*>(lds + p * kRows * K + to[j]) =
                        make_uint4(there ? x[p][j].x : 0, there ? x[p][j].y : 0, there ? x[p][j].z : 0, there ? x[p][j].w : 0);
        };
        auto load_table = [&](int64_t k, Piece (&x)[kSteps]) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) x[s] = *reinterpret_cast<const Piece*>(row + k + 32 * s);
        };
        f32x4 low[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        auto multiply = [&](const Piece (&x)[kSteps], const uint16_t* lds) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint32_t w[3][4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    uint32_t p[3], q[3];
                    three_parts(v < 2 ? x[s].lo[2 * v] : x[s].hi[2 * v - 4], p);
                    three_parts(v < 2 ? x[s].lo[2 * v + 1] : x[s].hi[2 * v - 3], q);
#pragma unroll
                    for (int k = 0; k < 3; ++k) w[k][v] = p[k] | q[k] << 16;
                }
                bf16x8 a[3];
#pragma unroll
                for (int k = 0; k < 3; ++k) a[k] = __builtin_bit_cast(bf16x8, make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint16_t* src = lds + (16 * j + n) * K + 8 * ((4 * s + g) ^ n);
                    bf16x8 b[3];
#pragma unroll
                    for (int k = 0; k < 3; ++k) b[k] = *reinterpret_cast<const bf16x8*>(src + k * kRows * K);
                    // the small products apart: what is added to the large sum is rounded at its size each time
                    f32x4& c = low[j];
                    c = mfma16(a[0], b[2], c);
                    c = mfma16(a[2], b[0], c);
                    c = mfma16(a[1], b[1], c);
                    c = mfma16(a[0], b[1], c);
                    c = mfma16(a[1], b[0], c);
                    acc[0][j] = mfma16(a[0], b[0], acc[0][j]);
                }
            }
        };
        acc[0][0] = acc[0][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int64_t whole = width / K * K;
        uint4 parts[3][kEach];
        Piece one[kSteps], two[kSteps];
        uint16_t *now = even, *then = odd;
        load_h(0, parts);
        if (whole > 0) load_table(0, one);
        put(0, parts, now);
        barrier();
        for (int64_t k = 0; k < whole; k += K) {
            // past the last whole step: h's rest, and the first step again, which nobody uses
            load_h(k + K, parts);
            load_table(k + K < whole ? k + K : 0, two);
            multiply(one, now);
            put(k + K, parts, then);
            barrier();
#pragma unroll
            for (int s = 0; s < kSteps; ++s) one[s] = two[s];
            uint16_t* x = now;
            now = then, then = x;
        }
        if (whole < width) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const int64_t c = whole + 32 * s + v;
                    const float y = c + 8 * g < width ? row[c] : 0.0f;
                    if (v < 4)
                        one[s].lo[v] = y;
                    else
                        one[s].hi[v - 4] = y;
                }
            multiply(one, now);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[0][j] += low[j];
        barrier();
    }
};

// One tile of the vocabulary against one of the rows; of every row the tile's largest logit and its
// sum of exponentials to that, which the next kernel joins over the tiles.  A cap of up to 60 bounds the logits, and
// exp(l) is summed as it is.  The products are 48 of a wide tile's 57 us at 2048 channels; the other 9, its first loads
// and its exponentials, nothing overlaps, since no second workgroup fits (fewer vector instructions there changed
// 0.1 to 0.4 percent).
template <class S>
__global__ void __launch_bounds__(S::kThreads) logits_kernel(LogitsArgs a)
{
    constexpr bool kStream = std::is_same_v<S, Shapes<2>::Thin>;
    constexpr int kBuffer = kStream ? Stream::kBuffer : S::kBuffer;
    __shared__ __attribute__((aligned(16))) uint16_t even[kBuffer], odd[kBuffer];
    int tm, tn;
    tile_of(int(a.tiles_m), int(a.tiles_n), tm, tn);
    f32x4 acc[S::MT][S::NT];
    if constexpr (kStream)
        Stream::run(a.whole, a.whole_stride, a.piece, a.width, a.h, int64_t(tm) * S::M, even, odd, acc);
    else
        Product<S, true, true>::run(a.table, a.h, tm, tn, 0, a.width, even, odd, acc);

    float* red = reinterpret_cast<float*>(even);
    const int64_t m0 = int64_t(tm) * S::M, n0 = int64_t(tn) * S::N;
    const int lane = int(threadIdx.x) % kWave, g = lane / 16, n = lane % 16;
    const int wave = int(threadIdx.x) / kWave, wm = wave / S::WN, wn = wave % S::WN;
    const int64_t v0 = a.first + m0 + wm * S::MT * 16;      // the wave's first row of the table
    const int here = int(min(a.first + a.piece - v0, int64_t(S::MT * 16)));     // its rows that exist (0 or less: none)
    if constexpr (S::Planes == 2 && !kStream) scale_back<S>(acc, a, m0 + wm * S::MT * 16, n0 + wn * S::NT * 16, g, n);
    float* red_m = red;           // [WM][N]
    float* red_s = red_m + S::WM * S::N;
    float* red_z = red_s + S::WM * S::N;
    int* red_v = reinterpret_cast<int*>(red_z + S::WM * S::N);

    if (a.best_z != nullptr) {
#pragma unroll
        for (int j = 0; j < S::NT; ++j) {
            float top = -kInf;
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, 16 * i + 4 * g + r < here ? acc[i][j][r] : -kInf);
            top = row_pair_max(top);
            int who = INT32_MAX;
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int v = 16 * i + 4 * g + r;
                    if (v < here && acc[i][j][r] == top) who = min(who, v);
                }
            who = row_pair_min(who);
            if (g == 0) {
                red_z[wm * S::N + (wn * S::NT + j) * 16 + n] = top;
                red_v[wm * S::N + (wn * S::NT + j) * 16 + n] = who == INT32_MAX ? who : int(v0) + who;
            }
        }
    }
    const bool plain = plain_cap(a.cap);        // then nothing has to be taken off the logits
    const float to_power = a.cap * kLog2e;      // tanh to the power of 2
    const NearTanh near(a.cap);
    const float inv = a.cap > 0.0f ? 1.0f / a.cap : 0.0f;
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
        const int64_t row = n0 + (wn * S::NT + j) * 16 + n;
        if (a.cap > 0.0f) {
            float far = 0.0f;
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) far = fmaxf(far, fabsf(acc[i][j][r]));
            if (!__any(far > near.edge)) {
#pragma unroll
                for (int i = 0; i < S::MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] = near(acc[i][j][r]);
            } else {
                float slope;
#pragma unroll
                for (int i = 0; i < S::MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] = any_tanh(near, acc[i][j][r], inv, slope);
            }
        }
        if (a.at != nullptr) {
            const int64_t t = row < a.rows ? token_at(a.targets, row) - v0 : -1;
            if (__any(t >= 0 && t < here)) {
#pragma unroll
                for (int i = 0; i < S::MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * i + 4 * g + r == t && t < here) a.at[row] = acc[i][j][r];
            }
        }
        if (here < S::MT * 16) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * i + 4 * g + r >= here) acc[i][j][r] = -kInf;
        }
        float top = 0.0f, sum = 0.0f;
        if (plain) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(acc[i][j][r] * to_power);
        } else {
            if (a.cap > 0.0f) {
#pragma unroll
                for (int i = 0; i < S::MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] *= a.cap;
            }
            top = -kInf;
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[i][j][r]);
            top = row_pair_max(top);
            // where every logit is -infinity (or there is none) the sum is 0, whatever they are taken to
            const float base = top == -kInf ? 0.0f : top;
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * kLog2e);
        }
        sum = row_pair_sums(sum);
        if (g == 0) {
            red_m[wm * S::N + (wn * S::NT + j) * 16 + n] = top;
            red_s[wm * S::N + (wn * S::NT + j) * 16 + n] = sum;
        }
    }
    __syncthreads();
    const int t = int(threadIdx.x);
    if (t < S::N && n0 + t < a.rows) {
        float top = red_m[t];
#pragma unroll
        for (int w = 1; w < S::WM; ++w) top = fmaxf(top, red_m[w * S::N + t]);
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < S::WM; ++w) {
            const float m = red_m[w * S::N + t];
            sum += red_s[w * S::N + t] * (m == top ? 1.0f : __builtin_amdgcn_exp2f((m - top) * kLog2e));
        }
        const int64_t to = (a.tile0 + tm) * a.rows + n0 + t;
        a.part[to] = make_float2(top, sum);
        if (a.best_z != nullptr) {
            float z = red_z[t];
            int v = red_v[t];
#pragma unroll
            for (int w = 1; w < S::WM; ++w) {
                const float zw = red_z[w * S::N + t];
                const int vw = red_v[w * S::N + t];
                if (zw > z || (zw == z && vw < v)) z = zw, v = vw;
            }
            a.best_z[to] = z;
            a.best_v[to] = v;
        }
    }
}

// The tiles' sums joined, in a fixed order: Rows rows a workgroup, 256 / Rows threads for the tiles of each.  Latency
// at all sizes: 4 to 5 us for up to 4000 rows, 9 for 16384 (26 MB).
struct JoinArgs {
    const float2* part;
    const float* best_z;
    const int32_t* best_v;
    const float* at;
    Tokens targets;
    float cap;
    int64_t rows, vocab, tiles;
    float* loss;
    float* lse;
    int32_t* best;
};
constexpr int kJoinThreads = 256, kJoinDepth = 4;

template <int Rows>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(JoinArgs a)
{
    constexpr int kSlices = kJoinThreads / Rows;
    __shared__ float2 red[kJoinThreads];
    __shared__ float red_z[kJoinThreads];
    __shared__ int red_v[kJoinThreads];
    const int r = int(threadIdx.x) % Rows, slice = int(threadIdx.x) / Rows;
    const int64_t row = int64_t(blockIdx.x) * Rows + r;
    float top = -kInf, sum = 0.0f, z = -kInf;
    int v = INT32_MAX;
    auto add = [&](float2 p) {
        const float m = fmaxf(top, p.x);
        // of what is all -infinity the sums are 0, or NaN
        const float before = top == m ? 1.0f : __builtin_amdgcn_exp2f((top - m) * kLog2e);
        sum = sum * before + p.y * (p.x == m ? 1.0f : __builtin_amdgcn_exp2f((p.x - m) * kLog2e));
        top = m;
    };
    auto better = [&](float zt, int vt) {
        if (zt > z || (zt == z && vt < v)) z = zt, v = vt;
    };
    if (row < a.rows) {
        for (int64_t t = slice; t < a.tiles; t += kSlices * kJoinDepth) {
            float2 p[kJoinDepth];
#pragma unroll
            for (int k = 0; k < kJoinDepth; ++k) p[k] = t + k * kSlices < a.tiles ? a.part[(t + k * kSlices) * a.rows + row] : make_float2(-kInf, 0.0f);
#pragma unroll
            for (int k = 0; k < kJoinDepth; ++k) add(p[k]);
            if (a.best != nullptr) {
#pragma unroll
                for (int k = 0; k < kJoinDepth; ++k)
                    if (t + k * kSlices < a.tiles) better(a.best_z[(t + k * kSlices) * a.rows + row], a.best_v[(t + k * kSlices) * a.rows + row]);
            }
        }
    }
#pragma unroll
    for (int half = kSlices / 2; half > 0; half /= 2) {
        red[threadIdx.x] = make_float2(top, sum);
        red_z[threadIdx.x] = z;
        red_v[threadIdx.x] = v;
        __syncthreads();
        if (slice < half) {
            const int other = int(threadIdx.x) + half * Rows;
            add(red[other]);
            better(red_z[other], red_v[other]);
        }
        __syncthreads();
    }
    if (slice != 0 || row >= a.rows) return;
    float lse = top + kLn2 * __builtin_amdgcn_logf(sum), loss = 0.0f;
    if (a.loss != nullptr) {
        const int64_t t = token_at(a.targets, row);
        if (t >= 0 && t < a.vocab) {
            // A small loss is the difference of two numbers that are not: it is formed from the sum in units of the
            // target's own exponential (to which the sum's element of it is equal), to some 2^-22, and lse from it
            // with one rounding.  The backward pass takes the same tanh, so its 1 - p is off by lse's rounding only.
            const float cap = a.cap > 0.0f ? a.cap : 1.0f, l = cap * a.at[row];
            const float away = plain_cap(a.cap) ? -a.at[row] * (cap * kLog2e) : (top - l) * kLog2e;
            const float q = sum * __builtin_amdgcn_exp2f(away);
            loss = lse - l;
            if (q < 8.0f) {
                loss = fmaxf(log1pf(q - 1.0f), 0.0f);
                lse = fmaf(cap, a.at[row], loss);
            }
        }
        a.loss[row] = loss;
    }
    a.lse[row] = lse;
    if (a.best != nullptr) a.best[row] = v == INT32_MAX ? -1 : v;
}

// ------------------------------------------------------------------ the gradient
// dz of one tile, from the same product: 503 us for 16384 rows by 8192 of 2048 channels (1093 TFLOP/s), of which the
// product alone is some 440; the rest are its exponentials and 268 MB written.
template <class S>
__global__ void __launch_bounds__(S::kThreads) logits_grad_kernel(LogitsArgs a)
{
    constexpr bool kStream = std::is_same_v<S, Shapes<2>::Thin>;
    constexpr int kBuffer = kStream ? Stream::kBuffer : S::kBuffer;
    __shared__ __attribute__((aligned(16))) uint16_t even[kBuffer], odd[kBuffer];
    int tm, tn;
    tile_of(int(a.tiles_m), int(a.tiles_n), tm, tn);
    f32x4 acc[S::MT][S::NT];
    if constexpr (kStream)
        Stream::run(a.whole, a.whole_stride, a.piece, a.width, a.h, int64_t(tm) * S::M, even, odd, acc);
    else
        Product<S, true, true>::run(a.table, a.h, tm, tn, 0, a.width, even, odd, acc);

    const int64_t m0 = int64_t(tm) * S::M, n0 = int64_t(tn) * S::N;
    const int lane = int(threadIdx.x) % kWave, g = lane / 16, n = lane % 16;
    const int wave = int(threadIdx.x) / kWave, wm = wave / S::WN, wn = wave % S::WN;
    const int64_t c0 = m0 + wm * S::MT * 16;                // the wave's first column of dz
    const int here = int(min(a.piece - c0, int64_t(S::MT * 16)));
    if constexpr (S::Planes == 2 && !kStream) scale_back<S>(acc, a, c0, n0 + wn * S::NT * 16, g, n);
    const float inv = a.cap > 0.0f ? 1.0f / a.cap : 0.0f, cap = a.cap > 0.0f ? a.cap : 1.0f;
    const NearTanh near(a.cap);
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
        const int64_t row = n0 + (wn * S::NT + j) * 16 + n;
        int64_t t = -1;
        bool counts = false;
        float lse = 0.0f, up = 0.0f;
        if (row < a.rows) {
            t = token_at(a.targets, row);
            counts = t >= 0 && t < a.vocab;
            if (counts) lse = a.lse[row], up = a.dloss[row];
        }
        const int64_t to = t - a.first - c0;
        const int mine = t < a.vocab && to >= 0 && to < here ? int(to) : -1;
        float far = 0.0f;
#pragma unroll
        for (int i = 0; i < S::MT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) far = fmaxf(far, fabsf(acc[i][j][r]));
        const bool all_near = a.cap > 0.0f && !__any(far > near.edge), target = __any(mine >= 0);
        // dz in the place of z: of near logits without a target among them tanh, its slope 1 - tanh^2 (at least
        // 0.68, so nothing cancels), exp and two products; else the target's element gets its -1 in place
        if (all_near && !target) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float y = near(acc[i][j][r]);
                    acc[i][j][r] = __builtin_amdgcn_exp2f(fmaf(y, cap, -lse) * kLog2e) * (fmaf(-y, y, 1.0f) * up);
                }
        } else {
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float slope = 1.0f, y = acc[i][j][r];
                    if (a.cap > 0.0f) y = any_tanh(near, y, inv, slope);
                    const float p = __builtin_amdgcn_exp2f(fmaf(y, cap, -lse) * kLog2e);
                    acc[i][j][r] = (16 * i + 4 * g + r == mine ? p - 1.0f : p) * (slope * up);
                }
        }
        if (here < S::MT * 16) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * i + 4 * g + r >= here) acc[i][j][r] = 0.0f;
        }
        // rows that do not count, and those that fill up the last step of 64: h is copied as zeros there, but the products
        // of those with an infinity or a NaN of the table are not 0
        if (!__all(counts)) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = counts ? acc[i][j][r] : 0.0f;
        }
        if (row >= a.dz_rows) continue;
        uint16_t* dst = a.dz + row * a.dz_ld + c0 + 4 * g;
        // Rounded to bf16 once for both products: 2^-8 of an element at most, at random over the sums.  But for the
        // target's, as large as all others of its row together: what its rounding takes off is kept, and both get it back.
        if constexpr (S::Planes == 1) {
            if (target) {
#pragma unroll
                for (int i = 0; i < S::MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * i + 4 * g + r == mine) a.rest[row] = acc[i][j][r] - __uint_as_float(pack_bf16(acc[i][j][r], 0.0f) << 16);
            }
#pragma unroll
            for (int i = 0; i < S::MT; ++i)
                *reinterpret_cast<uint2*>(dst + 16 * i) = make_uint2(pack_bf16(acc[i][j][0], acc[i][j][1]), pack_bf16(acc[i][j][2], acc[i][j][3]));
            if (a.twice) {
                auto left = [](float x) { return x - __uint_as_float(pack_bf16(x, 0.0f) << 16); };
#pragma unroll
                for (int i = 0; i < S::MT; ++i)
                    *reinterpret_cast<uint2*>(dst + a.dz_rows * a.dz_ld + 16 * i) =
                        make_uint2(pack_bf16(left(acc[i][j][0]), left(acc[i][j][1])), pack_bf16(left(acc[i][j][2]), left(acc[i][j][3])));
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::MT; ++i) {
                uint32_t p[4][3];
#pragma unroll
                for (int r = 0; r < 4; ++r) three_parts(acc[i][j][r], p[r]);
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    *reinterpret_cast<uint2*>(dst + k * a.dz_plane + 16 * i) = make_uint2(p[0][k] | p[1][k] << 16, p[2][k] | p[3][k] << 16);
                    // the other rows of the step of 64 that the table's gradient takes
                    if constexpr (kStream) *reinterpret_cast<uint2*>(dst + k * a.dz_plane + 32 * a.dz_ld + 16 * i) = make_uint2(0, 0);
                }
            }
        }
    }
}

// What a gradient's rows get at the end.  Of dh (targets.p not null), zeros where the target is none, else rest times
// their target's row of the table added (rest null: nothing).  Of the table (at not null), row at[row] - 1 of
// `sums` added, where at[row] is not 0: the sum of rest_n h_n over the rows n whose target it is.
struct Finish {
    Tokens targets;
    int64_t vocab;
    const float* rest;
    const uint16_t* table;
    int64_t table_stride;
    const float* sums;
    int64_t sums_ld;
    const int32_t* at;
};
__device__ __forceinline__ const float* sums_of(const Finish& f, int32_t at)
{
    return at > 0 ? f.sums + int64_t(at - 1) * f.sums_ld : nullptr;
}
struct RowEnd {
    bool counts;
    float rest;
    const uint16_t* target;      // its row of the table, or null
    __device__ RowEnd(const Finish& f, int64_t row) : counts(true), rest(0.0f), target(nullptr)
    {
        if (f.targets.p == nullptr) return;
        const int64_t t = token_at(f.targets, row);
        counts = t >= 0 && t < f.vocab;
        if (!counts || f.rest == nullptr) return;
        rest = f.rest[row];
        target = f.table + t * f.table_stride;
    }
    // Its channels m .. m + 3 (n of them exist) as they lie, and added to a sum.
    __device__ __forceinline__ uint2 load(int64_t m, int n) const
    {
        typedef uint32_t words_any __attribute__((ext_vector_type(2), aligned(2)));
        if (target == nullptr || n <= 0) return make_uint2(0, 0);
        if (n == 4) {
            const words_any w = *reinterpret_cast<const words_any*>(target + m);
            return make_uint2(w[0], w[1]);
        }
        return make_uint2(target[m] | (n > 1 ? uint32_t(target[m + 1]) << 16 : 0u), n > 2 ? target[m + 2] : 0u);
    }
    __device__ __forceinline__ f32x4 add(const f32x4& y, uint2 w) const
    {
        if (!counts) return f32x4{0.f, 0.f, 0.f, 0.f};
        return f32x4{fmaf(rest, __uint_as_float(w.x << 16), y[0]), fmaf(rest, __uint_as_float(w.x & 0xFFFF0000u), y[1]),
                     fmaf(rest, __uint_as_float(w.y << 16), y[2]), fmaf(rest, __uint_as_float(w.y & 0xFFFF0000u), y[3])};
    }
};

// out[n][m] = sum_k A(m, k) B(n, k): m a channel, n a row of dh or of the table's gradient.
struct GradArgs {
    Matrix a, b;
    int64_t k, k_split;       // k of a layer, a multiple of 64: blockIdx.y of them, none empty
    int64_t tiles_m, tiles_n;
    int64_t width, n;         // of the result
    // fp32 sums on the way: [layer][n][slab_ld], written (first) or added to; null: none
    float* slab;
    int64_t slab_ld, slab_layer;
    bool first;
    // the result, or null (then the slab is written): rows out_stride apart
    void* out;
    int64_t out_stride;
    Finish finish;
};

template <typename T>
__device__ __forceinline__ void put4(T* p, int n, bool wide, const f32x4& y)
{
    const float x[4] = {y[0], y[1], y[2], y[3]};
    if (wide)
        Lane4<T>::template store<true>(p, 0, n, x);
    else
        Lane4<T>::template store<false>(p, 0, n, x);
}

// AlongB: dh, whose k is the vocabulary, else the table's gradient, whose k are the rows; k lies across the
// memory's rows of A, and there of B too, and is read transposed from LDS.  16384 rows by 8192 of 2048 channels 470
// and 439 us (1170 and 1252 TFLOP/s).  Few tiles are cut into layers of k, added up by the next launch: dh of 3997 rows
// of 1000 by 32003 are 64 tiles, in four layers 250 us.  Both in one launch, so that the one's last tiles run
// beside the other's first, was slower (211 us for 204 of a pass over 777 rows, 11.8 ms for 11.5 over 16384).
template <class S, bool AlongB>
__global__ void __launch_bounds__(S::kThreads) grad_kernel(GradArgs a)
{
    using T = std::conditional_t<S::Planes == 1, bf16_t, float>;
    __shared__ __attribute__((aligned(16))) uint16_t even[S::kBuffer], odd[S::kBuffer];
    int tm, tn;
    tile_of(int(a.tiles_m), int(a.tiles_n), tm, tn);
    const int64_t k0 = int64_t(blockIdx.y) * a.k_split;
    f32x4 acc[S::MT][S::NT];
    Product<S, false, AlongB, AlongB>::run(a.a, a.b, tm, tn, k0, min(k0 + a.k_split, a.k), even, odd, acc);

    const int64_t m0 = int64_t(tm) * S::M, n0 = int64_t(tn) * S::N;
    const int lane = int(threadIdx.x) % kWave, g = lane / 16, n = lane % 16;
    const int wave = int(threadIdx.x) / kWave, wm = wave / S::WN, wn = wave % S::WN;
    // four channels in one access: the rows' pitch and the base allow it (the slab's always do)
    const bool wide = a.out != nullptr && (a.out_stride * int64_t(sizeof(T))) % (4 * sizeof(T)) == 0 && uintptr_t(a.out) % (4 * sizeof(T)) == 0;
    float* slab = a.slab == nullptr ? nullptr : a.slab + int64_t(blockIdx.y) * a.slab_layer;
    int32_t at[S::NT];      // of all rows together, ahead of what hangs on them: row by row their latency was 4 us of a wide tile
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
        at[j] = 0;
        if constexpr (!AlongB) {
            const int64_t row = n0 + (wn * S::NT + j) * 16 + n;
            if (a.out != nullptr && a.finish.at != nullptr && row < a.n) at[j] = a.finish.at[row];
        }
    }
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
        const int64_t row = n0 + (wn * S::NT + j) * 16 + n;
        if (row >= a.n) continue;
        const int64_t first = m0 + wm * S::MT * 16 + 4 * g;
        if (a.out == nullptr) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i) {
                if (first + 16 * i >= a.width) continue;
                f32x4* to = reinterpret_cast<f32x4*>(slab + row * a.slab_ld + first + 16 * i);
                *to = a.first ? acc[i][j] : acc[i][j] + *to;
            }
            continue;
        }
        if constexpr (!AlongB) {
            const float* more = sums_of(a.finish, at[j]);
            if (more != nullptr) {
                f32x4 x[S::MT];      // asked for together
#pragma unroll
                for (int i = 0; i < S::MT; ++i) x[i] = first + 16 * i < a.width ? *reinterpret_cast<const f32x4*>(more + first + 16 * i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < S::MT; ++i) acc[i][j] += x[i];
            }
#pragma unroll
            for (int i = 0; i < S::MT; ++i) {
                const int left = int(max(min(a.width - first - 16 * i, int64_t(4)), int64_t(0)));
                if (left > 0) put4(static_cast<T*>(a.out) + row * a.out_stride + first + 16 * i, left, wide && left == 4, acc[i][j]);
            }
            continue;
        }
        const RowEnd end(a.finish, row);
        uint2 w[S::MT];
        int left[S::MT];
#pragma unroll
        for (int i = 0; i < S::MT; ++i) {
            left[i] = int(max(min(a.width - first - 16 * i, int64_t(4)), int64_t(0)));
            w[i] = end.load(first + 16 * i, left[i]);
        }
#pragma unroll
        for (int i = 0; i < S::MT; ++i) {
            if (left[i] == 0) continue;
            f32x4 y = acc[i][j];
            if (slab != nullptr && !a.first) y += *reinterpret_cast<const f32x4*>(slab + row * a.slab_ld + first + 16 * i);
            put4(static_cast<T*>(a.out) + row * a.out_stride + first + 16 * i, left[i], wide && left[i] == 4, end.add(y, w[i]));
        }
    }
}

// The layers of a slab added in order: 5 to 15 us, what the launch and the slab's bytes take.
struct SumArgs {
    const float* slab;
    int64_t slab_ld, slab_layer, layers;
    int64_t n, width;
    void* out;
    int64_t out_stride;
    Finish finish;
};
constexpr int kSumThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kSumThreads) layer_sum_kernel(SumArgs a)
{
    const int64_t per = a.slab_ld / 4, i = int64_t(blockIdx.x) * kSumThreads + threadIdx.x;
    if (i >= a.n * per) return;
    const int64_t row = i / per, m = i % per * 4;
    if (m >= a.width) return;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    const float* src = a.slab + row * a.slab_ld + m;
#pragma unroll 4
    for (int64_t l = 0; l < a.layers; ++l) y += *reinterpret_cast<const f32x4*>(src + l * a.slab_layer);
    if (const float* more = sums_of(a.finish, a.finish.at == nullptr ? 0 : a.finish.at[row]); more != nullptr) y += *reinterpret_cast<const f32x4*>(more + m);
    T* p = static_cast<T*>(a.out) + row * a.out_stride + m;
    const int left = int(min(a.width - m, int64_t(4)));
    const RowEnd end(a.finish, row);
    put4(p, left, left == 4 && uintptr_t(p) % (4 * sizeof(T)) == 0, end.add(y, end.load(m, left)));
}

// ------------------------------------------------------------------ the tiles' launches
template <int Planes, class S>
constexpr bool planned(Shape s)
{
    return S::M == kTileRows[Planes - 1][s] && S::N == kTileColumns[Planes - 1][s] && S::K == step_of(Planes);
}
template <int Planes>
constexpr bool planned()
{
    using P = Shapes<Planes>;
    bool all = planned<Planes, typename P::Wide>(kWide) && planned<Planes, typename P::Middle>(kMiddle) && planned<Planes, typename P::Narrow>(kNarrow);
    if constexpr (Planes < 3) all = all && planned<Planes, typename P::Thin>(kThin);
    return all;
}
static_assert(planned<1>() && planned<2>() && planned<3>() && Stream::kRows == kStreamRows, "the tiles that the plans are made for");

template <int Planes, typename F>
hipError_t with_shape(Shape s, F f)
{
    using P = Shapes<Planes>;
    switch (s) {
        case kWide: return f(typename P::Wide{});
        case kMiddle: return f(typename P::Middle{});
        case kThin:
            if constexpr (Planes < 3) return f(typename P::Thin{});
            [[fallthrough]];
        default: return f(typename P::Narrow{});
    }
}
// A product of logits (bf16 or fp16 planes), and one of a gradient (bf16, one plane or three).
template <typename F>
hipError_t with_logits_shape(Shape s, int planes, F f)
{
    return planes == 1 ? with_shape<1>(s, f) : with_shape<2>(s, f);
}
template <typename F>
hipError_t with_grad_shape(Shape s, int planes, F f)
{
    return planes == 1 ? with_shape<1>(s, f) : with_shape<3>(s, f);
}

// A table or h that the products read where it lies: bf16 rows of whole steps in 16-byte pieces.
bool direct(const void* p, int64_t stride, int64_t width, int dtype)
{
    return may_lie(width, dtype) && stride % 8 == 0 && stride < (int64_t(1) << 22) && uintptr_t(p) % 16 == 0;
}

}  // namespace

int64_t cross_entropy_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype) { return ForwardPlan(rows, vocab, width, dtype).bytes; }

int64_t cross_entropy_grad_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype)
{
    return grad_bytes(rows, vocab, width, dtype);
}

hipError_t launch_cross_entropy(const CrossEntropyArgs& a, hipStream_t stream)
{
    const ForwardPlan plan(a.rows, a.vocab, a.width, a.dtype);
    const int planes = logit_planes(a.dtype);
    const int64_t ld = ceil_to(a.width, kStepK);
    char* ws = a.workspace;
    LogitsArgs k{};
    k.width = a.width;
    k.vocab = a.vocab;
    k.rows = a.rows;
    k.targets = a.targets;
    k.cap = a.cap;
    k.part = reinterpret_cast<float2*>(ws + plan.part);
    k.best_z = a.best == nullptr ? nullptr : reinterpret_cast<float*>(ws + plan.best_z);
    k.best_v = reinterpret_cast<int32_t*>(ws + plan.best_v);
    k.at = a.targets.p == nullptr ? nullptr : reinterpret_cast<float*>(ws + plan.at);
    k.h_e = reinterpret_cast<int32_t*>(ws + plan.h_e);
    k.table_e = reinterpret_cast<int32_t*>(ws + plan.table_e);
    uint16_t* h = reinterpret_cast<uint16_t*>(ws + plan.h);
    uint16_t* copy = reinterpret_cast<uint16_t*>(ws + plan.table);
    // h is copied, if at all, along with the table's first piece
    const bool h_as_is = direct(a.h, a.h_stride, a.width, a.dtype), as_is = direct(a.table, a.table_stride, a.width, a.dtype);
    k.h = h_as_is ? Matrix{static_cast<const uint16_t*>(a.h), a.h_stride, 0, a.rows, a.width} : Matrix{h, ld, a.rows * ld, a.rows, ld};
    const bool stream_table = streams(a.rows, planes);
    uint16_t* parts = stream_table ? reinterpret_cast<uint16_t*>(ws + plan.h_parts) : nullptr;
    if (stream_table) k.h = Matrix{parts, ld, a.rows * ld, a.rows, ld};
    int64_t most = as_is || stream_table ? a.vocab : copy_rows(a.vocab, a.width, a.dtype);
    const Shape shape = shape_of(most, a.rows, a.width, planes);
    k.tiles_n = ceil_div(a.rows, shape_n(shape, planes));
    most = std::min(most, kMostTiles / k.tiles_n * shape_m(shape, planes));
    for (int64_t first = 0; first < a.vocab; first += most) {
        k.first = first;
        k.piece = std::min(most, a.vocab - first);
        k.tile0 = first / shape_m(shape, planes);
        k.tiles_m = ceil_div(k.piece, shape_m(shape, planes));
        const uint16_t* src = static_cast<const uint16_t*>(a.table) + first * a.table_stride * planes;      // of fp32, two planes, twice the bytes
        k.table = as_is ? Matrix{src, a.table_stride, 0, k.piece, a.width} : Matrix{copy, ld, k.piece * ld, k.piece, ld};
        k.whole = reinterpret_cast<const float*>(src);
        k.whole_stride = a.table_stride;
        hipError_t e;
        if (planes == 1) {
            e = pack_copy(first > 0 || h_as_is ? PackArgs{} : PackArgs{static_cast<const uint16_t*>(a.h), a.rows, a.width, a.h_stride, {}, 0, h, a.rows, ld},
                          as_is ? PackArgs{} : PackArgs{src, k.piece, a.width, a.table_stride, {}, 0, copy, k.piece, ld}, stream);
        } else {
            e = pack_rows(first > 0 ? RowArgs{} : RowArgs{static_cast<const float*>(a.h), a.rows, a.width, a.h_stride, {}, 0, stream_table ? nullptr : h,
                                                           reinterpret_cast<int32_t*>(ws + plan.h_e), exponents_of(a.rows), parts, a.rows, ld},
                          stream_table ? RowArgs{} : RowArgs{reinterpret_cast<const float*>(src), k.piece, a.width, a.table_stride, {}, 0, copy,
                                                             reinterpret_cast<int32_t*>(ws + plan.table_e), exponents_of(k.piece), nullptr, k.piece, ld},
                          stream);
        }
        if (e != hipSuccess) return e;
        e = with_logits_shape(shape, planes, [&](auto s) {
            using S = decltype(s);
            if (!grid_fits(k.tiles_m * k.tiles_n, S::kThreads)) return hipErrorInvalidConfiguration;
            hipLaunchKernelGGL((logits_kernel<S>), dim3(unsigned(k.tiles_m * k.tiles_n)), dim3(S::kThreads), 0, stream, k);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    const JoinArgs j{k.part, k.best_z, k.best_v, k.at, a.targets, a.cap, a.rows, a.vocab,
                     ceil_div(a.vocab, shape_m(shape, planes)), a.targets.p == nullptr ? nullptr : a.loss, a.lse, a.best};
    // a workgroup for each of few rows; sixteen neighbours, whose sums lie side by side, of many (calls by 50257 of 64
    // channels: 256 rows 19.6 us against 23.6, 512 33.2 and 32.8, 1024 55.2 and 53.0, 2048 104 and 94)
    const bool few = a.rows < 512;
    const int64_t blocks = few ? a.rows : ceil_div(a.rows, 16);
    if (!grid_fits(blocks, kJoinThreads)) return hipErrorInvalidConfiguration;
    if (few)
        hipLaunchKernelGGL((join_kernel<1>), dim3(unsigned(blocks)), dim3(kJoinThreads), 0, stream, j);
    else
        hipLaunchKernelGGL((join_kernel<16>), dim3(unsigned(blocks)), dim3(kJoinThreads), 0, stream, j);
    return hipGetLastError();
}

namespace {

template <bool AlongB>
hipError_t launch_grad(const GradArgs& k, Shape shape, int64_t layers, int planes, hipStream_t stream)
{
    return with_grad_shape(shape, planes, [&](auto s) {
        using S = decltype(s);
        if (!grid_fits(k.tiles_m * k.tiles_n, S::kThreads)) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((grad_kernel<S, AlongB>), dim3(unsigned(k.tiles_m * k.tiles_n), unsigned(layers)), dim3(S::kThreads), 0, stream, k);
        return hipGetLastError();
    });
}

hipError_t launch_sum(const SumArgs& a, int dtype, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.n * (a.slab_ld / 4), kSumThreads);
    if (!grid_fits(blocks, kSumThreads)) return hipErrorInvalidConfiguration;
    if (dtype == kBf16)
        hipLaunchKernelGGL((layer_sum_kernel<bf16_t>), dim3(unsigned(blocks)), dim3(kSumThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((layer_sum_kernel<float>), dim3(unsigned(blocks)), dim3(kSumThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_entropy_grad(const CrossEntropyGradArgs& a, hipStream_t stream)
{
    if (a.rows == 0) {      // the table's gradient is the sum of nothing
        if (a.dtable == nullptr) return hipSuccess;
        const SumArgs none{nullptr, ceil_to(a.width, 4), 0, 0, a.vocab, a.width, a.dtable, a.dtable_stride, {}};
        return launch_sum(none, a.dtype, stream);
    }
    const bool as_is = direct(a.table, a.table_stride, a.width, a.dtype);
    const GradPlan plan(a.rows, a.vocab, a.width, a.dtype, !as_is);
    const int planes = grad_planes(a.dtype);
    const int64_t ld = plan.ld, es = planes == 1 ? 2 : 4;
    char* ws = a.workspace;
    auto words = [&](int64_t at) { return reinterpret_cast<uint16_t*>(ws + at); };
    uint16_t* dz = words(plan.dz);
    float* rest = planes == 1 ? reinterpret_cast<float*>(ws + plan.rest) : nullptr;
    const int64_t dz_plane = plan.dz_rows * plan.dz_ld;      // of fp32
    // dz's rest and h once more are for the table's gradient
    const bool twice = plan.deep > plan.dz_rows && a.dtable != nullptr;
    const int64_t deep = twice ? plan.deep : plan.dz_rows;
    const Matrix h{words(plan.h), ld, deep * ld, deep, ld};
    Finish more{};
    TokenSumArgs sums{};
    const bool sorts = plan.sorts && a.dtable != nullptr;
    if (sorts) {
        more.sums = sums.sums = reinterpret_cast<float*>(ws + plan.sums);
        more.sums_ld = sums.ld = ld;
        sums.at = reinterpret_cast<int32_t*>(ws + plan.at);
        sums.rows = a.rows;
        sums.width = a.width;
        sums.x = words(plan.h);
        sums.stride = ld;
        sums.weight = rest;
        sums.workspace = ws + plan.order;
        if (hipError_t e = launch_token_sort(a.targets, a.rows, a.vocab, a.width, Zeros{sums.at, a.vocab, 4, 4, 4}, sums.workspace, &sums.sorted, stream);
            e != hipSuccess)
            return e;
    }

    for (int64_t first = 0; first < a.vocab; first += plan.piece) {
        const int64_t piece = std::min(plan.piece, a.vocab - first);
        const bool last = first + piece == a.vocab;
        const char* src = static_cast<const char*>(a.table) + first * a.table_stride * es;
        const Matrix table = as_is ? Matrix{reinterpret_cast<const uint16_t*>(src), a.table_stride, 0, piece, a.width}
                                   : Matrix{words(plan.table), ld, piece * ld, piece, ld};
        // h is copied always: rows that do not count may hold anything, and the products over rows would meet it
        hipError_t e;
        LogitsArgs k{};
        if (planes == 1) {
            e = pack_copy(first > 0 ? PackArgs{} : PackArgs{static_cast<const uint16_t*>(a.h), a.rows, a.width, a.h_stride, a.targets, a.vocab,
                                                            words(plan.h), deep, ld, twice ? plan.dz_rows : 0},
                          as_is ? PackArgs{} : PackArgs{reinterpret_cast<const uint16_t*>(src), piece, a.width, a.table_stride, {}, 0, words(plan.table), piece, ld},
                          stream);
            k.table = table;
            k.h = h;
        } else {
            const bool streamed = streams(a.rows, logit_planes(a.dtype));
            int32_t *h_e = reinterpret_cast<int32_t*>(ws + plan.h_e), *table_e = reinterpret_cast<int32_t*>(ws + plan.table_e);
            // parts of h for the table's gradient, of the table for dh, and of few rows of h for the logits
            e = pack_rows(first > 0 ? RowArgs{} : RowArgs{static_cast<const float*>(a.h), a.rows, a.width, a.h_stride, a.targets, a.vocab,
                                                           streamed ? nullptr : words(plan.h16), h_e, exponents_of(plan.dz_rows),
                                                           streamed || a.dtable != nullptr ? words(plan.h) : nullptr, plan.dz_rows, ld},
                          RowArgs{reinterpret_cast<const float*>(src), piece, a.width, a.table_stride, {}, 0, streamed ? nullptr : words(plan.table16), table_e,
                                  exponents_of(piece), a.dh != nullptr ? words(plan.table) : nullptr, piece, ld},
                          stream);
            k.table = Matrix{words(plan.table16), ld, piece * ld, piece, ld};
            k.h = streamed ? h : Matrix{words(plan.h16), ld, plan.dz_rows * ld, plan.dz_rows, ld};
            k.whole = reinterpret_cast<const float*>(src);
            k.whole_stride = a.table_stride;
            k.h_e = h_e;
            k.table_e = table_e;
        }
        if (e != hipSuccess) return e;
        k.width = a.width;
        k.first = first;
        k.vocab = a.vocab;
        k.piece = piece;
        k.rows = a.rows;
        k.targets = a.targets;
        k.cap = a.cap;
        k.lse = a.lse;
        k.dloss = a.dloss;
        k.rest = rest;
        k.dz = dz;
        k.dz_ld = plan.dz_ld;
        k.dz_plane = dz_plane;
        k.dz_rows = plan.dz_rows;
        k.twice = twice;
        k.tiles_m = ceil_div(piece, shape_m(plan.logits, logit_planes(a.dtype)));
        k.tiles_n = streams(a.rows, logit_planes(a.dtype)) ? 1 : ceil_div(plan.dz_rows, shape_n(plan.logits, logit_planes(a.dtype)));
        e = with_logits_shape(plan.logits, logit_planes(a.dtype), [&](auto s) {
            using S = decltype(s);
            if (!grid_fits(k.tiles_m * k.tiles_n, S::kThreads)) return hipErrorInvalidConfiguration;
            hipLaunchKernelGGL((logits_grad_kernel<S>), dim3(unsigned(k.tiles_m * k.tiles_n)), dim3(S::kThreads), 0, stream, k);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
        const Matrix dz_rows{dz, plan.dz_ld, dz_plane, deep, plan.dz_ld};
        if (a.dh != nullptr) {
            const bool slab = plan.dh.layers > 1 || plan.piece < a.vocab;
            GradArgs d{};
            d.a = table;
            d.b = dz_rows;
            d.k = piece;
            d.k_split = ceil_to(ceil_div(std::min(plan.piece, a.vocab), plan.dh.layers), kStepK);
            const int64_t layers = ceil_div(std::min(plan.piece, a.vocab), d.k_split);      // that hold something
            d.tiles_m = ceil_div(a.width, shape_m(plan.dh.shape, planes));
            d.tiles_n = ceil_div(a.rows, shape_n(plan.dh.shape, planes));
            d.width = a.width;
            d.n = a.rows;
            d.slab = slab ? reinterpret_cast<float*>(ws + plan.slab_h) : nullptr;
            d.slab_ld = ld;
            d.slab_layer = a.rows * ld;
            d.first = first == 0;
            d.out = layers == 1 && last ? a.dh : nullptr;
            d.out_stride = a.dh_stride;
            d.finish = Finish{a.targets, a.vocab, rest, static_cast<const uint16_t*>(a.table), a.table_stride};
            if (e = launch_grad<true>(d, plan.dh.shape, ceil_div(d.k, d.k_split), planes, stream); e != hipSuccess) return e;
            if (last && layers > 1) {
                const SumArgs s{d.slab, ld, d.slab_layer, layers, a.rows, a.width, a.dh, a.dh_stride, d.finish};
                if (e = launch_sum(s, a.dtype, stream); e != hipSuccess) return e;
            }
        }
        if (a.dtable != nullptr) {
            const Cut cut = last ? plan.de_last : plan.de;
            const Shape shape = cut.shape;
            GradArgs d{};
            d.a = h;
            d.b = dz_rows;
            d.k = deep;
            d.k_split = ceil_to(ceil_div(deep, cut.layers), kStepK);
            const int64_t layers = ceil_div(d.k, d.k_split);
            d.tiles_m = ceil_div(a.width, shape_m(shape, planes));
            d.tiles_n = ceil_div(piece, shape_n(shape, planes));
            d.width = a.width;
            d.n = piece;
            d.slab = layers > 1 ? reinterpret_cast<float*>(ws + plan.slab_e) : nullptr;
            d.slab_ld = ld;
            d.slab_layer = piece * ld;
            d.first = true;
            if (sorts) {
                sums.first = uint32_t(first);
                sums.count = uint32_t(piece);
                if (e = launch_token_sums(sums, stream); e != hipSuccess) return e;
                more.at = sums.at + first;
            }
            d.finish = more;
            void* out = static_cast<char*>(a.dtable) + first * a.dtable_stride * es;
            d.out = layers == 1 ? out : nullptr;
            d.out_stride = a.dtable_stride;
            if (e = launch_grad<false>(d, shape, layers, planes, stream); e != hipSuccess) return e;
            if (layers > 1) {
                const SumArgs s{d.slab, ld, d.slab_layer, layers, piece, a.width, out, a.dtable_stride, more};
                if (e = launch_sum(s, a.dtype, stream); e != hipSuccess) return e;
            }
        }
    }
    return hipSuccess;
}

}  // namespace mesa
