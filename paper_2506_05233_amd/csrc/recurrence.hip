// The gated linear recurrence of a Hawk layer (the other layer of the paper's Hawk-Mesa
// hybrid), its backward pass and its one-token step.  For every sequence and channel
//     s_t = sigma(r_t),  l_t = -decay softplus(theta) s_t,  a_t = exp(l_t),  m_t = sqrt(1 - a_t^2)
//     h_t = a_t h_{t-1} + m_t sigma(i_t) x_t
// and, given dy and dh_T, with c_{T+1} = dh_T:
//     g_t = dy_t + c_{t+1},  c_t = a_t g_t,  dh_0 = c_1
//     dx = g m sigma(i),  di = dx x (1 - sigma(i))
//     dl = g (a h_{t-1} - a^2 / m sigma(i) x),  dr = dl l (1 - s)
//     dtheta = -decay sigma(theta) sum_{b,t} dl s
// A reset token has a_t = 0 and m_t = 1 and nothing before it is read.
//
// 1 - a^2 is -expm1(2 l): its series for a small argument, 1 - a a otherwise (the
// difference then keeps all but two bits).  l / m, which multiplies dl in dr, tends to 0
// with l although 1 / m does not stay finite, so the reciprocal root is formed once and
// is 0 where 1 - a^2 is.
//
// A span of tokens acts on the state as h -> A h + B, and spans compose, so time is cut:
// a lane holds kSub consecutive tokens of four channels in registers, a row of 16 lanes a
// token's 64 channels (128 bytes of bf16), a workgroup 32 such runs in time.  The runs'
// (A, B) are joined inside a wave by row swaps, across waves in LDS, across workgroups
// through the workspace: a first kernel writes every tile's (A, B), a second folds those
// before it and walks its tokens from the state that enters them.  A reset inside a span
// is kept as the sign of A (A is never negative otherwise), since 0 times a state that is
// not finite would not forget it.  All of it is fp32 and in a fixed order.
#include <algorithm>

#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"

namespace mesa {
namespace {

constexpr int kAcross = 16;            // lanes across a token's channels
constexpr int kCh = 4 * kAcross;       // channels of a workgroup
constexpr int kBlock = kRecurrenceBlock;

// What a span of tokens does to the state.
struct Span {
    float A, B;
};
template <bool Reset>
__device__ __forceinline__ float apply(Span s, float h)
{
    const float y = fmaf(s.A, h, s.B);
    return Reset && signbit(s.A) ? s.B : y;
}
// first `lo`, then `hi` (in the order in which the state passes through them)
template <bool Reset>
__device__ __forceinline__ Span join(Span lo, Span hi)
{
    const bool hard = Reset && signbit(hi.A);
    return {hard ? hi.A : lo.A * hi.A, apply<Reset>(hi, lo.B)};
}
__device__ __forceinline__ Span nothing() { return {1.0f, 0.0f}; }

// Rows (16 lanes) r of a wave: out lo[r] = v[r & ~1], hi[r] = v[r | 1]; and for pairs of rows.
__device__ __forceinline__ void swap_rows(float v, float& lo, float& hi)
{
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    lo = __uint_as_float(s[0]), hi = __uint_as_float(s[1]);
}
__device__ __forceinline__ void swap_halves(float v, float& lo, float& hi)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    lo = __uint_as_float(s[0]), hi = __uint_as_float(s[1]);
}

// Joins the spans of a wave's four rows in time order (Back: from the last row to the
// first): `before` the span of the rows that come before the lane's own, `all` that of all.
template <bool Reset, bool Back>
__device__ __forceinline__ void join_rows(Span own, int row, Span& before, Span& all)
{
    Span lo, hi;
    swap_rows(own.A, lo.A, hi.A);
    swap_rows(own.B, lo.B, hi.B);
    const bool second = Back ? (row & 1) == 0 : (row & 1) != 0;
    before = second ? (Back ? hi : lo) : nothing();
    const Span pair = Back ? join<Reset>(hi, lo) : join<Reset>(lo, hi);
    Span plo, phi;
    swap_halves(pair.A, plo.A, phi.A);
    swap_halves(pair.B, plo.B, phi.B);
    const bool later = Back ? row < 2 : row >= 2;
    if (later) before = join<Reset>(Back ? phi : plo, before);
    all = Back ? join<Reset>(phi, plo) : join<Reset>(plo, phi);
}

// The per-channel constants: log2 a_t = rate * s_t.
struct Rates {
    float v[4];
};
__device__ __forceinline__ Rates rates_of(const float* theta, float decay, int64_t ch, int n)
{
    Rates k;
#pragma unroll
    for (int v = 0; v < 4; ++v) k.v[v] = v < n ? -decay * kLog2e * softplus_both(theta[ch + v]) : 0.0f;
    return k;
}

// a = 2^z and 1 - a^2 for z <= 0
__device__ __forceinline__ float one_minus_square(float z, float a)
{
    const float u = -2.0f * kLn2 * z;   // a^2 = exp(-u)
    float p = 1.0f / 5040.0f;
    p = fmaf(p, u, -1.0f / 720.0f);
    p = fmaf(p, u, 1.0f / 120.0f);
    p = fmaf(p, u, -1.0f / 24.0f);
    p = fmaf(p, u, 1.0f / 6.0f);
    p = fmaf(p, u, -0.5f);
    p = fmaf(p, u, 1.0f);
    return u < 0.35f ? u * p : fmaf(-a, a, 1.0f);   // first term left out: u^7 / 8! < 2e-8
}

// One element's a and b (the state's input); hard: a reset token, a = -0
template <bool Reset>
__device__ __forceinline__ Span terms(float x, float r, float i, float rate, bool hard)
{
    const float z = rate * sigmoid_fast(r);
    const float a = __builtin_amdgcn_exp2f(z);
    const float m = __builtin_amdgcn_sqrtf(one_minus_square(z, a));
    const float in = sigmoid_fast(i) * x;
    if (Reset && hard) return {-0.0f, in};
    return {a, m * in};
}

// ---------------------------------------------------------------- forward
constexpr int kFwdSub = 8;                         // tokens of a lane
constexpr int kFwdThreads = 512;
constexpr int kFwdWaves = kFwdThreads / kWave;
constexpr int kFwdTile = kFwdWaves * 4 * kFwdSub;  // tokens of a workgroup
static_assert(kFwdTile == 2 * kBlock && kBlock % kFwdSub == 0, "a state block starts at a lane's first token");

// Folds spans [B, n_tiles, width] of tiles lo .. hi - 1, in that order (Back: reversed),
// onto the state h of four channels.
template <bool Reset, bool Vec, bool Back>
__device__ __forceinline__ void fold_tiles(const float2* spans, int64_t width, int lo, int hi, int n, float (&h)[4])
{
    for (int t = 0; t < hi - lo; ++t) {
        const float2* p = spans + int64_t(Back ? hi - 1 - t : lo + t) * width;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (v < n) {
                const float2 s = p[v];
                h[v] = apply<Reset>({s.x, s.y}, h[v]);
            }
    }
}

// Spans: the tiles' (A, B) only, into a.spans.  Otherwise the outputs.
template <typename T, bool Vec, bool Reset, bool Spans>
__global__ __launch_bounds__(kFwdThreads) void recurrence_kernel(RecurrenceArgs a)
{
    __shared__ float4 wave_A[kFwdWaves][kAcross], wave_B[kFwdWaves][kAcross];
    const int slabs = int((a.width + kCh - 1) / kCh);
    const int slab = blockIdx.x % slabs;
    const int tile = (blockIdx.x / slabs) % a.tiles;
    const int64_t b = blockIdx.x / slabs / a.tiles;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int row = lane / kAcross, col = lane % kAcross;
    const int64_t ch = int64_t(slab) * kCh + col * 4;
    const int n = int(max<int64_t>(0, min<int64_t>(4, a.width - ch)));   // channels of this lane
    const int64_t t0 = int64_t(tile) * kFwdTile + (wave * 4 + row) * kFwdSub;
    const int64_t at0 = (b * a.seq_len + t0) * a.stride + ch;

    // tokens past the end leave the state alone and are neither read nor written
    typename Lane4<T>::Raw rx[kFwdSub], rr[kFwdSub], ri[kFwdSub];
    bool hard[kFwdSub] = {};
#pragma unroll
    for (int j = 0; j < kFwdSub; ++j) {
        const int m = t0 + j < a.seq_len ? n : 0;
        rx[j] = Lane4<T>::template load<Vec>(a.x, at0 + j * a.stride, m);
        rr[j] = Lane4<T>::template load<Vec>(a.r, at0 + j * a.stride, m);
        ri[j] = Lane4<T>::template load<Vec>(a.i, at0 + j * a.stride, m);
        if (Reset) hard[j] = t0 + j < a.seq_len && a.reset[b * a.seq_len + t0 + j] != 0;
    }
    const Rates k = rates_of(a.theta, a.decay, ch, n);
    Span e[kFwdSub][4], own[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) own[v] = nothing();
#pragma unroll
    for (int j = 0; j < kFwdSub; ++j) {
        float x[4], r[4], i[4];
        Lane4<T>::widen(rx[j], x);
        Lane4<T>::widen(rr[j], r);
        Lane4<T>::widen(ri[j], i);
        const bool there = t0 + j < a.seq_len;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            e[j][v] = there ? terms<Reset>(x[v], r[v], i[v], k.v[v], hard[j]) : nothing();
            own[v] = join<Reset>(own[v], e[j][v]);
        }
    }
    Span before[4], all[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) join_rows<Reset, false>(own[v], row, before[v], all[v]);
    if (row == 0) {
        wave_A[wave][col] = make_float4(all[0].A, all[1].A, all[2].A, all[3].A);
        wave_B[wave][col] = make_float4(all[0].B, all[1].B, all[2].B, all[3].B);
    }
    __syncthreads();
    if constexpr (Spans) {
        if (wave == 0 && row == 0 && n > 0) {
            Span s[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) s[v] = nothing();
            for (int w = 0; w < kFwdWaves; ++w) {
                const float4 A = wave_A[w][col], B = wave_B[w][col];
                const Span t[4] = {{A.x, B.x}, {A.y, B.y}, {A.z, B.z}, {A.w, B.w}};
#pragma unroll
                for (int v = 0; v < 4; ++v) s[v] = join<Reset>(s[v], t[v]);
            }
            float2* out = a.spans + (b * a.tiles + tile) * a.width + ch;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (v < n) out[v] = make_float2(s[v].A, s[v].B);
        }
    } else {
        float h[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = a.h0 != nullptr && v < n ? a.h0[b * a.width + ch + v] : 0.0f;
        fold_tiles<Reset, Vec, false>(a.spans + b * a.tiles * a.width + ch, a.width, 0, tile, n, h);
        for (int w = 0; w < wave; ++w) {
            const float4 A = wave_A[w][col], B = wave_B[w][col];
            h[0] = apply<Reset>({A.x, B.x}, h[0]);
            h[1] = apply<Reset>({A.y, B.y}, h[1]);
            h[2] = apply<Reset>({A.z, B.z}, h[2]);
            h[3] = apply<Reset>({A.w, B.w}, h[3]);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = apply<Reset>(before[v], h[v]);
        if (a.states != nullptr && t0 % kBlock == 0 && t0 < a.seq_len)
            Lane4<float>::store<false>(a.states, (b * ((a.seq_len + kBlock - 1) / kBlock) + t0 / kBlock) * a.width + ch, n, h);
        const int64_t y0 = (b * a.seq_len + t0) * a.width + ch;
#pragma unroll
        for (int j = 0; j < kFwdSub; ++j) {
#pragma unroll
            for (int v = 0; v < 4; ++v) h[v] = apply<Reset>(e[j][v], h[v]);
            if (t0 + j < a.seq_len) {
                Lane4<T>::template store<Vec>(a.y, y0 + j * a.width, n, h);
                if (t0 + j == a.seq_len - 1 && a.final_h != nullptr) Lane4<float>::store<false>(a.final_h, b * a.width + ch, n, h);
            }
        }
        if (a.kept_x != nullptr) {
            // the checkpoint of this tile's inputs: eight lanes are a group of 32 channels
            const int64_t groups = (a.width + kGroup - 1) / kGroup;
            uint8_t* const kept[3] = {a.kept_x, a.kept_r, a.kept_i};
            const int64_t bytes_at = checkpoint_exponents_at(a.batch * a.seq_len, a.width);
#pragma unroll
            for (int j = 0; j < kFwdSub; ++j) {
                float val[3][4];
                Lane4<T>::widen(rx[j], val[0]);
                Lane4<T>::widen(rr[j], val[1]);
                Lane4<T>::widen(ri[j], val[2]);
                const int64_t token = b * a.seq_len + t0 + j;
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    uint32_t top = 0;
#pragma unroll
                    for (int v = 0; v < 4; ++v) top = max(top, abs_bits(val[q][v]));
                    top = max(top, uint32_t(dpp_i32<kDppQuadSwap1>(int(top), int(top))));
                    top = max(top, uint32_t(dpp_i32<kDppQuadSwap2>(int(top), int(top))));
                    top = max(top, uint32_t(dpp_i32<kDppRowHalfMirror>(int(top), int(top))));
                    const uint32_t byte = group_exponent(__uint_as_float(top));
                    const float inv = group_inverse(byte), most = group_most(byte);
                    int c[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) c[v] = group_code(val[q][v], inv, most);
                    if (t0 + j < a.seq_len && n > 0) {
                        uint8_t* out = kept[q] + token * a.width + ch;
                        if constexpr (Vec) {
                            *reinterpret_cast<uint32_t*>(out) = pack_codes(c);
                        } else {
#pragma unroll
                            for (int v = 0; v < 4; ++v)
                                if (v < n) out[v] = uint8_t(c[v]);
                        }
                        if (col % 8 == 0) kept[q][bytes_at + token * groups + ch / kGroup] = uint8_t(byte);
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------- one token
template <typename T, int Per>
__global__ __launch_bounds__(256) void recurrence_step_kernel(RecurrenceArgs a, float* state_out)
{
    const int64_t per_row = (a.width + Per - 1) / Per;
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (id >= a.batch * per_row) return;
    const int64_t b = id / per_row, ch = (id - b * per_row) * Per;
    constexpr bool Vec = Per == 4;
    float x[4], r[4], i[4], h[4];
    Lane4<T>::widen(Lane4<T>::template load<Vec>(a.x, b * a.stride + ch, Per), x);
    Lane4<T>::widen(Lane4<T>::template load<Vec>(a.r, b * a.stride + ch, Per), r);
    Lane4<T>::widen(Lane4<T>::template load<Vec>(a.i, b * a.stride + ch, Per), i);
    Lane4<float>::widen(Lane4<float>::load<Vec>(a.h0, b * a.width + ch, Per), h);
    const bool hard = a.reset != nullptr && a.reset[b] != 0;
    const Rates k = rates_of(a.theta, a.decay, ch, Per);
#pragma unroll
    for (int v = 0; v < Per; ++v) h[v] = apply<true>(terms<true>(x[v], r[v], i[v], k.v[v], hard), h[v]);
    Lane4<float>::store<Vec>(state_out, b * a.width + ch, Per, h);
    Lane4<T>::template store<Vec>(a.y, b * a.width + ch, Per, h);
}

// ---------------------------------------------------------------- backward
constexpr int kBwdSub = 4;
constexpr int kBwdThreads = 512;
constexpr int kBwdWaves = kBwdThreads / kWave;
constexpr int kBwdTile = kBwdWaves * 4 * kBwdSub;
static_assert(kBwdTile == kBlock, "a tile of the backward pass starts at a kept state");

// x, r or i of the backward pass: a tensor of T, or a checkpoint.
template <typename T>
struct Source {
    using Raw = typename Lane4<T>::Raw;
    template <bool Vec>
    __device__ static Raw load(const void* base, const RecurrenceGradArgs& a, int64_t token, int64_t ch, int n)
    {
        return Lane4<T>::template load<Vec>(base, token * a.stride + ch, n);
    }
    __device__ static void widen(const Raw& r, float (&x)[4]) { Lane4<T>::widen(r, x); }
};
template <>
struct Source<q8_t> {
    using Raw = Q8Raw;
    template <bool Vec>
    __device__ static Raw load(const void* base, const RecurrenceGradArgs& a, int64_t token, int64_t ch, int n)
    {
        if (n <= 0) return {0u, 0u};
        const uint8_t* bytes = static_cast<const uint8_t*>(base) + checkpoint_exponents_at(a.batch * a.seq_len, a.width);
        return {load_codes<Vec>(static_cast<const int8_t*>(base) + token * a.width + ch, n),
                bytes[token * ((a.width + kGroup - 1) / kGroup) + ch / kGroup]};
    }
    __device__ static void widen(const Raw& r, float (&x)[4]) { widen_q8(r.codes, group_scale(r.byte), x); }
};

// Spans: every tile's (A, B) of c -> A c + B, the walk from its last token to its first.
template <typename T, typename Tg, bool Vec, bool Reset, bool Spans>
__global__ __launch_bounds__(kBwdThreads) void recurrence_grad_kernel(RecurrenceGradArgs a)
{
    __shared__ float4 fwd_A[kBwdWaves][kAcross], fwd_B[kBwdWaves][kAcross];
    __shared__ float4 bwd_A[kBwdWaves][kAcross], bwd_B[kBwdWaves][kAcross];
    const int slabs = int((a.width + kCh - 1) / kCh);
    const int slab = blockIdx.x % slabs;
    const int tile = (blockIdx.x / slabs) % a.tiles;
    const int64_t b = blockIdx.x / slabs / a.tiles;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int row = lane / kAcross, col = lane % kAcross;
    const int64_t ch = int64_t(slab) * kCh + col * 4;
    const int n = int(max<int64_t>(0, min<int64_t>(4, a.width - ch)));
    const int64_t t0 = int64_t(tile) * kBwdTile + (wave * 4 + row) * kBwdSub;
    const int64_t token0 = b * a.seq_len + t0;

    typename Source<T>::Raw rx[kBwdSub], rr[kBwdSub], ri[kBwdSub];
    typename Lane4<Tg>::Raw rd[kBwdSub];
    bool hard[kBwdSub] = {};
#pragma unroll
    for (int j = 0; j < kBwdSub; ++j) {
        const int m = t0 + j < a.seq_len ? n : 0;
        rr[j] = Source<T>::template load<Vec>(a.r, a, token0 + j, ch, m);
        rd[j] = Lane4<Tg>::template load<Vec>(a.dy, (token0 + j) * a.width + ch, m);
        if (!Spans) {
            rx[j] = Source<T>::template load<Vec>(a.x, a, token0 + j, ch, m);
            ri[j] = Source<T>::template load<Vec>(a.i, a, token0 + j, ch, m);
        }
        if (Reset) hard[j] = t0 + j < a.seq_len && a.reset[token0 + j] != 0;
    }
    const Rates k = rates_of(a.theta, a.decay, ch, n);
    float ea[kBwdSub][4];
    Span fwd[4], bwd[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) fwd[v] = bwd[v] = nothing();
#pragma unroll
    for (int j = 0; j < kBwdSub; ++j) {
        float x[4], r[4], i[4];
        Source<T>::widen(rr[j], r);
        if (!Spans) {
            Source<T>::widen(rx[j], x);
            Source<T>::widen(ri[j], i);
        }
        const bool there = t0 + j < a.seq_len;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if constexpr (Spans) {
                const float z = k.v[v] * sigmoid_fast(r[v]);
                ea[j][v] = !there ? 1.0f : Reset && hard[j] ? -0.0f : __builtin_amdgcn_exp2f(z);
            } else {
                const Span s = there ? terms<Reset>(x[v], r[v], i[v], k.v[v], hard[j]) : nothing();
                ea[j][v] = s.A;
                fwd[v] = join<Reset>(fwd[v], s);
            }
        }
    }
#pragma unroll
    for (int j = kBwdSub - 1; j >= 0; --j) {
        float d[4];
        Lane4<Tg>::widen(rd[j], d);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            // c -> a (dy + c); a reset's c is 0 whatever comes after
            const bool cut = Reset && signbit(ea[j][v]);
            bwd[v] = cut ? Span{-0.0f, 0.0f} : Span{bwd[v].A * ea[j][v], ea[j][v] * (bwd[v].B + d[v])};
        }
    }
    Span fbefore[4], fall[4], bbefore[4], ball[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (!Spans) join_rows<Reset, false>(fwd[v], row, fbefore[v], fall[v]);
        join_rows<Reset, true>(bwd[v], row, bbefore[v], ball[v]);
    }
    if (row == 0) {
        if (!Spans) {
            fwd_A[wave][col] = make_float4(fall[0].A, fall[1].A, fall[2].A, fall[3].A);
            fwd_B[wave][col] = make_float4(fall[0].B, fall[1].B, fall[2].B, fall[3].B);
        }
        bwd_A[wave][col] = make_float4(ball[0].A, ball[1].A, ball[2].A, ball[3].A);
        bwd_B[wave][col] = make_float4(ball[0].B, ball[1].B, ball[2].B, ball[3].B);
    }
    __syncthreads();
    if constexpr (Spans) {
        if (wave == 0 && row == 0 && n > 0) {
            Span s[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) s[v] = nothing();
            for (int w = kBwdWaves - 1; w >= 0; --w) {
                const float4 A = bwd_A[w][col], B = bwd_B[w][col];
                const Span t[4] = {{A.x, B.x}, {A.y, B.y}, {A.z, B.z}, {A.w, B.w}};
#pragma unroll
                for (int v = 0; v < 4; ++v) s[v] = join<Reset>(s[v], t[v]);
            }
            float2* out = a.spans + (b * a.tiles + tile) * a.width + ch;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (v < n) out[v] = make_float2(s[v].A, s[v].B);
        }
        return;
    }
    float h[4], c[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        h[v] = v < n ? a.states[(b * a.tiles + tile) * a.width + ch + v] : 0.0f;
        c[v] = v < n && a.dfinal != nullptr ? a.dfinal[b * a.width + ch + v] : 0.0f;
    }
    fold_tiles<Reset, Vec, true>(a.spans + b * a.tiles * a.width + ch, a.width, tile + 1, a.tiles, n, c);
    for (int w = 0; w < wave; ++w) {
        const float4 A = fwd_A[w][col], B = fwd_B[w][col];
        h[0] = apply<Reset>({A.x, B.x}, h[0]);
        h[1] = apply<Reset>({A.y, B.y}, h[1]);
        h[2] = apply<Reset>({A.z, B.z}, h[2]);
        h[3] = apply<Reset>({A.w, B.w}, h[3]);
    }
    for (int w = kBwdWaves - 1; w > wave; --w) {
        const float4 A = bwd_A[w][col], B = bwd_B[w][col];
        c[0] = apply<Reset>({A.x, B.x}, c[0]);
        c[1] = apply<Reset>({A.y, B.y}, c[1]);
        c[2] = apply<Reset>({A.z, B.z}, c[2]);
        c[3] = apply<Reset>({A.w, B.w}, c[3]);
    }
    // the states before each of the lane's tokens, then the walk back
    float hp[kBwdSub][4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        h[v] = apply<Reset>(fbefore[v], h[v]);
        c[v] = apply<Reset>(bbefore[v], c[v]);
    }
#pragma unroll
    for (int j = 0; j < kBwdSub; ++j) {
        float x[4], r[4], i[4];
        Source<T>::widen(rx[j], x);
        Source<T>::widen(rr[j], r);
        Source<T>::widen(ri[j], i);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            hp[j][v] = h[v];
            h[v] = apply<Reset>(terms<Reset>(x[v], r[v], i[v], k.v[v], hard[j]), h[v]);
        }
    }
    float dth[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = kBwdSub - 1; j >= 0; --j) {
        float x[4], r[4], i[4], d[4], gx[4], gr[4], gi[4];
        Source<T>::widen(rx[j], x);
        Source<T>::widen(rr[j], r);
        Source<T>::widen(ri[j], i);
        Lane4<Tg>::widen(rd[j], d);
        const bool there = t0 + j < a.seq_len;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const bool cut = Reset && hard[j];
            float s_rest, i_rest;
            const float s = sigmoid_both(r[v], s_rest), si = sigmoid_both(i[v], i_rest);
            const float z = k.v[v] * s;
            const float at = __builtin_amdgcn_exp2f(z);
            const float m2 = one_minus_square(z, at);
            const float inv = m2 < kMinNormal ? 0.0f : __builtin_amdgcn_rsqf(m2);   // NaN for a NaN
            const float m = cut ? 1.0f : m2 * inv;
            const float g = d[v] + c[v];
            const float ix = si * x[v];
            gx[v] = g * m * si;
            gi[v] = gx[v] * x[v] * i_rest;
            const float dl = g * fmaf(at, hp[j][v], -at * at * inv * ix);
            gr[v] = cut ? 0.0f : dl * (z * kLn2) * s_rest;
            if (there && !cut) dth[v] = fmaf(dl, s, dth[v]);
            c[v] = cut ? 0.0f : there ? at * g : c[v];
        }
        if (there) {
            const int64_t at = (token0 + j) * a.grad_stride + ch;
            Lane4<Tg>::template store<Vec>(a.dx, at, n, gx);
            Lane4<Tg>::template store<Vec>(a.dr, at, n, gr);
            Lane4<Tg>::template store<Vec>(a.di, at, n, gi);
        }
    }
    if (a.dh0 != nullptr && t0 == 0) Lane4<float>::store<false>(a.dh0, b * a.width + ch, n, c);
    // dtheta: the tile's sum of dl s, one row of the partial sums
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        dth[v] = row_pair_sums(dth[v]);
    }
    if (row == 0) fwd_A[wave][col] = make_float4(dth[0], dth[1], dth[2], dth[3]);
    __syncthreads();
    if (wave == 0 && row == 0 && n > 0) {
        float4 s = fwd_A[0][col];
        for (int w = 1; w < kBwdWaves; ++w) {
            const float4 q = fwd_A[w][col];
            s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
        }
        const float o[4] = {s.x, s.y, s.z, s.w};
        Lane4<float>::store<false>(a.partial, (b * a.tiles + tile) * a.width + ch, n, o);
    }
}

// dtheta = -decay sigma(theta) times the column sums of the partial rows
__global__ __launch_bounds__(1024) void recurrence_dtheta_kernel(const float* partial, int64_t rows, const float* theta, float decay,
                                                                 int64_t width, float* dtheta)
{
    __shared__ float part[16][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t ch = int64_t(blockIdx.x) * kWave + lane;
    float s = 0.0f;
    if (ch < width)
        for (int64_t q = wave; q < rows; q += 16) s += partial[q * width + ch];
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || ch >= width) return;
    for (int w = 1; w < 16; ++w) s += part[w][lane];
    dtheta[ch] = -decay * sigmoid_fast(theta[ch]) * s;
}

// the final state of an empty sequence: the entering one
__global__ __launch_bounds__(256) void recurrence_copy_kernel(const float* from, float* to, int64_t n)
{
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) to[i] = from != nullptr ? from[i] : 0.0f;
}

bool aligned(const void* p, int bytes) { return uintptr_t(p) % uintptr_t(bytes) == 0; }

hipError_t copy_state(const float* from, float* to, int64_t n, hipStream_t stream)
{
    if (to == nullptr) return hipSuccess;
    hipLaunchKernelGGL(recurrence_copy_kernel, dim3(unsigned((n + 255) / 256)), dim3(256), 0, stream, from, to, n);
    return hipGetLastError();
}

template <typename T, bool Vec, bool Reset>
hipError_t launch_forward(const RecurrenceArgs& a, int64_t blocks, hipStream_t stream)
{
    const dim3 grid{unsigned(blocks)}, block{kFwdThreads};
    if (a.tiles > 1) hipLaunchKernelGGL((recurrence_kernel<T, Vec, Reset, true>), grid, block, 0, stream, a);
    hipLaunchKernelGGL((recurrence_kernel<T, Vec, Reset, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_forward_type(const RecurrenceArgs& a, hipStream_t stream)
{
    const int64_t blocks = a.batch * a.tiles * ((a.width + kCh - 1) / kCh);
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    constexpr int bytes = 4 * int(sizeof(T));
    const bool vec = a.width % 4 == 0 && a.stride % 4 == 0 && aligned(a.x, bytes) && aligned(a.r, bytes) &&
                     aligned(a.i, bytes) && aligned(a.y, bytes);
    if (a.reset != nullptr)
        return vec ? launch_forward<T, true, true>(a, blocks, stream) : launch_forward<T, false, true>(a, blocks, stream);
    return vec ? launch_forward<T, true, false>(a, blocks, stream) : launch_forward<T, false, false>(a, blocks, stream);
}

template <typename T>
hipError_t launch_step_type(const RecurrenceArgs& a, float* state_out, hipStream_t stream)
{
    constexpr int bytes = 4 * int(sizeof(T));
    const bool vec = a.width % 4 == 0 && a.stride % 4 == 0 && aligned(a.x, bytes) && aligned(a.r, bytes) &&
                     aligned(a.i, bytes) && aligned(a.y, bytes) && aligned(a.h0, 16) && aligned(state_out, 16);
    const int64_t threads = a.batch * (vec ? a.width / 4 : a.width), blocks = (threads + 255) / 256;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    if (vec)
        hipLaunchKernelGGL((recurrence_step_kernel<T, 4>), dim3(unsigned(blocks)), dim3(256), 0, stream, a, state_out);
    else
        hipLaunchKernelGGL((recurrence_step_kernel<T, 1>), dim3(unsigned(blocks)), dim3(256), 0, stream, a, state_out);
    return hipGetLastError();
}

template <typename T, typename Tg, bool Vec, bool Reset>
hipError_t launch_backward(const RecurrenceGradArgs& a, int64_t blocks, hipStream_t stream)
{
    const dim3 grid{unsigned(blocks)}, block{kBwdThreads};
    if (a.tiles > 1) hipLaunchKernelGGL((recurrence_grad_kernel<T, Tg, Vec, Reset, true>), grid, block, 0, stream, a);
    hipLaunchKernelGGL((recurrence_grad_kernel<T, Tg, Vec, Reset, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename T, typename Tg>
hipError_t launch_backward_types(const RecurrenceGradArgs& a, hipStream_t stream)
{
    const int64_t blocks = a.batch * a.tiles * ((a.width + kCh - 1) / kCh);
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    constexpr int in = 4 * int(sizeof(T)), out = 4 * int(sizeof(Tg));
    const bool vec = a.width % 4 == 0 && a.stride % 4 == 0 && a.grad_stride % 4 == 0 && aligned(a.x, in) &&
                     aligned(a.r, in) && aligned(a.i, in) && aligned(a.dy, out) && aligned(a.dx, out) &&
                     aligned(a.dr, out) && aligned(a.di, out);
    if (a.reset != nullptr)
        return vec ? launch_backward<T, Tg, true, true>(a, blocks, stream) : launch_backward<T, Tg, false, true>(a, blocks, stream);
    return vec ? launch_backward<T, Tg, true, false>(a, blocks, stream) : launch_backward<T, Tg, false, false>(a, blocks, stream);
}

}  // namespace

int64_t recurrence_tiles(int64_t seq_len) { return (seq_len + kFwdTile - 1) / kFwdTile; }

hipError_t launch_recurrence(const RecurrenceArgs& a, hipStream_t stream)
{
    if (a.batch * a.width == 0) return hipSuccess;
    if (a.seq_len == 0) return copy_state(a.h0, a.final_h, a.batch * a.width, stream);
    return a.dtype == kBf16 ? launch_forward_type<bf16_t>(a, stream) : launch_forward_type<float>(a, stream);
}

hipError_t launch_recurrence_step(const RecurrenceArgs& a, float* state_out, hipStream_t stream)
{
    if (a.batch * a.width == 0) return hipSuccess;
    return a.dtype == kBf16 ? launch_step_type<bf16_t>(a, state_out, stream) : launch_step_type<float>(a, state_out, stream);
}

hipError_t launch_recurrence_backward(const RecurrenceGradArgs& a, hipStream_t stream)
{
    if (a.width == 0) return hipSuccess;
    if (a.batch * a.seq_len > 0) {
        hipError_t e;
        if (a.dtype == kQ8)
            e = a.grad_dtype == kBf16 ? launch_backward_types<q8_t, bf16_t>(a, stream) : launch_backward_types<q8_t, float>(a, stream);
        else if (a.dtype == kBf16)
            e = a.grad_dtype == kBf16 ? launch_backward_types<bf16_t, bf16_t>(a, stream) : launch_backward_types<bf16_t, float>(a, stream);
        else
            e = a.grad_dtype == kBf16 ? launch_backward_types<float, bf16_t>(a, stream) : launch_backward_types<float, float>(a, stream);
        if (e != hipSuccess) return e;
    } else if (a.batch > 0) {
        const hipError_t e = copy_state(a.dfinal, a.dh0, a.batch * a.width, stream);
        if (e != hipSuccess) return e;
    }
    const int64_t rows = a.seq_len > 0 ? a.batch * a.tiles : 0;
    hipLaunchKernelGGL(recurrence_dtheta_kernel, dim3(unsigned((a.width + kWave - 1) / kWave)), dim3(1024), 0, stream,
                       a.partial, rows, a.theta, a.decay, a.width, a.dtheta);
    return hipGetLastError();
}

}  // namespace mesa
