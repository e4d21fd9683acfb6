// Gradients of the Mesa layer's front and back end (layer_ends.hip has the forward).
//
// Front end, per head and channel, with u = conv4(p), f = u sigma(u), n = 1 / sqrt(|f|^2 + eps)
// rebuilt from the projection p (kept as fp32, bf16 or an 8-bit checkpoint):
//     q, k:  df = n (dq - n^2 f (f . dq));    v: df = dv
//     du_t = df sigma(u) (1 + u (1 - sigma(u)))
//     dp_t = sum_{i=0..3} w_i du_{t+i},  dw_i = sum_{b,t} du_t p_{t-i}
//     da_beta = beta (1 - beta) (dbeta - 2 (1 - cap) dgamma sigma(a_gamma) beta)
//     da_gamma = dgamma (1 - (1 - cap) beta^2) sigma(a_gamma) (1 - sigma(a_gamma))
//     dtheta = dLambda sigma(theta)
// Back end, n = 1 / sqrt(mean(o^2) + eps), z = dy w:
//     do = n (z - n^2 o mean(z o)),  dw = sum_{b,t} dy o n
//
// One pass over each stream: a token of d channels is d / 4 lanes, and each such group of
// lanes walks its own run of consecutive tokens, holding the last three projections (for u
// and dw) and the last three du (for dp, which lags three tokens behind).  A run reads
// three tokens before it and recomputes du of three after it.  The filter's gradient stays
// in registers over the run, is added over a workgroup's runs in LDS and goes out as one
// partial row; a second small kernel adds the rows in order.
//
// Both are HBM-bound.  8 sequences of 16 heads of 128 channels, 2048 tokens, from checkpoints to
// bf16, no filter on the values: front end 145 to 148 us (680 MB, 4.6 TB/s; its vector units are busy
// for seven tenths of that), back end 43 us (236 MB, 5.5 TB/s), each with 5 us for the sums of the
// partial rows.
#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"

namespace mesa {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;     // tokens loaded together
constexpr int kHalo = 3;

constexpr int groups_of(int d) { return kThreads / (d / 4); }  // runs of a workgroup

// Tokens of a run: long runs repeat the three halo tokens less often, short ones give
// enough workgroups when there are few tokens.  With runs of 64, 32 and 16, sequences of 16 heads of
// 2048 tokens of 128 channels from 8 bits: front end 1 sequence 36, 24, 23 us, 2 42, 36, 38, 4 72, 75,
// 81, 8 147, 149, 157, 16 300, 310, 353; back end 24, 14, 10, 24, 16, 14, 37, 26, 25, 48, 43, 45 and 81, 88,
// 82.  2 x 4 heads of 777 fp32 tokens of 64 channels: 29, 17, 11 and 17, 10, 7.  The rule takes 16, 16,
// 16, 32, 64 and 16: the front end of 4 sequences alone would take longer ones.
int run_of(int64_t sequences, int64_t seq_len, int d)
{
    for (int run : {64, 32}) {
        const int64_t blocks = sequences * ((seq_len + int64_t(run) * groups_of(d) - 1) / (int64_t(run) * groups_of(d)));
        if (blocks >= 1024) return run;
    }
    return 16;
}
int64_t blocks_of(int64_t seq_len, int d, int run)
{
    const int64_t per = int64_t(run) * groups_of(d);
    return (seq_len + per - 1) / per;
}

// Sum over the 16 or 32 consecutive lanes of a group; every lane of it receives the sum.
template <int L>
__device__ __forceinline__ float group_sum(float v)
{
    static_assert(L == 16 || L == 32, "a row of lanes, or two");
    v += dpp_f32<kDppQuadSwap1>(v, v);
    v += dpp_f32<kDppQuadSwap2>(v, v);
    v += dpp_f32<kDppRowRor4>(v, v);
    v += dpp_f32<kDppRowRor8>(v, v);
    if constexpr (L == 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// 1 / sqrt(x) of a square sum and an eps.  The instruction takes a subnormal as 0, which it can be if
// nothing is added to tiny rows; Small: as the forward then, where it counts.
template <bool Small>
__device__ __forceinline__ float rsq(float x)
{
    return Small ? rsqrtf(x) : __builtin_amdgcn_rsqf(x);
}
// Whether an eps leaves subnormal sums as they are.
__host__ __device__ __forceinline__ bool small_eps(float eps) { return eps < 0x1p-126f; }

// Four channels at element `at` of a dense array of T, or of a checkpoint whose exponent
// bytes start at `bytes` (its width is a multiple of 32, so element e has byte e / 32).
template <typename T>
struct Held {
    using Raw = typename Lane4<T>::Raw;
    __device__ static Raw load(const void* base, int64_t, int64_t at) { return Lane4<T>::template load<true>(base, at, 4); }
    __device__ static void widen(const Raw& r, float (&x)[4]) { Lane4<T>::widen(r, x); }
};
template <>
struct Held<q8_t> {
    using Raw = Q8Raw;
    __device__ static Raw load(const void* base, int64_t bytes, int64_t at)
    {
        return {*reinterpret_cast<const uint32_t*>(static_cast<const int8_t*>(base) + at), static_cast<const uint8_t*>(base)[bytes + at / kGroup]};
    }
    __device__ static void widen(const Raw& r, float (&x)[4]) { widen_q8(r.codes, group_scale(r.byte), x); }
};

// One stream (kind 0 q, 1 k, 2 v) of one (sequence, head): `blk` its workgroup among those
// of the sequence.
template <typename T, typename Tg, int D, bool Small>
__device__ void stream_grad(const FrontGradArgs& a, int kind, int64_t bh, int64_t blk, int64_t blocks, int run, float* partial,
                            float (&red)[kThreads * 16])
{
    constexpr int LPT = D / 4;
    const int grp = threadIdx.x / LPT, cl = threadIdx.x % LPT;
    const int64_t t0 = (blk * groups_of(D) + grp) * run;
    const int64_t t1 = min<int64_t>(t0 + run, a.seq_len);   // may be <= t0: an idle group
    const int64_t b = bh / a.heads, h = bh % a.heads;
    const void* src = kind == 0 ? a.qp : kind == 1 ? a.kp : a.vp;
    const float* grad = (kind == 0 ? a.dq : kind == 1 ? a.dk : a.dv) + bh * a.seq_len * D + cl * 4;
    void* dst = kind == 0 ? a.dqp : kind == 1 ? a.dkp : a.dvp;
    const float* w = kind == 0 ? a.conv_q : kind == 1 ? a.conv_k : a.conv_v;
    const int64_t stride = a.heads * D;
    const int64_t at0 = b * a.seq_len * stride + h * D + cl * 4;
    const int64_t last = a.seq_len - 1;
    if (w == nullptr) {
        // values that passed through
        for (int s = 0; s < run; s += kBatch) {
            float4 g[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) g[u] = *reinterpret_cast<const float4*>(grad + min<int64_t>(t0 + s + u, last) * D);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int64_t t = t0 + s + u;
                const float y[4] = {g[u].x, g[u].y, g[u].z, g[u].w};
                if (t < t1) stream_store(static_cast<Tg*>(dst) + at0 + t * stride, Lane4<Tg>::narrow(y));
            }
        }
        return;
    }
    const int64_t bytes = checkpoint_exponents_at(a.batch * a.seq_len, stride);
    float wt[4][4], dw[4][4], prev[4][3], du[4][3];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float4 f = *reinterpret_cast<const float4*>(w + (h * D + cl * 4 + c) * 4);
        wt[c][0] = f.x, wt[c][1] = f.y, wt[c][2] = f.z, wt[c][3] = f.w;
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[c][i] = 0.0f;
#pragma unroll
        for (int i = 0; i < 3; ++i) prev[c][i] = du[c][i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const int64_t t = t0 - 1 - i;
        if (t >= 0 && t <= last) {
            float x[4];
            Held<T>::widen(Held<T>::load(src, bytes, at0 + t * stride), x);
#pragma unroll
            for (int c = 0; c < 4; ++c) prev[c][i] = x[c];
        }
    }
    // every group takes all the steps (the sums over a group need its lanes together)
#pragma unroll 1
    for (int s = 0; s < run + kHalo; s += kBatch) {
        typename Held<T>::Raw px[kBatch];
        float4 gx[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t t = min<int64_t>(t0 + s + u, last);
            px[u] = Held<T>::load(src, bytes, at0 + t * stride);
            gx[u] = *reinterpret_cast<const float4*>(grad + t * D);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t t = t0 + s + u;
            const bool there = t <= last;
            float x[4], uc[4], sg[4], f[4];
            Held<T>::widen(px[u], x);
            const float g[4] = {gx[u].x, gx[u].y, gx[u].z, gx[u].w};
            float ss = 0.0f, dot = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uc[c] = fmaf(wt[c][3], prev[c][2], fmaf(wt[c][2], prev[c][1], fmaf(wt[c][1], prev[c][0], wt[c][0] * x[c])));
                sg[c] = sigmoid_fast(uc[c]);
                f[c] = uc[c] * sg[c];
                ss = fmaf(f[c], f[c], ss);
                dot = fmaf(f[c], g[c], dot);
            }
            float n = 1.0f, pull = 0.0f;
            if (kind < 2) {
                n = rsq<Small>(group_sum<LPT>(ss) + a.l2_eps);
                pull = n * (n * group_sum<LPT>(dot));
            }
            float dp[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float df = n * fmaf(-pull, f[c], g[c]);
                const float d = there ? df * sg[c] * fmaf(uc[c], 1.0f - sg[c], 1.0f) : 0.0f;
                if (t < t1) {
                    dw[c][0] = fmaf(d, x[c], dw[c][0]);
                    dw[c][1] = fmaf(d, prev[c][0], dw[c][1]);
                    dw[c][2] = fmaf(d, prev[c][1], dw[c][2]);
                    dw[c][3] = fmaf(d, prev[c][2], dw[c][3]);
                }
                // du_{t-3}, du_{t-2}, du_{t-1} are du[2], du[1], du[0]
                dp[c] = fmaf(wt[c][3], d, fmaf(wt[c][2], du[c][0], fmaf(wt[c][1], du[c][1], wt[c][0] * du[c][2])));
                du[c][2] = du[c][1], du[c][1] = du[c][0], du[c][0] = d;
                prev[c][2] = prev[c][1], prev[c][1] = prev[c][0], prev[c][0] = x[c];
            }
            if (t - kHalo >= t0 && t - kHalo < t1)
                stream_store(static_cast<Tg*>(dst) + at0 + (t - kHalo) * stride, Lane4<Tg>::narrow(dp));
        }
    }
    // the workgroup's runs added: red[group][channel][tap]
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(&red[(grp * D + cl * 4 + c) * 4]) = make_float4(dw[c][0], dw[c][1], dw[c][2], dw[c][3]);
    __syncthreads();
    float* out = partial + ((b * blocks + blk) * a.heads + h) * D * 4;
    for (int e = threadIdx.x; e < D * 4; e += kThreads) {
        float s = red[e];
        for (int q = 1; q < groups_of(D); ++q) s += red[q * D * 4 + e];
        out[e] = s;
    }
}

// How the workgroups of a call are dealt out.
struct FrontPlan {
    int run_k, run_v;
    int64_t blocks_k, blocks_v;              // workgroups of a (sequence, head)
    int64_t part_k, part_v;                  // partial rows' floats of q or k, of v
    int64_t gate_blocks;
};
__host__ FrontPlan front_plan(int64_t batch, int64_t heads, int64_t seq_len, int d_k, int d_v)
{
    FrontPlan p;
    p.run_k = run_of(batch * heads, seq_len, d_k);
    p.run_v = run_of(batch * heads, seq_len, d_v);
    p.blocks_k = blocks_of(seq_len, d_k, p.run_k);
    p.blocks_v = blocks_of(seq_len, d_v, p.run_v);
    p.part_k = batch * p.blocks_k * heads * d_k * 4;
    p.part_v = batch * p.blocks_v * heads * d_v * 4;
    p.gate_blocks = (batch * seq_len * heads + kThreads - 1) / kThreads;
    return p;
}

template <typename T, typename Tg, int DK, int DV>
__global__ __launch_bounds__(kThreads) void frontend_grad_kernel(FrontGradArgs a, FrontPlan p)
{
    __shared__ __align__(16) float red[kThreads * 16];
    const int64_t bh_all = a.batch * a.heads;
    const int64_t nk = bh_all * p.blocks_k, nv = bh_all * p.blocks_v;
    int64_t id = blockIdx.x;
    if (id < 2 * nk) {
        const int kind = id < nk ? 0 : 1;
        id -= kind * nk;
        float* partial = a.partial + kind * p.part_k;
        // a form of its own, since the few instructions more cost both ends 200 us of 195 at the size above
        if (small_eps(a.l2_eps))
            stream_grad<T, Tg, DK, true>(a, kind, id / p.blocks_k, id % p.blocks_k, p.blocks_k, p.run_k, partial, red);
        else
            stream_grad<T, Tg, DK, false>(a, kind, id / p.blocks_k, id % p.blocks_k, p.blocks_k, p.run_k, partial, red);
        return;
    }
    id -= 2 * nk;
    if (id < nv) {
        stream_grad<T, Tg, DV, false>(a, 2, id / p.blocks_v, id % p.blocks_v, p.blocks_v, p.run_v, a.partial + 2 * p.part_k, red);
        return;
    }
    id -= nv;
    if (id < p.gate_blocks) {
        // one thread a gate, in the order of da_gamma and da_beta [B, T, H]
        const int64_t e = id * kThreads + threadIdx.x;
        if (e >= bh_all * a.seq_len) return;
        const int64_t h = e % a.heads, bt = e / a.heads;
        const int64_t at = ((bt / a.seq_len) * a.heads + h) * a.seq_len + bt % a.seq_len;
        float beta_rest, open_rest;
        const float beta = sigmoid_both(a.a_beta[e], beta_rest), open = sigmoid_both(a.a_gamma[e], open_rest);
        const float cut = 1.0f - a.gamma_cap, dg = a.dgamma[at];
        a.da_gamma[e] = dg * (1.0f - cut * beta * beta) * open * open_rest;
        a.da_beta[e] = beta * beta_rest * fmaf(-2.0f * cut * beta * open, dg, a.dbeta[at]);
        return;
    }
    const int64_t e = (id - p.gate_blocks) * kThreads + threadIdx.x;
    if (e < a.heads * DK) a.dtheta[e] = a.dlambda[e] * sigmoid_fast(a.theta[e]);
}

// out[c] = sum of rows of partial [rows, cols], for up to three arrays in one launch.
constexpr int kSumThreads = 1024;
struct Sums {
    const float* partial[3];
    float* out[3];
    int64_t rows[3], cols[3];
    int64_t blocks[3];
};
__global__ __launch_bounds__(kSumThreads) void partial_sum_kernel(Sums s)
{
    __shared__ float part[16][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int64_t id = blockIdx.x;
    int q = 0;
    while (q < 2 && id >= s.blocks[q]) id -= s.blocks[q++];
    const int64_t c = id * kWave + lane;
    float v = 0.0f;
    if (c < s.cols[q])
        for (int64_t r = wave; r < s.rows[q]; r += 16) v += s.partial[q][r * s.cols[q] + c];
    part[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || c >= s.cols[q]) return;
    for (int w = 1; w < 16; ++w) v += part[w][lane];
    s.out[q][c] = v;
}

int64_t blocks_of(const Sums& s) { return s.blocks[0] + s.blocks[1] + s.blocks[2]; }
hipError_t launch_sums(const Sums& s, hipStream_t stream)
{
    const int64_t blocks = blocks_of(s);
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL(partial_sum_kernel, dim3(unsigned(blocks)), dim3(kSumThreads), 0, stream, s);
    return hipGetLastError();
}

template <typename T, typename Tg, int DK, int DV>
hipError_t launch_front(const FrontGradArgs& a, hipStream_t stream)
{
    const FrontPlan p = front_plan(a.batch, a.heads, a.seq_len, DK, DV);
    const int64_t bh = a.batch * a.heads;
    const int64_t blocks = bh * (2 * p.blocks_k + p.blocks_v) + p.gate_blocks + (a.heads * DK + kThreads - 1) / kThreads;
    const int64_t ck = a.heads * DK * 4, cv = a.conv_v != nullptr ? a.heads * DV * 4 : 0;
    const Sums s{{a.partial, a.partial + p.part_k, a.partial + 2 * p.part_k},
                 {a.dconv_q, a.dconv_k, a.dconv_v},
                 {a.batch * p.blocks_k, a.batch * p.blocks_k, a.batch * p.blocks_v},
                 {ck, ck, cv},
                 {(ck + kWave - 1) / kWave, (ck + kWave - 1) / kWave, (cv + kWave - 1) / kWave}};
    if (!grid_fits(blocks, kThreads) || !grid_fits(blocks_of(s), kSumThreads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((frontend_grad_kernel<T, Tg, DK, DV>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    return launch_sums(s, stream);
}

template <typename T, typename Tg>
hipError_t launch_front_dims(const FrontGradArgs& a, hipStream_t stream)
{
    if (a.d_k == 64) return a.d_v == 64 ? launch_front<T, Tg, 64, 64>(a, stream) : launch_front<T, Tg, 64, 128>(a, stream);
    return a.d_v == 64 ? launch_front<T, Tg, 128, 64>(a, stream) : launch_front<T, Tg, 128, 128>(a, stream);
}

// ---------------------------------------------------------------- back end
template <typename T, typename Tg, int D>
__global__ __launch_bounds__(kThreads) void output_norm_grad_kernel(NormGradArgs a, int run, int64_t blocks)
{
    __shared__ __align__(16) float red[kThreads * 4];
    constexpr int LPT = D / 4;
    const int grp = threadIdx.x / LPT, cl = threadIdx.x % LPT;
    const int64_t bh = blockIdx.x / blocks, blk = blockIdx.x % blocks;
    const int64_t b = bh / a.heads, h = bh % a.heads;
    const int64_t t0 = (blk * groups_of(D) + grp) * run, t1 = min<int64_t>(t0 + run, a.seq_len), last = a.seq_len - 1;
    const int64_t bytes = checkpoint_exponents_at(a.batch * a.heads * a.seq_len, D);
    const int64_t o0 = bh * a.seq_len * D + cl * 4, y0 = (b * a.seq_len * a.heads + h) * D + cl * 4, stride = a.heads * D;
    const float4 w4 = *reinterpret_cast<const float4*>(a.weight + h * D + cl * 4);
    const float w[4] = {w4.x, w4.y, w4.z, w4.w};
    float dw[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int s = 0; s < run; s += kBatch) {
        typename Held<T>::Raw ro[kBatch];
        typename Lane4<Tg>::Raw ry[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t t = min<int64_t>(t0 + s + u, last);
            ro[u] = Held<T>::load(a.o, bytes, o0 + t * D);
            ry[u] = Lane4<Tg>::template load<true>(a.dy, y0 + t * stride, 4);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t t = t0 + s + u;
            float o[4], dy[4], z[4], out[4];
            Held<T>::widen(ro[u], o);
            Lane4<Tg>::widen(ry[u], dy);
            float ss = 0.0f, dot = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                z[c] = dy[c] * w[c];
                ss = fmaf(o[c], o[c], ss);
                dot = fmaf(z[c], o[c], dot);
            }
            // n^2 of a small row would overflow, n times the mean of z o is of z's order
            const float n = rsq<true>(group_sum<LPT>(ss) * (1.0f / D) + a.eps);   // no slower here
            const float pull = n * (n * (group_sum<LPT>(dot) * (1.0f / D)));
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                out[c] = n * fmaf(-pull, o[c], z[c]);
                if (t < t1) dw[c] = fmaf(dy[c], o[c] * n, dw[c]);
            }
            if (t < t1) Lane4<float>::store<true>(a.d_o, o0 + t * D, 4, out);
        }
    }
    *reinterpret_cast<float4*>(&red[threadIdx.x * 4]) = make_float4(dw[0], dw[1], dw[2], dw[3]);
    __syncthreads();
    for (int e = threadIdx.x; e < D; e += kThreads) {
        float s = red[e];
        for (int q = 1; q < groups_of(D); ++q) s += red[q * D + e];
        a.partial[((b * blocks + blk) * a.heads + h) * D + e] = s;
    }
}

template <typename T, typename Tg, int D>
hipError_t launch_norm(const NormGradArgs& a, hipStream_t stream)
{
    const int run = run_of(a.batch * a.heads, a.seq_len, D);
    const int64_t per = blocks_of(a.seq_len, D, run), blocks = a.batch * a.heads * per;
    const int64_t cols = a.heads * D;
    const Sums s{{a.partial, nullptr, nullptr}, {a.dweight, nullptr, nullptr}, {a.batch * per, 0, 0}, {cols, 0, 0},
                 {(cols + kWave - 1) / kWave, 0, 0}};
    if (!grid_fits(blocks, kThreads) || !grid_fits(blocks_of(s), kSumThreads)) return hipErrorInvalidConfiguration;
    if (blocks > 0) {
        hipLaunchKernelGGL((output_norm_grad_kernel<T, Tg, D>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a, run, per);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return launch_sums(s, stream);
}

template <typename T, typename Tg>
hipError_t launch_norm_dims(const NormGradArgs& a, hipStream_t stream)
{
    return a.d_v == 64 ? launch_norm<T, Tg, 64>(a, stream) : launch_norm<T, Tg, 128>(a, stream);
}

}  // namespace

int64_t front_grad_partial_floats(int64_t batch, int64_t heads, int64_t seq_len, int d_k, int d_v)
{
    const FrontPlan p = front_plan(batch, heads, seq_len, d_k, d_v);
    return 2 * p.part_k + p.part_v;
}

int64_t norm_grad_partial_floats(int64_t batch, int64_t heads, int64_t seq_len, int d_v)
{
    return batch * blocks_of(seq_len, d_v, run_of(batch * heads, seq_len, d_v)) * heads * d_v;
}

hipError_t launch_frontend_backward(const FrontGradArgs& a, hipStream_t stream)
{
    if (a.heads == 0) return hipSuccess;
    const bool g16 = a.grad_dtype == kBf16;
    if (a.dtype == kQ8) return g16 ? launch_front_dims<q8_t, bf16_t>(a, stream) : launch_front_dims<q8_t, float>(a, stream);
    if (a.dtype == kBf16) return g16 ? launch_front_dims<bf16_t, bf16_t>(a, stream) : launch_front_dims<bf16_t, float>(a, stream);
    return g16 ? launch_front_dims<float, bf16_t>(a, stream) : launch_front_dims<float, float>(a, stream);
}

hipError_t launch_output_norm_backward(const NormGradArgs& a, hipStream_t stream)
{
    if (a.heads == 0) return hipSuccess;
    const bool g16 = a.grad_dtype == kBf16;
    if (a.dtype == kQ8) return g16 ? launch_norm_dims<q8_t, bf16_t>(a, stream) : launch_norm_dims<q8_t, float>(a, stream);
    return g16 ? launch_norm_dims<float, bf16_t>(a, stream) : launch_norm_dims<float, float>(a, stream);
}

}  // namespace mesa
