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
// 1 - a^2 is -expm1(2 l): its series for a small argument, 1 - a a otherwise.
//
// A span of tokens acts on the state as h -> A h + B, and spans compose, so time is cut:
// a lane holds a few consecutive tokens of four channels in registers, a row of 16 lanes the
// 64 channels of such a run (128 bytes of bf16 a token), a workgroup 32 runs in time.  The runs'
// (A, B) meet in LDS, where one wave passes through them with a channel in each lane, and
// across workgroups in the workspace (below), so every input is read once.  A reset inside a
// span is kept as the sign of A (A is never negative otherwise), since 0 times a state that is
// not finite would not forget it.  All of it is fp32 and in a fixed order.
//
// 8 x 2048 tokens of 2048 bf16 channels: forward 51 us, 268 MB or 5.2 TB/s, what a copy of that
// size reaches; with the inputs' checkpoints written as well a forward of 4 x 2000 tokens of 1536
// packed channels takes 40 us (3.4 TB/s): 78 vector instructions an element, 45 of them for packing
// and resets.  Backward from checkpoints to bf16 gradients 95 to 98 us (3.9 TB/s): ten
// transcendentals and some sixty other instructions an element keep the vector units busy for four
// fifths of the time, and the rest is each workgroup waiting for its first loads and its walk; from
// bf16 tensors 108 us (4.4 TB/s).  fp32, 4 x 2048 tokens of 2048: forward 44 us, backward 86 us (6.1
// and 5.5 TB/s).  One row of 16381 tokens: 60 us, its 64 tiles one behind the other.  One token of
// 1 x 2048 or 256 x 2048 channels is one launch.
#include <algorithm>
#include <type_traits>

#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"

namespace mesa {

// The multiplication that takes 0 times anything as 0.
__device__ float mul_zero_wins(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

namespace {

constexpr int kRows = 32;              // runs of tokens of a workgroup, one to a row of lanes
// A workgroup of rows of Across lanes, four channels in each.
template <int Across>
struct Form {
    static constexpr int kAcross = Across, kCh = 4 * Across, kWaveRows = kWave / Across, kWaves = kRows / kWaveRows, kThreads = kWaves * kWave;
    static_assert(kCh <= kWave, "the walk has a channel in each lane");
};
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
// adds a token to the span (A, B) of those before it
template <bool Reset>
__device__ __forceinline__ void take(Span token, float& A, float& B)
{
    const Span s = join<Reset>({A, B}, token);
    A = s.A, B = s.B;
}

// The four theta of a lane whose first channel is channel c of a slab of cols; a channel past the
// last takes the last one's.
__device__ __forceinline__ void load_theta(const float* slab, int c, int cols, float (&t)[4])
{
#pragma unroll
    for (int v = 0; v < 4; ++v) t[v] = slab[uint32_t(min(c + v, cols - 1))];
}
// The per-channel constants: by = -decay: log a_t = k s_t; by = -decay log2(e): log2 a_t = k s_t.
__device__ __forceinline__ void rates_of(const float (&t)[4], float by, float (&k)[4])
{
#pragma unroll
    for (int v = 0; v < 4; ++v) k[v] = by * softplus_fast(t[v]);
}

// 1 - a^2 = 1 - 4^z for z <= 0 and a = 2^z as rounded: for u = -2 ln 2 z below 1/8 the series
// u - u^2/2 + u^3/6 - u^4/24 + u^5/120, written in z (what is left out is below u^6/720, 5e-8 of
// the sum); above, 1 - a a keeps all but three bits.
// `least` is added to the former.
__device__ __forceinline__ float one_minus_square(float z, float a, float least = 0.0f)
{
    constexpr float w = -2.0f * kLn2;
    float p = w * w * w * w * w / 120.0f;
    p = fmaf(p, z, -w * w * w * w / 24.0f);
    p = fmaf(p, z, w * w * w / 6.0f);
    p = fmaf(p, z, -w * w / 2.0f);
    p = fmaf(p, z, w);
    return z > 0.125f / w ? fmaf(p, z, least) : fmaf(-a, a, 1.0f);
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

// ---------------------------------------------------------------- the walk over tiles
// A tile's workgroup needs the state that enters it: the spans of the tiles before it,
// applied one after the other.  Tiles are taken in groups of kJoin: a tile publishes its span
// as soon as it knows it, without waiting for anything; the last tile of a group publishes
// the state that leaves the group instead, once it has it.  A tile reads the state that
// entered its group and the spans of the (at most kJoin - 1) tiles of the group before it.
//
// A workgroup takes its tile by drawing a ticket when it starts, and waits only for tiles of
// smaller tickets of its slab; those are held by workgroups that run already, and the smallest ticket
// not yet finished waits for nothing, so every wait ends whatever the order and the number
// of workgroups that fit the GPU.  A span and its "published" mark are one 8-byte word
// written and read with single relaxed accesses of agent scope, so no other memory has to be
// ordered.  The words start as kUnset, written by a fill kernel ahead on the stream.
constexpr int kJoin = 16;
constexpr int kLook = 8;   // words that a lane asks for at once
constexpr uint64_t kUnset = ~uint64_t(0);
// Ticket counters, one for each slab of channels, ahead of the spans, each in a cache line of
// its own; in 64-bit words.
constexpr int kCounterWords = 16;
__host__ __device__ inline int64_t ticket_words(int64_t slabs) { return slabs * kCounterWords; }

__device__ __forceinline__ void publish(uint64_t* at, Span s)
{
    uint64_t w = uint64_t(__float_as_uint(s.A)) | (uint64_t(__float_as_uint(s.B)) << 32);
    if (w == kUnset) w = 0xFFFFFFFF7FC00000ull;   // two NaNs with those very bits
    __hip_atomic_store(at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ uint64_t look(const uint64_t* at)
{
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The word at `at` of every lane that wants one, once all of them are published; w: what was
// there at a first look.
__device__ __forceinline__ Span await(const uint64_t* at, bool wanted, uint64_t w)
{
    while (__any(wanted && w == kUnset)) {
        __builtin_amdgcn_s_sleep(1);
        if (wanted) w = look(at);
    }
    return {__uint_as_float(uint32_t(w)), __uint_as_float(uint32_t(w >> 32))};
}

__global__ __launch_bounds__(256) void recurrence_fill_kernel(ulonglong2* words, int64_t n)
{
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) words[i] = make_ulonglong2(kUnset, kUnset);
}

// What the lane rows of a workgroup do to the state, in shared memory: a plane of their A and one
// of their B, by time.
template <int kCh>
using Plane = float[kRows][kCh];

template <int kCh>
__device__ __forceinline__ void put(Plane<kCh>& p, int r, int col, const float (&x)[4])
{
    *reinterpret_cast<float4*>(&p[r][col * 4]) = make_float4(x[0], x[1], x[2], x[3]);
}
template <int kCh>
__device__ __forceinline__ void get(const Plane<kCh>& p, int r, int col, float (&x)[4])
{
    const float4 f = *reinterpret_cast<const float4*>(&p[r][col * 4]);
    x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
}
// for a wave whose lanes take a channel each (Back: from the last row to the first): all rows
// together, and from the state ahead of them the one that enters each; returns the one that
// leaves them
template <bool Reset, bool Back, int kCh>
__device__ __forceinline__ Span join_rows(const Plane<kCh>& A, const Plane<kCh>& B, int lane)
{
    Span s = nothing();
#pragma unroll 8
    for (int r = 0; r < kRows; ++r) {
        const int at = Back ? kRows - 1 - r : r;
        s = join<Reset>(s, {A[at][lane], B[at][lane]});
    }
    return s;
}
template <bool Reset, bool Back, int kCh>
__device__ __forceinline__ float pass_rows(const Plane<kCh>& A, const Plane<kCh>& B, Plane<kCh>& in, int lane, float h)
{
#pragma unroll 8
    for (int r = 0; r < kRows; ++r) {
        const int at = Back ? kRows - 1 - r : r;
        const Span s = {A[at][lane], B[at][lane]};
        in[at][lane] = h;
        h = apply<Reset>(s, h);
    }
    return h;
}

// The workgroup's place in the call.  Its slab of channels goes by its index, so that the
// channels' constants are on their way while the ticket is drawn (a counter for each slab);
// the ticket gives the sequence and the step of the walk, steps slower than sequences, so
// that a tile's predecessors started long before it where there are many sequences.
struct Place {
    int64_t b;
    int step;
};
__device__ __forceinline__ int draw_ticket(uint64_t* words, bool many, int slab, int slabs)
{
    if (!many) return int(blockIdx.x) / slabs;
    if (threadIdx.x != 0) return 0;
    return int(__hip_atomic_fetch_add(reinterpret_cast<uint32_t*>(words + slab * kCounterWords), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u);
}
__device__ __forceinline__ Place place_of(int ticket, bool many, int64_t batch, int& shared)
{
    if (many) {
        if (threadIdx.x == 0) shared = ticket;
        __syncthreads();
        ticket = shared;
    }
    const uint32_t id = uint32_t(__builtin_amdgcn_readfirstlane(ticket)), step = id / uint32_t(batch);
    return {int64_t(id - step * uint32_t(batch)), int(step)};
}

// A tile's part in the walk, by waves with a channel in each lane.  `step` is the tile's place in
// the walk, `first` the state ahead of the whole walk.  The forward's first wave does all of it;
// in the backward pass, whose workgroups have longer to wait, a second one publishes meanwhile
// (gradients from checkpoints of 8 x 2048 tokens of 2048 102 us and 98; the forward, which would
// need a plane more for it, 52 and 55).
template <bool Reset, bool Back, class F>
struct Walk {
    uint64_t* spans;          // of the sequence's tiles, this lane's channel
    uint64_t* leaves;         // of its groups
    int64_t width;
    int step, steps;
    bool mine;                // the lane has a channel
    float start;              // entering the walk
    uint64_t seen[kLook];     // what the first words held: entry 0 the state entering the group, e the group's tile e - 1

    __device__ void find(uint64_t* words, int64_t batch, int64_t b, int step_, int steps_, int64_t width_, int slab)
    {
        step = step_, steps = steps_, width = width_;
        const int64_t slabs = (width + F::kCh - 1) / F::kCh, groups = steps / kJoin;
        const int lane = threadIdx.x % kWave;
        const int64_t ch = int64_t(slab) * F::kCh + lane;
        mine = lane < F::kCh && ch < width;
        spans = words + ticket_words(slabs) + b * steps * width + ch;
        leaves = words + ticket_words(slabs) + batch * steps * width + b * groups * width + ch;
    }
    // Taken before the barrier that makes the rows visible, so that the look's way to memory is
    // part of the wait for the other waves.
    __device__ void look_ahead(const float* first, int64_t b, int slab)
    {
        const int group = step / kJoin, at = step % kJoin;
        start = group == 0 && first != nullptr && mine ? first[b * width + int64_t(slab) * F::kCh + threadIdx.x % kWave] : 0.0f;
        seen[0] = group > 0 && mine ? look(leaves + int64_t(group - 1) * width) : 0;
#pragma unroll
        for (int e = 1; e < kLook; ++e) seen[e] = e <= at && mine ? look(entry(group, e)) : 0;
    }
    __device__ const uint64_t* entry(int group, int e) const { return spans + int64_t(group * kJoin + e - 1) * width; }

    // Publishes this tile's span.  It waits for nothing, so nobody waits for it in a circle.
    __device__ void tell(const Plane<F::kCh>& A, const Plane<F::kCh>& B)
    {
        const int lane = threadIdx.x % kWave;
        if (lane >= F::kCh || step % kJoin == kJoin - 1 || step + 1 >= steps) return;
        __builtin_amdgcn_s_setprio(3);   // other workgroups wait for it
        const Span s = join_rows<Reset, Back>(A, B, lane);
        if (mine) publish(spans + int64_t(step) * width, s);
        __builtin_amdgcn_s_setprio(0);
    }
    // The rows' entering states into the plane `in` (which may be B, once told): takes in what the
    // tiles before this one published, and passes through the rows.
    __device__ void pass(const Plane<F::kCh>& A, const Plane<F::kCh>& B, Plane<F::kCh>& in)
    {
        const int lane = threadIdx.x % kWave, group = step / kJoin, at = step % kJoin;
        if (lane >= F::kCh) return;
        __builtin_amdgcn_s_setprio(3);   // the other waves wait for it, and other workgroups
        float h = group > 0 ? await(leaves + int64_t(group - 1) * width, mine, seen[0]).B : start;
#pragma unroll
        for (int e = 1; e < kLook; ++e)
            if (e <= at) h = apply<Reset>(await(entry(group, e), mine, seen[e]), h);
#pragma unroll 1
        for (int e0 = kLook; e0 <= at; e0 += kLook) {
#pragma unroll
            for (int e = 0; e < kLook; ++e) seen[e] = e0 + e <= at && mine ? look(entry(group, e0 + e)) : 0;
#pragma unroll
            for (int e = 0; e < kLook; ++e)
                if (e0 + e <= at) h = apply<Reset>(await(entry(group, e0 + e), mine, seen[e]), h);
        }
        h = pass_rows<Reset, Back>(A, B, in, lane, h);
        if (mine && at == kJoin - 1 && step + 1 < steps) publish(leaves + int64_t(group) * width, {-0.0f, h});
        __builtin_amdgcn_s_setprio(0);
    }
};

// Makes a value opaque at this point: what is derived from it is derived here again, instead
// of being kept in registers from an earlier place.
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(uint32_t& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(uint2& r) { pin(r.x), pin(r.y); }
__device__ __forceinline__ void pin(float4& r) { pin(r.x), pin(r.y), pin(r.z), pin(r.w); }
__device__ __forceinline__ void pin(Q8Raw& r) { pin(r.codes); }

// ---------------------------------------------------------------- forward
// Tokens of a lane: eight where nothing but the state leaves the tile (8 x 2048 tokens of 2048
// bf16: 51 us, 58 with four); four where the inputs' codes do as well (4 x 2000 of 1536: 42 us
// with eight, 40 with four) and in the narrow form, whose calls are short (2 x 100 tokens of 768
// fp32: 7.6 us with eight, 6.0 with four).
template <class F, bool Kept>
constexpr int kFwdSub = F::kAcross == 16 && !Kept ? 8 : 4;
template <class F, bool Kept>
constexpr int kFwdTile = kRows * kFwdSub<F, Kept>;   // tokens of a workgroup

// A tile's rows are read and written, on the vector path, at an address that the whole wave
// shares plus an offset of the lane's own in 32 bits (rows at most kNearStride elements apart),
// made opaque at each use so that no 64-bit addresses are formed ahead and held.
constexpr int64_t kNearStride = int64_t(1) << 22;

template <typename R>
__device__ __forceinline__ R load_off(const void* base, uint32_t& off)
{
    pin(off);
    return *reinterpret_cast<const R*>(static_cast<const char*>(base) + off);
}
template <typename T>
__device__ __forceinline__ typename Lane4<T>::Raw load_row(const void* base, int64_t row, uint32_t& off)
{
    return load_off<typename Lane4<T>::Raw>(static_cast<const T*>(base) + row, off);
}
// Four channels of a token: on the vector path at the row's element `row` and off bytes from
// there, otherwise at element `at` of that row, n of them.
template <typename T, bool Vec>
__device__ __forceinline__ void store_row(void* base, int64_t row, uint32_t& off, int64_t at, int n, const float (&y)[4])
{
    if constexpr (Vec) {
        pin(off);
        if (n > 0) stream_store(reinterpret_cast<char*>(static_cast<T*>(base) + row) + off, Lane4<T>::narrow(y));
    } else {
        Lane4<T>::template store<false>(base, row + at, n, y);
    }
}

// A wave's token w0 and those after it: how many of a run of Sub tokens, the row-th of the wave, exist.
template <class F, int Sub>
__device__ __forceinline__ int there_are(int64_t seq_len, int64_t w0, int row)
{
    const int wave = int(max<int64_t>(0, min<int64_t>(seq_len - w0, F::kWaveRows * Sub)));
    return min(max(wave - row * Sub, 0), Sub);
}
// How many of a lane's four channels exist, from channel c of a slab of cols.
__device__ __forceinline__ int channels_of(int c, int cols) { return min(max(cols - c, 0), 4); }

// Eight lanes hold a group of 32 channels: its exponent byte and this lane's four codes.  A lane
// past the last channel (not mine) has no part in it.
__device__ __forceinline__ uint32_t pack_group(const float (&x)[4], bool mine, uint32_t& byte)
{
    uint32_t top = max(max(abs_bits(x[0]), abs_bits(x[1])), max(abs_bits(x[2]), abs_bits(x[3])));
    top = mine ? top : 0u;
    top = max(top, uint32_t(dpp_i32<kDppQuadSwap1>(int(top), int(top))));
    top = max(top, uint32_t(dpp_i32<kDppQuadSwap2>(int(top), int(top))));
    top = max(top, uint32_t(dpp_i32<kDppRowHalfMirror>(int(top), int(top))));
    byte = group_exponent(__uint_as_float(top));
    return pack_codes(x, byte);
}

// The resets of a wave's tokens, bit t for its token t, the same in every lane; few waves have
// any, and the others' arithmetic is that without resets.  Lane row `row` of Sub tokens:
// whether its token j is one, and whether token j of any row is.
template <bool Reset, class F, int Sub>
struct Cuts {
    static_assert(F::kWaveRows * Sub <= 64, "a wave's tokens are the bits of one ballot");
    uint64_t all;
    uint32_t mine;
    // The mark of the wave's token `lane`, asked for ahead of the tiles: loads return in order.
    __device__ static uint32_t ask(const uint8_t* reset, int64_t at, int64_t left)
    {
        const int lane = threadIdx.x % kWave;
        return Reset && reset != nullptr && lane < F::kWaveRows * Sub && lane < left ? reset[at + lane] : 0u;
    }
    __device__ Cuts(uint32_t mark, int row)
    {
        all = Reset ? __ballot(mark != 0) : 0;
        mine = uint32_t(all >> (row * Sub));
    }
    __device__ bool lane(int j) const { return Reset && ((mine >> j) & 1u) != 0; }
    __device__ bool any(int j) const
    {
        uint64_t rows = 0;
#pragma unroll
        for (int r = 0; r < F::kWaveRows; ++r) rows |= uint64_t(1) << (r * Sub);
        return Reset && (all & (rows << j)) != 0;
    }
};

template <typename T, bool Vec, bool Reset, bool Kept, class F>
__global__ __launch_bounds__(F::kThreads, (Vec ? 4 : 2)) void recurrence_kernel(RecurrenceArgs a)
{
    constexpr int kAcross = F::kAcross, kCh = F::kCh, kWaveRows = F::kWaveRows, kSub = kFwdSub<F, Kept>, kTile = kFwdTile<F, Kept>;
    static_assert(kTile % kBlock == 0 && kBlock % kSub == 0, "a state block starts at a lane's first token");
    __shared__ struct {
        Plane<kCh> A, B;
        int ticket;
    } sh;
    const int slabs = int((a.width + kCh - 1) / kCh);
    const int slab = int(blockIdx.x) % slabs, ticket = draw_ticket(a.words, a.tiles > 1, slab, slabs);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = lane / kAcross, col = lane % kAcross;
    const int64_t ch0 = int64_t(slab) * kCh, ch = ch0 + col * 4;
    const int cols = int(min<int64_t>(a.width - ch0, kCh)), n = channels_of(col * 4, cols);
    float theta[4], k[4];
    load_theta(a.theta + ch0, col * 4, cols, theta);
    const Place at = place_of(ticket, a.tiles > 1, a.batch, sh.ticket);
#pragma unroll
    for (int v = 0; v < 4; ++v) pin(theta[v]);   // here before the tile is asked for, or it would be waited for with it
    const int64_t w0 = int64_t(at.step) * kTile + wave * kWaveRows * kSub;  // the wave's first token
    const int64_t token0 = at.b * a.seq_len + w0;
    const int left = there_are<F, kSub>(a.seq_len, w0, row);  // of the lane's tokens
    const uint32_t mark = Cuts<Reset, F, kSub>::ask(a.reset, token0, a.seq_len - w0);

    // Tokens past the end come after all others, so the state that they would leave is used by
    // nobody: they and channels past the last are read as copies of existing ones.
    typename Lane4<T>::Raw rx[kSub], rr[kSub], ri[kSub];
    if (Vec && w0 + kWaveRows * kSub <= a.seq_len) {
        uint32_t off = (uint32_t(row * kSub) * uint32_t(a.stride) + (n > 0 ? col * 4 : 0)) * uint32_t(sizeof(T));
#pragma unroll
        for (int j = 0; j < kSub; ++j) {
            const int64_t at_row = (token0 + j) * a.stride + ch0;
            rx[j] = load_row<T>(a.x, at_row, off);
            rr[j] = load_row<T>(a.r, at_row, off);
            ri[j] = load_row<T>(a.i, at_row, off);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kSub; ++j) {
            const int64_t at_row = (at.b * a.seq_len + min<int64_t>(w0 + row * kSub + j, a.seq_len - 1)) * a.stride;
            rx[j] = Lane4<T>::template load_near<Vec>(a.x, at_row, ch, ch0, a.width - 1);
            rr[j] = Lane4<T>::template load_near<Vec>(a.r, at_row, ch, ch0, a.width - 1);
            ri[j] = Lane4<T>::template load_near<Vec>(a.i, at_row, ch, ch0, a.width - 1);
        }
    }
    const Cuts<Reset, F, kSub> cuts(mark, row);
    rates_of(theta, -a.decay * kLog2e, k);
    if constexpr (Kept) {
        // ordinary stores: the backward pass is the next to read them
        uint8_t* const kept[3] = {a.kept_x, a.kept_r, a.kept_i};
        const int64_t groups = (a.width + kGroup - 1) / kGroup;
        const int64_t codes_at = token0 * a.width + ch0;
        const int64_t bytes_at = checkpoint_exponents_at(a.batch * a.seq_len, a.width) + token0 * groups + ch0 / kGroup;
        const uint32_t c_off = uint32_t(row * kSub) * uint32_t(a.width) + col * 4, b_off = uint32_t(row * kSub) * uint32_t(groups) + col / 8;
#pragma unroll
        for (int j = 0; j < kSub; ++j) {
            uint32_t codes[3], byte[3];
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                float x[4];
                Lane4<T>::widen(q == 0 ? rx[j] : q == 1 ? rr[j] : ri[j], x);
                codes[q] = pack_group(x, n > 0, byte[q]);
            }
            if (j < left && n > 0) {
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    if constexpr (Vec) {
                        *reinterpret_cast<uint32_t*>(kept[q] + codes_at + j * a.width + c_off) = codes[q];
                    } else {
                        uint8_t* out = kept[q] + codes_at + (row * kSub + j) * a.width + col * 4;
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (v < n) out[v] = uint8_t(codes[q] >> (8 * v));
                    }
                }
                if (col % 8 == 0) {
#pragma unroll
                    for (int q = 0; q < 3; ++q) {
                        if constexpr (Vec)
                            kept[q][bytes_at + j * groups + b_off] = uint8_t(byte[q]);
                        else
                            kept[q][bytes_at + (row * kSub + j) * groups + col / 8] = uint8_t(byte[q]);
                    }
                }
            }
        }
    }
    Span e[kSub][4];
    float ownA[4], ownB[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) ownA[v] = 1.0f, ownB[v] = 0.0f;
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
        float x[4], r[4], i[4];
        pin(rx[j]), pin(rr[j]), pin(ri[j]);
        Lane4<T>::widen(rx[j], x);
        Lane4<T>::widen(rr[j], r);
        Lane4<T>::widen(ri[j], i);
#pragma unroll
        for (int v = 0; v < 4; ++v) e[j][v] = terms<false>(x[v], r[v], i[v], k[v], false);
        if (cuts.any(j)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                if (cuts.lane(j)) e[j][v] = terms<true>(x[v], r[v], i[v], k[v], true);
                take<true>(e[j][v], ownA[v], ownB[v]);
            }
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) take<false>(e[j][v], ownA[v], ownB[v]);
        }
    }
    put<kCh>(sh.A, wave * kWaveRows + row, col, ownA);
    put<kCh>(sh.B, wave * kWaveRows + row, col, ownB);
    Walk<Reset, false, F> walk;
    if (wave == 0) walk.find(a.words, a.batch, at.b, at.step, a.tiles, a.width, slab), walk.look_ahead(a.h0, at.b, slab);
    __syncthreads();
    if (wave == 0) walk.tell(sh.A, sh.B), walk.pass(sh.A, sh.B, sh.B);
    __syncthreads();
    float h[4];
    get<kCh>(sh.B, wave * kWaveRows + row, col, h);
    const int64_t t0 = w0 + row * kSub;
    if (a.states != nullptr && t0 % kBlock == 0 && left > 0)
        Lane4<float>::store<false>(a.states, (at.b * ((a.seq_len + kBlock - 1) / kBlock) + t0 / kBlock) * a.width + ch, n, h);
    uint32_t y_off = (uint32_t(row * kSub) * uint32_t(a.width) + col * 4) * uint32_t(sizeof(T));
    float* final_h = a.final_h != nullptr ? a.final_h + at.b * a.width + ch : nullptr;
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
        if (cuts.any(j)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) h[v] = apply<true>(e[j][v], h[v]);
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) h[v] = apply<false>(e[j][v], h[v]);
        }
        if (j < left) {
            store_row<T, Vec>(a.y, (token0 + j) * a.width + ch0, y_off, row * kSub * a.width + col * 4, n, h);
            if (final_h != nullptr && w0 + row * kSub + j == a.seq_len - 1) Lane4<float>::store<false>(final_h, 0, n, h);
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
    float theta[4], k[4];
    load_theta(a.theta + ch, 0, Per, theta);
    rates_of(theta, -a.decay * kLog2e, k);
#pragma unroll
    for (int v = 0; v < Per; ++v) h[v] = apply<true>(terms<true>(x[v], r[v], i[v], k[v], hard), h[v]);
    Lane4<float>::store<Vec>(state_out, b * a.width + ch, Per, h);
    Lane4<T>::template store<Vec>(a.y, b * a.width + ch, Per, h);
}

// ---------------------------------------------------------------- backward
constexpr int kBwdSub = 4;
constexpr int kBwdTile = kRows * kBwdSub;
static_assert(kBwdTile == kBlock, "a tile of the backward pass starts at a kept state");

// x, r or i of the backward pass: a tensor of T, or a checkpoint.  load: a token `row` tokens
// and four channels c4 groups of four past the one that the wave shares, which is what Off holds;
// load_near: any token.
template <typename T>
struct Source {
    using Raw = typename Lane4<T>::Raw;
    struct Off {
        uint32_t at;
        __device__ Off(const RecurrenceGradArgs& a, int row, int c4) : at((uint32_t(row) * uint32_t(a.stride) + c4 * 4) * uint32_t(sizeof(T))) {}
    };
    __device__ static Raw load(const void* base, const RecurrenceGradArgs& a, int64_t token, int64_t ch0, Off& off)
    {
        return load_row<T>(base, token * a.stride + ch0, off.at);
    }
    template <bool Vec>
    __device__ static Raw load_near(const void* base, const RecurrenceGradArgs& a, int64_t token, int64_t ch, int64_t ch0)
    {
        return Lane4<T>::template load_near<Vec>(base, token * a.stride, ch, ch0, a.width - 1);
    }
    // the values times `by`
    __device__ static void widen(const Raw& r, float by, float (&x)[4])
    {
        Lane4<T>::widen(r, x);
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] *= by;
    }
};
template <>
struct Source<q8_t> {
    using Raw = Q8Raw;
    struct Off {
        uint32_t code, byte;
        __device__ Off(const RecurrenceGradArgs& a, int row, int c4)
            : code(uint32_t(row) * uint32_t(a.width) + c4 * 4), byte(uint32_t(row) * uint32_t((a.width + kGroup - 1) / kGroup) + c4 / 8) {}
    };
    __device__ static Raw load(const void* base, const RecurrenceGradArgs& a, int64_t token, int64_t ch0, Off& off)
    {
        const int64_t groups = (a.width + kGroup - 1) / kGroup;
        const int8_t* codes = static_cast<const int8_t*>(base) + token * a.width + ch0;
        const uint8_t* bytes = static_cast<const uint8_t*>(base) + checkpoint_exponents_at(a.batch * a.seq_len, a.width) + token * groups + ch0 / kGroup;
        return {load_off<uint32_t>(codes, off.code), load_off<uint8_t>(bytes, off.byte)};
    }
    template <bool Vec>
    __device__ static Raw load_near(const void* base, const RecurrenceGradArgs& a, int64_t token, int64_t ch, int64_t ch0)
    {
        const int64_t groups = (a.width + kGroup - 1) / kGroup;
        const uint8_t* bytes = static_cast<const uint8_t*>(base) + checkpoint_exponents_at(a.batch * a.seq_len, a.width);
        return {load_codes_near<Vec>(static_cast<const int8_t*>(base) + token * a.width, ch, ch0, a.width - 1),
                bytes[token * groups + min(ch, a.width - 1) / kGroup]};
    }
    __device__ static void widen(const Raw& r, float by, float (&x)[4]) { widen_q8(r.codes, group_scale(r.byte) * by, x); }
};

// From e = exp(-x): sigma(x), and 1 - sigma(x) = e sigma(x) to its own accuracy.  Where e is
// infinite the product counts as 0 instead of the 1 that it is: it only ever multiplies sigma(x), which is 0 there.
__device__ __forceinline__ float gate_of(float e) { return __builtin_amdgcn_rcpf(1.0f + e); }
__device__ __forceinline__ float rest_of(float e, float s) { return mul_zero_wins(e, s); }

// What the walk back needs of an element, all that is kept of it in between.
struct Kept {
    float a, hp, m, er, ei;   // hp: the state's input at first, then the state before the token; exp(-r), exp(-i)
};

// Lean: 16-bit gradients of 8- or 16-bit inputs run two workgroups a compute unit, with 128
// registers a lane, and keep m in LDS.  Other types one workgroup of up to 256.  fp32 inputs, which
// with dy are 64 registers, spill in 128 (48 bytes a lane; 4 x 2048 tokens of 2048, fp32 gradients:
// 86 us so, 99 lean).  fp32 gradients of narrower inputs would be faster lean (from bf16 75 us so, 61
// lean, from 8 bits 81 and 63, of which the aligned forms without resets spill up to 20 bytes).
template <typename T, typename Tg>
constexpr bool kLean = sizeof(T) <= 2 && sizeof(Tg) == 2;

template <bool Lean, class F>
struct BackwardShared {
    Plane<F::kCh> A, on, back, in;    // a row's A is the same on the way forward and on the way back
    int ticket;
};
template <class F>
struct BackwardShared<true, F> : BackwardShared<false, F> {
    float4 m[kBwdSub][F::kThreads];
};

__device__ __forceinline__ float4 to_float4(const float (&x)[4]) { return make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void from_float4(const float4& f, float (&x)[4]) { x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w; }

template <typename T, typename Tg, bool Vec, bool Reset, class F>
__global__ __launch_bounds__(F::kThreads, (kLean<T, Tg> ? 4 : 2)) void recurrence_grad_kernel(RecurrenceGradArgs a)
{
    constexpr int kAcross = F::kAcross, kCh = F::kCh, kWaveRows = F::kWaveRows;
    constexpr bool Lean = kLean<T, Tg>;
    static_assert(F::kWaves >= 3, "a wave for each: the pass back, the states, and publishing, which later tiles wait for");
    __shared__ BackwardShared<Lean, F> sh;
    const int slabs = int((a.width + kCh - 1) / kCh);
    const int slab = int(blockIdx.x) % slabs, ticket = draw_ticket(a.words, a.tiles > 1, slab, slabs);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = lane / kAcross, col = lane % kAcross;
    const int64_t ch0 = int64_t(slab) * kCh, ch = ch0 + col * 4;
    const int cols = int(min<int64_t>(a.width - ch0, kCh)), n = channels_of(col * 4, cols);
    float theta[4], k[4];
    load_theta(a.theta + ch0, col * 4, cols, theta);
    const Place at = place_of(ticket, a.tiles > 1, a.batch, sh.ticket);
#pragma unroll
    for (int v = 0; v < 4; ++v) pin(theta[v]);   // here before the tile is asked for, or it would be waited for with it
    const int64_t tile = a.tiles - 1 - at.step;
    const int64_t w0 = tile * kBwdTile + wave * kWaveRows * kBwdSub;
    const int64_t token0 = at.b * a.seq_len + w0;
    const int left = there_are<F, kBwdSub>(a.seq_len, w0, row);
    const uint32_t mark = Cuts<Reset, F, kBwdSub>::ask(a.reset, token0, a.seq_len - w0);

    typename Source<T>::Raw rx[kBwdSub], rr[kBwdSub], ri[kBwdSub];
    typename Lane4<Tg>::Raw rd[kBwdSub];
    if (Vec && w0 + kWaveRows * kBwdSub <= a.seq_len) {
        typename Source<T>::Off off(a, row * kBwdSub, n > 0 ? col : 0);
        uint32_t d_off = (uint32_t(row * kBwdSub) * uint32_t(a.width) + (n > 0 ? col * 4 : 0)) * uint32_t(sizeof(Tg));
#pragma unroll
        for (int j = 0; j < kBwdSub; ++j) {
            rr[j] = Source<T>::load(a.r, a, token0 + j, ch0, off);
            rx[j] = Source<T>::load(a.x, a, token0 + j, ch0, off);
            ri[j] = Source<T>::load(a.i, a, token0 + j, ch0, off);
            rd[j] = load_row<Tg>(a.dy, (token0 + j) * a.width + ch0, d_off);
        }
    } else {
        // tokens past the end and channels past the last are read as copies of existing ones
#pragma unroll
        for (int j = 0; j < kBwdSub; ++j) {
            const int64_t token = at.b * a.seq_len + min<int64_t>(w0 + row * kBwdSub + j, a.seq_len - 1);
            rr[j] = Source<T>::template load_near<Vec>(a.r, a, token, ch, ch0);
            rx[j] = Source<T>::template load_near<Vec>(a.x, a, token, ch, ch0);
            ri[j] = Source<T>::template load_near<Vec>(a.i, a, token, ch, ch0);
            rd[j] = Lane4<Tg>::template load_near<Vec>(a.dy, token * a.width, ch, ch0, a.width - 1);
        }
    }
    const Cuts<Reset, F, kBwdSub> cuts(mark, row);
    rates_of(theta, -a.decay, k);
    // the lane's tokens: their factors, and what they do together to the state and, on the way
    // back, to its gradient; tokens past the end do nothing to either
    const bool whole = w0 + kWaveRows * kBwdSub <= a.seq_len;
    Kept e[kBwdSub][4];
    float A[4], on[4], back[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) A[v] = 1.0f, on[v] = back[v] = 0.0f;
#pragma unroll
    for (int j = 0; j < kBwdSub; ++j) {
        float x[4], r[4], i[4], m[4], in[4];
        pin(rx[j]), pin(rr[j]), pin(ri[j]);
        Source<T>::widen(rx[j], 1.0f, x);
        Source<T>::widen(rr[j], -kLog2e, r);
        Source<T>::widen(ri[j], -kLog2e, i);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            Kept& q = e[j][v];
            q.er = __builtin_amdgcn_exp2f(r[v]);
            q.ei = __builtin_amdgcn_exp2f(i[v]);
            const float z = k[v] * __builtin_amdgcn_rcpf(fmaf(q.er, kLn2, kLn2));   // s / ln 2
            q.a = __builtin_amdgcn_exp2f(z);
            // at least 2^-60, so that 1 / m is finite: where 1 - a^2 is less, its share of every
            // gradient is below fp32's resolution of the others
            m[v] = __builtin_amdgcn_sqrtf(one_minus_square(z, q.a, 0x1p-120f));
            in[v] = gate_of(q.ei) * x[v];
        }
        const bool cut = cuts.any(j);
        if (cut && cuts.lane(j)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) e[j][v].a = -0.0f, m[v] = 1.0f;
        }
        if (!whole && j >= left) {
#pragma unroll
            for (int v = 0; v < 4; ++v) e[j][v].a = m[v] = 1.0f, in[v] = 0.0f;
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            Kept& q = e[j][v];
            q.hp = m[v] * in[v];
            if (!Lean) q.m = m[v];
            pin(q.er), pin(q.ei);
        }
        if constexpr (Lean) sh.m[j][threadIdx.x] = to_float4(m);
        if (cut) {
#pragma unroll
            for (int v = 0; v < 4; ++v) take<true>({e[j][v].a, e[j][v].hp}, A[v], on[v]);
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) take<false>({e[j][v].a, e[j][v].hp}, A[v], on[v]);
        }
    }
#pragma unroll
    for (int j = kBwdSub - 1; j >= 0; --j) {
        float d[4];
        pin(rd[j]);
        Lane4<Tg>::widen(rd[j], d);
        if (!whole && j >= left) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) back[v] = e[j][v].a * (back[v] + d[v]);   // c -> a (dy + c)
        if (cuts.any(j) && cuts.lane(j)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) A[v] = -0.0f, back[v] = 0.0f;   // a reset's c is 0 whatever comes after (A may be a NaN by now)
        }
    }
    const int my_row = wave * kWaveRows + row;
    put<kCh>(sh.A, my_row, col, A);
    put<kCh>(sh.on, my_row, col, on);
    put<kCh>(sh.back, my_row, col, back);
    const int64_t my = ch0 + lane;
    float state = 0.0f;      // wave 1: the state entering the tile, a channel a lane
    if (wave == 1 && lane < kCh && my < a.width) state = a.states[(at.b * a.tiles + tile) * a.width + my];
    Walk<Reset, true, F> walk;
    if (wave == 0 || wave == 2) walk.find(a.words, a.batch, at.b, at.step, a.tiles, a.width, slab);
    if (wave == 0) walk.look_ahead(a.dfinal, at.b, slab);
    __syncthreads();
    if (wave == 0) walk.pass(sh.A, sh.back, sh.in);
    if (wave == 2) walk.tell(sh.A, sh.back);
    if (wave == 1 && lane < kCh) {
        __builtin_amdgcn_s_setprio(3);
        pass_rows<Reset, false>(sh.A, sh.on, sh.on, lane, state);
        __builtin_amdgcn_s_setprio(0);
    }
    __syncthreads();
    float h[4], c[4], dth[4] = {0.f, 0.f, 0.f, 0.f};
    get<kCh>(sh.on, my_row, col, h);
    get<kCh>(sh.in, my_row, col, c);
#pragma unroll
    for (int j = 0; j < kBwdSub; ++j) {
        float after[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) after[v] = apply<false>({e[j][v].a, e[j][v].hp}, h[v]);
        if (cuts.any(j)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) after[v] = apply<true>({e[j][v].a, e[j][v].hp}, h[v]);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) e[j][v].hp = h[v], h[v] = after[v];
    }
    uint32_t g_off = (uint32_t(row * kBwdSub) * uint32_t(a.grad_stride) + col * 4) * uint32_t(sizeof(Tg));
#pragma unroll
    for (int j = kBwdSub - 1; j >= 0; --j) {
        if (j >= left) continue;
        float x[4], d[4], m[4], gx[4], gr[4], gi[4], dls[4];
        pin(rx[j]), pin(rd[j]);
        Source<T>::widen(rx[j], 1.0f, x);
        Lane4<Tg>::widen(rd[j], d);
        if constexpr (Lean) {
            from_float4(sh.m[j][threadIdx.x], m);
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) m[v] = e[j][v].m;
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const Kept& q = e[j][v];
            const float s = gate_of(q.er), si = gate_of(q.ei);
            const float g = d[v] + c[v], ag = q.a * g;
            gx[v] = g * m[v] * si;
            gi[v] = gx[v] * x[v] * rest_of(q.ei, si);
            // dl s, with s / m first: it is at most m / (2 decay softplus(theta)), where 1 / m beside
            // a large x would overflow and then meet an s of 0
            dls[v] = ag * fmaf(-q.a * (s * __builtin_amdgcn_rcpf(m[v])), si * x[v], s * q.hp);
            gr[v] = dls[v] * (k[v] * rest_of(q.er, s));
            c[v] = ag;
        }
        if (cuts.any(j) && cuts.lane(j)) {
#pragma unroll
            for (int v = 0; v < 4; ++v) dls[v] = gr[v] = c[v] = 0.0f;
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) dth[v] += dls[v];
        const int64_t at_row = (token0 + j) * a.grad_stride + ch0, at = row * kBwdSub * a.grad_stride + col * 4;
        store_row<Tg, Vec>(a.dx, at_row, g_off, at, n, gx);
        store_row<Tg, Vec>(a.dr, at_row, g_off, at, n, gr);
        store_row<Tg, Vec>(a.di, at_row, g_off, at, n, gi);
    }
    if (a.dh0 != nullptr && tile == 0 && wave == 0 && row == 0) Lane4<float>::store<false>(a.dh0, at.b * a.width + ch, n, c);
    // dtheta: the tile's sum of dl s, one row of the partial sums; the rows' sums take the place
    // of their entering states
    put<kCh>(sh.on, my_row, col, dth);
    __syncthreads();
    if (wave == 0 && lane < kCh) {
        float s = 0.0f;
#pragma unroll 8
        for (int r = 0; r < kRows; ++r) s += sh.on[r][lane];
        if (my < a.width) a.partial[(at.b * a.tiles + tile) * a.width + my] = s;
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
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) to[i] = from != nullptr ? from[i] : 0.0f;
}

bool aligned(const void* p, int bytes) { return uintptr_t(p) % uintptr_t(bytes) == 0; }

hipError_t copy_state(const float* from, float* to, int64_t n, hipStream_t stream)
{
    if (to == nullptr) return hipSuccess;
    hipLaunchKernelGGL(recurrence_copy_kernel, dim3(unsigned(std::min<int64_t>((n + 255) / 256, 1 << 16))), dim3(256), 0, stream, from, to, n);
    return hipGetLastError();
}

// Marks every word of a walk as not yet published.
hipError_t clear_walk(uint64_t* words, int64_t batch, int64_t tiles, int64_t width, hipStream_t stream)
{
    const int64_t n = recurrence_walk_bytes(batch, tiles, width) / 16;
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL(recurrence_fill_kernel, dim3(unsigned(std::min<int64_t>((n + 255) / 256, 1024))), dim3(256), 0, stream,
                       reinterpret_cast<ulonglong2*>(words), n);
    return hipGetLastError();
}

// Workgroups of 64 channels read and write whole lines of memory; where there are fewer of
// them than compute units, workgroups of half the channels finish sooner or as soon (777 tokens of
// 2 x 321, fp32 gradient, 84 of the wide ones: 22.5 us wide, 16.2 narrow; 100 tokens of 2 x 768, fp32,
// 24: 8.3 and 6.0; 2048 tokens of 2 x 192 from 8 bits, 96: 13.0 both, 2 x 384, 192: 13.4 and 14.4; not
// from there on: 2 x 512, 256: 13.9 and 14.0, 2 x 1024 17.4 and 23.0, 8 x 2048 97 and 124, forward 50
// and 74).  The narrow ones always look for resets.
using Wide = Form<16>;
using Narrow = Form<8>;

template <class F>
int64_t workgroups(int64_t batch, int64_t tiles, int64_t width) { return batch * tiles * ((width + F::kCh - 1) / F::kCh); }
template <class F, bool Kept>
int64_t tiles_of(int64_t seq_len) { return (seq_len + kFwdTile<F, Kept> - 1) / kFwdTile<F, Kept>; }
bool narrow(int64_t batch, int64_t tiles, int64_t width) { return workgroups<Wide>(batch, tiles, width) < device_compute_units(); }

template <typename T, bool Vec, bool Reset, bool Kept, class F>
hipError_t launch_forward(RecurrenceArgs a, hipStream_t stream)
{
    a.tiles = tiles_of<F, Kept>(a.seq_len);
    if (!grid_fits(workgroups<F>(a.batch, a.tiles, a.width), F::kThreads)) return hipErrorInvalidConfiguration;
    if (hipError_t e = clear_walk(a.words, a.batch, a.tiles, a.width, stream); e != hipSuccess) return e;
    hipLaunchKernelGGL((recurrence_kernel<T, Vec, Reset, Kept, F>), dim3(unsigned(workgroups<F>(a.batch, a.tiles, a.width))),
                       dim3(F::kThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename T, bool Vec, bool Kept>
hipError_t launch_forward_form(const RecurrenceArgs& a, hipStream_t stream)
{
    if (narrow(a.batch, tiles_of<Wide, Kept>(a.seq_len), a.width)) return launch_forward<T, Vec, true, Kept, Narrow>(a, stream);
    return a.reset != nullptr ? launch_forward<T, Vec, true, Kept, Wide>(a, stream) : launch_forward<T, Vec, false, Kept, Wide>(a, stream);
}

template <typename T>
hipError_t launch_forward_type(const RecurrenceArgs& a, hipStream_t stream)
{
    constexpr int bytes = 4 * int(sizeof(T));
    const bool vec = a.width % 4 == 0 && a.stride % 4 == 0 && a.stride <= kNearStride && aligned(a.x, bytes) &&
                     aligned(a.r, bytes) && aligned(a.i, bytes) && aligned(a.y, bytes);
    if (a.kept_x != nullptr) return vec ? launch_forward_form<T, true, true>(a, stream) : launch_forward_form<T, false, true>(a, stream);
    return vec ? launch_forward_form<T, true, false>(a, stream) : launch_forward_form<T, false, false>(a, stream);
}

template <typename T>
hipError_t launch_step_type(const RecurrenceArgs& a, float* state_out, hipStream_t stream)
{
    constexpr int bytes = 4 * int(sizeof(T));
    const bool vec = a.width % 4 == 0 && a.stride % 4 == 0 && aligned(a.x, bytes) && aligned(a.r, bytes) &&
                     aligned(a.i, bytes) && aligned(a.y, bytes) && aligned(a.h0, 16) && aligned(state_out, 16);
    const int64_t threads = a.batch * (vec ? a.width / 4 : a.width), blocks = (threads + 255) / 256;
    if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
    if (vec)
        hipLaunchKernelGGL((recurrence_step_kernel<T, 4>), dim3(unsigned(blocks)), dim3(256), 0, stream, a, state_out);
    else
        hipLaunchKernelGGL((recurrence_step_kernel<T, 1>), dim3(unsigned(blocks)), dim3(256), 0, stream, a, state_out);
    return hipGetLastError();
}

template <typename T, typename Tg, bool Vec, bool Reset, class F>
hipError_t launch_backward(const RecurrenceGradArgs& a, hipStream_t stream)
{
    if (!grid_fits(workgroups<F>(a.batch, a.tiles, a.width), F::kThreads)) return hipErrorInvalidConfiguration;
    if (hipError_t e = clear_walk(a.words, a.batch, a.tiles, a.width, stream); e != hipSuccess) return e;
    hipLaunchKernelGGL((recurrence_grad_kernel<T, Tg, Vec, Reset, F>), dim3(unsigned(workgroups<F>(a.batch, a.tiles, a.width))),
                       dim3(F::kThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename T, typename Tg, bool Vec>
hipError_t launch_backward_form(const RecurrenceGradArgs& a, hipStream_t stream)
{
    if (narrow(a.batch, a.tiles, a.width)) return launch_backward<T, Tg, Vec, true, Narrow>(a, stream);
    return a.reset != nullptr ? launch_backward<T, Tg, Vec, true, Wide>(a, stream) : launch_backward<T, Tg, Vec, false, Wide>(a, stream);
}

template <typename T, typename Tg>
hipError_t launch_backward_types(const RecurrenceGradArgs& a, hipStream_t stream)
{
    constexpr int in = 4 * int(sizeof(T)), out = 4 * int(sizeof(Tg));
    const bool vec = a.width % 4 == 0 && a.stride % 4 == 0 && a.grad_stride % 4 == 0 && a.stride <= kNearStride &&
                     a.grad_stride <= kNearStride && aligned(a.x, in) && aligned(a.r, in) && aligned(a.i, in) &&
                     aligned(a.dy, out) && aligned(a.dx, out) && aligned(a.dr, out) && aligned(a.di, out);
    return vec ? launch_backward_form<T, Tg, true>(a, stream) : launch_backward_form<T, Tg, false>(a, stream);
}

}  // namespace

// the most that a forward pass of either form has
int64_t recurrence_tiles(int64_t seq_len) { return tiles_of<Narrow, true>(seq_len); }

int64_t recurrence_walk_bytes(int64_t batch, int64_t tiles, int64_t width)
{
    if (tiles <= 1) return 0;
    // counters for the narrow workgroups: enough for either form
    return (ticket_words((width + Narrow::kCh - 1) / Narrow::kCh) + batch * (tiles + tiles / kJoin) * width + 1) / 2 * 16;
}

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
    const int64_t sums = (a.width + kWave - 1) / kWave;
    if (!grid_fits(sums, 1024)) return hipErrorInvalidConfiguration;
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
    hipLaunchKernelGGL(recurrence_dtheta_kernel, dim3(unsigned(sums)), dim3(1024), 0, stream, a.partial, rows, a.theta,
                       a.decay, a.width, a.dtheta);
    return hipGetLastError();
}

}  // namespace mesa
