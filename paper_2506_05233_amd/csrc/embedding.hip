// Token embedding, y_n = scale E[t_n], and the gradient of its table, dE_v = scale sum_{n: t_n = v} dy_n.
//
// The look-up is a copy.  The gradient sorts the tokens (least significant digits first, stable), so
// that the rows of one token follow each other in the order in which they came, and every row of the
// table is then written once, by one group of lanes, which adds its token's rows in that order: no
// atomics on values, the same bits every time.  A token that fills whole pieces of 32 sorted
// positions has their sums from a launch before (and those of 32 such pieces from another), so that
// no group walks more than about a hundred rows, however frequent a token is.
#include <algorithm>

#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"
#include "vocab.hpp"

namespace mesa {
namespace {

constexpr int kThreads = 256;

// V consecutive channels as fp32, V 8 (16-byte pieces or two of them, aligned) or 1.
template <typename T, int V>
__device__ __forceinline__ void load_channels(const T* p, float (&x)[V])
{
    if constexpr (V == 8) {
        float lo[4], hi[4];
        if constexpr (sizeof(T) == 2) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            Lane4<T>::widen(make_uint2(w.x, w.y), lo);
            Lane4<T>::widen(make_uint2(w.z, w.w), hi);
        } else {
            Lane4<T>::widen(reinterpret_cast<const float4*>(p)[0], lo);
            Lane4<T>::widen(reinterpret_cast<const float4*>(p)[1], hi);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = lo[v], x[v + 4] = hi[v];
    } else {
        x[0] = to_f32(*p);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_channels(T* p, const float (&y)[V])
{
    if constexpr (V == 8 && sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
    } else if constexpr (V == 8) {
        reinterpret_cast<float4*>(p)[0] = make_float4(y[0], y[1], y[2], y[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else if constexpr (sizeof(T) == 2) {
        reinterpret_cast<uint16_t*>(p)[0] = uint16_t(pack_bf16(y[0], 0.0f));
    } else {
        *p = y[0];
    }
}

// A row's lanes: a power of two, as many as it has pieces of V channels, at most the workgroup.
struct Lanes {
    int log2;
    __host__ __device__ int rows() const { return kThreads >> log2; }     // rows a workgroup takes at once
    __device__ int row() const { return int(threadIdx.x) >> log2; }
    __device__ int lane() const { return int(threadIdx.x) & ((1 << log2) - 1); }
    __device__ int count() const { return 1 << log2; }
};
Lanes lanes_for(int64_t width, int v)
{
    Lanes l{0};
    while (l.log2 < 8 && (int64_t(v) << l.log2) < width) ++l.log2;
    return l;
}
bool wide_rows(const void* p, int64_t stride, int64_t width, int dtype)
{
    const int64_t row = stride * (dtype == kBf16 ? 2 : 4);
    return width % 8 == 0 && row % 16 == 0 && uintptr_t(p) % 16 == 0;
}

// ------------------------------------------------------------------ look-up
template <typename T, typename O, int V, int Each>
__global__ void __launch_bounds__(kThreads) embedding_kernel(EmbeddingArgs a, Lanes lanes)
{
    const int64_t row0 = (int64_t(blockIdx.x) * lanes.rows() + lanes.row()) * Each;
    int64_t t[Each];
#pragma unroll
    for (int e = 0; e < Each; ++e) t[e] = row0 + e < a.rows ? token_at(a.tokens, row0 + e) : -1;
    for (int64_t c = int64_t(lanes.lane()) * V; c < a.width; c += int64_t(lanes.count()) * V) {
        float x[Each][V];
#pragma unroll
        for (int e = 0; e < Each; ++e) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[e][v] = 0.0f;
            if (t[e] >= 0 && t[e] < a.vocab) load_channels<T, V>(static_cast<const T*>(a.table) + t[e] * a.table_stride + c, x[e]);
        }
#pragma unroll
        for (int e = 0; e < Each; ++e) {
            if (row0 + e >= a.rows) break;
            const bool there = t[e] >= 0 && t[e] < a.vocab;
#pragma unroll
            for (int v = 0; v < V; ++v) x[e][v] = there ? x[e][v] * a.scale : 0.0f;
            store_channels<O, V>(static_cast<O*>(a.out) + (row0 + e) * a.out_stride + c, x[e]);
        }
    }
}

template <typename T, typename O, int V>
hipError_t lookup(const EmbeddingArgs& a, hipStream_t stream)
{
    const Lanes lanes = lanes_for(a.width, V);
    // two rows a group keep two loads under way behind one look at the tokens; few rows are spread instead
    const bool many = a.rows >= 2048 * lanes.rows();
    const int64_t at_once = lanes.rows() * (many ? 2 : 1), blocks = (a.rows + at_once - 1) / at_once;
    if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
    if (many)
        hipLaunchKernelGGL((embedding_kernel<T, O, V, 2>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a, lanes);
    else
        hipLaunchKernelGGL((embedding_kernel<T, O, V, 1>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a, lanes);
    return hipGetLastError();
}

// ------------------------------------------------------------------ the tokens in order
constexpr int kTile = 2048;            // tokens a workgroup sorts
constexpr int kWaves = kThreads / kWave;
constexpr int kRounds = kTile / kThreads;
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kPiece = 32;             // sorted positions of a piece, pieces of a run of pieces

// A token's key: itself, or vocab for one that does not count, which comes last.
__device__ __forceinline__ uint32_t key_of(const Tokens& t, int64_t i, int64_t vocab)
{
    const int64_t v = token_at(t, i);
    return v >= 0 && v < vocab ? uint32_t(v) : uint32_t(vocab);
}

// Ranks of a tile's keys by one digit.  Wave w has keys w 512 + 64 k + lane; count[w][d] ends as the
// number of its keys with digit d and rank[k] as how many of them come before the lane's k-th.
__device__ __forceinline__ void digit_ranks(const uint32_t (&digit)[kRounds], const bool (&active)[kRounds], int bits,
                                            volatile uint32_t (*count)[kBins], uint32_t (&rank)[kRounds])
{
    const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
    for (int i = lane; i < kBins; i += kWave) count[wave][i] = 0;
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        uint64_t same = __ballot(active[k]);
        for (int b = 0; b < bits; ++b) {
            const bool bit = (digit[k] >> b) & 1;
            const uint64_t with = __ballot(bit);
            same &= bit ? with : ~with;
        }
        const uint32_t before = active[k] ? count[wave][digit[k]] : 0;
        const int lower = __popcll(same & ((uint64_t(1) << lane) - 1));
        rank[k] = before + uint32_t(lower);
        if (active[k] && lower == 0) count[wave][digit[k]] = before + uint32_t(__popcll(same));
    }
}

struct SortArgs {
    Tokens tokens;                 // first digit: keys come from here
    int64_t rows, vocab;
    const uint32_t* keys_in;       // null for the first digit
    const uint32_t* places_in;
    uint32_t* keys_out;
    uint32_t* places_out;
    uint32_t* hist;                // [tiles][kBins]
    int64_t tiles;
    int shift, bits;
    uint2* spans;                  // [vocab], cleared on the way when not null
    int digits;                    // of a whole key (a single tile sorts by all of them)
};

// Clears the spans, by workgroups tiles .. gridDim.x - 1.
__device__ __forceinline__ void clear_spans(uint2* spans, int64_t vocab, int64_t first)
{
    for (int64_t v = (int64_t(blockIdx.x) - first) * kThreads + threadIdx.x; v < vocab; v += (int64_t(gridDim.x) - first) * kThreads)
        spans[v] = make_uint2(0u, 0u);
}

// How many keys of a tile have each value of a digit.
__global__ void __launch_bounds__(kThreads) token_histogram_kernel(SortArgs a)
{
    if (int64_t(blockIdx.x) >= a.tiles) {
        clear_spans(a.spans, a.vocab, a.tiles);
        return;
    }
    __shared__ uint32_t bins[kBins];
    for (int i = int(threadIdx.x); i < kBins; i += kThreads) bins[i] = 0;
    __syncthreads();
    const int64_t first = int64_t(blockIdx.x) * kTile;
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int64_t i = first + k * kThreads + threadIdx.x;
        if (i < a.rows) {
            const uint32_t key = a.keys_in == nullptr ? key_of(a.tokens, i, a.vocab) : a.keys_in[i];
            atomicAdd(&bins[(key >> a.shift) & ((1u << a.bits) - 1u)], 1u);
        }
    }
    __syncthreads();
    for (int i = int(threadIdx.x); i < kBins; i += kThreads) a.hist[int64_t(blockIdx.x) * kBins + i] = bins[i];
}

// Exclusive prefix sums of kBins values in LDS, two a thread.
__device__ __forceinline__ void scan_bins(uint32_t* x, uint32_t* wave_total)
{
    const int t = int(threadIdx.x), lane = t % kWave, wave = t / kWave;
    const uint32_t a = x[2 * t], b = x[2 * t + 1];
    uint32_t s = a + b;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t o = uint32_t(__shfl_up(int(s), d));
        if (lane >= d) s += o;
    }
    if (lane == kWave - 1) wave_total[wave] = s;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < wave; ++w) base += wave_total[w];
    x[2 * t] = base + s - a - b;
    x[2 * t + 1] = base + s - b;
    __syncthreads();
}
static_assert(kBins == 2 * kThreads, "two bins a thread");

// A tile's keys to their places by one digit.
__global__ void __launch_bounds__(kThreads) token_scatter_kernel(SortArgs a)
{
    __shared__ uint32_t count[kWaves][kBins];
    __shared__ uint32_t base[kBins], before[kBins], wave_total[kWaves];
    const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
    const int64_t first = int64_t(blockIdx.x) * kTile + wave * (kTile / kWaves) + lane;
    uint32_t key[kRounds], place[kRounds], digit[kRounds], rank[kRounds];
    bool active[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int64_t i = first + k * kWave;
        active[k] = i < a.rows;
        key[k] = !active[k] ? 0u : a.keys_in == nullptr ? key_of(a.tokens, i, a.vocab) : a.keys_in[i];
        place[k] = !active[k] ? 0u : a.keys_in == nullptr ? uint32_t(i) : a.places_in[i];
        digit[k] = (key[k] >> a.shift) & ((1u << a.bits) - 1u);
    }
    // keys of a smaller digit, and of the same digit in earlier tiles
    for (int d = int(threadIdx.x); d < kBins; d += kThreads) {
        uint32_t all = 0, early = 0;
#pragma unroll 4
        for (int64_t t = 0; t < a.tiles; ++t) {
            const uint32_t n = a.hist[t * kBins + d];
            all += n;
            early += t < int64_t(blockIdx.x) ? n : 0u;
        }
        base[d] = all;
        before[d] = early;
    }
    digit_ranks(digit, active, a.bits, count, rank);
    __syncthreads();
    scan_bins(base, wave_total);
    for (int d = int(threadIdx.x); d < kBins; d += kThreads) {
        uint32_t at = base[d] + before[d];
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t n = count[w][d];
            count[w][d] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
        if (active[k]) {
            const uint32_t at = count[wave][digit[k]] + rank[k];
            a.keys_out[at] = key[k];
            a.places_out[at] = place[k];
        }
}

// All digits of at most one tile of tokens, by one workgroup; the others clear the spans.
__global__ void __launch_bounds__(kThreads) token_sort_kernel(SortArgs a)
{
    if (blockIdx.x > 0) {
        clear_spans(a.spans, a.vocab, 1);
        return;
    }
    __shared__ uint32_t count[kWaves][kBins];
    __shared__ uint32_t base[kBins], wave_total[kWaves];
    __shared__ uint32_t keys[kTile], places[kTile];
    const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
    const int first = wave * (kTile / kWaves) + lane;
    uint32_t key[kRounds], place[kRounds], digit[kRounds], rank[kRounds];
    bool active[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int i = first + k * kWave;
        active[k] = i < a.rows;
        key[k] = active[k] ? key_of(a.tokens, i, a.vocab) : 0u;
        place[k] = uint32_t(i);
    }
    for (int s = 0; s < a.digits; ++s) {
#pragma unroll
        for (int k = 0; k < kRounds; ++k) digit[k] = (key[k] >> (s * a.bits)) & ((1u << a.bits) - 1u);
        digit_ranks(digit, active, a.bits, count, rank);
        __syncthreads();
        for (int d = int(threadIdx.x); d < kBins; d += kThreads) {
            uint32_t n = 0;
            for (int w = 0; w < kWaves; ++w) n += count[w][d];
            base[d] = n;
        }
        __syncthreads();
        scan_bins(base, wave_total);
        for (int d = int(threadIdx.x); d < kBins; d += kThreads) {
            uint32_t at = base[d];
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t n = count[w][d];
                count[w][d] = at;
                at += n;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRounds; ++k)
            if (active[k]) {
                const uint32_t at = count[wave][digit[k]] + rank[k];
                keys[at] = key[k];
                places[at] = place[k];
            }
        __syncthreads();
        // the keys that exist fill the front again, so the same lanes are active
#pragma unroll
        for (int k = 0; k < kRounds; ++k)
            if (active[k]) key[k] = keys[first + k * kWave], place[k] = places[first + k * kWave];
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
        if (active[k]) {
            a.keys_out[first + k * kWave] = key[k];
            a.places_out[first + k * kWave] = place[k];
        }
}

// ------------------------------------------------------------------ the sums
struct SumArgs {
    const void* dy;
    int64_t rows, vocab, width, dy_stride, table_stride, ld;     // ld: of the pieces' sums
    float scale;
    bool accumulate;
    const uint32_t* keys;          // sorted, with the rows that they came from
    const uint32_t* places;
    uint2* spans;                  // [vocab]: first and past the last of a token's sorted positions
    float* pieces;                 // [rows / 32][ld]: sums of whole pieces of one token
    float* runs;                   // [rows / 1024][ld]: of 32 pieces
    void* dtable;
};

constexpr int kDepth = 4;          // rows asked for together

// Writes every token's span, and the sum of each piece that lies within one.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) token_piece_kernel(SumArgs a)
{
    const int64_t first = int64_t(blockIdx.x) * kPiece;
    const int t = int(threadIdx.x);
    if (t < kPiece && first + t < a.rows) {
        const int64_t i = first + t;
        const uint32_t k = a.keys[i];
        if (k < uint32_t(a.vocab)) {
            if (i == 0 || a.keys[i - 1] != k) a.spans[k].x = uint32_t(i);
            if (i + 1 == a.rows || a.keys[i + 1] != k) a.spans[k].y = uint32_t(i + 1);
        }
    }
    if (first + kPiece > a.rows) return;
    const uint32_t k = a.keys[first];
    if (k != a.keys[first + kPiece - 1] || k >= uint32_t(a.vocab)) return;
    for (int64_t c = int64_t(t) * V; c < a.width; c += kThreads * V) {
        float sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.0f;
        for (int r = 0; r < kPiece; r += kDepth) {
            float x[kDepth][V];
#pragma unroll
            for (int e = 0; e < kDepth; ++e) load_channels<T, V>(static_cast<const T*>(a.dy) + int64_t(a.places[first + r + e]) * a.dy_stride + c, x[e]);
#pragma unroll
            for (int e = 0; e < kDepth; ++e)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] += x[e][v];
        }
        store_channels<float, V>(a.pieces + int64_t(blockIdx.x) * a.ld + c, sum);
    }
}

// Sums of 32 pieces that lie within one token's span.
template <int V>
__global__ void __launch_bounds__(kThreads) token_run_kernel(SumArgs a)
{
    const int64_t first = int64_t(blockIdx.x) * kPiece * kPiece;
    if (first + kPiece * kPiece > a.rows) return;
    const uint32_t k = a.keys[first];
    if (k != a.keys[first + kPiece * kPiece - 1] || k >= uint32_t(a.vocab)) return;
    const float* src = a.pieces + int64_t(blockIdx.x) * kPiece * a.ld;
    for (int64_t c = int64_t(threadIdx.x) * V; c < a.width; c += kThreads * V) {
        float sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.0f;
        for (int r = 0; r < kPiece; r += kDepth) {
            float x[kDepth][V];
#pragma unroll
            for (int e = 0; e < kDepth; ++e) load_channels<float, V>(src + (r + e) * a.ld + c, x[e]);
#pragma unroll
            for (int e = 0; e < kDepth; ++e)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] += x[e][v];
        }
        store_channels<float, V>(a.runs + int64_t(blockIdx.x) * a.ld + c, sum);
    }
}

// Adds `n` rows at row(i) to the sum, several loads under way at a time, in order.
template <typename T, int V, typename Row>
__device__ __forceinline__ void add_rows(float (&sum)[V], int64_t n, Row row)
{
    int64_t i = 0;
    for (; i + kDepth <= n; i += kDepth) {
        float x[kDepth][V];
#pragma unroll
        for (int e = 0; e < kDepth; ++e) load_channels<T, V>(row(i + e), x[e]);
#pragma unroll
        for (int e = 0; e < kDepth; ++e)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += x[e][v];
    }
    for (; i < n; ++i) {
        float x[V];
        load_channels<T, V>(row(i), x);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += x[v];
    }
}

// Rows of the table's gradient, one a group of lanes.
template <typename T, typename O, int V>
__global__ void __launch_bounds__(kThreads) token_row_kernel(SumArgs a, Lanes lanes)
{
    const int64_t v0 = int64_t(blockIdx.x) * lanes.rows() + lanes.row();
    if (v0 >= a.vocab) return;
    const uint2 span = a.spans[v0];
    if (a.accumulate && span.x == span.y) return;
    // rows up to a piece's start, pieces up to a run's, runs, pieces, rows
    const int64_t lo = span.x, hi = span.y;
    const int64_t p0 = (lo + kPiece - 1) / kPiece, p1 = hi / kPiece;
    const bool pieces = p0 < p1;
    const int64_t head = pieces ? p0 * kPiece : hi;
    const int64_t r0 = (p0 + kPiece - 1) / kPiece, r1 = p1 / kPiece;
    const bool runs = pieces && r0 < r1;
    const int64_t mid = runs ? r0 * kPiece : p1;
    const T* dy = static_cast<const T*>(a.dy);
    for (int64_t c = int64_t(lanes.lane()) * V; c < a.width; c += int64_t(lanes.count()) * V) {
        float sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.0f;
        add_rows<T, V>(sum, head - lo, [&](int64_t i) { return dy + int64_t(a.places[lo + i]) * a.dy_stride + c; });
        if (pieces) {
            add_rows<float, V>(sum, mid - p0, [&](int64_t i) { return a.pieces + (p0 + i) * a.ld + c; });
            if (runs) {
                add_rows<float, V>(sum, r1 - r0, [&](int64_t i) { return a.runs + (r0 + i) * a.ld + c; });
                add_rows<float, V>(sum, p1 - r1 * kPiece, [&](int64_t i) { return a.pieces + (r1 * kPiece + i) * a.ld + c; });
            }
            add_rows<T, V>(sum, hi - p1 * kPiece, [&](int64_t i) { return dy + int64_t(a.places[p1 * kPiece + i]) * a.dy_stride + c; });
        }
        O* dst = static_cast<O*>(a.dtable) + v0 * a.table_stride + c;
        if (a.accumulate) {
            float x[V];
            load_channels<O, V>(dst, x);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] = x[v] + a.scale * sum[v];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] = span.x == span.y ? 0.0f : a.scale * sum[v];
        }
        store_channels<O, V>(dst, sum);
    }
}

int64_t ceil_to(int64_t x, int64_t n) { return (x + n - 1) / n * n; }

struct GradLayout {
    int64_t tiles, ld, hist, keys[2], places[2], spans, pieces, runs, bytes;
    GradLayout(int64_t rows, int64_t vocab, int64_t width)
    {
        tiles = (rows + kTile - 1) / kTile;
        ld = ceil_to(width, 8);
        int64_t at = 0;
        auto take = [&](int64_t n) {
            const int64_t p = at;
            at += ceil_to(n, 256);
            return p;
        };
        hist = take(tiles * kBins * 4);
        for (int k = 0; k < 2; ++k) keys[k] = take(rows * 4), places[k] = take(rows * 4);
        spans = take(vocab * 8);
        pieces = take(rows / kPiece * ld * 4);
        runs = take(rows / (kPiece * kPiece) * ld * 4);
        bytes = at;
    }
};

template <typename T, typename O, int V>
hipError_t sums(const SumArgs& a, hipStream_t stream)
{
    const int64_t pieces = (a.rows + kPiece - 1) / kPiece, runs = a.rows / (kPiece * kPiece);
    const Lanes lanes = lanes_for(a.width, V);
    const int64_t blocks = (a.vocab + lanes.rows() - 1) / lanes.rows();
    if (!grid_fits(blocks, kThreads) || !grid_fits(pieces, kThreads)) return hipErrorInvalidConfiguration;
    if (pieces > 0) hipLaunchKernelGGL((token_piece_kernel<T, V>), dim3(unsigned(pieces)), dim3(kThreads), 0, stream, a);
    if (runs > 0) hipLaunchKernelGGL((token_run_kernel<V>), dim3(unsigned(runs)), dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL((token_row_kernel<T, O, V>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, a, lanes);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t stream)
{
    const bool wide = wide_rows(a.table, a.table_stride, a.width, a.dtype) && wide_rows(a.out, a.out_stride, a.width, a.out_dtype);
    if (a.dtype == kBf16 && a.out_dtype == kBf16) return wide ? lookup<bf16_t, bf16_t, 8>(a, stream) : lookup<bf16_t, bf16_t, 1>(a, stream);
    if (a.dtype == kBf16) return wide ? lookup<bf16_t, float, 8>(a, stream) : lookup<bf16_t, float, 1>(a, stream);
    if (a.out_dtype == kBf16) return wide ? lookup<float, bf16_t, 8>(a, stream) : lookup<float, bf16_t, 1>(a, stream);
    return wide ? lookup<float, float, 8>(a, stream) : lookup<float, float, 1>(a, stream);
}

int64_t embedding_grad_bytes(int64_t rows, int64_t vocab, int64_t width) { return GradLayout(rows, vocab, width).bytes; }

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, hipStream_t stream)
{
    const GradLayout lay(a.rows, a.vocab, a.width);
    char* ws = a.workspace;
    int key_bits = 1;
    while (key_bits < 32 && (int64_t(1) << key_bits) <= a.vocab) ++key_bits;
    const int digits = (key_bits + kDigitBits - 1) / kDigitBits;
    SortArgs s{};
    s.tokens = a.tokens;
    s.rows = a.rows;
    s.vocab = a.vocab;
    s.hist = reinterpret_cast<uint32_t*>(ws + lay.hist);
    s.tiles = lay.tiles;
    s.bits = (key_bits + digits - 1) / digits;
    s.digits = digits;
    s.spans = reinterpret_cast<uint2*>(ws + lay.spans);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + lay.keys[0]), reinterpret_cast<uint32_t*>(ws + lay.keys[1])};
    uint32_t* places[2] = {reinterpret_cast<uint32_t*>(ws + lay.places[0]), reinterpret_cast<uint32_t*>(ws + lay.places[1])};
    const int64_t clear = std::min<int64_t>((a.vocab + 4 * kThreads - 1) / (4 * kThreads), 1024);
    int out = 0;
    if (!grid_fits(lay.tiles + clear, kThreads)) return hipErrorInvalidConfiguration;
    if (lay.tiles <= 1) {
        s.keys_out = keys[0];
        s.places_out = places[0];
        hipLaunchKernelGGL(token_sort_kernel, dim3(unsigned(1 + clear)), dim3(kThreads), 0, stream, s);
    } else {
        for (int d = 0; d < digits; ++d) {
            s.shift = d * s.bits;
            s.keys_in = d == 0 ? nullptr : keys[out];
            s.places_in = d == 0 ? nullptr : places[out];
            out = d == 0 ? 0 : 1 - out;
            s.keys_out = keys[out];
            s.places_out = places[out];
            hipLaunchKernelGGL(token_histogram_kernel, dim3(unsigned(lay.tiles + (d == 0 ? clear : 0))), dim3(kThreads), 0, stream, s);
            hipLaunchKernelGGL(token_scatter_kernel, dim3(unsigned(lay.tiles)), dim3(kThreads), 0, stream, s);
        }
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const SumArgs k{a.dy, a.rows, a.vocab, a.width, a.dy_stride, a.table_stride, lay.ld, a.scale, a.accumulate, keys[out], places[out],
                    s.spans, reinterpret_cast<float*>(ws + lay.pieces), reinterpret_cast<float*>(ws + lay.runs), a.dtable};
    const bool wide = wide_rows(a.dy, a.dy_stride, a.width, a.dtype) && wide_rows(a.dtable, a.table_stride, a.width, a.table_dtype);
    if (a.dtype == kBf16 && a.table_dtype == kBf16) return wide ? sums<bf16_t, bf16_t, 8>(k, stream) : sums<bf16_t, bf16_t, 1>(k, stream);
    if (a.dtype == kBf16) return wide ? sums<bf16_t, float, 8>(k, stream) : sums<bf16_t, float, 1>(k, stream);
    if (a.table_dtype == kBf16) return wide ? sums<float, bf16_t, 8>(k, stream) : sums<float, bf16_t, 1>(k, stream);
    return wide ? sums<float, float, 8>(k, stream) : sums<float, float, 1>(k, stream);
}

}  // namespace mesa
