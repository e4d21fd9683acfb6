// Token embedding, y_n = scale E[t_n], and the gradient of its table, dE_v = scale sum_{n: t_n = v} dy_n.
//
// The look-up is a copy.  The gradient sorts the tokens (least significant digits first, stable), so
// that the rows of one token follow each other in the order in which they came.  Then every piece of 8 or 16
// sorted positions is added up by one group of lanes, in order: tokens that begin and end in the piece
// are written to the table, and the sums of the piece's first and last token, where those go on past it,
// are kept; a last launch adds those up along each such token (of many rows over whole runs of 32 pieces).
// No atomics on values, the same bits every time, and no group walks far, however frequent a token is.
//
// Both are bound by memory: 16384 rows of 2048 bf16 channels are looked up in 18 us (134 MB, 7.2 TB/s, part of it from
// the last cache).  Their gradient for 50257 tokens takes 77 us of kernels, of which 47 are the sort's launches: it keeps 16 of
// the compute units busy, and the others fill the gradient with zeros in the same launches, which is most of
// its traffic (206 of 273 MB, 4.3 TB/s).  The pieces take 20 (67 MB read, 30 written), the join 9, which is latency.
// Few rows are launches and latency: 777 of 321 fp32 channels 14 us of kernels, 19 a call.
//
// The loss's gradient adds up weighted rows of sorted targets by the same kernels, a part of the vocabulary at a time.
#include <algorithm>

#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"
#include "vocab.hpp"
#include "vocab_plan.hpp"

namespace mesa {
namespace {

using namespace vocab;

constexpr int kThreads = 256;

// Sixteen bytes at an address that is aligned to an element only, which vector memory instructions take as well.
typedef uint32_t words_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float floats_any __attribute__((ext_vector_type(4), aligned(4)));

// V consecutive channels, V 8 or (rows of fewer) 1, as they lie in memory; widened when they are used.
template <typename T, int V>
struct Channels;
template <>
struct Channels<bf16_t, 8> {
    words_any w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const words_any*>(p); }
    __device__ __forceinline__ void widen(float (&x)[8]) const
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) x[2 * v] = __uint_as_float(w[v] << 16), x[2 * v + 1] = __uint_as_float(w[v] & 0xFFFF0000u);
    }
};
template <>
struct Channels<float, 8> {
    floats_any lo, hi;
    __device__ __forceinline__ void load(const float* p) { lo = reinterpret_cast<const floats_any*>(p)[0], hi = reinterpret_cast<const floats_any*>(p)[1]; }
    __device__ __forceinline__ void widen(float (&x)[8]) const
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = lo[v], x[v + 4] = hi[v];
    }
};
template <typename T>
struct Channels<T, 1> {
    T t;
    __device__ __forceinline__ void load(const T* p) { t = *p; }
    __device__ __forceinline__ void widen(float (&x)[1]) const { x[0] = to_f32(t); }
};
template <typename T, int V>
__device__ __forceinline__ void load_channels(const T* p, float (&x)[V])
{
    Channels<T, V> c;
    c.load(p);
    c.widen(x);
}
__device__ __forceinline__ void store_one(float* p, float y) { *p = y; }
__device__ __forceinline__ void store_one(bf16_t* p, float y) { p->bits = uint16_t(pack_bf16(y, 0.0f)); }
// Channels from `own` on.
template <typename T, int V>
__device__ __forceinline__ void store_channels(T* p, const float (&y)[V], int own)
{
    if (V == 1 || own > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v >= own) store_one(p + v, y[v]);
    } else if constexpr (V == 8 && sizeof(T) == 2) {
        *reinterpret_cast<words_any*>(p) = words_any{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
    } else if constexpr (V == 8) {
        reinterpret_cast<floats_any*>(p)[0] = floats_any{y[0], y[1], y[2], y[3]};
        reinterpret_cast<floats_any*>(p)[1] = floats_any{y[4], y[5], y[6], y[7]};
    }
}

// Which channels a lane takes: V from `at` on, of which those before `own` are another lane's too (the
// last V of a row whose width is no multiple of V) and not its to store.
struct Place {
    int64_t at;
    int own;
};
template <int V>
__device__ __forceinline__ Place place_of(int64_t c, int64_t width)
{
    const int64_t over = c + V - width;
    return over > 0 ? Place{c - over, int(over)} : Place{c, 0};
}

// A row's lanes: a power of two, as many as it has pieces of V channels, at most the workgroup.
struct Lanes {
    int log2;
    __host__ __device__ int rows() const { return kThreads >> log2; }     // rows a workgroup takes at once
    __device__ int row() const { return int(threadIdx.x) >> log2; }
    __device__ int lane() const { return int(threadIdx.x) & ((1 << log2) - 1); }
    __host__ __device__ int count() const { return 1 << log2; }
};
Lanes lanes_for(int64_t width, int v)
{
    Lanes l{0};
    while (l.log2 < 8 && (int64_t(v) << l.log2) < width) ++l.log2;
    return l;
}
// ------------------------------------------------------------------ look-up
template <typename T, typename O, int V, int Each>
__global__ void __launch_bounds__(kThreads) embedding_kernel(EmbeddingArgs a, Lanes lanes)
{
    const int64_t row0 = (int64_t(blockIdx.x) * lanes.rows() + lanes.row()) * Each;
    int64_t t[Each];
#pragma unroll
    for (int e = 0; e < Each; ++e) t[e] = row0 + e < a.rows ? token_at(a.tokens, row0 + e) : -1;
    for (int64_t first = int64_t(lanes.lane()) * V; first < a.width; first += int64_t(lanes.count()) * V) {
        const Place c = place_of<V>(first, a.width);
        float x[Each][V];
#pragma unroll
        for (int e = 0; e < Each; ++e) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[e][v] = 0.0f;
            if (t[e] >= 0 && t[e] < a.vocab) load_channels<T, V>(static_cast<const T*>(a.table) + t[e] * a.table_stride + c.at, x[e]);
        }
#pragma unroll
        for (int e = 0; e < Each; ++e) {
            if (row0 + e >= a.rows) break;
            const bool there = t[e] >= 0 && t[e] < a.vocab;
#pragma unroll
            for (int v = 0; v < V; ++v) x[e][v] = there ? x[e][v] * a.scale : 0.0f;
            store_channels<O, V>(static_cast<O*>(a.out) + (row0 + e) * a.out_stride + c.at, x[e], c.own);
        }
    }
}

template <typename T, typename O, int V>
hipError_t lookup(const EmbeddingArgs& a, hipStream_t stream)
{
    const Lanes lanes = lanes_for(a.width, V);
    // two rows a group keep two loads under way behind one look at the tokens: 65536 rows of 2048 bf16 channels take
    // 82 us so, 97 one by one, 16384 the same either way; fewer are spread over the card
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
constexpr int kWaves = kThreads / kWave;
constexpr int kRounds = kTile / kThreads;

// A token's key: itself, or vocab for one that does not count, which comes last.
__device__ __forceinline__ uint32_t key_of(const Tokens& t, int64_t i, int64_t vocab)
{
    const int64_t v = token_at(t, i);
    return v >= 0 && v < vocab ? uint32_t(v) : uint32_t(vocab);
}

// Ranks of a workgroup's keys by one digit.  Wave w has keys w 64 Rounds + 64 k + lane; count[w][d] ends
// as the number of its keys with digit d and rank[k] as how many of them come before the lane's k-th
// (bit k of live: it exists).
template <int Rounds>
__device__ __forceinline__ void digit_ranks(const uint32_t (&key)[Rounds], uint32_t live, int shift, uint32_t mask,
                                            volatile uint32_t (*count)[kBins], uint32_t (&rank)[Rounds])
{
    const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
    for (int i = lane; i < kBins; i += kWave) count[wave][i] = 0;
#pragma unroll
    for (int k = 0; k < Rounds; ++k) {
        const bool active = (live >> k) & 1;
        const uint32_t digit = (key[k] >> shift) & mask;
        uint64_t same = __ballot(active);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {      // bits past the digit's are 0 everywhere
            const bool bit = (digit >> b) & 1;
            const uint64_t with = __ballot(bit);
            same &= bit ? with : ~with;
        }
        const uint32_t before = active ? count[wave][digit] : 0;
        const int lower = __popcll(same & ((uint64_t(1) << lane) - 1));
        rank[k] = before + uint32_t(lower);
        if (active && lower == 0) count[wave][digit] = before + uint32_t(__popcll(same));
    }
}

// Inclusive prefix sum over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t o = uint32_t(__shfl_up(int(x), d));
        if (lane >= d) x += o;
    }
    return x;
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
    int digits;                    // of a whole key (a single workgroup sorts by all of them)
};

// `bytes` from p on by `threads` threads, of which this is the i-th.
__device__ __forceinline__ void fill_bytes(char* p, int64_t bytes, int element, int64_t i, int64_t threads)
{
    const int64_t whole = bytes / 16;
    for (int64_t k = i; k < whole; k += threads) *reinterpret_cast<words_any*>(p + 16 * k) = words_any{0u, 0u, 0u, 0u};
    const int64_t at = 16 * whole + i * element;
    if (at < bytes) {
        if (element == 4)
            *reinterpret_cast<uint32_t*>(p + at) = 0;
        else
            *reinterpret_cast<uint16_t*>(p + at) = 0;
    }
}
// Rows of zeros, in a launch's workgroups from `first` on.
__device__ __forceinline__ void fill_rows(const Zeros& f, int64_t first)
{
    char* to = static_cast<char*>(f.p);
    const int64_t block = int64_t(blockIdx.x) - first, blocks = int64_t(gridDim.x) - first;
    if (f.bytes == f.pitch) {        // dense rows are one run
        fill_bytes(to, f.rows * f.bytes, f.element, block * blockDim.x + threadIdx.x, blocks * blockDim.x);
        return;
    }
    for (int64_t row = block; row < f.rows; row += blocks) fill_bytes(to + row * f.pitch, f.bytes, f.element, threadIdx.x, blockDim.x);
}

// How many keys of a tile have each value of a digit.
__global__ void __launch_bounds__(kThreads) token_histogram_kernel(SortArgs a, Zeros fill)
{
    if (int64_t(blockIdx.x) >= a.tiles) {
        fill_rows(fill, a.tiles);
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
    const uint32_t s = wave_scan(a + b, lane);
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
__global__ void __launch_bounds__(kThreads) token_scatter_kernel(SortArgs a, Zeros fill)
{
    if (int64_t(blockIdx.x) >= a.tiles) {
        fill_rows(fill, a.tiles);
        return;
    }
    __shared__ uint32_t count[kWaves][kBins];
    __shared__ uint32_t base[kBins], before[kBins], wave_total[kWaves];
    const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
    const int64_t first = int64_t(blockIdx.x) * kTile + wave * (kTile / kWaves) + lane;
    const uint32_t mask = (1u << a.bits) - 1u;
    uint32_t key[kRounds], place[kRounds], rank[kRounds], live = 0;
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int64_t i = first + k * kWave;
        const bool active = i < a.rows;
        live |= uint32_t(active) << k;
        key[k] = !active ? 0u : a.keys_in == nullptr ? key_of(a.tokens, i, a.vocab) : a.keys_in[i];
        place[k] = !active ? 0u : a.keys_in == nullptr ? uint32_t(i) : a.places_in[i];
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
    digit_ranks<kRounds>(key, live, a.shift, mask, count, rank);
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
        if ((live >> k) & 1) {
            const uint32_t at = count[wave][(key[k] >> a.shift) & mask] + rank[k];
            a.keys_out[at] = key[k];
            a.places_out[at] = place[k];
        }
}

// All digits of up to 2048 tokens by one workgroup of 16 waves, Rounds keys a thread, which pass through
// LDS once a digit: 5.7 us for 777 tokens of 5003, where the launches by digit take 4 times 5 or more.
// (16 keys a thread, 16384 tokens, would take 54 against 30.)
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave, kSortRounds = 2;

template <int Rounds>
__global__ void __launch_bounds__(kSortThreads) token_sort_kernel(SortArgs a, Zeros fill)
{
    if (blockIdx.x > 0) {
        fill_rows(fill, 1);
        return;
    }
    __shared__ uint32_t count[kSortWaves][kBins];
    __shared__ uint32_t total[kBins / kWave];
    __shared__ uint32_t pass[Rounds * kSortThreads];
    const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
    const int first = wave * (Rounds * kWave) + lane;
    const uint32_t mask = (1u << a.bits) - 1u;
    uint32_t key[Rounds], place[Rounds], rank[Rounds], live = 0;
#pragma unroll
    for (int k = 0; k < Rounds; ++k) {
        const int i = first + k * kWave;
        live |= uint32_t(i < a.rows) << k;
        key[k] = i < a.rows ? key_of(a.tokens, i, a.vocab) : 0u;
        place[k] = uint32_t(i);
    }
    for (int s = 0; s < a.digits; ++s) {
        const int shift = s * a.bits;
        digit_ranks<Rounds>(key, live, shift, mask, count, rank);
        __syncthreads();
        // bin d: its keys in each wave come after those of smaller digits and of earlier waves
        const int d = int(threadIdx.x);
        uint32_t mine[kSortWaves], sum = 0;
        if (d < kBins) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) mine[w] = count[w][d];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t n = mine[w];
                mine[w] = sum;
                sum += n;
            }
        }
        const uint32_t upto = wave_scan(sum, lane);
        if (d < kBins && lane == kWave - 1) total[wave] = upto;
        __syncthreads();
        if (d < kBins) {
            uint32_t at = upto - sum;
            for (int w = 0; w < wave; ++w) at += total[w];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) count[w][d] = at + mine[w];
        }
        __syncthreads();
        // the keys that exist fill the front again, so the same lanes stay active
#pragma unroll
        for (int k = 0; k < Rounds; ++k) rank[k] += count[wave][(key[k] >> shift) & mask];
#pragma unroll
        for (int k = 0; k < Rounds; ++k)
            if ((live >> k) & 1) pass[rank[k]] = key[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < Rounds; ++k)
            if ((live >> k) & 1) key[k] = pass[first + k * kWave];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < Rounds; ++k)
            if ((live >> k) & 1) pass[rank[k]] = place[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < Rounds; ++k)
            if ((live >> k) & 1) place[k] = pass[first + k * kWave];
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < Rounds; ++k)
        if ((live >> k) & 1) {
            a.keys_out[first + k * kWave] = key[k];
            a.places_out[first + k * kWave] = place[k];
        }
}

// ------------------------------------------------------------------ the sums
struct SumArgs {
    const void* dy;
    int64_t rows, width, dy_stride, table_stride, ld;     // ld: of the pieces' sums
    uint32_t first, count;         // tokens whose sums are wanted (first 0 but for weighted rows)
    float scale;
    bool accumulate;
    const float* weight;           // of weighted rows: their weights,
    int32_t* at;                   // and where a token's sum is, plus one, in dtable, here a list of sums
    const uint32_t* keys;          // sorted, with the rows that they came from
    const uint32_t* places;
    float* entered;                // [pieces][ld]: of each piece its part of a token that begins before it
    float* left;                   // [pieces][ld]: and of one that begins in it and goes on after it
    float* runs;                   // [pieces / kRun][ld]: sums of kRun of `entered`, all of one token
    void* dtable;
};

constexpr int kDepth = 16;         // sums asked for together
constexpr uint32_t kNoKey = 0xFFFFFFFFu;

__device__ __forceinline__ bool wanted(const SumArgs& a, uint32_t key) { return key - a.first < a.count; }

// A token's sum to its row: the token's own, or of weighted rows that of its first sorted position.
template <typename O, int V>
__device__ __forceinline__ void write_row(const SumArgs& a, int64_t row, const Place& c, float (&sum)[V])
{
    O* dst = static_cast<O*>(a.dtable) + row * a.table_stride + c.at;
    float x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = 0.0f;
    if (a.accumulate) load_channels<O, V>(dst, x);
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] += a.scale * sum[v];
    store_channels<O, V>(dst, x, c.own);
}

// Each piece of sorted positions: its tokens' sums.
template <typename T, typename O, int V, int kPiece, bool Weighted>
__device__ __forceinline__ void add_piece(const SumArgs& a, const Lanes& lanes)
{
    const int64_t piece = int64_t(blockIdx.x) * lanes.rows() + lanes.row(), first = piece * kPiece;
    if (first >= a.rows) return;
    const int64_t from = (int64_t(blockIdx.y) * lanes.count() + lanes.lane()) * V;
    if (from >= a.width) return;
    const Place c = place_of<V>(from, a.width);
    const int n = int(min(int64_t(kPiece), a.rows - first));
    if (Weighted && a.keys[first + n - 1] < a.first) return;
    uint32_t key[kPiece], place[kPiece];
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        const int64_t i = min(first + e, a.rows - 1);
        key[e] = e < n ? a.keys[i] : kNoKey;
        place[e] = a.places[i];
    }
    const uint32_t before = first > 0 ? a.keys[first - 1] : kNoKey, after = first + n < a.rows ? a.keys[first + n] : kNoKey;
    if (key[0] >= a.first + a.count) return;      // only rows that do not count from here on
    // every row of the piece is asked for before the first is added (in the place of a row that does not count
    // one that does, for a sum that is not kept: those come last, and of weighted rows first, too)
    uint32_t some = place[0];
    if constexpr (Weighted) {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) some = wanted(a, key[e]) ? place[e] : some;
    }
    Channels<T, V> x[kPiece];
    float weight[kPiece];
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        const uint32_t row = wanted(a, key[e]) ? place[e] : some;
        x[e].load(static_cast<const T*>(a.dy) + int64_t(row) * a.dy_stride + c.at);
        if constexpr (Weighted) weight[e] = a.weight[row];
    }
    uint32_t token = key[0];
    int64_t begin = first;
    bool begins = token != before;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    auto flush = [&](bool ends) {
        if (Weighted && begins && from == 0) a.at[token] = int32_t(begin) + 1;
        if (begins && ends)
            write_row<O, V>(a, Weighted ? begin : int64_t(token), c, sum);
        else
            store_channels<float, V>((begins ? a.left : a.entered) + piece * a.ld + c.at, sum, c.own);
    };
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        if (key[e] != token) {
            if (wanted(a, token)) flush(true);
            token = key[e];
            begin = first + e;
            begins = true;
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] = 0.0f;
        }
        float y[V];
        x[e].widen(y);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = Weighted ? fmaf(weight[e], y[v], sum[v]) : sum[v] + y[v];
    }
    if (wanted(a, token)) flush(token != after);
}
template <typename T, typename O, int V, int kPiece>
__global__ void __launch_bounds__(kThreads) token_piece_kernel(SumArgs a, Lanes lanes)
{
    add_piece<T, O, V, kPiece, false>(a, lanes);
}
template <int V, int kPiece>
__global__ void __launch_bounds__(kThreads) weighted_piece_kernel(SumArgs a, Lanes lanes)
{
    add_piece<bf16_t, float, V, kPiece, true>(a, lanes);
}

// Sums of the runs of pieces that lie within one token's rows, the first of which come before them.
template <int V, int kPiece>
__global__ void __launch_bounds__(kThreads) token_run_kernel(SumArgs a)
{
    const int64_t first = int64_t(blockIdx.x) * kPiece * kRun;
    if (first == 0 || first + kPiece * kRun > a.rows) return;
    const uint32_t k = a.keys[first - 1];
    if (k != a.keys[first + kPiece * kRun - 1] || !wanted(a, k)) return;
    const float* src = a.entered + int64_t(blockIdx.x) * kRun * a.ld;
    for (int64_t from = int64_t(threadIdx.x) * V; from < a.width; from += kThreads * V) {
        const Place c = place_of<V>(from, a.width);
        float sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.0f;
        for (int r = 0; r < kRun; r += kDepth) {
            float x[kDepth][V];
#pragma unroll
            for (int e = 0; e < kDepth; ++e) load_channels<float, V>(src + (r + e) * a.ld + c.at, x[e]);
#pragma unroll
            for (int e = 0; e < kDepth; ++e)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] += x[e][v];
        }
        store_channels<float, V>(a.runs + int64_t(blockIdx.x) * a.ld + c.at, sum, c.own);
    }
}

// Adds rows lo .. hi - 1 of fp32 sums, several loads under way at a time, in order.
template <int V>
__device__ __forceinline__ void add_rows(float (&sum)[V], const float* rows, int64_t ld, int64_t lo, int64_t hi)
{
    for (int64_t i = lo; i < hi; i += kDepth) {
        float x[kDepth][V];
#pragma unroll
        for (int e = 0; e < kDepth; ++e) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[e][v] = 0.0f;
            if (i + e < hi) load_channels<float, V>(rows + (i + e) * ld, x[e]);
        }
#pragma unroll
        for (int e = 0; e < kDepth; ++e)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += x[e][v];
    }
}

// Past the last of the sorted positions from `at` on that have the same key.
template <int kPiece>
__device__ __forceinline__ int64_t end_of(const uint32_t* keys, int64_t at, int64_t rows)
{
    const uint32_t key = keys[at];
    int64_t lo = at, hi = rows;      // keys[lo] is the token's, keys[hi] is not (or there is none)
    for (int64_t step = kPiece; lo + step < rows; step *= 4) {
        if (keys[lo + step] != key) {
            hi = lo + step;
            break;
        }
        lo += step;
    }
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (keys[mid] == key)
            lo = mid;
        else
            hi = mid;
    }
    return hi;
}

// Past the last of the pieces that a token enters which goes on after position `last`, the end of a piece.
// A piece is entered where it begins with the token; a whole wave of one group looks at 64 of them at once.
template <int kPiece>
__device__ __forceinline__ int64_t pieces_entered(const SumArgs& a, uint32_t token, int64_t last, const Lanes& lanes)
{
    if (lanes.log2 < 6) return (end_of<kPiece>(a.keys, last, a.rows) + kPiece - 1) / kPiece;
    const int64_t pieces = (a.rows + kPiece - 1) / kPiece;
    for (int64_t p = last / kPiece + 1;; p += kWave) {
        const int64_t mine = p + int(threadIdx.x) % kWave;
        const uint64_t off = __ballot(mine >= pieces || a.keys[min(mine, pieces - 1) * kPiece] != token);
        if (off != 0) return p + __builtin_ctzll(off);
    }
}

// The tokens that begin in a piece and go on after it, one a group of lanes.
template <typename O, int V, int kPiece, bool Weighted>
__device__ __forceinline__ void join_pieces(const SumArgs& a, const Lanes& lanes)
{
    const int64_t piece = int64_t(blockIdx.x) * lanes.rows() + lanes.row(), first = piece * kPiece, last = first + kPiece - 1;
    if (last + 1 >= a.rows) return;
    const uint32_t token = a.keys[last];
    if (!wanted(a, token) || a.keys[last + 1] != token) return;
    if (first > 0 && a.keys[first - 1] == token) return;      // it begins before
    const int64_t p0 = piece + 1, p1 = pieces_entered<kPiece>(a, token, last, lanes);
    const int64_t from = (int64_t(blockIdx.y) * lanes.count() + lanes.lane()) * V;
    if (from >= a.width) return;
    const Place c = place_of<V>(from, a.width);
    float sum[V];
    load_channels<float, V>(a.left + piece * a.ld + c.at, sum);
    const int64_t r0 = (p0 + kRun - 1) / kRun, r1 = p1 / kRun;
    // a run is whole, the last one only if the token goes on to its end
    const bool runs = a.rows > kRunRows && r0 < r1;
    const int64_t r2 = runs && (r1 * kRun * kPiece > a.rows || a.keys[r1 * kRun * kPiece - 1] != token) ? r1 - 1 : r1;
    if (runs && r0 < r2) {
        add_rows<V>(sum, a.entered + c.at, a.ld, p0, r0 * kRun);
        add_rows<V>(sum, a.runs + c.at, a.ld, r0, r2);
        add_rows<V>(sum, a.entered + c.at, a.ld, r2 * kRun, p1);
    } else {
        add_rows<V>(sum, a.entered + c.at, a.ld, p0, p1);
    }
    write_row<O, V>(a, Weighted ? int64_t(a.at[token]) - 1 : int64_t(token), c, sum);
}
template <typename O, int V, int kPiece>
__global__ void __launch_bounds__(kThreads) token_join_kernel(SumArgs a, Lanes lanes)
{
    join_pieces<O, V, kPiece, false>(a, lanes);
}
template <int V, int kPiece>
__global__ void __launch_bounds__(kThreads) weighted_join_kernel(SumArgs a, Lanes lanes)
{
    join_pieces<float, V, kPiece, true>(a, lanes);
}

template <typename T, typename O, int V, int kPiece, bool Weighted>
hipError_t sums_of(const SumArgs& a, hipStream_t stream)
{
    const int64_t pieces = (a.rows + kPiece - 1) / kPiece, runs = a.rows <= kRunRows ? 0 : pieces / kRun;
    const Lanes lanes = lanes_for(a.width, V);
    const int64_t blocks = (pieces + lanes.rows() - 1) / lanes.rows();
    // a workgroup's lanes side by side, and along the second dimension of the grid
    const unsigned slabs = unsigned((a.width + lanes.count() * V - 1) / (lanes.count() * V));
    if (!grid_fits(blocks, kThreads) || !grid_fits(runs, kThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid(unsigned(blocks), slabs);
    if constexpr (Weighted)
        hipLaunchKernelGGL((weighted_piece_kernel<V, kPiece>), grid, dim3(kThreads), 0, stream, a, lanes);
    else
        hipLaunchKernelGGL((token_piece_kernel<T, O, V, kPiece>), grid, dim3(kThreads), 0, stream, a, lanes);
    if constexpr (kPiece == kManyPiece)
        if (runs > 0) hipLaunchKernelGGL((token_run_kernel<V, kPiece>), dim3(unsigned(runs)), dim3(kThreads), 0, stream, a);
    if (pieces > 1) {
        if constexpr (Weighted)
            hipLaunchKernelGGL((weighted_join_kernel<V, kPiece>), grid, dim3(kThreads), 0, stream, a, lanes);
        else
            hipLaunchKernelGGL((token_join_kernel<O, V, kPiece>), grid, dim3(kThreads), 0, stream, a, lanes);
    }
    return hipGetLastError();
}

template <typename T, typename O, int V, bool Weighted = false>
hipError_t sums(const SumArgs& a, hipStream_t stream)
{
    return piece_of(a.rows) == kFewPiece ? sums_of<T, O, V, kFewPiece, Weighted>(a, stream) : sums_of<T, O, V, kManyPiece, Weighted>(a, stream);
}

// Few sums have a lane each, so that there are waves enough for the loads' latency: 16384 rows of 64 bf16 channels
// take 30.8 us so and 35.8 with eight channels a lane, 1024 of 2048 14.2 and 16.0, 4096 of 1000 29.6 and 29.3,
// 16384 of 320 34.7 and 31.6.
bool eight_channels(int64_t rows, int64_t width) { return width >= 8 && rows * width >= (int64_t(1) << 22); }

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t stream)
{
    const bool wide = a.width >= 8;
    if (a.dtype == kBf16 && a.out_dtype == kBf16) return wide ? lookup<bf16_t, bf16_t, 8>(a, stream) : lookup<bf16_t, bf16_t, 1>(a, stream);
    if (a.dtype == kBf16) return wide ? lookup<bf16_t, float, 8>(a, stream) : lookup<bf16_t, float, 1>(a, stream);
    if (a.out_dtype == kBf16) return wide ? lookup<float, bf16_t, 8>(a, stream) : lookup<float, bf16_t, 1>(a, stream);
    return wide ? lookup<float, float, 8>(a, stream) : lookup<float, float, 1>(a, stream);
}

int64_t embedding_grad_bytes(int64_t rows, int64_t width) { return TokenSumLayout(rows, width).bytes; }

hipError_t launch_token_sort(const Tokens& tokens, int64_t rows, int64_t vocab, int64_t width, const Zeros& zeros, char* ws, Sorted* sorted,
                             hipStream_t stream)
{
    const TokenSumLayout lay(rows, width);
    int key_bits = 1;
    while (key_bits < 32 && (int64_t(1) << key_bits) <= vocab) ++key_bits;
    const int digits = (key_bits + kDigitBits - 1) / kDigitBits;
    SortArgs s{};
    s.tokens = tokens;
    s.rows = rows;
    s.vocab = vocab;
    s.hist = reinterpret_cast<uint32_t*>(ws + lay.hist);
    s.tiles = lay.tiles;
    s.bits = (key_bits + digits - 1) / digits;
    s.digits = digits;
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + lay.keys[0]), reinterpret_cast<uint32_t*>(ws + lay.keys[1])};
    uint32_t* places[2] = {reinterpret_cast<uint32_t*>(ws + lay.places[0]), reinterpret_cast<uint32_t*>(ws + lay.places[1])};
    // the rows of zeros are written in equal shares of the sort's launches
    const int shares = rows <= kSortRounds * kSortThreads ? 1 : 2 * digits;
    int share = 0;
    int64_t blocks = 0;
    auto next_fill = [&](int threads) {
        const int64_t r0 = zeros.rows * share / shares, r1 = zeros.rows * (share + 1) / shares;
        ++share;
        const Zeros f{static_cast<char*>(zeros.p) + r0 * zeros.pitch, r1 - r0, zeros.bytes, zeros.pitch, zeros.element};
        // about 64 KB a workgroup, at most eight a compute unit
        blocks = std::min<int64_t>(ceil_to(f.rows * f.bytes, 65536) / 65536, 2048 * kThreads / threads);
        return f;
    };
    int out = 0;
    if (!grid_fits(lay.tiles + 2048, kThreads)) return hipErrorInvalidConfiguration;
    if (shares == 1) {
        s.keys_out = keys[0];
        s.places_out = places[0];
        const Zeros fill = next_fill(kSortThreads);
        const dim3 grid(unsigned(1 + blocks)), block(kSortThreads);
        if (rows <= kSortThreads)
            hipLaunchKernelGGL(token_sort_kernel<1>, grid, block, 0, stream, s, fill);
        else
            hipLaunchKernelGGL(token_sort_kernel<kSortRounds>, grid, block, 0, stream, s, fill);
    } else {
        for (int d = 0; d < digits; ++d) {
            s.shift = d * s.bits;
            s.keys_in = d == 0 ? nullptr : keys[out];
            s.places_in = d == 0 ? nullptr : places[out];
            out = d == 0 ? 0 : 1 - out;
            s.keys_out = keys[out];
            s.places_out = places[out];
            const Zeros one = next_fill(kThreads);
            hipLaunchKernelGGL(token_histogram_kernel, dim3(unsigned(lay.tiles + blocks)), dim3(kThreads), 0, stream, s, one);
            const Zeros two = next_fill(kThreads);
            hipLaunchKernelGGL(token_scatter_kernel, dim3(unsigned(lay.tiles + blocks)), dim3(kThreads), 0, stream, s, two);
        }
    }
    *sorted = Sorted{keys[out], places[out]};
    return hipGetLastError();
}

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, hipStream_t stream)
{
    const TokenSumLayout lay(a.rows, a.width);
    char* ws = a.workspace;
    const int64_t es = a.table_dtype == kBf16 ? 2 : 4;
    Sorted sorted;
    const Zeros zeros{a.dtable, a.accumulate ? 0 : a.vocab, a.width * es, a.table_stride * es, int(es)};
    if (hipError_t e = launch_token_sort(a.tokens, a.rows, a.vocab, a.width, zeros, ws, &sorted, stream); e != hipSuccess || a.rows == 0) return e;
    const SumArgs k{a.dy, a.rows, a.width, a.dy_stride, a.table_stride, lay.ld, 0, uint32_t(a.vocab), a.scale, a.accumulate, nullptr, nullptr,
                    sorted.keys, sorted.places, reinterpret_cast<float*>(ws + lay.entered), reinterpret_cast<float*>(ws + lay.left),
                    reinterpret_cast<float*>(ws + lay.runs), a.dtable};
    const bool wide = eight_channels(a.rows, a.width);
    if (a.dtype == kBf16 && a.table_dtype == kBf16) return wide ? sums<bf16_t, bf16_t, 8>(k, stream) : sums<bf16_t, bf16_t, 1>(k, stream);
    if (a.dtype == kBf16) return wide ? sums<bf16_t, float, 8>(k, stream) : sums<bf16_t, float, 1>(k, stream);
    if (a.table_dtype == kBf16) return wide ? sums<float, bf16_t, 8>(k, stream) : sums<float, bf16_t, 1>(k, stream);
    return wide ? sums<float, float, 8>(k, stream) : sums<float, float, 1>(k, stream);
}

hipError_t launch_token_sums(const TokenSumArgs& a, hipStream_t stream)
{
    const TokenSumLayout lay(a.rows, a.width);
    char* ws = a.workspace;
    const SumArgs k{a.x, a.rows, a.width, a.stride, a.ld, lay.ld, a.first, a.count, 1.0f, false, a.weight, a.at,
                    a.sorted.keys, a.sorted.places, reinterpret_cast<float*>(ws + lay.entered), reinterpret_cast<float*>(ws + lay.left),
                    reinterpret_cast<float*>(ws + lay.runs), a.sums};
    return eight_channels(a.rows, a.width) ? sums<bf16_t, float, 8, true>(k, stream) : sums<bf16_t, float, 1, true>(k, stream);
}

}  // namespace mesa
