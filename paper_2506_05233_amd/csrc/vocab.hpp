// Host-side launchers of a language model's two ends: the token embedding and the cross entropy
// over a vocabulary, each with its gradient.  Sizes are checked by the C ABI (libmesa_vocab.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mesa {

// Token numbers, 4 or 8 bytes each.  One outside [0, vocab) stands for no token.
struct Tokens {
    const void* p;
    bool wide;
};

struct EmbeddingArgs {
    const void* table;        // [vocab] rows, table_stride elements apart
    Tokens tokens;            // [rows]
    float scale;
    int64_t rows, vocab, width, table_stride, out_stride;
    int dtype, out_dtype;     // kF32 or kBf16
    void* out;
};
hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t stream);

struct EmbeddingGradArgs {
    Tokens tokens;
    const void* dy;           // [rows] rows, dy_stride apart
    float scale;
    int64_t rows, vocab, width, dy_stride, table_stride;
    int dtype, table_dtype;   // of dy; of the table's gradient
    bool accumulate;
    void* dtable;
    char* workspace;          // embedding_grad_bytes, 16-byte aligned
};
int64_t embedding_grad_bytes(int64_t rows, int64_t width);
hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, hipStream_t stream);

// Its two stages apart, for sums that are wanted a part of the vocabulary at a time and of weighted rows.
struct Sorted {
    const uint32_t* keys;     // [rows] tokens in order (vocab for one that does not count)
    const uint32_t* places;   // and the rows that they came from
};
// Zeros for `rows` rows of `bytes`, `pitch` apart, of elements of 4 or 2 bytes.
struct Zeros {
    void* p;
    int64_t rows, bytes, pitch;
    int element;
};
// Sorts the tokens and writes the zeros.  The workspace, of embedding_grad_bytes(rows, width), holds what is sorted.
hipError_t launch_token_sort(const Tokens& tokens, int64_t rows, int64_t vocab, int64_t width, const Zeros& zeros, char* workspace, Sorted* sorted,
                             hipStream_t stream);
struct TokenSumArgs {
    Sorted sorted;
    int64_t rows, width;
    uint32_t first, count;    // the tokens [first, first + count)
    const uint16_t* x;        // [rows] bf16 rows, stride apart
    int64_t stride;
    const float* weight;      // [rows]
    // of each of those tokens that occurs sum weight_n x_n over its rows in their order, fp32, at row at[token] - 1 of `sums`
    // (where the first of its rows was sorted to), ld a multiple of 4; at[] of the others is left as it is
    float* sums;
    int64_t ld;
    int32_t* at;
    char* workspace;          // the sort's
};
hipError_t launch_token_sums(const TokenSumArgs& a, hipStream_t stream);

struct CrossEntropyArgs {
    const void* h;            // [rows] rows of width, h_stride apart
    const void* table;        // [vocab] rows of width, table_stride apart
    Tokens targets;           // p may be null: then neither are loss and at
    float cap;                // 0: none
    int64_t rows, vocab, width, h_stride, table_stride;
    int dtype;                // of h and table
    float* loss;              // [rows]
    float* lse;               // [rows]
    int32_t* best;            // [rows] or null
    char* workspace;          // cross_entropy_bytes, 16-byte aligned
};
int64_t cross_entropy_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype);
hipError_t launch_cross_entropy(const CrossEntropyArgs& a, hipStream_t stream);

struct CrossEntropyGradArgs {
    const void* h;
    const void* table;
    Tokens targets;
    float cap;
    int64_t rows, vocab, width, h_stride, table_stride, dh_stride, dtable_stride;
    int dtype;                // of h, table, dh and dtable
    const float* lse;         // [rows]
    const float* dloss;       // [rows]
    void* dh;                 // or null
    void* dtable;             // or null
    char* workspace;          // cross_entropy_grad_bytes, 16-byte aligned
};
int64_t cross_entropy_grad_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype);
hipError_t launch_cross_entropy_grad(const CrossEntropyGradArgs& a, hipStream_t stream);

__device__ __forceinline__ int64_t token_at(const Tokens& t, int64_t i)
{
    return t.wide ? static_cast<const int64_t*>(t.p)[i] : int64_t(static_cast<const int32_t*>(t.p)[i]);
}

}  // namespace mesa
