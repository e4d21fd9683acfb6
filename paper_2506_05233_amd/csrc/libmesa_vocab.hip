// libmesa C ABI: a language model's two ends, the token embedding and the cross entropy over a
// vocabulary, with their gradients.  Argument validation, workspace sizing and kernel launches; the
// contract of every entry point is documented in include/libmesa.h.
#include <math.h>

#include "mesa_abi.hpp"
#include "mesa_kernels.hpp"
#include "vocab.hpp"

namespace {

using mesa::aligned;
using mesa::all_aligned;
using mesa::any_null;
using mesa::bytes_of;
using mesa::clash;
using mesa::dense;
using mesa::float_type;
using mesa::product_ok;
using mesa::status_of;
using mesa::tokens;

// Sorted positions and rows of the table are counted in 32 bits; every workgroup of the sort adds up
// the tiles before its own, so the number of tokens is bounded too.
constexpr int64_t kMostRows = int64_t(1) << 24, kMostVocab = INT32_MAX - 1024, kMostWidth = int64_t(1) << 16;

bool token_type(int bytes) { return bytes == 4 || bytes == 8; }

int vocab_sizes(int64_t rows, int64_t vocab, int64_t width)
{
    if (rows < 0 || vocab < 0 || width < 0 || rows > kMostRows || vocab > kMostVocab || width > kMostWidth) return MESA_ERR_SHAPE;
    return product_ok({rows, width}) && product_ok({vocab, width}) ? MESA_OK : MESA_ERR_SHAPE;
}

bool stride_ok(int64_t rows, int64_t width, int64_t stride) { return rows <= 0 || (stride >= width && product_ok({rows, stride})); }

// A cap that a caller can mean: none, or one whose reciprocal is finite
bool cap_ok(float cap) { return cap == 0.0f || (isnormal(cap) && cap > 0.0f); }

bool loss_countable(int64_t rows, int64_t vocab, int64_t width, int dtype)
{
    return vocab_sizes(rows, vocab, width) == MESA_OK && float_type(dtype) && rows > 0 && vocab > 0 && width > 0;
}

}  // namespace

extern "C" {

int mesa_embedding(const void* table, const void* token, int token_bytes, float scale, int64_t rows, int64_t vocab, int64_t width,
                   int64_t table_stride, int dtype, int out_dtype, int64_t out_stride, void* out, void* stream)
{
    if (int st = vocab_sizes(rows, vocab, width); st != MESA_OK) return st;
    if (!float_type(dtype) || !float_type(out_dtype) || !token_type(token_bytes)) return MESA_ERR_UNSUPPORTED;
    if (!isfinite(scale)) return MESA_ERR_ARG;
    if (rows == 0 || width == 0) return MESA_OK;
    if (!stride_ok(vocab, width, table_stride) || !stride_ok(rows, width, out_stride)) return MESA_ERR_SHAPE;
    if (any_null({token, out}) || (vocab > 0 && table == nullptr)) return MESA_ERR_NULL;
    if (!aligned(table, bytes_of(dtype)) || !aligned(out, bytes_of(out_dtype)) || !aligned(token, token_bytes)) return MESA_ERR_ARG;
    if (clash({tokens(table, vocab, width, table_stride, dtype), dense(token, rows * token_bytes)},
              {tokens(out, rows, width, out_stride, out_dtype)}))
        return MESA_ERR_ARG;
    const mesa::EmbeddingArgs a{table, {token, token_bytes == 8}, scale, rows, vocab, width, table_stride, out_stride, dtype, out_dtype, out};
    return status_of(mesa::launch_embedding(a, static_cast<hipStream_t>(stream)), stream);
}

size_t mesa_embedding_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t width)
{
    if (vocab_sizes(rows, vocab, width) != MESA_OK || vocab == 0 || width == 0) return 0;
    return size_t(mesa::embedding_grad_bytes(rows, width));
}

int mesa_embedding_backward(const void* token, int token_bytes, const void* dy, float scale, int64_t rows, int64_t vocab, int64_t width,
                            int64_t dy_stride, int grad_dtype, int table_dtype, int64_t dtable_stride, int accumulate, void* dtable,
                            void* workspace, size_t workspace_bytes, void* stream)
{
    if (int st = vocab_sizes(rows, vocab, width); st != MESA_OK) return st;
    if (!float_type(grad_dtype) || !float_type(table_dtype) || !token_type(token_bytes)) return MESA_ERR_UNSUPPORTED;
    if (!isfinite(scale)) return MESA_ERR_ARG;
    if (vocab == 0 || width == 0 || (rows == 0 && accumulate != 0)) return MESA_OK;
    if (!stride_ok(rows, width, dy_stride) || !stride_ok(vocab, width, dtable_stride)) return MESA_ERR_SHAPE;
    const size_t need = mesa_embedding_backward_workspace_bytes(rows, vocab, width);
    if (dtable == nullptr || (need > 0 && workspace == nullptr) || (rows > 0 && any_null({token, dy}))) return MESA_ERR_NULL;
    if (workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!aligned(dy, bytes_of(grad_dtype)) || !aligned(dtable, bytes_of(table_dtype)) || !aligned(token, token_bytes) || !aligned(workspace, 16))
        return MESA_ERR_ARG;
    if (clash({dense(token, rows * token_bytes), tokens(dy, rows, width, dy_stride, grad_dtype)},
              {tokens(dtable, vocab, width, dtable_stride, table_dtype), dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    const mesa::EmbeddingGradArgs a{{token, token_bytes == 8}, dy, scale, rows, vocab, width, dy_stride, dtable_stride, grad_dtype, table_dtype,
                                    accumulate != 0, dtable, static_cast<char*>(workspace)};
    return status_of(mesa::launch_embedding_grad(a, static_cast<hipStream_t>(stream)), stream);
}

size_t mesa_cross_entropy_workspace_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype)
{
    if (!loss_countable(rows, vocab, width, dtype)) return 0;
    return size_t(mesa::cross_entropy_bytes(rows, vocab, width, dtype));
}

int mesa_cross_entropy(const void* h, const void* table, const void* target, int token_bytes, float cap, int64_t rows, int64_t vocab,
                       int64_t width, int64_t h_stride, int64_t table_stride, int dtype, float* loss, float* lse, int32_t* best,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    if (int st = vocab_sizes(rows, vocab, width); st != MESA_OK) return st;
    if (!float_type(dtype) || (target != nullptr && !token_type(token_bytes))) return MESA_ERR_UNSUPPORTED;
    if (!cap_ok(cap)) return MESA_ERR_ARG;
    if (rows == 0) return MESA_OK;
    if (vocab == 0 || width == 0 || !stride_ok(rows, width, h_stride) || !stride_ok(vocab, width, table_stride)) return MESA_ERR_SHAPE;
    if (any_null({h, table, lse, workspace}) || (target == nullptr) != (loss == nullptr)) return MESA_ERR_NULL;
    const size_t need = mesa_cross_entropy_workspace_bytes(rows, vocab, width, dtype);
    if (workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!all_aligned({h, table}, bytes_of(dtype)) || !all_aligned({loss, lse, best}, 4) || (target != nullptr && !aligned(target, token_bytes)) ||
        !aligned(workspace, 16))
        return MESA_ERR_ARG;
    if (clash({tokens(h, rows, width, h_stride, dtype), tokens(table, vocab, width, table_stride, dtype),
               dense(target, target == nullptr ? 0 : rows * token_bytes)},
              {dense(loss, rows * 4), dense(lse, rows * 4), dense(best, rows * 4), dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    const mesa::CrossEntropyArgs a{h, table, {target, token_bytes == 8}, cap, rows, vocab, width, h_stride, table_stride, dtype, loss, lse, best,
                                   static_cast<char*>(workspace)};
    return status_of(mesa::launch_cross_entropy(a, static_cast<hipStream_t>(stream)), stream);
}

size_t mesa_cross_entropy_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype)
{
    if (!loss_countable(rows, vocab, width, dtype)) return 0;
    return size_t(mesa::cross_entropy_grad_bytes(rows, vocab, width, dtype));
}

int mesa_cross_entropy_backward(const void* h, const void* table, const void* target, int token_bytes, const float* lse, const float* dloss,
                                float cap, int64_t rows, int64_t vocab, int64_t width, int64_t h_stride, int64_t table_stride, int dtype,
                                int64_t dh_stride, int64_t dtable_stride, void* dh, void* dtable, void* workspace, size_t workspace_bytes,
                                void* stream)
{
    if (int st = vocab_sizes(rows, vocab, width); st != MESA_OK) return st;
    if (!float_type(dtype) || !token_type(token_bytes)) return MESA_ERR_UNSUPPORTED;
    if (!cap_ok(cap)) return MESA_ERR_ARG;
    if (vocab == 0 || width == 0) return rows == 0 ? MESA_OK : MESA_ERR_SHAPE;
    if (!stride_ok(rows, width, h_stride) || !stride_ok(vocab, width, table_stride) || (dh != nullptr && !stride_ok(rows, width, dh_stride)) ||
        (dtable != nullptr && !stride_ok(vocab, width, dtable_stride)))
        return MESA_ERR_SHAPE;
    if (rows > 0 && any_null({h, table, target, lse, dloss, workspace})) return MESA_ERR_NULL;
    if (dh == nullptr && dtable == nullptr) return MESA_OK;
    const size_t need = mesa_cross_entropy_backward_workspace_bytes(rows, vocab, width, dtype);
    if (workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!all_aligned({h, table, dh, dtable}, bytes_of(dtype)) || !all_aligned({lse, dloss}, 4) || !aligned(target, token_bytes) ||
        !aligned(workspace, 16))
        return MESA_ERR_ARG;
    if (clash({tokens(h, rows, width, h_stride, dtype), tokens(table, vocab, width, table_stride, dtype), dense(target, rows * token_bytes),
               dense(lse, rows * 4), dense(dloss, rows * 4)},
              {tokens(dh, rows, width, dh_stride, dtype), tokens(dtable, vocab, width, dtable_stride, dtype), dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    const mesa::CrossEntropyGradArgs a{h, table, {target, token_bytes == 8}, cap, rows, vocab, width, h_stride, table_stride, dh_stride,
                                       dtable_stride, dtype, lse, dloss, dh, dtable, static_cast<char*>(workspace)};
    return status_of(mesa::launch_cross_entropy_grad(a, static_cast<hipStream_t>(stream)), stream);
}

}  // extern "C"
