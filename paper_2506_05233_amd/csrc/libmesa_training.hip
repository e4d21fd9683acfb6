// libmesa C ABI: the gated recurrence, the 8-bit checkpoints and the gradients of the
// layer's two ends.  Argument validation, workspace sizing and kernel launches; the contract
// of every entry point is documented in include/libmesa.h.
#include <math.h>

#include <initializer_list>

#include "mesa_abi.hpp"
#include "mesa_kernels.hpp"

namespace {

using mesa::finish;
using mesa::launch_status;
using mesa::overlaps;
using mesa::Range;
using mesa::range_of;

static_assert(MESA_RECURRENCE_BLOCK == mesa::kRecurrenceBlock, "the header's block of tokens");
static_assert(MESA_DTYPE_F32 == mesa::kF32 && MESA_DTYPE_BF16 == mesa::kBf16 && MESA_DTYPE_Q8 == mesa::kQ8, "the header's types");

constexpr int64_t kMostElements = int64_t(1) << 40;   // of one array: byte offsets stay far inside 64 bits

// Whether the product of non-negative factors stays within kMostElements.
bool product_ok(std::initializer_list<int64_t> factors)
{
    int64_t p = 1;
    for (int64_t f : factors) {
        if (f == 0) return true;
        if (f > kMostElements / p) return false;
        p *= f;
    }
    return true;
}

bool float_type(int dtype) { return dtype == MESA_DTYPE_F32 || dtype == MESA_DTYPE_BF16; }
int64_t bytes_of(int dtype) { return dtype == MESA_DTYPE_BF16 ? 2 : dtype == MESA_DTYPE_Q8 ? 1 : 4; }
bool aligned(const void* p, int64_t bytes) { return uintptr_t(p) % uintptr_t(bytes) == 0; }
bool all_aligned(std::initializer_list<const void*> ptrs, int64_t bytes)
{
    for (const void* p : ptrs)
        if (!aligned(p, bytes)) return false;
    return true;
}
bool any_null(std::initializer_list<const void*> ptrs)
{
    for (const void* p : ptrs)
        if (p == nullptr) return true;
    return false;
}

size_t checkpoint_bytes(int64_t rows, int64_t width)
{
    const int64_t groups = (width + MESA_CHECKPOINT_GROUP - 1) / MESA_CHECKPOINT_GROUP;
    return size_t((mesa::checkpoint_exponents_at(rows, width) + rows * groups + 15) / 16 * 16);
}

// A device array as `rows` pieces of `bytes`, `pitch` apart (absent: a null pointer or no bytes).
struct Rows {
    const void* p;
    int64_t rows, bytes, pitch;
    bool empty() const { return p == nullptr || rows <= 0 || bytes <= 0; }
    Range span() const { return range_of(p, (rows - 1) * pitch + bytes); }
};
Rows dense(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }
Rows tokens(const void* p, int64_t n, int64_t width, int64_t stride, int dtype)
{
    return {p, n, width * bytes_of(dtype), stride * bytes_of(dtype)};
}

// Whether two arrays share a byte.  Slices of one array (the same pitch) interleave freely.
bool touch(const Rows& a, const Rows& b)
{
    if (a.empty() || b.empty() || !overlaps(a.span(), b.span())) return false;
    if (a.pitch != b.pitch || a.rows == 1 || b.rows == 1) return true;
    int64_t d = (int64_t(uintptr_t(b.p)) - int64_t(uintptr_t(a.p))) % a.pitch;
    if (d < 0) d += a.pitch;
    return d < a.bytes || a.pitch - d < b.bytes;
}

// Outputs must overlap neither an input nor each other.
bool clash(std::initializer_list<Rows> ins, std::initializer_list<Rows> outs)
{
    for (const Rows* o = outs.begin(); o != outs.end(); ++o) {
        for (const Rows& i : ins)
            if (touch(*o, i)) return true;
        for (const Rows* q = o + 1; q != outs.end(); ++q)
            if (touch(*o, *q)) return true;
    }
    return false;
}

int status_of(hipError_t e, void* stream) { return finish(launch_status(e), stream); }

int checkpoint(const void* x, int64_t rows, int64_t width, int64_t stride, int dtype, const void* buffer, bool pack,
               void* stream)
{
    if (rows < 0 || width < 0) return MESA_ERR_SHAPE;
    if (!float_type(dtype)) return MESA_ERR_UNSUPPORTED;
    if (rows == 0 || width == 0) return MESA_OK;
    if (stride < width || !product_ok({rows, stride})) return MESA_ERR_SHAPE;
    if (any_null({x, buffer})) return MESA_ERR_NULL;
    if (!aligned(x, bytes_of(dtype)) || !aligned(buffer, 16)) return MESA_ERR_ARG;
    if (touch(tokens(x, rows, width, stride, dtype), dense(buffer, int64_t(checkpoint_bytes(rows, width))))) return MESA_ERR_ARG;
    char* base = static_cast<char*>(const_cast<void*>(buffer));
    const mesa::CheckpointArgs a{x, rows, width, stride, dtype == MESA_DTYPE_BF16, reinterpret_cast<int8_t*>(base),
                                 reinterpret_cast<uint8_t*>(base) + mesa::checkpoint_exponents_at(rows, width)};
    return status_of(mesa::launch_checkpoint(a, pack, static_cast<hipStream_t>(stream)), stream);
}

// Sizes shared by the recurrence's calls; tickets and tiles are counted in 32 bits, one of a slab
// of 32 channels and 128 tokens.
int recurrence_sizes(int64_t batch, int64_t seq_len, int64_t width, int64_t stride, float decay)
{
    if (batch < 0 || seq_len < 0 || width < 0 || seq_len > kMostElements || width > kMostElements) return MESA_ERR_SHAPE;
    if (!(isfinite(decay) && decay > 0.0f)) return MESA_ERR_ARG;
    if (batch > 0 && seq_len > 0 && stride < width) return MESA_ERR_SHAPE;
    const int64_t blocks = (seq_len + MESA_RECURRENCE_BLOCK - 1) / MESA_RECURRENCE_BLOCK, slabs = (width + 31) / 32;
    // the states are batch x width, however few the tokens
    if (!product_ok({batch, width}) || !product_ok({batch, blocks, slabs}) || batch * blocks * slabs > INT32_MAX) return MESA_ERR_SHAPE;
    return MESA_OK;
}

int64_t blocks_of(int64_t seq_len) { return (seq_len + MESA_RECURRENCE_BLOCK - 1) / MESA_RECURRENCE_BLOCK; }

bool sizes_countable(int64_t batch, int64_t seq_len, int64_t width)
{
    return batch > 0 && seq_len > 0 && width > 0 && product_ok({batch, seq_len, width});
}

}  // namespace

extern "C" {

size_t mesa_checkpoint_bytes(int64_t rows, int64_t width)
{
    if (rows <= 0 || width <= 0 || !product_ok({rows, width})) return 0;
    return checkpoint_bytes(rows, width);
}

int mesa_checkpoint_pack(const void* x, int64_t rows, int64_t width, int64_t stride, int dtype, void* buffer, void* stream)
{
    return checkpoint(x, rows, width, stride, dtype, buffer, true, stream);
}

int mesa_checkpoint_unpack(const void* buffer, int64_t rows, int64_t width, int64_t stride, int dtype, void* x, void* stream)
{
    return checkpoint(x, rows, width, stride, dtype, buffer, false, stream);
}

size_t mesa_recurrence_workspace_bytes(int64_t batch, int64_t seq_len, int64_t width)
{
    if (!sizes_countable(batch, seq_len, width)) return 0;
    return size_t(mesa::recurrence_walk_bytes(batch, mesa::recurrence_tiles(seq_len), width));
}

int mesa_recurrence(const void* x, const void* r, const void* i, const float* theta, float decay,
                    const uint8_t* reset, const float* h0, int64_t batch, int64_t seq_len, int64_t width,
                    int64_t stride, int dtype, void* y, float* final_h, float* states, void* kept_x, void* kept_r,
                    void* kept_i, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int st = recurrence_sizes(batch, seq_len, width, stride, decay); st != MESA_OK) return st;
    if (!float_type(dtype)) return MESA_ERR_UNSUPPORTED;
    if (batch == 0 || width == 0) return MESA_OK;
    if (!product_ok({batch, seq_len, seq_len > 0 ? stride : width})) return MESA_ERR_SHAPE;
    const int64_t n = batch * seq_len;
    if (seq_len > 0 && any_null({x, r, i, theta, y})) return MESA_ERR_NULL;
    const int kept = (kept_x != nullptr) + (kept_r != nullptr) + (kept_i != nullptr);
    if (n > 0 && kept != 0 && kept != 3) return MESA_ERR_NULL;
    const size_t need = mesa_recurrence_workspace_bytes(batch, seq_len, width);
    if (need > 0 && workspace == nullptr) return MESA_ERR_NULL;
    if (need > 0 && workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!all_aligned({x, r, i, y}, bytes_of(dtype)) || !all_aligned({theta, h0, final_h, states}, 4) ||
        !all_aligned({kept_x, kept_r, kept_i, workspace}, 16))
        return MESA_ERR_ARG;
    const int64_t state = batch * width * 4, held = n > 0 ? int64_t(checkpoint_bytes(n, width)) : 0;
    if (clash({tokens(x, n, width, stride, dtype), tokens(r, n, width, stride, dtype), tokens(i, n, width, stride, dtype),
               dense(theta, width * 4), dense(reset, n), dense(h0, state)},
              {tokens(y, n, width, width, dtype), dense(final_h, state), dense(states, state * blocks_of(seq_len)),
               dense(kept_x, held), dense(kept_r, held), dense(kept_i, held), dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    const mesa::RecurrenceArgs a{batch, seq_len, width, stride, dtype, x, r, i, theta, decay, reset, h0, y, final_h,
                                 states, static_cast<uint8_t*>(kept_x), static_cast<uint8_t*>(kept_r),
                                 static_cast<uint8_t*>(kept_i), int(mesa::recurrence_tiles(seq_len)),
                                 static_cast<uint64_t*>(workspace)};
    return status_of(mesa::launch_recurrence(a, static_cast<hipStream_t>(stream)), stream);
}

int mesa_recurrence_step(const float* state, const void* x, const void* r, const void* i, const float* theta,
                         float decay, const uint8_t* reset, int64_t batch, int64_t width, int64_t stride, int dtype,
                         float* state_out, void* y, void* stream)
{
    if (int st = recurrence_sizes(batch, 1, width, stride, decay); st != MESA_OK) return st;
    if (!float_type(dtype)) return MESA_ERR_UNSUPPORTED;
    if (batch == 0 || width == 0) return MESA_OK;
    if (!product_ok({batch, stride})) return MESA_ERR_SHAPE;
    if (any_null({state, x, r, i, theta, state_out, y})) return MESA_ERR_NULL;
    if (!all_aligned({x, r, i, y}, bytes_of(dtype)) || !all_aligned({theta, state, state_out}, 4)) return MESA_ERR_ARG;
    const Rows old = dense(state, batch * width * 4);
    if (clash({tokens(x, batch, width, stride, dtype), tokens(r, batch, width, stride, dtype),
               tokens(i, batch, width, stride, dtype), dense(theta, width * 4), dense(reset, batch),
               state_out == state ? Rows{} : old},
              {tokens(y, batch, width, width, dtype), dense(state_out, batch * width * 4)}))
        return MESA_ERR_ARG;
    const mesa::RecurrenceArgs a{batch, 1, width, stride, dtype, x, r, i, theta, decay, reset, state, y, nullptr,
                                 nullptr, nullptr, nullptr, nullptr, 1, nullptr};
    return status_of(mesa::launch_recurrence_step(a, state_out, static_cast<hipStream_t>(stream)), stream);
}

size_t mesa_recurrence_backward_workspace_bytes(int64_t batch, int64_t seq_len, int64_t width)
{
    if (!sizes_countable(batch, seq_len, width)) return 0;
    const int64_t tiles = blocks_of(seq_len);
    return size_t(mesa::recurrence_walk_bytes(batch, tiles, width) + (batch * tiles * width * 4 + 15) / 16 * 16);
}

int mesa_recurrence_backward(const void* x, const void* r, const void* i, const float* theta, float decay,
                             const uint8_t* reset, const float* states, const void* dy, const float* dfinal,
                             int64_t batch, int64_t seq_len, int64_t width, int64_t stride, int dtype, int grad_dtype,
                             int64_t grad_stride, void* dx, void* dr, void* di, float* dtheta, float* dh0,
                             void* workspace, size_t workspace_bytes, void* stream)
{
    if (dtype == MESA_DTYPE_Q8) stride = width;   // a checkpoint's rows are dense
    if (int st = recurrence_sizes(batch, seq_len, width, stride, decay); st != MESA_OK) return st;
    const int64_t n = batch * seq_len;
    if (batch > 0 && seq_len > 0 && grad_stride < width) return MESA_ERR_SHAPE;
    if ((!float_type(dtype) && dtype != MESA_DTYPE_Q8) || !float_type(grad_dtype)) return MESA_ERR_UNSUPPORTED;
    if (width == 0) return MESA_OK;
    if (n > 0 && (!product_ok({batch, seq_len, stride}) || !product_ok({batch, seq_len, grad_stride}))) return MESA_ERR_SHAPE;
    if (any_null({theta, dtheta}) || (n > 0 && any_null({x, r, i, states, dy, dx, dr, di}))) return MESA_ERR_NULL;
    const size_t need = mesa_recurrence_backward_workspace_bytes(batch, seq_len, width);
    if (need > 0 && workspace == nullptr) return MESA_ERR_NULL;
    if (need > 0 && workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!all_aligned({x, r, i}, dtype == MESA_DTYPE_Q8 ? 16 : bytes_of(dtype)) || !all_aligned({dy, dx, dr, di}, bytes_of(grad_dtype)) ||
        !all_aligned({theta, states, dfinal, dtheta, dh0}, 4) || !aligned(workspace, 16))
        return MESA_ERR_ARG;
    const int64_t tiles = blocks_of(seq_len), state = batch * width * 4;
    const int64_t held = n > 0 ? int64_t(checkpoint_bytes(n, width)) : 0;
    const bool q8 = dtype == MESA_DTYPE_Q8;
    if (clash({q8 ? dense(x, held) : tokens(x, n, width, stride, dtype), q8 ? dense(r, held) : tokens(r, n, width, stride, dtype),
               q8 ? dense(i, held) : tokens(i, n, width, stride, dtype), dense(theta, width * 4), dense(reset, n),
               dense(states, state * tiles), tokens(dy, n, width, width, grad_dtype), dense(dfinal, state)},
              {tokens(dx, n, width, grad_stride, grad_dtype), tokens(dr, n, width, grad_stride, grad_dtype),
               tokens(di, n, width, grad_stride, grad_dtype), dense(dtheta, width * 4), dense(dh0, state),
               dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    char* ws = static_cast<char*>(workspace);
    const mesa::RecurrenceGradArgs a{batch, seq_len, width, stride, grad_stride, dtype, grad_dtype, x, r, i, theta,
                                     decay, reset, states, dy, dfinal, dx, dr, di, dtheta, dh0, int(tiles),
                                     reinterpret_cast<uint64_t*>(ws),
                                     reinterpret_cast<float*>(ws + mesa::recurrence_walk_bytes(batch, tiles, width))};
    return status_of(mesa::launch_recurrence_backward(a, static_cast<hipStream_t>(stream)), stream);
}

}  // extern "C"

namespace {

bool dim_ok(int64_t d) { return d == 64 || d == 128; }

int ends_sizes(int64_t batch, int64_t heads, int64_t seq_len, int64_t d_k, int64_t d_v)
{
    if (batch < 0 || heads < 0 || seq_len < 0 || d_k < 0 || d_v < 0) return MESA_ERR_SHAPE;
    if (!dim_ok(d_k) || !dim_ok(d_v)) return MESA_ERR_UNSUPPORTED;
    // a workgroup of the ends takes at least 128 tokens of a (sequence, head)
    if (!product_ok({batch, heads, 128}) || !product_ok({batch, heads, seq_len, 128}) || !product_ok({heads, 128, 4}) ||
        batch * heads * ((seq_len + 127) / 128) > INT32_MAX / 4 || heads > INT32_MAX / 16)
        return MESA_ERR_SHAPE;
    return MESA_OK;
}

bool ends_countable(int64_t batch, int64_t heads, int64_t seq_len, int64_t d_k, int64_t d_v)
{
    return ends_sizes(batch, heads, seq_len, d_k, d_v) == MESA_OK && batch > 0 && heads > 0 && seq_len > 0;
}

}  // namespace

extern "C" {

size_t mesa_frontend_backward_workspace_bytes(int64_t batch, int64_t heads, int64_t seq_len, int64_t d_k, int64_t d_v)
{
    if (!ends_countable(batch, heads, seq_len, d_k, d_v)) return 0;
    return size_t(mesa::front_grad_partial_floats(batch, heads, seq_len, int(d_k), int(d_v))) * 4;
}

int mesa_frontend_backward(const void* qp, const void* kp, const void* vp, const float* conv_q, const float* conv_k,
                           const float* conv_v, const float* a_gamma, const float* a_beta, const float* theta,
                           float gamma_cap, float l2_eps, int64_t batch, int64_t heads, int64_t seq_len, int64_t d_k,
                           int64_t d_v, int dtype, const float* dq, const float* dk, const float* dv,
                           const float* dgamma, const float* dbeta, const float* dlambda, int grad_dtype, void* dqp,
                           void* dkp, void* dvp, float* dconv_q, float* dconv_k, float* dconv_v, float* da_gamma,
                           float* da_beta, float* dtheta, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int st = ends_sizes(batch, heads, seq_len, d_k, d_v); st != MESA_OK) return st;
    if ((!float_type(dtype) && dtype != MESA_DTYPE_Q8) || !float_type(grad_dtype)) return MESA_ERR_UNSUPPORTED;
    if (!(isfinite(gamma_cap) && gamma_cap >= 0.0f && gamma_cap <= 1.0f)) return MESA_ERR_ARG;
    if (!(isfinite(l2_eps) && l2_eps >= 0.0f)) return MESA_ERR_ARG;
    if (heads == 0) return MESA_OK;
    const int64_t n = batch * heads * seq_len;
    if (any_null({theta, dlambda, dtheta, conv_q, conv_k, dconv_q, dconv_k}) || (conv_v != nullptr && dconv_v == nullptr))
        return MESA_ERR_NULL;
    if (n > 0 && (any_null({qp, kp, a_gamma, a_beta, dq, dk, dv, dgamma, dbeta, dqp, dkp, dvp, da_gamma, da_beta}) ||
                  (conv_v != nullptr && vp == nullptr)))
        return MESA_ERR_NULL;
    const size_t need = mesa_frontend_backward_workspace_bytes(batch, heads, seq_len, d_k, d_v);
    if (need > 0 && workspace == nullptr) return MESA_ERR_NULL;
    if (need > 0 && workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!all_aligned({qp, kp, vp, conv_q, conv_k, conv_v, dq, dk, dv, dqp, dkp, dvp, workspace}, 16) ||
        !all_aligned({a_gamma, a_beta, theta, dgamma, dbeta, dlambda, dconv_q, dconv_k, dconv_v, da_gamma, da_beta, dtheta}, 4))
        return MESA_ERR_ARG;
    const int64_t rows = batch * seq_len, gs = bytes_of(grad_dtype);
    auto held = [&](const void* p, int64_t d) {
        return dense(p, dtype != MESA_DTYPE_Q8 ? n * d * bytes_of(dtype) : n > 0 ? int64_t(checkpoint_bytes(rows, heads * d)) : 0);
    };
    if (clash({held(qp, d_k), held(kp, d_k), held(vp, d_v), dense(conv_q, heads * d_k * 16), dense(conv_k, heads * d_k * 16),
               dense(conv_v, heads * d_v * 16), dense(a_gamma, n * 4), dense(a_beta, n * 4), dense(theta, heads * d_k * 4),
               dense(dq, n * d_k * 4), dense(dk, n * d_k * 4), dense(dv, n * d_v * 4), dense(dgamma, n * 4),
               dense(dbeta, n * 4), dense(dlambda, heads * d_k * 4)},
              {dense(dqp, n * d_k * gs), dense(dkp, n * d_k * gs), dense(dvp, n * d_v * gs), dense(dconv_q, heads * d_k * 16),
               dense(dconv_k, heads * d_k * 16), dense(conv_v != nullptr ? dconv_v : nullptr, heads * d_v * 16),
               dense(da_gamma, n * 4), dense(da_beta, n * 4), dense(dtheta, heads * d_k * 4),
               dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    const mesa::FrontGradArgs a{batch, heads, seq_len, int(d_k), int(d_v), dtype, grad_dtype, qp, kp, vp, conv_q, conv_k,
                                conv_v, a_gamma, a_beta, theta, gamma_cap, l2_eps, dq, dk, dv, dgamma, dbeta, dlambda, dqp,
                                dkp, dvp, dconv_q, dconv_k, dconv_v, da_gamma, da_beta, dtheta,
                                static_cast<float*>(workspace)};
    return status_of(mesa::launch_frontend_backward(a, static_cast<hipStream_t>(stream)), stream);
}

size_t mesa_output_norm_backward_workspace_bytes(int64_t batch, int64_t heads, int64_t seq_len, int64_t d_v)
{
    if (!ends_countable(batch, heads, seq_len, d_v, d_v)) return 0;
    return size_t(mesa::norm_grad_partial_floats(batch, heads, seq_len, int(d_v))) * 4;
}

int mesa_output_norm_backward(const void* o, const float* weight, float eps, const void* dy, int64_t batch,
                              int64_t heads, int64_t seq_len, int64_t d_v, int dtype, int grad_dtype, float* d_o,
                              float* dweight, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int st = ends_sizes(batch, heads, seq_len, d_v, d_v); st != MESA_OK) return st;
    if ((dtype != MESA_DTYPE_F32 && dtype != MESA_DTYPE_Q8) || !float_type(grad_dtype)) return MESA_ERR_UNSUPPORTED;
    if (!(isfinite(eps) && eps >= 0.0f)) return MESA_ERR_ARG;
    if (heads == 0) return MESA_OK;
    const int64_t n = batch * heads * seq_len;
    if (any_null({weight, dweight}) || (n > 0 && any_null({o, dy, d_o}))) return MESA_ERR_NULL;
    const size_t need = mesa_output_norm_backward_workspace_bytes(batch, heads, seq_len, d_v);
    if (need > 0 && workspace == nullptr) return MESA_ERR_NULL;
    if (need > 0 && workspace_bytes < need) return MESA_ERR_WORKSPACE;
    if (!all_aligned({o, weight, dy, d_o, workspace}, 16) || !aligned(dweight, 4)) return MESA_ERR_ARG;
    const int64_t held = n == 0 ? 0 : dtype == MESA_DTYPE_Q8 ? int64_t(checkpoint_bytes(n, d_v)) : n * d_v * 4;
    if (clash({dense(o, held), dense(weight, heads * d_v * 4), dense(dy, n * d_v * bytes_of(grad_dtype))},
              {dense(d_o, n * d_v * 4), dense(dweight, heads * d_v * 4), dense(workspace, int64_t(need))}))
        return MESA_ERR_ARG;
    const mesa::NormGradArgs a{batch, heads, seq_len, int(d_v), dtype, grad_dtype, o, weight, eps, dy, d_o, dweight,
                               static_cast<float*>(workspace)};
    return status_of(mesa::launch_output_norm_backward(a, static_cast<hipStream_t>(stream)), stream);
}

}  // extern "C"
