// Host-side launchers of the libmesa kernels.  Each kernel source file defines
// its kernels and the launcher declared here; the C ABI (libmesa.hip) validates
// arguments and calls the launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mesa {

// Shapes of one forward call.  Token (b, h, t) lives at row (b*heads + h)*seq_len + t.
struct ForwardShape {
    int64_t batch, heads, seq_len;
    int d_k, d_v, chunk;
    int n_chunks;  // ceil(seq_len / chunk)
    bool bf16;     // q, k, v element type
};

// Chunk-state scan: writes the states entering every chunk when store_chunks,
// and the fp32 states after the last token (final_H [B*H, d_k, d_k], final_G
// [B*H, d_v, d_k]) when those pointers are non-null.  Two layouts of the
// chunk states:
//   plain (frag == false): fp32 Hs [B*H, n_chunks, d_k, d_k], Gs [B*H, n_chunks, d_v, d_k];
//   fragment (frag == true, bf16 inputs, chunk 64): bf16 MFMA A-operand
//     fragments, Hs as [B*H, n_chunks, d_k/16, d_k/32, 64 lanes, 8] and Gs as
//     [B*H, n_chunks, d_v/16, d_k/32, 64 lanes, 8]; fragment (t, s) lane
//     (g, m) element e holds X[16t + m][32s + (e < 4 ? 4g + e : 16 + 4g + e - 4)].
struct StateArgs {
    ForwardShape s;
    const void* k;
    const void* v;
    const float* gamma;
    const float* beta;
    void* Hs;
    void* Gs;
    float* final_H;
    float* final_G;
    bool store_chunks;
    bool frag;
    // Scratch for the scan of few sequences (may be null: then one segment), seg_bytes
    // bytes: the fp32 totals and decays of its segments, or, where every chunk's total
    // stands at a bf16 fragment state's place, the second half of each.  Used by the
    // bf16 scan only.
    float* seg_ws = nullptr;
    size_t seg_bytes = 0;
    // With frag: also the same chunk states as plain fp32 (layout of frag == false), from
    // the same fp32-accurate pass (may be null).
    float* Hs32 = nullptr;
    float* Gs32 = nullptr;
    // Split-operand layout (bf16 inputs, chunk 64; instead of frag), fp32-accurate:
    // Hs fp32 H_c fragments, half e of fragment f = (t, s), lane l at
    // [B*H, n_chunks][(2 f + e) * 64 + l][4]; Gs the bf16 G_c fragments (high parts)
    // followed by a second plane of the same shape with the low parts bf16(x - hi).
    bool x3 = false;
};
bool chunk_state_frag_supported(const ForwardShape& s);
hipError_t launch_chunk_state(const StateArgs& a, hipStream_t stream);

// dst[0 .. n) = 0 with a fill kernel (no memset node, so the call can be graph-captured).
hipError_t launch_fill_zero(float* dst, int64_t n, hipStream_t stream);

// Chunked CG + read-out: q*_t for every token and o_t = G_t q*_t.
struct CgArgs {
    ForwardShape s;
    const void* q;
    const void* k;
    const void* v;
    const float* gamma;
    const float* beta;
    const float* lambda;
    const void* Hs;   // chunk states, plain fp32 (fp32 path) or bf16 fragments (bf16 path)
    const void* Gs;
    int n_cg;        // at most n_cg CG iterations per token
    float* out;
    float* qstar;    // may be null
    float eps2;      // Alg. 1 relative tolerance, squared: stop once |r|^2 <= eps2 |r_0|^2
    int32_t* steps;  // may be null: [B, H, T] iterations each token used
    // fp32 right-hand sides [B, H, T, d_k] solved for instead of q (fp32 path only),
    // may be null; with out null the read-out is skipped and only qstar is written
    const float* rhs = nullptr;
};
hipError_t launch_chunk_cg_f32(const CgArgs& a, hipStream_t stream);
// its chunk 64, d_k = 64 case (see chunk_cg_f32_split.hip)
hipError_t launch_chunk_cg_f32_split(const CgArgs& a, hipStream_t stream);

// Backward pass (fp32, chunk 64), in stages on one stream: 0 the right-hand sides
// u_t = G_t^T e_t, 1 the reverse adjoint scan, 2 the per-chunk gradients, 3 the
// Lambda reduction (the chunk-state scan and the solve for e* run between, through
// launch_chunk_state and launch_chunk_cg_f32).
struct BwdArgs {
    ForwardShape s;        // chunk 64
    const void* k;
    const void* v;
    const float* gamma;
    const float* beta;
    const float* qstar;    // [B, H, T, d_k]
    const float* dout;     // [B, H, T, d_v]: e_t
    const float* estar;    // [B, H, T, d_k]: e*_t
    const float* Hs;       // forward chunk states, plain fp32 [B*H, n_chunks, d_k, d_k]
    const float* Gs;       // [B*H, n_chunks, d_v, d_k]
    float* SH;             // symmetric H adjoint arriving at each chunk's end [B*H, n_chunks, d_k, d_k]
    float* AG;             // G adjoint [B*H, n_chunks, d_v, d_k]
    float* u;              // [B, H, T, d_k]
    uint16_t* u16;         // if non-null, u is written here instead, rounded to bf16
    float* dk;
    float* dv;
    float* dgamma;
    float* dbeta;
    float* dlam_part;      // [B*H, n_chunks, d_k]
    float* dlam;           // [H, d_k]
};
hipError_t launch_backward_stage(const BwdArgs& a, int stage, hipStream_t stream);
hipError_t launch_chunk_cg_bf16(const CgArgs& a, hipStream_t stream);
bool chunk_cg_bf16_supported(const ForwardShape& s);
// The same solve and read-out with split operands (hi + lo bf16 pairs, three matrix-core
// passes per product) from the split-operand chunk-state layout.
hipError_t launch_chunk_cg_x3(const CgArgs& a, hipStream_t stream);
bool chunk_cg_x3_supported(const ForwardShape& s);

// One recurrent decode step for batch*heads pairs.
struct DecodeArgs {
    int64_t batch, heads;
    int d_k, d_v;
    bool bf16;
    float* H;
    float* G;
    const void* q;
    const void* k;
    const void* v;
    const float* gamma;
    const float* beta;
    const float* lambda;
    int n_cg;
    float* out;
    float eps2;      // Alg. 1 relative tolerance, squared (0: fixed steps)
    int32_t* steps;  // may be null: [batch, heads] iterations each pair used
    bool packed = false;  // H in the packed symmetric layout (see launch_pack_state)
};
hipError_t launch_decode_step(const DecodeArgs& a, hipStream_t stream);

// Packed symmetric decode state: HP [pairs, d_k/2 + 1, d_k] with
// HP[k][i] = H[i][(i + k) mod d_k] (row k = the k-th cyclic diagonal).  Every
// unordered pair {i, j} is stored once, except on the last diagonal (k = d_k/2),
// where the copy at i < d_k/2 is the one read and written.
hipError_t launch_pack_state(const float* H, float* HP, int64_t pairs, int d_k, hipStream_t stream);
hipError_t launch_unpack_state(const float* HP, float* H, int64_t pairs, int d_k, hipStream_t stream);

// The layer's front end (App. E; gate cap and Lambda floor of App. G.5), one launch:
// q, k [B, H, T, d_k] and v [B, H, T, d_v] (element type of the projections) from the
// projections qp, kp [B, T, H, d_k], vp [B, T, H, d_v]; gamma, beta [B, H, T] from the
// gate projections a_gamma, a_beta [B, T, H]; lambda [H, d_k] from theta [H, d_k].
// conv_q, conv_k [H * d_k, 4], conv_v [H * d_v, 4] or null (values unchanged).
struct FrontArgs {
    int64_t batch, heads, seq_len;
    int d_k, d_v;
    bool bf16;
    const void* qp;
    const void* kp;
    const void* vp;
    const float* conv_q;
    const float* conv_k;
    const float* conv_v;
    const float* a_gamma;
    const float* a_beta;
    const float* theta;
    float gamma_cap, l2_eps;
    void* q;
    void* k;
    void* v;
    float* gamma;
    float* beta;
    float* lambda;
};
hipError_t launch_frontend(const FrontArgs& a, hipStream_t stream);

// The back end: per-head RMSNorm, o [B, H, T, d_v] fp32 -> y [B, T, H, d_v] (fp32 or
// bf16), weight [H, d_v].
struct NormArgs {
    int64_t batch, heads, seq_len;
    int d_v;
    bool bf16_out;
    const float* o;
    const float* weight;
    float eps;
    void* y;
};
hipError_t launch_output_norm(const NormArgs& a, hipStream_t stream);

// Element types of the calls below (MESA_DTYPE_*).
constexpr int kF32 = 0, kBf16 = 1, kQ8 = 2;

// An 8-bit checkpoint of rows x width values: the int8 codes [rows, width], then, from the
// next multiple of 16 bytes, the exponent bytes [rows, ceil(width / 32)].
__host__ __device__ inline int64_t checkpoint_exponents_at(int64_t rows, int64_t width) { return (rows * width + 15) / 16 * 16; }

// pack: x [rows, stride >= width] (fp32 or bf16) -> codes, exponents; else the other way.
struct CheckpointArgs {
    const void* x;
    int64_t rows, width, stride;
    bool bf16;
    int8_t* codes;
    uint8_t* exponents;
};
hipError_t launch_checkpoint(const CheckpointArgs& a, bool pack, hipStream_t stream);

// The gated recurrence over [batch, seq_len, width]: token (b, t) of x, r, i at element
// (b * seq_len + t) * stride, of y at (b * seq_len + t) * width.
constexpr int kRecurrenceBlock = 128;  // tokens between the states that `states` keeps
struct RecurrenceArgs {
    int64_t batch, seq_len, width, stride;
    int dtype;                // kF32 or kBf16: x, r, i and y
    const void* x;
    const void* r;
    const void* i;
    const float* theta;       // [width]
    float decay;
    const uint8_t* reset;     // [batch, seq_len] ([batch] for a step) or null
    const float* h0;          // [batch, width]; null: zeros (a step always has it)
    void* y;
    float* final_h;           // [batch, width] or null
    float* states;            // [batch, ceil(seq_len / kRecurrenceBlock), width] or null
    uint8_t* kept_x;          // checkpoints of x, r, i, all three or null
    uint8_t* kept_r;
    uint8_t* kept_i;
    int tiles;                // recurrence_tiles(seq_len) or fewer: the launch sets it
    uint64_t* words;          // recurrence_walk_bytes(batch, tiles, width), 16-byte aligned
};
int64_t recurrence_tiles(int64_t seq_len);
int64_t recurrence_walk_bytes(int64_t batch, int64_t tiles, int64_t width);
hipError_t launch_recurrence(const RecurrenceArgs& a, hipStream_t stream);
hipError_t launch_recurrence_step(const RecurrenceArgs& a, float* state_out, hipStream_t stream);

struct RecurrenceGradArgs {
    int64_t batch, seq_len, width, stride, grad_stride;
    int dtype, grad_dtype;    // x, r, i (kQ8: checkpoints); dy, dx, dr, di
    const void* x;
    const void* r;
    const void* i;
    const float* theta;
    float decay;
    const uint8_t* reset;
    const float* states;
    const void* dy;           // [batch, seq_len, width]
    const float* dfinal;      // [batch, width] or null
    void* dx;                 // token (b, t) at element (b * seq_len + t) * grad_stride
    void* dr;
    void* di;
    float* dtheta;            // [width]
    float* dh0;               // [batch, width] or null
    int tiles;                // ceil(seq_len / kRecurrenceBlock)
    uint64_t* words;          // recurrence_walk_bytes(batch, tiles, width), 16-byte aligned
    float* partial;           // [batch, tiles, width]
};
hipError_t launch_recurrence_backward(const RecurrenceGradArgs& a, hipStream_t stream);

// Gradients of the layer's front end (see FrontArgs).
struct FrontGradArgs {
    int64_t batch, heads, seq_len;
    int d_k, d_v;
    int dtype, grad_dtype;    // qp, kp, vp (kQ8: checkpoints of [batch * seq_len, heads * d]); dqp, dkp, dvp
    const void* qp;
    const void* kp;
    const void* vp;
    const float* conv_q;
    const float* conv_k;
    const float* conv_v;      // or null: the values pass through
    const float* a_gamma;
    const float* a_beta;
    const float* theta;
    float gamma_cap, l2_eps;
    const float* dq;          // [batch, heads, seq_len, d]
    const float* dk;
    const float* dv;
    const float* dgamma;      // [batch, heads, seq_len]
    const float* dbeta;
    const float* dlambda;     // [heads, d_k]
    void* dqp;                // [batch, seq_len, heads, d]
    void* dkp;
    void* dvp;
    float* dconv_q;           // [heads * d, 4]
    float* dconv_k;
    float* dconv_v;
    float* da_gamma;          // [batch, seq_len, heads]
    float* da_beta;
    float* dtheta;            // [heads, d_k]
    float* partial;           // front_grad_partial_floats
};
int64_t front_grad_partial_floats(int64_t batch, int64_t heads, int64_t seq_len, int d_k, int d_v);
hipError_t launch_frontend_backward(const FrontGradArgs& a, hipStream_t stream);

// Gradients of the back end (see NormArgs).
struct NormGradArgs {
    int64_t batch, heads, seq_len;
    int d_v;
    int dtype, grad_dtype;    // o (kF32, or kQ8: a checkpoint of [batch * heads * seq_len, d_v]); dy
    const void* o;
    const float* weight;
    float eps;
    const void* dy;           // [batch, seq_len, heads, d_v]
    float* d_o;               // [batch, heads, seq_len, d_v]
    float* dweight;           // [heads, d_v]
    float* partial;           // norm_grad_partial_floats
};
int64_t norm_grad_partial_floats(int64_t batch, int64_t heads, int64_t seq_len, int d_v);
hipError_t launch_output_norm_backward(const NormGradArgs& a, hipStream_t stream);

// Whether `blocks` workgroups of `threads` can be launched at once.  The runtime counts a launch's
// threads in 32 bits and past that starts the remainder alone, without an error (of 8388616
// workgroups of 512 threads eight ran), so such a launch has to be refused before it is made.
inline bool grid_fits(int64_t blocks, int threads) { return blocks <= int64_t(UINT32_MAX) / threads; }

// Compute units of the current device (queried once per device), for the persistent
// kernels that launch one workgroup per unit.
int device_compute_units();

}  // namespace mesa
