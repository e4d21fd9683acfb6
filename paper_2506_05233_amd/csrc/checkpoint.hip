// Activation checkpoints in 8 bits: rows of `width` values in groups of 32 channels, each
// group with one power of two 2^E and its values as int8 codes rint(x / 2^E).
//
// A power of two makes both directions exact but for the one rounding: x 2^-E and code 2^E
// are exact products, the codes are the same however they are computed, restoring to bf16
// loses nothing (seven bits fit its eight), and the scale is one byte for 32 values.  The
// error of a value is at most 2^E / 2 <= amax / 127 (2^-127 where E stops at -126, and up to 2^E for
// magnitudes that the largest exponent's codes stop short of); a free scale amax / 127 would halve
// that at best, at four bytes a group and with codes that hang on the rounding of a quotient.
//
// Both kernels are HBM-bound: 3.03 (bf16) or 5.03 (fp32) bytes an element each way.  A lane
// moves eight consecutive values (16 bytes of bf16), so a group is four lanes and its
// maximum two exchanges inside a quad.  16384 rows of 2048 bf16: 17.7 us to pack, 16.0 to
// unpack (102 MB, 5.7 and 6.4 TB/s, part of it out of the last-level cache), 8192 rows of fp32 13.5
// and 16.8 (101 MB).  Anything but dense rows of whole groups on aligned memory goes element by
// element, three to four times as long: the same 16384 rows as thirds of rows of 6144 52 and 59 us, the
// fp32 ones 37 and 52, 33554 bf16 rows of 1000 or of 1001 57 and 64.  33 fp32 rows of 1000 take 7 and 8
// us, all latency.
#include "mesa_kernels.hpp"
#include "mesa_lanes.hpp"

namespace mesa {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;      // values a lane
constexpr int kIter = 4;     // such pieces a lane, their loads in flight together

// Eight consecutive values, n (0..8) of them present when not Vec (the others 0).
template <bool Vec>
__device__ __forceinline__ void load8(const float* p, int n, float (&x)[8])
{
    if constexpr (Vec) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) x[v] = v < n ? p[v] : 0.0f;
    }
}
template <bool Vec>
__device__ __forceinline__ void load8(const bf16_t* p, int n, float (&x)[8])
{
    if constexpr (Vec) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int v = 0; v < 4; ++v) x[2 * v] = __uint_as_float(q[v] << 16), x[2 * v + 1] = __uint_as_float(q[v] & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) x[v] = v < n ? to_f32(p[v]) : 0.0f;
    }
}
template <bool Vec>
__device__ __forceinline__ void store8(float* p, int n, const float (&y)[8])
{
    if constexpr (Vec) {
        reinterpret_cast<float4*>(p)[0] = make_float4(y[0], y[1], y[2], y[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v)
            if (v < n) p[v] = y[v];
    }
}
template <bool Vec>
__device__ __forceinline__ void store8(bf16_t* p, int n, const float (&y)[8])
{
    const uint4 w = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
    if constexpr (Vec) {
        *reinterpret_cast<uint4*>(p) = w;
    } else {
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int v = 0; v < 8; ++v)
            if (v < n) p[v].bits = uint16_t(q[v / 2] >> (16 * (v & 1)));
    }
}

// Where piece `i` (a quarter of a group) lies: the offset of its first value in x, of its
// codes, of its group's byte, and how many of its eight values exist.
struct Place {
    int64_t x, code, byte;
    int n;
};
template <bool Flat>
__device__ __forceinline__ Place place_of(const CheckpointArgs& a, int64_t i)
{
    if constexpr (Flat) return {i * kPer, i * kPer, i / 4, kPer};
    const int64_t groups = (a.width + kGroup - 1) / kGroup;
    const int64_t group = i / 4, row = group / groups;
    const int64_t ch = (group - row * groups) * kGroup + (i & 3) * kPer;
    const int64_t left = a.width - ch;
    return {row * a.stride + ch, row * a.width + ch, group, left >= kPer ? kPer : left > 0 ? int(left) : 0};
}

template <typename T, bool Flat>
__global__ __launch_bounds__(kThreads) void checkpoint_pack_kernel(CheckpointArgs a, int64_t pieces)
{
    const int64_t first = int64_t(blockIdx.x) * (kThreads * kIter) + threadIdx.x;
    const T* x = static_cast<const T*>(a.x);
    float v[kIter][8];
    Place at[kIter];
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
        const int64_t i = first + k * kThreads;
        if (i < pieces) {
            at[k] = place_of<Flat>(a, i);
            load8<Flat>(x + at[k].x, at[k].n, v[k]);
        }
    }
    // a quad is one group, so all four of its lanes pass the test together
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
        if (first + k * kThreads >= pieces) break;
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, abs_bits(v[k][e]));
        top = max(top, uint32_t(dpp_i32<kDppQuadSwap1>(int(top), int(top))));
        top = max(top, uint32_t(dpp_i32<kDppQuadSwap2>(int(top), int(top))));
        const uint32_t byte = group_exponent(__uint_as_float(top));
        const float lo[4] = {v[k][0], v[k][1], v[k][2], v[k][3]}, hi[4] = {v[k][4], v[k][5], v[k][6], v[k][7]};
        const uint32_t w[2] = {pack_codes(lo, byte), pack_codes(hi, byte)};
        int8_t* out = a.codes + at[k].code;
        if constexpr (Flat) {
            *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < at[k].n) out[e] = int8_t(w[e / 4] >> (8 * (e % 4)));
        }
        if ((threadIdx.x & 3) == 0) a.exponents[at[k].byte] = uint8_t(byte);
    }
}

template <typename T, bool Flat>
__global__ __launch_bounds__(kThreads) void checkpoint_unpack_kernel(CheckpointArgs a, int64_t pieces)
{
    const int64_t first = int64_t(blockIdx.x) * (kThreads * kIter) + threadIdx.x;
    T* x = static_cast<T*>(const_cast<void*>(a.x));
    uint2 w[kIter];
    uint32_t byte[kIter];
    Place at[kIter];
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
        const int64_t i = first + k * kThreads;
        if (i < pieces) {
            at[k] = place_of<Flat>(a, i);
            const int8_t* in = a.codes + at[k].code;
            if constexpr (Flat)
                w[k] = *reinterpret_cast<const uint2*>(in);
            else
                w[k] = make_uint2(load_codes_scalar(in, at[k].n), load_codes_scalar(in + 4, at[k].n - 4));
            byte[k] = a.exponents[at[k].byte];
        }
    }
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
        if (first + k * kThreads >= pieces) break;
        float lo[4], hi[4];
        widen_q8(w[k].x, group_scale(byte[k]), lo);
        widen_q8(w[k].y, group_scale(byte[k]), hi);
        const float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        store8<Flat>(x + at[k].x, at[k].n, y);
    }
}

template <typename T>
hipError_t launch(const CheckpointArgs& a, bool pack, hipStream_t stream)
{
    // dense rows of whole groups on aligned memory are one run of groups: no division, 16
    // bytes a lane (both forms' times above)
    const bool flat = a.width % kGroup == 0 && a.stride == a.width && uintptr_t(a.x) % 16 == 0;
    const int64_t pieces = a.rows * ((a.width + kGroup - 1) / kGroup) * (kGroup / kPer);
    const int64_t blocks = (pieces + kThreads * kIter - 1) / (kThreads * kIter);
    if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid{unsigned(blocks)}, block{kThreads};
    if (pack && flat)
        hipLaunchKernelGGL((checkpoint_pack_kernel<T, true>), grid, block, 0, stream, a, pieces);
    else if (pack)
        hipLaunchKernelGGL((checkpoint_pack_kernel<T, false>), grid, block, 0, stream, a, pieces);
    else if (flat)
        hipLaunchKernelGGL((checkpoint_unpack_kernel<T, true>), grid, block, 0, stream, a, pieces);
    else
        hipLaunchKernelGGL((checkpoint_unpack_kernel<T, false>), grid, block, 0, stream, a, pieces);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_checkpoint(const CheckpointArgs& a, bool pack, hipStream_t stream)
{
    if (a.rows == 0 || a.width == 0) return hipSuccess;
    return a.bf16 ? launch<bf16_t>(a, pack, stream) : launch<float>(a, pack, stream);
}

}  // namespace mesa
