// Device helpers of the elementwise and scan kernels: four consecutive channels of a token
// per lane, held as fp32, bf16 or an 8-bit checkpoint, and the gate functions.
#pragma once

#include "mesa_device.hpp"

namespace mesa {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;

// Element tag of an 8-bit checkpoint (see the layout at launch_checkpoint_pack): int8 codes
// and, for every group of kGroup channels of a row, the exponent byte of their common scale.
struct q8_t {
    int8_t code;
};
constexpr int kGroup = 32;

// The exponent byte of a group whose largest magnitude is amax: E + 127 for the least E >=
// -126 with rint(amax 2^-E) <= 127; 255 if amax is not finite.  127.5 = 1.9921875 * 2^6 is
// the first magnitude that no longer fits at E = 0, so adding 1/128 to the significand
// carries into the exponent exactly there.
__device__ __forceinline__ uint32_t group_exponent(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = int((u + 0x10000u) >> 23) - 6;
    return u >= 0x7F800000u ? 255u : uint32_t(max(e, 1));
}
// 2^E, and infinity for byte 255, which turns every code of that group (all 0) into NaN
__device__ __forceinline__ float group_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// 2^-E for the bytes 1..249 (byte 255: no matter what, its codes are set to 0)
__device__ __forceinline__ float group_inverse(uint32_t byte) { return __uint_as_float(((254u - byte) & 0xFFu) << 23); }
// Codes of a group are at most 127 by the choice of E, but for the bytes from kRareByte on: at
// the largest exponent they stop at 63, since 64 * 2^122 is past fp32, and a group that is
// not finite has codes 0.
constexpr uint32_t kRareByte = 249;
__device__ __forceinline__ float group_most(uint32_t byte) { return byte == 255u ? 0.0f : 63.0f; }

// rint(x 2^-E), half to even, in the low byte: x 2^-E is exact (or rounds to a magnitude far
// below 1/2), and adding 1.5 * 2^23 leaves an integer's two's complement in the low bits.
__device__ __forceinline__ uint32_t group_code(float x, float inv) { return __float_as_uint(fmaf(x, inv, 12582912.0f)); }
// the same for a group with byte >= kRareByte
__device__ __forceinline__ uint32_t group_code_rare(float x, float inv, float most)
{
    const float c = __builtin_rintf(x * inv);
    return uint32_t(int(fminf(fmaxf(c, -most), most)));
}
// the low bytes of four words, first to last
__device__ __forceinline__ uint32_t pack_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0C0C0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000C0Cu);
    return lo | hi;
}
__device__ __forceinline__ uint32_t pack_codes(const float (&x)[4], uint32_t byte)
{
    const float inv = group_inverse(byte);
    if (__any(byte >= kRareByte)) {
        const float most = byte >= kRareByte ? group_most(byte) : 127.0f;
        return pack_codes(group_code_rare(x[0], inv, most), group_code_rare(x[1], inv, most), group_code_rare(x[2], inv, most),
                          group_code_rare(x[3], inv, most));
    }
    return pack_codes(group_code(x[0], inv), group_code(x[1], inv), group_code(x[2], inv), group_code(x[3], inv));
}

// max |x| with a NaN or an infinity coming out as infinity (fmaxf would drop a NaN): the
// bits of |x| order as the values do, NaNs above infinity.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Two fp32 values rounded to bf16 (nearest even, NaN stays NaN), packed low to high.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// Four channels of one token.  Vec: the address is aligned to the four elements and all four
// exist; otherwise n (0..4) of them are read or written one by one, the others read as 0.
// load_near reads channels ch .. ch + 3 of the row at element `row`, the row's last channel
// in the place of those past it (and, with Vec, its slab's first four, ch0, in the place of
// four that are), so that it asks nothing.
template <typename T>
struct Lane4;

template <>
struct Lane4<float> {
    using Raw = float4;
    template <bool Vec>
    __device__ static Raw load(const void* base, int64_t at, int n)
    {
        const float* p = static_cast<const float*>(base) + at;
        if constexpr (Vec) return n > 0 ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
        return make_float4(n > 0 ? p[0] : 0.f, n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, n > 3 ? p[3] : 0.f);
    }
    template <bool Vec>
    __device__ static Raw load_near(const void* base, int64_t row, int64_t ch, int64_t ch0, int64_t last)
    {
        const float* p = static_cast<const float*>(base) + row;
        if constexpr (Vec) return *reinterpret_cast<const float4*>(p + (ch <= last ? ch : ch0));
        return make_float4(p[min(ch, last)], p[min(ch + 1, last)], p[min(ch + 2, last)], p[min(ch + 3, last)]);
    }
    __device__ static void widen(const Raw& r, float (&x)[4]) { x[0] = r.x, x[1] = r.y, x[2] = r.z, x[3] = r.w; }
    __device__ static float4 narrow(const float (&y)[4]) { return make_float4(y[0], y[1], y[2], y[3]); }
    template <bool Vec>
    __device__ static void store(void* base, int64_t at, int n, const float (&y)[4])
    {
        float* p = static_cast<float*>(base) + at;
        if constexpr (Vec) {
            if (n > 0) *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (v < n) p[v] = y[v];
        }
    }
};

template <>
struct Lane4<bf16_t> {
    using Raw = uint2;
    template <bool Vec>
    __device__ static Raw load(const void* base, int64_t at, int n)
    {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        if constexpr (Vec) return n > 0 ? *reinterpret_cast<const uint2*>(p) : make_uint2(0u, 0u);
        const uint32_t a = n > 0 ? p[0] : 0u, b = n > 1 ? p[1] : 0u, c = n > 2 ? p[2] : 0u, d = n > 3 ? p[3] : 0u;
        return make_uint2(a | (b << 16), c | (d << 16));
    }
    template <bool Vec>
    __device__ static Raw load_near(const void* base, int64_t row, int64_t ch, int64_t ch0, int64_t last)
    {
        const uint16_t* p = static_cast<const uint16_t*>(base) + row;
        if constexpr (Vec) return *reinterpret_cast<const uint2*>(p + (ch <= last ? ch : ch0));
        return make_uint2(p[min(ch, last)] | (uint32_t(p[min(ch + 1, last)]) << 16),
                          p[min(ch + 2, last)] | (uint32_t(p[min(ch + 3, last)]) << 16));
    }
    __device__ static void widen(const Raw& r, float (&x)[4])
    {
        x[0] = __uint_as_float(r.x << 16), x[1] = __uint_as_float(r.x & 0xFFFF0000u);
        x[2] = __uint_as_float(r.y << 16), x[3] = __uint_as_float(r.y & 0xFFFF0000u);
    }
    __device__ static uint2 narrow(const float (&y)[4]) { return make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])); }
    template <bool Vec>
    __device__ static void store(void* base, int64_t at, int n, const float (&y)[4])
    {
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        const uint2 w = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
        if constexpr (Vec) {
            if (n > 0) *reinterpret_cast<uint2*>(p) = w;
        } else {
            if (n > 0) p[0] = uint16_t(w.x);
            if (n > 1) p[1] = uint16_t(w.x >> 16);
            if (n > 2) p[2] = uint16_t(w.y);
            if (n > 3) p[3] = uint16_t(w.y >> 16);
        }
    }
};

// Codes of four channels and their group's exponent byte.
struct Q8Raw {
    uint32_t codes, byte;
};
__device__ __forceinline__ void widen_q8(uint32_t codes, float scale, float (&x)[4])
{
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = float(int8_t(codes >> (8 * v))) * scale;
}
__device__ __forceinline__ uint32_t load_codes_scalar(const int8_t* p, int n)
{
    uint32_t w = 0;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (v < n) w |= uint32_t(uint8_t(p[v])) << (8 * v);
    return w;
}
template <bool Vec>
__device__ __forceinline__ uint32_t load_codes_near(const int8_t* p, int64_t ch, int64_t ch0, int64_t last)
{
    if constexpr (Vec) return *reinterpret_cast<const uint32_t*>(p + (ch <= last ? ch : ch0));
    return uint8_t(p[min(ch, last)]) | (uint32_t(uint8_t(p[min(ch + 1, last)])) << 8) | (uint32_t(uint8_t(p[min(ch + 2, last)])) << 16) |
           (uint32_t(uint8_t(p[min(ch + 3, last)])) << 24);
}

// sigma(x); exp(-x) = inf gives 0
__device__ __forceinline__ float sigmoid_fast(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }
// sigma(x) and 1 - sigma(x), each to fp32 accuracy relative to itself
__device__ __forceinline__ float sigmoid_both(float x, float& rest)
{
    const float e = __builtin_amdgcn_exp2f(-kLog2e * x);
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    rest = x > 0.0f ? e * s : 1.0f - s;
    return s;
}
// log(1 + exp(x)) = max(x, 0) + log(1 + e), e = exp(-|x|).  With u = 1 + e as rounded, log(u) e / (u - 1)
// is log(1 + e) to fp32 accuracy however small e is, and e itself where u is 1.  A NaN stays one.
__device__ __forceinline__ float softplus_fast(float x)
{
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(x));
    const float u = 1.0f + e, d = u - 1.0f;
    const float tail = d == 0.0f ? e : kLn2 * __builtin_amdgcn_logf(u) * e * __builtin_amdgcn_rcpf(d);
    return x > 0.0f ? x + tail : tail;
}

}  // namespace mesa
