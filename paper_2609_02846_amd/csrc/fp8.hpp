// 8-bit floating point on the device: block scales, conversion of four values
// to a word, and the layout of the scale arrays.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace ue5m3 {
namespace {

constexpr float kE4M3Top = 448.0f, kE5M2Top = 57344.0f;

// Elements of one row of a 1D scale array (one row for each block of 128):
// whole groups of 16, so that a kernel's vector loads stay aligned.
__host__ __device__ __forceinline__ int64_t scale_pitch(int64_t rows) { return (rows + 15) / 16 * 16; }

// Largest of the 16 lanes of a DPP row, in each of them.
__device__ __forceinline__ float row16_max(float v) {
    auto step = [&](auto ctl) {
        constexpr int kCtl = decltype(ctl)::value;
        const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtl, 0xF, 0xF, false);
        v = fmaxf(v, __int_as_float(o));
    };
    step(std::integral_constant<int, 0x128>{});      // rotate right by 8, 4, 2, 1
    step(std::integral_constant<int, 0x124>{});
    step(std::integral_constant<int, 0x122>{});
    step(std::integral_constant<int, 0x121>{});
    return v;
}

// |x|, or 0 for an infinity or a NaN.
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a <= 3.4028234663852886e38f ? a : 0.0f;
}

// A block's scale and what its elements are divided by.
template <bool E8>
struct BlockScale;

template <>
struct BlockScale<true> {                            // E8M0: powers of two
    uint32_t c;
    float inv;
    // a: the block's largest finite magnitude.  p = 2^e with e the least such
    // that a <= F 2^e, F = 1.75 2^8 or 1.75 2^15: the exponent of a less that
    // of F, one more where the fraction of a is above 1.75.
    __device__ __forceinline__ static BlockScale of(float a, bool e5m2) {
        const int bits = __float_as_int(a), top = e5m2 ? 15 : 8;
        int e = (bits >> 23) - 127 - top + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
        e = max(e, -126);                            // a subnormal a lands there too
        if (bits == 0) e = 0;
        BlockScale s;
        s.c = (uint32_t)(e + 127);
        s.inv = __int_as_float((127 - e) << 23);
        return s;
    }
    // exact; the second term is 0, or NaN for an infinity
    __device__ __forceinline__ float value(float x) const { return __builtin_fmaf(x, 0.0f, x * inv); }
    __device__ __forceinline__ uint32_t code() const { return c; }
    __device__ __forceinline__ float scale() const { return __uint_as_float(c << 23); }
    // What value() takes, as four numbers, and back.
    __device__ __forceinline__ float4 pack() const { return make_float4(inv, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ static BlockScale unpack(const float4& v) {
        BlockScale s;
        s.inv = v.x;
        return s;
    }
};

template <>
struct BlockScale<false> {                           // binary32
    float s, f, a, ra;
    // Elements and block maximum are brought to the middle of the exponent
    // range together, where neither F x nor 1 / a over- or underflows.
    __device__ __forceinline__ static BlockScale of(float m, bool e5m2) {
        const float top = e5m2 ? kE5M2Top : kE4M3Top;
        m = m > 0.0f ? fmaxf(m, top * 0x1p-126f) : top;
        const float k = m > 0x1p60f ? 0x1p-64f : m < 0x1p-60f ? 0x1p64f : 1.0f;
        BlockScale b;
        b.s = m / top;
        b.f = top * k;
        b.a = m * k;
        b.ra = 1.0f / b.a;
        return b;
    }
    __device__ __forceinline__ float value(float x) const {
        const float t = x * f, y = t * ra;
        // the correction of -0 adds +0 to it: the sign is x's
        return __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-y, a, t), ra, y), x);
    }
    __device__ __forceinline__ uint32_t code() const { return 0; }
    __device__ __forceinline__ float scale() const { return s; }
    __device__ __forceinline__ float4 pack() const { return make_float4(f, a, ra, 0.0f); }
    __device__ __forceinline__ static BlockScale unpack(const float4& v) {
        BlockScale s;
        s.f = v.x;
        s.a = v.y;
        s.ra = v.z;
        return s;
    }
};

// Four values, at most the format's largest (up to the last binary32 bit),
// to its bytes: nearest, ties to even; NaN stays NaN.
template <bool E5M2>
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
    int w = 0;
    if (E5M2) {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

}  // namespace
}  // namespace ue5m3
