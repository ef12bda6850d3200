// Vectors of eight elements of the operators' tensor types, at any element
// alignment: a row of an odd number of 16-bit elements starts at any even
// address, and the device's global loads and stores take such addresses.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fp4_decode.hpp"
#include "launch.hpp"

namespace ue5m3 {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

// Eight elements as the 32-bit words that hold them (as an array of elements
// the compiler gives each 16-bit one a register of its own).
template <typename T>
struct Vec8 {
    static constexpr int kWords = sizeof(T) * 2;
    uint32_t w[kWords];

    __device__ __forceinline__ float get(int e) const {
        if constexpr (std::is_same_v<T, float>) return __uint_as_float(w[e]);
        if constexpr (std::is_same_v<T, bf16>) return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        return (float)__builtin_bit_cast(f16, (uint16_t)(w[e / 2] >> (16 * (e & 1))));
    }
    // Each value rounded to nearest, ties to even.
    __device__ __forceinline__ static Vec8 of(const float (&f)[8]) {
        Vec8 v;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (std::is_same_v<T, float>) v.w[i] = __float_as_uint(f[i]);
            else if constexpr (std::is_same_v<T, bf16>) v.w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
            else
                v.w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (f16)f[2 * i]) |
                         (uint32_t)__builtin_bit_cast(uint16_t, (f16)f[2 * i + 1]) << 16;
        }
        return v;
    }
    // Its first s elements gone, the others at their places, zeros after them.
    __device__ __forceinline__ Vec8 shifted(int s) const {
        Vec8 v;
        if constexpr (sizeof(T) == 2) {
            // by half words, then by words
            uint32_t t[kWords + 1];
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                t[i] = s & 1 ? w[i] >> 16 | (i + 1 < kWords ? w[i + 1] << 16 : 0u) : w[i];
            s >>= 1;
#pragma unroll
            for (int k = 2; k > 0; k >>= 1)
#pragma unroll
                for (int i = 0; i < kWords; ++i) t[i] = s & k ? (i + k < kWords ? t[i + k] : 0u) : t[i];
#pragma unroll
            for (int i = 0; i < kWords; ++i) v.w[i] = s < kWords ? t[i] : 0u;
        } else {
            v = *this;
#pragma unroll
            for (int k = 4; k > 0; k >>= 1)
#pragma unroll
                for (int i = 0; i < kWords; ++i) v.w[i] = s & k ? (i + k < kWords ? v.w[i + k] : 0u) : v.w[i];
#pragma unroll
            for (int i = 0; i < kWords; ++i) v.w[i] = s < kWords ? v.w[i] : 0u;
        }
        return v;
    }
};

// Elements i .. i+7 of the n at p; those past the end read as zero.
template <typename T>
__device__ __forceinline__ Vec8<T> load8(const T* p, int64_t i, int64_t n) {
    Vec8<T> v;
    if (i + 8 <= n) {
        __builtin_memcpy(&v, p + i, sizeof v);
    } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = i + j < n ? (float)p[i + j] : 0.0f;
        v = Vec8<T>::of(f);                          // (exact)
    }
    return v;
}

// The same for a row of n >= 8 elements, any i >= 0, without a branch: loads
// that lie in branches of their own are waited for one by one, and a kernel that
// streams rows lives by how many it has in flight.  The last elements come as
// the row's last eight, shifted.
template <typename T>
__device__ __forceinline__ Vec8<T> load8_row(const T* row, int i, int n) {
    const int at = min(i, n - 8);
    Vec8<T> v;
    __builtin_memcpy(&v, row + at, sizeof v);
    return v.shifted(i - at);
}

// v to elements i .. i+7 of the n at p; those past the end are dropped.
template <typename T>
__device__ __forceinline__ void store8(T* p, int64_t i, int64_t n, const Vec8<T>& v) {
    if (i + 8 <= n) {
        __builtin_memcpy(p + i, &v, sizeof v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < n) p[i + j] = (T)v.get(j);   // (exact)
    }
}

// v, as values that the compiler knows nothing of.
template <typename T>
__device__ __forceinline__ void forget(Vec8<T>& v) {
#pragma unroll
    for (int i = 0; i < Vec8<T>::kWords; ++i) asm volatile("" : "+v"(v.w[i]));
}

// Sum over the 64 lanes, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Calls f with a null pointer of the element type.
template <typename F>
hipError_t with_type(DType t, F&& f) {
    switch (t) {
        case DType::BF16: return f((bf16*)nullptr);
        case DType::F16: return f((f16*)nullptr);
        case DType::F32: return f((float*)nullptr);
    }
    return hipErrorInvalidValue;
}

}  // namespace
}  // namespace ue5m3
