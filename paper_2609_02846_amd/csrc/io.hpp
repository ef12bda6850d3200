// Vectors of eight elements of the operators' tensor types, at any element
// alignment: a row of an odd number of 16-bit elements starts at any even
// address, and the device's global loads and stores take such addresses.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.hpp"

namespace ue5m3 {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

template <typename T>
struct Vec8 {
    T e[8];
};

// Elements i .. i+7 of the n at p; those past the end read as zero.
template <typename T>
__device__ __forceinline__ Vec8<T> load8(const T* p, int64_t i, int64_t n) {
    Vec8<T> v;
    if (i + 8 <= n) {
        __builtin_memcpy(&v, p + i, sizeof v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v.e[j] = i + j < n ? p[i + j] : (T)0.0f;
    }
    return v;
}

// v to elements i .. i+7 of the n at p; those past the end are dropped.
template <typename T>
__device__ __forceinline__ void store8(T* p, int64_t i, int64_t n, const Vec8<T>& v) {
    if (i + 8 <= n) {
        __builtin_memcpy(p + i, &v, sizeof v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < n) p[i + j] = v.e[j];
    }
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
