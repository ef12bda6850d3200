// What the 8-bit product kernels share: register types and the store of four
// neighbouring outputs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp4_decode.hpp"

namespace ue5m3 {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Outputs (m, n .. n+3) of a [., N] row-major C, those past N dropped.
template <bool OUT_BF16>
__device__ __forceinline__ void store4(void* C, int64_t m, int64_t n, int64_t N, const f32x4& v) {
    if (OUT_BF16) {
        uint16_t* d = (uint16_t*)C + m * N + n;
        const uint32_t lo = pack_bf16x2(v[0], v[1]), hi = pack_bf16x2(v[2], v[3]);
        if (n + 4 <= N) {
            const uint2 w = make_uint2(lo, hi);
            __builtin_memcpy(d, &w, 8);
        } else {
            if (n < N) d[0] = (uint16_t)lo;
            if (n + 1 < N) d[1] = (uint16_t)(lo >> 16);
            if (n + 2 < N) d[2] = (uint16_t)hi;
        }
    } else {
        float* d = (float*)C + m * N + n;
        if (n + 4 <= N) {
            __builtin_memcpy(d, &v, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < N) d[e] = v[e];
        }
    }
}

}  // namespace
}  // namespace ue5m3
