// What the 8-bit product kernels share: register types, direct loads to LDS,
// and the store of four neighbouring outputs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp4_decode.hpp"
#include "gemm_regs.hpp"

namespace ue5m3 {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
    return (uint64_t)(uint32_t)uniform((int)(uint32_t)(v >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)v);
}

// Direct loads to LDS.  m0 holds the LDS address, and the compiler does not
// track it: each load writes it in its own statement, with the state between
// that the write needs.  The immediate offset OFF counts for both sides.

// 16 bytes a lane from voff + soff + OFF to LDS at lds + OFF + 16 lane.
template <int OFF>
__device__ __forceinline__ void dma_rows(i32x4_t rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen offset:%3 lds"
                 :: "v"(voff), "s"(rsrc), "s"(soff), "n"(OFF), "s"(lds) : "memory", "m0");
}

// One dword (E8: byte, as a dword) a lane to LDS at lds + 4 lane.
template <bool E8>
__device__ __forceinline__ void dma_scale(i32x4_t rsrc, uint32_t voff, uint32_t lds) {
    if (E8)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_ubyte %0, %1, 0 offen lds"
                     :: "v"(voff), "s"(rsrc), "s"(lds) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds"
                     :: "v"(voff), "s"(rsrc), "s"(lds) : "memory", "m0");
}

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
