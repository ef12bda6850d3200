// Dropout from a counter-based generator: the mask is a function of (seed,
// tensor id, element), so it is computed where it is needed, in the forward
// and in the backward pass, and never stored.
//
// Element i takes 16 of the 128 bits that Philox4x32-10 gives for the counter
// (i / 8 in 64 bits, tensor id, 1): bits 16 (i % 2) .. +15 of word (i % 8) / 2.
// (The last counter word keeps the stream apart from stochastic rounding's,
// which has 0 there.)  The element is dropped when those 16 bits are below
// round(65536 p), so p is taken to the nearest 2^-16 and the survivors are
// scaled by the reciprocal of what that leaves: the expectation is exact.
// A dropped element is replaced, not multiplied, so a NaN or infinity there
// gives 0.
//
// Bound: HBM (read, optional residual, write), with the generator close
// behind: ten rounds cost about 20 multiplies of 64 bits and 20 XORs for eight
// elements; 32 bits for each element would double that.  8192 x 4096 bf16 with a
// residual 38 us (5.3 TB/s), without 23.6 (5.7): what a large copy reaches.
#include <cmath>

#include "codec.hpp"
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kDropThreads = 256;

template <typename T, bool RES>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const T* x, const T* res, int64_t n,
                                                               uint32_t drop, float up, uint32_t key0, uint32_t key1,
                                                               uint32_t tensor_id, T* y) {
    const int64_t chunks = (n + 7) / 8, stride = (int64_t)gridDim.x * kDropThreads;
    for (int64_t j = (int64_t)blockIdx.x * kDropThreads + threadIdx.x; j < chunks; j += stride) {
        const Vec8<T> v = load8(x, 8 * j, n);
        Vec8<T> r;
        float o[8];
        if (RES) r = load8(res, 8 * j, n);
        const uint4 c = philox4x32_10(make_uint4((uint32_t)j, (uint32_t)((uint64_t)j >> 32), tensor_id, 1u), key0, key1);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = e % 2 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFFu;
            float f = bits >= drop ? v.get(e) * up : 0.0f;
            if (RES) f = r.get(e) + f;
            o[e] = f;
        }
        store8(y, 8 * j, n, Vec8<T>::of(o));
    }
}

}  // namespace

hipError_t launch_dropout(DType type, const void* x, int64_t n, double p, uint64_t seed, uint32_t tensor_id,
                          const void* residual, void* y, hipStream_t s) {
    const uint32_t drop = (uint32_t)std::nearbyint(p * 65536.0);
    const float up = drop < 65536u ? (float)(65536.0 / (65536.0 - drop)) : 0.0f;
    const int64_t blocks = ((n + 7) / 8 + kDropThreads - 1) / kDropThreads;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
    return with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (residual != nullptr)
            hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(kDropThreads), 0, s, (const T*)x,
                               (const T*)residual, n, drop, up, (uint32_t)seed, (uint32_t)(seed >> 32), tensor_id,
                               (T*)y);
        else
            hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(kDropThreads), 0, s, (const T*)x,
                               (const T*)nullptr, n, drop, up, (uint32_t)seed, (uint32_t)(seed >> 32), tensor_id,
                               (T*)y);
        return hipGetLastError();
    });
}

}  // namespace ue5m3
