// Copies of pages within a cache: page src[i] to dst[i] in every plane (the keys
// and the values of every layer), as a fork's last page or a compaction needs.
//
// The page numbers come from the host (who keeps the tables) and go to the kernel
// by value, 256 pairs a launch: there is no copy of them to the device that a
// captured graph or a later call could find overwritten.
//
// Bound: HBM, each byte read and written once (268 MB moved: 54 us, 5.0 TB/s).
#include <algorithm>

#include "attention.hpp"

namespace ue5m3 {
namespace {

constexpr int kCopyThreads = 256, kPairs = 256;

struct Pairs {
    int32_t src[kPairs], dst[kPairs];
};

// V: what a thread moves at once.  A workgroup takes `chunk` of them of one page
// of one plane.
template <typename V>
__global__ __launch_bounds__(kCopyThreads) void copy_pages_kernel(V* base, int64_t plane, int64_t page, int64_t chunk,
                                                                  int64_t planes, Pairs pairs) {
    const int64_t from = (int64_t)blockIdx.x * chunk, to = min(from + chunk, page);
    const int64_t s = pairs.src[blockIdx.y], d = pairs.dst[blockIdx.y];
    for (int64_t p = blockIdx.z; p < planes; p += gridDim.z) {
        const V* x = base + p * plane + s * page;
        V* y = base + p * plane + d * page;
#pragma unroll 4
        for (int64_t i = from + threadIdx.x; i < to; i += kCopyThreads) y[i] = x[i];
    }
}

template <typename V>
hipError_t copy(void* base, int64_t planes, int64_t plane, int64_t page, const Pairs& pairs, int n, hipStream_t s) {
    plane /= sizeof(V);
    page /= sizeof(V);
    const int64_t chunk = std::max<int64_t>(kCopyThreads, ((page + 1023) / 1024 + kCopyThreads - 1) / kCopyThreads * kCopyThreads);
    const dim3 grid((unsigned)((page + chunk - 1) / chunk), (unsigned)n, (unsigned)std::min<int64_t>(planes, 1024));
    hipLaunchKernelGGL((copy_pages_kernel<V>), grid, dim3(kCopyThreads), 0, s, (V*)base, plane, page, chunk, planes, pairs);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_copy_pages(void* base, int64_t planes, int64_t plane, int64_t page, const int32_t* src,
                             const int32_t* dst, int64_t n, hipStream_t s) {
    const bool wide = (reinterpret_cast<uintptr_t>(base) | (uintptr_t)plane | (uintptr_t)page) % 16 == 0;
    for (int64_t i = 0; i < n; i += kPairs) {
        Pairs pairs;
        const int m = (int)std::min<int64_t>(n - i, kPairs);
        std::copy(src + i, src + i + m, pairs.src);
        std::copy(dst + i, dst + i + m, pairs.dst);
        std::fill(pairs.src + m, pairs.src + kPairs, 0);
        std::fill(pairs.dst + m, pairs.dst + kPairs, 0);
        const hipError_t e = wide ? copy<uint4>(base, planes, plane, page, pairs, m, s)
                                  : copy<uint16_t>(base, planes, plane, page, pairs, m, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ue5m3
