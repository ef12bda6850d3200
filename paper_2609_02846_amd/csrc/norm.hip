// Layer norm over rows of C elements, forward and backward.
//
//   mean = sum(x) / C, rstd = 1 / sqrt(sum((x - mean)^2) / C + eps),
//   h = (x - mean) rstd, y = h w + b
//   g = dy w, dx = rstd (g - sum(g) / C - h sum(g h) / C) [+ the residual's
//   gradient], dw = sum over rows of dy h, db = sum over rows of dy
//
// All in binary32; x, dy and the outputs are read and written once, rounded
// once.  A row stays in the registers of NW waves (U vectors of eight elements
// a lane), so the variance is the sum of squared distances from the mean that
// is already known, and the backward pass reads each tensor once.
//
// Bound: HBM.  The backward pass's column sums stay in registers too (rows of up
// to 8192), over all the rows that a workgroup takes; each workgroup then writes
// one row of partial sums, and a second kernel adds those rows in order, so the
// result does not depend on which workgroup ended first.
//
// 8192 x 4096 bf16 out of HBM: forward 32 us (4.2 TB/s), backward 52 us (3.9
// TB/s) and its sum 4; a large copy reaches 5.2 TB/s.  One row: 3 us of kernel.
// Longer rows, backward with its sum: 8192 x 16384 301 us (2.7 TB/s), 2000 x 21504
// 100 (2.6).
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kBwdThreads = 1024;

// Sum of v over the NW waves that share a row, in each of their lanes.  `red`
// holds one float for each wave of the workgroup; the caller alternates two
// of them, so that one barrier a sum is enough: a slot is written again only
// after the next sum's barrier.
template <int NW>
__device__ __forceinline__ float row_sum(float v, float* red, int wave) {
    v = wave_sum(v);
    if (NW == 1) return v;
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    const int first = wave / NW * NW;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < NW; ++k) s += red[first + k];
    return s;
}

// Rows by length: below eight elements (NW = U = 1), whole vectors of eight, any
// other.
enum class Len : int { Tiny, Whole, Ragged };

template <Len L, typename T>
__device__ __forceinline__ Vec8<T> row8(const T* row, int c, int C) {
    if constexpr (L == Len::Tiny) return load8(row, c, C);
    if constexpr (L == Len::Ragged) return load8_row(row, c, C);
    Vec8<T> v;
    __builtin_memcpy(&v, row + (c < C ? c : 0), sizeof v);
#pragma unroll
    for (int i = 0; i < Vec8<T>::kWords; ++i) v.w[i] = c < C ? v.w[i] : 0u;
    return v;
}

template <typename T, typename P, int NW, int U, Len L>
__global__ __launch_bounds__(NW > 4 ? 64 * NW : 256) void norm_fwd_kernel(const T* __restrict__ x,
                                                                          const P* __restrict__ w,
                                                                          const P* __restrict__ b, T* __restrict__ y,
                                                                          float* __restrict__ mean_out,
                                                                          float* __restrict__ rstd_out, int64_t rows,
                                                                          int C, float eps) {
    constexpr int kThreads = NW > 4 ? 64 * NW : 256, kRows = kThreads / 64 / NW;
    __shared__ float red[2][kThreads / 64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c0 = ((wave % NW) * 64 + (threadIdx.x & 63)) * 8;
    const float inv = 1.0f / (float)C;
    // a workgroup's waves take the same number of turns (they share barriers)
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < rows; r0 += (int64_t)gridDim.x * kRows) {
        const bool live = r0 + wave / NW < rows;
        const int64_t r = live ? r0 + wave / NW : rows - 1;
        Vec8<T> v[U];
        Vec8<P> wv[U], bv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW * 512;
            v[u] = row8<L>(x + r * C, c, C);
            if (U <= 2 && w != nullptr) wv[u] = row8<L>(w, c, C);
            if (U <= 2 && b != nullptr) bv[u] = row8<L>(b, c, C);
        }
        float sum = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[u].get(e);
        const float mean = row_sum<NW>(sum, red[0], wave) * inv;
        float sq = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (U > 2) forget(v[u]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = v[u].get(e) - mean;
                sq += c0 + u * NW * 512 + e < C ? d * d : 0.0f;
            }
            if (U > 2) __builtin_amdgcn_sched_barrier(0);
        }
        const float rstd = 1.0f / sqrtf(row_sum<NW>(sq, red[1], wave) * inv + eps);
        if (!live) continue;
        if (c0 == 0) {
            if (mean_out != nullptr) mean_out[r] = mean;
            if (rstd_out != nullptr) rstd_out[r] = rstd;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW * 512;
            if (c >= C) break;
            if (U > 2) {                             // (no registers for them before)
                forget(v[u]);
                if (w != nullptr) wv[u] = row8<L>(w, c, C);
                if (b != nullptr) bv[u] = row8<L>(b, c, C);
            }
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float h = (v[u].get(e) - mean) * rstd;
                if (w != nullptr) h *= wv[u].get(e);
                if (b != nullptr) h += bv[u].get(e);
                o[e] = h;
            }
            store8(y + r * C, c, C, Vec8<T>::of(o));
            if (U > 2) __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Rows too long for the registers: one workgroup a row, which it reads three
// times (the second and third time from the caches).
template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(const T* __restrict__ x, const P* __restrict__ w,
                                                             const P* __restrict__ b, T* __restrict__ y,
                                                             float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                             int64_t rows, int64_t C, float eps) {
    __shared__ float red[2][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float inv = 1.0f / (float)C;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* xr = x + r * C;
        float sum = 0.0f;
        for (int64_t c = 8 * (int64_t)threadIdx.x; c < C; c += 8192) {
            const Vec8<T> v = load8(xr, c, C);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v.get(e);
        }
        const float mean = row_sum<16>(sum, red[0], wave) * inv;
        float sq = 0.0f;
        for (int64_t c = 8 * (int64_t)threadIdx.x; c < C; c += 8192) {
            const Vec8<T> v = load8(xr, c, C);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = v.get(e) - mean;
                sq += c + e < C ? d * d : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<16>(sq, red[1], wave) * inv + eps);
        if (threadIdx.x == 0) {
            if (mean_out != nullptr) mean_out[r] = mean;
            if (rstd_out != nullptr) rstd_out[r] = rstd;
        }
        for (int64_t c = 8 * (int64_t)threadIdx.x; c < C; c += 8192) {
            const Vec8<T> v = load8(xr, c, C);
            Vec8<P> wv, bv;
            if (w != nullptr) wv = load8(w, c, C);
            if (b != nullptr) bv = load8(b, c, C);
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float h = (v.get(e) - mean) * rstd;
                if (w != nullptr) h *= wv.get(e);
                if (b != nullptr) h += bv.get(e);
                o[e] = h;
            }
            store8(y + r * C, c, C, Vec8<T>::of(o));
        }
    }
}

// One workgroup takes rows b, b + grid, ... in groups of kRows, writes dx and
// keeps the column sums of dy h and dy; part: [grid][2][C].
template <typename T, typename P, int NW, int U, Len L>
__global__ __launch_bounds__(kBwdThreads) void norm_bwd_kernel(const T* __restrict__ x, const T* __restrict__ dy,
                                                               const P* __restrict__ w, const float* __restrict__ mean,
                                                               const float* __restrict__ rstd,
                                                               const T* __restrict__ res, T* __restrict__ dx,
                                                               float* __restrict__ part, int64_t rows, int C) {
    constexpr int kRows = kBwdThreads / 64 / NW;
    __shared__ float red[2][2][kBwdThreads / 64];
    __shared__ float col[kRows > 1 ? NW * 512 : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c0 = ((wave % NW) * 64 + (threadIdx.x & 63)) * 8;
    const float inv = 1.0f / (float)C;
    float dw[U][8], db[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[u][e] = db[u][e] = 0.0f;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < rows; r0 += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const bool live = r0 + wave / NW < rows;
        const int64_t r = live ? r0 + wave / NW : rows - 1;
        const float mu = mean[r], rs = rstd[r];
        Vec8<T> xv[U], gv[U], rv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW * 512;
            xv[u] = row8<L>(x + r * C, c, C);
            gv[u] = row8<L>(dy + r * C, c, C);
            if (res != nullptr) rv[u] = row8<L>(res + r * C, c, C);
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW * 512;
            Vec8<P> wv;
            if (w != nullptr) wv = row8<L>(w, c, C);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (past the row's end dy is 0, and so must h be: a NaN there would count)
                const float d = live ? gv[u].get(e) : 0.0f;
                const float h = c + e < C && live ? (xv[u].get(e) - mu) * rs : 0.0f;
                const float g = w != nullptr ? d * wv.get(e) : d;
                s1 += g;
                s2 += g * h;
                dw[u][e] += d * h;
                db[u][e] += d;
            }
            __builtin_amdgcn_sched_barrier(0);       // one vector's numbers at a time
        }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if (NW > 1) {
            if ((threadIdx.x & 63) == 0) red[turn][0][wave] = s1, red[turn][1][wave] = s2;
            __syncthreads();
            const int first = wave / NW * NW;
            s1 = s2 = 0.0f;
#pragma unroll
            for (int k = 0; k < NW; ++k) s1 += red[turn][0][first + k], s2 += red[turn][1][first + k];
        }
        s1 *= inv;
        s2 *= inv;
        if (!live || dx == nullptr) continue;
        // the row is converted again from its 16-bit (or 32-bit) elements: kept as
        // numbers since before the sums it takes more registers than there are
#pragma unroll
        for (int u = 0; u < U; ++u) {
            forget(xv[u]);
            forget(gv[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW * 512;
            if (c >= C) break;
            Vec8<P> wv;
            if (w != nullptr) wv = row8<L>(w, c, C);
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = gv[u].get(e), h = (xv[u].get(e) - mu) * rs;
                const float g = w != nullptr ? d * wv.get(e) : d;
                float v = (g - s1 - h * s2) * rs;
                if (res != nullptr) v += rv[u].get(e);
                o[e] = v;
            }
            store8(dx + r * C, c, C, Vec8<T>::of(o));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (part == nullptr) return;
    // the row groups' sums, in order, then one row of partials
    float* out = part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + u * NW * 512;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float(&acc)[8] = k == 0 ? dw[u] : db[u];
            for (int g = 1; g < kRows; ++g) {
                __syncthreads();
                if (wave / NW == g)
#pragma unroll
                    for (int e = 0; e < 8; ++e) col[c0 + e] = acc[e];
                __syncthreads();
                if (wave / NW == 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += col[c0 + e];
            }
            if (wave / NW == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < C) out[k * (int64_t)C + c + e] = acc[e];
        }
    }
}

// Rows too long for the registers: dx with one workgroup a row ...
template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(const T* __restrict__ x, const T* __restrict__ dy,
                                                             const P* __restrict__ w, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, const T* __restrict__ res,
                                                             T* __restrict__ dx, int64_t rows, int64_t C) {
    __shared__ float red[2][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float inv = 1.0f / (float)C;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = 8 * (int64_t)threadIdx.x; c < C; c += 8192) {
            const Vec8<T> xv = load8(x + r * C, c, C), gv = load8(dy + r * C, c, C);
            Vec8<P> wv;
            if (w != nullptr) wv = load8(w, c, C);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = gv.get(e) * (w != nullptr ? wv.get(e) : 1.0f);
                s1 += g;
                s2 += c + e < C ? g * ((xv.get(e) - mu) * rs) : 0.0f;
            }
        }
        s1 = row_sum<16>(s1, red[0], wave) * inv;
        s2 = row_sum<16>(s2, red[1], wave) * inv;
        for (int64_t c = 8 * (int64_t)threadIdx.x; c < C; c += 8192) {
            const Vec8<T> xv = load8(x + r * C, c, C), gv = load8(dy + r * C, c, C);
            Vec8<P> wv;
            Vec8<T> rv;
            float o[8];
            if (w != nullptr) wv = load8(w, c, C);
            if (res != nullptr) rv = load8(res + r * C, c, C);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = gv.get(e) * (w != nullptr ? wv.get(e) : 1.0f);
                float v = (g - s1 - (xv.get(e) - mu) * rs * s2) * rs;
                if (res != nullptr) v += rv.get(e);
                o[e] = v;
            }
            store8(dx + r * C, c, C, Vec8<T>::of(o));
        }
    }
}

// ... and the column sums, one workgroup for 512 columns and each of gridDim.y
// shares of the rows; part: [gridDim.y][2][C].
template <typename T>
__global__ __launch_bounds__(64) void norm_cols_kernel(const T* __restrict__ x, const T* __restrict__ dy,
                                                       const float* __restrict__ mean, const float* __restrict__ rstd,
                                                       float* __restrict__ part, int64_t rows, int64_t C) {
    const int64_t c = ((int64_t)blockIdx.x * 64 + threadIdx.x) * 8;
    if (c >= C) return;
    float dw[8] = {}, db[8] = {};
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const float mu = mean[r], rs = rstd[r];
        const Vec8<T> xv = load8(x + r * C, c, C), gv = load8(dy + r * C, c, C);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = gv.get(e);
            dw[e] += d * ((xv.get(e) - mu) * rs);
            db[e] += d;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < C) {
            part[(int64_t)blockIdx.y * 2 * C + c + e] = dw[e];
            part[((int64_t)blockIdx.y * 2 + 1) * C + c + e] = db[e];
        }
}

// dw and db from the rows of partials: 16 waves take every 16th row of 64
// columns, then add up in order; c0: the launch's first column.
template <typename P>
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* __restrict__ part, int n, int64_t c0, int64_t C,
                                                        P* __restrict__ dw, P* __restrict__ db) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = c0 + (int64_t)blockIdx.x * 64 + lane;
    P* const out = blockIdx.y == 0 ? dw : db;
    if (out == nullptr) return;
    float v = 0.0f;
    const float* const in = part + (int64_t)blockIdx.y * C + (c < C ? c : 0);
    for (int i = wave; i < n; i += 128) {            // eight loads in flight
        float t[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = in[(int64_t)min(i + 16 * k, n - 1) * 2 * C];
#pragma unroll
        for (int k = 0; k < 8; ++k) v += i + 16 * k < n ? t[k] : 0.0f;
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || c >= C) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) v += s[k][lane];
    out[c] = (P)v;
}

constexpr int64_t kRegCols = 24576, kBwdRegCols = 8192;   // the longest row held in registers
constexpr int kMaxParts = 256;
constexpr int64_t kMaxSumGrid = 1 << 21;

// Element type of the parameters: x's own or fp32.
template <typename F>
hipError_t with_types(DType x, DType p, F&& f) {
    return with_type(x, [&](auto* t) {
        if (p == DType::F32) return f(t, (float*)nullptr);
        return f(t, t);
    });
}

template <typename T, typename P, int NW, int U, Len L>
hipError_t fwd_l(const T* x, int64_t rows, int64_t C, const P* w, const P* b, float eps, T* y, float* mean, float* rstd,
               hipStream_t s) {
    constexpr int kThreads = NW > 4 ? 64 * NW : 256, kRows = kThreads / 64 / NW;
    const int64_t blocks = (rows + kRows - 1) / kRows;
    hipLaunchKernelGGL((norm_fwd_kernel<T, P, NW, U, L>), dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))),
                       dim3(kThreads), 0, s, x, w, b, y, mean, rstd, rows, (int)C, eps);
    return hipGetLastError();
}

template <typename T, typename P, int NW, int U, Len L>
hipError_t bwd_l(const T* x, const T* dy, int64_t rows, int64_t C, const P* w, const float* mean, const float* rstd,
               const T* res, T* dx, float* part, int blocks, hipStream_t s) {
    hipLaunchKernelGGL((norm_bwd_kernel<T, P, NW, U, L>), dim3((unsigned)blocks), dim3(kBwdThreads), 0, s, x, dy, w, mean,
                       rstd, res, dx, part, rows, (int)C);
    return hipGetLastError();
}

template <typename T, typename P, int NW, int U>
hipError_t fwd(const T* x, int64_t rows, int64_t C, const P* w, const P* b, float eps, T* y, float* mean, float* rstd,
               hipStream_t s) {
    return C % 8 == 0 ? fwd_l<T, P, NW, U, Len::Whole>(x, rows, C, w, b, eps, y, mean, rstd, s)
                      : fwd_l<T, P, NW, U, Len::Ragged>(x, rows, C, w, b, eps, y, mean, rstd, s);
}

template <typename T, typename P, int NW, int U>
hipError_t bwd(const T* x, const T* dy, int64_t rows, int64_t C, const P* w, const float* mean, const float* rstd,
               const T* res, T* dx, float* part, int blocks, hipStream_t s) {
    return C % 8 == 0 ? bwd_l<T, P, NW, U, Len::Whole>(x, dy, rows, C, w, mean, rstd, res, dx, part, blocks, s)
                      : bwd_l<T, P, NW, U, Len::Ragged>(x, dy, rows, C, w, mean, rstd, res, dx, part, blocks, s);
}

}  // namespace

hipError_t launch_norm(DType type, const void* x_, int64_t rows, int64_t C, DType ptype, const void* w_,
                       const void* b_, float eps, void* y_, float* mean, float* rstd, hipStream_t s) {
    return with_types(type, ptype, [&](auto* t, auto* p) {
        using T = std::remove_pointer_t<decltype(t)>;
        using P = std::remove_pointer_t<decltype(p)>;
        const T* x = (const T*)x_;
        const P *w = (const P*)w_, *b = (const P*)b_;
        T* y = (T*)y_;
        // Waves a row and vectors a lane.  Many rows: as few waves as hold a row
        // without many registers (8192 rows out of HBM, us: C = 1024 1 x 2 9.8, 2 x 1
        // 10.9; 2048 2 x 2 16.9, 4 x 1 17.8, 1 x 4 17.9; 4096 4 x 2 29, 8 x 1 36, 2 x 4
        // 32; 8192 8 x 2 58, 4 x 4 57, 16 x 1 99).  Where the workgroups are fewer than
        // the CUs twice over, latency: twice the waves, worth little (64 rows: 1024 4.64
        // against 4.76, 4096 4.60, 4.68; 512 rows of 4096 5.1, 5.2).  From 8193 columns on
        // the whole workgroup; against the streaming form it is the faster one for few
        // rows and not for many: 256 rows of 12288 6.3, 6.9, of 21504 9.1, 9.7; 4096
        // rows 67, 58 and 95, 95.
        const bool few = rows <= 512;
        if (C < 8) return fwd_l<T, P, 1, 1, Len::Tiny>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= 512) return fwd<T, P, 1, 1>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= 1024) return few ? fwd<T, P, 2, 1>(x, rows, C, w, b, eps, y, mean, rstd, s)
                                  : fwd<T, P, 1, 2>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= 2048) return few ? fwd<T, P, 4, 1>(x, rows, C, w, b, eps, y, mean, rstd, s)
                                  : fwd<T, P, 2, 2>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= 4096) return few ? fwd<T, P, 8, 1>(x, rows, C, w, b, eps, y, mean, rstd, s)
                                  : fwd<T, P, 4, 2>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= 8192) return fwd<T, P, 8, 2>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= 16384) return fwd<T, P, 16, 2>(x, rows, C, w, b, eps, y, mean, rstd, s);
        if (C <= kRegCols) return fwd<T, P, 16, 3>(x, rows, C, w, b, eps, y, mean, rstd, s);
        hipLaunchKernelGGL((norm_fwd_long_kernel<T, P>), dim3((unsigned)(rows < (1 << 20) ? rows : (1 << 20))),
                           dim3(1024), 0, s, x, w, b, y, mean, rstd, rows, C, eps);
        return hipGetLastError();
    });
}

hipError_t launch_norm_grad(DType type, const void* x_, const void* dy_, int64_t rows, int64_t C, DType ptype,
                            const void* w_, const float* mean, const float* rstd, const void* res_, void* dx_,
                            void* dw, void* db, hipStream_t s) {
    return with_types(type, ptype, [&](auto* t, auto* p) {
        using T = std::remove_pointer_t<decltype(t)>;
        using P = std::remove_pointer_t<decltype(p)>;
        const T *x = (const T*)x_, *dy = (const T*)dy_, *res = (const T*)res_;
        const P* w = (const P*)w_;
        T* dx = (T*)dx_;
        const bool sums = dw != nullptr || db != nullptr;
        // Waves a row, one vector a lane (8192 rows out of HBM, us, with the sum: C =
        // 1024 2 x 1 21, 1 x 2 25; 4096 8 x 1 53, 4 x 2 54, 2 x 4 184, whose registers
        // spill; 8192 16 x 1 101, 8 x 2 110), and how many workgroups of 1024 threads
        // take the rows.  Longer rows would take two vectors a lane of 16 waves, which
        // spill, and are streamed (2 and 3 vectors against the streaming form: 1 x 8200
        // 21.9, 9.3; 4096 x 8200 147, 99; 8192 x 16384 403, 301; 2000 x 21504 260, 100).
        const int nw = C <= 512 ? 1 : C <= 1024 ? 2 : C <= 2048 ? 4 : C <= 4096 ? 8 : 16;
        const int64_t groups = (rows + 16 / nw - 1) / (16 / nw);
        int parts = (int)(groups < kMaxParts ? groups : kMaxParts);
        if (C > kBwdRegCols) parts = (int)(rows < 64 ? rows : 64);
        if (parts < 1) parts = 1;                    // no rows: sums of nothing
        Workspace held;
        float* part = nullptr;
        hipError_t e = hipSuccess;
        if (sums) e = held.take(kWsNorm, s, (size_t)parts * 2 * (size_t)C * sizeof(float), (void**)&part);
        if (e != hipSuccess) return e;
        if (C < 8) e = bwd_l<T, P, 1, 1, Len::Tiny>(x, dy, rows, C, w, mean, rstd, res, dx, part, parts, s);
        else if (C <= 512) e = bwd<T, P, 1, 1>(x, dy, rows, C, w, mean, rstd, res, dx, part, parts, s);
        else if (C <= 1024) e = bwd<T, P, 2, 1>(x, dy, rows, C, w, mean, rstd, res, dx, part, parts, s);
        else if (C <= 2048) e = bwd<T, P, 4, 1>(x, dy, rows, C, w, mean, rstd, res, dx, part, parts, s);
        else if (C <= 4096) e = bwd<T, P, 8, 1>(x, dy, rows, C, w, mean, rstd, res, dx, part, parts, s);
        else if (C <= kBwdRegCols) e = bwd<T, P, 16, 1>(x, dy, rows, C, w, mean, rstd, res, dx, part, parts, s);
        else {
            if (dx != nullptr && rows > 0)
                hipLaunchKernelGGL((norm_bwd_long_kernel<T, P>), dim3((unsigned)(rows < (1 << 20) ? rows : (1 << 20))),
                                   dim3(1024), 0, s, x, dy, w, mean, rstd, res, dx, rows, C);
            e = hipGetLastError();
            if (e == hipSuccess && sums) {
                hipLaunchKernelGGL((norm_cols_kernel<T>), dim3((unsigned)((C + 511) / 512), (unsigned)parts), dim3(64),
                                   0, s, x, dy, mean, rstd, part, rows, C);
                e = hipGetLastError();
            }
        }
        if (e != hipSuccess || !sums) return e;
        // (a launch takes fewer than 2^32 work-items)
        for (int64_t c0 = 0; c0 < C && e == hipSuccess; c0 += 64 * kMaxSumGrid) {
            const int64_t left = (C - c0 + 63) / 64;
            hipLaunchKernelGGL((norm_sum_kernel<P>), dim3((unsigned)(left < kMaxSumGrid ? left : kMaxSumGrid), 2),
                               dim3(1024), 0, s, part, parts, c0, C, (P*)dw, (P*)db);
            e = hipGetLastError();
        }
        return e;
    });
}

}  // namespace ue5m3
