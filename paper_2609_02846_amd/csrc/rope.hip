// Norms of queries and keys for each head, with the rotation by position in the
// same pass; the gradients; and the serving form, which writes keys and values
// into the pages of a cache.
//
// Of a head's row x of D elements, with the norm
//     n = x r w,  r = 1 / sqrt(mean(x^2) + eps)
// (without it n = x), and for each of P <= D / 2 pairs (a, b) = (n_p, n_{p+P}) or
// (n_2p, n_{2p+1}), at the angle t = position f_p,
//     a' = A (a cos t - b sin t),  b' = A (a sin t + b cos t);
// the elements past 2 P pass.  The gradient turns by -t, g = A (turned dy), and
//     dx = r (g w - x r^2 mean(g w x)),  dw = sum over rows of g x r.
// All in binary32, rounded once; the angle in binary64, since far positions
// times the first frequencies are thousands of turns: in quarter turns, less the
// nearest whole number of them, it is rounded to binary32 with an error of 2^-27
// of a quarter turn.
#include <algorithm>
#include <cmath>

#include "attention.hpp"
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kRopeThreads = 256, kRopeWaves = 4;

// cos and sin of position f.
__device__ __forceinline__ float2 turn(int64_t position, float f) {
    const double t = (double)position * ((double)f * 0.63661977236758134308);    // quarter turns
    const double n = rint(t);
    float s, c;
    sincospif((float)(t - n) * 0.5f, &s, &c);
    switch ((int)((int64_t)n & 3)) {
        case 0: return make_float2(c, s);
        case 1: return make_float2(-s, c);
        case 2: return make_float2(-c, -s);
        default: return make_float2(s, -c);
    }
}

__device__ __forceinline__ int64_t position_of(const ue5m3_rope_t& a, int64_t t) {
    return a.positions != nullptr ? a.positions[t] : t % a.period;
}

// Where token t's key or value goes in a cache, or a null pointer for a slot
// outside of it.
template <typename T>
__device__ __forceinline__ T* slot_row(const ue5m3_pages_t& c, void* base, int64_t slot, int head) {
    const int shift = __builtin_ctz(c.page_size);
    if (slot < 0 || slot >> shift >= c.pages) return nullptr;
    return (T*)base + (slot >> shift) * c.page + (slot & (c.page_size - 1)) * c.token + head * c.head;
}

// A wave for each row of a head: any size, two pairs a lane and up to four of
// the elements that pass.
template <typename T>
struct Row {
    float a[2], b[2], c[4];
    template <typename F>
    __device__ __forceinline__ static void each(const ue5m3_rope_t& r, int lane, F&& f) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int p = lane + 64 * j;
            if (p < r.pairs) f(j, r.interleaved ? 2 * p : p, r.interleaved ? 2 * p + 1 : p + r.pairs, p);
        }
    }
    template <typename F>
    __device__ __forceinline__ static void rest(const ue5m3_rope_t& r, int lane, F&& f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 2 * r.pairs + lane + 64 * j;
            if (e < r.dim) f(j, e);
        }
    }
    __device__ __forceinline__ void load(const ue5m3_rope_t& r, const T* x, int lane) {
#pragma unroll
        for (int j = 0; j < 2; ++j) a[j] = b[j] = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = 0.0f;
        each(r, lane, [&](int j, int i0, int i1, int) { a[j] = (float)x[i0], b[j] = (float)x[i1]; });
        rest(r, lane, [&](int j, int e) { c[j] = (float)x[e]; });
    }
    __device__ __forceinline__ void store(const ue5m3_rope_t& r, T* y, int lane) const {
        each(r, lane, [&](int j, int i0, int i1, int) { y[i0] = (T)a[j], y[i1] = (T)b[j]; });
        rest(r, lane, [&](int j, int e) { y[e] = (T)c[j]; });
    }
    __device__ __forceinline__ float dot(const Row& o) const {
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j) v += a[j] * o.a[j] + b[j] * o.b[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) v += c[j] * o.c[j];
        return wave_sum(v);
    }
    __device__ __forceinline__ void times(const Row& o) {
#pragma unroll
        for (int j = 0; j < 2; ++j) a[j] *= o.a[j], b[j] *= o.b[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] *= o.c[j];
    }
    __device__ __forceinline__ void times(float f) {
#pragma unroll
        for (int j = 0; j < 2; ++j) a[j] *= f, b[j] *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] *= f;
    }
    __device__ __forceinline__ void add(const Row& o) {
#pragma unroll
        for (int j = 0; j < 2; ++j) a[j] += o.a[j], b[j] += o.b[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] += o.c[j];
    }
    __device__ __forceinline__ void rotate(const ue5m3_rope_t& r, int64_t position, bool back, int lane) {
        each(r, lane, [&](int j, int, int, int p) {
            float2 cs = turn(position, r.freqs[p]);
            if (back) cs.y = -cs.y;
            const float u = a[j] * cs.x - b[j] * cs.y, v = a[j] * cs.y + b[j] * cs.x;
            a[j] = u * r.amplitude, b[j] = v * r.amplitude;
        });
    }
    // As its elements are numbered in a row.
    template <typename F>
    __device__ __forceinline__ void elements(const ue5m3_rope_t& r, int lane, F&& f) const {
        each(r, lane, [&](int j, int i0, int i1, int) { f(i0, a[j]), f(i1, b[j]); });
        rest(r, lane, [&](int j, int e) { f(e, c[j]); });
    }
};

// The weight of a head kind: ones where there is none.
template <typename T, typename W>
__device__ __forceinline__ Row<T> weight_row(const ue5m3_rope_t& r, const void* w, int lane) {
    Row<W> v;
    if (w != nullptr) v.load(r, (const W*)w, lane);
    Row<T> o;
#pragma unroll
    for (int j = 0; j < 2; ++j) o.a[j] = w != nullptr ? v.a[j] : 1.0f, o.b[j] = w != nullptr ? v.b[j] : 1.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o.c[j] = w != nullptr ? v.c[j] : 1.0f;
    return o;
}

template <typename T, typename W, bool APPEND>
__global__ __launch_bounds__(kRopeThreads) void rope_rows_kernel(ue5m3_rope_t r, Append ap) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int heads = r.q_heads + (APPEND ? 2 : 1) * r.kv_heads;
    const int64_t rows = r.tokens * heads, step = (int64_t)gridDim.x * kRopeWaves;
    for (int64_t at = (int64_t)blockIdx.x * kRopeWaves + wave; at < rows; at += step) {
        const int64_t t = at / heads;
        const int h = (int)(at - t * heads), kh = h - r.q_heads, vh = kh - r.kv_heads;
        const T* x = kh < 0 ? (const T*)r.q + t * r.q_token + h * r.q_head
                            : vh < 0 ? (const T*)r.k + t * r.k_token + kh * r.k_head
                                     : (const T*)ap.v + t * ap.v_token + vh * ap.v_head;
        T* y = (T*)r.q_out + t * r.q_out_token + h * r.q_out_head;
        if (kh >= 0) {
            if (APPEND) y = slot_row<T>(ap.cache, vh < 0 ? ap.cache.k : ap.cache.v, ap.slots[t], vh < 0 ? kh : vh);
            else y = (T*)r.k_out + t * r.k_out_token + kh * r.k_out_head;
        }
        if (y == nullptr) continue;
        Row<T> n;
        n.load(r, x, lane);
        if (!APPEND || vh < 0) {
            if (r.norm) {
                n.times(1.0f / sqrtf(n.dot(n) / (float)r.dim + r.eps));
                n.times(weight_row<T, W>(r, kh < 0 ? r.q_weight : r.k_weight, lane));
            }
            if (r.pairs > 0) n.rotate(r, position_of(r, t), false, lane);
        }
        n.store(r, y, lane);
    }
}

// Sums of a workgroup's rows for both weights: part [workgroup][2][dim].
template <typename T, typename W>
__global__ __launch_bounds__(kRopeThreads) void rope_rows_grad_kernel(ue5m3_rope_t r, const T* __restrict__ gq,
                                                                      const T* __restrict__ gk, float* part) {
    __shared__ float sums[kRopeWaves][2][kMaxRopeDim];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int heads = r.q_heads + r.kv_heads;
    const int64_t rows = r.tokens * heads, step = (int64_t)gridDim.x * kRopeWaves;
    Row<T> dw[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) dw[i].a[j] = dw[i].b[j] = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i].c[j] = 0.0f;
    }
    for (int64_t at = (int64_t)blockIdx.x * kRopeWaves + wave; at < rows; at += step) {
        const int64_t t = at / heads;
        const int h = (int)(at - t * heads), kh = h - r.q_heads;
        const T* dy = kh < 0 ? gq + (t * r.q_heads + h) * r.dim : gk + (t * r.kv_heads + kh) * r.dim;
        T* dx = kh < 0 ? (T*)r.q_out : (T*)r.k_out;
        if (dx != nullptr) dx += kh < 0 ? t * r.q_out_token + h * r.q_out_head : t * r.k_out_token + kh * r.k_out_head;
        Row<T> g;
        g.load(r, dy, lane);
        if (r.pairs > 0) g.rotate(r, position_of(r, t), true, lane);
        if (r.norm) {
            Row<T> x;
            x.load(r, kh < 0 ? (const T*)r.q + t * r.q_token + h * r.q_head : (const T*)r.k + t * r.k_token + kh * r.k_head,
                   lane);
            const float rstd = 1.0f / sqrtf(x.dot(x) / (float)r.dim + r.eps);
            x.times(rstd);
            Row<T> e = g;
            e.times(x);
            // (a lane's own register, not an index that the wave's head decides)
            if (kh < 0) dw[0].add(e);
            else dw[1].add(e);
            g.times(weight_row<T, W>(r, kh < 0 ? r.q_weight : r.k_weight, lane));
            x.times(-g.dot(x) / (float)r.dim);
            g.add(x);
            g.times(rstd);
        }
        if (dx != nullptr) g.store(r, dx, lane);
    }
    if (part == nullptr) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) dw[i].elements(r, lane, [&](int e, float v) { sums[wave][i][e] = v; });
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * r.dim; e += kRopeThreads) {
        const int i = e / r.dim, j = e - i * r.dim;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kRopeWaves; ++w) v += sums[w][i][j];
        part[(int64_t)blockIdx.x * 2 * r.dim + e] = v;
    }
}

// dw [2][dim] from n partial rows, in their order: a wave for 16 columns, four
// lanes a column, each a quarter of the rows.
template <typename W>
__global__ __launch_bounds__(64) void rope_sum_kernel(const float* __restrict__ part, int n, int dim, W* dqw, W* dkw) {
    const int e = blockIdx.x * 16 + (threadIdx.x & 15), quarter = threadIdx.x >> 4;
    float v = 0.0f;
    if (e < 2 * dim)
        for (int i = quarter; i < n; i += 4) v += part[(int64_t)i * 2 * dim + e];
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    if (quarter != 0 || e >= 2 * dim) return;
    W* w = e < dim ? dqw : dkw;
    if (w != nullptr) w[e < dim ? e : e - dim] = (W)v;
}

// Calls f with null pointers of the element and the weight type (x's own or
// binary32).
template <typename F>
hipError_t with_types(DType x, DType w, F&& f) {
    return with_type(x, [&](auto* t) {
        return w == x ? f(t, t) : f(t, (float*)nullptr);
    });
}

}  // namespace

int rope_grad_rows(int64_t tokens, int heads) {
    return (int)std::min<int64_t>((tokens * heads + kRopeWaves - 1) / kRopeWaves, kRopeGradRows);
}

hipError_t launch_rope(const ue5m3_rope_t& r, const Append* ap, hipStream_t s) {
    const int64_t rows = r.tokens * (r.q_heads + (ap != nullptr ? 2 : 1) * (int64_t)r.kv_heads);
    const dim3 grid((unsigned)std::min<int64_t>((rows + kRopeWaves - 1) / kRopeWaves, 1 << 20));
    return with_types((DType)r.type, (DType)r.weight_type, [&](auto* t, auto* w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        if (ap != nullptr) hipLaunchKernelGGL((rope_rows_kernel<T, W, true>), grid, dim3(kRopeThreads), 0, s, r, *ap);
        else hipLaunchKernelGGL((rope_rows_kernel<T, W, false>), grid, dim3(kRopeThreads), 0, s, r, Append{});
        return hipGetLastError();
    });
}

hipError_t launch_rope_grad(const ue5m3_rope_t& r, const void* gq, const void* gk, void* dqw, void* dkw, float* scratch,
                            hipStream_t s) {
    const bool sums = r.norm && (dqw != nullptr || dkw != nullptr);
    const int n = rope_grad_rows(r.tokens, r.q_heads + r.kv_heads);
    return with_types((DType)r.type, (DType)r.weight_type, [&](auto* t, auto* w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        hipError_t e = hipSuccess;
        if (n > 0) {
            hipLaunchKernelGGL((rope_rows_grad_kernel<T, W>), dim3(n), dim3(kRopeThreads), 0, s, r, (const T*)gq,
                               (const T*)gk, sums ? scratch : nullptr);
            e = hipGetLastError();
        }
        if (sums && e == hipSuccess) {
            hipLaunchKernelGGL((rope_sum_kernel<W>), dim3((2 * r.dim + 15) / 16), dim3(64), 0, s, scratch, n, r.dim,
                               (W*)dqw, (W*)dkw);
            e = hipGetLastError();
        }
        return e;
    });
}

}  // namespace ue5m3
