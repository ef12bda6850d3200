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
// nearest whole number of them, it is at most 1/2 and rounded to binary32 with an
// error of up to 2^-26 of a quarter turn.
#include <algorithm>
#include <cmath>

#include "attention.hpp"
#include "gemm_regs.hpp"
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
__device__ __forceinline__ T* slot_row(const ue5m3_pages_t& c, void* base, int64_t slot) {
    const int shift = __builtin_ctz(c.page_size);
    if (slot < 0 || slot >> shift >= c.pages) return nullptr;
    return (T*)base + (slot >> shift) * c.page + (slot & (c.page_size - 1)) * c.token;
}

// ---- heads of a multiple of 8 elements, pairs of a multiple of 4 ----
// 8 to 32 lanes hold a head's row (LPH), eight elements each, as two groups of
// four: of the pairs 4 c .. 4 c + 3 their first and their second elements (in halves), or
// eight neighbours.  So a pair's elements are one lane's, and so are its cos and sin: a
// wave works them out once for its token, a pair a lane, and hands them round through
// LDS; they stay in registers over all heads.  Loads of kBatch rows are under way
// together.
//
// Bound: HBM.  8192 tokens of 40 heads of 128, bf16 (168 MB): 41 us, 4.1 TB/s; the
// gradients (252 MB) 52 us, 4.8 TB/s, and 5 us for the weights' sums.
constexpr int kBatch = 4, kGradBatch = 2;

template <int LPH>
struct Lane {
    int c, sub, o0, o1;                              // lane of its head, head of the wave's, elements
    bool active, turns;
    __device__ __forceinline__ Lane(const ue5m3_rope_t& r, int lane) : c(lane % LPH), sub(lane / LPH) {
        active = 8 * c < r.dim;
        turns = 8 * c < 2 * r.pairs;
        o0 = !active ? 0 : turns && !r.interleaved ? 4 * c : 8 * c;
        o1 = !active ? 0 : turns && !r.interleaved ? r.pairs + 4 * c : 8 * c + 4;
    }
    // Sum over a head's lanes, in each.
    __device__ __forceinline__ static float sum(float v) {
#pragma unroll
        for (int off = LPH / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
        return v;
    }
};

// Eight elements of a row as they lie in memory: the loads, and later the values.
template <typename T>
struct Raw {
    uint32_t w[sizeof(T) * 2];
    __device__ __forceinline__ void load(const T* x, int o0, int o1) {
        __builtin_memcpy(w, x + o0, sizeof(T) * 4);
        __builtin_memcpy(w + sizeof(T), x + o1, sizeof(T) * 4);
    }
    // (the values come into being here: the compiler would else work on all rows of a
    // batch together, in twice the registers)
    __device__ __forceinline__ void get(float (&f)[8]) const {
        Vec8<T> v;
        __builtin_memcpy(&v, w, sizeof v);
        forget(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v.get(i);
    }
    __device__ __forceinline__ void put(T* y, int o0, int o1) const {
        __builtin_memcpy(y + o0, w, sizeof(T) * 4);
        __builtin_memcpy(y + o1, w + sizeof(T), sizeof(T) * 4);
    }
    __device__ __forceinline__ static void store(T* y, int o0, int o1, const float (&f)[8]) {
        const Vec8<T> v = Vec8<T>::of(f);
        __builtin_memcpy(y + o0, v.w, sizeof(T) * 4);
        __builtin_memcpy(y + o1, v.w + sizeof(T), sizeof(T) * 4);
    }
};

// cos and sin, times the amplitude, of the lane's four pairs at a position; `table` is
// the wave's.
__device__ __forceinline__ void turns_of(const ue5m3_rope_t& r, int64_t position, float2* table, int lane, int c, bool turns,
                                         float2 (&cs)[4]) {
    wave_lds_sync();                                 // (the last token's have been read)
    for (int p = lane; p < r.pairs; p += 64) {
        const float2 t = turn(position, r.freqs[p]);
        table[p] = make_float2(t.x * r.amplitude, t.y * r.amplitude);
    }
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = turns ? table[4 * c + i] : make_float2(1.0f, 0.0f);
}

// Turned by the angles (back: by their negatives); NEAR: pairs of neighbours.
template <bool NEAR>
__device__ __forceinline__ void rotate8(float (&f)[8], const float2 (&cs)[4], bool back) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float s = back ? -cs[i].y : cs[i].y;
        const float a = NEAR ? f[2 * i] : f[i], b = NEAR ? f[2 * i + 1] : f[4 + i];
        const float u = a * cs[i].x - b * s, v = a * s + b * cs[i].x;
        f[NEAR ? 2 * i : i] = u, f[NEAR ? 2 * i + 1 : 4 + i] = v;
    }
}

// Elements of a weight, which has the rows' type or binary32; ones where there is none.
template <typename T>
__device__ __forceinline__ float weight_at(const ue5m3_rope_t& r, const void* w, int e) {
    if (!r.norm || w == nullptr) return 1.0f;
    return r.weight_type == UE5M3_F32 ? ((const float*)w)[e] : (float)((const T*)w)[e];
}
template <typename T>
__device__ __forceinline__ void weight8(const ue5m3_rope_t& r, const void* w, int o0, int o1, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 1.0f;
    if (!r.norm || w == nullptr) return;
    if (r.weight_type == UE5M3_F32) {
        Raw<float> v;
        v.load((const float*)w, o0, o1);
        v.get(f);
    } else {
        Raw<T> v;
        v.load((const T*)w, o0, o1);
        v.get(f);
    }
}

// Units from .. to - 1 of a token's heads of one kind, kHeads heads each, kBatch units at
// a time: load(i, h) loads the lane's row of head h as the batch's i-th, use(i, h, ok)
// works on it; lanes past the heads load the last one's (no load in a branch of its
// own: it would be waited for alone) and are not ok.
template <int LPH, int kBatch, typename Load, typename Use>
__device__ __forceinline__ void each_head(const Lane<LPH>& at, int heads, int from, int to, Load&& load, Use&& use) {
    constexpr int kHeads = 64 / LPH;
    for (int u = from; u < to; u += kBatch) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) load(i, min((u + i) * kHeads + at.sub, heads - 1));
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int h = (u + i) * kHeads + at.sub;
            use(i, h, u + i < to && h < heads && at.active);
        }
    }
}

// A wave takes a token's heads, or with few tokens one of `segments` shares of them.
template <typename T, bool APPEND, bool NEAR, int LPH>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(ue5m3_rope_t r, Append ap, int segments) {
    constexpr int kHeads = 64 / LPH;                 // of a wave at once
    __shared__ float2 tables[kRopeWaves][kMaxRopeDim / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const Lane<LPH> at(r, lane);
    const int q_units = (r.q_heads + kHeads - 1) / kHeads, k_units = (r.kv_heads + kHeads - 1) / kHeads;
    const int units = q_units + (APPEND ? 2 : 1) * k_units;
    float wq[8], wk[8];
    weight8<T>(r, r.q_weight, at.o0, at.o1, wq);
    weight8<T>(r, r.k_weight, at.o0, at.o1, wk);
    const int64_t items = r.tokens * segments, step = (int64_t)gridDim.x * kRopeWaves;
    for (int64_t item = (int64_t)blockIdx.x * kRopeWaves + wave; item < items; item += step) {
        const int64_t t = item / segments;
        const int part = (int)(item - t * segments);
        const int u0 = (int)((int64_t)units * part / segments), u1 = (int)((int64_t)units * (part + 1) / segments);
        const int64_t slot = APPEND ? ap.slots[t] : 0;
        float2 cs[4];
        if (r.pairs > 0) turns_of(r, position_of(r, t), tables[wave], lane, at.c, at.turns, cs);
        Raw<T> raw[kBatch];
        auto turned = [&](const Raw<T>& x, const float (&w)[8], float (&f)[8]) {
            x.get(f);
            if (r.norm) {
                float sq = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sq += at.active ? f[j] * f[j] : 0.0f;
                const float rstd = 1.0f / sqrtf(Lane<LPH>::sum(sq) / (float)r.dim + r.eps);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = f[j] * rstd * w[j];
            }
            if (r.pairs > 0) rotate8<NEAR>(f, cs, false);
        };
        const T* const q = (const T*)r.q + t * r.q_token;
        T* const qo = (T*)r.q_out + t * r.q_out_token;
        each_head<LPH, kBatch>(at, r.q_heads, u0, min(u1, q_units),
                       [&](int i, int h) { raw[i].load(q + h * r.q_head, at.o0, at.o1); },
                       [&](int i, int h, bool ok) {
                           float f[8];
                           turned(raw[i], wq, f);
                           if (ok) Raw<T>::store(qo + h * r.q_out_head, at.o0, at.o1, f);
                       });
        const T* const k = (const T*)r.k + t * r.k_token;
        T* const ko = APPEND ? slot_row<T>(ap.cache, ap.cache.k, slot) : (T*)r.k_out + t * r.k_out_token;
        const int64_t ko_head = APPEND ? ap.cache.head : r.k_out_head;
        if (APPEND && ko == nullptr) continue;
        each_head<LPH, kBatch>(at, r.kv_heads, max(u0 - q_units, 0), min(u1 - q_units, k_units),
                       [&](int i, int h) { raw[i].load(k + h * r.k_head, at.o0, at.o1); },
                       [&](int i, int h, bool ok) {
                           float f[8];
                           turned(raw[i], wk, f);
                           if (ok) Raw<T>::store(ko + h * ko_head, at.o0, at.o1, f);
                       });
        if (!APPEND) continue;
        const T* const v = (const T*)ap.v + t * ap.v_token;
        T* const vo = slot_row<T>(ap.cache, ap.cache.v, slot);
        each_head<LPH, kBatch>(at, r.kv_heads, max(u0 - q_units - k_units, 0), u1 - q_units - k_units,
                       [&](int i, int h) { raw[i].load(v + h * ap.v_head, at.o0, at.o1); },
                       [&](int i, int h, bool ok) {
                           if (ok) raw[i].put(vo + h * ap.cache.head, at.o0, at.o1);
                       });
    }
}

// Sums of a workgroup's rows for both weights: part [workgroup][2][dim].
template <typename T, bool NORM, bool NEAR, int LPH>
__global__ __launch_bounds__(kRopeThreads) void rope_grad_kernel(ue5m3_rope_t r, const T* gq, const T* gk, float* part) {
    constexpr int kHeads = 64 / LPH;
    __shared__ float2 tables[kRopeWaves][kMaxRopeDim / 2];
    __shared__ float sums[kRopeWaves][2][kMaxRopeDim];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const Lane<LPH> at(r, lane);
    float wq[8], wk[8], dw[2][8];
    weight8<T>(r, r.q_weight, at.o0, at.o1, wq);
    weight8<T>(r, r.k_weight, at.o0, at.o1, wk);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[0][j] = dw[1][j] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * kRopeWaves;
    for (int64_t t = (int64_t)blockIdx.x * kRopeWaves + wave; t < r.tokens; t += step) {
        float2 cs[4];
        if (r.pairs > 0) turns_of(r, position_of(r, t), tables[wave], lane, at.c, at.turns, cs);
        Raw<T> raw[kGradBatch], in[kGradBatch];
        auto side = [&](int heads, const T* g, const T* x, int64_t x_head, T* dx, int64_t dx_head, const float (&w)[8],
                        float (&sum)[8]) {
            each_head<LPH, kGradBatch>(at, heads, 0, (heads + kHeads - 1) / kHeads,
                           [&](int i, int h) {
                               raw[i].load(g + h * r.dim, at.o0, at.o1);
                               if (NORM) in[i].load(x + h * x_head, at.o0, at.o1);
                           },
                           [&](int i, int h, bool ok) {
                               float f[8];
                               raw[i].get(f);
                               if (r.pairs > 0) rotate8<NEAR>(f, cs, true);
                               if (NORM) {
                                   float hat[8], sq = 0.0f, dot = 0.0f;
                                   in[i].get(hat);
#pragma unroll
                                   for (int j = 0; j < 8; ++j) sq += at.active ? hat[j] * hat[j] : 0.0f;
                                   const float rstd = 1.0f / sqrtf(Lane<LPH>::sum(sq) / (float)r.dim + r.eps);
#pragma unroll
                                   for (int j = 0; j < 8; ++j) {
                                       hat[j] *= rstd;
                                       sum[j] += ok ? f[j] * hat[j] : 0.0f;
                                       f[j] *= w[j];
                                       dot += at.active ? f[j] * hat[j] : 0.0f;
                                   }
                                   const float mean = Lane<LPH>::sum(dot) / (float)r.dim;
#pragma unroll
                                   for (int j = 0; j < 8; ++j) f[j] = rstd * (f[j] - hat[j] * mean);
                               }
                               if (ok && dx != nullptr) Raw<T>::store(dx + h * dx_head, at.o0, at.o1, f);
                           });
        };
        side(r.q_heads, gq + t * r.q_heads * r.dim, (const T*)r.q + t * r.q_token, r.q_head,
             r.q_out != nullptr ? (T*)r.q_out + t * r.q_out_token : nullptr, r.q_out_head, wq, dw[0]);
        side(r.kv_heads, gk + t * r.kv_heads * r.dim, (const T*)r.k + t * r.k_token, r.k_head,
             r.k_out != nullptr ? (T*)r.k_out + t * r.k_out_token : nullptr, r.k_out_head, wk, dw[1]);
    }
    if (part == nullptr) return;
    // the wave's heads, then the waves, in their order
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = dw[k][j];
#pragma unroll
            for (int off = LPH; off < 64; off <<= 1) v += __shfl_xor(v, off);
            if (at.sub == 0 && at.active) sums[wave][k][j < 4 ? at.o0 + j : at.o1 + j - 4] = v;
        }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * r.dim; e += kRopeThreads) {
        const int k = e / r.dim, j = e - k * r.dim;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kRopeWaves; ++w) v += sums[w][k][j];
        part[(int64_t)blockIdx.x * 2 * r.dim + e] = v;
    }
}

// ---- any other heads ----
// A wave for each row of a head: any size, two pairs a lane and up to four of
// the elements that pass.  Bound: the angles in binary64, which each row works out for
// itself, and loads of one element a lane: 8192 tokens of 40 heads of 100, bf16 (131 MB) take
// 161 us (heads of 128 by lanes of eight, of the same tensors again and again, 34), with
// gradients 443 (94); heads of 50 as long.
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

template <typename T>
__device__ __forceinline__ Row<T> weight_row(const ue5m3_rope_t& r, const void* w, int lane) {
    Row<T> o;
#pragma unroll
    for (int j = 0; j < 2; ++j) o.a[j] = o.b[j] = 1.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o.c[j] = 1.0f;
    Row<T>::each(r, lane, [&](int j, int i0, int i1, int) { o.a[j] = weight_at<T>(r, w, i0), o.b[j] = weight_at<T>(r, w, i1); });
    Row<T>::rest(r, lane, [&](int j, int e) { o.c[j] = weight_at<T>(r, w, e); });
    return o;
}

template <typename T, bool APPEND>
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
            if (APPEND) {
                y = slot_row<T>(ap.cache, vh < 0 ? ap.cache.k : ap.cache.v, ap.slots[t]);
                if (y != nullptr) y += (vh < 0 ? kh : vh) * ap.cache.head;
            } else y = (T*)r.k_out + t * r.k_out_token + kh * r.k_out_head;
        }
        if (y == nullptr) continue;
        Row<T> n;
        n.load(r, x, lane);
        if (!APPEND || vh < 0) {
            if (r.norm) {
                n.times(1.0f / sqrtf(n.dot(n) / (float)r.dim + r.eps));
                n.times(weight_row<T>(r, kh < 0 ? r.q_weight : r.k_weight, lane));
            }
            if (r.pairs > 0) n.rotate(r, position_of(r, t), false, lane);
        }
        n.store(r, y, lane);
    }
}

// Sums of a workgroup's rows for both weights: part [workgroup][2][dim].
template <typename T>
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
            g.times(weight_row<T>(r, kh < 0 ? r.q_weight : r.k_weight, lane));
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

// dw [2][dim] from n partial rows: 16 columns a workgroup, 16 of its threads a column,
// each every 16th row; then those, in a fixed order.
template <typename W>
__global__ __launch_bounds__(kRopeThreads) void rope_sum_kernel(const float* __restrict__ part, int n, int dim, W* dqw, W* dkw) {
    __shared__ float sums[16][17];
    const int col = threadIdx.x & 15, first = threadIdx.x >> 4, e = blockIdx.x * 16 + col;
    float v = 0.0f;
    if (e < 2 * dim) {
#pragma unroll 8
        for (int i = first; i < n; i += 16) v += part[(int64_t)i * 2 * dim + e];
    }
    sums[first][col] = v;
    __syncthreads();
    if (first != 0 || e >= 2 * dim) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += sums[i][col];
    W* w = e < dim ? dqw : dkw;
    if (w != nullptr) w[e < dim ? e : e - dim] = (W)v;
}

// Whether heads are held by lanes of eight elements, and by how many.
bool by_eights(const ue5m3_rope_t& r) { return r.dim % 8 == 0 && r.pairs % 4 == 0; }

// Calls f(lanes of a head, whether pairs are neighbours).
template <typename F>
hipError_t with_lanes(const ue5m3_rope_t& r, F&& f) {
    auto sized = [&](auto near) {
        if (r.dim <= 64) return f(std::integral_constant<int, 8>{}, near);
        if (r.dim <= 128) return f(std::integral_constant<int, 16>{}, near);
        return f(std::integral_constant<int, 32>{}, near);
    };
    return r.interleaved ? sized(std::true_type{}) : sized(std::false_type{});
}

// Shares of a token's heads: enough waves for every SIMD where tokens are few.
int segments_of(int64_t tokens, int units) { return (int)std::max<int64_t>(1, std::min<int64_t>(units, 1024 / std::max<int64_t>(tokens, 1))); }

}  // namespace

int rope_grad_rows(int64_t tokens, int heads) {
    return (int)std::min<int64_t>((tokens * heads + kRopeWaves - 1) / kRopeWaves, kRopeGradRows);
}

hipError_t launch_rope(const ue5m3_rope_t& r, const Append* ap, hipStream_t s) {
    const int heads = r.q_heads + (ap != nullptr ? 2 : 1) * r.kv_heads;
    const Append none{};
    return with_type((DType)r.type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (by_eights(r))
            return with_lanes(r, [&](auto lanes, auto near) {
                constexpr int LPH = decltype(lanes)::value;
                constexpr bool NEAR = decltype(near)::value;
                const int n = segments_of(r.tokens, (heads + 64 / LPH - 1) / (64 / LPH));
                const dim3 grid((unsigned)std::min<int64_t>((r.tokens * n + kRopeWaves - 1) / kRopeWaves, 1 << 20));
                if (ap != nullptr)
                    hipLaunchKernelGGL((rope_kernel<T, true, NEAR, LPH>), grid, dim3(kRopeThreads), 0, s, r, *ap, n);
                else
                    hipLaunchKernelGGL((rope_kernel<T, false, NEAR, LPH>), grid, dim3(kRopeThreads), 0, s, r, none, n);
                return hipGetLastError();
            });
        const dim3 grid((unsigned)std::min<int64_t>((r.tokens * heads + kRopeWaves - 1) / kRopeWaves, 1 << 20));
        if (ap != nullptr) hipLaunchKernelGGL((rope_rows_kernel<T, true>), grid, dim3(kRopeThreads), 0, s, r, *ap);
        else hipLaunchKernelGGL((rope_rows_kernel<T, false>), grid, dim3(kRopeThreads), 0, s, r, none);
        return hipGetLastError();
    });
}

hipError_t launch_rope_grad(const ue5m3_rope_t& r, const void* gq, const void* gk, void* dqw, void* dkw, float* scratch,
                            hipStream_t s) {
    const bool sums = r.norm && (dqw != nullptr || dkw != nullptr);
    const int n = rope_grad_rows(r.tokens, r.q_heads + r.kv_heads);
    float* const part = sums ? scratch : nullptr;
    hipError_t e = hipSuccess;
    if (n > 0)
        e = with_type((DType)r.type, [&](auto* t) {
            using T = std::remove_pointer_t<decltype(t)>;
            if (by_eights(r))
                return with_lanes(r, [&](auto lanes, auto near) {
                    constexpr int LPH = decltype(lanes)::value;
                    constexpr bool NEAR = decltype(near)::value;
                    if (r.norm)
                        hipLaunchKernelGGL((rope_grad_kernel<T, true, NEAR, LPH>), dim3(n), dim3(kRopeThreads), 0, s, r,
                                           (const T*)gq, (const T*)gk, part);
                    else
                        hipLaunchKernelGGL((rope_grad_kernel<T, false, NEAR, LPH>), dim3(n), dim3(kRopeThreads), 0, s, r,
                                           (const T*)gq, (const T*)gk, part);
                    return hipGetLastError();
                });
            hipLaunchKernelGGL((rope_rows_grad_kernel<T>), dim3(n), dim3(kRopeThreads), 0, s, r, (const T*)gq, (const T*)gk, part);
            return hipGetLastError();
        });
    if (e != hipSuccess || !sums) return e;
    return with_type((DType)r.weight_type, [&](auto* w) {
        using W = std::remove_pointer_t<decltype(w)>;
        hipLaunchKernelGGL((rope_sum_kernel<W>), dim3((2 * r.dim + 15) / 16), dim3(kRopeThreads), 0, s, scratch, n, r.dim,
                           (W*)dqw, (W*)dkw);
        return hipGetLastError();
    });
}

}  // namespace ue5m3
