// The 8-bit product for few rows of A (up to 64: tokens being decoded): every
// weight is read once, straight into registers, so this is as fast as HBM
// gives B.
//
// A workgroup takes 16 rows of B and splits the contraction over its waves; a
// wave's v_mfma_f32_16x16x128_f8f6f4 takes a block of those 16 rows (two
// 16-byte loads a lane, whole 128-byte lines) and of 16 rows of A, MT times.
// The waves' sums meet in LDS.  A lane's 32 bytes are consecutive k here; A is
// read the same way.
//
// FUSED: A is bf16, a few thousand elements in all, and every workgroup
// quantizes it for itself, into LDS, while its first weights are on their way:
// one launch, and nothing to wait for, instead of two.
#include <algorithm>

#include "fp8.hpp"
#include "fp8_tile.hpp"
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kFusedBytes = 16384;               // quantized tokens that a workgroup keeps

struct SkinnyArgs {
    const uint8_t* a;                            // payload, or bf16 tokens (FUSED)
    const void* as;
    const uint8_t* b;
    const void* bs;
    void* c;
    int64_t N;
    int M, K, KB;
};

__device__ __forceinline__ i32x8 load32(const uint8_t* p) {
    const uint4 lo = *reinterpret_cast<const uint4*>(p), hi = *reinterpret_cast<const uint4*>(p + 16);
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

template <int NW, int MT, int AF, bool E8, bool TILED, bool FUSED, bool OUT_BF16>
__global__ __launch_bounds__(64 * NW) void gemm_fp8_skinny_kernel(const SkinnyArgs g) {
    constexpr int kU = MT > 2 ? 2 : 4;           // blocks of a turn, all loaded before the first is used
    __shared__ __attribute__((aligned(16))) f32x4 sums[NW][MT][64];
    extern __shared__ __attribute__((aligned(16))) uint8_t dyn[];    // FUSED: payload rows, then scales
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q = lane >> 4, KB = g.KB;
    const int64_t Kp = (int64_t)KB * 128, n0 = (int64_t)blockIdx.x * 16, pb = scale_pitch(g.N);
    const int row = (int)Kp + 16;                // FUSED: bytes of a payload row in LDS
    using El = std::conditional_t<E8, uint8_t, float>;
    const El* const bs = (const El*)g.bs;
    const El* const as = (const El*)g.as;
    El* const sA = (El*)(dyn + g.M * row);

    const uint8_t* const wrow = g.b + min(n0 + l16, g.N - 1) * Kp + q * 32;
    const uint8_t* arow[MT];
    int at[MT];                                  // the lane's rows of A
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        at[t] = min(16 * t + l16, g.M - 1);
        arow[t] = FUSED ? dyn + at[t] * row + q * 32 : g.a + at[t] * Kp + q * 32;
    }
    const int64_t pa = scale_pitch(g.M);
    const int64_t bn = min(n0 + (E8 ? l16 : 4 * q), E8 ? g.N - 1 : pb - 4);
    struct Block {
        i32x8 w;
        El s;
        f32x4 s4;
    };
    auto fetch = [&](Block& f, int kb) {
        kb = min(kb, KB - 1);
        f.w = load32(wrow + (int64_t)kb * 128);
        if (TILED) f.s = bs[n0 / 128 * KB + kb];
        else if (E8) f.s = bs[kb * pb + bn];
        else f.s4 = *reinterpret_cast<const f32x4*>((const float*)g.bs + kb * pb + bn);
    };

    Block f[kU];
    i32x8 a[FUSED ? 1 : kU][MT];                 // FUSED: read from LDS at the product
    El sa[FUSED ? 1 : kU][MT];
    auto fetch_a = [&](int u, int kb) {
        kb = min(kb, KB - 1);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            a[u][t] = load32(arow[t] + (int64_t)kb * 128);
            sa[u][t] = FUSED ? sA[at[t] * KB + kb] : as[kb * pa + at[t]];
        }
    };
#pragma unroll
    for (int u = 0; u < kU; ++u) fetch(f[u], wave + u * NW);

    if constexpr (FUSED) {
        const bf16* const x = (const bf16*)g.a;
        for (int blk = threadIdx.x >> 4; blk < g.M * KB; blk += 4 * NW) {
            const int t = blk / KB, kb = blk - t * KB, k = kb * 128 + l16 * 8;
            const Vec8<bf16> v = load8(x + (int64_t)t * g.K, k, g.K);
            float a = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) a = fmaxf(a, finite_abs(v.get(e)));
            const BlockScale<E8> s = BlockScale<E8>::of(row16_max(a), false);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = s.value(v.get(e));
            *reinterpret_cast<uint2*>(dyn + t * row + k) =
                make_uint2(pack_fp8<false>(y[0], y[1], y[2], y[3]), pack_fp8<false>(y[4], y[5], y[6], y[7]));
            if (l16 == 0) sA[t * KB + kb] = E8 ? (El)s.code() : (El)s.scale();
        }
        __syncthreads();
    }

    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = wave; k0 < KB; k0 += kU * NW) {
        if (!FUSED)
#pragma unroll
            for (int u = 0; u < kU; ++u) fetch_a(u, k0 + u * NW);
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int kb = k0 + u * NW;
            if (kb >= KB) break;
            const Block w = f[u];
            if (FUSED) fetch_a(0, kb);
            constexpr int kStep = FUSED ? 0 : 1;
            const int v = u * kStep;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if (E8) {
                    acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.w, a[v][t], acc[t], 0, AF, 0, (int)w.s, 0,
                                                                             (int)sa[v][t]);
                } else {
                    const f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        w.w, a[v][t], f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, AF, 0, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[t][e] = __builtin_fmaf(p[e], (float)sa[v][t] * (TILED ? (float)w.s : w.s4[e]), acc[t][e]);
                }
            }
        }
        if (k0 + kU * NW < KB)
#pragma unroll
            for (int u = 0; u < kU; ++u) fetch(f[u], k0 + (kU + u) * NW);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 64; i += 64 * NW) {
        const int t = i >> 6, l = i & 63, m = 16 * t + (l & 15);
        f32x4 v = sums[0][t][l];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += sums[w][t][l];
        if (m < g.M) store4<OUT_BF16>(g.c, m, n0 + 4 * (l >> 4), g.N, v);
    }
}

template <bool FUSED>
hipError_t launch(const SkinnyArgs& g, bool e5m2, bool tiled, bool e8, bool c_bf16, hipStream_t s) {
    const int mt = (g.M + 15) / 16;
    const unsigned grid = (unsigned)((g.N + 15) / 16);
    const size_t dyn = FUSED ? (size_t)g.M * (g.KB * 128 + 16) + (size_t)g.M * g.KB * 4 : 0;
    using Y = std::true_type;
    using F = std::false_type;
    auto with = [](bool v, auto&& f) { return v ? f(Y{}) : f(F{}); };
    return with(e8, [&](auto e) {
        return with(c_bf16, [&](auto bf) {
            auto go = [&](auto nw, auto m, auto af, auto tl) {
                constexpr int kNW = decltype(nw)::value;
                hipLaunchKernelGGL((gemm_fp8_skinny_kernel<kNW, decltype(m)::value, decltype(af)::value,
                                                           decltype(e)::value, decltype(tl)::value, FUSED,
                                                           decltype(bf)::value>),
                                   dim3(grid), dim3(64 * kNW), dyn, s, g);
                return hipGetLastError();
            };
            // waves: at least four blocks of the contraction each
            auto waves = [&](auto m, auto af, auto tl) {
                if (g.KB >= 64) return go(std::integral_constant<int, 16>{}, m, af, tl);
                if (g.KB >= 16) return go(std::integral_constant<int, 8>{}, m, af, tl);
                return go(std::integral_constant<int, 4>{}, m, af, tl);
            };
            if constexpr (FUSED) {
                return waves(std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{}, Y{});
            } else {
                return with(tiled, [&](auto tl) {
                    return with(e5m2, [&](auto af) {
                        std::integral_constant<int, decltype(af)::value ? 1 : 0> fmt;
                        if (mt == 1) return waves(std::integral_constant<int, 1>{}, fmt, tl);
                        if (mt == 2) return waves(std::integral_constant<int, 2>{}, fmt, tl);
                        return waves(std::integral_constant<int, 4>{}, fmt, tl);
                    });
                });
            }
        });
    });
}

}  // namespace

bool fp8_skinny(int64_t M, int64_t K) { return M <= 64 && K > 0; }

hipError_t launch_gemm_fp8_skinny(int64_t M, int64_t N, int64_t K, const uint8_t* a, const void* as, Fp8 a_fmt,
                                  const uint8_t* b, const void* bs, bool tiled, bool e8, void* c, bool c_bf16,
                                  hipStream_t s) {
    const SkinnyArgs g{a, as, b, bs, c, N, (int)M, (int)K, (int)((K + 127) / 128)};
    return launch<false>(g, a_fmt == Fp8::E5M2, tiled, e8, c_bf16, s);
}

bool fp8_fused(int64_t T, int64_t K) { return K > 0 && T <= 16 && T * ((K + 127) / 128 * 128) <= kFusedBytes; }

hipError_t launch_linear_fp8_fused(const void* x, int64_t T, int64_t K, int64_t N, const uint8_t* w, const void* ws,
                                   bool e8, void* y, bool y_bf16, hipStream_t s) {
    const SkinnyArgs g{(const uint8_t*)x, nullptr, w, ws, y, N, (int)T, (int)K, (int)((K + 127) / 128)};
    return launch<true>(g, false, true, e8, y_bf16, s);
}

}  // namespace ue5m3
