// The 8-bit product for few rows of A (up to 64: tokens being decoded): every
// weight is read once, so this is as fast as HBM gives B.  The products are the
// instruction of the 128 x 128 tiles, which truncates (see fp8_gemm.hip).
//
// A workgroup takes 16 rows of B at a time and splits the contraction over its
// waves.  Each wave streams its own blocks through a ring of stages in LDS: whole
// 128-byte lines of 16 rows of B (and of the rows of A, from the L2) by direct
// loads, chunk c of row r at c ^ (r % 8).  (Loaded straight into the registers
// that the products take, a lane a row, each load touches 16 lines and the
// address unit is what bounds: 24 x 21504 x 4096 33 us.)  Workgroups are
// persistent: the ring runs on over the rows of B that they take next, so the
// waves' sums, which meet in LDS, and the stores overlap loads.
//
// FUSED: A is bf16, a few thousand elements in all, and every workgroup
// quantizes it for itself, into LDS, while its first weights are on their way:
// one launch, and nothing to wait for, instead of two (1 x 6144 x 4096 9.3 us, two
// launches 11.5; 1 x 3408 x 1360 4.4 and 6.0; but 4 x 6144 x 4096 12.7 and 10.7).
//
// Out of HBM: 1 x 6144 x 4096 9.4 - 10.3 us (2.5 - 2.7 TB/s: a wave holds six blocks,
// and the start and the sums are half of the time), 24 x 21504 x 4096 24 - 27 us (3.3 -
// 3.7 TB/s); a large copy reaches 5.2 TB/s.
#include <algorithm>
#include <atomic>

#include "fp8.hpp"
#include "fp8_tile.hpp"
#include "gemm_regs.hpp"
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kFusedBytes = 8192;               // quantized tokens that a workgroup keeps

struct SkinnyArgs {
    const uint8_t* a;                            // payload, or bf16 tokens (FUSED)
    const void* as;
    const uint8_t* b;
    const void* bs;
    void* c;
    int64_t N;
    int M, K, KB;
};

__device__ __forceinline__ i32x4_t rsrc_of(uint64_t at, uint32_t bytes) {
    return i32x4_t{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}

// Stages of a wave's ring (the LDS holds one workgroup of NW waves, or two).
template <int MT, bool FUSED>
constexpr int kRing = FUSED ? 6 : MT == 1 ? 4 : MT == 2 ? 5 : 3;

// Bytes of a stage: 16 rows of B, 16 MT of A, 64 scales of each.
template <int MT, bool FUSED>
constexpr int kStageBytes = 2048 + 256 + (FUSED ? 0 : MT * 2048 + 256);

template <int NW, int MT, int AF, bool E8, bool TILED, bool FUSED, bool OUT_BF16>
__global__ __launch_bounds__(64 * NW) void gemm_fp8_skinny_kernel(const SkinnyArgs g) {
    constexpr int kR = kRing<MT, FUSED>, kStage = kStageBytes<MT, FUSED>;
    constexpr int kScaleB = 2048 + (FUSED ? 0 : MT * 2048), kScaleA = kScaleB + 256;   // within a stage, after the rows
    constexpr int kLoads = 3 + (FUSED ? 0 : 2 * MT + 1);
    extern __shared__ __attribute__((aligned(16))) uint8_t dyn[];    // rings, sums, then FUSED: payload rows, scales
    uint8_t* const ring = dyn + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (kR * kStage);
    f32x4* const sums = reinterpret_cast<f32x4*>(dyn + NW * kR * kStage);     // [NW][MT][64]
    uint8_t* const sQ = dyn + NW * (kR * kStage + MT * 1024);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q = lane >> 4, KB = g.KB;
    const uint32_t Kp = (uint32_t)KB * 128u;
    const int row = (int)Kp + 16;                // FUSED: bytes of a payload row in LDS
    using El = std::conditional_t<E8, uint8_t, float>;
    constexpr uint32_t kEl = sizeof(El);
    El* const sA = (El*)(sQ + g.M * row);

    // The wave's blocks: wave, wave + NW, ... of each tile of 16 rows of B that
    // the workgroup takes; the cursor of the loads runs kR of them ahead.
    const int tiles = (int)((g.N + 15) / 16), grid = (int)gridDim.x;
    const uint64_t b = uniform64((uint64_t)(uintptr_t)g.b), bs = uniform64((uint64_t)(uintptr_t)g.bs);
    const uint64_t as = uniform64((uint64_t)(uintptr_t)g.as);
    const uint64_t pb = uniform64((uint64_t)scale_pitch(g.N) * kEl), pa = uniform64((uint64_t)scale_pitch(g.M) * kEl);
    const i32x4_t srcA = rsrc_of(uniform64((uint64_t)(uintptr_t)g.a), (uint32_t)g.M * Kp);
    // row 8h + lane / 8, chunk lane % 8: voff of load h is this + 8h rows, less its immediate offset
    const uint32_t voff = (uint32_t)(lane >> 3) * Kp + (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
    const uint32_t half = 8u * Kp - 1024u;
    const uint32_t lds = lds_addr(ring);
    const uint32_t arow = (uint32_t)min(lane, g.M - 1) * kEl;
    i32x4_t srcB;
    uint32_t brow = 0;
    uint64_t bsat = 0;
    // (a wave without a block of its own, KB < NW, runs one that counts for nothing)
    const bool idle = wave >= KB;
    const int first = idle ? 0 : wave;
    int lt = (int)blockIdx.x, lb = first;
    auto enter = [&]() {
        const int64_t n0 = (int64_t)lt * 16, left = g.N - n0;
        srcB = rsrc_of(uniform64(b + (uint64_t)n0 * Kp), (uint32_t)(left < 16 ? left : 16) * Kp);
        brow = TILED ? 0u : (uint32_t)min((int64_t)l16, left - 1) * kEl;
        bsat = uniform64(bs + (uint64_t)(TILED ? n0 / 128 * KB : n0) * kEl);
    };
    auto load = [&](int slot) {                  // the cursor's block, and on
        const uint32_t so = (uint32_t)lb * 128u, to = lds + (uint32_t)(slot * kStage);
        dma_rows<0>(srcB, voff, so, to);
        dma_rows<1024>(srcB, voff + half, so, to);
        if (!FUSED) {
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                dma_rows<0>(srcA, voff + t * 16u * Kp, so, to + 2048u + t * 2048u);
                dma_rows<1024>(srcA, voff + t * 16u * Kp + half, so, to + 2048u + t * 2048u);
            }
        }
        dma_scale<E8>(rsrc_of(bsat + (uint64_t)lb * (TILED ? kEl : pb), 64 * kEl), brow, to + kScaleB);
        if (!FUSED) dma_scale<E8>(rsrc_of(as + (uint64_t)lb * pa, 64 * kEl), arow, to + kScaleA);
        if (lb + NW < KB) {
            lb += NW;
        } else if (lt + grid < tiles) {          // past the last block the cursor stays on it
            lt += grid;
            lb = first;
            enter();
        }
    };
    enter();
#pragma unroll
    for (int s = 0; s < kR; ++s) load(s);

    if constexpr (FUSED) {
        const bf16* const x = (const bf16*)g.a;
        for (int blk = threadIdx.x >> 4; blk < g.M * KB; blk += 4 * NW) {
            const int t = blk / KB, kb = blk - t * KB, k = kb * 128 + l16 * 8;
            const Vec8<bf16> v = load8(x + (int64_t)t * g.K, k, g.K);
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v.get(e)));
            const BlockScale<E8> s = BlockScale<E8>::of(row16_max(m), false);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = s.value(v.get(e));
            *reinterpret_cast<uint2*>(sQ + t * row + k) =
                make_uint2(pack_fp8<false>(y[0], y[1], y[2], y[3]), pack_fp8<false>(y[4], y[5], y[6], y[7]));
            if (l16 == 0) sA[t * KB + kb] = E8 ? (El)s.code() : (El)s.scale();
        }
        __syncthreads();
    }

    // A lane's row l16, chunks q and q + 4 (which k they are does not matter as
    // long as both operands agree).
    const int c0 = l16 * 128 + ((q ^ (l16 & 7)) * 16), c1 = l16 * 128 + (((q + 4) ^ (l16 & 7)) * 16);
    auto frag = [&](const uint8_t* p, int lo_at, int hi_at) {
        const uint4 lo = *reinterpret_cast<const uint4*>(p + lo_at), hi = *reinterpret_cast<const uint4*>(p + hi_at);
        return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };
    int slot = 0;
    for (int tile = (int)blockIdx.x; tile < tiles; tile += grid) {
        f32x4 acc[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int kb = first; kb < (idle ? 1 : KB); kb += NW) {
            // this block has landed (stores that are still out only make it wait longer)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads * (kR - 1)) : "memory");
            const uint8_t* const st = ring + slot * kStage;
            const i32x8 w = frag(st, c0, c1);
            i32x8 a[MT];
            int ea[MT], eb = 0;
            float fa[MT];
            f32x4 fb;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int m = min(16 * t + l16, g.M - 1);
                a[t] = FUSED ? frag(sQ + m * row + kb * 128, q * 16, q * 16 + 64) : frag(st + 2048 + t * 2048, c0, c1);
                if (E8) ea[t] = FUSED ? (int)sA[m * KB + kb] : *reinterpret_cast<const int*>(st + kScaleA + (16 * t + l16) * 4);
                else fa[t] = FUSED ? (float)sA[m * KB + kb] : *reinterpret_cast<const float*>(st + kScaleA + (16 * t + l16) * 4);
            }
            if (E8) {
                eb = *reinterpret_cast<const int*>(st + kScaleB + (TILED ? 0 : l16) * 4);
            } else if (TILED) {
                const float v = *reinterpret_cast<const float*>(st + kScaleB);
                fb = f32x4{v, v, v, v};
            } else {
                fb = *reinterpret_cast<const f32x4*>(st + kScaleB + 16 * q);
            }
            // read, before the next block takes this slot
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            load(slot);
            slot = slot + 1 == kR ? 0 : slot + 1;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if (E8) {
                    acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a[t], acc[t], 0, AF, 0, eb, 0, ea[t]);
                } else {
                    const f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        w, a[t], f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, AF, 0, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][e] = __builtin_fmaf(p[e], fa[t] * fb[e], acc[t][e]);
                }
            }
        }
        // The last product may be read 12 states after its issue; across the loop's
        // branch the compiler leaves five.
        if (E8) asm volatile("s_nop 11" ::: "memory");
#pragma unroll
        for (int t = 0; t < MT; ++t) sums[(wave * MT + t) * 64 + lane] = acc[t];
        __syncthreads();
        const int waves = min(NW, KB);
        for (int i = threadIdx.x; i < MT * 64; i += 64 * NW) {
            const int t = i >> 6, l = i & 63, m = 16 * t + (l & 15);
            f32x4 v = sums[t * 64 + l];
            for (int u = 1; u < waves; ++u) v += sums[(u * MT + t) * 64 + l];
            if (m < g.M) store4<OUT_BF16>(g.c, m, (int64_t)tile * 16 + 4 * (l >> 4), g.N, v);
        }
        __syncthreads();                         // before the next tile's sums
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load outlives the kernel's LDS
}

template <bool FUSED>
hipError_t launch(const SkinnyArgs& g, int cus, bool e5m2, bool tiled, bool e8, bool c_bf16, hipStream_t s) {
    const int mt = (g.M + 15) / 16;
    const int64_t tiles = (g.N + 15) / 16;
    using Y = std::true_type;
    using F = std::false_type;
    auto with = [](bool v, auto&& f) { return v ? f(Y{}) : f(F{}); };
    return with(e8, [&](auto e) {
        return with(c_bf16, [&](auto bf) {
            auto go = [&](auto nw, auto m, auto af, auto tl) {
                constexpr int kNW = decltype(nw)::value, kM = decltype(m)::value;
                auto* const kernel = gemm_fp8_skinny_kernel<kNW, kM, decltype(af)::value, decltype(e)::value,
                                                            decltype(tl)::value, FUSED, decltype(bf)::value>;
                const size_t lds = kNW * (kRing<kM, FUSED> * kStageBytes<kM, FUSED> + kM * 1024) +
                                   (FUSED ? (size_t)g.M * (g.KB * 128 + 16) + (size_t)g.M * g.KB * 4 : 0);
                static std::atomic<bool> set[64];    // per device, the kernel's LDS limit
                int dev = 0;
                hipError_t err = hipGetDevice(&dev);
                if (err != hipSuccess) return err;
                if (dev < 0 || dev >= 64 || !set[dev].load(std::memory_order_acquire)) {
                    err = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
                    if (err != hipSuccess) return err;
                    if (dev >= 0 && dev < 64) set[dev].store(true, std::memory_order_release);
                }
                const int64_t most = cus * std::max<int64_t>(1, 160 * 1024 / (int64_t)lds);
                hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(tiles, most)), dim3(64 * kNW), lds, s, g);
                return hipGetLastError();
            };
            auto waves = [&](auto m, auto af, auto tl) {
                // Four waves, so that a CU holds two workgroups of 16 rows of A (16 x 21504
                // x 4096 23.6 us, eight waves 24.9); eight where there is not a tile for
                // every CU and each of them still has blocks enough (1 x 4096 x 16384 19,
                // four 21; but 16 x 4096 x 1024 6.5, four 5.6).
                if constexpr (decltype(m)::value == 1)
                    if (tiles <= cus && g.KB >= 32) return go(std::integral_constant<int, 8>{}, m, af, tl);
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

hipError_t launch_gemm_fp8_skinny(int64_t M, int64_t N, int64_t K, int cus, const uint8_t* a, const void* as, Fp8 a_fmt,
                                  const uint8_t* b, const void* bs, bool tiled, bool e8, void* c, bool c_bf16,
                                  hipStream_t s) {
    const SkinnyArgs g{a, as, b, bs, c, N, (int)M, (int)K, (int)((K + 127) / 128)};
    return launch<false>(g, cus, a_fmt == Fp8::E5M2, tiled, e8, c_bf16, s);
}

bool fp8_fused(int64_t T, int64_t K) { return K > 0 && T <= 16 && T * ((K + 127) / 128 * 128) <= kFusedBytes; }

hipError_t launch_linear_fp8_fused(const void* x, int64_t T, int64_t K, int64_t N, const uint8_t* w, const void* ws,
                                   bool e8, void* y, bool y_bf16, hipStream_t s) {
    const SkinnyArgs g{(const uint8_t*)x, nullptr, w, ws, y, N, (int)T, (int)K, (int)((K + 127) / 128)};
    int cus = 0;
    const hipError_t e = device_cus(&cus);
    if (e != hipSuccess) return e;
    return launch<true>(g, cus, false, true, e8, y_bf16, s);
}

}  // namespace ue5m3
