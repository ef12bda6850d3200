// C[m, n] = sum over blocks k of sa sb sum over the block of a b: operands in
// 8-bit floating point, rows of whole blocks of 128 along the contraction, one
// scale for each block of a row of A and for each block of a row (1D) or of
// 128 rows (tiles) of B.
//
// v_mfma_f32_16x16x128_f8f6f4 takes one whole block of 16 rows of each
// operand.  With E8M0 scales the instruction applies them (one byte a row) and
// accumulates in place; with binary32 scales its result starts from zero and
// sa sb times it is added to the accumulators, in binary32.  The products are
// issued as B x A^T: a lane then holds four consecutive columns n of one row m,
// so sa is one value a lane.
#include "fp8.hpp"
#include "gemm_regs.hpp"
#include "launch.hpp"

namespace ue5m3 {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 128, kRowBytes = 128, kStage = 2 * kTile * kRowBytes;

// A lane's 32 bytes of row `row`: chunks g and g + 4 of eight, which lie at
// their number XOR row % 8.  Which k they are does not matter as long as both
// operands agree.
__device__ __forceinline__ i32x8 read_frag(const uint8_t* rows, int row, int g) {
    const uint8_t* p = rows + row * kRowBytes;
    const uint4 lo = *reinterpret_cast<const uint4*>(p + ((g ^ (row & 7)) * 16));
    const uint4 hi = *reinterpret_cast<const uint4*>(p + (((g + 4) ^ (row & 7)) * 16));
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

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

// 128 x 128 output tiles, four waves of 64 x 64, two stages of one block each.
template <int AF, bool E8, bool TILED, bool OUT_BF16>
__global__ __launch_bounds__(256, 2) void gemm_fp8_kernel(int64_t M, int64_t N, int64_t KB, int64_t tiles_n,
                                                          const uint8_t* __restrict__ A, const void* __restrict__ As,
                                                          const uint8_t* __restrict__ B, const void* __restrict__ Bs,
                                                          void* __restrict__ C) {
    __shared__ __attribute__((aligned(16))) uint8_t sP[2 * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, g = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x / tiles_n * kTile, n0 = (int64_t)blockIdx.x % tiles_n * kTile;
    const uint32_t Kp = (uint32_t)KB * 128u;

    // waves 0, 1 bring A rows, waves 2, 3 B rows: 64 rows each, 8 rows a load
    const bool isA = wave < 2;
    const int64_t left = isA ? M - m0 : N - n0;
    const i32x4_t src = buffer_rsrc(isA ? A + m0 * Kp : B + n0 * Kp, (uint32_t)(left < kTile ? left : kTile) * Kp);
    const uint32_t voff = (uint32_t)(64 * (wave & 1) + (lane >> 3)) * Kp + (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
    const uint32_t lds = lds_addr(sP) + (uint32_t)wave * 64u * kRowBytes;
    auto load = [&](int64_t kb, int buf) {
        const uint32_t vo = voff + (uint32_t)kb * 128u, to = lds + (uint32_t)(buf * kStage);
        static_for<0, 8>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            dma_buf_x4<i * 1024>(src, vo + i * 8 * Kp, 0u, to);
        });
    };

    const int64_t pa = scale_pitch(M), pb = scale_pitch(N), nb = n0 / 128;
    float fa[4], fb[E8 || TILED ? 1 : 16];
    int ea[4], eb[4];
    auto scales = [&](int64_t kb) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t m = min(m0 + wm * 64 + 16 * i + l16, M - 1);
            if (E8) ea[i] = ((const uint8_t*)As)[kb * pa + m];
            else fa[i] = ((const float*)As)[kb * pa + m];
        }
        if (TILED) {
            if (E8) eb[0] = ((const uint8_t*)Bs)[nb * KB + kb];
            else fb[0] = ((const float*)Bs)[nb * KB + kb];
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (E8) {
                eb[j] = ((const uint8_t*)Bs)[kb * pb + min(n0 + wn * 64 + 16 * j + l16, N - 1)];
            } else {
                const float4 v = *reinterpret_cast<const float4*>((const float*)Bs + kb * pb +
                                                                  min(n0 + wn * 64 + 16 * j + 4 * g, pb - 4));
                fb[4 * j] = v.x; fb[4 * j + 1] = v.y; fb[4 * j + 2] = v.z; fb[4 * j + 3] = v.w;
            }
        }
    };

    f32x4 acc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    if (KB > 0) load(0, 0);
    for (int64_t kb = 0; kb < KB; ++kb) {
        // this stage has landed everywhere and every wave has left the other
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        scales(kb);
        if (kb + 1 < KB) load(kb + 1, (int)(kb + 1) & 1);
        const uint8_t* const rows = sP + ((int)kb & 1) * kStage;
        i32x8 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = read_frag(rows, wm * 64 + 16 * i + l16, g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const i32x8 b = read_frag(rows, kTile + wn * 64 + 16 * j + l16, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (E8) {
                    acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a[i], acc[j][i], 0, AF, 0,
                                                                                eb[TILED ? 0 : j], 0, ea[i]);
                } else {
                    const f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        b, a[i], f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, AF, 0, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[j][i][e] = __builtin_fmaf(p[e], fa[i] * fb[TILED ? 0 : 4 * j + e], acc[j][i][e]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + wm * 64 + 16 * i + l16;
        if (m >= M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) store4<OUT_BF16>(C, m, n0 + wn * 64 + 16 * j + 4 * g, N, acc[j][i]);
    }
}

}  // namespace

hipError_t launch_gemm_fp8(int64_t M, int64_t N, int64_t K, const uint8_t* a, const void* as, Fp8 a_fmt,
                           const uint8_t* b, const void* bs, bool tiled, bool e8, void* c, bool c_bf16,
                           hipStream_t s) {
    const int64_t KB = (K + 127) / 128, tm = (M + kTile - 1) / kTile, tn = (N + kTile - 1) / kTile;
    auto go = [&](auto af, auto e, auto tl, auto bf) {
        hipLaunchKernelGGL((gemm_fp8_kernel<decltype(af)::value, decltype(e)::value, decltype(tl)::value, decltype(bf)::value>),
                           dim3((unsigned)(tm * tn)), dim3(256), 0, s, M, N, KB, tn, a, as, b, bs, c);
        return hipGetLastError();
    };
    using Y = std::true_type;
    using F = std::false_type;
    auto with = [](bool v, auto&& f) { return v ? f(Y{}) : f(F{}); };
    return with(a_fmt == Fp8::E5M2, [&](auto af) {
        return with(e8, [&](auto e) {
            return with(tiled, [&](auto tl) { return with(c_bf16, [&](auto bf) { return go(af, e, tl, bf); }); });
        });
    });
}

hipError_t launch_linear_fp8(const void* x, int64_t T, int64_t K, int64_t N, const uint8_t* w, const void* ws,
                             bool e8, void* y, bool y_bf16, hipStream_t s) {
    const int64_t KB = (K + 127) / 128;
    const size_t payload = (size_t)(T * KB * 128), scales = (size_t)(KB * scale_pitch(T)) * (e8 ? 1 : 4);
    Workspace held;                                  // until the product is enqueued
    uint8_t* q = nullptr;
    hipError_t e = hipSuccess;
    if (K > 0) {
        e = held.take(kWsTokens, s, payload + scales, (void**)&q);
        if (e == hipSuccess)
            e = launch_quant_fp8(DType::BF16, Fp8::E4M3, e8, x, T, K, q, q + payload, nullptr, nullptr, s);
        if (e != hipSuccess) return e;
    }
    return launch_gemm_fp8(T, N, K, q, q + payload, Fp8::E4M3, w, ws, true, e8, y, y_bf16, s);
}

}  // namespace ue5m3
