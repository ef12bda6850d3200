// Quantizers to 8-bit floating point (OCP E4M3 or E5M2) with one scale for
// each block of 128: along the rows, down the columns (stored transposed),
// both from one read, or in 128 x 128 tiles with the transposed copy.
//
// With a the largest finite magnitude of a block and F the format's largest
// value (448, 57344):
//   F32 scales:   a' = max(a, F 2^-126), scale = a' / F, value = x F / a'
//   E8M0 scales:  the least power of two p >= a / F, 2^-126 at least, value = x / p
//   a = 0:        scale 1
// each value rounded to the nearest of the format's, ties to even.  The
// quotient of the first line is taken to the last bit (one correction of
// x F times 1 / a'): 16-bit inputs hit exact ties often, and a product with a
// rounded reciprocal would send half of those the wrong way.  An infinity or
// a NaN becomes a NaN of the format and leaves its block's scale alone.
//
// Bound: HBM (2 bytes read, 1 written for each blocking).  A workgroup holds
// one 128 x 128 tile in registers, 8 x 8 elements a thread, so that every block
// of either direction ends inside it: a row's block is 16 lanes (DPP), a
// column's 16 threads of four waves (LDS).  The transposed bytes pass through
// 16 KB of LDS, 8-byte chunk k of column c at k ^ (c / 8 % 16), and leave as
// whole 128-byte rows.  Rows alone need no tile: their kernel gives a block to
// 16 lanes, so that few rows still spread over many waves.
//
// 8192 x 21504 both ways 144 - 152 us (4.6 - 4.9 TB/s; a large copy 5.2), 8192 x 4096 30
// (4.5), tiles with the transposed copy of 21504 x 4096 61 (5.8); 1999 x 3408 both ways
// 14 - 15 (1.8 - 2.0: 432 workgroups, a tile each, with nothing behind them).
#include "codec.hpp"
#include "fp8.hpp"
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kThreads = 256;

// Which outputs a launch writes.
enum class Form : int { Rows, Cols, Dual, Tiles, TilesT };   // Rows: a kernel of its own

struct QuantOut {
    uint8_t *rows, *cols;                            // payloads [R][pad(C)], [C][pad(R)]
    void *rows_scale, *cols_scale;                   // [C / 128][pitch(R)], [R / 128][pitch(C)], or the tiles'
};

template <bool E8>
__device__ __forceinline__ void put_scale(void* p, int64_t i, const BlockScale<E8>& s) {
    if (E8)
        ((uint8_t*)p)[i] = (uint8_t)s.code();
    else
        ((float*)p)[i] = s.scale();
}

template <typename T, bool E5M2, bool E8, Form F>
__global__ __launch_bounds__(kThreads) void quant_fp8_kernel(const T* __restrict__ x, int64_t R, int64_t C,
                                                             int64_t blocks_c, QuantOut out) {
    constexpr bool kRows = F == Form::Dual, kCols = F == Form::Cols || F == Form::Dual;
    constexpr bool kTiles = F == Form::Tiles || F == Form::TilesT, kT = kCols || F == Form::TilesT;
    __shared__ float smax[5][128];                   // columns of the four waves, rows
    __shared__ float4 sPar[kCols ? 2 : 1][kTiles ? 1 : 128];   // what rows and columns are divided by
    __shared__ __attribute__((aligned(16))) uint8_t sT[kT ? 128 * 128 : 16];
    const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wave = t >> 6;
    const int64_t br = (int64_t)blockIdx.x / blocks_c, bc = (int64_t)blockIdx.x % blocks_c;
    const int64_t r0 = br * 128 + rg * 8, c0 = bc * 128 + cg * 8;
    const int64_t Cp = blocks_c * 128, Rp = (R + 127) / 128 * 128;

    Vec8<T> v[8];
    if (C >= 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = load8_row(x + min(r0 + i, R - 1) * C, (int)c0, (int)C);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < Vec8<T>::kWords; ++k) v[i].w[k] = r0 + i < R ? v[i].w[k] : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = load8(x + (r0 + i) * C, c0, r0 + i < R ? C : 0);
    }

    float rmax[8], cmax[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        rmax[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = finite_abs(v[i].get(j));
            rmax[i] = fmaxf(rmax[i], a);
            if (kCols) cmax[j] = fmaxf(cmax[j], a);
        }
    }

    BlockScale<E8> tile;
    if (kTiles) {
        float a = rmax[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) a = fmaxf(a, rmax[i]);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) a = fmaxf(a, __shfl_xor(a, off));
        if ((t & 63) == 0) smax[0][wave] = a;
        __syncthreads();
        a = fmaxf(fmaxf(smax[0][0], smax[0][1]), fmaxf(smax[0][2], smax[0][3]));
        tile = BlockScale<E8>::of(a, E5M2);
        if (t == 0) {
            put_scale(out.rows_scale, br * blocks_c + bc, tile);
            if (kT) put_scale(out.cols_scale, bc * (Rp / 128) + br, tile);
        }
    }
    if (!kTiles) {
        // One thread works out the scale of each row and of each column (a
        // division or two: too dear for every thread to do its sixteen).
        if (kRows) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = row16_max(rmax[i]);
                if (cg == i) smax[4][rg * 8 + i] = a;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float a = cmax[j];
            a = fmaxf(a, __shfl_xor(a, 16));
            cmax[j] = fmaxf(a, __shfl_xor(a, 32));
        }
        if ((t & 63) < 16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) smax[wave][cg * 8 + j] = cmax[j];
        }
        __syncthreads();
        const int i = t & 127;
        if (t < 128) {
            const BlockScale<E8> s =
                BlockScale<E8>::of(fmaxf(fmaxf(smax[0][i], smax[1][i]), fmaxf(smax[2][i], smax[3][i])), E5M2);
            sPar[0][i] = s.pack();
            if (bc * 128 + i < C) put_scale(out.cols_scale, br * scale_pitch(C) + bc * 128 + i, s);
        } else if (kRows) {
            const BlockScale<E8> s = BlockScale<E8>::of(smax[4][i], E5M2);
            sPar[kCols ? 1 : 0][i] = s.pack();
            if (br * 128 + i < R) put_scale(out.rows_scale, bc * scale_pitch(R) + br * 128 + i, s);
        }
        __syncthreads();
    }
    if (kRows || kTiles) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            forget(v[i]);
            const BlockScale<E8> s = kTiles ? tile : BlockScale<E8>::unpack(sPar[kCols ? 1 : 0][kTiles ? 0 : rg * 8 + i]);
            if (r0 + i < R) {
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = s.value(v[i].get(j));
                const uint2 w = make_uint2(pack_fp8<E5M2>(q[0], q[1], q[2], q[3]), pack_fp8<E5M2>(q[4], q[5], q[6], q[7]));
                *reinterpret_cast<uint2*>(out.rows + (r0 + i) * Cp + c0) = w;
            }
        }
    }
    if (!kT) return;
    // (converted again: kept as numbers the tile takes twice the registers)
#pragma unroll
    for (int i = 0; i < 8; ++i) forget(v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const BlockScale<E8> s = kTiles ? tile : BlockScale<E8>::unpack(sPar[0][kTiles ? 0 : cg * 8 + j]);
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = s.value(v[i].get(j));
        *reinterpret_cast<uint2*>(sT + (cg * 8 + j) * 128 + ((rg ^ cg) & 15) * 8) =
            make_uint2(pack_fp8<E5M2>(q[0], q[1], q[2], q[3]), pack_fp8<E5M2>(q[4], q[5], q[6], q[7]));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int col = k * 32 + (t >> 3), q = t & 7, sw = (col >> 3) & 15;
        uint4 w = *reinterpret_cast<const uint4*>(sT + col * 128 + ((2 * q ^ sw) & 14) * 8);
        if (sw & 1) w = make_uint4(w.z, w.w, w.x, w.y);
        if (bc * 128 + col < C)
            *reinterpret_cast<uint4*>(out.cols + (bc * 128 + col) * Rp + br * 128 + q * 16) = w;
    }
}

// Row blocks alone: 16 lanes a block, one block a thread group, so that a few
// rows still spread over many waves.  A workgroup takes 16 rows of one block
// column (the rows' scales are neighbours).
template <typename T, bool E5M2, bool E8>
__global__ __launch_bounds__(kThreads) void quant_fp8_rows_kernel(const T* __restrict__ x, int64_t R, int64_t C,
                                                                  int64_t blocks_c, uint8_t* __restrict__ out,
                                                                  void* __restrict__ scales) {
    const int t = threadIdx.x & 15;
    const int64_t br = (int64_t)blockIdx.x / blocks_c, bc = (int64_t)blockIdx.x % blocks_c;
    const int64_t r = br * 16 + (threadIdx.x >> 4), c = bc * 128 + t * 8;
    const Vec8<T> v = load8(x + r * C, c, r < R ? C : 0);
    float a = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) a = fmaxf(a, finite_abs(v.get(j)));
    const BlockScale<E8> s = BlockScale<E8>::of(row16_max(a), E5M2);
    if (r >= R) return;
    float q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = s.value(v.get(j));
    *reinterpret_cast<uint2*>(out + r * (blocks_c * 128) + c) =
        make_uint2(pack_fp8<E5M2>(q[0], q[1], q[2], q[3]), pack_fp8<E5M2>(q[4], q[5], q[6], q[7]));
    if (t == 0) put_scale(scales, bc * scale_pitch(R) + r, s);
}

template <Form F>
hipError_t launch(DType type, bool e5m2, bool e8, const void* x, int64_t R, int64_t C, const QuantOut& out,
                  hipStream_t s) {
    const int64_t bc = (C + 127) / 128, br = (R + 127) / 128;
    return with_type(type, [&](auto* tp) {
        using T = std::remove_pointer_t<decltype(tp)>;
        auto go = [&](auto f5, auto f8) {
            if constexpr (F == Form::Rows)
                hipLaunchKernelGGL((quant_fp8_rows_kernel<T, decltype(f5)::value, decltype(f8)::value>),
                                   dim3((unsigned)((R + 15) / 16 * bc)), dim3(kThreads), 0, s, (const T*)x, R, C, bc,
                                   out.rows, out.rows_scale);
            else
                hipLaunchKernelGGL((quant_fp8_kernel<T, decltype(f5)::value, decltype(f8)::value, F>),
                                   dim3((unsigned)(br * bc)), dim3(kThreads), 0, s, (const T*)x, R, C, bc, out);
            return hipGetLastError();
        };
        using Y = std::true_type;
        using N = std::false_type;
        if (e5m2) return e8 ? go(Y{}, Y{}) : go(Y{}, N{});
        return e8 ? go(N{}, Y{}) : go(N{}, N{});
    });
}

}  // namespace

hipError_t launch_quant_fp8(DType type, Fp8 fmt, bool e8, const void* x, int64_t R, int64_t C, uint8_t* rows,
                            void* rows_scale, uint8_t* cols, void* cols_scale, hipStream_t s) {
    const QuantOut out{rows, cols, rows_scale, cols_scale};
    const bool e5 = fmt == Fp8::E5M2;
    if (cols == nullptr) return launch<Form::Rows>(type, e5, e8, x, R, C, out, s);
    if (rows == nullptr) return launch<Form::Cols>(type, e5, e8, x, R, C, out, s);
    return launch<Form::Dual>(type, e5, e8, x, R, C, out, s);
}

hipError_t launch_quant_fp8_tiles(DType type, bool e8, const void* w, int64_t R, int64_t C, uint8_t* payload,
                                  void* scales, uint8_t* payload_t, void* scales_t, hipStream_t s) {
    const QuantOut out{payload, payload_t, scales, scales_t};
    if (payload_t == nullptr) return launch<Form::Tiles>(type, false, e8, w, R, C, out, s);
    return launch<Form::TilesT>(type, false, e8, w, R, C, out, s);
}

}  // namespace ue5m3
