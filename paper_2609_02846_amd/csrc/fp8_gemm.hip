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
//
// The instruction truncates: of eight products of consecutive k each goes toward
// zero to a multiple of 2^(E - 13), E the largest sum of two exponents among
// them.  That is taken for its rate: 4e-5 to 7e-5 of the result in L2 norm on
// normal values, where the operands' own rounding is 2.6e-2 each and bf16 output's
// 1.7e-3; the 16-bit instructions, which would keep the products, have half
// the rate and want every operand converted.  All sums are binary32.
//
// Bound: in the 128 x 128 tiles a CU's 512 cycles of the matrix pipe a block stand
// against as many of the loads (32 KB at 64 bytes a cycle) and of LDS reads (64 KB at
// 128), with one wave a SIMD to issue all of it: about 1270 cycles a block.  The
// 256 x 128 tiles halve the loads of B, and two waves a SIMD fill each other's gaps:
// out of HBM, under F32 scales 8192^3 495 us (2220 TFLOP/s; 128 x 128 623), 8192 x
// 4096 x 21504 631 (778); under E8M0 2000 x 4096 x 4096 34 (43).  The small tiles
// stay for products of few tiles: 1999 x 1360 x 3408 F32 20, the large 29.
#include <algorithm>

#include "fp8.hpp"
#include "fp8_tile.hpp"
#include "gemm_regs.hpp"
#include "launch.hpp"

namespace ue5m3 {
namespace {

constexpr int kTile = 128, kRowBytes = 128;

// Output tiles of 64 WM x 128, 2 WM waves of 64 x 64 (WM = 2 or 4), a ring of
// stages of one block each.  While a wave multiplies a stage out of registers it
// reads the next one from LDS, and the stages after that are on their way: at the
// barrier that opens turn k, stage k + 1 has landed and stage k has left the LDS,
// so stage k + kRing takes its place.  Scales travel with their stage, one dword
// for each row (an E8M0 byte is loaded as one).
// (WM = 4 under one-dimensional F32 scales spills three or four registers, before
// and after the loop's full turns; what is read back makes a wait there stricter.)
template <int WM>
struct Tile {
    static constexpr int kM = 64 * WM, kThreads = 128 * WM, kRing = WM == 2 ? 4 : 3;
    static constexpr int kStage = (kM + kTile) * kRowBytes, kStageAll = kStage + 2 * WM * 256;
    static constexpr int kLoadsB = 8 / WM;           // of a wave for one stage: rows of A 4, of B, scales 1
    static constexpr int kLoads = 5 + kLoadsB;
    static constexpr int kGroup = WM == 2 ? 8 : 4;   // tile rows, see tile_of()
};

// One product from zero, into registers that a VALU instruction can read (the
// compiler's own choice are accumulation registers, from where each value is
// moved first).  It does not model this instruction: a product of 8 passes may be
// read 12 instructions later, which the callers' order keeps.
template <int AF>
__device__ __forceinline__ void product(f32x4& d, const i32x8& b, const i32x8& a) {
    if (AF == 0)
        asm volatile("v_mfma_f32_16x16x128_f8f6f4 %0, %1, %2, 0" : "=&v"(d) : "v"(b), "v"(a));
    else
        asm volatile("v_mfma_f32_16x16x128_f8f6f4 %0, %1, %2, 0 blgp:1" : "=&v"(d) : "v"(b), "v"(a));
}

// One product times 2^(eb - 127) 2^(ea - 127), added in place (see product()).
template <int AF>
__device__ __forceinline__ void accumulate(f32x4& d, const i32x8& b, const i32x8& a, int eb, int ea) {
    if (AF == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                     : "+v"(d) : "v"(b), "v"(a), "v"(eb), "v"(ea));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] blgp:1"
                     : "+v"(d) : "v"(b), "v"(a), "v"(eb), "v"(ea));
}

// Registers of one stage: a lane's share of 64 rows of each operand, and their
// scales (E8: codes; else sa of each A row and, tiled, the tile's).
template <bool E8, bool TILED>
struct Frag {
    i32x8 a[4], b[4];
    float sa[4], st;
    int ea[4], eb[4];
};

// Workgroups are dealt to the XCDs in turn: the one of each XCD's own range of
// `n` pieces of work that workgroup b takes.
__device__ __forceinline__ int xcd_order(int b, int n) {
    const int x = b % kXcds, q = n / kXcds, r = n % kXcds;
    return x * q + min(x, r) + b / kXcds;
}

// Tiles in groups of `height` tile rows, down the columns of a group: the 32 tiles
// that an XCD works on together then share 1024 rows of A and 512 or 1024 of B in
// its L2.
__device__ __forceinline__ void tile_of(int t, int height, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int group = uniform(t / (height * tiles_n)), first = group * height, rows = min(tiles_m - first, height);
    const int in = t - group * height * tiles_n;
    tn = uniform(in / rows);
    tm = first + in - tn * rows;
}

template <int WM, int AF, bool E8, bool TILED, bool OUT_BF16>
__global__ __launch_bounds__(128 * WM, 1) void gemm_fp8_kernel(int64_t M, int64_t N, int KB, int tiles_m, int tiles_n,
                                                          const uint8_t* __restrict__ A, const void* __restrict__ As,
                                                          const uint8_t* __restrict__ B, const void* __restrict__ Bs,
                                                          void* __restrict__ C, int parts, float* __restrict__ part) {
    using L = Tile<WM>;
    constexpr int kRing = L::kRing, kStage = L::kStage, kStageAll = L::kStageAll, kLoads = L::kLoads;
    __shared__ __attribute__((aligned(16))) uint8_t sP[kRing * kStageAll];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, g = lane >> 4;
    // (divisions run in vector registers: back to scalars)
    const int work = xcd_order((int)blockIdx.x, (int)gridDim.x), tiles = tiles_m * tiles_n;
    const int p = uniform(work / tiles), item = work - p * tiles;
    int tm, tn;
    tile_of(item, L::kGroup, tiles_m, tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * L::kM, n0 = (int64_t)tn * kTile;
    const int kb0 = uniform(KB * p / parts), kb1 = uniform(KB * (p + 1) / parts);
    const uint32_t Kp = (uint32_t)KB * 128u;
    constexpr uint32_t kEl = E8 ? 1 : 4;

    // a wave brings 32 rows of A and its share of B's, 8 rows a load
    const i32x4_t srcA = buffer_rsrc(A + m0 * Kp, (uint32_t)uniform((int)min(M - m0, (int64_t)L::kM)) * Kp);
    const i32x4_t srcB = buffer_rsrc(B + n0 * Kp, (uint32_t)uniform((int)min(N - n0, (int64_t)kTile)) * Kp);
    uint32_t voff[4 + L::kLoadsB];                   // of load i, less its immediate offset
#pragma unroll
    for (int i = 0; i < 4 + L::kLoadsB; ++i)
        voff[i] = (uint32_t)((i < 4 ? 32 : 8 * L::kLoadsB) * wave + 8 * (i & 3) + (lane >> 3)) * Kp +
                  (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16) - (uint32_t)((i & 3) * 1024);
    const uint32_t lds = lds_addr(sP) + (uint32_t)wave * 32u * kRowBytes;
    const uint32_t lds_b = lds_addr(sP) + (uint32_t)(L::kM + 8 * L::kLoadsB * wave) * kRowBytes;
    const uint32_t lds_s = lds_addr(sP) + kStage + wave * 256u;
    // scales of 64 rows of one operand, one row of the array a stage; of a tile, the
    // one scale (A's by the first WM waves, B's by two more, again, unused, by the rest)
    const bool isA = wave < WM, tile_scale = TILED && !isA;
    const int64_t rows = isA ? M : N, x0 = isA ? m0 : n0;
    const uint64_t sstep = uniform64((uint64_t)((tile_scale ? 1 : scale_pitch(rows)) * kEl));
    uint64_t sat = uniform64((uint64_t)(uintptr_t)(isA ? As : Bs) +       // of the stage that is loaded next
                             (uint64_t)(tile_scale ? (int64_t)tn * KB + kb0 : kb0 * scale_pitch(rows) + x0) * kEl);
    const uint32_t srow =
        tile_scale ? 0u : (uint32_t)min((int64_t)(64 * (isA ? wave : wave & 1) + lane), rows - x0 - 1) * kEl;
    // step i of stage kb's loads (8 rows each, at last the scales)
    auto load = [&](auto ic, int kb, int slot) {
        constexpr int i = decltype(ic)::value;
        const uint32_t to = (uint32_t)(slot * kStageAll);
        if constexpr (i < kLoads - 1) {
            dma_rows<(i & 3) * 1024>(i < 4 ? srcA : srcB, voff[i], (uint32_t)kb * 128u, (i < 4 ? lds : lds_b) + to);
        } else {
            dma_scale<E8>(i32x4_t{(int)(uint32_t)sat, (int)(uint32_t)(sat >> 32), (int)(L::kM * kEl), 0x00020000}, srow,
                          lds_s + to);
            sat += kb + 1 < kb1 ? sstep : 0;
        }
    };
    using F = Frag<E8, TILED>;
    // Half h of a lane's 32 bytes of row group i: chunks g and g + 4 of eight,
    // which lie at their number XOR row % 8 (which k they are does not matter
    // as long as both operands agree).  Slots 0, 1 and 2, 3 have base pointers of
    // their own: what is added to them fits the instructions' offsets.
    const uint8_t* base[2][2][2];                    // [slot pair][operand][half]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            const int at = s2 * 2 * kStageAll + ((g + 4 * h) ^ (l16 & 7)) * 16 + l16 * kRowBytes;
            base[s2][0][h] = sP + at + wm * 64 * kRowBytes;
            base[s2][1][h] = sP + at + (L::kM + wn * 64) * kRowBytes;
        }
    auto frag = [&](i32x8& f, int op, int i, int h, int slot) {
        const uint4 v = *reinterpret_cast<const uint4*>(base[slot / 2][op][h] + (slot % 2) * kStageAll + i * 16 * kRowBytes);
        f[4 * h] = (int)v.x; f[4 * h + 1] = (int)v.y; f[4 * h + 2] = (int)v.z; f[4 * h + 3] = (int)v.w;
    };
    const uint8_t* scales[2][2];                     // [slot pair][operand]
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
        scales[s2][0] = sP + s2 * 2 * kStageAll + kStage + wm * 256 + l16 * 4;
        scales[s2][1] = sP + s2 * 2 * kStageAll + kStage + (WM + wn) * 256 + (TILED ? 0 : (E8 ? l16 : 4 * g) * 4);
    }
    auto read_scales = [&](F& f, int slot) {
        const uint8_t* const a = scales[slot / 2][0] + (slot % 2) * kStageAll;
        const uint8_t* const b = scales[slot / 2][1] + (slot % 2) * kStageAll;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (E8) f.ea[i] = *reinterpret_cast<const int*>(a + i * 64);
            else f.sa[i] = *reinterpret_cast<const float*>(a + i * 64);
            if (E8 && (!TILED || i == 0)) f.eb[i] = *reinterpret_cast<const int*>(b + i * 64);
        }
        if (TILED && !E8) f.st = *reinterpret_cast<const float*>(b);
    };

    // sb of four rows for each of a lane's row groups: held once, the next stage's
    // read when the last product that takes them is added
    f32x4 sb[TILED || E8 ? 1 : 4];
    auto read_sb = [&](int j, int slot) {
        if (!E8 && !TILED)
            sb[TILED || E8 ? 0 : j] =
                *reinterpret_cast<const f32x4*>(scales[slot / 2][1] + (slot % 2) * kStageAll + j * 64);
    };

    f32x4 acc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // 16 products of stage registers f; between them the next stage is read into
    // n and the loads of stage `kb` are issued.  A binary32 product is added three
    // products later, when it has left the matrix pipe (at least 14 instructions
    // after its own, whatever else stands between them).
    auto turn = [&](F& f, F& n, int slot, int kb, int to) __attribute__((always_inline)) {
        if (TILED && !E8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f.sa[i] *= f.st;
        }
        f32x4 q[E8 ? 1 : 4];
        auto add = [&](auto xc) {
            constexpr int x = decltype(xc)::value, j = x / 4, i = x % 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[j][i][e] = __builtin_fmaf(q[E8 ? 0 : x % 4][e], TILED ? f.sa[i] : f.sa[i] * sb[TILED || E8 ? 0 : j][e], acc[j][i][e]);
        };
        read_scales(n, slot);
        static_for<0, 16>([&](auto xc) {
            constexpr int x = decltype(xc)::value, j = x / 4, i = x % 4;
            if constexpr (E8)
                accumulate<AF>(acc[j][i], f.b[j], f.a[i], f.eb[TILED ? 0 : j], f.ea[i]);
            else
                product<AF>(q[x % 4], f.b[j], f.a[i]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (x < kLoads) load(xc, kb, to);
            frag(x < 8 ? n.a[x / 2 % 4] : n.b[x / 2 % 4], x / 8, x / 2 % 4, x % 2, slot);
            if constexpr (!E8 && x == 3) {           // no additions stand before this one
                asm volatile("s_nop 5");
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (!E8 && x >= 3) add(std::integral_constant<int, x - 3>{});
            if constexpr (x >= 6 && x % 4 == 2) read_sb((x - 6) / 4, slot);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (!E8) {
            asm volatile("s_nop 11");                // the last three leave the matrix pipe
            __builtin_amdgcn_sched_barrier(0);
            add(std::integral_constant<int, 13>{});
            add(std::integral_constant<int, 14>{});
            add(std::integral_constant<int, 15>{});
            read_sb(3, slot);
        }
    };

    const int n = kb1 - kb0;
    // past the last stage that one is loaded and read again, unused, so that the
    // waits count the same loads in every turn
    if (n > 0) {
#pragma unroll
        for (int k = 0; k < kRing; ++k)
            static_for<0, kLoads>([&](auto ic) { load(ic, min(kb0 + k, kb1 - 1), k); });
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoads * (kRing - 1)) : "memory");
        F f, h;
        read_scales(f, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) read_sb(j, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            frag(f.a[i / 2], 0, i / 2, i % 2, 0);
            frag(f.b[i / 2], 1, i / 2, i % 2, 0);
        }
        auto step = [&](F& cur, F& nxt, int k, int slot) __attribute__((always_inline)) {
            // stage k + 1 has landed everywhere, every wave holds stage k
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads * (kRing - 2)) : "memory");
            turn(cur, nxt, (slot + 1) % kRing, min(kb0 + k + kRing, kb1 - 1), slot);
        };
        constexpr int kTurns = kRing % 2 ? 2 * kRing : kRing;    // an even number: f and h change places
        int k = 0;
        auto turns = [&](auto ic, int at) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            if constexpr (i % 2 == 0) step(f, h, at + i, i % kRing);
            else step(h, f, at + i, i % kRing);
        };
        for (; k + kTurns <= n; k += kTurns)
            static_for<0, kTurns>([&](auto ic) { turns(ic, k); });
        static_for<0, kTurns - 1>([&](auto ic) {
            if (k + decltype(ic)::value < n) turns(ic, k);
        });
        // no load outlives the kernel's LDS, and the last products have landed
        asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    if (parts > 1) {
        // this part's sums as [item][part][wave][j][i][lane][4]
        float* out = part + ((int64_t)item * parts + p) * (L::kM * kTile) + wave * 4096 + lane * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(out + (j * 4 + i) * 256) = acc[j][i];
        return;
    }
    // The tile goes through LDS: a lane holds four columns of one row, and whole
    // rows (256 or 512 bytes) make whole lines.
    constexpr int kEs = OUT_BF16 ? 2 : 4, kPitch = kTile * kEs + 16, kPer = 16 / kEs;   // elements of a 16-byte piece
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint8_t* const at = sP + (wm * 64 + 16 * i + l16) * kPitch + (wn * 64 + 4 * g) * kEs;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (OUT_BF16)
                *reinterpret_cast<uint2*>(at + 16 * j * kEs) =
                    make_uint2(pack_bf16x2(acc[j][i][0], acc[j][i][1]), pack_bf16x2(acc[j][i][2], acc[j][i][3]));
            else
                *reinterpret_cast<f32x4*>(at + 16 * j * kEs) = acc[j][i];
        }
    }
    __syncthreads();
    constexpr int kPieces = kTile / kPer;            // of a row
    const int c = threadIdx.x % kPieces;
    const int64_t col = n0 + c * kPer;
    if (col >= N) return;
#pragma unroll 4
    for (int r = threadIdx.x / kPieces; r < L::kM; r += L::kThreads / kPieces) {
        if (m0 + r >= M) break;
        const uint4 v = *reinterpret_cast<const uint4*>(sP + r * kPitch + c * 16);
        uint8_t* const d = (uint8_t*)C + ((m0 + r) * N + col) * kEs;
        if (col + kPer <= N) {
            __builtin_memcpy(d, &v, 16);
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (col + e < N) {
                    if (OUT_BF16) ((uint16_t*)d)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                    else ((uint32_t*)d)[e] = w[e & 3];
                }
        }
    }
}

// The parts' sums of 1024 elements of a tile, in order.
template <int WM, bool OUT_BF16>
__global__ __launch_bounds__(256) void gemm_fp8_sum_kernel(int64_t M, int64_t N, int tiles_m, int tiles_n,
                                                           void* __restrict__ C, int parts,
                                                           const float* __restrict__ part) {
    using L = Tile<WM>;
    constexpr int kPer = L::kM * kTile / 1024;
    const int64_t item = blockIdx.x / kPer;
    int tm, tn;
    tile_of((int)item, L::kGroup, tiles_m, tiles_n, tm, tn);
    const int at = (blockIdx.x % kPer) * 256 + threadIdx.x, lane = at & 63, ji = at >> 6 & 15, wave = at >> 10;
    const float* in = part + item * parts * (L::kM * kTile) + at * 4;
    f32x4 v = *reinterpret_cast<const f32x4*>(in);
    for (int p = 1; p < parts; ++p) v += *reinterpret_cast<const f32x4*>(in + (int64_t)p * (L::kM * kTile));
    const int64_t m = (int64_t)tm * L::kM + (wave >> 1) * 64 + (ji & 3) * 16 + (lane & 15);
    const int64_t n = (int64_t)tn * kTile + (wave & 1) * 64 + (ji >> 2) * 16 + (lane >> 4) * 4;
    if (m < M) store4<OUT_BF16>(C, m, n, N, v);
}

}  // namespace

// Which kernel takes a product, and in how many parts along K the tiles here take
// it (never more than one workgroup a CU).  bytes: what the parts' sums take.
struct Plan {
    enum { Skinny, Wide, Tiles } kernel = Tiles;
    int cus = 0, wm = 2;
    int64_t tm = 0, tn = 0, parts = 1;
    size_t bytes = 0;
};

// The fastest by modelled times in us: rounds of one tile a CU, each with a fixed
// part and one for each block, and for split tiles the sum's launch and the
// partial sums' way out and back.  Model / measured on 256 CUs out of HBM, M x N x K
// (F32: 128, 256 rows; E8M0: 128, 256, wide):
//   8192 x 21504 x 4096   F32 908 / 914, 706 / 713    E8M0 881 / 882, 650 / 655, 588 / 568
//   8192 x 4096 x 21504   F32 782 / 778, 635 / 631    E8M0 755 / 757, 543 / 563, 515 / 517
//   2000 x 4096 x 4096    F32 43 / 45, 34 / 37        E8M0 42 / 43, 31 / 34, 54 / 49
//   777 x 4096 x 21504    F32 98 / 99, 99 / 94        E8M0 94 / 97, 88 / 88, 258 / 211
//   1999 x 1360 x 3408    F32 19 / 20, 29 / 29        E8M0 18 / 19, 27 / 27, 46 / 42
//   1999 x 3408 x 1360    F32 20 / 24, 14 / 18        E8M0 19 / 23, 15 / 17, 22 / 25
static hipError_t make_plan(int64_t M, int64_t N, int64_t K, bool e8, Plan& p) {
    const hipError_t err = device_cus(&p.cus);
    if (err != hipSuccess) return err;
    const int64_t KB = (K + 127) / 128, cus = p.cus;
    if (fp8_skinny(M, K)) {
        p.kernel = Plan::Skinny;
        return hipSuccess;
    }
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    double best = 1e30;
    for (int wm = 2; wm <= 4; wm += 2) {
        const int64_t tm = up(M, 64 * wm), tn = up(N, kTile), tiles = tm * tn;
        const double fixed = wm == 2 ? 3.7 : e8 ? 6.3 : 4.2;
        const double each = wm == 2 ? (e8 ? 0.54 : 0.56) : e8 ? 0.77 : 0.92;
        const int64_t most = std::max<int64_t>(std::min<int64_t>(cus / tiles, KB / 8), 1);
        for (int64_t parts : {(int64_t)1, most}) {                    // whole, or split as far as it goes
            const double bytes = parts > 1 ? (double)(tiles * parts) * (64 * wm) * kTile * 4 : 0.0;
            const double us = (double)up(tiles * parts, cus) * (fixed + each * (double)up(KB, parts)) +
                              (parts > 1 ? 4.0 + 2.0 * bytes / 5e6 : 0.0);
            if (us < best) {
                best = us;
                p.wm = wm, p.tm = tm, p.tn = tn, p.parts = parts, p.bytes = (size_t)bytes;
            }
        }
    }
    if (e8 && KB > 0 && (double)up(up(M, 256) * up(N, 256), cus) * (5.5 + 1.5 * (double)KB) < best) {
        p.kernel = Plan::Wide;
        p.parts = 1, p.bytes = 0;
    }
    return hipSuccess;
}

// part: p.bytes of workspace
static hipError_t run_plan(const Plan& p, int64_t M, int64_t N, int64_t K, const uint8_t* a, const void* as, Fp8 a_fmt,
                           const uint8_t* b, const void* bs, bool tiled, bool e8, void* c, bool c_bf16, float* part,
                           hipStream_t s) {
    if (p.kernel == Plan::Skinny)
        return launch_gemm_fp8_skinny(M, N, K, p.cus, a, as, a_fmt, b, bs, tiled, e8, c, c_bf16, s);
    if (p.kernel == Plan::Wide)
        return launch_gemm_fp8_wide(M, N, K, p.cus, a, as, a_fmt, b, bs, tiled, c, c_bf16, s);
    const int64_t KB = (K + 127) / 128, tm = p.tm, tn = p.tn, parts = p.parts;
    auto go = [&](auto wm, auto af, auto e, auto tl, auto bf) {
        constexpr int kWM = decltype(wm)::value;
        hipLaunchKernelGGL((gemm_fp8_kernel<kWM, decltype(af)::value, decltype(e)::value, decltype(tl)::value, decltype(bf)::value>),
                           dim3((unsigned)(tm * tn * parts)), dim3(128 * kWM), 0, s, M, N, (int)KB, (int)tm, (int)tn, a,
                           as, b, bs, c, (int)parts, part);
        hipError_t e2 = hipGetLastError();
        if (e2 != hipSuccess || parts == 1) return e2;
        hipLaunchKernelGGL((gemm_fp8_sum_kernel<kWM, decltype(bf)::value>), dim3((unsigned)(tm * tn * 8 * kWM)), dim3(256),
                           0, s, M, N, (int)tm, (int)tn, c, (int)parts, part);
        return hipGetLastError();
    };
    using Y = std::true_type;
    using F = std::false_type;
    auto with = [](bool v, auto&& f) { return v ? f(Y{}) : f(F{}); };
    return with(a_fmt == Fp8::E5M2, [&](auto af) {
        return with(e8, [&](auto e) {
            return with(tiled, [&](auto tl) {
                return with(c_bf16, [&](auto bf) {
                    if (p.wm == 4) return go(std::integral_constant<int, 4>{}, af, e, tl, bf);
                    return go(std::integral_constant<int, 2>{}, af, e, tl, bf);
                });
            });
        });
    });
}

hipError_t launch_gemm_fp8(int64_t M, int64_t N, int64_t K, const uint8_t* a, const void* as, Fp8 a_fmt,
                           const uint8_t* b, const void* bs, bool tiled, bool e8, void* c, bool c_bf16,
                           hipStream_t s) {
    Plan p;
    Workspace held;                                  // until the sum is enqueued
    void* part = nullptr;
    hipError_t e = make_plan(M, N, K, e8, p);
    if (e == hipSuccess && p.bytes > 0) e = held.take(kWsFp8, s, p.bytes, &part);
    if (e != hipSuccess) return e;
    return run_plan(p, M, N, K, a, as, a_fmt, b, bs, tiled, e8, c, c_bf16, (float*)part, s);
}

// One workspace holds the parts' sums, the payload and the scales, so that
// nothing is enqueued unless all of it is there.
hipError_t launch_linear_fp8(const void* x, int64_t T, int64_t K, int64_t N, const uint8_t* w, const void* ws,
                             bool e8, void* y, bool y_bf16, hipStream_t s) {
    if (fp8_fused(T, K)) return launch_linear_fp8_fused(x, T, K, N, w, ws, e8, y, y_bf16, s);
    const int64_t KB = (K + 127) / 128;
    const size_t payload = (size_t)(T * KB * 128), scales = (size_t)(KB * scale_pitch(T)) * (e8 ? 1 : 4);
    Plan p;
    Workspace held;                                  // until the product is enqueued
    uint8_t* base = nullptr;
    hipError_t e = make_plan(T, N, K, e8, p);
    if (e == hipSuccess && K > 0) e = held.take(kWsTokens, s, p.bytes + payload + scales, (void**)&base);
    if (e != hipSuccess) return e;
    uint8_t* q = base + p.bytes;
    if (K > 0) e = launch_quant_fp8(DType::BF16, Fp8::E4M3, e8, x, T, K, q, q + payload, nullptr, nullptr, s);
    if (e != hipSuccess) return e;
    return run_plan(p, T, N, K, q, q + payload, Fp8::E4M3, w, ws, true, e8, y, y_bf16, (float*)base, s);
}

}  // namespace ue5m3
