// The 8-bit product under E8M0 scales in 256 x 256 output tiles, for large
// products.
//
// Four waves of 128 x 128 accumulate in place in the accumulation registers,
// with v_mfma_scale_f32_32x32x64_f8f6f4, which applies the scales: lane l
// supplies row l % 32 and 32 of the 64 k of a slice, as two 16-byte chunks, and
// its row's scale byte.  (It truncates small products next to large ones, as the
// instruction of the smaller tiles does; see fp8_gemm.hip.)  A stage is one block of 128 k, two slices; its 512 rows
// of 128 bytes lie in LDS with chunk c at c ^ (row % 8).  Workgroups are
// persistent: the loads run two stages ahead over the stages of all of a
// workgroup's tiles, so a tile's epilogue and the next one's start overlap them.
// (With fp32 output four registers spill over the K loop: to read them back at a
// tile's end waits for every load, and that overlap is lost.)
//
// Bound: a CU takes in 64 KB for 2048 cycles of the matrix pipe, half of what
// the 128 x 128 tiles need for as many products, which were held up there by
// the loads (half of each wave's time it waited to issue one).  LDS reads and
// loads stand between the products, one of each, so that neither comes in bursts.
// Out of HBM 8192 x 21504 x 4096 568 - 577 us (2500 - 2540 TFLOP/s; within a training
// step 595 - 607), 8192 x 4096 x 21504 517 - 535, 8192^3 402 - 413 (2660 - 2730; without
// the lines fetched ahead into L2 12% slower), where the library's product under
// one scale for each tensor takes 393.
#include "fp8.hpp"
#include "fp8_tile.hpp"
#include "gemm_regs.hpp"
#include "launch.hpp"

namespace ue5m3 {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kRow = 128, kRows = BM + BN, kStage = kRows * kRow, kScale = kRows * 4;
constexpr int kEpi = 4096;                           // of a wave, for the epilogue's transposition
constexpr int kAhead = 3;                            // stages from the loads to the lines fetched into L2

// One product added in place, times 2^(sb - 127) 2^(sa - 127).  The compiler
// does not model it: accesses of its accumulator keep clear of it by the
// kernel's own order (16 passes: 20 wait states).
template <int AF>
__device__ __forceinline__ void accumulate(f32x16& d, const i32x8& b, const i32x8& a, int sb, int sa) {
    if (AF == 0)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                     : "+a"(d) : "v"(b), "v"(a), "v"(sb), "v"(sa));
    else
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] blgp:1"
                     : "+a"(d) : "v"(b), "v"(a), "v"(sb), "v"(sa));
}

template <int AF, bool TILED, bool OUT_BF16>
__global__ __launch_bounds__(256, 1) void gemm_fp8_wide_kernel(int64_t M, int64_t N, int KB, int tiles_m, int tiles_n,
                                                               const uint8_t* __restrict__ A,
                                                               const uint8_t* __restrict__ As,
                                                               const uint8_t* __restrict__ B,
                                                               const uint8_t* __restrict__ Bs, void* __restrict__ C) {
    __shared__ __attribute__((aligned(16))) uint8_t sP[2 * kStage];
    __shared__ __attribute__((aligned(16))) uint8_t sS[2 * kScale];
    __shared__ __attribute__((aligned(16))) uint8_t sE[4 * kEpi];
    __shared__ __attribute__((aligned(16))) uint8_t sD[4 * 256];   // what ahead() loads
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, r = lane & 31, hi = lane >> 5;
    const uint32_t Kp = (uint32_t)KB * 128u;
    const int tiles = tiles_m * tiles_n, grid = (int)gridDim.x;
    const int nw = (tiles - (int)blockIdx.x + grid - 1) / grid;      // tiles of this workgroup

    // ---- loads ------------------------------------------------------------
    // Waves 0, 1 bring A rows, 2, 3 B rows: 128 each, 8 a load, and their codes,
    // 64 a load (of tiled B: the tile's one, for every row).
    const bool isA = wave < 2;
    const int half = 128 * (wave & 1);
    const int64_t rows = isA ? M : N;
    const bool tile_code = TILED && !isA;
    const uint64_t pay = uniform64((uint64_t)(uintptr_t)(isA ? A : B)), cod = uniform64((uint64_t)(uintptr_t)(isA ? As : Bs));
    const uint64_t cstep = uniform64(tile_code ? 1 : (uint64_t)scale_pitch(rows));
    // (one register: what is added for load i goes in at the load, as the compiler
    // would keep all sixteen sums; not in the scalar offset, which the range
    // check leaves out)
    const uint32_t voff = (uint32_t)(half + (lane >> 3)) * Kp + (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
    const uint32_t lds = lds_addr(sP) + 128u * kRow * wave, lds_c = lds_addr(sS) + 512u * wave, lds_d = lds_addr(sD) + 256u * wave;
    i32x4_t src;                                     // the cursor's tile: rows, codes of its stage, lanes' codes
    uint64_t cat = 0;
    int cleft = 0;                                   // rows from the wave's first on, less one
    int lk = 0, lb = 0;                              // the cursor: tile of the workgroup, block
    auto rows_of = [&](int64_t x0) {                 // the (up to 256) rows from x0 on
        const uint64_t p = uniform64(pay + (uint64_t)x0 * Kp);
        return i32x4_t{(int)(uint32_t)p, (int)(uint32_t)(p >> 32), uniform((int)((uint32_t)min(rows - x0, (int64_t)256) * Kp)),
                       0x00020000};
    };
    auto enter = [&](int k) {
        int64_t m0, n0;
        tile_origin((int)blockIdx.x + k * grid, tiles_m, tiles_n, m0, n0);
        const int64_t x0 = isA ? m0 : n0, left = rows - x0;
        src = rows_of(x0);
        // of 128 rows of B that lie past N there is no tile code: the last one's is read, unused
        cat = uniform64(cod + (uint64_t)(tile_code ? min((x0 + half) / 128, (N - 1) / 128) * KB : x0));
        cleft = uniform((int)min(left - 1, (int64_t)255));
    };
    auto advance = [&]() {                           // past the last stage the cursor stays
        if (lb + 1 < KB) {
            ++lb;
            cat += cstep;
        } else if (lk + 1 < nw) {
            lb = 0;
            enter(++lk);
        }
    };
    // step i of the cursor's stage into buffer b
    auto load = [&](auto ic, int b) {
        constexpr int i = decltype(ic)::value;
        if constexpr (i < 16) {
            // (dma_rows(), with the sum in the place of its wait state)
            uint32_t vo;
            asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %3\n\tbuffer_load_dwordx4 %0, %4, %5 offen offset:%6 lds"
                         : "=&v"(vo) : "s"(lds + (uint32_t)(b * kStage) + (i & 12) * 1024u),
                           "s"((uint32_t)i * 8u * Kp - (i & 3) * 1024u), "v"(voff), "s"(src), "s"((uint32_t)lb * 128u),
                           "n"((i & 3) * 1024) : "memory", "m0");
        } else {
            uint32_t row;                            // the lane's, the last one past the operand's end
            asm volatile("v_add_u32 %0, %1, %2\n\tv_min_i32 %0, %3, %0"
                         : "=&v"(row) : "s"(half + 64 * (i - 16)), "v"(lane), "s"(cleft));
            if (tile_code) row = 0;
            dma_scale<true>(i32x4_t{(int)(uint32_t)cat, (int)(uint32_t)(cat >> 32), 256, 0x00020000}, row,
                            lds_c + (uint32_t)(b * kScale) + (i - 16) * 256u);
        }
    };
    // Lines of a later stage into the L2 (and to LDS that nobody reads): the eight
    // workgroups of an XCD that share a tile row of A take 32 of its rows each,
    // the four that share one of B 64 (tile_origin's groups).  The loads proper
    // then find them there; a miss would hold up all four waves at the barrier.
    i32x4_t fsrc;                                    // the tile that the lines are of
    uint32_t frow = 0;
    int fk = 0, fb = 0;                              // tile of the workgroup, block
    auto enter_ahead = [&]() {
        int64_t m0, n0;
        tile_origin((int)blockIdx.x + fk * grid, tiles_m, tiles_n, m0, n0);
        const int64_t x0 = isA ? m0 : n0;
        fsrc = rows_of(x0);
        const int64_t share = isA ? n0 / BN % 8 * 32 + 16 * (wave & 1) + (lane & 15)
                                  : m0 / BM % 4 * 64 + 32 * (wave & 1) + (lane & 31);
        frow = (uint32_t)min(share, rows - x0 - 1) * Kp;
    };
    auto ahead = [&]() {
        asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds"
                     :: "v"(frow), "s"(fsrc), "s"((uint32_t)fb * 128u), "s"(lds_d) : "memory", "m0");
        if (fb + 1 < KB) {
            ++fb;
        } else if (fk + 1 < nw) {
            fb = 0;
            ++fk;
            enter_ahead();
        }
    };

    // ---- fragments ----------------------------------------------------------
    // offset of chunk c of slice s in a lane's first row of operand `op`: chunk
    // (4s + 2hi + c) ^ (r % 8), from that of chunk 0 of slice 0 (two registers)
    const int first[2] = {(wm * 128 + r) * kRow + ((2 * hi) ^ (r & 7)) * 16,
                          (BM + wn * 128 + r) * kRow + ((2 * hi) ^ (r & 7)) * 16};
    auto chunk = [&](int op, int s, int c, int b) {
        int at;
        if (s == 0 && c == 0) asm volatile("v_mov_b32 %0, %1" : "=v"(at) : "v"(first[op]));
        else if (s == 0) asm volatile("v_xor_b32 %0, 16, %1" : "=v"(at) : "v"(first[op]));
        else if (c == 0) asm volatile("v_xor_b32 %0, 64, %1" : "=v"(at) : "v"(first[op]));
        else asm volatile("v_xor_b32 %0, 0x50, %1" : "=v"(at) : "v"(first[op]));
        return at + b * kStage;
    };
    struct Slice {
        i32x8 v[8];                                  // groups 0..3: A rows 32i + r, 4..7: B rows
    };
    // read q of 16: half q % 2 of group q / 2
    int from[2];
    auto read = [&](auto qc, Slice& f, int s, int b) {
        constexpr int q = decltype(qc)::value, g = q / 2, c = q % 2;
        if constexpr (g % 4 == 0) from[c] = chunk(g / 4, s, c, b);
        const uint4 v = *reinterpret_cast<const uint4*>(sP + from[c] + (g & 3) * 32 * kRow);
        f.v[g][4 * c] = (int)v.x; f.v[g][4 * c + 1] = (int)v.y; f.v[g][4 * c + 2] = (int)v.z; f.v[g][4 * c + 3] = (int)v.w;
    };
    const uint8_t* const ca = sS + (wm * 128 + r) * 4;
    const uint8_t* const cb = sS + (BM + wn * 128 + r) * 4;
    auto code = [&](int g, int b) {
        return *reinterpret_cast<const int*>((g < 4 ? ca : cb) + b * kScale + (g & 3) * 128);
    };

    f32x16 acc[4][4];
    Slice R0, R1;
    int sc[8], scn[8];

    enter(0);
    enter_ahead();
    fb = min(1 + kAhead, KB - 1);
    static_for<0, 18>([&](auto ic) { load(ic, 0); });
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    static_for<0, 16>([&](auto qc) { read(qc, R0, 0, 0); });
#pragma unroll
    for (int g = 0; g < 8; ++g) sc[g] = code(g, 0);
    advance();
    static_for<0, 18>([&](auto ic) { load(ic, 1); });
    // (as in every turn: the first one's wait leaves one load out, and the last code
    // of stage 1 must not be that one)
    ahead();

    int b = 0;
    for (int k = 0; k < nw; ++k) {
        float zero = 0.0f;
        asm volatile("" : "+v"(zero));               // (as a constant it becomes sixteen kept registers)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = zero;
                asm volatile("" : "+a"(acc[i][j]));
            }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 4" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        for (int kb = 0; kb < KB; ++kb) {
            // slice 0 of this stage, its slice 1 read in between
            static_for<0, 16>([&](auto qc) {
                constexpr int q = decltype(qc)::value, i = q / 4, j = q % 4;
                accumulate<AF>(acc[i][j], R0.v[4 + j], R0.v[i], sc[4 + j], sc[i]);
                read(qc, R1, 1, b);
                __builtin_amdgcn_sched_barrier(0);
            });
            // every wave has read this stage, the next one has landed
            // (all but the one load ahead: loads come in order, and stores that are
            // still out only make this wait longer)
            asm volatile("s_waitcnt vmcnt(1) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int bn = b ^ 1;
            advance();
            // slice 1, the next stage's slice 0 and codes and the loads of the one after
            static_for<0, 16>([&](auto qc) {
                constexpr int q = decltype(qc)::value, i = q / 4, j = q % 4;
                accumulate<AF>(acc[i][j], R1.v[4 + j], R1.v[i], sc[4 + j], sc[i]);
                if constexpr (q < 2) load(std::integral_constant<int, 2 * q>{}, b);
                load(std::integral_constant<int, q < 2 ? 2 * q + 1 : q + 2>{}, b);
                if constexpr (q == 15) ahead();
                read(qc, R0, 0, bn);
                if constexpr (q < 8) scn[q] = code(q, bn);
                __builtin_amdgcn_sched_barrier(0);
            });
            // the last product has landed before anything the compiler may put
            // where this loop closes
            asm volatile("s_nop 15\n\ts_nop 4" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int g = 0; g < 8; ++g) sc[g] = scn[g];
            b = bn;
        }
        __builtin_amdgcn_sched_barrier(0);

        // ---- epilogue: element e of acc[i][j] is row 32i + r, column 32j +
        // 8(e / 4) + 4 hi + e % 4 of the wave's 128 x 128.  32 rows x 128 bytes
        // at a time through the wave's LDS, chunk c of row x at c ^ (x / 2 % 8).
        int64_t m0, n0;
        tile_origin((int)blockIdx.x + k * grid, tiles_m, tiles_n, m0, n0);
        constexpr int kEs = OUT_BF16 ? 2 : 4, kPer = 16 / kEs, kJ = OUT_BF16 ? 2 : 1;   // kJ accumulators a round
        int l = lane;
        asm volatile("" : "+v"(l));                  // its addresses are not kept over the loop above
        const int r = l & 31, hi = l >> 5, rr = l >> 3, rc = l & 7;
        uint8_t* const ep = sE + wave * kEpi;
        const int64_t mw = m0 + wm * 128, nc = n0 + wn * 128 + rc * kPer;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; j += kJ) {
#pragma unroll
                for (int jj = 0; jj < kJ; ++jj) {
                    asm volatile("" : "+v"(acc[i][j + jj]));     // read out here, once
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x16& a = acc[i][j + jj];
                        if (OUT_BF16) {
                            const int c = (4 * jj + g) ^ (r >> 1 & 7);
                            *reinterpret_cast<uint2*>(ep + r * 128 + c * 16 + hi * 8) =
                                make_uint2(pack_bf16x2(a[4 * g], a[4 * g + 1]), pack_bf16x2(a[4 * g + 2], a[4 * g + 3]));
                        } else {
                            const int c = (2 * g + hi) ^ (r >> 1 & 7);
                            *reinterpret_cast<f32x4*>(ep + r * 128 + c * 16) = f32x4{a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]};
                        }
                    }
                }
                wave_lds_sync();
                uint4 v[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int x = rr + 8 * t;
                    v[t] = *reinterpret_cast<const uint4*>(ep + x * 128 + ((rc ^ (x >> 1 & 7)) * 16));
                }
                wave_lds_sync();
                const int64_t col = nc + 32 * j;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int64_t m = mw + 32 * i + rr + 8 * t;
                    uint8_t* const d = (uint8_t*)C + (m * N + col) * kEs;
                    if (m >= M || col >= N) continue;
                    if (col + kPer <= N) {
                        __builtin_memcpy(d, &v[t], 16);
                    } else {
                        const uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w};
#pragma unroll
                        for (int e = 0; e < kPer; ++e)
                            if (col + e < N) {
                                if (OUT_BF16) ((uint16_t*)d)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                                else ((uint32_t*)d)[e] = w[e & 3];
                            }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);   // one round's registers at a time
            }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load outlives the kernel's LDS
}

}  // namespace

hipError_t launch_gemm_fp8_wide(int64_t M, int64_t N, int64_t K, int cus, const uint8_t* a, const void* as, Fp8 a_fmt,
                                const uint8_t* b, const void* bs, bool tiled, void* c, bool c_bf16, hipStream_t s) {
    const int KB = (int)((K + 127) / 128), tm = (int)((M + BM - 1) / BM), tn = (int)((N + BN - 1) / BN);
    auto go = [&](auto af, auto tl, auto bf) {
        hipLaunchKernelGGL((gemm_fp8_wide_kernel<decltype(af)::value, decltype(tl)::value, decltype(bf)::value>),
                           dim3((unsigned)(tm * tn < cus ? tm * tn : cus)), dim3(256), 0, s, M, N, KB, tm, tn, a,
                           (const uint8_t*)as, b, (const uint8_t*)bs, c);
        return hipGetLastError();
    };
    using Y = std::true_type;
    using F = std::false_type;
    auto with = [](bool v, auto&& f) { return v ? f(Y{}) : f(F{}); };
    return with(a_fmt == Fp8::E5M2, [&](auto af) {
        return with(tiled, [&](auto tl) { return with(c_bf16, [&](auto bf) { return go(af, tl, bf); }); });
    });
}

}  // namespace ue5m3
