// What the attention kernels share: matrix instructions on 16-bit operands, tiles
// of rows in LDS, direct loads to them, and reads of them along and across rows.
//
// Matrix instructions (lane l, h = l / 32, or g = l / 16): of a 32 x 32 x 16
// product lane l holds A[l % 32][8 h + j], B[8 h + j][l % 32] (j < 8) and
// C[8 (i / 4) + 4 h + i % 4][l % 32] (i < 16); of a 16 x 16 x 32 one
// A[l % 16][8 g + j], B[8 g + j][l % 16] and C[4 g + i][l % 16] (i < 4).
//
// So a product C of scores, with the contraction of the next product along its
// rows, is that product's B operand as it lies in the registers: lane l's eight
// values of 16 rows r0 .. r0 + 15 are rows r0 + 4 h + {0 .. 3} and r0 + 8 + 4 h +
// {0 .. 3}, and a contraction may run in any order, as long as A is read in the
// same one (read_across).
//
// A tile holds rows of DT = 64 or 128 elements (heads of other sizes are padded),
// in chunks of 16 bytes; chunk c of row r lies at place c ^ swizzle(r) of the row,
// which spreads over the banks both the reads along rows (one chunk of 32 rows) and
// those across them (64 bytes of 8 rows).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gemm_regs.hpp"

namespace ue5m3 {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kSgTrans = 0x400;                    // (an instruction class, as in gemm_regs.hpp)
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(uint32_t)((uint64_t)v >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)v));
}

template <typename T>
__device__ __forceinline__ f32x16 product32(const u32x4& a, const u32x4& b, const f32x16& c) {
    if constexpr (std::is_same_v<T, bf16>)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <typename T>
__device__ __forceinline__ f32x4 product16(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (std::is_same_v<T, bf16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two values as 16-bit numbers, each rounded to nearest, ties to even.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (std::is_same_v<T, bf16>) {
        return pack_bf16x2(a, b);
    } else {
        return (uint32_t)__builtin_bit_cast(uint16_t, (f16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (f16)b) << 16;
    }
}

// The two values of a word.
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if constexpr (std::is_same_v<T, bf16>)
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    else
        return make_float2((float)__builtin_bit_cast(f16, (uint16_t)w), (float)__builtin_bit_cast(f16, (uint16_t)(w >> 16)));
}

// The sum of a word's two numbers, and of a third, in binary32.
template <typename T>
__device__ __forceinline__ float add_pair(uint32_t w, float c) {
    typedef std::conditional_t<std::is_same_v<T, bf16>, __bf16, _Float16> T2 __attribute__((ext_vector_type(2)));
    if constexpr (std::is_same_v<T, bf16>)
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(T2, w), T2{1.0f, 1.0f}, c, false);
    else
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(T2, w), T2{1.0f, 1.0f}, c, false);
}

// 2^x, small results flushed to zero.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The value of the lane in the other half of the wave.
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Number v, as a value that the compiler works out where it is used: kept over a loop, a
// kernel's addresses would fill its registers.
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// ---- tiles in LDS ---------------------------------------------------------
template <int DT>
__device__ __forceinline__ int swizzle(int row) {
    return DT == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
}

// Byte offset of chunk c of a row.
template <int DT>
__device__ __forceinline__ int place(int row, int c) { return row * (2 * DT) + ((c ^ swizzle<DT>(row)) << 4); }

// Lane l's operand of rows r0 + l % 32 (r0 a multiple of 32), elements 16 s + 8 h ..
template <int DT>
__device__ __forceinline__ u32x4 read_along(const uint8_t* tile, int r0, int s, int l) {
    return *(const u32x4*)(tile + r0 * (2 * DT) + (place<DT>(l & 31, l >> 5) ^ 32 * s));
}

// Lane l's operand across 16 rows from r0 on (a multiple of 16), column 32 b + l % 32:
// rows r0 + 4 h + {0 .. 3}, then r0 + 8 + 4 h + {0 .. 3}.  The read hands each
// group of 16 lanes four rows of 16 columns, transposed.
template <int DT>
__device__ __forceinline__ u32x4 read_across(const uint8_t* tile, int r0, int b, int l) {
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    const int c = 4 * b + 2 * (l >> 4 & 1) + (l >> 1 & 1), row = 4 * (l >> 5) + (l >> 2 & 3);
    const uint8_t* p = tile + r0 * (2 * DT) + 8 * (l & 1);
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + place<DT>(row, c))));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + place<DT>(row + 8, c))));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// ---- direct loads to LDS --------------------------------------------------
// The compiler does not model these loads (it would wait for all of them before
// any read of LDS): the kernels wait themselves.  m0 is written in the load's own
// statement, and the descriptor may come from a vector instruction: five states.

// 16 bytes a lane from the resource at voff to lds + 16 lane.
__device__ __forceinline__ void load_rows(i32x4_t rsrc, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :: "v"(voff), "s"(rsrc), "s"(lds) : "memory", "m0");
}

// 16 bytes, or a dword, a lane from an address of its own.
__device__ __forceinline__ void load_16(const void* p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(p), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void load_4(const void* p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dword %0, off" :: "v"(p), "s"(lds) : "memory", "m0");
}

// Waits until at most n of the wave's loads are under way.
template <int n>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(n) : "memory");
}

// Every wave's LDS accesses before it come before those after it.
__device__ __forceinline__ void barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A wave's share of the loads of a tile of ROWS rows, four waves loading: kN loads of
// kRpi rows each.  Past `rows` the last row is read again: what is masked has to
// be finite, as 0 times it is added.  A chunk past the head's end is replaced by the
// first one.
template <int DT, int ROWS = 64>
struct TileLoads {
    static constexpr int kChunks = DT / 8, kRpi = 64 / kChunks, kN = ROWS / kRpi / 4;
    uint32_t voff[kN];                               // of a whole tile

    __device__ __forceinline__ static uint32_t offset(int n, int rows, uint32_t row_bytes, int wave, int lane, int dim) {
        const int row = (wave * kN + n) * kRpi + lane / kChunks, c = lane % kChunks ^ swizzle<DT>(row);
        return (uint32_t)min(row, rows - 1) * row_bytes + (uint32_t)(8 * c < dim ? 16 * c : 0);
    }
    __device__ __forceinline__ TileLoads(uint32_t row_bytes, int wave, int lane, int dim) {
#pragma unroll
        for (int n = 0; n < kN; ++n) voff[n] = offset(n, ROWS, row_bytes, wave, lane, dim);
    }
    // The tile whose first row is at `first`; `rows` > 0 of its rows are there.
    __device__ __forceinline__ void issue(const void* first, uint32_t row_bytes, int rows, uint32_t lds, int wave,
                                          int dim) const {
        const i32x4_t rsrc = buffer_rsrc(first, 0x7FFFFFFF);
        lds += (uint32_t)wave * kN * 1024;
        if (rows >= ROWS) {
#pragma unroll
            for (int n = 0; n < kN; ++n) load_rows(rsrc, voff[n], lds + n * 1024);
        } else {
            const int lane = here((int)(threadIdx.x & 63));
#pragma unroll
            for (int n = 0; n < kN; ++n) load_rows(rsrc, offset(n, rows, row_bytes, wave, lane, dim), lds + n * 1024);
        }
    }
};

// ---- which sequence a workgroup serves --------------------------------------
struct Span {
    int64_t q0, k0;                                  // its first query and key
    int rows, keys;                                  // how many it has
    int tile;                                        // -1: none, the workgroup is `extra` past the last tile
    int extra;
};

// Sequence starts read from the device, kept within [0, tokens].
__device__ __forceinline__ void bounds(const int32_t* starts, int64_t i, int64_t tokens, int64_t& from, int64_t& to) {
    from = min(max((int64_t)starts[i], (int64_t)0), tokens);
    to = min(max((int64_t)starts[i + 1], from), tokens);
}

// Sequence `seq`, at its first tile.
__device__ __forceinline__ Span span_of(int64_t seq, int64_t n, const int32_t* q_starts, const int32_t* k_starts, int64_t q_tokens,
                                        int64_t k_tokens) {
    int64_t q0 = seq * (q_tokens / n), k0 = seq * (k_tokens / n), q1 = q0 + q_tokens / n, k1 = k0 + k_tokens / n;
    if (q_starts != nullptr) {
        bounds(q_starts, seq, q_tokens, q0, q1);
        bounds(k_starts, seq, k_tokens, k0, k1);
    }
    return Span{q0, k0, (int)(q1 - q0), (int)(k1 - k0), 0, 0};
}

// Work item `id` of all sequences' tiles of TILE rows, of queries or (KEYS) of
// keys; with DOWN the last tiles first.  All lanes of a wave call it.
template <int TILE, bool KEYS, bool DOWN>
__device__ __forceinline__ Span find_span(int id, int64_t n, const int32_t* q_starts, const int32_t* k_starts,
                                          int64_t q_tokens, int64_t k_tokens) {
    Span s{0, 0, 0, 0, -1, 0};
    if (q_starts == nullptr) {                       // equal lengths
        s.rows = (int)(q_tokens / n);
        s.keys = (int)(k_tokens / n);
        const int per = ((KEYS ? s.keys : s.rows) + TILE - 1) / TILE;
        const int seq = per > 0 ? id / per : 0;
        if (per == 0 || seq >= n) {
            s.extra = (int)(id - per * n);
            return s;
        }
        s.tile = DOWN ? per - 1 - id % per : id % per;
        s.q0 = (int64_t)seq * s.rows;
        s.k0 = (int64_t)seq * s.keys;
        return s;
    }
    const int lane = threadIdx.x & 63;
    const int32_t* starts = KEYS ? k_starts : q_starts;
    const int64_t tokens = KEYS ? k_tokens : q_tokens;
    int total = 0, want = id;
    for (int pass = DOWN ? 0 : 1; pass < 2; ++pass) {    // DOWN: how many there are, first
        int before = 0;
        for (int64_t base = 0; base < n; base += 64) {
            int tiles = 0;
            if (base + lane < n) {
                int64_t from, to;
                bounds(starts, base + lane, tokens, from, to);
                tiles = (int)((to - from + TILE - 1) / TILE);
            }
            int upto = tiles;                        // tiles of this chunk's sequences up to the lane's
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int v = __shfl_up(upto, off);
                if (lane >= off) upto += v;
            }
            const int here = uniform(__shfl(upto, 63));
            if (pass == 1 && want < before + here) {
                const uint64_t later = __ballot(before + upto > want);
                const int at = (int)__builtin_ctzll(later);
                const int64_t seq = uniform((int)(base + at));
                s.tile = uniform(want - before - (__shfl(upto, at) - __shfl(tiles, at)));
                int64_t from, to;
                bounds(q_starts, seq, q_tokens, from, to);
                s.q0 = uniform(from);
                s.rows = uniform((int)(to - from));
                bounds(k_starts, seq, k_tokens, from, to);
                s.k0 = uniform(from);
                s.keys = uniform((int)(to - from));
                return s;
            }
            before += here;
        }
        total = before;
        if (id >= total) {
            s.extra = id - total;
            return s;
        }
        want = total - 1 - id;
    }
    return s;
}

}  // namespace
}  // namespace ue5m3
