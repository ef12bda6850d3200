// Attention of ragged sequences, forward: of each query, the softmax over the keys
// it sees times their values, in one pass over the keys with the running maximum
// and sum.  Query i of a sequence of L queries and S keys stands at position
// p = i + S - L; it sees key j when j <= p and, under a window, p - j < window or
// j < sinks.  A row that sees nothing gives zeros; one sees something wherever it has a last
// key, and where all that it sees scores -inf its softmax is 0 / 0.
//
// A workgroup of four waves takes 128 queries of a head, 32 a wave, and walks
// through the keys 64 at a time.  Scores are computed transposed (keys x
// queries), so that a lane has 32 scores of one query and P^T is the second
// product's operand as it lies in its registers; the output is accumulated
// transposed too.  P is rounded to the inputs' type, as the matrix instructions
// take it, and its values are divided by the sum of what was rounded: with one key the
// output is its value exactly, and the gradients' do . o cancels dP as far as the formula
// says (without, dQ of sequences of 3 to 10 tokens is up to 2.9e-3 from the exact one
// instead of 2.2e-3, and not 0 for one token; it costs 3 to 5% of this kernel).  The sum
// before the rounding goes to lse.  Scores, sums and the output are binary32.
//
// Bound: the two products and, in their shadow, the exponentials: the scores of the next
// tile are computed between this one's (before values that are not finite were cared for and
// the second sum was kept, 8192 tokens 594 us, one after the other 639, in one run).
// 8192 tokens, causal, 32 heads of 128, bf16: 580 us in a warm run, 600 to 655 in the first
// passes of a process; 950 TFLOP/s of the 1443 that a large product reaches.  The matrix pipe
// works in 41% of the cycles, LDS in 22%; 40% of a wave's go by at waits (a tile's loads and
// its barrier), 23% at instructions that others' take the place of.  Not causal: 1100 us, 1000
// TFLOP/s.  Heads of other sizes take the products of 64 or 128: 96 561 us, 80 535, of 64 330,
// 32 313.
//
// With heads of 64 the scores are computed where they are needed: four workgroups fit a CU
// then, not three, and have nothing to do before their first tile (8192 tokens, 16 heads:
// window 1024 64 us, with the next tile's ahead 74; no window 195 and 191).
#include <algorithm>
#include <cfloat>

#include "attention.hpp"
#include "attn_tile.hpp"
#include "io.hpp"

namespace ue5m3 {
namespace {

constexpr int kAttnThreads = 256, kRows = 128, kKeys = 64;
constexpr int kCus = 256;                            // of the device

// The reference of a row's exponentials follows its maximum only where that has
// grown by more than 2^8: until then P is at most 2^8, which loses nothing in
// binary floating point, and the sums need no correction.
constexpr float kSlack = 8.0f;

struct Sight {                                       // what the rows of a sequence see
    int keys, window, sinks;
    bool causal;
    // The keys j that position p sees: j <= last and (j > before or j < sinks).
    __device__ __forceinline__ int last(int p) const { return causal ? min(p, keys - 1) : keys - 1; }
    __device__ __forceinline__ int before(int p) const { return causal && window != 0 ? p - window : -1; }
};

// Which tiles of keys the rows of a wave, at positions lo .. hi, see: some of those from
// key j on if j < some_hi and (j + kKeys > some_lo or j < sinks), all if j + kKeys <=
// all_hi and (j >= all_lo or j + kKeys <= sinks).
struct WaveSight {
    int some_lo, some_hi, all_lo, all_hi, sinks;
    __device__ __forceinline__ WaveSight(const Sight& s, int lo, int hi) : sinks(s.sinks) {
        some_hi = s.causal ? min(hi + 1, s.keys) : s.keys;
        all_hi = s.causal ? min(lo + 1, s.keys) : s.keys;
        const bool limited = s.causal && s.window != 0;
        some_lo = limited ? lo - s.window + 1 : 0;
        all_lo = limited ? hi - s.window + 1 : 0;
    }
    __device__ __forceinline__ bool none(int j) const { return j >= some_hi || (j + kKeys <= some_lo && j >= sinks); }
    __device__ __forceinline__ bool all(int j) const { return j + kKeys <= all_hi && (j >= all_lo || j + kKeys <= sinks); }
};

// (selects without a branch)
__device__ __forceinline__ bool seen(int j, int last, int before, int sinks) {
    return (j <= last) & ((j > before) | (j < sinks));
}

// The key tiles that rows at positions lo .. hi see: `sinks` first ones, then those
// from `from` on.
struct KeyTiles {
    int sinks, from, n;
    __device__ __forceinline__ KeyTiles(const Sight& s, int lo, int hi) {
        const int end = s.causal ? min(max(hi + 1, 0), s.keys) : s.keys;
        from = s.causal && s.window != 0 ? max(0, lo - s.window + 1) / kKeys : 0;
        const int to = (end + kKeys - 1) / kKeys;
        sinks = min((min(s.sinks, end) + kKeys - 1) / kKeys, from);
        n = sinks + max(0, to - from);
    }
    __device__ __forceinline__ int operator[](int i) const { return i < sinks ? i : from + i - sinks; }
};

__device__ __forceinline__ Sight sight(const ue5m3_attention_t& a, int keys) {
    return Sight{keys, a.window < keys ? (int)a.window : 0, (int)min(a.sinks, (int64_t)keys), a.causal != 0};
}

// Head of work item id, so that the query heads of a key-value head meet on one XCD:
// workgroups go round the eight.
__device__ __forceinline__ int head_of(int id, int q_heads, int kv_heads) {
    const int at = id % q_heads;
    return at % kv_heads * (q_heads / kv_heads) + at / kv_heads;
}

// Lane l's operand of a row in global memory: elements 16 s + 8 h .., zeros past dim.
template <int DT>
__device__ __forceinline__ void load_operand(u32x4 (&f)[DT / 16], const void* row, int dim) {
    const int h = (int)(threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < DT / 16; ++s) {
        f[s] = u32x4{0, 0, 0, 0};
        if (16 * s + 8 * h < dim) __builtin_memcpy(&f[s], (const uint16_t*)row + 16 * s + 8 * h, 16);
    }
}

// Whether the two numbers of a word are not finite: bits 15 and 31 of the result.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t kExponent = std::is_same_v<T, bf16> ? 0x7F807F80u : 0x7C007C00u;
    return (w & kExponent) + (std::is_same_v<T, bf16> ? 0x00800080u : 0x04000400u);
}

// The n lowest bits.
__device__ __forceinline__ uint64_t below(int n) { return n >= 64 ? ~(uint64_t)0 : n <= 0 ? 0 : ((uint64_t)1 << n) - 1; }

// A transposed accumulator's column (a lane pair's row of the tensor) times f.
template <typename T, int DT>
__device__ __forceinline__ void store_column(T* row, const f32x16 (&o)[DT / 32], float f, int dim) {
    const int h = (int)(threadIdx.x & 63) >> 5;
#pragma unroll
    for (int b = 0; b < DT / 32; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * b + 8 * g + 4 * h;
            const u32x2 w = {pack2<T>(o[b][4 * g] * f, o[b][4 * g + 1] * f), pack2<T>(o[b][4 * g + 2] * f, o[b][4 * g + 3] * f)};
            if (d < dim) __builtin_memcpy(row + d, &w, 8);
        }
}

// Rows of no sequence: zeros in this head's share of an output (each workgroup past
// the tiles takes every `extras`-th row), and -inf for `lse`, or that and a sum of 0.
__device__ __forceinline__ void empty_row(float& lse) { lse = -__builtin_inff(); }
__device__ __forceinline__ void empty_row(float2& ml) { ml = make_float2(-__builtin_inff(), 0.0f); }
template <typename T, typename L>
__device__ __forceinline__ void clear_outside(T* out, int64_t token, const int32_t* starts, int64_t n, int64_t tokens,
                                              int dim, int extra, int extras, L* lse) {
    if (starts == nullptr) return;
    const int64_t before = min(max((int64_t)starts[0], (int64_t)0), tokens);
    const int64_t after = min(max((int64_t)starts[n], before), tokens);
    for (int64_t i = extra; i < before + tokens - after; i += extras) {
        const int64_t t = i < before ? i : after + i - before;
        if constexpr (!std::is_same_v<T, float2>)
            for (int d = threadIdx.x; d < dim; d += kAttnThreads) out[t * token + d] = (T)0.0f;
        if (lse != nullptr && threadIdx.x == 0) empty_row(lse[t]);
    }
}

// Of the forward call's scratch memory: the parts' outputs [parts][tokens][heads][dim],
// then their rows' references and sums [parts][heads][tokens][2].
__host__ __device__ inline int64_t o_floats(const ue5m3_attention_t& a) { return a.q_tokens * a.q_heads * a.dim; }

template <typename T, int DT>
__global__ __launch_bounds__(kAttnThreads, DT == 64 ? 4 : 2) void attention_kernel(ue5m3_attention_t a, int items, int parts,
                                                                                  float* scratch) {
    constexpr int kTile = kKeys * DT * 2, kB = DT / 32, kS = DT / 16;
    constexpr bool AHEAD = DT == 128;
    __shared__ __attribute__((aligned(16))) uint8_t sK[2 * kTile];
    __shared__ __attribute__((aligned(16))) uint8_t sV[2 * kTile];
    __shared__ uint32_t sSpoilt[2][2];               // keys of a tile whose values are not all finite
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
    const int head = head_of(blockIdx.x, a.q_heads, a.kv_heads), kv = head / (a.q_heads / a.kv_heads);
    const int part = blockIdx.x / a.q_heads % parts, item = blockIdx.x / (a.q_heads * parts);
    const Span w = find_span<kRows, false, true>(item, a.sequences, a.q_starts, a.k_starts, a.q_tokens, a.k_tokens);
    // this head's part, and its rows' references and sums
    float* const part_o = scratch + (int64_t)part * o_floats(a) + (int64_t)head * a.dim;
    float2* const part_ml = (float2*)(scratch + parts * o_floats(a)) + ((int64_t)part * a.q_heads + head) * a.q_tokens;
    T* const o_head = (T*)a.o + (int64_t)head * a.dim;
    const int64_t o_token = (int64_t)a.q_heads * a.dim;
    float* const lse_head = a.lse != nullptr ? a.lse + head * a.q_tokens : nullptr;
    if (w.tile < 0) {
        const int extras = items - (item - w.extra);
        if (parts > 1) clear_outside((float2*)nullptr, 0, a.q_starts, a.sequences, a.q_tokens, 0, w.extra, extras, part_ml);
        else clear_outside(o_head, o_token, a.q_starts, a.sequences, a.q_tokens, a.dim, w.extra, extras, lse_head);
        return;
    }
    const int off = w.keys - w.rows, r0 = w.tile * kRows, row = r0 + wave * 32 + (lane & 31);
    const Sight sees = sight(a, w.keys);
    const KeyTiles tiles(sees, r0 + off, min(r0 + kRows, w.rows) - 1 + off);
    const int i0 = (int)((int64_t)tiles.n * part / parts), i1 = (int)((int64_t)tiles.n * (part + 1) / parts);
    const WaveSight mine(sees, r0 + wave * 32 + off, min(r0 + wave * 32 + 31, w.rows - 1) + off);
    const WaveSight ours(sees, r0 + off, min(r0 + kRows, w.rows) - 1 + off);     // the whole workgroup's
    const int last = sees.last(row + off), before = sees.before(row + off);

    u32x4 q[kS];
    load_operand<DT>(q, (const T*)a.q + (w.q0 + min(row, w.rows - 1)) * a.q_token + head * a.q_head, a.dim);

    const uint32_t k_bytes = (uint32_t)a.k_token * 2, v_bytes = (uint32_t)a.v_token * 2;
    const TileLoads<DT> lk(k_bytes, wave, lane, a.dim), lv(v_bytes, wave, lane, a.dim);
    const T* const k_head = (const T*)a.k + w.k0 * a.k_token + kv * a.k_head;
    const T* const v_head = (const T*)a.v + w.k0 * a.v_token + kv * a.v_head;
    const uint32_t ldsK = lds_addr(sK), ldsV = lds_addr(sV);
    auto issue_k = [&](int t, int buffer) {
        const int64_t j = (int64_t)t * kKeys;
        lk.issue(k_head + j * a.k_token, k_bytes, w.keys - (int)j, ldsK + buffer * kTile, wave, a.dim);
    };
    auto issue_v = [&](int t, int buffer) {
        const int64_t j = (int64_t)t * kKeys;
        lv.issue(v_head + j * a.v_token, v_bytes, w.keys - (int)j, ldsV + buffer * kTile, wave, a.dim);
    };

    f32x16 o[kB], s[2];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
    const float c = a.scale * kLog2e;
    float m = -__builtin_inff();                     // reference, in powers of two
    float sum = 0.0f, rounded = 0.0f;                // this lane's sums of P, before and after its rounding

    // One 16 elements' step of the scores of the tile in tk.
    auto score = [&](const uint8_t* tk, int x, f32x16 (&to)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) to[b] = product32<T>(read_along<DT>(tk, 32 * b, x, lane), q[x], to[b]);
    };
    auto clear = [](f32x16 (&to)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) to[b][e] = 0.0f;
    };
    // Of a tile that some rows see in part: 0 times a value that is not finite would reach
    // rows that do not see it.  In LDS zeros take the place of such values, each wave's of what
    // it loaded, and the rows that see one become NaN as a whole.
    auto clean = [&](uint8_t* tv, uint32_t* spoilt, int j0) {
        constexpr int kN = kTile / 4096;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            u32x4* const p = (u32x4*)(tv + (wave * kN + n) * 1024 + lane * 16);
            u32x4 f = *p;
            uint32_t any = 0;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const uint32_t e = not_finite<T>(f[y]) >> 15 & 0x00010001u;
                any |= e;
                f[y] &= ~(e * 0xFFFFu);
            }
            if (any != 0) {
                const int key = (wave * kN + n) * (1024 / (2 * DT)) + lane / (DT / 8);
                atomicOr(&spoilt[key / 32], 1u << key % 32);
                *p = f;
            }
        }
        barrier();
        const uint64_t keys = (uint64_t)spoilt[1] << 32 | spoilt[0];
        if (keys != 0) {
            const uint64_t seen = below(last - j0 + 1) & (~below(before - j0 + 1) | below(sees.sinks - j0));
            if ((keys & seen) != 0) sum = rounded = __builtin_nanf("");
        }
    };
    // One tile: with AHEAD its scores are there, and the next one's are computed between its
    // exponentials.  The buffer is known when this is compiled, so that the addresses of
    // all reads are a few registers and constants.
    int i = i0;
    auto turn = [&](auto buffer) __attribute__((always_inline)) {
        constexpr int B = decltype(buffer)::value;   // of this tile's values, and the tile's after the next keys
        wait_loads<0>();
        barrier();
        const int j0 = tiles[i] * kKeys;
        ++i;
        if (AHEAD && i + 1 < i1) issue_k(tiles[i + 1], B);
        if (!AHEAD && i < i1) issue_k(tiles[i], B ^ 1);
        if (i < i1) issue_v(tiles[i], B ^ 1);
        const uint8_t *tk = sK + (AHEAD ? B ^ 1 : B) * kTile, *tv = sV + B * kTile;
        if (threadIdx.x < 2) sSpoilt[B ^ 1][threadIdx.x] = 0;       // (of the last turn: all waves have read it)
        if (!ours.all(j0)) clean(sV + B * kTile, sSpoilt[B], j0);
        f32x16 ahead[2];
        if (AHEAD) clear(ahead);
        if (mine.none(j0)) {
            if (!AHEAD) return;
#pragma unroll
            for (int x = 0; x < kS; ++x) score(tk, x, ahead);
        } else {
            if (!AHEAD) {
                clear(s);
#pragma unroll
                for (int x = 0; x < kS; ++x) score(tk, x, s);
            }
            if (!mine.all(j0)) {
                const int end = last - j0 - 4 * h, start = before - j0 - 4 * h, sinks = sees.sinks - j0 - 4 * h;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        s[b][e] = seen(32 * b + 8 * (e / 4) + e % 4, end, start, sinks) ? s[b][e] : -__builtin_inff();
            }
            float top = s[0][0];
#pragma unroll
            for (int e = 1; e < 32; ++e) top = fmaxf(top, s[e / 16][e % 16]);
            top = fmaxf(top, other_half(top)) * c;
            if (__ballot(top > m + kSlack) != 0) {   // (each row by itself: none depends on its neighbours)
                const float next = top > m + kSlack ? top : m, f = exp2_fast(m - next);
                const float scale = m == next ? 1.0f : f;
                m = next;
                sum *= scale;
                rounded *= scale;
#pragma unroll
                for (int b = 0; b < kB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[b][e] *= scale;
            }
            const float ref = m == -__builtin_inff() ? 0.0f : m;
            u32x4 pt[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float u = exp2_fast(fmaf(s[x / 2][8 * (x % 2) + 2 * y], c, -ref));
                    const float v = exp2_fast(fmaf(s[x / 2][8 * (x % 2) + 2 * y + 1], c, -ref));
                    sum += u + v;
                    pt[x][y] = pack2<T>(u, v);
                    rounded = add_pair<T>(pt[x][y], rounded);
                }
                if (AHEAD) {
#pragma unroll
                    for (int z = 0; z < kS / 4; ++z) score(tk, x * (kS / 4) + z, ahead);
                }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int b = 0; b < kB; ++b) o[b] = product32<T>(read_across<DT>(tv, 16 * x, b, lane), pt[x], o[b]);
            if (AHEAD) {                             // products and exponentials in turn, operands read ahead of both
                __builtin_amdgcn_sched_group_barrier(kSgDsRead, 4, 0);
#pragma unroll
                for (int x = 0; x < 2 * kS; ++x) {
                    __builtin_amdgcn_sched_group_barrier(kSgMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSgDsRead, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSgValu, 80 / (2 * kS), 0);
                    __builtin_amdgcn_sched_group_barrier(kSgTrans, 32 / (2 * kS), 0);
                }
#pragma unroll
                for (int x = 0; x < 4 * kB; ++x) {
                    __builtin_amdgcn_sched_group_barrier(kSgMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSgDsRead, 2, 0);
                }
            }
        }
        if (AHEAD) {
#pragma unroll
            for (int b = 0; b < 2; ++b) s[b] = ahead[b];
        }
    };
    if (threadIdx.x < 4) sSpoilt[threadIdx.x / 2][threadIdx.x % 2] = 0;
    if (i0 < i1) {
        issue_k(tiles[i0], 0);
        issue_v(tiles[i0], 0);
        if (AHEAD) {
            if (i0 + 1 < i1) issue_k(tiles[i0 + 1], 1);
            wait_loads<0>();
            barrier();
            clear(s);
#pragma unroll
            for (int x = 0; x < kS; ++x) score(sK, x, s);
        }
    }
    while (i < i1) {
        turn(std::integral_constant<int, 0>{});
        if (i >= i1) break;
        turn(std::integral_constant<int, 1>{});
    }
    sum += other_half(sum);
    rounded += other_half(rounded);
    if (row >= w.rows) return;
    if (parts > 1) {
        const float f = sum == 0.0f ? 0.0f : sum / rounded;      // (the joining divides by `sum`)
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int x = 32 * b + 8 * e + 4 * h;
                if (x < a.dim)
                    *(f32x4*)(part_o + (w.q0 + row) * o_token + x) =
                        f32x4{o[b][4 * e] * f, o[b][4 * e + 1] * f, o[b][4 * e + 2] * f, o[b][4 * e + 3] * f};
            }
        // (a row whose keys here all score -inf is not one that sees nothing)
        if (h == 0) part_ml[w.q0 + row] = make_float2(last >= 0 ? fmaxf(m, -FLT_MAX) : m, sum);
        return;
    }
    const float inv = last < 0 ? 0.0f : 1.0f / rounded;          // (0 / 0 where all seen keys score -inf)
    store_column<T, DT>(o_head + (w.q0 + row) * o_token, o, inv, a.dim);
    if (a.o_rest != nullptr) {
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] = o[b][e] * inv - (float)(T)(o[b][e] * inv);
        store_column<T, DT>((T*)a.o_rest + (w.q0 + row) * o_token + (int64_t)head * a.dim, o, 1.0f, a.dim);
    }
    if (lse_head != nullptr && h == 0) lse_head[w.q0 + row] = sum == 0.0f ? -__builtin_inff() : m * kLn2 + logf(sum);
}

// Outputs from the parts of the keys, in their order; a thread four elements.  Only a row
// that sees nothing has no reference but -inf.
template <typename T>
__global__ __launch_bounds__(kAttnThreads) void attention_join_kernel(ue5m3_attention_t a, int parts, const float* __restrict__ scratch) {
    const int64_t n = o_floats(a), i = ((int64_t)blockIdx.x * kAttnThreads + threadIdx.x) * 4;
    if (i >= n) return;
    const int64_t row = i / a.dim, token = row / a.q_heads;
    const int d = (int)(i - row * a.dim), head = (int)(row - token * a.q_heads);
    const int64_t step = (int64_t)a.q_heads * a.q_tokens;
    const float2* ml = (const float2*)(scratch + parts * n) + head * a.q_tokens + token;
    float m = -__builtin_inff(), l = 0.0f;
    for (int p = 0; p < parts; ++p) m = fmaxf(m, ml[p * step].x);
    const float ref = m == -__builtin_inff() ? 0.0f : m;
    f32x4 v = {0, 0, 0, 0};
    for (int p = 0; p < parts; ++p) {
        const float2 x = ml[p * step];
        const float f = exp2_fast(x.x - ref);
        l += x.y * f;
        v += *(const f32x4*)(scratch + p * n + i) * f;
    }
    const float inv = 1.0f / l;
    u32x2 w, rest;
#pragma unroll
    for (int y = 0; y < 4; ++y) v[y] = m == -__builtin_inff() ? 0.0f : v[y] * inv;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        w[y] = pack2<T>(v[2 * y], v[2 * y + 1]);
        const float2 r = unpack2<T>(w[y]);
        rest[y] = pack2<T>(v[2 * y] - r.x, v[2 * y + 1] - r.y);
    }
    __builtin_memcpy((T*)a.o + i, &w, 8);
    if (a.o_rest != nullptr) __builtin_memcpy((T*)a.o_rest + i, &rest, 8);
    if (a.lse != nullptr && d == 0) a.lse[head * a.q_tokens + token] = l == 0.0f ? -__builtin_inff() : m * kLn2 + logf(l);
}

// Half x of a lane's 16 values, each as two numbers of the type: its rounding, and the
// rounding of what that left.
template <typename T>
__device__ __forceinline__ void two_numbers(const f32x16& s, int x, u32x4& first, u32x4& rest) {
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const float u = s[8 * x + 2 * y], v = s[8 * x + 2 * y + 1];
        first[y] = pack2<T>(u, v);
        const float2 r = unpack2<T>(first[y]);
        rest[y] = pack2<T>(u - r.x, v - r.y);
    }
}

// dQ, and the rows' sums do . o, which both halves of the backward pass take.
// As the forward kernel; P is exp(score - lse) and dS = P (dP - do . o) goes to its
// product as two numbers of the inputs' type, its rounding and the rounding of what that
// left (one product more for each operand read: 730 us against 916, 8% of a training
// step).  dP and do . o often nearly cancel, so the rounding of o would be the largest
// error of dS: the forward pass keeps what it left, too.  In relative L2 norm dQ and dK of
// 8192 tokens are 1.7e-3 from the exact ones, which is their own rounding; with dS in one
// number dQ is 2.6e-3 off and dK 2.4e-3, with o as it was rounded dQ 3.4e-3.
//
// Bound: the products.  8192 tokens, 32 heads of 128: 900 us for 0.82 TF, 1.10 with the
// second number, 1220 TFLOP/s; the matrix pipe works in 63% of the cycles, LDS in 24%.
template <typename T, int DT>
__global__ __launch_bounds__(kAttnThreads, 2) void attention_dq_kernel(ue5m3_attention_t a, ue5m3_attention_grad_t g, int items) {
    constexpr int kTile = kKeys * DT * 2, kB = DT / 32, kS = DT / 16;
    __shared__ __attribute__((aligned(16))) uint8_t sK[2 * kTile];
    __shared__ __attribute__((aligned(16))) uint8_t sV[2 * kTile];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
    const int head = head_of(blockIdx.x, a.q_heads, a.kv_heads), kv = head / (a.q_heads / a.kv_heads);
    const Span w = find_span<kRows, false, true>((int)(blockIdx.x / a.q_heads), a.sequences, a.q_starts, a.k_starts,
                                                 a.q_tokens, a.k_tokens);
    if (w.tile < 0) {
        const int extras = items - ((int)(blockIdx.x / a.q_heads) - w.extra);
        if (g.dq != nullptr)
            clear_outside((T*)g.dq + head * g.dq_head, g.dq_token, a.q_starts, a.sequences, a.q_tokens, a.dim, w.extra,
                          extras, (float*)nullptr);
        return;
    }
    const int off = w.keys - w.rows, r0 = w.tile * kRows, row = r0 + wave * 32 + (lane & 31);
    const Sight sees = sight(a, w.keys);
    const KeyTiles tiles(sees, r0 + off, min(r0 + kRows, w.rows) - 1 + off);
    const WaveSight mine(sees, r0 + wave * 32 + off, min(r0 + wave * 32 + 31, w.rows - 1) + off);
    const int last = sees.last(row + off), before = sees.before(row + off);
    const int64_t at = w.q0 + min(row, w.rows - 1), dense = (at * a.q_heads + head) * a.dim;

    u32x4 q[kS], d[kS];
    load_operand<DT>(q, (const T*)a.q + at * a.q_token + head * a.q_head, a.dim);
    load_operand<DT>(d, (const T*)g.d_o + dense, a.dim);
    float delta = 0.0f;
    {
        u32x4 o[kS], rest[kS];
        load_operand<DT>(o, (const T*)a.o + dense, a.dim);
        load_operand<DT>(rest, (const T*)a.o_rest + dense, a.dim);
#pragma unroll
        for (int x = 0; x < kS; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float2 u = unpack2<T>(o[x][y]), r = unpack2<T>(rest[x][y]), v = unpack2<T>(d[x][y]);
                delta += (u.x + r.x) * v.x + (u.y + r.y) * v.y;
            }
    }
    delta += other_half(delta);
    // (of a row that sees nothing the reference makes every P 0)
    const float lse = a.lse[head * a.q_tokens + at];
    const float ref = lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e;
    if (h == 0 && row < w.rows) {
        ((float*)g.scratch)[head * a.q_tokens + at] = delta;
        ((float*)g.scratch)[(a.q_heads + head) * a.q_tokens + at] = ref;
    }
    if (g.dq == nullptr) return;

    const uint32_t k_bytes = (uint32_t)a.k_token * 2, v_bytes = (uint32_t)a.v_token * 2;
    const TileLoads<DT> lk(k_bytes, wave, lane, a.dim), lv(v_bytes, wave, lane, a.dim);
    const T* const k_head = (const T*)a.k + w.k0 * a.k_token + kv * a.k_head;
    const T* const v_head = (const T*)a.v + w.k0 * a.v_token + kv * a.v_head;
    const uint32_t ldsK = lds_addr(sK), ldsV = lds_addr(sV);
    auto issue = [&](int t, int buffer) {
        const int64_t j = (int64_t)t * kKeys;
        lk.issue(k_head + j * a.k_token, k_bytes, w.keys - (int)j, ldsK + buffer * kTile, wave, a.dim);
        lv.issue(v_head + j * a.v_token, v_bytes, w.keys - (int)j, ldsV + buffer * kTile, wave, a.dim);
    };
    f32x16 dq[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[b][i] = 0.0f;
    const float c = a.scale * kLog2e;

    int i = 0;
    auto turn = [&](auto buffer) __attribute__((always_inline)) {
        constexpr int B = decltype(buffer)::value;
        wait_loads<0>();
        barrier();
        const int j0 = tiles[i] * kKeys;
        if (++i < tiles.n) issue(tiles[i], B ^ 1);
        if (mine.none(j0)) return;
        const uint8_t *tk = sK + B * kTile, *tv = sV + B * kTile;
        const bool all = mine.all(j0);
        const int end = last - j0 - 4 * h, start = before - j0 - 4 * h, sinks = sees.sinks - j0 - 4 * h;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x16 s, t;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = t[e] = 0.0f;
#pragma unroll
            for (int x = 0; x < kS; ++x) {
                s = product32<T>(read_along<DT>(tk, 32 * b, x, lane), q[x], s);
                t = product32<T>(read_along<DT>(tv, 32 * b, x, lane), d[x], t);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = exp2_fast(fmaf(s[e], c, -ref)) * (t[e] - delta);
            if (!all) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = seen(32 * b + 8 * (e / 4) + e % 4, end, start, sinks) ? s[e] : 0.0f;
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                u32x4 ds, rest;
                two_numbers<T>(s, x, ds, rest);
#pragma unroll
                for (int y = 0; y < kB; ++y) {
                    const u32x4 f = read_across<DT>(tk, 32 * b + 16 * x, y, lane);
                    dq[y] = product32<T>(f, ds, dq[y]);
                    dq[y] = product32<T>(f, rest, dq[y]);
                }
            }
        }
    };
    if (tiles.n > 0) issue(tiles[0], 0);
    while (i < tiles.n) {
        turn(std::integral_constant<int, 0>{});
        if (i >= tiles.n) break;
        turn(std::integral_constant<int, 1>{});
    }
    if (row < w.rows) store_column<T, DT>((T*)g.dq + at * g.dq_token + head * g.dq_head, dq, a.scale, a.dim);
}

// Of the gradient's scratch memory: delta and the references [2][heads][tokens], then
// the parts of dK and dV [parts][2][tokens][kv_heads][dim], then those of the sinks from
// the rows far from them [far][2][sequences][sinks][kv_heads][dim].
__host__ __device__ inline int64_t dkv_floats(const ue5m3_attention_t& a) { return a.k_tokens * a.kv_heads * a.dim; }
__host__ __device__ inline int64_t delta_floats(const ue5m3_attention_t& a) { return (2 * a.q_heads * a.q_tokens + 3) / 4 * 4; }
__device__ __forceinline__ float* dkv_parts(const ue5m3_attention_t& a, const ue5m3_attention_grad_t& g) {
    return (float*)g.scratch + delta_floats(a);
}
__host__ __device__ inline int64_t far_floats(const ue5m3_attention_t& a) { return a.sequences * a.sinks * a.kv_heads * a.dim; }

// dK and dV: a workgroup takes 128 keys of a key-value head, 32 a wave, and walks
// through the queries that see them, 32 at a time, of each query head that shares
// it in turn: the sum over those heads is made here, in a fixed order.
//
// Scores are queries x keys here, so that P and dS are the operands of the products that
// contract over queries.  P goes to dV's in one number (dV is 2.2e-3 off, 1.7e-3 of which its
// own rounding makes, and 2.5e-3 at most over sequences of all lengths), dS to dK's in two, as
// for dQ (in one dK is 2.4e-3 off, of a few tokens up to 3.2e-3, twice its own rounding; it is
// a fifth product, for operands that are read anyway: a training step of 8192 tokens 2660 us
// without, 2840 with it).  A wave's keys stay in registers, its values in LDS: with both in
// registers there would be room for one wave a SIMD only, and nothing to fill its waits
// (8192 tokens, 32 heads of 128, 8 of keys, dS in one number: 1730 us against 1230).
//
// Bound: the products, 4 of 2 pairs x heads x dim operations and one more for dS's second
// number: those 1.37 TF take 1270 us (1080 TFLOP/s).  The matrix pipe works in 49% of the
// cycles and LDS, which holds Q and dO for two reads each, in 30%; 46% of a wave's go by at
// waits, for reads of LDS and at the barrier of a tile.  With heads of 64 three workgroups
// fit a CU, which is worth more than products ordered between the exponentials by hand, for
// which there are registers with two only (packed sequences of 8192 tokens, window 1024, 4
// sinks, dS in one number: 108 us against 119; in two 120).
//
// Under a window the first tile of a sequence has all rows to visit where the others have
// the window's: the rows that see its sinks only are cut into `far` parts of their own.
template <typename T, int DT>
__global__ __launch_bounds__(kAttnThreads, DT == 64 ? 3 : 2) void attention_dkv_kernel(ue5m3_attention_t a, ue5m3_attention_grad_t g, int items,
                                                                       int parts, int far) {
    constexpr int kQ = 32, kTile = kQ * DT * 2, kB = DT / 32, kS = DT / 16;
    __shared__ __attribute__((aligned(16))) uint8_t sQ[2 * kTile];
    __shared__ __attribute__((aligned(16))) uint8_t sD[2 * kTile];
    __shared__ __attribute__((aligned(16))) uint8_t sV[kRows * DT * 2];
    __shared__ __attribute__((aligned(16))) float sR[2 * 64];        // delta of the tile's rows, then their references
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 5;
    const int kv = blockIdx.x % a.kv_heads, group = a.q_heads / a.kv_heads;
    const int far_groups = far * (int)a.sequences, id = (int)(blockIdx.x / a.kv_heads) - far_groups;
    const bool is_far = id < 0, staged = parts > 1 || far > 0;
    const int shares = is_far ? far : parts, at_id = is_far ? id + far_groups : id;
    const int part = at_id % shares, item = at_id / shares;      // (of the far ones the sequence)
    const Span w = is_far ? span_of(item, a.sequences, a.q_starts, a.k_starts, a.q_tokens, a.k_tokens)
                          : find_span<kRows, true, false>(item, a.sequences, a.q_starts, a.k_starts, a.q_tokens, a.k_tokens);
    if (is_far && w.keys == 0) return;
    float* const delta = (float*)g.scratch;
    float* part_dk = dkv_parts(a, g) + (int64_t)kv * a.dim;
    part_dk += is_far ? parts * 2 * dkv_floats(a) + part * 2 * far_floats(a) : part * 2 * dkv_floats(a);
    float* const part_dv = part_dk + (is_far ? far_floats(a) : dkv_floats(a));
    T* const dk_head = (T*)g.dk + kv * g.dk_head;
    T* const dv_head = (T*)g.dv + kv * g.dv_head;
    const int64_t token = (int64_t)a.kv_heads * a.dim;   // of the parts
    if (w.tile < 0) {
        const int extras = items - (item - w.extra);
        if (staged) {
            clear_outside(part_dk, token, a.k_starts, a.sequences, a.k_tokens, a.dim, w.extra, extras, (float*)nullptr);
            clear_outside(part_dv, token, a.k_starts, a.sequences, a.k_tokens, a.dim, w.extra, extras, (float*)nullptr);
        } else {
            clear_outside(dk_head, g.dk_token, a.k_starts, a.sequences, a.k_tokens, a.dim, w.extra, extras, (float*)nullptr);
            clear_outside(dv_head, g.dv_token, a.k_starts, a.sequences, a.k_tokens, a.dim, w.extra, extras, (float*)nullptr);
        }
        return;
    }
    const int off = w.keys - w.rows, c0 = w.tile * kRows, key = c0 + wave * 32 + (lane & 31);
    const Sight sees = sight(a, w.keys);
    const int64_t at = w.k0 + min(key, w.keys - 1);
    // the rows that see the lane's key
    const int first = sees.causal ? max(key - off, 0) : 0;
    const int last = sees.causal && sees.window != 0 && key >= sees.sinks
                         ? (int)min((int64_t)key + sees.window - 1 - off, (int64_t)w.rows - 1) : w.rows - 1;
    // of the wave's keys the rows that see some (from some_lo, before some_hi), and all
    const int wlo = c0 + wave * 32, whi = wlo + 31;
    const bool limited = sees.causal && sees.window != 0;
    const int some_lo = sees.causal ? max(0, wlo - off) : 0, all_lo = sees.causal ? max(0, whi - off) : 0;
    int some_hi = w.rows, all_hi = w.rows;
    if (limited && wlo >= sees.sinks) some_hi = (int)min((int64_t)w.rows, (int64_t)min(whi, w.keys - 1) + sees.window - off);
    if (limited && whi >= sees.sinks) all_hi = (int)min((int64_t)w.rows, (int64_t)wlo + sees.window - off);
    if (wlo >= w.keys) some_hi = 0;
    if (whi >= w.keys) all_hi = 0;

    // tiles of each head whose rows see some of the workgroup's keys
    const int end = min(c0 + kRows, w.keys) - 1;
    int from = 0, to = w.rows;
    if (sees.causal) from = max(0, c0 - off);
    if (limited && (c0 >= sees.sinks || far > 0)) to = (int)min((int64_t)to, (int64_t)end + sees.window - off);
    from = from / kQ;
    if (is_far) from = (max(to, 0) + kQ - 1) / kQ, to = w.rows;
    // of all heads' tiles, one after the other, this part's share
    const int per = max(0, (to + kQ - 1) / kQ - from);
    const int i0 = (int)((int64_t)per * group * part / shares), n = (int)((int64_t)per * group * (part + 1) / shares) - i0;

    const uint32_t ldsQ = lds_addr(sQ), ldsD = lds_addr(sD), ldsR = lds_addr(sR);
    if (n > 0) {                                     // (the first turn waits for them)
        const uint32_t v_bytes = (uint32_t)a.v_token * 2;
        const TileLoads<DT> lv(v_bytes, wave, lane, a.dim);
#pragma unroll
        for (int i = 0; i < kRows / 64; ++i)
            if (c0 + 64 * i < w.keys)
                lv.issue((const T*)a.v + (w.k0 + c0 + 64 * i) * a.v_token + kv * a.v_head, v_bytes, w.keys - c0 - 64 * i,
                         lds_addr(sV) + i * 64 * DT * 2, wave, a.dim);
    }
    u32x4 k[kS];
    load_operand<DT>(k, (const T*)a.k + at * a.k_token + kv * a.k_head, a.dim);

    // The tiles of a head come from its last to its first: causal workgroups then begin
    // with the same rows and an XCD's L2 holds what they read (measured, the order makes no
    // difference: from the first on 2053 us against 2041, before there were parts).
    // The next loads: the rows from `next` on, at q_at, d_at and r_at.
    const int top = (from + per - 1) * kQ;           // first row of the last tile
    const int head = kv * group + (per > 0 ? i0 / per : 0), skip = per > 0 ? i0 % per * kQ : 0;
    const int64_t o_token = (int64_t)a.q_heads * a.dim, row0 = w.q0 + top;
    const uint32_t q_bytes = (uint32_t)a.q_token * 2, d_bytes = (uint32_t)o_token * 2;
    const TileLoads<DT, kQ> lq(q_bytes, wave, lane, a.dim), ld(d_bytes, wave, lane, a.dim);
    const T* q_last = (const T*)a.q + row0 * a.q_token + head * a.q_head;
    const T* d_last = (const T*)g.d_o + row0 * o_token + (int64_t)head * a.dim;
    const float* r_last = delta + head * a.q_tokens + row0 + (int64_t)h * a.q_heads * a.q_tokens + (lane & 31);
    const T *q_at = q_last - skip * a.q_token, *d_at = d_last - skip * o_token;
    int next = top - skip;
    auto issue = [&](int buffer) {
        const int rows = w.rows - next;
        lq.issue(q_at, q_bytes, rows, ldsQ + buffer * kTile, wave, a.dim);
        ld.issue(d_at, d_bytes, rows, ldsD + buffer * kTile, wave, a.dim);
        if (wave == 0) load_4(r_last + (next - top) - max((lane & 31) - (rows - 1), 0), ldsR + buffer * 256);
        next -= kQ;
        q_at -= (int64_t)kQ * a.q_token;
        d_at -= (int64_t)kQ * o_token;
        if (next < from * kQ) {
            next = top;
            q_at = q_last += a.q_head;
            d_at = d_last += a.dim;
            r_last += a.q_tokens;
        }
    };
    f32x16 dk[kB], dv[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[b][i] = dv[b][i] = 0.0f;
    const float c = a.scale * kLog2e;

    if (n > 0) issue(0);
    if (a.dim < DT && n > 0) {                       // values past the head's end: zeros, as nothing else clears them here
        wait_loads<0>();
        barrier();
        for (int e = lane; e < 32 * (DT / 8); e += 64)
            if (8 * (e % (DT / 8)) >= a.dim)
                *(u32x4*)(sV + wave * (32 * DT * 2) + place<DT>(e / (DT / 8), e % (DT / 8))) = u32x4{0, 0, 0, 0};
    }
    int rb = top - skip, left = n;
    // One tile, in a buffer that is known when this is compiled, so that the addresses
    // of all reads are a few registers and constants.
    auto work = [&](auto buffer, bool masked, int r0) __attribute__((always_inline)) {
        constexpr int B = decltype(buffer)::value;
        const uint8_t *tq = sQ + B * kTile, *td = sD + B * kTile, *tv = sV + wave * (32 * DT * 2);
        const float* tr = sR + B * 64 + 4 * h;
        const int lo = first - r0 - 4 * h, hi = last - r0 - 4 * h;
        f32x16 s, t;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = t[e] = 0.0f;
#pragma unroll
        for (int x = 0; x < kS; ++x) s = product32<T>(read_along<DT>(tq, 0, x, lane), k[x], s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x4 ref = *(const f32x4*)(tr + 32 + 8 * e);
#pragma unroll
            for (int y = 0; y < 4; ++y) s[4 * e + y] = exp2_fast(fmaf(s[4 * e + y], c, -ref[y]));
        }
        if (masked) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 8 * (e / 4) + e % 4;
                s[e] = (r >= lo) & (r <= hi) ? s[e] : 0.0f;
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            u32x4 pt;
#pragma unroll
            for (int y = 0; y < 4; ++y) pt[y] = pack2<T>(s[8 * x + 2 * y], s[8 * x + 2 * y + 1]);
#pragma unroll
            for (int y = 0; y < kB; ++y) dv[y] = product32<T>(read_across<DT>(td, 16 * x, y, lane), pt, dv[y]);
        }
#pragma unroll
        for (int x = 0; x < kS; ++x) t = product32<T>(read_along<DT>(td, 0, x, lane), read_along<DT>(tv, 0, x, lane), t);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x4 delta = *(const f32x4*)(tr + 8 * e);
#pragma unroll
            for (int y = 0; y < 4; ++y) s[4 * e + y] *= t[4 * e + y] - delta[y];
        }
        if (masked) {                                // (0 times what is not finite)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 8 * (e / 4) + e % 4;
                s[e] = (r >= lo) & (r <= hi) ? s[e] : 0.0f;
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            u32x4 ds, rest;
            two_numbers<T>(s, x, ds, rest);
#pragma unroll
            for (int y = 0; y < kB; ++y) {
                const u32x4 f = read_across<DT>(tq, 16 * x, y, lane);
                dk[y] = product32<T>(f, ds, dk[y]);
                dk[y] = product32<T>(f, rest, dk[y]);
            }
        }
    };
    auto turn = [&](auto buffer) __attribute__((always_inline)) {
        wait_loads<0>();
        barrier();
        if (left > 1) issue(decltype(buffer)::value ^ 1);
        const int r0 = rb;
        rb = rb > from * kQ ? rb - kQ : top;
        if (r0 + kQ <= some_lo || r0 >= some_hi) return;
        work(buffer, r0 < all_lo || r0 + kQ > all_hi, r0);
    };
    while (left > 0) {
        turn(std::integral_constant<int, 0>{});
        if (--left == 0) break;
        turn(std::integral_constant<int, 1>{});
        --left;
    }
    if (key >= w.keys || (is_far && key >= sees.sinks)) return;
    if (staged) {
        const int64_t row = is_far ? item * a.sinks + key : at;
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 32 * b + 8 * e + 4 * h;
                if (d < a.dim) {
                    *(f32x4*)(part_dk + row * token + d) = f32x4{dk[b][4 * e], dk[b][4 * e + 1], dk[b][4 * e + 2], dk[b][4 * e + 3]};
                    *(f32x4*)(part_dv + row * token + d) = f32x4{dv[b][4 * e], dv[b][4 * e + 1], dv[b][4 * e + 2], dv[b][4 * e + 3]};
                }
            }
    } else {
        store_column<T, DT>(dk_head + at * g.dk_token, dk, a.scale, a.dim);
        store_column<T, DT>(dv_head + at * g.dv_token, dv, 1.0f, a.dim);
    }
}

// The sinks' parts from the rows far from them, in their order, added to the first part of
// the rest; a thread four elements of both.
__global__ __launch_bounds__(kAttnThreads) void attention_sink_sum_kernel(ue5m3_attention_t a, ue5m3_attention_grad_t g, int parts,
                                                                         int far) {
    const int64_t n = far_floats(a), i = ((int64_t)blockIdx.x * kAttnThreads + threadIdx.x) * 4;
    if (i >= n) return;
    const int64_t token = (int64_t)a.kv_heads * a.dim, row = i / token, seq = row / a.sinks, key = row - seq * a.sinks;
    const Span w = span_of(seq, a.sequences, a.q_starts, a.k_starts, a.q_tokens, a.k_tokens);
    if (key >= w.keys) return;
    const float* p = dkv_parts(a, g) + parts * 2 * dkv_floats(a) + i;
    float* const to = dkv_parts(a, g) + (w.k0 + key) * token + i % token;
    f32x4 dk = *(const f32x4*)to, dv = *(const f32x4*)(to + dkv_floats(a));
#pragma unroll 8
    for (int k = 0; k < far; ++k, p += 2 * n) {
        dk += *(const f32x4*)p;
        dv += *(const f32x4*)(p + n);
    }
    *(f32x4*)to = dk;
    *(f32x4*)(to + dkv_floats(a)) = dv;
}

// dK and dV from their parts, in their order; a thread four elements of both.
template <typename T>
__global__ __launch_bounds__(kAttnThreads) void attention_dkv_sum_kernel(ue5m3_attention_t a, ue5m3_attention_grad_t g, int parts) {
    const int64_t n = dkv_floats(a), i = ((int64_t)blockIdx.x * kAttnThreads + threadIdx.x) * 4;
    if (i >= n) return;
    const float* p = dkv_parts(a, g) + i;
    f32x4 dk = {0, 0, 0, 0}, dv = {0, 0, 0, 0};
    for (int k = 0; k < parts; ++k, p += 2 * n) {
        dk += *(const f32x4*)p;
        dv += *(const f32x4*)(p + n);
    }
    const int64_t row = i / a.dim, token = row / a.kv_heads;
    const int d = (int)(i - row * a.dim), kv = (int)(row - token * a.kv_heads);
    dk *= a.scale;
    const u32x2 k2 = {pack2<T>(dk[0], dk[1]), pack2<T>(dk[2], dk[3])}, v2 = {pack2<T>(dv[0], dv[1]), pack2<T>(dv[2], dv[3])};
    __builtin_memcpy((T*)g.dk + token * g.dk_token + kv * g.dk_head + d, &k2, 8);
    __builtin_memcpy((T*)g.dv + token * g.dv_token + kv * g.dv_head + d, &v2, 8);
}

// Calls f(null pointer of the type, the padded head size).
template <typename T, typename F>
hipError_t with_size(T* t, int dim, F&& f) {
    return dim <= 64 ? f(t, std::integral_constant<int, 64>{}) : f(t, std::integral_constant<int, 128>{});
}
template <typename F>
hipError_t with_head(DType type, int dim, F&& f) {
    return type == DType::BF16 ? with_size((bf16*)nullptr, dim, f) : with_size((f16*)nullptr, dim, f);
}

}  // namespace

// (of ragged ones one more, for rows of none)
int64_t attention_items(int64_t tokens, int64_t sequences, bool ragged) {
    return ragged ? tokens / kRows + sequences + 1 : sequences * ((tokens / sequences + kRows - 1) / kRows);
}

// Parts that the keys of a query tile are cut into: two workgroups for each CU where there
// are fewer tiles than that, and 8 tiles of keys for each by the sequences' mean length
// (777 queries over 5001 keys, 32 heads: one part 145 us, two 106 with their joining).
int attention_parts(const ue5m3_attention_t& a) {
    if (a.q_tokens == 0 || a.k_tokens == 0) return 1;
    const int64_t work = std::max<int64_t>((a.q_tokens + kRows - 1) / kRows, a.sequences) * a.q_heads;
    int64_t keys = a.k_tokens / a.sequences;
    if (a.causal && a.window != 0) keys = std::min(keys, std::min(a.window, keys) + std::min(a.sinks, keys) + kRows);
    return (int)std::max<int64_t>(1, std::min<int64_t>({8, 2 * kCus / work, keys / (8 * kKeys)}));
}

int64_t attention_scratch(const ue5m3_attention_t& a) {
    const int parts = attention_parts(a);
    return parts > 1 ? parts * (o_floats(a) + 2 * a.q_heads * a.q_tokens) * 4 : 0;
}

hipError_t launch_attention(const ue5m3_attention_t& a, float* scratch, hipStream_t s) {
    const int64_t items = attention_items(a.q_tokens, a.sequences, a.q_starts != nullptr);
    const int parts = attention_parts(a);
    return with_head((DType)a.type, a.dim, [&](auto* t, auto d) {
        using T = std::remove_pointer_t<decltype(t)>;
        hipLaunchKernelGGL((attention_kernel<T, decltype(d)::value>), dim3((unsigned)(items * parts * a.q_heads)),
                           dim3(kAttnThreads), 0, s, a, (int)items, parts, scratch);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || parts == 1) return e;
        const int64_t threads = (o_floats(a) + 3) / 4;
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3((unsigned)((threads + kAttnThreads - 1) / kAttnThreads)),
                           dim3(kAttnThreads), 0, s, a, parts, scratch);
        return hipGetLastError();
    });
}

// Parts that a key tile's queries are cut into.  Causal tiles differ in length, and two
// workgroups run on a CU: with four for each CU, the longest first, all CUs end together
// (8192 tokens, 8 key-value heads, dS in one number: one part 2041 us, two 1241 with their
// sum).  A part has
// 16 tiles of queries at least, by the sequences' mean length.
int dkv_parts_of(const ue5m3_attention_t& a) {
    if (a.q_tokens == 0 || a.k_tokens == 0) return 1;
    const int64_t tiles = std::max<int64_t>((a.k_tokens + kRows - 1) / kRows, a.sequences), work = tiles * a.kv_heads;
    const int64_t rows = a.q_tokens / a.sequences, turns = (rows + 31) / 32 * (a.q_heads / a.kv_heads);
    return (int)std::max<int64_t>(1, std::min<int64_t>({8, (4 * kCus + work - 1) / work, turns / 16}));
}

// Parts that the rows are cut into that see of a sequence's first tile the sinks only (0:
// they stay with the others): of the longest that a sequence can be, about as many turns
// each as a part of the other tiles has, two for each sequence at least, and no more of
// them than memory for two parts of all keys holds (8192 tokens, window 1024, 4 sinks, 32
// heads of 128, 8 of keys, forward and gradients, dS of dK in one number: 1550 us with them
// among the others, 899 apart; 16 heads of 64 494 and 303).
int far_parts_of(const ue5m3_attention_t& a, int parts) {
    if (!a.causal || a.window == 0 || a.sinks == 0 || a.sinks > kRows || a.sequences * a.kv_heads >= 1 << 21) return 0;
    const int64_t n = a.q_starts != nullptr ? 1 : a.sequences, group = a.q_heads / a.kv_heads;
    const int64_t keys = a.k_tokens / n, window = std::min(a.window, keys), rows = std::min(a.q_tokens / n, keys - window - kRows);
    if (rows <= 0) return 0;
    const int64_t turns = (window + kRows) / 32 * group / parts, want = rows / 32 * group / std::max<int64_t>(turns, 16);
    const int64_t room = 2 * a.k_tokens / (a.sequences * a.sinks);
    const int64_t far = std::min<int64_t>({want, room, 64, std::max<int64_t>(2, 4 * kCus / (a.sequences * a.kv_heads))});
    return far < 2 ? 0 : (int)far;
}

int64_t attention_grad_scratch(const ue5m3_attention_t& a) {
    const int parts = dkv_parts_of(a), far = far_parts_of(a, parts);
    const int64_t sinks = far > 0 ? 2 * far * far_floats(a) : 0;     // (any number of sinks may be asked for where there are none)
    return (delta_floats(a) + (parts > 1 || far > 0 ? 2 * parts * dkv_floats(a) + sinks : 0)) * 4;
}

hipError_t launch_attention_grad(const ue5m3_attention_t& a, const ue5m3_attention_grad_t& g, hipStream_t s) {
    const int64_t rows = attention_items(a.q_tokens, a.sequences, a.q_starts != nullptr);
    const int64_t keys = attention_items(a.k_tokens, a.sequences, a.k_starts != nullptr);
    const int parts = dkv_parts_of(a), far = far_parts_of(a, parts);
    return with_size((bf16*)nullptr, a.dim, [&](auto* t, auto d) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int DT = decltype(d)::value;
        hipError_t e = hipSuccess;
        if (a.q_tokens > 0) {
            hipLaunchKernelGGL((attention_dq_kernel<T, DT>), dim3((unsigned)(rows * a.q_heads)), dim3(kAttnThreads), 0, s, a,
                               g, (int)rows);
            e = hipGetLastError();
        }
        if (e != hipSuccess || g.dk == nullptr || a.k_tokens == 0) return e;
        hipLaunchKernelGGL((attention_dkv_kernel<T, DT>), dim3((unsigned)((keys * parts + far * a.sequences) * a.kv_heads)),
                           dim3(kAttnThreads), 0, s, a, g, (int)keys, parts, far);
        e = hipGetLastError();
        if (e == hipSuccess && far > 0) {
            const int64_t threads = far_floats(a) / 4;
            hipLaunchKernelGGL(attention_sink_sum_kernel, dim3((unsigned)((threads + kAttnThreads - 1) / kAttnThreads)),
                               dim3(kAttnThreads), 0, s, a, g, parts, far);
            e = hipGetLastError();
        }
        if (e != hipSuccess || (parts == 1 && far == 0)) return e;
        const int64_t threads = (dkv_floats(a) + 3) / 4;
        hipLaunchKernelGGL((attention_dkv_sum_kernel<T>), dim3((unsigned)((threads + kAttnThreads - 1) / kAttnThreads)),
                           dim3(kAttnThreads), 0, s, a, g, parts);
        return hipGetLastError();
    });
}

}  // namespace ue5m3
