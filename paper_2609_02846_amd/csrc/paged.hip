// Attention of one new token for each of several sequences over the pages of a
// cache: the softmax over the keys that the token sees (all of its sequence's, or
// under a window the last `window` and the `sinks` first ones) times their values.
//
// A workgroup takes up to 16 query heads that share a key-value head, and one part
// of a sequence's tiles of 32 keys; its four waves take every fourth tile.  The
// scores are 16 x 16 x 32 products with the queries as the columns (heads of one
// key-value head fill them up to 16); keys go from HBM to registers as that
// product's operand, values to LDS, whence they are read transposed.  Both are
// loaded a tile ahead, their pages' numbers two.  P is rounded to the queries' type,
// as the matrix instructions take it, and its product is divided by the sum of the
// rounded values, as the prompt's attention does it: a row's weights add up to one.  Parts
// are joined by a second launch, in their order.
//
// Bound: HBM, each key and value read once.  One token over 32768 of 8 heads of 128
// (134 MB): 26.4 us, 5.1 TB/s, what a copy reaches, and 5.0 for the joining; 24 rows of
// up to 8191 (232 MB): 62 us, 3.7 TB/s, as parts are cut by the table's width: the short
// rows' end early and leave CUs idle (24 rows of 8192: 157 us, 5.1 TB/s).  On a cache that
// lies in the chip's own one: the 24 rows 54 us, under a window of 1024 with 4 sinks 21 (62
// MB), with heads of 80 46 (145 MB), of 64 31 (116 MB).
#include <algorithm>

#include "attention.hpp"
#include "attn_tile.hpp"

namespace ue5m3 {
namespace {

constexpr int kWaves = 4, kTileKeys = 32, kCols = 16;
constexpr int kLeastKeys = 512;                      // of a part: four tiles a wave
constexpr int kMaxParts = 128, kMaxHead = 128;

// Chunk c of a row of the values' tile lies at c ^ place: reads across rows take 32
// bytes of 16 of them.
template <int DT>
__device__ __forceinline__ int value_swizzle(int row) { return DT == 128 ? (row & 7) << 1 : (row >> 1 & 3) << 1; }

// The keys of a row of the batch, as two ranges [0, first) and [from, to).
struct Seen {
    int first, from, to, tiles_first, tiles;
    __device__ __forceinline__ Seen(int length, int64_t window, int64_t sinks) {
        to = length;
        from = window != 0 && window < length ? length - (int)window : 0;
        first = (int)min(sinks, (int64_t)from);
        tiles_first = (first + kTileKeys - 1) / kTileKeys;
        tiles = tiles_first + (to - from + kTileKeys - 1) / kTileKeys;
    }
    // Tile t: its first key and the end of its range.
    __device__ __forceinline__ void tile(int t, int& j, int& end) const {
        const bool a = t < tiles_first;
        j = a ? t * kTileKeys : from + (t - tiles_first) * kTileKeys;
        end = a ? first : to;
    }
};

template <typename T, int DT>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_kernel(ue5m3_paged_attention_t a, int parts, int blocks,
                                                                        float* part_o, float* part_ml) {
    constexpr int kS = DT / 32, kB = DT / 16, kChunks = DT / 8, kTile = kTileKeys * DT * 2, kLoads = kTile / 1024;
    __shared__ __attribute__((aligned(16))) uint8_t sV[kWaves * 2 * kTile];
    __shared__ float sM[kWaves][kCols], sL[kWaves][kCols];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), col = lane & 15, g = lane >> 4;
    const int group = a.q_heads / a.kv_heads;
    // (key-value heads innermost: neighbours in memory run together, one on each XCD)
    int id = blockIdx.x;
    const int kv = id % a.kv_heads;
    id /= a.kv_heads;
    const int block = id % blocks;
    id /= blocks;
    const int part = id % parts;
    const int64_t row = id / parts;

    const int shift = __builtin_ctz(a.cache.page_size);
    const int64_t capacity = a.width << shift;
    const int asked = a.lengths[row], length = (int)min((int64_t)max(asked, 0), capacity);
    bool bad = asked > length;                       // longer than its pages
    const Seen seen(length, a.window, a.sinks);
    const int t0 = (int)((int64_t)seen.tiles * part / parts), t1 = (int)((int64_t)seen.tiles * (part + 1) / parts);

    const int head = kv * group + block * kCols + col;
    const bool has = block * kCols + col < group;
    u32x4 q[kS];
    {
        const uint16_t* p = (const uint16_t*)a.q + row * a.q_token + head * a.q_head;
#pragma unroll
        for (int s = 0; s < kS; ++s) {
            q[s] = u32x4{0, 0, 0, 0};
            if (has && 32 * s + 8 * g < a.dim) __builtin_memcpy(&q[s], p + 32 * s + 8 * g, 16);
        }
    }
    const int32_t* const table = a.table + row * a.table_row;
    const int mask = a.cache.page_size - 1;
    const uint16_t* const k_head = (const uint16_t*)a.cache.k + kv * a.cache.head;
    const uint16_t* const v_head = (const uint16_t*)a.cache.v + kv * a.cache.head;
    // Element offset of key j's row, whose page's number is n; a number outside the
    // cache is noted, and page 0 read.
    auto offset = [&](int j, int n) {
        const bool ok = (uint32_t)n < (uint64_t)a.cache.pages;
        bad |= !ok;
        return (int64_t)(ok ? n : 0) * a.cache.page + (int64_t)(j & mask) * a.cache.token;
    };
    // Keys of a tile that a lane needs: two for its operand of the scores, kLoads for
    // the values (the last key of the range in the place of those past it).
    struct Pages2 {
        int k[2], v[kLoads];
    };
    auto key_at = [&](int j, int end, int i) { return min(j + i, end - 1); };
    auto value_row = [&](int n) { return n * (64 / kChunks) + lane / kChunks; };
    auto numbers = [&](int t) {
        Pages2 n;
        int j, end;
        seen.tile(t, j, end);
#pragma unroll
        for (int i = 0; i < 2; ++i) n.k[i] = table[key_at(j, end, 16 * i + col) >> shift];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) n.v[i] = table[key_at(j, end, value_row(i)) >> shift];
        return n;
    };
    const uint32_t lds = lds_addr(sV) + wave * 2 * kTile;
    u32x4 k[2][kS];
    auto load = [&](int t, const Pages2& n, int buffer, u32x4 (&to)[2][kS]) {
        int j, end;
        seen.tile(t, j, end);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = value_row(i), c = lane % kChunks ^ value_swizzle<DT>(r);
            const int key = key_at(j, end, r);
            load_16(v_head + offset(key, n.v[i]) + (8 * c < a.dim ? 8 * c : 0), lds + buffer * kTile + i * 1024);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int key = key_at(j, end, 16 * i + col);
            const uint16_t* p = k_head + offset(key, n.k[i]);
#pragma unroll
            for (int s = 0; s < kS; ++s) __builtin_memcpy(&to[i][s], p + (32 * s + 8 * g < a.dim ? 32 * s + 8 * g : 0), 16);
        }
    };

    f32x4 o[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b) o[b] = f32x4{0, 0, 0, 0};
    const float c = a.scale * kLog2e;
    float m = -__builtin_inff(), sum = 0.0f;

    int t = t0 + wave, buffer = 0;
    if (t < t1) {
        const Pages2 first = numbers(t);
        load(t, first, 0, k);
        Pages2 next = first;
        if (t + kWaves < t1) next = numbers(t + kWaves);
        for (; t < t1; t += kWaves, buffer ^= 1) {
            u32x4 ahead[2][kS];
            Pages2 later = next;
            const bool more = t + kWaves < t1;
            if (more) {
                if (t + 2 * kWaves < t1) later = numbers(t + 2 * kWaves);
                load(t + kWaves, next, buffer ^ 1, ahead);
            }
            next = later;
            int j, end;
            seen.tile(t, j, end);
            f32x4 s[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s[i] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int x = 0; x < kS; ++x) s[i] = product16<T>(k[i][x], q[x], s[i]);
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = j + 16 * (e / 4) + 4 * g + e % 4;
                s[e / 4][e % 4] = key < end ? s[e / 4][e % 4] * c : -__builtin_inff();
                top = fmaxf(top, s[e / 4][e % 4]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, other_half(top));
            if (__ballot(top > m) != 0) {
                const float up = fmaxf(m, top), f = m == up ? 1.0f : exp2_fast(m - up);
                m = up;
                sum *= f;
#pragma unroll
                for (int b = 0; b < kB; ++b) o[b] *= f;
            }
            const float ref = m == -__builtin_inff() ? 0.0f : m;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = exp2_fast(s[e / 4][e % 4] - ref);
            const u32x4 pt = {pack2<T>(p[0], p[1]), pack2<T>(p[2], p[3]), pack2<T>(p[4], p[5]), pack2<T>(p[6], p[7])};
#pragma unroll
            for (int y = 0; y < 4; ++y) sum = add_pair<T>(pt[y], sum);
            // this tile's values are older than the next one's loads
            if (more) wait_loads<kLoads + 2 * kS>();
            else wait_loads<0>();
            typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
            const uint8_t* tv = sV + (wave * 2 + buffer) * kTile + 8 * (lane & 1);
            const int r = 4 * g + (lane >> 2 & 3);
#pragma unroll
            for (int b = 0; b < kB; ++b) {
                const int ch = 2 * b + (lane >> 1 & 1);
                const uint8_t* lo = tv + r * (2 * DT) + ((ch ^ value_swizzle<DT>(r)) << 4);
                const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)lo));
                const u32x2 y = __builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lo + 16 * (2 * DT))));   // (16 rows on: the same places)
                o[b] = product16<T>(u32x4{x[0], x[1], y[0], y[1]}, pt, o[b]);
            }
            // (read before the loads of the turn after next overwrite them)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 0; x < kS; ++x) k[i][x] = ahead[i][x];
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += other_half(sum);
    if (__ballot(bad) != 0) sum = __builtin_nanf("");

    // ---- the waves' parts, in their order ----
    __syncthreads();                                 // (values have been read)
    float* const so = (float*)sV;                    // [wave][col][DT]
    static_assert(kWaves * kCols * DT * 4 <= kWaves * 2 * kTile, "the waves' parts fit where the values were");
#pragma unroll
    for (int b = 0; b < kB; ++b) *(f32x4*)(so + (wave * kCols + col) * DT + 16 * b + 4 * g) = o[b];
    if (g == 0) sM[wave][col] = m, sL[wave][col] = sum;
    __syncthreads();
    const int heads = min(group - block * kCols, kCols);
    for (int i = threadIdx.x; i < heads * a.dim; i += 64 * kWaves) {
        const int hc = i / a.dim, d = i - hc * a.dim;
        float top = sM[0][hc];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sM[w][hc]);
        const float ref = top == -__builtin_inff() ? 0.0f : top;
        float v = 0.0f, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = exp2_fast(sM[w][hc] - ref);
            v += so[(w * kCols + hc) * DT + d] * f;
            l += sL[w][hc] * f;
        }
        const int64_t out = row * a.q_heads + kv * group + block * kCols + hc;
        if (parts == 1) {
            ((T*)a.o)[out * a.dim + d] = (T)(asked <= 0 ? 0.0f : v / l);     // (0 / 0 where all keys score -inf)
        } else {
            part_o[(out * parts + part) * a.dim + d] = v;
            if (d == 0) part_ml[(out * parts + part) * 2] = top, part_ml[(out * parts + part) * 2 + 1] = l;
        }
    }
}

// The parts of a head's output joined: a workgroup for each, its parts in eight
// groups (part mod 8) of 32 threads, four elements a thread; then the groups, in a
// fixed order.
constexpr int kJoinGroups = 8, kJoinThreads = 256;

template <typename T>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(const float* __restrict__ part_o,
                                                                  const float* __restrict__ part_ml, int parts, int dim,
                                                                  const int32_t* __restrict__ lengths, int q_heads,
                                                                  T* __restrict__ out) {
    __shared__ float so[kJoinGroups][kMaxHead], sl[kJoinGroups], sm[kMaxParts];
    const int64_t at = blockIdx.x;
    const float* ml = part_ml + at * parts * 2;
    const int group = threadIdx.x >> 5, d = 4 * (threadIdx.x & 31);
    if ((int)threadIdx.x < parts) sm[threadIdx.x] = ml[2 * threadIdx.x];
    __syncthreads();
    float top = -__builtin_inff();
    for (int p = 0; p < parts; ++p) top = fmaxf(top, sm[p]);
    const float ref = top == -__builtin_inff() ? 0.0f : top;
    f32x4 v = {0, 0, 0, 0};
    float l = 0.0f;
#pragma unroll 4
    for (int p = group; p < parts; p += kJoinGroups) {
        const float f = exp2_fast(sm[p] - ref);
        l += ml[2 * p + 1] * f;
        if (d < dim) v += *(const f32x4*)(part_o + (at * parts + p) * dim + d) * f;
    }
    if (d < dim) *(f32x4*)(&so[group][d]) = v;
    if (d == 0) sl[group] = l;
    __syncthreads();
    const int e = threadIdx.x;
    if (e >= dim) return;
    float o = 0.0f, sum = 0.0f;
#pragma unroll
    for (int g = 0; g < kJoinGroups; ++g) o += so[g][e], sum += sl[g];
    out[at * dim + e] = (T)(lengths[at / q_heads] <= 0 ? 0.0f : o / sum);
}

}  // namespace

// About eight workgroups for each CU, of rows that differ in length (24 rows of up to 8191
// tokens, 8 key-value heads: with two for each CU 81 us, four 63, eight 62, sixteen 66),
// and no part of fewer than 512 keys (one row of 32768: 64 parts 31.4 us, 128 of 256 keys
// 35, as they take longer to join).
int paged_parts(int64_t rows, int q_heads, int kv_heads, int64_t capacity, int64_t window, int64_t sinks) {
    const int group = q_heads / kv_heads;
    const int64_t work = rows * kv_heads * ((group + kCols - 1) / kCols);
    const int64_t keys = window != 0 ? std::min(capacity, std::min(window, capacity) + std::min(sinks, capacity)) : capacity;
    const int64_t most = std::min<int64_t>((keys + kLeastKeys - 1) / kLeastKeys, kMaxParts);
    return (int)std::max<int64_t>(1, std::min(most, 2048 / std::max<int64_t>(work, 1)));
}

int64_t paged_groups(int64_t rows, int q_heads, int kv_heads, int parts) {
    return rows * parts * kv_heads * ((q_heads / kv_heads + kCols - 1) / kCols);
}

hipError_t launch_paged_attention(const ue5m3_paged_attention_t& a, float* scratch, hipStream_t s) {
    const int blocks = (a.q_heads / a.kv_heads + kCols - 1) / kCols;
    const int parts = paged_parts(a.rows, a.q_heads, a.kv_heads, a.width * a.cache.page_size, a.window, a.sinks);
    float* const part_ml = scratch + a.rows * a.q_heads * parts * a.dim;
    const dim3 grid((unsigned)paged_groups(a.rows, a.q_heads, a.kv_heads, parts)), threads(64 * kWaves);
    auto run = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (a.dim <= 64)
            hipLaunchKernelGGL((paged_attention_kernel<T, 64>), grid, threads, 0, s, a, parts, blocks, scratch, part_ml);
        else
            hipLaunchKernelGGL((paged_attention_kernel<T, 128>), grid, threads, 0, s, a, parts, blocks, scratch, part_ml);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && parts > 1) {
            hipLaunchKernelGGL((paged_join_kernel<T>), dim3((unsigned)(a.rows * a.q_heads)), dim3(kJoinThreads), 0, s, scratch,
                               part_ml, parts, a.dim, a.lengths, a.q_heads, (T*)a.o);
            e = hipGetLastError();
        }
        return e;
    };
    return a.type == UE5M3_BF16 ? run((bf16*)nullptr) : run((f16*)nullptr);
}

}  // namespace ue5m3
