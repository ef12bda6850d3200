// C ABI shim of the operators between the QKV and the output projection: argument
// validation, status mapping and dispatch.  See include/ue5m3.h for the contract of
// every entry point.
#include <cmath>
#include <cstdint>
#include <new>

#include "attention.hpp"

namespace {

constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;   // workgroups of 256 threads a launch takes
constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr int32_t kMaxHeads = 1 << 16;
constexpr int64_t kMaxStride = (int64_t)1 << 23;       // a tile's rows stay within 32-bit offsets
constexpr int64_t kMaxPages = (int64_t)1 << 31;        // a page's number has 31 bits

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline ue5m3_status_t status(hipError_t e) { return e == hipSuccess ? UE5M3_OK : UE5M3_EHIP; }
inline bool known(ue5m3_dtype_t t) { return t == UE5M3_BF16 || t == UE5M3_F16 || t == UE5M3_F32; }
inline uintptr_t size_of(ue5m3_dtype_t t) { return t == UE5M3_F32 ? 4 : 2; }
inline bool power_of_two(int32_t n) { return n > 0 && (n & (n - 1)) == 0; }
inline bool flag(int32_t f) { return f == 0 || f == 1; }

// What every rotation call checks; `append`: no queries, or nothing but a copy, are
// fine.
ue5m3_status_t rope_args(const ue5m3_rope_t* a, bool append) {
    if (a == nullptr || !known(a->type) || !known(a->weight_type) ||
        (a->weight_type != a->type && a->weight_type != UE5M3_F32) || !flag(a->norm) || !flag(a->interleaved))
        return UE5M3_EINVAL;
    if (a->tokens < 0 || a->tokens > (int64_t)1 << 40 || a->q_heads < (append ? 0 : 1) ||
        a->q_heads > kMaxHeads || a->kv_heads < 0 ||
        a->kv_heads > kMaxHeads || a->dim < 1 || a->dim > ue5m3::kMaxRopeDim || a->pairs < 0 || a->pairs > a->dim / 2)
        return UE5M3_ESHAPE;
    if (!append && !a->norm && a->pairs == 0) return UE5M3_EINVAL;
    if (a->norm && (!(a->eps >= 0.0f) || !std::isfinite(a->eps))) return UE5M3_EINVAL;
    if (a->pairs > 0 && (!std::isfinite(a->amplitude) || (a->positions == nullptr && a->period < 1))) return UE5M3_EINVAL;
    return UE5M3_OK;
}

ue5m3_status_t rope_pointers(const ue5m3_rope_t* a) {
    if ((a->q_heads > 0 && a->q == nullptr) || (a->kv_heads > 0 && a->k == nullptr) || (a->pairs > 0 && a->freqs == nullptr)) return UE5M3_EINVAL;
    const uintptr_t n = size_of(a->type), w = size_of(a->weight_type);
    if (!aligned(a->q, n) || !aligned(a->k, n) || !aligned(a->q_out, n) || !aligned(a->k_out, n) ||
        !aligned(a->q_weight, w) || !aligned(a->k_weight, w) || !aligned(a->freqs, 4) || !aligned(a->positions, 8))
        return UE5M3_EALIGN;
    return UE5M3_OK;
}

// The stride of n things: of one it reaches nothing and may be any number.
inline int64_t used(int64_t stride, int64_t n) { return n > 1 ? stride : 0; }

// A cache of 16-bit or 32-bit elements, `multiple` of which its strides are multiples of.
ue5m3_status_t cache_args(const ue5m3_pages_t* c, int32_t heads, int64_t multiple) {
    if (c == nullptr || !power_of_two(c->page_size)) return UE5M3_EINVAL;
    if (c->pages < 0 || c->pages > kMaxPages) return UE5M3_ESHAPE;
    if ((used(c->page, c->pages) | used(c->token, c->page_size) | used(c->head, heads)) % multiple != 0) return UE5M3_EALIGN;
    return UE5M3_OK;
}

bool stride_ok(int64_t token, int64_t head, int32_t dim, int64_t tokens, int32_t heads) {
    return (tokens <= 1 || (token >= dim && token < kMaxStride)) && (heads <= 1 || head >= dim);
}

// Sizes and types of attention over heads.
ue5m3_status_t head_args(ue5m3_dtype_t type, int32_t q_heads, int32_t kv_heads, int32_t dim, float scale, int64_t window,
                         int64_t sinks) {
    if ((type != UE5M3_BF16 && type != UE5M3_F16) || !(scale > 0.0f) || !std::isfinite(scale)) return UE5M3_EINVAL;
    if (q_heads < 1 || q_heads > kMaxHeads || kv_heads < 1 || q_heads % kv_heads != 0 || dim < 8 || dim > 128 ||
        dim % 8 != 0 || window < 0 || sinks < 0)
        return UE5M3_ESHAPE;
    return UE5M3_OK;
}

ue5m3_status_t attention_args(const ue5m3_attention_t* a) {
    if (a == nullptr) return UE5M3_EINVAL;
    const ue5m3_status_t st = head_args(a->type, a->q_heads, a->kv_heads, a->dim, a->scale, a->window, a->sinks);
    if (st != UE5M3_OK) return st;
    if (!flag(a->causal) || (!a->causal && a->window != 0) || (a->q_starts == nullptr) != (a->k_starts == nullptr))
        return UE5M3_EINVAL;
    if (a->q_tokens < 0 || a->k_tokens < 0 || a->q_tokens > kMaxTokens || a->k_tokens > kMaxTokens || a->sequences < 1 ||
        a->sequences > kMaxTokens)
        return UE5M3_ESHAPE;
    if (a->q_starts == nullptr && (a->q_tokens % a->sequences != 0 || a->k_tokens % a->sequences != 0)) return UE5M3_ESHAPE;
    if (!stride_ok(a->q_token, a->q_head, a->dim, a->q_tokens, a->q_heads) ||
        !stride_ok(a->k_token, a->k_head, a->dim, a->k_tokens, a->kv_heads) ||
        !stride_ok(a->v_token, a->v_head, a->dim, a->k_tokens, a->kv_heads) ||
        (int64_t)a->q_heads * a->dim >= kMaxStride)
        return UE5M3_ESHAPE;
    const bool ragged = a->q_starts != nullptr;
    if (ue5m3::attention_items(a->q_tokens, a->sequences, ragged) > kMaxGrid / 8 / a->q_heads ||
        ue5m3::attention_items(a->k_tokens, a->sequences, ragged) > kMaxGrid / 8 / a->kv_heads ||
        (a->q_tokens / 32 + 2) * (a->q_heads / a->kv_heads) > 0x7FFFFFFF)
        return UE5M3_ESHAPE;
    if (a->q_tokens > 0 && (a->q == nullptr || a->o == nullptr)) return UE5M3_EINVAL;
    if (a->k_tokens > 0 && (a->k == nullptr || a->v == nullptr)) return UE5M3_EINVAL;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->o, 16) || !aligned(a->o_rest, 16) || !aligned(a->lse, 4) ||
        !aligned(a->q_starts, 4) || !aligned(a->k_starts, 4) ||
        (used(a->q_token, a->q_tokens) | used(a->q_head, a->q_heads) | used(a->k_token, a->k_tokens) |
         used(a->k_head, a->kv_heads) | used(a->v_token, a->k_tokens) | used(a->v_head, a->kv_heads)) % 8 != 0)
        return UE5M3_EALIGN;
    return UE5M3_OK;
}

// Whether the sizes that scratch memory goes by are such.
bool sizes_ok(const ue5m3_attention_t* a) {
    return a != nullptr && a->q_tokens >= 0 && a->q_tokens <= kMaxTokens && a->k_tokens >= 0 && a->k_tokens <= kMaxTokens &&
           a->sequences >= 1 && a->sequences <= kMaxTokens && a->q_heads >= 1 && a->q_heads <= kMaxHeads && a->kv_heads >= 1 && a->kv_heads <= a->q_heads &&
           a->dim >= 1 && a->dim <= 128 && a->window >= 0 && a->sinks >= 0;
}

}  // namespace

extern "C" {

ue5m3_status_t ue5m3_qk_norm_rope(const ue5m3_rope_t* args, hipStream_t stream) {
    ue5m3_status_t st = rope_args(args, false);
    if (st != UE5M3_OK || args->tokens == 0) return st;
    if ((st = rope_pointers(args)) != UE5M3_OK) return st;
    if (args->q_out == nullptr || (args->kv_heads > 0 && args->k_out == nullptr)) return UE5M3_EINVAL;
    return status(ue5m3::launch_rope(*args, nullptr, stream));
}

int64_t ue5m3_qk_norm_rope_grad_scratch(int64_t tokens, int32_t heads, int32_t dim) {
    if (tokens <= 0 || heads <= 0 || dim <= 0) return 0;
    return (int64_t)ue5m3::rope_grad_rows(tokens, heads) * 2 * dim * 4;
}

ue5m3_status_t ue5m3_qk_norm_rope_grad(const ue5m3_rope_t* args, const void* dq_rotated, const void* dk_rotated,
                                       void* dq_weight, void* dk_weight, void* scratch, hipStream_t stream) {
    ue5m3_status_t st = rope_args(args, false);
    if (st != UE5M3_OK) return st;
    const bool sums = dq_weight != nullptr || dk_weight != nullptr;
    if (sums && !args->norm) return UE5M3_EINVAL;
    if (!aligned(dq_weight, size_of(args->weight_type)) || !aligned(dk_weight, size_of(args->weight_type)) ||
        !aligned(scratch, 16))
        return UE5M3_EALIGN;
    if (args->tokens > 0) {
        // (without the norm q and k are not read)
        ue5m3_rope_t p = *args;
        if (!args->norm) p.q = p.k = dq_rotated != nullptr ? dq_rotated : dk_rotated;
        if ((st = rope_pointers(&p)) != UE5M3_OK) return st;
        if (dq_rotated == nullptr || (args->kv_heads > 0 && dk_rotated == nullptr) || (sums && scratch == nullptr))
            return UE5M3_EINVAL;
        if (!aligned(dq_rotated, size_of(args->type)) || !aligned(dk_rotated, size_of(args->type))) return UE5M3_EALIGN;
    }
    return status(ue5m3::launch_rope_grad(*args, dq_rotated, dk_rotated, dq_weight, dk_weight, (float*)scratch, stream));
}

ue5m3_status_t ue5m3_qk_norm_rope_append(const ue5m3_rope_t* args, const void* v, int64_t v_token, int64_t v_head,
                                         const ue5m3_pages_t* cache, const int64_t* slots, hipStream_t stream) {
    ue5m3_status_t st = rope_args(args, true);
    if (st != UE5M3_OK) return st;
    if ((st = cache_args(cache, args->kv_heads, 1)) != UE5M3_OK) return st;
    if (args->kv_heads < 1) return UE5M3_ESHAPE;
    if (args->tokens == 0) return UE5M3_OK;
    if ((st = rope_pointers(args)) != UE5M3_OK) return st;
    if ((args->q_heads > 0 && args->q_out == nullptr) || v == nullptr || slots == nullptr ||
        (cache->pages > 0 && (cache->k == nullptr || cache->v == nullptr)))
        return UE5M3_EINVAL;
    const uintptr_t n = size_of(args->type);
    if (!aligned(v, n) || !aligned(cache->k, n) || !aligned(cache->v, n) || !aligned(slots, 8)) return UE5M3_EALIGN;
    const ue5m3::Append ap{v, v_token, v_head, slots, *cache};
    return status(ue5m3::launch_rope(*args, &ap, stream));
}

ue5m3_status_t ue5m3_copy_pages(void* base, int64_t planes, int64_t plane, int64_t pages, int64_t page,
                                const int32_t* src, const int32_t* dst, int64_t n, hipStream_t stream) {
    if (planes < 0 || plane < 0 || pages < 0 || page < 0 || n < 0 || pages > kMaxPages || n > pages) return UE5M3_ESHAPE;
    if (plane % 2 != 0 || page % 2 != 0) return UE5M3_ESHAPE;
    if (page > 0 && (pages > INT64_MAX / page || (planes > 1 && pages * page > plane))) return UE5M3_ESHAPE;
    if (n == 0) return UE5M3_OK;
    if (src == nullptr || dst == nullptr) return UE5M3_EINVAL;
    // which pages are written: none twice, and none that is read
    uint8_t* const written = new (std::nothrow) uint8_t[(size_t)pages]();
    if (written == nullptr) return UE5M3_EHIP;
    bool ok = true;
    for (int64_t i = 0; i < n && ok; ++i) {
        ok = src[i] >= 0 && src[i] < pages && dst[i] >= 0 && dst[i] < pages && written[dst[i]] == 0;
        if (ok) written[dst[i]] = 1;
    }
    for (int64_t i = 0; i < n && ok; ++i) ok = written[src[i]] == 0;
    delete[] written;
    if (!ok) return UE5M3_EINVAL;
    if (planes == 0 || page == 0) return UE5M3_OK;
    if (base == nullptr) return UE5M3_EINVAL;
    if (!aligned(base, 2)) return UE5M3_EALIGN;
    return status(ue5m3::launch_copy_pages(base, planes, plane, page, src, dst, n, stream));
}

ue5m3_status_t ue5m3_attention(const ue5m3_attention_t* args, void* scratch, hipStream_t stream) {
    const ue5m3_status_t st = attention_args(args);
    if (st != UE5M3_OK || args->q_tokens == 0) return st;
    if (ue5m3::attention_scratch(*args) > 0 && scratch == nullptr) return UE5M3_EINVAL;
    if (!aligned(scratch, 16)) return UE5M3_EALIGN;
    return status(ue5m3::launch_attention(*args, (float*)scratch, stream));
}

int64_t ue5m3_attention_scratch(const ue5m3_attention_t* args) {
    return sizes_ok(args) ? ue5m3::attention_scratch(*args) : 0;
}

int64_t ue5m3_attention_grad_scratch(const ue5m3_attention_t* args) {
    return sizes_ok(args) ? ue5m3::attention_grad_scratch(*args) : 0;
}

ue5m3_status_t ue5m3_attention_grad(const ue5m3_attention_t* args, const ue5m3_attention_grad_t* grad,
                                    hipStream_t stream) {
    const ue5m3_status_t st = attention_args(args);
    if (st != UE5M3_OK) return st;
    if (grad == nullptr || (grad->dk == nullptr) != (grad->dv == nullptr) || args->type != UE5M3_BF16) return UE5M3_EINVAL;
    const ue5m3_attention_grad_t& g = *grad;
    if (ue5m3::attention_grad_scratch(*args) > 0 && g.scratch == nullptr) return UE5M3_EINVAL;
    if (args->q_tokens > 0 && (g.d_o == nullptr || args->lse == nullptr || args->o_rest == nullptr)) return UE5M3_EINVAL;
    if (!aligned(g.d_o, 16) || !aligned(g.scratch, 16) || !aligned(g.dq, 16) || !aligned(g.dk, 16) || !aligned(g.dv, 16) ||
        (g.dq != nullptr && (g.dq_token | g.dq_head) % 8 != 0) ||
        (g.dk != nullptr && (g.dk_token | g.dk_head | g.dv_token | g.dv_head) % 8 != 0))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_attention_grad(*args, g, stream));
}

int64_t ue5m3_paged_attention_scratch(int64_t rows, int32_t q_heads, int32_t kv_heads, int32_t dim, int64_t capacity,
                                      int64_t window, int64_t sinks) {
    if (rows <= 0 || q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads != 0 || dim <= 0 || capacity <= 0 || window < 0 ||
        sinks < 0)
        return 0;
    const int parts = ue5m3::paged_parts(rows, q_heads, kv_heads, capacity, window, sinks);
    return parts == 1 ? 0 : rows * q_heads * parts * (dim + 2) * 4;
}

ue5m3_status_t ue5m3_paged_attention(const ue5m3_paged_attention_t* args, void* scratch, hipStream_t stream) {
    if (args == nullptr) return UE5M3_EINVAL;
    const ue5m3_paged_attention_t& a = *args;
    ue5m3_status_t st = head_args(a.type, a.q_heads, a.kv_heads, a.dim, a.scale, a.window, a.sinks);
    if (st != UE5M3_OK) return st;
    if ((st = cache_args(&a.cache, a.kv_heads, 8)) != UE5M3_OK) return st;
    if (a.rows < 0 || a.rows > kMaxTokens || a.width < 0 || a.width > kMaxTokens / a.cache.page_size ||
        (a.rows > 1 && a.table_row < a.width) || (a.rows > 0 && a.width > 0 && a.cache.pages < 1))
        return UE5M3_ESHAPE;
    if (a.rows == 0) return UE5M3_OK;
    const int64_t capacity = a.width * a.cache.page_size;
    const int parts = ue5m3::paged_parts(a.rows, a.q_heads, a.kv_heads, capacity, a.window, a.sinks);
    if (ue5m3::paged_groups(a.rows, a.q_heads, a.kv_heads, parts) > kMaxGrid || a.rows * a.q_heads > kMaxGrid)
        return UE5M3_ESHAPE;
    if (a.q == nullptr || a.o == nullptr || a.lengths == nullptr || (parts > 1 && scratch == nullptr) ||
        (a.width > 0 && (a.table == nullptr || a.cache.k == nullptr || a.cache.v == nullptr)))
        return UE5M3_EINVAL;
    if (!aligned(a.q, 16) || !aligned(a.o, 16) || !aligned(a.cache.k, 16) || !aligned(a.cache.v, 16) ||
        !aligned(a.table, 4) || !aligned(a.lengths, 4) || !aligned(scratch, 16) ||
        (used(a.q_token, a.rows) | used(a.q_head, a.q_heads)) % 8 != 0)
        return UE5M3_EALIGN;
    return status(ue5m3::launch_paged_attention(a, (float*)scratch, stream));
}

}  // extern "C"
