// Launchers of the operators between the QKV and the output projection.  Their
// arguments are the C ABI's structures, checked by its shim.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ue5m3.h"
#include "launch.hpp"

namespace ue5m3 {

constexpr int kMaxRopeDim = 256;
constexpr int kRopeGradRows = 1024;              // most partial rows of the weights' gradients

// The values that go into a cache with the keys, and each token's place there.
struct Append {
    const void* v;
    int64_t v_token, v_head;
    const int64_t* slots;
    ue5m3_pages_t cache;
};

hipError_t launch_rope(const ue5m3_rope_t& r, const Append* ap, hipStream_t s);

// gq, gk: the outputs' gradients.  scratch: rope_grad_rows() rows of 2 dim floats, for
// dqw and dkw.
int rope_grad_rows(int64_t tokens, int heads);
hipError_t launch_rope_grad(const ue5m3_rope_t& r, const void* gq, const void* gk, void* dqw, void* dkw, float* scratch,
                            hipStream_t s);

hipError_t launch_copy_pages(void* base, int64_t planes, int64_t plane, int64_t page, const int32_t* src,
                             const int32_t* dst, int64_t n, hipStream_t s);

// Workgroups' tiles of all sequences, at most.
int64_t attention_items(int64_t tokens, int64_t sequences, bool ragged);
int64_t attention_scratch(const ue5m3_attention_t& a);               // bytes
hipError_t launch_attention(const ue5m3_attention_t& a, float* scratch, hipStream_t s);
int64_t attention_grad_scratch(const ue5m3_attention_t& a);          // bytes
hipError_t launch_attention_grad(const ue5m3_attention_t& a, const ue5m3_attention_grad_t& g, hipStream_t s);

// Parts that each row's length is cut into (one needs no scratch).
int paged_parts(int64_t rows, int q_heads, int kv_heads, int64_t capacity, int64_t window, int64_t sinks);
int64_t paged_groups(int64_t rows, int q_heads, int kv_heads, int parts);     // workgroups
hipError_t launch_paged_attention(const ue5m3_paged_attention_t& a, float* scratch, hipStream_t s);

}  // namespace ue5m3
