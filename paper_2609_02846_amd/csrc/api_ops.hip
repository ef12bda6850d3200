// C ABI shim of the operators around the linear layers (layer norm, dropout,
// the products in 8-bit floating point): argument validation, status mapping
// and dispatch.  See include/ue5m3.h for the contract of every entry point.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/ue5m3.h"
#include "launch.hpp"

namespace {

using ue5m3::DType;
using ue5m3::Fp8;

constexpr int64_t kMaxK = (int64_t)1 << 22;      // a tile's rows stay within 32-bit offsets
constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;   // workgroups of 256 threads a launch takes

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline ue5m3_status_t status(hipError_t e) { return e == hipSuccess ? UE5M3_OK : UE5M3_EHIP; }
inline bool known(ue5m3_dtype_t t) { return t == UE5M3_BF16 || t == UE5M3_F16 || t == UE5M3_F32; }
inline bool known(ue5m3_fp8_t t) { return t == UE5M3_E4M3 || t == UE5M3_E5M2; }
inline bool known(ue5m3_fp8_scale_t t) { return t == UE5M3_FP8_SCALE_F32 || t == UE5M3_FP8_SCALE_E8M0; }
inline bool known(ue5m3_out_t t) { return t == UE5M3_OUT_F32 || t == UE5M3_OUT_BF16; }
inline uintptr_t size_of(ue5m3_dtype_t t) { return t == UE5M3_F32 ? 4 : 2; }
inline DType dtype(ue5m3_dtype_t t) { return static_cast<DType>(t); }
inline int64_t blocks(int64_t n) { return (n + 127) / 128; }
// Whether the quantizers' grids take a [rows, cols] tensor (16 rows a workgroup).
inline bool fits(int64_t rows, int64_t cols) { return (rows + 15) / 16 <= kMaxGrid / std::max<int64_t>(blocks(cols), 1); }

// Types, sizes and parameters common to layer norm and its gradient.
ue5m3_status_t norm_args(int64_t rows, int64_t cols, ue5m3_dtype_t xt, ue5m3_dtype_t pt) {
    if (!known(xt) || !known(pt) || (pt != xt && pt != UE5M3_F32)) return UE5M3_EINVAL;
    if (rows < 0 || cols < 0 || cols >= (int64_t)1 << 31) return UE5M3_ESHAPE;
    return UE5M3_OK;
}

// Whether a blocking of 128 runs along the contraction (rows_contracted: along
// its source's rows); EINVAL for one that is not of 128.
ue5m3_status_t along(ue5m3_blocking_t b, bool rows_contracted, bool tile_ok) {
    if (b != UE5M3_ROW128 && b != UE5M3_COL128T && b != UE5M3_TILE128) return UE5M3_EINVAL;
    if (b == UE5M3_TILE128) return tile_ok ? UE5M3_OK : UE5M3_ELAYOUT;
    return (b == UE5M3_ROW128) == rows_contracted ? UE5M3_OK : UE5M3_ELAYOUT;
}

}  // namespace

extern "C" {

ue5m3_status_t ue5m3_layer_norm(const void* x, int64_t rows, int64_t cols, ue5m3_dtype_t x_type, const void* weight,
                                const void* bias, ue5m3_dtype_t param_type, float eps, void* y, float* mean,
                                float* rstd, hipStream_t stream) {
    const ue5m3_status_t st = norm_args(rows, cols, x_type, param_type);
    if (st != UE5M3_OK) return st;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return UE5M3_EINVAL;
    if (rows == 0 || cols == 0) return UE5M3_OK;
    if (x == nullptr || y == nullptr) return UE5M3_EINVAL;
    if (!aligned(x, size_of(x_type)) || !aligned(y, size_of(x_type)) || !aligned(weight, size_of(param_type)) ||
        !aligned(bias, size_of(param_type)) || !aligned(mean, 4) || !aligned(rstd, 4))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_norm(dtype(x_type), x, rows, cols, dtype(param_type), weight, bias, eps, y, mean, rstd,
                                     stream));
}

ue5m3_status_t ue5m3_layer_norm_grad(const void* x, const void* dy, int64_t rows, int64_t cols, ue5m3_dtype_t x_type,
                                     const void* weight, ue5m3_dtype_t param_type, const float* mean,
                                     const float* rstd, const void* residual_grad, void* dx, void* dweight,
                                     void* dbias, hipStream_t stream) {
    const ue5m3_status_t st = norm_args(rows, cols, x_type, param_type);
    if (st != UE5M3_OK) return st;
    if (cols == 0 || (dx == nullptr && dweight == nullptr && dbias == nullptr)) return UE5M3_OK;
    if (rows == 0 && dweight == nullptr && dbias == nullptr) return UE5M3_OK;
    if (rows > 0 && (x == nullptr || dy == nullptr || mean == nullptr || rstd == nullptr)) return UE5M3_EINVAL;
    const uintptr_t xs = size_of(x_type), ps = size_of(param_type);
    if (!aligned(x, xs) || !aligned(dy, xs) || !aligned(residual_grad, xs) || !aligned(dx, xs) || !aligned(weight, ps) ||
        !aligned(dweight, ps) || !aligned(dbias, ps) || !aligned(mean, 4) || !aligned(rstd, 4))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_norm_grad(dtype(x_type), x, dy, rows, cols, dtype(param_type), weight, mean, rstd,
                                          residual_grad, dx, dweight, dbias, stream));
}

ue5m3_status_t ue5m3_dropout(const void* x, int64_t n, ue5m3_dtype_t type, double p, uint64_t seed,
                             uint32_t tensor_id, const void* residual, void* y, hipStream_t stream) {
    if (!known(type) || !(p >= 0.0 && p <= 1.0)) return UE5M3_EINVAL;
    if (n < 0) return UE5M3_ESHAPE;
    if (n == 0) return UE5M3_OK;
    if (x == nullptr || y == nullptr) return UE5M3_EINVAL;
    if (!aligned(x, size_of(type)) || !aligned(residual, size_of(type)) || !aligned(y, size_of(type)))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_dropout(dtype(type), x, n, p, seed, tensor_id, residual, y, stream));
}

ue5m3_status_t ue5m3_quantize_fp8(const void* x, int64_t rows, int64_t cols, ue5m3_dtype_t x_type, ue5m3_fp8_t format,
                                  ue5m3_fp8_scale_t scale_kind, uint8_t* payload_r, void* scales_r,
                                  uint8_t* payload_c, void* scales_c, hipStream_t stream) {
    if (!known(x_type) || !known(format) || !known(scale_kind)) return UE5M3_EINVAL;
    if ((payload_r == nullptr) != (scales_r == nullptr) || (payload_c == nullptr) != (scales_c == nullptr))
        return UE5M3_EINVAL;
    if (rows < 0 || cols < 0) return UE5M3_ESHAPE;
    if (rows == 0 || cols == 0) return UE5M3_OK;
    if (!fits(rows, cols)) return UE5M3_ESHAPE;
    if (x == nullptr || (payload_r == nullptr && payload_c == nullptr)) return UE5M3_EINVAL;
    if (!aligned(x, size_of(x_type)) || !aligned(payload_r, 16) || !aligned(scales_r, 16) || !aligned(payload_c, 16) ||
        !aligned(scales_c, 16))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_quant_fp8(dtype(x_type), static_cast<Fp8>(format), scale_kind == UE5M3_FP8_SCALE_E8M0,
                                          x, rows, cols, payload_r, scales_r, payload_c, scales_c, stream));
}

ue5m3_status_t ue5m3_quantize_fp8_tiles(const void* w, int64_t rows, int64_t cols, ue5m3_dtype_t w_type,
                                        ue5m3_fp8_scale_t scale_kind, uint8_t* payload, void* scales,
                                        uint8_t* payload_t, void* scales_t, hipStream_t stream) {
    if (!known(w_type) || !known(scale_kind) || (payload_t == nullptr) != (scales_t == nullptr)) return UE5M3_EINVAL;
    if (rows < 0 || cols < 0) return UE5M3_ESHAPE;
    if (rows == 0 || cols == 0) return UE5M3_OK;
    if (!fits(rows, cols)) return UE5M3_ESHAPE;
    if (w == nullptr || payload == nullptr || scales == nullptr) return UE5M3_EINVAL;
    if (!aligned(w, size_of(w_type)) || !aligned(payload, 16) || !aligned(scales, 16) || !aligned(payload_t, 16) ||
        !aligned(scales_t, 16))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_quant_fp8_tiles(dtype(w_type), scale_kind == UE5M3_FP8_SCALE_E8M0, w, rows, cols,
                                                payload, scales, payload_t, scales_t, stream));
}

ue5m3_status_t ue5m3_gemm_fp8(ue5m3_layout_t layout, int64_t M, int64_t N, int64_t K, const uint8_t* a,
                              const void* a_scales, ue5m3_blocking_t a_blk, ue5m3_fp8_t a_format, const uint8_t* b,
                              const void* b_scales, ue5m3_blocking_t b_blk, ue5m3_fp8_scale_t scale_kind, void* c,
                              ue5m3_out_t c_type, hipStream_t stream) {
    if (layout != UE5M3_NT && layout != UE5M3_NN && layout != UE5M3_TN) return UE5M3_ELAYOUT;
    if (!known(a_format) || !known(scale_kind) || !known(c_type)) return UE5M3_EINVAL;
    const ue5m3_status_t sa = along(a_blk, layout != UE5M3_TN, false), sb = along(b_blk, layout == UE5M3_NT, true);
    if (sa == UE5M3_EINVAL || sb == UE5M3_EINVAL) return UE5M3_EINVAL;
    if (sa != UE5M3_OK || sb != UE5M3_OK) return UE5M3_ELAYOUT;
    if (M < 0 || N < 0 || K < 0 || K > kMaxK) return UE5M3_ESHAPE;
    if (M == 0 || N == 0) return UE5M3_OK;
    if (blocks(M) > kMaxGrid / blocks(N)) return UE5M3_ESHAPE;
    if (c == nullptr || (K > 0 && (a == nullptr || a_scales == nullptr || b == nullptr || b_scales == nullptr)))
        return UE5M3_EINVAL;
    if (!aligned(c, 16) || (K > 0 && (!aligned(a, 16) || !aligned(a_scales, 16) || !aligned(b, 16) ||
                                      !aligned(b_scales, 16))))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_gemm_fp8(M, N, K, a, a_scales, static_cast<Fp8>(a_format), b, b_scales,
                                         b_blk == UE5M3_TILE128, scale_kind == UE5M3_FP8_SCALE_E8M0, c,
                                         c_type == UE5M3_OUT_BF16, stream));
}

ue5m3_status_t ue5m3_linear_fp8(const void* x_bf16, int64_t T, int64_t K, int64_t N, const uint8_t* w,
                                const void* w_scales, ue5m3_fp8_scale_t scale_kind, void* y, ue5m3_out_t y_type,
                                hipStream_t stream) {
    if (!known(scale_kind) || !known(y_type)) return UE5M3_EINVAL;
    if (T < 0 || N < 0 || K < 0 || K > kMaxK) return UE5M3_ESHAPE;
    if (T == 0 || N == 0) return UE5M3_OK;
    if (blocks(T) > kMaxGrid / blocks(N) || !fits(T, K)) return UE5M3_ESHAPE;
    if (y == nullptr || (K > 0 && (x_bf16 == nullptr || w == nullptr || w_scales == nullptr))) return UE5M3_EINVAL;
    if (!aligned(y, 16) || (K > 0 && (!aligned(x_bf16, 2) || !aligned(w, 16) || !aligned(w_scales, 16))))
        return UE5M3_EALIGN;
    return status(ue5m3::launch_linear_fp8(x_bf16, T, K, N, w, w_scales, scale_kind == UE5M3_FP8_SCALE_E8M0, y,
                                           y_type == UE5M3_OUT_BF16, stream));
}

}  // extern "C"
