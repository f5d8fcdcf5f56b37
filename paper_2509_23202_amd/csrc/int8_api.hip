// C ABI of the 8-bit integer layers: argument validation on the host, then dispatch to the kernel launchers.
#include "../../include/fp4mr.h"

#include "internal.hpp"

using namespace fp4mr;

namespace {

constexpr int64_t kMost = 1 << 24;
// (sums of kMostK products of two codes, -128 among them, have 32 bits; an output of 2^38 elements, or 2^31 rows of weights, is more than the memory of any device)
constexpr int64_t kMostK = FP4MR_INT8_MAX_K, kMostOutput = 1ll << 38, kMostWeightRows = 1ll << 31;
static_assert((kMostK << 14) < (1ll << 31), "");

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename... P>
bool aligned16(const P*... p) { return (aligned(p, 16) && ...); }

bool columns(int64_t K) { return K > 0 && K <= kMostK && K % 16 == 0; }
bool product(int64_t M, int64_t N, int64_t K) { return M >= 0 && M <= kMost && N > 0 && N <= kMost && columns(K) && M <= kMostOutput / N; }

uintptr_t element(uint32_t flags) { return flags & FP4MR_OUT_F32 ? 4 : 2; }

fp4mr_status_t status(hipError_t e) { return e == hipSuccess ? FP4MR_OK : FP4MR_ERR_DEVICE; }

}  // namespace

extern "C" {

fp4mr_status_t int8_rmsnorm_quantize(const void* x, int64_t x_stride, const void* residual, const void* weight, int64_t M, int64_t K, float eps, void* codes_out,
                                     float* scales_out, void* residual_out, void* norm_out, uint32_t flags, void* stream)
{
    if (flags) return FP4MR_ERR_FMT;
    if (M < 0 || M > kMost || !columns(K) || K > kInt8NormMaxK || x_stride < K || x_stride % 8 != 0 || !(eps >= 0.0f)) return FP4MR_ERR_SHAPE;
    if (M == 0) return FP4MR_OK;
    if (!x || !weight || !codes_out || !scales_out || !residual != !residual_out) return FP4MR_ERR_NULL;
    if (!aligned16(x, residual, weight, codes_out, residual_out, norm_out) || !aligned(scales_out, 4)) return FP4MR_ERR_ALIGN;
    return status(launch_int8_rmsnorm_quantize(x, x_stride, residual, weight, M, K, eps, codes_out, scales_out, residual_out, norm_out, static_cast<hipStream_t>(stream)));
}

fp4mr_status_t int8_quantize(const void* x, int64_t x_stride, int64_t M, int64_t K, void* codes_out, float* scales_out, uint32_t flags, void* stream)
{
    if (flags & ~(uint32_t)FP4MR_SILU_MUL) return FP4MR_ERR_FMT;
    const bool silu = (flags & FP4MR_SILU_MUL) != 0;
    if (M < 0 || M > kMostWeightRows || !columns(K) || x_stride < (silu ? 2 * K : K) || x_stride % 8 != 0) return FP4MR_ERR_SHAPE;
    if (M == 0) return FP4MR_OK;
    if (!x || !codes_out || !scales_out) return FP4MR_ERR_NULL;
    if (!aligned16(x, codes_out) || !aligned(scales_out, 4)) return FP4MR_ERR_ALIGN;
    return status(launch_int8_quantize(x, x_stride, M, K, silu, codes_out, scales_out, static_cast<hipStream_t>(stream)));
}

fp4mr_status_t int8_gemm(const void* a_codes, const float* a_scales, const void* w_codes, const float* w_scales, int64_t M, int64_t N, int64_t K, void* out,
                         void* workspace, size_t workspace_bytes, uint32_t flags, void* stream)
{
    if (flags & ~(uint32_t)FP4MR_OUT_F32) return FP4MR_ERR_FMT;
    if (!product(M, N, K)) return FP4MR_ERR_SHAPE;
    if (M == 0) return FP4MR_OK;
    if (!a_codes || !a_scales || !w_codes || !w_scales || !out) return FP4MR_ERR_NULL;
    if (!aligned16(a_codes, w_codes, workspace) || !aligned(a_scales, 4) || !aligned(w_scales, 4) || !aligned(out, element(flags))) return FP4MR_ERR_ALIGN;
    return status(launch_int8_gemm(a_codes, a_scales, w_codes, w_scales, M, N, K, out, (flags & FP4MR_OUT_F32) != 0, workspace, workspace ? workspace_bytes : 0,
                                   static_cast<hipStream_t>(stream)));
}

size_t int8_workspace_bytes(int64_t M, int64_t N, int64_t K) { return M > 0 && product(M, N, K) ? int8_gemm_partial_bytes(M, N, K) : 0; }

fp4mr_status_t int8_grouped_gemm(const void* a_codes, const float* a_scales, int64_t a_rows, const void* w_codes, const float* w_scales, const int32_t* offsets,
                                 const int32_t* index, int64_t rows, int64_t experts, int64_t N, int64_t K, void* out, uint32_t flags, void* stream)
{
    if (flags & ~(uint32_t)FP4MR_OUT_F32) return FP4MR_ERR_FMT;
    if (!product(rows, N, K) || !product(a_rows, 1, K) || experts <= 0 || experts > (1 << 16)) return FP4MR_ERR_SHAPE;
    if (index ? (rows > 0 && a_rows == 0) || a_rows > kMaxGathered / K : a_rows != rows) return FP4MR_ERR_SHAPE;
    if (experts > kMostWeightRows / N) return FP4MR_ERR_SHAPE;
    if (rows == 0) return FP4MR_OK;
    if (!a_codes || !a_scales || !w_codes || !w_scales || !offsets || !out) return FP4MR_ERR_NULL;
    if (!aligned16(a_codes, w_codes) || !aligned(a_scales, 4) || !aligned(w_scales, 4) || !aligned(out, element(flags)) || !aligned(offsets, 4) || !aligned(index, 4))
        return FP4MR_ERR_ALIGN;
    return status(launch_int8_grouped_gemm(a_codes, a_scales, a_rows, w_codes, w_scales, offsets, index, rows, experts, N, K, out, (flags & FP4MR_OUT_F32) != 0,
                                           static_cast<hipStream_t>(stream)));
}

}  // extern "C"
