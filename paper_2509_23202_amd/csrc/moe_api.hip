// C ABI of the router's operators: argument validation on the host, then dispatch to the kernel launchers.
#include "../../include/fp4mr.h"

#include "internal.hpp"

using namespace fp4mr;

namespace {

constexpr int64_t kMostTokens = 1 << 24, kMostPairs = 1 << 30, kMostExperts = 1024, kMostTop = 64, kMostGroups = 64, kMostCols = 1 << 24;

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool routed(int64_t T, int64_t experts, int64_t top) { return T >= 0 && T <= kMostTokens && experts > 0 && experts <= kMostExperts && top > 0 && top <= kMostTop && T <= kMostPairs / top; }

fp4mr_status_t status(hipError_t e) { return e == hipSuccess ? FP4MR_OK : FP4MR_ERR_DEVICE; }

}  // namespace

extern "C" {

size_t moe_workspace_bytes(int64_t T, int64_t experts, int64_t top) { return routed(T, experts, top) ? moe_count_bytes(T, experts, top) : 0; }

fp4mr_status_t moe_route(const void* logits, int64_t logits_stride, const float* bias, int64_t T, int64_t experts, int64_t top, int64_t groups, int64_t top_groups, float scale,
                         float* weights_out, int32_t* experts_out, int32_t* rows_out, int32_t* offsets_out, int32_t* places_out, void* workspace, size_t workspace_bytes, uint32_t flags,
                         void* stream)
{
    constexpr uint32_t known = FP4MR_INPUT_F32 | FP4MR_ROUTE_SIGMOID | FP4MR_ROUTE_RENORM | FP4MR_ROUTE_GROUP_SUM2;
    if (flags & ~known) return FP4MR_ERR_FMT;
    if (!routed(T, experts, top) || logits_stride < experts || groups <= 0 || groups > kMostGroups || experts % groups != 0 || top_groups <= 0 || top_groups > groups ||
        top > experts / groups * top_groups)
        return FP4MR_ERR_SHAPE;
    if (!offsets_out || (T > 0 && (!logits || !weights_out || !experts_out || !rows_out || !places_out))) return FP4MR_ERR_NULL;
    const bool f32 = (flags & FP4MR_INPUT_F32) != 0;
    if (!aligned(logits, f32 ? 4 : 2) || !aligned(bias, 4) || !aligned(weights_out, 4) || !aligned(experts_out, 4) || !aligned(rows_out, 4) || !aligned(offsets_out, 4) ||
        !aligned(places_out, 4) || !aligned(workspace, 16))
        return FP4MR_ERR_ALIGN;
    const size_t need = moe_count_bytes(T, experts, top);
    if (need && (!workspace || workspace_bytes < need)) return FP4MR_ERR_WORKSPACE;
    return status(launch_moe_route(logits, logits_stride, f32, bias, T, experts, top, groups, top_groups, scale, (flags & FP4MR_ROUTE_SIGMOID) != 0, (flags & FP4MR_ROUTE_RENORM) != 0,
                                   (flags & FP4MR_ROUTE_GROUP_SUM2) != 0, weights_out, experts_out, offsets_out, rows_out, places_out, workspace, static_cast<hipStream_t>(stream)));
}

fp4mr_status_t moe_combine(const void* y, int64_t y_rows, const int32_t* places, const float* weights, const void* shared, int64_t T, int64_t top, int64_t cols, void* out, uint32_t flags,
                           void* stream)
{
    constexpr uint32_t known = FP4MR_INPUT_F32 | FP4MR_SHARED_F32 | FP4MR_OUT_F32;
    if (flags & ~known || ((flags & FP4MR_SHARED_F32) && !shared)) return FP4MR_ERR_FMT;
    if (!routed(T, 1, top) || y_rows < 0 || y_rows > kMostPairs || cols <= 0 || cols > kMostCols) return FP4MR_ERR_SHAPE;
    if (T == 0) return FP4MR_OK;
    if ((!y && y_rows > 0) || !places || !weights || !out) return FP4MR_ERR_NULL;
    if (!aligned(y, flags & FP4MR_INPUT_F32 ? 4 : 2) || !aligned(places, 4) || !aligned(weights, 4) || !aligned(shared, flags & FP4MR_SHARED_F32 ? 4 : 2) ||
        !aligned(out, flags & FP4MR_OUT_F32 ? 4 : 2))
        return FP4MR_ERR_ALIGN;
    return status(launch_moe_combine(y, y_rows, (flags & FP4MR_INPUT_F32) != 0, places, weights, shared, (flags & FP4MR_SHARED_F32) != 0, T, top, cols, out, (flags & FP4MR_OUT_F32) != 0,
                                     static_cast<hipStream_t>(stream)));
}

}  // extern "C"
