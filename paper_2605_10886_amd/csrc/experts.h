// A layer of experts (include/loka.h): what its kernels share.
#pragma once

#include <type_traits>

#include "mxfp4.h"

namespace loka {

// ---- launches (arguments are checked in api.hip)
size_t route_workspace_bytes(const loka_route_desc* d);
loka_status route_launch(const loka_route_desc* d, const void* logits, int32_t* expert, float* weight, int32_t* slot, int32_t* row,
                         int32_t* offsets, void* ws, hipStream_t stream);
loka_status route_backward_launch(const loka_route_desc* d, const void* logits, const int32_t* expert, const float* dweight, void* dlogits,
                                  hipStream_t stream);
loka_status combine_launch(const loka_combine_desc* d, const void* y, const int32_t* slot, const float* weight, const void* residual,
                           void* out, hipStream_t stream);
loka_status combine_backward_launch(const loka_combine_desc* d, const void* dout, const void* y, const int32_t* slot, const float* weight,
                                    void* dy, float* dweight, hipStream_t stream);
loka_status grouped_quantize_launch(const loka_grouped_quantize_desc* d, const void* x, const int32_t* index, const int32_t* offsets, uint8_t* q,
                                    float* scales, uint8_t* qt, float* st, hipStream_t stream);
bool grouped_gemm_fits(const loka_grouped_desc* d);
loka_status grouped_gemm_launch(const loka_grouped_desc* d, const uint8_t* xq, const float* sx, const int32_t* index, const int32_t* offsets,
                                const uint8_t* wq, const float* sw, void* out, float* y, hipStream_t stream);
bool grouped_wgrad_fits(const loka_grouped_desc* d);
size_t grouped_wgrad_workspace_bytes(const loka_grouped_desc* d);
loka_status grouped_wgrad_launch(const loka_grouped_desc* d, const uint8_t* xt, const float* sxt, const uint8_t* dyt, const float* sdyt,
                                 const int32_t* offsets, void* dw, float* dw32, void* ws, size_t ws_bytes, hipStream_t stream);

constexpr int kGroupBlock = 128;       // elements that share a scale
static inline int64_t group_blocks(int64_t n) { return (n + kGroupBlock - 1) / kGroupBlock; }

#ifdef __HIPCC__
// The rows of a group from the device's offsets; whatever they hold, first and count stay within `rows`.
struct GroupRows { int first, count; };
__device__ __forceinline__ GroupRows group_rows(const int32_t* offsets, int g, int rows) {
    const int lo = offsets[g], hi = offsets[g + 1];
    const int a = lo < 0 ? 0 : lo > rows ? rows : lo, b = hi > rows ? rows : hi;
    return {a, b > a ? b - a : 0};
}
// inclusive sums over the wave's lanes
__device__ __forceinline__ int lanes_inclusive(int v) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}
// Units of `unit` rows that all groups take (each its own), by a wave; uniform.
__device__ __forceinline__ int units_of_all(const int32_t* offsets, int groups, int rows, int unit) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    int n = 0;
    for (int g = lane; g < groups; g += 64) n += (group_rows(offsets, g, rows).count + unit - 1) / unit;
    return __builtin_amdgcn_readlane(lanes_inclusive(n), 63);
}
// The group that holds unit `target`, and the units of the groups before it; group = -1: there are not so many.  By a wave; uniform.
struct UnitAt { int group, before, first, count; };
__device__ __forceinline__ UnitAt find_unit(const int32_t* offsets, int groups, int rows, int unit, int target) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    int base = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        const GroupRows r = g0 + lane < groups ? group_rows(offsets, g0 + lane, rows) : GroupRows{0, 0};
        const int n = (r.count + unit - 1) / unit, s = lanes_inclusive(n);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(base + s > target);
        if (past) {
            const int l = __builtin_ctzll(past), before = base + __builtin_amdgcn_readlane(s - n, l);
            // (always so, unless groups that overlap have made the sums overflow: then the unit is nobody's)
            const bool inside = target >= before && target - before < __builtin_amdgcn_readlane(n, l);
            return {inside ? g0 + l : -1, before, __builtin_amdgcn_readlane(r.first, l), __builtin_amdgcn_readlane(r.count, l)};
        }
        base += __builtin_amdgcn_readlane(s, 63);
    }
    return {-1, base, 0, 0};
}
// Units of the groups before `group`, by a wave; uniform.
__device__ __forceinline__ int units_before(const int32_t* offsets, int group, int rows, int unit) {
    return units_of_all(offsets, group, rows, unit);
}
#endif

}  // namespace loka
