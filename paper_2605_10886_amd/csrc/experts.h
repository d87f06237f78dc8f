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
bool grouped_linear_fused(const loka_grouped_desc* d);
loka_status grouped_linear_fused_launch(const loka_grouped_desc* d, const void* x, int64_t ld, const int32_t* index, const int32_t* offsets,
                                        const uint8_t* wq, const float* sw, void* out, float* y, hipStream_t stream);
loka_status grouped_gemm_launch(const loka_grouped_desc* d, const uint8_t* xq, const float* sx, const int32_t* index, const int32_t* offsets,
                                const uint8_t* wq, const float* sw, void* out, float* y, hipStream_t stream);
bool grouped_wgrad_fits(const loka_grouped_desc* d);
size_t grouped_wgrad_workspace_bytes(const loka_grouped_desc* d);
loka_status grouped_wgrad_launch(const loka_grouped_desc* d, const uint8_t* xt, const float* sxt, const uint8_t* dyt, const float* sdyt,
                                 const int32_t* offsets, void* dw, float* dw32, void* ws, hipStream_t stream);

constexpr int kGroupBlock = 128;       // elements that share a scale
constexpr int32_t kMostGroups = 1024;
static inline int64_t group_blocks(int64_t n) { return (n + kGroupBlock - 1) / kGroupBlock; }

#ifdef __HIPCC__
// Units of `unit` rows that `count` rows (0 .. 2^31 - 1) take; in unsigned numbers, as count + unit - 1 may be more than an int holds
__host__ __device__ constexpr int units_of(int count, int unit) {
    return static_cast<int>((static_cast<uint32_t>(count) + static_cast<uint32_t>(unit) - 1u) / static_cast<uint32_t>(unit));
}
static_assert(units_of(0, 128) == 0 && units_of(1, 256) == 1 && units_of(INT32_MAX, 16) == 1 << 27 && units_of(INT32_MAX, 128) == 1 << 24 && units_of(INT32_MAX, 256) == 1 << 23);
// The rows of a group from the device's offsets; whatever they hold, first and count stay within `rows`.
struct GroupRows { int first, count; };
__device__ __forceinline__ GroupRows group_rows(const int32_t* offsets, int g, int rows) {
    const int lo = offsets[g], hi = offsets[g + 1];
    const int a = lo < 0 ? 0 : lo > rows ? rows : lo, b = hi > rows ? rows : hi;
    return {a, b > a ? b - a : 0};
}
// inclusive sums over the wave's lanes, by moves of the vector unit (a shuffle is an LDS round trip)
__device__ __forceinline__ int lanes_inclusive(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);         // within 16 lanes: 1, 2, 4, 8 to the left
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);        // lane 15 to the second 16, lane 47 to the fourth
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);        // lane 31 to the upper half
    return v;
}
// The group that holds unit `target`, and the units of the groups before it; group = -1: there are not so many.  By a wave; uniform.
struct UnitAt { int group, before, first, count; };
__device__ __forceinline__ UnitAt find_unit(const int32_t* offsets, int groups, int rows, int unit, int target) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    int base = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        const GroupRows r = g0 + lane < groups ? group_rows(offsets, g0 + lane, rows) : GroupRows{0, 0};
        const int n = units_of(r.count, unit), s = lanes_inclusive(n);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(base + s > target);
        if (past) {
            const int l = __builtin_ctzll(past), before = base + __builtin_amdgcn_readlane(s - n, l);
            // (always so, unless groups that overlap have made the sums overflow: then the unit is nobody's)
            const bool inside = target >= before && target - before < __builtin_amdgcn_readlane(n, l);
            // (as scalars: addresses that follow from them are)
            return {inside ? g0 + l : -1, before, __builtin_amdgcn_readlane(r.first, l), __builtin_amdgcn_readlane(r.count, l)};
        }
        base += __builtin_amdgcn_readlane(s, 63);
    }
    return {-1, base, 0, 0};
}
// Scale of 128 elements from the bits of their largest magnitude (a bf16's).  False where that is not finite: the scale is a NaN then, the codes are zeros.
__device__ __forceinline__ bool gq_scale(uint32_t amax, float& scale) {
    float inv;
    group_scale_pow2(bf16_bits_to_f32(amax), scale, inv);
    if (amax < 0x7F80u) return true;
    scale = __uint_as_float(0x7FC00000u);
    return false;
}
__device__ __forceinline__ uint32_t max_abs8(u32x4 v) {
    uint32_t a = max_abs_bf16x2(v.x & 0x7FFF7FFFu, v.y);
    a = max_abs_bf16x2(max_abs_bf16x2(a, v.z), v.w);
    return max_of_halves(a);
}
// Four elements (two words of two bf16) as codes: the instruction divides by the power of two exactly and rounds to nearest even; no quotient exceeds 448.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t gq_codes4(uint32_t a, uint32_t b, float scale) {
    s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, bf16_pair(a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, bf16_pair(b), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ u32x2 gq_codes8(u32x4 v, float scale, bool finite) {
    const u32x2 c{gq_codes4(v.x, v.y, scale), gq_codes4(v.z, v.w, scale)};
    return finite ? c : u32x2{0u, 0u};
}
#endif

}  // namespace loka
