// Stored form of MXFP4 operands (include/loka.h) and the conversions that the quantizing kernels share.
#pragma once

#include "common.h"

namespace loka {

constexpr int kMxGroup = 32;           // elements that share a scale
constexpr int kMxPad = 128;            // a stored row is a whole number of matrix instructions' K
constexpr int kMxNaN = 255;            // scale byte of a group with a NaN or an infinity

// A launch has fewer than 2^32 threads: workgroups 0 .. groups - 1 of `threads` threads in as many launches as that takes, each told its first
template <class F>
static inline loka_status in_launches(int64_t groups, int threads, F&& launch) {
    const int64_t most = (INT64_C(1) << 32) / threads - 1;
    for (int64_t from = 0; from < groups; from += most) {
        launch(from, static_cast<uint32_t>(groups - from < most ? groups - from : most));
        LOKA_HIP_TRY(hipGetLastError());
    }
    return LOKA_OK;
}

static inline int64_t mx_padded(int64_t cols) { return (cols + kMxPad - 1) / kMxPad * kMxPad; }

// Scale byte of a group from the bits of its largest magnitude as binary32 (a bf16's bits shifted up): the exponent field is
// floor(log2) + 127, two less of it the scale's own, none below 0 (subnormal maxima have exponent field 0).
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_f32_bits) {
    const uint32_t e = amax_f32_bits >> 23;
    return e == 255u ? static_cast<uint32_t>(kMxNaN) : e > 2u ? e - 2u : 0u;
}
// The scale as binary32 (2^-127 is subnormal); byte 255 gives a NaN.
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
    return __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7FC00000u : byte << 23);
}

// (by value: a bit cast of a vector's component takes the first one)
__device__ __forceinline__ bf16x2_t bf16_pair(uint32_t w) { return __builtin_bit_cast(bf16x2_t, w); }
// Eight elements -> eight codes of one word; the instruction divides by the scale exactly, rounds to nearest even, saturates.
__device__ __forceinline__ uint32_t mx_codes_bf16x8(const u32x4 w, float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16_pair(w.x), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16_pair(w.y), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16_pair(w.z), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16_pair(w.w), scale, 3);
    return r;
}
__device__ __forceinline__ uint32_t mx_codes_f32x8(const float (&v)[8], float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
    return r;
}

// the larger magnitudes of packed bf16, as packed 15-bit integers (a NaN is the largest)
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t a, uint32_t w) {
    const u16x2 r = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu));
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t max_of_halves(uint32_t a) {
    const uint32_t lo = a & 0xFFFFu, hi = a >> 16;
    return lo > hi ? lo : hi;
}
// maximum over groups of 4 consecutive lanes, in all of them
__device__ __forceinline__ uint32_t quad_max(uint32_t a) {
    uint32_t o;
    o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(a), 0xB1, 0xF, 0xF, false)); a = a > o ? a : o;      // lane ^ 1
    o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(a), 0x4E, 0xF, 0xF, false)); a = a > o ? a : o;      // lane ^ 2
    return a;
}
// Lanes 4k hold group k's byte (k of 16 lanes): the four bytes of the 16 lanes as one word, in lane 0 of them
__device__ __forceinline__ uint32_t quad_bytes(uint32_t byte) {
    uint32_t w = byte;
    w |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(byte), 0x104, 0xF, 0xF, true)) << 8;      // 4 lanes up (row_shl:4)
    w |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(byte), 0x108, 0xF, 0xF, true)) << 16;
    w |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(byte), 0x10C, 0xF, 0xF, true)) << 24;
    return w;
}

// Wide accesses that need no more than their elements' alignment: rows start anywhere (by elements, us: codes of 8191 x 4095 36.9, here
// 17.6; transposed 22.8 and 19.6; values 22.1 and 14.5)
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));

// The eight elements from `s` on of v and zeros behind it (s >= 0), without a branch
__device__ __forceinline__ u32x4 mx_from(u32x4 v, int64_t s) {
    const bool four = s & 4, two = s & 2, one = s & 1, none = s >= 8;
    v = four ? u32x4{v.z, v.w, 0u, 0u} : v;
    v = two ? u32x4{v.y, v.z, v.w, 0u} : v;
    v = one ? u32x4{__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16), __builtin_amdgcn_alignbit(v.w, v.z, 16), v.w >> 16} : v;
    return none ? u32x4{0u, 0u, 0u, 0u} : v;
}

// Eight consecutive elements of a row from column c on, zeros from `cols` on; STREAMED past the caches.  A run that the row's end
// cuts comes from the row's last eight.
template <bool STREAMED = false>
__device__ __forceinline__ u32x4 mx_load8(const uint16_t* row, int64_t c, int64_t cols) {
    if (c + 8 <= cols) {
        if (STREAMED) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + c));
        return *reinterpret_cast<const u32x4_any*>(row + c);
    }
    if (c >= cols) return u32x4{0u, 0u, 0u, 0u};
    if (cols >= 8) return mx_from(*reinterpret_cast<const u32x4_any*>(row + cols - 8), c + 8 - cols);
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? row[c + i] : 0u;
    return u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
}

}  // namespace loka
