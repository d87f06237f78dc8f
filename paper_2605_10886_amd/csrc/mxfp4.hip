// MXFP4 quantization and its inverse (include/loka.h, "MXFP4"): bandwidth-bound streaming kernels.
//
// A group's scale is the exponent field of its largest magnitude less 2, so the maximum is taken on the bits (an integer
// maximum of packed halves) and no division or logarithm is needed; the codes come from the gfx950 conversion, which divides
// by the power of two, rounds and saturates in one instruction per two elements.
#include "mxfp4.h"

namespace loka {

// ---------------------------------------------------------------------------------
// Groups along the row.  16 lanes take one stored block of 128 elements (8 each: one 16-byte load, one word of codes); four
// lanes share a group; the 16 lanes' four scale bytes leave as one word.  A workgroup takes 16 * U consecutive blocks of the
// matrix, so that short rows fill it too; U loads of a lane are in flight together.
template <int U, bool STREAMED>
__global__ __launch_bounds__(256) void mx_quant_rows_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t cols,
                                                            int64_t ld, uint32_t* __restrict__ q, uint32_t* __restrict__ scales, int64_t first_wg) {
    const int t = static_cast<int>(threadIdx.x), l16 = t & 15;
    const int64_t nb = (cols + kMxPad - 1) / kMxPad, total = rows * nb;
    const int64_t first = (first_wg + blockIdx.x) * (16 * U) + (t >> 4);
    int64_t row = first / nb, b = first - row * nb;
    const int64_t step_row = 16 / nb, step_b = 16 - step_row * nb;
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (row < rows) v[u] = mx_load8<STREAMED>(x + row * ld, b * kMxPad + l16 * 8, cols);
        row += step_row;
        b += step_b;
        if (b >= nb) { b -= nb; ++row; }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t unit = first + u * 16;
        if (unit < total) {
            uint32_t a = max_abs_bf16x2(v[u].x & 0x7FFF7FFFu, v[u].y);
            a = max_abs_bf16x2(max_abs_bf16x2(a, v[u].z), v[u].w);
            const uint32_t byte = mx_scale_byte(quad_max(max_of_halves(a)) << 16);
            const uint32_t codes = mx_codes_bf16x8(v[u], mx_scale_value(byte));
            const uint32_t four = quad_bytes(byte);
            q[unit * 16 + l16] = byte == kMxNaN ? 0u : codes;
            if (l16 == 0) scales[unit] = four;
        }
    }
}

// ---------------------------------------------------------------------------------
// Groups down the columns, written transposed.  A workgroup of 8 waves takes 256 rows x 128 columns; wave w's lanes hold two
// columns of rows 32 w ..: a whole group each, so its maximum needs no exchange.  The codes turn in LDS and leave as up to
// 128 consecutive bytes of an output row.
constexpr int kTurnRows = 256, kTurnCols = 128, kTurnPitch = kTurnRows / 2 + 16;      // (pitch: 16 bytes more, so that columns start on other banks)
template <bool STREAMED>
__global__ __launch_bounds__(512) void mx_quant_turned_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t cols,
                                                              int64_t ld, uint8_t* __restrict__ q, uint8_t* __restrict__ scales, int64_t first_wg) {
    __shared__ __align__(16) uint8_t codes[kTurnCols * kTurnPitch];
    __shared__ __align__(8) uint8_t bytes[kTurnCols * 8];
    const int t = static_cast<int>(threadIdx.x), lane = t & 63, wave = t >> 6;
    const int64_t rowsp = (rows + kMxPad - 1) / kMxPad * kMxPad;
    const int64_t nct = (cols + kTurnCols - 1) / kTurnCols;
    const int64_t rt = (first_wg + blockIdx.x) / nct, ct = first_wg + blockIdx.x - rt * nct;
    const int64_t r0 = rt * kTurnRows + wave * kMxGroup, c = ct * kTurnCols + lane * 2;
    uint32_t w[kMxGroup];              // (element of column c, of column c + 1) of each row
#pragma unroll
    for (int r = 0; r < kMxGroup; ++r) {
        w[r] = 0u;
        const uint16_t* p = x + (r0 + r) * ld + c;
        if (r0 + r < rows) {
            if (c + 1 < cols) w[r] = STREAMED ? __builtin_nontemporal_load(reinterpret_cast<const u32_any*>(p)) : *reinterpret_cast<const u32_any*>(p);
            else if (c < cols) w[r] = p[0];
        }
    }
    uint32_t a = 0u;
#pragma unroll
    for (int r = 0; r < kMxGroup; ++r) a = max_abs_bf16x2(a, w[r]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t byte = mx_scale_byte((h ? a >> 16 : a & 0xFFFFu) << 16);
        const float s = mx_scale_value(byte);
        u32x4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            u32x4 e;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = w[k * 8 + 2 * i], hi = w[k * 8 + 2 * i + 1];
                e[i] = h ? (lo >> 16) | (hi & 0xFFFF0000u) : (lo & 0xFFFFu) | (hi << 16);
            }
            o[k] = byte == kMxNaN ? 0u : mx_codes_bf16x8(e, s);
        }
        *reinterpret_cast<u32x4*>(codes + (lane * 2 + h) * kTurnPitch + wave * 16) = o;
        bytes[(lane * 2 + h) * 8 + wave] = static_cast<uint8_t>(byte);
    }
    __syncthreads();
    // 128 columns x 8 pieces of 16 bytes; pieces past the stored row end are not written
    const int64_t pieces = (rowsp - rt * kTurnRows) / kMxGroup;          // (a multiple of 4)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = t + k * 512, col = i >> 3, piece = i & 7;
        if (ct * kTurnCols + col < cols && piece < pieces)
            *reinterpret_cast<u32x4*>(q + (ct * kTurnCols + col) * (rowsp / 2) + rt * (kTurnRows / 2) + piece * 16) =
                *reinterpret_cast<const u32x4*>(codes + col * kTurnPitch + piece * 16);
    }
    if (t < 256) {
        const int col = t >> 1, half = t & 1;
        if (ct * kTurnCols + col < cols && half * 4 < pieces)
            *reinterpret_cast<uint32_t*>(scales + (ct * kTurnCols + col) * (rowsp / kMxGroup) + rt * 8 + half * 4) =
                *reinterpret_cast<const uint32_t*>(bytes + col * 8 + half * 4);
    }
}

// ---------------------------------------------------------------------------------
// The values of eight codes, in pairs of bf16
__device__ __forceinline__ u32x4 mx_values8(uint32_t codes, uint32_t byte) {
    const float f = mx_scale_value(byte);
    u32x4 o;
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 0));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 1));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 2));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 3));
    return byte == kMxNaN ? u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u} : o;
}

// The values of stored codes: a lane turns one word (8 codes) into 16 bytes.
template <int U>
__global__ __launch_bounds__(256) void mx_dequant_kernel(const uint32_t* __restrict__ q, const uint8_t* __restrict__ scales, int64_t rows,
                                                         int64_t cols, uint16_t* __restrict__ out, int64_t ld, int64_t first_wg) {
    const int t = static_cast<int>(threadIdx.x), l16 = t & 15;
    const int64_t nb = (cols + kMxPad - 1) / kMxPad, total = rows * nb;
    const int64_t first = (first_wg + blockIdx.x) * (16 * U) + (t >> 4);
    int64_t row = first / nb, b = first - row * nb;
    const int64_t step_row = 16 / nb, step_b = 16 - step_row * nb;
    uint32_t v[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t unit = first + u * 16;
        v[u] = unit < total ? q[unit * 16 + l16] : 0u;
        s[u] = unit < total ? scales[unit * 4 + (l16 >> 2)] : 0u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t c = b * kMxPad + l16 * 8;
        if (row < rows && c < cols) {
            u32x4 o = mx_values8(v[u], s[u]);
            uint16_t* p = out + row * ld + c;
            if (c + 8 <= cols) *reinterpret_cast<u32x4_any*>(p) = o;
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < cols) p[i] = static_cast<uint16_t>(o[i >> 1] >> ((i & 1) * 16));
            }
        }
        row += step_row;
        b += step_b;
        if (b >= nb) { b -= nb; ++row; }
    }
}

// ---------------------------------------------------------------------------------
loka_status mxfp4_quantize_launch(const void* x_bf16, int64_t rows, int64_t cols, int64_t ld, int transpose_out, uint8_t* q,
                                  uint8_t* scales, hipStream_t stream) {
    const uint16_t* x = static_cast<const uint16_t*>(x_bf16);
    // An input that the 256 MB of last-level cache cannot hold is read past it: 32768 x 4096 62 -> 58 us, turned 72 -> 65. A smaller one may
    // lie there already, and loses: 16384 x 4096 27.8 -> 31.8 us when its values were read just before, and 31.3 -> 31.4 when not.
    const bool streamed = rows * cols >= INT64_C(1) << 27;
    if (transpose_out) {
        const int64_t groups = ((rows + kTurnRows - 1) / kTurnRows) * ((cols + kTurnCols - 1) / kTurnCols);
        return in_launches(groups, 512, [&](int64_t from, uint32_t grid) {
            if (streamed) mx_quant_turned_kernel<true><<<grid, 512, 0, stream>>>(x, rows, cols, ld, q, scales, from);
            else mx_quant_turned_kernel<false><<<grid, 512, 0, stream>>>(x, rows, cols, ld, q, scales, from);
        });
    }
    constexpr int U = 4;
    uint32_t* qw = reinterpret_cast<uint32_t*>(q);
    uint32_t* sw = reinterpret_cast<uint32_t*>(scales);
    return in_launches((rows * (mx_padded(cols) / kMxPad) + 16 * U - 1) / (16 * U), 256, [&](int64_t from, uint32_t grid) {
        if (streamed) mx_quant_rows_kernel<U, true><<<grid, 256, 0, stream>>>(x, rows, cols, ld, qw, sw, from);
        else mx_quant_rows_kernel<U, false><<<grid, 256, 0, stream>>>(x, rows, cols, ld, qw, sw, from);
    });
}

loka_status mxfp4_dequantize_launch(const uint8_t* q, const uint8_t* scales, int64_t rows, int64_t cols, void* out_bf16, int64_t ld,
                                    hipStream_t stream) {
    constexpr int U = 4;
    const uint32_t* qw = reinterpret_cast<const uint32_t*>(q);
    uint16_t* out = static_cast<uint16_t*>(out_bf16);
    return in_launches((rows * (mx_padded(cols) / kMxPad) + 16 * U - 1) / (16 * U), 256, [&](int64_t from, uint32_t grid) {
        mx_dequant_kernel<U><<<grid, 256, 0, stream>>>(qw, scales, rows, cols, out, ld, from);
    });
}

}  // namespace loka
