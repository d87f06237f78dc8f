// 8-bit operands of grouped products in their two stored forms (include/loka.h, loka_grouped_quantize): scale = the least power of two s with
// max |x| / s <= 448 over 128 elements, code = x / s.  Bytes only: 2 read and 1 + 1/32 written per element and form, and both forms from one read.
#include "experts.h"

namespace loka {

struct GqArgs {
    const uint16_t* x;
    const int32_t *index, *offsets;
    uint8_t *q, *qt;
    float *scales, *st;
    int64_t rows, cols, ld, x_rows, first_wg;
    int64_t per_group, blocks_per_group;           // offsets == nullptr
    int groups, col_tiles;
};

// the source row of row p, or -1: a row of zeros
__device__ __forceinline__ int64_t gq_source(const GqArgs& a, int64_t p) {
    if (!a.index) return p;
    const int64_t s = a.index[p];
    return s >= 0 && s < a.x_rows ? s : -1;
}

// Sources of 2^27 elements and more pass the last-level cache (256 MB) by, which cannot hold them (32768 x 4096: 61.5 us, else 72.0, both forms 90.5 and 105;
// 16384 x 4096: 33.4 and 30.3, both forms 49.5 and 48.5).  What counts is the source that is read, not the rows made of it: gathered rows come back to it
// (through the cache and past it, along / turned / both: 16384 x 1024, each row 8 times, 59.7 / 46.0 / 78.8 and 67.2 / 65.8 / 95.4; 16384 x 4096, 8 times, 220 / 227 / 431
// and 284 / 298 / 426; 24000 x 4096, 4 times, 176 / 176 / 283 and 212 / 211 / 305; both forms of 16384 x 4096, twice, are the exception: 109 and 95).
template <bool STREAMED>
__device__ __forceinline__ u32x4 gq_load8(const uint16_t* p) {
    if (STREAMED) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
    return *reinterpret_cast<const u32x4_any*>(p);
}

// ALONG: 16 lanes take 128 elements of a row, 8 each; U such blocks at a time, 16 blocks apart.  (One division, of 32 bits where they do.)
// WHOLE: no run of 8 is cut by a row's end.  16384 x 4096: 30 us (203 MB, 6.7 TB/s).
template <int U, bool WHOLE, bool STREAMED>
__global__ __launch_bounds__(256) void gq_along_kernel(const GqArgs a) {
    const int t = static_cast<int>(threadIdx.x), l = t & 15;
    const int nb = a.col_tiles;
    int64_t rows = a.rows;
    if (a.offsets) {
        const int last = a.offsets[a.groups];
        rows = last < 0 ? 0 : last < rows ? last : rows;
    }
    const int64_t total = rows * nb, first = (a.first_wg + blockIdx.x) * (16 * U) + (t >> 4);
    int64_t row = first >> 32 ? first / nb : static_cast<int64_t>(static_cast<uint32_t>(first) / static_cast<uint32_t>(nb));
    int b = static_cast<int>(first - row * nb);
    const int step_row = 16 / nb, step_b = 16 - step_row * nb;
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (first + u * 16 < total) {
            const int64_t s = gq_source(a, row);
            const int c = b * kGroupBlock + l * 8;
            if (WHOLE) {
                if (s >= 0 && c < a.cols) v[u] = gq_load8<STREAMED>(a.x + s * a.ld + c);
            } else if (s >= 0) {
                v[u] = mx_load8(a.x + s * a.ld, c, a.cols);
            }
        }
        row += step_row;
        b += step_b;
        if (b >= nb) { b -= nb; ++row; }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t unit = first + u * 16;
        float scale;
        const bool finite = gq_scale(lanes_max_bits<16>(max_abs8(v[u])), scale);
        const u32x2 c = gq_codes8(v[u], scale, finite);
        if (unit < total) {
            *reinterpret_cast<u32x2*>(a.q + unit * kGroupBlock + l * 8) = c;
            if (l == 0) a.scales[unit] = scale;
        }
    }
}

// TURNED, and ALONG from the same read: a workgroup takes a block of 128 rows of one group x 128 columns; a thread 8 rows x 8 columns.
// Maxima down a column cross the wave by lane exchanges and the waves through LDS; the codes turn in LDS (runs of 8 rows of a
// column, run r at place r ^ (column / 8)) and leave in whole lines.  Both forms of 16384 x 4096: 49 us (272 MB, 5.5 TB/s), of 32768 x
// 4096 90 us (6.0 TB/s); the turned one alone of 32768 gathered rows x 1024 18 us.
template <bool ALONG, bool STREAMED>
__global__ __launch_bounds__(256) void gq_turned_kernel(const GqArgs a) {
    __shared__ __align__(16) uint8_t codes[128 * 128];
    __shared__ __align__(16) u32x4 maxima[4][16];
    __shared__ __align__(16) int source[128];              // rows of x, -1 for zeros
    const int t = static_cast<int>(threadIdx.x), cg = t & 15, rg = t >> 4, wave = t >> 6;
    const int64_t wg = a.first_wg + blockIdx.x;
    const int64_t block = wg >> 32 ? wg / a.col_tiles : static_cast<int64_t>(static_cast<uint32_t>(wg) / static_cast<uint32_t>(a.col_tiles)), ct = wg - block * a.col_tiles;
    int64_t row0;
    int count;
    if (a.offsets) {
        const UnitAt at = find_unit(a.offsets, a.groups, static_cast<int>(a.rows), kGroupBlock, static_cast<int>(block));
        if (at.group < 0) return;
        const int skip = (static_cast<int>(block) - at.before) * kGroupBlock;
        row0 = at.first + skip;
        count = at.count - skip;
    } else {
        const int64_t g = static_cast<uint32_t>(block) / static_cast<uint32_t>(a.blocks_per_group), skip = (block - g * a.blocks_per_group) * kGroupBlock;
        row0 = g * a.per_group + skip;
        count = static_cast<int>(a.per_group - skip < kGroupBlock ? a.per_group - skip : kGroupBlock);
    }
    if (count > kGroupBlock) count = kGroupBlock;
    if (t < 128) source[t] = t < count ? static_cast<int>(gq_source(a, row0 + t)) : -1;
    __syncthreads();
    const int64_t c = ct * 128 + cg * 8;
    u32x4 v[8];
    {
        // (a run that the row's end cuts comes from the row's last eight)
        const bool few = a.cols < 8;
        const int64_t at = c + 8 <= a.cols || few ? c : a.cols - 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t s = source[rg * 8 + i];
            v[i] = u32x4{0u, 0u, 0u, 0u};
            if (s >= 0 && !few) v[i] = gq_load8<STREAMED>(a.x + s * a.ld + at);
        }
        if (ct * 128 + 128 > a.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (few) {
                    const int64_t s = source[rg * 8 + i];
                    if (s >= 0) v[i] = mx_load8(a.x + s * a.ld, c, a.cols);
                } else {
                    v[i] = mx_from(v[i], c - at);
                }
            }
        }
    }
    u32x4 m = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = max_abs_bf16x2(m[e], v[i][e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m[e] = max_abs_bf16x2(m[e], __shfl_xor(m[e], 16, 64));
        m[e] = max_abs_bf16x2(m[e], __shfl_xor(m[e], 32, 64));
    }
    if ((t & 63) < 16) maxima[wave][cg] = m;
    if (ALONG) {
        const int64_t kb = (a.cols + kGroupBlock - 1) / kGroupBlock;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float scale;
            const bool finite = gq_scale(lanes_max_bits<16>(max_abs8(v[i])), scale);
            const int r = rg * 8 + i;
            if (r < count) {
                const int64_t unit = (row0 + r) * kb + ct;
                *reinterpret_cast<u32x2*>(a.q + unit * kGroupBlock + cg * 8) = gq_codes8(v[i], scale, finite);
                if (cg == 0) a.scales[unit] = scale;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const u32x4 o = maxima[w][cg];
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = max_abs_bf16x2(m[e], o[e]);
    }
    float scale[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const bool finite = gq_scale((k & 1) ? m[k >> 1] >> 16 : m[k >> 1] & 0xFFFFu, scale[k]);
        // (the column's elements of two rows as a word)
        auto two = [&](int i) __attribute__((always_inline)) { return __builtin_amdgcn_perm(v[i + 1][k >> 1], v[i][k >> 1], (k & 1) ? 0x07060302u : 0x05040100u); };
        const u32x2 o{gq_codes4(two(0), two(2), scale[k]), gq_codes4(two(4), two(6), scale[k])};
        *reinterpret_cast<u32x2*>(codes + (cg * 8 + k) * 128 + ((rg ^ cg) * 8)) = finite ? o : u32x2{0u, 0u};
    }
    if (rg == 0) {
        float* const st = a.st + block * a.cols + c;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < a.cols) st[k] = scale[k];
    }
    __syncthreads();
    uint8_t* const out = a.qt + (block * a.cols + ct * 128) * 128;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = t + k * 256, col = i >> 3, p = i & 7, g = col >> 3;
        if (ct * 128 + col < a.cols) {
            const u32x2 lo = *reinterpret_cast<const u32x2*>(codes + col * 128 + ((2 * p) ^ g) * 8);
            const u32x2 hi = *reinterpret_cast<const u32x2*>(codes + col * 128 + ((2 * p + 1) ^ g) * 8);
            *reinterpret_cast<u32x4*>(out + col * 128 + p * 16) = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    }
}

loka_status grouped_quantize_launch(const loka_grouped_quantize_desc* d, const void* x, const int32_t* index, const int32_t* offsets, uint8_t* q,
                                    float* scales, uint8_t* qt, float* st, hipStream_t stream) {
    GqArgs a{};
    a.x = static_cast<const uint16_t*>(x);
    a.index = index;
    a.offsets = offsets;
    a.q = q;
    a.scales = scales;
    a.qt = qt;
    a.st = st;
    a.rows = d->rows;
    a.cols = d->cols;
    a.ld = d->ld;
    a.x_rows = d->x_rows;
    a.groups = d->groups;
    a.col_tiles = static_cast<int>(group_blocks(d->cols));
    a.per_group = d->rows / d->groups;
    a.blocks_per_group = group_blocks(a.per_group);
    const bool streamed = (index && a.x_rows < a.rows ? a.x_rows : a.rows) * a.cols >= INT64_C(1) << 27;
    if (!qt) {
        // (blocks a thread: 4 in flight where there are many: 16384 x 1024 8.9 us, with 1 10.3; 1 where 4 leave CUs idle: 1024 x 1024 2.4 us, with 4 3.2)
        const int64_t units = d->rows * a.col_tiles;
        auto go = [&](auto u, auto whole, auto past) {
            return in_launches((units + 16 * u.value - 1) / (16 * u.value), 256, [&](int64_t from, uint32_t grid) {
                a.first_wg = from;
                gq_along_kernel<u.value, whole.value, past.value><<<grid, 256, 0, stream>>>(a);
            });
        };
        const bool many = units >= 131072;
        using std::integral_constant;
        const std::true_type yes;
        const std::false_type no;
        if (d->cols % 8 == 0 && streamed) return go(integral_constant<int, 4>{}, yes, yes);
        if (d->cols % 8 == 0) return many ? go(integral_constant<int, 4>{}, yes, no) : go(integral_constant<int, 1>{}, yes, no);
        return many ? go(integral_constant<int, 4>{}, no, no) : go(integral_constant<int, 1>{}, no, no);
    }
    const int64_t blocks = offsets ? loka_grouped_blocks(d->rows, d->groups) : a.blocks_per_group * d->groups;
    return in_launches(blocks * a.col_tiles, 256, [&](int64_t from, uint32_t grid) {
        a.first_wg = from;
        if (q && streamed) gq_turned_kernel<true, true><<<grid, 256, 0, stream>>>(a);
        else if (q) gq_turned_kernel<true, false><<<grid, 256, 0, stream>>>(a);
        else if (streamed) gq_turned_kernel<false, true><<<grid, 256, 0, stream>>>(a);
        else gq_turned_kernel<false, false><<<grid, 256, 0, stream>>>(a);
    });
}

}  // namespace loka
