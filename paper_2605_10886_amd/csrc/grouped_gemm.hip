// Products of ragged groups of rows with their group's weights, and the weights' gradients (include/loka.h: loka_grouped_gemm,
// loka_grouped_linear, loka_grouped_wgrad), on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A lane of that instruction holds 32 codes of one row of each operand (row l % 16) and one scale byte for them; with a scale per 128
// elements the four lanes of a row pass the same byte, the exponent field of the stored fp32 power of two.  The weights are the
// first operand and their rows are dealt so that a lane holds 8 neighbouring columns of one row of the result per two instructions.
#include "experts.h"
#include "gemm_common.h"

namespace loka {

struct GgArgs {
    const uint8_t *xq, *wq;
    const float *sx, *sw;
    const int32_t *index, *offsets;
    uint16_t* out;
    float* y;
    int64_t N;
    int rows, x_rows, groups, ksteps;  // ksteps: K in steps of 128
    int M, blocks;                     // weight gradient: rows of a result; blocks of 128 rows that the operands have
    // element (row r, step k) of an operand lies r * row + k * step bytes from its start (scales: floats), a group's part of it `group` further on
    int64_t x_row, x_step, sx_row, sx_step, w_row, w_step, w_group, sw_row, sw_step, sw_group;
    int tiles_n, tiles_m;              // (tiles_m: weight gradient)
    bool wide;                         // rows of whole 16-byte runs
};

__device__ __forceinline__ v4f gg_mfma(const v8i a, const v8i b, v4f c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}
__device__ __forceinline__ v8i join(u32x4 a, u32x4 b) {
    return v8i{static_cast<int>(a.x), static_cast<int>(a.y), static_cast<int>(a.z), static_cast<int>(a.w),
               static_cast<int>(b.x), static_cast<int>(b.y), static_cast<int>(b.z), static_cast<int>(b.w)};
}
// the scale operand from a stored scale (byte 255 where that is a NaN)
__device__ __forceinline__ int scale_byte(uint32_t bits) { return static_cast<int>(bits >> 23); }

// Eight columns n .. n + 7 of a row of N
__device__ __forceinline__ void put8(uint16_t* row, int64_t n, int64_t N, const float (&f)[8]) {
    const u32x4 v{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    if (n + 8 <= N) *reinterpret_cast<u32x4_any*>(row + n) = v;
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < N) row[n + e] = static_cast<uint16_t>(v[e >> 1] >> ((e & 1) * 16));
}
__device__ __forceinline__ void put8(float* row, int64_t n, int64_t N, const float (&f)[8]) {
    if (n + 8 <= N) {
        *reinterpret_cast<u32x4_any*>(row + n) = __builtin_bit_cast(u32x4, v4f{f[0], f[1], f[2], f[3]});
        *reinterpret_cast<u32x4_any*>(row + n + 4) = __builtin_bit_cast(u32x4, v4f{f[4], f[5], f[6], f[7]});
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < N) row[n + e] = f[e];
    }
}

// ---------------------------------------------------------------------------------
// Tiles in LDS.  A workgroup of WM x WN waves computes BM x BN values, each wave TM x TN tiles of 16 x 16, in steps of 128 along the
// contraction: 128 bytes a row, two steps in LDS.  The 16-byte chunks of a row lie permuted so that the 16 rows of a read use all
// banks: chunk c of X's row r at place c ^ (r / 2 % 8), of W's row r, whose reads take rows 8 apart, at c ^ (bits 1, 3 and 4 of r).
template <int TM_, int TN_, int WM_, int WN_>
struct GgTile {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, NW = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16;
    static constexpr int OFF_W = BM * 128, OFF_SX = OFF_W + BN * 128, OFF_SW = OFF_SX + BM * 4, STAGE = OFF_SW + BN * 4, LDS = 2 * STAGE;
    static constexpr int LX = BM / (8 * NW), LW = BN / (8 * NW), SROWS = (BM + BN) / 64;
    static constexpr int PER_CU = 163840 / LDS;
    static_assert(SROWS == NW && TM % 4 == 0 && TN % 2 == 0 && (NW == 4 || NW == 8));
};

template <class C, bool WGRAD>
__device__ __forceinline__ void gg_tiles(const GgArgs& a, uint8_t* smem) {
    constexpr int TM = C::TM, TN = C::TN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int wm = wave / C::WN, wn = wave % C::WN;

    // ---- which tile: rows m0 .. m0 + m_count - 1 of the result's rows, columns from n0 on, of `group`
    int group, tm, tn, m_first, m_count, ksteps;
    int64_t block0 = 0;                // weight gradient: the group's first block of 128 rows
    if (WGRAD) {
        const int per = a.tiles_m * a.tiles_n, t = xcd_contiguous(blockIdx.x, gridDim.x);
        group = t / per;
        banded_tile(t - group * per, a.tiles_m, a.tiles_n, tm, tn);
        // (of groups that overlap: no more blocks than there are)
        const int first = units_before(a.offsets, group, a.rows, kGroupBlock), own = (group_rows(a.offsets, group, a.rows).count + kGroupBlock - 1) / kGroupBlock;
        block0 = first < 0 ? 0 : first < a.blocks ? first : a.blocks;
        ksteps = a.blocks - static_cast<int>(block0) < own ? a.blocks - static_cast<int>(block0) : own;
        m_first = tm * C::BM;
        m_count = a.M - m_first < C::BM ? a.M - m_first : C::BM;
    } else {
        const int total = units_of_all(a.offsets, a.groups, a.rows, C::BM) * a.tiles_n;
        if (static_cast<int>(blockIdx.x) >= total) return;
        const int t = xcd_contiguous(blockIdx.x, total);
        const UnitAt at = find_unit(a.offsets, a.groups, a.rows, C::BM, t / a.tiles_n);
        if (at.group < 0) return;
        group = at.group;
        banded_tile(t - at.before * a.tiles_n, (at.count + C::BM - 1) / C::BM, a.tiles_n, tm, tn);
        m_first = at.first + tm * C::BM;
        m_count = at.count - tm * C::BM < C::BM ? at.count - tm * C::BM : C::BM;
        ksteps = a.ksteps;
    }
    const int n0 = tn * C::BN, n_count = a.N - n0 < C::BN ? static_cast<int>(a.N - n0) : C::BN;

    // ---- where the wave's loads find things: 8 rows of 128 bytes a load
    // (rows past the end: X reads the last one, W zeros; what they give is not written)
    auto x_source = [&](int row) __attribute__((always_inline)) {
        int64_t s = m_first + (row < m_count ? row : m_count - 1);
        if (!WGRAD && a.index) {
            s = a.index[s];
            s = s < 0 ? 0 : s >= a.x_rows ? a.x_rows - 1 : s;
        }
        return s;
    };
    const uint8_t* xp[C::LX];
#pragma unroll
    for (int i = 0; i < C::LX; ++i) {
        const int row = (i * C::NW + wave) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((lane >> 4) | ((wave & 1) << 2));
        xp[i] = a.xq + block0 * a.x_step + x_source(row) * a.x_row + chunk * 16;
    }
    const int w_chunk = (lane & 7) ^ ((lane >> 4) & 1) ^ ((wave & 3) << 1);
    const int w_lane = (lane >> 3) * static_cast<int>(a.w_row) + w_chunk * 16;
    const uint8_t* wp = a.wq + (WGRAD ? block0 * a.w_step : group * a.w_group) + static_cast<int64_t>(n0) * a.w_row;
    const int w_bytes = (n_count - 1) * static_cast<int>(a.w_row) + 128;
    // scales: 64 rows a load, those of X by the first waves
    const bool scales_of_x = wave < C::BM / 64;
    const float* sxp = a.sx + block0 * a.sx_step + x_source(scales_of_x ? wave * 64 + lane : 0) * a.sx_row;
    const int sw_local = (wave - C::BM / 64) * 64 + lane;
    const float* swp = a.sw + (WGRAD ? block0 * a.sw_step : group * a.sw_group) + (n0 + (!scales_of_x && sw_local < n_count ? sw_local : 0)) * a.sw_row;
    const float* sp = scales_of_x ? sxp : swp;
    const int64_t s_step = scales_of_x ? a.sx_step : a.sw_step;

    auto to_lds = [&](const void* p, int at, auto size) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p, (__attribute__((address_space(3))) void*)(smem + at), size.value, 0, 0);
    };
    auto request = [&](int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C::LX; ++i) {
            to_lds(xp[i], stage + (i * C::NW + wave) * 1024, std::integral_constant<int, 16>{});
            xp[i] += a.x_step;
        }
        const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(wp), 0, w_bytes, 0x00020000);
#pragma unroll
        for (int i = 0; i < C::LW; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (__attribute__((address_space(3))) void*)(smem + stage + C::OFF_W + (i * C::NW + wave) * 1024), 16,
                                                     w_lane, (i * C::NW + wave) * 8 * static_cast<int>(a.w_row), 0, 0);
        wp += a.w_step;
        to_lds(sp, stage + C::OFF_SX + wave * 256, std::integral_constant<int, 4>{});
        sp += s_step;
    };

    // ---- where it reads operands
    const int w_r = (r >> 2) * 8 + (r & 3);                // column, of the 32 of two tiles, that row r of the first one stands for
    int x_off[2], w_off[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        x_off[h] = (wm * TM * 16 + r) * 128 + ((2 * g + h) ^ ((r >> 1) & 7)) * 16;
        w_off[h] = C::OFF_W + (wn * TN * 16 + w_r) * 128 + ((2 * g + h) ^ (((r >> 1) & 1) | ((r >> 2) << 1))) * 16;
    }
    const int sx_off = C::OFF_SX + (wm * TM * 16 + r) * 4, sw_off = C::OFF_SW + (wn * TN * 16 + w_r) * 4;
    v4f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    if (ksteps > 0) request(0);
    for (int k = 0; k < ksteps; ++k) {
        const int stage = (k & 1) * C::STAGE;
        if (k + 1 < ksteps) {
            request(C::STAGE - stage);
            wait_vmcnt<C::LX + C::LW + 1>();
        } else {
            wait_vmcnt<0>();
        }
        lds_barrier();
        v8i w[TN];
        int sw[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const uint8_t* p = smem + stage + coff_of(j) * 128;
            w[j] = join(*reinterpret_cast<const u32x4*>(p + w_off[0]), *reinterpret_cast<const u32x4*>(p + w_off[1]));
            sw[j] = scale_byte(*reinterpret_cast<const uint32_t*>(smem + stage + sw_off + coff_of(j) * 4));
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint8_t* p = smem + stage + i * 2048;
            const v8i x = join(*reinterpret_cast<const u32x4*>(p + x_off[0]), *reinterpret_cast<const u32x4*>(p + x_off[1]));
            const int sx = scale_byte(*reinterpret_cast<const uint32_t*>(smem + stage + sx_off + i * 64));
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = gg_mfma(w[j], x, acc[i][j], sw[j], sx);
        }
        lds_barrier();
    }

    // ---- lane (r, g) holds row 16 i + r, columns 32 (j / 2) + 8 g + 0 .. 7
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = (wm * TM + i) * 16 + r;
        if (row >= m_count) continue;
        const int64_t at = (WGRAD ? static_cast<int64_t>(group) * a.M + m_first + row : static_cast<int64_t>(m_first) + row) * a.N;
#pragma unroll
        for (int j = 0; j < TN; j += 2) {
            const int64_t n = n0 + wn * TN * 16 + j * 16 + g * 8;
            const float f[8] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], acc[i][j + 1][0], acc[i][j + 1][1], acc[i][j + 1][2], acc[i][j + 1][3]};
            if (a.out) put8(a.out + at, n, a.N, f);
            if (a.y) put8(a.y + at, n, a.N, f);
        }
    }
}

template <class C, bool WGRAD>
__global__ __launch_bounds__(64 * C::NW, C::NW * C::PER_CU / 4) void gg_tile_kernel(const GgArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    gg_tiles<C, WGRAD>(a, smem);
}

using GgLarge = GgTile<8, 4, 2, 4>;
using GgSmall = GgTile<4, 4, 2, 2>;

template <class C>
static int64_t tiles_of(const loka_grouped_desc* d) {       // that the groups can take
    const int64_t some = d->rows < d->groups ? d->rows : d->groups;
    return (d->rows + (C::BM - 1) * some) / C::BM * ((d->N + C::BN - 1) / C::BN);
}
template <class C>
static int64_t wgrad_tiles_of(const loka_grouped_desc* d) { return (d->K + C::BM - 1) / C::BM * ((d->N + C::BN - 1) / C::BN) * d->groups; }

bool grouped_gemm_fits(const loka_grouped_desc* d) { return tiles_of<GgSmall>(d) <= INT32_MAX / 512; }
bool grouped_wgrad_fits(const loka_grouped_desc* d) { return wgrad_tiles_of<GgSmall>(d) <= INT32_MAX / 512; }

template <class C, bool WGRAD>
static loka_status gg_launch(GgArgs& a, int64_t grid, hipStream_t stream) {
    a.tiles_n = static_cast<int>((a.N + C::BN - 1) / C::BN);
    a.tiles_m = WGRAD ? (a.M + C::BM - 1) / C::BM : 0;
    LOKA_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&gg_tile_kernel<C, WGRAD>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS));
    gg_tile_kernel<C, WGRAD><<<static_cast<uint32_t>(grid), 64 * C::NW, C::LDS, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

loka_status grouped_gemm_launch(const loka_grouped_desc* d, const uint8_t* xq, const float* sx, const int32_t* index, const int32_t* offsets,
                                const uint8_t* wq, const float* sw, void* out, float* y, hipStream_t stream) {
    GgArgs a{};
    const int64_t kb = group_blocks(d->K), N = d->N;
    a.xq = xq;
    a.sx = sx;
    a.wq = wq;
    a.sw = sw;
    a.index = index;
    a.offsets = offsets;
    a.out = static_cast<uint16_t*>(out);
    a.y = y;
    a.N = N;
    a.rows = static_cast<int>(d->rows);
    a.x_rows = index ? static_cast<int>(d->x_rows) : a.rows;
    a.groups = d->groups;
    a.ksteps = static_cast<int>(kb);
    a.x_row = kb * kGroupBlock;
    a.x_step = kGroupBlock;
    a.sx_row = kb;
    a.sx_step = 1;
    const bool turned = d->w_form == LOKA_W_TURNED;
    a.w_row = turned ? kGroupBlock : kb * kGroupBlock;
    a.w_step = turned ? N * kGroupBlock : kGroupBlock;
    a.w_group = N * kb * kGroupBlock;
    a.sw_row = turned ? 1 : kb;
    a.sw_step = turned ? N : 1;
    a.sw_group = N * kb;
    if (d->rows >= 192 * static_cast<int64_t>(d->groups) && N > 128) return gg_launch<GgLarge, false>(a, tiles_of<GgLarge>(d), stream);
    return gg_launch<GgSmall, false>(a, tiles_of<GgSmall>(d), stream);
}

size_t grouped_wgrad_workspace_bytes(const loka_grouped_desc*) { return 0; }

loka_status grouped_wgrad_launch(const loka_grouped_desc* d, const uint8_t* xt, const float* sxt, const uint8_t* dyt, const float* sdyt,
                                 const int32_t* offsets, void* dw, float* dw32, void*, size_t, hipStream_t stream) {
    GgArgs a{};
    a.xq = xt;
    a.sx = sxt;
    a.wq = dyt;
    a.sw = sdyt;
    a.offsets = offsets;
    a.out = static_cast<uint16_t*>(dw);
    a.y = dw32;
    a.N = d->N;
    a.M = static_cast<int>(d->K);
    a.blocks = static_cast<int>(loka_grouped_blocks(d->rows, d->groups));
    a.rows = static_cast<int>(d->rows);
    a.groups = d->groups;
    a.x_row = a.w_row = kGroupBlock;
    a.x_step = d->K * kGroupBlock;
    a.w_step = d->N * kGroupBlock;
    a.sx_row = a.sw_row = 1;
    a.sx_step = d->K;
    a.sw_step = d->N;
    if (d->K > 128 && d->N > 128 && wgrad_tiles_of<GgLarge>(d) >= 256) return gg_launch<GgLarge, true>(a, wgrad_tiles_of<GgLarge>(d), stream);
    return gg_launch<GgSmall, true>(a, wgrad_tiles_of<GgSmall>(d), stream);
}

}  // namespace loka
