// Products of ragged groups of rows with their group's weights, and the weights' gradients (include/loka.h: loka_grouped_gemm,
// loka_grouped_linear, loka_grouped_wgrad), on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A lane of that instruction holds 32 codes of one row of each operand (row l % 16) and one scale byte for them; with a scale per 128
// elements the four lanes of a row pass the same byte, the exponent field of the stored fp32 power of two.
//
// Eight products at a time are cut to multiples of 2^-13 of the power of two of the largest of them before they are added, in fp32 from there on: what the
// FP8 instructions of this chip do, in every kernel of this library but the exact-product ones.  Against 64 bits that is 1e-5 to 8e-5 of a result in
// the norm, 1 to 3 in a hundred of the bf16 results by one step; e4m3's own rounding is 3e-2.
#include "experts.h"
#include "gemm_common.h"

#include <cmath>

namespace loka {

struct GgArgs {
    const uint8_t *xq, *wq;
    const float *sx, *sw;
    const int32_t *index, *offsets;
    uint16_t* out;
    float* y;
    int64_t N;
    int rows, x_rows, groups, ksteps;  // x_rows: of the operand X; ksteps: K in steps of 128
    int M, blocks, splits;             // weight gradient: rows of a result; blocks of 128 rows that the operands have; ranges of a group's blocks, whose sums go to y
    // element (row r, step k) of an operand lies r * row + k * step bytes from its start (scales: floats), a group's part of it `group` further on
    int64_t x_row, x_step, sx_row, sx_step, w_row, w_step, w_group, sw_row, sw_step, sw_group;
    int tiles_n, tiles_m, tiles;       // (tiles_m: weight gradient); tiles that there can be
    bool wide;                         // rows of whole runs of 4 columns
    const uint16_t* x;                 // few rows, quantized in the kernel: bf16 [x_rows, ldx]
    int64_t ldx, K;
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

// Four columns n .. n + 3 of a row of N
__device__ __forceinline__ void put4(uint16_t* row, int64_t n, int64_t N, v4f f) {
    if (n + 4 <= N) *reinterpret_cast<u32x2_any*>(row + n) = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) row[n + e] = static_cast<uint16_t>(f32_to_bf16_rne(f[e]));
}
__device__ __forceinline__ void put4(float* row, int64_t n, int64_t N, v4f f) {
    if (n + 4 <= N) *reinterpret_cast<u32x4_any*>(row + n) = __builtin_bit_cast(u32x4, f);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) row[n + e] = f[e];
}

// ---------------------------------------------------------------------------------
// Tiles in LDS.  A workgroup of WM x WN waves computes BM x BN values, each wave TM x TN tiles of 16 x 16, in steps of 128 along the
// contraction: 128 bytes a row, two steps in LDS (of the scales three).  The 16-byte chunks of a row lie permuted so that the 16 rows of a read use all
// banks: chunk c of row r at place c ^ (r / 2 % 8).  W's rows are dealt: row 16 j + r of a wave's 64 is column 4 r + j, so that a lane's four values of a row
// are neighbours and 16 lanes store 128 bytes of it (with 64 bytes of each of 16 rows from 16 lanes each, 32768 rows x 1024 x 4096 took 192 us, so 177).
//
// A step is TM / 2 pairs of X's 16-row fragments against all of the wave's W fragments; a pair is read while the pair before it is
// multiplied, W's fragments and the first pair of the next step during the last.  Two barriers a step, in front of the second pair and
// of the last, give LDS back as soon as it is read: behind the first one W and the first two pairs of X of the step after next are
// requested, behind the second X's other pairs, and each is awaited 1.5 steps later (a round trip through L2 under load is longer than a
// step; with one barrier, and one step, 32768 rows x 4096 x 4096 took 583 us where this took 555).  With two pairs to a step there is one barrier.  Workgroups are
// persistent, and the stream of steps does not stop between result tiles: the next tile's first steps arrive while this one's
// values are stored, and nothing waits for the stores where their number is known.
//
// Bound by the matrix cores and the power they draw: 32768 rows x 16 groups x 4096 x 4096 (256 x 256 tiles) 555 .. 590 us by the card, 1.86 .. 1.98 PFLOP/s at
// 1.9 GHz; loka_fp8_gemm_norm's kernel for one group of these sizes 490, this one 497: the rest is tiles that a group's end cuts and the last round.
// x 1024 x 4096 177 us (158 without its stores), weight gradient 137, 2.0 PFLOP/s.  Tiles of 128 x 128, two workgroups a CU, where those would be few:
// 4096 rows x 8 groups x 256 x 768 7 us.
template <int TM_, int TN_, int WM_, int WN_>
struct GgTile {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, NW = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16;
    static constexpr int OFF_W = BM * 128, STAGE = OFF_W + BN * 128, OFF_S = 2 * STAGE, SCALES = (BM + BN) * 4, LDS = OFF_S + 3 * SCALES;
    static constexpr int PAIRS = TM / 2, LX = BM / (8 * NW), LW = BN / (8 * NW), SROWS = (BM + BN) / 64, LOADS = LX + LW + 1;
    static constexpr int FIRST = PAIRS == 4 ? LW + LX / 2 + 1 : LOADS, SECOND = LOADS - FIRST;      // loads behind the first barrier, and the second
    static constexpr int MOST_LDS = LDS + 12 * kMostGroups, PER_CU = 163840 / MOST_LDS;     // (with the table of the groups)
    static_assert(SROWS == NW && (PAIRS == 2 || PAIRS == 4) && LX == 4 && WM == 2 && TN == 4 && (NW == 4 || NW == 8));
};

template <class C, bool WGRAD>
__device__ __forceinline__ void gg_tiles(const GgArgs& a, uint8_t* smem) {
    constexpr int TM = C::TM, TN = C::TN, PAIRS = C::PAIRS, MM = 2 * TN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int wm = wave / C::WN, wn = wave % C::WN;

    // ---- the groups: cum[i] = units (tiles of BM rows; weight gradient: blocks of 128) of groups 0 .. i, and their rows
    int* const cum = reinterpret_cast<int*>(smem + C::LDS);
    int* const off = cum + a.groups;
    // (up to 64 groups: a lane each, ranked without another pass.  More take their own order, which costs uneven ones: 32768 rows x 1024 x 4096 of 66 / 128 / 256 groups
    // with a router's loads 280 / 359 / 606 us, the same groups longest first 236 / 343 / 568)
    const bool sorted = WGRAD && a.groups <= 64 && a.tiles > static_cast<int>(gridDim.x);
    {
        int base = 0, units_here = 0;
        constexpr int UNIT = WGRAD ? kGroupBlock : C::BM;
        for (int g0 = 0; g0 < a.groups; g0 += 64) {        // (every wave by itself, the same values)
            const int i = g0 + lane;
            const GroupRows q = i < a.groups ? group_rows(a.offsets, i, a.rows) : GroupRows{0, 0};
            units_here = units_of(q.count, UNIT);
            const int s = base + lanes_inclusive(units_here);
            if (i < a.groups) {
                cum[i] = s;
                off[2 * i] = q.first;
                off[2 * i + 1] = q.count;
            }
            base = __builtin_amdgcn_readlane(s, 63);
        }
        if (sorted) {                                      // off[i]: the group with the i-th most blocks
            const int n = lane < a.groups ? units_here : -1;
            int rank = 0;
            for (int j = 0; j < a.groups; ++j) {
                const int o = __builtin_amdgcn_readlane(n, j);
                rank += o > n || (o == n && j < lane) ? 1 : 0;
            }
            if (lane < a.groups) off[rank] = lane;
        }
        __syncthreads();
    }
    // (groups that overlap would have more tiles than there are, or so many that their number overflows: no more than there are are taken,
    // and every one of them lies within its group)
    const int units = cum[a.groups - 1], most = a.tiles / a.tiles_n;
    const int total = __builtin_amdgcn_readfirstlane(WGRAD ? a.tiles : (units < 0 ? 0 : units < most ? units : most) * a.tiles_n);
    const int workers = static_cast<int>(gridDim.x) < total ? static_cast<int>(gridDim.x) : total;
    if (static_cast<int>(blockIdx.x) >= workers) return;

    // ---- a tile: rows m_first .. of the operand X (forward: of the routed order), columns n0 .., steps of its contraction
    struct Place { int group, m_first, m_count, n0, n_count, steps, block0, split; };
    auto locate = [&](int t) __attribute__((always_inline)) {
        Place p;
        int tm, tn;
        if (WGRAD) {
            // groups of most steps first, and every other round of tiles from its end: who takes a long one takes a short one next
            // (32768 rows over 16 groups x 1024 x 4096 137 us, in the order of the groups 165)
            const int per = a.tiles_m * a.tiles_n, round = t / workers, from = round * workers;
            const int turned = (round & 1) && from + workers <= total ? from + workers - 1 - (t - from) : t;
            const int range = turned / per;
            banded_tile(turned - range * per, a.tiles_m, a.tiles_n, tm, tn);
            p.group = range / a.splits;
            p.split = range - p.group * a.splits;
            if (sorted) p.group = off[p.group];
            int first = p.group ? cum[p.group - 1] : 0, last = cum[p.group];
            const int each = (last - first + a.splits - 1) / a.splits;
            first += p.split * each;
            last = last < first + each ? last : first + each;
            // (of groups that overlap: no more blocks than there are)
            p.block0 = __builtin_amdgcn_readfirstlane(first < 0 ? 0 : first < a.blocks ? first : a.blocks);
            const int own = last - first, left = a.blocks - p.block0;
            p.steps = __builtin_amdgcn_readfirstlane(own < left ? own : left);
            p.m_first = tm * C::BM;
            p.m_count = a.M - p.m_first;
        } else {
            const int u = t / a.tiles_n;
            int g0 = 0;
            unsigned long long past;
            for (;; g0 += 64) {
                past = __builtin_amdgcn_ballot_w64(g0 + lane < a.groups && cum[g0 + lane < a.groups ? g0 + lane : 0] > u);
                if (past || g0 + 64 >= a.groups) break;
            }
            p.group = g0 + __builtin_ctzll(past);          // (u is less than the last sum)
            const int before = p.group ? cum[p.group - 1] : 0;
            const int first = __builtin_amdgcn_readfirstlane(off[2 * p.group]), count = __builtin_amdgcn_readfirstlane(off[2 * p.group + 1]);
            const int tiles_m = units_of(count, C::BM);
            const int local = t - __builtin_amdgcn_readfirstlane(before) * a.tiles_n;
            banded_tile(local, tiles_m, a.tiles_n, tm, tn);
            p.m_first = first + tm * C::BM;
            p.m_count = count - tm * C::BM;
            p.steps = a.ksteps;
            p.block0 = p.split = 0;
        }
        p.m_count = p.m_count < C::BM ? p.m_count : C::BM;
        p.n0 = tn * C::BN;
        p.n_count = a.N - p.n0 < C::BN ? static_cast<int>(a.N - p.n0) : C::BN;
        // (all of it in scalar registers)
        for (int* v : {&p.group, &p.m_first, &p.m_count, &p.n0, &p.n_count, &p.steps, &p.block0, &p.split}) *v = __builtin_amdgcn_readfirstlane(*v);
        return p;
    };

    // ---- the stream of steps: `ld` is the tile whose steps are requested, `next` the one behind it
    // (rows past the end: X reads the last one, W zeros; what they give is not written)
    const bool scales_of_x = wave < C::BM / 64;            // 64 rows' scales a load, those of X by the first waves
    // row, of the tile, of load i of X: a pair's rows of both halves of the tile (2 TM / LX pairs to a load)
    auto x_row_of = [&](int i) __attribute__((always_inline)) {       // (of lane 0)
        return PAIRS == 4 ? (wave >> 2) * 128 + i * 32 + (wave & 3) * 8 : (i & 1) * 64 + (i >> 1) * 32 + wave * 8;
    };
    int src[C::LX], src_s = 0;         // X's rows of a tile, loaded a tile ahead
    auto x_rows = [&](const Place& p) __attribute__((always_inline)) {
        auto source = [&](int row) __attribute__((always_inline)) {
            const int s = p.m_first + (row < p.m_count ? row : p.m_count - 1);
            return !WGRAD && a.index ? a.index[s] : s;
        };
#pragma unroll
        for (int i = 0; i < C::LX; ++i) src[i] = source(x_row_of(i) + (lane >> 3));
        if (scales_of_x) src_s = source(wave * 64 + lane);
    };
    const uint8_t *xp[C::LX], *wp;
    const float* sp;
    int w_bytes;
    const int x_chunk = ((lane & 7) ^ ((lane >> 4) | ((wave & 1) << 2))) * 16;
    const int w_row = static_cast<int>(a.w_row), w_lane = (lane >> 3) * 4 * w_row + x_chunk;
    auto aim = [&](const Place& p) __attribute__((always_inline)) {
        auto inside = [&](int s) __attribute__((always_inline)) { return static_cast<int64_t>(s < 0 ? 0 : s >= a.x_rows ? a.x_rows - 1 : s); };
#pragma unroll
        for (int i = 0; i < C::LX; ++i) xp[i] = a.xq + p.block0 * a.x_step + inside(src[i]) * a.x_row + x_chunk;
        wp = a.wq + (WGRAD ? p.block0 * a.w_step : p.group * a.w_group) + static_cast<int64_t>(p.n0) * a.w_row;
        w_bytes = (p.n_count - 1) * w_row + 128;
        const int local = (wave - C::BM / 64) * 64 + lane;
        if (scales_of_x) sp = a.sx + p.block0 * a.sx_step + inside(src_s) * a.sx_row;
        else sp = a.sw + (WGRAD ? p.block0 * a.sw_step : p.group * a.sw_group) + (p.n0 + (local < p.n_count ? local : 0)) * a.sw_row;
    };
    const int64_t s_step = scales_of_x ? a.sx_step : a.sw_step;
    auto to_lds = [&](const void* p, int at, auto size) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p, (__attribute__((address_space(3))) void*)(smem + at), size.value, 0, 0);
    };
    // load i of a step: W's, X's first half, the scales; X's second half
    int ld_s = 0;                      // the scales' place
    auto request_x = [&](int stage, int i) __attribute__((always_inline)) {
        to_lds(xp[i], stage + x_row_of(i) * 128, std::integral_constant<int, 16>{});
        xp[i] += a.x_step;
    };
    auto request_one = [&](int stage, int i) __attribute__((always_inline)) {
        if (i < C::LW) {
            const int k = i * C::NW + wave, column = (k >> 3) * 64 + (k & 1) * 32 + ((k >> 1) & 3);
            const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(wp), 0, w_bytes, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (__attribute__((address_space(3))) void*)(smem + stage + C::OFF_W + k * 1024), 16, w_lane, column * w_row, 0, 0);
            if (i == C::LW - 1) wp += a.w_step;
        } else if (i < C::LW + C::LX / 2) {
            request_x(stage, i - C::LW);
        } else if (i == C::LW + C::LX / 2) {
            to_lds(sp, C::OFF_S + ld_s + wave * 256, std::integral_constant<int, 4>{});
            sp += s_step;
            ld_s = ld_s == 2 * C::SCALES ? 0 : ld_s + C::SCALES;
        } else {
            request_x(stage, i - C::LW - 1);
        }
    };
    // the first tile from t on that has steps (weight gradient: an empty group's has none), total where there is none
    auto with_steps = [&](int t, Place& p) __attribute__((always_inline)) {
        while (t < total) {
            p = locate(t);
            if (!WGRAD || p.steps > 0) break;
            t += workers;
        }
        return t;
    };
    const int first_tile = xcd_contiguous(blockIdx.x, workers);
    Place ld, next;
    int ld_k = 0, next_tile = with_steps(first_tile, ld);
    const bool any = next_tile < total;
    auto look_ahead = [&]() __attribute__((always_inline)) {
        if (next_tile < total) next_tile = with_steps(next_tile + workers, next);
        if (next_tile < total) x_rows(next);
    };
    if (any) {
        x_rows(ld);
        aim(ld);
        look_ahead();
    }
    // behind the last tile's steps the same again, so that every step requests as many loads
    auto advance = [&]() __attribute__((always_inline)) {
        if (++ld_k < ld.steps) return;
        ld_k = 0;
        if (next_tile < total) ld = next;
        aim(ld);
        look_ahead();
    };

    // ---- operands
    int x_off[2], w_off[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        x_off[h] = (wm * TM * 16 + r) * 128 + ((g + 4 * h) ^ ((r >> 1) & 7)) * 16;
        w_off[h] = C::OFF_W + (wn * TN * 16 + r) * 128 + ((g + 4 * h) ^ ((r >> 1) & 7)) * 16;
    }
    const int sx_off = C::OFF_S + (wm * TM * 16 + r) * 4, sw_off = C::OFF_S + C::BM * 4 + (wn * TN * 16 + r * 4) * 4;
    u32x4 fx[2][2][2], fw[TN][2];
    uint32_t sx[2][2], sw[TN];
    int scales = 0;                    // where the scales lie that are read
    // read i (of 6) of pair p into its set; of W fragment j (of 3)
    auto read_x = [&](int stage, int p, int i) __attribute__((always_inline)) {
        const int f = i / 3, k = i % 3;
        if (k < 2) fx[p & 1][f][k] = *reinterpret_cast<const u32x4*>(smem + stage + (2 * p + f) * 2048 + x_off[k]);
        else sx[p & 1][f] = *reinterpret_cast<const uint32_t*>(smem + scales + sx_off + (2 * p + f) * 64);
    };
    auto read_w = [&](int stage, int j, int k) __attribute__((always_inline)) {
        if (k < 2) fw[j][k] = *reinterpret_cast<const u32x4*>(smem + stage + j * 2048 + w_off[k]);
        else sw[j] = *reinterpret_cast<const uint32_t*>(smem + scales + sw_off + j * 4);
    };
    v4f acc[TM][TN];
    auto multiply = [&](int p, int i) __attribute__((always_inline)) {
        const int j = i >> 1, f = i & 1;
        acc[2 * p + f][j] = gg_mfma(join(fx[p & 1][f][0], fx[p & 1][f][1]), join(fw[j][0], fw[j][1]), acc[2 * p + f][j], scale_byte(sx[p & 1][f]), scale_byte(sw[j]));
    };

    int stage = 0;
    if (any) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i) request_one(k * C::STAGE, i);
            if (k == 0) advance();
        }
        wait_vmcnt<C::SECOND + C::LOADS>();
        lds_barrier();
#pragma unroll
        for (int i = 0; i < 6; ++i) read_x(0, 0, i);
#pragma unroll
        for (int j = 0; j < TN - 1; ++j)
#pragma unroll
            for (int k = 0; k < 3; ++k) read_w(0, j, k);
    }
    // Where a tile's values left in STORES stores, the loads that were requested before them are awaited with the stores in flight.
    constexpr int STORES = TM * 4, NEWER = PAIRS == 4 ? C::LOADS : 0;
    int late = 0;
    auto landed = [&]() __attribute__((always_inline)) {
        if (late > 0) { --late; wait_vmcnt<NEWER + STORES>(); }
        else wait_vmcnt<NEWER>();
        lds_barrier();
    };
    // the matrix instructions of pair p, and between them the LDS reads of the pair behind it (a burst would hold the issue stage up)
    // and `count` of the loads from `from` on into `freed`
    auto pair = [&](int p, int freed, int from, int count) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MM; ++i) {
            multiply(p, i);
            __builtin_amdgcn_sched_barrier(0);
            if (p == 0 && i == 0)
#pragma unroll
                for (int q = 0; q < 3; ++q) read_w(stage, TN - 1, q);
            if (i < 6) read_x(stage, p + 1, i);
#pragma unroll
            for (int l = from + count * i / MM; l < from + count * (i + 1) / MM; ++l) request_one(freed, l);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    Place at = locate(first_tile);
    for (int tile = first_tile; tile < total; tile += workers) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < at.steps; ++k) {
            pair(0, 0, 0, 0);
            advance();                                         // (of the loads, which are two steps ahead)
            if constexpr (PAIRS == 4) {
                landed();                                      // this step's other pairs; everyone has W and the first two
                pair(1, stage, 0, C::FIRST / 2 + 1);
                pair(2, stage, C::FIRST / 2 + 1, C::FIRST - C::FIRST / 2 - 1);
            }
            landed();                                          // the next step's W and first pairs; everyone has this one's operands
            const int freed = stage;
            constexpr int FROM = PAIRS == 4 ? C::FIRST : 0;
            stage = C::STAGE - stage;
            scales = scales == 2 * C::SCALES ? 0 : scales + C::SCALES;
#pragma unroll
            for (int i = 0; i < MM; ++i) {
                multiply(PAIRS - 1, i);
                __builtin_amdgcn_sched_barrier(0);
                if (i < 6) read_x(stage, 0, i);
                if ((i & 1) && i < MM - 1)                     // (the last one behind the next step's first instruction, which does not wait for it)
#pragma unroll
                    for (int q = 0; q < 3; ++q) read_w(stage, i >> 1, q);
#pragma unroll
                for (int l = FROM + (C::LOADS - FROM) * i / MM; l < FROM + (C::LOADS - FROM) * (i + 1) / MM; ++l) request_one(freed, l);
                __builtin_amdgcn_sched_barrier(0);
            }
        }

        // ---- lane (r, g) holds rows 16 i + 4 g + q, columns 4 r + j
        const int64_t row0 = WGRAD ? (static_cast<int64_t>(at.split) * a.groups + at.group) * a.M + at.m_first : static_cast<int64_t>(at.m_first);
        if (a.wide) {                  // whole runs of 4 columns; what is past the result is dropped
            const int N = static_cast<int>(a.N), n_lane = at.n0 + wn * 64 + r * 4, o_lane = (wm * TM * 16 + g * 4) * N + n_lane;
            // (the offset is the vector register's alone: behind a 16-byte store with a scalar offset the compiler lets the next
            // instruction overwrite the data, and now and then the last lanes of its first register left with the new value)
            if (a.out) {
                const __amdgpu_buffer_rsrc_t o = __builtin_amdgcn_make_buffer_rsrc(a.out + row0 * a.N, 0, at.m_count * N * 2, 0x00020000);
                int to = n_lane < N ? o_lane * 2 : 0x40000000;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const u32x2 w{pack_bf16x2(acc[i][0][q], acc[i][1][q]), pack_bf16x2(acc[i][2][q], acc[i][3][q])};
                        __builtin_amdgcn_raw_buffer_store_b64(w, o, to, 0, 0);
                        to += q < 3 ? N * 2 : N * 26;
                        asm volatile("" : "+v"(to));           // (else all rows' offsets are kept through the steps, in registers that these need)
                    }
                }
            }
            if (a.y) {
                const __amdgpu_buffer_rsrc_t o = __builtin_amdgcn_make_buffer_rsrc(a.y + row0 * a.N, 0, at.m_count * N * 4, 0x00020000);
                int to = n_lane < N ? o_lane * 4 : 0x40000000;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v4f{acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]}), o, to, 0, 0);
                        to += q < 3 ? N * 4 : N * 52;
                        asm volatile("" : "+v"(to));
                    }
                }
            }
            late = a.out && !a.y ? (PAIRS == 4 ? 3 : 1) : 0;
        } else {
            int first = wm * TM * 16 + g * 4;
            asm volatile("" : "+v"(first));
            const int64_t n = at.n0 + wn * 64 + r * 4;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = first + i * 16 + q;
                    if (row >= at.m_count) continue;
                    const v4f f{acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]};
                    if (a.out) put4(a.out + (row0 + row) * a.N, n, a.N, f);
                    if (a.y) put4(a.y + (row0 + row) * a.N, n, a.N, f);
                }
            late = 0;
        }
        if (tile + workers < total) at = locate(tile + workers);
    }
    wait_vmcnt<0>();
}

template <class C, bool WGRAD>
__global__ __launch_bounds__(64 * C::NW, C::NW * C::PER_CU / 4) void gg_tile_kernel(const GgArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    gg_tiles<C, WGRAD>(a, smem);
}

using GgLarge = GgTile<8, 4, 2, 4>;
using GgSmall = GgTile<4, 4, 2, 2>;

// ---------------------------------------------------------------------------------
// Few rows a group: bound by the weights' traffic.  A workgroup of 8 waves owns 16 MT rows x 16 NT columns of a group; the waves take the
// steps of the contraction in turn, straight from memory into registers, U of them in flight, and add their sums in LDS in wave order.
// FUSED: X is quantized here: a lane holds 32 of a row's 128 elements, and the row's four lanes share the maximum.
// 8 rows x 64 groups x 1024 x 4096: 7.8 us (35 MB, 4.4 TB/s; most of the rest is the launch and the journeys of offsets, index, operands);
// 26 rows x 8 groups x 4096 x 16384: 89 us (549 MB, 6.2 TB/s).
constexpr int kStreamWaves = 8;

// the larger of the four lanes l % 16 + 0, 16, 32, 48, in all of them
__device__ __forceinline__ uint32_t row_lanes_max(uint32_t v) {
    u32_pair r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = r.x > r.y ? r.x : r.y;
    r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return r.x > r.y ? r.x : r.y;
}

template <int MT, int NT, bool FUSED>
__device__ __forceinline__ void gg_stream(const GgArgs& a, uint8_t* smem) {
    v4f* const part = reinterpret_cast<v4f*>(smem);        // [wave][MT * NT][64]
    constexpr int U = FUSED ? 2 : NT * MT >= 8 ? 1 : NT * MT >= 4 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int u = static_cast<int>(blockIdx.x) / a.tiles_n, nt = static_cast<int>(blockIdx.x) - u * a.tiles_n;
    const UnitAt at = find_unit(a.offsets, a.groups, a.rows, 16 * MT, u);
    if (at.group < 0) return;
    const int skip = (u - at.before) * (16 * MT), m_first = at.first + skip, m_count = at.count - skip;
    const int64_t n0 = static_cast<int64_t>(nt) * (16 * NT);

    // rows past the end: of W zeros, of X the last one; what they give is not written
    const int n_count = a.N - n0 < 16 * NT ? static_cast<int>(a.N - n0) : 16 * NT, w_row = static_cast<int>(a.w_row), sw_row = static_cast<int>(a.sw_row) * 4;
    const uint8_t* const wp = a.wq + at.group * a.w_group + n0 * a.w_row;
    const float* const swp = a.sw + at.group * a.sw_group + n0 * a.sw_row;
    const int w_lane = r * w_row + g * 32, sw_lane = r * sw_row, w_bytes = (n_count - 1) * w_row + 128, sw_bytes = (n_count - 1) * sw_row + 4;
    const uint8_t* xp[MT];
    const float* sxp[MT];
    const uint16_t* xb[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m_first + (i * 16 + r < m_count ? i * 16 + r : m_count - 1);
        int64_t s = a.index ? a.index[m] : m;
        s = s < 0 ? 0 : s >= a.x_rows ? a.x_rows - 1 : s;
        if (FUSED) {
            xb[i] = a.x + s * a.ldx;
        } else {
            xp[i] = a.xq + s * a.x_row + g * 32;
            sxp[i] = a.sx + s * a.sx_row;
        }
    }
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    // steps k0, k0 + 8, ... of the contraction, so many at a time
    auto steps = [&](int k0, auto n) __attribute__((always_inline)) {
        constexpr int S = n.value;
        v8i w[S][NT], x[S][MT];
        int sw[S][NT], sx[S][MT];
        u32x4 raw[FUSED ? S : 1][FUSED ? MT : 1][4];
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int k = k0 + q * kStreamWaves;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if constexpr (FUSED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) raw[q][i][e] = mx_load8(xb[i], static_cast<int64_t>(k) * kGroupBlock + g * 32 + e * 8, a.K);
                } else {
                    const u32x4* p = reinterpret_cast<const u32x4*>(xp[i] + k * a.x_step);
                    x[q][i] = join(p[0], p[1]);
                    sx[q][i] = scale_byte(__float_as_uint(sxp[i][k * a.sx_step]));
                }
            }
            const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(wp + k * a.w_step), 0, w_bytes, 0x00020000);
            const __amdgpu_buffer_rsrc_t swr = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(swp + k * a.sw_step), 0, sw_bytes, 0x00020000);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const u32x4 lo = __builtin_amdgcn_raw_buffer_load_b128(wr, w_lane, j * 16 * w_row, 0), hi = __builtin_amdgcn_raw_buffer_load_b128(wr, w_lane + 16, j * 16 * w_row, 0);
                w[q][j] = join(lo, hi);
                sw[q][j] = scale_byte(__builtin_amdgcn_raw_buffer_load_b32(swr, sw_lane, j * 16 * sw_row, 0));
            }
        }
#pragma unroll
        for (int q = 0; q < S; ++q) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if constexpr (FUSED) {
                    uint32_t m = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t o = max_abs8(raw[q][i][e]);
                        m = o > m ? o : m;
                    }
                    float scale;
                    const bool finite = gq_scale(row_lanes_max(m), scale);
                    sx[q][i] = scale_byte(__float_as_uint(scale));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const u32x2 c = gq_codes8(raw[q][i][e], scale, finite);
                        x[q][i][2 * e] = static_cast<int>(c.x);
                        x[q][i][2 * e + 1] = static_cast<int>(c.y);
                    }
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = gg_mfma(w[q][j], x[q][i], acc[i][j], sw[q][j], sx[q][i]);
            }
        }
    };
    int k0 = wave;
    if constexpr (U > 1)
        for (; k0 + (U - 1) * kStreamWaves < a.ksteps; k0 += U * kStreamWaves) steps(k0, std::integral_constant<int, U>{});
    for (; k0 < a.ksteps; k0 += kStreamWaves) steps(k0, std::integral_constant<int, 1>{});
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[(wave * MT * NT + i * NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // value (m, n) of tile (i, j) lies in lane (n % 16) / 4 * 16 + m % 16, component n % 4
    for (int k = threadIdx.x; k < MT * NT * 64; k += 64 * kStreamWaves) {
        const int tile = k >> 6, l = k & 63, m = (tile / NT) * 16 + (l & 15);
        if (m >= m_count) continue;
        v4f s = part[tile * 64 + l];
#pragma unroll
        for (int v = 1; v < kStreamWaves; ++v) s += part[(v * MT * NT + tile) * 64 + l];
        const int64_t n = n0 + (tile % NT) * 16 + (l >> 4) * 4, o = static_cast<int64_t>(m_first + m) * a.N + n;
        if (n + 4 <= a.N) {
            if (a.out) *reinterpret_cast<u32x2_any*>(a.out + o) = u32x2{pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w)};
            if (a.y) *reinterpret_cast<u32x4_any*>(a.y + o) = __builtin_bit_cast(u32x4, s);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < a.N) {
                    if (a.out) a.out[o + e] = static_cast<uint16_t>(f32_to_bf16_rne(s[e]));
                    if (a.y) a.y[o + e] = s[e];
                }
        }
    }
}

// (512 threads, 4 waves on a SIMD: 128 registers, so that two workgroups share a CU)
template <int MT, int NT, bool FUSED>
__global__ __launch_bounds__(64 * kStreamWaves, 4) void gg_stream_kernel(const GgArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    gg_stream<MT, NT, FUSED>(a, smem);
}

template <int MT, int NT, bool FUSED>
static loka_status stream_launch(GgArgs& a, hipStream_t stream) {
    constexpr int LDS = kStreamWaves * MT * NT * 1024;
    const int64_t some = a.rows < a.groups ? a.rows : a.groups;
    a.tiles_n = static_cast<int>((a.N + 16 * NT - 1) / (16 * NT));
    const int64_t grid = (a.rows + (16 * MT - 1) * some) / (16 * MT) * a.tiles_n;
    gg_stream_kernel<MT, NT, FUSED><<<static_cast<uint32_t>(grid), 64 * kStreamWaves, LDS, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

template <class C>
static int64_t tiles_of(const loka_grouped_desc* d) {       // that the groups can take
    const int64_t some = d->rows < d->groups ? d->rows : d->groups;
    return (d->rows + (C::BM - 1) * some) / C::BM * ((d->N + C::BN - 1) / C::BN);
}
template <class C>
static int64_t wgrad_tiles_of(const loka_grouped_desc* d) { return (d->K + C::BM - 1) / C::BM * ((d->N + C::BN - 1) / C::BN) * d->groups; }

// (tiles are counted in 32 bits)
bool grouped_gemm_fits(const loka_grouped_desc* d) { return tiles_of<GgSmall>(d) <= INT32_MAX / 2; }
bool grouped_wgrad_fits(const loka_grouped_desc* d) { return wgrad_tiles_of<GgSmall>(d) <= INT32_MAX / 2; }

template <class C, bool WGRAD>
static loka_status gg_launch(GgArgs& a, int64_t tiles, hipStream_t stream) {
    a.tiles_n = static_cast<int>((a.N + C::BN - 1) / C::BN);
    a.tiles_m = WGRAD ? (a.M + C::BM - 1) / C::BM : 0;
    a.wide = a.N % 4 == 0;
    a.tiles = static_cast<int>(tiles);
    const int lds = C::LDS + 12 * a.groups;
    const int64_t slots = 256 * C::PER_CU;
    // (on every call, a host-side table write, and correct on whichever device is current; the same value whatever the call's groups, as another
    // thread may set it between this and the launch)
    LOKA_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&gg_tile_kernel<C, WGRAD>), hipFuncAttributeMaxDynamicSharedMemorySize, C::MOST_LDS));
    gg_tile_kernel<C, WGRAD><<<static_cast<uint32_t>(tiles < slots ? tiles : slots), 64 * C::NW, lds, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

static GgArgs gemm_args(const loka_grouped_desc* d, const int32_t* index, const int32_t* offsets, const uint8_t* wq, const float* sw, void* out, float* y) {
    GgArgs a{};
    const int64_t kb = group_blocks(d->K), N = d->N;
    a.wq = wq;
    a.sw = sw;
    a.index = index;
    a.offsets = offsets;
    a.out = static_cast<uint16_t*>(out);
    a.y = y;
    a.N = N;
    a.K = d->K;
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
    return a;
}

// What runs a product: the form whose microseconds, fitted to launches, are fewest.  How the rows spread over the groups is not known here: units are
// counted as if every group left half a one empty.  Estimated / measured (rows x groups x K x N; MT x NT: columns of 16 rows and columns each):
//   large tiles  3000 x 4 x 512 x 1024 15.5 / 14.4, 3000 x 4 x 4096 x 1024 51 / 50, 12000 x 4 x 4096 x 1024 51 / 53, 10026 x 23 x 1008 x 720 20.5 / 21.7
//   small tiles  3000 x 4 x 512 x 1024 7.4 / 8.0, 12000 x 4 x 4096 x 1024 73 / 74, 256 x 16 x 1024 x 4096 15.0 / 15.1, 128 x 8 x 4096 x 4096 25.8 / 26.7
//   1 x 1, 1 x 2 and 1 x 4   8 x 64 x 1024 x 4096 12.3 / 12.4, 9.2 / 9.3 and 7.6 / 7.8;  8 x 64 x 4096 x 1024 10.5 / 9.3, 8.3 / 8.1 and 12.1 / 12.2
//   2 x 4        256 x 16 x 1024 x 4096 16.1 / 17.2, 128 x 8 x 4096 x 4096 26.4 / 26.2 (1 x 4: 31.9 / 32.7)
// One choice for both entries: the linear's results are the bits of the quantization and the product of stored operands, which another form's order of sums would change.
struct GgForm { bool tiles; int mt, nt; };                  // tiles: mt = 2 the large ones, 1 the small ones; else 16 mt rows x 16 nt columns a workgroup
static double large_us(double tiles, double steps) { return 7.5 + std::ceil(tiles / 256) * (3.0 + 1.25 * steps); }
static double small_us(double tiles, double steps) {
    return tiles <= 256 ? 5.0 + (0.45 + 0.2 * tiles / 256) * steps : 5.5 + std::ceil(tiles / 512) * (1.5 + steps);
}
static GgForm gemm_form(const loka_grouped_desc* d) {
    const double rows = static_cast<double>(d->rows), some = static_cast<double>(d->rows < d->groups ? d->rows : d->groups), N = static_cast<double>(d->N);
    const double steps = std::ceil(static_cast<double>(d->K) / kGroupBlock), floor = some * N * steps * kGroupBlock / 6.5e6;      // (of the weights' bytes)
    auto units = [&](double b) { return std::fmax(some, rows / b + some / 2); };
    GgForm best{true, 1, 0};
    double least = 1e30;
    auto offer = [&](double us, GgForm f) {
        if (us >= least) return;
        least = us;
        best = f;
    };
    auto stream = [&](int mt, int nt) {
        const double rounds = std::ceil(units(16 * mt) * std::ceil(N / (16 * nt)) / 256);
        return std::fmax(floor, 2.2 + rounds * (0.06 * (mt + nt) * steps + 0.3 * mt));
    };
    // (2 us: the others' quantization is a launch before them where the rows come as bf16; stored operands have none and are given the same form)
    if ((rows / 16 + some) * std::ceil(N / 16) < 4194304.0) {                               // (workgroups of 512 threads in one launch)
        for (int nt = 4; nt >= 1; nt /= 2) offer(stream(1, nt), GgForm{false, 1, nt});
        offer(stream(2, 4) + 2.0, GgForm{false, 2, 4});
    }
    offer(std::fmax(floor, small_us(units(128) * std::ceil(N / 128), steps)) + 2.0, GgForm{true, 1, 0});
    offer(std::fmax(floor, large_us(units(256) * std::ceil(N / 256), steps)) + 2.0, GgForm{true, 2, 0});
    return best;
}
template <bool FUSED>
static loka_status stream16(int nt, GgArgs& a, hipStream_t stream) {
    return nt == 4 ? stream_launch<1, 4, FUSED>(a, stream) : nt == 2 ? stream_launch<1, 2, FUSED>(a, stream) : stream_launch<1, 1, FUSED>(a, stream);
}

loka_status grouped_gemm_launch(const loka_grouped_desc* d, const uint8_t* xq, const float* sx, const int32_t* index, const int32_t* offsets,
                                const uint8_t* wq, const float* sw, void* out, float* y, hipStream_t stream) {
    GgArgs a = gemm_args(d, index, offsets, wq, sw, out, y);
    a.xq = xq;
    a.sx = sx;
    const GgForm f = gemm_form(d);
    if (!f.tiles) return f.mt == 1 ? stream16<false>(f.nt, a, stream) : stream_launch<2, 4, false>(a, stream);
    return f.mt == 2 ? gg_launch<GgLarge, false>(a, tiles_of<GgLarge>(d), stream) : gg_launch<GgSmall, false>(a, tiles_of<GgSmall>(d), stream);
}

bool grouped_linear_fused(const loka_grouped_desc* d) {
    const GgForm f = gemm_form(d);
    return !f.tiles && f.mt == 1;
}

loka_status grouped_linear_fused_launch(const loka_grouped_desc* d, const void* x, int64_t ld, const int32_t* index, const int32_t* offsets,
                                        const uint8_t* wq, const float* sw, void* out, float* y, hipStream_t stream) {
    GgArgs a = gemm_args(d, index, offsets, wq, sw, out, y);
    a.x = static_cast<const uint16_t*>(x);
    a.ldx = ld;
    return stream16<true>(gemm_form(d).nt, a, stream);
}

// Sums of the ranges' partial results, in order.
__global__ __launch_bounds__(256) void gg_join_kernel(const float* __restrict__ part, int splits, int64_t n, int64_t first_wg, uint16_t* __restrict__ out,
                                                      float* __restrict__ y) {
    const int64_t i = (first_wg + blockIdx.x) * 256 + threadIdx.x;
    if (i >= n) return;
    float s = part[i];
#pragma unroll 8
    for (int k = 1; k < splits; ++k) s += part[k * n + i];
    if (out) out[i] = static_cast<uint16_t>(f32_to_bf16_rne(s));
    if (y) y[i] = s;
}

// Tile and ranges of a weight gradient.  Where the results are few tiles, a group's blocks are split over workgroups, as far as that saves more than the
// partial sums cost (rows x groups x K x N: 16384 x 1 x 256 x 256 in 32 ranges 14.5 us, in one 80; 16384 x 2 x
// 64 x 100 12.3 and 41).
struct WgradPlan { bool large; int splits; };
static WgradPlan wgrad_plan(const loka_grouped_desc* d) {
    const double steps = std::ceil(static_cast<double>(d->rows) / static_cast<double>(d->groups) / kGroupBlock + 0.5);
    const double small = static_cast<double>(wgrad_tiles_of<GgSmall>(d)), bytes = static_cast<double>(d->groups) * static_cast<double>(d->K) * static_cast<double>(d->N) * 4;
    WgradPlan p{large_us(static_cast<double>(wgrad_tiles_of<GgLarge>(d)), steps) < small_us(small, steps), 1};
    if (p.large) return p;
    double best = 1e30;
    for (int s = 1; s <= 32 && (s == 1 || small * s <= 512); s *= 2) {
        const double us = (small * s <= 256 ? 0.55 : 1.0) * std::ceil(steps / s) + (s > 1 ? 4.0 + bytes * s / 2e6 : 0.0);
        if (us < best) {
            best = us;
            p.splits = s;
        }
    }
    return p;
}

size_t grouped_wgrad_workspace_bytes(const loka_grouped_desc* d) {
    const int splits = wgrad_plan(d).splits;
    return splits > 1 ? static_cast<size_t>(splits) * static_cast<size_t>(d->groups) * static_cast<size_t>(d->K) * static_cast<size_t>(d->N) * 4 : 0;
}

loka_status grouped_wgrad_launch(const loka_grouped_desc* d, const uint8_t* xt, const float* sxt, const uint8_t* dyt, const float* sdyt,
                                 const int32_t* offsets, void* dw, float* dw32, void* ws, hipStream_t stream) {
    GgArgs a{};
    a.xq = xt;
    a.sx = sxt;
    a.wq = dyt;
    a.sw = sdyt;
    a.offsets = offsets;
    a.out = static_cast<uint16_t*>(dw);
    a.y = dw32;
    a.N = d->N;
    a.M = a.x_rows = static_cast<int>(d->K);
    a.blocks = static_cast<int>(loka_grouped_blocks(d->rows, d->groups));
    a.rows = static_cast<int>(d->rows);
    a.groups = d->groups;
    a.x_row = a.w_row = kGroupBlock;
    a.x_step = d->K * kGroupBlock;
    a.w_step = d->N * kGroupBlock;
    a.sx_row = a.sw_row = 1;
    a.sx_step = d->K;
    a.sw_step = d->N;
    const WgradPlan p = wgrad_plan(d);
    a.splits = p.splits;
    if (p.large) return gg_launch<GgLarge, true>(a, wgrad_tiles_of<GgLarge>(d), stream);
    if (p.splits == 1) return gg_launch<GgSmall, true>(a, wgrad_tiles_of<GgSmall>(d), stream);
    a.out = nullptr;
    a.y = static_cast<float*>(ws);
    const loka_status st = gg_launch<GgSmall, true>(a, wgrad_tiles_of<GgSmall>(d) * p.splits, stream);
    if (st != LOKA_OK) return st;
    const int64_t n = d->groups * d->K * d->N;
    return in_launches((n + 255) / 256, 256, [&](int64_t from, uint32_t grid) {
        gg_join_kernel<<<grid, 256, 0, stream>>>(static_cast<const float*>(ws), p.splits, n, from, static_cast<uint16_t*>(dw), dw32);
    });
}

}  // namespace loka
