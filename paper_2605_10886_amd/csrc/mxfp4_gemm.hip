// Products of MXFP4 operands (include/loka.h, loka_mxfp4_gemm / loka_mxfp4_linear) on the scaled matrix instructions.
//
// With 4-bit operands a lane of v_mfma_scale_f32_16x16x128_f8f6f4 holds row l % 16 and codes 32 (l / 16) .. + 31, and of the
// 32x32x64 form row l % 32 and codes 32 (l / 32) .. + 31, in 16 bytes, with one scale byte: a lane's operand IS one stored group and its
// scale.  The weights are the first operand, so that a lane holds neighbouring columns n of one row m of the result.
//
// Which 32-groups of a row meet in one instruction is free as long as both operands agree: the four instructions of 512 (256)
// consecutive elements take groups 4 g + s (g: lane / 16 or lane / 32, s: instruction), so a lane's four scale bytes are one word,
// from which the instruction picks by its byte selector.
//
// Two kernels: few rows stream the weights from memory into registers (16 x 16 x 128), many rows work on tiles in LDS (32 x 32 x 64).
#include "gemm_common.h"
#include "mxfp4.h"

#include <cmath>
#include <type_traits>

namespace loka {

typedef float v16f __attribute__((ext_vector_type(16)));

struct MxArgs {
    const uint8_t *xq, *sx, *wq, *sw;
    const uint16_t* x;                 // fused quantization: bf16 [M, ldx]
    uint16_t* out;
    float* y;
    int64_t M, N, K, Kp;               // Kp: stored row length in elements
    int64_t ldx;
    int64_t strideX, strideW, strideO; // elements between problems
    int64_t n_tiles, m_tiles, first_wg; // stream kernel
    bool x_whole;                      // rows of x start on multiples of 16 bytes, and are a whole number of 16-byte runs
    // tile kernel: result tiles of a problem, K ranges and their length in K tiles, all tiles
    int64_t batch;
    int tiles_m, tiles_n, splits, k_per_split, total;
    float* part;                       // [splits][batch][M][N]
    bool wide;                         // rows of whole 16-byte runs, a tile's within 32-bit offsets
    bool streamed;                     // bf16 values past the caches
};

template <int S>
__device__ __forceinline__ v4f mx_mfma(const u32x4 a, const u32x4 b, v4f c, uint32_t sa, uint32_t sb) {
    const v8i A = {static_cast<int>(a.x), static_cast<int>(a.y), static_cast<int>(a.z), static_cast<int>(a.w), 0, 0, 0, 0};
    const v8i B = {static_cast<int>(b.x), static_cast<int>(b.y), static_cast<int>(b.z), static_cast<int>(b.w), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, S, static_cast<int>(sa), S, static_cast<int>(sb));
}

template <int S>
__device__ __forceinline__ v16f mx_mfma32(const u32x4 a, const u32x4 b, v16f c, uint32_t sa, uint32_t sb) {
    const v8i A = {static_cast<int>(a.x), static_cast<int>(a.y), static_cast<int>(a.z), static_cast<int>(a.w), 0, 0, 0, 0};
    const v8i B = {static_cast<int>(b.x), static_cast<int>(b.y), static_cast<int>(b.z), static_cast<int>(b.w), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 4, S, static_cast<int>(sa), S, static_cast<int>(sb));
}

// A lane's four groups of 512 elements: codes and the word of their scale bytes.  Groups past the stored row are zero codes
// with scale 1 (the stored row is a whole number of four groups, so a lane has all of its four or none).
struct MxPiece {
    u32x4 c[4];
    uint32_t s;
};
__device__ __forceinline__ MxPiece mx_read_piece(const uint8_t* q, const uint8_t* scales, int64_t row, int64_t Kp, int64_t group) {
    MxPiece p;
    const bool in = group < (Kp >> 5);
    const int64_t g = in ? group : 0;
    const u32x4* src = reinterpret_cast<const u32x4*>(q + row * (Kp >> 1) + g * 16);
    const uint32_t s = *reinterpret_cast<const uint32_t*>(scales + row * (Kp >> 5) + g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32x4 v = src[i];
        p.c[i] = in ? v : u32x4{0u, 0u, 0u, 0u};
    }
    p.s = in ? s : 0x7F7F7F7Fu;
    return p;
}
// The same from bf16 rows, two ways.  One or two rows: the wave quantizes 512 elements of a row at a time, 8 a lane as
// they lie in memory, and turns the codes in its part of LDS (a lane that read its own row's groups would make every
// 16-byte load a cache line of its own).
constexpr int kTurn = 256 + 16;        // bytes of a row there: codes, scales
__device__ __forceinline__ MxPiece mx_quantize_rows(const uint16_t* x, int64_t ldx, int rows, int64_t first, int64_t K, bool whole, uint8_t* turn,
                                                    int lane) {
    constexpr int ROWS = 2;
    u32x4 v[ROWS];
    const int64_t c = first + lane * 8;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (i >= rows) continue;
        if (whole) {                   // no run of 8 is cut by the row's end
            const u32x4 w = *reinterpret_cast<const u32x4*>(x + i * ldx + (c < K ? c : 0));
            v[i] = c < K ? w : u32x4{0u, 0u, 0u, 0u};
        } else v[i] = mx_load8(x + i * ldx, c, K);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (i >= rows) continue;
        uint32_t a = max_abs_bf16x2(v[i].x & 0x7FFF7FFFu, v[i].y);
        a = max_abs_bf16x2(max_abs_bf16x2(a, v[i].z), v[i].w);
        const uint32_t byte = mx_scale_byte(quad_max(max_of_halves(a)) << 16);
        const uint32_t codes = mx_codes_bf16x8(v[i], mx_scale_value(byte)), four = quad_bytes(byte);
        *reinterpret_cast<uint32_t*>(turn + i * kTurn + lane * 4) = byte == kMxNaN ? 0u : codes;
        if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(turn + i * kTurn + 256 + (lane >> 4) * 4) = four;
    }
    const int r = lane & 15, g = lane >> 4;
    MxPiece p;                         // (rows that are not there: whatever lies there, for results that are not written)
#pragma unroll
    for (int i = 0; i < 4; ++i) p.c[i] = *reinterpret_cast<const u32x4*>(turn + r * kTurn + g * 64 + i * 16);
    p.s = *reinterpret_cast<const uint32_t*>(turn + r * kTurn + 256 + g * 4);
    return p;
}
// Up to 16 rows: loads bring 512 elements of each row into LDS (16-byte run c of row i at place c ^ i: the 16 rows of a read
// use all banks), and each lane quantizes its four groups from there: a third of the instructions of the other way's lanes, which
// share a group by four.
constexpr int kRaw = 16 * 1024;
__device__ __forceinline__ void mx_request_rows(const uint16_t* x, int64_t ldx, int rows, int64_t first, int64_t K, uint8_t* raw, int lane) {
    for (int i = 0; i < rows; ++i) {
        const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(x + i * ldx), 0, static_cast<int>(K) * 2, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (__attribute__((address_space(3))) void*)(raw + i * 1024), 16, static_cast<int>(first) * 2 + (lane ^ i) * 16, 0, 0, 0);
    }
}
// ... rows that start or end anywhere through registers (rows x columns x K: 16 x 14000 x 3001 9.5 us; quantized by rows, 4 lanes a group, 24.4)
__device__ __forceinline__ void mx_load_rows(const uint16_t* x, int64_t ldx, int rows, int64_t first, int64_t K, int lane, u32x4 (&v)[16]) {
    const int64_t c = first + lane * 8;
    if (K >= 8) {
        const int64_t at = c + 8 <= K ? c : K - 8;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = *reinterpret_cast<const u32x4_any*>(x + (i < rows ? i : 0) * ldx + at);
    } else {
        for (int i = 0; i < 16; ++i) v[i] = mx_load8(x + (i < rows ? i : 0) * ldx, c, K);
    }
}
__device__ __forceinline__ void mx_put_rows(u32x4 (&v)[16], int64_t first, int64_t K, uint8_t* raw, int lane) {
    const int64_t c = first + lane * 8;
    if (K >= 8 && first + 512 > K) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = mx_from(v[i], c + 8 <= K ? 0 : c + 8 - K);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) *reinterpret_cast<u32x4*>(raw + i * 1024 + (lane ^ i) * 16) = v[i];
}
__device__ __forceinline__ MxPiece mx_quantize_groups(const uint8_t* raw, int lane) {
    const int r = lane & 15, g = lane >> 4;
    MxPiece p;
    p.s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const u32x4*>(raw + r * 1024 + ((g * 16 + i * 4 + j) ^ r) * 16);
        uint32_t a = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) a = max_abs_bf16x2(a, v[j][e]);
        const uint32_t byte = mx_scale_byte(max_of_halves(a) << 16);
        const float s = mx_scale_value(byte);
#pragma unroll
        for (int j = 0; j < 4; ++j) p.c[i][j] = byte == kMxNaN ? 0u : mx_codes_bf16x8(v[j], s);
        p.s |= byte << (8 * i);
    }
    return p;
}

// No access to memory is moved across
__device__ __forceinline__ void in_order() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// ---------------------------------------------------------------------------------
// Few rows: bound by the weights' traffic (rows x columns x K here and below: 16 x 16384 x 4096 9.5 us with the quantization of x, 3.8 TB/s of
// codes; 16 x 28672 x 8192 35 us).  A workgroup of NW waves owns 16 NT columns x 16 MT rows of the result; the waves
// take 512-element pieces of the contraction in turn, straight from memory into registers, and add their partial sums in LDS
// in wave order.
// QUANT 0: stored X.  1, 2, 3: bf16 X of up to 16 rows (MT = 1): by groups; by rows (up to 2); by groups, rows that start or end anywhere.
template <int MT, int NT, int NW, int QUANT>
__global__ __launch_bounds__(64 * NW) void mx_stream_kernel(const MxArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];       // partial sums [NW][MT * NT][64]; before them, the waves' rows of x
    v4f* const part = reinterpret_cast<v4f*>(smem);
    uint8_t* const own = smem + (threadIdx.x >> 6) * (QUANT == 2 ? 16 * kTurn : kRaw);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    int64_t id = a.first_wg + blockIdx.x;
    const int64_t nt = id % a.n_tiles;
    id /= a.n_tiles;
    const int64_t mt = id % a.m_tiles, prob = id / a.m_tiles;
    const uint8_t* xq = a.xq + prob * (a.strideX >> 1);
    const uint8_t* sx = a.sx + prob * (a.strideX >> 5);
    const uint8_t* wq = a.wq + prob * (a.strideW >> 1);
    const uint8_t* sw = a.sw + prob * (a.strideW >> 5);
    const int64_t n0 = nt * (16 * NT), m0 = mt * (16 * MT);
    int64_t wrow[NT], xrow[MT];        // rows past the end read the last one; what they give is not written
#pragma unroll
    for (int j = 0; j < NT; ++j) wrow[j] = n0 + j * 16 + r < a.N ? n0 + j * 16 + r : a.N - 1;
#pragma unroll
    for (int i = 0; i < MT; ++i) xrow[i] = m0 + i * 16 + r < a.M ? m0 + i * 16 + r : a.M - 1;
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    const int64_t pieces = (a.Kp + 511) >> 9;
    for (int64_t p = wave; p < pieces; p += NW) {
        const int64_t group = p * 16 + g * 4;
        MxPiece w[NT], x[MT];
        if (QUANT == 1) {
            mx_request_rows(a.x, a.ldx, static_cast<int>(a.M), p << 9, a.K, own, lane);
            in_order();
        }
        u32x4 v[QUANT == 3 ? 16 : 1];
        if constexpr (QUANT == 3) {
            mx_load_rows(a.x, a.ldx, static_cast<int>(a.M), p << 9, a.K, lane, v);
            in_order();
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) w[j] = mx_read_piece(wq, sw, wrow[j], a.Kp, group);
        if constexpr (QUANT == 0) {
#pragma unroll
            for (int i = 0; i < MT; ++i) x[i] = mx_read_piece(xq, sx, xrow[i], a.Kp, group);
        } else if constexpr (QUANT == 1) {
            in_order();
            wait_vmcnt<5 * NT>();      // the rows, which were requested before the weights' five loads a tile
            in_order();
            x[0] = mx_quantize_groups(own, lane);
        } else if constexpr (QUANT == 3) {
            mx_put_rows(v, p << 9, a.K, own, lane);
            x[0] = mx_quantize_groups(own, lane);
        } else {
            x[0] = mx_quantize_rows(a.x, a.ldx, static_cast<int>(a.M), p << 9, a.K, a.x_whole, own, lane);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[i][j] = mx_mfma<0>(w[j].c[0], x[i].c[0], acc[i][j], w[j].s, x[i].s);
                acc[i][j] = mx_mfma<1>(w[j].c[1], x[i].c[1], acc[i][j], w[j].s, x[i].s);
                acc[i][j] = mx_mfma<2>(w[j].c[2], x[i].c[2], acc[i][j], w[j].s, x[i].s);
                acc[i][j] = mx_mfma<3>(w[j].c[3], x[i].c[3], acc[i][j], w[j].s, x[i].s);
            }
    }
    if (QUANT) __syncthreads();        // (the partial sums take the place of other waves' rows)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[(wave * MT * NT + i * NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // value (m, n) of tile (i, j) lies in lane (n % 16) / 4 * 16 + m % 16, component n % 4
    constexpr int total = MT * NT * 64;
    for (int k = threadIdx.x; k < total; k += 64 * NW) {
        const int tile = k >> 6, l = k & 63;
        v4f s = part[tile * 64 + l];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += part[(w * MT * NT + tile) * 64 + l];
        const int64_t m = m0 + (tile / NT) * 16 + (l & 15), n = n0 + (tile % NT) * 16 + (l >> 4) * 4;
        if (m >= a.M) continue;
        const int64_t o = prob * a.strideO + m * a.N + n;
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

// ---------------------------------------------------------------------------------
// Many rows: a workgroup of WM x WN x WK waves computes a tile of the result, each wave TM x TN tiles of 32 x 32, on K tiles of
// 256 elements (128 bytes of codes a row) that loads bring straight into LDS, R of them in a ring.  The 16-byte chunks of a
// row lie permuted, chunk c at place c ^ (row / 2 % 8), so that the rows that an LDS read serves at once use all 64 banks.
//
// v_mfma_scale_f32_32x32x64_f8f6f4: lane l holds row r = l % 32, one group of 32 elements (of the two: h = l / 32) and its scale
// byte.  The four instructions of a K tile (quarters s) take groups 4 h + s, so a lane's four scale bytes are one word.
// From registers, on changing operands, this form sustains 6.0 - 6.3 PFLOP/s on 4-bit codes and the 16 x 16 x 128 form 6.4 - 6.8; here
// half as many instructions, and longer runs to store, win: 32768 x 4096 x 4096 358 -> 344 us, 8192 x 8192 x 8192 the same.
// WK = 1: a wave multiplies all quarters; WK = 2: two of them, and two waves add up at the end (two waves on a SIMD where the
// tile gives only four).
// W's rows are dealt to the instruction's so that a lane's values are two runs of 8 columns.
//
// One barrier a K tile: its last operands are in registers when the barrier is passed, so the loads of a K tile R further on
// may go where this one lay, and the first operands of the next K tile are read between the matrix instructions that follow.
// (The barrier costs some 800 cycles of a K tile's 3800: K tiles of 128 elements, with four in the ring, took 8192 x 8192 x
// 8192 from 300 to 388 us.)  Workgroups are persistent, and the ring does not stop between result tiles: the next tile's first
// K tiles arrive while this one's values are stored, and nothing waits for the stores where their number is known (see `late`).
template <int TM_, int TN_, int WM_, int WN_, int WK_, int R_, bool WORDS_ = false>
struct MxTile {
    static constexpr bool WORDS = WORDS_;                           // bf16 rows that start inside a word leave in whole words (below)
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, WK = WK_, R = R_, NW = WM * WN * WK, BM = WM * TM * 32, BN = WN * TN * 32;
    static constexpr int OFF_W = BM * 128, OFF_SX = OFF_W + BN * 128, OFF_SW = OFF_SX + BM * 8, STAGE = OFF_SW + BN * 8;
    static constexpr int XCH = WM * WN * 64 * 64;                   // WK = 2: one 32 x 32 tile of every wave
    static constexpr int LDS = R * STAGE + (WK == 2 ? 2 * XCH : 0), PER_CU = 163840 / LDS;
    static_assert(NW % 2 == 0 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && (BM + BN) % (32 * NW) == 0);
    static_assert(WK == 1 || (WK == 2 && TM == 2));
};

template <class C, bool SPLIT>
__device__ __forceinline__ void mx_tiles(const MxArgs& a, uint8_t* smem) {
    constexpr int TM = C::TM, TN = C::TN, Q = 4 / C::WK;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
    const int kg = C::WK == 2 ? wave / (C::WM * C::WN) : 0, wmn = C::WK == 2 ? wave % (C::WM * C::WN) : wave;
    const int wm = wmn / C::WN, wn = wmn % C::WN;
    const int row_bytes = static_cast<int>(a.Kp >> 1), scale_bytes = static_cast<int>(a.Kp >> 5);
    const int ktiles_all = static_cast<int>((a.Kp + 255) >> 8);
    const bool ragged = (a.Kp & 255) != 0;
    const int total = a.total;

    // column, of the 32, that row r of the instruction's result stands for
    const int n_of = (r >> 4) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);
    // where this wave's loads find things (8 rows a load, every NW-th group of them: of one parity)
    const int chunk = (lane & 7) ^ (((wave & 1) << 2) | (lane >> 4)), c_lane = (lane >> 3) * row_bytes + chunk * 16;
    // (scales of 32 rows a load: the four bytes of h = 0 of each, then those of h = 1, W's in the order of the instruction's rows)
    const int sx_lane = r * scale_bytes + h * 4, sw_lane = n_of * scale_bytes + h * 4;
    // where it reads operands
    const int x_row = wm * TM * 32 + r, w_row = wn * TN * 32 + n_of;
    int x_off[Q], w_off[Q];
#pragma unroll
    for (int s = 0; s < Q; ++s) {
        x_off[s] = x_row * 128 + ((4 * h + kg * 2 + s) ^ ((r >> 1) & 7)) * 16;
        w_off[s] = C::OFF_W + w_row * 128 + ((4 * h + kg * 2 + s) ^ ((n_of >> 1) & 7)) * 16;
    }
    const int sx_off = C::OFF_SX + wm * TM * 256 + h * 128 + r * 4 + kg * 2, sw_off = C::OFF_SW + wn * TN * 256 + h * 128 + r * 4 + kg * 2;

    struct Place { int m0, n0, k_first, k_count, split; int64_t prob; };
    auto locate = [&](int t) __attribute__((always_inline)) {
        Place p;
        const int per = a.tiles_m * a.tiles_n;
        const int o = t / per;
        int tm, tn;
        banded_tile(t - o * per, a.tiles_m, a.tiles_n, tm, tn);
        p.prob = SPLIT ? o / a.splits : o;
        p.split = SPLIT ? o - static_cast<int>(p.prob) * a.splits : 0;
        p.k_first = p.split * a.k_per_split;
        p.k_count = !SPLIT || p.k_first + a.k_per_split > ktiles_all ? ktiles_all - p.k_first : a.k_per_split;
        p.m0 = tm * C::BM;
        p.n0 = tn * C::BN;
        return p;
    };

    // ---- the stream of K tiles: `ld` is the next one to request
    int ld_tile = xcd_contiguous(blockIdx.x, gridDim.x), ld_k = 0;      // (every XCD starts on consecutive tiles, which share operands)
    if (ld_tile >= total) return;
    Place ld = locate(ld_tile);
    __amdgpu_buffer_rsrc_t xr, wr, sxr, swr;
    auto aim = [&]() __attribute__((always_inline)) {
        const int64_t rows_x = a.M - ld.m0 < C::BM ? a.M - ld.m0 : C::BM, rows_w = a.N - ld.n0 < C::BN ? a.N - ld.n0 : C::BN;
        const bool on = ld_tile < total;                   // (past the end: zeros, so that every K tile requests as many loads)
        auto make = [&](const uint8_t* base, int64_t bytes) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, on ? static_cast<int>(bytes) : 0, 0x00020000);
        };
        xr = make(a.xq + ld.prob * (a.strideX >> 1) + static_cast<int64_t>(ld.m0) * row_bytes, rows_x * row_bytes);
        wr = make(a.wq + ld.prob * (a.strideW >> 1) + static_cast<int64_t>(ld.n0) * row_bytes, rows_w * row_bytes);
        sxr = make(a.sx + ld.prob * (a.strideX >> 5) + static_cast<int64_t>(ld.m0) * scale_bytes, rows_x * scale_bytes);
        swr = make(a.sw + ld.prob * (a.strideW >> 5) + static_cast<int64_t>(ld.n0) * scale_bytes, rows_w * scale_bytes);
    };
    aim();
    // load i of a wave's share of a K tile: X codes, W codes, scales of X, then of W
    constexpr int LX = C::BM / (8 * C::NW), LW = C::BN / (8 * C::NW), SROWS = (C::BM + C::BN) / 32, LS = SROWS / C::NW, LOADS = LX + LW + LS;
    int ld_c, ld_sx, ld_sw, ld_off, ld_soff;
    auto begin_request = [&]() __attribute__((always_inline)) {
        const int kt = ld.k_first + ld_k;
        const bool tail = ragged && kt == ktiles_all - 1;           // the last K tile is half one: the other half reads zeros
        ld_c = tail && chunk >= 4 ? 0x7FFFFFFF : c_lane;
        ld_sx = tail && h ? 0x7FFFFFFF : sx_lane;
        ld_sw = tail && h ? 0x7FFFFFFF : sw_lane;
        ld_off = wave * 8 * row_bytes + kt * 128;
        ld_soff = kt * 8;
    };
    auto request_one = [&](int stage, int i) __attribute__((always_inline)) {
        if (i < LX) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (__attribute__((address_space(3))) void*)(smem + stage + (i * C::NW + wave) * 1024), 16, ld_c,
                                                     ld_off + i * C::NW * 8 * row_bytes, 0, 0);
        } else if (i < LX + LW) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (__attribute__((address_space(3))) void*)(smem + stage + C::OFF_W + ((i - LX) * C::NW + wave) * 1024), 16, ld_c,
                                                     ld_off + (i - LX) * C::NW * 8 * row_bytes, 0, 0);
        } else {                                           // 32 rows a load: those of X first, then those of W
            const int grp = (i - LX - LW) * C::NW + wave;
            if (grp < C::BM / 32)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(sxr, (__attribute__((address_space(3))) void*)(smem + stage + C::OFF_SX + grp * 256), 4, ld_sx,
                                                         ld_soff + grp * 32 * scale_bytes, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(swr, (__attribute__((address_space(3))) void*)(smem + stage + C::OFF_SX + grp * 256), 4, ld_sw,
                                                         ld_soff + (grp - C::BM / 32) * 32 * scale_bytes, 0, 0);
        }
    };
    auto advance = [&]() __attribute__((always_inline)) {
        if (++ld_k == ld.k_count) {
            ld_k = 0;
            ld_tile += gridDim.x;
            ld = locate(ld_tile < total ? ld_tile : 0);
            aim();
        }
    };

    // ---- operands: two sets, used in turn
    constexpr int READS = TM + TN, MM = TM * TN;
    u32x4 fx[2][TM], fw[2][TN];
    uint32_t sx[TM], sw[TN], sx_next[TM], sw_next[TN];
    // operand i of the wave's quarter q, in the order in which they are used: one X tile, the W tiles, the other X tiles
    auto read_one = [&](int stage, int q, int i) __attribute__((always_inline)) {
        const int set = q & 1, k = i == 0 ? 0 : i <= TN ? i - 1 : i - TN;
        if (i >= 1 && i <= TN) fw[set][k] = *reinterpret_cast<const u32x4*>(smem + stage + w_off[q] + k * 4096);
        else fx[set][k] = *reinterpret_cast<const u32x4*>(smem + stage + x_off[q] + k * 4096);
    };
    auto read_scales = [&](int stage) __attribute__((always_inline)) {
        auto one = [&](const uint8_t* p) __attribute__((always_inline)) {
            return C::WK == 2 ? static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p)) : *reinterpret_cast<const uint32_t*>(p);
        };
#pragma unroll
        for (int j = 0; j < TN; ++j) sw_next[j] = one(smem + stage + sw_off + j * 256);
#pragma unroll
        for (int i = 0; i < TM; ++i) sx_next[i] = one(smem + stage + sx_off + i * 256);
    };
    v16f acc[TM][TN];
    // matrix instructions first .. last - 1 of quarter q
    auto multiply = [&](auto q_c, int first, int last) __attribute__((always_inline)) {
        constexpr int q = decltype(q_c)::value;
#pragma unroll
        for (int k = 0; k < MM; ++k) {
            if (k < first || k >= last) continue;
            const int i = k / TN, j = k % TN;
            acc[i][j] = mx_mfma32<q>(fw[q & 1][j], fx[q & 1][i], acc[i][j], sw[j], sx[i]);
        }
    };

    int tile = ld_tile, stage = 0;
    Place at = ld;
    for (int k = 0; k < C::R; ++k) {
        begin_request();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) request_one(k * C::STAGE, i);
        advance();
    }
    wait_vmcnt<(C::R - 1) * LOADS>();
    lds_barrier();
#pragma unroll
    for (int i = 0; i < READS; ++i) read_one(0, 0, i);
    read_scales(0);
    // Where a tile's values left in STORES stores, the loads of the K tiles that were requested before them are awaited with the
    // stores in flight: `late` K tiles from there.
    constexpr int STORES = TM * TN * 2 / C::WK, NEWER = (C::R - 2) * LOADS;
    static_assert(NEWER + STORES <= 63);
    int late = 0;

    // A quarter's matrix instructions, and between them (a burst would hold the issue stage up) the LDS reads of the next
    // operands, early enough to be there when they are wanted, ...
    auto quarter = [&](auto q_c) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MM; ++i) {
            if (i < READS) read_one(stage, decltype(q_c)::value + 1, i);
            if (i == MM - 1)
#pragma unroll
                for (int k = MM; k < READS; ++k) read_one(stage, decltype(q_c)::value + 1, k);
            __builtin_amdgcn_sched_barrier(0);
            multiply(q_c, i, i + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // ... and, where a K tile ends, the loads into the place that it leaves.
    auto finish = [&]() __attribute__((always_inline)) {
        const std::integral_constant<int, Q - 1> last;
        if (late > 0) { --late; wait_vmcnt<NEWER + STORES>(); }
        else wait_vmcnt<NEWER>();                               // the next K tile has landed
        lds_barrier();                                          // ... for everyone, and everyone has this one's operands
        const int freed = stage;
        stage = stage + C::STAGE == C::R * C::STAGE ? 0 : stage + C::STAGE;
        begin_request();
#pragma unroll
        for (int i = 0; i < MM; ++i) {
            multiply(last, i, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            if (i < READS) read_one(stage, 0, i);
            if (i == MM - 1)
#pragma unroll
                for (int k = MM; k < READS; ++k) read_one(stage, 0, k);
#pragma unroll
            for (int l = LOADS * i / MM; l < LOADS * (i + 1) / MM; ++l) request_one(freed, l);
            if (i == (READS < MM ? READS : MM - 1)) read_scales(stage);
            __builtin_amdgcn_sched_barrier(0);
        }
        advance();
    };

    for (; tile < total; tile += gridDim.x) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        for (int k = 0; k < at.k_count; ++k) {
#pragma unroll
            for (int i = 0; i < TM; ++i) sx[i] = sx_next[i];
#pragma unroll
            for (int j = 0; j < TN; ++j) sw[j] = sw_next[j];
            quarter(std::integral_constant<int, 0>{});
            if constexpr (Q == 4) {
                quarter(std::integral_constant<int, 1>{});
                quarter(std::integral_constant<int, 2>{});
            }
            finish();
        }
        if constexpr (C::WK == 2) {
            // the two halves' sums: wave (kg) keeps the 32 x 32 tiles of row kg, and hands the others over
            v4f* const mine = reinterpret_cast<v4f*>(smem + C::R * C::STAGE + kg * C::XCH) + wmn * 64 + lane;
            const v4f* const theirs = reinterpret_cast<const v4f*>(smem + C::R * C::STAGE + (kg ^ 1) * C::XCH) + wmn * 64 + lane;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                if (j) lds_barrier();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v16f t = kg ? acc[0][j] : acc[1][j];
                    mine[e * (C::WM * C::WN * 64)] = v4f{t[4 * e], t[4 * e + 1], t[4 * e + 2], t[4 * e + 3]};
                }
                lds_barrier();
                if (kg) acc[0][j] = acc[1][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v4f t = theirs[e * (C::WM * C::WN * 64)];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[0][j][4 * e + i] += t[i];
                }
            }
        }
        // ---- lane (r, h) holds rows 32 i + r, columns 32 j + 8 h + 0 .. 7 and 16 more.  Lanes of 16 exchange halves of their runs, so
        // that four of them write 64 consecutive bytes of a row.
        constexpr int ROWS = TM / C::WK;
        const int m_wave = (wm * TM + kg * ROWS) * 32, n_wave = wn * TN * 32;
        float* const y = SPLIT ? a.part + (static_cast<int64_t>(at.split) * a.batch + at.prob) * a.M * a.N : a.y ? a.y + at.prob * a.strideO : nullptr;
        uint16_t* const out = SPLIT || !a.out ? nullptr : a.out + at.prob * a.strideO;
        const int el = lane_id(), er = el & 15, es = (el >> 4) & 1, eh = el >> 5;       // (not kept through the loop, nor what follows from them)
        // (where a run of a row lies in one lane: `first` of row er, `second` of row er + 16, both from column n on)
        auto turn = [&](u32x4& first, u32x4& second) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const u32_pair t = __builtin_amdgcn_permlane16_swap(first[e], second[e], false, false);
                first[e] = t.x;
                second[e] = t.y;
            }
        };
        // every run of the wave's tiles: bf16 in runs of 8 columns, fp32 in runs of 4
        auto bf16_runs = [&](auto store) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const v16f v = acc[i][j];
                    u32x4 first{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
                    u32x4 second{pack_bf16x2(v[8], v[9]), pack_bf16x2(v[10], v[11]), pack_bf16x2(v[12], v[13]), pack_bf16x2(v[14], v[15])};
                    turn(first, second);
                    store(first, second, i, j * 32 + es * 16, j);
                }
        };
        auto fp32_runs = [&](auto store) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
#pragma unroll
                for (int j = 0; j < 2 * TN; ++j) {
                    const v16f v = acc[i][j >> 1];
                    auto word = [&](int e) __attribute__((always_inline)) { return __float_as_uint(v[(j & 1) * 8 + e]); };
                    u32x4 first{word(0), word(1), word(2), word(3)}, second{word(4), word(5), word(6), word(7)};
                    turn(first, second);
                    store(first, second, i, j * 16 + es * 4, j);
                }
        };
        if (a.wide) {                  // whole runs of 8 columns, 32-bit offsets in a tile's rows; what is past the result is dropped
            const int64_t rows = a.M - at.m0 < C::BM ? a.M - at.m0 : C::BM;
            const int N = static_cast<int>(a.N), n_lane = at.n0 + n_wave + eh * 8, o_lane = (m_wave + er) * N + n_lane;
            // (the offset is the vector register's alone: behind a 16-byte store with a scalar offset the compiler lets the next
            // instruction overwrite the data, and now and then the last lanes of its first register left with the new value)
            auto into = [&](const __amdgpu_buffer_rsrc_t& o, int size, bool streamed) __attribute__((always_inline)) {
                return [=](u32x4 first, u32x4 second, int i, int n, int) __attribute__((always_inline)) {
                    const bool in = n_lane + n < N;
                    const int off = (o_lane + i * 32 * N + n) * size;
                    const int first_at = in ? off : 0x7FFFFFFF, second_at = in ? off + 16 * N * size : 0x7FFFFFFF;
                    if (streamed) {    // (how a store meets the caches is in its instruction; the lines keep the two from being joined)
                        __builtin_amdgcn_raw_buffer_store_b128(first, o, first_at, 0, 2);
                        __builtin_amdgcn_raw_buffer_store_b128(second, o, second_at, 0, 2);
                        asm volatile("; past the caches");
                    } else {
                        __builtin_amdgcn_raw_buffer_store_b128(first, o, first_at, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b128(second, o, second_at, 0, 0);
                        asm volatile("; into the caches");
                    }
                };
            };
            if (out) bf16_runs(into(__builtin_amdgcn_make_buffer_rsrc(out + at.m0 * a.N, 0, static_cast<int>(rows * a.N * 2), 0x00020000), 2, a.streamed));
            if (y) fp32_runs(into(__builtin_amdgcn_make_buffer_rsrc(y + at.m0 * a.N, 0, static_cast<int>(rows * a.N * 4), 0x00020000), 4, false));
            late = out && !y ? C::R - 1 : 0;
        } else {                       // rows that start anywhere (by elements, rows x columns x K: 16384 x 4098 x 1024 238 us, here 65; 4096 columns 57.  Past the
                                       // caches they lose: 65536 x 4098 x 512 264 -> 500)
            late = 0;
            const int64_t n_lane = at.n0 + n_wave + eh * 8, m_lane = at.m0 + m_wave + er;
            const int cols = a.N - n_lane > 256 ? 256 : static_cast<int>(a.N - n_lane), rows = a.M - m_lane > 256 ? 256 : static_cast<int>(a.M - m_lane);
            // elements first .. of v, a run of the row whose first column is n + n_lane, as far as the row goes
            auto put = [=](auto* base, u32x4 v, int row, int n, int first) __attribute__((always_inline)) {
                using T = std::remove_pointer_t<decltype(base)>;
                constexpr int PER = 16 / sizeof(T);
                T* const p = base + (m_lane + row) * a.N + n_lane + n;
                if (row >= rows) return;
                if (first == 0 && n + PER <= cols) *reinterpret_cast<u32x4_any*>(p) = v;
                else
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (e >= first && n + e < cols) {
                            if constexpr (sizeof(T) == 2) p[e] = static_cast<uint16_t>(v[e >> 1] >> ((e & 1) * 16));
                            else p[e] = __uint_as_float(v[e]);
                        }
            };
            const bool inside = C::WORDS && ((a.N | static_cast<int64_t>(reinterpret_cast<uintptr_t>(out) >> 1)) & 1);
            if (out && inside) {
                // Rows that start inside a word (all of a lane's rows, or none: they lie 16 apart) are stored one column to the left, in whole words: a
                // run's last element goes with the next run, the lane before it in the order (es, eh), or its own
                // value of the tile before.  (Inside words 16384 x 4097 x 1024 took 107 us, here 76.)
                const bool odd = (reinterpret_cast<uintptr_t>(out + m_lane * a.N) >> 1) & 1, first_run = es == 0 && eh == 0, last_run = es == 1 && eh == 1;
                const int from = (er + (eh ? es * 16 : 32 + (es ^ 1) * 16)) * 4;         // that lane
                uint32_t before[2] = {0u, 0u};
                bf16_runs([&](u32x4 first, u32x4 second, int i, int n, int j) __attribute__((always_inline)) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const u32x4 v = k ? second : first;
                        const uint32_t last = v[3], left = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(from, static_cast<int>(last_run ? before[k] : last)));
                        before[k] = last;
                        const u32x4 w{__builtin_amdgcn_alignbit(v[0], left, 16), __builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16),
                                      __builtin_amdgcn_alignbit(v[3], v[2], 16)};
                        const int row = i * 32 + k * 16;
                        put(out, odd ? w : v, row, odd ? n - 1 : n, odd && first_run && j == 0 ? 1 : 0);
                        if (odd && last_run && j == TN - 1 && row < rows && n + 7 < cols) out[(m_lane + row) * a.N + n_lane + n + 7] = static_cast<uint16_t>(last >> 16);
                    }
                });
            } else if (out) {
                bf16_runs([&](u32x4 first, u32x4 second, int i, int n, int) __attribute__((always_inline)) {
                    put(out, first, i * 32, n, 0);
                    put(out, second, i * 32 + 16, n, 0);
                });
            }
            if (y)
                fp32_runs([&](u32x4 first, u32x4 second, int i, int n, int) __attribute__((always_inline)) {
                    put(y, first, i * 32, n, 0);
                    put(y, second, i * 32 + 16, n, 0);
                });
        }
        if (tile + static_cast<int>(gridDim.x) < total) at = locate(tile + gridDim.x);
    }
    wait_vmcnt<0>();           // the requests past the end (zeros) land before the workgroup's LDS is given on
}

template <class C, bool SPLIT>
__global__ __launch_bounds__(64 * C::NW, C::NW * C::PER_CU / 4) void mx_tile_kernel(const MxArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    mx_tiles<C, SPLIT>(a, smem);
}

// Sums of the partial products of a split contraction, in order.
__global__ __launch_bounds__(256) void mx_join_kernel(const float* __restrict__ part, int splits, int64_t n, int64_t per_problem, int64_t stride_o,
                                                      uint16_t* __restrict__ out, float* __restrict__ y) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= n) return;
    float s = part[i];
    for (int k = 1; k < splits; ++k) s += part[k * n + i];
    const int64_t prob = i / per_problem, o = prob * stride_o + (i - prob * per_problem);
    if (out) out[o] = static_cast<uint16_t>(f32_to_bf16_rne(s));
    if (y) y[o] = s;
}

template <int MT, int NT, int QUANT>
static loka_status stream_launch(MxArgs a, int64_t batch, hipStream_t stream) {
    constexpr int NW = 8, SUMS = NW * MT * NT * 1024, OWN = QUANT == 0 ? 0 : NW * (QUANT == 2 ? 16 * kTurn : kRaw), LDS = SUMS > OWN ? SUMS : OWN;
    a.n_tiles = (a.N + 16 * NT - 1) / (16 * NT);
    a.m_tiles = (a.M + 16 * MT - 1) / (16 * MT);
    if (LDS > 65536) LOKA_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&mx_stream_kernel<MT, NT, NW, QUANT>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
    return in_launches(a.n_tiles * a.m_tiles * batch, 64 * NW, [&](int64_t from, uint32_t grid) {
        a.first_wg = from;
        mx_stream_kernel<MT, NT, NW, QUANT><<<grid, 64 * NW, LDS, stream>>>(a);
    });
}

// Columns of a workgroup.  Quantizing groups of x takes all of a CU's LDS, and x anew in every workgroup: as few columns as need no
// second round (us by 16 / 32 / 64 columns a workgroup: 16 x 4112 x 4096 8.6 / 6.6 / 8.6, 16 x 4096 x 4096 5.5 / 6.5 / 8.4, 16 x 12000 x 4096
// 13.9 / 11.7 / 9.0).
// Elsewhere several workgroups share a CU, and more columns in one pay only where there are many and K is not long (quantized
// by rows: 2 x 12000 x 4096 7.6 / 8.6 / 8.4, 2 x 16384 x 4096 10.1 / 8.9 / 9.0, 2 x 8192 x 16384 16.1 / 21.5 / 23.8, rows that start anywhere,
// which take longer, 2 x 14000 x 3001 8.8 / 7.3; stored X: 16 x 32768 x 1024 7.4 / 6.6 / 6.0, 16 x 8192 x 16384 20 / 41 / 28).
template <int MT, int QUANT>
static loka_status stream_columns(const MxArgs& a, int64_t batch, hipStream_t stream) {
    const int64_t runs = (a.N + 15) / 16 * batch;          // of 16 columns
    if constexpr (QUANT == 1 || QUANT == 3) {
        if (runs <= 256) return stream_launch<MT, 1, QUANT>(a, batch, stream);
        if (runs <= 512) return stream_launch<MT, 2, QUANT>(a, batch, stream);
        return stream_launch<MT, 4, QUANT>(a, batch, stream);
    } else if constexpr (QUANT == 2) {
        if (runs >= (a.x_whole ? 1024 : 512) && a.Kp <= 8192) return stream_launch<MT, 2, QUANT>(a, batch, stream);
    } else if constexpr (MT == 1) {
        if (runs >= 1024 && a.Kp <= 2048) return stream_launch<MT, 4, QUANT>(a, batch, stream);
    } else {
        if (runs >= 512) return stream_launch<MT, 2, QUANT>(a, batch, stream);
    }
    return stream_launch<MT, 1, QUANT>(a, batch, stream);
}

static MxArgs args_of(const loka_gemm_desc* d, const uint8_t* wq, const uint8_t* sw, void* out_bf16, float* y) {
    MxArgs a{};
    a.wq = wq;
    a.sw = sw;
    a.out = static_cast<uint16_t*>(out_bf16);
    a.y = y;
    a.M = d->M;
    a.N = d->N;
    a.K = d->K;
    a.Kp = mx_padded(d->K);
    a.strideX = d->strideX;
    a.strideW = d->strideW;
    a.strideO = d->batch > 1 ? d->strideO : 0;
    return a;
}

// What runs a product: the form expected to be fastest, and in how many ranges of K tiles.  The estimates are microseconds fitted to measured launches (rows x columns x K, measured / estimated): a result tile
// costs its form a fixed part and a part per K tile, times the rounds in which the chip takes them; the stream kernel costs by
// 512-element pieces of 16 columns, times the row tiles.
//   256 x 256            8192 x 8192 x 8192 295 / 294, 4096 x 4096 x 4096 43.5 / 43, 16384 x 4096 x 1024 60 / 60
//   128 x 128, K halves  8192 x 8192 x 8192 417 / 415, 4096 x 4096 x 4096 59 / 59, 1024 x 4096 x 16384 53.5 / 53, 2048^3 11.8 / 11.9
//   128 x 128, 4 waves   16384 x 4096 x 1024 68 / 67, 4096 x 4096 x 4096 53 / 55, 2048^3 11.5 / 11.5, 5013 x 720 x 1008 8.0 / 8.0, 2048 x 768 x 256 6.0 / 5.4
//   stream               16 x 4096 x 4096 4.6 / 5.5, 16 x 8192 x 16384 20 / 20, 32 x 4096 x 4096 5.8 / 6.0, 32 x 16384 x 4096 13.1 / 13.3, 64 x 4096 x 4096 8.3 / 8.0, 128 x 4096 x 4096 14.2 / 12.5,
//                        256 x 4096 x 4096 25 / 22, 256 x 768 x 2048 5.5 / 5.2
enum { MX_STREAM = 0, MX_LARGE = 1, MX_HALVES = 2, MX_SMALL = 3 };
struct MxPlan { int kind, tiles_m, tiles_n, splits, k_per_split; int64_t total; };
static MxPlan plan_of(const loka_gemm_desc* d) {
    MxPlan p{MX_STREAM, 0, 0, 1, 0, 0};
    const int64_t Kp = mx_padded(d->K), k = (Kp + 255) / 256;
    if (Kp >= (INT64_C(1) << 23)) return p;                            // (a tile's rows within 32-bit offsets)
    auto tiles = [&](int64_t b) { return static_cast<double>((d->M + b - 1) / b) * static_cast<double>((d->N + b - 1) / b) * static_cast<double>(d->batch); };
    auto rounds = [](double t, double slots) { return std::ceil(t / slots); };
    const double t256 = tiles(256), t128 = tiles(128), bytes = static_cast<double>(d->M) * static_cast<double>(d->N) * static_cast<double>(d->batch) * 8.0;
    if (t128 > 1e9) return p;
    const double rows = d->M <= 16 ? 16.0 : d->M <= 32 ? 32.0 : 64.0, piece = d->M <= 16 ? 0.0010 : d->M <= 32 ? 0.0012 : 0.0022;
    double best = 3.5 + std::ceil(static_cast<double>(d->M) / rows) * std::ceil(static_cast<double>(d->N) / 16.0) * static_cast<double>(d->batch) *
                            static_cast<double>((Kp + 511) / 512) * piece;
    auto take = [&](double us, int kind, int splits) {
        if (us >= best) return;
        best = us;
        p.kind = kind;
        p.splits = splits;
    };
    take(4.0 + rounds(t256, 256) * (5.5 + 2.1 * static_cast<double>(k)), MX_LARGE, 1);
    take(t128 <= 256 ? 4.5 + 0.88 * static_cast<double>(k) : 4.5 + rounds(t128, 512) * (2.0 + 1.45 * static_cast<double>(k)), MX_SMALL, 1);
    for (int64_t s = 1; s <= 64 && s <= k && (s == 1 || static_cast<double>(s) * t128 <= 1024); s *= 2) {
        const double per = std::ceil(static_cast<double>(k) / static_cast<double>(s));
        const double us = 4.0 + rounds(t128 * static_cast<double>(s), 256) * (2.0 + 0.74 * per) + (s > 1 ? 3.0 + bytes * static_cast<double>(s) / 4.5e6 : 0.0);
        take(us, MX_HALVES, static_cast<int>(s));
    }
    if (p.kind == MX_STREAM) return p;
    const int b = p.kind == MX_LARGE ? 256 : 128;
    p.tiles_m = static_cast<int>((d->M + b - 1) / b);
    p.tiles_n = static_cast<int>((d->N + b - 1) / b);
    p.k_per_split = static_cast<int>((k + p.splits - 1) / p.splits);
    p.splits = static_cast<int>((k + p.k_per_split - 1) / p.k_per_split);
    p.total = static_cast<int64_t>(tiles(b)) * p.splits;
    return p;
}

int mxfp4_gemm_form(const loka_gemm_desc* d) { return plan_of(d).kind; }

size_t mxfp4_gemm_workspace_bytes(const loka_gemm_desc* d) {
    const MxPlan p = plan_of(d);
    return p.splits > 1 ? static_cast<size_t>(p.splits) * d->batch * d->M * d->N * 4 : 0;
}

template <class C, bool SPLIT>
static loka_status tile_launch(const MxArgs& a, hipStream_t stream) {
    const int64_t slots = 256 * C::PER_CU;
    const uint32_t grid = static_cast<uint32_t>(a.total < slots ? a.total : slots);
    // (on every call, a host-side table write: no process-wide state, and correct on whichever device is current)
    LOKA_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&mx_tile_kernel<C, SPLIT>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS));
    mx_tile_kernel<C, SPLIT><<<grid, 64 * C::NW, C::LDS, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

loka_status mxfp4_gemm_launch(const loka_gemm_desc* d, const uint8_t* xq, const uint8_t* sx, const uint8_t* wq, const uint8_t* sw,
                              void* out_bf16, float* y, void* ws, size_t ws_bytes, hipStream_t stream) {
    MxArgs a = args_of(d, wq, sw, out_bf16, y);
    a.xq = xq;
    a.sx = sx;
    a.batch = d->batch;
    MxPlan p = plan_of(d);
    if (p.kind == MX_STREAM) {
        if (a.M <= 16) return stream_columns<1, 0>(a, d->batch, stream);
        if (a.M <= 32) return stream_columns<2, 0>(a, d->batch, stream);
        return stream_columns<4, 0>(a, d->batch, stream);
    }
    if (p.splits > 1 && ws_bytes < mxfp4_gemm_workspace_bytes(d)) {       // no room: unsplit
        p.total /= p.splits;
        p.splits = 1;
    }
    a.tiles_m = p.tiles_m;
    a.tiles_n = p.tiles_n;
    a.splits = p.splits;
    a.k_per_split = p.k_per_split;
    a.total = static_cast<int>(p.total);
    a.part = static_cast<float*>(ws);
    // A bf16 result that the 256 MB of last-level cache would not hold leaves that cache to the operands (rows x columns x K:
    // 32768 x 4096 x 4096 333 -> 303 us, 40000 x 4096 x 1000 161 -> 127, 65536 x 2048 x 1024 112 -> 103); smaller ones gain little or lose
    // (24576 x 4096 x 4096 240 -> 230, 49152 x 2048 x 2048 114 -> 119, 4096 x 4096 x 4096 42.9 -> 43.8), and the next kernel may read them there.
    a.streamed = a.M * a.N * d->batch >= INT64_C(1) << 27;
    a.wide = a.N % 8 == 0 && a.N < (INT64_C(1) << 21) && (d->batch == 1 || d->strideO % 8 == 0);
    using Large = MxTile<2, 4, 4, 2, 1, 2, true>;
    using Halves = MxTile<2, 2, 2, 2, 2, 3>;
    using Small = MxTile<2, 2, 2, 2, 1, 2>;
    using SmallWords = MxTile<2, 2, 2, 2, 1, 2, true>;
    if (p.kind == MX_LARGE) return tile_launch<Large, false>(a, stream);
    // (stores bound several rounds of small tiles: 65536 x 1025 x 256 71 -> 52 us by words; one round loses, 5013 x 721 x 1008 8.3 -> 8.5, and the longer
    // kernel by itself costs 5013 x 720 x 1008 3 %)
    const bool odd = a.out && ((a.N & 1) || (d->batch > 1 && (d->strideO & 1)));
    if (p.kind == MX_SMALL && odd && a.total > 256 * Small::PER_CU) return tile_launch<SmallWords, false>(a, stream);
    if (p.kind == MX_SMALL) return tile_launch<Small, false>(a, stream);
    if (p.splits == 1) return tile_launch<Halves, false>(a, stream);
    const loka_status st = tile_launch<Halves, true>(a, stream);
    if (st != LOKA_OK) return st;
    const int64_t per = a.M * a.N, n = per * d->batch;
    mx_join_kernel<<<static_cast<uint32_t>((n + 255) / 256), 256, 0, stream>>>(a.part, p.splits, n, per, d->batch > 1 ? d->strideO : per, a.out, a.y);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

bool mxfp4_linear_fused(const loka_gemm_desc* d) { return d->M <= 16; }

loka_status mxfp4_linear_fused_launch(const loka_gemm_desc* d, const void* x_bf16, int64_t ld, const uint8_t* wq, const uint8_t* sw,
                                      void* out_bf16, float* y, hipStream_t stream) {
    MxArgs a = args_of(d, wq, sw, out_bf16, y);
    a.strideX = a.strideW = a.strideO = 0;
    a.x = static_cast<const uint16_t*>(x_bf16);
    a.ldx = ld;
    a.x_whole = aligned16(x_bf16) && ld % 8 == 0 && a.K % 8 == 0;
    // (rows x columns x K, us by rows / by groups: 1 x 4096 x 4096 4.0 / 4.5, 2 x 4096 x 4096 4.2 / 4.5, 3 x 4096 x 4096 4.5 / 4.5, 4 x 4096 x 4096
    // 4.8 / 4.4, 1 x 4096 x 16384 9.2 / 10.7)
    if (a.M <= 2) return stream_columns<1, 2>(a, 1, stream);
    if (a.x_whole && a.K < (INT64_C(1) << 30)) return stream_columns<1, 1>(a, 1, stream);
    return stream_columns<1, 3>(a, 1, stream);
}

}  // namespace loka
