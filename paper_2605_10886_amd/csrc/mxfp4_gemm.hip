// Products of MXFP4 operands (include/loka.h, loka_mxfp4_gemm / loka_mxfp4_linear) on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// The instruction takes 16 x 128 codes of each operand: lane l holds row l % 16, codes 32 (l / 16) .. + 31 in 16 bytes and that
// group's scale byte, so a lane's operand IS one stored group and its scale.  The weights are the first operand: a lane then
// holds four consecutive columns n of one row m of the result, which leave as one packed store.
//
// Which 32-groups of a row meet in one instruction is free as long as both operands agree: the four instructions of 512
// consecutive elements take groups 4 g + s (g: lane / 16, s: instruction), so a lane reads 64 consecutive bytes of codes and
// one word with the four scale bytes, which the instruction picks by its byte selector.
#include "mxfp4.h"

namespace loka {

constexpr int64_t kMaxThreads = INT64_C(1) << 32;       // of one launch

struct MxArgs {
    const uint8_t *xq, *sx, *wq, *sw;
    const uint16_t* x;                 // fused quantization: bf16 [M, ldx]
    uint16_t* out;
    float* y;
    int64_t M, N, K, Kp;               // Kp: stored row length in elements
    int64_t ldx;
    int64_t strideX, strideW, strideO; // elements between problems
    int64_t n_tiles, m_tiles;
    bool x_wide;                       // rows of x start on multiples of 16 bytes
};

template <int S>
__device__ __forceinline__ v4f mx_mfma(const u32x4 a, const u32x4 b, v4f c, uint32_t sa, uint32_t sb) {
    const v8i A = {static_cast<int>(a.x), static_cast<int>(a.y), static_cast<int>(a.z), static_cast<int>(a.w), 0, 0, 0, 0};
    const v8i B = {static_cast<int>(b.x), static_cast<int>(b.y), static_cast<int>(b.z), static_cast<int>(b.w), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, S, static_cast<int>(sa), S, static_cast<int>(sb));
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
// The same from a bf16 row: each group is quantized in the lane that holds it (loka_mxfp4_quantize's codes).
__device__ __forceinline__ MxPiece mx_quantize_piece(const uint16_t* x, int64_t K, int64_t group, bool wide) {
    MxPiece p;
    p.s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t k = (group + i) * kMxGroup;
        u32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = wide ? mx_load8<true>(x, k + j * 8, K) : mx_load8<false>(x, k + j * 8, K);
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

// ---------------------------------------------------------------------------------
// Few rows: bound by the weights' traffic.  A workgroup of NW waves owns 16 NT columns x 16 MT rows of the result; the waves
// take 512-element pieces of the contraction in turn, straight from memory into registers, and add their partial sums in LDS
// in wave order.
template <int MT, int NT, int NW, bool FUSED>
__global__ __launch_bounds__(64 * NW) void mx_stream_kernel(const MxArgs a) {
    __shared__ v4f part[NW][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    int64_t id = blockIdx.x;
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
#pragma unroll
        for (int j = 0; j < NT; ++j) w[j] = mx_read_piece(wq, sw, wrow[j], a.Kp, group);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (FUSED) x[i] = mx_quantize_piece(a.x + xrow[i] * a.ldx, a.K, group, a.x_wide);
            else x[i] = mx_read_piece(xq, sx, xrow[i], a.Kp, group);
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
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    // value (m, n) of tile (i, j) lies in lane (n % 16) / 4 * 16 + m % 16, component n % 4
    constexpr int total = MT * NT * 64;
    for (int k = threadIdx.x; k < total; k += 64 * NW) {
        const int tile = k >> 6, l = k & 63;
        v4f s = part[0][tile][l];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += part[w][tile][l];
        const int64_t m = m0 + (tile / NT) * 16 + (l & 15), n = n0 + (tile % NT) * 16 + (l >> 4) * 4;
        if (m >= a.M) continue;
        const int64_t o = prob * a.strideO + m * a.N + n;
        if (n + 4 <= a.N && (a.N & 3) == 0) {
            if (a.out) *reinterpret_cast<u32x2*>(a.out + o) = u32x2{pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w)};
            if (a.y) *reinterpret_cast<v4f*>(a.y + o) = s;
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

template <int MT, int NT, bool FUSED>
static loka_status stream_launch(MxArgs a, int64_t batch, hipStream_t stream) {
    constexpr int NW = 8;
    a.n_tiles = (a.N + 16 * NT - 1) / (16 * NT);
    a.m_tiles = (a.M + 16 * MT - 1) / (16 * MT);
    if (a.m_tiles > kMaxThreads || a.n_tiles * a.m_tiles >= kMaxThreads / (64 * NW) / batch) return LOKA_ERR_SHAPE;
    mx_stream_kernel<MT, NT, NW, FUSED><<<static_cast<uint32_t>(a.n_tiles * a.m_tiles * batch), 64 * NW, 0, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
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
    a.strideO = d->strideO;
    return a;
}

size_t mxfp4_gemm_workspace_bytes(const loka_gemm_desc*) { return 0; }

loka_status mxfp4_gemm_launch(const loka_gemm_desc* d, const uint8_t* xq, const uint8_t* sx, const uint8_t* wq, const uint8_t* sw,
                              void* out_bf16, float* y, void*, size_t, hipStream_t stream) {
    MxArgs a = args_of(d, wq, sw, out_bf16, y);
    a.xq = xq;
    a.sx = sx;
    if (a.M <= 16) return stream_launch<1, 1, false>(a, d->batch, stream);
    return stream_launch<2, 2, false>(a, d->batch, stream);
}

bool mxfp4_linear_fused(const loka_gemm_desc* d) { return d->M <= 16; }

loka_status mxfp4_linear_fused_launch(const loka_gemm_desc* d, const void* x_bf16, int64_t ld, const uint8_t* wq, const uint8_t* sw,
                                      void* out_bf16, float* y, hipStream_t stream) {
    MxArgs a = args_of(d, wq, sw, out_bf16, y);
    a.strideX = a.strideW = a.strideO = 0;
    a.x = static_cast<const uint16_t*>(x_bf16);
    a.ldx = ld;
    a.x_wide = aligned16(x_bf16) && ld % 8 == 0;
    return stream_launch<1, 1, true>(a, 1, stream);
}

}  // namespace loka
