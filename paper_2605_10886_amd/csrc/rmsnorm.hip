// Residual addition + RMSNorm + quantization, and its backward pass from an 8-bit checkpoint (include/loka.h,
// loka_add_rmsnorm / loka_rmsnorm_backward).  Bound by HBM: one pass over the rows, which stay in registers between the
// statistics and the stores.
#include "mxfp4.h"

namespace loka {

constexpr int kModeRow = 0, kModeBlock = 1, kModePow2 = 2, kModeNone = 3;      // of scales, as the kernels see them

struct RmsArgs {
    const uint16_t *x, *res, *gamma;
    uint16_t *h_out, *y_bf16;
    uint32_t* y_codes;
    float* y_scales;                   // (MXFP4: bytes)
    uint32_t* hq;
    float *hs, *rstd;
    int64_t rows, ld_x, ld_r, first_wg;
    int cols;
    int out, out_mode, ckpt_mode;
    float eps;
};

// ---- sums and maxima over the T threads of a row (T <= 64: lanes of a wave; else the workgroup)
template <int T>
__device__ __forceinline__ float lanes_sum(float a) {
#pragma unroll
    for (int m = 1; m < (T < 64 ? T : 64); m <<= 1) a += __shfl_xor(a, m, 64);
    return a;
}
template <int T>
__device__ __forceinline__ float lanes_most(float a) {     // of magnitudes, a NaN being the largest
    return __uint_as_float(lanes_max_bits<(T < 64 ? T : 64)>(__float_as_uint(a)));
}
__device__ __forceinline__ float most(float a, float b) {  // of magnitudes, a NaN being the largest
    return __uint_as_float(__float_as_uint(a) > __float_as_uint(b) ? __float_as_uint(a) : __float_as_uint(b));
}

// A row's inputs and results, STREAMED past the caches
template <bool STREAMED>
__device__ __forceinline__ u32x4 load16(const uint16_t* p) {
    return STREAMED ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)) : *reinterpret_cast<const u32x4*>(p);
}
template <bool STREAMED>
__device__ __forceinline__ void store16(uint16_t* p, u32x4 v) {
    if (STREAMED) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = v;
}

__device__ __forceinline__ void unpack8(const u32x4 w, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
}

// Scale and factor of an e4m3 group of y = v * rstd whose largest |v| is `am` (rstd = 1, or a power of two: of v itself, in its unit).  Away from the floor
// amax / 448 and 448 / amax: rstd cancels in the factor, so a code has one rounding fewer than v * rstd, then * 448 / amax
// (32768 x 4096, row scales: 122 codes are not the 64-bit formula's, where torch's fp32 operations leave 176).
// A group with an infinite or NaN value gets a NaN scale.
__device__ __forceinline__ void e4m3_group(bool pow2, float am, float rstd, float& scale, float& inv) {
    const float top = am * rstd;
    if (pow2) {
        group_scale_pow2(top, scale, inv);
        inv *= rstd;                   // (a power of two: exact)
    } else {
        group_scale(top, scale, inv);
        inv = top >= kAmaxFloor ? kE4M3Max / am : inv * rstd;
    }
    if (__float_as_uint(top) >= 0x7F800000u) scale = __uint_as_float(0x7FC00000u);
}

// A sum of squares from here on has fp32's precision (each of up to 32768 terms below 2^-126 is off by at most 2^-150), and beside an eps from
// here on a smaller sum's errors do not matter.  For a smaller eps another instance of the kernel looks at every sum: its branch, and
// what is not moved over it, cost rows that do not need it 0.1 us a launch and up to 3 % (5984 x 1280 12.6 -> 12.9 us, 32768 x 4096 the same).
constexpr float kLeast = 0x1p-90f;

// ---------------------------------------------------------------------------------
// T threads take a row (T = 16, 32, 64: several rows a wave or one; 256, 1024: a workgroup per row), CPL chunks of 8
// consecutive elements each, chunk j of thread t at 8 (t + j T): a group of 128 elements is 16 neighbouring lanes, one of 32 a quad.
template <int T, int CPL, bool STREAMED, bool RANGE>
__global__ __launch_bounds__(T < 256 ? 256 : T) void add_rmsnorm_kernel(const RmsArgs a) {
    constexpr int WG = T < 256 ? 256 : T;
    __shared__ float red[3][WG / 64];
    const int tid = static_cast<int>(threadIdx.x), t = tid % T;
    const int64_t row = (a.first_wg + blockIdx.x) * (WG / T) + tid / T;
    const bool live = row < a.rows;
    const int chunks = a.cols >> 3;
    float h[CPL][8], sum = 0.f, am_y = 0.f, am_h = 0.f;
    u32x4 g[CPL];
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
        const int c = t + j * T;
        u32x4 xv = u32x4{0u, 0u, 0u, 0u}, rv = u32x4{0u, 0u, 0u, 0u};
        g[j] = u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
        if (live && c < chunks) {
            xv = load16<STREAMED>(a.x + row * a.ld_x + c * 8);
            if (a.res) rv = load16<STREAMED>(a.res + row * a.ld_r + c * 8);
            if (a.gamma) g[j] = *reinterpret_cast<const u32x4*>(a.gamma + c * 8);
        }
        unpack8(xv, h[j]);
        if (a.res) {
            float r[8];
            unpack8(rv, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] += r[i];
        }
        if (a.h_out && live && c < chunks) {
            u32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(h[j][2 * i], h[j][2 * i + 1]);
            store16<STREAMED>(a.h_out + row * a.cols + c * 8, o);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[j][i], h[j][i], sum);
    }
    // the row's sum of squares, and its largest magnitudes where a scale is per row
    const bool row_y = a.out == LOKA_RMS_OUT_E4M3 && a.out_mode == kModeRow, row_h = a.ckpt_mode == kModeRow;
    auto over_row = [&]() __attribute__((always_inline)) {
        if (row_y) {
            am_y = 0.f;
#pragma unroll
            for (int j = 0; j < CPL; ++j) {
                float gf[8];
                unpack8(g[j], gf);
#pragma unroll
                for (int i = 0; i < 8; ++i) am_y = most(am_y, fabsf(h[j][i] * gf[i]));
            }
            am_y = lanes_most<T>(am_y);
        }
        if (row_h) {
            am_h = 0.f;
#pragma unroll
            for (int j = 0; j < CPL; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) am_h = most(am_h, fabsf(h[j][i]));
            am_h = lanes_most<T>(am_h);
        }
        sum = lanes_sum<T>(sum);
        if (T > 64) {
            if ((tid & 63) == 0) {
                red[0][tid >> 6] = sum;
                red[1][tid >> 6] = am_y;
                red[2][tid >> 6] = am_h;
            }
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < WG / 64; ++w) {
                sum += red[0][w];
                am_y = most(am_y, red[1][w]);
                am_h = most(am_h, red[2][w]);
            }
        }
    };
    over_row();
    // RANGE: a row whose squares fp32 does not hold (all of its lanes see the same sum) is taken up or down by a power of two, which is
    // exact; from here on h and 1 / rstd are in that unit.
    float up = 1.0f, down = 1.0f;
    if (RANGE && __builtin_expect(!(sum < 0x1p126f && sum >= kLeast), 0)) {
        const bool small = sum < 1.0f;
        up = small ? 0x1p96f : 0x1p-72f;
        down = small ? 0x1p-96f : 0x1p72f;
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < CPL; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[j][i] *= up;
                sum = __builtin_fmaf(h[j][i], h[j][i], sum);
            }
#pragma unroll
        for (int j = 0; j < CPL; ++j) asm volatile("" : "+v"(g[j]));       // (or gamma is unpacked once for both paths, and held: 72 registers for 62)
        if (T > 64) __syncthreads();   // (everyone has read the first sums)
        over_row();
    }
    if (!live) return;
    const float rstd = 1.0f / sqrtf(sum / static_cast<float>(a.cols) + a.eps * up * up);
    if (a.rstd && t == 0) a.rstd[row] = rstd * up;

    float sy = 0.f, iy = 0.f, sh = 0.f, ih = 0.f;
    if (row_y) {
        e4m3_group(false, am_y, rstd, sy, iy);
        if (t == 0) a.y_scales[row] = sy;
    }
    if (row_h) {
        e4m3_group(false, am_h, down, sh, ih);
        if (t == 0) a.hs[row] = sh;
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
        const int c = t + j * T;
        const int64_t at = row * chunks + c;             // chunk of the contiguous outputs
        if (a.ckpt_mode != kModeNone) {
            if (!row_h) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) m = most(m, fabsf(h[j][i]));
                m = lanes_most<16>(m);
                e4m3_group(a.ckpt_mode == kModePow2, m, down, sh, ih);
                if ((t & 15) == 0 && c < chunks) a.hs[row * (a.cols >> 7) + (c >> 4)] = sh;
            }
            // (past the caches too where y is bf16, 32768 x 4096 217 -> 187 us; beside codes it costs: e4m3 172 -> 176, MXFP4 158 -> 168)
            const u32x2 o = u32x2{e4m3x4(h[j][0] * ih, h[j][1] * ih, h[j][2] * ih, h[j][3] * ih), e4m3x4(h[j][4] * ih, h[j][5] * ih, h[j][6] * ih, h[j][7] * ih)};
            if (c < chunks) {
                if (STREAMED && a.out == LOKA_RMS_OUT_BF16) {
                    asm volatile("; past the caches");         // (or the two stores become one through the caches)
                    __builtin_nontemporal_store(o, reinterpret_cast<u32x2*>(a.hq + at * 2));
                    asm volatile("; past the caches");
                } else {
                    *reinterpret_cast<u32x2*>(a.hq + at * 2) = o;
                }
            }
        }
        float gf[8], v[8];
        unpack8(g[j], gf);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = h[j][i] * gf[i];
        if (a.out == LOKA_RMS_OUT_BF16) {
            u32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(v[2 * i] * rstd, v[2 * i + 1] * rstd);
            if (c < chunks) store16<false>(a.y_bf16 + at * 8, o);
        } else if (a.out == LOKA_RMS_OUT_E4M3) {
            if (!row_y) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) m = most(m, fabsf(v[i]));
                m = lanes_most<16>(m);
                e4m3_group(a.out_mode == kModePow2, m, rstd, sy, iy);
                if ((t & 15) == 0 && c < chunks) a.y_scales[row * (a.cols >> 7) + (c >> 4)] = sy;
            }
            if (c < chunks)
                *reinterpret_cast<u32x2*>(a.y_codes + at * 2) = u32x2{e4m3x4(v[0] * iy, v[1] * iy, v[2] * iy, v[3] * iy),
                                                                       e4m3x4(v[4] * iy, v[5] * iy, v[6] * iy, v[7] * iy)};
        } else {
            // the stored row is a multiple of 128 elements: 16 lanes write a whole block of it, zeros past cols
            const int blocks = (a.cols + kMxPad - 1) / kMxPad, blk = c >> 4;
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) { v[i] *= rstd; m = most(m, fabsf(v[i])); }
            if (c >= chunks) m = 0.f;
            const uint32_t byte = mx_scale_byte(quad_max(__float_as_uint(m)));
            const uint32_t codes = mx_codes_f32x8(v, mx_scale_value(byte)), four = quad_bytes(byte);
            if (blk < blocks) {
                a.y_codes[(row * blocks + blk) * 16 + (c & 15)] = byte == kMxNaN || c >= chunks ? 0u : codes;
                if ((t & 15) == 0) reinterpret_cast<uint32_t*>(a.y_scales)[row * blocks + blk] = four;
            }
        }
    }
}

// ---------------------------------------------------------------------------------
struct RmsBackArgs {
    const uint16_t *dy, *gamma, *dh;
    const uint8_t* hq;
    const float *hs, *rstd;
    uint16_t* dx;
    float* partial;                    // [workgroups][cols], or NULL
    int64_t rows, ld_dy, ld_dh;
    int cols, ckpt_mode;
};

// Eight e4m3 codes (two words) as floats
__device__ __forceinline__ void e4m3_values(const u32x2 w, float (&f)[8]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[k]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[k]), true);
        f[4 * k] = lo.x; f[4 * k + 1] = lo.y; f[4 * k + 2] = hi.x; f[4 * k + 3] = hi.y;
    }
}

// Layout of rows and chunks as above; a workgroup walks over rows, adding dgamma's terms of its columns in registers, and
// leaves one row of partial sums.  A row stays in its loaded form (11 registers a chunk, 16 as fp32) between its two
// uses, so that the next row's loads are in flight while this one is reduced (PREFETCH; not beyond 16384 elements, whose 1024 threads
// hold four chunks each in half the registers).
template <int T, int CPL, bool PREFETCH, bool STREAMED>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rmsnorm_backward_kernel(const RmsBackArgs a) {
    constexpr int WG = T < 256 ? 256 : T, RPW = WG / T;
    __shared__ float red[2][WG / 64];
    const int tid = static_cast<int>(threadIdx.x), t = tid % T, sub = tid / T;
    const int chunks = a.cols >> 3;
    struct Row { u32x4 dy[CPL], dh[CPL]; u32x2 q[CPL]; float s[CPL], rstd; };
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        Row v;
        v.rstd = row < a.rows ? a.rstd[row] : 0.f;
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
            const int c = t + j * T;
            v.dy[j] = v.dh[j] = u32x4{0u, 0u, 0u, 0u};
            v.q[j] = u32x2{0u, 0u};
            v.s[j] = 0.f;
            if (row < a.rows && c < chunks) {
                v.dy[j] = load16<STREAMED>(a.dy + row * a.ld_dy + c * 8);
                v.q[j] = *reinterpret_cast<const u32x2*>(a.hq + (row * chunks + c) * 8);
                v.s[j] = a.ckpt_mode == kModeRow ? a.hs[row] : a.hs[row * (a.cols >> 7) + (c >> 4)];
                if (PREFETCH && a.dh) v.dh[j] = load16<STREAMED>(a.dh + row * a.ld_dh + c * 8);
            }
        }
        return v;
    };
    auto gamma_of = [&](int j) __attribute__((always_inline)) {
        if (a.gamma && t + j * T < chunks) return *reinterpret_cast<const u32x4*>(a.gamma + (t + j * T) * 8);
        return u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    };
    constexpr bool KEEP = T < 1024;    // gamma in registers (1024 threads have half as many: read again for each row)
    float dg[CPL][8];
    u32x4 g[KEEP ? CPL : 1];
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[j][i] = 0.f;
        if (KEEP) g[j] = gamma_of(j);
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * RPW;
    int64_t base = static_cast<int64_t>(blockIdx.x) * RPW;
    Row v = load(base + sub);
    for (int turn = 0; base < a.rows; base += step, turn ^= 1) {
        const int64_t row = base + sub;
        Row next;
        if (PREFETCH) next = load(row + step);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
            float d[8], n[8], gf[8];
            unpack8(v.dy[j], d);
            e4m3_values(v.q[j], n);
            unpack8(KEEP ? g[KEEP ? j : 0] : gamma_of(j), gf);
            v.s[j] *= v.rstd;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] *= v.s[j];
                dg[j][i] = __builtin_fmaf(d[i], n[i], dg[j][i]);
                sum = __builtin_fmaf(d[i] * gf[i], n[i], sum);
            }
        }
        sum = lanes_sum<T>(sum);
        if (T > 64) {                  // (two sets: a row's sums are written while slow waves still read the last row's)
            if ((tid & 63) == 0) red[turn][tid >> 6] = sum;
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < WG / 64; ++w) sum += red[turn][w];
        }
        const float mean = sum / static_cast<float>(a.cols);
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
            const int c = t + j * T;
            if (row < a.rows && c < chunks) {
                float d[8], n[8], gf[8], e[8];
                unpack8(v.dy[j], d);
                e4m3_values(v.q[j], n);
                unpack8(KEEP ? g[KEEP ? j : 0] : gamma_of(j), gf);
                if (!PREFETCH && a.dh) v.dh[j] = load16<STREAMED>(a.dh + row * a.ld_dh + c * 8);
                unpack8(v.dh[j], e);
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = __builtin_fmaf(v.rstd, __builtin_fmaf(-mean, n[i] * v.s[j], d[i] * gf[i]), e[i]);
                u32x4 o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(e[2 * i], e[2 * i + 1]);
                store16<STREAMED>(a.dx + row * a.cols + c * 8, o);
            }
        }
        if (PREFETCH) v = next;
        else v = load(row + step);
    }
    if (!a.partial) return;
    float* const mine = a.partial + static_cast<int64_t>(blockIdx.x) * a.cols;
    if (T >= WG) {
#pragma unroll
        for (int j = 0; j < CPL; ++j)
            if (t + j * T < chunks) {
                float* p = mine + (t + j * T) * 8;
                *reinterpret_cast<v4f*>(p) = v4f{dg[j][0], dg[j][1], dg[j][2], dg[j][3]};
                *reinterpret_cast<v4f*>(p + 4) = v4f{dg[j][4], dg[j][5], dg[j][6], dg[j][7]};
            }
    } else {
        // several rows at once: their sums join in LDS, row group after row group
        __shared__ __align__(16) float joined[T < 256 ? T * CPL * 8 : 8];
        for (int k = 0; k < RPW; ++k) {
            if (sub == k) {
#pragma unroll
                for (int j = 0; j < CPL; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        v4f* p = reinterpret_cast<v4f*>(joined + (t + j * T) * 8 + 4 * i);
                        const v4f x = v4f{dg[j][4 * i], dg[j][4 * i + 1], dg[j][4 * i + 2], dg[j][4 * i + 3]};
                        *p = k ? *p + x : x;
                    }
            }
            __syncthreads();
        }
        for (int c = tid * 4; c < a.cols; c += WG * 4) *reinterpret_cast<v4f*>(mine + c) = *reinterpret_cast<const v4f*>(joined + c);
    }
}

// dgamma: 32 columns a workgroup (8 lanes of 4), 32 slices of the partial rows, added in order
__global__ __launch_bounds__(256) void rmsnorm_dgamma_kernel(const float* __restrict__ partial, int n, int cols, float* __restrict__ dgamma) {
    __shared__ float red[32][33];
    const int k = (threadIdx.x & 7) * 4, s = threadIdx.x >> 3;
    const int c = blockIdx.x * 32 + k;
    v4f sum = v4f{0.f, 0.f, 0.f, 0.f};
    if (c < cols) {
#pragma unroll 4
        for (int i = s; i < n; i += 32) sum += *reinterpret_cast<const v4f*>(partial + static_cast<int64_t>(i) * cols + c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[s][k + i] = sum[i];
    __syncthreads();
    const int col = static_cast<int>(threadIdx.x);
    if (col < 32 && blockIdx.x * 32 + col < cols) {
        float total = red[0][col];
#pragma unroll
        for (int i = 1; i < 32; ++i) total += red[i][col];
        dgamma[blockIdx.x * 32 + col] = total;
    }
}

// ---------------------------------------------------------------------------------
static int kernel_mode(int mode) {
    return mode == LOKA_SCALE_ROW ? kModeRow : mode == LOKA_SCALE_BLOCK_1x128 ? kModeBlock : kModePow2;
}

// From here on the 256 MB of last-level cache cannot hold what a call moves (5 to 8 bytes an element), and rows that pass it by are
// faster (8192 x 8192: forward 87 -> 76 us, with the checkpoint 100 -> 87, backward 93 -> 84); below they lose (8192 x 4096: 36 -> 41,
// 43 -> 47, 39 -> 42).  y goes through
// the caches: the next product reads it, and the call itself is faster (32768 x 4096: codes past them too 148 -> 160 us, bf16 158 -> 184).
static bool streamed(int64_t rows, int64_t cols) { return rows * cols >= INT64_C(1) << 26; }

template <int T, int CPL>
static loka_status forward_launch(RmsArgs a, hipStream_t stream) {
    constexpr int WG = T < 256 ? 256 : T;
    return in_launches((a.rows + WG / T - 1) / (WG / T), WG, [&](int64_t from, uint32_t grid) {
        a.first_wg = from;
        const bool past = streamed(a.rows, a.cols);
        if (a.eps < kLeast) {
            if (past) add_rmsnorm_kernel<T, CPL, true, true><<<grid, WG, 0, stream>>>(a);
            else add_rmsnorm_kernel<T, CPL, false, true><<<grid, WG, 0, stream>>>(a);
        } else {
            if (past) add_rmsnorm_kernel<T, CPL, true, false><<<grid, WG, 0, stream>>>(a);
            else add_rmsnorm_kernel<T, CPL, false, false><<<grid, WG, 0, stream>>>(a);
        }
    });
}

loka_status add_rmsnorm_launch(const loka_rms_desc* d, const void* x, const void* residual, const void* gamma, void* h_out, void* y_out,
                               void* y_scales, uint8_t* hq, float* hs, float* rstd, hipStream_t stream) {
    RmsArgs a{};
    a.x = static_cast<const uint16_t*>(x);
    a.res = static_cast<const uint16_t*>(residual);
    a.gamma = static_cast<const uint16_t*>(gamma);
    a.h_out = static_cast<uint16_t*>(h_out);
    a.y_bf16 = static_cast<uint16_t*>(y_out);
    a.y_codes = static_cast<uint32_t*>(y_out);
    a.y_scales = static_cast<float*>(y_scales);
    a.hq = reinterpret_cast<uint32_t*>(hq);
    a.hs = hs;
    a.rstd = rstd;
    a.rows = d->rows;
    a.ld_x = d->ld_x;
    a.ld_r = d->ld_r;
    a.cols = static_cast<int>(d->cols);
    a.out = d->out;
    a.out_mode = d->out == LOKA_RMS_OUT_E4M3 ? kernel_mode(d->out_mode) : kModeNone;
    a.ckpt_mode = hq ? kernel_mode(d->ckpt_mode) : kModeNone;
    a.eps = d->eps;
    // One or two chunks a lane wherever lanes suffice: more rows than registers hold at once stay in flight (a wave a row, 8 chunks a
    // lane: 32768 x 4096 with the checkpoint 217 us, here 193, both through the caches; 4096 x 2048 15.1 and 12.9).
    const int chunks = a.cols / 8;
    if (chunks <= 16) return forward_launch<16, 1>(a, stream);
    if (chunks <= 32) return forward_launch<32, 1>(a, stream);
    if (chunks <= 64) return forward_launch<64, 1>(a, stream);
    if (chunks <= 128) return forward_launch<64, 2>(a, stream);
    if (chunks <= 256) return forward_launch<256, 1>(a, stream);
    if (chunks <= 512) return forward_launch<256, 2>(a, stream);
    if (chunks <= 1024) return forward_launch<512, 2>(a, stream);
    if (chunks <= 2048) return forward_launch<512, 4>(a, stream);
    return forward_launch<1024, 4>(a, stream);
}

// Workgroups of the backward pass: two a CU, which keep enough loads in flight, so that the partial sums stay small beside the rows
// (32768 x 4096 through the caches: 169 us, with three 185, with four 197; 5013 x 1008 10.8, 12.7, 12.7)
static int64_t backward_groups(int64_t rows, int cols) {
    const int rpw = cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 1024 ? 4 : 1;
    const int64_t most = (rows + rpw - 1) / rpw;
    return most < 512 ? most : 512;
}

size_t rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    return static_cast<size_t>(backward_groups(rows, static_cast<int>(cols))) * static_cast<size_t>(cols) * 4;
}

template <int T, int CPL, bool PREFETCH = true>
static void backward_launch(const RmsBackArgs& a, int64_t groups, hipStream_t stream) {
    constexpr int WG = T < 256 ? 256 : T;
    if (streamed(a.rows, a.cols)) rmsnorm_backward_kernel<T, CPL, PREFETCH, true><<<static_cast<uint32_t>(groups), WG, 0, stream>>>(a);
    else rmsnorm_backward_kernel<T, CPL, PREFETCH, false><<<static_cast<uint32_t>(groups), WG, 0, stream>>>(a);
}

loka_status rmsnorm_backward_launch(const loka_rms_desc* d, const void* dy, const uint8_t* hq, const float* hs, const float* rstd,
                                    const void* gamma, const void* dh, void* dx, float* dgamma, void* workspace, hipStream_t stream) {
    RmsBackArgs a{};
    a.dy = static_cast<const uint16_t*>(dy);
    a.gamma = static_cast<const uint16_t*>(gamma);
    a.dh = static_cast<const uint16_t*>(dh);
    a.hq = hq;
    a.hs = hs;
    a.rstd = rstd;
    a.dx = static_cast<uint16_t*>(dx);
    a.partial = dgamma ? static_cast<float*>(workspace) : nullptr;
    a.rows = d->rows;
    a.ld_dy = d->ld_x;
    a.ld_dh = d->ld_r;
    a.cols = static_cast<int>(d->cols);
    a.ckpt_mode = kernel_mode(d->ckpt_mode);
    const int64_t groups = backward_groups(a.rows, a.cols);
    const int chunks = a.cols / 8;
    if (chunks <= 16) backward_launch<16, 1>(a, groups, stream);
    else if (chunks <= 32) backward_launch<32, 1>(a, groups, stream);
    else if (chunks <= 64) backward_launch<64, 1>(a, groups, stream);
    else if (chunks <= 128) backward_launch<64, 2>(a, groups, stream);
    else if (chunks <= 256) backward_launch<256, 1>(a, groups, stream);
    else if (chunks <= 512) backward_launch<256, 2>(a, groups, stream);
    else if (chunks <= 1024) backward_launch<256, 4>(a, groups, stream);
    else if (chunks <= 2048) backward_launch<1024, 2>(a, groups, stream);
    else backward_launch<1024, 4, false>(a, groups, stream);
    LOKA_HIP_TRY(hipGetLastError());
    if (dgamma) {
        rmsnorm_dgamma_kernel<<<static_cast<uint32_t>((a.cols + 31) / 32), 256, 0, stream>>>(a.partial, static_cast<int>(groups), a.cols, dgamma);
        LOKA_HIP_TRY(hipGetLastError());
    }
    return LOKA_OK;
}

}  // namespace loka
