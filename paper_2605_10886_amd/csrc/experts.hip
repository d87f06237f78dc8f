// The choice of experts, and the sum of their results (include/loka.h: loka_route, loka_combine and their backward passes).
#include "experts.h"

#include <cmath>

namespace loka {

// ---------------------------------------------------------------------------------
// The choice.  L lanes hold a token's logits, V each (entry lane + L v), as keys whose order as unsigned integers is the logits'
// order: 0 for what may not be chosen.  A choice is the largest key over the lanes, then the lowest entry that has it.
constexpr int kRouteChunk = 128;       // tokens of a workgroup
constexpr int kRouteThreads = 256;

__device__ __forceinline__ uint32_t key_of(float x) {
    if (x != x) return 0xFFC00000u;                        // above plus infinity
    const uint32_t b = __float_as_uint(x + 0.0f);          // (-0 and +0 are equal)
    return b == 0xFF800000u ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int m = 1; m < L; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}
template <bool BF16>
__device__ __forceinline__ float logit_at(const void* logits, int64_t i) {
    return BF16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(logits)[i]) : static_cast<const float*>(logits)[i];
}

struct RouteArgs {
    const void* logits;
    int64_t tokens, ld;
    int experts, top_k, score, renorm;
    float scale;
    int32_t *expert, *slot, *row, *offsets;
    float* weight;
    int32_t* counts;                   // [chunks + 1][experts]: of a chunk's tokens, then the same of all earlier chunks; the last: of all
    int chunks;
    const float* dweight;
    void* dlogits;
};

// Exclusive sums of v over the workgroup's threads, in their order
template <int THREADS>
__device__ __forceinline__ int block_exclusive(int v, int* lds, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(s, d, 64);
        if (lane >= d) s += o;
    }
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    __syncthreads();
    return before + s - v;
}

// first[e] = rows of the experts before e, from the counts of all (in LDS); returns their sum
__device__ __forceinline__ int first_rows(const int* count, int* first, int experts, int* lds) {
    int base = 0;
    for (int e0 = 0; e0 < experts; e0 += kRouteThreads) {
        const int e = e0 + static_cast<int>(threadIdx.x);
        int total;
        const int s = block_exclusive<kRouteThreads>(e < experts ? count[e] : 0, lds, total);
        if (e < experts) first[e] = base + s;
        base += total;
    }
    return base;
}

// Choices and weights of a chunk's tokens, and each choice's place among those of the chunk with the same expert: a 128-bit mask
// of tokens per expert (atomic OR: no order), whose bits below a token's are counted.  One chunk alone is finished here.
template <int L, int V, bool BF16>
__global__ __launch_bounds__(kRouteThreads) void route_choose_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    unsigned long long* const mask = reinterpret_cast<unsigned long long*>(smem);          // [experts][2]
    int* const count = reinterpret_cast<int*>(mask + 2 * a.experts);
    int* const first = count + a.experts;
    int* const lds = first + a.experts;
    const int t = static_cast<int>(threadIdx.x), l = t % L, k = a.top_k;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRouteChunk;
    const int tokens = a.tokens - t0 < kRouteChunk ? static_cast<int>(a.tokens - t0) : kRouteChunk;
    for (int i = t; i < 2 * a.experts; i += kRouteThreads) mask[i] = 0;
    __syncthreads();
    constexpr int PER = kRouteThreads / L;
    for (int i = t / L; i < (tokens + PER - 1) / PER * PER; i += PER) {       // (whole waves: the lanes' exchanges need all of them)
        const bool in = i < tokens;
        const int64_t at = (t0 + (in ? i : 0)) * a.ld;
        uint32_t key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = l + L * v < a.experts ? key_of(logit_at<BF16>(a.logits, at + l + L * v)) : 0u;
        float all = 0.f;
        if (a.score == LOKA_SCORE_SOFTMAX && !a.renorm) {
            uint32_t m = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) m = key[v] > m ? key[v] : m;
            const float top = value_of(lanes_max_bits<L>(m));
#pragma unroll
            for (int v = 0; v < V; ++v) all += key[v] ? expf(value_of(key[v]) - top) : 0.f;
            all = lanes_sum<L>(all);
        }
        int mine = -1;                 // lane j: choice j
        uint32_t mine_key = 0, top_key = 0;
        for (int j = 0; j < k; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) m = key[v] > m ? key[v] : m;
            m = lanes_max_bits<L>(m);
            unsigned low = 0;          // 65535 - entry
#pragma unroll
            for (int v = V - 1; v >= 0; --v) low = key[v] == m ? 65535u - static_cast<unsigned>(l + L * v) : low;
            const int e = 65535 - static_cast<int>(lanes_max_bits<L>(low));
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = l + L * v == e ? 0u : key[v];
            if (j == 0) top_key = m;
            if (l == j && m) { mine = e; mine_key = m; }
        }
        const float x = value_of(mine_key), top = value_of(top_key);
        float w = 0.f;
        if (a.score == LOKA_SCORE_SOFTMAX) {
            w = mine >= 0 ? expf(x - top) : 0.f;
            const float sum = lanes_sum<L>(w);
            w = w / (a.renorm ? sum : all);
        } else if (!a.renorm) {
            w = 1.f / (1.f + expf(-x));
        } else {
            // sigmoid(x) = e^x / (1 + e^x), all by the same factor e^-min(top, 0), so that none of a row's vanishes for being small
            const float shift = top < 0.f ? top : 0.f;
            w = mine < 0 ? 0.f : x < 0.f ? expf(x - shift) / (1.f + expf(x)) : 1.f / (1.f + expf(-x));
            const float sum = lanes_sum<L>(w);
            w = w / sum;
        }
        if (in && l < k) {
            const int64_t o = (t0 + i) * k + l;
            a.expert[o] = mine;
            a.weight[o] = mine >= 0 ? a.scale * w : 0.f;
            if (mine >= 0) atomicOr(mask + 2 * mine + (i >> 6), 1ull << (i & 63));
        }
    }
    __syncthreads();
    for (int e = t; e < a.experts; e += kRouteThreads) {
        const int n = __popcll(mask[2 * e]) + __popcll(mask[2 * e + 1]);
        count[e] = n;
        if (a.chunks > 1) a.counts[static_cast<int64_t>(blockIdx.x) * a.experts + e] = n;
    }
    __syncthreads();
    const bool alone = a.chunks == 1;
    int total = 0;
    if (alone) total = first_rows(count, first, a.experts, lds);
    __syncthreads();
    for (int i = t; i < tokens * k; i += kRouteThreads) {
        const int e = a.expert[t0 * k + i], m = i / k;
        if (e >= 0) {
            const unsigned long long below = (1ull << (m & 63)) - 1;
            const int rank = m < 64 ? __popcll(mask[2 * e] & below) : __popcll(mask[2 * e]) + __popcll(mask[2 * e + 1] & below);
            a.slot[t0 * k + i] = alone ? first[e] + rank : rank;
            if (alone) a.row[first[e] + rank] = m;
        } else {
            a.slot[t0 * k + i] = -1;
        }
        if (alone && i >= total) a.row[i] = -1;
    }
    if (alone) {
        for (int e = t; e < a.experts; e += kRouteThreads) a.offsets[e] = first[e];
        if (t == 0) a.offsets[a.experts] = total;
    }
}

// Counts of the chunks -> of all earlier chunks, and of all.  A workgroup takes one expert.
__global__ __launch_bounds__(kRouteThreads) void route_scan_kernel(const RouteArgs a) {
    __shared__ int lds[kRouteThreads / 64];
    const int e = static_cast<int>(blockIdx.x);
    int base = 0;
    for (int c0 = 0; c0 < a.chunks; c0 += kRouteThreads) {
        const int c = c0 + static_cast<int>(threadIdx.x);
        int total;
        int32_t* const p = a.counts + static_cast<int64_t>(c) * a.experts + e;
        const int s = block_exclusive<kRouteThreads>(c < a.chunks ? *p : 0, lds, total);
        if (c < a.chunks) *p = base + s;
        base += total;
    }
    if (threadIdx.x == 0) a.counts[static_cast<int64_t>(a.chunks) * a.experts + e] = base;
}

__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    int* const count = reinterpret_cast<int*>(smem);
    int* const first = count + a.experts;
    int* const lds = first + a.experts;
    const int t = static_cast<int>(threadIdx.x), k = a.top_k;
    for (int e = t; e < a.experts; e += kRouteThreads) count[e] = a.counts[static_cast<int64_t>(a.chunks) * a.experts + e];
    __syncthreads();
    const int total = first_rows(count, first, a.experts, lds);
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = t; e < a.experts; e += kRouteThreads) a.offsets[e] = first[e];
        if (t == 0) a.offsets[a.experts] = total;
    }
    for (int e = t; e < a.experts; e += kRouteThreads) first[e] += a.counts[static_cast<int64_t>(blockIdx.x) * a.experts + e];
    __syncthreads();
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRouteChunk;
    const int tokens = a.tokens - t0 < kRouteChunk ? static_cast<int>(a.tokens - t0) : kRouteChunk;
    for (int i = t; i < tokens * k; i += kRouteThreads) {
        const int64_t o = t0 * k + i;
        const int e = a.expert[o];
        if (e >= 0) {
            const int s = first[e] + a.slot[o];
            a.slot[o] = s;
            a.row[s] = static_cast<int32_t>(t0 + i / k);
        }
        if (o >= total) a.row[o] = -1;
    }
}

// q: the weights without `scale` (softmax, and sigmoids with renorm); dl of a chosen entry:
//   softmax, renorm   q_j (g_j - sum_i g_i q_i)                      others 0
//   softmax           q_e (g_e - sum_i g_i q_i), g_e = 0 where not chosen
//   sigmoid, renorm   q_j (g_j - sum_i g_i q_i) (1 - s_j)            others 0
//   sigmoid           g_j s_j (1 - s_j)                              others 0
template <int L, int V, bool BF16>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(const RouteArgs a) {
    const int t = static_cast<int>(threadIdx.x), l = t % L, k = a.top_k;
    constexpr int PER = kRouteThreads / L;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * PER + t / L;
    const bool in = token < a.tokens;
    const int64_t at = (in ? token : a.tokens - 1) * a.ld, o = (in ? token : a.tokens - 1) * k + (l < k ? l : 0);
    int mine = l < k ? a.expert[o] : -1;
    if (mine >= a.experts) mine = -1;
    const float g = mine >= 0 ? a.scale * a.dweight[o] : 0.f;
    const float x = mine >= 0 ? logit_at<BF16>(a.logits, at + mine) : -INFINITY;
    const bool dense = a.score == LOKA_SCORE_SOFTMAX && !a.renorm;
    float lx[V], top = -INFINITY, all = 0.f;
    if (dense) {
        uint32_t m = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            lx[v] = l + L * v < a.experts ? logit_at<BF16>(a.logits, at + l + L * v) : -INFINITY;
            const uint32_t key = key_of(lx[v]);
            m = key > m ? key : m;
        }
        m = lanes_max_bits<L>(m);
        top = value_of(m);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            lx[v] = lx[v] == -INFINITY ? 0.f : expf(lx[v] - top);
            all += lx[v];
        }
        all = lanes_sum<L>(all);
    } else {
        top = value_of(lanes_max_bits<L>(key_of(x)));
    }
    float q = 0.f, d;                  // of this lane's choice
    if (a.score == LOKA_SCORE_SOFTMAX) {
        q = mine >= 0 ? expf(x - top) : 0.f;
        const float sum = a.renorm ? lanes_sum<L>(q) : all;
        q = mine >= 0 ? q / sum : 0.f;
        const float inner = lanes_sum<L>(g * q);
        d = a.renorm ? q * (g - inner) : g * q;
        if (dense)
#pragma unroll
            for (int v = 0; v < V; ++v) lx[v] = lx[v] == 0.f ? 0.f : -(lx[v] / all) * inner;
    } else {
        const float s = 1.f / (1.f + expf(-x)), rest = 1.f / (1.f + expf(x));              // sigmoid, and 1 - sigmoid
        if (a.renorm) {
            const float shift = top < 0.f ? top : 0.f;
            q = mine < 0 ? 0.f : x < 0.f ? expf(x - shift) / (1.f + expf(x)) : s;
            const float sum = lanes_sum<L>(q);
            q = mine >= 0 ? q / sum : 0.f;
            const float inner = lanes_sum<L>(g * q);
            d = q * (g - inner) * rest;
        } else {
            d = mine >= 0 ? g * s * rest : 0.f;
        }
    }
    if (!dense)
#pragma unroll
        for (int v = 0; v < V; ++v) lx[v] = 0.f;
    for (int j = 0; j < k; ++j) {
        const int e = __shfl(mine, j, L);
        const float dj = __shfl(d, j, L);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (l + L * v == e) lx[v] += dj;
    }
    if (!in) return;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (l + L * v < a.experts) {
            const int64_t at_out = token * a.experts + l + L * v;
            if (BF16) static_cast<uint16_t*>(a.dlogits)[at_out] = static_cast<uint16_t>(f32_to_bf16_rne(lx[v]));
            else static_cast<float*>(a.dlogits)[at_out] = lx[v];
        }
}

size_t route_workspace_bytes(const loka_route_desc* d) {
    const int64_t chunks = (d->tokens + kRouteChunk - 1) / kRouteChunk;
    return chunks > 1 ? static_cast<size_t>(chunks + 1) * static_cast<size_t>(d->experts) * 4 : 0;
}

// Lanes and logits a lane, by the number of experts
template <class F>
static void by_experts(int experts, F&& f) {
    using std::integral_constant;
    if (experts <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (experts <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (experts <= 256) f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else if (experts <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

static RouteArgs args_of(const loka_route_desc* d, const void* logits) {
    RouteArgs a{};
    a.logits = logits;
    a.tokens = d->tokens;
    a.ld = d->ld;
    a.experts = d->experts;
    a.top_k = d->top_k;
    a.score = d->score;
    a.renorm = d->renorm != 0;
    a.scale = d->scale;
    a.chunks = static_cast<int>((d->tokens + kRouteChunk - 1) / kRouteChunk);
    return a;
}

loka_status route_launch(const loka_route_desc* d, const void* logits, int32_t* expert, float* weight, int32_t* slot, int32_t* row,
                         int32_t* offsets, void* ws, hipStream_t stream) {
    RouteArgs a = args_of(d, logits);
    a.expert = expert;
    a.weight = weight;
    a.slot = slot;
    a.row = row;
    a.offsets = offsets;
    a.counts = static_cast<int32_t*>(ws);
    const size_t lds = static_cast<size_t>(d->experts) * 24 + 64;
    by_experts(d->experts, [&](auto l, auto v) {
        if (d->bf16) route_choose_kernel<l.value, v.value, true><<<a.chunks, kRouteThreads, lds, stream>>>(a);
        else route_choose_kernel<l.value, v.value, false><<<a.chunks, kRouteThreads, lds, stream>>>(a);
    });
    LOKA_HIP_TRY(hipGetLastError());
    if (a.chunks == 1) return LOKA_OK;
    route_scan_kernel<<<d->experts, kRouteThreads, 0, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    route_place_kernel<<<a.chunks, kRouteThreads, static_cast<size_t>(d->experts) * 8 + 64, stream>>>(a);
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

loka_status route_backward_launch(const loka_route_desc* d, const void* logits, const int32_t* expert, const float* dweight, void* dlogits,
                                  hipStream_t stream) {
    RouteArgs a = args_of(d, logits);
    a.expert = const_cast<int32_t*>(expert);
    a.dweight = dweight;
    a.dlogits = dlogits;
    by_experts(d->experts, [&](auto l, auto v) {
        const uint32_t grid = static_cast<uint32_t>((d->tokens * l.value + kRouteThreads - 1) / kRouteThreads);
        if (d->bf16) route_backward_kernel<l.value, v.value, true><<<grid, kRouteThreads, 0, stream>>>(a);
        else route_backward_kernel<l.value, v.value, false><<<grid, kRouteThreads, 0, stream>>>(a);
    });
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

// ---------------------------------------------------------------------------------
// The sum of a token's results.  A lane takes 8 columns of a token; bytes only.
struct CombineArgs {
    const uint16_t *y, *residual, *dout;
    const int32_t* slot;
    const float* weight;
    uint16_t *out, *dy;
    float* dweight;
    int64_t tokens, cols, rows;
    int64_t runs;                      // of 8 columns of a token
    int64_t first_wg;
    int top_k;
};

// Eight columns from c on; a row may start anywhere
__device__ __forceinline__ void store8(uint16_t* row, int64_t c, int64_t cols, u32x4 v) {
    if (c + 8 <= cols) { *reinterpret_cast<u32x4_any*>(row + c) = v; return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < cols) row[c + e] = static_cast<uint16_t>(v[e >> 1] >> ((e & 1) * 16));
}
__device__ __forceinline__ void widen(u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo(v[i]);
        f[2 * i + 1] = bf16_hi(v[i]);
    }
}
__device__ __forceinline__ u32x4 narrow(const float (&f)[8]) {
    return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}

__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
    const int64_t i = (a.first_wg + blockIdx.x) * 256 + threadIdx.x;
    const int64_t t = i / a.runs, c = (i - t * a.runs) * 8;
    if (t >= a.tokens) return;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.top_k; ++j) {
        const int64_t slot = a.slot[t * a.top_k + j];
        if (slot < 0 || slot >= a.rows) continue;
        const float w = a.weight ? a.weight[t * a.top_k + j] : 1.f;
        float f[8];
        widen(mx_load8(a.y + slot * a.cols, c, a.cols), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = fmaf(w, f[e], s[e]);
    }
    if (a.residual) {
        float f[8];
        widen(mx_load8(a.residual + t * a.cols, c, a.cols), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += f[e];
    }
    store8(a.out + t * a.cols, c, a.cols, narrow(s));
}

// A workgroup takes a token, so that its threads' parts of dweight meet in it.
__global__ __launch_bounds__(256) void combine_backward_kernel(const CombineArgs a) {
    __shared__ float part[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = a.first_wg + blockIdx.x;
    for (int j = 0; j < a.top_k; ++j) {
        const int64_t slot = a.slot[t * a.top_k + j];
        const bool live = slot >= 0 && slot < a.rows;
        const float w = a.weight ? a.weight[t * a.top_k + j] : 1.f;
        float sum = 0.f;
        if (live)
            for (int64_t c = threadIdx.x * 8; c < a.cols; c += 2048) {
                float d[8], o[8];
                widen(mx_load8(a.dout + t * a.cols, c, a.cols), d);
                if (a.dweight) {
                    float f[8];
                    widen(mx_load8(a.y + slot * a.cols, c, a.cols), f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(d[e], f[e], sum);
                }
                if (a.dy) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = w * d[e];
                    store8(a.dy + slot * a.cols, c, a.cols, narrow(o));
                }
            }
        sum = lanes_sum<64>(sum);
        if (lane == 0) part[wave][j] = sum;
    }
    __syncthreads();
    const int j = static_cast<int>(threadIdx.x);
    if (a.dweight && j < a.top_k) a.dweight[t * a.top_k + j] = (part[0][j] + part[1][j]) + (part[2][j] + part[3][j]);
}

static CombineArgs args_of(const loka_combine_desc* d, const int32_t* slot, const float* weight) {
    CombineArgs a{};
    a.slot = slot;
    a.weight = weight;
    a.tokens = d->tokens;
    a.cols = d->cols;
    a.rows = d->rows;
    a.top_k = d->top_k;
    a.runs = (d->cols + 7) / 8;
    return a;
}

loka_status combine_launch(const loka_combine_desc* d, const void* y, const int32_t* slot, const float* weight, const void* residual,
                           void* out, hipStream_t stream) {
    CombineArgs a = args_of(d, slot, weight);
    a.y = static_cast<const uint16_t*>(y);
    a.residual = static_cast<const uint16_t*>(residual);
    a.out = static_cast<uint16_t*>(out);
    return in_launches((a.tokens * a.runs + 255) / 256, 256, [&](int64_t from, uint32_t grid) {
        a.first_wg = from;
        combine_kernel<<<grid, 256, 0, stream>>>(a);
    });
}

loka_status combine_backward_launch(const loka_combine_desc* d, const void* dout, const void* y, const int32_t* slot, const float* weight,
                                    void* dy, float* dweight, hipStream_t stream) {
    CombineArgs a = args_of(d, slot, weight);
    a.dout = static_cast<const uint16_t*>(dout);
    a.y = static_cast<const uint16_t*>(y);
    a.dy = static_cast<uint16_t*>(dy);
    a.dweight = dweight;
    return in_launches(a.tokens, 256, [&](int64_t from, uint32_t grid) {
        a.first_wg = from;
        combine_backward_kernel<<<grid, 256, 0, stream>>>(a);
    });
}

}  // namespace loka
