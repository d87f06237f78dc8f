// The choice of experts, and the sum of their results (include/loka.h: loka_route, loka_combine and their backward passes).
#include "experts.h"

#include <algorithm>
#include <cmath>

namespace loka {

// ---------------------------------------------------------------------------------
// The choice.  L lanes hold a token's logits, V each, in runs of R that follow each other in memory, as keys whose order as unsigned
// integers is the logits' order: 0 for what may not be chosen.  A choice is the largest key over the lanes, then the lowest entry that has it.  A
// bf16's key has room for the entry as well, so that all keys differ and the largest one is the choice; the next one is the largest below
// it, and no key has to be struck out.
//
// Bound by the vector unit's top_k passes over the keys: 32768 x 256 bf16 logits, 8 choices, 13.5 us (the 17 MB read alone: 3), their
// places 7.6.  A token alone: 5.2 us with the launch, of which the logits' journey and top_k exchanges are most.
constexpr int kRouteMostChunk = 128;   // tokens of a workgroup, at most
constexpr int kRouteThreads = 256;     // ... and its threads, of a small call and of the gradient
constexpr int kRouteMost = 1024;       // ... of a call of more tokens

__device__ __forceinline__ uint32_t key_of(float x) {
    x += 0.0f;                                             // (-0 and +0 are equal)
    const uint32_t b = x != x ? 0x7FC00000u : __float_as_uint(x);          // (a NaN: above plus infinity)
    return (b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u)) - 0x007FFFFFu;       // (of minus infinity, the least: 0)
}
__device__ __forceinline__ float value_of(uint32_t key) {
    const uint32_t k = key + 0x007FFFFFu;
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
// A bf16's key, and 1023 - its entry in the lower bits; below kNone: may not be chosen.  The upper bits that key_of gives a bf16 (0x7F80 to plus zero) say which it was.
constexpr uint32_t kNone = 1024;
__device__ __forceinline__ uint32_t short_key(uint32_t key, int entry) { return ((key >> 6) & ~1023u) | (1023u - static_cast<unsigned>(entry)); }
__device__ __forceinline__ float value_of_short(uint32_t k) { return value_of((k >> 10 << 16) | (k >= 0x7F80u << 10 ? 1u : 0u)); }

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
// entry v of lane l
template <int L, int R>
__device__ __forceinline__ int entry_of(int l, int v) { return ((v / R) * L + l) * R + v % R; }
// A lane's logits of the row at element `at`; minus infinity past the experts
template <int L, int V, int R, bool BF16>
__device__ __forceinline__ void load_logits(const void* logits, int64_t at, int experts, int l, float (&x)[V]) {
#pragma unroll
    for (int b = 0; b < V; b += R) {
        const int e = entry_of<L, R>(l, b);
        if constexpr (R == 1) {
            x[b] = e < experts ? logit_at<BF16>(logits, at + e) : -INFINITY;
        } else {                       // (runs are whole)
            const bool in = e < experts;
            const int64_t i = at + (in ? e : 0);
            if constexpr (!BF16) {
                const v4f v = *reinterpret_cast<const v4f*>(static_cast<const float*>(logits) + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[b + k] = in ? v[k] : -INFINITY;
            } else {
                uint32_t w[R / 2];
                if constexpr (R == 8) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(logits) + i);
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = v[k];
                } else {
                    const u32x2 v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(logits) + i);
                    w[0] = v.x;
                    w[1] = v.y;
                }
#pragma unroll
                for (int k = 0; k < R / 2; ++k) {
                    x[b + 2 * k] = in ? bf16_lo(w[k]) : -INFINITY;
                    x[b + 2 * k + 1] = in ? bf16_hi(w[k]) : -INFINITY;
                }
            }
        }
    }
}

struct RouteArgs {
    const void* logits;
    int64_t tokens, ld;
    int experts, top_k, score, renorm;
    float scale;
    int32_t *expert, *slot, *row, *offsets;
    float* weight;
    int32_t* counts;                   // [chunks + 1][pitch]: of a chunk's tokens; scanned: of all earlier chunks, the last of all
    int chunks, chunk_tokens, pitch;   // pitch: experts up to a power of two, 4 at least
    const float* dweight;
    void* dlogits;
};

// Exclusive sums of v over the workgroup's threads, in their order
template <int THREADS>
__device__ __forceinline__ int block_exclusive(int v, int* lds, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int s = lanes_inclusive(v);
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
template <int THREADS>
__device__ __forceinline__ int first_rows(const int* count, int* first, int experts, int* lds) {
    int base = 0;
    for (int e0 = 0; e0 < experts; e0 += THREADS) {
        const int e = e0 + static_cast<int>(threadIdx.x);
        int total;
        const int s = block_exclusive<THREADS>(e < experts ? count[e] : 0, lds, total);
        if (e < experts) first[e] = base + s;
        base += total;
    }
    return base;
}

// Choices and weights of a chunk's tokens, and each choice's place among those of the chunk with the same expert: a 128-bit mask
// of tokens per expert (atomic OR: no order), whose bits below a token's are counted.  One chunk alone is finished here.
template <int L, int V, int R, bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void route_choose_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    unsigned long long* const mask = reinterpret_cast<unsigned long long*>(smem);          // [experts][2]
    int* const count = reinterpret_cast<int*>(mask + 2 * a.experts);
    int* const first = count + a.experts;
    int* const lds = first + a.experts;
    const int t = static_cast<int>(threadIdx.x), l = t % L, k = a.top_k;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * a.chunk_tokens;
    const int tokens = a.tokens - t0 < a.chunk_tokens ? static_cast<int>(a.tokens - t0) : a.chunk_tokens;
    for (int i = t; i < 2 * a.experts; i += THREADS) mask[i] = 0;
    __syncthreads();
    constexpr int PER = THREADS / L;
    for (int i = t / L; i < (tokens + PER - 1) / PER * PER; i += PER) {       // (whole waves: the lanes' exchanges need all of them)
        const bool in = i < tokens;
        const int64_t at = (t0 + (in ? i : 0)) * a.ld;
        uint32_t key[V];
        {
            float x[V];
            load_logits<L, V, R, BF16>(a.logits, at, a.experts, l, x);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                key[v] = key_of(x[v]);
                if (BF16) key[v] = short_key(key[v], entry_of<L, R>(l, v));
            }
        }
        auto number = [](uint32_t k) __attribute__((always_inline)) { return BF16 ? value_of_short(k) : value_of(k); };
        constexpr uint32_t LEAST = BF16 ? kNone : 1;       // key of what may be chosen
        float all = 0.f;
        if (a.score == LOKA_SCORE_SOFTMAX && !a.renorm) {
            uint32_t m = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) m = key[v] > m ? key[v] : m;
            const float top = number(lanes_max_bits<L>(m));
#pragma unroll
            for (int v = 0; v < V; ++v) all += key[v] >= LEAST ? expf(number(key[v]) - top) : 0.f;
            all = lanes_sum<L>(all);
        }
        int mine = -1;                 // lane j: choice j
        uint32_t mine_key = 0, top_key = 0;
        uint32_t m = BF16 ? 1u << 26 : 0u;                 // the choice before
        for (int j = 0; j < k; ++j) {
            int e;
            if (BF16) {
                // the largest key below it: of the differences, as unsigned numbers, those of smaller keys are the large ones
                uint32_t d = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) d = key[v] - m > d ? key[v] - m : d;
                d = lanes_max_bits<L>(d);
                m = d >> 31 ? m + d : 0u;
                e = 1023 - static_cast<int>(m & 1023u);
            } else {
                m = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) m = key[v] > m ? key[v] : m;
                m = lanes_max_bits<L>(m);
                unsigned low = 0;      // 65535 - entry
#pragma unroll
                for (int v = V - 1; v >= 0; --v) low = key[v] == m ? 65535u - static_cast<unsigned>(entry_of<L, R>(l, v)) : low;
                e = 65535 - static_cast<int>(lanes_max_bits<L>(low));
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = entry_of<L, R>(l, v) == e ? 0u : key[v];
            }
            if (j == 0) top_key = m;
            if (l == j && m >= LEAST) { mine = e; mine_key = m; }
        }
        const float x = number(mine_key), top = number(top_key);
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
    for (int e = t; e < a.experts; e += THREADS) {
        const int n = __popcll(mask[2 * e]) + __popcll(mask[2 * e + 1]);
        count[e] = n;
        if (a.chunks > 1) a.counts[static_cast<int64_t>(blockIdx.x) * a.pitch + e] = n;
    }
    __syncthreads();
    const bool alone = a.chunks == 1;
    int total = 0;
    if (alone) total = first_rows<THREADS>(count, first, a.experts, lds);
    __syncthreads();
    for (int i = t; i < tokens * k; i += THREADS) {
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
        for (int e = t; e < a.experts; e += THREADS) a.offsets[e] = first[e];
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
        int32_t* const p = a.counts + static_cast<int64_t>(c) * a.pitch + e;
        const int s = block_exclusive<kRouteThreads>(c < a.chunks ? *p : 0, lds, total);
        if (c < a.chunks) *p = base + s;
        base += total;
    }
    if (threadIdx.x == 0) a.counts[static_cast<int64_t>(a.chunks) * a.pitch + e] = base;
}

// Rows of the routed order.  The chunks' counts are added up here (SCANNED: by route_scan_kernel): threads take four experts of
// every so many-th chunk, and their sums meet in LDS.
template <bool SCANNED>
__global__ __launch_bounds__(kRouteMost) void route_place_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    int* const count = reinterpret_cast<int*>(smem);
    int* const first = count + a.experts;
    int* const before = first + a.experts;                 // of earlier chunks
    int* const lds = before + a.experts;
    const int t = static_cast<int>(threadIdx.x), k = a.top_k, chunk = static_cast<int>(blockIdx.x);
    const int64_t t0 = static_cast<int64_t>(chunk) * a.chunk_tokens;
    const int tokens = a.tokens - t0 < a.chunk_tokens ? static_cast<int>(a.tokens - t0) : a.chunk_tokens;
    // (a thread's first choice travels while the counts are added up)
    const int my_expert = t < tokens * k ? a.expert[t0 * k + t] : -1, my_rank = t < tokens * k ? a.slot[t0 * k + t] : 0;
    if (SCANNED) {
        for (int e = t; e < a.experts; e += kRouteMost) {
            count[e] = a.counts[static_cast<int64_t>(a.chunks) * a.pitch + e];
            before[e] = a.counts[static_cast<int64_t>(chunk) * a.pitch + e];
        }
    } else {
        for (int e = t; e < a.experts; e += kRouteMost) count[e] = before[e] = 0;
        __syncthreads();
        const int quads = a.pitch / 4, parts = kRouteMost / quads;         // (pitch: a power of two)
        const int q = t & (quads - 1);
        v4i all = {0, 0, 0, 0}, own = {0, 0, 0, 0};
        constexpr int U = 8;           // loads in flight
        for (int c0 = t / quads; c0 < a.chunks; c0 += parts * U) {
            v4i n[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * parts;
                n[u] = v4i{0, 0, 0, 0};
                if (c < a.chunks) n[u] = *reinterpret_cast<const v4i*>(a.counts + static_cast<int64_t>(c) * a.pitch + q * 4);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                all += n[u];
                if (c0 + u * parts < chunk) own += n[u];
            }
        }
        // lanes of a wave with the same experts add up first
        for (int d = quads; d < 64; d <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                all[i] += __shfl_xor(all[i], d, 64);
                own[i] += __shfl_xor(own[i], d, 64);
            }
        if ((t & 63) < quads)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (q * 4 + i < a.experts) {
                    if (all[i]) atomicAdd(count + q * 4 + i, all[i]);      // (whole numbers: no order)
                    if (own[i]) atomicAdd(before + q * 4 + i, own[i]);
                }
    }
    __syncthreads();
    const int total = first_rows<kRouteMost>(count, first, a.experts, lds);
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = t; e < a.experts; e += kRouteMost) a.offsets[e] = first[e];
        if (t == 0) a.offsets[a.experts] = total;
    }
    for (int e = t; e < a.experts; e += kRouteMost) before[e] += first[e];
    __syncthreads();
    for (int i = t; i < tokens * k; i += kRouteMost) {
        const int64_t o = t0 * k + i;
        const int e = i == t ? my_expert : a.expert[o];
        if (e >= 0) {
            const int s = before[e] + (i == t ? my_rank : a.slot[o]);
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
// Bytes only: 32768 x 256 bf16 7.8 us (17 MB written and nearly as many read: eight chosen entries touch 3.6 of a row's 4 lines of 128 bytes), softmax over all
// 13.5 (an exponential each).
template <int L, int V, int R, bool BF16>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(const RouteArgs a) {
    constexpr int PER = kRouteThreads / L;
    __shared__ __align__(16) float rows[PER * L * V];
    const int t = static_cast<int>(threadIdx.x), l = t % L, k = a.top_k;
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
        load_logits<L, V, R, BF16>(a.logits, at, a.experts, l, lx);
#pragma unroll
        for (int v = 0; v < V; ++v) {
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
        d = q * (g - inner);
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
    // the chosen entries' values over the others', through LDS (in registers every choice would be compared with every entry)
    float* const row = rows + (t / L) * (L * V);
#pragma unroll
    for (int b = 0; b < V; b += R)
#pragma unroll
        for (int i = 0; i < R; ++i) row[entry_of<L, R>(l, b + i)] = lx[b + i];
    __syncthreads();
    if (mine >= 0) row[mine] = d;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < V; b += R)
#pragma unroll
        for (int i = 0; i < R; ++i) lx[b + i] = row[entry_of<L, R>(l, b + i)];
    if (!in) return;
#pragma unroll
    for (int b = 0; b < V; b += R) {
        const int e = entry_of<L, R>(l, b);
        if (e >= a.experts) continue;
        const int64_t o = token * a.experts + e;
        if constexpr (!BF16) {
            float* const p = static_cast<float*>(a.dlogits) + o;
            if constexpr (R == 4) *reinterpret_cast<v4f*>(p) = v4f{lx[b], lx[b + 1], lx[b + 2], lx[b + 3]};
            else *p = lx[b];
        } else {
            uint16_t* const p = static_cast<uint16_t*>(a.dlogits) + o;
            if constexpr (R == 8)
                *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(lx[b], lx[b + 1]), pack_bf16x2(lx[b + 2], lx[b + 3]), pack_bf16x2(lx[b + 4], lx[b + 5]), pack_bf16x2(lx[b + 6], lx[b + 7])};
            else if constexpr (R == 4) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(lx[b], lx[b + 1]), pack_bf16x2(lx[b + 2], lx[b + 3])};
            else *p = static_cast<uint16_t>(f32_to_bf16_rne(lx[b]));
        }
    }
}

static int route_pitch(int experts) {
    int p = 4;
    while (p < experts) p *= 2;
    return p;
}
// Tokens of a workgroup: all of a small call's (one launch: 64 tokens of 64 experts, 8 choices, 5.3 us, in two launches 7.2), else as few as leave
// 256 workgroups, each of which adds up the counts of all (300 tokens of 160 experts, 6 choices, 8.2 us with 16 of a workgroup, 12.8 with 128;
// 32768 of 256, 8 choices, 34.8 with 16, 19.9 with 128).
static int64_t route_chunk(const loka_route_desc* d) {
    if (d->tokens <= 64) return 64;
    int64_t c = 16;
    while (c < kRouteMostChunk && d->tokens > 256 * c) c *= 2;
    return c;
}
size_t route_workspace_bytes(const loka_route_desc* d) {
    const int64_t c = route_chunk(d), chunks = (d->tokens + c - 1) / c;
    return chunks > 1 ? static_cast<size_t>(chunks + 1) * static_cast<size_t>(route_pitch(d->experts)) * 4 : 0;
}

// Lanes, logits a lane and their runs: by the number of experts, and in runs of 16 bytes (8 where a lane has four bf16) where rows are whole runs.
// 16 lanes a token keep its exchanges inside the vector unit's rows and share a wave among four tokens (32768 x 256, 8 choices, 19.7 us; 32 lanes
// 23.7, 64 lanes 32.8); more than 256 logits are too many for them (32768 x 512 on 64 lanes 39.9 us and the gradient of a softmax over all 25.3, on 32
// 39.9 and 35.0).
template <class F>
static void by_experts(const loka_route_desc* d, const void* logits, const void* dlogits, F&& f) {
    auto with = [&](auto l, auto v) {
        auto typed = [&](auto bf16) {
            constexpr int run = bf16.value ? (v.value < 8 ? v.value : 8) : 4;
            if (d->experts % run == 0 && d->ld % run == 0 && aligned16(logits) && aligned16(dlogits)) f(l, v, std::integral_constant<int, run>{}, bf16);
            else f(l, v, std::integral_constant<int, 1>{}, bf16);
        };
        if (d->bf16) typed(std::true_type{});
        else typed(std::false_type{});
    };
    using std::integral_constant;
    if (d->experts <= 64) with(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (d->experts <= 128) with(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (d->experts <= 256) with(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else if (d->experts <= 512) with(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else with(integral_constant<int, 64>{}, integral_constant<int, 16>{});
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
    a.chunk_tokens = static_cast<int>(route_chunk(d));
    a.chunks = static_cast<int>((d->tokens + a.chunk_tokens - 1) / a.chunk_tokens);
    a.pitch = route_pitch(d->experts);
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
    by_experts(d, logits, nullptr, [&](auto l, auto v, auto r, auto bf16) {
        if (std::min<int64_t>(a.chunk_tokens, d->tokens) * l.value <= kRouteThreads) route_choose_kernel<l.value, v.value, r.value, bf16.value, kRouteThreads><<<a.chunks, kRouteThreads, lds, stream>>>(a);
        else route_choose_kernel<l.value, v.value, r.value, bf16.value, kRouteMost><<<a.chunks, kRouteMost, lds, stream>>>(a);
    });
    LOKA_HIP_TRY(hipGetLastError());
    if (a.chunks == 1) return LOKA_OK;
    const size_t place = static_cast<size_t>(d->experts) * 12 + 64;
    // A workgroup adds up every chunk's counts, chunks^2 in all, where that takes no longer than a launch that does it once (32768 x 64, 8
    // choices, 13.6 us, with the launch 14.1; 65536 x 256 37.6 and 32.7)
    if (a.chunks <= 256) {
        route_place_kernel<false><<<a.chunks, kRouteMost, place, stream>>>(a);
    } else {
        route_scan_kernel<<<d->experts, kRouteThreads, 0, stream>>>(a);
        LOKA_HIP_TRY(hipGetLastError());
        route_place_kernel<true><<<a.chunks, kRouteMost, place, stream>>>(a);
    }
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

loka_status route_backward_launch(const loka_route_desc* d, const void* logits, const int32_t* expert, const float* dweight, void* dlogits,
                                  hipStream_t stream) {
    RouteArgs a = args_of(d, logits);
    a.expert = const_cast<int32_t*>(expert);
    a.dweight = dweight;
    a.dlogits = dlogits;
    by_experts(d, logits, dlogits, [&](auto l, auto v, auto r, auto bf16) {
        const uint32_t grid = static_cast<uint32_t>((d->tokens * l.value + kRouteThreads - 1) / kRouteThreads);
        route_backward_kernel<l.value, v.value, r.value, bf16.value><<<grid, kRouteThreads, 0, stream>>>(a);
    });
    LOKA_HIP_TRY(hipGetLastError());
    return LOKA_OK;
}

// ---------------------------------------------------------------------------------
// The sum of a token's results, and its gradients.  A lane takes 8 columns of a token; bytes only, so a token's rows (K of them at
// most) are all requested before the first is used.  Tokens of more than 256 columns: a wave takes 512 of them, and its token's slots and weights are
// scalars; narrower ones share a wave, 2^lg lanes each.  16384 tokens x 4 choices x 4096: 135 .. 138 us (805 MB, 5.9 TB/s), backward 233 .. 239 (1.2 GB, 5.1 TB/s).
struct CombineArgs {
    const uint16_t *y, *residual, *dout;
    const int32_t* slot;
    const float* weight;
    uint16_t *out, *dy;
    float* dweight;
    int64_t tokens, cols, rows, first_wg;
    int segments;                      // of 512 columns of a token
    int top_k, lg;
};

// Eight columns from c on; a row may start anywhere
template <bool STREAMED>
__device__ __forceinline__ void store8(uint16_t* row, int64_t c, int64_t cols, u32x4 v) {
    if (c + 8 <= cols) {
        if (STREAMED) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(row + c));
        else *reinterpret_cast<u32x4_any*>(row + c) = v;
        return;
    }
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
// Eight columns of a row from c on, zeros behind the last: whole runs by one load, from the row's last eight where the row's end cuts
template <bool STREAMED>
__device__ __forceinline__ u32x4 load8(const uint16_t* row, int64_t c, int64_t cols) {
    if (c + 8 <= cols) {
        if (STREAMED) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + c));
        return *reinterpret_cast<const u32x4_any*>(row + c);
    }
    return mx_load8(row, c, cols);
}

// Slots (-1: none) and weights of token t
template <int K, bool WAVE>
__device__ __forceinline__ void choices(const CombineArgs& a, int64_t t, int64_t (&slot)[K], float (&w)[K]) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
        int s = -1;
        float f = 0.f;
        if (j < a.top_k) {
            s = a.slot[t * a.top_k + j];
            f = a.weight ? a.weight[t * a.top_k + j] : 1.f;
        }
        if (WAVE) s = __builtin_amdgcn_readfirstlane(s);
        slot[j] = s < 0 || s >= a.rows ? -1 : s;
        w[j] = f;
    }
}
template <bool WAVE>
__device__ __forceinline__ int64_t my_token(const CombineArgs& a, int64_t& c) {
    const int64_t wg = a.first_wg + blockIdx.x;
    if (!WAVE) {
        c = (static_cast<int>(threadIdx.x) & ((1 << a.lg) - 1)) * 8;
        return (wg * 256 + threadIdx.x) >> a.lg;
    }
    const int64_t unit = wg * 4 + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int64_t t = unit >> 32 ? unit / a.segments : static_cast<int64_t>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(a.segments));
    c = (unit - t * a.segments) * 512 + (threadIdx.x & 63) * 8;
    return t;
}

template <int K, bool WAVE, bool STREAMED>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
    int64_t c;
    const int64_t t = my_token<WAVE>(a, c);
    if (t >= a.tokens) return;
    int64_t slot[K];
    float w[K];
    choices<K, WAVE>(a, t, slot, w);
    if (c >= a.cols) return;
    u32x4 v[K], res = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < K; ++j) {
        v[j] = u32x4{0u, 0u, 0u, 0u};
        if (slot[j] >= 0) v[j] = load8<STREAMED>(a.y + slot[j] * a.cols, c, a.cols);
    }
    if (a.residual) res = load8<STREAMED>(a.residual + t * a.cols, c, a.cols);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, f[8];
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (slot[j] >= 0) {
            widen(v[j], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = fmaf(w[j], f[e], s[e]);
        }
    if (a.residual) {
        widen(res, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += f[e];
    }
    store8<false>(a.out + t * a.cols, c, a.cols, narrow(s));
}

// WAVE: a workgroup takes a token, 2048 columns at a time, so that its threads' parts of dweight meet in it; else 2^lg lanes do.
template <int K, bool WAVE, bool STREAMED>
__global__ __launch_bounds__(256) void combine_backward_kernel(const CombineArgs a) {
    __shared__ float part[4][K];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = WAVE ? a.first_wg + blockIdx.x : ((a.first_wg + blockIdx.x) * 256 + threadIdx.x) >> a.lg;
    const bool in = first < a.tokens;
    const int64_t t = in ? first : a.tokens - 1;
    int64_t slot[K];
    float w[K], sum[K];
    choices<K, WAVE>(a, t, slot, w);
#pragma unroll
    for (int j = 0; j < K; ++j) sum[j] = 0.f;
    const int64_t c0 = WAVE ? threadIdx.x * 8 : (threadIdx.x & ((1 << a.lg) - 1)) * 8;
    if (in)
        for (int64_t c = c0; c < a.cols; c += 2048) {
            u32x4 v[K];
            const u32x4 dv = load8<STREAMED>(a.dout + t * a.cols, c, a.cols);
            if (a.dweight)
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    v[j] = u32x4{0u, 0u, 0u, 0u};
                    if (slot[j] >= 0) v[j] = load8<STREAMED>(a.y + slot[j] * a.cols, c, a.cols);
                }
            float d[8], f[8];
            widen(dv, d);
            if (a.dy)
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (slot[j] >= 0) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = w[j] * d[e];
                        store8<STREAMED>(a.dy + slot[j] * a.cols, c, a.cols, narrow(f));
                    }
            if (a.dweight)
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    widen(v[j], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[j] = fmaf(d[e], f[e], sum[j]);
                }
        }
    if (!a.dweight) return;
    if (WAVE) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            sum[j] = lanes_sum<64>(sum[j]);
            if (lane == 0) part[wave][j] = sum[j];
        }
        __syncthreads();
        const int j = static_cast<int>(threadIdx.x);
        // (a dead choice has no row: its sum is of zeros, unless dout is not finite)
        if (j < a.top_k) {
            const int s = a.slot[t * a.top_k + j];
            a.dweight[t * a.top_k + j] = s < 0 || s >= a.rows ? 0.f : (part[0][j] + part[1][j]) + (part[2][j] + part[3][j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            for (int m = 1; m < (1 << a.lg); m <<= 1) sum[j] += __shfl_xor(sum[j], m, 64);
            if (in && j < a.top_k && (threadIdx.x & ((1 << a.lg) - 1)) == 0) a.dweight[t * a.top_k + j] = slot[j] < 0 ? 0.f : sum[j];
        }
    }
}

static CombineArgs args_of(const loka_combine_desc* d, const int32_t* slot, const float* weight) {
    CombineArgs a{};
    a.slot = slot;
    a.weight = weight;
    a.tokens = d->tokens;
    a.cols = d->cols;
    a.rows = d->rows;
    a.top_k = d->top_k;
    a.segments = static_cast<int>((d->cols + 511) / 512);
    while ((8 << a.lg) < d->cols) ++a.lg;
    return a;
}
// f(K, WAVE, STREAMED) for a call whose matrices of tokens * top_k rows have `cols` columns.  Results of 2^27 elements and more, which the 256 MB of last-level
// cache cannot hold, pass it by (8192 tokens x 4 x 4096: 67.7 us, else 78.6, backward 118 and 123; half the tokens: 35.0 and 30.4, backward 58 and 50).
template <class F>
static loka_status by_choices(const loka_combine_desc* d, F&& f) {
    using std::integral_constant;
    const bool streamed = d->tokens * d->top_k * d->cols >= INT64_C(1) << 27;
    auto with = [&](auto k) {
        if (d->cols <= 256) return f(k, std::false_type{}, std::false_type{});
        return streamed ? f(k, std::true_type{}, std::true_type{}) : f(k, std::true_type{}, std::false_type{});
    };
    if (d->top_k <= 1) return with(integral_constant<int, 1>{});
    if (d->top_k <= 2) return with(integral_constant<int, 2>{});
    if (d->top_k <= 4) return with(integral_constant<int, 4>{});
    if (d->top_k <= 8) return with(integral_constant<int, 8>{});
    return with(integral_constant<int, 16>{});
}

loka_status combine_launch(const loka_combine_desc* d, const void* y, const int32_t* slot, const float* weight, const void* residual,
                           void* out, hipStream_t stream) {
    CombineArgs a = args_of(d, slot, weight);
    a.y = static_cast<const uint16_t*>(y);
    a.residual = static_cast<const uint16_t*>(residual);
    a.out = static_cast<uint16_t*>(out);
    return by_choices(d, [&](auto k, auto wave, auto streamed) {
        const int64_t groups = wave.value ? (a.tokens * a.segments + 3) / 4 : ((a.tokens << a.lg) + 255) / 256;
        return in_launches(groups, 256, [&](int64_t from, uint32_t grid) {
            a.first_wg = from;
            combine_kernel<k.value, wave.value, streamed.value><<<grid, 256, 0, stream>>>(a);
        });
    });
}

loka_status combine_backward_launch(const loka_combine_desc* d, const void* dout, const void* y, const int32_t* slot, const float* weight,
                                    void* dy, float* dweight, hipStream_t stream) {
    CombineArgs a = args_of(d, slot, weight);
    a.dout = static_cast<const uint16_t*>(dout);
    a.y = static_cast<const uint16_t*>(y);
    a.dy = static_cast<uint16_t*>(dy);
    a.dweight = dweight;
    return by_choices(d, [&](auto k, auto wave, auto streamed) {
        const int64_t groups = wave.value ? a.tokens : ((a.tokens << a.lg) + 255) / 256;
        return in_launches(groups, 256, [&](int64_t from, uint32_t grid) {
            a.first_wg = from;
            combine_backward_kernel<k.value, wave.value, streamed.value><<<grid, 256, 0, stream>>>(a);
        });
    });
}

}  // namespace loka
