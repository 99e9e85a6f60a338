// Routing: the choice of experts and their weights, the experts' order, the rows' way there and back.
// One pass over each array, no floating-point atomics, and every sum in an order that does not depend on timing.
// What bounds it, and measured: the choice by instruction issue (16384 tokens, 128 experts, top 8: choice and places 19 us,
// the gradient 6), a decoding step by its launches (16 tokens, 64 experts: 5.7 us), the exchange by HBM (8192 rows of 4096,
// top 2: there 32 us, 6.3 TB/s, back 37 us, 5.4 TB/s; 4096 rows of 1024, top 8, its gradient 26 us, 5.4 TB/s).
#pragma once
#include "half.cuh"
#include "ptx.cuh"

namespace nk {

struct RouteParams {
    int tokens, experts, topk, renormalise;
    int logits_type;            // 0 FP32, 1 BF16, 2 FP16
    long long ld_logits;
    const void* logits;
    float* gates;
    int* chosen;                // [tokens][topk]
    int* offsets;               // [experts + 1]
    int* slots;                 // [tokens][topk]
    int* counts;                // [blocks][experts]: pairs of a block of tokens, by expert
    int per_block;              // tokens of a block
};

// A token's logits: lane l holds experts l, l + 32, ...; `none` where there is no expert.
template <int V>
__device__ __forceinline__ void route_fetch(const RouteParams& p, int t, int lane, float none, float (&z)[V]) {
    const size_t o = static_cast<size_t>(t) * p.ld_logits + lane;
    if (p.logits_type == 0) {
        const float* x = static_cast<const float*>(p.logits) + o;
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = lane + 32 * i < p.experts ? x[32 * i] : none;
    } else {
        const uint16_t* x = static_cast<const uint16_t*>(p.logits) + o;
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = lane + 32 * i < p.experts ? half_bits_to_f32(x[32 * i], p.logits_type == 2) : none;
    }
}

// Unsigned key in the order of the numbers: both zeros alike, NaN below every number (1), 0 left for "taken".
__device__ __forceinline__ uint32_t route_key(float z) {
    if (z != z) return 1u;
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float route_unkey(uint32_t k) {
    return __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k);
}

// One warp, one token: lane l holds experts l, l + 32, ...  (V of them).  topk rounds of a warp-wide maximum of the
// keys and a minimum of the indices that have it.
template <int V>
__device__ __forceinline__ int route_token(const RouteParams& p, int t, int lane, const float (&z)[V]) {
    uint32_t key[V];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool there = lane + 32 * i < p.experts;
        nan |= there && z[i] != z[i];
        key[i] = there ? route_key(z[i]) : 0u;
    }
    nan = __any_sync(~0u, nan);
    uint32_t own_key = 0u;                     // lane j keeps choice j
    int own = 0;
    uint32_t first_key = 0u;
    uint32_t live[V];
#pragma unroll
    for (int i = 0; i < V; ++i) live[i] = key[i];
    for (int j = 0; j < p.topk; ++j) {
        uint32_t best = 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) best = max(best, live[i]);
        const uint32_t top = __reduce_max_sync(~0u, best);
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int i = V - 1; i >= 0; --i)
            if (live[i] == top) at = lane + 32 * i;
        const uint32_t e = __reduce_min_sync(~0u, at);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (static_cast<uint32_t>(lane + 32 * i) == e) live[i] = 0u;
        if (lane == j) { own_key = top; own = static_cast<int>(e); }
        if (j == 0) first_key = top;
    }
    // weights: exp(z - max) over the sum
    const float m = route_unkey(first_key);
    const float mine = lane < p.topk && own_key > 1u ? expf(route_unkey(own_key) - m) : 0.0f;
    float sum = 0.0f;
    if (p.renormalise) {
        sum = mine;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (key[i]) sum += expf(z[i] - m);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    if (lane < p.topk) {
        const size_t o = static_cast<size_t>(t) * p.topk + lane;
        const bool none = m == -INFINITY;      // nothing may be chosen
        p.gates[o] = nan ? __int_as_float(0x7FC00000) : none ? 0.0f : mine / sum;
        p.chosen[o] = own;
    }
    return own;
}

// exclusive scan of s[0..n) in place by the whole block (n <= 1024, at least 32 threads); returns the total
__device__ __forceinline__ int block_scan(int* s, int n, int* part) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int chunks = (n + 31) / 32;
    for (int c = warp; c < chunks; c += warps) {
        const int i = c * 32 + lane;
        const int x = i < n ? s[i] : 0;
        int v = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(~0u, v, d);
            if (lane >= d) v += o;
        }
        if (i < n) s[i] = v - x;
        if (lane == 31) part[c] = v;
    }
    __syncthreads();
    if (warp == 0) {
        const int x = lane < chunks ? part[lane] : 0;
        int v = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(~0u, v, d);
            if (lane >= d) v += o;
        }
        if (lane < chunks) part[lane] = v - x;
        if (lane == 31) part[32] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) s[i] += part[i >> 5];
    __syncthreads();
    return part[32];
}

// The places of the tokens [t0, t1) of one block: `base[e]` is the place of its first pair of expert e.  Each warp
// has a contiguous run of tokens and a row of counts; after a scan over the warps it walks its tokens in order.
__device__ __forceinline__ void route_places(const RouteParams& p, int t0, int t1, const int* base, int* rows) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int E = p.experts, run = (t1 - t0 + warps - 1) / warps;
    const int lo = min(t1, t0 + warp * run), hi = min(t1, lo + run);
    int* mine = rows + warp * E;
    for (int e = lane; e < E; e += 32) mine[e] = 0;
    __syncwarp();
    for (int i = lo * p.topk + lane; i < hi * p.topk; i += 32) atomicAdd(mine + p.chosen[i], 1);
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        int at = base[e];
        for (int w = 0; w < warps; ++w) {
            const int n = rows[w * E + e];
            rows[w * E + e] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int t = lo; t < hi; t += 4) {             // four tokens' choices on the way at a time
        const size_t o = static_cast<size_t>(t) * p.topk + lane;
        int e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = lane < p.topk && t + i < hi ? p.chosen[o + i * p.topk] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (e[i] >= 0) p.slots[o + i * p.topk] = mine[e[i]]++;      // a token's experts are distinct
            __syncwarp();
        }
    }
}

constexpr int ROUTE_THREADS = 1024;                // of both kernels; a lane of route_select_kernel that holds 16 experts or more
                                                   // needs the registers of 512
__host__ __device__ constexpr int route_threads(int v) { return v >= 16 ? 512 : ROUTE_THREADS; }
constexpr int ROUTE_ONE_BLOCK = 64;                // up to this many tokens one block does everything
__host__ __device__ constexpr int route_smem(int experts) { return (ROUTE_THREADS / 32 * experts + 2 * experts + 64) * 4; }

// A block of tokens: choices, weights, and the block's counts by expert.  ONE: the only block; it goes on to the places.
template <int V, bool ONE>
__global__ void __launch_bounds__(route_threads(V)) route_select_kernel(const RouteParams p) {
    constexpr int THREADS = route_threads(V), WARPS = THREADS / 32;
    extern __shared__ int route_sm[];
    int* hist = route_sm;                          // [experts]
    int* part = hist + p.experts;                  // [64]
    int* rows = part + 64;                         // [warps][experts] (ONE)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t0 = blockIdx.x * p.per_block, t1 = min(p.tokens, t0 + p.per_block);
    for (int e = threadIdx.x; e < p.experts; e += THREADS) hist[e] = 0;
    launch_wait();
    launch_next();
    __syncthreads();
    // the next token's logits are on the way while one is worked on
    float z[V];
    if (t0 + warp < t1) route_fetch<V>(p, t0 + warp, lane, 0.0f, z);
    for (int t = t0 + warp; t < t1; t += WARPS) {
        float now[V];
#pragma unroll
        for (int i = 0; i < V; ++i) now[i] = z[i];
        if (t + WARPS < t1) route_fetch<V>(p, t + WARPS, lane, 0.0f, z);
        const int e = route_token<V>(p, t, lane, now);
        if (lane < p.topk) atomicAdd(hist + e, 1);
    }
    __syncthreads();
    if (ONE) {
        const int total = block_scan(hist, p.experts, part);
        for (int e = threadIdx.x; e < p.experts; e += THREADS) p.offsets[e] = hist[e];
        if (threadIdx.x == 0) p.offsets[p.experts] = total;
        route_places(p, t0, t1, hist, rows);
    } else {
        for (int e = threadIdx.x; e < p.experts; e += THREADS) p.counts[static_cast<size_t>(blockIdx.x) * p.experts + e] = hist[e];
    }
}

// The places of a block's pairs from every block's counts: the pairs of lower experts, then those of earlier blocks.
__global__ void __launch_bounds__(ROUTE_THREADS) route_place_kernel(const RouteParams p) {
    extern __shared__ int route_sm[];
    int* total = route_sm;                         // [experts]
    int* part = total + p.experts;                 // [64]
    int* rows = part + 64;                         // [warps][experts]
    int* before = rows + ROUTE_THREADS / 32 * p.experts;   // [experts]
    const int blocks = gridDim.x, E = p.experts;
    for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) total[e] = before[e] = 0;
    launch_wait();
    launch_next();
    __syncthreads();
    // threads of a row of counts side by side, rows dealt out over what threads are left (integer sums: any order)
    const int lanes = min(E, ROUTE_THREADS), rowsets = ROUTE_THREADS / lanes;
    const int set = threadIdx.x / lanes;
    if (set < rowsets) {
        for (int e = threadIdx.x - set * lanes; e < E; e += lanes) {
            int all = 0, early = 0;
#pragma unroll 8
            for (int b = set; b < blocks; b += rowsets) {
                const int n = p.counts[static_cast<size_t>(b) * E + e];
                all += n;
                if (b < static_cast<int>(blockIdx.x)) early += n;
            }
            atomicAdd(total + e, all);
            atomicAdd(before + e, early);
        }
    }
    __syncthreads();
    const int sum = block_scan(total, E, part);
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) p.offsets[e] = total[e];
        if (threadIdx.x == 0) p.offsets[E] = sum;
    }
    for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) total[e] += before[e];
    __syncthreads();
    const int t0 = blockIdx.x * p.per_block, t1 = min(p.tokens, t0 + p.per_block);
    route_places(p, t0, t1, total, rows);
}

// dz_e = p_e (d_e - sum_j d_j g_j): one warp per token, the row's softmax taken again (cheaper than keeping it)
template <int V>
__global__ void __launch_bounds__(256) route_backward_kernel(const RouteParams p, const float* dgates, float* dlogits) {
    const int lane = threadIdx.x & 31;
    const int t = blockIdx.x * 8 + (threadIdx.x >> 5);
    launch_wait();
    launch_next();
    if (t >= p.tokens) return;
    // the chosen experts' gradients by way of shared memory: a row of (gradient, 1) by expert for each warp
    extern __shared__ float2 route_d[];
    float2* row = route_d + (threadIdx.x >> 5) * (32 * V);
    const size_t o = static_cast<size_t>(t) * p.topk;
    const int own = lane < p.topk ? p.chosen[o + lane] : -1;
    const float own_d = lane < p.topk ? dgates[o + lane] : 0.0f;
    float z[V], d[V];
    route_fetch<V>(p, t, lane, -INFINITY, z);
#pragma unroll
    for (int i = 0; i < V; ++i) row[lane + 32 * i] = make_float2(0.0f, 0.0f);
    __syncwarp();
    if (own >= 0 && own < p.experts) row[own] = make_float2(own_d, 1.0f);
    __syncwarp();
    uint32_t top = 0u, taken = 0u;                 // taken, bit i: this lane's expert i is one of the chosen
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 x = row[lane + 32 * i];
        d[i] = x.x;
        taken |= x.y != 0.0f ? 1u << i : 0u;
        nan |= z[i] != z[i];
        top = max(top, route_key(z[i]));
    }
    nan = __any_sync(~0u, nan);
    const float m = route_unkey(__reduce_max_sync(~0u, top));
    float sum = 0.0f, inner = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool in = !p.renormalise || ((taken >> i) & 1u);
        z[i] = in ? expf(z[i] - m) : 0.0f;
        sum += z[i];
        inner += z[i] * d[i];
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, s);
        inner += __shfl_xor_sync(~0u, inner, s);
    }
    const bool none = m == -INFINITY && !nan;
    const float inv = 1.0f / sum;
    inner *= inv;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        if (e < p.experts) {
            float x = z[i] * inv * (d[i] - inner);
            if (p.renormalise && !((taken >> i) & 1u)) x = 0.0f;
            dlogits[static_cast<size_t>(t) * p.experts + e] = nan ? __int_as_float(0x7FC00000) : none ? 0.0f : x;
        }
    }
}

// ---------------------------------------------------------------- rows to their experts' order and back
struct ExchangeParams {
    int tokens, topk, vecs;     // vecs: 16-byte pieces of a row
    int lanes_log2;             // threads to a row of dispatch and combine
    long long ld_tokens, ld_slots;   // in 16-byte pieces
    const int* slots;
    const float* gates;
};

template <bool F16>
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = half_bits_to_f32(w[i] & 0xFFFFu, F16);
        x[2 * i + 1] = half_bits_to_f32(w[i] >> 16, F16);
    }
}
template <bool F16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_half2(x[0], x[1], F16), pack_half2(x[2], x[3], F16), pack_half2(x[4], x[5], F16), pack_half2(x[6], x[7], F16));
}

// A block of 256 threads has the rows of 256 >> p.lanes_log2 tokens, 1 << p.lanes_log2 threads to a row.  (One index over all
// pieces of all rows and a division by a row's pieces cost as many instructions as the sum itself.)
__device__ __forceinline__ int exchange_token(const ExchangeParams& p) {
    return blockIdx.x * (256 >> p.lanes_log2) + (threadIdx.x >> p.lanes_log2);
}

// a thread reads four pieces of a token's row and writes them to the topk places
__global__ void __launch_bounds__(256) dispatch_kernel(const ExchangeParams p, const uint4* x, uint4* xs) {
    const int t = exchange_token(p), lanes = 1 << p.lanes_log2;
    launch_wait();
    launch_next();
    if (t >= p.tokens) return;
    const int* slots = p.slots + static_cast<size_t>(t) * p.topk;
    const unsigned pairs = static_cast<unsigned>(p.tokens) * p.topk;
    x += t * p.ld_tokens;
    for (int v = threadIdx.x & (lanes - 1); v < p.vecs; v += 4 * lanes) {
        uint4 piece[4];
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (v + n * lanes < p.vecs) piece[n] = __ldcs(x + v + n * lanes);
        for (int j = 0; j < p.topk; ++j) {
            const unsigned s = __ldg(slots + j);
            if (s >= pairs) continue;
            uint4* row = xs + s * p.ld_slots + v;
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (v + n * lanes < p.vecs) row[n * lanes] = piece[n];
        }
    }
}

// a thread adds four pieces of the topk rows of a token
template <bool F16>
__global__ void __launch_bounds__(256) combine_kernel(const ExchangeParams p, const uint4* ys, uint4* y) {
    const int t = exchange_token(p), lanes = 1 << p.lanes_log2;
    launch_wait();
    launch_next();
    if (t >= p.tokens) return;
    const int* slots = p.slots + static_cast<size_t>(t) * p.topk;
    const float* gates = p.gates ? p.gates + static_cast<size_t>(t) * p.topk : nullptr;
    const unsigned pairs = static_cast<unsigned>(p.tokens) * p.topk;
    y += t * p.ld_tokens;
    // four pieces of a row at a time: where the rows are is known only after the slots have come, and then every load
    // that can be on the way has to be
    for (int v = threadIdx.x & (lanes - 1); v < p.vecs; v += 4 * lanes) {
        float sum[4][8];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[n][q] = 0.0f;
#pragma unroll 2
        for (int j = 0; j < p.topk; ++j) {
            const unsigned s = __ldg(slots + j);
            if (s >= pairs) continue;
            const float g = gates ? __ldg(gates + j) : 1.0f;
            const uint4* row = ys + s * p.ld_slots + v;
            uint4 piece[4];
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (v + n * lanes < p.vecs) piece[n] = __ldcs(row + n * lanes);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                float r[8];
                unpack8<F16>(piece[n], r);
#pragma unroll
                for (int q = 0; q < 8; ++q) sum[n][q] += g * r[q];
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (v + n * lanes < p.vecs) y[v + n * lanes] = pack8<F16>(sum[n]);
    }
}

// a warp per (token, j): the pair's row of dYs, and the product of two rows for its dgates
template <bool F16>
__global__ void __launch_bounds__(256) combine_backward_kernel(const ExchangeParams p, const uint4* dy, const uint4* ys, uint4* dys, float* dgates) {
    const int lane = threadIdx.x & 31;
    const unsigned pairs = static_cast<unsigned>(p.tokens) * p.topk;
    const unsigned i = blockIdx.x * 8u + (threadIdx.x >> 5);
    launch_wait();
    launch_next();
    if (i >= pairs) return;
    const unsigned t = i / static_cast<unsigned>(p.topk), s = p.slots[i];
    if (s >= pairs) {
        if (lane == 0) dgates[i] = 0.0f;
        return;
    }
    const float g = p.gates[i];
    dy += t * p.ld_tokens;
    ys += s * p.ld_slots;
    dys += s * p.ld_slots;
    float dot = 0.0f;
#pragma unroll 4
    for (int v = lane; v < p.vecs; v += 32) {
        float a[8], b[8];
        unpack8<F16>(dy[v], a);
        unpack8<F16>(ys[v], b);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            dot += a[q] * b[q];
            a[q] *= g;
        }
        dys[v] = pack8<F16>(a);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(~0u, dot, d);
    if (lane == 0) dgates[i] = dot;
}

}  // namespace nk
