// The balance of a router's loads: how many rows each expert got, its mean probability, the two losses made of them and
// their gradient.  Over the n tokens that count (mask), with c_e the choices of expert e and p_te the softmax of a row:
//   P_e = 1/n sum_t p_te,  balance = E / (n k) sum_e c_e P_e,  size = 1/n sum_t lse_t^2,  lse_t = log sum_e exp z_te
//   dz_te = p_te (g0 E / (n^2 k) (c_e - sum_j c_j p_tj) + g1 2/n lse_t)
// A warp has a token, a lane the experts l, l + 32, ..., and adds up the probabilities of its tokens in registers: one pass
// over the logits each way.  Sums of at most 64 tokens, of a block's warps and of the experts are FP32, those over blocks 64
// bits; every sum has one order (counts are integers, added in any).
// Bound by instruction issue (65 to 74 % of the slots) and by each launch's start and end: 16384 x 128 FP32 logits, 8.4 MB or 1.3 us of
// HBM, take 8.6 us (two launches), the way back (8.4 MB more) 5.8; 16 x 64 take 3.4 (one launch) and 2.2.
#pragma once
#include "route.cuh"

namespace nk {

struct BalanceParams {
    const uint8_t* mask;        // [tokens], 0: the token does not count; null: all do
    int* counts;                // [experts + 1]; the last: tokens that count
    float* share;               // [experts]
    float* losses;              // [2]
    float* partial;             // [blocks][2 experts + 2]: sums of probabilities, counts, sum of lse^2, tokens
    int blocks, per_block;
};
constexpr int BALANCE_RUN = 64;                    // tokens of a warp at most

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

// the largest of a warp's numbers, NaN if there is one
__device__ __forceinline__ float warp_max_nan(float x) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// A row's softmax in place: z becomes the probabilities; returns the row's log-sum-exp.  A row whose logits are all minus
// infinity has neither: zeros.
template <int V>
__device__ __forceinline__ float row_softmax(float (&z)[V]) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(z[i]));
    m = warp_max_nan(m);
    if (!(m > -INFINITY)) {
        const float x = m != m ? m : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = x;
        return x;
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        z[i] = expf(z[i] - m);
        sum += z[i];
    }
    sum = warp_sum(sum);
    const float inv = 1.0f / sum;
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] *= inv;
    return m + logf(sum);
}

// The losses from sums and counts in shared memory (experts of them), by the whole block; `part`: 32 doubles.
__device__ __forceinline__ void balance_finish(const RouteParams& p, const BalanceParams& b, const double* sum, const int* count, double size,
                                               int tokens, double* part) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const double n = tokens;
    double loss = 0.0;
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
        const double s = tokens ? sum[e] / n : 0.0;
        b.share[e] = static_cast<float>(s);
        b.counts[e] = count[e];
        loss += s * count[e];
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) loss += __shfl_xor_sync(~0u, loss, d);
    if (lane == 0) part[warp] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < warps; ++w) loss += part[w];
        b.losses[0] = tokens ? static_cast<float>(loss * p.experts / (n * p.topk)) : 0.0f;
        b.losses[1] = tokens ? static_cast<float>(size / n) : 0.0f;
        b.counts[p.experts] = tokens;
    }
}

// shared memory of balance_kernel: a row of probabilities for each warp, then sums, counts, the warps' two numbers
__host__ __device__ constexpr int balance_smem(int v) { return route_threads(v) / 32 * (32 * v * 4 + 8) + 32 * v * (8 + 4) + 32 * 8 + 16; }

template <int V, bool ONE>
__global__ void __launch_bounds__(route_threads(V)) balance_kernel(const RouteParams p, const BalanceParams b) {
    constexpr int THREADS = route_threads(V), WARPS = THREADS / 32;
    extern __shared__ double balance_sm[];
    double* total = balance_sm;                                  // [32 V]
    double* part = total + 32 * V;                               // [32]
    float* rows = reinterpret_cast<float*>(part + 32);           // [WARPS][32 V]
    int* hist = reinterpret_cast<int*>(rows + WARPS * 32 * V);   // [32 V]
    float* sizes = reinterpret_cast<float*>(hist + 32 * V);      // [WARPS]
    int* alive = reinterpret_cast<int*>(sizes + WARPS);          // [WARPS]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = p.experts;
    const int t0 = blockIdx.x * b.per_block, t1 = min(p.tokens, t0 + b.per_block);
    for (int e = threadIdx.x; e < E; e += THREADS) hist[e] = 0;
    launch_wait();
    launch_next();
    __syncthreads();
    float acc[V], size = 0.0f;
    int n = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    for (int t = t0 + warp; t < t1; t += WARPS) {
        if (b.mask && !b.mask[t]) continue;
        float z[V];
        route_fetch<V>(p, t, lane, -INFINITY, z);
        const int e = lane < p.topk ? p.chosen[static_cast<size_t>(t) * p.topk + lane] : -1;
        const float lse = row_softmax<V>(z);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += z[i];
        size += lse * lse;
        ++n;
        if (e >= 0 && e < E) atomicAdd(hist + e, 1);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) rows[warp * 32 * V + lane + 32 * i] = acc[i];
    if (lane == 0) { sizes[warp] = size; alive[warp] = n; }
    __syncthreads();
    if (ONE) {
        for (int e = threadIdx.x; e < E; e += THREADS) {
            double s = 0.0;
            for (int w = 0; w < WARPS; ++w) s += rows[w * 32 * V + e];
            total[e] = s;
        }
        double s = 0.0;
        int m = 0;
        if (threadIdx.x == 0)
            for (int w = 0; w < WARPS; ++w) { s += sizes[w]; m += alive[w]; }
        if (threadIdx.x == 0) alive[0] = m;
        __syncthreads();
        balance_finish(p, b, total, hist, s, alive[0], part);
    } else {
        float* out = b.partial + static_cast<size_t>(blockIdx.x) * (2 * E + 2);
        for (int e = threadIdx.x; e < E; e += THREADS) {
            float s = 0.0f;
            for (int w = 0; w < WARPS; ++w) s += rows[w * 32 * V + e];
            out[e] = s;
            out[E + e] = __int_as_float(hist[e]);
        }
        if (threadIdx.x == 0) {
            float s = 0.0f;
            int m = 0;
            for (int w = 0; w < WARPS; ++w) { s += sizes[w]; m += alive[w]; }
            out[2 * E] = s;
            out[2 * E + 1] = __int_as_float(m);
        }
    }
}

// The blocks' sums into the results: a cluster of eight, each an eighth of the experts, 2^narrow of them to a row of a warp's lanes; a warp of its
// own has the tokens.  (Short code: it runs once, and what it costs is mostly its fetch.  By one block, or with 64-bit divisions, 5 to 7 us; ten
// loads ahead instead of five 0.5 us more, the tokens' sums in front of the experts' 1.4.)
constexpr int BALANCE_CLUSTER = 8, BALANCE_TOTAL = 512;
__global__ void __launch_bounds__(BALANCE_TOTAL) __cluster_dims__(BALANCE_CLUSTER, 1, 1)
balance_total_kernel(const RouteParams p, const BalanceParams b, int narrow) {
    constexpr int WARPS = BALANCE_TOTAL / 32 - 1, AHEAD = 5;               // warps of the experts; the last has the tokens
    __shared__ double part[WARPS][32];
    __shared__ int count[WARPS][32], all;
    __shared__ __align__(16) float4 losses[BALANCE_CLUSTER];               // of the first block: everyone's part
    const int E = p.experts, rank = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int each = (E + BALANCE_CLUSTER - 1) / BALANCE_CLUSTER, first = rank * each, last = min(E, first + each);
    const int at = lane & ((1 << narrow) - 1), row = (warp << (5 - narrow)) + (lane >> narrow), rows = WARPS << (5 - narrow);
    const size_t pitch = 2 * E + 2;
    double s, size = 0.0;
    int c;
    // a column's sums (in s and c) of the blocks `from`, from + by, ..: numbers and, `gap` further on, counts
    auto add = [&](const float* x, int from, int by, int gap) {
        for (int i = from; i < b.blocks; i += AHEAD * by) {
            float v[AHEAD];
            int n[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const float* y = x + (i + j * by) * pitch;
                v[j] = i + j * by < b.blocks ? y[0] : 0.0f;
                n[j] = i + j * by < b.blocks ? __float_as_int(y[gap]) : 0;
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                s += v[j];
                c += n[j];
            }
        }
    };
    cluster_arrive();                                                      // everyone has started, once this is waited for: the stores below need it
    launch_wait();
    launch_next();
    if (warp == WARPS) {
        s = 0.0;
        c = 0;
        add(b.partial + 2 * E, lane, 32, 1);
        c = static_cast<int>(__reduce_add_sync(~0u, static_cast<unsigned>(c)));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
        size = s;
        if (lane == 0) all = c;
    }
    float loss = 0.0f;
    for (int e0 = first; e0 < last; e0 += 1 << narrow) {
        const int e = e0 + at;
        s = 0.0;
        c = 0;
        if (warp < WARPS && e < last) add(b.partial + e, row, rows, E);
        if (e0 > first) __syncthreads();
        if (warp < WARPS) {
            part[warp][lane] = s;
            count[warp][lane] = c;
        }
        __syncthreads();
        if (warp == 0) {
            s = 0.0;
            c = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                s += part[w][lane];
                c += count[w][lane];
            }
            for (int d = 16; d >= 1 << narrow; d >>= 1) {
                s += __shfl_xor_sync(~0u, s, d);
                c += __shfl_xor_sync(~0u, c, d);
            }
            if (e < last && lane >> narrow == 0) {
                const float mean = all ? static_cast<float>(s) / static_cast<float>(all) : 0.0f;
                b.share[e] = mean;
                b.counts[e] = c;
                loss += mean * static_cast<float>(c);
            }
        }
    }
    cluster_wait();
    if (warp == 0) {
        loss = warp_sum(loss);
        if (lane == 0) st_cluster_v4(map_to_cta(smem_u32(losses + rank), 0), __float_as_uint(loss), 0u, 0u, 0u);
    }
    cluster_sync_all();
    if (rank == 0 && threadIdx.x == WARPS * 32) {
        loss = 0.0f;
        for (int r = 0; r < BALANCE_CLUSTER; ++r) loss += losses[r].x;
        const float tokens = static_cast<float>(all);
        b.losses[0] = all ? loss / tokens * (static_cast<float>(E) / static_cast<float>(p.topk)) : 0.0f;
        b.losses[1] = all ? static_cast<float>(size) / tokens : 0.0f;
        b.counts[E] = all;
    }
}

// One warp per token.  The counts are taken from their mean, which changes nothing (the probabilities of a row add up to 1)
// but leaves the differences of even loads their digits.
template <int V>
__global__ void __launch_bounds__(256) balance_backward_kernel(const RouteParams p, const BalanceParams b, const float* dlosses, float* dlogits, int accumulate) {
    const int lane = threadIdx.x & 31;
    const int t = blockIdx.x * 8 + (threadIdx.x >> 5);
    launch_wait();
    launch_next();
    if (t >= p.tokens) return;
    float* out = dlogits + static_cast<size_t>(t) * p.experts;
    if (b.mask && !b.mask[t]) {
        if (!accumulate)
            for (int e = lane; e < p.experts; e += 32) out[e] = 0.0f;
        return;
    }
    float z[V];
    route_fetch<V>(p, t, lane, -INFINITY, z);
    const int n = b.counts[p.experts];
    const int mean = static_cast<int>(static_cast<long long>(n) * p.topk / p.experts);
    const float lse = row_softmax<V>(z);
    float c[V], inner = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        c[i] = e < p.experts ? static_cast<float>(b.counts[e] - mean) : 0.0f;
        inner += c[i] * z[i];
    }
    inner = warp_sum(inner);
    const float per = 1.0f / static_cast<float>(n);
    const float up = dlosses[0] * (static_cast<float>(p.experts) / static_cast<float>(p.topk)) * per * per, size = dlosses[1] * 2.0f * per * lse;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        if (e < p.experts) {
            const float x = z[i] * (up * (c[i] - inner) + size);
            out[e] = accumulate ? out[e] + x : x;
        }
    }
}

}  // namespace nk
