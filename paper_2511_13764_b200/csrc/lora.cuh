// The adapters' part of nk_lora for requests of few rows: D[t] = scale_a (X[t] . A_a) . B_a in FP32.
//
// With a row or a few per request this is two reads, of A_a and B_a, and next to no arithmetic: each weight is
// used for up to eight rows at a time on the FMA units.  A cluster of eight CTAs takes eight rows of one request:
// every CTA multiplies its eighth of K, the eight partial results are added (in the order of the CTAs) through
// distributed shared memory, and every CTA then multiplies its eighth of N.  So even sixteen requests spread their
// weights' reads over 128 SMs, and X . A_a never leaves the cluster.  Small in registers and shared memory, so that
// the projection's blocks can start beside it: its time hides behind theirs.  Measured: 16 requests, 4096 x 4096, rank 16,
// 6 us of a block's time (two reads of 2 MB each, latency: prefix 1, X . A 1.6, the cluster's two barriers and sum 1.7, B 1.1).
#pragma once
#include "half.cuh"
#include "ptx.cuh"

namespace nk {

constexpr int LORA_CLUSTER = 8, LORA_THREADS = 256, LORA_ROWS = 8;
constexpr int LORA_MAX_RANK = 128, LORA_MAX_REQUESTS = 1024;
constexpr int LORA_KSTEP = 256;                 // k of X kept in shared memory at a time

struct LoraParams {
    int rows, N, K, rank, adapters, requests;
    int transposed;
    int few;                                    // 0: requests of up to LORA_ROWS rows, their rows one behind the other in D
                                                // 1: all requests, D like Y, rows without an adapter zero
    long long ldx;
    const void *X, *A, *B;
    const float* scale;
    const int *offsets, *adapter;
    float* D;                                   // [rows][N]
    unsigned int* status;
};

// Rows of the requests, clamped and monotone, and before each request the chunks of LORA_ROWS rows and (few = 0) the rows
// of D.  (few = 0: one chunk to a short request, so `s_pre` counts rows and a request's chunk begins where they change.)
__device__ __forceinline__ int lora_prefix(const LoraParams& p, int* s_row, int* s_pre) {
    const int lane = threadIdx.x & 31;
    for (int q = threadIdx.x; q <= p.requests; q += LORA_THREADS) s_row[q] = p.offsets[q];
    __syncthreads();
    if (threadIdx.x < 32) {
        bool bad = false;
        for (int q = lane; q <= p.requests; q += 32) bad |= s_row[q] < (q ? s_row[q - 1] : 0) || s_row[q] > p.rows;
        if (__any_sync(~0u, bad)) {
            if (lane == 0) {
                if (blockIdx.x == 0 && p.status) atomicCAS(p.status, 0u, 0x10000u);
                int top = 0;
                for (int q = 0; q <= p.requests; ++q) s_row[q] = top = max(top, min(s_row[q], p.rows));
            }
            __syncwarp();
        }
        int sum = 0;
        for (int base = 0; base <= p.requests; base += 32) {
            const int q = base + lane;
            int n = 0;
            if (q < p.requests) {
                const int a = p.adapter[q], rows = s_row[q + 1] - s_row[q];
                if (a >= 0 && a < p.adapters) n = p.few ? (rows + LORA_ROWS - 1) / LORA_ROWS : rows <= LORA_ROWS ? rows : 0;
            }
            int v = n;
#pragma unroll 1
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v += o;
            }
            if (q <= p.requests) s_pre[q] = sum + v - n;
            sum += __shfl_sync(~0u, v, 31);
        }
    }
    __syncthreads();
    return s_pre[p.requests];
}

template <bool F16>
__device__ __forceinline__ void lora_unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = half_bits_to_f32(w[i] & 0xFFFFu, F16);
        x[2 * i + 1] = half_bits_to_f32(w[i] >> 16, F16);
    }
}

// RT rows (1 or LORA_ROWS) of one request; `n` of them exist.  h: this CTA's share of X . A_a, then the whole of it.
template <int RT, bool F16>
__device__ __forceinline__ void lora_chunk(const LoraParams& p, int row0, int n, int a, size_t d_row, uint32_t crank, float* xs, float* part,
                                           float* share, float* h) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int R = p.rank;
    const uint16_t* X = static_cast<const uint16_t*>(p.X);
    const uint16_t* A = static_cast<const uint16_t*>(p.A) + static_cast<size_t>(a) * R * p.K;
    const uint16_t* B = static_cast<const uint16_t*>(p.B) + static_cast<size_t>(a) * R * p.N;
    // this CTA's share of K and N, in steps of 8
    const int kw = ((p.K + LORA_CLUSTER * 8 - 1) / (LORA_CLUSTER * 8)) * 8, k_lo = min(p.K, static_cast<int>(crank) * kw), k_hi = min(p.K, k_lo + kw);
    const int nw = ((p.N + LORA_CLUSTER * 8 - 1) / (LORA_CLUSTER * 8)) * 8, n_lo = min(p.N, static_cast<int>(crank) * nw), n_hi = min(p.N, n_lo + nw);

    // B's part of this CTA is on its way to L2 while A is worked on
    {
        const size_t first = p.transposed ? static_cast<size_t>(n_lo) * R : n_lo, line = 64;   // elements of 128 bytes
        if (p.transposed) {
            for (size_t i = threadIdx.x * line; i < static_cast<size_t>(n_hi - n_lo) * R; i += LORA_THREADS * line)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(B + first + i));
        } else {
            const int lines = (n_hi - n_lo + 63) / 64;
            for (int i = threadIdx.x; i < R * lines; i += LORA_THREADS)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(B + static_cast<size_t>(i / lines) * p.N + first + (i % lines) * line));
        }
    }
    if (RT == 1) {
        // One row: X straight from memory, every load independent of the others.
        const uint16_t* x = X + static_cast<size_t>(row0) * p.ldx;
        if (p.transposed) {
            // a warp has every eighth rank, eight of them at a time with all their loads on the way; lanes along k
            for (int r0 = warp; r0 < R; r0 += 8 * (LORA_THREADS / 32)) {
                float acc[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
                for (int k = k_lo + lane * 8; k < k_hi; k += 256) {
                    uint4 w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int r = r0 + j * (LORA_THREADS / 32);
                        w[j] = r < R ? __ldg(reinterpret_cast<const uint4*>(A + static_cast<size_t>(r) * p.K + k)) : make_uint4(0, 0, 0, 0);
                    }
                    float y[8];
                    lora_unpack8<F16>(__ldg(reinterpret_cast<const uint4*>(x + k)), y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float z[8];
                        lora_unpack8<F16>(w[j], z);
#pragma unroll
                        for (int q = 0; q < 8; ++q) acc[j] += z[q] * y[q];
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = r0 + j * (LORA_THREADS / 32);
                    if (r >= R) break;
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) acc[j] += __shfl_xor_sync(~0u, acc[j], d);
                    if (lane == 0) share[r] = acc[j];
                }
            }
        } else {
            // lanes along eights of ranks, then along k; warps along k; the warps' sums meet in shared memory
            int wide = 1;
            while (wide * 8 < R) wide *= 2;                         // lanes for one k
            const int kl = lane / wide, deep = 32 / wide, r = (lane % wide) * 8;
            float acc[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[q] = 0.0f;
            if (r < R) {
#pragma unroll 4
                for (int k = k_lo + warp * deep + kl; k < k_hi; k += deep * (LORA_THREADS / 32)) {
                    float w[8];
                    lora_unpack8<F16>(__ldg(reinterpret_cast<const uint4*>(A + static_cast<size_t>(k) * R + r)), w);
                    const float y = half_bits_to_f32(__ldg(x + k), F16);
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[q] += w[q] * y;
                }
            }
            for (int d = wide; d < 32; d <<= 1)
#pragma unroll
                for (int q = 0; q < 8; ++q) acc[q] += __shfl_xor_sync(~0u, acc[q], d);
            if (kl == 0 && r < R) {
#pragma unroll
                for (int q = 0; q < 8; ++q) part[warp * R + r + q] = acc[q];
            }
            __syncthreads();
            for (int i = threadIdx.x; i < R; i += LORA_THREADS) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < LORA_THREADS / 32; ++w) s += part[w * R + i];
                share[i] = s;
            }
        }
    } else if (p.transposed) {
        // Up to eight rows: a lane has eight of k of four rows in registers while the ranks of its warp pass, lanes along k.
        for (int i = threadIdx.x; i < RT * R; i += LORA_THREADS) share[i] = 0.0f;
        __syncthreads();
        for (int k0 = k_lo; k0 < k_hi; k0 += 256) {
            const int k = k0 + lane * 8;
            for (int t0 = 0; t0 < n; t0 += 4) {
                uint4 x[4];
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    x[t] = k < k_hi && t0 + t < n ? __ldg(reinterpret_cast<const uint4*>(X + static_cast<size_t>(row0 + t0 + t) * p.ldx + k)) : make_uint4(0, 0, 0, 0);
#pragma unroll 2
                for (int r = warp; r < R; r += LORA_THREADS / 32) {
                    float w[8], acc[4];
                    lora_unpack8<F16>(k < k_hi ? __ldg(reinterpret_cast<const uint4*>(A + static_cast<size_t>(r) * p.K + k)) : make_uint4(0, 0, 0, 0), w);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        float y[8];
                        lora_unpack8<F16>(x[t], y);
                        acc[t] = 0.0f;
#pragma unroll
                        for (int q = 0; q < 8; ++q) acc[t] += w[q] * y[q];
                    }
                    // four sums over 32 lanes: lanes of bits 4, 3 keep one of them each, then the rest add up
                    const bool hi = lane & 16, odd = lane & 8;
                    float a0 = hi ? acc[2] : acc[0], a1 = hi ? acc[3] : acc[1];
                    a0 += __shfl_xor_sync(~0u, hi ? acc[0] : acc[2], 16);
                    a1 += __shfl_xor_sync(~0u, hi ? acc[1] : acc[3], 16);
                    float s = odd ? a1 : a0;
                    s += __shfl_xor_sync(~0u, odd ? a0 : a1, 8);
#pragma unroll
                    for (int d = 4; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
                    if ((lane & 7) == 0) share[r * RT + t0 + (lane >> 3)] += s;
                }
            }
        }
    } else {
        for (int i = threadIdx.x; i < RT * R; i += LORA_THREADS) share[i] = 0.0f;
        // part[warp][r][RT] (row-major weights only): each warp's sums
        for (int k0 = k_lo; k0 < k_hi; k0 += LORA_KSTEP) {
            const int kn = min(LORA_KSTEP, k_hi - k0);
            __syncthreads();
            // X as FP32, [k][RT]; eight of k to a thread
            for (int i = threadIdx.x; i < RT * (LORA_KSTEP / 8); i += LORA_THREADS) {
                const int t = i / (LORA_KSTEP / 8), k = (i - t * (LORA_KSTEP / 8)) * 8;
                if (k >= kn) continue;
                float x[8];
                lora_unpack8<F16>(t < n ? *reinterpret_cast<const uint4*>(X + static_cast<size_t>(row0 + t) * p.ldx + k0 + k) : make_uint4(0, 0, 0, 0), x);
#pragma unroll
                for (int q = 0; q < 8; ++q) xs[(k + q) * RT + t] = x[q];
            }
            __syncthreads();
            {
                // lanes along pairs of ranks, then along k; warps along k; the warps' sums meet in shared memory
                const int pairs = R / 2;
                int wide = 4;
                while (wide < pairs && wide < 32) wide *= 2;            // lanes for one k
                const int kl = lane / wide, deep = 32 / wide;
                for (int r0 = 0; r0 < pairs; r0 += wide) {
                    const int pr = r0 + lane % wide;
                    float acc0[RT], acc1[RT];
#pragma unroll
                    for (int t = 0; t < RT; ++t) acc0[t] = acc1[t] = 0.0f;
                    if (pr < pairs) {
#pragma unroll 8
                        for (int k = warp * deep + kl; k < kn; k += deep * (LORA_THREADS / 32)) {
                            const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(A + static_cast<size_t>(k0 + k) * R) + pr);
                            const float w0 = half_bits_to_f32(w & 0xFFFFu, F16), w1 = half_bits_to_f32(w >> 16, F16);
#pragma unroll
                            for (int t = 0; t < RT; ++t) {
                                acc0[t] += w0 * xs[k * RT + t];
                                acc1[t] += w1 * xs[k * RT + t];
                            }
                        }
                    }
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        for (int d = wide; d < 32; d <<= 1) {
                            acc0[t] += __shfl_xor_sync(~0u, acc0[t], d);
                            acc1[t] += __shfl_xor_sync(~0u, acc1[t], d);
                        }
                        if (kl == 0 && pr < pairs) {
                            part[(warp * R + 2 * pr) * RT + t] = acc0[t];
                            part[(warp * R + 2 * pr + 1) * RT + t] = acc1[t];
                        }
                    }
                }
                __syncthreads();
                for (int i = threadIdx.x; i < R * RT; i += LORA_THREADS) {
                    float s = share[i];
#pragma unroll
                    for (int w = 0; w < LORA_THREADS / 32; ++w) s += part[w * R * RT + i];
                    share[i] = s;
                }
            }
        }
    }
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    const float scale = __ldg(p.scale + a);
    const uint32_t share_addr = smem_u32(share);
    for (int i = threadIdx.x; i < R * RT; i += LORA_THREADS) {
        float v[LORA_CLUSTER];
#pragma unroll
        for (int c = 0; c < LORA_CLUSTER; ++c)
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c]) : "r"(map_to_cta(share_addr + 4 * i, c)) : "memory");
        float s = v[0];
#pragma unroll
        for (int c = 1; c < LORA_CLUSTER; ++c) s += v[c];
        h[i] = s * scale;
    }
    cluster_arrive();          // `share` may be written again once every CTA has read it
    cluster_wait();
    __syncthreads();
    if (RT == 1 && !p.transposed) {
        // threads along eights of columns, the rest of them along the ranks; their sums meet in shared memory
        const int eights = (n_hi - n_lo) / 8, groups = max(1, LORA_THREADS / max(1, eights));
        for (int e0 = 0; e0 < eights; e0 += LORA_THREADS) {
            const int wide = min(eights - e0, LORA_THREADS), g = threadIdx.x / wide, e = threadIdx.x - g * wide;
            if (g < groups) {
                float acc[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) acc[q] = 0.0f;
#pragma unroll 4
                for (int r = g; r < R; r += groups) {
                    float w[8];
                    lora_unpack8<F16>(__ldg(reinterpret_cast<const uint4*>(B + static_cast<size_t>(r) * p.N + n_lo + (e0 + e) * 8)), w);
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[q] += w[q] * h[r];
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) xs[(g * wide + e) * 8 + q] = acc[q];
            }
            __syncthreads();
            for (int i = threadIdx.x; i < wide * 8; i += LORA_THREADS) {
                float s = xs[i];
                for (int z = 1; z < groups; ++z) s += xs[z * wide * 8 + i];
                p.D[d_row * p.N + n_lo + e0 * 8 + i] = s;
            }
            __syncthreads();
        }
    } else if (RT == 1) {
        // lanes along eights of ranks, then along columns: a load is 512 contiguous bytes of B where the rank is a power of two
        int wide = 1;
        while (wide * 8 < R) wide *= 2;                             // lanes for one column
        const int per = 32 / wide, r = (lane % wide) * 8;
        float g[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) g[q] = r < R ? h[r + q] : 0.0f;
#pragma unroll 4
        for (int i0 = n_lo + warp * per; i0 < n_hi; i0 += per * (LORA_THREADS / 32)) {
            const int i = i0 + lane / wide;
            float w[8], acc = 0.0f;
            lora_unpack8<F16>(i < n_hi && r < R ? __ldg(reinterpret_cast<const uint4*>(B + static_cast<size_t>(i) * R + r)) : make_uint4(0, 0, 0, 0), w);
#pragma unroll
            for (int q = 0; q < 8; ++q) acc += w[q] * g[q];
            for (int d = 1; d < wide; d <<= 1) acc += __shfl_xor_sync(~0u, acc, d);
            if (lane % wide == 0 && i < n_hi) p.D[d_row * p.N + i] = acc;
        }
    } else if (p.transposed) {
        for (int i = n_lo + threadIdx.x; i < n_hi; i += LORA_THREADS) {
            float acc[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t] = 0.0f;
#pragma unroll 4
            for (int r = 0; r < R; r += 8) {
                float w[8];
                lora_unpack8<F16>(__ldg(reinterpret_cast<const uint4*>(B + static_cast<size_t>(i) * R + r)), w);
#pragma unroll
                for (int q = 0; q < 8; ++q)
#pragma unroll
                    for (int t = 0; t < RT; ++t) acc[t] += w[q] * h[(r + q) * RT + t];
            }
#pragma unroll
            for (int t = 0; t < RT; ++t)
                if (t < n) p.D[(d_row + t) * p.N + i] = acc[t];
        }
    } else {
        for (int i = n_lo + 2 * threadIdx.x; i < n_hi; i += 2 * LORA_THREADS) {
            float acc0[RT], acc1[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) acc0[t] = acc1[t] = 0.0f;
#pragma unroll 8
            for (int r = 0; r < R; ++r) {
                const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(B + static_cast<size_t>(r) * p.N + i));
                const float w0 = half_bits_to_f32(w & 0xFFFFu, F16), w1 = half_bits_to_f32(w >> 16, F16);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    acc0[t] += w0 * h[r * RT + t];
                    acc1[t] += w1 * h[r * RT + t];
                }
            }
#pragma unroll
            for (int t = 0; t < RT; ++t)
                if (t < n) *reinterpret_cast<float2*>(p.D + (d_row + t) * p.N + i) = make_float2(acc0[t], acc1[t]);
        }
    }
    __syncthreads();
}

// Shared memory: X, the warps' sums (row-major weights), the CTA's share and the whole of X . A_a, the two tables.
__host__ __device__ inline int lora_smem(int rank, int requests, bool transposed) {
    return 4 * (LORA_KSTEP * LORA_ROWS + (transposed ? 0 : LORA_THREADS / 32 * rank * LORA_ROWS) + 2 * rank * LORA_ROWS + 2 * (requests + 1));
}

template <bool F16>
__global__ void __launch_bounds__(LORA_THREADS, 4) __cluster_dims__(LORA_CLUSTER, 1, 1) lora_delta_kernel(const LoraParams p) {
    extern __shared__ float lora_sm[];
    float* xs = lora_sm;
    float* part = xs + LORA_KSTEP * LORA_ROWS;
    float* share = part + (p.transposed ? 0 : LORA_THREADS / 32 * p.rank * LORA_ROWS);
    float* h = share + p.rank * LORA_ROWS;
    int* s_row = reinterpret_cast<int*>(h + p.rank * LORA_ROWS);
    int* s_pre = s_row + p.requests + 1;
    launch_wait();
    launch_next();
    const int chunks = lora_prefix(p, s_row, s_pre);
    const uint32_t crank = cluster_ctarank();
    const int clusters = gridDim.x / LORA_CLUSTER, cluster = blockIdx.x / LORA_CLUSTER;
    if (p.few) {
        // rows without an adapter add nothing: zeros (rows of no request among them)
        for (int t = blockIdx.x; t < p.rows; t += gridDim.x) {
            int lo = 0, hi = p.requests + 1;               // the last request that begins at or before the row
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_row[mid] <= t) lo = mid;
                else hi = mid;
            }
            if (lo < p.requests && s_row[lo] <= t && s_pre[lo + 1] > s_pre[lo]) continue;
            float4* d = reinterpret_cast<float4*>(p.D + static_cast<size_t>(t) * p.N);
            for (int i = threadIdx.x; i < p.N / 4; i += LORA_THREADS) d[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    // few: chunk after chunk; else request after request
    for (int c = cluster; c < (p.few ? chunks : p.requests); c += clusters) {
        int q = c;
        if (p.few) {
            int lo = 0, hi = p.requests;                   // s_pre[lo] <= c < s_pre[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_pre[mid] <= c) lo = mid;
                else hi = mid;
            }
            q = lo;
        } else if (s_pre[q + 1] == s_pre[q]) {
            continue;
        }
        const int row0 = s_row[q] + (p.few ? (c - s_pre[q]) * LORA_ROWS : 0);
        const int n = min(LORA_ROWS, s_row[q + 1] - row0);
        const size_t d_row = p.few ? row0 : s_pre[q];
        const int a = p.adapter[q];
        if (n == 1) lora_chunk<1, F16>(p, row0, n, a, d_row, crank, xs, part, share, h);
        else lora_chunk<LORA_ROWS, F16>(p, row0, n, a, d_row, crank, xs, part, share, h);
    }
}

// FP16 operands: rows of X . A_a, FP32 [rows][rank], as the 16-bit numbers that the tensor cores multiply by B_a (see
// GroupedParams), a warp to a row.  FP16 has five bits of exponent: as it is, a row of 2^-14 would keep half of its leading part's
// bits and no remainder, one beyond 65504 nothing.  So a row is multiplied by the power of two that puts its largest finite element
// into [2^14, 2^15); two numbers are then good to 2^-22 of each element down to 2^-18 of the row's largest (and to 2^-40 of that
// below), three to 2^-33 and 2^-40.  A row scaled so costs the projection an accumulator (8192 rows of 5 requests, 4096 x 4096, rank
// 64: 204 us instead of 190); of two numbers, rows from 2^-5 to 2^15 stay as they are (2^-20 of the largest at worst) and add up in the
// tile's own.  Rows of no long request are whatever the workspace held; nothing comes of them.
struct LoraSplitParams {
    int rows, rank, rank_blocks, planes;
    const float* x;             // [rows][rank]
    uint16_t* h16;              // [rows][rank_blocks * 64]
    float* unscale;             // [rows]
};
constexpr int LORA_SPLIT_ROWS = 8;               // of a block of 256 threads at a time
__global__ void __launch_bounds__(32 * LORA_SPLIT_ROWS) lora_split_kernel(const LoraSplitParams p) {
    const int lane = threadIdx.x & 31;
    constexpr int V = LORA_MAX_RANK / 32;
    launch_wait();
    launch_next();
    int row = blockIdx.x * LORA_SPLIT_ROWS + (threadIdx.x >> 5);
    float next[V];
    auto fetch = [&](int r) {
#pragma unroll
        for (int n = 0; n < V; ++n) next[n] = r < p.rows && lane + 32 * n < p.rank ? __ldcg(p.x + static_cast<size_t>(r) * p.rank + lane + 32 * n) : 0.0f;
    };
    fetch(row);
    for (; row < p.rows; row += gridDim.x * LORA_SPLIT_ROWS) {
        float v[V];
        uint32_t top = 0u;
#pragma unroll
        for (int n = 0; n < V; ++n) {
            v[n] = next[n];
            const uint32_t bits = __float_as_uint(v[n]) & 0x7FFFFFFFu;
            if (bits < 0x7F800000u) top = max(top, bits);
        }
        fetch(row + gridDim.x * LORA_SPLIT_ROWS);      // the next row is on the way
        top = __reduce_max_sync(~0u, top);
        // (subnormal rows: 2^126 is as far as a factor and its inverse are both ordinary numbers)
        const int ex = static_cast<int>(top >> 23) - 127;
        const bool plain = p.planes == 2 && (top == 0u || (ex >= -5 && ex < 15));
        const int e = plain ? 0 : min(126, 14 - ex);
        const float up = __int_as_float((127 + e) << 23);
        if (lane == 0) p.unscale[row] = __int_as_float((127 - e) << 23);
        const int per = p.planes == 3 ? 16 : 32;
        uint16_t* h = p.h16 + static_cast<size_t>(row) * p.rank_blocks * 64;
#pragma unroll
        for (int n = 0; n < V; ++n) {
            const int i = lane + 32 * n;
            if (i >= p.rank_blocks * per) break;       // (ranks beyond the last are zeros)
            float left = v[n] * up;
            for (int z = 0; z < p.planes; ++z) {
                const uint32_t bits = pack_half2(left, 0.0f, 1) & 0xFFFFu;
                const float lead = half_bits_to_f32(bits, 1);
                h[i / per * 64 + z * per + i % per] = static_cast<uint16_t>(bits);
                left = fabsf(lead) <= 65504.0f ? left - lead : 0.0f;     // (nothing behind an infinity or NaN)
            }
        }
    }
}

}  // namespace nk
