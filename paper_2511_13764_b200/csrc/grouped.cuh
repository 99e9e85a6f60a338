// Products whose weight goes by the row: ragged groups of rows, one weight per group.
//
//   ROWS      C[t][i] = sum_k W_g[k][i] X[t][k]      for the rows t of group g (the contraction is dense)
//   WEIGHTS   C_g[j][i] = sum_t B[t][i] A[t][j]      over the rows t of group g (the contraction is ragged)
//
// Both are one kernel.  The MMA's M dimension is the one that is contiguous in C (i: the features of the
// output), its N dimension the rows of C (ROWS: the group's rows, WEIGHTS: j).  So it is the ragged
// dimension of ROWS that is the MMA's N, which the instruction takes in steps of 16: a group's last tile
// pays for its rows rounded up to 32, not to 128 or 256, and an expert with one row streams its weight
// through a 256 x 32 tile at the speed of memory.  And the accumulator's lanes are consecutive features:
// 32 lanes of a store write 32 consecutive elements of a row of C, wherever the group's rows begin.
//
// A CTA pair (cta_group::2) computes a tile of 256 features x up to 256 rows: each CTA holds 128 features
// of the MMA's A operand and half of the columns of its B operand, and drains 128 accumulator lanes.  The
// groups' offsets are read on the device: every CTA turns them into a prefix of tile counts at its start
// (a few hundred clocks), so no launch, size or plan depends on how the rows are spread.
//
// Warps: 0 TMA producer, 1 MMA issuer, 2-9 epilogue (warps 2-5 take the even 32-column chunks, 6-9 the odd
// ones), 10 (WEIGHTS) clears the rows of a group's last k-block that belong to the next group.
// All waits are bounded (see mbar_wait).
#pragma once
#include "grouped_launch.cuh"
#include "half.cuh"
#include "ptx.cuh"

namespace nk {

// Work of one unit.
struct GroupedUnit {
    int g, i0, c0;         // group, first feature, first row of C (ROWS: in the whole array, WEIGHTS: in C_g)
    int cols, jn;          // rows of C in the tile, and the MMA's N (cols rounded up to 32)
    int kb0, kb1;          // k-blocks
    int row0, rows;        // WEIGHTS: the group's rows
    int tile, split;
};

__device__ __forceinline__ int round32(int x) { return (x + 31) & ~31; }

// C[row][i] += for one 32 x 32 piece (lane = feature, v[j] = row c0 + j)
__device__ __forceinline__ void grouped_store(const GroupedParams& p, const uint32_t (&v)[32], size_t base, int i, int cols,
                                              const float* add) {
    if (i >= p.I) return;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (j >= cols) break;                            // warp-uniform
        const size_t o = base + static_cast<size_t>(j) * p.ldc + i;
        float x = __uint_as_float(v[j]);
        if (add) x += add[static_cast<size_t>(j) * p.I + i];
        if (p.out16) {
            uint16_t* c = static_cast<uint16_t*>(p.C) + o;
            if (p.beta) x += half_bits_to_f32(*c, p.f16);
            *c = static_cast<uint16_t>(pack_half2(x, 0.0f, p.f16) & 0xFFFFu);
        } else {
            float* c = static_cast<float*>(p.C) + o;
            if (p.beta) x += *c;
            *c = x;
        }
    }
}

// WEIGHTS: contraction over the rows of a group.  A_MN: the features' operand is MN-major (row-major weights
// [K][I], or rows [t][I]), else K-major (weights [I][K]).
template <bool WEIGHTS, bool A_MN>
__global__ void __launch_bounds__(GRP_THREADS, 1) __cluster_dims__(2, 1, 1)
grouped_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
               const __grid_constant__ CUtensorMap tmap_b16, const GroupedParams p) {
    static_assert(!WEIGHTS || A_MN, "rows are contiguous in their features");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
    int* s_row = reinterpret_cast<int*>(gen_base + GRP_STAGES * GRP_STAGE);   // first row of each group, clamped and monotone
    int* s_pre = s_row + GRP_MAX_GROUPS + 1;                                  // units before each group
    const uint32_t bar_base = smem_base + GRP_STAGES * GRP_STAGE + 2 * 4 * (GRP_MAX_GROUPS + 1);
    constexpr int S = GRP_STAGES;
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };
    auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * S + a); };
    auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * S + 2 + a); };
    auto raw_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + s); };    // WEIGHTS, last block of a group: this CTA's boxes have landed
    auto tail_bar = [&](int s) { return bar_base + 8u * (3 * S + 4 + s); };   // leader: both CTAs have cleared the rows beyond the group
    constexpr int NB = 4 * S + 4;
    static_assert(NB <= 32, "one barrier per lane");
    const uint32_t peer_ready_bar = bar_base + 8u * NB;
    uint8_t* after = gen_base + GRP_STAGES * GRP_STAGE + 2 * 4 * (GRP_MAX_GROUPS + 1) + 8 * (NB + 1);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(after);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile uint32_t* last_flag = tmem_slot + 2;       // this CTA is the last of its tile's K splits

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair_id = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    auto give_up = [&](unsigned int code) {
        *abort_flag = 1;
        if (p.status) atomicCAS(p.status, 0u, code);
    };

    // offsets -> shared memory
    for (int g = threadIdx.x; g <= p.groups; g += GRP_THREADS) s_row[g] = p.offsets ? p.offsets[g] : g == 0 ? 0 : p.rows;
    if (warp == 0) {
        if (lane < NB) {
            // tempty: one arrival per epilogue warp of both CTAs; tail: one per CTA
            const uint32_t count = lane >= 2 * S + 2 && lane < 2 * S + 4 ? 16 : lane >= 3 * S + 4 ? 2 : 1;
            mbar_init(bar_base + 8u * lane, count);
        }
        if (lane == 31) mbar_init(peer_ready_bar, 1);
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
        __syncwarp();
    } else if (warp == 2 && lane == 0) {
        tma_prefetch_desc(&tmap_a);
        tma_prefetch_desc(&tmap_b);
        if (!WEIGHTS) tma_prefetch_desc(&tmap_b16);
    } else if (warp == 1) {
        tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 2) {
        // running maximum of the clamped offsets, then the prefix of the unit counts
        int top = 0, units = 0;
        bool bad = false;
        for (int base = 0; base <= p.groups; base += 32) {
            const int g = base + lane;
            const int raw = g <= p.groups ? s_row[g] : 0;
            int v = min(max(raw, 0), p.rows);
            bool off = g <= p.groups && v != raw;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v = max(v, o);
            }
            v = max(v, top);
            if (g <= p.groups) {
                off |= v != raw;
                s_row[g] = v;
            }
            bad |= off;
            top = __shfl_sync(~0u, v, 31);
        }
        if (__any_sync(~0u, bad) && lane == 0 && blockIdx.x == 0 && p.status) atomicCAS(p.status, 0u, 0x10000u);
        __syncwarp();
        for (int base = 0; base <= p.groups; base += 32) {
            const int g = base + lane;
            const int n = g < p.groups ? (WEIGHTS ? p.tiles_i * p.tiles_j : (s_row[g + 1] - s_row[g] + GRP_TILE - 1) / GRP_TILE * p.tiles_i) : 0;
            int v = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v += o;
            }
            if (g <= p.groups) s_pre[g] = units + v - n;
            units += __shfl_sync(~0u, v, 31);
        }
    }
    cluster_arrive();
    cluster_wait();          // the barriers of both CTAs are initialised
    __syncthreads();         // the prefix is there
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    if (warp == 1 && rank == 1 && lane == 0) mbar_arrive_cluster_cta_release(map_to_cta(peer_ready_bar, 0));

    const int tiles = s_pre[p.groups];
    // K splits where there are fewer tiles than pairs (a split has at least four k-blocks); every pair then has one unit at most
    int splits = 1, per_split = p.kb_total;
    if (!WEIGHTS && p.partial && tiles > 0 && 2 * tiles <= num_pairs) {
        splits = min(min(num_pairs / tiles, p.kb_total / 4), GRP_MAX_SPLITS);
        splits = max(splits, 1);
        per_split = (p.kb_total + splits - 1) / splits;
        splits = (p.kb_total + per_split - 1) / per_split;
    }
    const int total_units = tiles * splits;
    auto decode = [&](int unit) {
        GroupedUnit u;
        u.tile = splits > 1 ? div_small(unit, splits) : unit;
        u.split = unit - u.tile * splits;
        if (WEIGHTS) {
            const int per = p.tiles_i * p.tiles_j;
            u.g = div_small(unit, per);
            const int rel = unit - u.g * per;
            const int ti = div_small(rel, p.tiles_j);
            u.i0 = ti * GRP_TILE;
            u.c0 = (rel - ti * p.tiles_j) * GRP_TILE;
            u.cols = min(GRP_TILE, p.J - u.c0);
            u.row0 = s_row[u.g];
            u.rows = s_row[u.g + 1] - u.row0;
            u.kb0 = 0;
            u.kb1 = (u.rows + GRP_BK - 1) / GRP_BK;
        } else {
            int lo = 0, hi = p.groups;                    // s_pre[lo] <= tile < s_pre[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_pre[mid] <= u.tile) lo = mid;
                else hi = mid;
            }
            u.g = lo;
            const int rel = u.tile - s_pre[lo];
            u.row0 = s_row[lo];
            u.rows = s_row[lo + 1] - u.row0;
            // the group's rows cut into equal tiles; eight of them sweep the features together
            const int nt = (u.rows + GRP_TILE - 1) / GRP_TILE;
            const int jt = round32((u.rows + nt - 1) / nt);
            const int per = 8 * p.tiles_i;
            const int block = div_small(rel, per);
            const int within = rel - block * per;
            const int wide = min(8, nt - block * 8);
            const int ti = div_small(within, wide);
            const int tj = block * 8 + within - ti * wide;
            u.i0 = ti * GRP_TILE;
            u.c0 = u.row0 + tj * jt;
            u.cols = min(jt, u.row0 + u.rows - u.c0);
            u.kb0 = u.split * per_split;
            u.kb1 = min(p.kb_total, u.kb0 + per_split);
        }
        u.jn = round32(u.cols);
        return u;
    };
    // WEIGHTS: 16-row steps of k-block kb, and whether rows beyond the group have to be cleared in the last of them
    auto tail_rows = [&](const GroupedUnit& u, int kb) { return min(GRP_BK, u.rows - kb * GRP_BK); };

    if (warp == 0) {
        // ------------------------------------------------ TMA producer (both CTAs)
        const uint32_t lead_full0 = map_to_cta(full_bar(0), 0);
        const uint32_t elected = elect_one();
        const uint32_t lead_elected = rank == 0 ? elected : 0u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int unit = pair_id; ok && unit < total_units; unit += num_pairs) {
            const GroupedUnit u = decode(unit);
            const int half = u.jn >> 1;
            const int i = u.i0 + static_cast<int>(rank) * 128;
            const int c = u.c0 + static_cast<int>(rank) * half;      // first column of this CTA's B operand
            const int boxes = WEIGHTS ? (half + 63) >> 6 : half >> 4;
            const uint32_t bytes = GRP_A_BYTES + (WEIGHTS ? boxes * 8192u : half * 128u);
            for (int kb = u.kb0; kb < u.kb1; ++kb) {
                if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) {
                    if (lane == 0) give_up(0x100u + stage);
                    ok = false;
                    break;
                }
                const uint32_t sa = smem_base + stage * GRP_STAGE, sb = sa + GRP_A_BYTES;
                const uint32_t fb = full_bar(stage), lfb = lead_full0 + 8u * stage;
                if (WEIGHTS) {
                    const int t = u.row0 + kb * GRP_BK;
                    if (tail_rows(u, kb) & 15) {
                        // on this CTA's own barrier: warp 10 clears what belongs to the next group, then reports to the leader
                        mbar_arrive_expect_tx_if(raw_bar(stage), bytes, elected);
                        if (rank == 0 && elected) mbar_arrive(fb);
                        __syncwarp();
                        tma_load_3d_if(sa, &tmap_a, raw_bar(stage), i, t, 0, elected);
                        tma_load_3d_if(sa + 8192, &tmap_a, raw_bar(stage), i + 64, t, 0, elected);
                        for (int b = 0; b < boxes; ++b) tma_load_3d_if(sb + b * 8192, &tmap_b, raw_bar(stage), c + b * 64, t, 0, elected);
                    } else {
                        mbar_arrive_expect_tx_if(fb, 2u * bytes, lead_elected);
                        tma_load_3d_pair_if(sa, &tmap_a, lfb, i, t, 0, elected);
                        tma_load_3d_pair_if(sa + 8192, &tmap_a, lfb, i + 64, t, 0, elected);
                        for (int b = 0; b < boxes; ++b) tma_load_3d_pair_if(sb + b * 8192, &tmap_b, lfb, c + b * 64, t, 0, elected);
                    }
                } else {
                    const int kx = kb * GRP_BK;
                    mbar_arrive_expect_tx_if(fb, 2u * bytes, lead_elected);
                    if (A_MN) {
                        tma_load_3d_pair_if(sa, &tmap_a, lfb, i, kx, u.g, elected);
                        tma_load_3d_pair_if(sa + 8192, &tmap_a, lfb, i + 64, kx, u.g, elected);
                    } else {
                        tma_load_3d_pair_if(sa, &tmap_a, lfb, kx, i, u.g, elected);
                    }
                    if (half == 128) {
                        tma_load_3d_pair_if(sb, &tmap_b, lfb, kx, c, 0, elected);
                    } else {
                        for (int b = 0; b < boxes; ++b) tma_load_3d_pair_if(sb + b * 2048, &tmap_b16, lfb, kx, c + b * 16, 0, elected);
                    }
                }
                __syncwarp();
                if (++stage == S) { stage = 0; phase ^= 1u; }
            }
        }
        if (ok) {   // drain: every stage this CTA filled has been consumed
            for (int s = 0; s < S; ++s) {
                if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) break;
                if (++stage == S) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer (leader only)
        if (rank == 0) {
            const uint64_t da = A_MN ? make_smem_desc(smem_base, 8192, 1024, 2) : make_smem_desc(smem_base, 16, 1024, 2);
            const uint64_t db = WEIGHTS ? make_smem_desc(smem_base + GRP_A_BYTES, 8192, 1024, 2)
                                        : make_smem_desc(smem_base + GRP_A_BYTES, 16, 1024, 2);
            const uint32_t a_hi = static_cast<uint32_t>(da >> 32), b_hi = static_cast<uint32_t>(db >> 32);
            const uint32_t a_lo0 = static_cast<uint32_t>(da), b_lo0 = static_cast<uint32_t>(db);
            constexpr uint32_t a_s = A_MN ? 128u : 2u, b_s = WEIGHTS ? 128u : 2u;   // 16 of k, in 16-byte units
            const uint32_t elected = elect_one();
            int stage = 0, local = 0;
            uint32_t phase = 0, tail_phase = 0;
            bool ok = true;
            if (!mbar_wait(peer_ready_bar, 0u, abort_flag)) {
                if (lane == 0) give_up(0x700u);
                ok = false;
            }
            for (int unit = pair_id; ok && unit < total_units; unit += num_pairs, ++local) {
                const GroupedUnit u = decode(unit);
                const int acc = local & 1;
                if (!mbar_wait(tempty_bar(acc), ((local >> 1) & 1u) ^ 1u, abort_flag)) {
                    if (lane == 0) give_up(0x200u + acc);
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + acc * GRP_TILE;
                const uint32_t idesc = p.idesc | (static_cast<uint32_t>(u.jn >> 3) << 17);
                uint32_t accumulate = 0u;
                for (int kb = u.kb0; kb < u.kb1; ++kb) {
                    if (!mbar_wait(full_bar(stage), phase, abort_flag)) {
                        if (lane == 0) give_up(0x300u + stage);
                        ok = false;
                        break;
                    }
                    int steps = 4;
                    if (WEIGHTS) {
                        const int rem = tail_rows(u, kb);
                        steps = (rem + 15) >> 4;
                        if (rem & 15) {
                            if (!mbar_wait(tail_bar(stage), (tail_phase >> stage) & 1u, abort_flag)) {
                                if (lane == 0) give_up(0x600u + stage);
                                ok = false;
                                break;
                            }
                            tail_phase ^= 1u << stage;
                        }
                    }
                    tc_fence_after_sync();
                    const uint32_t a_lo = a_lo0 + stage * (GRP_STAGE >> 4), b_lo = b_lo0 + stage * (GRP_STAGE >> 4);
                    umma_pair_if<0>(d_tmem, a_lo, a_hi, b_lo, b_hi, idesc, accumulate, elected);
                    if (!WEIGHTS || steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + b_s, b_hi, idesc, 1u, elected);
                    if (!WEIGHTS || steps > 2) umma_pair_if<0>(d_tmem, a_lo + 2 * a_s, a_hi, b_lo + 2 * b_s, b_hi, idesc, 1u, elected);
                    if (!WEIGHTS || steps > 3) umma_pair_if<0>(d_tmem, a_lo + 3 * a_s, a_hi, b_lo + 3 * b_s, b_hi, idesc, 1u, elected);
                    umma_commit_pair_if(empty_bar(stage), 3, elected);
                    if (kb == u.kb1 - 1) umma_commit_pair_if(tfull_bar(acc), 3, elected);
                    accumulate = 1u;
                    __syncwarp();
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
                if (u.kb1 <= u.kb0) umma_commit_pair_if(tfull_bar(acc), 3, elected);
            }
        }
    } else if (warp < 10) {
        // ------------------------------------------------ epilogue (both CTAs, own 128 features)
        const int set = warp >= 6 ? 1 : 0;
        const int quarter = warp & 3;
        int local = 0;
        for (int unit = pair_id; unit < total_units; unit += num_pairs, ++local) {
            const GroupedUnit u = decode(unit);
            const int acc = local & 1;
            if (!mbar_wait(tfull_bar(acc), (local >> 1) & 1u, abort_flag)) {
                if (lane == 0) give_up(0x400u + acc);
                break;
            }
            tc_fence_after_sync();
            const int i = u.i0 + static_cast<int>(rank) * 128 + quarter * 32 + lane;
            const uint32_t taddr = tmem_base + acc * GRP_TILE + (static_cast<uint32_t>(quarter * 32) << 16);
            const bool empty_k = u.kb1 <= u.kb0;
            const size_t slab = 2 * 128 * GRP_TILE;           // partials of one (unit, split): two CTAs
            float* part = p.partial + (static_cast<size_t>(u.tile) * splits + u.split) * slab + rank * (slab / 2) + quarter * 32 + lane;
            for (int c = set * 32; c < u.cols; c += 64) {
                uint32_t v[32];
                tmem_ld_32x32(taddr + c, v);
                tmem_ld_wait();
                if (empty_k) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0u;
                }
                const int n = min(32, u.cols - c);
                if (splits > 1) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) part[(c + j) * 128] = __uint_as_float(v[j]);
                } else {
                    const size_t base = (WEIGHTS ? static_cast<size_t>(u.g) * p.stride_c : 0) + static_cast<size_t>(u.c0 + c) * p.ldc;
                    grouped_store(p, v, base, i, n, p.add ? p.add + static_cast<size_t>(u.c0 + c) * p.I : nullptr);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_cta_release(map_to_cta(tempty_bar(acc), 0));
            if (!WEIGHTS && splits > 1) {
                // the CTA that finishes a tile last adds its K splits in their order and stores: nobody waits
                __threadfence();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (warp == 2 && lane == 0) {
                    const unsigned int old = atomicAdd(p.counter + 2 * u.tile + rank, 1u);
                    *last_flag = old == static_cast<unsigned int>(splits) - 1u;
                    if (old == static_cast<unsigned int>(splits) - 1u) p.counter[2 * u.tile + rank] = 0;
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (*last_flag) {
                    __threadfence();
                    const float* src = p.partial + static_cast<size_t>(u.tile) * splits * slab + rank * (slab / 2) + quarter * 32 + lane;
                    for (int c = set * 32; c < u.cols; c += 64) {
                        uint32_t v[32];
                        float sum[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[j] = __ldcg(src + (c + j) * 128);
                        for (int s = 1; s < splits; ++s)
#pragma unroll
                            for (int j = 0; j < 32; ++j) sum[j] += __ldcg(src + s * slab + (c + j) * 128);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(sum[j]);
                        grouped_store(p, v, static_cast<size_t>(u.c0 + c) * p.ldc, i, min(32, u.cols - c),
                                      p.add ? p.add + static_cast<size_t>(u.c0 + c) * p.I : nullptr);
                    }
                }
            }
        }
    } else if (WEIGHTS) {
        // ------------------------------------------------ rows of the next group in a group's last k-block
        const uint32_t lead_tail0 = map_to_cta(tail_bar(0), 0);
        int stage = 0;
        uint32_t raw_phase = 0;
        for (int unit = pair_id; unit < total_units; unit += num_pairs) {
            const GroupedUnit u = decode(unit);
            if (u.kb1 == 0) continue;
            stage = (stage + u.kb1 - 1) % S;
            const int rem = tail_rows(u, u.kb1 - 1);
            if (rem & 15) {
                if (!mbar_wait(raw_bar(stage), (raw_phase >> stage) & 1u, abort_flag)) {
                    if (lane == 0) give_up(0x500u + stage);
                    break;
                }
                raw_phase ^= 1u << stage;
                const int boxes = 2 + ((u.jn >> 1) + 63) / 64;
                const int first = rem * 8, last = ((rem + 15) & ~15) * 8;   // 16-byte pieces of a box's rows of 128 bytes
                for (int b = 0; b < boxes; ++b)
                    for (int x = first + lane; x < last; x += 32)
                        st_shared_v4(smem_base + stage * GRP_STAGE + b * 8192 + x * 16, 0u, 0u, 0u, 0u);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_cta_release(lead_tail0 + 8u * stage);
            }
            stage = (stage + 1) % S;
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

}  // namespace nk
