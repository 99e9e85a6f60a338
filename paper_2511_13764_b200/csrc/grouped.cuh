// Products whose weight goes by the row: ragged groups of rows, one weight per group.
//
//   ROWS      C[t][i] = sum_k W_g[k][i] X[t][k]      for the rows t of group g (the contraction is dense)
//   WEIGHTS   C_g[j][i] = sum_t B[t][i] A[t][j]      over the rows t of group g (the contraction is ragged)
//   LORA      ROWS with one weight, and for every request q a rank-r product of its rows on top
//
// All are one kernel.  The MMA's M dimension is the one that is contiguous in C (i: the features of the
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
// Schedule.  Whole waves of tiles go to the pairs in turn.  What is left (less than two waves) is laid end to
// end along k and shared out evenly, where that saves more k-blocks than a cut tile costs; the pieces of a
// cut tile meet in global memory, and the warp that finishes a 32 x 32 piece last adds its parts in k order
// and stores it: nobody waits, and the sum does not depend on who was last.
//
// FP32 results (p.chunk): the tensor core's accumulator is cut short, not rounded, at every step, an error
// that grows with the number of steps; so after `chunk` k-blocks the accumulator is added to an FP32 sum in
// the epilogue's registers while the other accumulator is being filled.  16-bit results do not need it.
//
// Warps: 0 TMA producer, 1 MMA issuer, 2-9 epilogue (warps 2-5 take the even 32-column chunks, 6-9 the odd
// ones), 10 (WEIGHTS) clears the rows of a group's last k-block that belong to the next group.
// All waits are bounded (see mbar_wait).
#pragma once
#include "grouped_launch.cuh"
#include "half.cuh"
#include "ptx.cuh"

namespace nk {

// One piece of work: k-blocks kb0 .. kb1-1 of a tile.
struct GroupedUnit {
    int g, w, i0, c0;      // group, its weight, first feature, first row of C (ROWS: in the whole array, WEIGHTS: in C_g)
    int cols, jn;          // rows of C in the tile, and the MMA's N (cols rounded up to 32)
    int kb0, kb1, kbs;     // k-blocks of this piece, and of the whole tile
    int row0, rows;        // the group's rows
    int cut, parts, part, first_pair;   // a cut tile: its number among the tail's tiles, its parts, this one, the pair of part 0
};

// LORA: the first request of a tile, the k-blocks of the one that has all of its rows, how many have some of them
struct GroupedRequests {
    int first, whole, parts;
};

__device__ __forceinline__ int round32(int x) { return (x + 31) & ~31; }

// One 32 x 32 piece of C, lane l holding feature l, v[j] row j.  Where all of its rows are stored it goes through
// shared memory: a TMA store writes the box (and clips what lies beyond C's edges), which takes a third of the
// instructions of stores from registers; with a short contraction the epilogue's issue slots bound the kernel.
//
// 16-bit results: a lane packs its feature of rows j and j + 1 and exchanges words with its neighbour; even lanes then
// hold row j of features (l, l + 1), odd lanes row j + 1 of (l - 1, l): two rows of 64 bytes per store, no bank twice.
template <bool F16>
__device__ __forceinline__ void grouped_stage16(const float (&v)[32], uint32_t dst) {
    const uint32_t odd = threadIdx.x & 1, l = threadIdx.x & 31;
    const uint32_t pick = odd ? 0x3276u : 0x5410u;
    dst += odd * 64 + (l >> 1) * 4;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint32_t w = pack_half2(v[2 * j], v[2 * j + 1], F16);
        const uint32_t got = __shfl_xor_sync(~0u, w, 1);
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + j * 128), "r"(__byte_perm(w, got, pick)) : "memory");
    }
}
__device__ __forceinline__ void grouped_stage32(const float (&v)[32], uint32_t dst) {
    dst += (threadIdx.x & 31) * 4;
#pragma unroll
    for (int j = 0; j < 32; ++j) asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + j * 128), "r"(__float_as_uint(v[j])) : "memory");
}

// The rows [0, rows) of a piece from registers; c points at row 0, this lane's feature.
__device__ __forceinline__ void grouped_store_rows(const GroupedParams& p, const float (&v)[32], size_t at, int rows) {
    if (p.out16) {
        uint16_t* c = static_cast<uint16_t*>(p.C) + at;
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < rows) c[j * p.ldc] = static_cast<uint16_t>(pack_half2(v[j], 0.0f, p.f16) & 0xFFFFu);
    } else {
        float* c = static_cast<float*>(p.C) + at;
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < rows) c[j * p.ldc] = v[j];
    }
}

// h16: leading part and remainder of the scaled product; an infinite leading part has no remainder
__device__ __forceinline__ void grouped_store_h(const GroupedParams& p, const float (&v)[32], int row0, int i, int cols, float scale) {
    if (i >= p.rank_blocks * 32) return;
    uint16_t* h = p.h16 + static_cast<size_t>(row0) * (p.rank_blocks * 64) + (i >> 5) * 64 + (i & 31);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (j >= cols) break;
        const float x = i < p.I ? v[j] * scale : 0.0f;
        const uint32_t hi = pack_half2(x, 0.0f, p.f16) & 0xFFFFu;
        const float back = half_bits_to_f32(hi, p.f16);
        const uint32_t lo = fabsf(back) <= 3.4028235e38f ? pack_half2(x - back, 0.0f, p.f16) & 0xFFFFu : 0u;
        h[static_cast<size_t>(j) * (p.rank_blocks * 64)] = static_cast<uint16_t>(hi);
        h[static_cast<size_t>(j) * (p.rank_blocks * 64) + 32] = static_cast<uint16_t>(lo);
    }
}

// MODE: GroupedMode.  A_MN: the features' operand is MN-major (row-major weights [K][I], or rows [t][I]), else
// K-major (weights [I][K]).
template <int MODE, bool A_MN>
__global__ void __launch_bounds__(GRP_THREADS, 1) __cluster_dims__(2, 1, 1)
grouped_kernel(const __grid_constant__ GroupedMaps maps, const __grid_constant__ GroupedParams p) {
    constexpr bool WEIGHTS = MODE == GRP_WEIGHTS, LORA = MODE == GRP_LORA;
    static_assert(!WEIGHTS || A_MN, "rows are contiguous in their features");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
    int* s_row = reinterpret_cast<int*>(gen_base + GRP_STAGES * GRP_STAGE + GRP_STAGING);   // first row of each group (LORA: request), clamped and monotone
    int* s_pre = s_row + GRP_MAX_GROUPS + 1;                                  // tiles before each group
    int* s_alt = s_pre + GRP_MAX_GROUPS + 1;                                  // ROWS: weight of the group; LORA: adapter of the request; -1: none.  WEIGHTS: k-blocks before each group
    const uint32_t bar_base = smem_base + GRP_STAGES * GRP_STAGE + GRP_STAGING + 3 * GRP_TABLE + 4;   // (8-byte aligned: a table is 4 mod 8 bytes)
    constexpr int S = GRP_STAGES;
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };
    auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * S + a); };
    auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * S + 2 + a); };
    auto raw_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + s); };    // a block with rows to clear: this CTA's boxes have landed
    auto tail_bar = [&](int s) { return bar_base + 8u * (3 * S + 4 + s); };   // leader: both CTAs have cleared theirs
    constexpr int NB = 4 * S + 4;
    static_assert(NB <= 32, "one barrier per lane");
    static_assert((3 * GRP_TABLE + 4) % 8 == 0, "barriers are 8-byte aligned");
    const uint32_t peer_ready_bar = bar_base + 8u * NB;
    uint8_t* after = gen_base + (bar_base - smem_base) + 8 * (NB + 1);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(after);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile int* s_most = reinterpret_cast<volatile int*>(after + 8);       // rows of the largest group

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair_id = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    auto give_up = [&](unsigned int code) {
        *abort_flag = 1;
        if (p.status) atomicCAS(p.status, 0u, code);
    };

    // offsets -> shared memory (LORA: the requests'; its one group is all the rows)
    const int* offsets = LORA ? p.request_offsets : p.offsets;
    const int entries = LORA ? p.requests : p.groups;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int g = threadIdx.x; g <= entries; g += GRP_THREADS) {
        s_row[g] = offsets ? offsets[g] : g == 0 ? 0 : p.rows;
        if (!WEIGHTS) {
            const int a = p.index && g < entries ? p.index[g] : g;
            s_alt[g] = p.index && (a < 0 || a >= p.index_max) ? -1 : a;
        }
    }
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
        tma_prefetch_desc(&maps.a);
        tma_prefetch_desc(&maps.b[0]);
    } else if (warp == 1) {
        tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 2) {
        // running maximum of the clamped offsets, then the prefix of the tile counts
        int top = 0, units = 0, blocks = 0, most = 0;
        bool bad = false;
        for (int base = 0; base <= entries; base += 32) {
            const int g = base + lane;
            const int raw = g <= entries ? s_row[g] : 0;
            int v = min(max(raw, 0), p.rows);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v = max(v, o);
            }
            v = max(v, top);
            if (g <= entries) {
                bad |= v != raw;
                s_row[g] = v;
            }
            top = __shfl_sync(~0u, v, 31);
        }
        if (__any_sync(~0u, bad) && lane == 0 && blockIdx.x == 0 && p.status) atomicCAS(p.status, 0u, 0x10000u);
        __syncwarp();
        for (int base = 0; !LORA && base <= p.groups; base += 32) {
            const int g = base + lane;
            const int rows = g < p.groups ? s_row[g + 1] - s_row[g] : 0;
            most = max(most, rows);
            const int n = g >= p.groups ? 0 : WEIGHTS ? p.tiles_i * p.tiles_j : s_alt[g] < 0 ? 0 : (rows + GRP_TILE - 1) / GRP_TILE * p.tiles_i;
            const int b = WEIGHTS ? n * max(1, (rows + GRP_BK - 1) / GRP_BK) : 0;
            int v = n, w = b;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d), x = __shfl_up_sync(~0u, w, d);
                if (lane >= d) { v += o; w += x; }
            }
            if (g <= p.groups) {
                s_pre[g] = units + v - n;
                if (WEIGHTS) s_alt[g] = blocks + w - b;
            }
            units += __shfl_sync(~0u, v, 31);
            blocks += __shfl_sync(~0u, w, 31);
        }
        if (LORA) {
            most = p.rows;
            if (lane == 0) { s_pre[0] = 0; s_pre[1] = (p.rows + GRP_TILE - 1) / GRP_TILE * p.tiles_i; }
        }
        most = static_cast<int>(__reduce_max_sync(~0u, static_cast<unsigned>(most)));
        if (lane == 0) *s_most = most;
    }
    cluster_arrive();
    cluster_wait();          // the barriers of both CTAs are initialised
    __syncthreads();         // the prefix is there
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    if (warp == 1 && rank == 1 && lane == 0) mbar_arrive_cluster_cta_release(map_to_cta(peer_ready_bar, 0));

    // ---------------------------------------------------- the schedule
    const int tiles = s_pre[p.groups];
    const int most_kbs = WEIGHTS ? (*s_most + GRP_BK - 1) / GRP_BK : p.kb_total;      // k-blocks of the longest tile
    // whole tiles in turn, then the tail [tail_from, tiles): `tail_len` k-blocks, `share` of them to each pair
    const int full_waves = tiles / num_pairs;
    int tail_from = tiles, tail_len = 0, share = 0, tail_base = 0;
    if (p.partial && tiles > full_waves * num_pairs) {
        const int from = full_waves > 1 ? (full_waves - 1) * num_pairs : 0;
        if (WEIGHTS) {
            int lo = 0, hi = p.groups;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_pre[mid] <= from) lo = mid;
                else hi = mid;
            }
            tail_base = s_alt[lo] + (from - s_pre[lo]) * max(1, (s_row[lo + 1] - s_row[lo] + GRP_BK - 1) / GRP_BK);
            tail_len = s_alt[p.groups] - tail_base;
        } else {
            tail_len = (tiles - from) * p.kb_total;
        }
        share = max(4, (tail_len + num_pairs - 1) / num_pairs);
        // a cut tile writes its sums to memory and reads them back: about as long as 8 k-blocks, and one more for
        // every 32 columns
        const int rounds = (tiles - from + num_pairs - 1) / num_pairs;
        const int columns = WEIGHTS ? min(p.J, GRP_TILE) : min(*s_most, GRP_TILE);
        if (rounds * most_kbs - share > 8 + columns / 32) tail_from = from;
    }
    const int tail_lo = pair_id * share, tail_hi = min(tail_lo + share, tail_len);
    // n counts this pair's whole tiles, x is its place in the tail
    int next_tile = pair_id, x = tail_lo;
    auto reset = [&]() { next_tile = pair_id; x = tail_lo; };
    auto next = [&](GroupedUnit& u) -> bool {
        int tile;
        u.cut = -1;
        u.parts = 1;
        u.part = 0;
        u.first_pair = 0;
        int at = 0;                                       // k-block of the tile to begin with
        if (next_tile < tail_from) {
            tile = next_tile;
            next_tile += num_pairs;
        } else {
            if (tail_from == tiles || x >= tail_hi) return false;
            if (WEIGHTS) {
                const int y = tail_base + x;
                int lo = 0, hi = p.groups;                // s_alt[lo] <= y < s_alt[hi]
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_alt[mid] <= y) lo = mid;
                    else hi = mid;
                }
                const int len = max(1, (s_row[lo + 1] - s_row[lo] + GRP_BK - 1) / GRP_BK);
                const int rel = (y - s_alt[lo]) / len;
                tile = s_pre[lo] + rel;
                at = y - s_alt[lo] - rel * len;
            } else {
                const int rel = x / p.kb_total;
                tile = tail_from + rel;
                at = x - rel * p.kb_total;
            }
        }
        if (WEIGHTS) {
            const int per = p.tiles_i * p.tiles_j;
            u.g = div_small(tile, per);
            u.w = 0;
            const int rel = tile - u.g * per;
            const int ti = div_small(rel, p.tiles_j);
            u.i0 = ti * GRP_TILE;
            u.c0 = (rel - ti * p.tiles_j) * GRP_TILE;
            u.cols = min(GRP_TILE, p.J - u.c0);
            u.row0 = s_row[u.g];
            u.rows = s_row[u.g + 1] - u.row0;
            u.kbs = (u.rows + GRP_BK - 1) / GRP_BK;
        } else {
            int lo = 0, hi = p.groups;                    // s_pre[lo] <= tile < s_pre[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_pre[mid] <= tile) lo = mid;
                else hi = mid;
            }
            u.g = lo;
            u.w = LORA ? 0 : s_alt[lo];
            const int rel = tile - s_pre[lo];
            u.row0 = LORA ? 0 : s_row[lo];
            u.rows = LORA ? p.rows : s_row[lo + 1] - u.row0;
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
            u.kbs = p.kb_total;
        }
        u.jn = round32(u.cols);
        u.kb0 = 0;
        u.kb1 = u.kbs;
        if (tile >= tail_from) {
            const int len = max(1, u.kbs), start = x - at;            // the tile's place in the tail
            u.kb0 = min(at, u.kbs);
            u.kb1 = min(u.kbs, at + tail_hi - x);
            x += min(len - at, tail_hi - x);
            u.first_pair = start / share;
            const int last_pair = (start + len - 1) / share;
            u.parts = last_pair - u.first_pair + 1;
            u.part = pair_id - u.first_pair;
            u.cut = tile - tail_from;
        }
        return true;
    };
    // WEIGHTS: rows of the group in k-block kb
    auto rows_of = [&](const GroupedUnit& u, int kb) { return min(GRP_BK, u.rows - kb * GRP_BK); };

    // LORA: the requests' blocks follow the last k-block of a tile.  A request that has all of the tile's rows goes into
    // the tile's own accumulator.  Of the others each gets an accumulator of its own, of which the epilogue adds the
    // request's columns to the tile's sum: an adapter of infinities or NaN cannot reach another request's rows.
    auto first_request = [&](const GroupedUnit& u) {
        int lo = 0, hi = p.requests;                      // the first q with s_row[q + 1] > c0
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_row[mid + 1] > u.c0) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    };
    auto in_tile = [&](const GroupedUnit& u, int q) { return q < p.requests && s_row[q] < u.c0 + u.cols; };
    auto has_part = [&](int q) { return s_alt[q] >= 0 && s_row[q + 1] > s_row[q]; };
    auto look = [&](const GroupedUnit& u) {
        GroupedRequests r = {0, 0, 0};
        if (!LORA || u.kb1 != u.kbs) return r;
        r.first = first_request(u);
        if (r.first >= p.requests) return r;
        if (s_row[r.first] <= u.c0 && s_row[r.first + 1] >= u.c0 + u.cols) {
            r.whole = s_alt[r.first] >= 0 ? p.rank_blocks : 0;
            return r;
        }
        int n = 0;
        for (int q = r.first + lane; in_tile(u, q); q += 32) n += has_part(q) ? 1 : 0;
        r.parts = static_cast<int>(__reduce_add_sync(~0u, static_cast<unsigned>(n)));
        return r;
    };

    if (warp == 0) {
        // ------------------------------------------------ TMA producer (both CTAs)
        const uint32_t lead_full0 = map_to_cta(full_bar(0), 0);
        const uint32_t elected = elect_one();
        const uint32_t lead_elected = rank == 0 ? elected : 0u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true, waited = false;
        GroupedUnit u = {};
        reset();
        while (ok && next(u)) {
            const int half = u.jn >> 1;
            const int i = u.i0 + static_cast<int>(rank) * 128;
            const int c = u.c0 + static_cast<int>(rank) * half;      // first column of this CTA's B operand
            const int boxes = (half + 63) >> 6;                       // WEIGHTS
            const uint32_t b_bytes = WEIGHTS ? boxes * 8192u : half * 128u;
            // half rows (a multiple of 16, up to 128) of 128 bytes each, in the fewest boxes of 16, 32, 64 or 128 rows
            auto rows_boxes = [&](const CUtensorMap (&map)[4], uint32_t dst, uint32_t bar, int x0) {
                int row = c;
#pragma unroll
                for (int z = 3; z >= 0; --z)
                    if (half & (16 << z)) {
                        tma_load_3d_pair_if(dst, &map[z], bar, x0, row, 0, elected);
                        dst += 2048u << z;
                        row += 16 << z;
                    }
            };
            auto acquire = [&]() {
                if (mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) return true;
                if (lane == 0) give_up(0x100u + stage);
                return false;
            };
            auto advance = [&]() {
                __syncwarp();
                if (++stage == S) { stage = 0; phase ^= 1u; }
            };
            for (int kb = u.kb0; kb < u.kb1; ++kb) {
                if (!acquire()) { ok = false; break; }
                const uint32_t sa = smem_base + stage * GRP_STAGE, sb = sa + GRP_A_BYTES;
                const uint32_t fb = full_bar(stage), lfb = lead_full0 + 8u * stage;
                const uint32_t bytes = GRP_A_BYTES + b_bytes;
                if (WEIGHTS) {
                    const int t = u.row0 + kb * GRP_BK;
                    if (rows_of(u, kb) & 15) {
                        // on this CTA's own barrier: warp 10 clears what belongs to the next group, then reports to the leader
                        mbar_arrive_expect_tx_if(raw_bar(stage), bytes, elected);
                        if (rank == 0 && elected) mbar_arrive(fb);
                        __syncwarp();
                        if (p.a_slabs) {
                            tma_load_4d_if(sa, &maps.a, raw_bar(stage), 0, t, i >> 6, 0, elected);
                        } else {
                            tma_load_3d_if(sa, &maps.a, raw_bar(stage), i, t, 0, elected);
                            tma_load_3d_if(sa + 8192, &maps.a, raw_bar(stage), i + 64, t, 0, elected);
                        }
                        for (int b = 0; b < boxes; ++b) tma_load_3d_if(sb + b * 8192, &maps.b[0], raw_bar(stage), c + b * 64, t, 0, elected);
                    } else {
                        mbar_arrive_expect_tx_if(fb, 2u * bytes, lead_elected);
                        if (p.a_slabs) {
                            tma_load_4d_pair_if(sa, &maps.a, lfb, 0, t, i >> 6, 0, elected);
                        } else {
                            tma_load_3d_pair_if(sa, &maps.a, lfb, i, t, 0, elected);
                            tma_load_3d_pair_if(sa + 8192, &maps.a, lfb, i + 64, t, 0, elected);
                        }
                        if (p.b_slabs && half == 128) {
                            tma_load_4d_pair_if(sb, &maps.b[1], lfb, 0, t, c >> 6, 0, elected);
                        } else {
                            for (int b = 0; b < boxes; ++b) tma_load_3d_pair_if(sb + b * 8192, &maps.b[0], lfb, c + b * 64, t, 0, elected);
                        }
                    }
                } else {
                    const int kx = kb * GRP_BK;
                    mbar_arrive_expect_tx_if(fb, 2u * bytes, lead_elected);
                    if (A_MN && p.a_slabs) {
                        tma_load_4d_pair_if(sa, &maps.a, lfb, 0, kx, i >> 6, u.w, elected);
                    } else if (A_MN) {
                        tma_load_3d_pair_if(sa, &maps.a, lfb, i, kx, u.w, elected);
                        tma_load_3d_pair_if(sa + 8192, &maps.a, lfb, i + 64, kx, u.w, elected);
                    } else {
                        tma_load_3d_pair_if(sa, &maps.a, lfb, kx, i, u.w, elected);
                    }
                    rows_boxes(maps.b, sb, lfb, kx);
                }
                advance();
            }
            const GroupedRequests r = look(u);
            if (LORA && ok && r.whole + r.parts > 0) {
                // h16 comes from the kernel before this one
                if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
                waited = true;
                const uint32_t bytes = (A_MN ? 8192u : GRP_A_BYTES) + b_bytes;
                int q = r.first;
                for (int n = 0; ok && n < max(1, r.parts); ++n, ++q) {
                    while (!r.whole && !has_part(q)) ++q;
                    for (int rb = 0; rb < p.rank_blocks; ++rb) {
                        if (!acquire()) { ok = false; break; }
                        const uint32_t sa = smem_base + stage * GRP_STAGE, sb = sa + GRP_A_BYTES, lfb = lead_full0 + 8u * stage;
                        mbar_arrive_expect_tx_if(full_bar(stage), 2u * bytes, lead_elected);
                        if (A_MN) {
                            tma_load_3d_pair_if(sa, &maps.c, lfb, i, rb * 32, s_alt[q], elected);
                            tma_load_3d_pair_if(sa + 8192, &maps.c, lfb, i + 64, rb * 32, s_alt[q], elected);
                        } else {
                            tma_load_3d_pair_if(sa, &maps.c, lfb, rb * 32, i, s_alt[q], elected);
                        }
                        rows_boxes(maps.h, sb, lfb, rb * 64);
                        advance();
                    }
                }
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
            int stage = 0, local = 0;                     // local: accumulators filled so far
            uint32_t phase = 0, tail_phase = 0;
            bool ok = true;
            if (!mbar_wait(peer_ready_bar, 0u, abort_flag)) {
                if (lane == 0) give_up(0x700u);
                ok = false;
            }
            GroupedUnit u;
            reset();
            while (ok && next(u)) {
                const uint32_t idesc = p.idesc | (static_cast<uint32_t>(u.jn >> 3) << 17);
                const GroupedRequests r = look(u);
                const int base = u.kb1 - u.kb0, own = base + r.whole, blocks = own + r.parts * p.rank_blocks;
                const int chunk = p.chunk ? p.chunk : own;
                int in_chunk = 0, rb = 0;
                uint32_t d_tmem = 0;
                if (blocks == 0) {                        // (an empty group's gradient: the epilogue stores zeros)
                    const int acc = local & 1;
                    if (!mbar_wait(tempty_bar(acc), ((local >> 1) & 1u) ^ 1u, abort_flag)) {
                        if (lane == 0) give_up(0x200u + acc);
                        break;
                    }
                    umma_commit_pair_if(tfull_bar(acc), 3, elected);
                    ++local;
                    continue;
                }
                for (int n = 0; n < blocks; ++n) {
                    const int acc = local & 1;
                    if (in_chunk == 0) {
                        if (!mbar_wait(tempty_bar(acc), ((local >> 1) & 1u) ^ 1u, abort_flag)) {
                            if (lane == 0) give_up(0x200u + acc);
                            ok = false;
                            break;
                        }
                        tc_fence_after_sync();
                        d_tmem = tmem_base + acc * GRP_TILE;
                    }
                    const uint32_t accumulate = in_chunk > 0;
                    if (!mbar_wait(full_bar(stage), phase, abort_flag)) {
                        if (lane == 0) give_up(0x300u + stage);
                        ok = false;
                        break;
                    }
                    int steps = 4;
                    bool cleared = false;
                    const bool low_rank = LORA && n >= base;
                    if (WEIGHTS) {
                        const int rem = rows_of(u, u.kb0 + n);
                        steps = (rem + 15) >> 4;
                        cleared = rem & 15;
                    }
                    if (low_rank) {
                        steps = min(2, (p.rank - 32 * rb + 15) >> 4);
                        if (++rb == p.rank_blocks) rb = 0;
                    }
                    if (WEIGHTS && cleared) {
                        if (!mbar_wait(tail_bar(stage), (tail_phase >> stage) & 1u, abort_flag)) {
                            if (lane == 0) give_up(0x600u + stage);
                            ok = false;
                            break;
                        }
                        tail_phase ^= 1u << stage;
                    }
                    tc_fence_after_sync();
                    const uint32_t a_lo = a_lo0 + stage * (GRP_STAGE >> 4), b_lo = b_lo0 + stage * (GRP_STAGE >> 4);
                    umma_pair_if<0>(d_tmem, a_lo, a_hi, b_lo, b_hi, idesc, accumulate, elected);
                    if (low_rank) {
                        // 32 ranks: leading parts of h16 in the first 64 bytes of a row, remainders in the second
                        if (steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + b_s, b_hi, idesc, 1u, elected);
                        umma_pair_if<0>(d_tmem, a_lo, a_hi, b_lo + 2 * b_s, b_hi, idesc, 1u, elected);
                        if (steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + 3 * b_s, b_hi, idesc, 1u, elected);
                    } else {
                        if (!WEIGHTS || steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + b_s, b_hi, idesc, 1u, elected);
                        if (!WEIGHTS || steps > 2) umma_pair_if<0>(d_tmem, a_lo + 2 * a_s, a_hi, b_lo + 2 * b_s, b_hi, idesc, 1u, elected);
                        if (!WEIGHTS || steps > 3) umma_pair_if<0>(d_tmem, a_lo + 3 * a_s, a_hi, b_lo + 3 * b_s, b_hi, idesc, 1u, elected);
                    }
                    umma_commit_pair_if(empty_bar(stage), 3, elected);
                    if (++in_chunk == chunk || n == own - 1 || (LORA && n >= own && rb == 0)) {
                        umma_commit_pair_if(tfull_bar(acc), 3, elected);
                        in_chunk = 0;
                        ++local;
                    }
                    __syncwarp();
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp < 10) {
        // ------------------------------------------------ epilogue (both CTAs, own 128 features)
        const int set = warp >= 6 ? 1 : 0;
        const int quarter = warp & 3;
        const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t staging = smem_base + S * GRP_STAGE + (warp - 2) * 4096;
        uint32_t parity = 0;
        int local = 0;
        bool ok = true, waited = false;
        GroupedUnit u = {};
        auto await = [&]() {
            const int acc = local & 1;
            if (!mbar_wait(tfull_bar(acc), (local >> 1) & 1u, abort_flag)) {
                if (lane == 0) give_up(0x400u + acc);
                return false;
            }
            tc_fence_after_sync();
            return true;
        };
        auto release = [&]() {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_cta_release(map_to_cta(tempty_bar(local & 1), 0));
            ++local;
        };
        // one 32 x 32 piece (columns c .. c + 31 of the tile, this warp's 32 features) of a tile or of one part of a cut one
        auto deliver = [&](float (&v)[32], int c) {
            if (u.parts > 1) {
                const size_t slab = static_cast<size_t>(GRP_TILE) * p.slab_cols;
                const size_t at = (rank * static_cast<size_t>(p.slab_cols) + c) * 128 + quarter * 32 + lane;
                // the slab of a pair: 0 for the tile its share begins in, 1 for the one it ends in
                auto slab_of = [&](int part) { return p.partial + (2 * (u.first_pair + part) + (part > 0 ? 0 : 1)) * slab + at; };
                float* mine = slab_of(u.part);
#pragma unroll
                for (int j = 0; j < 32; ++j) __stcg(mine + j * 128, v[j]);
                __threadfence();
                __syncwarp();
                unsigned int* counter = p.counter + (u.cut * 2 + rank) * 8 + (c >> 5);
                unsigned int old = 0;
                if (lane == 0) old = (atomicAdd(counter, 1u << (8 * quarter)) >> (8 * quarter)) & 255u;
                old = __shfl_sync(~0u, old, 0);
                if (old != static_cast<unsigned>(u.parts) - 1u) return;
                if (lane == 0) atomicSub(counter, static_cast<unsigned>(u.parts) << (8 * quarter));
                __threadfence();
                const float* src = slab_of(0);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __ldcg(src + j * 128);
#pragma unroll 1
                for (int s = 1; s < u.parts; ++s) {
                    src = slab_of(s);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += __ldcg(src + j * 128);
                }
            }
            const int i = u.i0 + static_cast<int>(rank) * 128 + quarter * 32 + lane;
            const int n = min(32, u.cols - c);
            if (MODE == GRP_ROWS && p.h16) {
                grouped_store_h(p, v, u.c0 + c, i, n, __ldg(p.scale + u.w));
                return;
            }
            const bool live = i < p.I;
            if (MODE == GRP_ROWS && p.add) {
                if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");   // `add` comes from the kernel before this one
                waited = true;
                const float* add = p.add + static_cast<size_t>(u.c0 + c) * p.I + i;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (live && j < n) v[j] += add[static_cast<size_t>(j) * p.I];
            }
            const size_t base = (WEIGHTS ? static_cast<size_t>(u.g) * p.stride_c : 0) + static_cast<size_t>(u.c0 + c) * p.ldc + i;
            if (p.beta && live) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j < n)
                        v[j] += p.out16 ? half_bits_to_f32(static_cast<const uint16_t*>(p.C)[base + j * p.ldc], p.f16)
                                        : static_cast<const float*>(p.C)[base + j * p.ldc];
            }
            if (!WEIGHTS && n < 32) {                     // the next row is another group's
                grouped_store_rows(p, v, base, live ? n : 0);
                return;
            }
            // two boxes of 16-bit, one of 32-bit results fit this warp's 4 KB: wait until the store of the one before has been read
            const uint32_t box = staging + (p.out16 ? parity * 2048 : 0);
            if (lane == 0) {
                if (p.out16) bulk_wait_read<1>();
                else bulk_wait_read<0>();
            }
            __syncwarp();
            if (!p.out16) grouped_stage32(v, box);
            else if (p.f16) grouped_stage16<true>(v, box);
            else grouped_stage16<false>(v, box);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                tma_store_3d(&maps.out, box, i - lane, u.c0 + c, WEIGHTS ? u.g : 0);
                bulk_commit();
            }
            parity ^= 1u;
        };
        reset();
        while (ok && next(u)) {
            const GroupedRequests r = look(u);
            // the accumulators that make up the tile: chunks of its own k-blocks, then one for each request with some of its rows
            const int blocks = u.kb1 - u.kb0 + r.whole;
            const int chunks = p.chunk ? max(1, (blocks + p.chunk - 1) / p.chunk) : 1, all = chunks + r.parts;
            if (!await()) break;
            if (all > 1) {
                // all but the last are added in registers, and the sum goes back to the last one's place
                float sum[4][32];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[q][j] = 0.0f;
                int at = r.first;
#pragma unroll 1
                for (int n = 0; n < all; ++n) {
                    int lo = 0, hi = u.cols;              // the columns this accumulator has something for
                    if (LORA && n >= chunks) {
                        while (!has_part(at)) ++at;
                        lo = s_row[at] - u.c0;
                        hi = min(hi, s_row[at + 1] - u.c0);
                        ++at;
                    }
                    const uint32_t taddr = tmem_base + (local & 1) * GRP_TILE + lane_addr;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = set * 32 + q * 64;
                        if (c < hi && c + 32 > lo) {
                            uint32_t v[32];
                            tmem_ld_32x32(taddr + c, v);
                            tmem_ld_wait();
                            if (!LORA || (c >= lo && c + 32 <= hi)) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) sum[q][j] += __uint_as_float(v[j]);
                            } else {
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (c + j >= lo && c + j < hi) sum[q][j] += __uint_as_float(v[j]);
                            }
                        }
                    }
                    if (n < all - 1) {
                        release();
                        if (!await()) { ok = false; break; }
                    }
                }
                if (!ok) break;
                const uint32_t taddr = tmem_base + (local & 1) * GRP_TILE + lane_addr;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = set * 32 + q * 64;
                    if (c < u.cols) {
                        uint32_t v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(sum[q][j]);
                        tmem_st_32x32(taddr + c, v);
                    }
                }
                tmem_st_wait();
            }
            const uint32_t taddr = tmem_base + (local & 1) * GRP_TILE + lane_addr;
            // the parts of a cut tile begin with different columns, so that each finishes some of them last
            const int mine = (u.cols - set * 32 + 63) >> 6;
#pragma unroll 1
            for (int n = 0; n < mine; ++n) {
                int q = n + u.part;
                while (q >= mine) q -= mine;
                const int c = set * 32 + q * 64;
                uint32_t v[32];
                float f[32];
                tmem_ld_32x32(taddr + c, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
                if (WEIGHTS && blocks == 0) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = 0.0f;
                }
                deliver(f, c);
            }
            release();
        }
        if (lane == 0) bulk_wait_read<0>();               // the stores are done with this CTA's shared memory
        __syncwarp();
    } else if (WEIGHTS) {
        // ------------------------------------------------ rows of the next group in a group's last k-block
        const uint32_t lead_tail0 = map_to_cta(tail_bar(0), 0);
        int stage = 0;
        uint32_t raw_phase = 0;
        GroupedUnit u = {};
        reset();
        while (next(u)) {
            if (u.kb1 <= u.kb0) continue;
            stage = (stage + u.kb1 - u.kb0 - 1) % S;
            const int rem = rows_of(u, u.kb1 - 1);
            if (rem & 15) {
                if (!mbar_wait(raw_bar(stage), (raw_phase >> stage) & 1u, abort_flag)) {
                    if (lane == 0) give_up(0x500u + stage);
                    break;
                }
                raw_phase ^= 1u << stage;
                const int boxes = 2 + ((u.jn >> 1) + 63) / 64;
                const int first = rem * 8, last = ((rem + 15) & ~15) * 8;   // 16-byte pieces of a box's rows of 128 bytes
                for (int b = 0; b < boxes; ++b)
                    for (int y = first + lane; y < last; y += 32)
                        st_shared_v4(smem_base + stage * GRP_STAGE + b * 8192 + y * 16, 0u, 0u, 0u, 0u);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_cta_release(lead_tail0 + 8u * stage);
            }
            stage = (stage + 1) % S;
        }
    }

    if (warp == 0) asm volatile("griddepcontrol.wait;" ::: "memory");   // this launch ends after the one before it, whatever it read
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

}  // namespace nk
