// Products of 4-bit operands with block scales, of all rows with one weight or grouped by expert:
//   C[t][i] = ta tb sum_k X[t][k] W_g[i][k]      for the rows t of group g
// The shape of the kernel is that of the grouped products (grouped.cuh): the features are the MMA's M dimension and the ragged rows
// its N, a CTA pair computes 256 features x up to 256 rows, the groups' offsets are read on the device by a scheduler warp, and
// of one group the plan may have the tiles of the last, partial wave cut along k.  What is different:
//
// A k-block is 256 elements (128 bytes of a row), four MMAs of 64.  Its scales arrive by TMA as the tiles of 128 rows x 4 blocks that
// tensor memory wants and go there by tcgen05.cp, from a warp of its own that is some k-blocks ahead of the MMAs.  (Issued by the MMAs' warp the
// copies, twelve to a k-block of NVF4, took a third of its time: 8192^3 264 us, from their own warp 230.)  Each CTA has the scales of
// its own 128 features and of all the tile's rows.
//
// Tensor memory: two accumulators of 256 columns would leave no room for the scales.  So for tiles of more than 128 rows they share
// columns (NVF4 144, MXF4 96).  The epilogue takes the shared columns of an accumulator first, into
// registers, and gives them back; the next tile may begin then, while the rest is taken and stored.
//
// Tiles begin at multiples of 64 rows of a group (or at its first row): scales of 64 rows are two columns, by which the place of the
// rows' scales moves where a tile begins in the middle of 128.
//
// Warps: eight or sixteen of the epilogue (see mx_sets), in sets of four for the quarters of the lanes, which take the 32-column pieces in turn; then
// the TMA producer, the MMA issuer, one that copies the scales, the scheduler.
// All waits are bounded (see mbar_wait).
//
// Bound by the SMs' feed from L2, 46 bytes a clock: a k-block of 256 x 256 takes 0.45 us, the MMAs 0.28.  8192^3 to BF16: NVF4
// 198 to 206 us (5.4 PFLOP/s), MXF4 189 (5.8); without pauses 240, the power cap's.  8192 x 4096 x 1024 29 us.  Few rows wait for their
// weights: 16 x 16384 x 16384 31 us (4.9 TB/s), 16 x 4096 x 4096 9.2 (5.0 with one k-block, 0.27 for each more), 64 experts of 4096 x 1024 with 32
// rows 15.7.  Short contractions wait for the epilogue, whose stores are two bytes a lane: 8192 x 4096 x 1024 takes 3.5 us a tile, its feed 1.8.
#pragma once
#include "grouped.cuh"
#include "mx_format.cuh"
#include "mx_launch.cuh"

namespace nk {

// One piece of work: k-blocks kb0 .. kb1-1 of a tile.
struct __align__(16) MxUnit {
    int some;              // 0: no more work
    int g, i0;             // group (and its weight), first feature
    int c0, cols, jn;      // first row of C, rows of the tile, the MMA's N (rows rounded up to 32)
    int tile, shift;       // first tile of the rows' scales, columns before the first row's
    int kb0, kb1;
    int cut, parts, part, first_pair;   // a cut tile: its number among the tail's tiles, its parts, this one, the pair of part 0
};
constexpr int MX_UNITS = 4;             // of them on the way
// Tensor memory's columns.  A k-block's scales take a third of a place for the features and the rest for the rows; three places (NVF4) or four, so
// that copies are as far ahead of the MMAs as the ring of stages.  (With two, 8192^3 NVF4 took 230 us.)
__host__ __device__ constexpr int mx_places(bool nv) { return nv ? 3 : 4; }
__host__ __device__ constexpr int mx_place(bool nv) { return nv ? 48 : 24; }
__host__ __device__ constexpr int mx_scales(bool nv) { return 512 - mx_places(nv) * mx_place(nv); }    // first column of the scales
__host__ __device__ constexpr int mx_shared(bool nv) { return mx_scales(nv) - MX_TILE; }               // first of the columns that both accumulators have

// MODE: whole tiles only; tiles may be cut; they may be cut and be sums of several accumulators.
// A launch of 384 threads has 168 registers for each.  Sums take 128, so the epilogue's 256 threads get some of the others'
// (216 x 256 + 72 x 128 = 168 x 384; 4096 x 4096 x 16384 122 us, with 208 and 88 127, without 155, in 16 bits and one accumulator 104).
// The other kernels must do without, as the loops of the other warps are slower for it (4096 x 1024 x 4096 16.0 us instead of 14.0), and
// without spilling: there is next to no L1 beside this much shared memory (20 spilled registers: 8192 x 4096 x 256 38 us instead of 25).
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(MX_MORE_REGISTERS)); }
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(MX_FEWER_REGISTERS)); }

template <bool NV, int OUT, int MODE>
__global__ void __launch_bounds__(mx_threads(MODE, NV), 1) __cluster_dims__(2, 1, 1)
mx_kernel(const __grid_constant__ MxMaps maps, const __grid_constant__ MxParams p) {
    constexpr bool OUT16 = OUT != MX_OUT_F32, F16 = OUT == MX_OUT_F16;
    constexpr int SIZE = OUT16 ? 2 : 4;
    constexpr bool SUMS = MODE == MX_SUMS, CUT = MODE != MX_WHOLE_TILES;
    constexpr int SETS = mx_sets(MODE, NV), EPILOGUE = 4 * SETS, SPAN = 32 * SETS;       // sets of epilogue warps, warps, columns between a warp's pieces
    constexpr int PRODUCER = EPILOGUE, ISSUER = EPILOGUE + 1, COPIER = EPILOGUE + 2, SCHEDULER = EPILOGUE + 3;
    constexpr int S_BOX = NV ? 2048 : 1024;               // scales of 128 rows and a k-block
    constexpr int PLACES = mx_places(NV), PLACE = mx_place(NV), SCALES = mx_scales(NV), SHARED = mx_shared(NV);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
    int* s_row = reinterpret_cast<int*>(gen_base + MX_RING);   // first row of each group, clamped and monotone
    int* s_pre = s_row + MX_MAX_GROUPS + 1;                                  // tiles before each group
    const uint32_t bar_base = smem_base + MX_RING + 2 * MX_TABLE;
    static_assert(2 * MX_TABLE % 8 == 0, "barriers are 8-byte aligned");
    constexpr int MS = MX_MAX_STAGES;
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (MS + s); };
    auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * MS + a); };
    auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * MS + 2 + a); };
    auto ufull_bar = [&](int n) { return bar_base + 8u * (2 * MS + 4 + n); };    // a unit is there
    auto uempty_bar = [&](int n) { return bar_base + 8u * (2 * MS + 4 + MX_UNITS + n); };   // every role has read it
    auto sready_bar = [&](int n) { return bar_base + 8u * (2 * MS + 4 + 2 * MX_UNITS + n); };   // scales are in place n
    constexpr int NB = 2 * MS + 4 + 2 * MX_UNITS + PLACES;
    const uint32_t peer_ready_bar = bar_base + 8u * NB;
    uint8_t* after = gen_base + (bar_base - smem_base) + 8 * (NB + 1);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(after);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile int* s_width = reinterpret_cast<volatile int*>(after + 8);      // rows of a tile at most
    MxUnit* s_unit = reinterpret_cast<MxUnit*>(gen_base + ((MX_RING + 2 * MX_TABLE + 8 * (NB + 1) + 12 + 15) & ~15));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair_id = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    auto give_up = [&](unsigned int code) {
        *abort_flag = 1;
        if (p.status) atomicCAS(p.status, 0u, code);
    };
    // after a wait that ran out: what is still on its way into shared memory, or at work on it, needs some microseconds, and the pair
    // ends together
    auto settle = [&]() {
        const long long t0 = clock64();
        while (clock64() - t0 < (1ll << 20)) __nanosleep(1000);
    };

    if (warp == PRODUCER) {
        for (int n = lane; n < NB; n += 32) {
            // tempty: one arrival per epilogue warp of both CTAs; uempty: producer, epilogue warps, the leader's issuer and copier
            const uint32_t count = n >= 2 * MS + 2 && n < 2 * MS + 4                                      ? 2 * EPILOGUE
                                   : n >= 2 * MS + 4 + MX_UNITS && n < 2 * MS + 4 + 2 * MX_UNITS ? EPILOGUE + 1 + 2 * (rank == 0)
                                                                                                         : 1;
            mbar_init(bar_base + 8u * n, count);
        }
        if (lane == 31) mbar_init(peer_ready_bar, 1);
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
        __syncwarp();
    } else if (warp == 0) {
        if (lane < MX_BOXES) tma_prefetch_desc(&maps.b[lane]);
        if (lane == 8) tma_prefetch_desc(&maps.a);
        if (lane == 9) tma_prefetch_desc(&maps.sa);
        if (lane == 10) tma_prefetch_desc(&maps.sb);
    } else if (warp == ISSUER) {
        tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    cluster_arrive();
    // up to here the launch may have run beside the end of the one before it in the stream
    launch_wait();
    launch_next();
    for (int g = threadIdx.x; g <= p.groups; g += mx_threads(MODE, NV)) s_row[g] = p.offsets ? p.offsets[g] : g == 0 ? 0 : p.rows;
    __syncthreads();
    cluster_wait();          // the barriers of both CTAs are initialised
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    if (warp == ISSUER && rank == 1 && lane == 0) mbar_arrive_cluster_cta_release(map_to_cta(peer_ready_bar, 0));

    // the roles' view of the schedule: wait for the next unit, read it, give its place back
    int unit_at = 0;
    uint32_t unit_phase = 0;
    auto next = [&](MxUnit& u) -> bool {
        if (!mbar_wait(ufull_bar(unit_at), unit_phase, abort_flag)) {
            if (lane == 0) give_up(0x800u + warp);
            return false;
        }
        u = s_unit[unit_at];
        __syncwarp();
        if (lane == 0) mbar_arrive(uempty_bar(unit_at));
        if (++unit_at == MX_UNITS) { unit_at = 0; unit_phase ^= 1u; }
        return u.some != 0;
    };
    // settled once the first unit is there: stages of the ring, and whether the accumulators share columns
    int stage_bytes = 0, S = 1, apart = 128;
    bool sharing = false;
    auto ring = [&]() {
        const int width = *s_width;
        stage_bytes = mx_stage_bytes(width);
        S = min(MS, MX_RING / stage_bytes);
        sharing = width > 128;
        apart = sharing ? SHARED : 128;
    };

    if (SUMS && warp >= EPILOGUE) fewer_registers();
    if (warp == COPIER) {
        // ------------------------------------------------ scales into tensor memory (leader only)
        if (rank == 0) {
            const uint64_t ds = make_smem_desc(smem_base, 16, 128, 0);
            const uint32_t s_hi = static_cast<uint32_t>(ds >> 32), s_lo0 = static_cast<uint32_t>(ds);
            const uint32_t elected = elect_one();
            int stage = 0;
            uint32_t phase = 0, place = 0;
            int count = 0;
            bool ok = mbar_wait(peer_ready_bar, 0u, abort_flag);
            MxUnit u;
            while (ok && next(u)) {
                ring();
                const uint32_t s_off = (MX_A_BYTES + *s_width * 64) >> 4;
                const bool two = u.shift * 32 + u.jn > 128;
                for (int kb = u.kb0; kb < u.kb1; ++kb) {
                    // what the place held before was used PLACES k-blocks ago: those MMAs have to be done (a stage given back says so)
                    const int old = stage >= PLACES ? stage - PLACES : stage - PLACES + S;
                    const bool free = count < PLACES || mbar_wait(empty_bar(old), stage >= PLACES ? phase : phase ^ 1u, abort_flag);
                    if (!free || !mbar_wait(full_bar(stage), phase, abort_flag)) {
                        if (lane == 0) give_up(0x500u + stage);
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    count = min(count + 1, PLACES);
                    const int steps = min(4, p.steps - 4 * kb);
                    const uint32_t s_lo = s_lo0 + stage * (stage_bytes >> 4) + s_off;
                    const uint32_t sa_t = tmem_base + SCALES + place * PLACE, sb_t = sa_t + PLACE / 3;
                    // tiles of scales: four columns of the features' and four or eight of the rows', of one step (NV) or two
#pragma unroll
                    for (int s = 0; s < (NV ? 4 : 2); ++s) {
                        if (s > 0 && (NV ? s : 2 * s) >= steps) break;
                        tmem_copy_scales_pair_if(sa_t + 4 * s, s_lo + 32 * s, s_hi, elected);
                        tmem_copy_scales_pair_if(sb_t + 8 * s, s_lo + (MX_S_BYTES >> 4) + 32 * s, s_hi, elected);
                        if (two) tmem_copy_scales_pair_if(sb_t + 8 * s + 4, s_lo + (2 * MX_S_BYTES >> 4) + 32 * s, s_hi, elected);
                    }
                    umma_commit_pair_if(sready_bar(place), 1, elected);
                    if (++place == PLACES) place = 0;
                    __syncwarp();
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
            }
            if (*abort_flag) settle();
        }
    } else if (warp == SCHEDULER) {
        // ------------------------------------------------ scheduler (both CTAs of a pair come to the same schedule)
        // offsets that break their rule are clamped to the running maximum
        bool bad = false;
        for (int g = lane; g <= p.groups; g += 32) bad |= s_row[g] < (g ? s_row[g - 1] : 0) || s_row[g] > p.rows;
        if (__any_sync(~0u, bad)) {
            if (lane == 0) {
                if (blockIdx.x == 0 && p.status) atomicCAS(p.status, 0u, 0x10000u);
                int top = 0;
                for (int g = 0; g <= p.groups; ++g) s_row[g] = top = max(top, min(s_row[g], p.rows));
            }
            __syncwarp();
        }
        auto rows_in = [&](int g) { return s_row[g + 1] - s_row[g]; };
        // The width of the tiles: the plan's (one group), or that of the least estimated time of whole waves (lane l looks at 64 (l + 1) rows)
        int width = p.width;
        if (!width) {
            int most = 0;
            for (int g = lane; g < p.groups; g += 32) most = max(most, rows_in(g));
            most = static_cast<int>(__reduce_max_sync(~0u, static_cast<unsigned>(most)));
            width = most <= 32 ? 32 : 64;
            if (most > 64) {
                const int limit = min(MX_TILE, (most + 63) & ~63), w = min(64 * ((lane & 3) + 1), limit);
                int n = 0;
                for (int g = lane >> 2; g < p.groups; g += 8) n += (rows_in(g) + w - 1) / w;
                n += __shfl_xor_sync(~0u, n, 4);
                n += __shfl_xor_sync(~0u, n, 8);
                n += __shfl_xor_sync(~0u, n, 16);
                const float waves = static_cast<float>((n * p.tiles_i + num_pairs - 1) / num_pairs);
                const float t = waves * (static_cast<float>(p.kb_total) * static_cast<float>(mx_block_clocks(w)) + MX_TILE_CLOCKS) + static_cast<float>(MX_ROW_CLOCKS * w);
                // the smallest; of equals the widest: a time's upper bits, then the width
                const unsigned won = __reduce_min_sync(~0u, (__float_as_uint(t) & ~7u) | (4u - static_cast<unsigned>(w >> 6)));
                width = static_cast<int>(4u - (won & 7u)) << 6;
            }
        }
        if (lane == 0) *s_width = width;
        // tiles before each group
        int tiles = 0;
        for (int base = 0; base <= p.groups; base += 32) {
            const int g = base + lane;
            const int n = g >= p.groups ? 0 : (rows_in(g) + width - 1) / width * p.tiles_i;
            int v = n;
#pragma unroll 1
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v += o;
            }
            if (g <= p.groups) s_pre[g] = tiles + v - n;
            tiles += __shfl_sync(~0u, v, 31);
        }
        __syncwarp();
        // Whole tiles in turn, then the tail [tail_from, tiles), the last, partial wave: `tail_len` k-blocks, `share` of them to each pair; a
        // tile counts `padded` k-blocks there, a whole number of shares.
        const int from = tiles / num_pairs * num_pairs;
        int tail_from = tiles, tail_len = 0, share = 1, padded = p.kb_total;
        if (CUT && p.parts > 1) {
            tail_from = from;
            share = (p.kb_total + p.parts - 1) / p.parts;
            padded = (p.kb_total + share - 1) / share * share;
            tail_len = (tiles - from) * padded;
        }
        int next_tile = pair_id, x = pair_id * share;     // this pair's next whole tile, its place in the tail
        const int tail_hi = min(x + share, tail_len);
        MxUnit u = {};
        for (u.some = 1; u.some;) {
            int tile = 0, at = 0;                         // `at`: the tile's k-block to begin with
            // (tiles come in order: the group is found from the one before, 32 at a time)
            if (next_tile < tail_from) {
                tile = next_tile;
                next_tile += num_pairs;
            } else if (CUT && tail_from < tiles && x < tail_hi) {
                const int rel = x / padded;
                tile = tail_from + rel;
                at = x - rel * padded;
            } else {
                u.some = 0;
            }
            if (u.some) {
                for (;;) {
                    const int g = u.g + lane;
                    const unsigned before = __ballot_sync(~0u, g < p.groups && s_pre[g + 1] <= tile);
                    u.g += __popc(before);
                    if (before != ~0u) break;
                }
                const int rel = tile - s_pre[u.g], row0 = s_row[u.g], rows = rows_in(u.g);
                int ti = rel, first = 0;
                u.cols = rows;
                if (rows > width) {
                    // eight tiles of a group's rows sweep the features together
                    const int nt = (rows + width - 1) / width, jt = ((rows + nt - 1) / nt + 63) & ~63;    // cut evenly, in steps of 64
                    const int block = div_small(rel, 8 * p.tiles_i);
                    const int within = rel - block * 8 * p.tiles_i;
                    const int wide = min(8, nt - block * 8);
                    ti = div_small(within, wide);
                    first = (block * 8 + within - ti * wide) * jt;
                    u.cols = min(jt, rows - first);       // (at least 1: rows > width (nt - 1) >= jt (nt - 1))
                }
                u.c0 = row0 + first;
                u.tile = mx_group_tile(row0, u.g) + (first >> 7);
                u.shift = (first & 127) >> 5;
                u.i0 = ti * MX_TILE;
                u.jn = round32(u.cols);
                u.kb0 = 0;
                u.kb1 = p.kb_total;
                u.parts = 1;
                u.part = 0;
                if (CUT && tile >= tail_from) {
                    const int start = x - at;             // the tile's place in the tail
                    u.kb0 = min(at, p.kb_total);
                    u.kb1 = min(p.kb_total, at + tail_hi - x);
                    x += min(padded - at, tail_hi - x);
                    u.first_pair = start / share;
                    u.parts = (start + p.kb_total - 1) / share - u.first_pair + 1;
                    u.part = pair_id - u.first_pair;
                    u.cut = tile - tail_from;
                }
            }
            if (!mbar_wait(uempty_bar(unit_at), unit_phase ^ 1u, abort_flag)) {
                if (lane == 0) give_up(0x900u);
                break;
            }
            if (lane == 0) {
                s_unit[unit_at] = u;
                mbar_arrive(ufull_bar(unit_at));
            }
            __syncwarp();
            if (++unit_at == MX_UNITS) { unit_at = 0; unit_phase ^= 1u; }
        }
    } else if (warp == PRODUCER) {
        // ------------------------------------------------ TMA producer (both CTAs)
        const uint32_t lead_full0 = map_to_cta(full_bar(0), 0);
        const uint32_t elected = elect_one();
        const uint32_t lead_elected = rank == 0 ? elected : 0u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        MxUnit u = {};
        while (ok && next(u)) {
            ring();
            const int half = u.jn >> 1, high = mx_box(half);          // rows of this CTA, and the map whose boxes have them
            const int i = u.i0 + static_cast<int>(rank) * 128, c = u.c0 + static_cast<int>(rank) * half;
            const int s_tile = u.g * p.scale_tiles + (i >> 7);
            const bool two = u.shift * 32 + u.jn > 128;               // tiles of the rows' scales
            const uint32_t bytes = 2u * (MX_A_BYTES + mx_box_rows(high) * 128u + (two ? 3u : 2u) * S_BOX);
            const int s_off = MX_A_BYTES + *s_width * 64;
            for (int kb = u.kb0; kb < u.kb1; ++kb) {
                if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) {
                    if (lane == 0) give_up(0x100u + stage);
                    ok = false;
                    break;
                }
                const uint32_t sa = smem_base + stage * stage_bytes, lfb = lead_full0 + 8u * stage, ss = sa + s_off;
                const int kx = kb * (MX_BK / 2), ks = kb * (S_BOX / MX_TILE_BYTES);
                mbar_arrive_expect_tx_if(full_bar(stage), bytes, lead_elected);
                tma_load_3d_pair_if(sa, &maps.a, lfb, kx, i, u.g, elected);
                tma_load_3d_pair_if(sa + MX_A_BYTES, &maps.b[high], lfb, kx, c, 0, elected);
                tma_load_3d_pair_if(ss, &maps.sa, lfb, 0, ks, s_tile, elected);
                tma_load_3d_pair_if(ss + MX_S_BYTES, &maps.sb, lfb, 0, ks, u.tile, elected);
                if (two) tma_load_3d_pair_if(ss + 2 * MX_S_BYTES, &maps.sb, lfb, 0, ks, u.tile + 1, elected);
                __syncwarp();
                if (++stage == S) { stage = 0; phase ^= 1u; }
            }
        }
        for (int s = 0; ok && s < S; ++s) {   // drain: every stage this CTA filled has been consumed
            ok = mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag);
            if (++stage == S) { stage = 0; phase ^= 1u; }
        }
        if (!ok) settle();
    } else if (warp == ISSUER) {
        // ------------------------------------------------ MMA issuer (leader only)
        if (rank == 0) {
            const uint64_t da = make_smem_desc(smem_base, 16, 1024, 2);
            const uint32_t hi = static_cast<uint32_t>(da >> 32), a_lo0 = static_cast<uint32_t>(da);
            const uint32_t elected = elect_one();
            int stage = 0, local = 0;                     // local: accumulators filled so far
            uint32_t phase = 0, place = 0, place_phase = 0;   // place: of the scales
            bool ok = true;
            if (!mbar_wait(peer_ready_bar, 0u, abort_flag)) {
                if (lane == 0) give_up(0x700u);
                ok = false;
            }
            MxUnit u;
            while (ok && next(u)) {
                ring();
                const uint32_t idesc = p.idesc | (static_cast<uint32_t>(u.jn >> 3) << 17);
                int in_chunk = 0;
                uint32_t d_tmem = 0;
                for (int kb = u.kb0; kb < u.kb1; ++kb) {
                    const int acc = local & 1;
                    if (in_chunk == 0) {
                        // sharing: the accumulator before this one has given the shared columns back (and so its predecessor all of its own);
                        // else: the one before that is free
                        const bool free = !sharing ? mbar_wait(tempty_bar(acc), ((local >> 1) & 1u) ^ 1u, abort_flag)
                                                   : local == 0 || mbar_wait(tempty_bar(acc ^ 1), ((local - 1) >> 1) & 1u, abort_flag);
                        if (!free) {
                            if (lane == 0) give_up(0x200u + acc);
                            ok = false;
                            break;
                        }
                        tc_fence_after_sync();
                        d_tmem = tmem_base + acc * apart;
                    }
                    if (!mbar_wait(full_bar(stage), phase, abort_flag)) {
                        if (lane == 0) give_up(0x300u + stage);
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    const int steps = min(4, p.steps - 4 * kb);
                    const uint32_t a_lo = a_lo0 + stage * (stage_bytes >> 4), b_lo = a_lo + (MX_A_BYTES >> 4);
                    const uint32_t sa_t = tmem_base + SCALES + place * PLACE, sb_t = sa_t + PLACE / 3;
                    if (!mbar_wait(sready_bar(place), place_phase, abort_flag)) {
                        if (lane == 0) give_up(0x600u + place);
                        ok = false;
                        break;
                    }
                    if (++place == PLACES) { place = 0; place_phase ^= 1u; }
                    tc_fence_after_sync();
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        if (s > 0 && s >= steps) break;
                        // (two steps' scales in a column's word: the second's in its upper half)
                        const uint32_t id = NV ? 0u : (s & 1u) << 1, col = NV ? s : s >> 1;
                        umma_mx_pair_if<NV>(d_tmem, a_lo + 2 * s, hi, b_lo + 2 * s, hi, idesc | id << 4 | id << 29, sa_t + 4 * col,
                                            sb_t + 8 * col + u.shift, in_chunk > 0 || s > 0 ? 1u : 0u, elected);
                    }
                    umma_commit_pair_if(empty_bar(stage), 3, elected);
                    ++in_chunk;
                    if ((SUMS && in_chunk == p.chunk) || kb == u.kb1 - 1) {
                        umma_commit_pair_if(tfull_bar(acc), 3, elected);
                        in_chunk = 0;
                        ++local;
                    }
                    __syncwarp();
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
            }
            if (*abort_flag) settle();
        }
    } else {
        // ------------------------------------------------ epilogue (both CTAs, own 128 features)
        if (SUMS) more_registers();
        const int set = warp >> 2;
        const int quarter = warp & 3;
        const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
        int local = 0;
        bool ok = true;
        const float scale_a = p.scale_a ? __ldg(p.scale_a) : 1.0f;
        MxUnit u = {};
        float alpha = 1.0f;
        int group = -1;                                   // that alpha is of
        // Where the product of the two scales is no normal number (it is 0 or infinite, or has lost bits, though results may fit) a sum takes the larger
        // one before it is looked at, and the smaller is alpha.  A sum is 0 or 2^-20 to 2^54 in size, so with scales of packed operands (2^-100 to 2^120)
        // only what does not fit the result is lost on the way.  `group` stays -1 then, so that all of it is out of ordinary tiles' way (a test for
        // each piece cost 1.5 us of 21 at 8192 x 4096 x 256).
        auto larger_scale = [&]() {
            const float b = p.scale_b ? __ldg(p.scale_b + u.g) : 1.0f;
            alpha = fabsf(scale_a) > fabsf(b) ? b : scale_a;
            return fabsf(scale_a) > fabsf(b) ? scale_a : b;
        };
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
        };
        // Cut tiles.  The slab of a pair: 0 for the tile its share begins in, 1 for the one it ends in.  A piece is 4 KB of it,
        // lane after lane.
        auto slab_of = [&](int part, int c) {
            return reinterpret_cast<float4*>(p.partial) + (2 * (u.first_pair + part) + (part > 0 ? 0 : 1)) * (static_cast<size_t>(MX_TILE / 4) * p.slab_cols) +
                   ((rank * p.slab_cols + c) / 32 * 4 + quarter) * 256 + lane;
        };
        auto to_slab = [&](const float (&v)[32], int c) {
            float4* dst = slab_of(u.part, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) __stcg(dst + j * 32, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
        };
        // One 32 x 32 piece of C (columns c .. c + 31 of the tile, this warp's 32 features): lane l has feature l, v[j] is row j.  A store writes 32
        // consecutive features of a row.  (8192 x 4096 x 256 with 16-bit results: 20 us; pairs of features exchanged by shuffles and stored as
        // words, or transposed by way of shared memory into 16-byte stores, 25; by TMA stores, which wait behind the ring's loads, 38.)
        auto deliver = [&](float (&v)[32], int c) {
            const int n = min(32, u.cols - c), i0 = u.i0 + static_cast<int>(rank) * 128 + quarter * 32;
            const size_t base = static_cast<size_t>(u.c0 + c) * p.ldc + i0;
            if (p.bias) {
                const float bias = i0 + lane < p.I ? __ldg(p.bias + static_cast<size_t>(u.g) * p.I + i0 + lane) : 0.0f;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = fmaf(v[j], alpha, bias);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= alpha;
            }
            if (p.beta) {
                // C's old values, row after row (the pointer is kept from being computed for all of them at once, which spills)
                const char* old = static_cast<const char*>(p.C) + (base + lane) * SIZE;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (j % 8 == 0) asm volatile("" : "+l"(old)::"memory");
                    if (j < n && i0 + lane < p.I) v[j] += OUT16 ? half_bits_to_f32(*reinterpret_cast<const uint16_t*>(old), F16) : *reinterpret_cast<const float*>(old);
                    old += p.ldc * SIZE;
                }
            }
            if (p.relu) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];          // (a NaN stays)
            }
            const bool live = i0 + lane < p.I;
            char* dst = static_cast<char*>(p.C) + (base + lane) * SIZE;
            uint32_t w[16];                               // 16 bits: rows 2 j and 2 j + 1
#pragma unroll
            for (int j = 0; OUT16 && j < 16; ++j) w[j] = pack_half2(v[2 * j], v[2 * j + 1], F16);
            auto put = [&](int j) {
                if (OUT16) *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(j & 1 ? w[j >> 1] >> 16 : w[j >> 1]);
                else *reinterpret_cast<float*>(dst) = v[j];
                dst += p.ldc * SIZE;
            };
            if (n == 32 && i0 + 32 <= p.I) {
#pragma unroll
                for (int j = 0; j < 32; ++j) put(j);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (j % 8 == 0 && j >= n) break;
                    if (live && j < n) put(j);
                    else dst += p.ldc * SIZE;
                }
            }
        };
        while (ok && next(u)) {
            ring();
            if (u.g != group) {                           // (a load's latency for each tile otherwise)
                alpha = scale_a * (p.scale_b ? __ldg(p.scale_b + u.g) : 1.0f);
                group = NV && !(fabsf(alpha) >= 0x1p-126f && fabsf(alpha) < INFINITY) ? -1 : u.g;
            }
            // the accumulators that make up the unit
            const int blocks = u.kb1 - u.kb0, all = SUMS ? (blocks + p.chunk - 1) / p.chunk : 1;
            const int mine = (u.cols - set * 32 + SPAN - 1) / SPAN;   // pieces of this warp: columns set * 32 + SPAN q
            if (SUMS && all > 1) {
                // Accumulators are added in registers; the last one's place takes the sum, so that there is one way from here to C.  (Code that
                // runs once a launch costs its fetch: with a copy of that way for each piece of a sum this was 7 us slower.)
                float sum[4][32];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[q][j] = 0.0f;
#pragma unroll 1
                for (int n = 0; n < all; ++n) {
                    if (!await()) { ok = false; break; }
                    const uint32_t taddr = tmem_base + (local & 1) * apart + lane_addr + set * 32;
                    const bool end = n == all - 1;
                    auto take = [&](int q) {
                        if (q >= mine) return;
                        uint32_t v[32];
                        tmem_ld_32x32(taddr + q * 64, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[q][j] += __uint_as_float(v[j]);
                        if (end) {
                            tmem_st_32x16(taddr + q * 64, sum[q]);
                            tmem_st_32x16(taddr + q * 64 + 16, sum[q] + 16);
                        }
                    };
                    auto give = [&](bool now) { if (now && !end) release(); };
                    // the shared columns first: the last ones of the first accumulator, the first ones of the second
                    if (sharing && (local & 1) == 0) {
                        take(3);
                        take(2);
                        give(SHARED >= 128);
                        take(1);
                        give(SHARED < 128);
                        take(0);
                    } else {
                        take(0);
                        take(1);
                        give(sharing && SHARED >= 128);
                        take(2);
                        give(sharing && SHARED < 128);
                        take(3);
                        give(!sharing);
                    }
                    if (!end) ++local;
                }
                if (!ok) break;
                tmem_st_wait();
            } else if (!await()) {
                break;
            }
            // Pieces from tensor memory to C, the shared columns' first.
            const uint32_t taddr = tmem_base + (local & 1) * apart + lane_addr + set * 32;
            if (NV && group < 0 && !(CUT && u.parts > 1)) {
                const float large = larger_scale();
#pragma unroll 1
                for (int i = 0; i < 2 * mine; ++i) {         // half a piece
                    const uint32_t at = taddr + (i >> 1) * SPAN + (i & 1) * 16;
                    uint32_t v[16];
                    float x[16];
                    tmem_ld_32x16(at, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = __uint_as_float(v[j]) * large;
                    tmem_st_32x16(at, x);
                }
                tmem_st_wait();
            }
            const bool down = sharing && (local & 1) == 0;
            auto piece = [&](int i) { return down ? mine - 1 - i : i; };
            auto column = [&](int i) { return set * 32 + piece(i) * SPAN; };
            auto take = [&](float (&v)[32], int i) { tmem_ld_32x32(taddr + piece(i) * SPAN, reinterpret_cast<uint32_t (&)[32]>(v)); };
            auto emit = [&](float (&v)[32], int i) {
                if (CUT && u.parts > 1) to_slab(v, column(i));
                else deliver(v, column(i));
            };
            float f[32];
            if constexpr (SETS == 2) {                    // four pieces at most
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    if (i < mine) {
                        take(f, i);
                        tmem_ld_wait();
                    }
                    if (i == (!sharing ? 3 : SHARED >= 128 ? 1 : 2)) release();
                    if (i < mine) emit(f, i);
                }
            } else {
                // two pieces at most, and no more than one of them with shared columns
                static_assert(SETS == 2 || SHARED >= 128, "a warp's second piece has no shared columns");
#pragma unroll 1
                for (int i = 0; i < max(1, mine); ++i) {
                    if (i < mine) {
                        take(f, i);
                        tmem_ld_wait();
                    }
                    if (i == 0) release();
                    if (i < mine) emit(f, i);
                }
            }
            ++local;
            if (CUT && u.parts > 1) {
                // of a cut tile they went to this part's slab; one count for each of them says which have all their parts, and those are added up
                __syncwarp();
                bool done = false;
                if (lane < mine) {
                    unsigned int* counter = p.counter + (u.cut * 2 + rank) * 8 + set + SETS * lane;
                    const unsigned int old = (atomic_add_acq_rel(counter, 1u << (8 * quarter)) >> (8 * quarter)) & 255u;
                    done = old == static_cast<unsigned>(u.parts) - 1u;
                    if (done) atomicSub(counter, static_cast<unsigned>(u.parts) << (8 * quarter));
                }
                const unsigned int last = __ballot_sync(~0u, done);
                __syncwarp();                             // (a ballot orders no memory: what a lane acquired holds for the others from here on)
#pragma unroll 1
                for (int q = 0; q < mine; ++q) {
                    if (!((last >> q) & 1u)) continue;
                    const int c = set * 32 + q * SPAN;
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = 0.0f;
#pragma unroll 1
                    for (int s = 0; s < u.parts; ++s) {
                        const float4* src = slab_of(s, c);
                        float4 y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = __ldcg(src + j * 32);
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[4 * j] += y[j].x, f[4 * j + 1] += y[j].y, f[4 * j + 2] += y[j].z, f[4 * j + 3] += y[j].w;
                    }
                    if (NV && group < 0) {
                        const float large = larger_scale();
#pragma unroll
                        for (int j = 0; j < 32; ++j) f[j] *= large;
                    }
                    deliver(f, c);
                }
            }
        }
    }

    if (warp == PRODUCER) launch_wait();     // this launch ends after the one before it, whatever it read
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    if (warp == ISSUER) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

}  // namespace nk
