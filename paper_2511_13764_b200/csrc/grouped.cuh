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
// groups' offsets are read on the device: every CTA turns them into a prefix of tile counts at its start,
// so no launch, size or plan depends on how the rows are spread.
//
// Schedule.  Whole waves of tiles go to the pairs in turn.  The tiles of the last, partial wave are cut along k where that
// saves more than it costs (see `estimate`); the parts of a cut tile meet in global memory, and the warp that finishes a
// 32 x 32 piece last adds them in k order and stores it: nobody waits, and the sum does not depend on who was last.
//
// What bounds it, and measured: few rows a group, HBM (64 groups of one row, 4096 x 4096: 305 us, 7.0 TB/s); many rows, the
// operand feed from L2, 0.33-0.385 us a k-block of 256 x 256 (8 groups, 8192 x 4096 x 1024: 55 us, 1.25 PFLOP/s; one group,
// 8192^3: 720-755 us, 1.46-1.53 PFLOP/s); little work, a launch's start, schedule and end (one tile 5.4 us after another
// launch, 16 x 4096 x 4096 13.9 us).  The gradient of the weights of 8 groups, 8192 rows, 1024 x 4096: 54 us to BF16, 64 to FP32.
//
// The tensor core's accumulator is cut short, not rounded, at every step, an error that goes one way and grows with the number of steps.
// So after p.chunk k-blocks the accumulator is added to an FP32 sum in the epilogue's registers while the other accumulator is being
// filled.  FP32 results, chunks of 8 k-blocks (512 of the contraction): 8192 rows in one accumulator were 9.1e-6 off (relative 2-norm),
// so 4.1e-7, where FP32 FMAs are 2.4e-7 (chunks of 4: half of that, for 5 % of the gradient's time).  16-bit results, 64 (4096 of the
// contraction; shorter ones need no sums): 2^18 products of one sign were 1.6e-3 too small, so 2.6e-5, a twentieth of what FP16's rounding may be.
//
// Warps: 0 TMA producer, 1 MMA issuer, 2-9 epilogue (warps 2-5 take the even 32-column chunks, 6-9 the odd
// ones), 10 (WEIGHTS) clears the rows of a group's last k-block that belong to the next group, 11 scheduler: it alone
// reads the offsets and hands out the work (inlined in every role the schedule made the kernel's code several times
// as long, and a launch that does little pays for code that is not in the instruction cache yet).
// All waits are bounded (see mbar_wait).
#pragma once
#include "grouped_launch.cuh"
#include "half.cuh"
#include "ptx.cuh"
#include <type_traits>

namespace nk {

// One piece of work: k-blocks kb0 .. kb1-1 of a tile.  Made by the scheduler warp, handed to the others in shared memory.
struct __align__(16) GroupedUnit {
    int some;              // 0: no more work
    int g, w, i0;          // group, its weight, first feature
    int c0, cols, jn;      // first row of C (ROWS: in the whole array, WEIGHTS: in C_g), rows of C in the tile, the MMA's N (cols rounded up to 32)
    int kb0, kb1;
    int row0, rows;        // the group's rows
    int cut, parts, part, first_pair;   // a cut tile: its number among the tail's tiles, its parts, this one, the pair of part 0
    int req, req_whole, req_parts;      // LORA: the first request of the tile, k-blocks of the one with all of its rows, how many have some of them
    int shorts;            // LORA: short requests with rows in the tile
    int pad;
};
constexpr int GRP_UNITS = 4;            // of them on the way

// the last i of [0, n) with table[i] <= x (0 if there is none)
__device__ __forceinline__ int find_last(const int* table, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (table[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int round32(int x) { return (x + 31) & ~31; }

// MODE: GroupedMode.  A_MN: the features' operand is MN-major (row-major weights [K][I], or rows [t][I]), else
// K-major (weights [I][K]).
// OUT: type of C (GroupedOut).  SUMS: a tile may have several accumulators to add.  (The bound of 512 threads keeps the 16-bit ROWS
// kernels without sums at 128 registers, which leaves an SM room for a block of the adapters' kernel beside them.)
template <int MODE, bool A_MN, int OUT, bool SUMS>
__global__ void __launch_bounds__(MODE == GRP_ROWS && !SUMS ? 512 : GRP_THREADS, 1) __cluster_dims__(2, 1, 1)
grouped_kernel(const __grid_constant__ std::conditional_t<MODE == GRP_LORA, LoraMaps, GroupedMaps> maps, const __grid_constant__ GroupedParams p) {
    constexpr bool WEIGHTS = MODE == GRP_WEIGHTS, LORA = MODE == GRP_LORA;
    constexpr bool OUT16 = OUT == GRP_OUT_BF16 || OUT == GRP_OUT_F16, F16 = OUT == GRP_OUT_F16;
    constexpr bool SCALED = LORA && OUT != GRP_OUT_BF16;   // operands may be FP16: rows of h16 may have a factor (p.unscale)
    constexpr int STAGING = OUT == GRP_OUT_H ? 0 : GRP_STAGING;
    static_assert(SUMS || (!LORA && OUT != GRP_OUT_F32), "FP32 results, and adapters, are sums");
    static_assert(!WEIGHTS || A_MN, "rows are contiguous in their features");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
    int* s_row = reinterpret_cast<int*>(gen_base + GRP_RING + STAGING);   // first row of each group (LORA: request), clamped and monotone
    int* s_pre = s_row + GRP_MAX_GROUPS + 1;                                  // tiles before each group
    int* s_alt = s_pre + GRP_MAX_GROUPS + 1;                                  // ROWS: weight of the group; LORA: adapter of the request; -1: none.  WEIGHTS: k-blocks before each group
    const uint32_t bar_base = smem_base + GRP_RING + STAGING + 3 * GRP_TABLE + 4;   // (8-byte aligned: a table is 4 mod 8 bytes)
    constexpr int MS = GRP_MAX_STAGES, WS = 5;            // (WEIGHTS: always five stages)
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (MS + s); };
    auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * MS + a); };
    auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * MS + 2 + a); };
    auto raw_bar = [&](int s) { return bar_base + 8u * (2 * MS + 4 + s); };   // a block with rows to clear: this CTA's boxes have landed
    auto tail_bar = [&](int s) { return bar_base + 8u * (2 * MS + 4 + WS + s); };   // leader: both CTAs have cleared theirs
    auto ufull_bar = [&](int n) { return bar_base + 8u * (2 * MS + 4 + 2 * WS + n); };    // a unit is there
    auto uempty_bar = [&](int n) { return bar_base + 8u * (2 * MS + 4 + 2 * WS + GRP_UNITS + n); };   // every role has read it
    constexpr int NB = 2 * MS + 4 + 2 * WS + 2 * GRP_UNITS;
    static_assert((3 * GRP_TABLE + 4) % 8 == 0, "barriers are 8-byte aligned");
    const uint32_t peer_ready_bar = bar_base + 8u * NB;
    uint8_t* after = gen_base + (bar_base - smem_base) + 8 * (NB + 1);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(after);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile int* s_width = reinterpret_cast<volatile int*>(after + 8);      // rows of a tile at most
    GroupedUnit* s_unit = reinterpret_cast<GroupedUnit*>(gen_base + ((GRP_RING + STAGING + 3 * GRP_TABLE + 4 + 8 * (NB + 1) + 12 + 15) & ~15));

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

    // offsets -> shared memory (LORA: the requests'; its one group is all the rows)
    const int* offsets = LORA ? p.request_offsets : p.offsets;
    const int entries = LORA ? p.requests : p.groups;
    if (warp == 0) {
        for (int n = lane; n < NB; n += 32) {
            // tempty: one arrival per epilogue warp of both CTAs; tail: one per CTA; uempty: producer, epilogue warps, the leader's
            // MMA issuer and (WEIGHTS) the warp that clears rows
            const uint32_t count = n >= 2 * MS + 2 && n < 2 * MS + 4                            ? 16
                                   : n >= 2 * MS + 4 + WS && n < 2 * MS + 4 + 2 * WS            ? 2
                                   : n >= 2 * MS + 4 + 2 * WS + GRP_UNITS ? 9 + (rank == 0) + WEIGHTS
                                                                                                : 1;
            mbar_init(bar_base + 8u * n, count);
        }
        if (lane == 31) mbar_init(peer_ready_bar, 1);
        if (lane == 0) *abort_flag = 0;
        fence_mbar_init();
        __syncwarp();
    } else if (warp == 2) {
        if (lane < (WEIGHTS ? 1 : 8)) tma_prefetch_desc(&maps.b[lane]);
        if (lane == 8) tma_prefetch_desc(&maps.a);
    } else if (warp == 1) {
        tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    cluster_arrive();
    // up to here the launch may have run beside the end of the one before it in the stream
    if (!p.late) launch_wait();
    launch_next();
    for (int g = threadIdx.x; g <= entries; g += GRP_THREADS) {
        s_row[g] = offsets ? offsets[g] : g == 0 ? 0 : p.rows;
        if (!WEIGHTS) {
            const int a = p.index && g < entries ? p.index[g] : g;
            s_alt[g] = p.index && (a < 0 || a >= p.index_max) ? -1 : a;
        }
    }
    __syncthreads();
    cluster_wait();          // the barriers of both CTAs are initialised
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    if (warp == 1 && rank == 1 && lane == 0) mbar_arrive_cluster_cta_release(map_to_cta(peer_ready_bar, 0));

    // the roles' view of the schedule: wait for the next unit, read it, give its place back
    int unit_at = 0;
    uint32_t unit_phase = 0;
    auto next = [&](GroupedUnit& u) -> bool {
        if (!mbar_wait(ufull_bar(unit_at), unit_phase, abort_flag)) {
            if (lane == 0) give_up(0x800u + warp);
            return false;
        }
        u = s_unit[unit_at];
        __syncwarp();
        if (lane == 0) mbar_arrive(uempty_bar(unit_at));
        if (++unit_at == GRP_UNITS) { unit_at = 0; unit_phase ^= 1u; }
        return u.some != 0;
    };
    // stages of the ring: as many as tiles of the schedule's width leave room for
    int stage_bytes = 2 * GRP_A_BYTES, S = WS;
    auto ring = [&]() {
        if (WEIGHTS) return;
        stage_bytes = GRP_A_BYTES + *s_width * 64;
        S = min(MS, GRP_RING / stage_bytes);
    };
    // WEIGHTS: rows of the group in k-block kb
    auto rows_of = [&](const GroupedUnit& u, int kb) { return min(GRP_BK, u.rows - kb * GRP_BK); };

    // LORA: the requests' blocks follow the last k-block of a tile.  A request that has all of the tile's rows goes into
    // the tile's own accumulator, unless rows of it have a factor (p.unscale).  Of the others each gets an accumulator of its own, of
    // which the epilogue adds the request's columns to the tile's sum: an adapter of infinities or NaN cannot reach another
    // request's rows.  Requests of p.min_rows rows or fewer are not worth an accumulator: theirs comes in FP32 from the
    // kernel before (`add`).
    auto has_part = [&](int q) { return s_alt[q] >= 0 && s_row[q + 1] - s_row[q] > p.min_rows; };
    auto is_short = [&](int q) { return s_alt[q] >= 0 && s_row[q + 1] > s_row[q] && s_row[q + 1] - s_row[q] <= p.min_rows; };

    if (warp == GRP_THREADS / 32 - 1) {
        // ------------------------------------------------ scheduler (both CTAs of a pair come to the same schedule)
        // offsets that break their rule are clamped to the running maximum
        bool bad = false;
        for (int g = lane; g <= entries; g += 32) bad |= s_row[g] < (g ? s_row[g - 1] : 0) || s_row[g] > p.rows;
        if (__any_sync(~0u, bad)) {
            if (lane == 0) {
                if (blockIdx.x == 0 && p.status) atomicCAS(p.status, 0u, 0x10000u);
                int top = 0;
                for (int g = 0; g <= entries; ++g) s_row[g] = top = max(top, min(s_row[g], p.rows));
            }
            __syncwarp();
        }
        auto rows_in = [&](int g) {
            if (LORA) return p.rows;
            const int rows = s_row[g + 1] - s_row[g];
            return !WEIGHTS && (s_alt[g] < 0 || rows <= p.min_rows) ? 0 : rows;
        };
        // k-blocks of a tile of group g
        auto length = [&](int g) { return WEIGHTS ? max(1, (rows_in(g) + GRP_BK - 1) / GRP_BK) : p.kb_total; };
        int most = 0;
        for (int g = lane; g < p.groups; g += 32) most = max(most, rows_in(g));
        most = static_cast<int>(__reduce_max_sync(~0u, static_cast<unsigned>(most)));
        // Estimated time, in clocks, of n tiles of w rows, and into how many parts (1: none) the tiles of the last, partial wave are cut:
        // equal parts, so that no pair has parts of two tiles, where they fill at most half a wave.  A k-block of a tile costs about
        // 260 + 1.5 w (operand feed; the tensor core alone would need 2 w for w = 256), for which GRP_BLOCK stands where the width is
        // settled.  (600 + w / 8 held for a slower producer; with it 4099 rows in 8 groups took 43.2 us instead of 38.9 (a card below its power cap), 5000
        // rows 43.1 instead of 37.1, 4096 x 1024 both, and 29 groups of 35 rows, 2048 x 32, 13.2 instead of 14.0; with 400 at
        // least 32 groups of 64 rows, 2048 x 768, 28.6 instead of 27.0, those of 35 rows 13.2.)  Parts are written to memory
        // at the end and the last to arrive reads them all: about 4000 clocks, and for every part and row (64 at least: a warp's
        // pieces follow one another) 10 + t^2 / 450, t being the parts of all tiles, which share the way to memory and back.
        // So the best number of parts goes with the root of the contraction's length.  (Measured with the slower producer: 1024 rows, 4096 x 1024, whole tiles of 256
        // rows 28.8 us, in four parts 26.5, tiles of 128 in two parts 21.7; 48 tiles of 86 k-blocks in two or three parts each 44, whole 36.)
        auto share_of = [&](int w, int t) { return static_cast<float>(max(64, w)) * (10.0f + static_cast<float>(t) * t * (1.0f / 450)); };
        auto best_parts = [&](int kbs, int w, int t) {
            return max(1, min(__float2int_rn(sqrtf(__fdividef(static_cast<float>(kbs) * GRP_BLOCK, share_of(w, t)))), kbs / 4));
        };
        auto estimate = [&](int n, int w, int& parts) {
            const int waves = n / num_pairs, rest = n - waves * num_pairs, most_parts = rest ? num_pairs / rest : 1;
            const float kb = 260.0f + w * 1.5f, k = static_cast<float>(p.kb_total), whole = (waves + (rest ? 1 : 0)) * k * kb;
            parts = p.partial && most_parts > 1 ? min(most_parts, best_parts(p.kb_total, w, rest * most_parts)) : 1;
            const float cut = (waves * k + (p.kb_total + parts - 1) / parts) * kb + 4000.0f + share_of(w, rest * parts) * parts;
            if (parts > 1 && cut < whole) return cut;
            parts = 1;
            return whole;
        };
        int width = WEIGHTS ? GRP_TILE : max(32, min(GRP_TILE, round32(most))), parts = 1;
        if (!WEIGHTS && width > 32) {
            // the width of least estimated time: lane l looks at 32 (l + 1)
            const int w = min(32 * ((lane & 7) + 1), width);
            int n = 0;
            for (int g = lane >> 3; g < p.groups; g += 4) n += (rows_in(g) + w - 1) / w;
            n += __shfl_xor_sync(~0u, n, 8);
            n += __shfl_xor_sync(~0u, n, 16);
            const float t = estimate(n * p.tiles_i, w, parts);
            // the smallest; of equals the widest: a time's upper bits, then the width
            const unsigned won = __reduce_min_sync(~0u, (__float_as_uint(t) & ~15u) | (8u - static_cast<unsigned>(w >> 5)));
            width = static_cast<int>(8u - (won & 15u)) << 5;
        }
        if (lane == 0) *s_width = width;
        // tiles (and k-blocks) before each group
        int tiles = 0, blocks = 0;
        for (int base = 0; base <= p.groups; base += 32) {
            const int g = base + lane;
            int n = g >= p.groups ? 0 : WEIGHTS ? p.tiles_i * p.tiles_j : (rows_in(g) + width - 1) / width * p.tiles_i;
            const int m = WEIGHTS && g < p.groups ? n * length(g) : 0;
            int v = n, w = m;
#pragma unroll 1
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(~0u, v, d), y = WEIGHTS ? __shfl_up_sync(~0u, w, d) : 0;
                if (lane >= d) { v += o; w += y; }
            }
            if (!LORA && g <= p.groups) {
                s_pre[g] = tiles + v - n;
                if (WEIGHTS) s_alt[g] = blocks + w - m;
            }
            tiles += __shfl_sync(~0u, v, 31);
            if (WEIGHTS) blocks += __shfl_sync(~0u, w, 31);
        }
        if (LORA) {
            // rows of short requests before each request
            int sum = 0;
            for (int base = 0; base < p.requests; base += 32) {
                const int q = base + lane, n = q < p.requests && is_short(q) ? s_row[q + 1] - s_row[q] : 0;
                int v = n;
#pragma unroll 1
                for (int d = 1; d < 32; d <<= 1) {
                    const int o = __shfl_up_sync(~0u, v, d);
                    if (lane >= d) v += o;
                }
                if (q < p.requests) s_pre[q] = sum + v - n;
                sum += __shfl_sync(~0u, v, 31);
            }
        }
        __syncwarp();
        // Whole tiles in turn, then the tail [tail_from, tiles), the last, partial wave: `tail_len` k-blocks from `tail_base` on, `share` of them
        // to each pair.  (ROWS, LORA: a tile counts `padded` k-blocks there, a whole number of shares.)
        const int full_waves = tiles / num_pairs, from = full_waves * num_pairs;
        int tail_from = tiles, tail_len = 0, share = 1, tail_base = 0, padded = p.kb_total;
        if (WEIGHTS) {
            if (p.partial && tiles > from) {
                // tiles of different lengths: the wave's k-blocks laid end to end and shared out evenly (as long as the longest, uncut)
                const int g = find_last(s_pre, p.groups, from);
                tail_base = s_alt[g] + (from - s_pre[g]) * length(g);
                tail_len = blocks - tail_base;
                int longest = 0;
                for (int h = g + lane; h < p.groups; h += 32) longest = max(longest, length(h));
                longest = static_cast<int>(__reduce_max_sync(~0u, static_cast<unsigned>(longest)));
                const int w = min(p.J, GRP_TILE), n = tiles - from;
                const int most_parts = best_parts(longest, w, min(2 * n, num_pairs + n));
                share = max(max(4, (tail_len + num_pairs - 1) / num_pairs), (longest + most_parts - 1) / most_parts);
                const int tile_parts = (longest + share - 1) / share + 1, all_parts = min(n * tile_parts, num_pairs + n);
                if (static_cast<float>(longest - share) * GRP_BLOCK > 4000.0f + share_of(w, all_parts) * tile_parts) tail_from = from;
            }
        } else {
            estimate(tiles, width, parts);
            if (parts > 1) {
                tail_from = from;
                share = (p.kb_total + parts - 1) / parts;
                padded = (p.kb_total + share - 1) / share * share;
                tail_len = (tiles - from) * padded;
            }
        }
        bool waited = false, handed = false;              // `handed`: a unit, to the other warps
        int next_tile = pair_id, x = pair_id * share;     // this pair's next whole tile, its place in the tail
        const int tail_hi = min(x + share, tail_len);
        GroupedUnit u = {};
        for (u.some = 1; u.some;) {
            int tile = 0, at = 0;                         // `at`: the tile's k-block to begin with
            if (next_tile < tail_from) {
                tile = next_tile;
                next_tile += num_pairs;
                u.g = LORA ? 0 : find_last(s_pre, p.groups, tile);
            } else if (tail_from < tiles && x < tail_hi) {
                if (WEIGHTS) {
                    const int y = tail_base + x;
                    u.g = find_last(s_alt, p.groups, y);
                    const int rel = (y - s_alt[u.g]) / length(u.g);
                    tile = s_pre[u.g] + rel;
                    at = y - s_alt[u.g] - rel * length(u.g);
                } else {
                    const int rel = x / padded;
                    tile = tail_from + rel;
                    at = x - rel * padded;
                    u.g = LORA ? 0 : find_last(s_pre, p.groups, tile);
                }
            } else {
                u.some = 0;
            }
            if (u.some) {
                const int rel = LORA ? tile : tile - s_pre[u.g], len = length(u.g);
                u.row0 = LORA ? 0 : s_row[u.g];
                u.rows = rows_in(u.g);
                int ti, kbs = len;
                if (WEIGHTS) {
                    ti = div_small(rel, p.tiles_j);
                    u.c0 = (rel - ti * p.tiles_j) * GRP_TILE;
                    u.cols = min(GRP_TILE, p.J - u.c0);
                    kbs = u.rows > 0 ? len : 0;
                } else {
                    u.w = LORA ? 0 : s_alt[u.g];
                    // the group's rows cut into equal tiles; eight of them sweep the features together
                    const int nt = (u.rows + width - 1) / width;
                    const int jt = round32((u.rows + nt - 1) / nt);
                    const int block = div_small(rel, 8 * p.tiles_i);
                    const int within = rel - block * 8 * p.tiles_i;
                    const int wide = min(8, nt - block * 8);
                    ti = div_small(within, wide);
                    u.c0 = u.row0 + (block * 8 + within - ti * wide) * jt;
                    u.cols = min(jt, u.row0 + u.rows - u.c0);
                }
                u.i0 = ti * GRP_TILE;
                u.jn = round32(u.cols);
                u.kb0 = 0;
                u.kb1 = kbs;
                u.parts = 1;
                u.part = 0;
                if (tile >= tail_from) {
                    const int start = x - at, whole = WEIGHTS ? len : padded;    // the tile's place and extent in the tail
                    u.kb0 = min(at, kbs);
                    u.kb1 = min(kbs, at + tail_hi - x);
                    x += min(whole - at, tail_hi - x);
                    u.first_pair = start / share;
                    u.parts = (start + len - 1) / share - u.first_pair + 1;
                    u.part = pair_id - u.first_pair;
                    u.cut = tile - tail_from;
                }
                if (LORA) {
                    u.req_whole = u.req_parts = u.shorts = 0;
                    // (the first request with rows at or behind the tile's first; before the first request's rows it is that one)
                    u.req = find_last(s_row, p.requests + 1, u.c0);
                    int parts_of = 0, shorts = 0;
                    for (int q = u.req + lane; q < p.requests && s_row[q] < u.c0 + u.cols; q += 32) {
                        parts_of += has_part(q) ? 1 : 0;
                        shorts += is_short(q) ? 1 : 0;
                    }
                    parts_of = static_cast<int>(__reduce_add_sync(~0u, static_cast<unsigned>(parts_of)));
                    u.shorts = static_cast<int>(__reduce_add_sync(~0u, static_cast<unsigned>(shorts)));
                    if (u.kb1 == kbs && parts_of) {
                        bool whole = s_row[u.req] <= u.c0 && s_row[u.req + 1] >= u.c0 + u.cols;
                        if (SCALED && whole && p.unscale) {
                            // Which rows have a factor says the kernel before this one; the pair's first tile does not wait to know.
                            if (!handed) {
                                whole = false;
                            } else {
                                if (!waited) launch_wait();
                                waited = true;
                                bool plain = true;
                                for (int r = lane; r < u.cols; r += 32) plain &= __ldcg(p.unscale + u.c0 + r) == 1.0f;
                                whole = __all_sync(~0u, plain);
                            }
                        }
                        if (whole) u.req_whole = p.rank_blocks;
                        else u.req_parts = parts_of;
                    }
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
            handed = true;
            if (++unit_at == GRP_UNITS) { unit_at = 0; unit_phase ^= 1u; }
        }
    } else if (warp == 0) {
        // ------------------------------------------------ TMA producer (both CTAs)
        const uint32_t lead_full0 = map_to_cta(full_bar(0), 0);
        const uint32_t elected = elect_one();
        const uint32_t lead_elected = rank == 0 ? elected : 0u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true, waited = false;
        GroupedUnit u = {};
        while (ok && next(u)) {
            ring();
            const int half = u.jn >> 1;
            const int i = u.i0 + static_cast<int>(rank) * 128;
            const int c = u.c0 + static_cast<int>(rank) * half;      // first column of this CTA's B operand
            const int boxes = (half + 63) >> 6;                       // WEIGHTS
            const uint32_t b_bytes = WEIGHTS ? boxes * 8192u : half * 128u;
            // Not WEIGHTS: half rows (a multiple of 16, up to 128) in one box, of the map that has them.  (Put together from boxes of 16, 32,
            // 64 and 128 rows the loads kept this warp busy for 450 clocks a k-block, whatever the tile: 1024 rows,
            // 4096 x 1024 took 20.6 us instead of 18.8; 32 rows, 8192 x 256 13.1 instead of 11.8.)
            const int high = (half >> 4) - 1;
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
                const uint32_t sa = smem_base + stage * stage_bytes, sb = sa + GRP_A_BYTES;
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
                    tma_load_3d_pair_if(sb, &maps.b[high], lfb, kx, c, 0, elected);
                }
                advance();
            }
            if constexpr (LORA) if (ok && u.req_whole + u.req_parts > 0) {
                // h16 comes from the kernel before this one
                if (!waited) launch_wait();
                waited = true;
                const uint32_t bytes = (A_MN ? 8192u : GRP_A_BYTES) + b_bytes;
                const int ranks = p.planes == 3 ? 16 : 32;    // of a block
                int q = u.req;
                for (int n = 0; ok && n < max(1, u.req_parts); ++n, ++q) {
                    while (!u.req_whole && !has_part(q)) ++q;
                    for (int rb = 0; rb < p.rank_blocks; ++rb) {
                        if (!acquire()) { ok = false; break; }
                        const uint32_t sa = smem_base + stage * stage_bytes, sb = sa + GRP_A_BYTES, lfb = lead_full0 + 8u * stage;
                        mbar_arrive_expect_tx_if(full_bar(stage), 2u * bytes, lead_elected);
                        if (A_MN) {
                            tma_load_3d_pair_if(sa, &maps.c, lfb, i, rb * ranks, s_alt[q], elected);
                            tma_load_3d_pair_if(sa + 8192, &maps.c, lfb, i + 64, rb * ranks, s_alt[q], elected);
                        } else {
                            tma_load_3d_pair_if(sa, &maps.c, lfb, rb * ranks, i, s_alt[q], elected);
                        }
                        tma_load_3d_pair_if(sb, &maps.h[high], lfb, rb * 64, c, 0, elected);
                        advance();
                    }
                }
            }
        }
        for (int s = 0; ok && s < S; ++s) {   // drain: every stage this CTA filled has been consumed
            ok = mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag);
            if (++stage == S) { stage = 0; phase ^= 1u; }
        }
        if (!ok) settle();
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
            while (ok && next(u)) {
                ring();
                const uint32_t idesc = p.idesc | (static_cast<uint32_t>(u.jn >> 3) << 17);
                const int base = u.kb1 - u.kb0, own = base + u.req_whole, blocks = own + u.req_parts * p.rank_blocks;
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
                        steps = p.planes == 3 ? 1 : min(2, (p.rank - 32 * rb + 15) >> 4);
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
                    const uint32_t a_lo = a_lo0 + stage * (stage_bytes >> 4), b_lo = b_lo0 + stage * (stage_bytes >> 4);
                    umma_pair_if<0>(d_tmem, a_lo, a_hi, b_lo, b_hi, idesc, accumulate, elected);
                    if (low_rank) {
                        // 32 ranks: leading parts in the first 64 bytes of a row of h16, remainders in the second; or 16 ranks in 32 bytes each
                        const uint32_t second = p.planes == 3 ? b_s : 2 * b_s;
                        if (steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + b_s, b_hi, idesc, 1u, elected);
                        umma_pair_if<0>(d_tmem, a_lo, a_hi, b_lo + second, b_hi, idesc, 1u, elected);
                        if (p.planes == 3) umma_pair_if<0>(d_tmem, a_lo, a_hi, b_lo + 2 * b_s, b_hi, idesc, 1u, elected);
                        if (steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + 3 * b_s, b_hi, idesc, 1u, elected);
                    } else {
                        if (!WEIGHTS || steps > 1) umma_pair_if<0>(d_tmem, a_lo + a_s, a_hi, b_lo + b_s, b_hi, idesc, 1u, elected);
                        if (!WEIGHTS || steps > 2) umma_pair_if<0>(d_tmem, a_lo + 2 * a_s, a_hi, b_lo + 2 * b_s, b_hi, idesc, 1u, elected);
                        if (!WEIGHTS || steps > 3) umma_pair_if<0>(d_tmem, a_lo + 3 * a_s, a_hi, b_lo + 3 * b_s, b_hi, idesc, 1u, elected);
                    }
                    umma_commit_pair_if(empty_bar(stage), 3, elected);
                    // (a request's accumulator has all of its ranks, however short the tile's own chunks are: one with K <= 64 and
                    // ranks above 32 closed before its last block would leave the epilogue an accumulator nobody waits for)
                    ++in_chunk;
                    if (!LORA || n < own ? (SUMS && in_chunk == p.chunk) || n == own - 1 : rb == 0) {
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
    } else if (warp < 10) {
        // ------------------------------------------------ epilogue (both CTAs, own 128 features)
        const int set = warp >= 6 ? 1 : 0;
        const int quarter = warp & 3;
        const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t staging = smem_base + GRP_RING + (warp - 2) * 4096;
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
        // Cut tiles.  The slab of a pair: 0 for the tile its share begins in, 1 for the one it ends in.  A piece is 4 KB of it,
        // lane after lane.
        auto slab_of = [&](int part, int c) {
            return reinterpret_cast<float4*>(p.partial) + (2 * (u.first_pair + part) + (part > 0 ? 0 : 1)) * (static_cast<size_t>(GRP_TILE / 4) * p.slab_cols) +
                   ((rank * p.slab_cols + c) / 32 * 4 + quarter) * 256 + lane;
        };
        auto to_slab = [&](const float (&v)[32], int c) {
            float4* dst = slab_of(u.part, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) __stcg(dst + j * 32, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
        };
        // One 32 x 32 piece of C (columns c .. c + 31 of the tile, this warp's 32 features): lane l has feature l, v[j] is row j.
        // It goes through two 2 KB buffers of shared memory, from where a TMA store writes it (and clips what lies beyond C's
        // edges); of a piece that ends inside the box, because the next row is another group's, lanes write 16 bytes each.
        auto deliver = [&](float (&v)[32], int c) {
            const int n = min(32, u.cols - c), i0 = u.i0 + static_cast<int>(rank) * 128 + quarter * 32;
            const size_t row0 = static_cast<size_t>(u.c0 + c);
            if (OUT == GRP_OUT_H || (MODE == GRP_ROWS && OUT == GRP_OUT_F32 && p.h16)) {
                // X . A_a for the adapters: the scaled product as a leading BF16 part and one or two remainders (none behind an
                // infinite leading part); ranks beyond the last are zeros
                const float scale = __ldg(p.scale + u.w);
                const int pitch = p.rank_blocks * 64, per = p.planes == 3 ? 16 : 32, i = i0 + lane;
                uint16_t* h = p.h16 + row0 * pitch + i / per * 64 + i % per;
                if (i < p.rank_blocks * per) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        float x = i < p.I ? v[j] * scale : 0.0f;
                        if (j < n) {
#pragma unroll
                            for (int z = 0; z < 3; ++z) {
                                if (z == p.planes) break;
                                const uint32_t bits = pack_half2(x, 0.0f, 0) & 0xFFFFu;
                                const float lead = half_bits_to_f32(bits, 0);
                                h[z * per] = static_cast<uint16_t>(bits);
                                x = fabsf(lead) <= 3.4028235e38f ? x - lead : 0.0f;
                            }
                        }
                        h += pitch;
                    }
                }
                return;
            }
            const bool live = i0 + lane < p.I;
            if (MODE == GRP_ROWS && OUT == GRP_OUT_F32 && p.scale) {
                const float scale = __ldg(p.scale + u.w);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= scale;
            }
            if (MODE == GRP_ROWS && p.add) {
                if (!waited) launch_wait();
                waited = true;
                const float* add = p.add + row0 * p.I + i0 + lane;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (live && j < n) v[j] += __ldcg(add);
                    add += p.I;
                }
            }
            if (LORA && u.shorts) {
                // rows of short requests have theirs in `add`, in the order of the rows: which of these 32, and where the first is
                const int row = u.c0 + c + lane;
                const int q = find_last(s_row, p.requests + 1, row);
                const bool has = lane < n && row >= s_row[0] && q < p.requests && is_short(q);
                const unsigned mask = __ballot_sync(~0u, has);
                if (mask) {
                    if (!waited) launch_wait();
                    waited = true;
                    const int first = __shfl_sync(~0u, has ? s_pre[q] + row - s_row[q] : 0, __ffs(mask) - 1);
                    const float* add = p.add + static_cast<size_t>(first) * p.I + i0 + lane;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if ((mask >> j) & 1u) {
                            if (live) v[j] += __ldcg(add);
                            add += p.I;
                        }
                }
            }
            const size_t base = (WEIGHTS ? static_cast<size_t>(u.g) * p.stride_c : 0) + row0 * p.ldc + i0;
            if (p.beta) {
                const uint16_t* c16 = static_cast<const uint16_t*>(p.C) + base + lane;
                const float* c32 = static_cast<const float*>(p.C) + base + lane;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (live && j < n) v[j] += OUT16 ? half_bits_to_f32(*c16, F16) : *c32;
                    c16 += p.ldc;
                    c32 += p.ldc;
                }
            }
            constexpr int ROWS = OUT16 ? 32 : 16, PITCH = 2048 / ROWS;    // of a buffer; 64 or 128 bytes
#pragma unroll
            for (int half = 0; half < 32; half += ROWS) {
                if (half > 0 && half >= n) break;
                const uint32_t box = staging + parity * 2048;
                parity ^= 1u;
                if (lane == 0) bulk_wait_read<1>();       // the store before the last has read this buffer
                __syncwarp();
                if (OUT16) {
                    // a lane packs its feature of rows j and j + 1 and exchanges words with its neighbour: even lanes then hold row j of
                    // features (l, l + 1), odd lanes row j + 1 of (l - 1, l): two rows of 64 bytes per store, no bank twice
                    const uint32_t odd = lane & 1, pick = odd ? 0x3276u : 0x5410u, dst = box + odd * 64 + (lane >> 1) * 4;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t w = pack_half2(v[2 * j], v[2 * j + 1], F16);
                        const uint32_t got = __shfl_xor_sync(~0u, w, 1);
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + j * 128), "r"(__byte_perm(w, got, pick)) : "memory");
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < ROWS; ++j)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(box + lane * 4 + j * PITCH), "f"(v[half + j]) : "memory");
                }
                if (WEIGHTS || n >= half + ROWS) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) tma_store_3d(&maps.out, box, i0, static_cast<int>(row0) + half, WEIGHTS ? u.g : 0);
                } else {
                    __syncwarp();
                    constexpr int LANES = PITCH / 16, WIDE = OUT16 ? 8 : 4;       // lanes of a row, elements of a lane
                    const int f = (lane % LANES) * WIDE;
                    if (i0 + f < p.I) {                   // (the number of features is a multiple of 8)
#pragma unroll 1
                        for (int r = lane / LANES; r < n - half; r += 32 / LANES) {
                            uint32_t x[4];
                            ld_shared_v4(box + r * PITCH + (lane % LANES) * 16, x);
                            const size_t o = base + (half + r) * p.ldc + f;
                            uint4* dst = OUT16 ? reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.C) + o) : reinterpret_cast<uint4*>(static_cast<float*>(p.C) + o);
                            *dst = make_uint4(x[0], x[1], x[2], x[3]);
                        }
                    }
                    __syncwarp();
                }
                if (lane == 0) bulk_commit();             // (an empty group where nothing was stored: the buffers take turns)
            }
        };
        while (ok && next(u)) {
            // the accumulators that make up the tile: chunks of its own k-blocks, then one for each request with some of its rows
            bool held = true;                             // the sum is in tensor memory, not stored yet
            const int blocks = u.kb1 - u.kb0 + u.req_whole;
            const int chunks = !SUMS || blocks <= p.chunk ? 1 : (blocks + p.chunk - 1) / p.chunk, all = chunks + u.req_parts;
            if (!await()) break;
            if (SUMS && all > 1) {
                // they are added in registers
                float sum[4][32];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[q][j] = 0.0f;
                int at = u.req;
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
                    const bool unscale = SCALED && n >= chunks && p.unscale;
                    if (unscale && !waited) {
                        launch_wait();
                        waited = true;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = set * 32 + q * 64;
                        if (c < hi && c + 32 > lo) {
                            // lane l has the factor of the piece's row l
                            const float factor = unscale && lane < u.cols - c ? __ldcg(p.unscale + u.c0 + c + lane) : 0.0f;
#pragma unroll
                            for (int b = 0; b < 32; b += 16) {                   // (halves of a piece: fewer registers beside the sums)
                                uint32_t v[16];
                                tmem_ld_32x16(taddr + c + b, v);
                                tmem_ld_wait();
                                if (unscale) {
#pragma unroll
                                    for (int j = 0; j < 16; ++j) {
                                        const float f = __shfl_sync(~0u, factor, b + j);
                                        if (c + b + j >= lo && c + b + j < hi) sum[q][b + j] += __uint_as_float(v[j]) * f;
                                    }
                                } else if (!LORA || (c >= lo && c + 32 <= hi)) {
#pragma unroll
                                    for (int j = 0; j < 16; ++j) sum[q][b + j] += __uint_as_float(v[j]);
                                } else {
#pragma unroll
                                    for (int j = 0; j < 16; ++j)
                                        if (c + b + j >= lo && c + b + j < hi) sum[q][b + j] += __uint_as_float(v[j]);
                                }
                            }
                        }
                    }
                    if (n < all - 1) {
                        release();
                        if (!await()) { ok = false; break; }
                    }
                }
                if (!ok) break;
                release();                                // the next tile may have this accumulator while the sums are stored
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = set * 32 + q * 64;
                    if (c >= u.cols) continue;
                    if (u.parts > 1) to_slab(sum[q], c);
                    else deliver(sum[q], c);
                }
                held = false;
            }
            const uint32_t taddr = tmem_base + (local & 1) * GRP_TILE + lane_addr;
            const int mine = (u.cols - set * 32 + 63) >> 6;
            unsigned int last = (1u << max(0, mine)) - 1u;    // the pieces this warp stores
            if (u.parts > 1) {
                // this part's pieces go to its slab; then one count for each of them says which have all their parts
#pragma unroll 1
                for (int q = 0; held && q < mine; ++q) {
                    uint32_t v[32];
                    float f[32];
                    tmem_ld_32x32(taddr + set * 32 + q * 64, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
                    to_slab(f, set * 32 + q * 64);
                }
                if (held) release();
                __syncwarp();
                bool done = false;
                if (lane < mine) {
                    unsigned int* counter = p.counter + (u.cut * 2 + rank) * 8 + set + 2 * lane;
                    const unsigned int old = (atomic_add_acq_rel(counter, 1u << (8 * quarter)) >> (8 * quarter)) & 255u;
                    done = old == static_cast<unsigned>(u.parts) - 1u;
                    if (done) atomicSub(counter, static_cast<unsigned>(u.parts) << (8 * quarter));
                }
                last = __ballot_sync(~0u, done);
                __syncwarp();                                 // (a ballot orders no memory: what a lane acquired holds for the others from here on)
            }
#pragma unroll 1
            for (int q = 0; q < mine; ++q) {
                if (!((last >> q) & 1u) || !(held || u.parts > 1)) continue;
                const int c = set * 32 + q * 64;
                float f[32];
                if (u.parts > 1) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = 0.0f;
#pragma unroll 2
                    for (int s = 0; s < u.parts; ++s) {
                        const float4* src = slab_of(s, c);
                        float4 y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = __ldcg(src + j * 32);
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[4 * j] += y[j].x, f[4 * j + 1] += y[j].y, f[4 * j + 2] += y[j].z, f[4 * j + 3] += y[j].w;
                    }
                } else {
                    uint32_t v[32];
                    tmem_ld_32x32(taddr + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
                    if (WEIGHTS && blocks == 0) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) f[j] = 0.0f;
                    }
                }
                deliver(f, c);
            }
            if (held && u.parts == 1) release();
        }
        if (lane == 0) bulk_wait_read<0>();               // the stores are done with this CTA's shared memory
        __syncwarp();
    } else if (WEIGHTS) {
        // ------------------------------------------------ rows of the next group in a group's last k-block
        const uint32_t lead_tail0 = map_to_cta(tail_bar(0), 0);
        int stage = 0;
        uint32_t raw_phase = 0;
        GroupedUnit u = {};
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
                        st_shared_v4(smem_base + stage * stage_bytes + b * 8192 + y * 16, 0u, 0u, 0u, 0u);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_cta_release(lead_tail0 + 8u * stage);
            }
            stage = (stage + 1) % S;
        }
    }

    if (warp == 0) launch_wait();        // this launch ends after the one before it, whatever it read
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

}  // namespace nk
