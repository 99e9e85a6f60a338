// What the host code of the operators that run the grouped kernel shares: its parameters and its launch.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>

namespace nk {

constexpr int GRP_THREADS = 384;
constexpr int GRP_MAX_GROUPS = 1024;
constexpr int GRP_A_BYTES = 128 * 64 * 2;              // a stage: 16 KB of features, up to 16 KB of rows, per CTA
constexpr int GRP_RING = 5 * 2 * GRP_A_BYTES;          // five stages of 256 rows, more where the tiles are narrower
constexpr int GRP_MAX_STAGES = 8;
constexpr int GRP_BK = 64;
constexpr int GRP_TILE = 256;                          // features of a tile, and the most rows of one
constexpr int GRP_TABLE = 4 * (GRP_MAX_GROUPS + 1);    // bytes of a table by group
constexpr int GRP_STAGING = 8 * 4096;                  // of the stores: two buffers of 2 KB for each epilogue warp
constexpr int GRP_BLOCK = 600;                         // clocks of a k-block for the choice of parts (see grouped.cuh)
// (a kernel that only writes h16 has no staging: more room for other blocks beside it)
__host__ __device__ constexpr int grp_smem(bool staging) { return GRP_RING + (staging ? GRP_STAGING : 0) + 1024 + 3 * GRP_TABLE + 1024; }

// k-blocks between additions to the FP32 sums (see grouped.cuh): of FP32 results, and of 16-bit ones
constexpr int GRP_CHUNK = 8, GRP_CHUNK_16 = 64;

enum GroupedMode { GRP_ROWS = 0, GRP_WEIGHTS = 1, GRP_LORA = 2 };
enum GroupedOut { GRP_OUT_F32 = 0, GRP_OUT_BF16 = 1, GRP_OUT_F16 = 2, GRP_OUT_H = 3 };   // H: h16 only (see GroupedParams), from one accumulator

struct GroupedParams {
    int groups, rows;      // rows: extent of the row arrays; offsets are clamped to it
    int I, J;              // features (contiguous in C); WEIGHTS: rows of each C_g
    int kb_total;          // ROWS, LORA: k-blocks of the contraction
    int tiles_i;           // ceil(I / 256)
    int tiles_j;           // WEIGHTS: ceil(J / 256)
    int beta, f16;
    int chunk;             // k-blocks summed in tensor memory before they are added to an FP32 sum
    uint32_t idesc;        // without the N field
    int a_slabs, b_slabs;  // MN-major operands of whole 64-feature slabs: a CTA's 128 features in one box
    const int* offsets;    // [groups + 1]; null: one group of all rows
    const int* index;      // ROWS: weight of each group (outside [0, index_max): the group is skipped); null: its number
    int index_max;
    void* C;
    const float* add;      // FP32 [rows][I], added before the rounding; null: none.  LORA: rows of short requests only, one behind the other
    int late;              // what `add` and h16 hold comes from the kernel before this one, nothing else does: wait for it there only
    int min_rows;          // ROWS with index: groups of so few rows are skipped; LORA: such requests' part is in `add`
    long long ldc, stride_c;
    float* partial;        // slabs of tiles cut along k, two per CTA pair; null: no tile is cut
    int slab_cols;         // columns of a slab
    unsigned int* counter; // arrivals, a byte per (cut tile, CTA of the pair, 32-column piece, warp); zero before and after
    unsigned int* status;
    // adapters.  LORA: each request's rows of h16 times its B_a are further k-blocks of a tile.  A row of h16 is a row of X . A_a as two
    // or three 16-bit numbers (`planes`) that add up to it, each the rounding of what the ones before it leave: blocks of 64
    // to a row, of 32 (two) or 16 (three) ranks, plane after plane.
    // BF16: ROWS with h16 (out H, or F32: by chunks) stores the product times scale[weight] that way instead of C.
    // FP16: ROWS (out F32) stores the product times scale[weight] as C, from which lora_split_kernel makes h16, with rows that need it
    // multiplied by a power of two; LORA's epilogue multiplies their part by the inverse, `unscale`.
    uint16_t* h16;
    const float* scale;    // ROWS; null: none
    const float* unscale;  // FP32 [rows]; null: BF16
    int rank_blocks, rank, planes;
    int requests;
    const int* request_offsets;
};

// tcgen05 instruction descriptor without N: kind::f16, FP32 accumulator, M = 256 over the pair
inline uint32_t grouped_idesc(bool a_mn, bool b_mn, bool f16) {
    uint32_t d = 1u << 4;
    d |= (f16 ? 0u : 1u) << 7 | (f16 ? 0u : 1u) << 10;
    d |= (a_mn ? 1u : 0u) << 15 | (b_mn ? 1u : 0u) << 16;
    return d | (256u >> 4) << 24;
}

struct GroupedMaps {
    CUtensorMap a;         // the features' operand: boxes of 128 features x 64 of k; with a_slabs one box, else two
    CUtensorMap b[8];      // the rows' operand in boxes of 16, 32, .. 128 rows; WEIGHTS: [0] 64 features, [1] 128 of them (b_slabs)
    CUtensorMap out;       // C in boxes of 2 KB: 32 features x 32 (16-bit) or 16 (FP32) rows (not with h16)
};
struct LoraMaps : GroupedMaps {    // (LORA alone: another KB of arguments costs a small launch 0.9 us)
    CUtensorMap c, h[8];   // the adapters' B, and h16 in boxes like b's
};

// (grouped_rows.cu, grouped_weights.cu, grouped_lora.cu: the instantiations; nk_grouped.cu: the rest)
typedef void (*GroupedFunction)(GroupedMaps, GroupedParams);
typedef void (*LoraFunction)(LoraMaps, GroupedParams);
GroupedFunction grouped_rows_kernel(bool a_mn, GroupedOut out, bool sums);
GroupedFunction grouped_weights_kernel(GroupedOut out, bool sums);
LoraFunction grouped_lora_kernel(bool a_mn, GroupedOut out);
struct GroupedKernel {     // one instantiation
    GroupedMode mode;
    bool a_mn;
    GroupedOut out;
    bool sums;             // a contraction may be longer than a chunk
    int chunk() const { return out == GRP_OUT_F32 ? GRP_CHUNK : GRP_CHUNK_16; }
};
// (`longest`: of the contractions)
inline GroupedKernel grouped_choose(GroupedMode mode, bool a_mn, GroupedOut out, int64_t longest) {
    return {mode, a_mn, out, mode == GRP_LORA || out == GRP_OUT_F32 || longest > GRP_CHUNK_16 * GRP_BK};
}
inline GroupedOut grouped_out(bool out16, bool f16) { return !out16 ? GRP_OUT_F32 : f16 ? GRP_OUT_F16 : GRP_OUT_BF16; }
cudaError_t grouped_prepare(const GroupedKernel& k);     // once per kernel and device: its shared memory
cudaError_t grouped_launch(const GroupedKernel& k, int pairs, cudaStream_t st, const GroupedMaps& maps, const GroupedParams& p);   // (LORA: LoraMaps)
// Arrival counters of the tiles cut along k, zero between launches (the last arriver clears its own).  A plan holds a
// slot of a static table from create until its last run has ended (see slot_table.h); where none is free (null) it cuts no tile.
constexpr int SPLIT_COUNTERS = 1280;           // 16 for each CTA pair of the device (a cut tile is one of the last wave)
int take_split_slot(int device, int pairs, unsigned int** counters);      // (of the current device)
void give_split_slot(int device, int slot, bool in_flight, bool captured);
inline size_t grouped_partial_bytes(int pairs, int slab_cols) {
    return static_cast<size_t>(pairs) * 2 * GRP_TILE * slab_cols * sizeof(float);
}
inline int grouped_slab_cols(int64_t most_rows) { return most_rows >= GRP_TILE ? GRP_TILE : static_cast<int>((most_rows + 31) / 32 * 32); }

}  // namespace nk
