// What the host code of the operators that run the grouped kernel shares: its parameters and its launch.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>

namespace nk {

constexpr int GRP_THREADS = 352;
constexpr int GRP_MAX_GROUPS = 1024;
constexpr int GRP_STAGES = 6;
constexpr int GRP_A_BYTES = 128 * 64 * 2;
constexpr int GRP_STAGE = 2 * GRP_A_BYTES;             // 16 KB of features, up to 16 KB of rows, per CTA
constexpr int GRP_BK = 64;
constexpr int GRP_TILE = 256;                          // features of a tile, and the most rows of one
constexpr int GRP_MAX_SPLITS = 16;
constexpr int GRP_SMEM = GRP_STAGES * GRP_STAGE + 1024 + 2 * 4 * (GRP_MAX_GROUPS + 1) + 512;

struct GroupedParams {
    int groups, rows;      // rows: extent of the row arrays; offsets are clamped to it
    int I, J;              // features (contiguous in C); WEIGHTS: rows of each C_g
    int kb_total;          // ROWS: k-blocks of the contraction
    int tiles_i;           // ceil(I / 256)
    int tiles_j;           // WEIGHTS: ceil(J / 256)
    int beta, out16, f16;
    uint32_t idesc;        // without the N field
    const int* offsets;    // [groups + 1]; null: one group of all rows
    void* C;
    const float* add;      // ROWS: FP32 [rows][I], added before the rounding; null: none
    long long ldc, stride_c;
    float* partial;        // K splits: [unit][split][CTA of the pair][column][128 features]
    unsigned int* counter; // one per (unit, CTA of the pair); zero before and after every launch
    unsigned int* status;
};

// tcgen05 instruction descriptor without N: kind::f16, FP32 accumulator, M = 256 over the pair
inline uint32_t grouped_idesc(bool a_mn, bool b_mn, bool f16) {
    uint32_t d = 1u << 4;
    d |= (f16 ? 0u : 1u) << 7 | (f16 ? 0u : 1u) << 10;
    d |= (a_mn ? 1u : 0u) << 15 | (b_mn ? 1u : 0u) << 16;
    return d | (256u >> 4) << 24;
}

// (nk_grouped.cu)
cudaError_t grouped_prepare(bool weights, bool a_mn);     // once per kernel and device: its shared memory
cudaError_t grouped_launch(bool weights, bool a_mn, int pairs, cudaStream_t st, const CUtensorMap& a, const CUtensorMap& b,
                           const CUtensorMap& b16, const GroupedParams& p);
// Arrival counters of the K splits, zero between launches (the last arriver of a tile clears its own).  A plan holds a
// slot of a static table from create to destroy; where none is free (null) it runs without K splits.
constexpr int SPLIT_COUNTERS = 128;
int take_split_slot(unsigned int** counters);
void give_split_slot(int slot);
inline size_t grouped_partial_bytes(int pairs) { return static_cast<size_t>(pairs) * GRP_TILE * GRP_TILE * sizeof(float); }

}  // namespace nk
