// What the host code and the kernel of the 4-bit products share: parameters and shared memory.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>

namespace nk {

enum MxMode { MX_WHOLE_TILES = 0, MX_CUT = 1, MX_SUMS = 2 };   // (sums: may be cut, too)
// Sets of four epilogue warps, and all threads (with four more warps).  Four sets have two pieces of a tile each, and the accumulator goes back once the
// first are taken: 8192 x 4096 x 1024 MXF4 25.2 us, by two sets 26.0.  With NVF4, whose accumulators share more columns, one set of four would
// have to take both first: 28.3 and 27.9.
__host__ __device__ constexpr int mx_sets(int mode, bool nv) { return mode == MX_WHOLE_TILES && !nv ? 4 : 2; }
__host__ __device__ constexpr int mx_threads(int mode, bool nv) { return 32 * (4 * mx_sets(mode, nv) + 4); }
constexpr int MX_MORE_REGISTERS = 216, MX_FEWER_REGISTERS = 72;   // of a thread where accumulators are summed: the epilogue's 256, the other 128
constexpr int MX_MAX_GROUPS = 1024;
constexpr int MX_BK = 256;                              // of the contraction to a k-block: 128 bytes of a row
constexpr int MX_A_BYTES = 128 * 128;                   // a stage: 16 KB of features, up to 16 KB of rows, then 2 KB of the features' scales
constexpr int MX_S_BYTES = 2048;                        // and 2 KB for each 128 rows, per CTA
constexpr int MX_TILE = 256;                            // features of a tile, and the most rows of one
constexpr int MX_RING = 190 * 1024;                     // five stages of 256 rows, more where the tiles are narrower
constexpr int MX_MAX_STAGES = 8;
constexpr int MX_TABLE = 4 * (MX_MAX_GROUPS + 1);
constexpr int MX_SMEM = MX_RING + 1024 + 2 * MX_TABLE + 1024;
static_assert(MX_SMEM <= 227 * 1024, "shared memory of an SM");
__host__ __device__ constexpr int mx_stage_bytes(int width) { return MX_A_BYTES + 64 * width + MX_S_BYTES * (1 + (width + 127) / 128); }

// Clocks, for the choice of tiles.  A k-block of tiles of w rows when all pairs are at work (the operand feed; 8192^3: 64 rows 0.30 us, 128 0.33,
// 192 0.39, 256 0.455), and by a pair alone; the rest of a tile, and of the last one for each of its rows.
constexpr int MX_ALONE_CLOCKS = 460, MX_TILE_CLOCKS = 300, MX_ROW_CLOCKS = 8;
__host__ __device__ constexpr int mx_block_clocks(int w) { return 450 + w + w / 2; }

struct MxParams {
    int width, parts;      // one group: rows of a tile, and into how many parts the tiles of the last wave are cut (1: none); 0, 1: the kernel's choice
    int groups, rows;      // rows: extent of the row arrays; offsets are clamped to it
    int I;                 // features (contiguous in C)
    int kb_total;          // k-blocks of the contraction
    int steps;             // of 64, of the whole contraction
    int tiles_i;           // ceil(I / 256)
    int scale_tiles;       // of a weight along its features: ceil(I / 128)
    int beta, relu;
    int chunk;             // k-blocks summed in tensor memory before they are added to an FP32 sum
    uint32_t idesc;        // without the N field
    const int* offsets;    // [groups + 1]; null: one group of all rows
    const float *scale_a, *scale_b, *bias;   // [1], [groups], [groups][I]; null: 1, 1, 0
    void* C;
    long long ldc;
    float* partial;        // slabs of tiles cut along k, two per CTA pair; null: no tile is cut
    int slab_cols;         // columns of a slab
    unsigned int* counter; // arrivals, a byte per (cut tile, CTA of the pair, 32-column piece, warp); zero before and after
    unsigned int* status;
};

// Boxes of the rows' operand: a CTA's half of a tile's rows takes the smallest that has them, which is no more than half of the tiles' width.  (Rows that
// are loaded beyond them are not multiplied; a box for every sixteen rows would be three more maps among a launch's arguments.)
constexpr int MX_BOXES = 5;
__host__ __device__ constexpr int mx_box_rows(int z) { return z < 3 ? 16 << z : 32 * z; }                     // 16, 32, 64, 96, 128
__host__ __device__ constexpr int mx_box(int rows) { return rows <= 16 ? 0 : rows <= 32 ? 1 : (rows + 31) / 32; }

struct MxMaps {
    CUtensorMap a;         // the features' operand (bytes): boxes of 128 features x 256 of k
    CUtensorMap b[MX_BOXES];   // the rows' operand in boxes of mx_box_rows rows
    CUtensorMap sa, sb;    // scales: boxes of the tiles of one k-block
};

enum MxOut { MX_OUT_F32 = 0, MX_OUT_BF16 = 1, MX_OUT_F16 = 2 };
// K-blocks to an accumulator: contractions of more are summed in FP32, FP32 results by MX_CHUNK.  (What the tensor core drops of a sum of 4-bit
// products is little, as they have few bits: against 64 bits, relative 2-norm, 8192 products of one sign are 5.3e-8 off in one accumulator, 4.9e-8 in
// four, normal ones 2.5e-8; 65536 of one sign 4.5e-7 by 32 k-blocks, 7.3e-8 by 16.  Magnitudes spread over ten powers of two and more are the
// worst: 8192 of them 3.6e-7 to 7.9e-7, 65536 2.5e-6 by 32, 1.2e-6 by 16; FP32 sums 1.7e-7 and 4.4e-7.  Sums cost 5 us of 26 at 4096 x
// 1024 x 8192.)
constexpr int MX_WHOLE = 32, MX_WHOLE_16 = 64, MX_CHUNK = 16;

// tcgen05 instruction descriptor without N: block-scaled E2M1 operands, M = 256 over the pair, scales E8M0 or (nv) E4M3
inline uint32_t mx_idesc(bool nv) { return 1u << 7 | 1u << 10 | (nv ? 0u : 1u << 23) | (256u >> 7) << 27; }

typedef void (*MxFunction)(MxMaps, MxParams);
MxFunction mx_kernel_nv(MxOut out, MxMode mode);       // (mx_nv.cu, mx_mx.cu)
MxFunction mx_kernel_mx(MxOut out, MxMode mode);

}  // namespace nk
