/*
 * nk_mx — 4-bit floating-point operands with a scale for every block of elements, for NVIDIA B200 (sm_100a), beside the GEMM of
 * nk_gemm.h and the row-wise operators of nk_rows.h and in the same library:
 *
 *   nk_pack      matrices into 4-bit elements and block scales, along their rows or their columns; the scale of a whole tensor;
 *                reading back
 *   nk_mx        products of packed operands, of all rows with one weight or grouped by expert
 *
 * Conventions are those of nk_gemm.h and nk_rows.h: DEVICE pointers on the plan's device, nothing is allocated on the device,
 * nothing synchronises inside a run call, failures are status codes, and a plan (with its workspace) serves one stream at a time.
 *
 * Formats.  An element is an E2M1 number: a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  A block is a run of elements along the
 * contraction, counted from its start; the last one may be cut short by the end.
 *
 *   NK_MXF4   blocks of 32, scale 2^(floor(log2 m) - 2) with m the block's largest magnitude, held as E8M0 (the exponent + 127, at
 *             least 0): the OCP microscaling format MXFP4.  Magnitudes above 6 scales (up to 8) become 6.
 *   NK_NVF4   blocks of 16, scale s = m / (6 t) rounded to E4M3 (nearest even, at most 448), t an FP32 scale of the whole tensor
 *             (NULL: 1).  An element stands for s t e.  A scale that rounds to 0 makes the block zeros.
 *
 * An element is the E2M1 number nearest to x / scale, ties to the one with an even last bit; beyond 6 it is 6.  Every such decision is
 * that of exact arithmetic where t has at most 8 significant bits (nk_pack_scale's has); with another t a quotient within 2^-16 of a
 * border may go either way (a block's scale never does).  A block with an infinity or a NaN has the scale NaN (0xFF, 0x7F), and so have all blocks
 * if t is not between 2^-100 and 2^120.
 *
 * Packed arrays of a matrix of `outer` rows along the contraction of length L:
 *   data     [outer][Lp / 2] bytes, Lp = L rounded up to a multiple of 64; byte i holds element 2i in its low four bits, 2i + 1 above.
 *            Elements behind L are zeros.
 *   scales   tiles of 128 rows x 4 blocks, [ceil(outer / 128)][C][512] bytes, C = ceil(Lp / (4 block)); row r, block c of a tile is byte
 *            (r % 32) * 16 + r / 32 * 4 + c: what the tensor core reads.  Scales behind the last block or row are zeros.
 * A batch of matrices: one behind the other, data and scales.  Rows grouped by offsets (as for nk_grouped): data as of one matrix, but
 * the tiles of scales begin with every group: group g's at tile offsets[g] / 128 + g; there are rows / 128 + groups of them.
 */
#ifndef NK_MX_H
#define NK_MX_H

#include "nk_rows.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { NK_MXF4 = 0, NK_NVF4 = 1 } nk_mx_format_t;

/* ------------------------------------------------------------------ packing
 *
 * nk_pack_run: X [batch][rows][K] into packed arrays.  transposed = 0: along its rows (outer = rows, L = K).  transposed = 1: along its
 * columns, as the packed form of its transpose (outer = K, L = rows): what a product that contracts over the rows takes.
 * groups > 0 (batch 1, not transposed): rows grouped by `offsets`, groups + 1 non-decreasing INT32 row numbers on the device; rows
 * outside all groups are left alone, in data and scales.  Offsets that break the rule are clamped as for nk_grouped and
 * reported by nk_pack_check.  groups = 0: offsets is NULL.
 *
 * nk_pack_scale: scale[b] = max |X_b| / 2688 (6 x 448: no block scale saturates) rounded up to 8 significant bits, at least 2^-60; NaN if
 * X_b holds an infinity or a NaN.  All rows count, whatever the groups.  NK_MXF4 has no tensor scale: NK_ERR_UNSUPPORTED.
 *
 * nk_pack_values: Y [batch][outer][L] (dense) = what the packed arrays stand for, in FP32 or rounded once from it.
 */
typedef struct nk_pack_s* nk_pack_t;

typedef struct {
    int64_t rows;        /* 0 is allowed */
    int64_t K;           /* a multiple of 8 */
    int64_t batch;       /* 1 .. 65535; 0: 1 */
    int64_t groups;      /* 0 .. NK_GROUPED_MAX_GROUPS */
    int64_t ldx;         /* row stride of X in elements, a multiple of 8; 0: K */
    int64_t stride_x;    /* elements from X_b to X_b+1, a multiple of 8; 0: rows * ldx */
    int32_t format;      /* nk_mx_format_t */
    int32_t in_dtype;    /* NK_F32, NK_BF16 or NK_F16: X */
    int32_t value_dtype; /* the same: Y of nk_pack_values */
    int32_t transposed;  /* 0 or 1 */
    int32_t device;
} nk_pack_desc_t;

nk_status_t nk_pack_create(const nk_pack_desc_t* desc, nk_pack_t* out);
size_t nk_pack_data_bytes(nk_pack_t plan);
size_t nk_pack_scales_bytes(nk_pack_t plan);
size_t nk_pack_workspace_bytes(nk_pack_t plan); /* of nk_pack_scale; contents need no initialisation */
/* X, data, scales and Y 16-byte aligned; scale: `batch` FP32 numbers on the device, or NULL. */
nk_status_t nk_pack_scale(nk_pack_t plan, const void* X, float* scale, void* workspace, size_t workspace_bytes, void* cuda_stream);
nk_status_t nk_pack_run(nk_pack_t plan, const void* X, const float* scale, const int32_t* offsets, void* data, void* scales,
                        void* cuda_stream);
nk_status_t nk_pack_values(nk_pack_t plan, const void* data, const void* scales, const float* scale, const int32_t* offsets, void* Y,
                           void* cuda_stream);
nk_status_t nk_pack_check(nk_pack_t plan); /* as nk_grouped_check */
const char* nk_pack_kernel_name(nk_pack_t plan);
const char* nk_pack_last_cuda_error(nk_pack_t plan);
nk_status_t nk_pack_destroy(nk_pack_t plan);

/* ------------------------------------------------------------------ products
 *
 *   C[t][n] = epilogue( ta tb sum_k A[t][k] B[n][k] + beta C[t][n] )
 *
 * A [rows][K] and B [N][K] are packed along the contraction, in one format; ta and tb are their tensor scales (FP32 on the device; NULL: 1).
 * groups = 0: one B.  groups > 0: B, tb and bias are those of the row's group, B [groups][N][K] packed as a batch, A packed with the same
 * offsets; rows of C outside all groups are not touched.  FP32 accumulation, C in FP32 or rounded once to 16 bits.
 * NK_EPI_BIAS_RELU: max(0, .. + bias[n]), bias FP32 [N] (groups: [groups][N]); NULL: no bias.  The tensor scales of packed operands may be of any
 * size: where their product leaves FP32's range they are applied one after the other, and results that fit come out.
 *
 * Backward of Y = X . W^T: dX = dY . W is the same product with dY packed along its rows and W along its columns (transposed = 1); dW =
 * dY^T . X the same with both packed along their columns.  By expert: dX likewise; dW_g contracts over ragged rows, which have
 * no whole blocks, and is nk_grouped's (NK_GROUPED_WEIGHTS, 16-bit operands).
 *
 * The tensor core drops low bits of its FP32 accumulator at every step of 64 elements, so longer contractions than 8192 (FP32 C) or 16384
 * (16-bit C) are FP32 sums of accumulators of 4096 or 16384.  Measured against 64 bits (2-norm, FP32 C): normal operands 2.5e-8,
 * products of one sign up to 1e-7 however many, operands whose blocks differ by ten powers of two and more up to 1.2e-6.
 * Few tiles of one group with a long contraction are cut along it; such a plan takes one of the sets of counters of nk_rows.h, and one that
 * finds none cuts nothing (its kernel name ends in "_uncut"), which costs time and adds in another order.
 */
typedef struct nk_mx_s* nk_mx_t;

typedef struct {
    int64_t rows;      /* 0 is allowed */
    int64_t N;         /* a multiple of 8 */
    int64_t K;         /* the contraction's length: any, at least 1 */
    int64_t groups;    /* 0 .. NK_GROUPED_MAX_GROUPS */
    int64_t ldc;       /* row stride of C in elements, a multiple of 8; 0: N */
    int32_t format;    /* nk_mx_format_t */
    int32_t out_dtype; /* NK_F32, NK_BF16 or NK_F16 */
    int32_t epilogue;  /* nk_epilogue_t */
    int32_t beta;      /* 0 (C's old contents are never read) or 1 */
    int32_t device;
} nk_mx_desc_t;

nk_status_t nk_mx_create(const nk_mx_desc_t* desc, nk_mx_t* out);
size_t nk_mx_workspace_bytes(nk_mx_t plan); /* contents need no initialisation */
/* A, A_scales, B, B_scales, C and workspace 16-byte aligned. */
nk_status_t nk_mx_run(nk_mx_t plan, const void* A, const void* A_scales, const void* B, const void* B_scales, const float* scale_a,
                      const float* scale_b, const float* bias, const int32_t* offsets, void* C, void* workspace, size_t workspace_bytes,
                      void* cuda_stream);
nk_status_t nk_mx_check(nk_mx_t plan); /* as nk_grouped_check */
const char* nk_mx_kernel_name(nk_mx_t plan);
const char* nk_mx_last_cuda_error(nk_mx_t plan);
nk_status_t nk_mx_destroy(nk_mx_t plan);

#ifdef __cplusplus
}
#endif
#endif /* NK_MX_H */
