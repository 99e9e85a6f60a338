/*
 * nk_rows — layers whose weight is chosen row by row, for NVIDIA B200 (sm_100a), beside the dense GEMM of
 * nk_gemm.h and in the same library:
 *
 *   nk_route     which experts a row goes to and with what weight, the rows' way to their experts' order and
 *                back, and the gradients of both
 *   nk_grouped   products grouped by expert over ragged groups of rows, and their gradients
 *   nk_lora      a shared projection with the low-rank adapters of many requests beside it
 *
 * Conventions are those of nk_gemm.h: DEVICE pointers on the plan's device, nothing is allocated on the
 * device, nothing synchronises inside a run call, failures are status codes, and a plan (with its workspace)
 * serves one stream at a time: two runs of a plan whose work can overlap on the device race.
 * A plan may be destroyed while runs of it are queued or are held by a CUDA graph: they keep what they need, and the
 * counters they use in the library's static memory go to no other plan before they have ended (those of a captured run,
 * never).  A device has 1024 sets of counters: nk_grouped takes one, nk_lora one or two; a plan that finds none cuts no
 * tile along its contraction, which costs time where there are few tiles and adds FP32 sums in another order: its kernel
 * name ends in "_uncut", and its bits can differ from those of a plan with counters.  Bits of one plan are the same on every run.
 * The caller's buffers have to live as long as the runs, as always.
 * Matrices are row-major; "ld" fields are row strides in elements (0: dense).
 */
#ifndef NK_ROWS_H
#define NK_ROWS_H

#include "nk_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ products grouped by expert
 *
 * `offsets` is a device array of groups + 1 non-decreasing INT32 row numbers, 0 <= offsets[0],
 * offsets[groups] <= rows: group g owns the rows offsets[g] .. offsets[g+1]-1 of the row arrays (empty groups
 * are fine).  It is read by the kernel, never by the host, so a plan serves every way of spreading the rows.
 *
 *   NK_GROUPED_ROWS      C[t][0..N) = A[t][0..K) . B_g            for the rows t of every group g
 *                        B_g is [K][N] (layout_b NK_ROW_MAJOR) or kept as its transpose, [N][K]
 *                        (NK_TRANSPOSED, the [out][in] of a linear layer).  Rows of C outside all groups are
 *                        not touched.  The gradient of the rows, dA[t] = dC[t] . B_g^T, is the same product with
 *                        N and K exchanged and the other layout_b: no copy of the weights is made.
 *   NK_GROUPED_WEIGHTS   C_g[K][N] = sum over the rows t of group g of A[t][0..K)^T . B[t][0..N)
 *                        the gradient of the weights (A: the rows, B: the gradient of the result; exchange the
 *                        two for weights kept as [N][K]).  A group without rows gives zeros.
 *
 * 16-bit operands of one type, FP32 accumulation, C in FP32 or rounded once to the operands' type.  beta = 1
 * adds C's old values in FP32 before the rounding (accumulated gradients); with beta = 0 they are never read.
 * The tensor core drops low bits of its FP32 accumulator at every step, so the accumulator is emptied into an FP32 sum every 512
 * elements of the contraction for an FP32 C, every 4096 for a 16-bit one: products of one sign then add up to 2.3e-7 too little
 * on average (FP32), 2.6e-5 (16-bit, a tenth of half of FP16's spacing), however many there are.
 * With NK_GROUPED_ROWS a row of C depends on its own row of A and its group's weight only: infinities and NaN in
 * other rows, groups or beyond offsets[groups] stay there.
 * Offsets that are negative, beyond `rows` or decreasing are clamped to the running maximum within [0, rows] (no
 * access leaves the arrays) and reported by nk_grouped_check.
 */
typedef struct nk_grouped_s* nk_grouped_t;
typedef enum { NK_GROUPED_ROWS = 0, NK_GROUPED_WEIGHTS = 1 } nk_grouped_kind_t;
#define NK_GROUPED_MAX_GROUPS 1024

typedef struct {
    int64_t groups;    /* 1 .. NK_GROUPED_MAX_GROUPS */
    int64_t rows;      /* extent of the row arrays; 0 is allowed */
    int64_t N, K;      /* multiples of 8 */
    int32_t kind;      /* nk_grouped_kind_t */
    int32_t in_dtype;  /* NK_BF16 or NK_F16: A and B */
    int32_t out_dtype; /* NK_F32, or the operands' type */
    int32_t layout_b;  /* NK_GROUPED_ROWS: NK_ROW_MAJOR or NK_TRANSPOSED; NK_GROUPED_WEIGHTS: NK_ROW_MAJOR */
    int32_t beta;      /* 0 or 1 */
    int32_t device;
    int64_t lda, ldb, ldc; /* row strides of A, of B (of one B_g) and of C (of one C_g); multiples of 8; 0: dense */
    int64_t stride_g;      /* elements from B_g to B_g+1 (ROWS) or from C_g to C_g+1 (WEIGHTS); multiple of 8; 0: dense */
} nk_grouped_desc_t;

nk_status_t nk_grouped_create(const nk_grouped_desc_t* desc, nk_grouped_t* out);
/* Device scratch a run needs (FP32 partial sums where few tiles are cut along K); contents need no initialisation. */
size_t nk_grouped_workspace_bytes(nk_grouped_t plan);
/* A, B, C and workspace 16-byte aligned; A, B and C may be NULL where they have no element (rows = 0). */
nk_status_t nk_grouped_run(nk_grouped_t plan, const void* A, const void* B, void* C, const int32_t* offsets,
                           void* workspace, size_t workspace_bytes, void* cuda_stream);
/* Synchronise the device and report, once: NK_ERR_INVALID_ARG if a run met offsets that break the rule above,
 * NK_ERR_TIMEOUT if a bounded wait ran out (results undefined), else NK_OK. */
nk_status_t nk_grouped_check(nk_grouped_t plan);
const char* nk_grouped_kernel_name(nk_grouped_t plan);
const char* nk_grouped_last_cuda_error(nk_grouped_t plan);
nk_status_t nk_grouped_destroy(nk_grouped_t plan);

/* ------------------------------------------------------------------ routing of rows to experts
 *
 * nk_route_run: for every token t, from its row of logits z[t][0..experts):
 *   experts[t][j]  the indices of its topk largest logits, the largest first, ties by the lower index
 *   gates[t][j]    softmax(z[t]) at experts[t][j] (over all experts; renormalise = 0), or the softmax over the
 *                  chosen ones only (renormalise = 1), in FP32
 *   offsets[e]     (experts + 1 of them) how many (token, j) pairs go to experts below e: the row offsets that
 *                  nk_grouped takes
 *   slots[t][j]    the pair's place in the experts' order: offsets[e] + the number of tokens before t that chose e
 * Logits of minus infinity are experts that may not be chosen: they are chosen only where fewer than topk others
 * are left, with gate 0; a row with nothing else has all gates 0.  A NaN is smaller than every number in the
 * choice, and the gates of its row are NaN.
 *
 * nk_route_backward: dlogits[t][e] (FP32) from dgates[t][j] = dL / dgates[t][j], logits and experts of the run:
 *   dz_e = p_e (d_e - sum_j d_j gates_j), d_e = dgates[t][j] where e = experts[t][j], else 0; p the softmax above.
 *   A row whose logits are all minus infinity gets zeros.
 * nk_route_dispatch: Xs[slots[t][j]] = X[t].
 * nk_route_combine:  Y[t] = sum_j gates[t][j] * Ys[slots[t][j]], summed in j's order in FP32, rounded once; gates NULL:
 *   all ones, which is the gradient of nk_route_dispatch.
 * nk_route_combine_backward: dYs[slots[t][j]] = gates[t][j] * dY[t] and dgates[t][j] = <dY[t], Ys[slots[t][j]]> (FP32).
 * A slot outside [0, tokens * topk) is a dropped pair: nothing is written for it, it adds nothing to Y, its dgates
 * is 0.  X, Y, dY have `tokens` rows; Xs, Ys, dYs have tokens * topk rows; all of `width` 16-bit elements of one type.
 */
typedef struct nk_route_s* nk_route_t;
#define NK_ROUTE_MAX_EXPERTS 1024
#define NK_ROUTE_MAX_TOPK 32

typedef struct {
    int64_t tokens;       /* 0 .. 2^24 */
    int64_t experts;      /* 1 .. NK_ROUTE_MAX_EXPERTS */
    int64_t topk;         /* 1 .. min(experts, NK_ROUTE_MAX_TOPK) */
    int64_t width;        /* a multiple of 8; 0: only run and backward are used */
    int64_t ld_logits;    /* row stride of logits in elements; 0: experts */
    int64_t ld_tokens;    /* row stride of X, Y, dY; a multiple of 8; 0: width */
    int64_t ld_slots;     /* row stride of Xs, Ys, dYs; a multiple of 8; 0: width */
    int32_t logits_dtype; /* NK_F32, NK_BF16 or NK_F16 */
    int32_t dtype;        /* NK_BF16 or NK_F16: the rows */
    int32_t renormalise;  /* 0 or 1 */
    int32_t device;
} nk_route_desc_t;

nk_status_t nk_route_create(const nk_route_desc_t* desc, nk_route_t* out);
size_t nk_route_workspace_bytes(nk_route_t plan); /* of nk_route_run; contents need no initialisation */
nk_status_t nk_route_run(nk_route_t plan, const void* logits, float* gates, int32_t* experts, int32_t* offsets, int32_t* slots,
                         void* workspace, size_t workspace_bytes, void* cuda_stream);
nk_status_t nk_route_backward(nk_route_t plan, const void* logits, const int32_t* experts, const float* dgates, float* dlogits,
                              void* cuda_stream);
nk_status_t nk_route_dispatch(nk_route_t plan, const void* X, const int32_t* slots, void* Xs, void* cuda_stream);
nk_status_t nk_route_combine(nk_route_t plan, const void* Ys, const int32_t* slots, const float* gates, void* Y, void* cuda_stream);
nk_status_t nk_route_combine_backward(nk_route_t plan, const void* dY, const void* Ys, const int32_t* slots, const float* gates,
                                      void* dYs, float* dgates, void* cuda_stream);
nk_status_t nk_route_check(nk_route_t plan); /* synchronises the device */
const char* nk_route_kernel_name(nk_route_t plan);
const char* nk_route_last_cuda_error(nk_route_t plan);
nk_status_t nk_route_destroy(nk_route_t plan);

/* ------------------------------------------------------------------ low-rank adapters of many requests
 *
 *   Y[t] = X[t] . W + scale[a] * (X[t] . A_a) . B_a        a = adapter[q] of the request q that row t belongs to
 *
 * `offsets` is a device array of requests + 1 non-decreasing INT32 row numbers as for nk_grouped: request q owns the
 * rows offsets[q] .. offsets[q+1]-1 (one row each in a decoding step, many for a prompt, none is fine; any mix).
 * `adapter` is a device array of `requests` INT32 numbers; a number outside [0, adapters) means no adapter.  Rows
 * outside all requests get the shared projection alone.  `scale` is a device array of `adapters` FP32 numbers.
 *
 *   layout NK_ROW_MAJOR    W [K][N],  A [adapters][K][rank],  B [adapters][rank][N]
 *   layout NK_TRANSPOSED   W [N][K],  A [adapters][rank][K],  B [adapters][N][rank]   (linear layers' [out][in])
 *
 * The gradient of the rows, dX[t] = dY[t] . W^T + scale[a] (dY[t] . B_a^T) . A_a^T, is the same call: a plan with N and K exchanged
 * and the other layout, and dY, W, B, A in the places of X, W, A, B (no copy of the weights is made).
 * Adapters of a lower rank are padded with zeros.  16-bit operands of one type, FP32 accumulation, Y in FP32 or rounded
 * once to the operands' type, sums as in nk_grouped.  X . A_a is held in FP32, or where the tensor cores multiply it by B_a (requests of more than eight
 * rows) as the sum of 16-bit numbers.  NK_BF16: two, good to 2^-16 of each element, or for an FP32 Y three (2^-24).  NK_F16: two, good
 * to 2^-22 of each element and never worse than 2^-20 of its row's largest, or for an FP32 Y three (2^-33, 2^-40), whatever the
 * row's size: rows that FP16 has no range for are scaled by a power of two.  (An infinite element of B_a times such a sum is an
 * infinity or NaN.)
 * Offsets that break the rule are clamped and reported by nk_lora_check, as for nk_grouped.
 */
typedef struct nk_lora_s* nk_lora_t;
#define NK_LORA_MAX_RANK 128
#define NK_LORA_MAX_REQUESTS 1024

typedef struct {
    int64_t rows;      /* extent of X and Y; 0 is allowed */
    int64_t N, K;      /* multiples of 8 */
    int64_t rank;      /* a multiple of 8, up to NK_LORA_MAX_RANK */
    int64_t adapters;  /* 1 .. 65535 */
    int64_t requests;  /* 1 .. NK_LORA_MAX_REQUESTS */
    int32_t in_dtype;  /* NK_BF16 or NK_F16: X, W, A, B */
    int32_t out_dtype; /* NK_F32, or the operands' type */
    int32_t layout;    /* NK_ROW_MAJOR or NK_TRANSPOSED, of W, A and B alike */
    int32_t device;
    int64_t ldx, ldw, ldy; /* row strides of X, W and Y; multiples of 8; 0: dense.  A and B are dense */
} nk_lora_desc_t;

nk_status_t nk_lora_create(const nk_lora_desc_t* desc, nk_lora_t* out);
size_t nk_lora_workspace_bytes(nk_lora_t plan); /* contents need no initialisation */
nk_status_t nk_lora_run(nk_lora_t plan, const void* X, const void* W, const void* A, const void* B, const float* scale,
                        const int32_t* offsets, const int32_t* adapter, void* Y, void* workspace, size_t workspace_bytes,
                        void* cuda_stream);
nk_status_t nk_lora_check(nk_lora_t plan); /* as nk_grouped_check */
const char* nk_lora_kernel_name(nk_lora_t plan);
const char* nk_lora_last_cuda_error(nk_lora_t plan);
nk_status_t nk_lora_destroy(nk_lora_t plan);

#ifdef __cplusplus
}
#endif
#endif /* NK_ROWS_H */
