// Host-side pieces of the row-wise operators' plans: the device check, the status word, TMA maps.
#pragma once
#include "../../include/nk_rows.h"
#include "host_util.cuh"

#include <cstdio>
#include <cstring>
#include <mutex>
#include <new>

namespace nk {

constexpr unsigned int STATUS_BAD_OFFSETS = 0x10000u;

// What every plan of this family holds.
struct PlanBase {
    int device, sm_count;
    unsigned int* status_dev;
    bool in_flight, captured;     // a run may not have ended; a graph holds one
    char cuda_err[256];

    nk_status_t cuda(const char* what, cudaError_t e) {
        snprintf(cuda_err, sizeof(cuda_err), "%s: %s", what, cudaGetErrorString(e));
        return NK_ERR_CUDA;
    }
};

static inline bool is_half_type(int dt) { return dt == NK_BF16 || dt == NK_F16; }
static inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// An sm_100 device, made current by the caller's DeviceGuard afterwards.
static inline nk_status_t usable_device(int device, int* sm_count) {
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev <= 0) {
        cudaGetLastError();
        return NK_ERR_DEVICE;
    }
    if (device < 0 || device >= ndev) return NK_ERR_DEVICE;
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess || major != 10 ||
        cudaDeviceGetAttribute(sm_count, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return NK_ERR_DEVICE;
    }
    return NK_OK;
}

static inline nk_status_t base_init(PlanBase* p, int device, int sm_count) {
    p->device = device;
    p->sm_count = sm_count;
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    return take_status_slot(&p->status_dev);
}

// What a run leaves to know for the plan's end.
static inline void base_runs(PlanBase* p, cudaStream_t st) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &status) != cudaSuccess) cudaGetLastError();      // (the launch will say it)
    if (status != cudaStreamCaptureStatusNone) p->captured = true;
    p->in_flight = true;
}

// Synchronises and takes the status word: NK_OK, NK_ERR_INVALID_ARG (offsets) or NK_ERR_TIMEOUT.
static inline nk_status_t base_check(PlanBase* p) {
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return p->cuda("cudaDeviceSynchronize", e);
    p->in_flight = false;
    unsigned int w = 0;
    const unsigned int z = 0;
    if ((e = cudaMemcpy(&w, p->status_dev, sizeof(w), cudaMemcpyDeviceToHost)) != cudaSuccess) return p->cuda("status read", e);
    if (w == 0) return NK_OK;
    cudaMemcpy(p->status_dev, &z, sizeof(z), cudaMemcpyHostToDevice);
    if (w == STATUS_BAD_OFFSETS) {
        snprintf(p->cuda_err, sizeof(p->cuda_err), "offsets out of range or decreasing");
        return NK_ERR_INVALID_ARG;
    }
    snprintf(p->cuda_err, sizeof(p->cuda_err), "device wait gave up, code 0x%x", w);
    return NK_ERR_TIMEOUT;
}

static inline EncodeTiledFn encode_tiled() {
    static EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}

// 16-bit [outer][mid][inner] array as boxes of `box_mid` rows of 64 elements (128 bytes, swizzled); what lies
// outside arrives as zeros.  Strides in elements.
static inline bool encode_map(CUtensorMap* m, const void* base, bool f16, int64_t inner, int64_t mid, int64_t outer,
                              int64_t ld, int64_t stride, int box_mid) {
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(mid), static_cast<cuuint64_t>(outer)};
    // (the outer stride of a single matrix only has to be legal)
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(outer > 1 ? stride : ld) * 2};
    cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_mid), 1};
    cuuint32_t es[3] = {1, 1, 1};
    return encode_tiled()(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base),
                          dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same array with rows of whole slabs of 64 elements seen as [outer][slab][mid][64]: a box is 64 rows of two slabs,
// one slab behind the other.
static inline bool encode_slabs(CUtensorMap* m, const void* base, bool f16, int64_t inner, int64_t mid, int64_t outer,
                                int64_t ld, int64_t stride) {
    cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(mid), static_cast<cuuint64_t>(inner / 64), static_cast<cuuint64_t>(outer)};
    cuuint64_t strides[3] = {static_cast<cuuint64_t>(ld) * 2, 128, static_cast<cuuint64_t>(outer > 1 ? stride : ld) * 2};
    cuuint32_t box[4] = {64, 64, 2, 1};
    cuuint32_t es[4] = {1, 1, 1, 1};
    return encode_tiled()(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base),
                          dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// C as boxes of 2 KB: 32 elements by 32 (16-bit) or 16 (FP32) rows, rows of a box behind one another.
static inline bool encode_out(CUtensorMap* m, void* base, int dtype, int64_t inner, int64_t mid, int64_t outer, int64_t ld, int64_t stride) {
    const int64_t esz = dtype == NK_F32 ? 4 : 2;
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(mid), static_cast<cuuint64_t>(outer)};
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld * esz), static_cast<cuuint64_t>((outer > 1 ? stride : ld) * esz)};
    cuuint32_t box[3] = {32, dtype == NK_F32 ? 16u : 32u, 1};
    cuuint32_t es[3] = {1, 1, 1};
    return encode_tiled()(m, dtype == NK_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == NK_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                          3, base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                          CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A rows' operand in boxes of 16, 32, .. 128 rows.
static inline bool encode_rows(CUtensorMap (&m)[8], const void* base, bool f16, int64_t inner, int64_t rows, int64_t ld) {
    for (int z = 0; z < 8; ++z)
        if (!encode_map(&m[z], base, f16, inner, rows, 1, ld, 0, 16 * (z + 1))) return false;
    return true;
}

}  // namespace nk
