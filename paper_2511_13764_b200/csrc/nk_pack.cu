// Host side of nk_pack: descriptor validation and the launches.
#include "rows_host.cuh"
#include "../../include/nk_mx.h"
#include "pack.cuh"

struct nk_pack_s : nk::PlanBase {
    nk_pack_desc_t d;             // strides filled in
    int outer, length;            // of the packed matrix
    int row_tiles, tiles;         // of scales
    int max_blocks;               // of the tensor's scale, for each matrix; one: a single launch
    char name[64];
};

using namespace nk;

namespace nk {

typedef void (*PackFunction)(PackParams);
template <int T>
static PackFunction pack_kernel(bool nv, bool columns) {
    return columns ? nv ? pack_columns_kernel<T, true> : pack_columns_kernel<T, false> : nv ? pack_rows_kernel<T, true> : pack_rows_kernel<T, false>;
}
static PackFunction pack_kernel_of(const nk_pack_desc_t& d) {
    const bool nv = d.format == NK_NVF4;
    return d.in_dtype == NK_F32 ? pack_kernel<0>(nv, d.transposed) : d.in_dtype == NK_BF16 ? pack_kernel<1>(nv, d.transposed) : pack_kernel<2>(nv, d.transposed);
}
static PackFunction values_kernel_of(const nk_pack_desc_t& d) {
    const bool nv = d.format == NK_NVF4;
    return d.value_dtype == NK_F32    ? nv ? pack_values_kernel<0, true> : pack_values_kernel<0, false>
           : d.value_dtype == NK_BF16 ? nv ? pack_values_kernel<1, true> : pack_values_kernel<1, false>
                                      : nv ? pack_values_kernel<2, true> : pack_values_kernel<2, false>;
}

static PackParams pack_params(const nk_pack_s* p) {
    PackParams r = {};
    r.nv = p->d.format == NK_NVF4;
    r.outer = p->outer;
    r.groups = static_cast<int>(p->d.groups);
    r.length = p->length;
    r.row_tiles = p->row_tiles;
    r.chunks = static_cast<int>(div_up(mx_padded(p->length), pack_chunk(r.nv)));
    r.tiles = p->tiles;
    r.ldx = p->d.ldx;
    r.stride_x = p->d.stride_x;
    r.status = p->status_dev;
    return r;
}

static inline bool float_type(int dt) { return dt == NK_F32 || is_half_type(dt); }

}  // namespace nk

extern "C" {

nk_status_t nk_pack_create(const nk_pack_desc_t* desc, nk_pack_t* out) {
    if (out) *out = nullptr;
    if (!desc || !out) return NK_ERR_INVALID_ARG;
    nk_pack_desc_t d = *desc;
    if (d.batch == 0) d.batch = 1;
    if (d.rows < 0 || d.K <= 0 || d.batch < 0 || d.groups < 0) return NK_ERR_INVALID_ARG;
    if ((d.format != NK_MXF4 && d.format != NK_NVF4) || (d.transposed != 0 && d.transposed != 1)) return NK_ERR_INVALID_ARG;
    if (d.in_dtype < NK_F32 || d.in_dtype > NK_E5M2 || d.value_dtype < NK_F32 || d.value_dtype > NK_E5M2) return NK_ERR_INVALID_ARG;
    if (!float_type(d.in_dtype) || !float_type(d.value_dtype)) return NK_ERR_UNSUPPORTED;
    if (d.groups > 0 && (d.batch > 1 || d.transposed)) return NK_ERR_UNSUPPORTED;
    if (d.K % 8 || d.ldx % 8 || d.stride_x % 8) return NK_ERR_MISALIGNED;
    if (d.ldx == 0) d.ldx = d.K;
    if (d.ldx < d.K) return NK_ERR_INVALID_ARG;
    if (d.rows >= (1ll << 31) - 4096 || d.K > (1 << 24) || d.ldx >= (1ll << 36) || d.batch > 65535 || d.groups > NK_GROUPED_MAX_GROUPS)
        return NK_ERR_UNSUPPORTED;
    if (d.stride_x == 0) d.stride_x = d.rows * d.ldx;
    if (d.batch > 1 && d.stride_x < (d.rows ? (d.rows - 1) * d.ldx + d.K : 0)) return NK_ERR_INVALID_ARG;   // matrices overlap
    const int64_t outer = d.transposed ? d.K : d.rows, length = d.transposed ? d.rows : d.K;
    // grids: along the rows (and reading back) tiles x pieces, below 2^31; along the columns pieces in y
    if (d.transposed && div_up(mx_padded(length), PACK_TURN) > 65535) return NK_ERR_UNSUPPORTED;
    if ((outer / MX_TILE_ROWS + (d.groups ? d.groups : 1)) * div_up(mx_padded(length), 128) >= (1ll << 31)) return NK_ERR_UNSUPPORTED;
    int sms = 0;
    nk_status_t s = usable_device(d.device, &sms);
    if (s != NK_OK) return s;
    nk_pack_s* p = new (std::nothrow) nk_pack_s();
    if (!p) return NK_ERR_INVALID_ARG;
    p->d = d;
    if ((s = base_init(p, d.device, sms)) != NK_OK) { delete p; return s; }
    p->outer = static_cast<int>(outer);
    p->length = static_cast<int>(length);
    p->row_tiles = static_cast<int>(d.groups ? outer / MX_TILE_ROWS + d.groups : div_up(outer, MX_TILE_ROWS));
    p->tiles = static_cast<int>(mx_tiles(length, d.format == NK_NVF4));
    // the tensor's scale: up to half a million elements are one cluster's (a second launch costs more: 16 x 4096 2.9 us instead of 3.7); else
    // blocks of 256, a turn of 64 elements to a thread (FP32: 32) each at least, four to an SM over the whole batch
    const int64_t turns = div_up(d.rows * d.K, PACK_THREADS * (d.in_dtype == NK_F32 ? 32 : 64)), most = div_up(4 * static_cast<int64_t>(sms), d.batch);
    p->max_blocks = static_cast<int>(d.rows * d.K <= (1 << 19) ? 1 : turns < most ? turns : most);
    DeviceGuard guard(d.device);
    if (d.transposed && cudaFuncSetAttribute(pack_kernel_of(d), cudaFuncAttributeMaxDynamicSharedMemorySize, pack_columns_smem(d.in_dtype == NK_F32 ? 0 : 1)) != cudaSuccess) {
        delete p;
        return NK_ERR_CUDA;
    }
    snprintf(p->name, sizeof(p->name), "pack_%s_%s%s", d.format == NK_NVF4 ? "nvf4" : "mxf4", d.transposed ? "columns" : "rows", d.groups ? "_grouped" : "");
    *out = p;
    return NK_OK;
}

size_t nk_pack_data_bytes(nk_pack_t p) {
    return p ? static_cast<size_t>(p->d.batch) * p->outer * (mx_padded(p->length) / 2) : 0;
}
size_t nk_pack_scales_bytes(nk_pack_t p) {
    return p ? static_cast<size_t>(p->d.batch) * p->row_tiles * p->tiles * MX_TILE_BYTES : 0;
}
size_t nk_pack_workspace_bytes(nk_pack_t p) {
    return p && p->d.format == NK_NVF4 && p->max_blocks > 1 ? static_cast<size_t>(p->d.batch) * p->max_blocks * sizeof(uint32_t) : 0;
}

nk_status_t nk_pack_scale(nk_pack_t p, const void* X, float* scale, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!p || !scale || (p->d.rows > 0 && !X)) return NK_ERR_INVALID_ARG;
    if (p->d.format != NK_NVF4) return NK_ERR_UNSUPPORTED;
    if (misaligned16(X) || (reinterpret_cast<uintptr_t>(scale) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 3u)) return NK_ERR_MISALIGNED;
    const size_t need = nk_pack_workspace_bytes(p);
    if (need && (!workspace || workspace_bytes < need)) return NK_ERR_WORKSPACE;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    PackParams r = pack_params(p);
    r.x = X;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const dim3 grid(p->max_blocks, static_cast<unsigned>(p->d.batch));
    uint32_t* partial = static_cast<uint32_t*>(workspace);
    const int rows = static_cast<int>(p->d.rows), width = static_cast<int>(p->d.K);
    cudaError_t e;
    if (p->max_blocks == 1)
        e = launch_beside(p->d.in_dtype == NK_F32 ? tensor_cluster_kernel<0> : p->d.in_dtype == NK_BF16 ? tensor_cluster_kernel<1> : tensor_cluster_kernel<2>,
                          dim3(SCALE_CLUSTER, static_cast<unsigned>(p->d.batch)), SCALE_THREADS, 0, st, r, rows, width, scale);
    else
        e = launch_beside(p->d.in_dtype == NK_F32 ? tensor_max_kernel<0> : p->d.in_dtype == NK_BF16 ? tensor_max_kernel<1> : tensor_max_kernel<2>, grid,
                          PACK_THREADS, 0, st, r, rows, width, partial);
    if (e != cudaSuccess) return p->cuda("tensor max launch", e);
    if (p->max_blocks > 1 && (e = launch_beside(tensor_scale_kernel, static_cast<unsigned>(p->d.batch), PACK_THREADS, 0, st, partial, p->max_blocks, scale)) != cudaSuccess)
        return p->cuda("tensor scale launch", e);
    return NK_OK;
}

nk_status_t nk_pack_run(nk_pack_t p, const void* X, const float* scale, const int32_t* offsets, void* data, void* scales, void* cuda_stream) {
    if (!p || (p->d.groups > 0) != (offsets != nullptr)) return NK_ERR_INVALID_ARG;
    if (scale && p->d.format != NK_NVF4) return NK_ERR_INVALID_ARG;
    if (p->d.rows == 0) return NK_OK;
    if (!X || !data || !scales) return NK_ERR_INVALID_ARG;
    if (misaligned16(X) || misaligned16(data) || misaligned16(scales) || (reinterpret_cast<uintptr_t>(scale) & 3u) || (reinterpret_cast<uintptr_t>(offsets) & 3u))
        return NK_ERR_MISALIGNED;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    PackParams r = pack_params(p);
    r.x = X;
    r.scale = scale;
    r.offsets = offsets;
    r.data = static_cast<uint8_t*>(data);
    r.scales = static_cast<uint8_t*>(scales);
    const dim3 grid = p->d.transposed ? dim3(p->row_tiles, static_cast<unsigned>(div_up(mx_padded(p->length), PACK_TURN)), static_cast<unsigned>(p->d.batch))
                                      : dim3(static_cast<unsigned>(p->row_tiles) * r.chunks, 1, static_cast<unsigned>(p->d.batch));
    const cudaError_t e = launch_beside(pack_kernel_of(p->d), grid, PACK_THREADS, p->d.transposed ? pack_columns_smem(p->d.in_dtype == NK_F32 ? 0 : 1) : 0,
                                        static_cast<cudaStream_t>(cuda_stream), r);
    return e == cudaSuccess ? NK_OK : p->cuda("pack launch", e);
}

nk_status_t nk_pack_values(nk_pack_t p, const void* data, const void* scales, const float* scale, const int32_t* offsets, void* Y, void* cuda_stream) {
    if (!p || (p->d.groups > 0) != (offsets != nullptr)) return NK_ERR_INVALID_ARG;
    if (scale && p->d.format != NK_NVF4) return NK_ERR_INVALID_ARG;
    if (p->d.rows == 0) return NK_OK;
    if (!data || !scales || !Y) return NK_ERR_INVALID_ARG;
    if (misaligned16(data) || misaligned16(scales) || misaligned16(Y) || (reinterpret_cast<uintptr_t>(scale) & 3u) || (reinterpret_cast<uintptr_t>(offsets) & 3u))
        return NK_ERR_MISALIGNED;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    PackParams r = pack_params(p);
    r.scale = scale;
    r.offsets = offsets;
    r.data = static_cast<uint8_t*>(const_cast<void*>(data));
    r.scales = static_cast<uint8_t*>(const_cast<void*>(scales));
    r.values = Y;
    r.chunks = static_cast<int>(div_up(mx_padded(p->length), PACK_LINE));
    const dim3 grid(static_cast<unsigned>(p->row_tiles) * r.chunks, 1, static_cast<unsigned>(p->d.batch));
    const cudaError_t e = launch_beside(values_kernel_of(p->d), grid, PACK_THREADS, 0, static_cast<cudaStream_t>(cuda_stream), r);
    return e == cudaSuccess ? NK_OK : p->cuda("values launch", e);
}

nk_status_t nk_pack_check(nk_pack_t p) { return p ? base_check(p) : NK_ERR_INVALID_ARG; }
const char* nk_pack_kernel_name(nk_pack_t p) { return p ? p->name : ""; }
const char* nk_pack_last_cuda_error(nk_pack_t p) { return p ? p->cuda_err : ""; }

nk_status_t nk_pack_destroy(nk_pack_t p) {
    delete p;
    return NK_OK;
}

}  // extern "C"
