// Host side of nk_lora: descriptor validation, TMA maps, the launches.
#include "rows_host.cuh"
#include "grouped_launch.cuh"
#include "lora.cuh"

struct nk_lora_s : nk::PlanBase {
    nk_lora_desc_t d;             // strides filled in
    int pairs, split_slot;
    unsigned int* counters;
    CUtensorMap map_w, map_x, map_x16;
    const void *cached_x, *cached_w;
    char name[64];
};

using namespace nk;

namespace nk {

static size_t align256(size_t x) { return (x + 255) / 256 * 256; }
static size_t lora_delta_bytes(const nk_lora_desc_t& d) { return align256(static_cast<size_t>(d.rows) * d.N * sizeof(float)); }

}  // namespace nk

extern "C" {

nk_status_t nk_lora_create(const nk_lora_desc_t* desc, nk_lora_t* out) {
    if (out) *out = nullptr;
    if (!desc || !out) return NK_ERR_INVALID_ARG;
    nk_lora_desc_t d = *desc;
    if (d.rows < 0 || d.N <= 0 || d.K <= 0 || d.rank <= 0 || d.adapters <= 0 || d.requests <= 0) return NK_ERR_INVALID_ARG;
    if (d.in_dtype < NK_F32 || d.in_dtype > NK_E5M2) return NK_ERR_INVALID_ARG;
    if (!is_half_type(d.in_dtype)) return NK_ERR_UNSUPPORTED;
    if (d.out_dtype != NK_F32 && d.out_dtype != d.in_dtype) return NK_ERR_INVALID_ARG;
    if (d.layout != NK_ROW_MAJOR && d.layout != NK_TRANSPOSED && d.layout != NK_BLOCKED32) return NK_ERR_INVALID_ARG;
    if (d.layout == NK_BLOCKED32) return NK_ERR_UNSUPPORTED;
    if (d.rank > NK_LORA_MAX_RANK || d.requests > NK_LORA_MAX_REQUESTS || d.adapters > 65535) return NK_ERR_UNSUPPORTED;
    if (d.rows > (1 << 24) || d.N > (1 << 24) || d.K > (1 << 24)) return NK_ERR_UNSUPPORTED;
    if (d.N % 8 || d.K % 8 || d.rank % 8 || d.ldx % 8 || d.ldw % 8 || d.ldy % 8) return NK_ERR_MISALIGNED;
    const int64_t w_cols = d.layout == NK_ROW_MAJOR ? d.N : d.K;
    if (d.ldx == 0) d.ldx = d.K;
    if (d.ldw == 0) d.ldw = w_cols;
    if (d.ldy == 0) d.ldy = d.N;
    if (d.ldx < d.K || d.ldw < w_cols || d.ldy < d.N) return NK_ERR_INVALID_ARG;
    if (d.ldx >= (1ll << 38) || d.ldw >= (1ll << 38)) return NK_ERR_UNSUPPORTED;
    if ((d.rows / 256 + 1) * div_up(d.N, 256) >= (1 << 24)) return NK_ERR_UNSUPPORTED;
    int sms = 0;
    nk_status_t s = usable_device(d.device, &sms);
    if (s != NK_OK) return s;
    nk_lora_s* p = new (std::nothrow) nk_lora_s();
    if (!p) return NK_ERR_INVALID_ARG;
    p->d = d;
    p->split_slot = -1;
    if ((s = base_init(p, d.device, sms)) != NK_OK) { delete p; return s; }
    DeviceGuard guard(d.device);
    if (!encode_tiled() || grouped_prepare(false, d.layout == NK_ROW_MAJOR) != cudaSuccess ||
        cudaFuncSetAttribute(lora_delta_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LORA_SMEM) != cudaSuccess) {
        delete p;
        return NK_ERR_CUDA;
    }
    p->pairs = sms / 2;
    p->split_slot = take_split_slot(&p->counters);
    snprintf(p->name, sizeof(p->name), "lora_delta_%s", d.layout == NK_TRANSPOSED ? "rows_t" : "rows");
    *out = p;
    return NK_OK;
}

size_t nk_lora_workspace_bytes(nk_lora_t p) {
    if (!p) return 0;
    return lora_delta_bytes(p->d) + (p->split_slot < 0 ? 0 : grouped_partial_bytes(p->pairs));
}

nk_status_t nk_lora_run(nk_lora_t p, const void* X, const void* W, const void* A, const void* B, const float* scale,
                        const int32_t* offsets, const int32_t* adapter, void* Y, void* workspace, size_t workspace_bytes,
                        void* cuda_stream) {
    if (!p) return NK_ERR_INVALID_ARG;
    const nk_lora_desc_t& d = p->d;
    if (d.rows == 0) return NK_OK;
    if (!X || !W || !A || !B || !scale || !offsets || !adapter || !Y) return NK_ERR_INVALID_ARG;
    if (misaligned16(X) || misaligned16(W) || misaligned16(A) || misaligned16(B) || misaligned16(Y) || misaligned16(workspace) ||
        ((reinterpret_cast<uintptr_t>(scale) | reinterpret_cast<uintptr_t>(offsets) | reinterpret_cast<uintptr_t>(adapter)) & 3u))
        return NK_ERR_MISALIGNED;
    if (!workspace || workspace_bytes < nk_lora_workspace_bytes(p)) return NK_ERR_WORKSPACE;
    DeviceGuard guard(d.device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    const bool f16 = d.in_dtype == NK_F16;
    if (p->cached_x != X || p->cached_w != W) {
        p->cached_x = nullptr;
        const bool ok = (d.layout == NK_ROW_MAJOR ? encode_map(&p->map_w, W, f16, d.N, d.K, 1, d.ldw, 0, 64)
                                                  : encode_map(&p->map_w, W, f16, d.K, d.N, 1, d.ldw, 0, 128)) &&
                        encode_map(&p->map_x, X, f16, d.K, d.rows, 1, d.ldx, 0, 128) &&
                        encode_map(&p->map_x16, X, f16, d.K, d.rows, 1, d.ldx, 0, 16);
        if (!ok) {
            snprintf(p->cuda_err, sizeof(p->cuda_err), "cuTensorMapEncodeTiled failed");
            return NK_ERR_CUDA;
        }
        p->cached_x = X;
        p->cached_w = W;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    float* delta = static_cast<float*>(workspace);
    LoraParams l = {};
    l.rows = static_cast<int>(d.rows);
    l.N = static_cast<int>(d.N);
    l.K = static_cast<int>(d.K);
    l.rank = static_cast<int>(d.rank);
    l.adapters = static_cast<int>(d.adapters);
    l.requests = static_cast<int>(d.requests);
    l.transposed = d.layout == NK_TRANSPOSED;
    l.f16 = f16;
    l.ldx = d.ldx;
    l.X = X;
    l.A = A;
    l.B = B;
    l.scale = scale;
    l.offsets = offsets;
    l.adapter = adapter;
    l.D = delta;
    l.status = p->status_dev;
    // clusters: no more than there can be chunks of rows, and a few for every SM
    const int64_t chunks = d.rows / LORA_ROWS + (d.rows < d.requests ? d.rows : d.requests);
    const int64_t most = 4 * p->sm_count / LORA_CLUSTER;
    lora_delta_kernel<<<static_cast<unsigned>((chunks < most ? chunks : most) * LORA_CLUSTER), LORA_THREADS, LORA_SMEM, st>>>(l);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return p->cuda("lora delta launch", e);

    GroupedParams g = {};
    g.groups = 1;
    g.rows = l.rows;
    g.I = l.N;
    g.J = l.K;
    g.kb_total = static_cast<int>(div_up(d.K, GRP_BK));
    g.tiles_i = static_cast<int>(div_up(d.N, GRP_TILE));
    g.out16 = d.out_dtype != NK_F32;
    g.f16 = f16;
    g.idesc = grouped_idesc(d.layout == NK_ROW_MAJOR, false, f16);
    g.C = Y;
    g.ldc = d.ldy;
    g.add = delta;
    g.partial = p->split_slot < 0 ? nullptr : reinterpret_cast<float*>(static_cast<char*>(workspace) + lora_delta_bytes(d));
    g.counter = p->counters;
    g.status = p->status_dev;
    e = grouped_launch(false, d.layout == NK_ROW_MAJOR, p->pairs, st, p->map_w, p->map_x, p->map_x16, g);
    return e == cudaSuccess ? NK_OK : p->cuda("lora projection launch", e);
}

nk_status_t nk_lora_check(nk_lora_t p) {
    if (!p) return NK_ERR_INVALID_ARG;
    const nk_status_t s = base_check(p);
    if (s == NK_ERR_TIMEOUT && p->counters) {
        DeviceGuard guard(p->device);
        cudaMemset(p->counters, 0, SPLIT_COUNTERS * sizeof(unsigned int));   // an abandoned tile may have left a count
    }
    return s;
}

const char* nk_lora_kernel_name(nk_lora_t p) { return p ? p->name : ""; }
const char* nk_lora_last_cuda_error(nk_lora_t p) { return p ? p->cuda_err : ""; }

nk_status_t nk_lora_destroy(nk_lora_t p) {
    if (p) give_split_slot(p->split_slot);
    delete p;
    return NK_OK;
}

}  // extern "C"
