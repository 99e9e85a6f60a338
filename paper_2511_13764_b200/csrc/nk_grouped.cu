// Host side of nk_grouped: descriptor validation, TMA maps, the launch.
#include "rows_host.cuh"
#include "grouped_launch.cuh"
#include "slot_table.h"

namespace nk {

__device__ unsigned int g_split_counter[SlotTable::SLOTS][SPLIT_COUNTERS];
constexpr int MAX_DEVICES = 64;
static SlotTable g_split_slots[MAX_DEVICES];      // (the words are in every device's memory)

int take_split_slot(int device, int pairs, unsigned int** counters) {
    *counters = nullptr;
    void* sym = nullptr;
    if (device >= MAX_DEVICES || 16 * pairs > SPLIT_COUNTERS || cudaGetSymbolAddress(&sym, g_split_counter) != cudaSuccess) {
        cudaGetLastError();
        return -1;
    }
    const int slot = g_split_slots[device].take([] { return cudaDeviceSynchronize() == cudaSuccess; });
    if (slot < 0) {
        cudaGetLastError();
        return -1;
    }
    // zero, whatever the plan before has left (a launch that gave up and was never checked leaves counts), and before any stream's run
    unsigned int* words = static_cast<unsigned int*>(sym) + slot * SPLIT_COUNTERS;
    if (cudaMemset(words, 0, SPLIT_COUNTERS * sizeof(unsigned int)) != cudaSuccess || cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) {
        cudaGetLastError();
        g_split_slots[device].give(slot, false, false);
        return -1;
    }
    *counters = words;
    return slot;
}
void give_split_slot(int device, int slot, bool in_flight, bool captured) {
    if (slot >= 0) g_split_slots[device].give(slot, in_flight, captured);
}

static GroupedFunction function_of(const GroupedKernel& k) {
    return k.mode == GRP_WEIGHTS ? grouped_weights_kernel(k.out, k.sums) : grouped_rows_kernel(k.a_mn, k.out, k.sums);
}
cudaError_t grouped_prepare(const GroupedKernel& k) {
    const int smem = grp_smem(k.out != GRP_OUT_H);
    if (k.mode == GRP_LORA) return cudaFuncSetAttribute(grouped_lora_kernel(k.a_mn, k.out), cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return cudaFuncSetAttribute(function_of(k), cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
}
cudaError_t grouped_launch(const GroupedKernel& k, int pairs, cudaStream_t st, const GroupedMaps& maps, const GroupedParams& p) {
    if (k.mode == GRP_LORA)
        return launch_beside(grouped_lora_kernel(k.a_mn, k.out), 2 * pairs, GRP_THREADS, grp_smem(true), st, static_cast<const LoraMaps&>(maps), p);
    return launch_beside(function_of(k), 2 * pairs, GRP_THREADS, grp_smem(k.out != GRP_OUT_H), st, maps, p);
}

}  // namespace nk

struct nk_grouped_s : nk::PlanBase {
    nk_grouped_desc_t d;          // strides filled in
    int pairs;                    // CTA pairs that fit the device
    nk::GroupedKernel kernel;
    int split_slot;
    unsigned int* counters;
    nk::GroupedMaps maps;
    int slab_cols;                // columns of a slab of partial sums
    const void *cached_a, *cached_b, *cached_c;
    char name[64];
};

using namespace nk;

extern "C" {

nk_status_t nk_grouped_create(const nk_grouped_desc_t* desc, nk_grouped_t* out) {
    if (out) *out = nullptr;
    if (!desc || !out) return NK_ERR_INVALID_ARG;
    nk_grouped_desc_t d = *desc;
    if (d.groups <= 0 || d.rows < 0 || d.N <= 0 || d.K <= 0) return NK_ERR_INVALID_ARG;
    if (d.kind != NK_GROUPED_ROWS && d.kind != NK_GROUPED_WEIGHTS) return NK_ERR_INVALID_ARG;
    if (d.in_dtype < NK_F32 || d.in_dtype > NK_E5M2) return NK_ERR_INVALID_ARG;
    if (!is_half_type(d.in_dtype)) return NK_ERR_UNSUPPORTED;
    if (d.out_dtype != NK_F32 && d.out_dtype != d.in_dtype) return NK_ERR_INVALID_ARG;
    if (d.layout_b != NK_ROW_MAJOR && d.layout_b != NK_TRANSPOSED && d.layout_b != NK_BLOCKED32) return NK_ERR_INVALID_ARG;
    if (d.layout_b == NK_BLOCKED32 || (d.kind == NK_GROUPED_WEIGHTS && d.layout_b != NK_ROW_MAJOR)) return NK_ERR_UNSUPPORTED;
    if (d.beta != 0 && d.beta != 1) return NK_ERR_INVALID_ARG;
    if (d.groups > NK_GROUPED_MAX_GROUPS || d.N > (1 << 24) || d.K > (1 << 24) || d.rows >= (1ll << 31) - 4096) return NK_ERR_UNSUPPORTED;
    if (d.N % 8 || d.K % 8 || d.lda % 8 || d.ldb % 8 || d.ldc % 8 || d.stride_g % 8) return NK_ERR_MISALIGNED;
    const bool weights = d.kind == NK_GROUPED_WEIGHTS;
    const int64_t b_cols = weights || d.layout_b == NK_ROW_MAJOR ? d.N : d.K;       // width of B's rows
    const int64_t b_rows = d.layout_b == NK_ROW_MAJOR ? d.K : d.N;                  // rows of one B_g
    if (d.lda == 0) d.lda = d.K;
    if (d.ldb == 0) d.ldb = b_cols;
    if (d.ldc == 0) d.ldc = d.N;
    if (d.lda < d.K || d.ldb < b_cols || d.ldc < d.N) return NK_ERR_INVALID_ARG;
    const int64_t item = weights ? d.K * d.ldc : b_rows * d.ldb;
    if (d.stride_g == 0) d.stride_g = item;
    if (d.stride_g < item) return NK_ERR_INVALID_ARG;                               // items overlap
    // TMA strides are below 2^40 bytes; unit numbers stay below 2^24
    if (d.lda >= (1ll << 37) || d.ldb >= (1ll << 37) || d.ldc >= (1ll << 37) || d.stride_g >= (1ll << 37)) return NK_ERR_UNSUPPORTED;
    const int64_t tiles = weights ? d.groups * div_up(d.N, 256) * div_up(d.K, 256) : (d.rows / 32 + d.groups) * div_up(d.N, 256);
    if (tiles >= (1 << 24)) return NK_ERR_UNSUPPORTED;
    if (weights && (d.rows / 64 + d.groups) * div_up(d.N, 256) * div_up(d.K, 256) >= (1ll << 31)) return NK_ERR_UNSUPPORTED;   // k-blocks of all tiles

    int sms = 0;
    nk_status_t s = usable_device(d.device, &sms);
    if (s != NK_OK) return s;
    nk_grouped_s* p = new (std::nothrow) nk_grouped_s();
    if (!p) return NK_ERR_INVALID_ARG;
    p->d = d;
    p->split_slot = -1;
    if ((s = base_init(p, d.device, sms)) != NK_OK) { delete p; return s; }
    DeviceGuard guard(d.device);
    if (!encode_tiled()) { delete p; return NK_ERR_CUDA; }
    p->kernel = grouped_choose(weights ? GRP_WEIGHTS : GRP_ROWS, weights || d.layout_b == NK_ROW_MAJOR,
                               grouped_out(d.out_dtype != NK_F32, d.in_dtype == NK_F16), weights ? d.rows : d.K);
    if (grouped_prepare(p->kernel) != cudaSuccess) { delete p; return NK_ERR_CUDA; }
    p->pairs = sms / 2;
    p->slab_cols = grouped_slab_cols(weights ? d.K : d.rows);
    p->split_slot = take_split_slot(d.device, p->pairs, &p->counters);
    snprintf(p->name, sizeof(p->name), "grouped_%s_256x256x64_pair%s", weights ? "weights" : d.layout_b == NK_TRANSPOSED ? "rows_t" : "rows",
             p->split_slot < 0 ? "_uncut" : "");
    *out = p;
    return NK_OK;
}

// partial sums of cut tiles: two FP32 slabs for each pair
size_t nk_grouped_workspace_bytes(nk_grouped_t p) {
    if (!p || p->split_slot < 0) return 0;
    return grouped_partial_bytes(p->pairs, p->slab_cols);
}

nk_status_t nk_grouped_run(nk_grouped_t p, const void* A, const void* B, void* C, const int32_t* offsets, void* workspace,
                           size_t workspace_bytes, void* cuda_stream) {
    if (!p || !offsets) return NK_ERR_INVALID_ARG;
    const nk_grouped_desc_t& d = p->d;
    const bool weights = d.kind == NK_GROUPED_WEIGHTS;
    if (!weights && d.rows == 0) return NK_OK;
    if (!C || (d.rows > 0 && (!A || !B))) return NK_ERR_INVALID_ARG;
    if (misaligned16(A) || misaligned16(B) || misaligned16(C) || misaligned16(workspace) || (reinterpret_cast<uintptr_t>(offsets) & 3u))
        return NK_ERR_MISALIGNED;
    const size_t need = nk_grouped_workspace_bytes(p);
    if (need && (!workspace || workspace_bytes < need)) return NK_ERR_WORKSPACE;
    DeviceGuard guard(d.device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    if (d.rows == 0) A = B = C;        // no row is loaded; the maps only need an address
    const int64_t rows = d.rows ? d.rows : 1;
    if (p->cached_c != C || p->cached_a != A || p->cached_b != B) {
        const bool f16 = d.in_dtype == NK_F16;
        bool ok;
        GroupedMaps& m = p->maps;
        if (weights) {
            ok = encode_out(&m.out, C, d.out_dtype, d.N, d.K, d.groups, d.ldc, d.stride_g) &&
                 (d.N % 64 == 0 ? encode_slabs(&m.a, B, f16, d.N, rows, 1, d.ldb, 0) : encode_map(&m.a, B, f16, d.N, rows, 1, d.ldb, 0, 64)) &&
                 encode_map(&m.b[0], A, f16, d.K, rows, 1, d.lda, 0, 64) && (d.K % 64 != 0 || encode_slabs(&m.b[1], A, f16, d.K, rows, 1, d.lda, 0));
        } else {
            ok = encode_rows(m.b, A, f16, d.K, rows, d.lda) && encode_out(&m.out, C, d.out_dtype, d.N, rows, 1, d.ldc, 0) &&
                 (d.layout_b == NK_TRANSPOSED ? encode_map(&m.a, B, f16, d.K, d.N, d.groups, d.ldb, d.stride_g, 128)
                  : d.N % 64 == 0             ? encode_slabs(&m.a, B, f16, d.N, d.K, d.groups, d.ldb, d.stride_g)
                                              : encode_map(&m.a, B, f16, d.N, d.K, d.groups, d.ldb, d.stride_g, 64));
        }
        if (!ok) {
            p->cached_c = nullptr;
            snprintf(p->cuda_err, sizeof(p->cuda_err), "cuTensorMapEncodeTiled failed");
            return NK_ERR_CUDA;
        }
        p->cached_a = A;
        p->cached_b = B;
        p->cached_c = C;               // (C is never null: the maps are valid)
    }
    GroupedParams g = {};
    g.groups = static_cast<int>(d.groups);
    g.rows = static_cast<int>(d.rows);
    g.I = static_cast<int>(d.N);
    g.J = static_cast<int>(d.K);
    g.kb_total = static_cast<int>(div_up(d.K, GRP_BK));
    g.tiles_i = static_cast<int>(div_up(d.N, GRP_TILE));
    g.tiles_j = static_cast<int>(div_up(d.K, GRP_TILE));
    g.beta = d.beta;
    g.f16 = d.in_dtype == NK_F16;
    g.idesc = grouped_idesc(weights || d.layout_b == NK_ROW_MAJOR, weights, g.f16);
    g.offsets = offsets;
    g.C = C;
    g.ldc = d.ldc;
    g.stride_c = d.stride_g;
    g.partial = need ? static_cast<float*>(workspace) : nullptr;
    g.counter = p->counters;
    g.status = p->status_dev;
    g.slab_cols = p->slab_cols;
    g.a_slabs = d.N % 64 == 0;
    g.b_slabs = d.K % 64 == 0;
    g.chunk = p->kernel.chunk();
    base_runs(p, static_cast<cudaStream_t>(cuda_stream));
    const cudaError_t e = grouped_launch(p->kernel, p->pairs, static_cast<cudaStream_t>(cuda_stream), p->maps, g);
    return e == cudaSuccess ? NK_OK : p->cuda("grouped launch", e);
}

nk_status_t nk_grouped_check(nk_grouped_t p) {
    if (!p) return NK_ERR_INVALID_ARG;
    const nk_status_t s = base_check(p);
    if (s == NK_ERR_TIMEOUT && p->counters) {
        DeviceGuard guard(p->device);
        cudaMemset(p->counters, 0, SPLIT_COUNTERS * sizeof(unsigned int));   // an abandoned tile may have left a count
    }
    return s;
}

const char* nk_grouped_kernel_name(nk_grouped_t p) { return p ? p->name : ""; }
const char* nk_grouped_last_cuda_error(nk_grouped_t p) { return p ? p->cuda_err : ""; }

nk_status_t nk_grouped_destroy(nk_grouped_t p) {
    if (p) give_split_slot(p->device, p->split_slot, p->in_flight, p->captured);
    delete p;
    return NK_OK;
}

}  // extern "C"
