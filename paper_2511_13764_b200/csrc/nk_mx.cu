// Host side of nk_mx: descriptor validation, TMA maps, the launch.
#include "rows_host.cuh"
#include "../../include/nk_mx.h"
#include "grouped_launch.cuh"
#include "mx_format.cuh"
#include "mx_launch.cuh"

namespace nk {

// bytes [outer][mid][inner] as boxes of `box_mid` rows of 128 bytes, swizzled; what lies outside arrives as zeros
static bool encode_packed(CUtensorMap* m, const void* base, int64_t inner, int64_t mid, int64_t outer, int box_mid) {
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(mid), static_cast<cuuint64_t>(outer)};
    // (the outer stride of a single matrix only has to be legal)
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(outer > 1 ? inner * mid : inner)};
    cuuint32_t box[3] = {128, static_cast<cuuint32_t>(box_mid), 1};
    cuuint32_t es[3] = {1, 1, 1};
    return encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// tiles of scales [rows][tiles][512 bytes] as boxes of `box` tiles of a row
static bool encode_scales(CUtensorMap* m, const void* base, int64_t tiles, int64_t rows, int box_tiles) {
    cuuint64_t dims[3] = {MX_TILE_BYTES / 4, static_cast<cuuint64_t>(tiles), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[2] = {MX_TILE_BYTES, static_cast<cuuint64_t>(MX_TILE_BYTES * tiles)};
    cuuint32_t box[3] = {MX_TILE_BYTES / 4, static_cast<cuuint32_t>(box_tiles), 1};
    cuuint32_t es[3] = {1, 1, 1};
    return encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of one group of rows: their width, and into how many parts those of the last, partial wave are cut, by the least estimated time.
// Joining parts costs 2900 clocks and 700 a part, and what is written and read again of them at 3500 bytes a clock.  (16 rows, 4096
// features: K 4096 10.0 us uncut, 9.7 in four parts, K 8192 14.8 and 11.5; 128 rows, K 4096 10.8 uncut, 12.1 in four.  Groups' tiles are never
// cut: their number is known on the device alone, where the choice costs every launch 1.5 us.  Below K = 8192 cuts gained nothing there; what
// longer contractions with few tiles would gain, as one group's do, was not measured.)
static void mx_tiles_of(int64_t rows, int tiles_i, int kbs, int pairs, bool cut, int* width, int* parts) {
    double best = 1e300;
    for (int w = rows <= 32 ? 32 : 64; w <= MX_TILE; w += w < 64 ? 32 : 64) {
        const int64_t n = div_up(rows, w) * tiles_i, waves = n / pairs, rest = n % pairs;
        auto block = [&](int64_t active) {
            return MX_ALONE_CLOCKS + (mx_block_clocks(w) - MX_ALONE_CLOCKS) * (active < pairs ? static_cast<double>(active) / pairs : 1.0);
        };
        const double full = static_cast<double>(waves) * (kbs * block(pairs) + MX_TILE_CLOCKS), end = MX_TILE_CLOCKS + MX_ROW_CLOCKS * w;
        for (int c = 1; c == 1 || (cut && rest && c <= 8 && c <= kbs && c * rest <= pairs); ++c) {
            const double join = c > 1 ? 2900.0 + 700.0 * c + static_cast<double>(rest * c) * w * (2048.0 / 3500.0) : 0.0;
            const double t = full + (rest ? div_up(kbs, c) * block(rest * c) : 0.0) + end + join;
            if (t < best * 0.999 || (t <= best * 1.001 && c == 1 && *parts == 1)) {      // (of equals the widest)
                best = t < best ? t : best;
                *width = w;
                *parts = c;
            }
        }
        if (w >= rows) break;
    }
}

}  // namespace nk

struct nk_mx_s : nk::PlanBase {
    nk_mx_desc_t d;               // strides filled in
    int pairs;                    // CTA pairs that fit the device
    nk::MxFunction kernel;
    int chunk;
    nk::MxMode mode;
    int width, parts;             // of one group's tiles; groups: 0, 1
    int split_slot;
    unsigned int* counters;
    nk::MxMaps maps;
    int slab_cols;                // columns of a slab of partial sums
    const void* cached[4];        // what the maps are of: A, its scales, B, its scales
    char name[64];
};

using namespace nk;

extern "C" {

nk_status_t nk_mx_create(const nk_mx_desc_t* desc, nk_mx_t* out) {
    if (out) *out = nullptr;
    if (!desc || !out) return NK_ERR_INVALID_ARG;
    nk_mx_desc_t d = *desc;
    if (d.groups < 0 || d.rows < 0 || d.N <= 0 || d.K <= 0) return NK_ERR_INVALID_ARG;
    if ((d.format != NK_MXF4 && d.format != NK_NVF4) || d.out_dtype < NK_F32 || d.out_dtype > NK_E5M2) return NK_ERR_INVALID_ARG;
    if (d.out_dtype != NK_F32 && !is_half_type(d.out_dtype)) return NK_ERR_UNSUPPORTED;
    if ((d.epilogue != NK_EPI_NONE && d.epilogue != NK_EPI_BIAS_RELU) || (d.beta != 0 && d.beta != 1)) return NK_ERR_INVALID_ARG;
    if (d.groups > NK_GROUPED_MAX_GROUPS || d.N > (1 << 24) || d.K >= (1ll << 31) - 4096 || d.rows >= (1ll << 31) - 4096) return NK_ERR_UNSUPPORTED;
    if (d.N % 8 || d.ldc % 8) return NK_ERR_MISALIGNED;
    if (d.ldc == 0) d.ldc = d.N;
    if (d.ldc < d.N) return NK_ERR_INVALID_ARG;
    const int64_t groups = d.groups ? d.groups : 1;
    // TMA strides are below 2^40 bytes; unit numbers stay below 2^24
    if (d.ldc >= (1ll << 37) || d.N * mx_padded(d.K) >= (1ll << 40)) return NK_ERR_UNSUPPORTED;
    if ((d.rows / 64 + groups) * div_up(d.N, MX_TILE) >= (1 << 24)) return NK_ERR_UNSUPPORTED;
    int sms = 0;
    nk_status_t s = usable_device(d.device, &sms);
    if (s != NK_OK) return s;
    nk_mx_s* p = new (std::nothrow) nk_mx_s();
    if (!p) return NK_ERR_INVALID_ARG;
    p->d = d;
    p->split_slot = -1;
    if ((s = base_init(p, d.device, sms)) != NK_OK) { delete p; return s; }
    DeviceGuard guard(d.device);
    if (!encode_tiled()) { delete p; return NK_ERR_CUDA; }
    const MxOut type = d.out_dtype == NK_F32 ? MX_OUT_F32 : d.out_dtype == NK_BF16 ? MX_OUT_BF16 : MX_OUT_F16;
    const bool sums = div_up(d.K, MX_BK) > (type == MX_OUT_F32 ? MX_WHOLE : MX_WHOLE_16);
    p->chunk = type == MX_OUT_F32 ? MX_CHUNK : MX_WHOLE_16;
    bool uncut = false;
    p->pairs = sms / 2;
    p->slab_cols = static_cast<int>(d.rows >= MX_TILE ? MX_TILE : div_up(d.rows, 32) * 32);
    p->parts = 1;
    if (!d.groups) {
        const int tiles_i = static_cast<int>(div_up(d.N, MX_TILE)), kbs = static_cast<int>(div_up(d.K, MX_BK));
        mx_tiles_of(d.rows, tiles_i, kbs, p->pairs, true, &p->width, &p->parts);
        if (p->parts > 1) p->split_slot = take_split_slot(d.device, p->pairs, &p->counters);
        if (p->parts > 1 && p->split_slot < 0) {         // no counters: uncut
            uncut = true;
            mx_tiles_of(d.rows, tiles_i, kbs, p->pairs, false, &p->width, &p->parts);
        }
    }
    const MxMode mode = sums ? MX_SUMS : p->parts > 1 ? MX_CUT : MX_WHOLE_TILES;
    p->mode = mode;
    p->kernel = d.format == NK_NVF4 ? mx_kernel_nv(type, mode) : mx_kernel_mx(type, mode);
    if (cudaFuncSetAttribute(p->kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MX_SMEM) != cudaSuccess) {
        give_split_slot(d.device, p->split_slot, false, false);
        delete p;
        return NK_ERR_CUDA;
    }
    // the epilogue's registers come from the launch's own (see mx.cuh): a kernel built with fewer would wait for them without end
    cudaFuncAttributes built = {};
    if (mode == MX_SUMS && (cudaFuncGetAttributes(&built, p->kernel) != cudaSuccess ||
                            built.numRegs * mx_threads(mode, d.format == NK_NVF4) < MX_MORE_REGISTERS * 256 + MX_FEWER_REGISTERS * 128)) {
        give_split_slot(d.device, p->split_slot, false, false);
        delete p;
        return NK_ERR_CUDA;
    }
    snprintf(p->name, sizeof(p->name), "mx_%s%s_256x256x256_pair%s", d.format == NK_NVF4 ? "nvf4" : "mxf4", d.groups ? "_grouped" : "", uncut ? "_uncut" : "");
    *out = p;
    return NK_OK;
}

// partial sums of cut tiles: two FP32 slabs for each pair
size_t nk_mx_workspace_bytes(nk_mx_t p) {
    if (!p || p->split_slot < 0) return 0;
    return grouped_partial_bytes(p->pairs, p->slab_cols);
}

nk_status_t nk_mx_run(nk_mx_t p, const void* A, const void* A_scales, const void* B, const void* B_scales, const float* scale_a,
                      const float* scale_b, const float* bias, const int32_t* offsets, void* C, void* workspace, size_t workspace_bytes,
                      void* cuda_stream) {
    if (!p || (p->d.groups > 0) != (offsets != nullptr)) return NK_ERR_INVALID_ARG;
    const nk_mx_desc_t& d = p->d;
    if ((d.format != NK_NVF4 && (scale_a || scale_b)) || (d.epilogue == NK_EPI_NONE && bias)) return NK_ERR_INVALID_ARG;
    if (d.rows == 0) return NK_OK;
    if (!A || !A_scales || !B || !B_scales || !C) return NK_ERR_INVALID_ARG;
    auto misaligned4 = [](const void* x) { return (reinterpret_cast<uintptr_t>(x) & 3u) != 0; };
    if (misaligned16(A) || misaligned16(A_scales) || misaligned16(B) || misaligned16(B_scales) || misaligned16(C) || misaligned16(workspace) ||
        misaligned4(scale_a) || misaligned4(scale_b) || misaligned4(bias) || misaligned4(offsets))
        return NK_ERR_MISALIGNED;
    const size_t need = nk_mx_workspace_bytes(p);
    if (need && (!workspace || workspace_bytes < need)) return NK_ERR_WORKSPACE;
    DeviceGuard guard(d.device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    const int64_t groups = d.groups ? d.groups : 1;
    const bool nv = d.format == NK_NVF4;
    const void* now[4] = {A, A_scales, B, B_scales};
    if (memcmp(now, p->cached, sizeof(now)) != 0) {
        const int64_t pitch = mx_padded(d.K) / 2, tiles = mx_tiles(d.K, nv), box = nv ? 4 : 2;
        MxMaps& m = p->maps;
        bool ok = encode_packed(&m.a, B, pitch, d.N, groups, 128) && encode_scales(&m.sa, B_scales, tiles, groups * div_up(d.N, MX_TILE_ROWS), box) &&
                  encode_scales(&m.sb, A_scales, tiles, d.groups ? d.rows / MX_TILE_ROWS + groups : div_up(d.rows, MX_TILE_ROWS), box);
        for (int z = 0; ok && z < MX_BOXES; ++z) ok = encode_packed(&m.b[z], A, pitch, d.rows, 1, mx_box_rows(z));
        if (!ok) {
            memset(p->cached, 0, sizeof(p->cached));
            snprintf(p->cuda_err, sizeof(p->cuda_err), "cuTensorMapEncodeTiled failed");
            return NK_ERR_CUDA;
        }
        memcpy(p->cached, now, sizeof(now));     // (none is null: the maps are valid)
    }
    MxParams g = {};
    g.width = p->width;
    g.parts = p->parts;
    g.groups = static_cast<int>(groups);
    g.rows = static_cast<int>(d.rows);
    g.I = static_cast<int>(d.N);
    g.kb_total = static_cast<int>(div_up(d.K, MX_BK));
    g.steps = static_cast<int>(mx_padded(d.K) / 64);
    g.tiles_i = static_cast<int>(div_up(d.N, MX_TILE));
    g.scale_tiles = static_cast<int>(div_up(d.N, MX_TILE_ROWS));
    g.beta = d.beta;
    g.relu = d.epilogue == NK_EPI_BIAS_RELU;
    g.chunk = p->chunk;
    g.idesc = mx_idesc(nv);
    g.offsets = offsets;
    g.scale_a = scale_a;
    g.scale_b = scale_b;
    g.bias = bias;
    g.C = C;
    g.ldc = d.ldc;
    g.partial = need ? static_cast<float*>(workspace) : nullptr;
    g.slab_cols = p->slab_cols;
    g.counter = p->counters;
    g.status = p->status_dev;
    if (p->split_slot >= 0) base_runs(p, static_cast<cudaStream_t>(cuda_stream));       // (what has no counters leaves nothing behind)
    const cudaError_t e = launch_beside(p->kernel, 2 * p->pairs, mx_threads(p->mode, nv), MX_SMEM, static_cast<cudaStream_t>(cuda_stream), p->maps, g);
    return e == cudaSuccess ? NK_OK : p->cuda("mx launch", e);
}

nk_status_t nk_mx_check(nk_mx_t p) {
    if (!p) return NK_ERR_INVALID_ARG;
    const nk_status_t s = base_check(p);
    if (s == NK_ERR_TIMEOUT && p->counters) {
        DeviceGuard guard(p->device);
        cudaMemset(p->counters, 0, SPLIT_COUNTERS * sizeof(unsigned int));   // an abandoned tile may have left a count
    }
    return s;
}

const char* nk_mx_kernel_name(nk_mx_t p) { return p ? p->name : ""; }
const char* nk_mx_last_cuda_error(nk_mx_t p) { return p ? p->cuda_err : ""; }

nk_status_t nk_mx_destroy(nk_mx_t p) {
    if (p) give_split_slot(p->device, p->split_slot, p->in_flight, p->captured);
    delete p;
    return NK_OK;
}

}  // extern "C"
