// Host side of nk_lora: descriptor validation, TMA maps, the launches.
#include "rows_host.cuh"
#include "grouped_launch.cuh"
#include "lora.cuh"

struct nk_lora_s : nk::PlanBase {
    nk_lora_desc_t d;             // strides filled in
    bool few;                     // few rows to a request: FP32 contributions from lora_delta_kernel
    int pairs, rank_blocks, planes;
    int split_slot[2];            // of X . A and of the projection: the two overlap
    unsigned int* counters[2];
    size_t part_bytes[2], side_bytes;   // partial sums of the two; what lies before them:
    size_t h32_at, unscale_at, d_at;    // X . A in 16-bit numbers, then (FP16) in FP32 and the rows' factors, then the FP32 contributions
    nk::GroupedKernel projection, shrinking;
    nk::LoraMaps maps;            // of the projection
    nk::GroupedMaps shrink;       // of X . A
    const void *cached_x, *cached_w, *cached_a, *cached_b, *cached_ws, *cached_y;
    char name[64];
};

using namespace nk;

namespace nk {

static size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Which way the adapters' part goes.  Requests of up to LORA_ROWS rows are lora_delta_kernel's: their weights are all that
// counts, and its clusters read them at the speed of memory; more rows want the tensor cores: X . A_a as a grouped
// product, (X . A_a) . B_a as further k-blocks of the projection ("many").  A plan knows its rows and requests, not how the ones
// are spread over the others, so it leaves all of them to lora_delta_kernel ("few", one or two launches less), long ones too, where
// that costs little in the worst spread, one long request beside requests of one row.  Times in us, few against many, BF16, K = N = 4096
// unless said:
//   up to two rows to a request: 1000 of one row, rank 16: 237 / 300, rank 128: 888 / 954; 999 and one of 1001 rows: 335 / 389, 1175 / 1028
//   up to eight, rows x rank <= 48K: 64 requests of 8 rows, rank 16: 48 / 75, rank 64: 80 / 110; 63 and one of 400: 54 / 67, 84 / 74.
//     (Beyond: 256 of 8 rows, rank 128: 377 / 480, but 240 and 16 of 100 rows: 500 / 251; 1023 and one of 7000: 2189 / 919)
//   more, A as rows of K (16 bytes to a lane), few chunks of eight rows and a low rank: one of 240 rows, rank 16: 32 / 39, rank 32:
//     40 / 39, rank 64: 60 / 39; four of 12, rank 48: 29 / 33, rank 64: 34 / 33; N = K = 1024: 20 / 23, 22 / 23
static bool lora_few(int64_t rows, int64_t requests, int64_t rank, bool row) {
    const int64_t chunks = rows / LORA_ROWS + requests;
    return rows <= 2 * requests || (rows <= LORA_ROWS * requests && rows * rank <= 48 * 1024) ||
           (!row && rank <= 48 && chunks <= 32 && rank * chunks <= 640);
}

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
    if (d.ldx >= (1ll << 37) || d.ldw >= (1ll << 37) || d.ldy >= (1ll << 37)) return NK_ERR_UNSUPPORTED;
    if ((d.rows / 32 + 1) * div_up(d.N, 256) >= (1 << 24)) return NK_ERR_UNSUPPORTED;
    int sms = 0;
    nk_status_t s = usable_device(d.device, &sms);
    if (s != NK_OK) return s;
    nk_lora_s* p = new (std::nothrow) nk_lora_s();
    if (!p) return NK_ERR_INVALID_ARG;
    p->d = d;
    p->split_slot[0] = p->split_slot[1] = -1;
    if ((s = base_init(p, d.device, sms)) != NK_OK) { delete p; return s; }
    DeviceGuard guard(d.device);
    const bool row = d.layout == NK_ROW_MAJOR;
    p->few = lora_few(d.rows, d.requests, d.rank, row);
    p->projection = grouped_choose(p->few ? GRP_ROWS : GRP_LORA, row, grouped_out(d.out_dtype != NK_F32, d.in_dtype == NK_F16), d.K);
    // (BF16, a 16-bit Y and a K of one chunk: from one accumulator, in a kernel that leaves room for lora_delta_kernel's blocks; else
    // X . A_a is summed by the chunks of FP32 results)
    const bool f16 = d.in_dtype == NK_F16;
    p->shrinking = grouped_choose(GRP_ROWS, row, d.out_dtype == NK_F32 || f16 || d.K > GRP_CHUNK_16 * GRP_BK ? GRP_OUT_F32 : GRP_OUT_H, d.K);
    cudaError_t e = grouped_prepare(p->projection);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(d.in_dtype == NK_F16 ? lora_delta_kernel<true> : lora_delta_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, lora_smem(LORA_MAX_RANK, LORA_MAX_REQUESTS, false));
    if (e == cudaSuccess && !p->few) e = grouped_prepare(p->shrinking);
    if (e != cudaSuccess || !encode_tiled()) { delete p; return NK_ERR_CUDA; }
    p->pairs = sms / 2;
    // two 16-bit numbers hold X . A_a to 2^-16 (BF16) or 2^-22 (FP16) of it: enough for a 16-bit Y, not for an FP32 one, which gets
    // three (2^-24 and better)
    p->planes = d.out_dtype == NK_F32 ? 3 : 2;
    p->rank_blocks = static_cast<int>(div_up(d.rank, p->planes == 3 ? 16 : 32));
    const int64_t short_rows = p->few || d.rows < LORA_ROWS * d.requests ? d.rows : LORA_ROWS * d.requests;
    p->h32_at = p->few ? 0 : align256(static_cast<size_t>(d.rows) * p->rank_blocks * 128);
    p->unscale_at = p->h32_at + (p->few || !f16 ? 0 : align256(static_cast<size_t>(d.rows) * d.rank * sizeof(float)));
    p->d_at = p->unscale_at + (p->few || !f16 ? 0 : align256(static_cast<size_t>(d.rows) * sizeof(float)));
    p->side_bytes = p->d_at + align256(static_cast<size_t>(short_rows) * d.N * sizeof(float));
    for (int i = p->few ? 1 : 0; i < 2; ++i) {
        p->split_slot[i] = take_split_slot(d.device, p->pairs, &p->counters[i]);
        p->part_bytes[i] = p->split_slot[i] < 0 ? 0 : grouped_partial_bytes(p->pairs, grouped_slab_cols(d.rows));
    }
    snprintf(p->name, sizeof(p->name), "lora_%s_%s%s", p->few ? "few" : "many", row ? "rows" : "rows_t",
             p->split_slot[1] < 0 || (!p->few && p->split_slot[0] < 0) ? "_uncut" : "");
    *out = p;
    return NK_OK;
}

size_t nk_lora_workspace_bytes(nk_lora_t p) {
    if (!p) return 0;
    return p->side_bytes + p->part_bytes[0] + p->part_bytes[1];
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
    const bool f16 = d.in_dtype == NK_F16, row = d.layout == NK_ROW_MAJOR;
    if (p->cached_x != X || p->cached_w != W || p->cached_a != A || p->cached_b != B || p->cached_ws != workspace || p->cached_y != Y) {
        p->cached_x = nullptr;
        LoraMaps& m = p->maps;
        GroupedMaps& s = p->shrink;
        bool ok = encode_rows(m.b, X, f16, d.K, d.rows, d.ldx) && encode_out(&m.out, Y, d.out_dtype, d.N, d.rows, 1, d.ldy, 0) &&
                  (!row ? encode_map(&m.a, W, f16, d.K, d.N, 1, d.ldw, 0, 128)
                   : d.N % 64 == 0 ? encode_slabs(&m.a, W, f16, d.N, d.K, 1, d.ldw, 0) : encode_map(&m.a, W, f16, d.N, d.K, 1, d.ldw, 0, 64));
        if (!p->few) {
            const int64_t r = d.rank, h = p->rank_blocks * 64;
            ok = ok && encode_rows(m.h, workspace, f16, h, d.rows, h) &&
                 (row ? encode_map(&s.a, A, f16, r, d.K, d.adapters, r, r * d.K, 64) : encode_map(&s.a, A, f16, d.K, r, d.adapters, d.K, r * d.K, 128)) &&
                 (row ? encode_map(&m.c, B, f16, d.N, r, d.adapters, d.N, r * d.N, 32) : encode_map(&m.c, B, f16, r, d.N, d.adapters, r, r * d.N, 128));
            if (f16) ok = ok && encode_out(&s.out, static_cast<char*>(workspace) + p->h32_at, NK_F32, r, d.rows, 1, r, 0);
            memcpy(s.b, m.b, sizeof(s.b));
        }
        if (!ok) {
            snprintf(p->cuda_err, sizeof(p->cuda_err), "cuTensorMapEncodeTiled failed");
            return NK_ERR_CUDA;
        }
        p->cached_x = X;
        p->cached_w = W;
        p->cached_a = A;
        p->cached_b = B;
        p->cached_ws = workspace;
        p->cached_y = Y;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    base_runs(p, st);
    char* ws = static_cast<char*>(workspace);
    float* partial[2];
    for (int i = 0; i < 2; ++i) partial[i] = p->part_bytes[i] ? reinterpret_cast<float*>(ws + p->side_bytes + (i ? p->part_bytes[0] : 0)) : nullptr;
    GroupedParams g = {};
    g.rows = static_cast<int>(d.rows);
    g.kb_total = static_cast<int>(div_up(d.K, GRP_BK));
    g.f16 = f16;
    g.idesc = grouped_idesc(row, false, f16);
    g.slab_cols = grouped_slab_cols(d.rows);
    g.status = p->status_dev;
    g.rank = static_cast<int>(d.rank);
    g.rank_blocks = p->rank_blocks;
    g.planes = p->planes;
    LoraParams l = {};
    l.rows = g.rows;
    l.N = static_cast<int>(d.N);
    l.K = static_cast<int>(d.K);
    l.rank = g.rank;
    l.adapters = static_cast<int>(d.adapters);
    l.requests = static_cast<int>(d.requests);
    l.transposed = !row;
    l.few = p->few;
    l.ldx = d.ldx;
    l.X = X;
    l.A = A;
    l.B = B;
    l.scale = scale;
    l.offsets = offsets;
    l.adapter = adapter;
    l.D = reinterpret_cast<float*>(ws + p->d_at);
    l.status = p->status_dev;
    // Clusters: no more than there can be chunks of rows.  Up to two rounds of them go to as many clusters as fit with one block
    // to an SM (two in each of eight GPCs), beside which the projection's or X . A's blocks find room; more of them are bound by
    // memory and get four blocks to an SM.
    const int64_t chunks = p->few ? d.rows / LORA_ROWS + (d.rows < d.requests ? d.rows : d.requests) : d.requests;
    const int64_t single = p->sm_count / LORA_CLUSTER / 8 * 8, most = chunks <= 2 * single ? single : 4 * p->sm_count / LORA_CLUSTER;
    cudaError_t e = launch_beside(f16 ? lora_delta_kernel<true> : lora_delta_kernel<false>, static_cast<unsigned>((chunks < most ? chunks : most) * LORA_CLUSTER), LORA_THREADS,
                                  lora_smem(l.rank, l.requests, l.transposed), st, l);
    if (e != cudaSuccess) return p->cuda("lora delta launch", e);
    // The two products start beside it.  Neither touches what it writes before they wait for it, and what it waited for
    // before its start has ended before theirs.
    g.late = 1;
    g.add = l.D;
    if (!p->few) {
        // X . A_a: the requests are the groups, their adapters the weights
        GroupedParams h = g;
        h.add = nullptr;
        h.groups = l.requests;
        h.offsets = offsets;
        h.index = adapter;
        h.index_max = l.adapters;
        h.min_rows = LORA_ROWS;
        h.scale = scale;
        h.I = g.rank;
        h.tiles_i = 1;
        h.chunk = p->shrinking.chunk();
        LoraSplitParams split = {};
        if (f16) {
            h.C = ws + p->h32_at;
            h.ldc = d.rank;
            split = {h.rows, h.I, g.rank_blocks, g.planes, static_cast<const float*>(h.C), reinterpret_cast<uint16_t*>(ws), reinterpret_cast<float*>(ws + p->unscale_at)};
            g.unscale = split.unscale;
        } else {
            h.h16 = reinterpret_cast<uint16_t*>(ws);
        }
        h.partial = partial[0];
        h.counter = p->counters[0];
        e = grouped_launch(p->shrinking, p->pairs, st, p->shrink, h);
        if (e != cudaSuccess) return p->cuda("lora shrink launch", e);
        // (few blocks: the projection's start when all of them have, which they do where X . A_a is done first)
        const int64_t blocks = div_up(d.rows, LORA_SPLIT_ROWS), most_blocks = 2 * p->sm_count;
        if (f16 && (e = launch_beside(lora_split_kernel, static_cast<unsigned>(blocks < most_blocks ? blocks : most_blocks), 32 * LORA_SPLIT_ROWS, 0, st, split)) != cudaSuccess)
            return p->cuda("lora split launch", e);
        g.requests = h.groups;
        g.request_offsets = offsets;
        g.index = adapter;
        g.index_max = h.index_max;
        g.min_rows = LORA_ROWS;
    }
    g.groups = 1;
    g.I = static_cast<int>(d.N);
    g.tiles_i = static_cast<int>(div_up(d.N, GRP_TILE));
    g.a_slabs = d.N % 64 == 0;
    g.chunk = p->projection.chunk();
    g.C = Y;
    g.ldc = d.ldy;
    g.partial = partial[1];
    g.counter = p->counters[1];
    e = grouped_launch(p->projection, p->pairs, st, p->maps, g);
    return e == cudaSuccess ? NK_OK : p->cuda("lora projection launch", e);
}

nk_status_t nk_lora_check(nk_lora_t p) {
    if (!p) return NK_ERR_INVALID_ARG;
    const nk_status_t s = base_check(p);
    if (s == NK_ERR_TIMEOUT) {
        DeviceGuard guard(p->device);
        for (unsigned int* c : p->counters)
            if (c) cudaMemset(c, 0, SPLIT_COUNTERS * sizeof(unsigned int));   // an abandoned tile may have left a count
    }
    return s;
}

const char* nk_lora_kernel_name(nk_lora_t p) { return p ? p->name : ""; }
const char* nk_lora_last_cuda_error(nk_lora_t p) { return p ? p->cuda_err : ""; }

nk_status_t nk_lora_destroy(nk_lora_t p) {
    if (p) {
        for (int slot : p->split_slot) give_split_slot(p->device, slot, p->in_flight, p->captured);
    }
    delete p;
    return NK_OK;
}

}  // extern "C"
