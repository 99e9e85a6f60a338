// Host side of nk_route: descriptor validation and the launches.
#include "rows_host.cuh"
#include "route.cuh"

struct nk_route_s : nk::PlanBase {
    nk_route_desc_t d;            // strides filled in
    int blocks, per_block;        // of nk_route_run; one block: a single launch
};

using namespace nk;

namespace nk {

// experts a lane holds, rounded up to a power of two
static int route_width(int64_t experts) {
    int v = 1;
    while (32 * v < experts) v *= 2;
    return v;
}

template <bool ONE>
static void (*select_kernel(int v))(RouteParams) {
    switch (v) {
        case 1: return route_select_kernel<1, ONE>;
        case 2: return route_select_kernel<2, ONE>;
        case 4: return route_select_kernel<4, ONE>;
        case 8: return route_select_kernel<8, ONE>;
        case 16: return route_select_kernel<16, ONE>;
    }
    return route_select_kernel<32, ONE>;
}
static void (*backward_kernel(int v))(RouteParams, const float*, float*) {
    switch (v) {
        case 1: return route_backward_kernel<1>;
        case 2: return route_backward_kernel<2>;
        case 4: return route_backward_kernel<4>;
        case 8: return route_backward_kernel<8>;
        case 16: return route_backward_kernel<16>;
    }
    return route_backward_kernel<32>;
}

static RouteParams route_params(const nk_route_s* p) {
    RouteParams r = {};
    r.tokens = static_cast<int>(p->d.tokens);
    r.experts = static_cast<int>(p->d.experts);
    r.topk = static_cast<int>(p->d.topk);
    r.renormalise = p->d.renormalise;
    r.logits_type = p->d.logits_dtype == NK_F32 ? 0 : p->d.logits_dtype == NK_BF16 ? 1 : 2;
    r.ld_logits = p->d.ld_logits;
    r.per_block = p->per_block;
    return r;
}

static ExchangeParams exchange_params(const nk_route_s* p, const int32_t* slots, const float* gates) {
    ExchangeParams x = {};
    x.tokens = static_cast<int>(p->d.tokens);
    x.topk = static_cast<int>(p->d.topk);
    x.vecs = static_cast<int>(p->d.width / 8);
    // four pieces to a thread, but eight threads (128 bytes) to a row at least
    while (x.lanes_log2 < 8 && (1 << x.lanes_log2) < x.vecs && (x.lanes_log2 < 3 || (4 << x.lanes_log2) < x.vecs)) ++x.lanes_log2;
    x.ld_tokens = p->d.ld_tokens / 8;
    x.ld_slots = p->d.ld_slots / 8;
    x.slots = slots;
    x.gates = gates;
    return x;
}

static inline bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace nk

extern "C" {

nk_status_t nk_route_create(const nk_route_desc_t* desc, nk_route_t* out) {
    if (out) *out = nullptr;
    if (!desc || !out) return NK_ERR_INVALID_ARG;
    nk_route_desc_t d = *desc;
    if (d.tokens < 0 || d.experts <= 0 || d.topk <= 0 || d.topk > d.experts || d.width < 0) return NK_ERR_INVALID_ARG;
    if (d.logits_dtype < NK_F32 || d.logits_dtype > NK_E5M2 || d.dtype < NK_F32 || d.dtype > NK_E5M2) return NK_ERR_INVALID_ARG;
    if (d.renormalise != 0 && d.renormalise != 1) return NK_ERR_INVALID_ARG;
    if (d.logits_dtype != NK_F32 && !is_half_type(d.logits_dtype)) return NK_ERR_UNSUPPORTED;
    if (!is_half_type(d.dtype)) return NK_ERR_UNSUPPORTED;
    if (d.tokens > (1 << 24) || d.experts > NK_ROUTE_MAX_EXPERTS || d.topk > NK_ROUTE_MAX_TOPK || d.width > (1 << 24)) return NK_ERR_UNSUPPORTED;
    // (2^24 tokens of 32 choices: pairs stay below 2^31)
    if (d.width % 8 || d.ld_tokens % 8 || d.ld_slots % 8) return NK_ERR_MISALIGNED;
    if (d.ld_logits == 0) d.ld_logits = d.experts;
    if (d.ld_tokens == 0) d.ld_tokens = d.width;
    if (d.ld_slots == 0) d.ld_slots = d.width;
    if (d.ld_logits < d.experts || d.ld_tokens < d.width || d.ld_slots < d.width) return NK_ERR_INVALID_ARG;
    if (d.ld_logits >= (1ll << 36) || d.ld_tokens >= (1ll << 36) || d.ld_slots >= (1ll << 36)) return NK_ERR_UNSUPPORTED;
    int sms = 0;
    nk_status_t s = usable_device(d.device, &sms);
    if (s != NK_OK) return s;
    nk_route_s* p = new (std::nothrow) nk_route_s();
    if (!p) return NK_ERR_INVALID_ARG;
    p->d = d;
    if ((s = base_init(p, d.device, sms)) != NK_OK) { delete p; return s; }
    p->per_block = static_cast<int>(d.tokens <= ROUTE_ONE_BLOCK ? ROUTE_ONE_BLOCK : div_up(d.tokens, sms) < 32 ? 32 : div_up(d.tokens, sms));
    p->blocks = static_cast<int>(d.tokens <= ROUTE_ONE_BLOCK ? 1 : div_up(d.tokens, p->per_block));
    DeviceGuard guard(d.device);
    const int v = route_width(d.experts);
    if (cudaFuncSetAttribute(backward_kernel(v), cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * 32 * 32 * sizeof(float2)) != cudaSuccess) {
        delete p;
        return NK_ERR_CUDA;
    }
    const auto first = p->blocks == 1 ? select_kernel<true>(v) : select_kernel<false>(v);
    if (cudaFuncSetAttribute(first, cudaFuncAttributeMaxDynamicSharedMemorySize, route_smem(NK_ROUTE_MAX_EXPERTS)) != cudaSuccess ||
        cudaFuncSetAttribute(route_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, route_smem(NK_ROUTE_MAX_EXPERTS)) != cudaSuccess) {
        delete p;
        return NK_ERR_CUDA;
    }
    *out = p;
    return NK_OK;
}

size_t nk_route_workspace_bytes(nk_route_t p) {
    if (!p || p->blocks == 1) return 0;
    return static_cast<size_t>(p->blocks) * p->d.experts * sizeof(int);
}

nk_status_t nk_route_run(nk_route_t p, const void* logits, float* gates, int32_t* experts, int32_t* offsets, int32_t* slots,
                         void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!p || !offsets) return NK_ERR_INVALID_ARG;
    if (p->d.tokens > 0 && (!logits || !gates || !experts || !slots)) return NK_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(logits) & (p->d.logits_dtype == NK_F32 ? 3u : 1u)) || misaligned4(gates) || misaligned4(experts) ||
        misaligned4(offsets) || misaligned4(slots) || misaligned4(workspace))
        return NK_ERR_MISALIGNED;
    const size_t need = nk_route_workspace_bytes(p);
    if (need && (!workspace || workspace_bytes < need)) return NK_ERR_WORKSPACE;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    RouteParams r = route_params(p);
    r.logits = logits;
    r.gates = gates;
    r.chosen = experts;
    r.offsets = offsets;
    r.slots = slots;
    r.counts = static_cast<int*>(workspace);
    const int v = route_width(p->d.experts), smem = route_smem(r.experts);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = launch_beside(p->blocks == 1 ? select_kernel<true>(v) : select_kernel<false>(v), p->blocks, route_threads(v), smem, st, r);
    if (e != cudaSuccess) return p->cuda("route select launch", e);
    if (p->blocks > 1) {
        if ((e = launch_beside(route_place_kernel, p->blocks, ROUTE_THREADS, smem, st, r)) != cudaSuccess) return p->cuda("route place launch", e);
    }
    return NK_OK;
}

nk_status_t nk_route_backward(nk_route_t p, const void* logits, const int32_t* experts, const float* dgates, float* dlogits,
                              void* cuda_stream) {
    if (!p) return NK_ERR_INVALID_ARG;
    if (p->d.tokens == 0) return NK_OK;
    if (!logits || !experts || !dgates || !dlogits) return NK_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(logits) & (p->d.logits_dtype == NK_F32 ? 3u : 1u)) || misaligned4(experts) || misaligned4(dgates) ||
        misaligned4(dlogits))
        return NK_ERR_MISALIGNED;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    RouteParams r = route_params(p);
    r.logits = logits;
    r.chosen = const_cast<int32_t*>(experts);
    const cudaError_t e = launch_beside(backward_kernel(route_width(p->d.experts)), static_cast<unsigned>(div_up(r.tokens, 8)), 256, 8 * 32 * route_width(p->d.experts) * sizeof(float2),
                                        static_cast<cudaStream_t>(cuda_stream), r, dgates, dlogits);
    return e == cudaSuccess ? NK_OK : p->cuda("route backward launch", e);
}

nk_status_t nk_route_dispatch(nk_route_t p, const void* X, const int32_t* slots, void* Xs, void* cuda_stream) {
    if (!p || p->d.width == 0) return NK_ERR_INVALID_ARG;
    if (p->d.tokens == 0) return NK_OK;
    if (!X || !slots || !Xs) return NK_ERR_INVALID_ARG;
    if (misaligned16(X) || misaligned16(Xs) || misaligned4(slots)) return NK_ERR_MISALIGNED;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    const ExchangeParams x = exchange_params(p, slots, nullptr);
    const cudaError_t e = launch_beside(dispatch_kernel, static_cast<unsigned>(div_up(x.tokens, 256 >> x.lanes_log2)), 256, 0,
                                        static_cast<cudaStream_t>(cuda_stream), x, static_cast<const uint4*>(X), static_cast<uint4*>(Xs));
    return e == cudaSuccess ? NK_OK : p->cuda("dispatch launch", e);
}

nk_status_t nk_route_combine(nk_route_t p, const void* Ys, const int32_t* slots, const float* gates, void* Y, void* cuda_stream) {
    if (!p || p->d.width == 0) return NK_ERR_INVALID_ARG;
    if (p->d.tokens == 0) return NK_OK;
    if (!Ys || !slots || !Y) return NK_ERR_INVALID_ARG;
    if (misaligned16(Ys) || misaligned16(Y) || misaligned4(slots) || misaligned4(gates)) return NK_ERR_MISALIGNED;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    const ExchangeParams x = exchange_params(p, slots, gates);
    const cudaError_t e = launch_beside(p->d.dtype == NK_F16 ? combine_kernel<true> : combine_kernel<false>,
                                        static_cast<unsigned>(div_up(x.tokens, 256 >> x.lanes_log2)), 256, 0, static_cast<cudaStream_t>(cuda_stream), x,
                                        static_cast<const uint4*>(Ys), static_cast<uint4*>(Y));
    return e == cudaSuccess ? NK_OK : p->cuda("combine launch", e);
}

nk_status_t nk_route_combine_backward(nk_route_t p, const void* dY, const void* Ys, const int32_t* slots, const float* gates,
                                      void* dYs, float* dgates, void* cuda_stream) {
    if (!p || p->d.width == 0) return NK_ERR_INVALID_ARG;
    if (p->d.tokens == 0) return NK_OK;
    if (!dY || !Ys || !slots || !gates || !dYs || !dgates) return NK_ERR_INVALID_ARG;
    if (misaligned16(dY) || misaligned16(Ys) || misaligned16(dYs) || misaligned4(slots) || misaligned4(gates) || misaligned4(dgates))
        return NK_ERR_MISALIGNED;
    DeviceGuard guard(p->device);
    if (guard.err != cudaSuccess) return NK_ERR_DEVICE;
    const ExchangeParams x = exchange_params(p, slots, gates);
    const cudaError_t e = launch_beside(p->d.dtype == NK_F16 ? combine_backward_kernel<true> : combine_backward_kernel<false>, static_cast<unsigned>(div_up(p->d.tokens * p->d.topk, 8)), 256, 0, static_cast<cudaStream_t>(cuda_stream),
                                        x, static_cast<const uint4*>(dY), static_cast<const uint4*>(Ys), static_cast<uint4*>(dYs), dgates);
    return e == cudaSuccess ? NK_OK : p->cuda("combine backward launch", e);
}

nk_status_t nk_route_check(nk_route_t p) { return p ? base_check(p) : NK_ERR_INVALID_ARG; }
const char* nk_route_kernel_name(nk_route_t p) { return !p ? "" : p->blocks == 1 ? "route_one_block" : "route_select_place"; }
const char* nk_route_last_cuda_error(nk_route_t p) { return p ? p->cuda_err : ""; }

nk_status_t nk_route_destroy(nk_route_t p) {
    delete p;
    return NK_OK;
}

}  // extern "C"
