// The kernels of nk_mx for NVF4 operands.
#include "mx.cuh"

namespace nk {

MxFunction mx_kernel_nv(MxOut out, bool sums) {
    if (out == MX_OUT_F32) return sums ? mx_kernel<true, MX_OUT_F32, true> : mx_kernel<true, MX_OUT_F32, false>;
    if (out == MX_OUT_BF16) return sums ? mx_kernel<true, MX_OUT_BF16, true> : mx_kernel<true, MX_OUT_BF16, false>;
    return sums ? mx_kernel<true, MX_OUT_F16, true> : mx_kernel<true, MX_OUT_F16, false>;
}

}  // namespace nk
