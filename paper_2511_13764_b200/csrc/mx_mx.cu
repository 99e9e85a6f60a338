// The kernels of nk_mx for MXF4 operands.
#include "mx.cuh"

namespace nk {

MxFunction mx_kernel_mx(MxOut out, bool sums) {
    if (out == MX_OUT_F32) return sums ? mx_kernel<false, MX_OUT_F32, true> : mx_kernel<false, MX_OUT_F32, false>;
    if (out == MX_OUT_BF16) return sums ? mx_kernel<false, MX_OUT_BF16, true> : mx_kernel<false, MX_OUT_BF16, false>;
    return sums ? mx_kernel<false, MX_OUT_F16, true> : mx_kernel<false, MX_OUT_F16, false>;
}

}  // namespace nk
