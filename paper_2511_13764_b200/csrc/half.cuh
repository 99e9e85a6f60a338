// The two 16-bit floating-point element types as bits in registers.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace nk {

// A 16-bit element is BF16 (its bits are the upper half of the FP32 pattern) or, with `f16`
// set, IEEE binary16.  Both widen exactly to FP32; a result is rounded once (RNE) on the way out.
__device__ __forceinline__ float half_bits_to_f32(uint32_t h, int f16) {
    return f16 ? __half2float(__ushort_as_half(static_cast<unsigned short>(h))) : __uint_as_float(h << 16);
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi, int f16) {
    if (f16) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// eight elements of 16 bytes
template <bool F16>
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = half_bits_to_f32(w[i] & 0xFFFFu, F16);
        x[2 * i + 1] = half_bits_to_f32(w[i] >> 16, F16);
    }
}
template <bool F16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_half2(x[0], x[1], F16), pack_half2(x[2], x[3], F16), pack_half2(x[4], x[5], F16), pack_half2(x[6], x[7], F16));
}

}  // namespace nk
