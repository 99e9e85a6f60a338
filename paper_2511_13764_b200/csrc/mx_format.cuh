// The 4-bit formats: geometry of packed arrays (host and device) and conversions of scales and elements.
#pragma once
#ifdef __CUDACC__
#include "half.cuh"
#endif

namespace nk {

constexpr int MX_TILE_ROWS = 128, MX_TILE_BYTES = 512;          // a tile of scales: 128 rows x 4 blocks
__host__ __device__ constexpr int mx_block(int nv) { return nv ? 16 : 32; }
__host__ __device__ constexpr long long mx_padded(long long length) { return (length + 63) / 64 * 64; }
// tiles of scales along the contraction
__host__ __device__ constexpr long long mx_tiles(long long length, int nv) {
    return (mx_padded(length) + 4 * mx_block(nv) - 1) / (4 * mx_block(nv));
}
// first tile of scales of a group whose rows begin at row0: groups' tiles never meet, since ceil(n / 128) <= (row0 + n) / 128 - row0 / 128 + 1
__host__ __device__ constexpr int mx_group_tile(int row0, int g) { return row0 / MX_TILE_ROWS + g; }
// rows that the tile `at` tiles behind the first of a group of `rows` rows has; 0: it is none of the group's.  (`at` counts tiles of all groups, of
// which there are up to 2^24 + 1024: 128 times that may pass 2^31, so it is not formed before `at` is known to be the group's.)
__host__ __device__ constexpr int mx_tile_rows(int at, int rows) {
    if (at < 0 || at >= (rows + MX_TILE_ROWS - 1) / MX_TILE_ROWS) return 0;
    return rows - at * MX_TILE_ROWS < MX_TILE_ROWS ? rows - at * MX_TILE_ROWS : MX_TILE_ROWS;
}

#ifdef __CUDACC__
// E8M0 byte to its number (2^-127 is a subnormal)
__device__ __forceinline__ float e8m0_to_f32(uint32_t b) { return __uint_as_float(b == 255u ? 0x7FC00000u : max(b << 23, 0x00400000u)); }
__device__ __forceinline__ uint32_t f32_to_e4m3(float x) {       // round to nearest even, at most 448; NaN: 0x7F
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(x));
    return r & 0xFFu;
}
__device__ __forceinline__ float e4m3_to_f32(uint32_t b) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(b)));
    return half_bits_to_f32(r & 0xFFFFu, 1);
}
// two FP32 operations in one instruction
__device__ __forceinline__ unsigned long long pair_bits(float2 x) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x.x), "f"(x.y));
    return r;
}
__device__ __forceinline__ float2 pair_of(unsigned long long r) {
    float2 x;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x.x), "=f"(x.y) : "l"(r));
    return x;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return pair_of(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
// 1 / x to within one of its last places (x neither subnormal nor beyond 2^126)
__device__ __forceinline__ float rcp_approx(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// eight numbers to E2M1 (nearest even, at most 6 in size), the first in the lowest four bits
__device__ __forceinline__ uint32_t f32_to_e2m1x8(const float2 (&x)[4]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(x[0].x), "f"(x[0].y), "f"(x[1].x), "f"(x[1].y), "f"(x[2].x), "f"(x[2].y), "f"(x[3].x), "f"(x[3].y));
    return r;
}
__device__ __forceinline__ void e2m1x8_to_f32(uint32_t w, float (&x)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = half_bits_to_f32(h[i] & 0xFFFFu, 1);
        x[2 * i + 1] = half_bits_to_f32(h[i] >> 16, 1);
    }
}
#endif

}  // namespace nk
