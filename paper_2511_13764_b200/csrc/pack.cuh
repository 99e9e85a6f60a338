// Packing into 4-bit elements with block scales, the scale of a tensor, and reading back.
//   MXF4   scale 2^(floor(log2 m) - 2): bits of m's exponent; x / scale is exact
//   NVF4   scale s = RN_e4m3(m / (6 t)), element RN_e2m1(x / (s t))
// The element's decision has to be that of exact arithmetic.  With t of 8 significant bits d = s t has 12 and is exact, a border b of
// the elements (0.25 .. 5) times d has 15, so for x of a 16-bit type x / d is either b or at least 2^-14 away from it.  x times the
// FP32 reciprocal of d is within 2^-20 of the quotient; rounded to a multiple of 2^-16 (one FMA onto 192 and a subtraction) it is b
// exactly where the quotient is, and on the quotient's side of b elsewhere.  So there is no division for an element.  FP32 x take one: a
// correctly rounded x / d is b only where the quotient is (24 bits against 15: the next quotient is more than half a step away).
//
// A block of threads has a tile of scales' 128 rows, so that the scales of 256 of the contraction leave as 2 KB in one piece; a warp reads
// 256 consecutive elements of a row (8 to a lane), and a block's maximum is one or two shuffles.  Along the columns a tile of 128 x
// 128 goes through shared memory, where a thread has a word of adjacent features.  Bound by memory.
#pragma once
#include "mx_format.cuh"
#include "ptx.cuh"

namespace nk {

constexpr int PACK_THREADS = 256, PACK_CHUNK = 256;      // along rows: threads, elements of the contraction to a block
constexpr int PACK_TURN = 128;                           // along columns: a tile's side
constexpr int PACK_MAX_GROUPS = 1024;

struct PackParams {
    int nv;                    // 1 NVF4, 0 MXF4
    int outer;                 // rows of the packed matrix (of one of the batch)
    int groups;                // 0: none
    int length;                // of the contraction
    int row_tiles, tiles;      // tiles of scales: along the rows of a matrix (groups: of all), along the contraction
    long long ldx, stride_x;   // in elements
    const void* x;
    const float* scale;        // [batch]; null: 1
    const int* offsets;
    uint8_t* data;             // [batch][outer][padded / 2]
    uint8_t* scales;
    void* values;
    unsigned int* status;
};

// The element types by number: 0 FP32, 1 BF16, 2 FP16.  Magnitudes are compared as the bits of an element: those of infinities and
// NaN are the largest.
template <int T> __device__ __forceinline__ constexpr uint32_t pack_not_finite() { return T == 0 ? 0x7F800000u : T == 1 ? 0x7F80u : 0x7C00u; }
template <int T> __device__ __forceinline__ float pack_widen(uint32_t bits) { return T == 0 ? __uint_as_float(bits) : half_bits_to_f32(bits, T == 2); }

struct PackScale {
    float t, six_t;            // NVF4
    bool bad;
};
__device__ __forceinline__ PackScale pack_scale(const PackParams& p, int item) {
    PackScale s = {1.0f, 6.0f, false};
    if (p.nv && p.scale) {
        s.t = p.scale[item];
        s.six_t = 6.0f * s.t;
        s.bad = !(s.t > 0.0f && s.t < INFINITY);
    }
    return s;
}

// m / (6 t) to E4M3.  The FP32 quotient is off by 2 of its last places (6 t is rounded, too), so one that close to the border of two
// scales is decided by the border itself: border x 6 t is exact in 64 bits (5 + 2 + 24).
__device__ __forceinline__ uint32_t pack_e4m3(float m, const PackScale& s) {
    float q = __fdiv_rn(m, s.six_t);
    const uint32_t bits = __float_as_uint(q) + 4u;
    float border = 0.0f;
    if (q >= 0x1p-6f) {
        if (((bits - 0x80000u) & 0xFFFFFu) <= 8u) border = __uint_as_float(bits & ~0x7FFFFu);     // halfway between steps of 1/8
    } else {
        const float n = rintf(q * 1024.0f);                                // subnormals: odd multiples of 2^-10
        if ((static_cast<int>(n) & 1) && fabsf(q * 1024.0f - n) <= n * 0x1p-21f) border = n * 0x1p-10f;
    }
    if (border > 0.0f) {
        const double at = static_cast<double>(border) * 6.0 * static_cast<double>(s.t), x = m;
        q = x > at ? __uint_as_float(__float_as_uint(border) + 1u) : x < at ? __uint_as_float(__float_as_uint(border) - 1u) : border;
    }
    return f32_to_e4m3(q);
}

// A block's scale from the bits of its largest magnitude: the byte, and what the elements are multiplied by (FP32, NVF4: divided by).
template <int T, bool NV>
__device__ __forceinline__ uint32_t pack_block(uint32_t most, const PackScale& s, float& factor) {
    factor = 0.0f;
    if (most >= pack_not_finite<T>() || s.bad) return NV ? 0x7Fu : 0xFFu;
    const float m = pack_widen<T>(most);
    if (!NV) {
        const uint32_t e = __float_as_uint(m) >> 23, byte = e > 2u ? e - 2u : 0u;
        factor = __uint_as_float((254u - byte) << 23);
        return byte;
    }
    const uint32_t byte = pack_e4m3(m, s);
    const float d = e4m3_to_f32(byte) * s.t;
    factor = T == 0 ? d : d > 0.0f ? __frcp_rn(d) : 0.0f;
    return byte;
}
template <int T, bool NV>
__device__ __forceinline__ float pack_quotient(float x, float factor) {
    if (!NV) return x * factor;
    if (T == 0) return factor > 0.0f ? __fdiv_rn(x, factor) : 0.0f;
    return fmaf(x, factor, 192.0f) - 192.0f;
}

// the rows of a tile of scales
struct PackRows {
    int first, count;          // rows of the arrays
};
// Which rows tile `tile` has; `count` 0: none.  With groups the block looks the tile's group up in the offsets.  (Every thread calls this.)
__device__ __forceinline__ PackRows pack_rows(const PackParams& p, int tile, int* s_off, int* s_found) {
    PackRows r;
    if (!p.groups) {
        r.first = tile * MX_TILE_ROWS;
        r.count = min(MX_TILE_ROWS, p.outer - r.first);
        return r;
    }
    bool bad = false;
    for (int g = threadIdx.x; g <= p.groups; g += PACK_THREADS) {
        const int o = p.offsets[g];
        s_off[g] = o;
        bad |= o < 0 || o > p.outer;
    }
    if (threadIdx.x == 0) s_found[0] = 0, s_found[1] = 0;
    __syncthreads();
    for (int g = threadIdx.x; g < p.groups; g += PACK_THREADS) bad |= s_off[g + 1] < s_off[g];
    if (__syncthreads_or(bad)) {
        // clamped to the running maximum
        if (threadIdx.x == 0) {
            if (p.status) atomicCAS(p.status, 0u, 0x10000u);
            int top = 0;
            for (int g = 0; g <= p.groups; ++g) s_off[g] = top = max(top, min(s_off[g], p.outer));
        }
        __syncthreads();
    }
    for (int g = threadIdx.x; g < p.groups; g += PACK_THREADS) {
        const int lo = s_off[g], hi = s_off[g + 1], from = mx_group_tile(lo, g), at = tile - from;
        if (at >= 0 && at * MX_TILE_ROWS < hi - lo) {
            s_found[0] = lo + at * MX_TILE_ROWS;
            s_found[1] = min(MX_TILE_ROWS, hi - lo - at * MX_TILE_ROWS);
        }
    }
    __syncthreads();
    r.first = s_found[0];
    r.count = s_found[1];
    return r;
}

// eight elements at x as bits; their largest magnitude
template <int T>
__device__ __forceinline__ void pack_load(const void* x, size_t at, uint32_t (&w)[T == 0 ? 8 : 4]) {
    if (T == 0) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(x) + at);
        const uint4 a = __ldcs(p), b = __ldcs(p + 1);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[T == 0 ? 4 : 0] = b.x, w[T == 0 ? 5 : 0] = b.y, w[T == 0 ? 6 : 0] = b.z, w[T == 0 ? 7 : 0] = b.w;
    } else {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + at));
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    }
}
template <int T, int N>
__device__ __forceinline__ uint32_t pack_most(const uint32_t (&w)[N]) {
    if (T == 0) {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < N; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
    return max(m & 0xFFFFu, m >> 16);
}
template <int T>
__device__ __forceinline__ float pack_element(const uint32_t (&w)[T == 0 ? 8 : 4], int i) {
    return T == 0 ? __uint_as_float(w[T == 0 ? i : 0]) : pack_widen<T>(i & 1 ? w[T == 0 ? 0 : i >> 1] >> 16 : w[T == 0 ? 0 : i >> 1] & 0xFFFFu);
}

// Along the rows: blockIdx.x a tile's rows, y 256 of the contraction, z the matrix.
template <int T, bool NV>
__global__ void __launch_bounds__(PACK_THREADS) pack_rows_kernel(const PackParams p) {
    constexpr int LANES = NV ? 2 : 4;                    // of a block
    constexpr int TILES = PACK_CHUNK / (4 * mx_block(NV));
    __shared__ int s_off[PACK_MAX_GROUPS + 1], s_found[2];
    __shared__ __align__(16) uint8_t s_scale[TILES * MX_TILE_BYTES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, item = blockIdx.z;
    launch_wait();
    launch_next();
    const PackRows rows = pack_rows(p, blockIdx.x, s_off, s_found);
    if (rows.count <= 0) return;
    const PackScale s = pack_scale(p, item);
    for (int i = threadIdx.x; i < TILES * MX_TILE_BYTES / 4; i += PACK_THREADS) reinterpret_cast<uint32_t*>(s_scale)[i] = 0u;
    __syncthreads();
    const int k = blockIdx.y * PACK_CHUNK + lane * 8, pitch = static_cast<int>(mx_padded(p.length) / 2);
    const bool there = k < p.length, kept = k < 2 * pitch;
    const size_t x0 = item * static_cast<size_t>(p.stride_x) + rows.first * static_cast<size_t>(p.ldx) + k;
    uint8_t* data = p.data + (static_cast<size_t>(item) * p.outer + rows.first) * pitch + k / 2;
    const int c = lane / LANES;                          // the block's place in the chunk
    constexpr int AHEAD = 4;                             // rows on the way
    for (int r0 = warp; r0 < rows.count; r0 += AHEAD * 8) {
        uint32_t w[AHEAD][T == 0 ? 8 : 4];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
#pragma unroll
            for (int i = 0; i < (T == 0 ? 8 : 4); ++i) w[n][i] = 0u;
            if (there && r0 + 8 * n < rows.count) pack_load<T>(p.x, x0 + (r0 + 8 * n) * static_cast<size_t>(p.ldx), w[n]);
        }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const int r = r0 + 8 * n;
            if (r >= rows.count) break;
            uint32_t most = pack_most<T>(w[n]);
            most = max(most, __shfl_xor_sync(~0u, most, 1));
            if (!NV) most = max(most, __shfl_xor_sync(~0u, most, 2));
            float factor, y[8];
            const uint32_t byte = pack_block<T, NV>(most, s, factor);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = pack_quotient<T, NV>(pack_element<T>(w[n], i), factor);
            // (a block that is not finite has factor 0 and may have products that are NaN)
            const uint32_t e = most >= pack_not_finite<T>() ? 0u : f32_to_e2m1x8(y);
            if (kept) *reinterpret_cast<uint32_t*>(data + static_cast<size_t>(r) * pitch) = e;
            if (there && lane % LANES == 0) s_scale[c / 4 * MX_TILE_BYTES + (r & 31) * 16 + (r >> 5) * 4 + (c & 3)] = static_cast<uint8_t>(byte);
        }
    }
    __syncthreads();
    const int first = blockIdx.y * TILES, n = min(TILES, p.tiles - first) * (MX_TILE_BYTES / 16);
    uint4* out = reinterpret_cast<uint4*>(p.scales + ((static_cast<size_t>(item) * p.row_tiles + blockIdx.x) * p.tiles + first) * MX_TILE_BYTES);
    for (int i = threadIdx.x; i < n; i += PACK_THREADS) out[i] = reinterpret_cast<const uint4*>(s_scale)[i];
}

// Along the columns: blockIdx.x 128 features (a tile's rows), y 128 rows of X, z the matrix.
template <int T, bool NV>
__global__ void __launch_bounds__(PACK_THREADS) pack_columns_kernel(const PackParams p) {
    constexpr int BLOCK = mx_block(NV), BLOCKS = PACK_TURN / BLOCK;           // of the contraction
    constexpr int WORDS = T == 0 ? PACK_TURN : PACK_TURN / 2;                 // 32-bit words of a row of the tile
    constexpr int EACH = T == 0 ? 1 : 2;                                      // features of a word
    constexpr int TILES = PACK_TURN / (4 * BLOCK);
    constexpr int OUT = PACK_TURN / 2 + 8;                                    // bytes of a feature's packed row, and 8 against bank conflicts
    extern __shared__ __align__(16) uint8_t pack_sm[];
    uint32_t* tile = reinterpret_cast<uint32_t*>(pack_sm);                    // [128][WORDS]
    uint8_t* out = pack_sm + PACK_TURN * WORDS * 4;                           // [128][OUT]
    uint8_t* s_scale = out + PACK_TURN * OUT;                                 // [TILES][512]
    const int item = blockIdx.z, f0 = blockIdx.x * PACK_TURN, t0 = blockIdx.y * PACK_TURN;
    const int features = min(PACK_TURN, p.outer - f0);
    launch_wait();
    launch_next();
    const PackScale s = pack_scale(p, item);
    // pieces of 16 bytes: a row of the tile has WORDS / 4
    constexpr int PIECES = WORDS / 4, PER = PACK_TURN * PIECES / PACK_THREADS;
    const uint8_t* x = static_cast<const uint8_t*>(p.x) + (item * static_cast<size_t>(p.stride_x) + f0) * (T == 0 ? 4 : 2);
    const int piece = threadIdx.x % PIECES, row = threadIdx.x / PIECES;
    const bool there = piece * (T == 0 ? 4 : 8) < features;                   // (the number of features is a multiple of 8)
#pragma unroll 8
    for (int n = 0; n < PER; ++n) {
        const int t = row + n * (PACK_THREADS / PIECES);
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (there && t0 + t < p.length)
            v = __ldcs(reinterpret_cast<const uint4*>(x + static_cast<size_t>(t0 + t) * p.ldx * (T == 0 ? 4 : 2) + piece * 16));
        reinterpret_cast<uint4*>(tile)[t * PIECES + piece] = v;
    }
    __syncthreads();
    for (int task = threadIdx.x; task < WORDS * BLOCKS; task += PACK_THREADS) {
        const int w = task % WORDS, b = task / WORDS;
        const uint32_t* at = tile + b * BLOCK * WORDS + w;
        uint32_t m = 0u;
        uint32_t v[BLOCK];
#pragma unroll
        for (int i = 0; i < BLOCK; ++i) {
            v[i] = at[i * WORDS];
            m = T == 0 ? max(m, v[i] & 0x7FFFFFFFu) : __vmaxu2(m, v[i] & 0x7FFF7FFFu);
        }
#pragma unroll
        for (int h = 0; h < EACH; ++h) {
            const uint32_t most = T == 0 ? m : h ? m >> 16 : m & 0xFFFFu;
            const int f = w * EACH + h;
            float factor;
            uint32_t byte = pack_block<T, NV>(most, s, factor);
#pragma unroll
            for (int q = 0; q < BLOCK / 8; ++q) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t bits = v[q * 8 + i];
                    y[i] = pack_quotient<T, NV>(pack_widen<T>(T == 0 ? bits : h ? bits >> 16 : bits & 0xFFFFu), factor);
                }
                const uint32_t e = most >= pack_not_finite<T>() ? 0u : f32_to_e2m1x8(y);
                *reinterpret_cast<uint32_t*>(out + f * OUT + b * (BLOCK / 2) + q * 4) = e;
            }
            if (f >= features || t0 + b * BLOCK >= p.length) byte = 0u;
            s_scale[b / 4 * MX_TILE_BYTES + (f & 31) * 16 + (f >> 5) * 4 + (b & 3)] = static_cast<uint8_t>(byte);
        }
    }
    __syncthreads();
    const size_t pitch = mx_padded(p.length) / 2;
    const int bytes = static_cast<int>(min(static_cast<long long>(PACK_TURN / 2), static_cast<long long>(pitch) - t0 / 2));
    uint8_t* data = p.data + (static_cast<size_t>(item) * p.outer + f0) * pitch + t0 / 2;
    for (int i = threadIdx.x; i < features * 8; i += PACK_THREADS) {
        const int f = i >> 3, o = (i & 7) * 8;
        if (o < bytes) *reinterpret_cast<uint2*>(data + f * pitch + o) = *reinterpret_cast<const uint2*>(out + f * OUT + o);
    }
    const int first = blockIdx.y * TILES, n = min(TILES, p.tiles - first) * (MX_TILE_BYTES / 16);
    uint4* sc = reinterpret_cast<uint4*>(p.scales + ((static_cast<size_t>(item) * p.row_tiles + blockIdx.x) * p.tiles + first) * MX_TILE_BYTES);
    for (int i = threadIdx.x; i < n; i += PACK_THREADS) sc[i] = reinterpret_cast<const uint4*>(s_scale)[i];
}
__host__ __device__ constexpr int pack_columns_smem(int type) { return PACK_TURN * PACK_TURN * (type == 0 ? 4 : 2) + PACK_TURN * (PACK_TURN / 2 + 8) + 2 * MX_TILE_BYTES; }

// Reading back: blocks as in pack_rows_kernel.  A lane has eight elements.
template <int T, bool NV>
__global__ void __launch_bounds__(PACK_THREADS) pack_values_kernel(const PackParams p) {
    constexpr int LANES = NV ? 2 : 4, TILES = PACK_CHUNK / (4 * mx_block(NV));
    __shared__ int s_off[PACK_MAX_GROUPS + 1], s_found[2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, item = blockIdx.z;
    launch_wait();
    launch_next();
    const PackRows rows = pack_rows(p, blockIdx.x, s_off, s_found);
    if (rows.count <= 0) return;
    const float t = NV && p.scale ? p.scale[item] : 1.0f;
    const int k = blockIdx.y * PACK_CHUNK + lane * 8, pitch = static_cast<int>(mx_padded(p.length) / 2), c = lane / LANES;
    if (k >= p.length) return;
    const uint8_t* data = p.data + (static_cast<size_t>(item) * p.outer + rows.first) * pitch + k / 2;
    const uint8_t* scales = p.scales + ((static_cast<size_t>(item) * p.row_tiles + blockIdx.x) * p.tiles + blockIdx.y * TILES + c / 4) * MX_TILE_BYTES + (c & 3);
    const size_t y0 = (static_cast<size_t>(item) * p.outer + rows.first) * p.length + k;
    const bool whole = p.length % 8 == 0;                // rows of Y are pieces of eight, 16-byte aligned
#pragma unroll 4
    for (int r = warp; r < rows.count; r += 8) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(data + static_cast<size_t>(r) * pitch);
        const uint32_t b = scales[(r & 31) * 16 + (r >> 5) * 4];
        const float s = NV ? e4m3_to_f32(b) : e8m0_to_f32(b);
        float x[8];
        e2m1x8_to_f32(w, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = NV ? x[i] * s * t : x[i] * s;
        const size_t y = y0 + static_cast<size_t>(r) * p.length;
        if (T == 0) {
            float* out = static_cast<float*>(p.values) + y;
            if (whole) {
                __stcs(reinterpret_cast<float4*>(out), make_float4(x[0], x[1], x[2], x[3]));
                __stcs(reinterpret_cast<float4*>(out) + 1, make_float4(x[4], x[5], x[6], x[7]));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k + i < p.length) out[i] = x[i];
            }
        } else {
            uint16_t* out = static_cast<uint16_t*>(p.values) + y;
            if (whole) {
                __stcs(reinterpret_cast<uint4*>(out), pack8<T == 2>(x));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k + i < p.length) out[i] = static_cast<uint16_t>(pack_half2(x[i], 0.0f, T == 2) & 0xFFFFu);
            }
        }
    }
}

// A tensor's scale from its largest magnitude: divided by 6 x 448, rounded up to 8 significant bits (both steps upwards: the same as
// one).
__device__ __forceinline__ float tensor_scale_of(float m) {
    if (!(m < INFINITY)) return __int_as_float(0x7FC00000);
    const float t = __uint_as_float((__float_as_uint(__fdiv_ru(m, 2688.0f)) + 0xFFFFu) & 0xFFFF0000u);
    return fmaxf(t, 0x1p-60f);
}
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* line) {
    m = __reduce_max_sync(~0u, m);
    if ((threadIdx.x & 31) == 0) line[threadIdx.x >> 5] = m;
    __syncthreads();
    m = threadIdx.x < blockDim.x / 32 ? line[threadIdx.x] : 0u;
    if (threadIdx.x < 32) m = __reduce_max_sync(~0u, m);
    return m;                                            // (of the first warp)
}

// blockIdx.x of gridDim.x takes every gridDim.x-th piece of 8 elements x 256 threads x 4; y the matrix.  ONE block writes the scale.
template <int T>
__global__ void __launch_bounds__(PACK_THREADS) tensor_max_kernel(const PackParams p, int rows, int width, uint32_t* partial, float* scale) {
    __shared__ uint32_t line[32];
    const size_t x0 = blockIdx.y * static_cast<size_t>(p.stride_x);
    const int per_row = width / 8;
    const long long pieces = static_cast<long long>(rows) * per_row, step = static_cast<long long>(gridDim.x) * PACK_THREADS;
    launch_wait();
    launch_next();
    uint32_t m = 0u;
    const bool dense = p.ldx == width;
    for (long long i = blockIdx.x * static_cast<long long>(PACK_THREADS) + threadIdx.x; i < pieces; i += 4 * step) {
        uint32_t w[4][T == 0 ? 8 : 4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const long long j = i + n * step;
#pragma unroll
            for (int q = 0; q < (T == 0 ? 8 : 4); ++q) w[n][q] = 0u;
            if (j < pieces) {
                const long long r = dense ? 0 : j / per_row;
                pack_load<T>(p.x, x0 + (dense ? j * 8 : r * p.ldx + (j - r * per_row) * 8), w[n]);
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) m = max(m, pack_most<T>(w[n]));
    }
    m = __float_as_uint(pack_widen<T>(m));               // (order of FP32 bits from here on)
    m = block_max(m, line);
    if (threadIdx.x == 0) {
        if (gridDim.x == 1) scale[blockIdx.y] = tensor_scale_of(__uint_as_float(m));
        else partial[blockIdx.y * gridDim.x + blockIdx.x] = m;
    }
}
__global__ void __launch_bounds__(PACK_THREADS) tensor_scale_kernel(const uint32_t* partial, int blocks, float* scale) {
    __shared__ uint32_t line[32];
    launch_wait();
    launch_next();
    uint32_t m = 0u;
    for (int i = threadIdx.x; i < blocks; i += PACK_THREADS) m = max(m, partial[blockIdx.x * blocks + i]);
    m = block_max(m, line);
    if (threadIdx.x == 0) scale[blockIdx.x] = tensor_scale_of(__uint_as_float(m));
}

}  // namespace nk
