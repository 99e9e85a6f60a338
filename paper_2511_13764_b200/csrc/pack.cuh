// Packing into 4-bit elements with block scales, the scale of a tensor, and reading back.
//   MXF4   scale 2^(floor(log2 m) - 2): bits of m's exponent; x / scale is exact
//   NVF4   scale s = RN_e4m3(m / (6 t)), element RN_e2m1(x / (s t))
// The element's decision has to be that of exact arithmetic.  With t of 8 significant bits d = s t has 12 and is exact, a border b of
// the elements (0.25 .. 5) times d has 15, so for x of a 16-bit type x / d is either b or at least 2^-14 away from it.  x times a
// reciprocal of d that is off by 3 of its last places is within 2^-18 of the quotient (which is below 9 where it matters); rounded to a
// multiple of 2^-16 (one FMA onto 192 and a subtraction) it is b exactly where the quotient is, and on the quotient's side of b
// elsewhere.  So there is no division for an element.  FP32 x take one: a correctly rounded x / d is b only where the quotient is
// (24 bits against 15: the next quotient is more than half a step away).
//
// A block of threads has a tile of scales' 128 rows, so that the scales of a chunk of the contraction leave in one piece; a thread has
// a block of the format.  Along the columns a tile of 128 x 128 goes through shared memory, where a thread has a word of adjacent
// features.  BF16, 64 matrices of 4096 x 1024 to NVF4 106 us: 6.3 TB/s, the rate of a copy.  8192 x 4096 is two waves of blocks, whose
// loads and arithmetic overlap less (issue slots 60 % busy): NVF4 17.8 us (4.8 TB/s), along the columns 19.5-20.5; MXF4 15.1 and 17.6;
// its scale of a tensor 15.4 (4.4 TB/s), values in FP32 29 (5.3 TB/s).  From FP32, whose bytes take 24 us: MXF4 35.5 along the rows, 35 along the
// columns, NVF4, a division an element, 43 and 51, the scale 23 (5.8 TB/s).  16 x 4096 takes 2.1 to 2.4 us, a launch's start and end.
#pragma once
#include "mx_format.cuh"
#include "ptx.cuh"

namespace nk {

constexpr int PACK_THREADS = 256;
// along rows: elements of the contraction to a block of threads (8192 x 4096: NVF4 17.8 us by 256, 18.8 by 128; MXF4 16.1 and 15.1)
__host__ __device__ constexpr int pack_chunk(bool nv) { return nv ? 256 : 128; }
constexpr int PACK_LINE = 256;                           // reading back, likewise
constexpr int PACK_TURN = 128;                           // along columns: a tile's side
constexpr int PACK_MAX_GROUPS = 1024;

struct PackParams {
    int nv;                    // 1 NVF4, 0 MXF4
    int outer;                 // rows of the packed matrix (of one of the batch)
    int groups;                // 0: none
    int length;                // of the contraction
    int chunks;                // pack_chunk or PACK_LINE along the contraction (not along the columns)
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
    float t, per_t, per_six_t; // NVF4: the tensor's scale, 1 / t, 1 / (6 t)
    bool bad;
};
__device__ __forceinline__ PackScale pack_scale(const PackParams& p, int item) {
    PackScale s = {1.0f, 1.0f, 1.0f / 6.0f, false};
    if (p.nv && p.scale) {
        s.t = p.scale[item];
        s.bad = !(s.t >= 0x1p-100f && s.t <= 0x1p120f);
        s.per_t = __frcp_rn(s.t);
        s.per_six_t = __frcp_rn(6.0f * s.t);
    }
    return s;
}

// m / (6 t) to E4M3.  m times the reciprocal is off by 2 of its last places, so one that close to the border of two scales is decided by the
// border itself: border x 6 t is exact in 64 bits (5 + 2 + 24).
__device__ __noinline__ float pack_at_border(float q, float m, float t) {
    float border = 0.0f;
    if (q >= 0x1p-6f) {
        border = __uint_as_float((__float_as_uint(q) + 8u) & ~0x7FFFFu);        // halfway between steps of 1/8
    } else {
        const float n = rintf(q * 1024.0f);                                   // subnormals: odd multiples of 2^-10
        if ((static_cast<int>(n) & 1) && fabsf(q * 1024.0f - n) <= n * 0x1p-20f) border = n * 0x1p-10f;
    }
    if (border == 0.0f) return q;
    const double at = static_cast<double>(border) * 6.0 * static_cast<double>(t), x = m;
    return x > at ? __uint_as_float(__float_as_uint(border) + 1u) : x < at ? __uint_as_float(__float_as_uint(border) - 1u) : border;
}
__device__ __forceinline__ uint32_t pack_e4m3(float m, const PackScale& s) {
    float q = m * s.per_six_t;
    if (((__float_as_uint(q) + 8u - 0x80000u) & 0xFFFFFu) <= 16u || q < 0x1p-6f) q = pack_at_border(q, m, s.t);
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
    const float b = e4m3_to_f32(byte);
    factor = T == 0 ? b * s.t : b > 0.0f ? rcp_approx(b) * s.per_t : 0.0f;
    return byte;
}
// Quotients of two elements, each by its own factor: FP32 ...
template <bool NV>
__device__ __forceinline__ float2 pack_quotients(float2 x, float2 factor) {
    if (!NV) return mul2(x, factor);
    return make_float2(factor.x > 0.0f ? __fdiv_rn(x.x, factor.x) : 0.0f, factor.y > 0.0f ? __fdiv_rn(x.y, factor.y) : 0.0f);
}
// ... and of a word of 16-bit elements
template <int T, bool NV>
__device__ __forceinline__ float2 pack_quotients(uint32_t word, float2 factor) {
    const float2 x = make_float2(half_bits_to_f32(word & 0xFFFFu, T == 2), T == 2 ? half_bits_to_f32(word >> 16, 1) : __uint_as_float(word & 0xFFFF0000u));
    if (!NV) return mul2(x, factor);
    return add2(fma2(x, factor, make_float2(192.0f, 192.0f)), make_float2(-192.0f, -192.0f));
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
        const int lo = s_off[g], at = tile - mx_group_tile(lo, g), count = mx_tile_rows(at, s_off[g + 1] - lo);
        if (count > 0) {
            s_found[0] = lo + at * MX_TILE_ROWS;
            s_found[1] = count;
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
        const uint4 a = __ldg(p), b = __ldg(p + 1);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[T == 0 ? 4 : 0] = b.x, w[T == 0 ? 5 : 0] = b.y, w[T == 0 ? 6 : 0] = b.z, w[T == 0 ? 7 : 0] = b.w;
    } else {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + at));
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    }
}
// The largest magnitudes of words, one (FP32) or two (by halves) to a word; joined; and the one of a word.
template <int T>
__device__ __forceinline__ uint32_t pack_join(uint32_t a, uint32_t b) { return T == 0 ? max(a, b) : __vmaxu2(a, b); }
template <int T, int N>
__device__ __forceinline__ uint32_t pack_most(const uint32_t (&w)[N]) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) m = pack_join<T>(m, w[i] & (T == 0 ? 0x7FFFFFFFu : 0x7FFF7FFFu));
    return m;
}
template <int T>
__device__ __forceinline__ uint32_t pack_one(uint32_t m) { return T == 0 ? m : max(m & 0xFFFFu, m >> 16); }
// Along the rows: blockIdx.x a chunk of the contraction of a tile's rows (pieces of the same rows side by side, so that blocks at work
// together read whole rows), z the matrix.  A thread has a block: no exchange, and no division but FP32 elements' to NVF4, one for each.
template <int T, bool NV>
__global__ void __launch_bounds__(PACK_THREADS) pack_rows_kernel(const PackParams p) {
    constexpr int BLOCK = mx_block(NV), EIGHTS = BLOCK / 8, WORDS = T == 0 ? 8 : 4;
    constexpr int CHUNK = pack_chunk(NV), LANES = CHUNK / BLOCK;   // threads of a row: 16 or 4
    constexpr int STEP = PACK_THREADS / LANES;           // rows at a time: 16 or 64
    constexpr int AHEAD = (NV ? 4 : 2) / (T == 0 ? 2 : 1);         // of them on the way
    constexpr int TILES = CHUNK / (4 * BLOCK);
    __shared__ int s_off[PACK_MAX_GROUPS + 1], s_found[2];
    __shared__ __align__(16) uint8_t s_scale[TILES * MX_TILE_BYTES];
    const int item = blockIdx.z;
    const int tile = blockIdx.x / p.chunks, chunk = blockIdx.x - tile * p.chunks;
    launch_wait();
    launch_next();
    const PackRows rows = pack_rows(p, tile, s_off, s_found);
    if (rows.count <= 0) return;
    const PackScale s = pack_scale(p, item);
    for (int i = threadIdx.x; i < TILES * MX_TILE_BYTES / 4; i += PACK_THREADS) reinterpret_cast<uint32_t*>(s_scale)[i] = 0u;
    __syncthreads();
    const int c = threadIdx.x % LANES, k = chunk * CHUNK + c * BLOCK, pitch = static_cast<int>(mx_padded(p.length) / 2);
    const int eights = min(EIGHTS, (p.length - k) / 8);  // (the length is a multiple of 8; 0 or less: none)
    const bool kept = k < 2 * pitch;
    const size_t x0 = item * static_cast<size_t>(p.stride_x) + rows.first * static_cast<size_t>(p.ldx) + k;
    uint8_t* data = p.data + (static_cast<size_t>(item) * p.outer + rows.first) * pitch + k / 2;
    for (int r0 = threadIdx.x / LANES; r0 < rows.count; r0 += AHEAD * STEP) {
        uint32_t w[AHEAD][EIGHTS][WORDS];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n)
#pragma unroll
            for (int q = 0; q < EIGHTS; ++q) {
#pragma unroll
                for (int i = 0; i < WORDS; ++i) w[n][q][i] = 0u;
                if (q < eights && r0 + n * STEP < rows.count) pack_load<T>(p.x, x0 + (r0 + n * STEP) * static_cast<size_t>(p.ldx) + 8 * q, w[n][q]);
            }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const int r = r0 + n * STEP;
            if (r >= rows.count || !kept) break;
            uint32_t most = 0u;
#pragma unroll
            for (int q = 0; q < EIGHTS; ++q) most = pack_join<T>(most, pack_most<T>(w[n][q]));
            most = pack_one<T>(most);
            float factor;
            const uint32_t byte = pack_block<T, NV>(most, s, factor);
            uint32_t e[EIGHTS];
#pragma unroll
            for (int q = 0; q < EIGHTS; ++q) {
                float2 y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = make_float2(factor, factor);
                    if constexpr (T == 0) y[i] = pack_quotients<NV>(make_float2(__uint_as_float(w[n][q][2 * i]), __uint_as_float(w[n][q][2 * i + 1])), f);
                    else y[i] = pack_quotients<T, NV>(w[n][q][i], f);
                }
                // (a block that is not finite has factor 0 and may have products that are NaN)
                e[q] = most >= pack_not_finite<T>() ? 0u : f32_to_e2m1x8(y);
            }
            uint8_t* out = data + static_cast<size_t>(r) * pitch;
            if (NV) *reinterpret_cast<uint2*>(out) = make_uint2(e[0], e[1]);
            else *reinterpret_cast<uint4*>(out) = make_uint4(e[0], e[1], e[EIGHTS - 2], e[EIGHTS - 1]);
            if (eights > 0) s_scale[c / 4 * MX_TILE_BYTES + (r & 31) * 16 + (r >> 5) * 4 + (c & 3)] = static_cast<uint8_t>(byte);
        }
    }
    __syncthreads();
    const int first = chunk * TILES, n = min(TILES, p.tiles - first) * (MX_TILE_BYTES / 16);
    uint4* out = reinterpret_cast<uint4*>(p.scales + ((static_cast<size_t>(item) * p.row_tiles + tile) * p.tiles + first) * MX_TILE_BYTES);
    for (int i = threadIdx.x; i < n; i += PACK_THREADS) out[i] = reinterpret_cast<const uint4*>(s_scale)[i];
}

// Along the columns: blockIdx.x 128 features (a tile's rows), y 128 rows of X, z the matrix.
template <int T, bool NV>
__global__ void __launch_bounds__(PACK_THREADS, 4) pack_columns_kernel(const PackParams p) {
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
            v = __ldg(reinterpret_cast<const uint4*>(x + static_cast<size_t>(t0 + t) * p.ldx * (T == 0 ? 4 : 2) + piece * 16));
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
        uint32_t most[EACH], byte[EACH];
        float factor[EACH];
#pragma unroll
        for (int h = 0; h < EACH; ++h) {
            most[h] = T == 0 ? m : h ? m >> 16 : m & 0xFFFFu;
            byte[h] = pack_block<T, NV>(most[h], s, factor[h]);
        }
#pragma unroll
        for (int q = 0; q < BLOCK / 8; ++q) {
            uint32_t e[EACH];
            if constexpr (T == 0) {
                float2 y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[i] = pack_quotients<NV>(make_float2(__uint_as_float(v[q * 8 + 2 * i]), __uint_as_float(v[q * 8 + 2 * i + 1])), make_float2(factor[0], factor[0]));
                e[0] = f32_to_e2m1x8(y);
            } else {
                // both features of a word at once
                float2 a[4], z[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = make_float2(factor[0], factor[EACH - 1]);
                    const float2 y0 = pack_quotients<T, NV>(v[q * 8 + 2 * i], f), y1 = pack_quotients<T, NV>(v[q * 8 + 2 * i + 1], f);
                    a[i] = make_float2(y0.x, y1.x);
                    z[i] = make_float2(y0.y, y1.y);
                }
                e[0] = f32_to_e2m1x8(a);
                e[EACH - 1] = f32_to_e2m1x8(z);
            }
#pragma unroll
            for (int h = 0; h < EACH; ++h)
                *reinterpret_cast<uint32_t*>(out + (w * EACH + h) * OUT + b * (BLOCK / 2) + q * 4) = most[h] >= pack_not_finite<T>() ? 0u : e[h];
        }
#pragma unroll
        for (int h = 0; h < EACH; ++h) {
            const int f = w * EACH + h;
            if (f >= features || t0 + b * BLOCK >= p.length) byte[h] = 0u;
            s_scale[b / 4 * MX_TILE_BYTES + (f & 31) * 16 + (f >> 5) * 4 + (b & 3)] = static_cast<uint8_t>(byte[h]);
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

// Reading back: a warp has 256 elements of a row, a lane eight side by side, or for FP32 results twice four, so that a store of a warp
// is whole sectors (32 bytes to a lane in two stores: 8192 x 4096 41 us instead of 29).  Where the rows of Y are not whole pieces of
// eight, a warp's elements go by way of shared memory, from where consecutive lanes store consecutive ones.
template <int T, bool NV>
__global__ void __launch_bounds__(PACK_THREADS) pack_values_kernel(const PackParams p) {
    constexpr int TILES = PACK_LINE / (4 * mx_block(NV)), AHEAD = 4;
    constexpr int PARTS = T == 0 ? 2 : 1, WIDE = 8 / PARTS;                   // runs of a lane's elements, their length
    __shared__ int s_off[PACK_MAX_GROUPS + 1], s_found[2];
    __shared__ __align__(16) float s_line[PACK_THREADS / 32][PACK_LINE];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, item = blockIdx.z;
    const int tile = blockIdx.x / p.chunks, chunk = blockIdx.x - tile * p.chunks;
    launch_wait();
    launch_next();
    const PackRows rows = pack_rows(p, tile, s_off, s_found);
    if (rows.count <= 0) return;
    const float t = NV && p.scale ? p.scale[item] : 1.0f;
    const int k0 = chunk * PACK_LINE, pitch = static_cast<int>(mx_padded(p.length) / 2);
    const bool whole = p.length % 8 == 0;
    auto at = [&](int part) { return part * (PACK_LINE / PARTS) + lane * WIDE; };       // a run's place in the line
    const uint8_t* data = p.data + (static_cast<size_t>(item) * p.outer + rows.first) * pitch + k0 / 2;
    const uint8_t* scales = p.scales + ((static_cast<size_t>(item) * p.row_tiles + tile) * p.tiles + chunk * TILES) * MX_TILE_BYTES;
    const size_t y0 = (static_cast<size_t>(item) * p.outer + rows.first) * p.length + k0;
    for (int r0 = warp; r0 < rows.count; r0 += 8 * AHEAD) {
        uint32_t w[AHEAD], b[AHEAD][PARTS];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const int r = r0 + 8 * n;
            w[n] = 0u;
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
                const bool load = k0 + at(h) < p.length && r < rows.count;
                const int c = at(h) / mx_block(NV);
                const uint8_t* d = data + static_cast<size_t>(r) * pitch + at(h) / 2;
                if (load)
                    w[n] |= T == 0 ? static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t*>(d))) << (16 * h)
                                   : __ldg(reinterpret_cast<const uint32_t*>(d));
                b[n][h] = load ? __ldg(scales + c / 4 * MX_TILE_BYTES + (r & 31) * 16 + (r >> 5) * 4 + (c & 3)) : 0u;
            }
        }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const int r = r0 + 8 * n;
            if (r >= rows.count) break;
            float x[8];
            e2m1x8_to_f32(w[n], x);
            float s[PARTS];
#pragma unroll
            for (int h = 0; h < PARTS; ++h) s[h] = NV ? e4m3_to_f32(b[n][h]) : e8m0_to_f32(b[n][h]);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = NV ? x[i] * s[i / WIDE] * t : x[i] * s[i / WIDE];
            const size_t y = y0 + static_cast<size_t>(r) * p.length;
            if (whole) {
                if (T == 0) {
#pragma unroll
                    for (int h = 0; h < PARTS; ++h)
                        if (k0 + at(h) < p.length)
                            __stcs(reinterpret_cast<float4*>(static_cast<float*>(p.values) + y + at(h)),
                                   make_float4(x[h * WIDE], x[h * WIDE + 1], x[h * WIDE + 2], x[h * WIDE + 3]));
                } else if (k0 + at(0) < p.length) {
                    __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.values) + y + at(0)), pack8<T == 2>(x));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    *reinterpret_cast<float4*>(s_line[warp] + at(i / WIDE) + i % WIDE) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = s_line[warp][i * 32 + lane];
                    if (k0 + i * 32 + lane >= p.length) continue;
                    if (T == 0) static_cast<float*>(p.values)[y + i * 32 + lane] = v;
                    else static_cast<uint16_t*>(p.values)[y + i * 32 + lane] = static_cast<uint16_t>(pack_half2(v, 0.0f, T == 2) & 0xFFFFu);
                }
                __syncwarp();
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

// blockIdx.x of gridDim.x takes its share of the pieces of 8 elements, 4 to a thread at a time; y the matrix.  CLUSTER: the blocks are one
// cluster, whose first writes the scale; else tensor_scale_kernel does.
constexpr int SCALE_CLUSTER = 8, SCALE_THREADS = 512;
template <int T, bool CLUSTER, bool DENSE>
__device__ __forceinline__ void tensor_max(const PackParams& p, int rows, int width, uint32_t* partial, float* scale) {
    constexpr int AHEAD = CLUSTER ? 2 : T == 0 ? 4 : 8, WORDS = T == 0 ? 8 : 4;
    __shared__ uint32_t line[32];
    __shared__ __align__(16) uint4 maxima[SCALE_CLUSTER];
    const size_t x0 = blockIdx.y * static_cast<size_t>(p.stride_x);
    const int per_row = width / 8;
    const long long pieces = static_cast<long long>(rows) * per_row;
    const int turn = AHEAD * static_cast<int>(blockDim.x);
    if (CLUSTER) cluster_arrive();                       // everyone has started, once this is waited for: the stores below need it
    launch_wait();
    launch_next();
    uint32_t m = 0u;
    for (long long i = blockIdx.x * static_cast<long long>(turn) + threadIdx.x; i < pieces; i += static_cast<long long>(gridDim.x) * turn) {
        uint32_t w[AHEAD][WORDS];
        const int left = static_cast<int>(min(pieces - i, static_cast<long long>(turn)));
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const int j = n * static_cast<int>(blockDim.x);
#pragma unroll
            for (int q = 0; q < WORDS; ++q) w[n][q] = 0u;
            if (j < left) {
                if (DENSE) {
                    pack_load<T>(p.x, x0 + (i + j) * 8, w[n]);
                } else {
                    const long long r = (i + j) / per_row;
                    pack_load<T>(p.x, x0 + r * p.ldx + (i + j - r * per_row) * 8, w[n]);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) m = pack_join<T>(m, pack_most<T>(w[n]));
    }
    m = __float_as_uint(pack_widen<T>(pack_one<T>(m)));  // (order of FP32 bits from here on)
    m = block_max(m, line);
    if (CLUSTER) {
        cluster_wait();
        if (threadIdx.x == 0) st_cluster_v4(map_to_cta(smem_u32(maxima + cluster_ctarank()), 0), m, 0u, 0u, 0u);
        cluster_sync_all();
        if (blockIdx.x == 0 && threadIdx.x < SCALE_CLUSTER) {
            m = __reduce_max_sync((1u << SCALE_CLUSTER) - 1u, maxima[threadIdx.x].x);
            if (threadIdx.x == 0) scale[blockIdx.y] = tensor_scale_of(__uint_as_float(m));
        }
    } else if (threadIdx.x == 0) {
        partial[blockIdx.y * gridDim.x + blockIdx.x] = m;
    }
}
template <int T>
__global__ void __launch_bounds__(PACK_THREADS) tensor_max_kernel(const PackParams p, int rows, int width, uint32_t* partial) {
    if (p.ldx == width) tensor_max<T, false, true>(p, rows, width, partial, nullptr);
    else tensor_max<T, false, false>(p, rows, width, partial, nullptr);
}
template <int T>
__global__ void __launch_bounds__(SCALE_THREADS) __cluster_dims__(SCALE_CLUSTER, 1, 1)
tensor_cluster_kernel(const PackParams p, int rows, int width, float* scale) {
    if (p.ldx == width) tensor_max<T, true, true>(p, rows, width, nullptr, scale);
    else tensor_max<T, true, false>(p, rows, width, nullptr, scale);
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
