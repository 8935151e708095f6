// Microscaled matrices (OCP Microscaling Formats 1.0): layout, scales and elements, shared by the quantiser, the norms and the products.
//
// 32 neighbours v of a row share a power of two 2^X, X = floor(log2 max|v|) - emax, held to -127 .. 127 (E8M0: one byte, X + 127); an element is
// v 2^-X rounded to the nearest e4m3 (emax 8, up to 448) or e2m1 (emax 2, up to 6), ties to even, magnitudes above the largest to the largest.
//
// Memory.  Elements: row-major, rows of whole 128 elements (pitch 128 or 64 bytes a group), zeros behind the last column; element 2 i of an
// e2m1 row is the low half of byte i.  Scales: 512 bytes for 128 rows x 128 columns, row r and block b (of 32 columns) of such a tile at
// 16 (r % 32) + 4 (r / 32) + b, tiles of the same rows next to each other.  That is the order in which the tensor cores take them: thirty-two
// lanes of sixteen bytes, a column of tensor memory for each 32 rows, so a tile goes from memory to tensor memory as it is.
#pragma once
#include "bnn_real.cuh"

constexpr int BNN_MX_BLOCK = 32, BNN_MX_GROUP = 128, BNN_MX_TILE = 512;

static inline bool bnn_mx_known(int format) { return format == BNN_MX_E4M3 || format == BNN_MX_E2M1; }
static inline int64_t bnn_mx_groups(int64_t cols) { return (cols + BNN_MX_GROUP - 1) / BNN_MX_GROUP; }
static inline int64_t bnn_mx_pitch(int format, int64_t cols) { return bnn_mx_groups(cols) * (format == BNN_MX_E2M1 ? 64 : 128); }
static inline int bnn_check_mx(const bnn_mx_matrix *q) {
    if (!q || !bnn_mx_known(q->format) || !bnn_real_dim(q->rows) || !bnn_real_dim(q->cols)) return BNN_ERR_INVALID_ARG;
    if (q->rows == 0 || q->cols == 0) return BNN_OK;
    if (!q->values || !q->scales) return BNN_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(q->values) % 32 || reinterpret_cast<uintptr_t>(q->scales) % 16) return BNN_ERR_ALIGNMENT;
    return BNN_OK;
}

#ifdef __CUDACC__
__device__ __forceinline__ int64_t mx_scale_at(int64_t row, int64_t block, int64_t groups) {
    return ((row >> 7) * groups + (block >> 2)) * BNN_MX_TILE + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}
// The scale's byte from the bits of max|v|.  Bits of magnitudes are ordered like the magnitudes, infinities and NaN above all: a block that holds one is
// NaN (byte 255).  Subnormal maxima have exponent bits 0 and are below 2^-126, where X is -127 whatever they are.
template <bool FOUR> __device__ __forceinline__ uint32_t mx_scale(uint32_t amax) {
    const uint32_t e = amax >> 23, emax = FOUR ? 2 : 8;
    return e == 255u ? 255u : e > emax ? e - emax : 0u;
}
__device__ __forceinline__ float mx_down(uint32_t scale) { return __uint_as_float(scale == 255u ? 0x7fffffffu : (254u - scale) << 23); }                    // 2^-X, exact
__device__ __forceinline__ float mx_up(uint32_t scale) { return __uint_as_float(scale == 255u ? 0x7fffffffu : scale ? scale << 23 : 0x00400000u); }        // 2^X
// Eight scaled values as elements: two words (e4m3) or one (e2m1), the first value lowest.
__device__ __forceinline__ uint32_t mx_e4m3x4(float a, float b, float c, float d) {
    uint32_t w;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
    return w;
}
__device__ __forceinline__ uint32_t mx_e2m1x8(const float (&v)[8]) {
    uint32_t w;
    asm("{\n\t.reg .b8 p, q, r, s;\n\tcvt.rn.satfinite.e2m1x2.f32 p, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 q, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 r, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 s, %8, %7;\n\tmov.b32 %0, {p, q, r, s};\n\t}"
        : "=r"(w) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}
template <bool FOUR> __device__ __forceinline__ void mx_encode8(const float (&v)[8], uint32_t (&w)[2]) {
    if constexpr (FOUR) { w[0] = mx_e2m1x8(v); w[1] = 0; }
    else { w[0] = mx_e4m3x4(v[0], v[1], v[2], v[3]); w[1] = mx_e4m3x4(v[4], v[5], v[6], v[7]); }
}
// And back, unscaled (exact: both formats fit half precision).
template <bool FOUR> __device__ __forceinline__ void mx_decode8(const uint32_t (&w)[2], float (&v)[8]) {
    uint32_t h[4];
    if constexpr (FOUR) {
        // The three bits of a magnitude are the lowest two exponent bits and the highest mantissa bit of a half 2^14 times smaller, subnormals included.
        // (Taken apart by shifts: bytes packed by one instruction and taken apart by another came back with the upper two zero.)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t b = w[0] >> (8 * i);
            h[i] = (b & 7u) << 9 | (b & 8u) << 12 | (b & 0x70u) << 21 | (b & 0x80u) << 24;
        }
    } else
        asm("{\n\t.reg .b16 p, q, r, s;\n\tmov.b32 {p, q}, %4;\n\tmov.b32 {r, s}, %5;\n\tcvt.rn.f16x2.e4m3x2 %0, p;\n\tcvt.rn.f16x2.e4m3x2 %1, q;\n\t"
            "cvt.rn.f16x2.e4m3x2 %2, r;\n\tcvt.rn.f16x2.e4m3x2 %3, s;\n\t}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w[0]), "r"(w[1]));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<__half>(h[i]);
        v[2 * i] = FOUR ? f.x * 16384.0f : f.x;
        v[2 * i + 1] = FOUR ? f.y * 16384.0f : f.y;
    }
}
__device__ __forceinline__ uint32_t mx_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// One row's columns c .. c + 7 (c a multiple of 8; zeros behind the last column) of every lane of a warp, lanes next to each other: four neighbouring lanes
// hold a block, sixteen a group.  All lanes take part; those with c >= limit (the row's pitch in elements, a multiple of 128) write nothing.
// On return v holds the values that the elements stand for.
template <bool FOUR> __device__ __forceinline__ void mx_write8(uint8_t *values, uint8_t *scales, int64_t row, int64_t c, int64_t limit, float (&v)[8], bool back) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, mx_magnitude(v[j]));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t scale = mx_scale<FOUR>(top);
    const float down = mx_down(scale);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= down;
    uint32_t w[2];
    mx_encode8<FOUR>(v, w);
    const int lane = threadIdx.x & 31;
    uint32_t four = scale << (8 * ((lane >> 2) & 3));           // the group's scales in the order of its blocks
    four |= __shfl_xor_sync(0xffffffffu, four, 4);
    four |= __shfl_xor_sync(0xffffffffu, four, 8);
    if (c < limit) {
        if constexpr (FOUR) *reinterpret_cast<uint32_t *>(values + row * (limit / 2) + c / 2) = w[0];
        else *reinterpret_cast<uint2 *>(values + row * limit + c) = make_uint2(w[0], w[1]);
        if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(scales + mx_scale_at(row, c >> 5, limit >> 7)) = four;
    }
    if (back) {
        const float up = mx_up(scale);
        mx_decode8<FOUR>(w, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= up;
    }
}
// The same for one column per lane: the warp's 32 columns c (c of lane 0 a multiple of 32) are a block.
template <bool FOUR> __device__ __forceinline__ void mx_write1(uint8_t *values, uint8_t *scales, int64_t row, int64_t c, int64_t limit, float &v, bool back) {
    const uint32_t scale = mx_scale<FOUR>(__reduce_max_sync(0xffffffffu, mx_magnitude(v)));
    const float e[8] = {v * mx_down(scale), 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t w[2];
    mx_encode8<FOUR>(e, w);
    const int lane = threadIdx.x & 31;
    if constexpr (FOUR) {
        const uint32_t next = __shfl_down_sync(0xffffffffu, w[0] & 15u, 1);
        if (c < limit && !(lane & 1)) values[row * (limit / 2) + c / 2] = (uint8_t)((w[0] & 15u) | next << 4);
    } else if (c < limit) values[row * limit + c] = (uint8_t)w[0];
    if (c < limit && lane == 0) scales[mx_scale_at(row, c >> 5, limit >> 7)] = (uint8_t)scale;
    if (back) {
        float d[8];
        mx_decode8<FOUR>(w, d);
        v = d[0] * mx_up(scale);
    }
}
#endif
