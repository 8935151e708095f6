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
// Whether a microscaled matrix shares memory with `bytes` bytes at p; with a row-major matrix; with another one.  Results are written while other parts of the inputs are still to be
// read, so that a call whose result shares memory with an input is refused.
static inline bool bnn_mx_touches(const bnn_mx_matrix *q, const void *p, uint64_t bytes) {
    if (!p || !bytes || q->rows == 0 || q->cols == 0) return false;
    const auto meet = [&](const void *a, uint64_t n) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(p);
        return x < y ? y - x < n : x - y < bytes;
    };
    return meet(q->values, (uint64_t)q->rows * (uint64_t)bnn_mx_pitch(q->format, q->cols)) || meet(q->scales, bnn_mx_scale_bytes(q->rows, q->cols));
}
static inline bool bnn_mx_touches(const bnn_mx_matrix *q, const void *p, int64_t ld, int64_t rows, int64_t cols, int size) {
    return rows > 0 && cols > 0 && bnn_mx_touches(q, p, ((uint64_t)(rows - 1) * (uint64_t)(rows > 1 ? ld : 0) + (uint64_t)cols) * (uint64_t)size);
}
static inline bool bnn_mx_touches(const bnn_mx_matrix *q, const bnn_mx_matrix *other) {
    if (other->rows == 0 || other->cols == 0) return false;
    return bnn_mx_touches(q, other->values, (uint64_t)other->rows * (uint64_t)bnn_mx_pitch(other->format, other->cols)) ||
           bnn_mx_touches(q, other->scales, bnn_mx_scale_bytes(other->rows, other->cols));
}

#ifdef __CUDACC__
// Two float32 values in one instruction.
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
    unsigned long long w;
    asm("mov.b64 %0, {%1, %2};" : "=l"(w) : "f"(a), "f"(b));
    return w;
}
__device__ __forceinline__ void pair_out(unsigned long long w, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(w)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ unsigned long long both(float v) { return pair_of(v, v); }

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
        // Taken apart by shifts: where one kernel both packs four bytes by mov.b32 {p, q, r, s} (mx_e2m1x8) and takes a word apart by its reverse, nvcc 12.9.86 makes one of the two and
        // loses the upper bytes, also with an opaque step between them (a kernel of nothing else: 32 of 32 words).  Either of them alone is right.
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

// Eight neighbouring elements of a row that begins at `row` and has `cols`, from column c on, packed as in memory; zeros behind the end.  Rows off the 16-byte rule are
// read as aligned words of four bytes, shifted into place where they begin in the middle of one; the half words at both ends of a row are read alone.
template <typename T> __device__ __forceinline__ void mx_read_words(const T *row, int64_t c, int64_t cols, uint32_t (&w)[2 * sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = c + i < cols ? __float_as_uint(row[c + i]) : 0u;
    } else {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(row), end = begin + 2 * (uintptr_t)cols, at = begin + 2 * (uintptr_t)c, from = at & ~uintptr_t(3);
        const bool odd = at & 2;
        uint32_t t[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const uintptr_t p = from + 4 * i;
            t[i] = 0u;
            if (i == 4 && !odd) continue;
            if (p >= begin && p + 4 <= end) t[i] = *reinterpret_cast<const uint32_t *>(p);
            else if (p >= begin && p < end) t[i] = *reinterpret_cast<const uint16_t *>(p);
            else if (p < begin && p + 2 < end) t[i] = (uint32_t)*reinterpret_cast<const uint16_t *>(p + 2) << 16;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = odd ? __funnelshift_r(t[i], t[i + 1], 16) : t[i];
    }
}
// Eight values of each lane, neighbouring lanes at neighbouring columns from c0 on, to a row off the 16-byte rule: through the warp's shared memory (256 elements), so that
// neighbouring lanes write neighbouring elements.  The warp is together.
template <typename T> __device__ __forceinline__ void mx_spread8(T *row, int64_t c0, int64_t cols, const float (&v)[8], T *stage) {
    const int lane = threadIdx.x & 31;
    store8(stage + lane * 8, v);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c0 + j * 32 + lane < cols) row[c0 + j * 32 + lane] = stage[j * 32 + lane];
    __syncwarp();
}

// Values that are float32 as they stand; or float32 roundings of others: rest.held().lack(j, v) is then what v lacks.  Whether such a value is on this or that side of a border
// (of two elements; of two shared exponents, where it is the block's largest) is decided by the exact one, which differs from v by MX_NEAR of it at most: whatever lies farther
// from a border is on the same side as v.  What lies closer than rest.tie of it can't be told from the border and counts as on it.  (One in 2^20 values rounds to a border.)
struct MxExact { static constexpr bool rounded = false; };
constexpr float MX_NEAR = 1.0f / (1 << 22);

// The element that a scaled value is converted to, as a value.
template <bool FOUR> __device__ __forceinline__ float mx_element(float v) {
    float e[8] = {v, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t w[2];
    mx_encode8<FOUR>(e, w);
    mx_decode8<FOUR>(w, e);
    return e[0];
}

// Eight values of a lane one of which may be beside a border: their elements, and their block's scale from its largest magnitude.  The block's four lanes come together where its
// largest is beside a power of two.  Out of line and in a loop, arrays in memory: one in two thousand lanes gets here, and inlined it took registers from all of them.
constexpr uint32_t MX_UNITS = 2;
struct MxCodes { uint32_t w[2], scale; };
__device__ __forceinline__ bool mx_beside_power(uint32_t top) { return ((top + MX_UNITS) ^ (top - MX_UNITS)) & 0xff800000u; }
template <bool FOUR, typename H> __device__ __noinline__ MxCodes mx_decide(const float *v, uint32_t top, const H *rest) {
    if (mx_beside_power(top) && top - 0x00800000u < 0x7e800000u) {
        // The largest reaches the power of two if one of the block's exact values does.
        const uint32_t power = (top + MX_UNITS) & 0x7f800000u;
        const float border = __uint_as_float(power);
        bool reached = false;
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
            const float size = fabsf(v[j]);
            if (__float_as_uint(size) + MX_UNITS >= power) reached |= (size - border) + copysignf(1.0f, v[j]) * rest->lack(j, v[j]) >= -rest->tie * border;
        }
        top = __any_sync(0xfu << (threadIdx.x & 28), reached) ? max(top, power) : power - 1;
    }
    const uint32_t scale = mx_scale<FOUR>(top);
    const float down = mx_down(scale);
    float e[8];
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
        const float low = mx_element<FOUR>(v[j] * (down * (1.0f - MX_NEAR))), high = mx_element<FOUR>(v[j] * (down * (1.0f + MX_NEAR))), edge = 0.5f * (low + high);
        e[j] = low;
        if (low == high) continue;
        const float d = copysignf(1.0f, v[j]) * ((v[j] * down - edge) + rest->lack(j, v[j]) * down);
        e[j] = fabsf(d) <= rest->tie * fabsf(edge) ? edge : d > 0.0f ? high : low;           // (an edge is converted to the even one)
    }
    MxCodes out;
    mx_encode8<FOUR>(e, out.w);
    out.scale = scale;
    return out;
}

// One row's columns c .. c + 7 (c a multiple of 8; zeros behind the last column) of every lane of a warp, lanes next to each other: four neighbouring lanes
// hold a block, sixteen a group.  All lanes take part; those with c >= limit (the row's pitch in elements, a multiple of 128) write nothing.
// On return v holds the values that the elements stand for, where they are asked back.
template <bool FOUR, typename F> __device__ __forceinline__ void mx_write8(uint8_t *values, uint8_t *scales, int64_t row, int64_t c, int64_t limit, float (&v)[8], bool back, const F &rest) {
    const int lane = threadIdx.x & 31;
    uint32_t top = F::rounded ? MX_UNITS : 0;                       // (a block of zeros is beside no power of two)
#pragma unroll
    for (int j = 0; j < 8; j += 2) top = __vimax3_u32(top, mx_magnitude(v[j]), mx_magnitude(v[j + 1]));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    uint32_t scale = mx_scale<FOUR>(top), w[2];
    const float down = mx_down(scale);
    if constexpr (F::rounded) {
        // Elements of the values moved by MX_NEAR towards zero and away from it are alike where no border is near, and so is the exponent of the largest one moved by MX_UNITS.
        float in[8], away[8];
        uint32_t w_away[2];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const unsigned long long t = pair_of(v[j], v[j + 1]);
            pair_out(mul2(t, both(down * (1.0f - MX_NEAR))), in[j], in[j + 1]);
            pair_out(mul2(t, both(down * (1.0f + MX_NEAR))), away[j], away[j + 1]);
        }
        mx_encode8<FOUR>(in, w);
        mx_encode8<FOUR>(away, w_away);
        if (__builtin_expect((w[0] != w_away[0]) | (w[1] != w_away[1]) | mx_beside_power(top), 0)) {
            const auto held = rest.held();
            float mine[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[j] = v[j];
            const MxCodes codes = mx_decide<FOUR>(mine, top, &held);
            w[0] = codes.w[0]; w[1] = codes.w[1]; scale = codes.scale;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j += 2) pair_out(mul2(pair_of(v[j], v[j + 1]), both(down)), v[j], v[j + 1]);
        mx_encode8<FOUR>(v, w);
    }
    const float up = mx_up(scale);
    uint32_t four = scale << (8 * ((lane >> 2) & 3));           // the group's scales in the order of its blocks
    four |= __shfl_xor_sync(0xffffffffu, four, 4);
    four |= __shfl_xor_sync(0xffffffffu, four, 8);
    if (c < limit) {
        if constexpr (FOUR) *reinterpret_cast<uint32_t *>(values + row * (limit / 2) + c / 2) = w[0];
        else *reinterpret_cast<uint2 *>(values + row * limit + c) = make_uint2(w[0], w[1]);
        if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(scales + mx_scale_at(row, c >> 5, limit >> 7)) = four;
    }
    if (back) {
        mx_decode8<FOUR>(w, v);
#pragma unroll
        for (int j = 0; j < 8; j += 2) pair_out(mul2(pair_of(v[j], v[j + 1]), both(up)), v[j], v[j + 1]);
    }
}
#endif
