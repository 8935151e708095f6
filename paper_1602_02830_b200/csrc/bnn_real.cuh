// Shared pieces of the real-valued operators (dense, gated, norm, dropout): element types, activations and their slopes,
// argument checks.
#pragma once
#include "bnn_common.cuh"
#include <cuda_bf16.h>
#include <cuda_fp16.h>

static inline int bnn_real_size(int dtype) { return dtype == BNN_F32 ? 4 : (dtype == BNN_F16 || dtype == BNN_BF16) ? 2 : 0; }
// Sizes stay far enough below 2^31 that tile coordinates past an edge fit 32 bits; offsets are 64-bit.
constexpr int64_t BNN_REAL_MAX = 0x7fff0000;
static inline bool bnn_real_dim(int64_t n) { return n >= 0 && n <= BNN_REAL_MAX; }
// A row-major matrix: needed unless one of its dimensions is 0; a single row may have any leading dimension.
static inline int bnn_check_real(const void *p, int64_t ld, int64_t rows, int64_t cols, int size) {
    if (rows == 0 || cols == 0) return BNN_OK;
    if (!p) return BNN_ERR_INVALID_ARG;
    if (rows > 1 && ld < cols) return BNN_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)size) return BNN_ERR_ALIGNMENT;
    return BNN_OK;
}
static inline int bnn_check_real_opt(const void *p, int64_t ld, int64_t rows, int64_t cols, int size) {
    return p ? bnn_check_real(p, ld, rows, cols, size) : BNN_OK;
}
// Rows that can be read in 16-byte groups: base and row pitch are multiples of 16 bytes.
static inline bool bnn_rows16(const void *p, int64_t ld, int64_t rows, int size) {
    return bnn_aligned16(p) && (rows <= 1 || (ld * size) % 16 == 0);
}
static inline bool bnn_act_known(int act) { return act >= BNN_ACT_NONE && act <= BNN_ACT_HTANH; }

#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two values as one 32-bit word, first value in the low half; and back.
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// Eight consecutive values in 16-byte accesses.
template <typename T> __device__ __forceinline__ void unpack8(const uint4 *w, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(w[0].x); v[1] = __uint_as_float(w[0].y); v[2] = __uint_as_float(w[0].z); v[3] = __uint_as_float(w[0].w);
        v[4] = __uint_as_float(w[1].x); v[5] = __uint_as_float(w[1].y); v[6] = __uint_as_float(w[1].z); v[7] = __uint_as_float(w[1].w);
    } else {
        const float2 f0 = unpack2<T>(w[0].x), f1 = unpack2<T>(w[0].y), f2 = unpack2<T>(w[0].z), f3 = unpack2<T>(w[0].w);
        v[0] = f0.x; v[1] = f0.y; v[2] = f1.x; v[3] = f1.y; v[4] = f2.x; v[5] = f2.y; v[6] = f3.x; v[7] = f3.y;
    }
}
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    unpack8<T>(w, v);
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    }
}

// act(z).  exp and the division are the fast forms (relative error a few 2^-23): results are rounded to 8 or 11 bits.
// A NaN stays a NaN in every branch.
__device__ __forceinline__ float sigmoid_f(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
// The normal distribution: cdf Phi(z) and density phi(z).  Phi(-|z|) = e^(-z^2 / 2) t P(t), t = 1 / (1 + 0.375 |z| / sqrt 2), the form of Hastings (1955); P of
// degree 6 is a least-squares fit of 0 <= |z| <= 14.5, reweighted until the largest RELATIVE error is smallest (Lawson 1961): 6.4e-7, 1.0e-6 in float32.  bfloat16
// has float32's range, so that a tail like gelu(-8) = -5e-15 is a result like any other; Hastings' own coefficients are for the absolute error and were
// 1 % off there.  The exponential is the density's.  (erff and a separate exp made the slope of gelu compute-bound: 8192 x 4096 in 84 us.)
__device__ __forceinline__ float normal_cdf(float z, float &density) {
    const float e = __expf(-0.5f * z * z), t = __fdividef(1.0f, 1.0f + 0.26516503f * fabsf(z));
    const float p = 0.105669729f + t * (0.107844487f + t * (0.0833328068f + t * (0.141529396f + t * (-0.0647966936f + t * (0.193967491f - 0.0675475374f * t)))));
    const float half = t * p * e;
    density = 0.3989422804014327f * e;
    return z < 0.0f ? half : 1.0f - half;
}
// The tanh form of gelu, z (1 + tanh u) / 2 with u = sqrt(2 / pi) (z + 0.044715 z^3), as z sigmoid(2 u): the same function without the difference that
// cancels below z = -3 (20 % off at -5).
constexpr float GELU_2C = 1.5957691216057308f /* 2 sqrt(2 / pi) */, GELU_A = 0.044715f;
__device__ __forceinline__ float gelu_tanh_share(float z) { return sigmoid_f(GELU_2C * (z + GELU_A * z * z * z)); }
__device__ __forceinline__ float act_value(int act, float z) {
    switch (act) {
        case BNN_ACT_RELU: return z < 0.0f ? 0.0f : z;
        case BNN_ACT_GELU: { float density; return z * normal_cdf(z, density); }
        case BNN_ACT_GELU_TANH: return z * gelu_tanh_share(z);
        case BNN_ACT_SILU: return z * sigmoid_f(z);
        case BNN_ACT_SIGMOID: return sigmoid_f(z);
        case BNN_ACT_HTANH: return z > 1.0f ? 1.0f : (z < -1.0f ? -1.0f : z);
        default: return z;
    }
}
// act(z) and act'(z).  Far out on the tanh form its two factors 0 and infinity are not multiplied: the slope is 0 or 1 there.
__device__ __forceinline__ float act_slope(int act, float z, float &value) {
    switch (act) {
        case BNN_ACT_RELU: value = z < 0.0f ? 0.0f : z; return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
        case BNN_ACT_GELU: {
            float density;
            const float cdf = normal_cdf(z, density);
            value = z * cdf;
            return cdf + z * density;
        }
        case BNN_ACT_GELU_TANH: {
            const float p = gelu_tanh_share(z);
            value = z * p;
            if (fabsf(z) > 100.0f) return z > 0.0f ? 1.0f : 0.0f;
            return p * (1.0f + z * (1.0f - p) * GELU_2C * (1.0f + 3.0f * GELU_A * z * z));
        }
        case BNN_ACT_SILU: {
            const float p = sigmoid_f(z);
            value = z * p;
            return p * (1.0f + z * (1.0f - p));
        }
        case BNN_ACT_SIGMOID: {
            const float p = sigmoid_f(z);
            value = p;
            return p * (1.0f - p);
        }
        case BNN_ACT_HTANH:
            value = z > 1.0f ? 1.0f : (z < -1.0f ? -1.0f : z);
            return fabsf(z) <= 1.0f ? 1.0f : (fabsf(z) > 1.0f ? 0.0f : z);
        default: value = z; return 1.0f;
    }
}
#endif
