// What the norms share (bnn_norm.cu, bnn_norm_mx.cu): arguments, and eight columns of a row per thread and slot.
#pragma once
#include "bnn_real.cuh"

namespace bnn_norm {

struct NormArgs {
    const void *x, *block;
    int64_t ldx, ldb;
    void *stream, *normed;
    int64_t lds, ldn;
    float *stats;                      // M x 4: mean_b, r_b, mean_s, r_s
    int64_t M;
    int D;
    float eps, alpha, inv_d;
    int layer, post, pre;
    const void *post_w, *post_c, *pre_w, *pre_c, *gate;
    int64_t ld_gate, rows_per_gate;
    // backward
    const void *ds, *dn;
    int64_t ldds, lddn;
    void *dx, *db, *dgate;
    int64_t lddx, lddb, ld_dgate;
    float *part, *part_gate;           // partial column sums: [CTA][4][D], [unit][D]
    int want;                          // which of the four parameter sums are wanted (bits: pre_w, pre_c, post_w, post_c)
    int64_t groups, chunks, chunk_rows, units;
    // microscaled output: elements, scales, pitch in elements; normed receives the represented values
    uint8_t *mx_values, *mx_scales;
    int mx_limit, mx_four;
    double inv;                        // 1 / D
};

// Eight columns of one row per thread and slot, as they are in memory.  VEC: neighbouring columns in 16-byte accesses; otherwise
// (odd pitches or widths) columns a team apart, so that neighbouring threads still touch neighbouring elements.
template <typename T> struct Eight {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
        else { const float2 f = unpack2<T>(w[j >> 1]); return (j & 1) ? f.y : f.x; }
    }
    __device__ __forceinline__ void fill(float v) {
#pragma unroll
        for (int i = 0; i < (int)(2 * sizeof(T)); ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v);
            else w[i] = pack2<T>(v, v);
        }
    }
};
template <bool VEC> __device__ __forceinline__ int column(int slot, int j, int tid, int team) {
    return VEC ? (slot * team + tid) * 8 + j : (slot * 8 + j) * team + tid;
}
template <typename T, bool VEC> __device__ __forceinline__ Eight<T> read8(const T *row, int slot, int tid, int team, int D) {
    Eight<T> e;
    if constexpr (VEC) {
        const int c = column<true>(slot, 0, tid, team);
        // a predicated load instead of a branch: the branches around 28 accesses a row were a sixth of the instructions
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
                         "@p ld.global.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
                         : "=&r"(e.w[4 * i]), "=&r"(e.w[4 * i + 1]), "=&r"(e.w[4 * i + 2]), "=&r"(e.w[4 * i + 3])
                         : "l"(reinterpret_cast<const uint4 *>(row + c) + i), "r"((uint32_t)(c < D)) : "memory");
    } else {
#pragma unroll
        for (int j = 0; j < 8; j += 8 / (2 * (int)sizeof(T))) {
            // requests without a branch, which would wait for each: beyond D the last column again
            const int c = column<false>(slot, j, tid, team), c1 = c + team;
            if constexpr (sizeof(T) == 4) {
                const uint32_t v = __float_as_uint(row[c < D ? c : D - 1]);
                e.w[j] = c < D ? v : 0u;
            } else {
                const uint16_t *bits = reinterpret_cast<const uint16_t *>(row);
                const uint32_t v = bits[c < D ? c : D - 1], v1 = bits[c1 < D ? c1 : D - 1];
                e.w[j >> 1] = (c < D ? v : 0u) | (c1 < D ? v1 << 16 : 0u);
            }
        }
    }
    return e;
}
template <typename T, bool VEC>
__device__ __forceinline__ void write8(T *row, int slot, int tid, int team, int D, const float (&v)[8]) {
    if constexpr (VEC) {
        const int c = column<true>(slot, 0, tid, team);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            uint32_t w[4];
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = __float_as_uint(v[4 * i + k]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = pack2<T>(v[2 * k], v[2 * k + 1]);
            }
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p st.global.v4.u32 [%4], {%0,%1,%2,%3};\n\t}"
                         ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "l"(reinterpret_cast<uint4 *>(row + c) + i), "r"((uint32_t)(c < D)) : "memory");
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = column<false>(slot, j, tid, team);
            if (c < D) row[c] = from_f32<T>(v[j]);
        }
    }
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace bnn_norm

// The forward pass with the stream's norm microscaled: vec as in bnn_norm.cu (bnn_norm_mx.cu).
int bnn_launch_norm_mx(bnn_ctx *ctx, const bnn_norm::NormArgs &a, int dtype, bool vec);
