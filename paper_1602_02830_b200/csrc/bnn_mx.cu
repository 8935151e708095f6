// Microscaled matrices: quantisation of rows and the way back (formats and layout: bnn_mx.cuh).
//
// Bound: HBM.  One pass: an element is read once, its code and, where asked for, the value that the code stands for are written once.  Measured: 8192 x 4096 bf16 to
// e4m3 with represented values 28.0 us = 6.0 TB/s, without 20.0 us = 5.1 TB/s, to e2m1 19.7 us; 1000 x 4100 float16 (rows off the 16-byte rule) 5.5 us, lane by lane
// instead of by words 12.8; one row 1.7 us.
#include "bnn_mx.cuh"

namespace {

struct MxArgs {
    const void *x;          // rows to quantise, or NULL
    void *out;              // values: the represented ones, or NULL
    int64_t ldx, ldo, rows, cols, limit;
    uint8_t *values, *scales;
    int64_t chunks;         // of 256 columns
};

// A warp takes 256 columns of a row, ROWS rows one after another, all of which it requests before it computes.  (Four rows: as fast at 8192 x 4096, 48 x 2048 1.8 -> 2.4 us.)
constexpr int WARPS = 8, ROWS = 2, CHUNK = 256;

template <typename T, bool VEC, bool FOUR>
__global__ void __launch_bounds__(WARPS * 32) k_mx_quantize(const __grid_constant__ MxArgs p) {
    constexpr int WORDS = (int)sizeof(T) / 2;
    __shared__ __align__(16) uint4 stage[VEC ? 1 : WARPS][VEC ? 1 : 32 * WORDS];
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    const int64_t group = blockIdx.x / p.chunks, c0 = (blockIdx.x - group * p.chunks) * CHUNK;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = (group * WARPS + warp) * ROWS, c = c0 + lane * 8;
    const T *x = static_cast<const T *>(p.x);
    T *out = static_cast<T *>(p.out);
    uint4 w[ROWS][WORDS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[r][i] = make_uint4(0u, 0u, 0u, 0u);
        if (first + r >= p.rows || c >= p.cols) continue;
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[r][i] = reinterpret_cast<const uint4 *>(x + (first + r) * p.ldx + c)[i];
        } else {
            uint32_t t[4 * WORDS];
            mx_read_words<T>(x + (first + r) * p.ldx, c, p.cols, t);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[r][i] = make_uint4(t[4 * i], t[4 * i + 1], t[4 * i + 2], t[4 * i + 3]);
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (first + r >= p.rows) break;
        float v[8];
        unpack8<T>(w[r], v);
        mx_write8<FOUR>(p.values, p.scales, first + r, c, p.limit, v, out != nullptr, MxExact());
        if (!out) continue;
        if constexpr (VEC) {
            if (c < p.cols) store8(out + (first + r) * p.ldo + c, v);
        } else {
            mx_spread8(out + (first + r) * p.ldo, c0, p.cols, v, reinterpret_cast<T *>(stage[warp]));
        }
    }
}

template <typename T, bool VEC, bool FOUR>
__global__ void __launch_bounds__(WARPS * 32) k_mx_values(const __grid_constant__ MxArgs p) {
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    const int64_t group = blockIdx.x / p.chunks, c = (blockIdx.x - group * p.chunks) * CHUNK + (threadIdx.x & 31) * 8;
    const int64_t first = (group * WARPS + (threadIdx.x >> 5)) * ROWS;
    if (c >= p.cols) return;
    T *out = static_cast<T *>(p.out);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t row = first + r;
        if (row >= p.rows) break;
        uint32_t w[2];
        if constexpr (FOUR) { w[0] = *reinterpret_cast<const uint32_t *>(p.values + row * (p.limit / 2) + c / 2); w[1] = 0; }
        else {
            const uint2 t = *reinterpret_cast<const uint2 *>(p.values + row * p.limit + c);
            w[0] = t.x; w[1] = t.y;
        }
        const float up = mx_up(p.scales[mx_scale_at(row, c >> 5, p.limit >> 7)]);
        float v[8];
        mx_decode8<FOUR>(w, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= up;
        T *to = out + row * p.ldo + c;
        if (VEC) store8(to, v);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < p.cols) to[j] = from_f32<T>(v[j]);
        }
    }
}

// Whether every row is made of whole 16-byte groups of eight columns.
bool whole(const void *p, int64_t ld, int64_t rows, int64_t cols, int size) { return !p || (cols % 8 == 0 && bnn_rows16(p, ld, rows, size)); }

template <typename T, bool VEC> int launch(bnn_ctx *ctx, const MxArgs &a, bool four) {
    const int64_t blocks = (a.rows + WARPS * ROWS - 1) / (WARPS * ROWS) * a.chunks;
    if (blocks > 0x7fffffff) return BNN_ERR_INVALID_ARG;
    auto kernel = a.x ? (four ? k_mx_quantize<T, VEC, true> : k_mx_quantize<T, VEC, false>) : (four ? k_mx_values<T, VEC, true> : k_mx_values<T, VEC, false>);
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, dim3((unsigned)blocks), dim3(WARPS * 32), 0, ctx->stream, a));
    return bnn_check_launch(ctx);
}
int run(bnn_ctx *ctx, int dtype, MxArgs &a, const bnn_mx_matrix *q) {
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (q->rows == 0 || q->cols == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    a.rows = q->rows; a.cols = q->cols;
    a.values = static_cast<uint8_t *>(q->values); a.scales = static_cast<uint8_t *>(q->scales);
    a.limit = bnn_mx_groups(q->cols) * BNN_MX_GROUP;
    a.chunks = (q->cols + CHUNK - 1) / CHUNK;
    const bool four = q->format == BNN_MX_E2M1;
    const int size = bnn_real_size(dtype);
    const bool vec = whole(a.x, a.ldx, q->rows, q->cols, size) && whole(a.out, a.ldo, q->rows, q->cols, size);
    if (dtype == BNN_F32) return vec ? launch<float, true>(ctx, a, four) : launch<float, false>(ctx, a, four);
    if (dtype == BNN_F16) return vec ? launch<__half, true>(ctx, a, four) : launch<__half, false>(ctx, a, four);
    return vec ? launch<__nv_bfloat16, true>(ctx, a, four) : launch<__nv_bfloat16, false>(ctx, a, four);
}

}  // namespace

extern "C" int64_t bnn_mx_ld(int format, int64_t cols) { return bnn_mx_known(format) && bnn_real_dim(cols) ? bnn_mx_pitch(format, cols) : 0; }
extern "C" size_t bnn_mx_scale_bytes(int64_t rows, int64_t cols) {
    if (!bnn_real_dim(rows) || !bnn_real_dim(cols)) return 0;
    return (size_t)((rows + 127) / 128) * (size_t)bnn_mx_groups(cols) * BNN_MX_TILE;
}

extern "C" int bnn_mx_quantize(bnn_ctx *ctx, int dtype, const void *x, int64_t ldx, const bnn_mx_matrix *q, void *represented, int64_t ldv) {
    if (int st = bnn_check_mx(q)) return st;
    const int size = bnn_real_size(dtype);
    if (!size) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(x, ldx, q->rows, q->cols, size)) return st;
    if (int st = bnn_check_real_opt(represented, ldv, q->rows, q->cols, size)) return st;
    if (bnn_mx_touches(q, x, ldx, q->rows, q->cols, size) || bnn_mx_touches(q, represented, ldv, q->rows, q->cols, size)) return BNN_ERR_INVALID_ARG;
    MxArgs a{};
    a.x = x; a.ldx = ldx; a.out = represented; a.ldo = ldv;
    return run(ctx, dtype, a, q);
}

extern "C" int bnn_mx_values(bnn_ctx *ctx, const bnn_mx_matrix *q, int dtype, void *out, int64_t ldo) {
    if (int st = bnn_check_mx(q)) return st;
    const int size = bnn_real_size(dtype);
    if (!size) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(out, ldo, q->rows, q->cols, size)) return st;
    if (bnn_mx_touches(q, out, ldo, q->rows, q->cols, size)) return BNN_ERR_INVALID_ARG;
    MxArgs a{};
    a.out = out; a.ldo = ldo;
    return run(ctx, dtype, a, q);
}
