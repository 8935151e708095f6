// Dropout whose mask is never stored.  y = residual + (kept ? x / (1 - p) : 0); the mask is a pure function of
// (rows, cols, seed, offset), so the backward pass is the same call on dy and recomputes it.
//
// Mathematics: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds
//   (c0, c1, c2, c3) -> (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)),  keys advanced by Weyl constants,
// give four 32-bit words per counter; word e % 4 at counter e / 4 decides element e.
// Bound: HBM.  Per element 2 (3 with a residual) x the element size.  The generator costs 20 wide multiplies and 20
// three-input logic operations per four elements.
#include "bnn_real.cuh"
#include <cmath>

namespace {

struct DropArgs {
    const void *x, *residual;
    void *y;
    int64_t ldx, ldr, ldy, rows, cols;
    uint32_t thr;             // kept when the word is >= thr
    int drop_all;             // p = 1 (its threshold 2^32 does not fit a word)
    float scale;
    uint32_t k0, k1, o0, o1;  // seed and offset words
    int vec;                  // every group of 8 elements lies in one row and on 16-byte boundaries
};

__device__ __forceinline__ uint4 philox4x32(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b; c3 = (uint32_t)a; c0 = n0; c2 = n2;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// One thread per 8 consecutive elements (two counters).  The row is requested before the generator runs, which covers the wait.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout(const DropArgs p) {
    const int64_t total = p.rows * p.cols;
    const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x, e0 = g * 8;
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    if (e0 >= total) return;
    const T *x = static_cast<const T *>(p.x), *res = static_cast<const T *>(p.residual);
    T *y = static_cast<T *>(p.y);
    int64_t row = 0, col = e0;
    if (p.rows > 1) {
        row = total <= 0xffffffffll ? (int64_t)((uint32_t)e0 / (uint32_t)p.cols) : e0 / p.cols;
        col = e0 - row * p.cols;
    }
    const bool whole = p.vec && e0 + 8 <= total;
    uint4 xw[sizeof(T) / 2], rw[sizeof(T) / 2];
    if (whole) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            xw[i] = __ldcs(reinterpret_cast<const uint4 *>(x + row * p.ldx + col) + i);
            if (res) rw[i] = __ldcs(reinterpret_cast<const uint4 *>(res + row * p.ldr + col) + i);
        }
    }
    const uint64_t c = (uint64_t)g * 2;
    const uint4 a = philox4x32((uint32_t)c, (uint32_t)(c >> 32), p.o0, p.o1, p.k0, p.k1);
    const uint4 b = philox4x32((uint32_t)(c + 1), (uint32_t)((c + 1) >> 32), p.o0, p.o1, p.k0, p.k1);
    const uint32_t word[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (whole) {
        float v[8], r[8];
        unpack8<T>(xw, v);
        if (res) unpack8<T>(rw, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = (word[j] >= p.thr && !p.drop_all) ? v[j] * p.scale : 0.0f;
            if (res) v[j] += r[j];
        }
        store8(y + row * p.ldy + col, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (e0 + j < total) {
                float v = (word[j] >= p.thr && !p.drop_all) ? to_f32(x[row * p.ldx + col]) * p.scale : 0.0f;
                if (res) v += to_f32(res[row * p.ldr + col]);
                y[row * p.ldy + col] = from_f32<T>(v);
                if (++col == p.cols) { col = 0; ++row; }
            }
        }
    }
}

}  // namespace

extern "C" int bnn_dropout(bnn_ctx *ctx, int dtype, const void *x, int64_t ldx, const void *residual, int64_t ldr, void *y, int64_t ldy,
                           int64_t rows, int64_t cols, double p, uint64_t seed, uint64_t offset) {
    const int size = bnn_real_size(dtype);
    if (!size || !bnn_real_dim(rows) || !bnn_real_dim(cols) || !(p >= 0.0 && p <= 1.0)) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(x, ldx, rows, cols, size)) return st;
    if (int st = bnn_check_real_opt(residual, ldr, rows, cols, size)) return st;
    if (int st = bnn_check_real(y, ldy, rows, cols, size)) return st;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    DropArgs a{};
    a.x = x; a.residual = residual; a.y = y;
    a.ldx = ldx; a.ldr = ldr; a.ldy = ldy; a.rows = rows; a.cols = cols;
    const double words = std::rint(p * 4294967296.0);
    a.drop_all = words >= 4294967296.0;
    a.thr = a.drop_all ? 0xffffffffu : (uint32_t)words;
    a.scale = a.drop_all ? 0.0f : (float)(1.0 / (1.0 - p));
    a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32); a.o0 = (uint32_t)offset; a.o1 = (uint32_t)(offset >> 32);
    if (rows == 1 || (ldx == cols && ldy == cols && (!residual || ldr == cols))) { a.cols = rows * cols; a.rows = 1; }   // one long row
    a.vec = (a.rows == 1 || a.cols % 8 == 0) && bnn_rows16(x, ldx, a.rows, size) && bnn_rows16(y, ldy, a.rows, size) &&
            (!residual || bnn_rows16(residual, ldr, a.rows, size));
    const int64_t blocks = (rows * cols + 2047) / 2048;
    if (blocks > BNN_REAL_MAX) return BNN_ERR_INVALID_ARG;
    const dim3 grid((unsigned)blocks);
    auto kernel = dtype == BNN_F32 ? k_dropout<float> : dtype == BNN_F16 ? k_dropout<__half> : k_dropout<__nv_bfloat16>;
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, grid, dim3(256), 0, ctx->stream, a));
    return bnn_check_launch(ctx);
}
