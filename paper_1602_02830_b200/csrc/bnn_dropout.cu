// Dropout whose mask is never stored.  y = residual + (kept ? x / (1 - p) : 0); the mask is a pure function of
// (rows, cols, seed, offset), so the backward pass is the same call on dy and recomputes it.
//
// Mathematics: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds
//   (c0, c1, c2, c3) -> (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)),  keys advanced by Weyl constants,
// give four 32-bit words per counter; word e % 4 at counter e / 4 decides element e.
// Bound: HBM (2 elements moved per element, 3 with a residual), with the integer pipes close behind: the generator costs 18 wide
// multiplies and about as many three-input logic operations per four elements.  Measured, bf16: 16384 x 4096 with a residual and the same again
// without one (the backward pass), 671 MB, 138 us = 4.9 TB/s; 333 x 1011 float32, both passes, 15.5 us, which is the two calls' launches.
// Sixteen elements a thread: four independent chains of multiplies cover each other's latency.
#include "bnn_real.cuh"
#include <cmath>

namespace {

constexpr uint32_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u, W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;

struct DropArgs {
    const void *x, *residual;
    void *y;
    int64_t ldx, ldr, ldy, rows, cols;
    int64_t first, total;     // elements of this launch: first .. total - 1 (one value of the counter's high word)
    uint32_t thr;             // kept when the word is >= thr
    float scale;
    uint32_t key0[10], key1[10];
    uint32_t first2, second0, second2, second3;      // what rounds 1 and 2 make of the counter's other three words, see philox
    int vec;                  // every group of 8 elements lies in one row and on 16-byte boundaries
};

// The counter's words 1 .. 3 (high word of the index, offset) are the same for the whole launch, so half of the products of the first
// two rounds are as well: the host makes them, and the round keys, once.
//   round 1: (c, c1, o0, o1) -> (hi(M1 o0) ^ c1 ^ k, lo(M1 o0), hi(M0 c) ^ first2, lo(M0 c))
//   round 2: (u0, u1, v, w)  -> (hi(M1 v) ^ second0, lo(M1 v), second2 ^ w, second3)
void philox_constants(DropArgs &a, uint32_t c1, uint32_t o0, uint32_t o1, uint32_t k0, uint32_t k1) {
    for (int r = 0; r < 10; ++r) { a.key0[r] = k0 + (uint32_t)r * W0; a.key1[r] = k1 + (uint32_t)r * W1; }
    const uint64_t b = (uint64_t)M1 * o0;
    const uint32_t u0 = (uint32_t)(b >> 32) ^ c1 ^ a.key0[0];
    const uint64_t n = (uint64_t)M0 * u0;
    a.first2 = o1 ^ a.key1[0];
    a.second0 = (uint32_t)b ^ a.key0[1];
    a.second2 = (uint32_t)(n >> 32) ^ a.key1[1];
    a.second3 = (uint32_t)n;
}
__device__ __forceinline__ void philox(const DropArgs &p, uint32_t c, uint32_t (&w)[4]) {
    const uint64_t a = (uint64_t)M0 * c, b = (uint64_t)M1 * ((uint32_t)(a >> 32) ^ p.first2);
    uint32_t c0 = (uint32_t)(b >> 32) ^ p.second0, c1 = (uint32_t)b, c2 = p.second2 ^ (uint32_t)a, c3 = p.second3;
#pragma unroll
    for (int r = 2; r < 10; ++r) {
        const uint64_t s = (uint64_t)M0 * c0, t = (uint64_t)M1 * c2;
        c0 = (uint32_t)(t >> 32) ^ c1 ^ p.key0[r];
        c2 = (uint32_t)(s >> 32) ^ c3 ^ p.key1[r];
        c1 = (uint32_t)t; c3 = (uint32_t)s;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// One thread per 16 consecutive elements (four counters).  The row is requested before the generator runs, which covers the wait.
constexpr int PER = 16;
template <typename T, bool ADD>
__global__ void __launch_bounds__(256) k_dropout(const __grid_constant__ DropArgs p) {
    constexpr int WORDS = PER * (int)sizeof(T) / 16;
    const int64_t e0 = p.first + ((int64_t)blockIdx.x * 256 + threadIdx.x) * PER;
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    if (e0 >= p.total) return;
    const T *x = static_cast<const T *>(p.x), *res = static_cast<const T *>(p.residual);
    T *y = static_cast<T *>(p.y);
    int64_t row = 0, col = e0;
    if (p.rows > 1) {
        row = p.total <= 0xffffffffll ? (int64_t)((uint32_t)e0 / (uint32_t)p.cols) : e0 / p.cols;
        col = e0 - row * p.cols;
    }
    const bool whole = p.vec && e0 + PER <= p.total;
    // the second half of the sixteen may begin the next row
    const int64_t row2 = whole && p.rows > 1 && col + 8 >= p.cols ? row + 1 : row, col2 = row2 > row ? 0 : col + 8;
    uint4 xw[WORDS], rw[WORDS];
    if (whole) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const bool half = i >= WORDS / 2;
            const int64_t r = half ? row2 : row, c = half ? col2 : col;
            const int at = half ? i - WORDS / 2 : i;
            xw[i] = __ldcs(reinterpret_cast<const uint4 *>(x + r * p.ldx + c) + at);
            if (ADD) rw[i] = __ldcs(reinterpret_cast<const uint4 *>(res + r * p.ldr + c) + at);
        }
    }
    uint32_t word[PER / 4][4];
    const uint32_t c = (uint32_t)((uint64_t)e0 / 4);
#pragma unroll
    for (int i = 0; i < PER / 4; ++i) philox(p, c + i, word[i]);
    if (whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8], r[8];
            unpack8<T>(xw + h * WORDS / 2, v);
            if (ADD) unpack8<T>(rw + h * WORDS / 2, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = word[2 * h + j / 4][j % 4] >= p.thr ? v[j] * p.scale : 0.0f;
                if (ADD) v[j] += r[j];
            }
            store8(y + (h ? row2 : row) * p.ldy + (h ? col2 : col), v);
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (e0 + j < p.total) {
                float v = word[j / 4][j % 4] >= p.thr ? to_f32(x[row * p.ldx + col]) * p.scale : 0.0f;
                if (ADD) v += to_f32(res[row * p.ldr + col]);
                y[row * p.ldy + col] = from_f32<T>(v);
                if (++col == p.cols) { col = 0; ++row; }
            }
        }
    }
}

template <typename T> int launch(bnn_ctx *ctx, const DropArgs &a) {
    const unsigned blocks = (unsigned)((a.total - a.first + 256 * PER - 1) / (256 * PER));
    auto kernel = a.residual ? k_dropout<T, true> : k_dropout<T, false>;
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, dim3(blocks), dim3(256), 0, ctx->stream, a));
    return bnn_check_launch(ctx);
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
    const double words = std::rint(p * 4294967296.0);
    if (words >= 4294967296.0) {          // everything dropped: y is the residual, or zero
        const size_t width = (size_t)cols * size, pitch = (size_t)(rows > 1 ? ldy : cols) * size;
        if (!residual) BNN_CUDA_TRY(ctx, cudaMemset2DAsync(y, pitch, 0, width, (size_t)rows, ctx->stream));
        else if (residual != y)
            BNN_CUDA_TRY(ctx, cudaMemcpy2DAsync(y, pitch, residual, (size_t)(rows > 1 ? ldr : cols) * size, width, (size_t)rows,
                                                cudaMemcpyDeviceToDevice, ctx->stream));
        return BNN_OK;
    }
    DropArgs a{};
    a.x = x; a.residual = residual; a.y = y;
    a.ldx = ldx; a.ldr = ldr; a.ldy = ldy; a.rows = rows; a.cols = cols;
    a.thr = (uint32_t)words;
    a.scale = (float)(1.0 / (1.0 - p));
    if (rows == 1 || (ldx == cols && ldy == cols && (!residual || ldr == cols))) { a.cols = rows * cols; a.rows = 1; }   // one long row
    a.vec = (a.rows == 1 || a.cols % 8 == 0) && bnn_rows16(x, ldx, a.rows, size) && bnn_rows16(y, ldy, a.rows, size) &&
            (!residual || bnn_rows16(residual, ldr, a.rows, size));
    const int64_t total = rows * cols, span = int64_t(1) << 34;      // elements that share the high word of the counter
    for (int64_t first = 0; first < total; first += span) {
        a.first = first;
        a.total = first + span < total ? first + span : total;
        philox_constants(a, (uint32_t)(first >> 34), (uint32_t)offset, (uint32_t)(offset >> 32), (uint32_t)seed, (uint32_t)(seed >> 32));
        const int st = dtype == BNN_F32 ? launch<float>(ctx, a) : dtype == BNN_F16 ? launch<__half>(ctx, a) : launch<__nv_bfloat16>(ctx, a);
        if (st) return st;
    }
    return BNN_OK;
}
