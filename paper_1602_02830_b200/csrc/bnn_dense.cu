// Real-valued dense layer and gated projections, forward and backward.
//
//   linear:  z = x W^T + bias, y = residual + act(z);   dz = dy act'(z), dx = dz W, dW = dz^T x, dbias = sum dz
//   gated:   g = x Wg^T, u = x Wu^T, h = act(g) u;      dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x
//
// Every product is bnn_product with an epilogue; dz (dg, du) is rounded to 16 bits once, the operand type of the products that read it.
#include "bnn_internal.cuh"
#include "bnn_product.cuh"

namespace {

// d *= act'(z), eight at a time; the choice of the activation is made once.
template <int ACT> __device__ __forceinline__ void slopes8_of(const float (&z)[8], float (&d)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float value;
        d[j] *= act_slope(ACT, z[j], value);
    }
}
__device__ __forceinline__ void slopes8(int act, const float (&z)[8], float (&d)[8]) {
    switch (act) {
        case BNN_ACT_RELU: slopes8_of<BNN_ACT_RELU>(z, d); break;
        case BNN_ACT_GELU: slopes8_of<BNN_ACT_GELU>(z, d); break;
        case BNN_ACT_GELU_TANH: slopes8_of<BNN_ACT_GELU_TANH>(z, d); break;
        case BNN_ACT_SILU: slopes8_of<BNN_ACT_SILU>(z, d); break;
        case BNN_ACT_SIGMOID: slopes8_of<BNN_ACT_SIGMOID>(z, d); break;
        case BNN_ACT_HTANH: slopes8_of<BNN_ACT_HTANH>(z, d); break;
        default: break;
    }
}
// a = g, b = u, d = dh -> a = dg, b = du.
template <int ACT> __device__ __forceinline__ void gated8_of(const float (&d)[8], float (&a)[8], float (&b)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float value;
        const float slope = act_slope(ACT, a[j], value);
        a[j] = d[j] * b[j] * slope;
        b[j] = d[j] * value;
    }
}
__device__ __forceinline__ void gated8(int act, const float (&d)[8], float (&a)[8], float (&b)[8]) {
    switch (act) {
        case BNN_ACT_RELU: gated8_of<BNN_ACT_RELU>(d, a, b); break;
        case BNN_ACT_GELU: gated8_of<BNN_ACT_GELU>(d, a, b); break;
        case BNN_ACT_GELU_TANH: gated8_of<BNN_ACT_GELU_TANH>(d, a, b); break;
        case BNN_ACT_SILU: gated8_of<BNN_ACT_SILU>(d, a, b); break;
        case BNN_ACT_SIGMOID: gated8_of<BNN_ACT_SIGMOID>(d, a, b); break;
        case BNN_ACT_HTANH: gated8_of<BNN_ACT_HTANH>(d, a, b); break;
        default: gated8_of<BNN_ACT_NONE>(d, a, b); break;
    }
}

// Copies matrices whose rows are not whole 16-byte groups to ones whose rows are: what TMA can read.  Bound: HBM.  One thread per 16
// bytes written: it reads the one or two aligned 16-byte groups that hold them and shifts (single elements at the very ends of the
// matrix, where a group would reach outside).  The copied row's padding up to a whole group is written as zero.
struct RepitchArgs {
    const uint16_t *src[3];
    uint16_t *dst[3];
    int64_t ld[3], pitch[3], rows[3], cols[3];
    int64_t groups[3];            // per row
    int64_t first[4];             // first group of each matrix in the launch's numbering
    int count;
};
template <int WORD> __device__ __forceinline__ void shifted(const uint4 &a, const uint4 &b, uint32_t half, uint32_t (&w)[4]) {
    const uint32_t v[9] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, 0u};
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(v[k + WORD], v[k + WORD + 1], half);
}
__global__ void __launch_bounds__(256) k_repitch(const __grid_constant__ RepitchArgs p) {
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < p.first[p.count]; t += (int64_t)gridDim.x * 256) {
        int i = 0;
        while (i + 1 < p.count && t >= p.first[i + 1]) ++i;
        const int64_t at = t - p.first[i], gpr = p.groups[i];
        const int64_t m = p.first[p.count] <= 0xffffffffll ? (int64_t)((uint32_t)at / (uint32_t)gpr) : at / gpr, c = (at - m * gpr) * 8;
        const uint16_t *from = p.src[i] + m * p.ld[i] + c;
        const int n = (int)(p.cols[i] - c < 8 ? p.cols[i] - c : 8);
        const uintptr_t begin = reinterpret_cast<uintptr_t>(from), low = begin & ~uintptr_t(15), high = (begin + 2 * n - 1) & ~uintptr_t(15);
        const uintptr_t matrix = reinterpret_cast<uintptr_t>(p.src[i]), limit = reinterpret_cast<uintptr_t>(p.src[i] + (p.rows[i] - 1) * p.ld[i] + p.cols[i]);
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (low >= matrix && high + 16 <= limit) {
            const uint4 a = *reinterpret_cast<const uint4 *>(low), b = *reinterpret_cast<const uint4 *>(high);
            const uint32_t skip = (uint32_t)(begin - low) >> 1, half = (skip & 1) * 16;
            switch (skip >> 1) {                      // the same for a whole row
                case 0: shifted<0>(a, b, half, w); break;
                case 1: shifted<1>(a, b, half, w); break;
                case 2: shifted<2>(a, b, half, w); break;
                default: shifted<3>(a, b, half, w); break;
            }
            if (n < 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] &= 2 * k + 1 < n ? 0xffffffffu : 2 * k < n ? 0xffffu : 0u;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) w[k >> 1] |= (uint32_t)from[k] << (16 * (k & 1));
        }
        *reinterpret_cast<uint4 *>(p.dst[i] + m * p.pitch[i] + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// dz = dy act'(pre) and/or the column sums of dz: a block takes 64 columns (8 per thread) of one chunk of rows, 32 rows at a time.  With
// a single chunk the sums are the bias gradient itself, otherwise partial sums.  With `pre` the sums take dz
// before it is rounded; without, dz is given (dy itself, or recomputed and rounded) and only the sums are taken.  Bound: HBM.  8192 x 4096 bf16 with GELU and the sums 56 us = 4.8 TB/s (blocks in whole rounds of two per SM; a
// round more took 67), the sums alone 13 us = 5.2 TB/s; 4096 x 5393 (rows off the 16-byte rule) 69 us.  VEC: rows of dy, pre and dz in 16-byte groups, N % 8 == 0.
struct SlopeArgs {
    const void *dy; int64_t lddy;
    const float *pre; int64_t ldp;
    void *dz; int64_t lddz;
    float *part;                       // [chunk][N] or NULL
    void *sum;                         // N or NULL
    int64_t M, N, chunk_rows;
    int act;
};
constexpr int SUM_COLS = 64, SUM_ROWS = 32;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256, VEC ? 2 : 4) k_act_backward(const SlopeArgs p) {
    __shared__ float sums[SUM_ROWS][SUM_COLS + 1];
    const int cx = threadIdx.x & 7, ry = threadIdx.x >> 3;
    const int64_t c0 = (int64_t)blockIdx.x * SUM_COLS + cx * 8;
    const int64_t first = (int64_t)blockIdx.y * p.chunk_rows, end = first + p.chunk_rows < p.M ? first + p.chunk_rows : p.M;
    const T *dy = static_cast<const T *>(p.dy);
    T *dz = static_cast<T *>(p.dz);
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    float s[8] = {};
    if (VEC && c0 < p.N) {
        constexpr int AT_ONCE = 4;               // rows on their way
        for (int64_t m0 = first + ry; m0 < end; m0 += SUM_ROWS * AT_ONCE) {
            uint4 dw[AT_ONCE], zw[AT_ONCE][2];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int64_t m = m0 + i * SUM_ROWS;
                if (m >= end) break;
                dw[i] = *reinterpret_cast<const uint4 *>(dy + m * p.lddy + c0);
                if (p.pre) {
                    zw[i][0] = __ldcs(reinterpret_cast<const uint4 *>(p.pre + m * p.ldp + c0));
                    zw[i][1] = __ldcs(reinterpret_cast<const uint4 *>(p.pre + m * p.ldp + c0) + 1);
                }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int64_t m = m0 + i * SUM_ROWS;
                if (m >= end) break;
                float d[8], z[8];
                unpack8<T>(&dw[i], d);
                if (p.pre) {
                    unpack8<float>(zw[i], z);
                    slopes8(p.act, z, d);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += d[j];
                if (dz) store8(dz + m * p.lddz + c0, d);
            }
        }
    } else if (!VEC) {                         // a warp takes half of the columns and every fourth row, a lane one column of eight rows at a time
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int64_t c = (int64_t)blockIdx.x * SUM_COLS + 32 * (warp & 1) + lane;
        for (int64_t m0 = first + (warp >> 1); c < p.N && m0 < end; m0 += 32) {
            T bits[8];
            float d[8], z[8] = {};
#pragma unroll
            for (int j = 0; j < 8; ++j) {            // requests without a branch, which would wait for each: beyond the end the last row again
                const int64_t m = m0 + 4 * j < end ? m0 + 4 * j : end - 1;
                bits[j] = dy[m * p.lddy + c];
                if (p.pre) z[j] = p.pre[m * p.ldp + c];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = m0 + 4 * j < end ? to_f32(bits[j]) : 0.0f;
            if (p.pre) slopes8(p.act, z, d);
            T *to = dz + m0 * p.lddz + c;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[0] += d[j];
                if (dz && m0 + 4 * j < end) to[4 * j * p.lddz] = from_f32<T>(d[j]);
            }
        }
    }
    if (!p.part && !p.sum) return;
    if (VEC) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[ry][cx * 8 + j] = s[j];
    } else {
        sums[threadIdx.x >> 6][threadIdx.x & 63] = s[0];
    }
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * SUM_COLS + threadIdx.x;
    if (threadIdx.x < SUM_COLS && c < p.N) {
        float t = 0.0f;
        constexpr int rows = VEC ? SUM_ROWS : 4;
#pragma unroll
        for (int k = 0; k < rows; ++k) t += sums[k][threadIdx.x];
        if (p.sum) static_cast<T *>(p.sum)[c] = from_f32<T>(t);
        else p.part[(int64_t)blockIdx.y * p.N + c] = t;
    }
}

// dg = dh u act'(g), du = dh act(g) from the kept g and u: one thread per 8 columns, neighbouring ones or (rows that are not whole 16-byte
// groups) every eighth of 64, so that neighbouring lanes touch neighbouring elements.
struct GatedSlopeArgs {
    const void *dh; int64_t lddh;
    const float *pre; int64_t ldp;
    void *dg, *du; int64_t ldd;
    int64_t M, N;
    uint32_t groups;                   // threads of a row
    int act, vec;
};
template <typename T>
__global__ void __launch_bounds__(256) k_gated_slopes(const GatedSlopeArgs p) {
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    const int64_t total = p.M * p.groups, stride = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += stride) {
        const int64_t m = total <= 0xffffffffll ? (int64_t)((uint32_t)i / p.groups) : i / p.groups, at = i - m * p.groups;
        const int64_t c0 = p.vec ? at * 8 : at / 8 * 64 + at % 8;
        const T *dh = static_cast<const T *>(p.dh) + m * p.lddh + c0;
        const float *g = p.pre + m * p.ldp + c0, *u = p.pre + (p.M + m) * p.ldp + c0;
        T *dg = static_cast<T *>(p.dg) + m * p.ldd + c0, *du = static_cast<T *>(p.du) + m * p.ldd + c0;
        float d[8], a[8], b[8];
        if (p.vec) { load8(dh, d); load8(g, a); load8(u, b); }
        else {
            T bits[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {            // requests without a branch, which would wait for each: beyond N the last column again
                const int64_t c = c0 + 8 * j < p.N ? 8 * j : p.N - 1 - c0;
                bits[j] = dh[c]; a[j] = g[c]; b[j] = u[c];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = to_f32(bits[j]);
        }
        gated8(p.act, d, a, b);
        if (p.vec) { store8(dg, a); store8(du, b); }
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + 8 * j < p.N) { dg[8 * j] = from_f32<T>(a[j]); du[8 * j] = from_f32<T>(b[j]); }
        }
    }
}

// Pitch of 16-bit rows in the scratch: whole 128-byte lines, what one row of a TMA box reads (1000 x 1008 x 4104 with rows of 8208 bytes
// 21 us, of whole lines 17).
int64_t pitch16(int64_t n) { return (n + 63) & ~int64_t(63); }
size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

// Rows per chunk of the column sums: about four blocks per SM, whole rounds of two, while there are at most 296 blocks of columns (18944 outputs); above, one
// chunk, whose last round may be nearly empty (2048 rows: 18944 outputs 70 us, 22016 103, 37888 118).  Up to 256 rows one chunk as well, which needs no
// second kernel to join the partial sums.
int64_t sum_chunk_rows(int64_t M, int64_t N) {
    if (M <= 256) return M;
    const int64_t blocks_n = (N + SUM_COLS - 1) / SUM_COLS, want = blocks_n < 592 ? 592 / blocks_n : 1;
    const int64_t rows = (M + want - 1) / want;
    return (rows + SUM_ROWS - 1) / SUM_ROWS * SUM_ROWS;
}
int64_t sum_chunks(int64_t M, int64_t N) { const int64_t r = sum_chunk_rows(M, N); return (M + r - 1) / r; }

int check_linear(const bnn_linear_desc *l, int64_t M) {
    if (!l || (l->dtype != BNN_F16 && l->dtype != BNN_BF16) || !bnn_act_known(l->act)) return BNN_ERR_INVALID_ARG;
    if (!bnn_real_dim(l->K) || !bnn_real_dim(l->N) || !bnn_real_dim(M)) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(l->W, l->ldw, l->N, l->K, 2)) return st;
    return bnn_check_real_opt(l->bias, l->N, 1, l->N, 2);
}
int check_gated(const bnn_gated_desc *l, int64_t M) {
    if (!l || (l->dtype != BNN_F16 && l->dtype != BNN_BF16) || !bnn_act_known(l->act)) return BNN_ERR_INVALID_ARG;
    if (!bnn_real_dim(l->K) || !bnn_real_dim(l->N) || !bnn_real_dim(M)) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(l->Wg, l->ldg, l->N, l->K, 2)) return st;
    return bnn_check_real(l->Wu, l->ldu, l->N, l->K, 2);
}
size_t dz_bytes(int64_t M, int64_t N) { return round256((size_t)M * pitch16(N) * 2); }
size_t sums_bytes(int64_t M, int64_t N) { return M <= 256 ? 0 : round256((size_t)sum_chunks(M, N) * N * 4); }

// Scratch of one call, handed out in order.  What does not fit is noticed at the end (`ok`), before anything is launched.
struct Scratch {
    bnn_ctx *ctx;
    size_t used = 0;
    explicit Scratch(bnn_ctx *c) : ctx(c) {}
    uint8_t *take(size_t bytes) {
        uint8_t *p = static_cast<uint8_t *>(ctx->ws) + used;
        used += bytes;
        return p;
    }
    bool ok() const { return used == 0 || (ctx->ws && ctx->ws_bytes >= used); }
};
// Operands as TMA can read them: themselves, or copies in the scratch (made by `copy`, in one launch, once the scratch is known to suffice).
struct Readable {
    Scratch &scratch;
    RepitchArgs r{};
    explicit Readable(Scratch &s) : scratch(s) {}
    BnnOperand operator()(const void *p, int64_t ld, int64_t rows, int64_t cols) {
        if (rows == 0 || cols == 0 || bnn_rows16(p, ld, rows, 2)) return {p, ld};
        const int i = r.count++;
        r.src[i] = static_cast<const uint16_t *>(p); r.ld[i] = rows > 1 ? ld : cols; r.rows[i] = rows; r.cols[i] = cols;
        r.dst[i] = reinterpret_cast<uint16_t *>(scratch.take(dz_bytes(rows, cols))); r.pitch[i] = pitch16(cols);
        r.groups[i] = (cols + 7) / 8;
        r.first[i + 1] = r.first[i] + rows * r.groups[i];
        return {r.dst[i], r.pitch[i]};
    }
    int copy(bnn_ctx *ctx) {
        if (!r.count) return BNN_OK;
        const int64_t blocks = (r.first[r.count] + 255) / 256, most = 148 * 8 * 4;
        BNN_CUDA_TRY(ctx, bnn_launch_dependent(k_repitch, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, ctx->stream, r));
        return bnn_check_launch(ctx);
    }
};

// The gradients of a layer: in one launch, so that the tiles of all of them fill the GPU together, or some of them on the kernel for few
// rows.  The choice is made for all of them and then what is not wanted (out[0] NULL) is left out, so that a gradient has the same
// bits whatever is asked for beside it.
int gradients(bnn_ctx *ctx, int dtype, BnnProduct *g, int n) {
    if (n == 0) return BNN_OK;
    for (int i = 0; i < n; ++i) { g[i].dtype = dtype; g[i].epilogue = BNN_EPI_LINEAR; if (!g[i].pairs) g[i].pairs = 1; }
    bool few[3] = {};
    if (!bnn_product_apart(ctx, g, n, few)) few[0] = few[1] = few[2] = false;
    int kept = 0;
    for (int i = 0; i < n; ++i) {
        if (!g[i].out[0]) continue;
        g[i].kernel = few[i] ? BNN_FEW : BNN_PAIR;
        if (few[i]) { if (int st = bnn_product(ctx, g + i, 1)) return st; }
        else g[kept++] = g[i];
    }
    return kept ? bnn_product(ctx, g, kept) : BNN_OK;
}

}  // namespace

extern "C" size_t bnn_linear_workspace_bytes(const bnn_linear_desc *l, int64_t M, int backward, int aligned) {
    if (check_linear(l, M) || M == 0 || l->N == 0) return 0;
    size_t n = aligned ? 0 : dz_bytes(M, l->K) + dz_bytes(l->N, l->K);
    if (backward) n += (l->act == BNN_ACT_NONE ? (aligned ? 0 : dz_bytes(M, l->N)) : dz_bytes(M, l->N)) + (l->bias ? sums_bytes(M, l->N) : 0);
    return n;
}

extern "C" int bnn_linear(bnn_ctx *ctx, const bnn_linear_desc *l, const void *x, int64_t ldx, int64_t M, const void *residual, int64_t ldr,
                          void *y, int64_t ldy, float *pre, int64_t ldp) {
    if (int st = check_linear(l, M)) return st;
    if (int st = bnn_check_real(x, ldx, M, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(residual, ldr, M, l->N, 2)) return st;
    if (int st = bnn_check_real(y, ldy, M, l->N, 2)) return st;
    if (int st = bnn_check_real_opt(pre, ldp, M, l->N, 4)) return st;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (M == 0 || l->N == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    Scratch scratch(ctx);
    Readable readable(scratch);
    const BnnOperand rx = readable(x, ldx, M, l->K), rw = readable(l->W, l->ldw, l->N, l->K);
    if (!scratch.ok()) return BNN_ERR_WORKSPACE;
    if (int st = readable.copy(ctx)) return st;
    BnnProduct p{};
    p.dtype = l->dtype; p.epilogue = BNN_EPI_LINEAR; p.pairs = 1;
    p.a[0] = rx; p.b[0] = rw; p.M = M; p.N = l->N; p.K = l->K;
    p.bias = l->bias; p.add = residual; p.ld_add = ldr; p.out[0] = y; p.ldo[0] = ldy; p.pre = pre; p.ldp = ldp; p.act = l->act;
    return bnn_product(ctx, &p, 1);
}

extern "C" int bnn_linear_backward(bnn_ctx *ctx, const bnn_linear_desc *l, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                                   int64_t M, const float *pre, int64_t ldp, void *dx, int64_t lddx, void *dW, int64_t lddw, void *dbias) {
    if (int st = check_linear(l, M)) return st;
    if (int st = bnn_check_real(dy, lddy, M, l->N, 2)) return st;
    if (int st = bnn_check_real(x, ldx, M, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(pre, ldp, M, l->N, 4)) return st;
    if (int st = bnn_check_real_opt(dx, lddx, M, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(dW, lddw, l->N, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(dbias, l->N, 1, l->N, 2)) return st;
    if (dbias && !l->bias) return BNN_ERR_INVALID_ARG;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    if (dbias && M == 0 && l->N > 0) BNN_CUDA_TRY(ctx, cudaMemsetAsync(dbias, 0, (size_t)l->N * 2, ctx->stream));
    const bool some = M > 0 && l->N > 0, slopes = l->act != BNN_ACT_NONE && some, sums = dbias && some, again = slopes && !pre;
    const bool products = (dx && M > 0 && l->K > 0) || (dW && l->N > 0 && l->K > 0);
    if (!products && !sums) return BNN_OK;
    Scratch scratch(ctx);
    BnnOperand dz{dy, lddy};
    if (slopes) dz = {scratch.take(dz_bytes(M, l->N)), pitch16(l->N)};
    Readable readable(scratch);
    // an empty product reads neither operand, and bnn_linear_workspace_bytes counts no copies for it
    const BnnOperand rz = readable(dz.p, dz.ld, products && !slopes ? M : 0, l->N), rx = readable(x, ldx, some && (dW || again) ? M : 0, l->K),
                     rw = readable(l->W, l->ldw, some && (dx || again) ? l->N : 0, l->K);
    const int64_t chunks = sums ? sum_chunks(M, l->N) : 0;
    float *part = chunks > 1 ? reinterpret_cast<float *>(scratch.take(sums_bytes(M, l->N))) : nullptr;
    if (!scratch.ok()) return BNN_ERR_WORKSPACE;
    if (int st = readable.copy(ctx)) return st;
    BnnProduct p{};
    p.dtype = l->dtype; p.pairs = 1;
    if (again) {
        p.epilogue = BNN_EPI_LINEAR_BACK;
        p.a[0] = rx; p.b[0] = rw; p.M = M; p.N = l->N; p.K = l->K;
        p.bias = l->bias; p.add = dy; p.ld_add = lddy; p.out[0] = const_cast<void *>(dz.p); p.ldo[0] = dz.ld; p.act = l->act;
        if (int st = bnn_product(ctx, &p, 1)) return st;
    }
    const bool kept = slopes && pre;
    if (kept || sums) {
        SlopeArgs s{};
        s.dy = kept ? dy : dz.p; s.lddy = kept ? lddy : dz.ld;
        s.pre = kept ? pre : nullptr; s.ldp = ldp;
        s.dz = kept ? const_cast<void *>(dz.p) : nullptr; s.lddz = dz.ld;
        s.part = part; s.sum = chunks == 1 ? dbias : nullptr;
        s.M = M; s.N = l->N; s.chunk_rows = sum_chunk_rows(M, l->N); s.act = l->act;
        const bool vec = l->N % 8 == 0 && bnn_rows16(s.dy, s.lddy, M, 2) && (!kept || bnn_rows16(pre, ldp, M, 4));
        const dim3 grid((unsigned)((l->N + SUM_COLS - 1) / SUM_COLS), (unsigned)sum_chunks(M, l->N));
        auto kernel = l->dtype == BNN_F16 ? (vec ? k_act_backward<__half, true> : k_act_backward<__half, false>)
                                            : (vec ? k_act_backward<__nv_bfloat16, true> : k_act_backward<__nv_bfloat16, false>);
        BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, grid, dim3(256), 0, ctx->stream, s));
        if (int st = bnn_check_launch(ctx)) return st;
        if (part)
            if (int st = bnn_join_columns(ctx, l->dtype, part, l->N, chunks, dbias, l->N)) return st;
    }
    const BnnOperand z = slopes ? dz : rz;
    BnnProduct g[2] = {};
    int n = 0;
    if (M > 0 && l->K > 0) {
        BnnProduct &d = g[n++];
        d.a[0] = z; d.b[0] = rw; d.b_mn = 1;
        d.M = M; d.N = l->K; d.K = l->N; d.out[0] = dx; d.ldo[0] = lddx;
    }
    if (l->N > 0 && l->K > 0) {
        BnnProduct &d = g[n++];
        d.a[0] = z; d.b[0] = rx; d.a_mn = d.b_mn = 1;
        d.M = l->N; d.N = l->K; d.K = M; d.out[0] = dW; d.ldo[0] = lddw;
    }
    return gradients(ctx, l->dtype, g, n);
}

extern "C" size_t bnn_gated_workspace_bytes(const bnn_gated_desc *l, int64_t M, int backward, int aligned) {
    if (check_gated(l, M) || M == 0 || l->N == 0) return 0;
    return (aligned ? 0 : dz_bytes(M, l->K) + 2 * dz_bytes(l->N, l->K)) + (backward ? 2 * dz_bytes(M, l->N) : 0);
}

extern "C" int bnn_gated(bnn_ctx *ctx, const bnn_gated_desc *l, const void *x, int64_t ldx, int64_t M, void *h, int64_t ldh, float *pre,
                         int64_t ldp) {
    if (int st = check_gated(l, M)) return st;
    if (int st = bnn_check_real(x, ldx, M, l->K, 2)) return st;
    if (int st = bnn_check_real(h, ldh, M, l->N, 2)) return st;
    if (int st = bnn_check_real_opt(pre, ldp, 2 * M, l->N, 4)) return st;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (M == 0 || l->N == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    Scratch scratch(ctx);
    Readable readable(scratch);
    const BnnOperand rx = readable(x, ldx, M, l->K), rg = readable(l->Wg, l->ldg, l->N, l->K), ru = readable(l->Wu, l->ldu, l->N, l->K);
    if (!scratch.ok()) return BNN_ERR_WORKSPACE;
    if (int st = readable.copy(ctx)) return st;
    BnnProduct p{};
    p.dtype = l->dtype; p.epilogue = BNN_EPI_GATED; p.pairs = 1;
    p.a[0] = rx; p.b[0] = rg; p.b[1] = ru; p.M = M; p.N = l->N; p.K = l->K;
    p.out[0] = h; p.ldo[0] = ldh; p.pre = pre; p.ldp = ldp; p.act = l->act;
    return bnn_product(ctx, &p, 1);
}

extern "C" int bnn_gated_backward(bnn_ctx *ctx, const bnn_gated_desc *l, const void *dh, int64_t lddh, const void *x, int64_t ldx, int64_t M,
                                  const float *pre, int64_t ldp, void *dx, int64_t lddx, void *dWg, int64_t lddg, void *dWu, int64_t lddu) {
    if (int st = check_gated(l, M)) return st;
    if (int st = bnn_check_real(dh, lddh, M, l->N, 2)) return st;
    if (int st = bnn_check_real(x, ldx, M, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(pre, ldp, 2 * M, l->N, 4)) return st;
    if (int st = bnn_check_real_opt(dx, lddx, M, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(dWg, lddg, l->N, l->K, 2)) return st;
    if (int st = bnn_check_real_opt(dWu, lddu, l->N, l->K, 2)) return st;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    const bool some = M > 0 && l->N > 0, again = some && !pre;
    if (!(dx && M > 0 && l->K > 0) && !((dWg || dWu) && l->N > 0 && l->K > 0)) return BNN_OK;
    Scratch scratch(ctx);
    const int64_t ldd = pitch16(l->N);
    void *dg = scratch.take(dz_bytes(M, l->N)), *du = scratch.take(dz_bytes(M, l->N));
    Readable readable(scratch);
    const BnnOperand rx = readable(x, ldx, some && (dWg || dWu || again) ? M : 0, l->K), rg = readable(l->Wg, l->ldg, some && (dx || again) ? l->N : 0, l->K),
                     ru = readable(l->Wu, l->ldu, some && (dx || again) ? l->N : 0, l->K);     // an empty product reads no operand
    if (!scratch.ok()) return BNN_ERR_WORKSPACE;
    if (int st = readable.copy(ctx)) return st;
    BnnProduct p{};
    p.dtype = l->dtype; p.pairs = 1;
    if (again) {
        p.epilogue = BNN_EPI_GATED_BACK;
        p.a[0] = rx; p.b[0] = rg; p.b[1] = ru; p.M = M; p.N = l->N; p.K = l->K;
        p.add = dh; p.ld_add = lddh; p.out[0] = dg; p.out[1] = du; p.ldo[0] = p.ldo[1] = ldd; p.act = l->act;
        if (int st = bnn_product(ctx, &p, 1)) return st;
    } else if (some) {
        GatedSlopeArgs s{};
        s.dh = dh; s.lddh = lddh; s.pre = pre; s.ldp = ldp; s.dg = dg; s.du = du; s.ldd = ldd; s.M = M; s.N = l->N; s.act = l->act;
        s.vec = l->N % 8 == 0 && bnn_rows16(dh, lddh, M, 2) && bnn_rows16(pre, ldp, 2 * M, 4);
        s.groups = (uint32_t)(s.vec ? l->N / 8 : (l->N + 63) / 64 * 8);
        const int64_t blocks = (M * s.groups + 255) / 256, most = 8 * 148;
        auto kernel = l->dtype == BNN_F16 ? k_gated_slopes<__half> : k_gated_slopes<__nv_bfloat16>;
        BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, ctx->stream, s));
        if (int st = bnn_check_launch(ctx)) return st;
    }
    BnnProduct g[3] = {};
    int n = 0;
    if (M > 0 && l->K > 0) {
        BnnProduct &d = g[n++];
        d.a[0] = {dg, ldd}; d.a[1] = {du, ldd}; d.b[0] = rg; d.b[1] = ru; d.b_mn = 1; d.pairs = 2;
        d.M = M; d.N = l->K; d.K = l->N; d.out[0] = dx; d.ldo[0] = lddx;
    }
    void *const dw[2] = {dWg, dWu};
    const int64_t ldw[2] = {lddg, lddu};
    for (int k = 0; k < 2; ++k) {
        if (l->N == 0 || l->K == 0) continue;
        BnnProduct &d = g[n++];
        d.a[0] = {k ? du : dg, ldd}; d.b[0] = rx; d.a_mn = d.b_mn = 1;
        d.M = l->N; d.N = l->K; d.K = M; d.out[0] = dw[k]; d.ldo[0] = ldw[k];
    }
    return gradients(ctx, l->dtype, g, n);
}
