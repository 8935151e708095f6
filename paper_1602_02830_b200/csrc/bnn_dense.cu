// Real-valued dense layer and gated projections, forward and backward.
//
//   linear:  z = x W^T + bias, y = residual + act(z);   dz = dy act'(z), dx = dz W, dW = dz^T x, dbias = sum dz
//   gated:   g = x Wg^T, u = x Wu^T, h = act(g) u;      dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x
//
// Every product is k_product with an epilogue; dz (dg, du) is rounded to 16 bits once, the operand type of the products that read it.
#include "bnn_real.cuh"
#include "bnn_internal.cuh"

namespace {

enum Epilogue { EPI_LINEAR, EPI_LINEAR_BACK, EPI_GATED, EPI_GATED_BACK };

struct Operand { const void *p; int64_t row, k; };        // element (i, k) at p[i * row + k * k]
struct ProductArgs {
    Operand a[2], b[2];      // EPI_GATED*: two products with one accumulator each; otherwise their sum (the second may be absent)
    int pairs;
    int64_t M, N, K;
    const void *bias;
    const void *add; int64_t ld_add;      // EPI_LINEAR: residual; *_BACK: the gradient dy / dh
    void *out[2]; int64_t ldo;
    float *pre; int64_t ldp;
    int act;
};

template <typename T, int EPI>
__global__ void __launch_bounds__(256) k_product(const ProductArgs p) {
    constexpr int ACCS = (EPI == EPI_GATED || EPI == EPI_GATED_BACK) ? 2 : 1;
    __shared__ float sa[16][65], sb[16][65];
    float acc[ACCS][4][4] = {};
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t m0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        if (pair >= p.pairs) break;
        const T *A = static_cast<const T *>(p.a[pair].p), *B = static_cast<const T *>(p.b[pair].p);
        for (int64_t k0 = 0; k0 < p.K; k0 += 16) {
            for (int i = threadIdx.x; i < 1024; i += 256) {
                const int r = i >> 4, k = i & 15;
                sa[k][r] = (m0 + r < p.M && k0 + k < p.K) ? to_f32(A[(m0 + r) * p.a[pair].row + (k0 + k) * p.a[pair].k]) : 0.0f;
                sb[k][r] = (n0 + r < p.N && k0 + k < p.K) ? to_f32(B[(n0 + r) * p.b[pair].row + (k0 + k) * p.b[pair].k]) : 0.0f;
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[ACCS == 2 ? pair : 0][i][j] += sa[k][ty * 4 + i] * sb[k][tx * 4 + j];
            __syncthreads();
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
            if (m >= p.M || n >= p.N) continue;
            float z = acc[0][i][j], value;
            if constexpr (ACCS == 1) {
                if (p.bias) z += to_f32(static_cast<const T *>(p.bias)[n]);
                T *out = static_cast<T *>(p.out[0]) + m * p.ldo + n;
                if constexpr (EPI == EPI_LINEAR) {
                    if (p.pre) p.pre[m * p.ldp + n] = z;
                    value = act_value(p.act, z);
                    if (p.add) value += to_f32(static_cast<const T *>(p.add)[m * p.ld_add + n]);
                } else {
                    value = to_f32(static_cast<const T *>(p.add)[m * p.ld_add + n]) * act_slope(p.act, z, z);
                }
                *out = from_f32<T>(value);
            } else {
                const float u = acc[ACCS - 1][i][j];
                if constexpr (EPI == EPI_GATED) {
                    if (p.pre) { p.pre[m * p.ldp + n] = z; p.pre[(p.M + m) * p.ldp + n] = u; }
                    static_cast<T *>(p.out[0])[m * p.ldo + n] = from_f32<T>(act_value(p.act, z) * u);
                } else {
                    const float d = to_f32(static_cast<const T *>(p.add)[m * p.ld_add + n]);
                    const float slope = act_slope(p.act, z, value);
                    static_cast<T *>(p.out[0])[m * p.ldo + n] = from_f32<T>(d * u * slope);
                    static_cast<T *>(p.out[1])[m * p.ldo + n] = from_f32<T>(d * value);
                }
            }
        }
}

template <int EPI> int product(bnn_ctx *ctx, int dtype, const ProductArgs &a) {
    if (a.M == 0 || a.N == 0) return BNN_OK;
    const dim3 grid((unsigned)((a.N + 63) / 64), (unsigned)((a.M + 63) / 64));
    if (dtype == BNN_F16) k_product<__half, EPI><<<grid, 256, 0, ctx->stream>>>(a);
    else k_product<__nv_bfloat16, EPI><<<grid, 256, 0, ctx->stream>>>(a);
    return bnn_check_launch(ctx);
}

// dz = dy act'(pre) and/or the partial column sums of dz: a block takes 256 columns (8 per thread) of one chunk of rows, eight
// rows at a time.  Without `pre` dz is dy itself and only the sums are taken.
struct SlopeArgs {
    const void *dy; int64_t lddy;
    const float *pre; int64_t ldp;
    void *dz; int64_t lddz;
    float *part;                       // [chunk][N] or NULL
    int64_t M, N, chunk_rows;
    int act, vec;                      // vec: rows of dy, pre and dz in 16-byte groups, N % 8 == 0
};
template <typename T>
__global__ void __launch_bounds__(256) k_act_backward(const SlopeArgs p) {
    __shared__ float sums[8][256 + 8];
    const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
    const int64_t c0 = (int64_t)blockIdx.x * 256 + cx * 8;
    const int64_t first = (int64_t)blockIdx.y * p.chunk_rows, end = first + p.chunk_rows < p.M ? first + p.chunk_rows : p.M;
    const T *dy = static_cast<const T *>(p.dy);
    T *dz = static_cast<T *>(p.dz);
    float s[8] = {};
    for (int64_t m = first + ry; m < end; m += 8) {
        if (c0 >= p.N) break;
        float d[8], z[8];
        if (p.vec) {
            load8(dy + m * p.lddy + c0, d);
            if (p.pre) load8(p.pre + m * p.ldp + c0, z);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[j] = c0 + j < p.N ? to_f32(dy[m * p.lddy + c0 + j]) : 0.0f;
                z[j] = p.pre && c0 + j < p.N ? p.pre[m * p.ldp + c0 + j] : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float value;
            if (p.pre && (p.vec || c0 + j < p.N)) d[j] *= act_slope(p.act, z[j], value);
            s[j] += d[j];
        }
        if (dz) {
            if (p.vec) store8(dz + m * p.lddz + c0, d);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c0 + j < p.N) dz[m * p.lddz + c0 + j] = from_f32<T>(d[j]);
            }
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[ry][cx * 8 + j] = s[j];
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c < p.N) {
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += sums[k][threadIdx.x];
        p.part[(int64_t)blockIdx.y * p.N + c] = t;
    }
}

// dg = dh u act'(g), du = dh act(g) from the kept g and u: one thread per 8 columns.
struct GatedSlopeArgs {
    const void *dh; int64_t lddh;
    const float *pre; int64_t ldp;
    void *dg, *du; int64_t ldd;
    int64_t M, N;
    int act, vec;
};
template <typename T>
__global__ void __launch_bounds__(256) k_gated_slopes(const GatedSlopeArgs p) {
    const int64_t c0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (c0 >= p.N) return;
    for (int64_t m = blockIdx.y; m < p.M; m += gridDim.y) {
        const T *dh = static_cast<const T *>(p.dh) + m * p.lddh + c0;
        const float *g = p.pre + m * p.ldp + c0, *u = p.pre + (p.M + m) * p.ldp + c0;
        T *dg = static_cast<T *>(p.dg) + m * p.ldd + c0, *du = static_cast<T *>(p.du) + m * p.ldd + c0;
        if (p.vec) {
            float d[8], a[8], b[8];
            load8(dh, d); load8(g, a); load8(u, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float value;
                const float slope = act_slope(p.act, a[j], value);
                a[j] = d[j] * b[j] * slope;
                b[j] = d[j] * value;
            }
            store8(dg, a); store8(du, b);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (c0 + j >= p.N) break;
                float value;
                const float d = to_f32(dh[j]), slope = act_slope(p.act, g[j], value);
                dg[j] = from_f32<T>(d * u[j] * slope);
                du[j] = from_f32<T>(d * value);
            }
        }
    }
}

int64_t pitch16(int64_t n) { return (n + 7) & ~int64_t(7); }            // 16-bit rows of whole 16-byte groups
size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

// Rows per chunk of the column sums: about four blocks per SM, at least eight rows each.
int64_t sum_chunk_rows(int64_t M, int64_t N) {
    const int64_t blocks_n = (N + 255) / 256, want = 592 / blocks_n + 1;
    const int64_t rows = (M + want - 1) / want;
    return (rows + 7) & ~int64_t(7);
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
// Scratch of the backward passes: dz (or dg and du), then the partial column sums of the bias gradient.
size_t dz_bytes(int64_t M, int64_t N) { return round256((size_t)M * pitch16(N) * 2); }

}  // namespace

extern "C" size_t bnn_linear_workspace_bytes(const bnn_linear_desc *l, int64_t M, int backward, int aligned) {
    if (check_linear(l, M) || M == 0 || l->N == 0) return 0;
    (void)aligned;
    if (!backward) return 0;
    return (l->act == BNN_ACT_NONE ? 0 : dz_bytes(M, l->N)) + (l->bias ? round256((size_t)sum_chunks(M, l->N) * l->N * 4) : 0);
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
    ProductArgs a{};
    a.a[0] = {x, ldx, 1}; a.b[0] = {l->W, l->ldw, 1}; a.pairs = 1;
    a.M = M; a.N = l->N; a.K = l->K;
    a.bias = l->bias; a.add = residual; a.ld_add = ldr; a.out[0] = y; a.ldo = ldy; a.pre = pre; a.ldp = ldp; a.act = l->act;
    return product<EPI_LINEAR>(ctx, l->dtype, a);
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
    const bool slopes = l->act != BNN_ACT_NONE && M > 0 && l->N > 0;
    const bool sums = dbias && M > 0 && l->N > 0;
    const size_t need = (slopes ? dz_bytes(M, l->N) : 0) + (sums ? round256((size_t)sum_chunks(M, l->N) * l->N * 4) : 0);
    if (need && (!ctx->ws || ctx->ws_bytes < need)) return BNN_ERR_WORKSPACE;
    uint8_t *ws = static_cast<uint8_t *>(ctx->ws);
    const void *dz = dy;
    int64_t lddz = lddy;
    float *part = sums ? reinterpret_cast<float *>(ws + (slopes ? dz_bytes(M, l->N) : 0)) : nullptr;
    if (slopes) {
        dz = ws; lddz = pitch16(l->N);
        if (!pre) {
            ProductArgs a{};
            a.a[0] = {x, ldx, 1}; a.b[0] = {l->W, l->ldw, 1}; a.pairs = 1;
            a.M = M; a.N = l->N; a.K = l->K;
            a.bias = l->bias; a.add = dy; a.ld_add = lddy; a.out[0] = ws; a.ldo = lddz; a.act = l->act;
            if (int st = product<EPI_LINEAR_BACK>(ctx, l->dtype, a)) return st;
        }
    }
    if ((slopes && pre) || sums) {
        SlopeArgs s{};
        const bool kept = slopes && pre;
        s.dy = kept ? dy : dz; s.lddy = kept ? lddy : lddz;
        s.pre = kept ? pre : nullptr; s.ldp = ldp;
        s.dz = kept ? ws : nullptr; s.lddz = lddz;
        s.part = part; s.M = M; s.N = l->N; s.chunk_rows = sum_chunk_rows(M, l->N); s.act = l->act;
        s.vec = l->N % 8 == 0 && bnn_rows16(s.dy, s.lddy, M, 2) && (!kept || bnn_rows16(pre, ldp, M, 4));
        const dim3 grid((unsigned)((l->N + 255) / 256), (unsigned)sum_chunks(M, l->N));
        if (l->dtype == BNN_F16) k_act_backward<__half><<<grid, 256, 0, ctx->stream>>>(s);
        else k_act_backward<__nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(s);
        if (int st = bnn_check_launch(ctx)) return st;
        if (sums)
            if (int st = bnn_join_columns(ctx, l->dtype, part, l->N, sum_chunks(M, l->N), dbias, l->N)) return st;
    }
    if (dx) {
        ProductArgs a{};
        a.a[0] = {dz, lddz, 1}; a.b[0] = {l->W, 1, l->ldw}; a.pairs = 1;
        a.M = M; a.N = l->K; a.K = l->N; a.out[0] = dx; a.ldo = lddx;
        if (int st = product<EPI_LINEAR>(ctx, l->dtype, a)) return st;
    }
    if (dW) {
        ProductArgs a{};
        a.a[0] = {dz, 1, lddz}; a.b[0] = {x, 1, ldx}; a.pairs = 1;
        a.M = l->N; a.N = l->K; a.K = M; a.out[0] = dW; a.ldo = lddw;
        if (int st = product<EPI_LINEAR>(ctx, l->dtype, a)) return st;
    }
    return BNN_OK;
}

extern "C" size_t bnn_gated_workspace_bytes(const bnn_gated_desc *l, int64_t M, int backward, int aligned) {
    if (check_gated(l, M) || M == 0 || l->N == 0) return 0;
    (void)aligned;
    return backward ? 2 * dz_bytes(M, l->N) : 0;
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
    ProductArgs a{};
    a.a[0] = a.a[1] = {x, ldx, 1}; a.b[0] = {l->Wg, l->ldg, 1}; a.b[1] = {l->Wu, l->ldu, 1}; a.pairs = 2;
    a.M = M; a.N = l->N; a.K = l->K;
    a.out[0] = h; a.ldo = ldh; a.pre = pre; a.ldp = ldp; a.act = l->act;
    return product<EPI_GATED>(ctx, l->dtype, a);
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
    const size_t one = dz_bytes(M, l->N);
    if (one && (!ctx->ws || ctx->ws_bytes < 2 * one)) return BNN_ERR_WORKSPACE;
    uint8_t *dg = static_cast<uint8_t *>(ctx->ws), *du = dg + one;
    const int64_t ldd = pitch16(l->N);
    if (one && pre) {
        GatedSlopeArgs s{};
        s.dh = dh; s.lddh = lddh; s.pre = pre; s.ldp = ldp; s.dg = dg; s.du = du; s.ldd = ldd; s.M = M; s.N = l->N; s.act = l->act;
        s.vec = l->N % 8 == 0 && bnn_rows16(dh, lddh, M, 2) && bnn_rows16(pre, ldp, 2 * M, 4);
        const dim3 grid((unsigned)((l->N + 2047) / 2048), (unsigned)(M < 65535 ? M : 65535));
        if (l->dtype == BNN_F16) k_gated_slopes<__half><<<grid, 256, 0, ctx->stream>>>(s);
        else k_gated_slopes<__nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(s);
        if (int st = bnn_check_launch(ctx)) return st;
    } else if (one) {
        ProductArgs a{};
        a.a[0] = a.a[1] = {x, ldx, 1}; a.b[0] = {l->Wg, l->ldg, 1}; a.b[1] = {l->Wu, l->ldu, 1}; a.pairs = 2;
        a.M = M; a.N = l->N; a.K = l->K;
        a.add = dh; a.ld_add = lddh; a.out[0] = dg; a.out[1] = du; a.ldo = ldd; a.act = l->act;
        if (int st = product<EPI_GATED_BACK>(ctx, l->dtype, a)) return st;
    }
    if (dx) {
        ProductArgs a{};
        a.a[0] = {dg, ldd, 1}; a.b[0] = {l->Wg, 1, l->ldg}; a.a[1] = {du, ldd, 1}; a.b[1] = {l->Wu, 1, l->ldu}; a.pairs = 2;
        a.M = M; a.N = l->K; a.K = l->N; a.out[0] = dx; a.ldo = lddx;
        if (int st = product<EPI_LINEAR>(ctx, l->dtype, a)) return st;
    }
    void *dw[2] = {dWg, dWu};
    const int64_t ldw[2] = {lddg, lddu};
    for (int k = 0; k < 2; ++k) {
        if (!dw[k]) continue;
        ProductArgs a{};
        a.a[0] = {k ? du : dg, 1, ldd}; a.b[0] = {x, 1, ldx}; a.pairs = 1;
        a.M = l->N; a.N = l->K; a.K = M; a.out[0] = dw[k]; a.ldo = ldw[k];
        if (int st = product<EPI_LINEAR>(ctx, l->dtype, a)) return st;
    }
    return BNN_OK;
}
