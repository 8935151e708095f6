// Norms around a block fused with the block's gate and the residual scale, forward and backward.
//
// Mathematics, per row of D values:
//   p = post ? Norm(b) w_post + c_post : b;   s = alpha x + gate p;   n = Norm(s) w_pre + c_pre
// backward, with unit rows bh = (b - mean_b) r_b, sh = (s - mean_s) r_s (recomputed from x, b and the saved statistics) and
//   back(e; u, r) = r (e - u mean(e u) - mean(e))      (the last term for layer norm only)
//   T = ds + back(dn w_pre; sh, r_s);  dx = alpha T;  dp = gate T;  db = post ? back(dp w_post; bh, r_b) : dp
//   dw_pre = sum dn sh, dc_pre = sum dn, dw_post = sum dp bh, dc_post = sum dp, dgate = sum T p       (sums over rows)
// Bound: HBM.  Forward moves 4 rows of D (reads x, b, writes s, n), backward 6 (reads x, b, ds, dn, writes dx, db).
//
// A row lives in the registers of one team of threads: every value is read once and written once.  Sums are float32;
// the variance is taken around the mean (two reductions), not as a difference of squares.
#include "bnn_real.cuh"
#include "bnn_internal.cuh"

namespace {

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
};

constexpr int PRE_W = 1, PRE_C = 2, POST_W = 4, POST_C = 8;

// Eight columns of one row per thread and slot.  VEC: eight neighbouring columns in 16-byte accesses; otherwise (odd pitches
// or widths) columns a team apart, so that neighbouring threads still read neighbouring elements.
template <bool VEC> __device__ __forceinline__ int column(int slot, int j, int tid, int team) {
    return VEC ? (slot * team + tid) * 8 + j : (slot * 8 + j) * team + tid;
}
template <typename T, bool VEC>
__device__ __forceinline__ void read_row(const T *row, int slot, int tid, int team, int D, float (&v)[8]) {
    if constexpr (VEC) {
        const int c = column<true>(slot, 0, tid, team);
        if (c < D) load8(row + c, v);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = column<false>(slot, j, tid, team);
            v[j] = c < D ? to_f32(row[c]) : 0.0f;
        }
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void write_row(T *row, int slot, int tid, int team, int D, const float (&v)[8]) {
    if constexpr (VEC) {
        const int c = column<true>(slot, 0, tid, team);
        if (c < D) store8(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = column<false>(slot, j, tid, team);
            if (c < D) row[c] = from_f32<T>(v[j]);
        }
    }
}
// VEC rows have D % 8 == 0: a slot is inside the row or outside as a whole.
template <bool VEC> __device__ __forceinline__ bool inside(int slot, int j, int tid, int team, int D) { return column<VEC>(slot, j, tid, team) < D; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sums of two values over the block, in a fixed order; `slots` alternates between two buffers so that one barrier per sum is enough.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 *buf, int warps, int warp, int lane) {
    a = warp_sum(a); b = warp_sum(b);
    if (warps == 1) return make_float2(a, b);
    if (lane == 0) buf[warp] = make_float2(a, b);
    __syncthreads();
    const float2 t = lane < warps ? buf[lane] : make_float2(0.0f, 0.0f);
    return make_float2(warp_sum(t.x), warp_sum(t.y));
}

template <typename T, int SLOTS, bool VEC>
__global__ void __launch_bounds__(1024) k_block_norm(const NormArgs p) {
    __shared__ float2 buf[4][32];
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = static_cast<const T *>(p.post_w), *pc = static_cast<const T *>(p.post_c);
    const T *nw = static_cast<const T *>(p.pre_w), *nc = static_cast<const T *>(p.pre_c);
    for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
        float s[SLOTS][8];
        {
            const T *x = static_cast<const T *>(p.x) + m * p.ldx;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                read_row<T, VEC>(x, i, tid, team, p.D, s[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[i][j] *= p.alpha;
            }
        }
        if (p.block) {
            const T *b = static_cast<const T *>(p.block) + m * p.ldb;
            const T *gate = p.gate ? static_cast<const T *>(p.gate) + (m / p.rows_per_gate) * p.ld_gate : nullptr;
            float v[SLOTS][8];
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) read_row<T, VEC>(b, i, tid, team, p.D, v[i]);
            if (p.post) {
                float mean = 0.0f;
                if (p.layer) {
                    float t = 0.0f;
#pragma unroll
                    for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) t += v[i][j];
                    mean = block_sum2(t, 0.0f, buf[0], warps, warp, lane).x * p.inv_d;
                }
                float q = 0.0f;
#pragma unroll
                for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[i][j] = inside<VEC>(i, j, tid, team, p.D) ? v[i][j] - mean : 0.0f;
                        q += v[i][j] * v[i][j];
                    }
                const float r = 1.0f / sqrtf(block_sum2(q, 0.0f, buf[1], warps, warp, lane).x * p.inv_d + p.eps);
                if (p.stats && tid == 0) { p.stats[4 * m] = mean; p.stats[4 * m + 1] = r; }
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) {
                    float w[8], c[8];
                    if (pw) read_row<T, VEC>(pw, i, tid, team, p.D, w);
                    if (pc) read_row<T, VEC>(pc, i, tid, team, p.D, c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[i][j] *= r;
                        if (pw) v[i][j] *= w[j];
                        if (pc) v[i][j] += c[j];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                float g[8];
                if (gate) read_row<T, VEC>(gate, i, tid, team, p.D, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[i][j] += gate ? g[j] * v[i][j] : v[i][j];
            }
        }
        if (p.stream) {
            T *out = static_cast<T *>(p.stream) + m * p.lds;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) write_row<T, VEC>(out, i, tid, team, p.D, s[i]);
        }
        if (p.pre) {
            float mean = 0.0f;
            if (p.layer) {
                float t = 0.0f;
#pragma unroll
                for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) t += inside<VEC>(i, j, tid, team, p.D) ? s[i][j] : 0.0f;
                mean = block_sum2(t, 0.0f, buf[2], warps, warp, lane).x * p.inv_d;
            }
            float q = 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s[i][j] = inside<VEC>(i, j, tid, team, p.D) ? s[i][j] - mean : 0.0f;
                    q += s[i][j] * s[i][j];
                }
            const float r = 1.0f / sqrtf(block_sum2(q, 0.0f, buf[3], warps, warp, lane).x * p.inv_d + p.eps);
            if (p.stats && tid == 0) { p.stats[4 * m + 2] = mean; p.stats[4 * m + 3] = r; }
            if (p.normed) {
                T *out = static_cast<T *>(p.normed) + m * p.ldn;
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) {
                    float w[8], c[8];
                    if (nw) read_row<T, VEC>(nw, i, tid, team, p.D, w);
                    if (nc) read_row<T, VEC>(nc, i, tid, team, p.D, c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        s[i][j] *= r;
                        if (nw) s[i][j] *= w[j];
                        if (nc) s[i][j] += c[j];
                    }
                    write_row<T, VEC>(out, i, tid, team, p.D, s[i]);
                }
            }
        }
        if (warps > 1) __syncthreads();      // the next row reuses the buffers
    }
}

// A CTA takes whole units (a unit: chunk_rows rows that share one gate row), so every thread keeps the column sums of its own
// columns in registers from row to row: the four parameter sums for all its units, the gate's for one unit.
template <typename T, int SLOTS, bool VEC, int THREADS>
__global__ void __launch_bounds__(THREADS) k_block_norm_backward(const NormArgs p) {
    __shared__ float2 buf[2][32];
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = static_cast<const T *>(p.post_w), *pc = static_cast<const T *>(p.post_c), *nw = static_cast<const T *>(p.pre_w);
    float sum_nw[SLOTS][8], sum_nc[SLOTS][8], sum_pw[SLOTS][8], sum_pc[SLOTS][8], sum_g[SLOTS][8];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) { sum_nw[i][j] = 0.0f; sum_nc[i][j] = 0.0f; sum_pw[i][j] = 0.0f; sum_pc[i][j] = 0.0f; }
    for (int64_t unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const int64_t group = unit / p.chunks, chunk = unit - group * p.chunks;
        const int64_t first = group * p.rows_per_gate + chunk * p.chunk_rows;
        const int64_t group_end = (group + 1) * p.rows_per_gate < p.M ? (group + 1) * p.rows_per_gate : p.M;
        const int64_t end = first + p.chunk_rows < group_end ? first + p.chunk_rows : group_end;
        const T *gate = p.gate ? static_cast<const T *>(p.gate) + group * p.ld_gate : nullptr;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum_g[i][j] = 0.0f;
        for (int64_t m = first; m < end; ++m) {
            float e[SLOTS][8], u[SLOTS][8], bh[SLOTS][8], dn[SLOTS][8];      // dn w_pre; unit rows of the stream and of the block; dn
            float4 st = make_float4(0.0f, 1.0f, 0.0f, 1.0f);
            if (p.stats) st = make_float4(p.stats[4 * m], p.stats[4 * m + 1], p.stats[4 * m + 2], p.stats[4 * m + 3]);
            const float mean_b = p.post ? st.x : 0.0f, r_b = p.post ? st.y : 1.0f;
            float a1 = 0.0f, a2 = 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                if (p.block) {
                    read_row<T, VEC>(static_cast<const T *>(p.block) + m * p.ldb, i, tid, team, p.D, bh[i]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) bh[i][j] = (bh[i][j] - mean_b) * r_b;
                }
                if (p.pre && p.dn) {
                    read_row<T, VEC>(static_cast<const T *>(p.x) + m * p.ldx, i, tid, team, p.D, u[i]);
                    read_row<T, VEC>(static_cast<const T *>(p.dn) + m * p.lddn, i, tid, team, p.D, dn[i]);
                    float w[8], c[8], g[8], v[8];
                    if (pw) read_row<T, VEC>(pw, i, tid, team, p.D, w);
                    if (pc) read_row<T, VEC>(pc, i, tid, team, p.D, c);
                    if (gate) read_row<T, VEC>(gate, i, tid, team, p.D, g);
                    if (nw) read_row<T, VEC>(nw, i, tid, team, p.D, v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float q = 0.0f;
                        if (p.block) {
                            q = bh[i][j];
                            if (p.post && pw) q *= w[j];
                            if (p.post && pc) q += c[j];
                            if (gate) q *= g[j];
                        }
                        const bool in = inside<VEC>(i, j, tid, team, p.D);
                        u[i][j] = in ? (p.alpha * u[i][j] + q - st.z) * st.w : 0.0f;
                        e[i][j] = nw ? dn[i][j] * v[j] : dn[i][j];
                        a1 += e[i][j] * u[i][j];
                        a2 += e[i][j];
                        sum_nw[i][j] += dn[i][j] * u[i][j];
                        sum_nc[i][j] += dn[i][j];
                    }
                }
            }
            if (p.pre && p.dn) {
                const float2 t = block_sum2(a1, p.layer ? a2 : 0.0f, buf[0], warps, warp, lane);
                const float m1 = t.x * p.inv_d, m2 = t.y * p.inv_d;
#pragma unroll
                for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[i][j] = st.w * (e[i][j] - u[i][j] * m1 - m2);
            } else {
#pragma unroll
                for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[i][j] = 0.0f;
            }
            // u becomes T, e becomes dp, then its product with w_post
            float b1 = 0.0f, b2 = 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                if (p.ds) {
                    float d[8];
                    read_row<T, VEC>(static_cast<const T *>(p.ds) + m * p.ldds, i, tid, team, p.D, d);
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[i][j] += d[j];
                }
                if (p.dx) {
                    float d[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] = p.alpha * u[i][j];
                    write_row<T, VEC>(static_cast<T *>(p.dx) + m * p.lddx, i, tid, team, p.D, d);
                }
                if (p.block) {
                    float w[8], c[8], g[8];
                    if (pw) read_row<T, VEC>(pw, i, tid, team, p.D, w);
                    if (pc) read_row<T, VEC>(pc, i, tid, team, p.D, c);
                    if (gate) read_row<T, VEC>(gate, i, tid, team, p.D, g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool in = inside<VEC>(i, j, tid, team, p.D);
                        const float tj = in ? u[i][j] : 0.0f;
                        const float unit_b = in ? bh[i][j] : 0.0f;
                        float q = unit_b;
                        if (p.post && pw) q *= w[j];
                        if (p.post && pc) q += c[j];
                        sum_g[i][j] += tj * q;
                        const float dp = gate ? g[j] * tj : tj;
                        e[i][j] = dp;
                        bh[i][j] = unit_b;
                        if (p.post) {
                            sum_pw[i][j] += dp * unit_b;
                            sum_pc[i][j] += dp;
                            e[i][j] = pw ? dp * w[j] : dp;
                            b1 += e[i][j] * unit_b;
                            b2 += e[i][j];
                        }
                    }
                }
            }
            if (p.block && p.db) {
                float m1 = 0.0f, m2 = 0.0f;
                if (p.post) {
                    const float2 t = block_sum2(b1, p.layer ? b2 : 0.0f, buf[1], warps, warp, lane);
                    m1 = t.x * p.inv_d; m2 = t.y * p.inv_d;
                }
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) {
                    float d[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] = p.post ? r_b * (e[i][j] - bh[i][j] * m1 - m2) : e[i][j];
                    write_row<T, VEC>(static_cast<T *>(p.db) + m * p.lddb, i, tid, team, p.D, d);
                }
            }
            if (warps > 1) __syncthreads();
        }
        if (p.dgate) {
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                if (p.chunks == 1) write_row<T, VEC>(static_cast<T *>(p.dgate) + group * p.ld_dgate, i, tid, team, p.D, sum_g[i]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int c = column<VEC>(i, j, tid, team);
                        if (c < p.D) p.part_gate[unit * p.D + c] = sum_g[i][j];
                    }
                }
            }
        }
    }
    float *part = p.part + (int64_t)blockIdx.x * 4 * p.D;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = column<VEC>(i, j, tid, team);
            if (c >= p.D) continue;
            if (p.want & PRE_W) part[c] = sum_nw[i][j];
            if (p.want & PRE_C) part[p.D + c] = sum_nc[i][j];
            if (p.want & POST_W) part[2 * p.D + c] = sum_pw[i][j];
            if (p.want & POST_C) part[3 * p.D + c] = sum_pc[i][j];
        }
}

// Joins partial column sums in the order of their index: out[o][c] = sum_i part[(o * count + i) * pitch + c].
struct JoinArgs {
    const float *part[5];
    void *out[5];
    int64_t pitch[5], count[5], ldo[5];
    int outs[5];             // rows of out (gate rows; 1 for the parameters)
    int D;
};
template <typename T>
__global__ void __launch_bounds__(256) k_join_columns(const JoinArgs p) {
    __shared__ float sum[8][33];
    const int which = blockIdx.y, cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
    if (!p.out[which]) return;
    const int c = blockIdx.x * 32 + cx;
    for (int64_t o = blockIdx.z; o < p.outs[which]; o += gridDim.z) {
        float t = 0.0f;
        if (c < p.D)
            for (int64_t i = ry; i < p.count[which]; i += 8) t += p.part[which][(o * p.count[which] + i) * p.pitch[which] + c];
        sum[ry][cx] = t;
        __syncthreads();
        if (ry == 0 && c < p.D) {
            t = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += sum[k][cx];
            static_cast<T *>(p.out[which])[o * p.ldo[which] + c] = from_f32<T>(t);
        }
        __syncthreads();
    }
}

int launch_join(bnn_ctx *ctx, int dtype, const JoinArgs &j, int sums) {
    const int outs = j.outs[sums - 1];
    const dim3 grid((unsigned)((j.D + 31) / 32), (unsigned)sums, (unsigned)(outs > 1 ? (outs < 1024 ? outs : 1024) : 1));
    if (dtype == BNN_F32) k_join_columns<float><<<grid, 256, 0, ctx->stream>>>(j);
    else if (dtype == BNN_F16) k_join_columns<__half><<<grid, 256, 0, ctx->stream>>>(j);
    else k_join_columns<__nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(j);
    return bnn_check_launch(ctx);
}

constexpr int NORM_MAX_D = 32768;

int check_norm(const bnn_block_norm_desc *n, int64_t M) {
    if (!n || !bnn_real_size(n->dtype) || (n->kind != BNN_NORM_RMS && n->kind != BNN_NORM_LAYER)) return BNN_ERR_INVALID_ARG;
    if (n->D < 1 || n->D > NORM_MAX_D || !bnn_real_dim(M) || !(n->eps >= 0.0f)) return BNN_ERR_INVALID_ARG;
    if ((n->post != 0 && n->post != 1) || (n->pre != 0 && n->pre != 1)) return BNN_ERR_INVALID_ARG;
    if (n->gate && n->rows_per_gate < 1) return BNN_ERR_INVALID_ARG;
    const int size = bnn_real_size(n->dtype);
    const void *vectors[] = {n->post_weight, n->post_shift, n->pre_weight, n->pre_shift};
    for (const void *v : vectors)
        if (int st = bnn_check_real_opt(v, n->D, 1, n->D, size)) return st;
    const int64_t gates = n->gate ? (M + n->rows_per_gate - 1) / n->rows_per_gate : 0;
    return bnn_check_real_opt(n->gate, n->ld_gate, gates, n->D, size);
}
NormArgs norm_args(const bnn_block_norm_desc *n, int64_t M) {
    NormArgs a{};
    a.M = M; a.D = (int)n->D; a.eps = n->eps; a.alpha = n->alpha; a.inv_d = 1.0f / (float)n->D;
    a.layer = n->kind == BNN_NORM_LAYER; a.post = n->post; a.pre = n->pre;
    a.post_w = n->post ? n->post_weight : nullptr; a.post_c = n->post ? n->post_shift : nullptr;
    a.pre_w = n->pre ? n->pre_weight : nullptr; a.pre_c = n->pre ? n->pre_shift : nullptr;
    a.gate = n->gate; a.ld_gate = n->ld_gate;
    a.rows_per_gate = n->gate ? n->rows_per_gate : (M > 0 ? M : 1);
    return a;
}
// Whole 16-byte groups everywhere a row is touched.
bool norm_vec(const bnn_block_norm_desc *n, int64_t M, const NormArgs &a) {
    const int size = bnn_real_size(n->dtype);
    if (n->D % 8) return false;
    const void *vectors[] = {a.post_w, a.post_c, a.pre_w, a.pre_c};
    for (const void *v : vectors)
        if (!bnn_aligned16(v)) return false;
    const struct { const void *p; int64_t ld; } rows[] = {{a.x, a.ldx}, {a.block, a.ldb}, {a.stream, a.lds}, {a.normed, a.ldn}, {a.ds, a.ldds},
        {a.dn, a.lddn}, {a.dx, a.lddx}, {a.db, a.lddb}, {a.gate, a.ld_gate}, {a.dgate, a.ld_dgate}};
    for (const auto &r : rows)
        if (r.p && !bnn_rows16(r.p, r.ld, r.p == a.gate || r.p == a.dgate ? 2 : M, size)) return false;
    return true;
}

template <typename T, bool VEC> void launch_forward(bnn_ctx *ctx, const NormArgs &a) {
    const int groups = (a.D + 7) / 8;
    const int slots = groups <= 1024 ? 1 : groups <= 2048 ? 2 : 4;
    const int team = ((groups + slots - 1) / slots + 31) & ~31;
    const int64_t most = (int64_t)ctx->sm_count * 16;
    const dim3 grid((unsigned)(a.M < most ? a.M : most));
    if (slots == 1) k_block_norm<T, 1, VEC><<<grid, team, 0, ctx->stream>>>(a);
    else if (slots == 2) k_block_norm<T, 2, VEC><<<grid, team, 0, ctx->stream>>>(a);
    else k_block_norm<T, 4, VEC><<<grid, team, 0, ctx->stream>>>(a);
}
template <typename T, bool VEC> void launch_backward(bnn_ctx *ctx, const NormArgs &a, unsigned ctas) {
    const int groups = (a.D + 7) / 8;
    const int slots = groups <= 1024 ? 1 : groups <= 2048 ? 2 : 4;
    const int team = ((groups + slots - 1) / slots + 31) & ~31;
    if (slots == 1 && team <= 512) k_block_norm_backward<T, 1, VEC, 512><<<ctas, team, 0, ctx->stream>>>(a);
    else if (slots == 1) k_block_norm_backward<T, 1, VEC, 1024><<<ctas, team, 0, ctx->stream>>>(a);
    else if (slots == 2) k_block_norm_backward<T, 2, VEC, 1024><<<ctas, team, 0, ctx->stream>>>(a);
    else k_block_norm_backward<T, 4, VEC, 1024><<<ctas, team, 0, ctx->stream>>>(a);
}

// How the rows of the backward pass are divided: units of rows that share a gate row, at least `ctas` of them if the rows allow.
struct Division { int64_t groups, chunks, chunk_rows, units, ctas; };
Division divide_rows(int64_t M, int64_t rows_per_gate, int64_t ctas) {
    Division d{};
    d.groups = (M + rows_per_gate - 1) / rows_per_gate;
    const int64_t rows = rows_per_gate < M ? rows_per_gate : M;           // of one group
    d.chunks = d.groups >= ctas ? 1 : (ctas + d.groups - 1) / d.groups;
    if (d.chunks > rows) d.chunks = rows;
    d.chunk_rows = (rows + d.chunks - 1) / d.chunks;
    d.chunks = (rows + d.chunk_rows - 1) / d.chunk_rows;
    d.units = d.groups * d.chunks;
    d.ctas = d.units < ctas ? d.units : ctas;
    return d;
}
constexpr int64_t NORM_CTAS = 296;          // two per SM
size_t norm_part_floats(const Division &d, int64_t D) { return (size_t)d.ctas * 4 * D + (d.chunks > 1 ? (size_t)d.units * D : 0); }

}  // namespace

int bnn_join_columns(bnn_ctx *ctx, int dtype, const float *part, int64_t pitch, int64_t count, void *out, int64_t columns) {
    JoinArgs j{};
    j.D = (int)columns; j.part[0] = part; j.out[0] = out; j.pitch[0] = pitch; j.count[0] = count; j.outs[0] = 1;
    return launch_join(ctx, dtype, j, 1);
}

extern "C" int bnn_block_norm(bnn_ctx *ctx, const bnn_block_norm_desc *norm, const void *x, int64_t ldx, const void *block, int64_t ldb,
                              int64_t M, void *stream, int64_t lds, void *normed, int64_t ldn, float *stats) {
    if (int st = check_norm(norm, M)) return st;
    const int size = bnn_real_size(norm->dtype);
    if (!block && M > 0 && (norm->post || norm->gate)) return BNN_ERR_INVALID_ARG;
    if (normed && !norm->pre) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(x, ldx, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(block, ldb, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(stream, lds, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(normed, ldn, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(stats, 4, M, 4, 4)) return st;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (M == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    NormArgs a = norm_args(norm, M);
    a.x = x; a.ldx = ldx; a.block = block; a.ldb = ldb; a.stream = stream; a.lds = lds; a.normed = normed; a.ldn = ldn; a.stats = stats;
    const bool vec = norm_vec(norm, M, a);
    if (norm->dtype == BNN_F32) vec ? launch_forward<float, true>(ctx, a) : launch_forward<float, false>(ctx, a);
    else if (norm->dtype == BNN_F16) vec ? launch_forward<__half, true>(ctx, a) : launch_forward<__half, false>(ctx, a);
    else vec ? launch_forward<__nv_bfloat16, true>(ctx, a) : launch_forward<__nv_bfloat16, false>(ctx, a);
    return bnn_check_launch(ctx);
}

extern "C" size_t bnn_block_norm_workspace_bytes(const bnn_block_norm_desc *norm, int64_t M) {
    if (check_norm(norm, M) || M == 0) return 0;
    return (norm_part_floats(divide_rows(M, norm->gate ? norm->rows_per_gate : M, NORM_CTAS), norm->D) * 4 + 255) & ~size_t(255);
}

extern "C" int bnn_block_norm_backward(bnn_ctx *ctx, const bnn_block_norm_desc *norm, const void *dstream, int64_t ldds, const void *dnormed,
                                       int64_t lddn, const void *x, int64_t ldx, const void *block, int64_t ldb, const float *stats,
                                       int64_t M, const bnn_block_norm_grads *g) {
    if (int st = check_norm(norm, M)) return st;
    if (!g) return BNN_ERR_INVALID_ARG;
    const int size = bnn_real_size(norm->dtype);
    if (!block && M > 0 && (norm->post || norm->gate || g->dblock || g->dgate)) return BNN_ERR_INVALID_ARG;
    if ((g->dgate && !norm->gate) || ((g->dpost_weight || g->dpost_shift) && !norm->post) || ((g->dpre_weight || g->dpre_shift || dnormed) && !norm->pre))
        return BNN_ERR_INVALID_ARG;
    if (M > 0 && !stats && (norm->post || norm->pre)) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(x, ldx, M, norm->D, size)) return st;
    const struct { const void *p; int64_t ld; } rows[] = {{block, ldb}, {dstream, ldds}, {dnormed, lddn}, {g->dx, g->lddx}, {g->dblock, g->lddb}};
    for (const auto &r : rows)
        if (int st = bnn_check_real_opt(r.p, r.ld, M, norm->D, size)) return st;
    const void *vectors[] = {g->dpost_weight, g->dpost_shift, g->dpre_weight, g->dpre_shift};
    for (const void *v : vectors)
        if (int st = bnn_check_real_opt(v, norm->D, 1, norm->D, size)) return st;
    const int64_t gates = norm->gate ? (M + norm->rows_per_gate - 1) / norm->rows_per_gate : 0;
    if (int st = bnn_check_real_opt(g->dgate, g->ld_dgate, gates, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(stats, 4, M, 4, 4)) return st;
    if (!ctx) return BNN_ERR_INVALID_ARG;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    void *sums[] = {g->dpre_weight, g->dpre_shift, g->dpost_weight, g->dpost_shift};
    if (M == 0) {
        for (void *v : sums)
            if (v) BNN_CUDA_TRY(ctx, cudaMemsetAsync(v, 0, (size_t)norm->D * size, ctx->stream));
        return BNN_OK;
    }
    NormArgs a = norm_args(norm, M);
    a.x = x; a.ldx = ldx; a.block = block; a.ldb = ldb; a.stats = const_cast<float *>(stats);
    a.ds = dstream; a.ldds = ldds; a.dn = dnormed; a.lddn = lddn;
    a.dx = g->dx; a.lddx = g->lddx; a.db = g->dblock; a.lddb = g->lddb; a.dgate = g->dgate; a.ld_dgate = g->ld_dgate;
    for (int k = 0; k < 4; ++k) a.want |= sums[k] ? (1 << k) : 0;
    const Division d = divide_rows(M, a.rows_per_gate, NORM_CTAS);
    a.groups = d.groups; a.chunks = d.chunks; a.chunk_rows = d.chunk_rows; a.units = d.units;
    const bool joins = a.want || (a.dgate && d.chunks > 1);
    if (joins && (!ctx->ws || ctx->ws_bytes < norm_part_floats(d, norm->D) * 4)) return BNN_ERR_WORKSPACE;
    a.part = static_cast<float *>(ctx->ws);
    a.part_gate = a.part + (size_t)d.ctas * 4 * norm->D;
    const bool vec = norm_vec(norm, M, a);
    if (norm->dtype == BNN_F32) vec ? launch_backward<float, true>(ctx, a, (unsigned)d.ctas) : launch_backward<float, false>(ctx, a, (unsigned)d.ctas);
    else if (norm->dtype == BNN_F16) vec ? launch_backward<__half, true>(ctx, a, (unsigned)d.ctas) : launch_backward<__half, false>(ctx, a, (unsigned)d.ctas);
    else vec ? launch_backward<__nv_bfloat16, true>(ctx, a, (unsigned)d.ctas) : launch_backward<__nv_bfloat16, false>(ctx, a, (unsigned)d.ctas);
    if (int st = bnn_check_launch(ctx)) return st;
    if (!joins) return BNN_OK;
    JoinArgs j{};
    j.D = (int)norm->D;
    for (int k = 0; k < 4; ++k) {
        j.part[k] = a.part + k * norm->D; j.out[k] = sums[k]; j.pitch[k] = 4 * norm->D; j.count[k] = d.ctas; j.outs[k] = 1;
    }
    if (a.dgate && d.chunks > 1) {
        j.part[4] = a.part_gate; j.out[4] = a.dgate; j.pitch[4] = norm->D; j.count[4] = d.chunks; j.outs[4] = (int)d.groups; j.ldo[4] = a.ld_dgate;
    }
    return launch_join(ctx, norm->dtype, j, 5);
}
