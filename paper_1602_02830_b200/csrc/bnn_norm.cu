// Norms around a block fused with the block's gate and the residual scale, forward and backward.
//
// Mathematics, per row of D values:
//   p = post ? Norm(b) w_post + c_post : b;   s = alpha x + gate p;   n = Norm(s) w_pre + c_pre
// backward, with unit rows bh = (b - mean_b) r_b, sh = (s - mean_s) r_s (recomputed from x, b and the saved statistics) and
//   back(e; u, r) = r (e - u mean(e u) - mean(e))      (the last term for layer norm only)
//   T = ds + back(dn w_pre; sh, r_s);  dx = alpha T;  dp = gate T;  db = post ? back(dp w_post; bh, r_b) : dp
//   dw_pre = sum dn sh, dc_pre = sum dn, dw_post = sum dp bh, dc_post = sum dp, dgate = sum T p       (sums over rows)
// Bound: HBM.  Forward moves 4 rows of D (reads x, b, writes s, n), backward 6 (reads x, b, ds, dn, writes dx, db).  Measured, RMS norms:
// 4096 x 4096 bf16 forward 23.6 us = 5.7 TB/s, backward 39.5 us = 5.1 TB/s; float32 51 us = 5.2 TB/s and 116 us = 3.5 TB/s (one CTA of 512
// threads per SM: registers); layer norm bf16 32 and 65 us; rows off the 16-byte rule (4097 columns, bf16) 93 and 175 us.
//
// A row lives in the registers of one team of threads: every value is read once and written once.  Sums are float32;
// the variance is taken around the mean (two reductions), not as a difference of squares.
#include "bnn_norm.cuh"
#include "bnn_internal.cuh"
#include "bnn_mx.cuh"
#include <mutex>

namespace {
using namespace bnn_norm;

constexpr int PRE_W = 1, PRE_C = 2, POST_W = 4, POST_C = 8;

// Sum over the block in a fixed order.  One barrier each: successive sums use different buffers.
__device__ __forceinline__ float block_sum(float a, float *buf, int warps, int warp, int lane) {
    a = warp_sum(a);
    if (warps == 1) return a;
    if (lane == 0) buf[warp] = a;
    __syncthreads();
    return warp_sum(lane < warps ? buf[lane] : 0.0f);
}
// N = 4 or 8 sums over the block at once, in a fixed order, with one barrier.  While several sums are left, half of them go to the
// partner lane at every exchange, so N sums cost N + log2(32 / N) - 1 shuffles a warp instead of 5 N.
template <int N> __device__ __forceinline__ void block_sums(float (&v)[N], float *buf, int warps, int warp, int lane) {
    constexpr int G = 32 / N;                       // lanes that end up with the same sum: lane / G
#pragma unroll
    for (int o = 16, n = N; n > 1; o >>= 1, n >>= 1) {
#pragma unroll
        for (int k = 0; k < n / 2; ++k) {
            const bool up = lane & o;
            const float give = up ? v[k] : v[k + n / 2], keep = up ? v[k + n / 2] : v[k];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    float t = v[0];
#pragma unroll
    for (int o = G / 2; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (warps > 1) {
        const int sum = lane / G, sub = lane - sum * G;
        if (sub == 0) buf[warp * N + sum] = t;
        __syncthreads();
        t = 0.0f;
        for (int w = sub; w < warps; w += G) t += buf[w * N + sum];
#pragma unroll
        for (int o = G / 2; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, t, k * G);
}

// One row per CTA: both rows are requested before anything is computed from them.
// PLAIN: BNN_NORM_RMS without shifts, with a block, both outputs wanted.  Columns beyond D read as zero, which adds nothing to the sums of squares; around a mean
// (layer norm) they have to be left out.
template <typename T, int SLOTS, bool VEC> __device__ __forceinline__ void plain_row(const NormArgs &p, int64_t m, float (&buf)[4][32]) {
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = static_cast<const T *>(p.post_w), *nw = static_cast<const T *>(p.pre_w);
    // everything is there and nothing is optional inside the loops: weights that are not given are ones
    Eight<T> rx[SLOTS], rb[SLOTS];
    const T *X = static_cast<const T *>(p.x) + m * p.ldx, *B = static_cast<const T *>(p.block) + m * p.ldb;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) { rx[i] = read8<T, VEC>(X, i, tid, team, p.D); rb[i] = read8<T, VEC>(B, i, tid, team, p.D); }
    const T *gate = p.gate ? static_cast<const T *>(p.gate) + (m / p.rows_per_gate) * p.ld_gate : nullptr;
    float r = 1.0f, q = 0.0f;
    if (p.post) {
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) q += rb[i][j] * rb[i][j];
        r = 1.0f / sqrtf(block_sum(q, buf[1], warps, warp, lane) * p.inv_d + p.eps);
    }
    float s[SLOTS][8];
    q = 0.0f;
    T *out = static_cast<T *>(p.stream) + m * p.lds;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        Eight<T> w, g;
        w.fill(1.0f); g.fill(1.0f);
        if (pw) w = read8<T, VEC>(pw, i, tid, team, p.D);
        if (gate) g = read8<T, VEC>(gate, i, tid, team, p.D);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[i][j] = p.alpha * rx[i][j] + rb[i][j] * r * (w[j] * g[j]);
            q += s[i][j] * s[i][j];
        }
        write8<T, VEC>(out, i, tid, team, p.D, s[i]);
    }
    const float r_s = 1.0f / sqrtf(block_sum(q, buf[3], warps, warp, lane) * p.inv_d + p.eps);
    if (p.stats && tid == 0) { p.stats[4 * m] = 0.0f; p.stats[4 * m + 1] = r; p.stats[4 * m + 2] = 0.0f; p.stats[4 * m + 3] = r_s; }
    out = static_cast<T *>(p.normed) + m * p.ldn;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        Eight<T> w;
        w.fill(1.0f);
        if (nw) w = read8<T, VEC>(nw, i, tid, team, p.D);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] *= r_s * w[j];
        write8<T, VEC>(out, i, tid, team, p.D, s[i]);
    }
}
template <typename T, int SLOTS, bool VEC> __device__ __forceinline__ void any_row(const NormArgs &p, int64_t m, float (&buf)[4][32]) {
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = static_cast<const T *>(p.post_w), *pc = static_cast<const T *>(p.post_c);
    const T *nw = static_cast<const T *>(p.pre_w), *nc = static_cast<const T *>(p.pre_c);
    const bool layer = p.layer;
    Eight<T> rx[SLOTS], rb[SLOTS];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        rx[i] = read8<T, VEC>(static_cast<const T *>(p.x) + m * p.ldx, i, tid, team, p.D);
        if (p.block) rb[i] = read8<T, VEC>(static_cast<const T *>(p.block) + m * p.ldb, i, tid, team, p.D);
    }
    const T *gate = p.gate ? static_cast<const T *>(p.gate) + (m / p.rows_per_gate) * p.ld_gate : nullptr;
    float mean = 0.0f, r = 1.0f;
    if (p.block && p.post) {
        if (layer) {
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) t += rb[i][j];
            mean = block_sum(t, buf[0], warps, warp, lane) * p.inv_d;
        }
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            if (VEC && column<VEC>(i, 0, tid, team) >= p.D) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = rb[i][j];
                v = VEC || column<VEC>(i, j, tid, team) < p.D ? v - mean : 0.0f;
                q += v * v;
            }
        }
        r = 1.0f / sqrtf(block_sum(q, buf[1], warps, warp, lane) * p.inv_d + p.eps);
        if (p.stats && tid == 0) { p.stats[4 * m] = mean; p.stats[4 * m + 1] = r; }
    }
    float s[SLOTS][8];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        float v[8];
        if (p.block) {
            Eight<T> w, c, g;
            if (pw) w = read8<T, VEC>(pw, i, tid, team, p.D);
            if (pc) c = read8<T, VEC>(pc, i, tid, team, p.D);
            if (gate) g = read8<T, VEC>(gate, i, tid, team, p.D);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (rb[i][j] - mean) * r;
            if (pw)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= w[j];
            if (pc)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += c[j];
            if (gate)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= g[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] = p.block ? p.alpha * rx[i][j] + v[j] : p.alpha * rx[i][j];
        if (p.stream) write8<T, VEC>(static_cast<T *>(p.stream) + m * p.lds, i, tid, team, p.D, s[i]);
    }
    if (!p.pre) return;
    mean = 0.0f;
    if (layer) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (column<VEC>(i, VEC ? 0 : j, tid, team) < p.D) t += s[i][j];
        mean = block_sum(t, buf[2], warps, warp, lane) * p.inv_d;
    }
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        if (VEC && column<VEC>(i, 0, tid, team) >= p.D) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = s[i][j];
            v = VEC || column<VEC>(i, j, tid, team) < p.D ? v - mean : 0.0f;
            q += v * v;
        }
    }
    r = 1.0f / sqrtf(block_sum(q, buf[3], warps, warp, lane) * p.inv_d + p.eps);
    if (p.stats && tid == 0) { p.stats[4 * m + 2] = mean; p.stats[4 * m + 3] = r; }
    if (!p.normed) return;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        Eight<T> w, c;
        if (nw) w = read8<T, VEC>(nw, i, tid, team, p.D);
        if (nc) c = read8<T, VEC>(nc, i, tid, team, p.D);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] = (s[i][j] - mean) * r;
        if (nw)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] *= w[j];
        if (nc)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] += c[j];
        write8<T, VEC>(static_cast<T *>(p.normed) + m * p.ldn, i, tid, team, p.D, s[i]);
    }
}
template <typename T, int SLOTS, int THREADS, bool VEC, bool PLAIN>
__global__ void __launch_bounds__(THREADS, THREADS <= 256 ? 3 : 1) k_block_norm(const NormArgs p) {
    __shared__ float buf[4][32];
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    if constexpr (PLAIN) plain_row<T, SLOTS, VEC>(p, blockIdx.x, buf);
    else any_row<T, SLOTS, VEC>(p, blockIdx.x, buf);
}

// A CTA takes whole units (a unit: chunk_rows rows that share one gate row), so every thread keeps the column sums of its own
// columns in registers from row to row.  STAGES > 0 (VEC): the rows ahead are on their way to shared memory by cp.async, each thread's
// sixteen bytes to its own place, so that no register waits for memory; otherwise a row is read when it is its turn.
// One reduction per row: with y = gate w_post bh and z = ds + r_s e, the row's T is z - r_s (m1 u + m2), linear in the means m1 = mean(e u) and
// m2 = mean(e) of the stream's norm, so the two sums that the block's norm needs, of T y and of T gate w_post, follow from sums that
// are taken together with those of e u and e.  Of the parameter sums only sum T bh (and sum T) is kept per unit: the gate's gradient is
// w_post times it, the post weight's the gate times it.
// PLAIN: no means and no shifts (BNN_NORM_RMS without shift vectors or their gradients), and all four inputs and both row gradients are there,
// so that nothing is optional inside the row loop.
// Sixteen bytes, or zeros without an access where `bytes` is 0.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <typename T, int SLOTS, int THREADS, int CTAS, bool VEC, bool PLAIN, int STAGES>
__global__ void __launch_bounds__(THREADS, CTAS) k_block_norm_backward(const NormArgs p) {
    constexpr int SUMS = PLAIN ? 4 : 8, PIECES = (int)sizeof(T) / 2;        // 16-byte pieces of eight values
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float buf[2][32 * SUMS];
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = static_cast<const T *>(p.post_w), *pc = PLAIN ? nullptr : static_cast<const T *>(p.post_c), *nw = static_cast<const T *>(p.pre_w);
    const T *X = static_cast<const T *>(p.x), *B = static_cast<const T *>(p.block), *S = static_cast<const T *>(p.ds), *N = static_cast<const T *>(p.dn);
    const bool inner = PLAIN || (p.pre && p.dn), has_b = PLAIN || B, has_s = PLAIN || S;
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    Eight<T> w_pre[SLOTS];
    float sum_nw[SLOTS][8], sum_nc[SLOTS][8];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        w_pre[i].fill(1.0f);
        if (nw) w_pre[i] = read8<T, VEC>(nw, i, tid, team, p.D);
#pragma unroll
        for (int j = 0; j < 8; ++j) { sum_nw[i][j] = 0.0f; sum_nc[i][j] = 0.0f; }
    }
    float *part = p.part + (int64_t)blockIdx.x * 4 * p.D;
    // this thread's place in a stage: [array][slot][piece], a team's width apart
    const uint32_t place = STAGES ? (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)tid * 16 : 0;
    const uint32_t step = (uint32_t)team * 16, stage_bytes = step * 4 * SLOTS * PIECES;
    uint32_t turn = 0;                     // rows done: alternates the buffers of the sums
    for (int64_t unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const int64_t group = unit / p.chunks, chunk = unit - group * p.chunks;
        const int64_t first = group * p.rows_per_gate + chunk * p.chunk_rows;
        const int64_t group_end = (group + 1) * p.rows_per_gate < p.M ? (group + 1) * p.rows_per_gate : p.M;
        const int64_t end = first + p.chunk_rows < group_end ? first + p.chunk_rows : group_end;
        // gate w_post (0 beyond D, which keeps those columns out of every sum), gate c_post, and what is summed over the unit
        float gw[SLOTS][8], gc[SLOTS][8], sum_tb[SLOTS][8], sum_t[SLOTS][8];
        auto parameters = [&](int i, Eight<T> &w, Eight<T> &c, Eight<T> &g) {
            w.fill(1.0f); c.fill(0.0f); g.fill(1.0f);
            if (pw) w = read8<T, VEC>(pw, i, tid, team, p.D);
            if (pc) c = read8<T, VEC>(pc, i, tid, team, p.D);
            if (p.gate) g = read8<T, VEC>(static_cast<const T *>(p.gate) + group * p.ld_gate, i, tid, team, p.D);
        };
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            Eight<T> w, c, g;
            parameters(i, w, c, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                gw[i][j] = column<VEC>(i, VEC ? 0 : j, tid, team) < p.D ? w[j] * g[j] : 0.0f;
                gc[i][j] = c[j] * g[j];
                sum_tb[i][j] = 0.0f; sum_t[i][j] = 0.0f;
            }
        }
        // a row's four arrays in the order block, x, dn, ds
        auto ahead = [&](int64_t m, uint32_t stage) {
            if (m < end) {
                const T *const rows[4] = {B + m * p.ldb, X + m * p.ldx, N + m * p.lddn, S + m * p.ldds};
                const bool has[4] = {has_b, inner, inner, has_s};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (!has[k]) continue;
#pragma unroll
                    for (int i = 0; i < SLOTS; ++i) {
                        const int c = column<VEC>(i, 0, tid, team);
#pragma unroll
                        for (int h = 0; h < PIECES; ++h)
                            copy16(place + stage * stage_bytes + ((k * SLOTS + i) * PIECES + h) * step,
                                   reinterpret_cast<const uint4 *>(rows[k] + (c < p.D ? c : 0)) + h, c < p.D ? 16u : 0u);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        auto arrived = [&](uint32_t stage, int k, int i) {
            Eight<T> e;                       // columns beyond D arrive as zeros
#pragma unroll
            for (int h = 0; h < PIECES; ++h)
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(e.w[4 * h]), "=r"(e.w[4 * h + 1]), "=r"(e.w[4 * h + 2]), "=r"(e.w[4 * h + 3])
                             : "r"(place + stage * stage_bytes + ((k * SLOTS + i) * PIECES + h) * step) : "memory");
            return e;
        };
        auto statistics = [&](int64_t m) {          // read a row ahead
            if (!p.stats || m >= end) return make_float4(0.0f, 1.0f, 0.0f, 1.0f);
            const float *at = p.stats + 4 * m;
            return make_float4(__ldg(at), __ldg(at + 1), __ldg(at + 2), __ldg(at + 3));
        };
        float4 next = statistics(first);
        uint32_t stage = 0, fill = 0;
        if (STAGES) {
#pragma unroll
            for (int k = 0; k < STAGES - 1; ++k) ahead(first + k, (uint32_t)k);
            fill = (uint32_t)(STAGES > 0 ? STAGES - 1 : 0);
        }
        for (int64_t m = first; m < end; ++m, turn ^= 1u) {
            const float4 st = next;
            next = statistics(m + 1);
            if (STAGES) {
                ahead(m + STAGES - 1, fill);
                fill = fill + 1 == STAGES ? 0 : fill + 1;
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES > 0 ? STAGES - 1 : 0) : "memory");
            }
            const float mean_b = p.post ? st.x : 0.0f, r_b = p.post ? st.y : 1.0f, mean_s = p.pre ? st.z : 0.0f, r_s = p.pre ? st.w : 1.0f;
            if (!STAGES && m + 1 < end) {              // the next row comes to L2: a 128-byte line per thread and array
                constexpr int LINE = 128 / (int)sizeof(T);
                if (tid * LINE < p.D) {
                    if (has_b) asm volatile("prefetch.global.L2 [%0];" ::"l"(B + (m + 1) * p.ldb + tid * LINE));
                    if (inner) {
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(X + (m + 1) * p.ldx + tid * LINE));
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(N + (m + 1) * p.lddn + tid * LINE));
                    }
                    if (has_s) asm volatile("prefetch.global.L2 [%0];" ::"l"(S + (m + 1) * p.ldds + tid * LINE));
                }
            }
            Eight<T> rb[SLOTS];
            float u[SLOTS][8], z[SLOTS][8], v[SUMS];
#pragma unroll
            for (int k = 0; k < SUMS; ++k) v[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                Eight<T> rx, rn, rs;
                if (!PLAIN) { rb[i].fill(0.0f); rx.fill(0.0f); rn.fill(0.0f); rs.fill(0.0f); }
                if (has_b) rb[i] = STAGES ? arrived(stage, 0, i) : read8<T, VEC>(B + m * p.ldb, i, tid, team, p.D);
                if (inner) {
                    rx = STAGES ? arrived(stage, 1, i) : read8<T, VEC>(X + m * p.ldx, i, tid, team, p.D);
                    rn = STAGES ? arrived(stage, 2, i) : read8<T, VEC>(N + m * p.lddn, i, tid, team, p.D);
                }
                if (has_s) rs = STAGES ? arrived(stage, 3, i) : read8<T, VEC>(S + m * p.ldds, i, tid, team, p.D);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float bh = PLAIN ? rb[i][j] * r_b : (rb[i][j] - mean_b) * r_b;
                    const float y = gw[i][j] * bh, d = rn[j], e = d * w_pre[i][j];
                    if (PLAIN) u[i][j] = (p.alpha * rx[j] + y) * r_s;
                    else u[i][j] = (p.alpha * rx[j] + y + gc[i][j] - mean_s) * r_s;
                    z[i][j] = rs[j] + r_s * e;
                    v[0] += e * u[i][j];
                    v[1] += y * z[i][j];
                    v[2] += y * u[i][j];
                    sum_nw[i][j] += d * u[i][j];
                    if (!PLAIN) {
                        sum_nc[i][j] += d;
                        v[3] += e;
                        v[SUMS - 4] += y;
                        v[SUMS - 3] += gw[i][j] * z[i][j];
                        v[SUMS - 2] += gw[i][j] * u[i][j];
                        v[SUMS - 1] += gw[i][j];
                    }
                }
            }
            if (STAGES) stage = stage + 1 == STAGES ? 0 : stage + 1;
            block_sums<SUMS>(v, buf[turn], warps, warp, lane);
            const float rm1 = inner ? r_s * (v[0] * p.inv_d) : 0.0f, rm2 = !PLAIN && inner && p.layer ? r_s * (v[3] * p.inv_d) : 0.0f;
            float b1 = v[1] - rm1 * v[2], b2 = 0.0f;
            if (!PLAIN) { b1 -= rm2 * v[SUMS - 4]; b2 = v[SUMS - 3] - rm1 * v[SUMS - 2] - rm2 * v[SUMS - 1]; }
            b1 = p.post ? r_b * (b1 * p.inv_d) : 0.0f;
            b2 = !PLAIN && p.post && p.layer ? r_b * (b2 * p.inv_d) : 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                float d[8], bh[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    bh[j] = PLAIN ? rb[i][j] * r_b : (rb[i][j] - mean_b) * r_b;
                    float t = z[i][j];
                    if (inner) t -= PLAIN ? rm1 * u[i][j] : rm1 * u[i][j] + rm2;
                    z[i][j] = t;
                    d[j] = p.alpha * t;
                    sum_tb[i][j] += t * bh[j];
                    if (!PLAIN) sum_t[i][j] += t;
                }
                if (PLAIN || p.dx) write8<T, VEC>(static_cast<T *>(p.dx) + m * p.lddx, i, tid, team, p.D, d);
                if (PLAIN || (B && p.db)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        d[j] = r_b * (gw[i][j] * z[i][j]);
                        if (PLAIN) d[j] -= b1 * bh[j];          // b1 = 0 without a post norm
                        else if (p.post) d[j] -= b1 * bh[j] + b2;
                    }
                    write8<T, VEC>(static_cast<T *>(p.db) + m * p.lddb, i, tid, team, p.D, d);
                }
            }
        }
        if (STAGES) asm volatile("cp.async.wait_group 0;" ::: "memory");
        // the unit's sums: the gate's gradient, and the post norm's parameters added to what earlier units of this CTA left
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            Eight<T> w, c, g;
            parameters(i, w, c, g);
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[j] = w[j] * sum_tb[i][j];
                if (!PLAIN) d[j] += c[j] * sum_t[i][j];
                const int at = column<VEC>(i, j, tid, team);
                if (at >= p.D) continue;
                if (p.want & POST_W) part[2 * p.D + at] = g[j] * sum_tb[i][j] + (unit == blockIdx.x ? 0.0f : part[2 * p.D + at]);
                if (!PLAIN && (p.want & POST_C)) part[3 * p.D + at] = g[j] * sum_t[i][j] + (unit == blockIdx.x ? 0.0f : part[3 * p.D + at]);
                if (p.dgate && p.chunks > 1) p.part_gate[unit * p.D + at] = d[j];
            }
            if (p.dgate && p.chunks == 1) write8<T, VEC>(static_cast<T *>(p.dgate) + group * p.ld_dgate, i, tid, team, p.D, d);
        }
    }
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = column<VEC>(i, j, tid, team);
            if (c >= p.D) continue;
            if (p.want & PRE_W) part[c] = sum_nw[i][j];
            if (!PLAIN && (p.want & PRE_C)) part[p.D + c] = sum_nc[i][j];
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
constexpr int JOIN_LANES = 8, JOIN_AHEAD = 16;      // threads per column; loads a thread has on their way
template <typename T>
__global__ void __launch_bounds__(32 * JOIN_LANES) k_join_columns(const JoinArgs p) {
    __shared__ float sum[JOIN_LANES][33];
    const int which = blockIdx.y, cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    if (!p.out[which]) return;
    const int c = blockIdx.x * 32 + cx;
    const int64_t count = p.count[which], pitch = p.pitch[which];
    for (int64_t o = blockIdx.z; o < p.outs[which]; o += gridDim.z) {
        float t = 0.0f;
        if (c < p.D) {
            const float *part = p.part[which] + o * count * pitch + c;
            for (int64_t i = ry; i < count; i += JOIN_LANES * JOIN_AHEAD) {
                float v[JOIN_AHEAD];
#pragma unroll
                for (int k = 0; k < JOIN_AHEAD; ++k) v[k] = i + k * JOIN_LANES < count ? part[(i + k * JOIN_LANES) * pitch] : 0.0f;
#pragma unroll
                for (int k = 0; k < JOIN_AHEAD; ++k) t += v[k];
            }
        }
        sum[ry][cx] = t;
        __syncthreads();
        if (ry == 0 && c < p.D) {
            t = 0.0f;
#pragma unroll
            for (int k = 0; k < JOIN_LANES; ++k) t += sum[k][cx];
            static_cast<T *>(p.out[which])[o * p.ldo[which] + c] = from_f32<T>(t);
        }
        __syncthreads();
    }
}

int launch_join(bnn_ctx *ctx, int dtype, const JoinArgs &j, int sums) {
    const int outs = j.outs[sums - 1];
    const dim3 grid((unsigned)((j.D + 31) / 32), (unsigned)sums, (unsigned)(outs > 1 ? (outs < 1024 ? outs : 1024) : 1));
    auto kernel = dtype == BNN_F32 ? k_join_columns<float> : dtype == BNN_F16 ? k_join_columns<__half> : k_join_columns<__nv_bfloat16>;
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, grid, dim3(32 * JOIN_LANES), 0, ctx->stream, j));
    return bnn_check_launch(ctx);
}

constexpr int NORM_MAX_D = 32768;

// Rows of the stream that share a gate row, and gate rows.  Any number from M on means one gate row: it is brought down to M, so that nothing
// computed from it overflows.
int64_t rows_per_gate(const bnn_block_norm_desc *n, int64_t M) {
    const int64_t most = M > 0 ? M : 1;
    return n->gate && n->rows_per_gate < most ? n->rows_per_gate : most;
}
int64_t gate_rows(const bnn_block_norm_desc *n, int64_t M) { return n->gate ? (M + rows_per_gate(n, M) - 1) / rows_per_gate(n, M) : 0; }
int check_norm(const bnn_block_norm_desc *n, int64_t M) {
    if (!n || !bnn_real_size(n->dtype) || (n->kind != BNN_NORM_RMS && n->kind != BNN_NORM_LAYER)) return BNN_ERR_INVALID_ARG;
    if (n->D < 1 || n->D > NORM_MAX_D || !bnn_real_dim(M) || !(n->eps >= 0.0f)) return BNN_ERR_INVALID_ARG;
    if ((n->post != 0 && n->post != 1) || (n->pre != 0 && n->pre != 1)) return BNN_ERR_INVALID_ARG;
    if (n->gate && n->rows_per_gate < 1) return BNN_ERR_INVALID_ARG;
    const int size = bnn_real_size(n->dtype);
    const void *vectors[] = {n->post_weight, n->post_shift, n->pre_weight, n->pre_shift};
    for (const void *v : vectors)
        if (int st = bnn_check_real_opt(v, n->D, 1, n->D, size)) return st;
    return bnn_check_real_opt(n->gate, n->ld_gate, gate_rows(n, M), n->D, size);
}
NormArgs norm_args(const bnn_block_norm_desc *n, int64_t M) {
    NormArgs a{};
    a.M = M; a.D = (int)n->D; a.eps = n->eps; a.alpha = n->alpha; a.inv_d = 1.0f / (float)n->D;
    a.layer = n->kind == BNN_NORM_LAYER; a.post = n->post; a.pre = n->pre;
    a.post_w = n->post ? n->post_weight : nullptr; a.post_c = n->post ? n->post_shift : nullptr;
    a.pre_w = n->pre ? n->pre_weight : nullptr; a.pre_c = n->pre ? n->pre_shift : nullptr;
    a.gate = n->gate; a.ld_gate = n->ld_gate;
    a.rows_per_gate = rows_per_gate(n, M);
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

// Teams.  Forward: many rows take four slots a thread (few warps per row, few barriers, many rows in flight); few rows one slot (the
// shortest chain).  Rows of single elements: one slot up to 2048 columns (1000 x 1011 float32, both passes: 41 us with four, 34 with one), then two and four,
// so that at most 256 threads wait at a barrier and several rows share an SM (4096 x 4097 bf16: 119 us with one, 93 with four).
template <typename T, bool VEC> int launch_forward(bnn_ctx *ctx, const NormArgs &a) {
    const int groups = (a.D + 7) / 8;
    const bool few = a.M <= 2 * ctx->sm_count || (!VEC && groups <= 256);
    const int slots = groups > 1024 ? 4 : (few || groups <= 32) ? 1 : groups <= (VEC ? 64 : 512) ? 2 : 4;
    const int team = ((groups + slots - 1) / slots + 31) & ~31;
    const dim3 grid((unsigned)a.M), block(team);
    const bool plain = VEC && !a.layer && !a.post_c && !a.pre_c && a.block && a.stream && a.pre && a.normed;
#define BNN_FORWARD(SLOTS, THREADS) BNN_CUDA_TRY(ctx, bnn_launch_dependent(plain ? k_block_norm<T, SLOTS, THREADS, VEC, VEC> : k_block_norm<T, SLOTS, THREADS, VEC, false>, \
                                                                           grid, block, 0, ctx->stream, a))
    if (slots == 1) BNN_FORWARD(1, 1024);
    else if (slots == 2) BNN_FORWARD(2, 256);
    else if (team <= 256) BNN_FORWARD(4, 256);
    else BNN_FORWARD(4, 1024);
#undef BNN_FORWARD
    return bnn_check_launch(ctx);
}
// Backward.  TWICE, 16-bit rows of 16-byte groups without means and shifts: two slots a thread (one below 257 columns), at most 256 threads
// up to 4096 columns, so that two CTAs share an SM and one computes while the other waits at its barrier.  ONCE, other rows of 16-byte
// groups: their state and float32 rows fill the registers of two slots, so one slot up to 4096 columns (4096 rows, layer norm, 1016
// columns of bf16: 29 us, 42 with two; RMS norm, 2048 columns of float32: 61 us, 69 with two).  ELEMENTS: one slot, more threads; single
// elements are not fetched ahead, and more warps cover the wait (1000 x 1011: 34 us for the whole step, 52 with two slots).
enum Rows { ELEMENTS, ONCE, TWICE, ROWS_KINDS };
int backward_slots(int64_t D, int rows) {
    if (D <= (rows == TWICE ? 256 : rows == ONCE ? 4096 : 8192)) return 1;
    return D <= 16384 ? 2 : 4;
}
int backward_team(int64_t D, int rows) {
    const int groups = (int)((D + 7) / 8), slots = backward_slots(D, rows);
    return ((groups + slots - 1) / slots + 31) & ~31;
}
Rows backward_rows(const NormArgs &a, int size, bool vec) { return !vec ? ELEMENTS : size == 4 || a.layer || a.post_c || a.pre_c ? ONCE : TWICE; }
// Shared memory past 48 KB has to be opted in to.  The setting belongs to the kernel and not to a call, and contexts of several host threads
// launch the same kernel at different widths: it is made once per device, for the widest team.
template <typename T, int SLOTS, int THREADS, int CTAS, bool VEC, bool PLAIN, int DEEP>
int launch_rows(bnn_ctx *ctx, const NormArgs &a, unsigned ctas, int team) {
    auto kernel = k_block_norm_backward<T, SLOTS, THREADS, CTAS, VEC, PLAIN, DEEP>;
    constexpr size_t PER_THREAD = (size_t)DEEP * 64 * SLOTS * (sizeof(T) / 2);
    if constexpr (PER_THREAD * THREADS > 40 * 1024) {     // with the kernel's own shared memory below the 48 KB that need no opting in
        static std::mutex lock;
        static bool ready[64];
        if (ctx->device < 0 || ctx->device >= 64) return BNN_ERR_INVALID_ARG;
        std::lock_guard<std::mutex> guard(lock);
        if (!ready[ctx->device]) BNN_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(PER_THREAD * THREADS)));
        ready[ctx->device] = true;
    }
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, dim3(ctas), dim3(team), PER_THREAD * team, ctx->stream, a));
    return bnn_check_launch(ctx);
}
template <typename T, bool VEC> int launch_backward(bnn_ctx *ctx, const NormArgs &a, unsigned ctas) {
    const Rows rows = backward_rows(a, (int)sizeof(T), VEC);
    const int slots = backward_slots(a.D, rows), team = backward_team(a.D, rows);
    const bool plain = VEC && !a.layer && !a.post_c && !(a.want & (PRE_C | POST_C)) && a.block && a.pre && a.dn && a.ds && a.dx && a.db;
    constexpr int STAGES = VEC ? 3 : 0, WIDE = VEC && sizeof(T) == 2 ? 2 : 0;      // rows of all four arrays that fit
#define BNN_BACKWARD(SLOTS, THREADS, CTAS, PLAIN, DEEP) launch_rows<T, SLOTS, THREADS, CTAS, VEC, PLAIN, DEEP>(ctx, a, ctas, team)
    if constexpr (VEC) {
        if (slots == 1) return plain ? BNN_BACKWARD(1, 512, 1, true, STAGES) : BNN_BACKWARD(1, 512, 1, false, STAGES);
        if constexpr (sizeof(T) == 2)
            if (team <= 256) return plain ? BNN_BACKWARD(2, 256, 2, true, STAGES) : BNN_BACKWARD(2, 256, 1, false, STAGES);
        if (team <= 512) return plain ? BNN_BACKWARD(2, 512, 1, true, WIDE) : BNN_BACKWARD(2, 512, 1, false, WIDE);
    } else if (slots == 1 && team <= 512) return BNN_BACKWARD(1, 512, 1, false, 0);
    else if (slots == 1) return BNN_BACKWARD(1, 1024, 1, false, 0);
    if (slots == 2) return BNN_BACKWARD(2, 1024, 1, false, 0);
    return BNN_BACKWARD(4, 1024, 1, false, 0);
#undef BNN_BACKWARD
}

// How the rows of the backward pass are divided: units of rows that share a gate row, at least `ctas` of them if the rows allow.
struct Division { int64_t groups, chunks, chunk_rows, units, ctas; };
Division divide_rows(int64_t M, int64_t rows, int64_t ctas) {             // rows of one group
    Division d{};
    d.groups = (M + rows - 1) / rows;
    d.chunks = d.groups >= ctas ? 1 : (ctas + d.groups - 1) / d.groups;
    if (d.chunks > rows) d.chunks = rows;
    d.chunk_rows = (rows + d.chunks - 1) / d.chunks;
    d.chunks = (rows + d.chunk_rows - 1) / d.chunk_rows;
    d.units = d.groups * d.chunks;
    d.ctas = d.units < ctas ? d.units : ctas;
    return d;
}
// CTAs of the backward pass: 512 threads per SM (their registers hold the column sums), at most sixteen CTAs; at least two rows
// each, or joining the partial sums takes longer than making them.
int64_t norm_ctas(int64_t D, int64_t M, int rows_kind) {
    const int per = 512 / backward_team(D, rows_kind);
    const int64_t most = 148 * (per < 1 ? 1 : per > 16 ? 16 : per), rows = (M + 1) / 2;
    return rows < most ? rows : most;
}
size_t norm_part_floats(const Division &d, int64_t D) { return (size_t)d.ctas * 4 * D + (d.chunks > 1 ? (size_t)d.units * D : 0); }

}  // namespace

int bnn_join_columns(bnn_ctx *ctx, int dtype, const float *part, int64_t pitch, int64_t count, void *out, int64_t columns) {
    JoinArgs j{};
    j.D = (int)columns; j.part[0] = part; j.out[0] = out; j.pitch[0] = pitch; j.count[0] = count; j.outs[0] = 1;
    return launch_join(ctx, dtype, j, 1);
}

namespace {
// The forward pass of both entry points: normed as it is, or microscaled into q with normed for the represented values.
template <bool MX> int block_norm(bnn_ctx *ctx, const bnn_block_norm_desc *norm, const void *x, int64_t ldx, const void *block, int64_t ldb, int64_t M, void *stream,
                                  int64_t lds, const bnn_mx_matrix *q, void *normed, int64_t ldn, float *stats) {
    if (int st = check_norm(norm, M)) return st;
    const int size = bnn_real_size(norm->dtype);
    if (!block && M > 0 && (norm->post || norm->gate)) return BNN_ERR_INVALID_ARG;
    if ((MX || normed) && !norm->pre) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_real(x, ldx, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(block, ldb, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(stream, lds, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(normed, ldn, M, norm->D, size)) return st;
    if (int st = bnn_check_real_opt(stats, 4, M, 4, 4)) return st;
    if (MX) {
        if (int st = bnn_check_mx(q)) return st;
        if (q->rows != M || q->cols != norm->D) return BNN_ERR_INVALID_ARG;
        if (bnn_mx_touches(q, x, ldx, M, norm->D, size) || bnn_mx_touches(q, block, ldb, M, norm->D, size) || bnn_mx_touches(q, stream, lds, M, norm->D, size) ||
            bnn_mx_touches(q, normed, ldn, M, norm->D, size)) return BNN_ERR_INVALID_ARG;
    }
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (M == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    NormArgs a = norm_args(norm, M);
    a.x = x; a.ldx = ldx; a.block = block; a.ldb = ldb; a.stream = stream; a.lds = lds; a.normed = normed; a.ldn = ldn; a.stats = stats;
    if (MX) {
        a.mx_values = static_cast<uint8_t *>(q->values); a.mx_scales = static_cast<uint8_t *>(q->scales);
        a.inv = 1.0 / (double)norm->D;
        a.mx_limit = (int)bnn_mx_groups(norm->D) * BNN_MX_GROUP; a.mx_four = q->format == BNN_MX_E2M1;
    }
    const bool vec = norm_vec(norm, M, a);
    if (MX) return bnn_launch_norm_mx(ctx, a, norm->dtype, vec);
    const auto launch = [&](auto zero) {
        using T = decltype(zero);
        return vec ? launch_forward<T, true>(ctx, a) : launch_forward<T, false>(ctx, a);
    };
    return norm->dtype == BNN_F32 ? launch(0.0f) : norm->dtype == BNN_F16 ? launch(__half()) : launch(__nv_bfloat16());
}
}  // namespace

extern "C" int bnn_block_norm(bnn_ctx *ctx, const bnn_block_norm_desc *norm, const void *x, int64_t ldx, const void *block, int64_t ldb,
                              int64_t M, void *stream, int64_t lds, void *normed, int64_t ldn, float *stats) {
    return block_norm<false>(ctx, norm, x, ldx, block, ldb, M, stream, lds, nullptr, normed, ldn, stats);
}
extern "C" int bnn_block_norm_mx(bnn_ctx *ctx, const bnn_block_norm_desc *norm, const void *x, int64_t ldx, const void *block, int64_t ldb, int64_t M,
                                 void *stream, int64_t lds, const bnn_mx_matrix *normed, void *represented, int64_t ldv, float *stats) {
    return block_norm<true>(ctx, norm, x, ldx, block, ldb, M, stream, lds, normed, represented, ldv, stats);
}

extern "C" size_t bnn_block_norm_workspace_bytes(const bnn_block_norm_desc *norm, int64_t M) {
    if (check_norm(norm, M) || M == 0) return 0;
    size_t most = 0;                         // of all kinds of rows
    for (int rows = 0; rows < ROWS_KINDS; ++rows) {
        const size_t n = norm_part_floats(divide_rows(M, rows_per_gate(norm, M), norm_ctas(norm->D, M, rows)), norm->D);
        if (n > most) most = n;
    }
    return (most * 4 + 255) & ~size_t(255);
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
    if (int st = bnn_check_real_opt(g->dgate, g->ld_dgate, gate_rows(norm, M), norm->D, size)) return st;
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
    const bool vec = norm_vec(norm, M, a);
    const Division d = divide_rows(M, a.rows_per_gate, norm_ctas(norm->D, M, backward_rows(a, size, vec)));
    a.groups = d.groups; a.chunks = d.chunks; a.chunk_rows = d.chunk_rows; a.units = d.units;
    const bool joins = a.want || (a.dgate && d.chunks > 1);
    if (joins && (!ctx->ws || ctx->ws_bytes < norm_part_floats(d, norm->D) * 4)) return BNN_ERR_WORKSPACE;
    a.part = static_cast<float *>(ctx->ws);
    a.part_gate = a.part + (size_t)d.ctas * 4 * norm->D;
    const unsigned ctas = (unsigned)d.ctas;
    int st;
    if (norm->dtype == BNN_F32) st = vec ? launch_backward<float, true>(ctx, a, ctas) : launch_backward<float, false>(ctx, a, ctas);
    else if (norm->dtype == BNN_F16) st = vec ? launch_backward<__half, true>(ctx, a, ctas) : launch_backward<__half, false>(ctx, a, ctas);
    else st = vec ? launch_backward<__nv_bfloat16, true>(ctx, a, ctas) : launch_backward<__nv_bfloat16, false>(ctx, a, ctas);
    if (st) return st;
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
