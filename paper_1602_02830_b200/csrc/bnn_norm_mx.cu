// Norms around a block with the stream's norm microscaled (bnn_mx.cuh); the mathematics is that of bnn_norm.cu.  Eight neighbouring columns a thread and slot
// whatever the alignment, so that four lanes hold a block.
// Elements have three or one bits behind the point: what decides an element is on which side of a border its value lies.  So the sums of the warps, the mean square
// and the reciprocal root are kept in two float32 each (a value and what it lacks), and what a value's float32 rounding lacks is known where it lies beside a border.
// Bound: HBM, and the issue slots beside it (41 instructions an element where everything is optional).  8192 x 4096 bf16: residual and norm 41.3 us = 5.7 TB/s, with represented
// values 48.2 us = 6.3 TB/s (BARE; 48.4 and 53.6 with a predicate for every access and optional weights); with a block norm 55.7 us.  Elements off the 64-bit result: 3 of 33.5
// million, 20 in float32 alone.
#include "bnn_norm.cuh"
#include "bnn_mx.cuh"

namespace {
using namespace bnn_norm;

struct Two { float high, low; };
__device__ __forceinline__ Two two_sum(float a, float b) {       // a + b exactly (Knuth)
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two two_product(float a, float b) {
    const float s = __fmul_rn(a, b);
    return {s, fmaf(a, b, -s)};
}
// Mean over the row of the block's sum of `a`, with `add` (eps or 0); 1 / D is inv + inv_low.
__device__ __forceinline__ Two block_mean(float a, float add, float inv, float inv_low, float *buf, int warps, int warp, int lane) {
    a = warp_sum(a);
    Two s{a, 0.0f};
    if (warps > 1) {
        if (lane == 0) buf[warp] = a;
        __syncthreads();
        s = {buf[0], 0.0f};
        for (int w = 1; w < warps; ++w) {
            const Two t = two_sum(s.high, buf[w]);
            s = {t.high, s.low + t.low};
        }
    }
    const Two t = two_product(s.high, inv), u = two_sum(t.high, add);
    return {u.high, u.low + (t.low + (s.high * inv_low + s.low * inv))};
}
__device__ __forceinline__ Two inverse_root(Two v) {
    if (!(v.high > 1e-30f && v.high < 1e30f)) return {1.0f / sqrtf(v.high), 0.0f};
    // r (1 + e / 2), e = 1 - v r^2
    const float r = rsqrtf(v.high);
    const Two s = two_product(r, r), t = two_product(v.high, s.high);
    const float e = ((1.0f - t.high) - t.low) - v.high * s.low - v.low * s.high, low = 0.5f * r * e, high = __fadd_rn(r, low);
    return {high, __fsub_rn(low, __fsub_rn(high, r))};
}
// WHOLE: the team's slots are the row's columns exactly, nothing is asked.
template <typename T, bool VEC, bool WHOLE = false> __device__ __forceinline__ Eight<T> take8(const T *row, int slot, int tid, int team, int D) {
    if constexpr (WHOLE) {
        Eight<T> e;
        const uint4 *from = reinterpret_cast<const uint4 *>(row + column<true>(slot, 0, tid, team));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 w = from[i];
            e.w[4 * i] = w.x; e.w[4 * i + 1] = w.y; e.w[4 * i + 2] = w.z; e.w[4 * i + 3] = w.w;
        }
        return e;
    } else if constexpr (VEC) return read8<T, true>(row, slot, tid, team, D);
    else {
        Eight<T> e;
        mx_read_words<T>(row, column<true>(slot, 0, tid, team), D, e.w);
        return e;
    }
}
template <typename T, bool VEC, bool WHOLE = false> __device__ __forceinline__ void give8(T *row, int slot, int tid, int team, int D, const float (&v)[8], T *stage) {
    if constexpr (WHOLE) store8(row + column<true>(slot, 0, tid, team), v);
    else if constexpr (VEC) write8<T, true>(row, slot, tid, team, D, v);
    else mx_spread8(row, column<true>(slot, 0, tid & ~31, team), D, v, stage + (tid >> 5) * 256);
}
// What u = round(t r + c), t = round(s w), lacks: s w is t and its own rest, r two parts.
struct NormRest {
    static constexpr bool rounded = true;
    const float (&s)[8];
    const float (&w)[8];
    const float (&c)[8];
    Two r;
    __device__ __forceinline__ float operator()(int j, float u) const {
        const float t = __fmul_rn(s[j], w[j]);
        return fmaf(fmaf(s[j], w[j], -t), r.high, fmaf(t, r.low, fmaf(t, r.high, c[j] - u)));
    }
};
template <typename T, bool VEC> __device__ __forceinline__ void spread(const Eight<T> &e, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e[j];
}
// ANY; PLAIN: BNN_NORM_RMS without shifts, with a block and a stream; BARE: that without a norm of the block and a gate, with a weight, rows of whole teams.
enum NormKind { ANY, PLAIN_ROWS, BARE };
template <typename T, int SLOTS, int THREADS, bool VEC, int KIND, bool FOUR>
__global__ void __launch_bounds__(THREADS, THREADS <= 256 ? 3 : 1) k_block_norm_mx(const NormArgs p) {
    constexpr bool PLAIN = KIND != ANY, WHOLE = KIND == BARE;
    __shared__ float buf[4][32];
    __shared__ __align__(16) T stage[VEC ? 8 : THREADS * 8];
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = WHOLE ? nullptr : static_cast<const T *>(p.post_w), *pc = PLAIN ? nullptr : static_cast<const T *>(p.post_c);
    const T *nw = static_cast<const T *>(p.pre_w), *nc = PLAIN ? nullptr : static_cast<const T *>(p.pre_c);
    const bool layer = !PLAIN && p.layer, blocks = PLAIN || p.block, post = !WHOLE && p.post;
    Eight<T> rx[SLOTS], rb[SLOTS];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        rx[i] = take8<T, VEC, WHOLE>(static_cast<const T *>(p.x) + m * p.ldx, i, tid, team, p.D);
        if (blocks) rb[i] = take8<T, VEC, WHOLE>(static_cast<const T *>(p.block) + m * p.ldb, i, tid, team, p.D);
    }
    const T *gate = !WHOLE && p.gate ? static_cast<const T *>(p.gate) + (m / p.rows_per_gate) * p.ld_gate : nullptr;
    // the block's norm: mean and reciprocal deviation.  Columns behind D are zeros: around a mean they are left out of the sums.
    float mean = 0.0f;
    Two r{1.0f, 0.0f};
    if (blocks && post) {
        if (layer) {
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                float v = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) v += rb[i][j];
                t += v;
            }
            mean = block_mean(t, 0.0f, p.inv_d, p.inv_low, buf[0], warps, warp, lane).high;
        }
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            float v = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = !layer || column<true>(i, j, tid, team) < p.D ? rb[i][j] - mean : 0.0f;
                v = fmaf(d, d, v);
            }
            q += v;
        }
        r = inverse_root(block_mean(q, p.eps, p.inv_d, p.inv_low, buf[1], warps, warp, lane));
    }
    if (p.stats && tid == 0) { p.stats[4 * m] = mean; p.stats[4 * m + 1] = r.high; }
    float s[SLOTS][8], q = 0.0f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        Eight<T> w, g, c;
        w.fill(1.0f); g.fill(1.0f);
        if (blocks && pw) w = take8<T, VEC, WHOLE>(pw, i, tid, team, p.D);
        if (gate) g = take8<T, VEC, WHOLE>(gate, i, tid, team, p.D);
        if (blocks && pc) c = take8<T, VEC, WHOLE>(pc, i, tid, team, p.D);
        float v = 0.0f;
        if constexpr (PLAIN) {
            unsigned long long squares = both(0.0f);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                unsigned long long add = pair_of(rb[i][j], rb[i][j + 1]);
                if (!WHOLE) add = mul2(add, pair_of(w[j], w[j + 1]));
                if (post) add = fma2(add, both(r.high), mul2(add, both(r.low)));
                if (gate) add = mul2(add, pair_of(g[j], g[j + 1]));
                const unsigned long long sum = fma2(both(p.alpha), pair_of(rx[i][j], rx[i][j + 1]), add);
                squares = fma2(sum, sum, squares);
                pair_out(sum, s[i][j], s[i][j + 1]);
            }
            float odd;
            pair_out(squares, v, odd);
            v += odd;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float add = 0.0f;
                if (blocks) {
                    const float t = (rb[i][j] - mean) * w[j];
                    add = post ? fmaf(t, r.high, t * r.low) : t;
                    if (pc) add += c[j];
                    if (gate) add *= g[j];
                }
                s[i][j] = fmaf(p.alpha, rx[i][j], add);
                if (layer && column<true>(i, j, tid, team) >= p.D) s[i][j] = 0.0f;      // the block's mean is taken off zeros there
                v = layer ? v + s[i][j] : fmaf(s[i][j], s[i][j], v);
            }
        }
        q += v;
        if (PLAIN || p.stream) give8<T, VEC, WHOLE>(static_cast<T *>(p.stream) + m * p.lds, i, tid, team, p.D, s[i], stage);
    }
    // the stream's
    mean = 0.0f;
    Two of = block_mean(q, layer ? 0.0f : p.eps, p.inv_d, p.inv_low, buf[2], warps, warp, lane);
    if (layer) {
        mean = of.high;
        q = 0.0f;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            float v = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[i][j] = column<true>(i, j, tid, team) < p.D ? (s[i][j] - mean) - of.low : 0.0f;
                v = fmaf(s[i][j], s[i][j], v);
            }
            q += v;
        }
        of = block_mean(q, p.eps, p.inv_d, p.inv_low, buf[3], warps, warp, lane);
    }
    r = inverse_root(of);
    if (p.stats && tid == 0) { p.stats[4 * m + 2] = mean; p.stats[4 * m + 3] = r.high; }
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int c0 = column<true>(i, 0, tid, team);
        Eight<T> e;
        e.fill(1.0f);
        if (WHOLE || nw) e = take8<T, VEC, WHOLE>(nw, i, tid, team, p.D);
        float w[8], c[8], u[8];
        spread<T, VEC>(e, w);
        e.fill(0.0f);
        if (nc) e = take8<T, VEC, WHOLE>(nc, i, tid, team, p.D);
        spread<T, VEC>(e, c);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const unsigned long long t = mul2(pair_of(s[i][j], s[i][j + 1]), pair_of(w[j], w[j + 1]));
            pair_out(fma2(t, both(r.high), nc ? fma2(t, both(r.low), pair_of(c[j], c[j + 1])) : mul2(t, both(r.low))), u[j], u[j + 1]);
        }
        if (layer) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j >= p.D) u[j] = 0.0f;
        }
        const NormRest rest{s[i], w, c, r};
        mx_write8<FOUR>(p.mx_values, p.mx_scales, m, c0, p.mx_limit, u, p.normed != nullptr, rest);
        if (p.normed) give8<T, VEC, WHOLE>(static_cast<T *>(p.normed) + m * p.ldn, i, tid, team, p.D, u, stage);
    }
}

// Teams as in bnn_norm.cu.
template <typename T, bool VEC, bool FOUR> int launch_forward_mx(bnn_ctx *ctx, const NormArgs &a) {
    const int groups = (a.D + 7) / 8;
    const bool few = a.M <= 2 * ctx->sm_count;
    const int slots = groups > 1024 ? 4 : (few || groups <= 32) ? 1 : groups <= 64 ? 2 : 4;
    const int team = ((groups + slots - 1) / slots + 31) & ~31;
    const dim3 grid((unsigned)a.M), block(team);
    const bool plain = VEC && !a.layer && !a.post_c && !a.pre_c && a.block && a.stream, bare = plain && !a.post && !a.gate && a.pre_w && a.D == slots * team * 8;
#define BNN_FORWARD(SLOTS, THREADS) BNN_CUDA_TRY(ctx, bnn_launch_dependent(bare ? k_block_norm_mx<T, SLOTS, THREADS, VEC, VEC ? BARE : ANY, FOUR> : \
                                                                           plain ? k_block_norm_mx<T, SLOTS, THREADS, VEC, VEC ? PLAIN_ROWS : ANY, FOUR> : \
                                                                           k_block_norm_mx<T, SLOTS, THREADS, VEC, ANY, FOUR>, grid, block, 0, ctx->stream, a))
    if (slots == 1) BNN_FORWARD(1, 1024);
    else if (slots == 2) BNN_FORWARD(2, 256);
    else if (team <= 256) BNN_FORWARD(4, 256);
    else BNN_FORWARD(4, 1024);
#undef BNN_FORWARD
    return bnn_check_launch(ctx);
}
template <typename T> int launch(bnn_ctx *ctx, const NormArgs &a, bool vec) {
    if (a.mx_four) return vec ? launch_forward_mx<T, true, true>(ctx, a) : launch_forward_mx<T, false, true>(ctx, a);
    return vec ? launch_forward_mx<T, true, false>(ctx, a) : launch_forward_mx<T, false, false>(ctx, a);
}

}  // namespace

int bnn_launch_norm_mx(bnn_ctx *ctx, const NormArgs &a, int dtype, bool vec) {
    return dtype == BNN_F32 ? launch<float>(ctx, a, vec) : dtype == BNN_F16 ? launch<__half>(ctx, a, vec) : launch<__nv_bfloat16>(ctx, a, vec);
}
