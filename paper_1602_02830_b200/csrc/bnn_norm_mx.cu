// Norms around a block with the stream's norm microscaled (bnn_mx.cuh); the mathematics is that of bnn_norm.cu.  Eight neighbouring columns a thread and slot
// whatever the alignment, so that four lanes hold a block.
// Elements have three or one bits behind the point: what decides an element is on which side of a border its value lies, and likewise the block's exponent.  So the row's squares are
// added up in float64, the reciprocal root is kept as a float32 and what it lacks, and what a value's float32 rounding lacks is known where it lies beside a border.  In the RMS form
// without shifts that decides every border by the row s in float32 (x + block of 16 bits: their exact sum, unless they are 2^16 apart).  A row with a block norm, a gate or alpha
// beside 1 is rounded to float32 before, the layer form's row around its mean as well; a shift that cancels most of the value leaves more than the border's surroundings cover.
// Bound: HBM, and the issue slots beside it.  8192 x 4096 bf16: residual and norm 41.7 us = 5.7 TB/s, with represented values 48.9 us = 6.2 TB/s (BARE); with a block norm 57.0 us; layer
// norm 75, with block norm, shifts and represented values 98; 2560 columns, not whole teams, 37.6; float16 rows of 1011 31.5; float32 4096 x 4096 37.7, layer norm 50.  2048 x 16384: 47 us,
// float32 75.  Elements off the 64-bit result: none of 33.5 million; 20 in float32 alone, 9 with float32 sums in a thread and the borders of normal elements only.
#include "bnn_norm.cuh"
#include "bnn_mx.cuh"

namespace {
using namespace bnn_norm;

struct Two { float high, low; };
__device__ __forceinline__ Two two(double v) { const float high = (float)v; return {high, (float)(v - (double)high)}; }
// Mean over the row of the block's sum of `a`, with `add` (eps or 0).
__device__ __forceinline__ double block_mean(double a, double add, double inv, double *buf, int warps, int warp, int lane) {
#pragma unroll
    for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    if (warps > 1) {
        if (lane == 0) buf[warp] = a;
        __syncthreads();
        a = buf[0];
        for (int w = 1; w < warps; ++w) a += buf[w];
    }
    return fma(a, inv, add);
}
// From float32's root by r (1 - e)^(-1/2), e = 1 - v r^2, to the second order: e is below 2^-21.
__device__ __forceinline__ Two inverse_root(double v) {
    const bool small = v < 1e-30, large = v > 1e30;
    v *= small ? 0x1p192 : large ? 0x1p-160 : 1.0;                       // squares of any float32 are then in its range
    const float first = rsqrtf((float)v);
    if (!(first > 0.0f && first < 1e30f)) return {first, 0.0f};        // zero, infinity, NaN
    const double r = (double)first, e = fma(-(v * r), r, 1.0);
    return two(fma(r * e, fma(0.375, e, 0.5), r) * (small ? 0x1p96 : large ? 0x1p-80 : 1.0));
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
// What u = round(t r + c), t = round(s w), lacks: s w is t and its own rest, r two parts.  The rest is good to 2^-44 of u with float64 sums of squares, of LAYER_TIE where the
// row around its mean is a float32 rounding itself and its sums are float32.
constexpr float RMS_TIE = 1.0f / (1ll << 44), LAYER_TIE = 1.0f / (1 << 23);
struct NormHeld {
    float s[8], w[8], c[8];
    Two r;
    float tie;
    __device__ __forceinline__ float lack(int j, float u) const {
        const float t = __fmul_rn(s[j], w[j]);
        return fmaf(fmaf(s[j], w[j], -t), r.high, fmaf(t, r.low, fmaf(t, r.high, c[j] - u)));
    }
};
struct NormRest {
    static constexpr bool rounded = true;
    const float (&s)[8];
    const float (&w)[8];
    const float (&c)[8];
    Two r;
    float tie;
    __device__ __forceinline__ NormHeld held() const {
        NormHeld h;
#pragma unroll
        for (int j = 0; j < 8; ++j) { h.s[j] = s[j]; h.w[j] = w[j]; h.c[j] = c[j]; }
        h.r = r; h.tie = tie;
        return h;
    }
};
template <typename T, bool VEC> __device__ __forceinline__ void spread(const Eight<T> &e, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e[j];
}
// LAYER, RMS: the two norms; PLAIN_ROWS: BNN_NORM_RMS without shifts, with a block and a stream; BARE: that without a norm of the block and a gate, with a weight, rows of whole
// teams.  (The two norms in one kernel kept float32 and float64 sums beside each other: layer norm of 4096 x 4096 float32 68 us.)
enum NormKind { LAYER, RMS, PLAIN_ROWS, BARE };
template <typename T, int SLOTS, int THREADS, bool VEC, int KIND, bool FOUR>
// (Four CTAs of 256 an SM, 64 registers: 44.0 -> 41.7 us; float32 rows and the layer norm lose by it, 37.7 -> 39.3 and 75.2 -> 76.9.)
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : sizeof(T) == 2 && KIND != LAYER ? 4 : 3) k_block_norm_mx(const NormArgs p) {
    constexpr bool PLAIN = KIND == PLAIN_ROWS || KIND == BARE, WHOLE = KIND == BARE, layer = KIND == LAYER;
    __shared__ double buf[4][32];
    __shared__ __align__(16) T stage[VEC ? 8 : THREADS * 8];
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x, team = blockDim.x, warps = team >> 5, warp = tid >> 5, lane = tid & 31;
    const T *pw = WHOLE ? nullptr : static_cast<const T *>(p.post_w), *pc = PLAIN ? nullptr : static_cast<const T *>(p.post_c);
    const T *nw = static_cast<const T *>(p.pre_w), *nc = PLAIN ? nullptr : static_cast<const T *>(p.pre_c);
    const bool blocks = PLAIN || p.block, post = !WHOLE && p.post;
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
            mean = (float)block_mean(t, 0.0, p.inv, buf[0], warps, warp, lane);
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
        r = inverse_root(block_mean(q, p.eps, p.inv, buf[1], warps, warp, lane));
    }
    if (p.stats && tid == 0) { p.stats[4 * m] = mean; p.stats[4 * m + 1] = r.high; }
    float s[SLOTS][8];
    double q = 0.0;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        Eight<T> w, g, c;
        w.fill(1.0f); g.fill(1.0f);
        if (blocks && pw) w = take8<T, VEC, WHOLE>(pw, i, tid, team, p.D);
        if (gate) g = take8<T, VEC, WHOLE>(gate, i, tid, team, p.D);
        if (blocks && pc) c = take8<T, VEC, WHOLE>(pc, i, tid, team, p.D);
        double even = 0.0, odd = 0.0;                               // of the squares; a float32 sum of the values where a mean comes first
        float sum = 0.0f;
        if constexpr (PLAIN) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                unsigned long long add = pair_of(rb[i][j], rb[i][j + 1]);
                if (!WHOLE) add = mul2(add, pair_of(w[j], w[j + 1]));
                if (post) add = fma2(add, both(r.high), mul2(add, both(r.low)));
                if (gate) add = mul2(add, pair_of(g[j], g[j + 1]));
                const unsigned long long both_sums = fma2(both(p.alpha), pair_of(rx[i][j], rx[i][j + 1]), add);
                pair_out(both_sums, s[i][j], s[i][j + 1]);
                even = fma((double)s[i][j], (double)s[i][j], even);
                odd = fma((double)s[i][j + 1], (double)s[i][j + 1], odd);
            }
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
                if (layer) sum += s[i][j];
                else even = fma((double)s[i][j], (double)s[i][j], even);
            }
        }
        q += layer ? (double)sum : even + odd;
        if (PLAIN || p.stream) give8<T, VEC, WHOLE>(static_cast<T *>(p.stream) + m * p.lds, i, tid, team, p.D, s[i], stage);
    }
    // the stream's
    mean = 0.0f;
    double of = block_mean(q, layer ? 0.0 : (double)p.eps, p.inv, buf[2], warps, warp, lane);
    if (layer) {
        const Two m = two(of);
        mean = m.high;
        q = 0.0;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            float v = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[i][j] = column<true>(i, j, tid, team) < p.D ? (s[i][j] - mean) - m.low : 0.0f;
                v = fmaf(s[i][j], s[i][j], v);
            }
            q += (double)v;
        }
        of = block_mean(q, p.eps, p.inv, buf[3], warps, warp, lane);
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
        const NormRest rest{s[i], w, c, r, layer ? LAYER_TIE : RMS_TIE};
        mx_write8<FOUR>(p.mx_values, p.mx_scales, m, c0, p.mx_limit, u, p.normed != nullptr, rest);
        if (p.normed) give8<T, VEC, WHOLE>(static_cast<T *>(p.normed) + m * p.ldn, i, tid, team, p.D, u, stage);
    }
}

template <int N> struct Int { static constexpr int value = N; };
// Teams as in bnn_norm.cu.
template <typename T, bool VEC, bool FOUR> int launch_forward_mx(bnn_ctx *ctx, const NormArgs &a) {
    const int groups = (a.D + 7) / 8;
    const bool few = a.M <= 2 * ctx->sm_count;
    const int slots = groups > 1024 ? 4 : (few || groups <= 32) ? 1 : groups <= 64 ? 2 : 4;
    const int team = ((groups + slots - 1) / slots + 31) & ~31;
    const dim3 grid((unsigned)a.M), block(team);
    const bool plain = VEC && !a.layer && !a.post_c && !a.pre_c && a.block && a.stream, bare = plain && !a.post && !a.gate && a.pre_w && a.D == slots * team * 8;
#define BNN_KERNEL(KIND) k_block_norm_mx<T, SLOTS, THREADS, VEC, KIND, FOUR>
    const auto run = [&](auto slots_of, auto threads_of) -> int {
        constexpr int SLOTS = decltype(slots_of)::value, THREADS = decltype(threads_of)::value;
        auto kernel = a.layer ? BNN_KERNEL(LAYER) : BNN_KERNEL(RMS);
        if constexpr (VEC) kernel = bare ? BNN_KERNEL(BARE) : plain ? BNN_KERNEL(PLAIN_ROWS) : kernel;
        BNN_CUDA_TRY(ctx, bnn_launch_dependent(kernel, grid, block, 0, ctx->stream, a));
        return bnn_check_launch(ctx);
    };
#undef BNN_KERNEL
    if (slots == 1) return run(Int<1>(), Int<1024>());
    if (slots == 2) return run(Int<2>(), Int<256>());
    return team <= 256 ? run(Int<4>(), Int<256>()) : run(Int<4>(), Int<1024>());
}
template <typename T> int launch(bnn_ctx *ctx, const NormArgs &a, bool vec) {
    if (a.mx_four) return vec ? launch_forward_mx<T, true, true>(ctx, a) : launch_forward_mx<T, false, true>(ctx, a);
    return vec ? launch_forward_mx<T, true, false>(ctx, a) : launch_forward_mx<T, false, false>(ctx, a);
}

}  // namespace

int bnn_launch_norm_mx(bnn_ctx *ctx, const NormArgs &a, int dtype, bool vec) {
    return dtype == BNN_F32 ? launch<float>(ctx, a, vec) : dtype == BNN_F16 ? launch<__half>(ctx, a, vec) : launch<__nv_bfloat16>(ctx, a, vec);
}
