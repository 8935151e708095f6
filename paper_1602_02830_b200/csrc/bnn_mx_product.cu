// Products of microscaled operands on the 5th-generation tensor cores: dense layer and gated projections in 8 and 4 bits.
//
//   sum_k x[m][k] w[n][k],  x and w e4m3 or e2m1 elements times a power of two for each 32 of them along k, float32 accumulators.
// tcgen05.mma multiplies by the scales itself (block_scale): it reads them from tensor memory, one byte per row and block, where tcgen05.cp brings
// them from shared memory as they lie in memory.  Two kinds: mxf4 (e2m1 x e2m1, packed, 64 of K an instruction) and mxf8f6f4 (bytes, 32 of K); the latter takes e2m1
// beside e4m3 when its nibbles lie in the low eight bytes of every sixteen, which the tensor map does on the way (16U4_ALIGN16B).
// One stage is a row of 128 bytes of shared memory: 256 of K packed, 128 otherwise.
//
// Bound: many rows, the tensor pipe and the part's power limit (8192 x 8192 x 8192 of random values: 182 us = 6.0 PFLOP/s in 4 bits, 363 us = 3.0 PFLOP/s in 8 bits, 352 with 4-bit
// weights, in bursts; 216, 435 and 404 after seconds on end at the power limit, 1250 to 1360 MHz; 8192 x 4096 -> 8192 in 4 bits 101 us, with a residual 116; gated, 4096 rows, 4096 -> 8192 twice, microscaled result 176 us = 3.1 PFLOP/s).  Short
// sums: the epilogue (4096 x 128 -> 4096 13.5 to 19 us, gelu 27 to 42).  Fewer rows: mostly the operands' way from L2 (at pair_cost; 512 x 4096 -> 4096 13.8 us, in 4 bits
// 9.4); a token, 4096 -> 4096 with 4-bit weights, 7.1 us, of which 3.5 are launch, set-up and tail.
// Nothing is rounded between the sums and the one conversion of a result: to 16 bits, or to an element of a microscaled result.
#include "bnn_epilogue.cuh"
#include "bnn_internal.cuh"
#include "bnn_mx.cuh"
#include <mutex>

namespace {

__device__ int g_mx_error;               // 0 = fine; otherwise a code saying which wait gave up

// Maps of the operands: x rows, its scales; weights (gated: gate, up) and theirs.
struct MxMaps { CUtensorMap x, xs, w[2], ws[2]; };
struct MxCommon : Common {
    int four;                            // both operands packed e2m1: kind mxf4
    int last;                            // instructions of the last K step
    uint32_t w_bytes;                    // what a copy of 128 weight rows counts on its barrier: elements as they are in memory, nibbles on their way to bytes half of what they fill
    uint32_t idesc;
    uint8_t *q_values, *q_scales;        // microscaled output
    int64_t q_limit;
    int q_four;
};

constexpr uint32_t ROWS128 = 128 * 128;  // bytes of 128 rows of a stage

// One lane of a warp that is together.  What leads the tensor cores and the copies runs warp-wide and lets one lane issue: descriptors, addresses and counters are then the
// same for all lanes and stay in the registers that those instructions take them from.
__device__ __forceinline__ bool elected() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d_2sm(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// 512 bytes of scales (32 lanes of 16 bytes, groups of eight lanes 128 bytes apart, no swizzle) to four columns of tensor memory, in all four lane quadrants.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) { return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(128u >> 4) << 32 | 1ull << 46; }
template <int CTAS> __device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    if constexpr (CTAS == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
#define BNN_MX_MMA(GROUP, KIND)                                                                                                                                  \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::" GROUP ".kind::" KIND ".block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}" \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory")
template <int CTAS, bool FOUR> __device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if constexpr (CTAS == 2) {
        if constexpr (FOUR) BNN_MX_MMA("2", "mxf4");
        else BNN_MX_MMA("2", "mxf8f6f4");
    } else {
        if constexpr (FOUR) BNN_MX_MMA("1", "mxf4");
        else BNN_MX_MMA("1", "mxf8f6f4");
    }
}
// One K step: instruction k of up to four, scales of A and B in tensor memory at sa and sb, `pitch` columns a group of 128 of K further.  The bytes of an
// instruction's blocks within a column's words are named in the descriptor: one byte (32 of K), or the lower or upper two (64 of K).
template <int CTAS, bool FOUR> __device__ __forceinline__ void step_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t pitch_b, int count, bool first) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (k >= count) break;
        const uint32_t id = FOUR ? 2u * (k & 1) : (uint32_t)k, group = FOUR ? k >> 1 : 0;
        mma_mx<CTAS, FOUR>(d, a + 2 * k, b + 2 * k, idesc | id << 4 | id << 29, sa + 4 * group, sb + pitch_b * group, first && k == 0 ? 0u : 1u);
    }
}

__device__ __forceinline__ float exp2_of(float v) { float r; asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float inverse_of(float v) { float r; asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
constexpr float LOG2E = 1.44269504f;
// z sigmoid(u), u given as -u log2 e.
__device__ __forceinline__ unsigned long long times_sigmoid(unsigned long long z, unsigned long long minus_u) {
    float a, b;
    pair_out(minus_u, a, b);
    const unsigned long long d = add2(pair_of(exp2_of(a), exp2_of(b)), both(1.0f));
    pair_out(d, a, b);
    return mul2(z, pair_of(inverse_of(a), inverse_of(b)));
}
// gelu(z) = max(z, 0) - |z| Phi(-|z|), Phi as in normal_cdf (bnn_real.cuh).  Above z = 100 the second term is 0 and stays 0; of minus infinity it is infinity times 0, a NaN as in
// z Phi(z).
__device__ __forceinline__ unsigned long long gelu2(unsigned long long z) {
    float a, b;
    pair_out(z, a, b);
    const float ra = a < 0.0f ? 0.0f : a, rb = b < 0.0f ? 0.0f : b;
    const unsigned long long size = pair_of(fabsf(fminf(a, 100.0f)), fabsf(fminf(b, 100.0f)));
    pair_out(mul2(mul2(z, z), both(-0.5f * LOG2E)), a, b);
    const unsigned long long e = pair_of(exp2_of(a), exp2_of(b));
    pair_out(fma2(size, both(0.26516503f), both(1.0f)), a, b);
    const unsigned long long t = pair_of(inverse_of(a), inverse_of(b));
    unsigned long long s = fma2(t, both(-0.0675475374f), both(0.193967491f));
    s = fma2(t, s, both(-0.0647966936f));
    s = fma2(t, s, both(0.141529396f));
    s = fma2(t, s, both(0.0833328068f));
    s = fma2(t, s, both(0.107844487f));
    s = fma2(t, s, both(0.105669729f));
    s = mul2(mul2(mul2(t, s), e), size);
    pair_out(s, a, b);
    return pair_of(ra - a, rb - b);
}
// The activation of sixteen values; both forms of GELU two values an instruction (4096 x 2048 -> 4096: gelu 35.0 us, one at a time 37.5; its tanh form 32.3 and 34.2).
// SILU has little but its exponential and reciprocal, sixteen a clock and SM either way, and is faster without the pairs (gated 48.8 and 50.6).
__device__ __forceinline__ void activate(int act, float (&v)[16]) {
#define BNN_EACH_PAIR(EXPRESSION)                              \
    _Pragma("unroll") for (int j = 0; j < 16; j += 2) {        \
        const unsigned long long z = pair_of(v[j], v[j + 1]);  \
        pair_out(EXPRESSION, v[j], v[j + 1]);                  \
    }
    switch (act) {
        case BNN_ACT_NONE: break;
        case BNN_ACT_GELU: BNN_EACH_PAIR(gelu2(z)); break;
        case BNN_ACT_GELU_TANH:
            BNN_EACH_PAIR(times_sigmoid(z, mul2(z, fma2(mul2(z, z), both(-GELU_2C * GELU_A * LOG2E), both(-GELU_2C * LOG2E)))));
            break;
        case BNN_ACT_SILU: act16<BNN_ACT_SILU>(v); break;
        case BNN_ACT_SIGMOID: act16<BNN_ACT_SIGMOID>(v); break;
        case BNN_ACT_RELU: act16<BNN_ACT_RELU>(v); break;
        default: act16<BNN_ACT_HTANH>(v); break;
    }
#undef BNN_EACH_PAIR
}

// Results that are microscaled: a lane's 32 columns are a block.  Columns behind the last are zeros whatever the accumulators hold (scales of weight rows
// that do not exist may be NaN); the row's padding up to 128 columns is written too.
__device__ __forceinline__ void write_block(const MxCommon &p, const Output &q, int64_t m, int64_t n0, float (&v)[32]) {
    const int n = (int)(q.N - n0 < 32 ? q.N - n0 : 32);
    if (n < 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = j < n ? v[j] : 0.0f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) top = max(top, mx_magnitude(v[j]));
    const uint32_t scale = p.q_four ? mx_scale<true>(top) : mx_scale<false>(top);
    const unsigned long long down = both(mx_down(scale));
#pragma unroll
    for (int j = 0; j < 32; j += 2) pair_out(mul2(pair_of(v[j], v[j + 1]), down), v[j], v[j + 1]);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float e[8];
        uint32_t t[2];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = v[8 * i + j];
        if (p.q_four) { mx_encode8<true>(e, t); w[i] = t[0]; }
        else { mx_encode8<false>(e, t); w[2 * i] = t[0]; w[2 * i + 1] = t[1]; }
    }
    if (m >= q.M || n0 >= p.q_limit) return;
    if (p.q_four) *reinterpret_cast<uint4 *>(p.q_values + m * (p.q_limit / 2) + n0 / 2) = make_uint4(w[0], w[1], w[2], w[3]);
    else {
        uint4 *to = reinterpret_cast<uint4 *>(p.q_values + m * p.q_limit + n0);
        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
    p.q_scales[mx_scale_at(m, n0 >> 5, p.q_limit >> 7)] = (uint8_t)scale;
}

// 32 bytes, one sector of memory.
__device__ __forceinline__ void read_sector(const void *from, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(from) : "memory");
}
__device__ __forceinline__ void write_sector(void *to, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
// What is added to a warp's 32 rows x 16 columns: the lane's row, 32 bytes.  Where rows are not whole sectors (vec below 3) or the piece of the matrix is not whole,
// it passes through the warp's piece of shared memory, neighbouring lanes at neighbouring elements.
__device__ __forceinline__ void read_added(uint32_t (&in)[8], const uint16_t *first, int64_t ld, int rows) {
    const int lane = threadIdx.x & 31;
    if (lane < rows) read_sector(first + lane * ld, in);
}
// (The functions that are not inlined take no arrays, which would have to be in memory.  The kernels are laid out not to spill, and the build refuses them otherwise; builds
// held to 64 and 72 registers, which spill 12 to 356 bytes around these calls, gave the same results.)
__device__ __noinline__ void land16(const uint16_t *first, int64_t ld, int rows, int n, uint8_t *piece) {
    const int lane = threadIdx.x & 31, c = lane & 15;
    uint16_t v[16];                                              // two rows a pass, all on their way
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = 2 * k + (lane >> 4) < rows && c < n ? first[(2 * k + (lane >> 4)) * ld + c] : (uint16_t)0;
#pragma unroll
    for (int k = 0; k < 16; ++k) *word_of<uint16_t>(piece, 2 * k + (lane >> 4), c) = v[k];
    __syncwarp();
}
__device__ __forceinline__ void pass_added(uint32_t (&in)[8], const uint16_t *first, int64_t ld, int rows, int n, uint8_t *piece) {
    land16(first, ld, rows, n, piece);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 w = *unit_of(piece, threadIdx.x & 31, i);
        in[4 * i] = w.x; in[4 * i + 1] = w.y; in[4 * i + 2] = w.z; in[4 * i + 3] = w.w;
    }
    __syncwarp();
}
__device__ __noinline__ void flush_out(uint16_t *first, int64_t ld, int vec, int rows, int n, uint8_t *piece) { flush<uint16_t, 16>(first, ld, vec, rows, n, piece); }
__device__ __forceinline__ void flush_pre(float *first, int64_t ld, int vec, int rows, int n, uint8_t *piece) { flush<float, 16>(first, ld, vec, rows, n, piece); }
// Sixteen values of the lane's row, as words, to rows that are not whole sectors.
__device__ __forceinline__ void pass_out(const uint32_t (&w)[8], uint16_t *first, int64_t ld, int vec, int rows, int n, uint8_t *piece) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *unit_of(piece, threadIdx.x & 31, i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    flush_out(first, ld, vec, rows, n, piece);
}
__device__ __forceinline__ void keep(const MxCommon &p, int64_t row, int64_t n0, int rows, int n, uint8_t *piece, const float (&v)[16]) {
    float *to = p.pre + row * p.ldp + n0;
    if (p.vec_pre == 3 && n == 16) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * i + j]);
            if ((int)(threadIdx.x & 31) < rows) write_sector(to + (threadIdx.x & 31) * p.ldp + 8 * i, w);
        }
    } else {
        put16<float>(piece, 0, v);
        flush_pre(to, p.ldp, p.vec_pre < 2 ? p.vec_pre : 2, rows, n, piece);
    }
}

// A warp's 32 rows from m0 on, sixteen columns from n0 on, one row a lane: accumulators a (and b: gated), what is added in `in`.  One short path that all
// warps run through again and again: blocks of 32 columns and both halves unrolled waited for instructions a fifth of the time.
enum { OUT_PLAIN, OUT_PRE, OUT_MX };
template <int EPI, typename T, bool PRE>
__device__ __forceinline__ void finish16(const MxCommon &p, const Output &q, int64_t m0, int64_t n0, bool adds, const uint32_t (&in)[8], uint8_t *piece, float (&a)[16], float (&b)[16]) {
    constexpr bool GATED = EPI == BNN_EPI_GATED;
    const int lane = threadIdx.x & 31, rows = (int)(q.M - m0 < 32 ? q.M - m0 : 32), n = (int)(q.N - n0 < 16 ? q.N - n0 : 16);
    if (!GATED && p.bias) add_bias16<T>(bias_of(p, n0, n), a);
    if constexpr (PRE) {
        keep(p, m0, n0, rows, n, piece, a);
        if constexpr (GATED) keep(p, q.M + m0, n0, rows, n, piece, b);
    }
    activate(p.act, a);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (GATED) { a[2 * j] *= b[2 * j]; a[2 * j + 1] *= b[2 * j + 1]; }
        else if (adds) {
            const float2 d = unpack2<T>(in[j]);
            a[2 * j] += d.x; a[2 * j + 1] += d.y;
        }
        w[j] = pack2<T>(a[2 * j], a[2 * j + 1]);
    }
    uint16_t *to = static_cast<uint16_t *>(q.out[0]) + m0 * q.ldo[0] + n0;
    if (q.vec_out == 3 && n == 16) {
        if (lane < rows) write_sector(to + lane * q.ldo[0], w);
    } else pass_out(w, to, q.ldo[0], q.vec_out < 2 ? q.vec_out : 2, rows, n, piece);
}
// 32 columns for a microscaled result.  held: its columns of the accumulator that has been taken out of tensor memory, the only one or, gated, the
// gate's (UP false) or the other (UP true); the second comes from `acc`.
template <int EPI, typename T, bool UP>
__device__ __forceinline__ void finish_mx(const MxCommon &p, const Output &q, int64_t m0, int64_t n0, uint32_t acc, const uint32_t (&held)[32]) {
    constexpr bool GATED = EPI == BNN_EPI_GATED;
    const int n = (int)(q.N - n0 < BLOCK ? q.N - n0 : BLOCK);
    float all[32];
#pragma unroll
    for (int c = 0; c < BLOCK; c += CHUNK) {
        float a[16], b[16];
        if constexpr (GATED) {
            uint32_t r[16];
            tmem_ld16(acc + c, r);
            tmem_ld_wait16(r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                a[j] = __uint_as_float(UP ? r[j] : held[c + j]);
                b[j] = __uint_as_float(UP ? held[c + j] : r[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) a[j] = __uint_as_float(held[c + j]);
            if (p.bias && n > c) add_bias16<T>(bias_of(p, n0 + c, n - c < 16 ? n - c : 16), a);
        }
        activate(p.act, a);
#pragma unroll
        for (int j = 0; j < 16; ++j) all[c + j] = GATED ? a[j] * b[j] : a[j];
    }
    write_block(p, q, m0 + (threadIdx.x & 31), n0, all);
}

// ---------------------------------------------------------------------------------------------------------
// Many rows: k_mx_pair, the pair kernel of the 16-bit products (two CTAs on one 256 x 256 tile, persistent) with scales beside the elements.
//   warp 0        TMA producer of x: 128 rows of this CTA and their scales
//   last warp     TMA producer of the weights: this CTA's half of the tile's columns, and the scales of all of them (each tensor core needs those of
//                 every column)
//   warp 1        MMA issuer (CTA 0): scales to tensor memory, then up to four instructions a stage
//   the others    epilogue
// Each of the two producers makes every K step, so the ring may have any number of stages: a stage is full with the bytes of all four.  (Six or eight stages instead of
// five changed nothing at any size.)  Issuer and producers run warp-wide with one elected lane: a single lane of a divergent warp took about 1100 clocks a K step
// of ten instructions, 8192 x 8192 x 8192 in 4 bits 287 us.  One issuing lane keeps the order of the additions fixed: the same call gives the same bits.
// Tensor memory: two accumulators of 256 columns and 48 of scales are more than there is.  The accumulators overlap by 64 columns: the epilogue
// takes the columns that they share first, from above in the first one and from below in the second, and hands them over before it computes (handed over after the
// first block instead: 8192 x 4096 -> 8192 in 4 bits 116 us).  A lane writes and adds whole 32-byte sectors of its own row; through shared memory, as rows that are not whole
// sectors go, the same took 24 instead of 19 us at K = 128.  The residual's lines brought to L2 during the tile before made it slower (117 -> 124 us).
constexpr int STAGES = 5, BAND = 8, EPI_WARPS = 16, PAIR_THREADS = (EPI_WARPS + 3) * 32;
constexpr uint32_t STAGE = 35 * 1024, X_SCALES = 2 * ROWS128, W_SCALES = X_SCALES + 1024;       // x, weights, scales of x, scales of weights
constexpr uint32_t ACC2 = 192, SCALES = 448, SCALE_SET = 32;      // columns: second accumulator, scales (two sets: 8 of x, 16 of weights)
constexpr int SHARED = 64;               // columns that both accumulators have
static_assert(ACC2 + SHARED == 256, "of 256 each");
// Half-width tiles (128 columns, dense layer only) where whole ones would leave half of the pairs without work: their accumulators share nothing.
template <int BN> constexpr uint32_t second_acc() { return BN == 256 ? ACC2 : 128; }

struct PairArgs : MxCommon {
    Output q;
    MxMaps maps;
    uint32_t tiles, tiles_m, tiles_n;
};
struct __align__(16) Control {
    uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty, drain;
    uint32_t tmem_base, failed;
};
__device__ __forceinline__ void fail(Control *ctl, int code) {
    *reinterpret_cast<volatile uint32_t *>(&ctl->failed) = (uint32_t)code;
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&ctl->failed)), "r"(cluster_ctarank() ^ 1u));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote), "r"((uint32_t)code) : "memory");
    atomicCAS(&g_mx_error, 0, code);
}
template <int WIDTH> __device__ __forceinline__ void tile_at(const PairArgs &p, uint32_t t, int &m0, int &n0) {
    const uint32_t band = t / (BAND * p.tiles_n), w = t - band * BAND * p.tiles_n;
    const uint32_t high = p.tiles_m - band * BAND < BAND ? p.tiles_m - band * BAND : BAND, n = w / high;
    m0 = (int)((band * BAND + w - n * high) * 256);
    n0 = (int)(n * WIDTH);
}

template <bool FOUR, int BN> __device__ __forceinline__ void issue_pair(const PairArgs &p, Control *ctl, uint8_t *tiles, uint32_t tmem, uint32_t pair, uint32_t pairs) {
    uint32_t stage = 0, phase = 0, count = 0, set = 0;
    bool ok = true;
    const uint64_t a0 = smem_desc_sw128(smem_u32(tiles)), b0 = smem_desc_sw128(smem_u32(tiles + ROWS128));
    const uint64_t xs0 = scale_desc(smem_u32(tiles + X_SCALES)), ws0 = scale_desc(smem_u32(tiles + W_SCALES));
    const int k_iters = p.q.k_iters;
    constexpr int GROUPS = FOUR ? 2 : 1;
    for (uint32_t t = pair; t < p.tiles && ok; t += pairs, ++count) {
        if (count > 0 && !warp_wait(ctl, p.wait_ns, &ctl->acc_empty, (count - 1) & 1)) { fail(ctl, 4); ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + (count & 1) * second_acc<BN>();
        for (int kit = 0; kit < k_iters; ++kit) {
            if (!warp_wait(ctl, p.wait_ns, &ctl->full[stage], phase)) { fail(ctl, 2); ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t at = (uint64_t)(stage * (STAGE >> 4));
            const uint32_t sx = tmem + SCALES + set * SCALE_SET, sw = sx + 8;
            if (elected()) {
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    copy_scales<2>(sx + 4 * g, xs0 + at + 32 * g);
                    copy_scales<2>(sw + 8 * g, ws0 + at + 32 * g);                        // columns 0 .. 127 of the tile
                    if (BN == 256) copy_scales<2>(sw + 8 * g + 4, ws0 + at + 32 * (GROUPS + g));         // and 128 .. 255
                }
                step_mx<2, FOUR>(d, a0 + at, b0 + at, p.idesc, sx, sw, 8, kit == k_iters - 1 ? p.last : 4, kit == 0);
                umma_commit_2sm(smem_u32(&ctl->empty[stage]));
            }
            __syncwarp();
            set ^= 1;
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (elected()) umma_commit_2sm(smem_u32(&ctl->acc_full[count & 1]));
        __syncwarp();
    }
    if (elected()) umma_commit_2sm(smem_u32(&ctl->drain));      // the MMAs issued end before tensor memory is given back, also where nobody waits for them any more
    __syncwarp();
    warp_wait(ctl, DRAIN_NS, &ctl->drain, 0, false);
}

template <int EPI, int OUT, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PAIR_THREADS, 1) k_mx_pair(const __grid_constant__ PairArgs p) {
    constexpr bool GATED = EPI == BNN_EPI_GATED;
    constexpr int WIDTH = GATED ? BN / 2 : BN, PARTS = EPI_WARPS / 4;
    static_assert(BN == 256 || (BN == 128 && !GATED), "gate and up rows of a tile begin with a tile of scales each");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Control *ctl = reinterpret_cast<Control *>(tiles + STAGES * STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        for (int b = 0; b < 2; ++b) mbar_init(smem_u32(&ctl->acc_full[b]), 1);
        mbar_init(smem_u32(&ctl->acc_empty), 2 * EPI_WARPS);
        mbar_init(smem_u32(&ctl->drain), 1);
        ctl->failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                          // both CTAs' barriers exist before anyone signals them
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = ctl->tmem_base;

    if (warp == 0 || warp == 2 + EPI_WARPS) {
        // ---------------- producers.  The "full" barrier of a stage (in CTA 0) completes with the arrival of CTA 0's first producer and the bytes of both
        // producers of both CTAs.
        if (!p.drop_loads) {
            const bool weights = warp != 0;
            const int groups = p.four ? 2 : 1;      // of 128 columns in a stage; the coordinate of the elements counts bytes, or nibbles on their way to bytes: 128 a stage
            bool ok = true;
            uint32_t stage = 0, lap = 0;
            bnn_pdl_wait();
            for (uint32_t t = pair; t < p.tiles && ok; t += pairs) {
                int m0, n0;
                tile_at<WIDTH>(p, t, m0, n0);
                m0 += (int)rank * 128;
                for (int kit = 0; kit < p.q.k_iters; ++kit) {
                    if (lap > 0 && !warp_wait(ctl, p.wait_ns, &ctl->empty[stage], (lap - 1) & 1)) { fail(ctl, 1); ok = false; break; }
                    const uint32_t dst = smem_u32(tiles + stage * STAGE), bar = smem_u32(&ctl->full[stage]) & PEER_MASK;
                    if (!elected()) {
                    } else if (!weights) {
                        if (rank == 0) mbar_expect_tx(smem_u32(&ctl->full[stage]), 2 * (ROWS128 + p.w_bytes * (BN / 2) / 128 + (1 + BN / 128) * groups * BNN_MX_TILE));
                        tma_load_2d_2sm(dst, &p.maps.x, kit * 128, m0, bar);
                        tma_load_3d_2sm(dst + X_SCALES, &p.maps.xs, 0, kit * groups, m0 >> 7, bar);
                    } else if (GATED) {
                        tma_load_2d_2sm(dst + ROWS128, &p.maps.w[rank], kit * 128, n0, bar);
                        tma_load_3d_2sm(dst + W_SCALES, &p.maps.ws[0], 0, kit * groups, n0 >> 7, bar);
                        tma_load_3d_2sm(dst + W_SCALES + groups * BNN_MX_TILE, &p.maps.ws[1], 0, kit * groups, n0 >> 7, bar);
                    } else {
                        tma_load_2d_2sm(dst + ROWS128, &p.maps.w[0], kit * 128, n0 + (int)rank * (BN / 2), bar);
                        tma_load_3d_2sm(dst + W_SCALES, &p.maps.ws[0], 0, kit * groups, n0 >> 7, bar);
                    }
                    __syncwarp();
                    if (++stage == STAGES) { stage = 0; ++lap; }
                }
            }
            // The copies in flight land before the CTA gives its shared memory up.  Waited for in every case: whether one of the other waits gives up
            // may be decided after this thread has requested everything.
            if (rank == 0)
                for (uint32_t i = 0, s = stage, l = lap; i < (uint32_t)STAGES; ++i) {      // this thread's last uses, newest first
                    if (s == 0) { if (l == 0) break; s = STAGES; --l; }
                    --s;
                    if (!warp_wait(ctl, DRAIN_NS, &ctl->full[s], l & 1, false)) break;
                }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            if (p.four) issue_pair<true, BN>(p, ctl, tiles, tmem_base, pair, pairs);
            else issue_pair<false, BN>(p, ctl, tiles, tmem_base, pair, pairs);
        }
    } else if (warp < 2 + EPI_WARPS) {
        bnn_pdl_wait();
        bnn_pdl_launch_next();
        const Output &q = p.q;
        const int quad = warp & 3, part = (warp - 2) >> 2;
        uint8_t *piece = reinterpret_cast<uint8_t *>(ctl + 1) + (warp - 2) * PIECE;
        uint32_t count = 0;
        for (uint32_t t = pair; t < p.tiles; t += pairs, ++count) {
            const uint32_t buf = count & 1;
            int tm0, tn0;
            tile_at<WIDTH>(p, t, tm0, tn0);
            const int64_t m0 = tm0 + (int)rank * 128 + 32 * quad;
            const int rows = (int)(q.M - m0 < 32 ? q.M - m0 : 32);
            const uint32_t acc = tmem_base + buf * second_acc<BN>() + ((uint32_t)(32 * quad) << 16);
            // the i-th piece of this warp: from above in the first accumulator, from below in the second, so that what they share comes first
            constexpr int EACH = OUT == OUT_MX ? BLOCK : CHUNK, PIECES = WIDTH / EACH, MINE = PIECES / PARTS;
            static_assert(SHARED / EACH <= PARTS, "what is shared is among the warps' first pieces");
            static_assert(PIECES % PARTS == 0, "every warp has as many pieces");
            const auto column_of = [&](int i) { const int k = i * PARTS + part; return (buf ? k : PIECES - 1 - k) * EACH; };
            const bool adds = OUT != OUT_MX && !GATED && p.add != nullptr;
            const uint16_t *add = static_cast<const uint16_t *>(p.add) + m0 * p.ld_add + tn0;
            uint32_t in[8];
            const auto ask = [&](int i) {
                const int c = column_of(i);
                if (adds && p.vec_add == 3 && rows > 0 && q.N - tn0 - c >= CHUNK) read_added(in, add + c, p.ld_add, rows);
            };
            // The residual is requested a piece ahead, the first one while the tile is being multiplied; not beside kept pre-activations (4096 x 2048 -> 4096, gelu: 55.0 us, ahead 58.6).
            constexpr bool AHEAD = OUT == OUT_PLAIN;
            if (AHEAD) ask(0);
            const auto hand_over = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_cta0(smem_u32(&ctl->acc_empty));
            };
            if (BN == 128) hand_over();                          // the tile before, whose columns the next one writes, is done
            if (!warp_wait(ctl, p.wait_ns, &ctl->acc_full[buf], (count >> 1) & 1)) { fail(ctl, 3); break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            // Gated: the accumulators share columns of the up rows of the first and of the gate rows of the second.
            const uint32_t first = acc + (GATED && !buf ? WIDTH : 0), second = acc + (GATED && buf ? WIDTH : 0);
#pragma unroll 1
            for (int i = 0; i < MINE; ++i) {
                const int c = column_of(i), n = (int)(q.N - tn0 - c);
                uint32_t r[EACH], other[CHUNK];
                if constexpr (OUT == OUT_MX) {
                    tmem_ld32(first + c, r);
                    tmem_ld_wait(r);
                } else {
                    tmem_ld16(acc + c, r);
                    if (GATED) tmem_ld16(acc + WIDTH + c, other);
                    tmem_ld_wait16(r);
                    if (GATED) tmem_ld_wait16(other);
                }
                if (BN == 256 && i == 0) hand_over();            // this warp has read its share of the columns that the next tile's MMAs write
                const bool there = rows > 0 && (OUT == OUT_MX ? tn0 + c < p.q_limit : n > 0);
                if constexpr (OUT == OUT_MX) {
                    if (!there) continue;
                    if (GATED && !buf) finish_mx<EPI, __nv_bfloat16, GATED>(p, q, m0, tn0 + c, second + c, r);      // without bias nothing is of the 16-bit type
                    else if (!GATED && p.f16) finish_mx<EPI, __half, false>(p, q, m0, tn0 + c, second + c, r);
                    else finish_mx<EPI, __nv_bfloat16, false>(p, q, m0, tn0 + c, second + c, r);
                } else if (there) {
                    if (!AHEAD) ask(i);
                    if (adds && (p.vec_add != 3 || n < CHUNK)) pass_added(in, add + c, p.ld_add, rows, n < CHUNK ? n : CHUNK, piece);
                    float a[CHUNK], b[CHUNK];
#pragma unroll
                    for (int j = 0; j < CHUNK; ++j) {
                        a[j] = __uint_as_float(r[j]);
                        if (GATED) b[j] = __uint_as_float(other[j]);
                    }
                    if (p.f16) finish16<EPI, __half, OUT == OUT_PRE>(p, q, m0, tn0 + c, adds, in, piece, a, b);
                    else finish16<EPI, __nv_bfloat16, OUT == OUT_PRE>(p, q, m0, tn0 + c, adds, in, piece, a, b);
                }
                if (AHEAD && i + 1 < MINE) ask(i + 1);
            }
        }
    }

    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (rank != 0 && threadIdx.x == 0) wait(ctl, DRAIN_NS, &ctl->drain, 0, false);       // the issuer's signals have reached this CTA as well
    __syncwarp();
    cluster_sync_all();                                          // nobody leaves while the peer may still reach its shared memory
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t *>(&ctl->failed) != 0u) {
        // After a failure one CTA may have requested a step that the other has not, whose barrier then never completes: both stay until such
        // copies have landed.
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < SETTLE_NS) {}
    }
    __syncwarp();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
    }
}
constexpr size_t PAIR_SMEM = (size_t)STAGES * STAGE + sizeof(Control) + EPI_WARPS * PIECE + 1024;
static_assert(PAIR_SMEM <= 227 * 1024, "fits the shared memory of an SM");
static_assert(BNN_MX_TILE * 3 * 2 + 2 * ROWS128 <= STAGE && STAGE % 1024 == 0, "a stage holds both operands and their scales");

// ---------------------------------------------------------------------------------------------------------
// Few rows (tokens): k_mx_few, the few-row kernel of the 16-bit products.  128 weight rows are the M side of the tile and the tokens its N side; the
// sum is split over a cluster, whose CTAs store their partial tiles into the shared memory of the CTAs that finish them.  Gated: 128 gate and the 128 up
// rows of the same hidden units, two accumulators.
//   warps 0 and 11  TMA producers, K steps in turn, warp 1  MMA issuer, warps 2 .. 9  partial tile to its finishers, all warps  sum and epilogue
constexpr int FEW_SMEM = 200 * 1024, FEW_THREADS = 384, FEW_STAGES = 12;
// A tile's tokens: all of them up to `whole`, otherwise 128 (gated: 64) or 64, so that a tile begins at the first or third column of a tile of scales.  Bounded so
// that a CTA takes at most half of tensor memory: CTAs of two clusters that share two SMs and wait there for each other's columns would wait for good.
constexpr int FEW_WHOLE = 192, FEW_WHOLE_GATED = 96, FEW_COLUMNS = 256;
// Shared memory that keeps an SM from holding more CTAs than its tensor memory has columns for (228 KB; 512 columns; registers allow two).
constexpr size_t FEW_SMEM_PER_COLUMN = 360;

struct FewArgs : MxCommon {
    Output q;
    MxMaps maps;
    uint32_t token_tiles;
    int tokens;                         // of a tile: N of the instructions, a multiple of 16 (several tiles: of 64)
    int stages;
    uint32_t stage_bytes, loaded, x_at, ws_at, xs_at;       // bytes of a stage and of its loads; tokens, scales of weights and of tokens in it
    uint32_t acc_up, scales, scale_set, x_pitch, tmem_cols; // columns: second accumulator, scales (two sets; a group's of the tokens), all
};
struct __align__(16) FewControl {
    uint64_t full[FEW_STAGES], empty[FEW_STAGES], acc_full;
    uint32_t tmem_base, failed;
};
__device__ __forceinline__ void few_fail(FewControl *ctl, int code) {
    *reinterpret_cast<volatile uint32_t *>(&ctl->failed) = (uint32_t)code;
    atomicCAS(&g_mx_error, 0, code);
}

template <bool FOUR, bool GATED> __device__ __forceinline__ void issue_few(const FewArgs &f, FewControl *ctl, uint8_t *tiles, uint32_t tmem, int first, int last, int shift) {
    constexpr int GROUPS = FOUR ? 2 : 1, HALVES = GATED ? 2 : 1;
    const uint64_t a0 = smem_desc_sw128(smem_u32(tiles)), b0 = smem_desc_sw128(smem_u32(tiles + f.x_at));
    const uint64_t ws0 = scale_desc(smem_u32(tiles + f.ws_at)), xs0 = scale_desc(smem_u32(tiles + f.xs_at));
    const int x_tiles = f.tokens > 128 ? 2 : 1;
    int stage = 0;
    uint32_t phase = 0, set = 0;
    for (int kit = first; kit < last; ++kit) {
        if (!warp_wait(ctl, f.wait_ns, &ctl->full[stage], phase)) { few_fail(ctl, 22); break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t at = (uint64_t)(stage * (f.stage_bytes >> 4));
        // a set: for each group of 128 of K four columns of each half's weights, then for each group those of the tokens
        const uint32_t sw = tmem + f.scales + set * f.scale_set, sx = sw + 4 * GROUPS * HALVES;
        const int count = kit == f.q.k_iters - 1 ? f.last : 4;
        if (elected()) {
#pragma unroll
            for (int i = 0; i < GROUPS * HALVES; ++i) copy_scales<1>(sw + 4 * i, ws0 + at + 32 * i);
            for (int i = 0; i < x_tiles; ++i)
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) copy_scales<1>(sx + f.x_pitch * g + 4 * i, xs0 + at + 32 * (i * GROUPS + g));
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
                step_mx<1, FOUR>(tmem + h * f.acc_up, a0 + at + h * (ROWS128 >> 4), b0 + at, f.idesc, sw + 4 * GROUPS * h, sx + shift, f.x_pitch, count, kit == first);
            mma_commit(&ctl->empty[stage]);
        }
        __syncwarp();
        set ^= 1;
        if (++stage == f.stages) { stage = 0; phase ^= 1; }
    }
    if (elected()) mma_commit(&ctl->acc_full);
    __syncwarp();
    warp_wait(ctl, DRAIN_NS, &ctl->acc_full, 0, false);       // the MMAs issued end before tensor memory is given back, also where the epilogue has given up
}

template <int ACT> __device__ __forceinline__ void act4(float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = act_value(ACT, v[j]);
}
// Four neighbouring outputs of one token from their sums; bias and what is added have been read.
template <int EPI, typename T>
__device__ __forceinline__ void finish_few(const MxCommon &p, const Output &q, int64_t m, int64_t n0, float (&a)[4], float (&b)[4], const float (&bias)[4], const float (&add)[4]) {
    constexpr bool GATED = EPI == BNN_EPI_GATED;
    const int n = (int)(q.N - n0 < 4 ? q.N - n0 : 4);
    if (!GATED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] += bias[j];
    }
    if (p.pre) {
        write4(p.pre + m * p.ldp + n0, n, p.vec_pre, a);
        if (GATED) write4(p.pre + (q.M + m) * p.ldp + n0, n, p.vec_pre, b);
    }
#define BNN_CALL(ACT) act4<ACT>(a)
    BNN_EACH_ACT(BNN_CALL)
#undef BNN_CALL
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = GATED ? a[j] * b[j] : a[j] + add[j];
    write4(static_cast<T *>(q.out[0]) + m * q.ldo[0] + n0, n, q.vec_out, a);
}
// The same, microscaled: eight neighbouring lanes hold a block.  All lanes of the warp take part; `there`: the token exists.
template <int EPI>
__device__ __forceinline__ void finish_few_mx(const MxCommon &p, const Output &q, int64_t m, int64_t n0, bool there, float (&a)[4], float (&b)[4], const float (&bias)[4]) {
    const int n = (int)(q.N - n0 < 4 ? (q.N > n0 ? q.N - n0 : 0) : 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] += EPI == BNN_EPI_GATED ? 0.0f : bias[j];
#define BNN_CALL(ACT) act4<ACT>(a)
    BNN_EACH_ACT(BNN_CALL)
#undef BNN_CALL
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (EPI == BNN_EPI_GATED) a[j] *= b[j];
        a[j] = j < n ? a[j] : 0.0f;
        top = max(top, mx_magnitude(a[j]));
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t scale = p.q_four ? mx_scale<true>(top) : mx_scale<false>(top);
    const float down = mx_down(scale), e[8] = {a[0] * down, a[1] * down, a[2] * down, a[3] * down, 0.0f, 0.0f, 0.0f, 0.0f};
    if (!there || n0 >= p.q_limit) return;
    uint32_t w[2];
    if (p.q_four) { mx_encode8<true>(e, w); *reinterpret_cast<uint16_t *>(p.q_values + m * (p.q_limit / 2) + n0 / 2) = (uint16_t)w[0]; }
    else { mx_encode8<false>(e, w); *reinterpret_cast<uint32_t *>(p.q_values + m * p.q_limit + n0) = w[0]; }
    if ((threadIdx.x & 7) == 0) p.q_scales[mx_scale_at(m, n0 >> 5, p.q_limit >> 7)] = (uint8_t)scale;
}
// Four 16-bit values as float32, n of them inside; zeros without a matrix.
__device__ __forceinline__ void read_half4(const MxCommon &p, const void *base, int64_t at, int n, int vec, float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = 0.0f;
    if (!base || n <= 0) return;
    if (p.f16) read4(static_cast<const __half *>(base) + at, n, vec, v);
    else read4(static_cast<const __nv_bfloat16 *>(base) + at, n, vec, v);
}

template <int EPI, bool MX> __global__ void __launch_bounds__(FEW_THREADS, 2) k_mx_few(const __grid_constant__ FewArgs f) {
    constexpr bool GATED = EPI == BNN_EPI_GATED;
    constexpr int HALVES = GATED ? 2 : 1;
    const Output &q = f.q;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ FewControl control;
    FewControl *ctl = &control;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    uint32_t split;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    const uint32_t tile = blockIdx.x / split, tn = tile / f.token_tiles, tt = tile - tn * f.token_tiles;     // tiles of the same weights next to each other
    const int64_t n0 = (int64_t)tn * 128, t0 = (int64_t)tt * f.tokens;
    const int first = (int)((int64_t)q.k_iters * rank / split), last = (int)((int64_t)q.k_iters * (rank + 1) / split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < f.stages; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        mbar_init(smem_u32(&ctl->acc_full), 1);
        ctl->failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(f.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = ctl->tmem_base;
    const bool loads = loads_here(f.drop_loads, split, rank);
    if ((warp == 0 || warp == FEW_THREADS / 32 - 1) && loads) {
        // While the kernel before this one runs, the first weights are brought to L2.  (Only to L2, where its writes are seen: it may have made them.)
        const int mine = warp == 0 ? 0 : 1, groups = f.four ? 2 : 1;
        if (elected())
            for (int kit = first + mine; kit < last && kit < first + f.stages; kit += 2)
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&f.maps.w[h]), "r"(kit * 128), "r"((int)n0) : "memory");
                    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(&f.maps.ws[h]), "r"(0), "r"(kit * groups), "r"((int)(n0 >> 7)) : "memory");
                }
        __syncwarp();
    }
    bnn_pdl_wait();
    bnn_pdl_launch_next();

    if (warp == 0 || warp == FEW_THREADS / 32 - 1) {
        if (loads) {
            const int mine = warp == 0 ? 0 : 1, groups = f.four ? 2 : 1;
            int stage = mine % f.stages, lap = mine / f.stages;
            for (int kit = first + mine; kit < last; kit += 2) {
                if (lap > 0 && !warp_wait(ctl, f.wait_ns, &ctl->empty[stage], (lap - 1) & 1)) { few_fail(ctl, 21); break; }
                const uint32_t dst = smem_u32(tiles) + stage * f.stage_bytes, bar = smem_u32(&ctl->full[stage]);
                if (elected()) {
                    mbar_expect_tx(bar, f.loaded);
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) {
                        tma_load_2d(dst + h * ROWS128, &f.maps.w[h], kit * 128, (int)n0, bar);
                        tma_load_3d(dst + f.ws_at + h * groups * BNN_MX_TILE, &f.maps.ws[h], 0, kit * groups, (int)(n0 >> 7), bar);
                    }
                    tma_load_2d(dst + f.x_at, &f.maps.x, kit * 128, (int)t0, bar);
                    tma_load_3d(dst + f.xs_at, &f.maps.xs, 0, kit * groups, (int)(t0 >> 7), bar);
                }
                __syncwarp();
                stage += 2;
                while (stage >= f.stages) { stage -= f.stages; ++lap; }
            }
            for (int i = 0, s = stage, l = lap; i < f.stages; i += 2) {            // copies in flight land before the shared memory is given up, as above
                s -= 2;
                while (s < 0) { s += f.stages; --l; }
                if (l < 0 || !warp_wait(ctl, DRAIN_NS, &ctl->full[s], l & 1, false)) break;
            }
        }
    } else if (warp == 1) {
        const int shift = (int)(t0 >> 5) & 3;        // columns of the first token within its tile of scales
        if (f.four) issue_few<true, GATED>(f, ctl, tiles, tmem_base, first, last, shift);
        else issue_few<false, GATED>(f, ctl, tiles, tmem_base, first, last, shift);
    }
    // Rank r finishes the tile's outputs r * out .. r * out + out - 1 of every token.  A lane of warps 2 .. 9 holds one weight row of the
    // partial tile and stores it where it is needed: parts[rank it comes from][token][row of the finishing rank's share], the gate rows of
    // a share before its up rows, in the finishing CTA's ring, which is free once all MMAs of the cluster are done (first barrier).
    const int log = split == 8 ? 3 : (int)split >> 1, out = 128 >> log, share = out * HALVES, pitch = f.tokens * share;
    float *parts = reinterpret_cast<float *>(tiles);
    const int valid = (int)(q.M - t0 < f.tokens ? q.M - t0 : f.tokens);
    // A thread finishes four outputs of token after token, the same four: their bias, and what is added to the first of them, are requested here.
    static_assert(FEW_THREADS % 32 == 0, "a multiple of out / 4 for every split");
    const int row = (int)threadIdx.x % (out / 4) * 4, n_mine = (int)(q.N - n0 - (int)rank * out - row);
    const int64_t n_at = n0 + (int)rank * out + row;
    float bias[4], add[4];
    if (!GATED) {
        read_half4(f, f.bias, n_at, n_mine < 4 ? n_mine : 4, f.vec_bias, bias);
        const int t = (int)threadIdx.x / (out / 4);
        if (!MX) read_half4(f, f.add, (t0 + t) * f.ld_add + n_at, t < valid ? (n_mine < 4 ? n_mine : 4) : 0, f.vec_add, add);
    }
    bool done = false;
    if (warp >= 2 && warp < 10) {
        done = warp_wait(ctl, 2 * f.wait_ns, &ctl->acc_full, 0, false);
        if (!done) few_fail(ctl, 23);
    }
    __syncwarp();
    if (split > 1) {
        cluster_sync_all();
        tell_cluster(ctl, split);
    } else __syncthreads();
    if (__all_sync(0xffffffffu, done && *reinterpret_cast<volatile uint32_t *>(&ctl->failed) == 0u)) {       // the flag may come from another CTA now
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int quad = warp & 3, row = 32 * quad + lane, owner = row / out;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const uint32_t to = in_cta(smem_u32(parts + (int)rank * pitch + row - owner * out + h * out), (uint32_t)owner);
            for (int c = warp < 6 ? 0 : 16; c < f.tokens; c += 32) {
                if (c >= valid) break;
                uint32_t r[16];
                tmem_ld16(tmem_base + h * f.acc_up + ((uint32_t)(32 * quad) << 16) + c, r);
                tmem_ld_wait16(r);
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (c + j < valid)
                        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + (uint32_t)((c + j) * share) * 4), "r"(last > first ? r[j] : 0u) : "memory");
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    if (split > 1) cluster_sync_all();
    else __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(f.tmem_cols) : "memory");
    }
    if (*reinterpret_cast<volatile uint32_t *>(&ctl->failed) != 0u) return;
    const int all = valid * (out / 4);
    if (!MX && n_mine <= 0) return;
    for (int i = threadIdx.x; MX ? i - lane < all : i < all; i += FEW_THREADS) {      // microscaled: a warp stays together
        const bool there = i < all;
        const int t = there ? i / (out / 4) : 0;
        float a[4], b[4];
        sum_parts(parts + t * share + row, (int)split, pitch, a);
        if (GATED) sum_parts(parts + t * share + out + row, (int)split, pitch, b);
        if constexpr (MX) finish_few_mx<EPI>(f, q, t0 + t, n_at, there, a, b, bias);
        else {
            if (!GATED && i != (int)threadIdx.x) read_half4(f, f.add, (t0 + t) * f.ld_add + n_at, n_mine < 4 ? n_mine : 4, f.vec_add, add);
            if (f.f16) finish_few<EPI, __half>(f, q, t0 + t, n_at, a, b, bias, add);
            else finish_few<EPI, __nv_bfloat16>(f, q, t0 + t, n_at, a, b, bias, add);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------
// Opts in to the shared memory and asks how many pairs fit the device, once per device and kernel; 0 = cannot run.
template <int EPI, int OUT, int BN> int pairs_of(int device, int sm_count) {
    static std::mutex lock;
    static int cached[64];
    if (device < 0 || device >= 64) return 0;
    std::lock_guard<std::mutex> guard(lock);
    if (cached[device] == 0) {
        auto kernel = k_mx_pair<EPI, OUT, BN>;
        int pairs = 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PAIR_SMEM) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(2 * sm_count); cfg.blockDim = dim3(PAIR_THREADS); cfg.dynamicSmemBytes = PAIR_SMEM;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
            cfg.attrs = &attr; cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&pairs, kernel, &cfg) != cudaSuccess) pairs = 0;
        }
        (void)cudaGetLastError();
        cached[device] = pairs > 0 ? pairs : -1;
    }
    return cached[device] > 0 ? cached[device] : 0;
}
template <int EPI, int OUT, int BN> int launch_pair(bnn_ctx *ctx, const PairArgs &a) {
    const int pairs = pairs_of<EPI, OUT, BN>(ctx->device, ctx->sm_count);
    if (pairs == 0) return BNN_ERR_CUDA;
    const unsigned n = a.tiles < (uint32_t)pairs ? a.tiles : (unsigned)pairs;
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(k_mx_pair<EPI, OUT, BN>, dim3(2 * n), dim3(PAIR_THREADS), PAIR_SMEM, ctx->stream, a));
    return bnn_check_launch(ctx);
}
template <int EPI, bool MX> int launch_few(bnn_ctx *ctx, const FewArgs &f, unsigned tiles, unsigned split) {
    auto kernel = k_mx_few<EPI, MX>;
    static std::mutex lock;
    static bool ready[64];
    if (ctx->device < 0 || ctx->device >= 64) return BNN_ERR_INVALID_ARG;
    {
        std::lock_guard<std::mutex> guard(lock);
        if (!ready[ctx->device]) BNN_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM + 1024));
        ready[ctx->device] = true;
    }
    cudaLaunchConfig_t cfg{};
    const size_t ring = (size_t)f.stages * f.stage_bytes, part = (size_t)f.tokens * 512 * (EPI == BNN_EPI_GATED ? 2 : 1);
    cfg.gridDim = dim3(tiles * split); cfg.blockDim = dim3(FEW_THREADS); cfg.stream = ctx->stream;
    cfg.dynamicSmemBytes = (ring > part ? ring : part) + 1024;
    if (cfg.dynamicSmemBytes < f.tmem_cols * FEW_SMEM_PER_COLUMN) cfg.dynamicSmemBytes = f.tmem_cols * FEW_SMEM_PER_COLUMN;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    BNN_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, kernel, f));
    return bnn_check_launch(ctx);
}

// A call: x and one or two weight matrices, and what the epilogue needs.
struct Call {
    int dtype, act, epilogue;
    const bnn_mx_matrix *x, *w[2];
    const void *bias, *add;
    int64_t ld_add;
    void *out;
    int64_t ldo;
    const bnn_mx_matrix *q;             // instead of out
    float *pre;
    int64_t ldp;
};
bool is_four(const Call &c) { return c.x->format == BNN_MX_E2M1; }
int64_t steps_of(const Call &c) { const int64_t groups = bnn_mx_groups(c.x->cols); return is_four(c) ? (groups + 1) / 2 : groups; }

// Elements: stages are rows of 128 bytes; packed nibbles as bytes, bytes as bytes, nibbles beside bytes on their way to bytes.
int map_elements(bnn_ctx *ctx, CUtensorMap *map, const bnn_mx_matrix *m, bool packed, int box_rows) {
    const int64_t pitch = bnn_mx_pitch(m->format, m->cols);
    const bool widen = m->format == BNN_MX_E2M1 && !packed;
    const uint64_t dims[2] = {(uint64_t)(widen ? 2 * pitch : pitch), (uint64_t)m->rows}, strides[1] = {(uint64_t)pitch};
    const uint32_t box[2] = {128, (uint32_t)box_rows};
    return bnn_tensor_map(ctx, map, widen ? CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m->values, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
int map_scales(bnn_ctx *ctx, CUtensorMap *map, const bnn_mx_matrix *m, int groups, int tiles) {
    const uint64_t all = (uint64_t)bnn_mx_groups(m->cols), dims[3] = {BNN_MX_TILE / 4, all, (uint64_t)((m->rows + 127) / 128)};
    const uint64_t strides[2] = {BNN_MX_TILE, all * BNN_MX_TILE};
    const uint32_t box[3] = {BNN_MX_TILE / 4, (uint32_t)groups, (uint32_t)tiles};
    return bnn_tensor_map(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, m->scales, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}
// float32 accumulators, scales E8M0 (bit 23), A m rows and B n rows; element types of the kind: mxf4 e2m1 1, mxf8f6f4 e4m3 0, e2m1 5.
uint32_t instruction(bool four, int a_format, int b_format, int n, int m) {
    const auto type = [four](int format) { return four ? 1u : format == BNN_MX_E2M1 ? 5u : 0u; };
    return type(a_format) << 7 | type(b_format) << 10 | (uint32_t)(n >> 3) << 17 | 1u << 23 | (uint32_t)(m >> 4) << 24;
}
void common_args(MxCommon &a, Output &q, bnn_ctx *ctx, const Call &c) {
    a.bias = c.bias; a.add = c.add; a.ld_add = c.ld_add; a.pre = c.pre; a.ldp = c.ldp; a.act = c.act; a.f16 = c.dtype == BNN_F16;
    a.wait_ns = ctx->wait_limit_ns; a.drop_loads = ctx->drop_loads;
    a.four = is_four(c);
    a.w_bytes = !a.four && c.w[0]->format == BNN_MX_E2M1 ? ROWS128 / 2 : ROWS128;
    q.M = c.x->rows; q.N = c.w[0]->rows; q.k_iters = (int)steps_of(c);
    q.out[0] = c.out; q.ldo[0] = c.ldo;
    const int per = a.four ? 64 : 32;
    a.last = c.x->cols ? (int)((c.x->cols - (int64_t)(q.k_iters - 1) * 4 * per + per - 1) / per) : 0;
    if (c.q) {
        a.q_values = static_cast<uint8_t *>(c.q->values); a.q_scales = static_cast<uint8_t *>(c.q->scales);
        a.q_limit = bnn_mx_groups(c.q->cols) * BNN_MX_GROUP; a.q_four = c.q->format == BNN_MX_E2M1;
    }
}
int map_operands(bnn_ctx *ctx, MxMaps &m, const Call &c, int x_rows, int x_tiles, int w_rows, int w_tiles) {
    if (c.x->cols == 0) return BNN_OK;
    const bool packed = is_four(c);
    const int groups = packed ? 2 : 1;
    if (int st = map_elements(ctx, &m.x, c.x, packed, x_rows)) return st;
    if (int st = map_scales(ctx, &m.xs, c.x, groups, x_tiles)) return st;
    for (int i = 0; i < 2; ++i) {
        if (!c.w[i]) continue;
        if (int st = map_elements(ctx, &m.w[i], c.w[i], packed, w_rows)) return st;
        if (int st = map_scales(ctx, &m.ws[i], c.w[i], groups, w_tiles)) return st;
    }
    return BNN_OK;
}

int64_t pair_tiles(const Call &c, int64_t width) { return (c.x->rows + 255) / 256 * ((c.w[0]->rows + width - 1) / width); }
bool half_width(const bnn_ctx *ctx, const Call &c) { return !c.w[1] && 2 * pair_tiles(c, 256) <= ctx->sm_count / 2; }
int product_pair(bnn_ctx *ctx, const Call &c) {
    PairArgs a{};
    common_args(a, a.q, ctx, c);
    const bool gated = c.epilogue == BNN_EPI_GATED, half = half_width(ctx, c);
    const int64_t width = gated || half ? 128 : 256, tiles = pair_tiles(c, width);
    if (tiles > 0x7fffffff) return BNN_ERR_INVALID_ARG;
    a.tiles_m = (uint32_t)((a.q.M + 255) / 256); a.tiles_n = (uint32_t)((a.q.N + width - 1) / width); a.tiles = (uint32_t)tiles;
    a.idesc = instruction(a.four, c.x->format, c.w[0]->format, half ? 128 : 256, 256);
    const auto sectors = [](const void *at, int64_t ld, int64_t rows) { return (reinterpret_cast<uintptr_t>(at) | (rows > 1 ? (uint64_t)ld * 2 : 0)) % 32 == 0 ? 3 : width_of(at, ld, rows, 2); };
    a.q.vec_out = sectors(c.out, c.ldo, a.q.M); a.vec_add = sectors(c.add, c.ld_add, a.q.M);
    a.vec_bias = width_of(c.bias, 0, 1, 2); a.vec_pre = width_of(c.pre, c.ldp, 2 * a.q.M, 4);
    if (int st = map_operands(ctx, a.maps, c, 128, 1, half ? 64 : 128, gated || half ? 1 : 2)) return st;
#define BNN_LAUNCH(EPI, BN) (c.pre ? launch_pair<EPI, OUT_PRE, BN>(ctx, a) : c.q ? launch_pair<EPI, OUT_MX, BN>(ctx, a) : launch_pair<EPI, OUT_PLAIN, BN>(ctx, a))
    return gated ? BNN_LAUNCH(BNN_EPI_GATED, 256) : half ? BNN_LAUNCH(BNN_EPI_LINEAR, 128) : BNN_LAUNCH(BNN_EPI_LINEAR, 256);
#undef BNN_LAUNCH
}

// Which kernel, and how k_mx_few divides the work, by estimates of both in microseconds, fitted to 1095 plans of seventy sizes (1 to 1000 rows, 256 x 256 to
// 8192 x 8192 weights in every pair of formats, gated ones too; calls that repeat the same weights, from L2).  The plan chosen takes 3 % longer than the best in the mean.
//   pair: 6.2 + 0.33 per K step and round of tiles; half-width tiles 4.4 + 0.29.
//   few:  4.2 for every round of CTAs, + per K step of an SM's CTAs 0.07 + 0.0022 per token of a tile, at least 0.29 where an SM has one CTA (gated 1.42 times that);
//         + 0.83 for every doubling of the split, + 0.036 per token of a CTA's share of the epilogue.
// Mostly the arrival of operands, by what was left out in copies of the pair kernel: 512 x 512 x 8192 and 512 x 4096 x 4096 in 8 bits took 20.0 and 14.0 us whole, 20.7 and
// 14.2 without the copies of scales, 20.3 and 13.8 without their loads, 17.6 and 11.8 with one of four MMAs; the rest is about 64 bytes a clock and SM from L2.
double pair_cost(const bnn_ctx *ctx, const Call &c) {
    const bool half = half_width(ctx, c);
    const int64_t tiles = pair_tiles(c, c.w[1] || half ? 128 : 256), pairs = ctx->sm_count / 2;
    return (half ? 4.4 : 6.2) + (half ? 0.29 : 0.33) * (double)steps_of(c) * (double)((tiles + pairs - 1) / pairs);
}
constexpr int FEW_RESIDENT[2][4] = {{148, 148, 132, 120}, {296, 296, 284, 264}};      // bnn_product.cu
struct FewPlan { int64_t tiles; int token_tiles, tokens, split, per_sm; double cost; };
FewPlan few_plan(const Call &c) {
    const int64_t steps = steps_of(c), weight_tiles = (c.w[0]->rows + 127) / 128, M = c.x->rows;
    const int halves = c.w[1] ? 2 : 1;
    FewPlan best{};
    best.cost = 1e30;
    int64_t last = 0;
    for (int most : {halves == 2 ? FEW_WHOLE_GATED : FEW_WHOLE, 128, 64}) {
        FewPlan f{};
        const int64_t token_tiles = (M + most - 1) / most;
        if (token_tiles == last || token_tiles > 1 << 20 || (token_tiles > 1 && most % 64) || (halves == 2 && most > FEW_WHOLE_GATED)) continue;
        if (token_tiles > 1 && most > 128) continue;
        last = token_tiles;
        f.token_tiles = (int)token_tiles;
        f.tokens = token_tiles > 1 ? most : (int)((M + 15) / 16 * 16);
        f.tiles = weight_tiles * token_tiles;
        for (int log = 0; log < (c.q ? 3 : 4); ++log) {            // microscaled results: a CTA finishes whole blocks
            f.split = 1 << log;
            if (log && steps < f.split * 2) break;
            const int64_t ctas = f.tiles * f.split;
            f.per_sm = ctas > FEW_RESIDENT[0][log] && f.tokens <= 64 ? 2 : 1;      // half of an SM's memory still holds four stages of 64 tokens
            const int64_t resident = FEW_RESIDENT[f.per_sm - 1][log], rounds = (ctas + resident - 1) / resident;
            const double load = (double)(rounds > 1 ? rounds * f.per_sm : (ctas + 147) / 148), cta_steps = (double)((steps + f.split - 1) / f.split);
            double step = 0.07 + 0.0022 * f.tokens;
            if (f.per_sm == 1 && step < 0.29) step = 0.29;
            f.cost = 4.2 * (double)rounds + load * cta_steps * step * (halves == 2 ? 1.42 : 1.0) + 0.83 * log - 0.7 + 0.036 * f.tokens * halves / f.split * load;
            if (f.cost < best.cost) best = f;
        }
    }
    return best;
}
int product_few(bnn_ctx *ctx, const Call &c, const FewPlan &plan) {
    if (plan.tiles * plan.split > 0x7fffffff) return BNN_ERR_INVALID_ARG;
    FewArgs f{};
    common_args(f, f.q, ctx, c);
    const auto fours = [](const void *at, int64_t ld, int64_t n, int size) { return reinterpret_cast<uintptr_t>(at) % (4 * size) == 0 && (n <= 1 || ld % 4 == 0); };
    f.vec_bias = fours(c.bias, 0, 1, 2); f.vec_add = fours(c.add, c.ld_add, f.q.M, 2); f.vec_pre = fours(c.pre, c.ldp, 2 * f.q.M, 4);
    f.q.vec_out = fours(c.out, c.ldo, f.q.M, 2);
    f.tokens = plan.tokens; f.token_tiles = (uint32_t)plan.token_tiles;
    f.idesc = instruction(f.four, c.w[0]->format, c.x->format, f.tokens, 128);
    const uint32_t halves = c.w[1] ? 2 : 1, groups = f.four ? 2 : 1, x_tiles = f.tokens > 128 ? 2 : 1;
    f.x_at = halves * ROWS128;
    f.ws_at = f.x_at + (uint32_t)f.tokens * 128;
    f.xs_at = f.ws_at + halves * groups * BNN_MX_TILE;
    f.stage_bytes = (f.xs_at + x_tiles * groups * BNN_MX_TILE + 1023) & ~1023u;
    f.loaded = halves * f.w_bytes + (uint32_t)f.tokens * 128 + (halves + x_tiles) * groups * BNN_MX_TILE;
    f.acc_up = (uint32_t)((f.tokens + 31) & ~31);
    f.scales = halves * f.acc_up;
    f.x_pitch = 4 * x_tiles;
    f.scale_set = groups * (4 * halves + f.x_pitch);
    f.tmem_cols = 32;
    while (f.tmem_cols < f.scales + 2 * f.scale_set) f.tmem_cols *= 2;
    if (f.tmem_cols > FEW_COLUMNS) return BNN_ERR_INVALID_ARG;          // not reached: FEW_WHOLE
    const int budget = plan.per_sm == 2 ? FEW_SMEM / 2 : FEW_SMEM, steps = (f.q.k_iters + plan.split - 1) / plan.split;
    f.stages = budget / (int)f.stage_bytes;
    f.stages = f.stages > FEW_STAGES ? FEW_STAGES : f.stages;
    if (f.stages > steps) f.stages = steps;
    f.stages = f.stages < 2 ? 2 : f.stages & ~1;
    if (int st = map_operands(ctx, f.maps, c, f.tokens, (int)x_tiles, 128, 1)) return st;
    const unsigned tiles = (unsigned)plan.tiles, split = (unsigned)plan.split;
    if (halves == 2) return c.q ? launch_few<BNN_EPI_GATED, true>(ctx, f, tiles, split) : launch_few<BNN_EPI_GATED, false>(ctx, f, tiles, split);
    return c.q ? launch_few<BNN_EPI_LINEAR, true>(ctx, f, tiles, split) : launch_few<BNN_EPI_LINEAR, false>(ctx, f, tiles, split);
}

int product(bnn_ctx *ctx, const Call &c) {
    if (!ctx) return BNN_ERR_INVALID_ARG;
    if (c.x->rows == 0 || c.w[0]->rows == 0) return BNN_OK;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    const FewPlan plan = few_plan(c);
    if (c.x->cols == 0 && plan.tiles == 0) return BNN_ERR_INVALID_ARG;        // the empty sum is the few-row kernel's, up to 2^26 rows
    return c.x->cols == 0 || plan.cost < pair_cost(ctx, c) ? product_few(ctx, c, plan) : product_pair(ctx, c);
}
// x e2m1: weights e2m1; x e4m3: weights of either format.
int check_operands(const bnn_mx_matrix *w, const bnn_mx_matrix *x) {
    if (w->cols != x->cols || (x->format == BNN_MX_E2M1 && w->format != BNN_MX_E2M1)) return BNN_ERR_INVALID_ARG;
    return BNN_OK;
}
int check_output(const bnn_mx_matrix *q, const void *y, const float *pre, const bnn_mx_matrix *x, const bnn_mx_matrix *w, const bnn_mx_matrix *w2) {
    if (!q) return BNN_OK;
    if (y || pre) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_mx(q)) return st;
    if (q->rows != x->rows || q->cols != w->rows) return BNN_ERR_INVALID_ARG;
    return bnn_mx_touches(q, x) || bnn_mx_touches(q, w) || (w2 && bnn_mx_touches(q, w2)) ? BNN_ERR_INVALID_ARG : BNN_OK;
}
bool is_half(int dtype) { return dtype == BNN_F16 || dtype == BNN_BF16; }

}  // namespace

int bnn_mx_product_status(bnn_ctx *ctx, int *code) {
    BNN_CUDA_TRY(ctx, cudaMemcpyFromSymbol(code, g_mx_error, sizeof(int)));
    const int zero = 0;
    if (*code) BNN_CUDA_TRY(ctx, cudaMemcpyToSymbol(g_mx_error, &zero, sizeof(int)));
    return BNN_OK;
}

extern "C" int bnn_mx_linear(bnn_ctx *ctx, const bnn_mx_linear_desc *layer, const bnn_mx_matrix *x, const void *residual, int64_t ldr, void *y, int64_t ldy,
                             float *pre, int64_t ldp, const bnn_mx_matrix *y_mx) {
    if (!layer || !is_half(layer->dtype) || !bnn_act_known(layer->act)) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_mx(&layer->W)) return st;
    if (int st = bnn_check_mx(x)) return st;
    if (int st = check_operands(&layer->W, x)) return st;
    const int64_t M = x->rows, N = layer->W.rows;
    if (int st = bnn_check_real_opt(layer->bias, N, 1, N, 2)) return st;
    if (int st = check_output(y_mx, y, pre, x, &layer->W, nullptr)) return st;
    if (y_mx && (residual || bnn_mx_touches(y_mx, layer->bias, 0, 1, N, 2))) return BNN_ERR_INVALID_ARG;
    if (!y_mx)
        if (int st = bnn_check_real(y, ldy, M, N, 2)) return st;
    if (int st = bnn_check_real_opt(residual, ldr, M, N, 2)) return st;
    if (int st = bnn_check_real_opt(pre, ldp, M, N, 4)) return st;
    Call c{};
    c.dtype = layer->dtype; c.act = layer->act; c.epilogue = BNN_EPI_LINEAR; c.x = x; c.w[0] = &layer->W; c.bias = layer->bias;
    c.add = residual; c.ld_add = ldr; c.out = y; c.ldo = ldy; c.q = y_mx; c.pre = pre; c.ldp = ldp;
    return product(ctx, c);
}

extern "C" int bnn_mx_gated(bnn_ctx *ctx, const bnn_mx_gated_desc *layer, const bnn_mx_matrix *x, void *h, int64_t ldh, float *pre, int64_t ldp,
                            const bnn_mx_matrix *h_mx) {
    if (!layer || !is_half(layer->dtype) || !bnn_act_known(layer->act)) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_mx(&layer->Wg)) return st;
    if (int st = bnn_check_mx(&layer->Wu)) return st;
    if (layer->Wg.rows != layer->Wu.rows || layer->Wg.cols != layer->Wu.cols || layer->Wg.format != layer->Wu.format) return BNN_ERR_INVALID_ARG;
    if (int st = bnn_check_mx(x)) return st;
    if (int st = check_operands(&layer->Wg, x)) return st;
    const int64_t M = x->rows, N = layer->Wg.rows;
    if (int st = check_output(h_mx, h, pre, x, &layer->Wg, &layer->Wu)) return st;
    if (!h_mx)
        if (int st = bnn_check_real(h, ldh, M, N, 2)) return st;
    if (int st = bnn_check_real_opt(pre, ldp, M > 0 && M < BNN_REAL_MAX / 2 ? 2 * M : M, N, 4)) return st;
    Call c{};
    c.dtype = layer->dtype; c.act = layer->act; c.epilogue = BNN_EPI_GATED; c.x = x; c.w[0] = &layer->Wg; c.w[1] = &layer->Wu;
    c.out = h; c.ldo = ldh; c.q = h_mx; c.pre = pre; c.ldp = ldp;
    return product(ctx, c);
}
