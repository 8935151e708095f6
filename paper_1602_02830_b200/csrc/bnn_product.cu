// 16-bit matrix product on the 5th-generation tensor cores with the epilogues of the dense layer and the gated projections.
//
//   out[m][n] = epilogue(sum_k A[m][k] B[n][k]),  float32 accumulators in tensor memory, one rounding at the end.
// All three products of a layer are this one: forward x W^T reads both operands along their rows; dx = dz W reads W against its
// rows, dW = dz^T x both.  The tensor cores take either order from shared memory (the descriptor's major bit), so nothing is
// transposed on the way.
//
// k_product_pair: a cluster of two CTAs works on one 256 x BN tile (tcgen05.mma cta_group::2): each CTA holds its 128 rows of A
// and half of the tile's columns of B, so a pair reads 256 + BN rows of operands for 256 x BN products.  Persistent, one CTA per
// SM, tiles in bands of eight tile rows so that the operands of the tiles in flight stay in L2.
//   warp 0, last warp  TMA producers, K steps in turn: 64-element K slices of both operands, 128-byte swizzle, a ring of stages
//   warp 1             MMA issuer (CTA 0 of the pair): four K = 16 MMAs per stage; tcgen05.commit frees the stage
//   the others         epilogue: two or four per TMEM lane quadrant, a share of the columns each, one output row per thread
// Two accumulator buffers: the epilogue of a tile runs under the MMAs of the next one.
// Gated projections: B's two halves are the gate rows (CTA 0) and the up rows (CTA 1), so columns 0 .. BN/2 - 1 of the
// accumulator are g and the others u of the same hidden units, and one thread holds both when it forms act(g) u.
// One issuing thread keeps the order of the additions fixed: the same call gives the same bits.
// Bound: the tensor pipe and, for seconds on end, the part's power limit.  Measured (bf16): 8192 x 4096 x 4096 213 us = 1.29 PFLOP/s, with a
// residual 227; 2048 x 4096 x 8192 109 us = 1.26 PFLOP/s; gated, 8192 rows, 4096 to 8192 twice, SiLU 800 us = 1.37 PFLOP/s; gradients
// of 8192 x 4096 x 4096 440 us = 1.25 PFLOP/s.  256 x 256 tiles read (256 + 256) x K of operands from L2 for 256 x 256 x K products, half
// of what 128 x 128 tiles of single CTAs read.  Short sums are bound by the epilogue and by writing: 3644 x 6416, K = 64, 25 us for 47 MB
// (a plain fill of as much takes 14).
// Every wait is bounded, as in the binary engine: a failure ends the kernel and shows in bnn_device_status.
#include "bnn_product.cuh"
#include "bnn_internal.cuh"
#include "bnn_ptx.cuh"
#include <mutex>

namespace {
using namespace bnn_ptx;

__device__ int g_product_error;          // 0 = fine; otherwise a code saying which wait gave up

constexpr int BK = 64;                   // elements of K per stage: one 128-byte row
constexpr int TM = 256;                  // tile rows of a pair
// Epilogue warps: sixteen or eight.  Eight where a thread needs more than the 104 registers that sixteen leave (kept pre-activations, the
// gated gradient: 8192 x 4096 x 4096 with GELU, residual and kept pre-activations 281 us with sixteen, 259 with eight) and, from LONG_SUM
// K steps on, where the epilogue has time (2048 x 4096 x 8192 112 us with sixteen, 110 with eight; 4096 x 4096 x 4096, both gradients 220
// and 216).  Shorter sums are bound by their epilogue (3584 x 6400 x 256 with residual and bias 42 with sixteen, 49 with eight; K = 1024 53 and 59, 2048 79 and 77).
constexpr int LONG_SUM = 32;
constexpr int pair_threads(int epi_warps) { return (2 + epi_warps + 1) * 32; }
constexpr uint32_t A_STAGE = 128 * BK * 2;
template <int BN> struct Ring {
    static constexpr uint32_t B_STAGE = (BN / 2) * BK * 2;
    static constexpr uint32_t STAGE = A_STAGE + B_STAGE;
    static constexpr int STAGES = BN == 256 ? 6 : 8;                // 192 KB
    static constexpr uint32_t TMEM = 2 * BN;
};
constexpr int STAGES_MAX = 8;             // even numbers of stages: each belongs to one of the two producers
constexpr int BAND = 8;                  // tile rows per band

// One product of a launch.  a_mn / b_mn: the operand is stored against the sum.
struct Problem {
    CUtensorMap a[2], b[2];
    int64_t M, N;
    int k_pair, k_iters;                 // K steps of the first pair of operands; of all
    uint32_t first, tiles_m, tiles_n;    // first tile of the launch's numbering; tile rows and columns
    uint32_t idesc;
    int a_mn, b_mn;
    void *out[2];
    int64_t ldo[2];
    int vec_out;                         // what every row is made of: 2 = 16-byte groups, 1 = 4-byte words, 0 = elements
};
constexpr int PROBLEMS = 3;              // a gated layer's gradients: dx, dWg, dWu
// What the epilogue of a single product needs beside the problem, and what every launch needs.
struct Common {
    const void *bias, *add;
    float *pre;
    int64_t ld_add, ldp;
    int act, f16;
    int vec_bias, vec_add, vec_pre;      // as vec_out; vec_pre 3 = 32-byte sectors
    unsigned long long wait_ns;
    int drop_loads;                      // test hook: the producers request nothing, every consumer's wait runs out
};
template <int N> struct ProductArgs : Common {
    Problem q[N];
    int problems;
    uint32_t tiles;
};

// How long a kernel waits at its end for copies and MMAs that it has issued, whatever the limit of its other waits; and for copies that no
// barrier of its own counts.
constexpr unsigned long long DRAIN_NS = 1000000000ull, SETTLE_NS = 2000000ull;

struct __align__(16) Control {
    uint64_t full[STAGES_MAX], empty[STAGES_MAX], acc_full[2], acc_empty[2], drain;
    uint32_t tmem_base, failed;
};

__device__ __forceinline__ void fail(Control *ctl, int code) {
    *reinterpret_cast<volatile uint32_t *>(&ctl->failed) = (uint32_t)code;
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&ctl->failed)), "r"(cluster_ctarank() ^ 1u));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote), "r"((uint32_t)code) : "memory");
    atomicCAS(&g_product_error, 0, code);
}
// Bounded wait on a phase parity; false once the limit has passed or another wait of the pair has given up (`look`: whether to ask).
template <typename C> __device__ __forceinline__ bool wait(const C *ctl, unsigned long long limit, const uint64_t *barrier, uint32_t parity, bool look = true) {
    const uint32_t bar = smem_u32(barrier);
    unsigned long long t0 = 0;
    for (uint32_t i = 0;; ++i) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if ((i & 63u) == 63u) {
            if (look && *reinterpret_cast<const volatile uint32_t *>(&ctl->failed) != 0u) return false;
            const unsigned long long now = global_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > limit) return false;
        }
    }
}
// The same by a whole warp, with one answer for all lanes: what follows (tcgen05.ld, __syncwarp) needs them together, and a lane that looked
// a moment earlier than another could have given up alone.
template <typename C> __device__ __forceinline__ bool warp_wait(const C *ctl, unsigned long long limit, const uint64_t *barrier, uint32_t parity, bool look = true) {
    return __all_sync(0xffffffffu, wait(ctl, limit, barrier, parity, look));
}
__device__ __forceinline__ void mma_f16_2sm(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Operand stored against the sum: boxes of 64 output rows (128 bytes) x 64 K rows, 8192 bytes each; groups of eight K rows 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
    return smem_desc_sw128(addr) | ((uint64_t)(8192u >> 4) << 16);
}

struct Tile { int problem, m0, n0; };
template <int WIDTH, int N> __device__ __forceinline__ Tile tile_at(const ProductArgs<N> &p, uint32_t t) {
    int i = 0;
    if (N > 1)
        while (i + 1 < p.problems && t >= p.q[i + 1].first) ++i;
    const Problem &q = p.q[i];
    t -= q.first;
    const uint32_t band = t / (BAND * q.tiles_n), w = t - band * BAND * q.tiles_n;
    const uint32_t high = q.tiles_m - band * BAND < BAND ? q.tiles_m - band * BAND : BAND;
    const uint32_t n = w / high;
    return {i, (int)((band * BAND + w - n * high) * TM), (int)(n * WIDTH)};
}

// A warp's block of 32 rows in memory passes through its piece of shared memory (32 rows of 64 bytes: 32 16-bit or 16 float columns), so that
// a lane computes on its own row while neighbouring lanes touch neighbouring bytes of memory.  Sixteen-byte units of a row are
// permuted by the row, which keeps both sides free of bank conflicts.
// vec: 2 = rows of whole 16-byte groups, 1 = of whole 4-byte words, 0 = single elements (lane-private rows of 2-byte accesses took five
// times as long: 3644 x 6417, K = 288, 281 us).
constexpr int PIECE = 32 * 64, BLOCK = 32, CHUNK = 16;      // columns of a block; of one pass through the registers
__device__ __forceinline__ uint4 *unit_of(uint8_t *piece, int row, int unit) { return reinterpret_cast<uint4 *>(piece + row * 64 + ((unit ^ ((row >> 1) & 3)) << 4)); }
template <typename W> __device__ __forceinline__ W *word_of(uint8_t *piece, int row, int word) {
    constexpr int PER = 16 / (int)sizeof(W);
    return reinterpret_cast<W *>(unit_of(piece, row, word / PER)) + word % PER;
}
// Writes a block: rows x n of its 32 x COLS elements exist, `first` is its first element.
template <typename T, int COLS> __device__ __forceinline__ void flush(T *first, int64_t ld, int vec, int rows, int n, uint8_t *piece) {
    constexpr int PER = 16 / (int)sizeof(T), UNITS = COLS / PER;
    const int lane = threadIdx.x & 31;
    __syncwarp();
    if (vec == 2) {
        const int u = lane % UNITS;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int r = i * (32 / UNITS) + lane / UNITS;
            if (r >= rows) continue;
            const uint4 w = *unit_of(piece, r, u);
            T *to = first + r * ld + u * PER;
            if ((u + 1) * PER <= n) __stcs(reinterpret_cast<uint4 *>(to), w);
            else
                for (int k = 0; k < n - u * PER; ++k) to[k] = *word_of<T>(piece, r, u * PER + k);
        }
    } else if (vec == 1) {
        constexpr int EACH = 4 / (int)sizeof(T), WORDS = COLS / EACH;                 // words of a row
        const int c = lane % WORDS;
#pragma unroll 8
        for (int i = 0; i < WORDS; ++i) {
            const int r = i * (32 / WORDS) + lane / WORDS;
            T *to = first + r * ld + c * EACH;
            if (r < rows) {
                if ((c + 1) * EACH <= n) __stcs(reinterpret_cast<uint32_t *>(to), *word_of<uint32_t>(piece, r, c));
                else if (c * EACH < n) *to = *word_of<T>(piece, r, c * EACH);
            }
        }
    } else {
        constexpr int PASSES = COLS;                                                   // COLS x 32 elements, 32 at a time
        const int c = lane % COLS;
#pragma unroll 8
        for (int i = 0; i < PASSES; ++i) {
            const int r = i * (32 / COLS) + lane / COLS;
            if (r < rows && c < n) first[r * ld + c] = *word_of<T>(piece, r, c);
        }
    }
    __syncwarp();
}
// A block of 16-bit elements comes in: `request` asks for its units, `land` puts them into the piece, from where each lane takes its row.
struct Incoming { uint4 w[4]; };
__device__ __forceinline__ void request(Incoming &in, const uint16_t *first, int64_t ld, int rows, int n) {
    const int lane = threadIdx.x & 31, u = lane & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 2);
        const uint16_t *from = first + r * ld + u * 8;
        in.w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r >= rows) continue;
        if ((u + 1) * 8 <= n) in.w[i] = *reinterpret_cast<const uint4 *>(from);
        else {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (u * 8 + k < n) w[k >> 1] |= (uint32_t)from[k] << (16 * (k & 1));
            in.w[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}
__device__ __forceinline__ void land(const Incoming &in, const uint16_t *first, int64_t ld, int vec, int rows, int n, uint8_t *piece) {
    const int lane = threadIdx.x & 31;
    if (vec == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *unit_of(piece, i * 8 + (lane >> 2), lane & 3) = in.w[i];
    } else {
        for (int i = 0; i < 32; i += 16) {                       // sixteen rows on their way
            uint16_t v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = i + k < rows && lane < n ? first[(i + k) * ld + lane] : (uint16_t)0;
#pragma unroll
            for (int k = 0; k < 16; ++k) *word_of<uint16_t>(piece, i + k, lane) = v[k];
        }
    }
    __syncwarp();
}
// Sixteen columns of the lane's row into the piece (16-bit ones from column `at` on, or floats), and out of it.
template <typename T> __device__ __forceinline__ void put16(uint8_t *piece, int at, const float (&v)[16]) {
    constexpr int PER = 16 / (int)sizeof(T);
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 16 / PER; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (sizeof(T) == 4) w[k] = __float_as_uint(v[4 * i + k]);
            else w[k] = pack2<T>(v[8 * i + 2 * k], v[8 * i + 2 * k + 1]);
        }
        *unit_of(piece, lane, at / PER + i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T> __device__ __forceinline__ void get16(uint8_t *piece, int at, float (&d)[16]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 w = *unit_of(piece, lane, at / 8 + i);
        float e[8];
        unpack8<T>(&w, e);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[8 * i + j] = e[j];
    }
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}

template <int ACT> __device__ __forceinline__ void act16(float (&v)[16]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = act_value(ACT, v[j]);
}
template <int ACT> __device__ __forceinline__ void back16(const float (&d)[16], float (&a)[16]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float value;
        a[j] = d[j] * act_slope(ACT, a[j], value);
    }
}
template <int ACT> __device__ __forceinline__ void gated_back16(const float (&d)[16], float (&a)[16], float (&b)[16]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float value;
        const float slope = act_slope(ACT, a[j], value);
        a[j] = d[j] * b[j] * slope;
        b[j] = d[j] * value;
    }
}
// The choice of the activation is made once for sixteen values.
#define BNN_EACH_ACT(CALL)                                        \
    switch (p.act) {                                              \
        case BNN_ACT_RELU: CALL(BNN_ACT_RELU); break;             \
        case BNN_ACT_GELU: CALL(BNN_ACT_GELU); break;             \
        case BNN_ACT_GELU_TANH: CALL(BNN_ACT_GELU_TANH); break;   \
        case BNN_ACT_SILU: CALL(BNN_ACT_SILU); break;             \
        case BNN_ACT_SIGMOID: CALL(BNN_ACT_SIGMOID); break;       \
        case BNN_ACT_HTANH: CALL(BNN_ACT_HTANH); break;           \
        default: CALL(BNN_ACT_NONE); break;                       \
    }
// Sixteen bias values.
struct Bias { uint4 w[2]; };
__device__ __forceinline__ Bias bias_of(const Common &p, int64_t n0, int n) {
    const uint16_t *bias = static_cast<const uint16_t *>(p.bias) + n0;
    Bias b;
    if (p.vec_bias == 2 && n >= 16) { b.w[0] = reinterpret_cast<const uint4 *>(bias)[0]; b.w[1] = reinterpret_cast<const uint4 *>(bias)[1]; }
    else {
        uint32_t w[8] = {};
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < n) w[j >> 1] |= (uint32_t)bias[j] << (16 * (j & 1));
        b.w[0] = make_uint4(w[0], w[1], w[2], w[3]); b.w[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
    return b;
}
template <typename T> __device__ __forceinline__ void add_bias16(const Bias &bias, float (&a)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c[8];
        unpack8<T>(&bias.w[i], c);
#pragma unroll
        for (int j = 0; j < 8; ++j) a[8 * i + j] += c[j];
    }
}
// Sixteen pre-activations of the lane's row, 64 bytes: directly where rows are whole 32-byte sectors (3), else through the piece.
__device__ __forceinline__ void keep16(float *first, int64_t ld, int vec, int rows, int n, uint8_t *piece, const float (&v)[16]) {
    const int lane = threadIdx.x & 31;
    if (vec == 3 && n >= 16) {
        if (lane < rows) {
            float *to = first + lane * ld;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                asm volatile("st.global.cs.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                             ::"l"(to + 8 * i), "r"(__float_as_uint(v[8 * i])), "r"(__float_as_uint(v[8 * i + 1])), "r"(__float_as_uint(v[8 * i + 2])),
                               "r"(__float_as_uint(v[8 * i + 3])), "r"(__float_as_uint(v[8 * i + 4])), "r"(__float_as_uint(v[8 * i + 5])),
                               "r"(__float_as_uint(v[8 * i + 6])), "r"(__float_as_uint(v[8 * i + 7])) : "memory");
        }
    } else {
        put16<float>(piece, 0, v);
        flush<float, 16>(first, ld, vec < 2 ? vec : 2, rows, n, piece);
    }
}

// A warp's block: 32 rows from m0 on, 32 columns from n0 on, accumulators at `acc` (and `acc2`: gated).  What is added has landed in the
// piece; a lane takes sixteen columns of it at a time and puts the result into their place, unless the piece has to pass something
// else on in between: the kept pre-activations (PRE: as floats) or the first of two outputs, which are then written sixteen columns at a
// time.  In those cases the incoming values are taken before.
template <int EPI, typename T, bool PRE>
__device__ __forceinline__ void finish_block(const Common &p, const Problem &q, int64_t m0, int64_t n0, uint32_t acc, uint32_t acc2, uint8_t *piece) {
    constexpr bool GATED = EPI == BNN_EPI_GATED || EPI == BNN_EPI_GATED_BACK, APART = PRE || EPI == BNN_EPI_GATED_BACK;
    const int rows = (int)(q.M - m0 < 32 ? q.M - m0 : 32), n = (int)(q.N - n0 < BLOCK ? q.N - n0 : BLOCK);
    T *out = static_cast<T *>(q.out[0]) + m0 * q.ldo[0] + n0;
    const bool adds = EPI != BNN_EPI_GATED && p.add;
    uint4 held[4];                                           // APART: the lane's row of what is added
    if (APART && adds) {
#pragma unroll
        for (int i = 0; i < 4; ++i) held[i] = *unit_of(piece, threadIdx.x & 31, i);
        __syncwarp();
    }
#pragma unroll
    for (int c = 0; c < BLOCK; c += CHUNK) {
        uint32_t ra[16], rb[16];
        float a[16], b[16], d[16];
        const int left = n - c < CHUNK ? n - c : CHUNK;
        if (left <= 0) break;
        tmem_ld16(acc + c, ra);
        if (GATED) tmem_ld16(acc2 + c, rb);
        tmem_ld_wait16(ra);
        if (GATED) tmem_ld_wait16(rb);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            a[j] = q.k_iters ? __uint_as_float(ra[j]) : 0.0f;
            if (GATED) b[j] = q.k_iters ? __uint_as_float(rb[j]) : 0.0f;
        }
        if (!GATED && p.bias) add_bias16<T>(bias_of(p, n0 + c, left), a);
        if (adds) {
            if constexpr (APART) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    unpack8<T>(&held[c / 8 + i], e);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[8 * i + j] = e[j];
                }
            } else get16<T>(piece, c, d);
        }
        if constexpr (PRE) {
            keep16(p.pre + m0 * p.ldp + n0 + c, p.ldp, p.vec_pre, rows, left, piece, a);
            if constexpr (GATED) keep16(p.pre + (q.M + m0) * p.ldp + n0 + c, p.ldp, p.vec_pre, rows, left, piece, b);
        }
        if constexpr (EPI == BNN_EPI_LINEAR || EPI == BNN_EPI_GATED) {
#define BNN_CALL(ACT) act16<ACT>(a)
            BNN_EACH_ACT(BNN_CALL)
#undef BNN_CALL
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (GATED) a[j] *= b[j];
                else if (adds) a[j] += d[j];
            }
        } else if constexpr (EPI == BNN_EPI_LINEAR_BACK) {
#define BNN_CALL(ACT) back16<ACT>(d, a)
            BNN_EACH_ACT(BNN_CALL)
#undef BNN_CALL
        } else {
#define BNN_CALL(ACT) gated_back16<ACT>(d, a, b)
            BNN_EACH_ACT(BNN_CALL)
#undef BNN_CALL
        }
        put16<T>(piece, APART ? 0 : c, a);
        if constexpr (APART) flush<T, 16>(out + c, q.ldo[0], q.vec_out, rows, left, piece);
        if constexpr (EPI == BNN_EPI_GATED_BACK) {
            put16<T>(piece, 0, b);
            flush<T, 16>(static_cast<T *>(q.out[1]) + m0 * q.ldo[1] + n0 + c, q.ldo[1], q.vec_out, rows, left, piece);
        }
    }
    if constexpr (!APART) flush<T, BLOCK>(out, q.ldo[0], q.vec_out, rows, n, piece);
}

template <int EPI, int BN, int N, bool PRE, int EPI_WARPS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads(EPI_WARPS), 1) k_product_pair(const __grid_constant__ ProductArgs<N> p) {
    constexpr bool GATED = EPI == BNN_EPI_GATED || EPI == BNN_EPI_GATED_BACK;
    constexpr int WIDTH = GATED ? BN / 2 : BN;                   // output columns of a tile
    constexpr int STAGES = Ring<BN>::STAGES, PARTS = EPI_WARPS / 4;
    constexpr uint32_t STAGE = Ring<BN>::STAGE, TMEM = Ring<BN>::TMEM;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Control *ctl = reinterpret_cast<Control *>(tiles + STAGES * STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl->acc_full[b]), 1); mbar_init(smem_u32(&ctl->acc_empty[b]), 2 * EPI_WARPS); }
        mbar_init(smem_u32(&ctl->drain), 1);
        ctl->failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                          // both CTAs' barriers exist before anyone signals them
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = ctl->tmem_base;

    if (warp == 0 || warp == 2 + EPI_WARPS) {
        // ---------------- producers: two threads take the K steps in turn.  One pass of this loop costs a thread about 480 clocks
        // (0.256 us a step alone, 0.144 two in turn; a further box 0.035), as much as the step's MMAs take.
        // The "full" barrier of a stage (in CTA 0) completes with the arrival of CTA 0's producer and the bytes of both CTAs.
        // The two need no order between them: the use before last of a stage is consumed whenever one of them gets to its next use.
        if (lane == 0 && !p.drop_loads) {
            const uint32_t mine = warp == 0 ? 0 : 1;
            bool ok = true;
            uint32_t step = 0, stage = mine, lap = 0;                // step: of the launch, before the current tile
            bnn_pdl_wait();
            for (uint32_t t = pair; t < p.tiles && ok; t += pairs) {
                const Tile tile = tile_at<WIDTH>(p, t);
                const Problem &q = p.q[tile.problem];
                const int m0 = tile.m0 + (int)rank * 128, n0 = tile.n0 + (GATED ? 0 : (int)rank * (BN / 2));
                const int k_pair = q.k_pair, k_iters = q.k_iters, a_mn = q.a_mn, b_mn = q.b_mn;
                for (int kit = (int)((mine + step) & 1u); kit < k_iters; kit += 2) {
                    if (lap > 0 && !wait(ctl, p.wait_ns, &ctl->empty[stage], (lap - 1) & 1)) { fail(ctl, 1); ok = false; break; }
                    const int second = kit >= k_pair ? 1 : 0, k = (kit - (second ? k_pair : 0)) * BK;
                    const uint32_t dst = smem_u32(tiles + stage * STAGE), bar = smem_u32(&ctl->full[stage]) & PEER_MASK;
                    if (rank == 0) mbar_expect_tx(smem_u32(&ctl->full[stage]), 2 * STAGE);
                    const CUtensorMap *am = &q.a[second], *bm = &q.b[GATED ? (int)rank : second];
                    if (a_mn) {
                        tma_load_2d_2sm(dst, am, m0, k, bar);
                        tma_load_2d_2sm(dst + 8192, am, m0 + 64, k, bar);
                    } else tma_load_2d_2sm(dst, am, k, m0, bar);
                    if (b_mn) {
                        tma_load_2d_2sm(dst + A_STAGE, bm, n0, k, bar);
                        if (BN == 256) tma_load_2d_2sm(dst + A_STAGE + 8192, bm, n0 + 64, k, bar);
                    } else tma_load_2d_2sm(dst + A_STAGE, bm, k, n0, bar);
                    stage += 2;
                    if (stage >= (uint32_t)STAGES) { stage -= STAGES; ++lap; }
                }
                step += (uint32_t)k_iters;
            }
            // The copies in flight land before the CTA gives its shared memory up.  Waited for in every case: whether one of the other waits gives up
            // may be decided after this thread has requested everything.
            if (rank == 0)
                for (uint32_t i = 0, s = stage, l = lap; i < (uint32_t)STAGES; i += 2) {      // this thread's last uses, newest first
                    if (s < 2) { if (l == 0) break; s += STAGES; --l; }
                    s -= 2;
                    if (!wait(ctl, DRAIN_NS, &ctl->full[s], l & 1, false)) break;
                }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t stage = 0, phase = 0, count = 0;
            bool ok = true;
            for (uint32_t t = pair; t < p.tiles && ok; t += pairs, ++count) {
                const uint32_t buf = count & 1, use = count >> 1;
                if (use > 0 && !wait(ctl, p.wait_ns, &ctl->acc_empty[buf], (use - 1) & 1)) { fail(ctl, 4); ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d = tmem_base + buf * BN;
                const Problem &q = p.q[tile_at<WIDTH>(p, t).problem];
                const uint64_t a0 = q.a_mn ? smem_desc_mn(smem_u32(tiles)) : smem_desc_sw128(smem_u32(tiles));
                const uint64_t b0 = q.b_mn ? smem_desc_mn(smem_u32(tiles + A_STAGE)) : smem_desc_sw128(smem_u32(tiles + A_STAGE));
                const uint64_t a_step = q.a_mn ? 2048 >> 4 : 32 >> 4, b_step = q.b_mn ? 2048 >> 4 : 32 >> 4;      // 16 elements of K
                const uint32_t idesc = q.idesc;
                const int k_iters = q.k_iters;
                for (int kit = 0; kit < k_iters; ++kit) {
                    if (!wait(ctl, p.wait_ns, &ctl->full[stage], phase)) { fail(ctl, 2); ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = a0 + (uint64_t)(stage * (STAGE >> 4)), b = b0 + (uint64_t)(stage * (STAGE >> 4));
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) mma_f16_2sm(d, a + k * a_step, b + k * b_step, idesc, (kit | k) != 0 ? 1u : 0u);
                    umma_commit_2sm(smem_u32(&ctl->empty[stage]));
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                umma_commit_2sm(smem_u32(&ctl->acc_full[buf]));
            }
            umma_commit_2sm(smem_u32(&ctl->drain));  // the MMAs issued end before tensor memory is given back, also where nobody waits for them any more
            wait(ctl, DRAIN_NS, &ctl->drain, 0, false);
        }
    } else if (warp < 2 + EPI_WARPS) {
        bnn_pdl_wait();
        bnn_pdl_launch_next();
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const uint32_t quadrant = (uint32_t)(32 * quad) << 16;
        uint8_t *piece = reinterpret_cast<uint8_t *>(ctl + 1) + (warp - 2) * PIECE;
        uint32_t count = 0;
        for (uint32_t t = pair; t < p.tiles; t += pairs, ++count) {
            const uint32_t buf = count & 1;
            const Tile tile = tile_at<WIDTH>(p, t);
            const Problem &q = p.q[tile.problem];
            const int64_t m0 = tile.m0 + (int)rank * 128 + 32 * quad;
            constexpr int SHARE = WIDTH / PARTS < BLOCK ? BLOCK : WIDTH / PARTS;       // a warp's columns of a tile (gated 128-wide tiles: two warps of four)
            const int first = part * SHARE < WIDTH ? part * SHARE : WIDTH, last = first + SHARE < WIDTH ? first + SHARE : WIDTH;
            const int rows = (int)(q.M - m0 < 32 ? q.M - m0 : 32);
            // what is added (the residual, an incoming gradient) is requested a block ahead, the first one while the tile is being multiplied
            const bool adds = EPI != BNN_EPI_GATED && p.add != nullptr;
            const uint16_t *add = static_cast<const uint16_t *>(p.add) + m0 * p.ld_add + tile.n0;
            Incoming in;
            if (adds && p.vec_add == 2 && rows > 0 && first < last) request(in, add + first, p.ld_add, rows, (int)(q.N - tile.n0 - first));
            if (!warp_wait(ctl, p.wait_ns, &ctl->acc_full[buf], (count >> 1) & 1)) { fail(ctl, 3); break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem_base + buf * BN + quadrant;
#pragma unroll 1
            for (int c = first; c < last; c += BLOCK) {
                const int n = (int)(q.N - tile.n0 - c);
                if (n <= 0 || rows <= 0) break;
                if (adds) {
                    land(in, add + c, p.ld_add, p.vec_add, rows, n, piece);
                    if (p.vec_add == 2 && c + BLOCK < last) request(in, add + c + BLOCK, p.ld_add, rows, n - BLOCK);
                }
                if (p.f16) finish_block<EPI, __half, PRE>(p, q, m0, tile.n0 + c, acc + c, acc + WIDTH + c, piece);
                else finish_block<EPI, __nv_bfloat16, PRE>(p, q, m0, tile.n0 + c, acc + c, acc + WIDTH + c, piece);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_cta0(smem_u32(&ctl->acc_empty[buf]));
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
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------------------
// Few output rows (tokens): k_product_few.  The roles are swapped -- 128 weight rows are the M side of the tensor-core tile and the
// tokens, 16 to 256 of them, its N side -- so a single token costs a tile of 16 columns and not of 256 rows, and every SM streams
// weights.  Bound: the weights' bytes (HBM) where they are more than L2 holds: one row by two 8192 x 4096 bf16 24.3 us for 134 MB = 5.5 TB/s.  Smaller weights stay in
// L2 between calls that repeat them, and launch and fill show: one row by 4096 x 4096, 33.6 MB, 9.4 us; 48 rows by two 5500 x 2048, 45 MB, 14.8 us.  With
// the weights rotated through 20 layers and the calls in a graph: 11.3 us = 3.0 TB/s and 14.5 us = 3.1 TB/s.  The sum is split over the CTAs of a cluster when there are too few tiles of
// weight rows to keep every SM loading: each takes a share of the K steps, stores its partial tile into the shared memory of the CTAs
// that finish it (distributed shared memory, a share of the rows each), and after a cluster barrier every CTA adds up the parts of its
// share in the order of the ranks: one launch, no workspace, the same bits every time.  (Reading the parts from the other CTAs
// instead cost a remote access's latency per pass: 4096 x 4096, 256 rows, 17.9 us.)
// Gated projections: 64 gate rows and the up rows of the same 64 hidden units form the 128 rows of a tile.
//   warps 0 and 11  TMA producers, warp 1  MMA issuer (cta_group::1), warps 2 .. 9  partial tile to its finishers, all warps  sum and epilogue
constexpr int FEW_SMEM = 200 * 1024;
constexpr int FEW_THREADS = 384;
constexpr int FEW_STAGES = 12;
constexpr int FEW_TOKENS = 256;
// Above so many 256 x 256 tiles the pair kernel is taken without a comparison.  That is right for many rows, whose tiles fill the GPU.  The tiles are counted
// whatever their rows, though, so it also holds for few tokens and more than 32768 outputs (gated: 16384), whose tiles are mostly padding: one token, 4096 inputs,
// 32768 outputs 46 us = 5.8 TB/s of weights on this kernel, 40960 outputs 86 us = 3.9 TB/s on the pair kernel.
constexpr int64_t FEW_TILES = 128;

struct FewArgs : Common {
    Problem q;                          // a: weights (a[1]: up rows, or the second pair), b: tokens; M tokens, N outputs
    uint32_t token_tiles;
    int tokens;                         // N of the MMA: tokens per tile, a multiple of 16
    int stages;
    uint32_t stage_bytes, tmem_cols;
};
struct __align__(16) FewControl {
    uint64_t full[FEW_STAGES], empty[FEW_STAGES], acc_full;
    uint32_t tmem_base, failed;
};
__device__ __forceinline__ void few_fail(FewControl *ctl, int code) {
    *reinterpret_cast<volatile uint32_t *>(&ctl->failed) = (uint32_t)code;
    atomicCAS(&g_product_error, 0, code);
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    return remote;
}
// The sum of four neighbouring values over the ranks' parts, in the order of the ranks, `pitch` floats apart.
__device__ __forceinline__ void sum_parts(const float *at, int split, int pitch, float (&v)[4]) {
    float4 t = *reinterpret_cast<const float4 *>(at);
    for (int i = 1; i < split; ++i) {
        const float4 r = *reinterpret_cast<const float4 *>(at + i * pitch);
        t.x += r.x; t.y += r.y; t.z += r.z; t.w += r.w;
    }
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
}

// Four neighbouring outputs of one token, n of them inside; vec: on 8-byte (pre: 16-byte) boundaries.
template <typename T> __device__ __forceinline__ void read4(const T *p, int n, int vec, float (&v)[4]) {
    if (vec && n >= 4) {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < n ? to_f32(p[j]) : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void write4(T *p, int n, int vec, const float (&v)[4]) {
    if (vec && n >= 4) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = from_f32<T>(v[j]);
    }
}
template <int EPI, typename T> __device__ __forceinline__ void finish4(const Common &p, const Problem &q, int64_t m, int64_t n0, float (&a)[4], float (&b)[4]) {
    const int n = (int)(q.N - n0 < 4 ? q.N - n0 : 4);
    const T *add = static_cast<const T *>(p.add) + m * p.ld_add + n0;
    T *out = static_cast<T *>(q.out[0]) + m * q.ldo[0] + n0;
    float d[4];
    if constexpr (EPI == BNN_EPI_LINEAR || EPI == BNN_EPI_LINEAR_BACK) {
        if (p.bias) {
            read4(static_cast<const T *>(p.bias) + n0, n, p.vec_bias, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] += d[j];
        }
    }
    if (EPI != BNN_EPI_GATED && p.add) read4(add, n, p.vec_add, d);
    if ((EPI == BNN_EPI_LINEAR || EPI == BNN_EPI_GATED) && p.pre) {
        write4(p.pre + m * p.ldp + n0, n, p.vec_pre, a);
        if (EPI == BNN_EPI_GATED) write4(p.pre + (q.M + m) * p.ldp + n0, n, p.vec_pre, b);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float value;
        if constexpr (EPI == BNN_EPI_LINEAR) {
            a[j] = act_value(p.act, a[j]);
            if (p.add) a[j] += d[j];
        } else if constexpr (EPI == BNN_EPI_LINEAR_BACK) {
            a[j] = d[j] * act_slope(p.act, a[j], value);
        } else if constexpr (EPI == BNN_EPI_GATED) {
            a[j] = act_value(p.act, a[j]) * b[j];
        } else {
            const float slope = act_slope(p.act, a[j], value);
            a[j] = d[j] * b[j] * slope;
            b[j] = d[j] * value;
        }
    }
    write4(out, n, q.vec_out, a);
    if constexpr (EPI == BNN_EPI_GATED_BACK) write4(static_cast<T *>(q.out[1]) + m * q.ldo[1] + n0, n, q.vec_out, b);
}

template <bool W_MN, bool T_MN, int EPI> __global__ void __launch_bounds__(FEW_THREADS, 2) k_product_few(const __grid_constant__ FewArgs f) {
    constexpr bool GATED = EPI == BNN_EPI_GATED || EPI == BNN_EPI_GATED_BACK;
    constexpr int ROWS = GATED ? 64 : 128;                        // outputs of a tile
    const Common &p = f;
    const Problem &q = f.q;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ FewControl control;
    FewControl *ctl = &control;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    uint32_t split;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    const uint32_t tile = blockIdx.x / split, tn = tile / f.token_tiles, tt = tile - tn * f.token_tiles;     // tiles of the same weights next to each other
    const int64_t n0 = (int64_t)tn * ROWS, t0 = (int64_t)tt * f.tokens;
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
    bnn_pdl_wait();
    bnn_pdl_launch_next();

    if (warp == 0 || warp == FEW_THREADS / 32 - 1) {              // two producers take the K steps in turn, as in the pair kernel
        if (lane == 0 && !p.drop_loads) {
            const int mine = warp == 0 ? 0 : 1;
            int stage = mine % f.stages, lap = mine / f.stages;
            for (int kit = first + mine; kit < last; kit += 2) {
                if (lap > 0 && !wait(ctl, p.wait_ns, &ctl->empty[stage], (lap - 1) & 1)) { few_fail(ctl, 21); break; }
                const int second = kit >= q.k_pair ? 1 : 0, k = (kit - (second ? q.k_pair : 0)) * BK;
                const uint32_t dst = smem_u32(tiles) + stage * f.stage_bytes, bar = smem_u32(&ctl->full[stage]);
                mbar_expect_tx(bar, f.stage_bytes);
                if constexpr (GATED) {
                    tma_load_2d(dst, &q.a[0], k, (int)n0, bar);
                    tma_load_2d(dst + 8192, &q.a[1], k, (int)n0, bar);
                } else if constexpr (W_MN) {
                    tma_load_2d(dst, &q.a[second], (int)n0, k, bar);
                    tma_load_2d(dst + 8192, &q.a[second], (int)n0 + 64, k, bar);
                } else tma_load_2d(dst, &q.a[second], k, (int)n0, bar);
                if constexpr (T_MN) {
                    for (int i = 0; i < f.tokens; i += 64) tma_load_2d(dst + A_STAGE + i * 128, &q.b[second], (int)t0 + i, k, bar);
                } else tma_load_2d(dst + A_STAGE, &q.b[second], k, (int)t0, bar);
                stage += 2;
                while (stage >= f.stages) { stage -= f.stages; ++lap; }
            }
            for (int i = 0, s = stage, l = lap; i < f.stages; i += 2) {            // copies in flight land before the shared memory is given up, as above
                s -= 2;
                while (s < 0) { s += f.stages; --l; }
                if (l < 0 || !wait(ctl, DRAIN_NS, &ctl->full[s], l & 1, false)) break;
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint64_t A_STEP = W_MN ? 2048 >> 4 : 32 >> 4;
            const uint64_t a0 = W_MN ? smem_desc_mn(smem_u32(tiles)) : smem_desc_sw128(smem_u32(tiles)), b0 = T_MN ? smem_desc_mn(smem_u32(tiles + A_STAGE)) : smem_desc_sw128(smem_u32(tiles + A_STAGE));
            constexpr uint64_t B_STEP = T_MN ? 2048 >> 4 : 32 >> 4;
            int stage = 0;
            uint32_t phase = 0;
            for (int kit = first; kit < last; ++kit) {
                if (!wait(ctl, p.wait_ns, &ctl->full[stage], phase)) { few_fail(ctl, 22); break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t at = (uint64_t)(stage * (f.stage_bytes >> 4));
#pragma unroll
                for (int k = 0; k < BK / 16; ++k) mma_f16(tmem_base, a0 + at + k * A_STEP, b0 + at + k * B_STEP, q.idesc, (kit > first || k) ? 1u : 0u);
                mma_commit(&ctl->empty[stage]);
                if (++stage == f.stages) { stage = 0; phase ^= 1; }
            }
            mma_commit(&ctl->acc_full);
            wait(ctl, DRAIN_NS, &ctl->acc_full, 0, false);       // the MMAs issued end before tensor memory is given back, also where the epilogue has given up
        }
    }
    // Rank r finishes the tile's outputs r * OUT .. r * OUT + OUT - 1 of every token.  A lane of warps 2 .. 9 holds one weight row of the
    // partial tile and stores it where it is needed: parts[rank it comes from][token][row of the finishing rank's share], the gate rows of
    // a share before its up rows, in the finishing CTA's ring, which is free once all MMAs of the cluster are done (first barrier).
    const int log = split == 8 ? 3 : (int)split >> 1, out = ROWS >> log, share = 128 >> log, pitch = f.tokens * share;
    float *parts = reinterpret_cast<float *>(tiles);
    const int valid = (int)(q.M - t0 < f.tokens ? q.M - t0 : f.tokens);
    {                                                             // what this thread's first outputs will need from memory is brought to L2
        const int t = (int)threadIdx.x / (out / 4);
        const int64_t n = n0 + (int)rank * out + ((int)threadIdx.x - t * (out / 4)) * 4;
        if (t < valid && n < q.N) {
            const uint16_t *add = static_cast<const uint16_t *>(p.add) + (t0 + t) * p.ld_add + n;
            if (EPI != BNN_EPI_GATED && p.add) asm volatile("prefetch.global.L2 [%0];" ::"l"(add));
            if (!GATED && p.bias) asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint16_t *>(p.bias) + n));
        }
    }
    bool done = false;
    if (warp >= 2 && warp < 10) {
        done = warp_wait(ctl, 2 * p.wait_ns, &ctl->acc_full, 0, false);
        if (!done) few_fail(ctl, 23);
    }
    __syncwarp();
    if (split > 1) cluster_sync_all();
    else __syncthreads();
    if (done && *reinterpret_cast<volatile uint32_t *>(&ctl->failed) == 0u) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int quad = warp & 3, row = 32 * quad + lane, unit = GATED ? row & 63 : row, owner = unit / out;
        const int place = unit - owner * out + (GATED && row >= 64 ? out : 0);
        const uint32_t to = in_cta(smem_u32(parts + (int)rank * pitch + place), (uint32_t)owner);
        for (int c = warp < 6 ? 0 : 16; c < f.tokens; c += 32) {
            if (c >= valid) break;
            uint32_t r[16];
            tmem_ld16(tmem_base + ((uint32_t)(32 * quad) << 16) + c, r);
            tmem_ld_wait16(r);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < valid)
                    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + (uint32_t)((c + j) * share) * 4), "r"(last > first ? r[j] : 0u) : "memory");
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
    for (int i = threadIdx.x; i < valid * (out / 4); i += FEW_THREADS) {
        const int t = i / (out / 4), row = (i - t * (out / 4)) * 4;
        const int64_t n = n0 + (int)rank * out + row;
        if (n >= q.N) continue;
        float a[4], b[4];
        sum_parts(parts + t * share + row, (int)split, pitch, a);
        if (GATED) sum_parts(parts + t * share + out + row, (int)split, pitch, b);
        if (p.f16) finish4<EPI, __half>(p, q, t0 + t, n, a, b);
        else finish4<EPI, __nv_bfloat16>(p, q, t0 + t, n, a, b);
    }
}

// ---------------------------------------------------------------------------------------------------------
template <int BN> constexpr size_t pair_smem(int epi_warps) {
    return (size_t)Ring<BN>::STAGES * Ring<BN>::STAGE + sizeof(Control) + epi_warps * PIECE + 1024;
}
static_assert(pair_smem<256>(16) <= 227 * 1024 && pair_smem<128>(16) <= 227 * 1024, "fits the shared memory of an SM");

// Opts in to the shared memory and asks how many pairs fit the device, once per device and kernel; 0 = cannot run.
template <int EPI, int BN, int N, bool PRE, int WARPS> int pairs_of(int device, int sm_count) {
    static std::mutex lock;
    static int cached[64];
    if (device < 0 || device >= 64) return 0;
    std::lock_guard<std::mutex> guard(lock);
    if (cached[device] == 0) {
        auto kernel = k_product_pair<EPI, BN, N, PRE, WARPS>;
        int pairs = 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pair_smem<BN>(WARPS)) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(2 * sm_count); cfg.blockDim = dim3(pair_threads(WARPS)); cfg.dynamicSmemBytes = pair_smem<BN>(WARPS);
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

template <int EPI, int BN, bool PRE, int WARPS, int N> int launch_warps(bnn_ctx *ctx, const ProductArgs<N> &a) {
    const int pairs = pairs_of<EPI, BN, N, PRE, WARPS>(ctx->device, ctx->sm_count);
    if (pairs == 0) return BNN_ERR_CUDA;
    const unsigned n = a.tiles < (uint32_t)pairs ? a.tiles : (unsigned)pairs;
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(k_product_pair<EPI, BN, N, PRE, WARPS>, dim3(2 * n), dim3(pair_threads(WARPS)), pair_smem<BN>(WARPS), ctx->stream, a));
    return bnn_check_launch(ctx);
}
template <int EPI, int BN, bool PRE, int N> int launch(bnn_ctx *ctx, const ProductArgs<N> &a) {      // q[0] has the longest sum
    if constexpr (!PRE && EPI != BNN_EPI_GATED_BACK)
        if (a.q[0].k_iters < LONG_SUM) return launch_warps<EPI, BN, PRE, 16>(ctx, a);
    return launch_warps<EPI, BN, PRE, 8>(ctx, a);
}

template <bool W_MN, bool T_MN, int EPI> int launch_few(bnn_ctx *ctx, const FewArgs &f, unsigned tiles, unsigned split) {
    auto kernel = k_product_few<W_MN, T_MN, EPI>;
    static std::mutex lock;
    static bool ready[64];
    if (ctx->device < 0 || ctx->device >= 64) return BNN_ERR_INVALID_ARG;
    {
        std::lock_guard<std::mutex> guard(lock);
        if (!ready[ctx->device]) BNN_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM + 1024));
        ready[ctx->device] = true;
    }
    cudaLaunchConfig_t cfg{};
    const size_t ring = (size_t)f.stages * f.stage_bytes, part = (size_t)f.tokens * 512;
    cfg.gridDim = dim3(tiles * split); cfg.blockDim = dim3(FEW_THREADS); cfg.dynamicSmemBytes = (ring > part ? ring : part) + 1024; cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    BNN_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, kernel, f));
    return bnn_check_launch(ctx);
}

int map16(bnn_ctx *ctx, CUtensorMap *map, const void *p, int64_t ld, int64_t rows, int64_t cols, int box_rows) {
    return bnn_tensor_map16(ctx, map, p, rows, cols, rows > 1 ? ld : (cols + 7) & ~int64_t(7), box_rows, BK);
}
int width_of(const void *p, int64_t ld, int64_t rows, int size) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint64_t pitch = rows > 1 ? (uint64_t)ld * size : 0;
    if (size == 4 && (at | pitch) % 32 == 0) return 3;
    return (at | pitch) % 16 == 0 ? 2 : (at | pitch) % 4 == 0 ? 1 : 0;
}

}  // namespace

int bnn_product_status(bnn_ctx *ctx, int *code) {
    BNN_CUDA_TRY(ctx, cudaMemcpyFromSymbol(code, g_product_error, sizeof(int)));
    const int zero = 0;
    if (*code) BNN_CUDA_TRY(ctx, cudaMemcpyToSymbol(g_product_error, &zero, sizeof(int)));
    return BNN_OK;
}

namespace {
bool is_gated(const BnnProduct &q) { return q.epilogue == BNN_EPI_GATED || q.epilogue == BNN_EPI_GATED_BACK; }
int64_t steps_of(const BnnProduct &q) { return (q.K + BK - 1) / BK * (is_gated(q) ? 1 : q.pairs); }
void common_args(Common &a, bnn_ctx *ctx, const BnnProduct &q) {
    a.bias = q.bias; a.add = q.add; a.ld_add = q.ld_add; a.pre = q.pre; a.ldp = q.ldp; a.act = q.act; a.f16 = q.dtype == BNN_F16;
    a.wait_ns = ctx->wait_limit_ns; a.drop_loads = ctx->drop_loads;
}
void common_problem(Problem &w, const BnnProduct &q) {
    w.M = q.M; w.N = q.N;
    w.k_pair = (int)((q.K + BK - 1) / BK); w.k_iters = (int)steps_of(q);
    w.a_mn = q.a_mn; w.b_mn = q.b_mn;
    for (int i = 0; i < 2; ++i) { w.out[i] = q.out[i]; w.ldo[i] = q.ldo[i]; }
}
// float32 accumulators, both operands of the call's type, N columns, M rows; whether each operand lies against the sum.
uint32_t instruction(int dtype, int a_mn, int b_mn, int n, int m) {
    const uint32_t type = dtype == BNN_BF16 ? 1u : 0u;
    return (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

int64_t pair_tiles(const BnnProduct &q, int bn) {
    const int64_t width = is_gated(q) ? bn / 2 : bn;
    return (q.M + TM - 1) / TM * ((q.N + width - 1) / width);
}
// Which kernel, and how k_product_few divides the work, by estimates of both in microseconds.  Fitted to times of calls that repeat the same weights, from L2
// as far as it holds them (N x K, rows, few / pair): 4096 x 4096, 1: 10.7 / 27.8, 128: 14.2 / 25.8, 384: 22.5 / 26.8, 768: 37.5 / 30.4; 512 x 8192, 512: 16.0 / 44.1; 8192 x 1024,
// 64: 9.5 / 10.6, 192: 14.1 / 11.3; 256 x 256, 1: 3.9 / 5.3, 128: 9.0 / 5.9.
//   pair: 5 + 0.30 per K step and round of tiles, or the weights at 3.3 TB/s (gated, 5500 x 2048 twice: 20.9) if that takes longer.
//   few:  3 for every round of CTAs, + per K step of an SM's CTAs 0.12 + 0.0012 per token of a tile, at least 0.28 (0.26 with
//         two CTAs per SM): what one SM draws from HBM (8192 x 8192, one row: 40 us on 64 SMs, 26 on all); + 1 (2 with a split sum) + 0.041 per token of a CTA's share of the epilogue.
// More, smaller token tiles keep more SMs busy, fewer read the weights less often; the sum is split while there are SMs left and
// every CTA keeps four K steps.
double pair_cost(const bnn_ctx *ctx, const BnnProduct &q) {
    const int64_t pairs = ctx->sm_count / 2;
    const double steps = 5.0 + 0.30 * (double)steps_of(q) * (double)((pair_tiles(q, 256) + pairs - 1) / pairs);
    const double weights = 5.0 + 2.0 * (double)q.N * (double)q.K * (is_gated(q) ? 2 : q.pairs) / 3.3e6;
    return steps > weights ? steps : weights;
}
// CTAs that are resident at once in clusters of 1, 2, 4 and 8, one or two per SM (cudaOccupancyMaxActiveClusters with the whole or half
// of the shared memory: the SMs of a GPC are not a multiple of the larger clusters).
constexpr int FEW_RESIDENT[2][4] = {{148, 148, 132, 120}, {296, 296, 284, 264}};
struct FewPlan { int64_t tiles; int token_tiles, tokens, split, per_sm; double cost; };
FewPlan few_plan(const BnnProduct &q) {
    const int64_t rows = is_gated(q) ? 64 : 128, steps = steps_of(q), weight_tiles = (q.N + rows - 1) / rows;
    FewPlan best{};
    best.cost = 1e30;
    int last = 0;
    const int unit = q.a_mn ? 64 : 16;                     // boxes of 64 when the token operand lies against the sum
    for (int most = FEW_TOKENS; most >= unit; most /= 2) {
        FewPlan f{};
        f.token_tiles = (int)((q.M + most - 1) / most);
        if (f.token_tiles == last) continue;
        last = f.token_tiles;
        f.tokens = (int)(((q.M + f.token_tiles - 1) / f.token_tiles + unit - 1) / unit * unit);
        f.tiles = weight_tiles * f.token_tiles;
        for (int log = 0; log < 4; ++log) {
            f.split = 1 << log;
            if (log && steps < f.split * 4) break;
            const int64_t ctas = f.tiles * f.split;
            f.per_sm = ctas > FEW_RESIDENT[0][log] && f.tokens <= 64 ? 2 : 1;      // half of an SM's memory still holds four stages of 64 tokens
            const int64_t resident = FEW_RESIDENT[f.per_sm - 1][log], rounds = (ctas + resident - 1) / resident;
            const double load = (double)(rounds > 1 ? rounds * f.per_sm : (ctas + 147) / 148), cta_steps = (double)((steps + f.split - 1) / f.split);
            double step = 0.12 + 0.0012 * f.tokens;
            if (step < (f.per_sm == 2 ? 0.26 : 0.28)) step = f.per_sm == 2 ? 0.26 : 0.28;
            f.cost = 3.0 * (double)rounds + load * cta_steps * step + (f.split > 1 ? 2.0 : 1.0) + 0.041 * f.tokens / f.split * load;
            if (f.cost < best.cost) best = f;
        }
    }
    return best;
}
int product_few(bnn_ctx *ctx, const BnnProduct &q) {
    const FewPlan plan = few_plan(q);
    if (plan.tiles * plan.split > 0x7fffffff) return BNN_ERR_INVALID_ARG;
    FewArgs f{};
    common_args(f, ctx, q);
    Problem &w = f.q;
    common_problem(w, q);
    const auto fours = [](const void *at, int64_t ld, int64_t n, int size) { return reinterpret_cast<uintptr_t>(at) % (4 * size) == 0 && (n <= 1 || ld % 4 == 0); };
    f.vec_bias = fours(q.bias, 0, 1, 2); f.vec_add = fours(q.add, q.ld_add, q.M, 2); f.vec_pre = fours(q.pre, q.ldp, 2 * q.M, 4);
    w.vec_out = fours(q.out[0], q.ldo[0], q.M, 2) && fours(q.out[1], q.ldo[1], q.M, 2);
    const int rows = is_gated(q) ? 64 : 128;
    f.tokens = plan.tokens; f.token_tiles = (uint32_t)plan.token_tiles;
    w.tiles_n = (uint32_t)((q.N + rows - 1) / rows);
    w.idesc = instruction(q.dtype, q.b_mn, q.a_mn, f.tokens, 128);
    f.stage_bytes = A_STAGE + (uint32_t)f.tokens * BK * 2;
    f.tmem_cols = 32;
    while ((int)f.tmem_cols < f.tokens) f.tmem_cols *= 2;
    const int budget = plan.per_sm == 2 ? FEW_SMEM / 2 : FEW_SMEM, steps = (w.k_iters + plan.split - 1) / plan.split;
    f.stages = budget / (int)f.stage_bytes;
    f.stages = f.stages > FEW_STAGES ? FEW_STAGES : f.stages;
    if (f.stages > steps) f.stages = steps;
    f.stages = f.stages < 2 ? 2 : f.stages & ~1;
    if (q.K > 0) {
        for (int i = 0; i < 2; ++i) {
            if (q.b[i].p)
                if (int st = q.b_mn ? map16(ctx, &w.a[i], q.b[i].p, q.b[i].ld, q.K, q.N, BK) : map16(ctx, &w.a[i], q.b[i].p, q.b[i].ld, q.N, q.K, rows)) return st;
            if (q.a[i].p)
                if (int st = q.a_mn ? map16(ctx, &w.b[i], q.a[i].p, q.a[i].ld, q.K, q.M, BK) : map16(ctx, &w.b[i], q.a[i].p, q.a[i].ld, q.M, q.K, f.tokens)) return st;
        }
    }
    const unsigned tiles = (unsigned)plan.tiles, split = (unsigned)plan.split;
    if (q.a_mn) return launch_few<true, true, BNN_EPI_LINEAR>(ctx, f, tiles, split);          // a weight gradient: both against the sum
    if (q.b_mn) return launch_few<true, false, BNN_EPI_LINEAR>(ctx, f, tiles, split);
    switch (q.epilogue) {
        case BNN_EPI_LINEAR: return launch_few<false, false, BNN_EPI_LINEAR>(ctx, f, tiles, split);
        case BNN_EPI_LINEAR_BACK: return launch_few<false, false, BNN_EPI_LINEAR_BACK>(ctx, f, tiles, split);
        case BNN_EPI_GATED: return launch_few<false, false, BNN_EPI_GATED>(ctx, f, tiles, split);
        default: return launch_few<false, false, BNN_EPI_GATED_BACK>(ctx, f, tiles, split);
    }
}
}  // namespace

// The cheapest way to make several products: each alone on either kernel, or all of them in one launch of the pair kernel.
// few[i]: product i runs on k_product_few.
bool bnn_product_apart(const bnn_ctx *ctx, const BnnProduct *list, int n, bool *few) {
    struct Load { int64_t longest = 0, total = 0; } rest, all;       // K steps: of one tile, of all tiles
    const auto add = [](Load &l, const BnnProduct &q) {
        const int64_t steps = steps_of(q);
        if (steps > l.longest) l.longest = steps;
        l.total += steps * pair_tiles(q, 256);
    };
    const auto cost = [&](const Load &l) {
        const int64_t even = (l.total + ctx->sm_count / 2 - 1) / (ctx->sm_count / 2);
        return l.longest ? 5.0 + 0.30 * (double)(even > l.longest ? even : l.longest) : 0.0;
    };
    double apart = 0.0;
    for (int i = 0; i < n; ++i) {
        const double f = pair_tiles(list[i], 256) <= FEW_TILES ? few_plan(list[i]).cost : 1e30;
        few[i] = f < pair_cost(ctx, list[i]);
        if (few[i]) apart += f;
        else add(rest, list[i]);
        add(all, list[i]);
    }
    return n == 1 || apart + cost(rest) < cost(all);
}

namespace {
template <int N> int product_pair(bnn_ctx *ctx, const BnnProduct *list, int count) {
    // Half-width tiles where whole ones would leave half of the pairs without work.
    int64_t whole = 0, tiles = 0;
    for (int i = 0; i < count; ++i) whole += pair_tiles(list[i], 256);
    const int bn = 2 * whole <= ctx->sm_count / 2 ? 128 : 256;
    ProductArgs<N> a{};
    common_args(a, ctx, list[0]);
    a.problems = count;
    const BnnProduct *order[N];
    for (int i = 0; i < count; ++i) order[i] = &list[i];
    for (int i = 1; i < count; ++i)                      // the longest sums first: short tiles fill the end of the launch
        for (int j = i; j > 0 && steps_of(*order[j]) > steps_of(*order[j - 1]); --j) { const BnnProduct *t = order[j]; order[j] = order[j - 1]; order[j - 1] = t; }
    for (int i = 0; i < count; ++i) {
        const BnnProduct &q = *order[i];
        Problem &w = a.q[i];
        common_problem(w, q);
        const int64_t width = is_gated(q) ? bn / 2 : bn;
        w.first = (uint32_t)tiles; w.tiles_m = (uint32_t)((q.M + TM - 1) / TM); w.tiles_n = (uint32_t)((q.N + width - 1) / width);
        tiles += pair_tiles(q, bn);
        if (tiles > 0x7fffffff) return BNN_ERR_INVALID_ARG;
        w.idesc = instruction(q.dtype, q.a_mn, q.b_mn, bn, TM);
        w.vec_out = width_of(q.out[0], q.ldo[0], q.M, 2);
        if (q.out[1]) { const int v = width_of(q.out[1], q.ldo[1], q.M, 2); w.vec_out = v < w.vec_out ? v : w.vec_out; }
        if (q.K == 0) continue;
        for (int k = 0; k < 2; ++k) {
            if (q.a[k].p)
                if (int st = q.a_mn ? map16(ctx, &w.a[k], q.a[k].p, q.a[k].ld, q.K, q.M, BK) : map16(ctx, &w.a[k], q.a[k].p, q.a[k].ld, q.M, q.K, 128)) return st;
            if (q.b[k].p)
                if (int st = q.b_mn ? map16(ctx, &w.b[k], q.b[k].p, q.b[k].ld, q.K, q.N, BK) : map16(ctx, &w.b[k], q.b[k].p, q.b[k].ld, q.N, q.K, bn / 2)) return st;
        }
    }
    a.tiles = (uint32_t)tiles;
    const BnnProduct &q = list[0];
    a.vec_bias = width_of(q.bias, 0, 1, 2); a.vec_add = width_of(q.add, q.ld_add, q.M, 2); a.vec_pre = width_of(q.pre, q.ldp, 2 * q.M, 4);
#define BNN_LAUNCH(EPI, PRE) (bn == 256 ? launch<EPI, 256, PRE>(ctx, a) : launch<EPI, 128, PRE>(ctx, a))
    if constexpr (N == 1) {
        if (q.epilogue == BNN_EPI_LINEAR_BACK) return BNN_LAUNCH(BNN_EPI_LINEAR_BACK, false);
        if (q.epilogue == BNN_EPI_GATED_BACK) return BNN_LAUNCH(BNN_EPI_GATED_BACK, false);
        if (q.epilogue == BNN_EPI_GATED) return q.pre ? BNN_LAUNCH(BNN_EPI_GATED, true) : BNN_LAUNCH(BNN_EPI_GATED, false);
        if (q.pre) return BNN_LAUNCH(BNN_EPI_LINEAR, true);
    }
    return BNN_LAUNCH(BNN_EPI_LINEAR, false);
#undef BNN_LAUNCH
}
}  // namespace

int bnn_product(bnn_ctx *ctx, const BnnProduct *list, int count) {
    if (count < 1 || count > PROBLEMS) return BNN_ERR_INVALID_ARG;
    if (count > 1) return product_pair<PROBLEMS>(ctx, list, count);
    bool few = list[0].kernel == BNN_FEW;
    if (list[0].kernel == BNN_CHEAPEST) bnn_product_apart(ctx, list, 1, &few);
    if (few) return product_few(ctx, list[0]);
    return product_pair<1>(ctx, list, 1);
}
