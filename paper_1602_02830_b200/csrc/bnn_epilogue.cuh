// What the tensor-core products of the real-valued operators share (16-bit and microscaled operands): what a launch is told, bounded waits, and
// epilogues from tensor memory (a warp's block of 32 x 32 outputs) and from partial sums (four neighbouring outputs of a token).
#pragma once
#include "bnn_product.cuh"
#include "bnn_ptx.cuh"

namespace {
using namespace bnn_ptx;

// What the epilogue has to know of a product.
struct Output {
    int64_t M, N;
    int k_iters;                         // K steps of all pairs of operands
    int vec_out;                         // what every row is made of: 2 = 16-byte groups, 1 = 4-byte words, 0 = elements
    void *out[2];
    int64_t ldo[2];
};
// One product of a launch.  a_mn / b_mn: the operand is stored against the sum.
struct Problem : Output {
    CUtensorMap a[2], b[2];
    int k_pair;                          // K steps of the first pair of operands
    uint32_t first, tiles_m, tiles_n;    // first tile of the launch's numbering; tile rows and columns
    uint32_t idesc;
    int a_mn, b_mn;
};
// What the epilogue of a single product needs beside the problem, and what every launch needs.
struct Common {
    const void *bias, *add;
    float *pre;
    int64_t ld_add, ldp;
    int act, f16;
    int vec_bias, vec_add, vec_pre;      // as vec_out; vec_pre 3 = 32-byte sectors
    unsigned long long wait_ns;
    int drop_loads;                      // test hook: the producers request nothing, every consumer's wait runs out (2: see loads_here)
};
// How long a kernel waits at its end for copies and MMAs that it has issued, whatever the limit of its other waits; and for copies that no
// barrier of its own counts.
constexpr unsigned long long DRAIN_NS = 1000000000ull, SETTLE_NS = 2000000ull;

// Whether the producers of a CTA of a split sum request anything (the test hook: 2 = the odd CTAs of a cluster do not).
__device__ __forceinline__ bool loads_here(int drop_loads, uint32_t split, uint32_t rank) { return drop_loads == 0 || (drop_loads == 2 && split > 1 && !(rank & 1)); }

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
__device__ __forceinline__ void finish_block(const Common &p, const Output &q, int64_t m0, int64_t n0, uint32_t acc, uint32_t acc2, uint8_t *piece) {
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

__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    return remote;
}
// Between the two barriers of a split sum's cluster: a CTA that has given up tells the others, none of which then writes outputs that lack its share.
template <typename C> __device__ __forceinline__ void tell_cluster(C *ctl, uint32_t split) {
    const uint32_t code = *reinterpret_cast<volatile uint32_t *>(&ctl->failed);
    if (code != 0u && threadIdx.x < split) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(smem_u32(&ctl->failed), threadIdx.x)), "r"(code) : "memory");
    __syncwarp();
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
template <int EPI, typename T> __device__ __forceinline__ void finish4(const Common &p, const Output &q, int64_t m, int64_t n0, float (&a)[4], float (&b)[4]) {
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

int width_of(const void *p, int64_t ld, int64_t rows, int size) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint64_t pitch = rows > 1 ? (uint64_t)ld * size : 0;
    if (size == 4 && (at | pitch) % 32 == 0) return 3;
    return (at | pitch) % 16 == 0 ? 2 : (at | pitch) % 4 == 0 ? 1 : 0;
}


}  // namespace
