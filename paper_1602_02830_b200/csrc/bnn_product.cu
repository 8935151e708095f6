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
//   warp 0, last warp  TMA producers (A and B): 64-element K slices, 128-byte swizzle, a ring of shared-memory stages
//   warp 1             MMA issuer (CTA 0 of the pair): four K = 16 MMAs per stage; tcgen05.commit frees the stage
//   warps 2 .. 9       epilogue: two per TMEM lane quadrant, each half of the columns, one output row per thread
// Two accumulator buffers: the epilogue of a tile runs under the MMAs of the next one.
// Gated projections: B's two halves are the gate rows (CTA 0) and the up rows (CTA 1), so columns 0 .. BN/2 - 1 of the
// accumulator are g and the others u of the same hidden units, and one thread holds both when it forms act(g) u.
// One issuing thread keeps the order of the additions fixed: the same call gives the same bits.
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
constexpr int EPI_WARPS = 8;
constexpr int THREADS = (2 + EPI_WARPS + 1) * 32;
constexpr uint32_t A_STAGE = 128 * BK * 2;
template <int BN> struct Ring {
    static constexpr uint32_t B_STAGE = (BN / 2) * BK * 2;
    static constexpr uint32_t STAGE = A_STAGE + B_STAGE;
    static constexpr int STAGES = BN == 256 ? 6 : 8;                // 192 KB
    static constexpr uint32_t TMEM = 2 * BN;
};
constexpr int STAGES_MAX = 8;
constexpr int BAND = 8;                  // tile rows per band

struct ProductArgs {
    CUtensorMap a[2], b[2];
    int64_t M, N;
    int k_pair, k_iters;                 // K steps of the first pair; of all
    int groups;
    uint32_t tiles_m, tiles_n, tiles;
    uint32_t idesc;
    const void *bias, *add;
    void *out[2];
    float *pre;
    int64_t ld_add, ldo[2], ldp;
    int act, f16;
    int vec_bias, vec_add, vec_out, vec_pre;   // widest access that every row allows: 2 = 32 bytes, 1 = 16 bytes, 0 = one element
    unsigned long long wait_ns;
    int drop_loads;                      // test hook: the producers request nothing, every consumer's wait runs out
};

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
__device__ __forceinline__ bool wait(const Control *ctl, unsigned long long limit, const uint64_t *barrier, uint32_t parity, bool look = true) {
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
__device__ __forceinline__ void mma_f16_2sm(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Operand stored against the sum: boxes of 64 output rows (128 bytes) x 64 K rows, 8192 bytes each; groups of eight K rows 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
    return smem_desc_sw128(addr) | ((uint64_t)(8192u >> 4) << 16);
}

struct Tile { int64_t m0, n0; int group; };
template <int WIDTH> __device__ __forceinline__ Tile tile_at(const ProductArgs &p, uint32_t t) {
    const uint32_t per = p.tiles_m * p.tiles_n, g = t / per;
    t -= g * per;
    const uint32_t band = t / (BAND * p.tiles_n), w = t - band * BAND * p.tiles_n;
    const uint32_t high = p.tiles_m - band * BAND < BAND ? p.tiles_m - band * BAND : BAND;
    const uint32_t n = w / high;
    return {(int64_t)(band * BAND + w - n * high) * TM, (int64_t)n * WIDTH, (int)g};
}

// 32 neighbouring elements of a row, n of them inside the matrix, as floats.
template <typename T> __device__ __forceinline__ void read32(const T *p, int n, int vec, float (&v)[32]) {
    if (vec && n >= 32) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 w = reinterpret_cast<const uint4 *>(p)[i];
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = unpack2<T>(u[j]);
                    v[8 * i + 2 * j] = f.x; v[8 * i + 2 * j + 1] = f.y;
                }
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = j < n ? to_f32(p[j]) : 0.0f;
    }
}
__device__ __forceinline__ void st256(void *p, const uint32_t *w) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
template <typename T> __device__ __forceinline__ void write32(T *p, int n, int vec, const float (&v)[32]) {
    if (vec && n >= 32) {
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = pack2<T>(v[2 * j], v[2 * j + 1]);
        if (vec == 2) { st256(p, w); st256(p + 16, w + 8); }
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < n) p[j] = from_f32<T>(v[j]);
    }
}
__device__ __forceinline__ void write32f(float *p, int n, int vec, const float (&v)[32]) {
    if (vec && n >= 32) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(v);
        if (vec == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) st256(p + 8 * i, w + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < n) p[j] = v[j];
    }
}

template <int ACT> __device__ __forceinline__ void act32(float (&v)[32]) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = act_value(ACT, v[j]);
}
__device__ __forceinline__ void act_values(int act, float (&v)[32]) {
    switch (act) {               // the choice is made once for 32 values
        case BNN_ACT_RELU: act32<BNN_ACT_RELU>(v); break;
        case BNN_ACT_GELU: act32<BNN_ACT_GELU>(v); break;
        case BNN_ACT_GELU_TANH: act32<BNN_ACT_GELU_TANH>(v); break;
        case BNN_ACT_SILU: act32<BNN_ACT_SILU>(v); break;
        case BNN_ACT_SIGMOID: act32<BNN_ACT_SIGMOID>(v); break;
        case BNN_ACT_HTANH: act32<BNN_ACT_HTANH>(v); break;
        default: break;
    }
}

// 32 columns of one row, from accumulators to memory.  b: the second accumulator of the gated epilogues.
template <int EPI, typename T>
__device__ __forceinline__ void finish32(const ProductArgs &p, int group, int64_t m, int64_t n0, float (&a)[32], float (&b)[32]) {
    const int n = (int)(p.N - n0 < 32 ? p.N - n0 : 32);
    float d[32];
    if constexpr (EPI == BNN_EPI_LINEAR || EPI == BNN_EPI_LINEAR_BACK) {
        if (p.bias) {
            read32(static_cast<const T *>(p.bias) + n0, n, p.vec_bias, d);
#pragma unroll
            for (int j = 0; j < 32; ++j) a[j] += d[j];
        }
    }
    if (m >= p.M) return;
    if constexpr (EPI == BNN_EPI_LINEAR) {
        if (p.pre) write32f(p.pre + m * p.ldp + n0, n, p.vec_pre, a);
        act_values(p.act, a);
        if (p.add) {
            read32(static_cast<const T *>(p.add) + m * p.ld_add + n0, n, p.vec_add, d);
#pragma unroll
            for (int j = 0; j < 32; ++j) a[j] += d[j];
        }
        write32(static_cast<T *>(p.out[group]) + m * p.ldo[group] + n0, n, p.vec_out, a);
    } else if constexpr (EPI == BNN_EPI_LINEAR_BACK) {
        read32(static_cast<const T *>(p.add) + m * p.ld_add + n0, n, p.vec_add, d);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float value;
            d[j] *= act_slope(p.act, a[j], value);
        }
        write32(static_cast<T *>(p.out[0]) + m * p.ldo[0] + n0, n, p.vec_out, d);
    } else if constexpr (EPI == BNN_EPI_GATED) {
        if (p.pre) {
            write32f(p.pre + m * p.ldp + n0, n, p.vec_pre, a);
            write32f(p.pre + (p.M + m) * p.ldp + n0, n, p.vec_pre, b);
        }
        act_values(p.act, a);
#pragma unroll
        for (int j = 0; j < 32; ++j) a[j] *= b[j];
        write32(static_cast<T *>(p.out[0]) + m * p.ldo[0] + n0, n, p.vec_out, a);
    } else {
        read32(static_cast<const T *>(p.add) + m * p.ld_add + n0, n, p.vec_add, d);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float value;
            const float slope = act_slope(p.act, a[j], value);
            a[j] = d[j] * b[j] * slope;
            b[j] = d[j] * value;
        }
        write32(static_cast<T *>(p.out[0]) + m * p.ldo[0] + n0, n, p.vec_out, a);
        write32(static_cast<T *>(p.out[1]) + m * p.ldo[1] + n0, n, p.vec_out, b);
    }
}

template <bool A_MN, bool B_MN, int EPI, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) k_product_pair(const __grid_constant__ ProductArgs p) {
    constexpr bool GATED = EPI == BNN_EPI_GATED || EPI == BNN_EPI_GATED_BACK;
    constexpr int WIDTH = GATED ? BN / 2 : BN;                   // output columns of a tile
    constexpr int STAGES = Ring<BN>::STAGES;
    constexpr uint32_t STAGE = Ring<BN>::STAGE, B_STAGE = Ring<BN>::B_STAGE, TMEM = Ring<BN>::TMEM;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Control *ctl = reinterpret_cast<Control *>(tiles + STAGES * STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&ctl->full[s]), 2); mbar_init(smem_u32(&ctl->empty[s]), 1); }
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
        // ---------------- producers: the thread of warp 0 loads A, the other one B.  The "full" barrier of a stage (in CTA 0)
        // completes with the arrivals of CTA 0's two producers and the bytes of both CTAs.
        if (lane == 0 && !p.drop_loads) {
            const bool is_a = warp == 0;
            bool ok = true;
            uint32_t stage = 0, lap = 0;
            bnn_pdl_wait();
            for (uint32_t t = pair; t < p.tiles && ok; t += pairs) {
                const Tile tile = tile_at<WIDTH>(p, t);
                const int m0 = (int)tile.m0 + (int)rank * 128;
                const int n0 = (int)tile.n0 + (GATED ? 0 : (int)rank * (BN / 2));
                for (int kit = 0; kit < p.k_iters; ++kit) {
                    if (lap > 0 && !wait(ctl, p.wait_ns, &ctl->empty[stage], (lap - 1) & 1)) { fail(ctl, 1); ok = false; break; }
                    const int second = kit >= p.k_pair ? 1 : 0, k = (kit - (second ? p.k_pair : 0)) * BK;
                    const uint32_t dst = smem_u32(tiles + stage * STAGE) + (is_a ? 0 : A_STAGE), bar = smem_u32(&ctl->full[stage]);
                    if (rank == 0) mbar_expect_tx(bar, 2 * (is_a ? A_STAGE : B_STAGE));
                    if (is_a) {
                        const CUtensorMap *map = &p.a[p.groups == 2 ? tile.group : second];
                        if constexpr (A_MN) {
                            tma_load_2d_2sm(dst, map, m0, k, bar & PEER_MASK);
                            tma_load_2d_2sm(dst + 8192, map, m0 + 64, k, bar & PEER_MASK);
                        } else tma_load_2d_2sm(dst, map, k, m0, bar & PEER_MASK);
                    } else {
                        const CUtensorMap *map = &p.b[GATED ? (int)rank : second];
                        if constexpr (B_MN) {
#pragma unroll
                            for (int i = 0; i < BN / 128; ++i) tma_load_2d_2sm(dst + i * 8192, map, n0 + i * 64, k, bar & PEER_MASK);
                        } else tma_load_2d_2sm(dst, map, k, n0, bar & PEER_MASK);
                    }
                    if (++stage == STAGES) { stage = 0; ++lap; }
                }
            }
            // after a failure: the copies still in flight land before the CTA gives its shared memory up
            if (is_a && rank == 0 && *reinterpret_cast<volatile uint32_t *>(&ctl->failed) != 0u) {
                const uint32_t issued = lap * STAGES + stage, first = issued > STAGES ? issued - STAGES : 0;
                for (uint32_t i = first; i < issued; ++i)
                    if (!wait(ctl, p.wait_ns, &ctl->full[i % STAGES], (i / STAGES) & 1, false)) break;
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint64_t a0 = A_MN ? smem_desc_mn(smem_u32(tiles)) : smem_desc_sw128(smem_u32(tiles));
            const uint64_t b0 = B_MN ? smem_desc_mn(smem_u32(tiles + A_STAGE)) : smem_desc_sw128(smem_u32(tiles + A_STAGE));
            constexpr uint64_t A_STEP = A_MN ? 2048 >> 4 : 32 >> 4, B_STEP = B_MN ? 2048 >> 4 : 32 >> 4;   // 16 elements of K
            uint32_t stage = 0, phase = 0, count = 0;
            bool ok = true;
            for (uint32_t t = pair; t < p.tiles && ok; t += pairs, ++count) {
                const uint32_t buf = count & 1, use = count >> 1;
                if (use > 0 && !wait(ctl, p.wait_ns, &ctl->acc_empty[buf], (use - 1) & 1)) { fail(ctl, 4); ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d = tmem_base + buf * BN;
                for (int kit = 0; kit < p.k_iters; ++kit) {
                    if (!wait(ctl, p.wait_ns, &ctl->full[stage], phase)) { fail(ctl, 2); ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = a0 + (uint64_t)(stage * (STAGE >> 4)), b = b0 + (uint64_t)(stage * (STAGE >> 4));
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) mma_f16_2sm(d, a + k * A_STEP, b + k * B_STEP, p.idesc, (kit | k) != 0 ? 1u : 0u);
                    umma_commit_2sm(smem_u32(&ctl->empty[stage]));
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                umma_commit_2sm(smem_u32(&ctl->acc_full[buf]));
            }
            if (!ok) {                               // the MMAs issued so far end before tensor memory is given back
                umma_commit_2sm(smem_u32(&ctl->drain));
                wait(ctl, p.wait_ns, &ctl->drain, 0, false);
            }
        }
    } else if (warp < 2 + EPI_WARPS) {
        bnn_pdl_wait();
        bnn_pdl_launch_next();
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t quadrant = (uint32_t)(32 * q) << 16;
        uint32_t count = 0;
        for (uint32_t t = pair; t < p.tiles; t += pairs, ++count) {
            const uint32_t buf = count & 1;
            const Tile tile = tile_at<WIDTH>(p, t);
            if (!wait(ctl, p.wait_ns, &ctl->acc_full[buf], (count >> 1) & 1)) { fail(ctl, 3); break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int64_t m = tile.m0 + rank * 128 + 32 * q + lane;
            const uint32_t acc = tmem_base + buf * BN + quadrant;
#pragma unroll 1
            for (int c = half * (WIDTH / 2); c < (half + 1) * (WIDTH / 2); c += 32) {
                if (tile.n0 + c >= p.N) break;
                uint32_t ra[32], rb[32];
                float a[32], b[32];
                tmem_ld32(acc + c, ra);
                if (GATED) tmem_ld32(acc + WIDTH + c, rb);
                tmem_ld_wait(ra);
                if (GATED) tmem_ld_wait(rb);
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    a[j] = p.k_iters ? __uint_as_float(ra[j]) : 0.0f;
                    if (GATED) b[j] = p.k_iters ? __uint_as_float(rb[j]) : 0.0f;
                }
                if (p.f16) finish32<EPI, __half>(p, tile.group, m, tile.n0 + c, a, b);
                else finish32<EPI, __nv_bfloat16>(p, tile.group, m, tile.n0 + c, a, b);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_cta0(smem_u32(&ctl->acc_empty[buf]));
        }
    }

    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                          // nobody leaves while the peer may still reach its shared memory
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------------------
template <int BN> constexpr size_t pair_smem() { return (size_t)Ring<BN>::STAGES * Ring<BN>::STAGE + sizeof(Control) + 1024; }

// Opts in to the shared memory and asks how many pairs fit the device, once per device and kernel; 0 = cannot run.
template <bool A_MN, bool B_MN, int EPI, int BN> int pairs_of(int device, int sm_count) {
    static std::mutex lock;
    static int cached[64];
    if (device < 0 || device >= 64) return 0;
    std::lock_guard<std::mutex> guard(lock);
    if (cached[device] == 0) {
        auto kernel = k_product_pair<A_MN, B_MN, EPI, BN>;
        int pairs = 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pair_smem<BN>()) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(2 * sm_count); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = pair_smem<BN>();
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

template <bool A_MN, bool B_MN, int EPI, int BN> int launch(bnn_ctx *ctx, const ProductArgs &a) {
    const int pairs = pairs_of<A_MN, B_MN, EPI, BN>(ctx->device, ctx->sm_count);
    if (pairs == 0) return BNN_ERR_CUDA;
    const unsigned n = a.tiles < (uint32_t)pairs ? a.tiles : (unsigned)pairs;
    BNN_CUDA_TRY(ctx, bnn_launch_dependent(k_product_pair<A_MN, B_MN, EPI, BN>, dim3(2 * n), dim3(THREADS), pair_smem<BN>(), ctx->stream, a));
    return bnn_check_launch(ctx);
}

int map16(bnn_ctx *ctx, CUtensorMap *map, const void *p, int64_t ld, int64_t rows, int64_t cols, int box_rows) {
    return bnn_tensor_map16(ctx, map, p, rows, cols, rows > 1 ? ld : (cols + 7) & ~int64_t(7), box_rows, BK);
}
int width_of(const void *p, int64_t ld, int64_t rows, int size) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint64_t pitch = rows > 1 ? (uint64_t)ld * size : 0;
    return (at | pitch) % 32 == 0 ? 2 : (at | pitch) % 16 == 0 ? 1 : 0;
}

}  // namespace

int bnn_product_status(bnn_ctx *ctx, int *code) {
    BNN_CUDA_TRY(ctx, cudaMemcpyFromSymbol(code, g_product_error, sizeof(int)));
    const int zero = 0;
    if (*code) BNN_CUDA_TRY(ctx, cudaMemcpyToSymbol(g_product_error, &zero, sizeof(int)));
    return BNN_OK;
}

int bnn_product(bnn_ctx *ctx, const BnnProduct &q) {
    const bool gated = q.epilogue == BNN_EPI_GATED || q.epilogue == BNN_EPI_GATED_BACK;
    const int bn = 256;
    ProductArgs a{};
    a.M = q.M; a.N = q.N;
    const int64_t steps = (q.K + BK - 1) / BK;
    a.k_pair = (int)steps; a.k_iters = (int)(steps * (gated ? 1 : q.pairs)); a.groups = q.groups;
    const int64_t width = gated ? bn / 2 : bn;
    const int64_t tm = (q.M + TM - 1) / TM, tn = (q.N + width - 1) / width;
    if (tm * tn * q.groups > 0x7fffffff) return BNN_ERR_INVALID_ARG;
    a.tiles_m = (uint32_t)tm; a.tiles_n = (uint32_t)tn; a.tiles = (uint32_t)(tm * tn * q.groups);
    const uint32_t type = q.dtype == BNN_BF16 ? 1u : 0u;
    a.idesc = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)q.a_mn << 15) | ((uint32_t)q.b_mn << 16) | ((uint32_t)(bn >> 3) << 17) |
              ((uint32_t)(TM >> 4) << 24);
    a.bias = q.bias; a.add = q.add; a.ld_add = q.ld_add; a.pre = q.pre; a.ldp = q.ldp; a.act = q.act; a.f16 = q.dtype == BNN_F16;
    for (int i = 0; i < 2; ++i) { a.out[i] = q.out[i]; a.ldo[i] = q.ldo[i]; }
    a.vec_bias = width_of(q.bias, 0, 1, 2); a.vec_add = width_of(q.add, q.ld_add, q.M, 2); a.vec_pre = width_of(q.pre, q.ldp, 2 * q.M, 4);
    a.vec_out = width_of(q.out[0], q.ldo[0], q.M, 2);
    if (q.out[1]) { const int v = width_of(q.out[1], q.ldo[1], q.M, 2); a.vec_out = v < a.vec_out ? v : a.vec_out; }
    a.wait_ns = ctx->wait_limit_ns; a.drop_loads = ctx->drop_loads;
    if (q.K > 0) {
        for (int i = 0; i < 2; ++i) {
            if (q.a[i].p)
                if (int st = q.a_mn ? map16(ctx, &a.a[i], q.a[i].p, q.a[i].ld, q.K, q.M, BK) : map16(ctx, &a.a[i], q.a[i].p, q.a[i].ld, q.M, q.K, 128)) return st;
            if (q.b[i].p)
                if (int st = q.b_mn ? map16(ctx, &a.b[i], q.b[i].p, q.b[i].ld, q.K, q.N, BK) : map16(ctx, &a.b[i], q.b[i].p, q.b[i].ld, q.N, q.K, bn / 2)) return st;
        }
    }
    if (q.a_mn) return launch<true, true, BNN_EPI_LINEAR, 256>(ctx, a);
    if (q.b_mn) return launch<false, true, BNN_EPI_LINEAR, 256>(ctx, a);
    switch (q.epilogue) {
        case BNN_EPI_LINEAR: return launch<false, false, BNN_EPI_LINEAR, 256>(ctx, a);
        case BNN_EPI_LINEAR_BACK: return launch<false, false, BNN_EPI_LINEAR_BACK, 256>(ctx, a);
        case BNN_EPI_GATED: return launch<false, false, BNN_EPI_GATED, 256>(ctx, a);
        default: return launch<false, false, BNN_EPI_GATED_BACK, 256>(ctx, a);
    }
}
