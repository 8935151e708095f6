// The norm of all gradients of a model together, and their clipping.
//
// Mathematics:  n = sqrt(sum over all tensors of g^2),  f = min(1, max_norm / (n + eps)),  out = f g.
// Bound: HBM.  Two launches: the sums of squares, then the factor (every block adds up the same partial sums in the same order) and the
// scaled values.  Every element is read twice and written once; the second launch goes backwards, so that what the first read last comes from L2.
// Squares are added in float32 over the 32 elements that a thread takes at a time, and those sums in float64: 2^-19 relative at most, whatever
// the number of elements.  Measured: 705 MB of bf16 in 49 tensors 347 us (squares 112 = 6.3 TB/s, then 1.41 GB at 6.0 TB/s), in place and not clipped 114 us; 4 MB in eight tensors
// 5.6 us, 8 with the host's call.  Blocks: four per SM (two 417, three 355, six 376 us).  Where a float32 sum of squares has left the range in which that holds (elements above 1.8e19 or all below 1e-15), the
// squares are formed in float64.
#include "bnn_real.cuh"

namespace {

constexpr int THREADS = 256, PER = 32, CHUNK = THREADS * PER, PER_SM = 4;
struct Entry {
    const void *g;
    void *out;
    int64_t n;
    uint32_t first;        // first chunk of the launch's numbering
    int32_t dtype;
};
template <int N> struct ClipArgs {
    Entry e[N];
    int count;
    uint32_t chunks;
    double *part;          // partial sums: of this launch from here on
    const double *parts;   // all of them
    int sums;
    float *norm;
    double max_norm, eps;
    int writes_norm, in_place;   // every tensor of the launch is its own output
};
constexpr int FEW = 24, MANY = 1000;      // tensors of a launch; its arguments are 0.9 or 32 KB

template <typename T> constexpr int group_of() { return 16 / (int)sizeof(T); }

// Elements in front of the first 16-byte boundary; -1 where reading and writing are not on the same footing.
template <typename T> __device__ __forceinline__ int head_of(const Entry &e, bool writes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(e.g), b = reinterpret_cast<uintptr_t>(e.out);
    if (writes && ((a ^ b) & 15)) return -1;
    const int64_t h = (int64_t)(((16 - (a & 15)) & 15) / sizeof(T));
    return (int)(h < e.n ? h : e.n);
}

template <typename T> __device__ __forceinline__ double square_sum(const float (&v)[PER]) {
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) q += v[i] * v[i];
    if (q >= 1e-28f && q <= 3e38f) return (double)q;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) d += (double)v[i] * (double)v[i];
    return d;
}

// The chunk's elements of this thread: PER of them, in 16-byte groups (head >= 0) or one by one a block's width apart; zeros behind the end.
// f: called with the values' index and the values of a group.
template <typename T> __device__ __forceinline__ void read_chunk(const Entry &e, int64_t base, int head, float (&v)[PER]) {
    constexpr int G = group_of<T>();
    const T *g = static_cast<const T *>(e.g);
    if (head >= 0) {
        const int64_t at = head + base;
        if (at + CHUNK <= e.n) {
            uint4 w[PER / G];
#pragma unroll
            for (int i = 0; i < PER / G; ++i) w[i] = reinterpret_cast<const uint4 *>(g + at)[i * THREADS + threadIdx.x];
#pragma unroll
            for (int i = 0; i < PER / 8; ++i) {
                float t[8];
                unpack8<T>(w + i * (8 / G), t);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[8 * i + j] = t[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER / G; ++i)
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    const int64_t k = at + (int64_t)(i * THREADS + threadIdx.x) * G + j;
                    v[G * i + j] = k < e.n ? to_f32(g[k]) : 0.0f;
                }
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t k = base + i * THREADS + threadIdx.x;
            v[i] = k < e.n ? to_f32(g[k]) : 0.0f;
        }
    }
}
template <typename T> __device__ __forceinline__ double chunk_squares(const Entry &e, int64_t base) {
    const int head = head_of<T>(e, false);
    float v[PER];
    read_chunk<T>(e, base, head, v);
    double d = square_sum<T>(v);
    if (base == 0 && (int)threadIdx.x < head) {
        const double t = (double)to_f32(static_cast<const T *>(e.g)[threadIdx.x]);
        d += t * t;
    }
    return d;
}
template <typename T> __device__ __forceinline__ void chunk_scale(const Entry &e, int64_t base, float f) {
    constexpr int G = group_of<T>();
    const int head = head_of<T>(e, true);
    float v[PER];
    read_chunk<T>(e, base, head, v);
    T *out = static_cast<T *>(e.out);
    if (head >= 0) {
        const int64_t at = head + base;
        if (at + CHUNK <= e.n) {
#pragma unroll
            for (int i = 0; i < PER / G; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (sizeof(T) == 4) w[k] = __float_as_uint(v[4 * i + k] * f);
                    else w[k] = pack2<T>(v[8 * i + 2 * k] * f, v[8 * i + 2 * k + 1] * f);
                }
                __stcs(reinterpret_cast<uint4 *>(out + at) + i * THREADS + threadIdx.x, make_uint4(w[0], w[1], w[2], w[3]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER / G; ++i)
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    const int64_t k = at + (int64_t)(i * THREADS + threadIdx.x) * G + j;
                    if (k < e.n) out[k] = from_f32<T>(v[G * i + j] * f);
                }
        }
        if (base == 0 && (int)threadIdx.x < head) out[threadIdx.x] = from_f32<T>(to_f32(static_cast<const T *>(e.g)[threadIdx.x]) * f);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t k = base + i * THREADS + threadIdx.x;
            if (k < e.n) out[k] = from_f32<T>(v[i] * f);
        }
    }
}

__device__ __forceinline__ double block_sum(double d, double *buf) {
#pragma unroll
    for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = d;
    __syncthreads();
    d = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) d += buf[w];
    return d;
}
template <int N> __device__ __forceinline__ int entry_of(const ClipArgs<N> &p, uint32_t chunk) {
    int low = 0, high = p.count - 1;
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (p.e[mid].first <= chunk) low = mid; else high = mid - 1;
    }
    return low;
}

template <int N> __global__ void __launch_bounds__(THREADS) k_clip_squares(const __grid_constant__ ClipArgs<N> p) {
    __shared__ double buf[THREADS / 32];
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    double d = 0.0;
    for (uint32_t c = blockIdx.x; c < p.chunks; c += gridDim.x) {
        const Entry &e = p.e[entry_of(p, c)];
        const int64_t base = (int64_t)(c - e.first) * CHUNK;
        d += e.dtype == BNN_F32 ? chunk_squares<float>(e, base) : e.dtype == BNN_F16 ? chunk_squares<__half>(e, base) : chunk_squares<__nv_bfloat16>(e, base);
    }
    d = block_sum(d, buf);
    if (threadIdx.x == 0) p.part[blockIdx.x] = d;
}
template <int N> __global__ void __launch_bounds__(THREADS) k_clip_scale(const __grid_constant__ ClipArgs<N> p) {
    __shared__ double buf[THREADS / 32];
    bnn_pdl_wait();
    bnn_pdl_launch_next();
    double d = 0.0;
    for (int i = threadIdx.x; i < p.sums; i += THREADS) d += p.parts[i];
    const double norm = sqrt(block_sum(d, buf));
    const double all = norm + p.eps, share = p.max_norm / all;
    const float f = all == 0.0 || share >= 1.0 ? 1.0f : (float)share;      // a NaN stays one
    if (blockIdx.x == 0 && threadIdx.x == 0 && p.writes_norm) *p.norm = (float)norm;
    if (f == 1.0f && p.in_place) return;                     // nothing to change
    for (uint32_t i = blockIdx.x; i < p.chunks; i += gridDim.x) {
        const uint32_t c = p.chunks - 1 - i;
        const Entry &e = p.e[entry_of(p, c)];
        if (f == 1.0f && e.out == e.g) continue;
        const int64_t base = (int64_t)(c - e.first) * CHUNK;
        if (e.dtype == BNN_F32) chunk_scale<float>(e, base, f);
        else if (e.dtype == BNN_F16) chunk_scale<__half>(e, base, f);
        else chunk_scale<__nv_bfloat16>(e, base, f);
    }
}

int64_t chunks_of(const bnn_gradient &g) { return g.n > 0 ? (g.n + CHUNK - 1) / CHUNK : 0; }
// Launches of the set, each of at most MANY tensors and 2^31 chunks.
int64_t launches_of(int64_t count) { return count > 0 ? (count + MANY - 1) / MANY : 1; }

template <int N> int fill(ClipArgs<N> &a, const bnn_gradient *list, int64_t from, int64_t to) {
    uint64_t chunks = 0;
    a.count = 0;
    a.in_place = 1;
    for (int64_t i = from; i < to; ++i) {
        if (list[i].n == 0) continue;
        Entry &e = a.e[a.count++];
        e.g = list[i].g; e.out = list[i].out; e.n = list[i].n; e.first = (uint32_t)chunks; e.dtype = list[i].dtype;
        if (e.out != e.g) a.in_place = 0;
        chunks += (uint64_t)chunks_of(list[i]);
        if (chunks > 0x7fffffffu) return BNN_ERR_INVALID_ARG;
    }
    a.chunks = (uint32_t)chunks;
    return BNN_OK;
}
template <int N> int clip(bnn_ctx *ctx, const bnn_gradient *list, int64_t count, double max_norm, double eps, float *norm) {
    const int64_t rounds = launches_of(count), most = (int64_t)ctx->sm_count * PER_SM;
    double *part = static_cast<double *>(ctx->ws);
    int sums = 0;
    for (int pass = 0; pass < 2; ++pass)
        for (int64_t k = 0; k < rounds; ++k) {
            const int64_t r = pass ? rounds - 1 - k : k;
            ClipArgs<N> a;
            if (int st = fill(a, list, r * MANY, (r + 1) * MANY < count ? (r + 1) * MANY : count)) return st;
            const unsigned blocks = a.chunks == 0 ? 1 : a.chunks < most ? a.chunks : (unsigned)most;
            a.part = part + sums; a.parts = part; a.sums = sums; a.norm = norm; a.max_norm = max_norm; a.eps = eps; a.writes_norm = k == 0;
            BNN_CUDA_TRY(ctx, bnn_launch_dependent(pass ? k_clip_scale<N> : k_clip_squares<N>, dim3(blocks), dim3(THREADS), 0, ctx->stream, a));
            if (int st = bnn_check_launch(ctx)) return st;
            if (!pass) sums += (int)blocks;
        }
    return BNN_OK;
}

}  // namespace

extern "C" size_t bnn_clip_workspace_bytes(int64_t count) {
    if (count < 0 || count > BNN_REAL_MAX) return 0;
    return ((size_t)launches_of(count) * 1024 * PER_SM * sizeof(double) + 255) & ~size_t(255);
}

extern "C" int bnn_clip_gradients(bnn_ctx *ctx, const bnn_gradient *list, int64_t count, double max_norm, double eps, float *norm) {
    if (count < 0 || count > BNN_REAL_MAX || (count > 0 && !list) || !norm || !(max_norm >= 0.0) || !(eps >= 0.0)) return BNN_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(norm) % 4) return BNN_ERR_ALIGNMENT;
    for (int64_t i = 0; i < count; ++i) {
        const int size = bnn_real_size(list[i].dtype);
        if (!size || list[i].n < 0) return BNN_ERR_INVALID_ARG;
        if (list[i].n == 0) continue;
        if (!list[i].g || !list[i].out) return BNN_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(list[i].g) % size || reinterpret_cast<uintptr_t>(list[i].out) % size) return BNN_ERR_ALIGNMENT;
    }
    if (!ctx) return BNN_ERR_INVALID_ARG;
    bnn_device_guard guard(ctx);
    if (!guard.ok) return BNN_ERR_CUDA;
    if (!ctx->ws || ctx->ws_bytes < bnn_clip_workspace_bytes(count)) return BNN_ERR_WORKSPACE;
    return count <= FEW ? clip<FEW>(ctx, list, count, max_norm, eps, norm) : clip<MANY>(ctx, list, count, max_norm, eps, norm);
}
