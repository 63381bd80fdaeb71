// Group norm with an activation over channels-last images [B, HW, C], forward and gradient.
//
//   xhat = (x - mean) rstd over the HW x C/G values of an image's group;  z = xhat weight + bias;  out = act(z)
//   g = d_out act'(z);  dbias_c = sum g;  dweight_c = sum g xhat;  dx = rstd (g w - mean(g w) - xhat mean(g w xhat))
//
// Memory bounds all of it, so an image's groups stay on chip between the statistics and their use wherever they fit: a cluster of up to
// eight blocks holds all rows of a slab of whole groups in shared memory (16-byte vectors, a thread's vectors all of the same channels), sums
// are exchanged through distributed shared memory, and every value crosses memory once in and once out.  Larger images go through
// it twice, in launches of their own.  Variances are sums of squares about a mean that is known: a block's own first, moved to the
// image's when blocks are joined, so that a mean far from zero costs no digits.  All sums run in a fixed order.
// 64 x 56 x 56 x 96 bf16 with SiLU (77 MB): 31 us, 0.38 of the rate of a copy: a block's phases follow one another (load, sums, cluster, results), two
// blocks an SM.  64 x 14 x 14 x 768: 18 us, its gradient with the parameters' 28 us.
#include <type_traits>

#include "gdr.h"
#include "ptx.cuh"

namespace vig {
namespace {

constexpr int kActNone = VIG_ACT_NONE, kActSilu = VIG_ACT_SILU, kActGelu = VIG_ACT_GELU;
constexpr int kThreads = 256;
constexpr int kMostBlocks = 8;   // of a cluster (portable)

template <typename T>
struct Wide {   // 16 bytes of T
    static constexpr int N = 16 / sizeof(T);
};
__device__ __forceinline__ void widen16(const uint4& r, float (&f)[4], const float*) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void widen16(const uint4& r, float (&f)[8], const __nv_bfloat16*) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ float one(const float* p, long long i, float none) { return p ? p[i] : none; }
__device__ __forceinline__ float one(const __nv_bfloat16* p, long long i, float none) { return p ? __bfloat162float(p[i]) : none; }
__device__ __forceinline__ void put(float* p, long long i, float x) { p[i] = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, long long i, float x) { p[i] = __float2bfloat16_rn(x); }

// The same as pairs of fp32: two values an instruction (all of it is issue-bound otherwise: 42 instructions a value, 94 us for 64 x 56 x 56 x 96).
__device__ __forceinline__ void widen16(const uint4& r, f32x2 (&f)[2], const float*) {
    f[0] = pack2(__uint_as_float(r.x), __uint_as_float(r.y));
    f[1] = pack2(__uint_as_float(r.z), __uint_as_float(r.w));
}
__device__ __forceinline__ void widen16(const uint4& r, f32x2 (&f)[4], const __nv_bfloat16*) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 narrow16(const f32x2 (&f)[2], const float*) {
    float a, b, c, d;
    unpack2(f[0], a, b);
    unpack2(f[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
}
__device__ __forceinline__ uint4 narrow16(const f32x2 (&f)[4], const __nv_bfloat16*) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpack2(f[i], a, b);
        u[i] = pack_bf16(a, b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ f32x2 both(float x) { return pack2(x, x); }
__device__ __forceinline__ f32x2 fsub2(f32x2 a, f32x2 b) { return ffma2(b, both(-1.f), a); }
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// FAST (results rounded to bf16): e^-z and the reciprocal from the special-function unit, relative error below 1e-6.
template <bool FAST>
__device__ __forceinline__ f32x2 sigmoid2(f32x2 z) {
    if constexpr (FAST) {
        float a, b;
        unpack2(fmul2(z, both(-1.4426950408889634f)), a, b);
        unpack2(fadd2(pack2(ex2(a), ex2(b)), both(1.f)), a, b);
        return pack2(rcp_approx(a), rcp_approx(b));   // (of infinity: 0)
    } else {
        float a, b;
        unpack2(z, a, b);
        return pack2(1.f / (1.f + expf(-a)), 1.f / (1.f + expf(-b)));
    }
}
__device__ __forceinline__ float gelu_cdf(float z) { return 0.5f * erfcf(-0.70710678118654752f * z); }
template <int ACT, bool FAST>
__device__ __forceinline__ f32x2 act2(f32x2 z) {
    if constexpr (ACT == kActSilu) return fmul2(z, sigmoid2<FAST>(z));
    else if constexpr (ACT == kActGelu) {
        float a, b;
        unpack2(z, a, b);
        return pack2(a * gelu_cdf(a), b * gelu_cdf(b));
    } else return z;
}
template <int ACT, bool FAST>
__device__ __forceinline__ f32x2 slope2(f32x2 z) {
    if constexpr (ACT == kActSilu) {
        const f32x2 s = sigmoid2<FAST>(z);
        return fmul2(s, ffma2(z, fsub2(both(1.f), s), both(1.f)));
    } else if constexpr (ACT == kActGelu) {
        float a, b;
        unpack2(z, a, b);
        auto one_slope = [](float x) {
            const float phi = 0.3989422804014327f * (FAST ? ex2(-0.7213475204444817f * x * x) : expf(-0.5f * x * x));
            return fmaf(x, phi, gelu_cdf(x));
        };
        return pack2(one_slope(a), one_slope(b));
    } else return both(1.f);
}

// x / d without the two dozen instructions of a division: x below 2^16, d from the host.
struct Div {
    uint32_t m;
    int d;
    Div() = default;
    explicit Div(int by) : m(by > 1 ? (uint32_t)((1ULL << 32) / by) + 1u : 0u), d(by) {}
    __device__ __forceinline__ int of(int x) const { return d == 1 ? x : (int)__umulhi((uint32_t)x, m); }
};

template <typename T>
struct Norm {
    const T *x, *weight, *bias, *d_out;
    T *out, *dx;
    float *mean, *rstd;      // [B][G]; forward: null where the caller does not want them
    const float *cmean, *crstd;   // the gradient's
    float2* part;            // scratch: [rows][C]
    int HW, C, per;          // per: channels of a group
    float eps;
    int slab, rows;          // channels of a block; rows of a block
    int blocks;              // of an image (on chip: slabs x blocks of a cluster; else chunks of rows)
    // on chip: row lanes, groups of the slab, entries of the slab and of a group, threads of an entry; divisors
    int lanes, groups, entries, width, parts;
    int held;                // floats of shared memory in front of the vectors
    Div by_vectors, by_entries, by_slab, by_per, by_lanes;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// This variable of another block of the cluster.  Blocks write what they have into each other's memory ahead of the one barrier that they then meet at
// (reading it from there behind the barrier, with another one before the end, was as fast when the vectors lay in registers: 40 us for 64 x 56 x 56 x 96).
__device__ __forceinline__ void put_peer(float2* p, uint32_t rank, float2 x) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(cluster_peer(smem_u32(p), rank)), "f"(x.x), "f"(x.y) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_await() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// A vector of the parameters, or `none` where there are none.
template <typename T>
__device__ __forceinline__ void params(const T* p, int c, float none, f32x2 (&f)[Wide<T>::N / 2]) {
    if (p) widen16(*reinterpret_cast<const uint4*>(p + c), f, p);
    else
#pragma unroll
        for (int e = 0; e < Wide<T>::N / 2; ++e) f[e] = both(none);
}
// f(pair, group of its first, group of its second) of a vector's channels c .. c + V - 1
template <int V, typename F>
__device__ __forceinline__ void over_pairs(int c, int g, int per, F f) {   // g: the first one's
    int r = c - g * per;
#pragma unroll
    for (int e = 0; e < V; e += 2) {
        const int g0 = g;
        if (++r == per) r = 0, ++g;
        const int g1 = g;
        if (++r == per) r = 0, ++g;
        f(e / 2, g0, g1);
    }
}
// On chip, threads leave what they have per entry, [row lane][entry of the slab]: an entry is a vector where a vector lies in one group (per a
// multiple of V), else a channel.  (Sums of an entry over its row lanes by several threads, then a warp per group: each a handful of steps.
// A warp per group straight away took 3400 cycles of a block's 20000.)
constexpr size_t on_chip_floats(int lanes, int slab, int groups) { return 2 * ((size_t)lanes * slab + (1 + kMostBlocks) * groups + (slab > kThreads ? slab : kThreads)); }

// A vector's channels in the gradient.
template <typename T>
struct Channels {
    static constexpr int V = Wide<T>::N;
    f32x2 m[V / 2], rs[V / 2], w[V / 2], b[V / 2];
    // c: the first channel; groups count from group0, whose first channel is c0
    __device__ __forceinline__ void load(const Norm<T>& a, long long group0, int c0, int c, bool live) {
        params(a.weight, live ? c0 + c : 0, 1.f, w);
        params(a.bias, live ? c0 + c : 0, 0.f, b);
        if (live)
            over_pairs<V>(c, c < 1 << 16 ? a.by_per.of(c) : c / a.per, a.per, [&](int e, int g0, int g1) {
                m[e] = pack2(a.cmean[group0 + g0], a.cmean[group0 + g1]);
                rs[e] = pack2(a.crstd[group0 + g0], a.crstd[group0 + g1]);
            });
    }
    // h = xhat, g = d_out act'(z)
    template <int ACT>
    __device__ __forceinline__ void grad(const uint4& x, const uint4& d, f32x2 (&h)[V / 2], f32x2 (&g)[V / 2]) const {
        f32x2 f[V / 2];
        widen16(x, f, (const T*)nullptr);
        widen16(d, g, (const T*)nullptr);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            h[e] = fmul2(fsub2(f[e], m[e]), rs[e]);
            if constexpr (ACT != kActNone) g[e] = fmul2(g[e], slope2<ACT, sizeof(T) == 2>(ffma2(h[e], w[e], b[e])));
        }
    }
    // g <- rstd (g w - m1 - h m2)
    __device__ __forceinline__ void dx(const f32x2 (&h)[V / 2], f32x2 (&g)[V / 2], const f32x2 (&m1)[V / 2], const f32x2 (&m2)[V / 2]) const {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) g[e] = fmul2(rs[e], fsub2(fsub2(fmul2(g[e], w[e]), m1[e]), fmul2(h[e], m2[e])));
    }
};

__device__ __forceinline__ void cp_async16(uint4* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_all() { asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory"); }

// ---- on chip: grid (blocks of a cluster x slabs x B) --------------------------------------------------------------------------
// A thread's vectors lie in shared memory, brought there by its own asynchronous copies and read by nobody else.  (In registers, 16 of them a thread: 40 us
// where this takes 35 with 16 and 31 with 24.)
template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads, 4) norm_kernel(Norm<T> a, int N) {
    constexpr int V = Wide<T>::N;
    extern __shared__ __align__(16) float smem[];
    const int lanes = a.lanes, tid = threadIdx.x, rl = a.by_vectors.of(tid), vc = tid - rl * a.by_vectors.d, groups = a.groups;
    const int entries = a.entries, width = a.width;
    const bool vectors = entries < a.slab;
    float2 *const red = reinterpret_cast<float2*>(smem), *const own = red + lanes * entries, *const all = own + kMostBlocks * groups, *const sums = all + groups;   // own: of every block of the cluster
    const long long image = blockIdx.x / a.blocks;
    const int slab = blockIdx.x % a.blocks / N, rank = blockIdx.x % N;
    const int c0 = slab * a.slab, row0 = rank * a.rows, rows = max(0, min(a.rows, a.HW - row0));
    const bool live = rl < lanes;
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    if (N > 1) cluster_arrive();   // (the others may write here from then on)
    pdl_wait();
    pdl_launch_dependents();
    uint4* const x = reinterpret_cast<uint4*>(smem + a.held) + tid;   // every kThreads-th
    const int full = a.by_lanes.of(rows), rest = rows - full * lanes;   // vectors of a row lane: full, or one more
    const int n = live ? full + (rl < rest) : 0;
    for (int i = 0; i < n; ++i) cp_async16(x + i * kThreads, a.x + base + (long long)(rl + i * lanes) * a.C);
    // this thread's mean and sum of squares about it per channel, in one pass about its own first value: as that value is one of them, the
    // sum about it is at most n + 1 times the sum about the mean, and so is what rounding costs
    f32x2 w[V / 2], b[V / 2], first[V / 2], sum[V / 2], sq[V / 2];
    params(a.weight, live ? c0 + vc * V : 0, 1.f, w);
    params(a.bias, live ? c0 + vc * V : 0, 0.f, b);
    cp_async_all();
    widen16(n > 0 ? x[0] : make_uint4(0u, 0u, 0u, 0u), first, a.x);
#pragma unroll
    for (int e = 0; e < V / 2; ++e) sum[e] = sq[e] = both(0.f);
#pragma unroll 2
    for (int i = 1; i < n; ++i) {
        f32x2 f[V / 2];
        widen16(x[i * kThreads], f, a.x);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            const f32x2 d = fsub2(f[e], first[e]);
            sum[e] = fadd2(sum[e], d);
            sq[e] = ffma2(d, d, sq[e]);
        }
    }
    if (live) {
        const float inv = n > 0 ? 1.f / (float)n : 0.f;
        float mean[V], m2[V];
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            float f0, f1, s0, s1, q0, q1;
            unpack2(first[e], f0, f1);
            unpack2(sum[e], s0, s1);
            unpack2(sq[e], q0, q1);
            mean[2 * e] = fmaf(s0, inv, f0);
            mean[2 * e + 1] = fmaf(s1, inv, f1);
            // (the product inside does not overflow by itself: not a number only where the mean is not finite either, which carries it)
            m2[2 * e] = fmaxf(fmaf(-s0 * inv, s0, q0), 0.f);
            m2[2 * e + 1] = fmaxf(fmaf(-s1 * inv, s1, q1), 0.f);
        }
        if (vectors) {
            float m = 0.f, q = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) m += mean[e];
            m *= 1.f / V;
#pragma unroll
            for (int e = 0; e < V; ++e) q += fmaf((mean[e] - m) * (float)n, mean[e] - m, m2[e]);
            red[rl * entries + vc] = make_float2(m, q);
        } else
#pragma unroll
            for (int e = 0; e < V; e += 2) *reinterpret_cast<float4*>(red + rl * entries + vc * V + e) = make_float4(mean[e], m2[e], mean[e + 1], m2[e + 1]);
    }
    __syncthreads();
    const float values = vectors ? (float)V : 1.f;               // of an entry and row
    // an entry over its row lanes, about the first one's mean; then per entry: mean and sum of squares about it
    const int parts = a.parts;
    for (int i = tid; i < entries * parts; i += blockDim.x) {
        const int part = a.by_entries.of(i), c = i - part * entries;
        const float first_mean = red[c].x;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll 4
        for (int r = part; r < lanes; r += parts) {
            const float2 y = red[r * entries + c];
            const float k = (float)(full + (r < rest)) * values, d = y.x - first_mean;
            s1 = fmaf(k, d, s1);
            s2 += fmaf(k * d, d, y.y);
        }
        sums[i] = make_float2(s1, s2);
    }
    __syncthreads();
    if (N > 1) cluster_await();
    const float per_entry = (float)rows * values, of_entry = rows > 0 ? 1.f / per_entry : 0.f, of_group = 1.f / (float)width;
    for (int j = tid >> 5; j < groups; j += blockDim.x >> 5) {
        auto entry = [&](int c, float& m, float& q) {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll 4
            for (int p = 0; p < parts; ++p) {
                const float2 y = sums[p * entries + c];
                s1 += y.x;
                s2 += y.y;
            }
            m = fmaf(s1, of_entry, red[c].x);
            q = fmaxf(fmaf(-s1 * of_entry, s1, s2), 0.f);
        };
        const int lane = tid & 31;
        float m = 0.f, q = 0.f;
        if (width <= 32) {
            float me = 0.f, qe = 0.f;
            if (lane < width) entry(j * width + lane, me, qe);
            m = warp_sum(me) * of_group;
            q = warp_sum(lane < width ? fmaf(per_entry * (me - m), me - m, qe) : 0.f);
        } else {
            for (int c = lane; c < width; c += 32) {
                float me, qe;
                entry(j * width + c, me, qe);
                m += me;
            }
            m = warp_sum(m) * of_group;
            for (int c = lane; c < width; c += 32) {
                float me, qe;
                entry(j * width + c, me, qe);
                q += fmaf(per_entry * (me - m), me - m, qe);
            }
            q = warp_sum(q);
        }
        if (N > 1) {
            if (lane < N) put_peer(own + rank * groups + j, lane, make_float2(m, q));
        } else if (lane == 0) own[j] = make_float2(m, q);
    }
    if (N > 1) {
        cluster_arrive();
        cluster_await();
    } else __syncthreads();
    for (int j = tid; j < groups; j += blockDim.x) {
        float m = own[j].x, q = own[j].y;
        if (N > 1) {
            float2 peer[kMostBlocks];
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) peer[p] = own[p * groups + j];
            auto share = [&](int p) { return (float)max(0, min(a.rows, a.HW - p * a.rows)); };   // rows of block p
            m = q = 0.f;
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) m = fmaf(share(p), peer[p].x, m);
            m /= (float)a.HW;
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) q += fmaf(share(p) * a.per * (peer[p].x - m), peer[p].x - m, peer[p].y);
        }
        const float rstd = rsqrtf(q / ((float)a.HW * a.per) + a.eps);
        all[j] = make_float2(m, rstd);
        if (rank == 0) {
            const long long at = image * (a.C / a.per) + c0 / a.per + j;
            if (a.mean) a.mean[at] = m;
            if (a.rstd) a.rstd[at] = rstd;
        }
    }
    __syncthreads();
    f32x2 m[V / 2];
    if (live)
        over_pairs<V>(vc * V, a.by_per.of(vc * V), a.per, [&](int e, int g0, int g1) {
            const float2 s0 = all[g0], s1 = all[g1];
            m[e] = pack2(s0.x, s1.x);
            w[e] = fmul2(w[e], pack2(s0.y, s1.y));
        });
#pragma unroll 2
    for (int i = 0; i < n; ++i) {
        f32x2 f[V / 2];
        widen16(x[i * kThreads], f, a.x);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) f[e] = act2<ACT, sizeof(T) == 2>(ffma2(fsub2(f[e], m[e]), w[e], b[e]));
        *reinterpret_cast<uint4*>(a.out + base + (long long)(rl + i * lanes) * a.C) = narrow16(f, a.x);
    }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads, 3) norm_grad_kernel(Norm<T> a, int N, int K) {   // K: vectors of a thread, at most
    constexpr int V = Wide<T>::N;
    extern __shared__ __align__(16) float smem[];
    const int lanes = a.lanes, tid = threadIdx.x, rl = a.by_vectors.of(tid), vc = tid - rl * a.by_vectors.d, groups = a.groups;
    float2 *const red = reinterpret_cast<float2*>(smem), *const own = red + lanes * a.slab, *const all = own + kMostBlocks * groups;   // own: of every block of the cluster
    const long long image = blockIdx.x / a.blocks;
    const int slab = blockIdx.x % a.blocks / N, rank = blockIdx.x % N;
    const int c0 = slab * a.slab, row0 = rank * a.rows, rows = max(0, min(a.rows, a.HW - row0));
    const bool live = rl < lanes;
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    if (N > 1) cluster_arrive();   // (the others may write here from then on)
    pdl_wait();
    pdl_launch_dependents();
    uint4 *const x = reinterpret_cast<uint4*>(smem + a.held) + tid, *const d = x + K * kThreads;
    const int full = a.by_lanes.of(rows), n = live ? full + (rl < rows - full * lanes) : 0;
    for (int i = 0; i < n; ++i) {
        const long long at = base + (long long)(rl + i * lanes) * a.C;
        cp_async16(x + i * kThreads, a.x + at);
        cp_async16(d + i * kThreads, a.d_out + at);
    }
    Channels<T> ch;
    ch.load(a, image * (a.C / a.per) + c0 / a.per, c0, vc * V, live);
    cp_async_all();
    constexpr bool kKeepG = sizeof(T) == 4;   // g takes d_out's place where it fits: no second pass through the activation
    f32x2 sg[V / 2], sx[V / 2];
#pragma unroll
    for (int e = 0; e < V / 2; ++e) sg[e] = sx[e] = both(0.f);
    for (int i = 0; i < n; ++i) {
        f32x2 h[V / 2], g[V / 2];
        ch.template grad<ACT>(x[i * kThreads], d[i * kThreads], h, g);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            sg[e] = fadd2(sg[e], g[e]);
            sx[e] = ffma2(g[e], h[e], sx[e]);
        }
        if constexpr (kKeepG) d[i * kThreads] = narrow16(g, a.x);
    }
    if (live)
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            float g0, g1, x0, x1;
            unpack2(sg[e], g0, g1);
            unpack2(sx[e], x0, x1);
            *reinterpret_cast<float4*>(red + rl * a.slab + vc * V + 2 * e) = make_float4(g0, x0, g1, x1);
        }
    __syncthreads();
    // a channel's sums over the block, several threads a channel: what the parameters' gradients and the group's means are made of
    const int parts = a.parts;
    for (int i = tid; i < a.slab * parts; i += blockDim.x) {
        const int part = a.by_slab.of(i), c = i - part * a.slab;
        float u = 0.f, v = 0.f;
#pragma unroll 4
        for (int l = part; l < lanes; l += parts) {
            const float2 y = red[l * a.slab + c];
            u += y.x;
            v += y.y;
        }
        red[part * a.slab + c] = make_float2(u, v);   // (row lane `part` of this very channel: read by this thread alone)
    }
    __syncthreads();
    if (N > 1) cluster_await();
    for (int j = tid >> 5; j < groups; j += blockDim.x >> 5) {
        float u = 0.f, v = 0.f;
        for (int c = j * a.per + (tid & 31); c < (j + 1) * a.per; c += 32) {
            float su = 0.f, sv = 0.f;
            for (int p = 0; p < parts; ++p) {
                const float2 y = red[p * a.slab + c];
                su += y.x;
                sv += y.y;
            }
            a.part[(image * N + rank) * a.C + c0 + c] = make_float2(su, sv);
            const float wc = one(a.weight, c0 + c, 1.f);
            u = fmaf(su, wc, u);
            v = fmaf(sv, wc, v);
        }
        u = warp_sum(u);
        v = warp_sum(v);
        if (N > 1) {
            if ((tid & 31) < N) put_peer(own + rank * groups + j, tid & 31, make_float2(u, v));
        } else if ((tid & 31) == 0) own[j] = make_float2(u, v);
    }
    if (N > 1) {
        cluster_arrive();
        cluster_await();
    } else __syncthreads();
    const float inv = 1.f / ((float)a.HW * a.per);
    for (int j = tid; j < groups; j += blockDim.x) {
        float2 sum = own[j];
        if (N > 1) {
            sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) {
                    const float2 y = own[p * groups + j];
                    sum.x += y.x;
                    sum.y += y.y;
                }
        }
        all[j] = make_float2(sum.x * inv, sum.y * inv);
    }
    __syncthreads();
    f32x2 m1[V / 2], m2[V / 2];
    if (live)
        over_pairs<V>(vc * V, a.by_per.of(vc * V), a.per, [&](int e, int g0, int g1) {
            const float2 s0 = all[g0], s1 = all[g1];
            m1[e] = pack2(s0.x, s1.x);
            m2[e] = pack2(s0.y, s1.y);
        });
    for (int i = 0; i < n; ++i) {
        f32x2 h[V / 2], g[V / 2];
        ch.template grad<kKeepG ? kActNone : ACT>(x[i * kThreads], d[i * kThreads], h, g);
        ch.dx(h, g, m1, m2);
        *reinterpret_cast<uint4*>(a.dx + base + (long long)(rl + i * lanes) * a.C) = narrow16(g, a.x);
    }
}

// ---- larger images: three launches.  Grid (chunks of rows x B, 1, slabs of at most 256 vectors) ------------------------------------
// A channel's mean over the chunk and sum of squares about it; four rows at a time, each four about their own mean.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_stats_kernel(Norm<T> a) {
    constexpr int V = Wide<T>::N;
    extern __shared__ __align__(16) float smem[];
    const int c0 = blockIdx.z * a.slab, slab = min(a.slab, a.C - c0);
    const int nv = slab / V, lanes = kThreads / nv, tid = threadIdx.x, vc = tid % nv, rl = tid / nv;
    const long long image = blockIdx.x / a.blocks;
    const int row0 = blockIdx.x % a.blocks * a.rows, rows = min(a.rows, a.HW - row0);
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    pdl_wait();
    pdl_launch_dependents();
    float mean[V] = {}, m2[V] = {};
    int n = 0;
    if (rl < lanes)
        for (int r = rl; r < rows; r += 4 * lanes) {
            float f[4][V];
            int k = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 y = make_uint4(0u, 0u, 0u, 0u);
                if (r + i * lanes < rows) {
                    y = *reinterpret_cast<const uint4*>(a.x + base + (long long)(r + i * lanes) * a.C);
                    k = i + 1;
                }
                widen16(y, f[i], a.x);
            }
            const float ik = 1.f / (float)k, share = (float)k / (float)(n + k), cross = share * (float)n;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float mk = (f[0][e] + f[1][e] + f[2][e] + f[3][e]) * ik;
                float q = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < k) q = fmaf(f[i][e] - mk, f[i][e] - mk, q);
                const float dm = mk - mean[e];
                m2[e] += fmaf(dm * dm, cross, q);
                mean[e] = fmaf(dm, share, mean[e]);
            }
            n += k;
        }
    float *rm = smem, *rq = smem + kThreads * V;
    if (rl < lanes)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            rm[rl * slab + vc * V + e] = mean[e];
            rq[rl * slab + vc * V + e] = m2[e];
        }
    __syncthreads();
    for (int c = tid; c < slab; c += kThreads) {
        float m = 0.f, q = 0.f;
        int cnt = 0;
        for (int l = 0; l < lanes; ++l) {
            const int k = l < rows ? (rows - l + lanes - 1) / lanes : 0;
            if (k == 0) break;
            const float dm = rm[l * slab + c] - m, share = (float)k / (float)(cnt + k);
            q += fmaf(dm * dm, share * (float)cnt, rq[l * slab + c]);
            m = fmaf(dm, share, m);
            cnt += k;
        }
        a.part[(long long)blockIdx.x * a.C + c0 + c] = make_float2(m, q);
    }
}
// Chunks' channels of an image's group joined by W threads: a warp, or a block where the entries (chunks x channels of the group) are many.  (A warp for any
// number of them, a chain of divisions: 1450 us for 1 x 56 x 56 x 768 in one group, 150000 entries.)
constexpr int kJoinWide = 1024;
constexpr long long kJoinWarp = 2048;   // entries that a warp takes
template <int W>
__device__ __forceinline__ float join_sum(float x, float* red) {   // over the W threads, in all of them
    x = warp_sum(x);
    if constexpr (W > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
        __syncthreads();
        x = warp_sum(red[threadIdx.x & 31]);
    }
    return x;
}
// f(chunk, channel of the group) for every W-th entry.
template <int W, typename F>
__device__ __forceinline__ void over_entries(int chunks, int per, F f) {
    int chunk = (threadIdx.x % W) / per, c = (threadIdx.x % W) - chunk * per;
    const int chunk_step = W / per, c_step = W - chunk_step * per;
#pragma unroll 4
    while (chunk < chunks) {
        f(chunk, c);
        chunk += chunk_step;
        c += c_step;
        if (c >= per) {
            c -= per;
            ++chunk;
        }
    }
}
// Mean first, then the squares about it.
template <typename T, int W>
__global__ void __launch_bounds__(W > 32 ? W : kThreads) norm_join_kernel(Norm<T> a, int chunks, long long total) {
    __shared__ float red[32];
    pdl_wait();
    pdl_launch_dependents();
    const long long at = W > 32 ? blockIdx.x : (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (at >= total) return;   // (whole warps; never where a block is at it)
    const int lane = threadIdx.x % W, G = a.C / a.per;
    const long long b = at / G;
    const float2* const part = a.part + b * chunks * a.C + at % G * a.per;
    auto over = [&](auto f) {   // sum of f(values of the entry, the entry)
        float x = 0.f;
        over_entries<W>(chunks, a.per, [&](int chunk, int c) { x += f((float)min(a.rows, a.HW - chunk * a.rows), part[(long long)chunk * a.C + c]); });
        return join_sum<W>(x, red);
    };
    const float n = (float)a.HW * a.per;
    const float m = over([](float k, float2 p) { return k * p.x; }) / n;
    const float q = over([m](float k, float2 p) { return fmaf(k * (p.x - m), p.x - m, p.y); });
    if (lane == 0) {
        a.mean[at] = m;
        a.rstd[at] = rsqrtf(q / n + a.eps);
    }
}
template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(Norm<T> a) {
    constexpr int V = Wide<T>::N;
    const int c0 = blockIdx.z * a.slab, slab = min(a.slab, a.C - c0);
    const int nv = slab / V, lanes = kThreads / nv, tid = threadIdx.x, vc = tid % nv, rl = tid / nv;
    const long long image = blockIdx.x / a.blocks;
    const int row0 = blockIdx.x % a.blocks * a.rows, rows = min(a.rows, a.HW - row0);
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    pdl_wait();
    pdl_launch_dependents();
    if (rl >= lanes) return;
    const long long at = image * (a.C / a.per);
    f32x2 m[V / 2], w[V / 2], b[V / 2];
    params(a.weight, c0 + vc * V, 1.f, w);
    params(a.bias, c0 + vc * V, 0.f, b);
    over_pairs<V>(c0 + vc * V, (c0 + vc * V) / a.per, a.per, [&](int e, int g0, int g1) {
        m[e] = pack2(a.mean[at + g0], a.mean[at + g1]);
        w[e] = fmul2(w[e], pack2(a.rstd[at + g0], a.rstd[at + g1]));
    });
    for (int r = rl; r < rows; r += 4 * lanes) {
        uint4 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i * lanes < rows) y[i] = *reinterpret_cast<const uint4*>(a.x + base + (long long)(r + i * lanes) * a.C);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i * lanes < rows) {
                f32x2 f[V / 2];
                widen16(y[i], f, a.x);
#pragma unroll
                for (int e = 0; e < V / 2; ++e) f[e] = act2<ACT, sizeof(T) == 2>(ffma2(fsub2(f[e], m[e]), w[e], b[e]));
                *reinterpret_cast<uint4*>(a.out + base + (long long)(r + i * lanes) * a.C) = narrow16(f, a.x);
            }
    }
}

// The gradient: sums of g and g xhat per channel and chunk (SUMS), or dx.
template <typename T, int ACT, bool SUMS>
__global__ void __launch_bounds__(kThreads) norm_grad_chunk_kernel(Norm<T> a, const float2* means) {
    constexpr int V = Wide<T>::N;
    extern __shared__ __align__(16) float smem[];
    const int c0 = blockIdx.z * a.slab, slab = min(a.slab, a.C - c0);
    const int nv = slab / V, lanes = kThreads / nv, tid = threadIdx.x, vc = tid % nv, rl = tid / nv;
    const long long image = blockIdx.x / a.blocks;
    const int row0 = blockIdx.x % a.blocks * a.rows, rows = min(a.rows, a.HW - row0);
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    pdl_wait();
    pdl_launch_dependents();
    const bool live = rl < lanes;
    const long long at = image * (a.C / a.per);
    Channels<T> ch;
    ch.load(a, at, 0, c0 + vc * V, live);
    f32x2 s1[V / 2], s2[V / 2];
#pragma unroll
    for (int e = 0; e < V / 2; ++e) s1[e] = s2[e] = both(0.f);
    if (!SUMS && live)
        over_pairs<V>(c0 + vc * V, (c0 + vc * V) / a.per, a.per, [&](int e, int g0, int g1) {
            const float2 p = means[at + g0], q = means[at + g1];
            s1[e] = pack2(p.x, q.x);
            s2[e] = pack2(p.y, q.y);
        });
    if (live)
        for (int r = rl; r < rows; r += 2 * lanes) {
            uint4 y[2], d[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (r + i * lanes < rows) {
                    y[i] = *reinterpret_cast<const uint4*>(a.x + base + (long long)(r + i * lanes) * a.C);
                    d[i] = *reinterpret_cast<const uint4*>(a.d_out + base + (long long)(r + i * lanes) * a.C);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (r + i * lanes < rows) {
                    f32x2 h[V / 2], g[V / 2];
                    ch.template grad<ACT>(y[i], d[i], h, g);
                    if constexpr (SUMS) {
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) {
                            s1[e] = fadd2(s1[e], g[e]);
                            s2[e] = ffma2(g[e], h[e], s2[e]);
                        }
                    } else {
                        ch.dx(h, g, s1, s2);
                        *reinterpret_cast<uint4*>(a.dx + base + (long long)(r + i * lanes) * a.C) = narrow16(g, a.x);
                    }
                }
        }
    if constexpr (SUMS) {
        float2* const red = reinterpret_cast<float2*>(smem);
        if (live)
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                float g0, g1, x0, x1;
                unpack2(s1[e], g0, g1);
                unpack2(s2[e], x0, x1);
                *reinterpret_cast<float4*>(red + rl * slab + vc * V + 2 * e) = make_float4(g0, x0, g1, x1);
            }
        __syncthreads();
        for (int c = tid; c < slab; c += kThreads) {
            float u = 0.f, v = 0.f;
            for (int l = 0; l < lanes; ++l) {
                const float2 y = red[l * slab + c];
                u += y.x;
                v += y.y;
            }
            a.part[(long long)blockIdx.x * a.C + c0 + c] = make_float2(u, v);
        }
    }
}
// Means of g w and g w xhat of an image's group, by W threads as above.
template <typename T, int W>
__global__ void __launch_bounds__(W > 32 ? W : kThreads) norm_grad_join_kernel(Norm<T> a, float2* means, int chunks, long long total) {
    __shared__ float red[32];
    pdl_wait();
    pdl_launch_dependents();
    const long long at = W > 32 ? blockIdx.x : (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (at >= total) return;
    const int lane = threadIdx.x % W, G = a.C / a.per;
    const long long b = at / G;
    const int c0 = (int)(at % G) * a.per;
    const float2* const part = a.part + b * chunks * a.C + c0;
    float u = 0.f, v = 0.f;
    over_entries<W>(chunks, a.per, [&](int chunk, int c) {
        const float2 p = part[(long long)chunk * a.C + c];
        const float w = one(a.weight, c0 + c, 1.f);
        u = fmaf(p.x, w, u);
        v = fmaf(p.y, w, v);
    });
    u = join_sum<W>(u, red);
    v = join_sum<W>(v, red);
    const float inv = 1.f / ((float)a.HW * a.per);
    if (lane == 0) means[at] = make_float2(u * inv, v * inv);
}
// The parameters' gradients: a channel's sums over all images and blocks.  Eight channels a block, 32 threads a channel.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_params_kernel(const float2* part, T* dweight, T* dbias, long long rows, int C) {
    __shared__ float2 red[32][8];
    pdl_wait();
    pdl_launch_dependents();
    const int c = blockIdx.x * 8 + (threadIdx.x & 7), l = threadIdx.x >> 3;
    float u = 0.f, v = 0.f;
    if (c < C)
        for (long long r = l; r < rows; r += 32) {
            const float2 p = part[r * C + c];
            u += p.x;
            v += p.y;
        }
    red[l][threadIdx.x & 7] = make_float2(u, v);
    __syncthreads();
    if (threadIdx.x < 8 && c < C) {
        u = v = 0.f;
        for (int i = 0; i < 32; ++i) {
            u += red[i][threadIdx.x].x;
            v += red[i][threadIdx.x].y;
        }
        if (dbias) put(dbias, c, u);
        if (dweight) put(dweight, c, v);
    }
}

// ---- which form, and its cut ---------------------------------------------------------------------------------------------
struct Plan {
    bool on_chip;
    int N, slab, slabs, rows, threads, K;   // on chip
    int chunks;                             // else
};

constexpr int kMostHeld = 48 * 1024, kMostVectors = 24;   // a block's shared memory: in front of the vectors; vectors of a thread, of all inputs together
constexpr size_t kMostSmem = kMostHeld + (size_t)kMostVectors * kThreads * 16;

int gcd(int a, int b) { return b == 0 ? a : gcd(b, a % b); }

Plan plan_of(int B, int HW, int C, int groups, int V, bool gradient) {
    Plan p = {};
    const int per = C / groups, base = per / gcd(per, V) * V, units = C / base, most = gradient ? kMostVectors / 2 : kMostVectors;   // 96 KB of a block's shared memory, two blocks an SM (64 KB: 35 us where this takes 31, fp32 57 and 49)
    for (int m = 1; m <= units; ++m) {
        if (units % m) continue;
        const int slab = base * m, nv = slab / V;
        if (nv > kThreads) break;
        // few images: not wider where that leaves SMs without a block (1 x 64 x 64 x 192: 6.7 us against 7.8)
        if (p.on_chip && (long long)B * (units / m) * kMostBlocks < 148) break;
        const int threads = kThreads / nv * nv, lanes = threads / nv;
        for (int N = 1; N <= kMostBlocks; N *= 2) {
            const int rows = (HW + N - 1) / N, K = (rows + lanes - 1) / lanes;
            // (no more shared memory than a block has without asking: slabs of many groups)
            if (K > most || on_chip_floats((threads + 31) / 32 * 32 / nv, slab, slab / per) * 4 > kMostHeld) continue;
            p = {true, N, slab, units / m, rows, (threads + 31) / 32 * 32, K, 0};
            break;
        }
        if (p.on_chip && slab * (16 / V) >= 64) break;   // rows of 64 bytes and more
    }
    if (p.on_chip) {
        const int lanes = kThreads / (p.slab / V);
        while (p.N < kMostBlocks && (long long)B * p.slabs * p.N < 2 * 148 && p.K > 1) {   // few blocks: smaller ones
            p.N *= 2;
            p.rows = (HW + p.N - 1) / p.N;
            p.K = (p.rows + lanes - 1) / lanes;
        }
        return p;
    }
    p.slab = (C < kThreads * V ? C : kThreads * V);
    p.slabs = (C + p.slab - 1) / p.slab;
    const int lanes = kThreads / (p.slab / V);
    long long want = (4LL * 148 + (long long)B * p.slabs - 1) / ((long long)B * p.slabs);   // chunks of an image
    const long long fewest = (HW + 32767) / 32768, finest = (HW + 8 * lanes - 1) / (8 * lanes);
    want = want > finest ? finest : want;
    want = want < fewest ? fewest : want;
    p.rows = (int)((HW + want - 1) / want);
    p.chunks = (HW + p.rows - 1) / p.rows;
    return p;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
void fill(Norm<T>& a, const Plan& p, int HW, int C, int groups, bool gradient) {
    constexpr int V = 16 / sizeof(T);
    a.HW = HW; a.C = C; a.per = C / groups; a.slab = p.slab; a.rows = p.rows;
    a.blocks = p.on_chip ? p.N * p.slabs : p.chunks;
    a.by_per = Div(a.per);
    if (!p.on_chip) return;
    const bool vectors = !gradient && a.per % V == 0;
    a.lanes = p.threads / (p.slab / V);
    a.groups = p.slab / a.per;
    a.entries = vectors ? p.slab / V : p.slab;
    a.width = vectors ? a.per / V : a.per;
    a.parts = p.threads / a.entries;
    a.parts = a.parts < 1 ? 1 : a.parts > a.lanes ? a.lanes : a.parts;
    a.by_vectors = Div(p.slab / V);
    a.by_entries = Div(a.entries);
    a.by_slab = Div(p.slab);
    a.by_lanes = Div(a.lanes);
    a.held = (int)((on_chip_floats(a.lanes, p.slab, a.groups) + 3) / 4 * 4);
}

template <typename F>
cudaError_t with_act(int act, F f) {
    if (act == kActSilu) return f(std::integral_constant<int, kActSilu>());
    if (act == kActGelu) return f(std::integral_constant<int, kActGelu>());
    return f(std::integral_constant<int, kActNone>());
}
}  // namespace

bool group_norm_supported(int B, int HW, int C, int groups, size_t elem) {
    if (C % (int)(16 / elem) != 0 || C > (1 << 20) || C % groups != 0) return false;
    for (int gradient = 0; gradient < 2; ++gradient) {
        const Plan p = plan_of(B > 0 ? B : 1, HW > 0 ? HW : 1, C, groups, (int)(16 / elem), gradient != 0);
        if ((long long)B * (p.on_chip ? p.N * p.slabs : p.chunks) > 0x7fffffffLL || p.slabs > 65535) return false;
    }
    return (long long)B * groups <= 0x7fffffffLL;
}

size_t group_norm_scratch_bytes(int B, int HW, int C, int groups, size_t elem, bool gradient) {
    const Plan p = plan_of(B, HW, C, groups, (int)(16 / elem), gradient);
    const size_t stats = up((size_t)B * groups * sizeof(float2));
    if (p.on_chip) return gradient ? up((size_t)B * p.N * C * sizeof(float2)) : 0;
    return up((size_t)B * p.chunks * C * sizeof(float2)) + stats;
}

template <typename T>
cudaError_t launch_group_norm(const T* x, const T* weight, const T* bias, T* out, float* mean, float* rstd, int B, int HW, int C, int groups,
                              float eps, int act, void* scratch, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const Plan p = plan_of(B, HW, C, groups, V, false);
    Norm<T> a = {};
    a.x = x; a.weight = weight; a.bias = bias; a.out = out; a.mean = mean; a.rstd = rstd;
    a.eps = eps;
    fill(a, p, HW, C, groups, false);
    if (p.on_chip)
        return with_act(act, [&](auto A) {
            const size_t smem = (size_t)a.held * 4 + (size_t)p.K * kThreads * 16;
            cudaError_t e = allow_smem<norm_kernel<T, decltype(A)::value>>(kMostSmem);
            if (e != cudaSuccess) return e;
            count_launch();
            return launch_pdl_cluster(norm_kernel<T, decltype(A)::value>, dim3((unsigned)((long long)a.blocks * B)), dim3(p.threads), smem, p.N, stream, a, p.N);
        });
    a.part = (float2*)scratch;
    float* stats = (float*)((char*)scratch + up((size_t)B * p.chunks * C * sizeof(float2)));
    const long long total = (long long)B * groups;
    if (!a.mean) a.mean = stats;
    if (!a.rstd) a.rstd = stats + total;
    const dim3 grid((unsigned)((long long)p.chunks * B), 1, p.slabs);
    cudaError_t e = launch_pdl(norm_stats_kernel<T>, grid, dim3(kThreads), 2 * kThreads * V * 4, stream, a);
    if (e != cudaSuccess) return e;
    e = (long long)p.chunks * a.per > kJoinWarp
            ? launch_pdl(norm_join_kernel<T, kJoinWide>, dim3((unsigned)total), dim3(kJoinWide), 0, stream, a, p.chunks, total)
            : launch_pdl(norm_join_kernel<T, 32>, dim3((unsigned)((total + 7) / 8)), dim3(kThreads), 0, stream, a, p.chunks, total);
    if (e != cudaSuccess) return e;
    count_launch(3);
    return with_act(act, [&](auto A) { return launch_pdl(norm_apply_kernel<T, decltype(A)::value>, grid, dim3(kThreads), 0, stream, a); });
}

template <typename T>
cudaError_t launch_group_norm_bwd(const T* x, const T* weight, const T* bias, const float* mean, const float* rstd, const T* d_out, T* dx, T* dweight,
                                  T* dbias, int B, int HW, int C, int groups, int act, void* scratch, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const Plan p = plan_of(B, HW, C, groups, V, true);
    Norm<T> a = {};
    a.x = x; a.weight = weight; a.bias = bias; a.d_out = d_out; a.dx = dx; a.cmean = mean; a.crstd = rstd;
    fill(a, p, HW, C, groups, true);
    a.part = (float2*)scratch;
    cudaError_t e;
    if (p.on_chip)
        e = with_act(act, [&](auto A) {
            const size_t smem = (size_t)a.held * 4 + (size_t)2 * p.K * kThreads * 16;
            cudaError_t r = allow_smem<norm_grad_kernel<T, decltype(A)::value>>(kMostSmem);
            if (r != cudaSuccess) return r;
            count_launch();
            return launch_pdl_cluster(norm_grad_kernel<T, decltype(A)::value>, dim3((unsigned)((long long)a.blocks * B)), dim3(p.threads), smem, p.N, stream, a, p.N, p.K);
        });
    else {
        float2* means = (float2*)((char*)scratch + up((size_t)B * p.chunks * C * sizeof(float2)));
        const long long total = (long long)B * groups;
        const dim3 grid((unsigned)((long long)p.chunks * B), 1, p.slabs);
        e = with_act(act, [&](auto A) {
            constexpr int kAct = decltype(A)::value;
            cudaError_t r = launch_pdl(norm_grad_chunk_kernel<T, kAct, true>, grid, dim3(kThreads), 2 * kThreads * V * 4, stream, a, nullptr);
            if (r == cudaSuccess)
                r = (long long)p.chunks * a.per > kJoinWarp
                        ? launch_pdl(norm_grad_join_kernel<T, kJoinWide>, dim3((unsigned)total), dim3(kJoinWide), 0, stream, a, means, p.chunks, total)
                        : launch_pdl(norm_grad_join_kernel<T, 32>, dim3((unsigned)((total + 7) / 8)), dim3(kThreads), 0, stream, a, means, p.chunks, total);
            if (r == cudaSuccess) r = launch_pdl(norm_grad_chunk_kernel<T, kAct, false>, grid, dim3(kThreads), 0, stream, a, means);
            count_launch(3);
            return r;
        });
    }
    if (e != cudaSuccess || (!dweight && !dbias)) return e;
    count_launch();
    return launch_pdl(norm_params_kernel<T>, dim3((C + 7) / 8), dim3(kThreads), 0, stream, a.part, dweight, dbias,
                      (long long)B * (p.on_chip ? p.N : p.chunks), C);
}

#define VIG_NORM(T)                                                                                                                               \
    template cudaError_t launch_group_norm<T>(const T*, const T*, const T*, T*, float*, float*, int, int, int, int, float, int, void*, cudaStream_t); \
    template cudaError_t launch_group_norm_bwd<T>(const T*, const T*, const T*, const float*, const float*, const T*, T*, T*, T*, int, int, int, int, \
                                                  int, void*, cudaStream_t);
VIG_NORM(float)
VIG_NORM(__nv_bfloat16)

}  // namespace vig
