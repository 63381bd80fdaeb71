// Group norm with an activation over channels-last images [B, HW, C], forward and gradient.
//
//   xhat = (x - mean) rstd over the HW x C/G values of an image's group;  z = xhat weight + bias;  out = act(z)
//   g = d_out act'(z);  dbias_c = sum g;  dweight_c = sum g xhat;  dx = rstd (g w - mean(g w) - xhat mean(g w xhat))
//
// Memory bounds all of it, so an image's groups stay on chip between the statistics and their use wherever they fit: a cluster of up to
// eight blocks holds all rows of a slab of whole groups in registers (16-byte vectors, a thread's vectors all of the same channels), sums
// are exchanged through distributed shared memory, and every value crosses memory once in and once out.  Larger images go through
// it twice, in launches of their own.  Variances are sums of squares about a mean that is known: a block's own first, moved to the
// image's when blocks are joined, so that a mean far from zero costs no digits.  All sums run in a fixed order.
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
__device__ __forceinline__ uint4 narrow16(const float (&f)[4], const float*) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 narrow16(const float (&f)[8], const __nv_bfloat16*) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ float one(const float* p, long long i, float none) { return p ? p[i] : none; }
__device__ __forceinline__ float one(const __nv_bfloat16* p, long long i, float none) { return p ? __bfloat162float(p[i]) : none; }
__device__ __forceinline__ void put(float* p, long long i, float x) { p[i] = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, long long i, float x) { p[i] = __float2bfloat16_rn(x); }

// FAST (results rounded to bf16): e^-z and the quotient from the special-function unit, relative error below 1e-6.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z) {
    if constexpr (FAST) return __fdividef(1.f, 1.f + ex2(-z * 1.4426950408889634f));   // (1 + inf: 0, as __fdividef has it from 2^126 on)
    else return 1.f / (1.f + expf(-z));
}
template <int ACT, bool FAST>
__device__ __forceinline__ float act(float z) {
    if constexpr (ACT == kActSilu) return z * sigmoid<FAST>(z);
    else if constexpr (ACT == kActGelu) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    else return z;
}
template <int ACT, bool FAST>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == kActSilu) {
        const float s = sigmoid<FAST>(z);
        return s * fmaf(z, 1.f - s, 1.f);
    } else if constexpr (ACT == kActGelu) {
        const float phi = 0.3989422804014327f * (FAST ? ex2(-0.7213475204444817f * z * z) : expf(-0.5f * z * z));
        return fmaf(z, phi, 0.5f * erfcf(-0.70710678118654752f * z));
    } else return 1.f;
}

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
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ float peer_f32(const float* p, uint32_t rank) {   // this variable of another block of the cluster
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(cluster_peer(smem_u32(p), rank)) : "memory");
    return x;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_await() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Shared memory of the forms that stay on chip: a partial sum per thread and channel ([row lane][channel of the slab]), what a group
// comes to in the block, and what it comes to over the cluster.
struct Shared {
    float *red, *own, *all;
    __device__ Shared(float* base, int lanes, int slab, int groups) {
        red = base;
        own = base + lanes * slab;
        all = own + 2 * groups;
    }
};
constexpr size_t on_chip_smem(int lanes, int slab, int groups) { return ((size_t)lanes * slab + 4 * groups) * 4; }

// Sums of the group over what all threads hold, a warp per group.
template <typename F>
__device__ __forceinline__ void over_groups(const float* red, int lanes, int slab, int per, int groups, F f) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int g = warp; g < groups; g += warps) {
        float s = 0.f;
        for (int i = lane; i < lanes * per; i += 32) s += red[(i / per) * slab + g * per + i % per];
        f(g, warp_sum(s));
    }
}

// ---- on chip: grid (blocks of a cluster x slabs x B); K vectors of 16 bytes a thread --------------------------------------
template <typename T, int ACT, int K>
__global__ void __launch_bounds__(kThreads) norm_kernel(Norm<T> a, int N) {
    constexpr int V = Wide<T>::N;
    extern __shared__ __align__(16) float smem[];
    const int nv = a.slab / V, lanes = blockDim.x / nv, tid = threadIdx.x, vc = tid % nv, rl = tid / nv;
    const int groups = a.slab / a.per;
    const Shared s(smem, lanes, a.slab, groups);
    const long long image = blockIdx.x / a.blocks;
    const int slab = blockIdx.x % a.blocks / N, rank = blockIdx.x % N;
    const int c0 = slab * a.slab, row0 = rank * a.rows, rows = min(a.rows, a.HW - row0);   // (may be none)
    const bool live = rl < lanes;
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    pdl_wait();
    pdl_launch_dependents();
    uint4 x[K];
    int n = 0;   // vectors of this thread
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int r = rl + i * lanes;
        if (live && r < rows) {
            x[i] = *reinterpret_cast<const uint4*>(a.x + base + (long long)r * a.C);
            n = i + 1;
        }
    }
    float acc[V] = {};
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < n) {
            float f[V];
            widen16(x[i], f, a.x);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += f[e];
        }
    if (live)
#pragma unroll
        for (int e = 0; e < V; ++e) s.red[rl * a.slab + vc * V + e] = acc[e];
    __syncthreads();
    const float mine = rows > 0 ? 1.f / ((float)rows * a.per) : 0.f;
    over_groups(s.red, lanes, a.slab, a.per, groups, [&](int g, float sum) {
        if ((tid & 31) == 0) s.own[2 * g] = sum * mine;
    });
    __syncthreads();
    int g[V];
    float m[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        g[e] = (vc * V + e) / a.per;
        m[e] = s.own[2 * g[e]];
        acc[e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < n) {
            float f[V];
            widen16(x[i], f, a.x);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = fmaf(f[e] - m[e], f[e] - m[e], acc[e]);
        }
    if (live)
#pragma unroll
        for (int e = 0; e < V; ++e) s.red[rl * a.slab + vc * V + e] = acc[e];
    __syncthreads();
    over_groups(s.red, lanes, a.slab, a.per, groups, [&](int g_, float sum) {
        if ((tid & 31) == 0) s.own[2 * g_ + 1] = sum;
    });
    if (N > 1) {
        cluster_arrive();
        cluster_await();
    } else __syncthreads();
    for (int j = tid; j < groups; j += blockDim.x) {
        float mean = s.own[2 * j], m2 = s.own[2 * j + 1];
        if (N > 1) {
            // blocks' means and sums of squares about them, joined: mean over rows, and every block's sum moved to it
            float bm[kMostBlocks], bs[kMostBlocks];
            mean = m2 = 0.f;
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) {
                    bm[p] = peer_f32(s.own + 2 * j, p);
                    bs[p] = peer_f32(s.own + 2 * j + 1, p);
                }
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) mean += bm[p] * ((float)max(0, min(a.rows, a.HW - p * a.rows)) / (float)a.HW);
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) m2 += bs[p] + (float)max(0, min(a.rows, a.HW - p * a.rows)) * a.per * (bm[p] - mean) * (bm[p] - mean);
        }
        const float rstd = rsqrtf(m2 / ((float)a.HW * a.per) + a.eps);
        s.all[2 * j] = mean;
        s.all[2 * j + 1] = rstd;
        if (rank == 0) {
            const long long at = image * (a.C / a.per) + c0 / a.per + j;
            if (a.mean) a.mean[at] = mean;
            if (a.rstd) a.rstd[at] = rstd;
        }
    }
    if (N > 1) cluster_arrive();   // has read the others' shared memory, which they keep until all have
    __syncthreads();
    float w[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = c0 + vc * V + e;
        m[e] = live ? s.all[2 * g[e]] : 0.f;
        w[e] = live ? one(a.weight, c, 1.f) * s.all[2 * g[e] + 1] : 0.f;
        b[e] = live ? one(a.bias, c, 0.f) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < n) {
            float f[V];
            widen16(x[i], f, a.x);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = act<ACT, sizeof(T) == 2>(fmaf(f[e] - m[e], w[e], b[e]));
            *reinterpret_cast<uint4*>(a.out + base + (long long)(rl + i * lanes) * a.C) = narrow16(f, a.x);
        }
    if (N > 1) cluster_await();
}

template <typename T, int ACT, int K>
__global__ void __launch_bounds__(kThreads) norm_grad_kernel(Norm<T> a, int N) {
    constexpr int V = Wide<T>::N;
    constexpr bool FAST = sizeof(T) == 2;
    extern __shared__ __align__(16) float smem[];
    const int nv = a.slab / V, lanes = blockDim.x / nv, tid = threadIdx.x, vc = tid % nv, rl = tid / nv;
    const int groups = a.slab / a.per;
    const Shared s(smem, lanes, a.slab, groups);
    float* const red2 = s.all + 2 * groups;   // [lanes][slab]
    const long long image = blockIdx.x / a.blocks;
    const int slab = blockIdx.x % a.blocks / N, rank = blockIdx.x % N;
    const int c0 = slab * a.slab, row0 = rank * a.rows, rows = min(a.rows, a.HW - row0);
    const bool live = rl < lanes;
    const long long base = (image * a.HW + row0) * a.C + c0 + vc * V;
    pdl_wait();
    pdl_launch_dependents();
    uint4 x[K], d[K];
    int n = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int r = rl + i * lanes;
        if (live && r < rows) {
            x[i] = *reinterpret_cast<const uint4*>(a.x + base + (long long)r * a.C);
            d[i] = *reinterpret_cast<const uint4*>(a.d_out + base + (long long)r * a.C);
            n = i + 1;
        }
    }
    float m[V], rs[V], w[V], b[V], sg[V] = {}, sx[V] = {};
    const long long at = image * (a.C / a.per) + c0 / a.per;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = vc * V + e;
        m[e] = live ? a.cmean[at + c / a.per] : 0.f;
        rs[e] = live ? a.crstd[at + c / a.per] : 0.f;
        w[e] = live ? one(a.weight, c0 + c, 1.f) : 0.f;
        b[e] = live ? one(a.bias, c0 + c, 0.f) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < n) {
            float f[V], o[V];
            widen16(x[i], f, a.x);
            widen16(d[i], o, a.x);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = (f[e] - m[e]) * rs[e], g = o[e] * slope<ACT, FAST>(fmaf(h, w[e], b[e]));
                sg[e] += g;
                sx[e] = fmaf(g, h, sx[e]);
            }
        }
    if (live)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s.red[rl * a.slab + vc * V + e] = sg[e];
            red2[rl * a.slab + vc * V + e] = sx[e];
        }
    __syncthreads();
    // a channel's sums over the block: what the parameters' gradients and the group's means are made of
    for (int c = tid; c < a.slab; c += blockDim.x) {
        float u = 0.f, v = 0.f;
        for (int l = 0; l < lanes; ++l) {
            u += s.red[l * a.slab + c];
            v += red2[l * a.slab + c];
        }
        a.part[(image * N + rank) * a.C + c0 + c] = make_float2(u, v);
        const float wc = one(a.weight, c0 + c, 1.f);
        s.red[c] = u * wc;    // row lane 0 of this very channel: read above by this thread alone
        red2[c] = v * wc;
    }
    __syncthreads();
    over_groups(s.red, 1, a.slab, a.per, groups, [&](int g, float sum) {
        if ((tid & 31) == 0) s.own[2 * g] = sum;
    });
    over_groups(red2, 1, a.slab, a.per, groups, [&](int g, float sum) {
        if ((tid & 31) == 0) s.own[2 * g + 1] = sum;
    });
    if (N > 1) {
        cluster_arrive();
        cluster_await();
    } else __syncthreads();
    const float inv = 1.f / ((float)a.HW * a.per);
    for (int j = tid; j < 2 * groups; j += blockDim.x) {
        float sum = 0.f;
        if (N > 1) {
#pragma unroll
            for (int p = 0; p < kMostBlocks; ++p)
                if (p < N) sum += peer_f32(s.own + j, p);
        } else sum = s.own[j];
        s.all[j] = sum * inv;
    }
    if (N > 1) cluster_arrive();
    __syncthreads();
    float m1[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int g = (vc * V + e) / a.per;
        m1[e] = live ? s.all[2 * g] : 0.f;
        m2[e] = live ? s.all[2 * g + 1] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < n) {
            float f[V], o[V];
            widen16(x[i], f, a.x);
            widen16(d[i], o, a.x);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = (f[e] - m[e]) * rs[e], g = o[e] * slope<ACT, FAST>(fmaf(h, w[e], b[e]));
                f[e] = rs[e] * (fmaf(g, w[e], -m1[e]) - h * m2[e]);
            }
            *reinterpret_cast<uint4*>(a.dx + base + (long long)(rl + i * lanes) * a.C) = narrow16(f, a.x);
        }
    if (N > 1) cluster_await();
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
// A warp per image and group: joins the chunks' channels.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_join_kernel(Norm<T> a, int chunks, long long total) {
    pdl_wait();
    pdl_launch_dependents();
    const long long at = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (at >= total) return;
    const int lane = threadIdx.x & 31, G = a.C / a.per;
    const long long b = at / G;
    const int c0 = (int)(at % G) * a.per;
    float n = 0.f, m = 0.f, q = 0.f;
    for (long long i = lane; i < (long long)chunks * a.per; i += 32) {
        const int chunk = (int)(i / a.per);
        const float2 p = a.part[(b * chunks + chunk) * a.C + c0 + i % a.per];
        const float k = (float)min(a.rows, a.HW - chunk * a.rows), dm = p.x - m, share = k / (n + k);
        q += fmaf(dm * dm, share * n, p.y);
        m = fmaf(dm, share, m);
        n += k;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float n2 = __shfl_xor_sync(0xffffffffu, n, o), m2 = __shfl_xor_sync(0xffffffffu, m, o), q2 = __shfl_xor_sync(0xffffffffu, q, o);
        const float sum = n + n2, share = sum > 0.f ? n2 / sum : 0.f, dm = m2 - m;
        q = q + q2 + dm * dm * (share * n);
        m = fmaf(dm, share, m);
        n = sum;
    }
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
    float m[V], w[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = c0 + vc * V + e;
        m[e] = a.mean[at + c / a.per];
        w[e] = one(a.weight, c, 1.f) * a.rstd[at + c / a.per];
        b[e] = one(a.bias, c, 0.f);
    }
    for (int r = rl; r < rows; r += 4 * lanes) {
        uint4 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i * lanes < rows) y[i] = *reinterpret_cast<const uint4*>(a.x + base + (long long)(r + i * lanes) * a.C);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i * lanes < rows) {
                float f[V];
                widen16(y[i], f, a.x);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = act<ACT, sizeof(T) == 2>(fmaf(f[e] - m[e], w[e], b[e]));
                *reinterpret_cast<uint4*>(a.out + base + (long long)(r + i * lanes) * a.C) = narrow16(f, a.x);
            }
    }
}

// The gradient: sums of g and g xhat per channel and chunk (SUMS), or dx.
template <typename T, int ACT, bool SUMS>
__global__ void __launch_bounds__(kThreads) norm_grad_chunk_kernel(Norm<T> a, const float2* means) {
    constexpr int V = Wide<T>::N;
    constexpr bool FAST = sizeof(T) == 2;
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
    float m[V], rs[V], w[V], b[V], s1[V], s2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = c0 + vc * V + e;
        m[e] = live ? a.cmean[at + c / a.per] : 0.f;
        rs[e] = live ? a.crstd[at + c / a.per] : 0.f;
        w[e] = live ? one(a.weight, c, 1.f) : 0.f;
        b[e] = live ? one(a.bias, c, 0.f) : 0.f;
        const float2 mm = !SUMS && live ? means[at + c / a.per] : make_float2(0.f, 0.f);
        s1[e] = mm.x;
        s2[e] = mm.y;
    }
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
                    float f[V], o[V];
                    widen16(y[i], f, a.x);
                    widen16(d[i], o, a.x);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float h = (f[e] - m[e]) * rs[e], g = o[e] * slope<ACT, FAST>(fmaf(h, w[e], b[e]));
                        if constexpr (SUMS) {
                            s1[e] += g;
                            s2[e] = fmaf(g, h, s2[e]);
                        } else f[e] = rs[e] * (fmaf(g, w[e], -s1[e]) - h * s2[e]);
                    }
                    if constexpr (!SUMS) *reinterpret_cast<uint4*>(a.dx + base + (long long)(r + i * lanes) * a.C) = narrow16(f, a.x);
                }
        }
    if constexpr (SUMS) {
        float *r1 = smem, *r2 = smem + kThreads * V;
        if (live)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                r1[rl * slab + vc * V + e] = s1[e];
                r2[rl * slab + vc * V + e] = s2[e];
            }
        __syncthreads();
        for (int c = tid; c < slab; c += kThreads) {
            float u = 0.f, v = 0.f;
            for (int l = 0; l < lanes; ++l) {
                u += r1[l * slab + c];
                v += r2[l * slab + c];
            }
            a.part[(long long)blockIdx.x * a.C + c0 + c] = make_float2(u, v);
        }
    }
}
// A warp per image and group: means of g w and g w xhat.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_grad_join_kernel(Norm<T> a, float2* means, int chunks, long long total) {
    pdl_wait();
    pdl_launch_dependents();
    const long long at = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (at >= total) return;
    const int lane = threadIdx.x & 31, G = a.C / a.per;
    const long long b = at / G;
    const int c0 = (int)(at % G) * a.per;
    float u = 0.f, v = 0.f;
    for (long long i = lane; i < (long long)chunks * a.per; i += 32) {
        const int c = c0 + (int)(i % a.per);
        const float2 p = a.part[(b * chunks + i / a.per) * a.C + c];
        const float w = one(a.weight, c, 1.f);
        u = fmaf(p.x, w, u);
        v = fmaf(p.y, w, v);
    }
    u = warp_sum(u);
    v = warp_sum(v);
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

int gcd(int a, int b) { return b == 0 ? a : gcd(b, a % b); }

Plan plan_of(int B, int HW, int C, int groups, int V, bool gradient) {
    Plan p = {};
    const int per = C / groups, base = per / gcd(per, V) * V, units = C / base, most = gradient ? 8 : 16;
    for (int m = 1; m <= units; ++m) {
        if (units % m) continue;
        const int slab = base * m, nv = slab / V;
        if (nv > kThreads) break;
        const int threads = kThreads / nv * nv, lanes = threads / nv;
        for (int N = 1; N <= kMostBlocks; N *= 2) {
            const int rows = (HW + N - 1) / N, K = (rows + lanes - 1) / lanes;
            if (K > most) continue;
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

template <typename F>
cudaError_t with_act(int act, F f) {
    if (act == kActSilu) return f(std::integral_constant<int, kActSilu>());
    if (act == kActGelu) return f(std::integral_constant<int, kActGelu>());
    return f(std::integral_constant<int, kActNone>());
}
template <typename F>
cudaError_t with_vectors(int K, F f) {
    if (K <= 1) return f(std::integral_constant<int, 1>());
    if (K <= 2) return f(std::integral_constant<int, 2>());
    if (K <= 4) return f(std::integral_constant<int, 4>());
    if (K <= 8) return f(std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 16>());
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
    a.HW = HW; a.C = C; a.per = C / groups; a.eps = eps; a.slab = p.slab; a.rows = p.rows; a.blocks = p.on_chip ? p.N * p.slabs : p.chunks;
    if (p.on_chip)
        return with_act(act, [&](auto A) {
            return with_vectors(p.K, [&](auto K) {
                count_launch();
                return launch_pdl_cluster(norm_kernel<T, decltype(A)::value, decltype(K)::value>, dim3((unsigned)((long long)a.blocks * B)), dim3(p.threads),
                                          on_chip_smem(p.threads / (p.slab / V), p.slab, p.slab / a.per), p.N, stream, a, p.N);
            });
        });
    a.part = (float2*)scratch;
    float* stats = (float*)((char*)scratch + up((size_t)B * p.chunks * C * sizeof(float2)));
    const long long total = (long long)B * groups;
    if (!a.mean) a.mean = stats;
    if (!a.rstd) a.rstd = stats + total;
    const dim3 grid((unsigned)((long long)p.chunks * B), 1, p.slabs);
    cudaError_t e = launch_pdl(norm_stats_kernel<T>, grid, dim3(kThreads), 2 * kThreads * V * 4, stream, a);
    if (e != cudaSuccess) return e;
    e = launch_pdl(norm_join_kernel<T>, dim3((unsigned)((total + 7) / 8)), dim3(kThreads), 0, stream, a, p.chunks, total);
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
    a.HW = HW; a.C = C; a.per = C / groups; a.slab = p.slab; a.rows = p.rows; a.blocks = p.on_chip ? p.N * p.slabs : p.chunks;
    a.part = (float2*)scratch;
    cudaError_t e;
    if (p.on_chip)
        e = with_act(act, [&](auto A) {
            return with_vectors(p.K, [&](auto K) -> cudaError_t {
                constexpr int k = decltype(K)::value;
                if constexpr (k > 8) return cudaErrorInvalidValue;   // (plans of the gradient stop at eight)
                else {
                    const int lanes = p.threads / (p.slab / V);
                    count_launch();
                    return launch_pdl_cluster(norm_grad_kernel<T, decltype(A)::value, k>, dim3((unsigned)((long long)a.blocks * B)), dim3(p.threads),
                                              on_chip_smem(lanes, p.slab, p.slab / a.per) + (size_t)lanes * p.slab * 4, p.N, stream, a, p.N);
                }
            });
        });
    else {
        float2* means = (float2*)((char*)scratch + up((size_t)B * p.chunks * C * sizeof(float2)));
        const long long total = (long long)B * groups;
        const dim3 grid((unsigned)((long long)p.chunks * B), 1, p.slabs);
        e = with_act(act, [&](auto A) {
            constexpr int kAct = decltype(A)::value;
            cudaError_t r = launch_pdl(norm_grad_chunk_kernel<T, kAct, true>, grid, dim3(kThreads), 2 * kThreads * V * 4, stream, a, nullptr);
            if (r == cudaSuccess)
                r = launch_pdl(norm_grad_join_kernel<T>, dim3((unsigned)((total + 7) / 8)), dim3(kThreads), 0, stream, a, means, p.chunks, total);
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
