// Pieces that the selective scan's kernels share.
//
// A block owns 64 channels of a group, a warp eight of them: lanes l, l + 8, l + 16, l + 24 hold a quarter each of the states of channel
// l < 8 (NS of them, as pairs of fp32).  Sums over the states cross these four lanes only, for four tokens together.  Element-wise work
// (step sizes, gates) is done once for every token and channel: thread i takes channels 4 (i % 16) .. + 3 of token i / 16 of a
// tile of 16 tokens, and hands over through shared memory.
#pragma once
#include "ssm.h"
#include "wide.cuh"

namespace vig {
namespace ssm {

constexpr int kThreads = 256, kTile = kSsmTile, kCh = kSsmChannels;
constexpr int kRow = kCh + 8;   // floats of a row of sums: the four tokens that a warp writes at a time lie in different banks

// Four neighbouring values.
__device__ __forceinline__ uint4 load4(const float* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint2 load4(const __nv_bfloat16* p) { return *reinterpret_cast<const uint2*>(p); }
__device__ __forceinline__ void widen4(const uint4& r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void widen4(const uint2& r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x << 16); f[1] = __uint_as_float(r.x & 0xffff0000u);
    f[2] = __uint_as_float(r.y << 16); f[3] = __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&f)[4]) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&f)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
}
template <typename T>
struct Four;
template <>
struct Four<float> { typedef uint4 Raw; };
template <>
struct Four<__nv_bfloat16> { typedef uint2 Raw; };

// e^-|v| and with it max(v, 0) + log(1 + e^-|v|) and 1 / (1 + e^-v).  The logarithm is 2 atanh(u / (2 + u)) by the series of atanh, whose
// argument is at most 1/3: its eighth term is below 2^-26 of the sum.
template <typename T>
__device__ __forceinline__ float exp_minus_abs(float v) { return sizeof(T) == 2 ? ex2(-kLog2E * fabsf(v)) : expf(-fabsf(v)); }
__device__ __forceinline__ float softplus_of(float v, float u) {
    const float s = u * reciprocal(2.f + u), q = s * s;
    float p = fmaf(q, 1.f / 13, 1.f / 11);
    p = fmaf(q, p, 1.f / 9);
    p = fmaf(q, p, 1.f / 7);
    p = fmaf(q, p, 1.f / 5);
    p = fmaf(q, p, 1.f / 3);
    p = fmaf(q, p, 1.f);
    return fmaf(s + s, p, fmaxf(v, 0.f));
}
template <typename T>
__device__ __forceinline__ float sigmoid_of(float v, float u) {
    const float r = sizeof(T) == 2 ? reciprocal(1.f + u) : 1.f / (1.f + u);
    return v >= 0.f ? r : u * r;
}

// What a block works on: sequence, segment, channels of a group.
struct Place {
    int b, seg, group, c0, live;   // live: channels of the block that exist (a multiple of four)
    template <typename T>
    __device__ __forceinline__ Place(const Ssm<T>& a, long long item) {
        const int cb = (int)(item % a.blocks);
        item /= a.blocks;
        group = (int)(item % a.G);
        item /= a.G;
        seg = (int)(item % a.segs);
        b = (int)(item / a.segs);
        c0 = group * a.per + cb * kCh;
        live = min(kCh, a.per - cb * kCh);
    }
};

// NS / 2 pairs of a lane's states of channel c; zero behind the last state.
template <int NS>
__device__ __forceinline__ void load_states(const float* p, int N, int n0, f32x2 (&h)[NS / 2]) {
#pragma unroll
    for (int i = 0; i < NS / 2; ++i) h[i] = pack2(n0 + 2 * i < N ? p[n0 + 2 * i] : 0.f, n0 + 2 * i + 1 < N ? p[n0 + 2 * i + 1] : 0.f);
}
template <int NS>
__device__ __forceinline__ void store_states(float* p, int N, int n0, const f32x2 (&h)[NS / 2]) {
#pragma unroll
    for (int i = 0; i < NS / 2; ++i) {
        float lo, hi;
        unpack2(h[i], lo, hi);
        if (n0 + 2 * i < N) p[n0 + 2 * i] = lo;
        if (n0 + 2 * i + 1 < N) p[n0 + 2 * i + 1] = hi;
    }
}
template <int NP>
__device__ __forceinline__ f32x2 lds2(const float* p) { return *reinterpret_cast<const f32x2*>(p); }
// NS floats (pairs) at 8- or 16-byte alignment.
template <int NS>
__device__ __forceinline__ void load_pairs(const float* p, f32x2 (&v)[NS / 2]) {
    if constexpr (NS == 2) {
        v[0] = *reinterpret_cast<const f32x2*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < NS / 4; ++i) {
            const ulonglong2 u = *reinterpret_cast<const ulonglong2*>(p + 4 * i);
            v[2 * i] = u.x;
            v[2 * i + 1] = u.y;
        }
    }
}
template <int NS>
__device__ __forceinline__ void store_pairs(float* p, const f32x2 (&v)[NS / 2]) {
    if constexpr (NS == 2) {
        *reinterpret_cast<f32x2*>(p) = v[0];
    } else {
#pragma unroll
        for (int i = 0; i < NS / 4; ++i) {
            ulonglong2 u;
            u.x = v[2 * i];
            u.y = v[2 * i + 1];
            *reinterpret_cast<ulonglong2*>(p + 4 * i) = u;
        }
    }
}
__device__ __forceinline__ f32x2 exp2_pair(f32x2 v) {
    float lo, hi;
    unpack2(v, lo, hi);
    return pack2(ex2(lo), ex2(hi));
}
// Sums over the four lanes of a channel of what they hold for four tokens: lane quarter q ends with token q's.
__device__ __forceinline__ float over_quarters(float p0, float p1, float p2, float p3, int quarter) {
    const bool hi = quarter & 2, lo = quarter & 1;
    float k0 = hi ? p2 : p0, k1 = hi ? p3 : p1;
    k0 += __shfl_xor_sync(0xffffffffu, hi ? p0 : p2, 16);
    k1 += __shfl_xor_sync(0xffffffffu, hi ? p1 : p3, 16);
    return (lo ? k1 : k0) + __shfl_xor_sync(0xffffffffu, lo ? k0 : k1, 8);
}

// A tile's rows of Bt and Ct, loaded a tile ahead by all threads of a block: E values of either a thread.
template <typename T, int NP>
struct Rows {
    static constexpr int E = (kTile * NP + kThreads - 1) / kThreads;
    T v[E];
    __device__ __forceinline__ void load(const T* p, const Ssm<T>& a, long long ld, const Place& at, int t0) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = threadIdx.x + e * kThreads, t = t0 + i / NP, n = i % NP;
            from_f32(&v[e], 0.f);
            if (i < kTile * NP && t < a.L && n < a.N) v[e] = p[a.row(at.b, t) * ld + at.group * a.N + n];
        }
    }
    __device__ __forceinline__ void put(float* to) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = threadIdx.x + e * kThreads;
            if (i < kTile * NP) to[i] = to_f32(v[e]);
        }
    }
};

}  // namespace ssm
}  // namespace vig
