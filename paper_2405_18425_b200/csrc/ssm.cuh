// Pieces that the selective scan's kernels share.
//
// A block owns 64 channels of a group.  Lanes l, l + 8, l + 16, l + 24 of a warp hold a quarter each of the states of K neighbouring channels,
// (l mod 8) K of the warp's 8 K, as pairs of fp32.  What a token's products take comes from shared memory, and that is where the SM's 128
// bytes a clock into registers count, broadcast or not: rows of Bt and Ct are read once for K channels, step sizes once for a quarter
// of the states, 32 / K + 8 values a token and channel (K = 1 was bound by it: 126 us for 64 x 196 x 1152 with 16 states).
// Element-wise work (step sizes, gates) is done once for every token and channel: thread i takes channels 4 (i % 16) .. + 3 of token
// i / 16 of a tile, and hands over through shared memory, as do the quarters their parts of sums over the states.
#pragma once
#include "ssm.h"
#include "wide.cuh"

namespace vig {
namespace ssm {

constexpr int kCh = kSsmChannels;
constexpr int kRow = kCh + 8;   // floats of a quarter's row of sums: the four that a warp writes at a time lie in different banks
__host__ __device__ constexpr int threads_of(int K) { return 4 * kCh / K; }
__host__ __device__ constexpr int tile_of(int K) { return 16 / K; }   // tokens of a tile: four values a thread

// Four neighbouring values.
__device__ __forceinline__ uint4 load4(const float* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint2 load4(const __nv_bfloat16* p) { return *reinterpret_cast<const uint2*>(p); }
template <typename T>
struct Four;
template <>
struct Four<float> { typedef uint4 Raw; };
template <>
struct Four<__nv_bfloat16> { typedef uint2 Raw; };

__device__ __forceinline__ void widen4(const uint4& r, f32x2 (&f)[2]) {
    f[0] = pack2(__uint_as_float(r.x), __uint_as_float(r.y));
    f[1] = pack2(__uint_as_float(r.z), __uint_as_float(r.w));
}
__device__ __forceinline__ void widen4(const uint2& r, f32x2 (&f)[2]) {
    f[0] = pack2(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u));
    f[1] = pack2(__uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, const f32x2 (&f)[2]) {
    ulonglong2 u;
    u.x = f[0];
    u.y = f[1];
    *reinterpret_cast<ulonglong2*>(p) = u;
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const f32x2 (&f)[2]) {
    float a, b, c, d;
    unpack2(f[0], a, b);
    unpack2(f[1], c, d);
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}
__device__ __forceinline__ f32x2 both(float x) { return pack2(x, x); }
__device__ __forceinline__ f32x2 neg_add2(f32x2 a, f32x2 b) { return ffma2(a, both(-1.f), b); }   // b - a

// e^-|v|, both of a pair.
template <typename T>
__device__ __forceinline__ f32x2 exp_minus_abs(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    if constexpr (sizeof(T) == 2) return pack2(ex2(-kLog2E * fabsf(a)), ex2(-kLog2E * fabsf(b)));
    else return pack2(expf(-fabsf(a)), expf(-fabsf(b)));
}
// max(v, 0) + log(1 + u) with u = e^-|v|.  log(1 + u) / u on [0, 1]: polynomial of least largest relative error among those that are one at zero,
// so that small steps keep their digits, 2^-24.8 (a fit of weighted least squares, the weights raised where the error was large until it was level;
// a coefficient rounded to fp32 and the higher ones fitted anew).
__device__ __forceinline__ f32x2 softplus2(f32x2 v, f32x2 u) {
    f32x2 p = ffma2(u, both(0.005365422461181879f), both(-0.030068300664424896f));
    p = ffma2(u, p, both(0.07920882850885391f));
    p = ffma2(u, p, both(-0.13754187524318695f));
    p = ffma2(u, p, both(0.1915384829044342f));
    p = ffma2(u, p, both(-0.24857217073440552f));
    p = ffma2(u, p, both(0.33321329951286316f));
    p = ffma2(u, p, both(-0.49999648332595825f));
    p = ffma2(u, p, both(1.f));
    float a, b;
    unpack2(v, a, b);
    return ffma2(u, p, pack2(fmaxf(a, 0.f), fmaxf(b, 0.f)));
}
// 1 / (1 + e^-v) with u = e^-|v|
template <typename T>
__device__ __forceinline__ f32x2 sigmoid2(f32x2 v, f32x2 u) {
    float a, b, x, y;
    unpack2(fadd2(u, both(1.f)), x, y);
    const f32x2 r = sizeof(T) == 2 ? pack2(reciprocal(x), reciprocal(y)) : pack2(1.f / x, 1.f / y);
    unpack2(v, a, b);
    unpack2(u, x, y);
    return fmul2(r, pack2(a >= 0.f ? 1.f : x, b >= 0.f ? 1.f : y));
}
// The same by itself: e^-v may overflow, the reciprocal is zero then.
template <typename T>
__device__ __forceinline__ f32x2 sigmoid2(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    if constexpr (sizeof(T) == 2) return pack2(sigmoid(a), sigmoid(b));
    else return pack2(1.f / (1.f + expf(-a)), 1.f / (1.f + expf(-b)));
}
template <typename T>
__device__ __forceinline__ float softplus_of(float v) {
    float a, b;
    const f32x2 w = both(v);
    unpack2(softplus2(w, exp_minus_abs<T>(w)), a, b);
    return a;
}
template <typename T>
__device__ __forceinline__ float sigmoid_of(float v) { return sizeof(T) == 2 ? sigmoid(v) : 1.f / (1.f + expf(-v)); }

template <int M>
__device__ __forceinline__ void load_floats(const float* p, float (&v)[M]) {
    if constexpr (M == 1) {
        v[0] = *p;
    } else if constexpr (M == 2) {
        const float2 u = *reinterpret_cast<const float2*>(p);
        v[0] = u.x; v[1] = u.y;
    } else {
#pragma unroll
        for (int i = 0; i < M / 4; ++i) {
            const float4 u = *reinterpret_cast<const float4*>(p + 4 * i);
            v[4 * i] = u.x; v[4 * i + 1] = u.y; v[4 * i + 2] = u.z; v[4 * i + 3] = u.w;
        }
    }
}
template <int M>
__device__ __forceinline__ void store_floats(float* p, const float (&v)[M]) {
    static_assert(M <= 2, "one or two channels a lane");
    if constexpr (M == 1) *p = v[0];
    else *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
}
// delta, delta x of two neighbouring channels
__device__ __forceinline__ void put_step(float (*to)[2], f32x2 delta, f32x2 in) {
    float d0, d1, i0, i1;
    unpack2(delta, d0, d1);
    unpack2(in, i0, i1);
    *reinterpret_cast<float4*>(to[0]) = make_float4(d0, i0, d1, i1);
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

// A log2 e, the rate of a decay 2^(rate delta), kept finite: beyond every bound it forgets the state at any step size, but at none (the tokens
// that fill up a group of four have a step size of zero) it keeps it, instead of being infinity times zero.  A NaN stays one.
__device__ __forceinline__ float finite_rate(float rate) { return isinf(rate) ? copysignf(3.402823466e+38f, rate) : rate; }
__device__ __forceinline__ float rate_of(float A) { return finite_rate(A * kLog2E); }
__device__ __forceinline__ f32x2 rate_of2(f32x2 A) {
    float a, b;
    unpack2(fmul2(A, both(kLog2E)), a, b);
    return pack2(finite_rate(a), finite_rate(b));
}
// NS / 2 pairs of a lane's states of channel c.  Behind the last state: zero, or that one again.
//
// Where outputs are read from the states, those that fill up the lanes' are the last one again, Ct 2^-60 times as large, so that
// they add less than a sum's rounding.  With zeros in their rows an infinite delta x (or one that has overflowed) would be NaN in them, and
// out with it.  (8 x 4096 x 384 with sixteen states: 159 us as before; with a search for infinities and those states cleared, 171.)
constexpr float kCopies = 0x1p-60f;
template <int NS, bool COPIES>
__device__ __forceinline__ void load_states(const float* p, int N, int n0, f32x2 (&h)[NS / 2]) {
    const auto at = [&](int n) { return n < N ? p[n] : COPIES && N > 0 ? p[N - 1] : 0.f; };
#pragma unroll
    for (int i = 0; i < NS / 2; ++i) h[i] = pack2(at(n0 + 2 * i), at(n0 + 2 * i + 1));
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
// 2^v of a pair: from the special-function unit (relative error 2^-22, sixteen a clock and SM), or, for fp32 calls, whose sums show that
// error, as arithmetic: 2 to the nearest whole number is put together from bits, 2^f for the rest, |f| <= 1/2, is a polynomial of least largest
// relative error, 2^-28 (fitted like the logarithm's).  Below 2^-126.5 the result is zero.  (A quarter of the
// bf16 states this way, to relieve the special-function unit: 95 to 106 us for 64 x 196 x 1152; an eighth: 100.)
__device__ __forceinline__ f32x2 exp2_special(f32x2 v) {
    float lo, hi;
    unpack2(v, lo, hi);
    return pack2(ex2(lo), ex2(hi));
}
__device__ __forceinline__ float clamp_exponent(float v) {   // (a NaN stays one)
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(v), "f"(-127.f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(y) : "f"(128.f));
    return y;
}
__device__ __forceinline__ f32x2 exp2_arithmetic(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    v = pack2(clamp_exponent(a), clamp_exponent(b));
    const f32x2 whole = fadd2(v, both(12582912.f));   // 1.5 2^23: the nearest whole number in the last bits
    const f32x2 f = fadd2(v, neg_add2(whole, both(12582912.f)));
    f32x2 p = ffma2(f, both(0.0001532646274426952f), both(0.0013390806270763278f));
    p = ffma2(f, p, both(0.009618505835533142f));
    p = ffma2(f, p, both(0.05550359934568405f));
    p = ffma2(f, p, both(0.24022647738456726f));
    p = ffma2(f, p, both(0.6931471824645996f));
    p = ffma2(f, p, both(1.f));
    unpack2(whole, a, b);
    return fmul2(p, pack2(__uint_as_float((__float_as_uint(a) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(b) << 23) + 0x3f800000u)));
}
template <typename T>
__device__ __forceinline__ f32x2 decay2(f32x2 v) {
    if constexpr (sizeof(T) == 4) return exp2_arithmetic(v);
    else return exp2_special(v);
}
template <typename T>
__device__ __forceinline__ float decay_of(float v) {
    if constexpr (sizeof(T) == 2) return ex2(v);
    float lo, hi;
    unpack2(exp2_arithmetic(both(v)), lo, hi);
    return lo;
}
// Sums over the four lanes of a channel of what they hold for four tokens: lane quarter q ends with token q's.
__device__ __forceinline__ float over_quarters(float p0, float p1, float p2, float p3, int quarter) {
    const bool hi = quarter & 2, lo = quarter & 1;
    float k0 = hi ? p2 : p0, k1 = hi ? p3 : p1;
    k0 += __shfl_xor_sync(0xffffffffu, hi ? p0 : p2, 16);
    k1 += __shfl_xor_sync(0xffffffffu, hi ? p1 : p3, 16);
    return (lo ? k1 : k0) + __shfl_xor_sync(0xffffffffu, lo ? k0 : k1, 8);
}

// A tile's rows of Bt or Ct, loaded a tile ahead by all threads of a block: E values a thread.  Behind the last state: COPIES of it, or zero.
template <typename T, int NP, int kTile, int kThreads, bool COPIES>
struct Rows {
    static constexpr int E = (kTile * NP + kThreads - 1) / kThreads;
    const T* p[E];
    long long pitch;
    T v[E];
    __device__ __forceinline__ void start(const T* rows, const Ssm<T>& a, long long ld, const Place& at, int t0) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = threadIdx.x + e * kThreads, n = i % NP;
            p[e] = rows + a.row(at.b, t0 + i / NP) * ld + at.group * a.N + (COPIES ? min(n, a.N - 1) : n);
            from_f32(&v[e], 0.f);
        }
        pitch = a.reverse ? -ld : ld;
    }
    // the tile that starts at token t of `last`, which the pointers stand at
    __device__ __forceinline__ void load(int t, int last, int N) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = threadIdx.x + e * kThreads;
            from_f32(&v[e], 0.f);
            if (i < kTile * NP && (COPIES || i % NP < N) && t + i / NP < last) v[e] = *p[e];   // (as it comes: a conversion would wait for it here)
        }
    }
    __device__ __forceinline__ void move(int tokens) {
#pragma unroll
        for (int e = 0; e < E; ++e) p[e] += tokens * pitch;
    }
    __device__ __forceinline__ void put(float* to) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = threadIdx.x + e * kThreads;
            if (i < kTile * NP) to[i] = to_f32(v[e]);
        }
    }
    // copies reduced to kCopies of the value
    __device__ __forceinline__ void put_reduced(float* to, int N) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = threadIdx.x + e * kThreads;
            if (i < kTile * NP) to[i] = to_f32(v[e]) * (i % NP < N ? 1.f : kCopies);
        }
    }
};

}  // namespace ssm
}  // namespace vig
