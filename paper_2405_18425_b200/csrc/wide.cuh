// 16-byte vectors of bf16 or fp32, and the sigmoid in two precisions: what the row-wise kernels (RMS norm, causal convolution, selective
// scan) share.
#pragma once
#include "ptx.cuh"

namespace vig {

template <typename T>
struct Vec {   // 16 bytes of T
    static constexpr int N = 16 / sizeof(T);
};
__device__ __forceinline__ void widen(const uint4& r, float (&f)[4], const float*) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void widen(const uint4& r, float (&f)[8], const __nv_bfloat16*) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 narrow(const float (&f)[4], const float*) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 narrow(const float (&f)[8], const __nv_bfloat16*) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p) { return *reinterpret_cast<const uint4*>(p); }
template <typename T>
__device__ __forceinline__ void store16(T* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ float reciprocal(float x) {   // one unit in the last place
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2E = 1.4426950408889634f;
// 1 / (1 + e^-z), both steps from the special-function unit: relative error below 2^-21 + |z| 2^-23.6 (the exponent's rounding; |z| counts where z
// is negative) where the result is a normal number.
__device__ __forceinline__ float sigmoid(float z) { return reciprocal(1.f + ex2(-kLog2E * z)); }

}  // namespace vig
