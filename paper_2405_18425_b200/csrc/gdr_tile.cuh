// Warp-level pieces of the gated delta rule on the tensor cores (mma.sync, fp16 operands, fp32 sums).
//
// Everything a chunk of up to 64 tokens does to V, U, O and S acts on their columns alike, so a warp owns sixteen columns and works
// transposed: the columns are the rows of its products (M = 16), tokens or key dimensions the columns, and the accumulator of one product is,
// packed, the A operand of the next.  K, Q and the small token-by-token matrices are B operands in shared memory, shared by all warps.
//
// Operands are fp16: eleven significant bits at the rate of bf16's eight.  What fp16 lacks is range, and that is supplied by powers of two:
// a row of K or Q is divided by 2^e of its largest element when it is staged (exact), and a warp's column of S and V by 2^y of the larger of
// its state and its step from outside (exact again), chunk by chunk.  With beta |k|^2 <= 2 nothing in a chunk then exceeds 47000 (the transition
// of a token has norm at most one: a column's norm is at most 11.3 M + 64 x 22.6 M for a largest element M, which is put at 8, and u at most
// twice that).  A warp that meets something larger, infinite or not a number all the same redoes its columns step by step in fp32.
#pragma once
#include <cuda_fp16.h>

#include "ptx.cuh"

namespace vig {
namespace gdr {

constexpr int kChunk = 64;

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void stsm_trans(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// Two adjacent accumulator tiles (sixteen columns) as an A operand; lo: what the first rounding left, eleven bits more.
__device__ __forceinline__ void pack_a(const float (&t0)[4], const float (&t1)[4], uint32_t (&a)[4]) {
    a[0] = pack_half(t0[0], t0[1]);
    a[1] = pack_half(t0[2], t0[3]);
    a[2] = pack_half(t1[0], t1[1]);
    a[3] = pack_half(t1[2], t1[3]);
}
__device__ __forceinline__ uint32_t rest_half(float x, float y, uint32_t hi) {
    const float2 h = unpack_half(hi);
    return pack_half(x - h.x, y - h.y);
}
__device__ __forceinline__ void pack_a_rest(const float (&t0)[4], const float (&t1)[4], const uint32_t (&a)[4], uint32_t (&lo)[4]) {
    lo[0] = rest_half(t0[0], t0[1], a[0]);
    lo[1] = rest_half(t0[2], t0[3], a[1]);
    lo[2] = rest_half(t1[0], t1[1], a[2]);
    lo[3] = rest_half(t1[2], t1[3], a[3]);
}

// Tiles in shared memory: rows of an odd number of 16-byte pieces, so that eight rows at one column never share a bank.
// Addresses of this lane for an ldmatrix of sixteen rows by sixteen columns (row0 and col0 multiples of 16):
//   b     the tile's rows as the columns of a B operand: rows 0-7 take (r[0], r[1]), rows 8-15 (r[2], r[3]); also an A operand's a0, a2, a1, a3
//   t     with a transposing load: B operand that contracts over the rows, columns 0-7 take (r[0], r[1]), columns 8-15 (r[2], r[3])
struct Lane {
    int b_row, b_col, t_row, t_col;
    __device__ __forceinline__ explicit Lane(int lane)
        : b_row((lane & 7) + ((lane >> 4) << 3)), b_col(((lane >> 3) & 1) * 8), t_row(lane & 15), t_col((lane >> 4) * 8) {}
};
template <int PITCH>   // bytes
__device__ __forceinline__ uint32_t at_b(const Lane& l, uint32_t tile, int row0, int col0) {
    return tile + (row0 + l.b_row) * PITCH + (col0 + l.b_col) * 2;
}
template <int PITCH>
__device__ __forceinline__ uint32_t at_t(const Lane& l, uint32_t tile, int row0, int col0) {
    return tile + (row0 + l.t_row) * PITCH + (col0 + l.t_col) * 2;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {   // zeros where !in
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Running maximum of an operand's magnitudes; NaN and what overflowed stay visible.
struct Largest {
    __half2 m = __float2half2_rn(0.f);
    __device__ __forceinline__ void see(const uint32_t (&a)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t& x = *reinterpret_cast<uint32_t*>(&m);
            asm("max.NaN.xorsign.abs.f16x2 %0, %0, %1;" : "+r"(x) : "r"(a[i]));   // (larger magnitude, the signs' product)
        }
    }
    __device__ __forceinline__ bool lost() const {   // infinite or not a number
        const float2 f = __half22float2(m);
        return !(fabsf(f.x) <= 65504.f) || !(fabsf(f.y) <= 65504.f);
    }
};

// Largest magnitude of eight bf16, as the bits of one.
__device__ __forceinline__ uint32_t largest_bf16(const uint4& v) {
    uint32_t m = v.x;
    asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.y));
    asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.z));
    asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.w));
    m &= 0x7fff7fffu;
    return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ f32x2 widen_bf16(uint32_t x) { return pack2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack_half(f32x2 x) {
    float a, b;
    unpack2(x, a, b);
    return pack_half(a, b);
}
__device__ __forceinline__ uint4 bf16_to_half(const uint4& v, float s) {   // times s
    const f32x2 ss = pack2(s, s);
    return make_uint4(pack_half(fmul2(widen_bf16(v.x), ss)), pack_half(fmul2(widen_bf16(v.y), ss)), pack_half(fmul2(widen_bf16(v.z), ss)),
                      pack_half(fmul2(widen_bf16(v.w), ss)));
}
// Two neighbouring values of an accumulator at a time.
__device__ __forceinline__ f32x2 pair(const float (&t)[4], int h) { return pack2(t[2 * h], t[2 * h + 1]); }
__device__ __forceinline__ void set_pair(float (&t)[4], int h, f32x2 x) { unpack2(x, t[2 * h], t[2 * h + 1]); }

// 2^-e and 2^e for the exponent e of a positive float's bits (1 and 1 where it has none: zero, subnormal, infinite, NaN).
__device__ __forceinline__ void power_of(uint32_t exponent, float& down, float& up) {
    const bool ok = exponent >= 1 && exponent <= 253;
    down = ok ? __uint_as_float((254u - exponent) << 23) : 1.f;
    up = ok ? __uint_as_float(exponent << 23) : 1.f;
}

}  // namespace gdr
}  // namespace vig
