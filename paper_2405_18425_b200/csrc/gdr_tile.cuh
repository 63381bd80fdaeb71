// Warp-level pieces of the gated delta rule on the tensor cores (mma.sync, bf16 operands, fp32 sums).
//
// Everything a chunk of up to 64 tokens does to V, U, O and S acts on their columns alike, so a warp owns sixteen columns and works
// transposed: the columns are the rows of its products (M = 16), tokens or key dimensions the columns, and the accumulator of one product is,
// packed, the A operand of the next.  K, Q and the small token-by-token matrices are B operands in shared memory, shared by all warps.
//
// K, Q, V and dO are bf16 as they come; what is computed is taken as a sum of bf16 terms: two (sixteen significant bits) where results are
// bf16, three (24) where fp32 states leave the call.  Each term has the range of fp32, so a value keeps its digits however small it is beside its
// neighbours; nothing is scaled.  (fp16 under a common power of two per column and chunk has eleven bits in one term, but loses what is 2^-17 of
// the largest value that shares the scale: values before and behind a gate that forgets, rows of the state, tokens of small loss.)
#pragma once
#include "ptx.cuh"

namespace vig {
namespace gdr {

constexpr int kChunk = 64;

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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
__device__ __forceinline__ f32x2 widen_bf16(uint32_t x) { return pack2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
// Two neighbouring values of an accumulator at a time.
__device__ __forceinline__ f32x2 pair(const float (&t)[4], int h) { return pack2(t[2 * h], t[2 * h + 1]); }
__device__ __forceinline__ void set_pair(float (&t)[4], int h, f32x2 x) { unpack2(x, t[2 * h], t[2 * h + 1]); }

// Two values as N terms: each takes what the ones before it left.
template <int N>
__device__ __forceinline__ void split(f32x2 x, uint32_t (&t)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
        float a, b;
        unpack2(x, a, b);
        t[n] = pack_bf16(a, b);
        if (n + 1 < N) x = ffma2(widen_bf16(t[n]), pack2(-1.f, -1.f), x);
    }
}
// Two adjacent accumulator tiles (sixteen columns) as an A operand of N terms.
template <int N>
__device__ __forceinline__ void pack_a(const float (&t0)[4], const float (&t1)[4], uint32_t (&a)[N][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t t[N];
        split<N>(pair(i < 2 ? t0 : t1, i & 1), t);
#pragma unroll
        for (int n = 0; n < N; ++n) a[n][i] = t[n];
    }
}

// Tiles in shared memory: rows of an odd number of 16-byte pieces, so that eight rows at one column never share a bank.
// Addresses of this lane for an ldmatrix of sixteen rows by sixteen columns (row0 and col0 multiples of 16):
//   b     the tile's rows as the columns of a B operand: rows 0-7 take (r[0], r[1]), rows 8-15 (r[2], r[3]); also an A operand's a0, a2, a1, a3
//   t     with a transposing load: B operand that contracts over the rows, columns 0-7 take (r[0], r[1]), columns 8-15 (r[2], r[3])
// Blocks of sixteen rows by sixteen columns lie without gaps, 32 bytes a row; the two pieces of rows 4-7 and 12-15 change places, for the banks' sake.
constexpr int kBlock = 16 * 32;
__device__ __forceinline__ int in_block(int row, int piece) { return row * 32 + ((piece ^ ((row >> 2) & 1)) << 4); }
struct Lane {
    int b_row, b_col, t_row, t_col, b_block, t_block;
    __device__ __forceinline__ explicit Lane(int lane)
        : b_row((lane & 7) + ((lane >> 4) << 3)), b_col(((lane >> 3) & 1) * 8), t_row(lane & 15), t_col((lane >> 4) * 8),
          b_block(in_block(b_row, b_col >> 3)), t_block(in_block(t_row, t_col >> 3)) {}
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

// Running sums of log2 alpha of a chunk as two floats: multiples of 2^-8, of which 64 add up exactly (a gate counts down to 2^-160, below which fp32
// keeps nothing of a state), and what is left, below 2^-3 in sum.  So a difference of two sums is as exact behind gates that forget as anywhere: of
// one float it had lost up to ten bits.
struct Sum {
    float h, l;
    __device__ __forceinline__ float to(const Sum& s) const { return (h - s.h) + (l - s.l); }   // from s to here
};
// The sums at tokens 2 lane and 2 lane + 1, and of the whole chunk, of natural logarithms la.
__device__ __forceinline__ void gate_sums(const float (&la)[2], Sum (&b)[2], Sum& all) {
    const int lane = threadIdx.x & 31;
    float h[2], l[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float x = la[i] * 1.4426950408889634f;
        x = x < -160.f ? -160.f : x;
        h[i] = rintf(x * 256.f) * 0x1p-8f;
        l[i] = x - h[i];
    }
    float rh = h[0] + h[1], rl = l[0] + l[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float yh = __shfl_up_sync(0xffffffffu, rh, o), yl = __shfl_up_sync(0xffffffffu, rl, o);
        if (lane >= o) {
            rh += yh;
            rl += yl;
        }
    }
    all = {__shfl_sync(0xffffffffu, rh, 31), __shfl_sync(0xffffffffu, rl, 31)};
    b[0] = {rh - h[1], rl - l[1]};
    b[1] = {rh, rl};
}

// Largest magnitudes of pairs of bf16; a NaN stays.
__device__ __forceinline__ void see(uint32_t& m, uint32_t x) { asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(x)); }   // (larger magnitude, the signs' product)
__device__ __forceinline__ bool within(uint32_t m, float limit) {   // false for what is not finite
    limit = fminf(limit, 3.3e38f);
    return fabsf(__uint_as_float(m << 16)) <= limit && fabsf(__uint_as_float(m & 0xffff0000u)) <= limit;
}
__device__ __forceinline__ float largest_of(uint32_t m) { return fmaxf(__uint_as_float((m & 0x7fffu) << 16), __uint_as_float(m & 0x7fff0000u)); }   // (of no NaN)
__device__ __forceinline__ void larger(uint32_t& m, uint32_t x) { asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(x)); }   // (a NaN is passed over)
__device__ __forceinline__ void larger(uint32_t& m, const uint4& v) {
    larger(m, v.x);
    larger(m, v.y);
    larger(m, v.z);
    larger(m, v.w);
}

}  // namespace gdr
}  // namespace vig
