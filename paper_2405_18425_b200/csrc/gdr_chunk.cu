// The gated delta rule in chunks of 64 tokens on the tensor cores (bf16 calls): what goes from chunk to chunk.
//
// With b the running sum of log alpha in a chunk, Gam_ts = e^{b_t - b_s}, N = strict_tril(K K^T . Gam), P = tril(Q K^T . Gam):
//   forwards    W = V - e^b K S - N U, U = beta W       O = e^b Q S + P U        S <- e^{b_C} S + (e^{b_C - b} K)^T U
//   backwards   dU = P^T dO + e^{b_C - b} K A - N^T R, R = beta dU (= dV)        A <- e^{b_C} A + (e^b Q)^T dO - (e^b K)^T R
// The triangular systems are solved sixteen tokens at a time: what the other sixteens contribute is a product with N, what the sixteen do to
// one another a product with the inverse of 1 + beta N of their own 16 x 16 block, which one warp computes by substitution in fp32.
// e^{b_t - b_s} is taken of the difference, never of its parts, so that no gate is out of range.
//
// A block runs through the chunks of a unit for up to 64 columns.  Four of its warps prepare: they bring the rows of K and Q, scale them and
// make N, P and the inverses of the next chunk while the others, a warp for every sixteen columns (gdr_tile.cuh), work on this one.  Two
// buffers, handed over by named barriers.  (All warps doing both in turn: 64 x 12 units of 196 tokens, 32 x 64, 70 us, 32 units of 4096, 24 x
// 48, 448 us: a chunk took 7 us from start to end.)
#include <type_traits>

#include "gdr.h"
#include "gdr_tile.cuh"

namespace vig {
namespace {

using namespace gdr;
using bf = __nv_bfloat16;

constexpr int kMostWarps = 4;       // with columns
constexpr int kPrepWarps = 4;
constexpr int kPrep = 32 * kPrepWarps;
constexpr int kBlockPitch = 48, kBlock = 16 * kBlockPitch, kColPitch = 48;
// Token-by-token matrices are kept as their lower triangle of 16 x 16 blocks.
__device__ __forceinline__ int block_of(int i, int j) { return (i * (i + 1) / 2 + j) * kBlock; }
constexpr int kBarFull = 1, kBarEmpty = 3, kBarPrep = 5;   // named barriers: two of the first two

enum class Way { kForward, kKeep, kBack };   // the call's result; the gradient's forward walk, which keeps W and the states; its way back

template <int DKP>
constexpr int key_pitch() { return DKP * 2 + 16; }

// Per token of a chunk, in shared memory: arrays of kChunk floats.
//   b running sum of log2 alpha; eb 2^b; dl 2^{b_C - b}; gv beta 2^e and gn beta 2^{2e} with 2^e the scale of the key's row (ku); qu the query's
enum { kB, kEb, kDl, kBeta, kGv, kGn, kKu, kQu, kGateRows };
__device__ __forceinline__ f32x2 gate_pair(const float* gates, int row, int t) { return *reinterpret_cast<const f32x2*>(gates + row * kChunk + t); }

// Shared memory, in bytes.
template <int DKP, bool EXACT, Way WAY>
struct Layout {
    static constexpr int kKeys = kChunk * key_pitch<DKP>(), kMat = 10 * kBlock, kInv = 4 * kBlock, kCols = kChunk * kColPitch;
    static constexpr bool kQ = WAY != Way::kKeep;   // queries, and P
    // of a buffer: keys, queries, N, P, inverses, gates, and what their first rounding left
    static constexpr int kQueries = kKeys, kN = kQueries + (kQ ? kKeys : 0), kP = kN + kMat, kInverse = kP + (kQ ? kMat : 0), kGates = kInverse + kInv,
                         kNLo = kGates + kChunk * kGateRows * 4, kPLo = kNLo + (EXACT ? kMat : 0),
                         kInvLo = kPLo + (EXACT && WAY == Way::kBack ? kMat : 0), kBuffer = kInvLo + (EXACT ? kInv : 0);
    static constexpr int x = 2 * kBuffer;                  // the diagonal blocks of beta N, transposed, rows of 20 floats
    static constexpr int cols = x + 4 * 16 * 20 * 4;       // a warp's columns of V or dO, two chunks
    static constexpr int k(int buf) { return buf * kBuffer; }
    static constexpr int q(int buf) { return buf * kBuffer + kQueries; }
    static constexpr int n(int buf) { return buf * kBuffer + kN; }
    static constexpr int p(int buf) { return buf * kBuffer + kP; }
    static constexpr int inv(int buf) { return buf * kBuffer + kInverse; }
    static constexpr int gates(int buf) { return buf * kBuffer + kGates; }
    static constexpr int n_lo(int buf) { return buf * kBuffer + kNLo; }
    static constexpr int p_lo(int buf) { return buf * kBuffer + kPLo; }
    static constexpr int inv_lo(int buf) { return buf * kBuffer + kInvLo; }
    static constexpr int total(int warps) { return cols + 2 * warps * kCols; }
};

// What the gradient's walks leave for its last launch, per unit and chunk (see gdr.h).
using Kept = GdrKept;

__device__ __forceinline__ void bar_arrive(int id, int count) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(count) : "memory"); }

// ---- the preparing warps ----------------------------------------------------------------------------------------------
template <int DKP, bool EXACT, Way WAY>
__device__ void prepare_chunks(const Gdr<bf>& a, unsigned char* smem, const Layout<DKP, EXACT, WAY>& lay, long long unit, int chunks, int threads) {
    constexpr int KP = key_pitch<DKP>(), KS = DKP / 16;
    constexpr bool Q = WAY != Way::kKeep;
    constexpr int kLanes = DKP <= 16 ? 2 : DKP <= 32 ? 4 : DKP <= 64 ? 8 : 16;   // of a row
    constexpr int kRows = kPrep / kLanes, kPasses = (Q ? 2 : 1) * kChunk / kRows;
    const int tid = threadIdx.x - (blockDim.x - kPrep), lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int e8 = tid % kLanes * 8, r0 = tid / kLanes;
    const uint32_t base = smem_u32(smem);
    const Lane ln(lane);
    uint4 rows[kPasses];
    float la[2], be[2];
    auto bring = [&](int n) {
        const int t0 = n * kChunk;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int r = p * kRows + r0, t = r & (kChunk - 1);
            rows[p] = make_uint4(0u, 0u, 0u, 0u);
            if (t0 + t < a.L && e8 < a.dk) rows[p] = *reinterpret_cast<const uint4*>((r < kChunk ? a.k : a.q) + a.row(unit, t0 + t) * a.dk + e8);
        }
        if (warp == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = t0 + 2 * lane + h;
                la[h] = t < a.L ? __bfloat162float(a.la[a.row(unit, t)]) : 0.f;
                be[h] = t < a.L ? __bfloat162float(a.beta[a.row(unit, t)]) : 0.f;
            }
    };
    bring(WAY == Way::kBack ? chunks - 1 : 0);
    for (int it = 0; it < chunks; ++it) {
        const int n = WAY == Way::kBack ? chunks - 1 - it : it, buf = it & 1, strips = (min(kChunk, a.L - n * kChunk) + 15) >> 4;
        if (it >= 2) named_bar(kBarEmpty + buf, threads);
        float* const gates = reinterpret_cast<float*>(smem + lay.gates(buf));
        if (warp == 0) {   // running sum of log2 alpha, two tokens a lane
            float l[2], s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // (below 2^-150 nothing of the state is left in fp32; the bound keeps sums of such gates exact to 2^-11)
                const float x = la[h] * 1.4426950408889634f;
                l[h] = x < -160.f ? -160.f : x;
            }
            s[0] = l[0];
            s[1] = l[0] + l[1];
            float run = s[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float y = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += y;
            }
            const float before = run - s[1], all = __shfl_sync(0xffffffffu, run, 31), b0 = before + s[0], b1 = before + s[1];
            auto two = [&](int row, float x, float y) { *reinterpret_cast<float2*>(gates + row * kChunk + 2 * lane) = make_float2(x, y); };
            two(kB, b0, b1);
            two(kEb, ex2(b0), ex2(b1));
            two(kDl, ex2(all - b0), ex2(all - b1));
            two(kBeta, be[0], be[1]);
        }
        // K and Q to fp16, each row over its largest element's power of two
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int r = p * kRows + r0, t = r & (kChunk - 1);
            const uint4 x = rows[p];
            uint32_t m = largest_bf16(x);
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            float down, up;
            power_of(m >> 7, down, up);
            if (e8 < DKP) *reinterpret_cast<uint4*>(smem + (r < kChunk ? lay.k(buf) : lay.q(buf)) + t * KP + e8 * 2) = bf16_to_half(x, down);
            if (e8 == 0) gates[(r < kChunk ? kKu : kQu) * kChunk + t] = up;
        }
        named_bar(kBarPrep, kPrep);
        if (tid < kChunk) {
            const float gv = gates[kBeta * kChunk + tid] * gates[kKu * kChunk + tid];
            gates[kGv * kChunk + tid] = gv;
            gates[kGn * kChunk + tid] = gv * gates[kKu * kChunk + tid];
        }
        if (it + 1 < chunks) bring(WAY == Way::kBack ? n - 1 : n + 1);
        // N and P by blocks of sixteen by sixteen: two of the diagonal's for each of the first two warps, with their inverses side by side; three
        // of the others for each of the other two
        const uint32_t kt = base + lay.k(buf), qt = base + lay.q(buf);
        auto products = [&](int i, int j, float (&nn)[2][4], float (&pp)[2][4]) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t kb[4], x[4];
                ldsm(at_b<KP>(ln, kt, j * 16, s * 16), kb);
                if constexpr (Q) {
                    ldsm(at_b<KP>(ln, qt, i * 16, s * 16), x);
                    const uint32_t qa[4] = {x[0], x[2], x[1], x[3]};
                    mma(pp[0], qa, kb[0], kb[1]);
                    mma(pp[1], qa, kb[2], kb[3]);
                }
                ldsm(at_b<KP>(ln, kt, i * 16, s * 16), x);
                const uint32_t ka[4] = {x[0], x[2], x[1], x[3]};
                mma(nn[0], ka, kb[0], kb[1]);
                mma(nn[1], ka, kb[2], kb[3]);
            }
        };
        auto put = [&](int hi_at, int lo_at, bool lo, int at, f32x2 x) {
            const uint32_t hi = pack_half(x);
            *reinterpret_cast<uint32_t*>(smem + hi_at + at) = hi;
            if (lo) {
                float u, v;
                unpack2(x, u, v);
                *reinterpret_cast<uint32_t*>(smem + lo_at + at) = rest_half(u, v, hi);
            }
        };
        if (warp < 2) {
            float* const xt = reinterpret_cast<float*>(smem + lay.x) + warp * 2 * 16 * 20;
#pragma unroll 1
            for (int d = 0; d < 2; ++d) {
                const int i = 2 * warp + d;
                if (i >= strips) break;
                float nn[2][4] = {}, pp[2][4] = {};
                products(i, i, nn, pp);
#pragma unroll
                for (int h = 0; h < 2; ++h) {   // rows g, g + 8
                    const int tt = g + 8 * h, t = i * 16 + tt;
                    const float bt = gates[kB * kChunk + t], ku = gates[kKu * kChunk + t], gn = gates[kBeta * kChunk + t] * ku * ku;
#pragma unroll
                    for (int m = 0; m < 2; ++m) {   // columns 8m + 2c, + 1
                        const int ss = 8 * m + 2 * c, at = block_of(i, i) + tt * kBlockPitch + ss * 2;
                        const float2 bs = *reinterpret_cast<const float2*>(gates + kB * kChunk + i * 16 + ss);
                        const float e0 = ss <= tt ? ex2(bt - bs.x) : 0.f, e1 = ss + 1 <= tt ? ex2(bt - bs.y) : 0.f;
                        // (selected, not multiplied: what is not finite stays out of earlier tokens)
                        if constexpr (Q) put(lay.p(buf), lay.p_lo(buf), EXACT && WAY == Way::kBack, at, pack2(ss <= tt ? pp[m][2 * h] * e0 : 0.f, ss + 1 <= tt ? pp[m][2 * h + 1] * e1 : 0.f));
                        const float n0 = ss < tt ? nn[m][2 * h] * e0 : 0.f, n1 = ss + 1 < tt ? nn[m][2 * h + 1] * e1 : 0.f;
                        if constexpr (WAY == Way::kKeep) put(lay.n(buf), 0, false, at, pack2(n0, n1));   // (W takes its own strip's off)
                        xt[(d * 16 + ss) * 20 + tt] = n0 * gn;   // beta N, transposed: row s, column t
                        xt[(d * 16 + ss + 1) * 20 + tt] = n1 * gn;
                    }
                }
            }
            __syncwarp();
            // (1 + beta N)^-1, a column a lane, a block a half warp: x_t -= (beta N)_ts x_s as soon as x_s is known
            const int cc = lane & 15, i = 2 * warp + (lane >> 4);
            const float* const own = xt + (lane >> 4) * 16 * 20;
            float x[16];
#pragma unroll
            for (int t = 0; t < 16; ++t) x[t] = t == cc ? 1.f : 0.f;
#pragma unroll
            for (int s = 0; s < 15; ++s) {
#pragma unroll
                for (int p = (s + 1) / 4; p < 4; ++p) {
                    const float4 r = *reinterpret_cast<const float4*>(own + s * 20 + 4 * p);
                    if (4 * p > s) x[4 * p] = fmaf(-r.x, x[s], x[4 * p]);
                    if (4 * p + 1 > s) x[4 * p + 1] = fmaf(-r.y, x[s], x[4 * p + 1]);
                    if (4 * p + 2 > s) x[4 * p + 2] = fmaf(-r.z, x[s], x[4 * p + 2]);
                    if (4 * p + 3 > s) x[4 * p + 3] = fmaf(-r.w, x[s], x[4 * p + 3]);
                }
            }
            if (i < strips)
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const __half hi = __float2half_rn(x[t]);
                    *reinterpret_cast<__half*>(smem + lay.inv(buf) + i * kBlock + t * kBlockPitch + cc * 2) = hi;
                    if constexpr (EXACT)
                        *reinterpret_cast<__half*>(smem + lay.inv_lo(buf) + i * kBlock + t * kBlockPitch + cc * 2) = __float2half_rn(x[t] - __half2float(hi));
                }
        } else {
#pragma unroll 1
            for (int w = 0; w < 3; ++w) {
                // (3,0) (3,1) (3,2), (1,0) (2,0) (2,1)
                const int i = warp == 2 ? 3 : w == 0 ? 1 : 2, j = warp == 2 ? w : w == 2 ? 1 : 0;
                if (i >= strips) continue;
                float nn[2][4] = {}, pp[2][4] = {};
                products(i, j, nn, pp);
                // e^{b_t - b_s} by way of the last token of s' sixteen: both factors are at most one
                const float ref = gates[kB * kChunk + j * 16 + 15];
                f32x2 ec[2];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const float2 bs = *reinterpret_cast<const float2*>(gates + kB * kChunk + j * 16 + 8 * m + 2 * c);
                    ec[m] = pack2(ex2(ref - bs.x), ex2(ref - bs.y));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float et = ex2(gates[kB * kChunk + i * 16 + g + 8 * h] - ref);
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const int at = block_of(i, j) + (g + 8 * h) * kBlockPitch + (8 * m + 2 * c) * 2;
                        const f32x2 e = fmul2(ec[m], pack2(et, et));
                        if constexpr (Q) put(lay.p(buf), lay.p_lo(buf), EXACT && WAY == Way::kBack, at, fmul2(pair(pp[m], h), e));
                        put(lay.n(buf), lay.n_lo(buf), EXACT, at, fmul2(pair(nn[m], h), e));
                    }
                }
            }
        }
        bar_arrive(kBarFull + buf, threads);
    }
}

// ---- the warps with columns ---------------------------------------------------------------------------------------------

// Columns of a warp step by step in fp32, two lanes a column: what leaves the range of the tiles.
template <int DKP>
__device__ __noinline__ void walk_sixteen(const Gdr<bf>& a, long long unit, int j, int half) {
    const bool valid = j < a.dv;
    const long long plane = (long long)a.dk * a.dv;
    float S[DKP / 2];
#pragma unroll 1
    for (int i = 0; i < DKP / 2; ++i) {
        const int e = 2 * i + half;
        S[i] = a.state_in && valid && e < a.dk ? a.state_in[unit * plane + (long long)e * a.dv + j] : 0.f;
    }
#pragma unroll 1
    for (int t = 0; t < a.L; ++t) {
        const long long r = a.row(unit, t);
        const float alpha = expf(__bfloat162float(a.la[r])), beta = __bfloat162float(a.beta[r]);
        float s = 0.f, o = 0.f;
#pragma unroll 1
        for (int i = 0; 2 * i + half < a.dk; ++i) {
            S[i] *= alpha;
            s = fmaf(__bfloat162float(a.k[r * a.dk + 2 * i + half]), S[i], s);
        }
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        const float u = valid ? beta * (__bfloat162float(a.v[r * a.dv + j]) - s) : 0.f;
#pragma unroll 1
        for (int i = 0; 2 * i + half < a.dk; ++i) {
            S[i] = fmaf(__bfloat162float(a.k[r * a.dk + 2 * i + half]), u, S[i]);
            o = fmaf(__bfloat162float(a.q[r * a.dk + 2 * i + half]), S[i], o);
        }
        o += __shfl_xor_sync(0xffffffffu, o, 16);
        if (valid && half == 0) a.out[r * a.dv + j] = __float2bfloat16_rn(o);
    }
    if (a.state_out && valid)
#pragma unroll 1
        for (int i = 0; 2 * i + half < a.dk; ++i) a.state_out[unit * plane + (long long)(2 * i + half) * a.dv + j] = S[i];
}

// The state of sixteen columns, transposed: tile n holds key dimensions 8n + 2c, + 1 of columns g (0, 1) and g + 8 (2, 3), times `scale`, a
// power of two per column.
template <int DKP>
struct State {
    float x[DKP / 8][4];
    float scale[2] = {1.f, 1.f};
    __device__ __forceinline__ void load(const float* from, long long unit, const Gdr<bf>& a, int col, int c) {
        const long long plane = (long long)a.dk * a.dv;
#pragma unroll
        for (int n = 0; n < DKP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = n * 8 + 2 * c + (e & 1), j = col + (e >> 1) * 8;
                x[n][e] = from && i < a.dk && j < a.dv ? from[unit * plane + (long long)i * a.dv + j] : 0.f;
            }
    }
    __device__ __forceinline__ void store(float* to, long long unit, const Gdr<bf>& a, int col, int c) const {
        const long long plane = (long long)a.dk * a.dv;
#pragma unroll
        for (int n = 0; n < DKP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = n * 8 + 2 * c + (e & 1), j = col + (e >> 1) * 8;
                if (i < a.dk && j < a.dv) to[unit * plane + (long long)i * a.dv + j] = x[n][e] / scale[e >> 1];
            }
    }
    // New scales: the larger of the state and `outside` (per column) to [2^TOP / 2, 2^TOP).  back: what undoes them.
    template <int TOP>
    __device__ __forceinline__ void rescale(const float (&outside)[2], float (&back)[2]) {
        float most[2] = {0.f, 0.f};
#pragma unroll
        for (int m = 0; m < DKP / 8; ++m) {
            most[0] = fmaxf(most[0], fmaxf(fabsf(x[m][0]), fabsf(x[m][1])));
            most[1] = fmaxf(most[1], fmaxf(fabsf(x[m][2]), fabsf(x[m][3])));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float m = fmaxf(outside[h], most[h] / scale[h]);   // (a power of two: exact)
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const uint32_t ex = min(max(__float_as_uint(m) >> 23, 10u), 244u);
            const float now = __uint_as_float((253u + TOP - ex) << 23), change = now / scale[h];
            back[h] = __uint_as_float((ex + 1u - TOP) << 23);
            scale[h] = now;
            if (__any_sync(0xffffffffu, change != 1.f)) {
                const f32x2 cc = pack2(change, change);
#pragma unroll
                for (int n = 0; n < DKP / 8; ++n) set_pair(x[n], h, fmul2(pair(x[n], h), cc));
            }
        }
    }
    __device__ __forceinline__ void decay(float s) {
        const f32x2 ss = pack2(s, s);
#pragma unroll
        for (int n = 0; n < DKP / 8; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(x[n], h, fmul2(pair(x[n], h), ss));
    }
};

// acc += A^T-operand x rows of a key tile: D[columns x tokens of the strip]
template <int DKP, int TERMS>
__device__ __forceinline__ void state_times_rows(float (&acc)[2][4], const uint32_t (*hi)[4], const uint32_t (*lo)[4], uint32_t tile, int strip, const Lane& ln) {
#pragma unroll
    for (int s = 0; s < DKP / 16; ++s) {
        uint32_t x[4];
        ldsm(at_b<key_pitch<DKP>()>(ln, tile, strip * 16, s * 16), x);
        mma(acc[0], hi[s], x[0], x[1]);
        mma(acc[1], hi[s], x[2], x[3]);
        if constexpr (TERMS == 2) {
            mma(acc[0], lo[s], x[0], x[1]);
            mma(acc[1], lo[s], x[2], x[3]);
        }
    }
}
// S += (sixteen tokens' operand) x their rows of a key tile
template <int DKP, int TERMS>
__device__ __forceinline__ void rows_into_state(State<DKP>& S, const uint32_t (&hi)[4], const uint32_t (&lo)[4], uint32_t tile, int strip, const Lane& ln) {
#pragma unroll
    for (int s = 0; s < DKP / 16; ++s) {
        uint32_t y[4];
        ldsm_trans(at_t<key_pitch<DKP>()>(ln, tile, strip * 16, s * 16), y);
        mma(S.x[2 * s], hi, y[0], y[1]);
        mma(S.x[2 * s + 1], hi, y[2], y[3]);
        if constexpr (TERMS == 2) {
            mma(S.x[2 * s], lo, y[0], y[1]);
            mma(S.x[2 * s + 1], lo, y[2], y[3]);
        }
    }
}
// acc += operand x a 16 x 16 block of a token-by-token matrix, contracted over its columns, or with TRANS over its rows
template <bool TRANS, int TERMS>
__device__ __forceinline__ void times_block(float (&acc)[2][4], const uint32_t (&hi)[4], const uint32_t (&lo)[4], uint32_t block, uint32_t block_lo,
                                            const Lane& ln) {
    uint32_t x[4];
    if constexpr (TRANS) ldsm_trans(at_t<kBlockPitch>(ln, block, 0, 0), x);
    else ldsm(at_b<kBlockPitch>(ln, block, 0, 0), x);
    mma(acc[0], hi, x[0], x[1]);
    mma(acc[1], hi, x[2], x[3]);
    if constexpr (TERMS == 2) {
        mma(acc[0], lo, x[0], x[1]);
        mma(acc[1], lo, x[2], x[3]);
        uint32_t y[4];
        if constexpr (TRANS) ldsm_trans(at_t<kBlockPitch>(ln, block_lo, 0, 0), y);
        else ldsm(at_b<kBlockPitch>(ln, block_lo, 0, 0), y);
        mma(acc[0], hi, y[0], y[1]);
        mma(acc[1], hi, y[2], y[3]);
    }
}
template <int TERMS>
__device__ __forceinline__ void pack_terms(const float (&t)[2][4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    pack_a(t[0], t[1], hi);
    if constexpr (TERMS == 2) pack_a_rest(t[0], t[1], hi, lo);
}
__device__ __forceinline__ float2 gate2(const float* gates, int row, int t) { return *reinterpret_cast<const float2*>(gates + row * kChunk + t); }

// One chunk of NS strips forwards.
template <int DKP, bool EXACT, Way WAY, int NS>
__device__ __forceinline__ void forward_chunk(State<DKP>& S, Largest& seen, const Gdr<bf>& a, const Kept& kept, unsigned char* smem,
                                              const Layout<DKP, EXACT, WAY>& lay, int buf, int cols, long long unit, int n, int chunks, int col0, int lane,
                                              const Lane& ln) {
    constexpr int KS = DKP / 16, TERMS = EXACT ? 2 : 1;
    constexpr bool OUT = WAY == Way::kForward;
    const int g = lane >> 2, c = lane & 3;
    const uint32_t base = smem_u32(smem), kt = base + lay.k(buf), qt = base + lay.q(buf), vt = base + cols;
    const float* const gates = reinterpret_cast<const float*>(smem + lay.gates(buf));
    float gmax = fmaxf(fabsf(gates[kGv * kChunk + lane]), fabsf(gates[kGv * kChunk + lane + 32])), vmax[2] = {0.f, 0.f}, back[2];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, o));
    if constexpr (!OUT) gmax = fmaxf(gmax, 1.f);   // W itself is kept too
    uint32_t vm[2] = {0u, 0u}, vv[NS][4];   // V transposed: strip i, columns g (0, 2), g + 8 (1, 3) of tokens 2c, 2c + 1 (0, 1), + 8 (2, 3)
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        uint32_t x[4];
        ldsm_trans(vt + (i * 16 + ln.t_row) * kColPitch + ln.t_col * 2, x);
        vv[i][0] = x[0]; vv[i][1] = x[2]; vv[i][2] = x[1]; vv[i][3] = x[3];
        asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(vm[0]) : "r"(vv[i][0]));
        asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(vm[1]) : "r"(vv[i][1]));
        asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(vm[0]) : "r"(vv[i][2]));
        asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(vm[1]) : "r"(vv[i][3]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) vmax[h] = fmaxf(__uint_as_float((vm[h] & 0x7fffu) << 16), __uint_as_float(vm[h] & 0x7fff0000u));
    vmax[0] *= gmax;
    vmax[1] *= gmax;
    S.template rescale<3>(vmax, back);
    uint32_t sa[KS][4], sl[EXACT ? KS : 1][4];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        pack_a(S.x[2 * s], S.x[2 * s + 1], sa[s]);   // (what does not fit shows in U)
        if constexpr (EXACT) pack_a_rest(S.x[2 * s], S.x[2 * s + 1], sa[s], sl[s]);
    }
    if constexpr (!OUT) kept.keep_state<DKP>(kept.S, kept.y, unit * (chunks + 1) + n, col0, sa, back, g, c);
    S.decay(gates[kEb * kChunk + kChunk - 1]);
    // products with S, of all strips; then strip by strip, what a strip's U means to the strips behind it as soon as it is there: the next
    // strip's chain (N, the step, the inverse) is what bounds a chunk, all else fills its gaps
    float w[NS][2][4] = {}, o[OUT ? NS : 1][2][4] = {};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        state_times_rows<DKP, TERMS>(w[i], sa, sl, kt, i, ln);
        if constexpr (OUT) state_times_rows<DKP, 1>(o[i], sa, sl, qt, i, ln);
    }
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 eb = gate_pair(gates, kEb, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                set_pair(w[i][m], h, fmul2(pair(w[i][m], h), eb));
                if constexpr (OUT) set_pair(o[i][m], h, fmul2(pair(o[i][m], h), eb));
            }
        }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        float r[2][4], uu[2][4] = {};
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 ku = gate_pair(gates, kKu, i * 16 + 8 * m + 2 * c), gv = gate_pair(gates, kGv, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 got = fmul2(pair(w[i][m], h), ku);
                const f32x2 y = ffma2(got, pack2(-1.f, -1.f), fmul2(widen_bf16(vv[i][2 * m + h]), pack2(S.scale[h], S.scale[h])));
                if constexpr (!OUT) set_pair(w[i][m], h, y);
                set_pair(r[m], h, fmul2(gv, y));
            }
        }
        uint32_t ra[4], rl[4], u[4], ul[4];
        pack_terms<TERMS>(r, ra, rl);
        times_block<false, TERMS>(uu, ra, rl, base + lay.inv(buf) + i * kBlock, base + lay.inv_lo(buf) + i * kBlock, ln);
        pack_terms<TERMS>(uu, u, ul);
        seen.see(u);
#pragma unroll
        for (int j = i + 1; j < NS; ++j) times_block<false, TERMS>(w[j], u, ul, base + lay.n(buf) + block_of(j, i), base + lay.n_lo(buf) + block_of(j, i), ln);
        if constexpr (OUT)
#pragma unroll
            for (int j = i; j < NS; ++j) times_block<false, 1>(o[j], u, ul, base + lay.p(buf) + block_of(j, i), 0, ln);
        // S += (e^{b_C - b} U)^T K
        uint32_t ud[4], udl[4];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 dl = gate_pair(gates, kDl, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(uu[m], h, fmul2(pair(uu[m], h), dl));
        }
        pack_terms<TERMS>(uu, ud, udl);
        rows_into_state<DKP, TERMS>(S, ud, udl, kt, i, ln);
        uint32_t res[2][2];
        if constexpr (OUT) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const f32x2 qu = gate_pair(gates, kQu, i * 16 + 8 * m + 2 * c);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x, y;
                    unpack2(fmul2(fmul2(pair(o[i][m], h), qu), pack2(back[h], back[h])), x, y);
                    res[m][h] = pack_bf16(x, y);
                }
            }
        } else {   // W of the strip: what its own block takes off
            float own[2][4] = {};
            times_block<false, 1>(own, u, ul, base + lay.n(buf) + block_of(i, i), 0, ln);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const float2 ku = gate2(gates, kKu, i * 16 + 8 * m + 2 * c);
#pragma unroll
                for (int h = 0; h < 2; ++h) res[m][h] = pack_half(fmaf(-ku.x, own[m][2 * h], w[i][m][2 * h]), fmaf(-ku.y, own[m][2 * h + 1], w[i][m][2 * h + 1]));
            }
            const uint32_t ws[4] = {res[0][0], res[0][1], res[1][0], res[1][1]};
            seen.see(ws);
        }
        // over the strip's values, and out from there in pieces of sixteen bytes
        stsm_trans(vt + (i * 16 + ln.t_row) * kColPitch + ln.t_col * 2, res[0][0], res[1][0], res[0][1], res[1][1]);
        __syncwarp();
        const int t = i * 16 + (lane >> 1), e = (lane & 1) * 8;
        const uint4 piece = *reinterpret_cast<const uint4*>(smem + cols + t * kColPitch + e * 2);
        if constexpr (OUT) {
            if (n * kChunk + t < a.L && col0 + e < a.dv) *reinterpret_cast<uint4*>(a.out + a.row(unit, n * kChunk + t) * a.dv + col0 + e) = piece;
        } else *reinterpret_cast<uint4*>(kept.w + ((unit * chunks + n) * kChunk + t) * kept.dvp + col0 + e) = piece;
    }
}

// One chunk of NS strips backwards: S is A, the columns are those of dO.
template <int DKP, bool EXACT, int NS>
__device__ __forceinline__ void backward_chunk(State<DKP>& A, Largest& seen, const Gdr<bf>& a, const Kept& kept, unsigned char* smem,
                                               const Layout<DKP, EXACT, Way::kBack>& lay, int buf, int cols, long long unit, int n, int chunks, int col0,
                                               int lane, const Lane& ln) {
    constexpr int KS = DKP / 16, TERMS = EXACT ? 2 : 1;
    const int g = lane >> 2, c = lane & 3;
    const uint32_t base = smem_u32(smem), kt = base + lay.k(buf), qt = base + lay.q(buf), vt = base + cols;
    const float* const gates = reinterpret_cast<const float*>(smem + lay.gates(buf));
    // dO, times the scale of its query's row: everything it meets is a product with that row
    float most[2] = {0.f, 0.f}, back[2];
    uint32_t dd[NS][4];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        uint32_t x[4];
        ldsm_trans(vt + (i * 16 + ln.t_row) * kColPitch + ln.t_col * 2, x);
        dd[i][0] = x[0]; dd[i][1] = x[2]; dd[i][2] = x[1]; dd[i][3] = x[3];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const float2 qu = gate2(gates, kQu, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                most[h] = fmaxf(most[h], fmaxf(fabsf(__uint_as_float(dd[i][2 * m + h] << 16)) * qu.x, fabsf(__uint_as_float(dd[i][2 * m + h] & 0xffff0000u)) * qu.y));
        }
    }
    A.template rescale<0>(most, back);
    uint32_t aa[KS][4], al[EXACT ? KS : 1][4];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        pack_a(A.x[2 * s], A.x[2 * s + 1], aa[s]);   // (what does not fit shows in dU)
        if constexpr (EXACT) pack_a_rest(A.x[2 * s], A.x[2 * s + 1], aa[s], al[s]);
    }
    kept.keep_state<DKP>(kept.A, kept.z, unit * chunks + n, col0, aa, back, g, c);
    A.decay(gates[kEb * kChunk + kChunk - 1]);
    auto d_out = [&](int i, float (&x)[2][4]) {   // scaled
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 qu = gate_pair(gates, kQu, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(x[m], h, fmul2(fmul2(widen_bf16(dd[i][2 * m + h]), qu), pack2(A.scale[h], A.scale[h])));
        }
    };
    float r[NS][2][4] = {};
#pragma unroll
    for (int i = 0; i < NS; ++i) state_times_rows<DKP, TERMS>(r[i], aa, al, kt, i, ln);
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 dl = gate_pair(gates, kDl, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(r[i][m], h, fmul2(pair(r[i][m], h), dl));
        }
#pragma unroll
    for (int j = NS - 1; j >= 0; --j) {
        float x[2][4];
        uint32_t db[4], dbl[4];
        d_out(j, x);
        pack_terms<TERMS>(x, db, dbl);
#pragma unroll
        for (int i = j; i >= 0; --i) times_block<true, TERMS>(r[i], db, dbl, base + lay.p(buf) + block_of(j, i), base + lay.p_lo(buf) + block_of(j, i), ln);
    }
#pragma unroll
    for (int i = NS - 1; i >= 0; --i) {
        uint32_t pa[4], pl[4];
        float du[2][4] = {}, x[2][4];
        pack_terms<TERMS>(r[i], pa, pl);
        times_block<true, TERMS>(du, pa, pl, base + lay.inv(buf) + i * kBlock, base + lay.inv_lo(buf) + i * kBlock, ln);
        uint32_t dv[2][2], dh[2][2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 gv = gate_pair(gates, kGv, i * 16 + 8 * m + 2 * c), gn = gate_pair(gates, kGn, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float p, q;
                unpack2(fmul2(fmul2(pair(du[m], h), gv), pack2(back[h], back[h])), p, q);
                dv[m][h] = pack_bf16(p, q);
                dh[m][h] = pack_half(du[m][2 * h], du[m][2 * h + 1]);
                set_pair(x[m], h, fmul2(fmul2(pair(du[m], h), gn), pack2(-1.f, -1.f)));
            }
        }
        const uint32_t ds[4] = {dh[0][0], dh[0][1], dh[1][0], dh[1][1]};
        seen.see(ds);
        uint32_t ra[4], rl[4];   // - 2^e R
        pack_terms<TERMS>(x, ra, rl);
        seen.see(ra);
#pragma unroll
        for (int j = i - 1; j >= 0; --j) times_block<true, TERMS>(r[j], ra, rl, base + lay.n(buf) + block_of(i, j), base + lay.n_lo(buf) + block_of(i, j), ln);
        // A += (e^b dO)^T Q - (e^b R)^T K
        uint32_t pe[4], pel[4];
        float y[2][4];
        d_out(i, y);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 eb = gate_pair(gates, kEb, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                set_pair(x[m], h, fmul2(pair(x[m], h), eb));
                set_pair(y[m], h, fmul2(pair(y[m], h), eb));
            }
        }
        pack_terms<TERMS>(x, pe, pel);
        rows_into_state<DKP, TERMS>(A, pe, pel, kt, i, ln);
        pack_terms<TERMS>(y, pe, pel);
        rows_into_state<DKP, TERMS>(A, pe, pel, qt, i, ln);
        // out: dv, then 2^-e dU, through the strip's rows
        const int t = i * 16 + (lane >> 1), e = (lane & 1) * 8;
        const uint32_t at = vt + (i * 16 + ln.t_row) * kColPitch + ln.t_col * 2;
        const uint4* const piece = reinterpret_cast<const uint4*>(smem + cols + t * kColPitch + e * 2);
        stsm_trans(at, dv[0][0], dv[1][0], dv[0][1], dv[1][1]);
        __syncwarp();
        if (n * kChunk + t < a.L && col0 + e < a.dv) *reinterpret_cast<uint4*>(a.dv_out + a.row(unit, n * kChunk + t) * a.dv + col0 + e) = *piece;
        __syncwarp();
        stsm_trans(at, dh[0][0], dh[1][0], dh[0][1], dh[1][1]);
        __syncwarp();
        *reinterpret_cast<uint4*>(kept.du + ((unit * chunks + n) * kChunk + t) * kept.dvp + col0 + e) = *piece;
    }
}

// Whether two blocks share an SM: their shared memory must.  Each then has 128 registers a thread, of which the preparing warps leave the
// others 48 (128 x (176 + 80) = 256 x 128).
template <int DKP, bool EXACT, Way WAY>
constexpr bool two_blocks() { return 2 * (Layout<DKP, EXACT, WAY>::total(kMostWarps) + 1024) <= 228 * 1024; }

// EXACT: states leave the call in fp32, so that what they are made of is taken with 22 bits (two fp16 an operand); otherwise only bf16
// results do, and eleven bits keep the error below a quarter of their rounding.
template <int DKP, bool EXACT, Way WAY>
__global__ void __launch_bounds__(32 * kMostWarps + kPrep, two_blocks<DKP, EXACT, WAY>() ? 2 : 1) gdr_chunk_kernel(Gdr<bf> a, Kept kept, int slabs, int warps, int* status) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = 32 * warps + kPrep;
    const Layout<DKP, EXACT, WAY> lay;
    const long long unit = blockIdx.x / slabs;
    const int chunks = (a.L + kChunk - 1) / kChunk;
    pdl_wait();
    pdl_launch_dependents();
    if (warp >= kMostWarps) {
        if constexpr (two_blocks<DKP, EXACT, WAY>()) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        prepare_chunks<DKP, EXACT, WAY>(a, smem, lay, unit, chunks, threads);
        return;
    }
    if constexpr (two_blocks<DKP, EXACT, WAY>()) asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    if (warp >= warps) return;   // (four warps split their registers together)
    const int col0 = (blockIdx.x % slabs * warps + warp) * 16, g = lane >> 2, c = lane & 3;
    const Lane ln(lane);
    const uint32_t base = smem_u32(smem);
    const int cols0 = lay.cols + warp * 2 * lay.kCols;
    auto cols = [&](int buf) { return cols0 + buf * lay.kCols; };
    const bf* const from = WAY == Way::kBack ? a.d_out : a.v;
    auto fetch = [&](int n, int buf) {   // this warp's columns of the chunk's rows: two pieces of sixteen bytes a row
        const int e = (lane & 1) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = i * 16 + (lane >> 1);
            const bool in = n * kChunk + t < a.L && col0 + e < a.dv;
            cp_async16(base + cols(buf) + t * kColPitch + e * 2, from + (in ? a.row(unit, n * kChunk + t) * a.dv + col0 + e : 0), in);
        }
        cp_async_commit();
    };
    State<DKP> S;
    Largest seen;
    fetch(WAY == Way::kBack ? chunks - 1 : 0, 0);
    S.load(WAY == Way::kBack ? a.d_state_out : a.state_in, unit, a, col0 + g, c);
    for (int it = 0; it < chunks; ++it) {
        const int n = WAY == Way::kBack ? chunks - 1 - it : it, buf = it & 1, strips = (min(kChunk, a.L - n * kChunk) + 15) >> 4;
        if (it + 1 < chunks) {
            fetch(WAY == Way::kBack ? n - 1 : n + 1, buf ^ 1);
            cp_async_wait<1>();
        } else cp_async_wait<0>();
        __syncwarp();
        named_bar(kBarFull + buf, threads);
        auto chunk = [&](auto NS) {
            constexpr int ns = decltype(NS)::value;
            if constexpr (WAY == Way::kBack) backward_chunk<DKP, EXACT, ns>(S, seen, a, kept, smem, lay, buf, cols(buf), unit, n, chunks, col0, lane, ln);
            else forward_chunk<DKP, EXACT, WAY, ns>(S, seen, a, kept, smem, lay, buf, cols(buf), unit, n, chunks, col0, lane, ln);
        };
        if (strips == 4) chunk(std::integral_constant<int, 4>());
        else if (strips == 1) chunk(std::integral_constant<int, 1>());
        else if (strips == 2) chunk(std::integral_constant<int, 2>());
        else chunk(std::integral_constant<int, 3>());
        if (it + 2 < chunks) bar_arrive(kBarEmpty + buf, threads);
        __syncwarp();
    }
    const bool lost = __any_sync(0xffffffffu, seen.lost());
    if constexpr (WAY == Way::kForward) {
        if (lost) {   // (this warp's own stores of its columns come before)
            __syncwarp();
            if (lane == 0) atomicAdd(status + 1, 1);
            walk_sixteen<DKP>(a, unit, col0 + (lane & 15), lane >> 4);
        } else if (a.state_out) S.store(a.state_out, unit, a, col0 + g, c);
    } else {
        if (lane == 0) {
            int* const flag = kept.lost + unit * (kept.dvp / 16) + col0 / 16;
            *flag = WAY == Way::kKeep ? lost : lost || *flag;
        }
        if constexpr (WAY == Way::kKeep) {   // the last state, for the gates' gradient
            float none[2] = {0.f, 0.f}, back[2];
            uint32_t sa[DKP / 16][4];
            S.template rescale<3>(none, back);
#pragma unroll
            for (int s = 0; s < DKP / 16; ++s) pack_a(S.x[2 * s], S.x[2 * s + 1], sa[s]);
            kept.keep_state<DKP>(kept.S, kept.y, unit * (chunks + 1) + chunks, col0, sa, back, g, c);
        } else if (a.d_state_in) S.store(a.d_state_in, unit, a, col0 + g, c);
    }
}

// f(DKP)
template <typename F>
cudaError_t with_keys(int dk, F f) {
    if (dk <= 16) return f(std::integral_constant<int, 16>());
    if (dk <= 32) return f(std::integral_constant<int, 32>());
    if (dk <= 48) return f(std::integral_constant<int, 48>());
    if (dk <= 64) return f(std::integral_constant<int, 64>());
    if (dk <= 96) return f(std::integral_constant<int, 96>());
    return f(std::integral_constant<int, 128>());
}

template <Way WAY>
cudaError_t launch_chunks(const Gdr<bf>& a, const Kept& kept, bool exact, cudaStream_t stream) {
    int* status = device_status_ptr();
    if (!status) return cudaErrorUnknown;
    const int all = (a.dv + 15) / 16, slabs = (all + kMostWarps - 1) / kMostWarps, warps = (all + slabs - 1) / slabs;   // (gdr_padded_columns)
    return with_keys(a.dk, [&](auto D) {
        constexpr int dkp = decltype(D)::value;
        auto go = [&](auto E) {
            constexpr bool ex = decltype(E)::value;
            const int smem = Layout<dkp, ex, WAY>::total(warps);
            auto kernel = gdr_chunk_kernel<dkp, ex, WAY>;
            cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
            if (e != cudaSuccess) return e;
            count_launch();
            return launch_pdl(kernel, dim3((unsigned)(a.units * slabs)), dim3(32 * kMostWarps + kPrep), smem, stream, a, kept, slabs, warps, status);
        };
        if constexpr (WAY != Way::kKeep)
            if (exact) return go(std::true_type());
        return go(std::false_type());
    });
}

}  // namespace

bool gdr_chunk_supported(int dk, int dv) { return dk % 8 == 0 && dv % 8 == 0; }
int gdr_padded_columns(int dv) {
    const int all = (dv + 15) / 16, slabs = (all + kMostWarps - 1) / kMostWarps;
    return (all + slabs - 1) / slabs * slabs * 16;
}
int gdr_padded_keys(int dk) {
    int padded = 0;
    with_keys(dk, [&](auto D) { padded = decltype(D)::value; return cudaSuccess; });
    return padded;
}

cudaError_t launch_gdr_chunk_fwd(const Gdr<__nv_bfloat16>& a, cudaStream_t stream) {
    return launch_chunks<Way::kForward>(a, Kept{}, a.state_out != nullptr, stream);
}
cudaError_t launch_gdr_chunk_walks(const Gdr<__nv_bfloat16>& a, const GdrKept& kept, cudaStream_t stream) {
    cudaError_t e = launch_chunks<Way::kKeep>(a, kept, false, stream);
    return e == cudaSuccess ? launch_chunks<Way::kBack>(a, kept, a.d_state_in != nullptr, stream) : e;
}

namespace {

constexpr size_t kRepairBytes = 64u << 20;   // of scratch, unless one unit takes more

int repair_slots(long long units, int L, int dk, int dv) {
    const long long fit = (long long)(kRepairBytes / gdr_repair_slot_bytes(L, dk, dv));
    return (int)(fit < 1 ? 1 : fit > units ? units : fit > 148 ? 148 : fit);
}
size_t up(size_t n) { return (n + 255) / 256 * 256; }

Kept cut_kept(char* base, long long units, int L, int dk, int dv, size_t* total) {
    Kept k = {};
    const size_t chunks = (L + kChunk - 1) / kChunk, dvp = gdr_padded_columns(dv), dkp = gdr_padded_keys(dk);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? base + at : nullptr;
        at += up(bytes);
        return p;
    };
    k.dvp = (int)dvp;
    k.w = (__half*)take(units * chunks * kChunk * dvp * 2);
    k.du = (__half*)take(units * chunks * kChunk * dvp * 2);
    k.S = (__half*)take(units * (chunks + 1) * dvp * dkp * 2);
    k.A = (__half*)take(units * chunks * dvp * dkp * 2);
    k.y = (float*)take(units * (chunks + 1) * dvp * 4);
    k.z = (float*)take(units * chunks * dvp * 4);
    k.lost = (int*)take(units * (dvp / 16) * 4);
    k.lost_grad = (int*)take(units * chunks * 4);
    *total = at;
    return k;
}

}  // namespace

size_t gdr_grad_scratch_bytes(long long units, int L, int dk, int dv) {
    size_t kept;
    cut_kept(nullptr, units, L, dk, dv, &kept);
    return kept + repair_slots(units, L, dk, dv) * gdr_repair_slot_bytes(L, dk, dv);
}
cudaError_t launch_gdr_chunk_bwd(const Gdr<__nv_bfloat16>& a, void* scratch, cudaStream_t stream) {
    size_t used;
    const Kept kept = cut_kept((char*)scratch, a.units, a.L, a.dk, a.dv, &used);
    cudaError_t e = launch_gdr_chunk_walks(a, kept, stream);
    if (e == cudaSuccess) e = launch_gdr_grad(a, kept, stream);
    if (e == cudaSuccess)
        e = launch_gdr_repair(a, kept.lost, kept.dvp / 16, kept.lost_grad, (a.L + kChunk - 1) / kChunk, (char*)scratch + used,
                              repair_slots(a.units, a.L, a.dk, a.dv), stream);
    return e;
}

}  // namespace vig
