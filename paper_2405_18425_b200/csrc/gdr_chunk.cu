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
// buffers, handed over by named barriers.  64 x 12 units of 196 tokens, 32 x 64 (58 MB): 48 us, 0.19 of the rate of a copy, bound by instruction issue
// (8400 warp instructions a chunk, 430 of them products) and a chunk's chain with two blocks an SM.  (All warps doing both in turn: 70 us; 32 units of
// 4096 tokens, 24 x 48, 448 us, 7 us a chunk; now 86 in segments, 2.4 us a chunk.)
#include <type_traits>

#include "gdr.h"
#include "gdr_tile.cuh"

namespace vig {
namespace {

using namespace gdr;
using bf = __nv_bfloat16;

constexpr int kMostWarps = 4;       // with columns
constexpr int kMostColumns = 16;    // sixteens of dv
constexpr int kMostSegmentKeys = 64;   // key dimensions of sequences in segments
constexpr int kPrepWarps = 4;
constexpr int kPrep = 32 * kPrepWarps;
constexpr int kBlockPitch = 48, kBlock = 16 * kBlockPitch, kColPitch = 48;
// Token-by-token matrices are kept as their lower triangle of 16 x 16 blocks.
__device__ __forceinline__ int block_of(int i, int j) { return (i * (i + 1) / 2 + j) * kBlock; }
constexpr int kBarFull = 1, kBarEmpty = 3, kBarPrep = 5;   // named barriers: two of the first two

// The call's result; the gradient's forward walk, which keeps W and the states; its way back; and what a segment does to a state: where few
// units leave SMs idle a long sequence is cut into segments that run side by side.  A first launch takes every segment from zero states and, as
// further columns without values, from the unit vectors (S behind it = T S + B: both are columns of one loop), a small one (gdr_fold_kernel)
// carries the true states from segment to segment, and the launch proper starts every segment from its own.  Backwards T^T serves.
enum class Way { kForward, kKeep, kBack, kSum, kBackSum };
constexpr bool is_back(Way w) { return w == Way::kBack || w == Way::kBackSum; }

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
    static constexpr bool kQ = WAY == Way::kForward || is_back(WAY);   // queries, and P
    // of a buffer: keys, queries, N, P, inverses, gates, and what their first rounding left
    static constexpr int kQueries = kKeys, kN = kQueries + (kQ ? kKeys : 0), kP = kN + kMat, kInverse = kP + (kQ ? kMat : 0), kGates = kInverse + kInv,
                         kNLo = kGates + kChunk * kGateRows * 4, kPLo = kNLo + (EXACT ? kMat : 0),
                         kInvLo = kPLo + (EXACT && is_back(WAY) ? kMat : 0), kBuffer = kInvLo + (EXACT ? kInv : 0);
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

// Segments of a unit: chunks of one; fp32 [units][segs][dk][dv] states before (backwards: behind) each, what they add, and [units][segs][dk][dk].
struct Segs {
    int n, per, sums;   // segments, chunks of one, segments that the first launch takes (the last one's transition serves backwards only)
    float *in, *sum, *trans;
    int* lost;   // [units][slots]: something left the range of fp16; a slot for every segment and warp of columns
    int slots;
};

// What the gradient's walks leave for its last launch, per unit and chunk (see gdr.h).
using Kept = GdrKept;

__device__ __forceinline__ void bar_arrive(int id, int count) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(count) : "memory"); }

// ---- the preparing warps ----------------------------------------------------------------------------------------------
template <int DKP, bool EXACT, Way WAY>
__device__ void prepare_chunks(const Gdr<bf>& a, unsigned char* smem, const Layout<DKP, EXACT, WAY>& lay, long long unit, int first, int count, int threads) {
    constexpr int KP = key_pitch<DKP>(), KS = DKP / 16;
    constexpr bool Q = Layout<DKP, EXACT, WAY>::kQ;
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
            if (t0 + t < a.L && e8 < a.ldk) rows[p] = *reinterpret_cast<const uint4*>((r < kChunk ? a.k : a.q) + a.row(unit, t0 + t) * a.ldk + e8);
        }
        if (warp == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = t0 + 2 * lane + h;
                la[h] = t < a.L ? __bfloat162float(a.la[a.row(unit, t)]) : 0.f;
                be[h] = t < a.L ? __bfloat162float(a.beta[a.row(unit, t)]) : 0.f;
            }
    };
    bring(first);
    for (int it = 0; it < count; ++it) {
        const int n = is_back(WAY) ? first - it : first + it, buf = it & 1, strips = (min(kChunk, a.L - n * kChunk) + 15) >> 4;
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
        if (it + 1 < count) bring(is_back(WAY) ? n - 1 : n + 1);
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
                        if constexpr (Q) put(lay.p(buf), lay.p_lo(buf), EXACT && is_back(WAY), at, pack2(ss <= tt ? pp[m][2 * h] * e0 : 0.f, ss + 1 <= tt ? pp[m][2 * h + 1] * e1 : 0.f));
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
                        if constexpr (Q) put(lay.p(buf), lay.p_lo(buf), EXACT && is_back(WAY), at, fmul2(pair(pp[m], h), e));
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
            s = fmaf(__bfloat162float(a.k[r * a.ldk + 2 * i + half]), S[i], s);
        }
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        const float u = valid ? beta * (__bfloat162float(a.v[r * a.ldv + j]) - s) : 0.f;
#pragma unroll 1
        for (int i = 0; 2 * i + half < a.dk; ++i) {
            S[i] = fmaf(__bfloat162float(a.k[r * a.ldk + 2 * i + half]), u, S[i]);
            o = fmaf(__bfloat162float(a.q[r * a.ldk + 2 * i + half]), S[i], o);
        }
        o += __shfl_xor_sync(0xffffffffu, o, 16);
        if (valid && half == 0) a.out[r * a.ldv + j] = __float2bfloat16_rn(o);
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
    // [dk][cols] fp32 at `from` (null: zero)
    __device__ __forceinline__ void load(const float* from, int dk, int cols, int col, int c) {
#pragma unroll
        for (int n = 0; n < DKP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = n * 8 + 2 * c + (e & 1), j = col + (e >> 1) * 8;
                x[n][e] = from && i < dk && j < cols ? from[(long long)i * cols + j] : 0.f;
            }
    }
    __device__ __forceinline__ void unit_vectors(int col, int c) {
#pragma unroll
        for (int n = 0; n < DKP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = n * 8 + 2 * c + (e & 1) == col + (e >> 1) * 8 ? 1.f : 0.f;
    }
    __device__ __forceinline__ void store(float* to, int dk, int cols, int col, int c) const {
#pragma unroll
        for (int n = 0; n < DKP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = n * 8 + 2 * c + (e & 1), j = col + (e >> 1) * 8;
                if (i < dk && j < cols) to[(long long)i * cols + j] = x[n][e] / scale[e >> 1];
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
            const float now = __uint_as_float((253u + TOP - ex) << 23), change = fminf(now / scale[h], 0x1p126f);   // (more only where the state is nothing beside either)
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

// acc of every strip += state operand x the strip's rows of a key tile.  Strips inside, so that a product never waits for the one before it.
template <int DKP, int TERMS, int NS>
__device__ __forceinline__ void state_times_rows(float (&acc)[NS][2][4], const uint32_t (&hi)[4], const uint32_t (&lo)[4], uint32_t tile, int s, const Lane& ln) {
    uint32_t x[NS][4];
#pragma unroll
    for (int i = 0; i < NS; ++i) ldsm(at_b<key_pitch<DKP>()>(ln, tile, i * 16, s * 16), x[i]);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        mma(acc[i][0], hi, x[i][0], x[i][1]);
        mma(acc[i][1], hi, x[i][2], x[i][3]);
    }
    if constexpr (TERMS == 2)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            mma(acc[i][0], lo, x[i][0], x[i][1]);
            mma(acc[i][1], lo, x[i][2], x[i][3]);
        }
}
// S += (sixteen tokens' operand) x their rows of a key tile
template <int DKP, int TERMS>
__device__ __forceinline__ void rows_into_state(State<DKP>& S, const uint32_t (&hi)[4], const uint32_t (&lo)[4], uint32_t tile, int strip, const Lane& ln) {
    constexpr int KS = DKP / 16, AT = KS % 4 == 0 ? 4 : KS % 2 == 0 ? 2 : 1;   // sixteens of keys at a time
#pragma unroll
    for (int s0 = 0; s0 < KS; s0 += AT) {
        uint32_t y[AT][4];
#pragma unroll
        for (int s = 0; s < AT; ++s) ldsm_trans(at_t<key_pitch<DKP>()>(ln, tile, strip * 16, (s0 + s) * 16), y[s]);
#pragma unroll
        for (int s = 0; s < AT; ++s) {
            mma(S.x[2 * (s0 + s)], hi, y[s][0], y[s][1]);
            mma(S.x[2 * (s0 + s) + 1], hi, y[s][2], y[s][3]);
        }
        if constexpr (TERMS == 2)
#pragma unroll
            for (int s = 0; s < AT; ++s) {
                mma(S.x[2 * (s0 + s)], lo, y[s][0], y[s][1]);
                mma(S.x[2 * (s0 + s) + 1], lo, y[s][2], y[s][3]);
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
    constexpr bool OUT = WAY == Way::kForward, KEEP = WAY == Way::kKeep;
    const int g = lane >> 2, c = lane & 3;
    const uint32_t base = smem_u32(smem), kt = base + lay.k(buf), qt = base + lay.q(buf), vt = base + cols;
    const float* const gates = reinterpret_cast<const float*>(smem + lay.gates(buf));
    float gmax = fmaxf(fabsf(gates[kGv * kChunk + lane]), fabsf(gates[kGv * kChunk + lane + 32])), vmax[2] = {0.f, 0.f}, back[2];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, o));
    if constexpr (KEEP) gmax = fmaxf(gmax, 1.f);   // W itself is kept too
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
    if constexpr (KEEP) kept.keep_state<DKP>(kept.S, kept.y, unit * (chunks + 1) + n, col0, sa, back, g, c, n > 0 || a.state_in);
    S.decay(gates[kEb * kChunk + kChunk - 1]);
    // products with S, of all strips; then strip by strip, what a strip's U means to the strips behind it as soon as it is there: the next
    // strip's chain (N, the step, the inverse) is what bounds a chunk, all else fills its gaps
    float w[NS][2][4] = {}, o[NS][2][4] = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        state_times_rows<DKP, TERMS, NS>(w, sa[s], sl[EXACT ? s : 0], kt, s, ln);
        if constexpr (OUT) state_times_rows<DKP, 1, NS>(o, sa[s], sa[s], qt, s, ln);
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
                if constexpr (KEEP) set_pair(w[i][m], h, y);
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
        uint32_t res[2][2] = {};
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
        } else if constexpr (KEEP) {   // W of the strip: what its own block takes off
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
        if constexpr (!OUT && !KEEP) continue;
        // over the strip's values, and out from there in pieces of sixteen bytes
        stsm_trans(vt + (i * 16 + ln.t_row) * kColPitch + ln.t_col * 2, res[0][0], res[1][0], res[0][1], res[1][1]);
        __syncwarp();
        const int t = i * 16 + (lane >> 1), e = (lane & 1) * 8;
        const uint4 piece = *reinterpret_cast<const uint4*>(smem + cols + t * kColPitch + e * 2);
        if constexpr (OUT) {
            if (n * kChunk + t < a.L && col0 + e < a.ldv) *reinterpret_cast<uint4*>(a.out + a.row(unit, n * kChunk + t) * a.ldv + col0 + e) = piece;
        } else *reinterpret_cast<uint4*>(kept.w + ((unit * chunks + n) * kChunk + t) * kept.dvp + col0 + e) = piece;
    }
}

// One chunk of NS strips backwards: S is A, the columns are those of dO.
template <int DKP, bool EXACT, Way WAY, int NS>
__device__ __forceinline__ void backward_chunk(State<DKP>& A, Largest& seen, const Gdr<bf>& a, const Kept& kept, unsigned char* smem,
                                               const Layout<DKP, EXACT, WAY>& lay, int buf, int cols, long long unit, int n, int chunks, int col0,
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
    if constexpr (WAY == Way::kBack) kept.keep_state<DKP>(kept.A, kept.z, unit * chunks + n, col0, aa, back, g, c, n + 1 < chunks || a.d_state_out);
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
    for (int s = 0; s < KS; ++s) state_times_rows<DKP, TERMS, NS>(r, aa[s], al[EXACT ? s : 0], kt, s, ln);
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
        if constexpr (WAY != Way::kBack) continue;
        // out: dv, then 2^-e dU, through the strip's rows
        const int t = i * 16 + (lane >> 1), e = (lane & 1) * 8;
        const uint32_t at = vt + (i * 16 + ln.t_row) * kColPitch + ln.t_col * 2;
        const uint4* const piece = reinterpret_cast<const uint4*>(smem + cols + t * kColPitch + e * 2);
        stsm_trans(at, dv[0][0], dv[1][0], dv[0][1], dv[1][1]);
        __syncwarp();
        if (n * kChunk + t < a.L && col0 + e < a.ldv) *reinterpret_cast<uint4*>(a.dv_out + a.row(unit, n * kChunk + t) * a.ldv + col0 + e) = *piece;
        __syncwarp();
        stsm_trans(at, dh[0][0], dh[1][0], dh[0][1], dh[1][1]);
        __syncwarp();
        *reinterpret_cast<uint4*>(kept.du + ((unit * chunks + n) * kChunk + t) * kept.dvp + col0 + e) = *piece;
    }
}

// Whether two blocks share an SM: their shared memory must.  Each then has 128 registers a thread.  (Unequal shares, 80 to 104 for the preparing
// warps and 176 to 152 for the others: 53 to 47 us for 64 x 12 units of 196 tokens, 32 x 64, against 46.)
template <int DKP, bool EXACT, Way WAY>
constexpr bool two_blocks() { return 2 * (Layout<DKP, EXACT, WAY>::total(kMostWarps) + 1024) <= 228 * 1024; }

// EXACT: states leave the call in fp32, so that what they are made of is taken with 22 bits (two fp16 an operand); otherwise only bf16
// results do, and eleven bits keep the error below a quarter of their rounding.
template <int DKP, bool EXACT, Way WAY>
__global__ void __launch_bounds__(32 * kMostWarps + kPrep, two_blocks<DKP, EXACT, WAY>() ? 2 : 1) gdr_chunk_kernel(Gdr<bf> a, Kept kept, Segs segs, int slabs, int warps, int* status) {
    constexpr bool BACK = is_back(WAY), PROPER = WAY != Way::kSum && WAY != Way::kBackSum;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = 32 * warps + kPrep;
    const Layout<DKP, EXACT, WAY> lay;
    // sums have further slabs for the unit vectors, backwards none, and leave out the first segment
    const int all = slabs + (WAY == Way::kSum ? (a.dk + warps * 16 - 1) / (warps * 16) : 0), runs = WAY == Way::kSum ? segs.sums : WAY == Way::kBackSum ? segs.n - 1 : segs.n;
    const int slab = blockIdx.x % all, seg = blockIdx.x / all % runs + (WAY == Way::kBackSum);
    const long long unit = blockIdx.x / all / runs;
    const int chunks = (a.L + kChunk - 1) / kChunk, from = seg * segs.per, to = min(chunks, from + segs.per), first = BACK ? to - 1 : from, count = to - from;
    const bool starts = seg == (BACK ? segs.n - 1 : 0), ends = seg == (BACK ? 0 : segs.n - 1);
    pdl_wait();
    pdl_launch_dependents();
    if (warp >= warps) {
        prepare_chunks<DKP, EXACT, WAY>(a, smem, lay, unit, first, count, threads);
        return;
    }
    const bool vectors = WAY == Way::kSum && slab >= slabs;   // columns that are unit vectors
    const int col0 = ((vectors ? slab - slabs : slab) * warps + warp) * 16, g = lane >> 2, c = lane & 3;
    const Lane ln(lane);
    const uint32_t base = smem_u32(smem);
    const int cols0 = lay.cols + warp * 2 * lay.kCols;
    auto cols = [&](int buf) { return cols0 + buf * lay.kCols; };
    const bf* const rows = BACK ? a.d_out : a.v;
    auto fetch = [&](int n, int buf) {   // this warp's columns of the chunk's rows: two pieces of sixteen bytes a row
        const int e = (lane & 1) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = i * 16 + (lane >> 1);
            const bool in = n * kChunk + t < a.L && col0 + e < a.ldv && !vectors;
            cp_async16(base + cols(buf) + t * kColPitch + e * 2, rows + (in ? a.row(unit, n * kChunk + t) * a.ldv + col0 + e : 0), in);
        }
        cp_async_commit();
    };
    const long long plane = (long long)a.dk * a.dv, at = unit * segs.n + seg;
    State<DKP> S;
    Largest seen;
    fetch(first, 0);
    if (vectors) S.unit_vectors(col0 + g, c);
    else {
        const float* const edge = BACK ? a.d_state_out : a.state_in;
        S.load(!PROPER ? nullptr : !starts ? segs.in + at * plane : edge ? edge + unit * plane : nullptr, a.dk, a.dv, col0 + g, c);
    }
    for (int it = 0; it < count; ++it) {
        const int n = BACK ? first - it : first + it, buf = it & 1, strips = (min(kChunk, a.L - n * kChunk) + 15) >> 4;
        if (it + 1 < count) {
            fetch(BACK ? n - 1 : n + 1, buf ^ 1);
            cp_async_wait<1>();
        } else cp_async_wait<0>();
        __syncwarp();
        named_bar(kBarFull + buf, threads);
        auto chunk = [&](auto NS) {
            constexpr int ns = decltype(NS)::value;
            if constexpr (BACK) backward_chunk<DKP, EXACT, WAY, ns>(S, seen, a, kept, smem, lay, buf, cols(buf), unit, n, chunks, col0, lane, ln);
            else forward_chunk<DKP, EXACT, WAY, ns>(S, seen, a, kept, smem, lay, buf, cols(buf), unit, n, chunks, col0, lane, ln);
        };
        if (strips == 4) chunk(std::integral_constant<int, 4>());
        else if (strips == 1) chunk(std::integral_constant<int, 1>());
        else if (strips == 2) chunk(std::integral_constant<int, 2>());
        else chunk(std::integral_constant<int, 3>());
        if (it + 2 < count) bar_arrive(kBarEmpty + buf, threads);
        __syncwarp();
    }
    const bool lost = __any_sync(0xffffffffu, seen.lost());
    if constexpr (WAY == Way::kForward) {
        if (segs.n == 1) {
            if (lost) {   // (this warp's own stores of its columns come before)
                __syncwarp();
                if (lane == 0) atomicAdd(status + 1, 1);
                walk_sixteen<DKP>(a, unit, col0 + (lane & 15), lane >> 4);
                return;
            }
        } else if (lost && lane == 0) segs.lost[unit * segs.slots + seg * kMostColumns + col0 / 16] = 1;
        if (a.state_out && ends) S.store(a.state_out + unit * plane, a.dk, a.dv, col0 + g, c);
    } else if constexpr (PROPER) {
        if (lane == 0) {
            int* const flag = segs.lost + unit * segs.slots + seg * kMostColumns + col0 / 16;
            if (WAY == Way::kKeep) *flag = lost;
            else if (lost) *flag = 1;
        }
        if constexpr (WAY == Way::kKeep) {   // the last state, for the gates' gradient
            if (ends && a.d_state_out) {
                float none[2] = {0.f, 0.f}, back[2];
                uint32_t sa[DKP / 16][4];
                S.template rescale<3>(none, back);
#pragma unroll
                for (int s = 0; s < DKP / 16; ++s) pack_a(S.x[2 * s], S.x[2 * s + 1], sa[s]);
                kept.keep_state<DKP>(kept.S, kept.y, unit * (chunks + 1) + chunks, col0, sa, back, g, c, true);
            }
        } else if (a.d_state_in && ends) S.store(a.d_state_in + unit * plane, a.dk, a.dv, col0 + g, c);
    } else {
        if (lost && lane == 0) segs.lost[unit * segs.slots + segs.n * kMostColumns] = 1;   // (whichever warp of the unit's)
        if (vectors) S.store(segs.trans + at * a.dk * a.dk, a.dk, a.dk, col0 + g, c);
        else S.store(segs.sum + at * plane, a.dk, a.dv, col0 + g, c);
    }
}

// The states between segments: a block takes sixteen columns of a unit.  S before the next = T S + B, backwards A behind the last = T^T A + C,
// in fp32; transitions and sums come by asynchronous copies a segment ahead.
__global__ void __launch_bounds__(256) gdr_fold_kernel(Gdr<bf> a, Segs segs, int slabs, bool back) {
    extern __shared__ __align__(16) float fold_smem[];
    const int dk = a.dk, pitch = dk + 4, tid = threadIdx.x, j0 = blockIdx.x % slabs * 16, mine = min(16, a.dv - j0);   // (dk, dv: multiples of eight)
    const long long unit = blockIdx.x / slabs, plane = (long long)dk * a.dv;
    const int size = dk * pitch + dk * 16;
    float* const X = fold_smem + 2 * size;   // [dk][16]
    const uint32_t base = smem_u32(fold_smem);
    auto segment = [&](int k) { return unit * segs.n + (back ? segs.n - 1 - k : k); };
    auto fetch = [&](int k) {   // [dk][pitch] transition, [dk][16] sum
        const uint32_t to = base + (k & 1) * size * 4;
        const float* const t = segs.trans + segment(k) * dk * dk;
        const int pieces = dk / 4;
        for (int i = tid; i < dk * pieces; i += 256) {
            const int r = i / pieces, p = i - r * pieces;
            cp_async16(to + (r * pitch + p * 4) * 4, t + i * 4, true);
        }
        for (int i = tid; i < dk * 4; i += 256) {
            const int r = i >> 2, p = (i & 3) * 4;
            cp_async16(to + (dk * pitch + r * 16 + p) * 4, segs.sum + segment(k) * plane + (p < mine ? (long long)r * a.dv + j0 + p : 0), p < mine);
        }
        cp_async_commit();
    };
    pdl_wait();
    pdl_launch_dependents();
    fetch(0);
    const float* const edge = back ? a.d_state_out : a.state_in;
    for (int i = tid; i < dk * 16; i += 256) X[i] = edge && (i & 15) < mine ? edge[unit * plane + (long long)(i >> 4) * a.dv + j0 + (i & 15)] : 0.f;
    for (int k = 0; k + 1 < segs.n; ++k) {
        if (k + 2 < segs.n) {
            fetch(k + 1);
            cp_async_wait<1>();
        } else cp_async_wait<0>();
        __syncthreads();
        const float *const T = fold_smem + (k & 1) * size, *const B = T + dk * pitch;
        const long long next = segment(k + 1);
        // row tid / 4, four columns; rows of 64 and more a second time
        float4 y[2];
        const int c0 = (tid & 3) * 4;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = (tid >> 2) + 64 * h;
            if (r >= dk) break;
            y[h] = *reinterpret_cast<const float4*>(B + r * 16 + c0);
#pragma unroll 4
            for (int i = 0; i < dk; ++i) {
                const float t = back ? T[i * pitch + r] : T[r * pitch + i];
                const float4 u = *reinterpret_cast<const float4*>(X + i * 16 + c0);
                y[h].x = fmaf(t, u.x, y[h].x); y[h].y = fmaf(t, u.y, y[h].y); y[h].z = fmaf(t, u.z, y[h].z); y[h].w = fmaf(t, u.w, y[h].w);
            }
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = (tid >> 2) + 64 * h;
            if (r >= dk) break;
            *reinterpret_cast<float4*>(X + r * 16 + c0) = y[h];
            if (c0 < mine) *reinterpret_cast<float4*>(segs.in + next * plane + (long long)r * a.dv + j0 + c0) = y[h];
        }
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
cudaError_t launch_chunks(const Gdr<bf>& a, const Kept& kept, const Segs& segs, bool exact, cudaStream_t stream) {
    int* status = device_status_ptr();
    if (!status) return cudaErrorUnknown;
    const int sixteens = gdr_padded_columns(a.dv) / 16;
    const int slabs = (sixteens + kMostWarps - 1) / kMostWarps, warps = sixteens / slabs;   // (narrower blocks for few units: 332 -> 414 us for 2 x 16 x 4096, 128 x 128)
    const long long blocks = a.units * (WAY == Way::kSum ? segs.sums : WAY == Way::kBackSum ? segs.n - 1 : segs.n) * (slabs + (WAY == Way::kSum ? (a.dk + warps * 16 - 1) / (warps * 16) : 0));
    return with_keys(a.dk, [&](auto D) {
        constexpr int dkp = decltype(D)::value;
        auto go = [&](auto E) {
            constexpr bool ex = decltype(E)::value;
            const int smem = Layout<dkp, ex, WAY>::total(warps);
            cudaError_t e = allow_smem<gdr_chunk_kernel<dkp, ex, WAY>>(Layout<dkp, ex, WAY>::total(kMostWarps));
            if (e != cudaSuccess) return e;
            count_launch();
            return launch_pdl(gdr_chunk_kernel<dkp, ex, WAY>, dim3((unsigned)blocks), dim3(32 * warps + kPrep), smem, stream, a, kept, segs, slabs, warps, status);
        };
        if constexpr (WAY != Way::kKeep)
            if (exact) return go(std::true_type());
        return go(std::false_type());
    });
}

cudaError_t launch_fold(const Gdr<bf>& a, const Segs& segs, bool back, cudaStream_t stream) {
    const int slabs = (a.dv + 15) / 16;
    auto bytes = [](int dk) { return ((size_t)2 * (dk * (dk + 4) + dk * 16) + dk * 16) * 4; };
    const size_t smem = bytes(a.dk);
    cudaError_t e = allow_smem<gdr_fold_kernel>(bytes(kMostSegmentKeys));
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(gdr_fold_kernel, dim3((unsigned)(a.units * slabs)), dim3(256), smem, stream, a, segs, slabs, back);
}

// Segments of a unit: as many as let the blocks of the launch proper run at once (two an SM), of four chunks and more, from three segments on:
// below, what the first launch adds is what the second saves.  (A block's time is its chunks' in a row, whether or not another shares its SM:
// 32 units of 4096 tokens, 24 x 48, 8 segments 49 + 39 us for the two launches, 5 segments, with which the first fits the chip too, 40 + 57.)
int segments(long long units, int L, int dk, int dv) {
    if (dk % 8 || dv % 8) return 1;   // (the states' copies between segments are whole pieces of sixteen bytes)
    if (dk > kMostSegmentKeys) return 1;   // (one block an SM, and as many columns for the transition as for the state: 2 x 16 units of 4096 tokens, 128 x 128, gain nothing)
    const long long blocks = units * ((dv + 16 * kMostWarps - 1) / (16 * kMostWarps)), chunks = (L + kChunk - 1) / kChunk;
    const long long fit = 2LL * 148 / blocks, n = fit < chunks / 4 ? fit : chunks / 4;
    return n < 3 ? 1 : (int)(n < 32 ? n : 32);
}
size_t up(size_t n) { return (n + 255) / 256 * 256; }

Segs cut_segments(char* base, long long units, int L, int dk, int dv, int n, bool back, size_t* total) {
    Segs s = {};
    const int chunks = (L + kChunk - 1) / kChunk;
    s.per = (chunks + n - 1) / n;
    s.n = (chunks + s.per - 1) / s.per;
    s.sums = back ? s.n : s.n - 1;
    s.slots = s.n > 1 ? s.n * kMostColumns + 1 : gdr_padded_columns(dv) / 16;   // (one segment: all of them are written)
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? base + at : nullptr;
        at += up(bytes);
        return p;
    };
    s.lost = (int*)take(units * s.slots * 4);
    if (s.n > 1) {
        s.in = (float*)take((size_t)units * s.n * dk * dv * 4);
        s.sum = (float*)take((size_t)units * s.n * dk * dv * 4);
        s.trans = (float*)take((size_t)units * s.n * dk * dk * 4);
    }
    *total = at;
    return s;
}

constexpr size_t kRepairBytes = 64u << 20;   // of scratch, unless one unit takes more

int repair_slots(long long units, int L, int dk, int dv) {
    const long long fit = (long long)(kRepairBytes / gdr_repair_slot_bytes(L, dk, dv));
    return (int)(fit < 1 ? 1 : fit > units ? units : fit > 148 ? 148 : fit);
}

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
    k.lost_grad = (int*)take(units * chunks * 4);
    *total = at;
    return k;
}

}  // namespace

int gdr_padded_columns(int dv) {
    const int all = (dv + 15) / 16, slabs = (all + kMostWarps - 1) / kMostWarps;
    return (all + slabs - 1) / slabs * slabs * 16;
}
int gdr_padded_keys(int dk) {
    int padded = 0;
    with_keys(dk, [&](auto D) { padded = decltype(D)::value; return cudaSuccess; });
    return padded;
}

size_t gdr_chunk_scratch_bytes(long long units, int L, int dk, int dv) {
    const int n = segments(units, L, dk, dv);
    size_t total = 0;
    if (n > 1) cut_segments(nullptr, units, L, dk, dv, n, false, &total);
    return total;
}
cudaError_t launch_gdr_chunk_fwd(const Gdr<__nv_bfloat16>& a, void* scratch, cudaStream_t stream) {
    const bool exact = a.state_out != nullptr;
    const int n = segments(a.units, a.L, a.dk, a.dv);
    if (n == 1) {
        Segs one = {};
        one.n = 1;
        one.per = (a.L + kChunk - 1) / kChunk;
        return launch_chunks<Way::kForward>(a, Kept{}, one, exact, stream);
    }
    size_t total;
    const Segs segs = cut_segments((char*)scratch, a.units, a.L, a.dk, a.dv, n, false, &total);
    cudaError_t e = cudaMemsetAsync(segs.lost, 0, a.units * segs.slots * 4, stream);
    if (e == cudaSuccess) e = launch_chunks<Way::kSum>(a, Kept{}, segs, exact, stream);
    if (e == cudaSuccess) e = launch_fold(a, segs, false, stream);
    if (e == cudaSuccess) e = launch_chunks<Way::kForward>(a, Kept{}, segs, exact, stream);
    if (e == cudaSuccess) e = launch_gdr_repair_fwd(a, segs.lost, segs.slots, stream);
    return e;
}

size_t gdr_grad_scratch_bytes(long long units, int L, int dk, int dv) {
    size_t kept, segs;
    cut_kept(nullptr, units, L, dk, dv, &kept);
    cut_segments(nullptr, units, L, dk, dv, segments(units, L, dk, dv), true, &segs);
    return kept + segs + repair_slots(units, L, dk, dv) * gdr_repair_slot_bytes(L, dk, dv);
}
cudaError_t launch_gdr_chunk_bwd(const Gdr<__nv_bfloat16>& a, void* scratch, cudaStream_t stream) {
    size_t used, more;
    const Kept kept = cut_kept((char*)scratch, a.units, a.L, a.dk, a.dv, &used);
    const Segs segs = cut_segments((char*)scratch + used, a.units, a.L, a.dk, a.dv, segments(a.units, a.L, a.dk, a.dv), true, &more);
    const bool exact = a.d_state_in != nullptr;
    cudaError_t e = cudaSuccess;
    if (segs.n > 1) {
        e = cudaMemsetAsync(segs.lost, 0, a.units * segs.slots * 4, stream);
        if (e == cudaSuccess) e = launch_chunks<Way::kSum>(a, kept, segs, exact, stream);
        if (e == cudaSuccess) e = launch_fold(a, segs, false, stream);
    }
    if (e == cudaSuccess) e = launch_chunks<Way::kKeep>(a, kept, segs, false, stream);
    if (segs.n > 1) {
        if (e == cudaSuccess) e = launch_chunks<Way::kBackSum>(a, kept, segs, exact, stream);
        if (e == cudaSuccess) e = launch_fold(a, segs, true, stream);
    }
    if (e == cudaSuccess) e = launch_chunks<Way::kBack>(a, kept, segs, exact, stream);
    if (e == cudaSuccess) e = launch_gdr_grad(a, kept, stream);
    if (e == cudaSuccess)
        e = launch_gdr_repair(a, segs.lost, segs.slots, kept.lost_grad, (a.L + kChunk - 1) / kChunk, (char*)scratch + used + more,
                              repair_slots(a.units, a.L, a.dk, a.dv), stream);
    return e;
}

}  // namespace vig
