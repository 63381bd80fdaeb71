// The gated delta rule in chunks of 64 tokens on the tensor cores (bf16 calls): what goes from chunk to chunk.
//
// With b the running sum of log alpha in a chunk, Gam_ts = e^{b_t - b_s}, N = strict_tril(K K^T . Gam), P = tril(Q K^T . Gam):
//   forwards    W = V - e^b K S - N U, U = beta W       O = e^b Q S + P U        S <- e^{b_C} S + (e^{b_C - b} K)^T U
//   backwards   dU = P^T dO + e^{b_C - b} K A - N^T R, R = beta dU (= dV)        A <- e^{b_C} A + (e^b Q)^T dO - (e^b K)^T R
// The triangular systems are solved sixteen tokens at a time: what the other sixteens contribute is a product with N, what the sixteen do to
// one another a product with the inverse of 1 + beta N of their own 16 x 16 block, which one warp computes by substitution in fp32.
// e^{b_t - b_s} is taken of the difference, never of its parts, so that no gate is out of range.
//
// A block runs through the chunks of a unit for up to 64 columns.  Four of its warps prepare: they bring the rows of K and Q and make N, P and the
// inverses of the next chunk while the others, a warp for every sixteen columns (gdr_tile.cuh), work on this one.  Two buffers, handed over by
// named barriers.  64 x 12 units of 196 tokens, 32 x 64 (58 MB): 56 us, 0.16 of the rate of a copy, bound by instruction issue and a chunk's chain with two
// blocks an SM.  (One term of fp16 an operand under powers of two: 50 us, but see gdr_tile.cuh.  32 units of 4096 tokens, 24 x 48, without segments 448 us,
// 7 us a chunk.)
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
//   b, bl running sum of log2 alpha (two floats); eb 2^b; dl 2^{b_C - b}; beta; and of the whole chunk the largest of K and of Q that each preparing warp met (at 0 and
//   4), and of beta (at 8)
enum { kB, kBl, kEb, kDl, kBeta, kMost, kGateRows };
__device__ __forceinline__ f32x2 gate_pair(const float* gates, int row, int t) { return *reinterpret_cast<const f32x2*>(gates + row * kChunk + t); }

// Terms of what is computed: states that leave the call in fp32 are made of three, bf16 results of two.
template <bool EXACT>
constexpr int terms() { return EXACT ? 3 : 2; }

// Shared memory, in bytes.
template <int DKP, bool EXACT, Way WAY>
struct Layout {
    static constexpr int kKeys = kChunk * key_pitch<DKP>(), kMat = 10 * kBlock, kInv = 4 * kBlock, kCols = kChunk * 32;
    static constexpr bool kQ = WAY == Way::kForward || is_back(WAY);   // queries, and P
    static constexpr int kTerms = terms<EXACT>(), kPTerms = is_back(WAY) ? kTerms : 2;   // (forwards P makes bf16 results only)
    // of a buffer: keys, queries, the terms of N, P and the inverses, gates
    static constexpr int kQueries = kKeys, kN = kQueries + (kQ ? kKeys : 0), kP = kN + kTerms * kMat, kInverse = kP + (kQ ? kPTerms * kMat : 0),
                         kGates = kInverse + kTerms * kInv, kBuffer = kGates + kChunk * kGateRows * 4;
    static constexpr int x = 2 * kBuffer;                  // the diagonal blocks of beta N, transposed, rows of 20 floats
    static constexpr int cols = x + 4 * 16 * 20 * 4;       // a warp's columns of V or dO, two chunks
    static constexpr int k(int buf) { return buf * kBuffer; }
    static constexpr int q(int buf) { return buf * kBuffer + kQueries; }
    static constexpr int n(int buf) { return buf * kBuffer + kN; }
    static constexpr int p(int buf) { return buf * kBuffer + kP; }
    static constexpr int inv(int buf) { return buf * kBuffer + kInverse; }
    static constexpr int gates(int buf) { return buf * kBuffer + kGates; }
    static constexpr int total(int warps) { return cols + 2 * warps * kCols; }
};

// Segments of a unit: chunks of one; fp32 [units][segs][dk][dv] states before (backwards: behind) each, what they add, and [units][segs][dk][dk].
struct Segs {
    int n, per, sums;   // segments, chunks of one, segments that the first launch takes (the last one's transition serves backwards only)
    float *in, *sum, *trans;
    int* lost;   // [units][slots]: something grew beyond the loop's digits or is not finite; a slot for every segment and warp of columns
    int slots;
};

// What the gradient's walks leave for its last launch, per unit and chunk (see gdr.h).
using Kept = GdrKept;

__device__ __forceinline__ void bar_arrive(int id, int count) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(count) : "memory"); }

// ---- the preparing warps ----------------------------------------------------------------------------------------------
template <int DKP, bool EXACT, Way WAY>
__device__ void prepare_chunks(const Gdr<bf>& a, unsigned char* smem, const Layout<DKP, EXACT, WAY>& lay, long long unit, int first, int count, int threads) {
    using Lay = Layout<DKP, EXACT, WAY>;
    constexpr int KP = key_pitch<DKP>(), KS = DKP / 16, TERMS = Lay::kTerms, PT = Lay::kPTerms;
    constexpr bool Q = Lay::kQ;
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
            Sum b[2], all;
            gate_sums(la, b, all);
            float step = fmaxf(fabsf(be[0]), fabsf(be[1]));
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) step = fmaxf(step, __shfl_xor_sync(0xffffffffu, step, o));
            auto two = [&](int row, float x, float y) { *reinterpret_cast<float2*>(gates + row * kChunk + 2 * lane) = make_float2(x, y); };
            two(kB, b[0].h, b[1].h);
            two(kBl, b[0].l, b[1].l);
            two(kEb, ex2(b[0].h + b[0].l), ex2(b[1].h + b[1].l));
            two(kDl, ex2(all.to(b[0])), ex2(all.to(b[1])));
            two(kBeta, be[0], be[1]);
            if (lane == 0) gates[kMost * kChunk + 8] = step;
        }
        // K and Q as they come, and the largest of each
        uint32_t most[2] = {0u, 0u};
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int r = p * kRows + r0, t = r & (kChunk - 1);
            larger(most[p * kRows >= kChunk], rows[p]);
            if (e8 < DKP) *reinterpret_cast<uint4*>(smem + (r < kChunk ? lay.k(buf) : lay.q(buf)) + t * KP + e8 * 2) = rows[p];
        }
#pragma unroll
        for (int m = 0; m < (Q ? 2 : 1); ++m) {
            float x = largest_of(most[m]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            if (lane == 0) gates[kMost * kChunk + 4 * m + warp] = x;
        }
        named_bar(kBarPrep, kPrep);
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
        auto put = [&](auto N, int matrix, int at, f32x2 x) {   // its terms, a matrix each
            constexpr int kN = decltype(N)::value;
            uint32_t t[kN];
            split<kN>(x, t);
#pragma unroll
            for (int m = 0; m < kN; ++m) *reinterpret_cast<uint32_t*>(smem + matrix + m * Lay::kMat + at) = t[m];
        };
        auto sum_at = [&](int t) { return Sum{gates[kB * kChunk + t], gates[kBl * kChunk + t]}; };
        auto sums_at = [&](int t, Sum& x, Sum& y) {   // of two neighbours
            const float2 h = *reinterpret_cast<const float2*>(gates + kB * kChunk + t), l = *reinterpret_cast<const float2*>(gates + kBl * kChunk + t);
            x = {h.x, l.x};
            y = {h.y, l.y};
        };
        const std::integral_constant<int, TERMS> terms_n;
        const std::integral_constant<int, PT> terms_p;
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
                    const Sum bt = sum_at(t);
                    const float beta = gates[kBeta * kChunk + t];
#pragma unroll
                    for (int m = 0; m < 2; ++m) {   // columns 8m + 2c, + 1
                        const int ss = 8 * m + 2 * c, at = block_of(i, i) + in_block(tt, m) + 4 * c;
                        Sum b0, b1;
                        sums_at(i * 16 + ss, b0, b1);
                        const float e0 = ss <= tt ? ex2(bt.to(b0)) : 0.f, e1 = ss + 1 <= tt ? ex2(bt.to(b1)) : 0.f;
                        // (selected, not multiplied: what is not finite stays out of earlier tokens)
                        if constexpr (Q) put(terms_p, lay.p(buf), at, pack2(ss <= tt ? pp[m][2 * h] * e0 : 0.f, ss + 1 <= tt ? pp[m][2 * h + 1] * e1 : 0.f));
                        const float n0 = ss < tt ? nn[m][2 * h] * e0 : 0.f, n1 = ss + 1 < tt ? nn[m][2 * h + 1] * e1 : 0.f;
                        if constexpr (WAY == Way::kKeep) put(terms_n, lay.n(buf), at, pack2(n0, n1));   // (W takes its own strip's off)
                        xt[(d * 16 + ss) * 20 + tt] = n0 * beta;   // beta N, transposed: row s, column t
                        xt[(d * 16 + ss + 1) * 20 + tt] = n1 * beta;
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
                for (int t = 0; t < 16; t += 2) {
                    uint32_t y[TERMS];
                    split<TERMS>(pack2(x[t], x[t + 1]), y);
#pragma unroll
                    for (int m = 0; m < TERMS; ++m) {
                        unsigned char* const at = smem + lay.inv(buf) + m * Lay::kInv + i * kBlock + (cc & 7) * 2;
                        *reinterpret_cast<unsigned short*>(at + in_block(t, cc >> 3)) = (unsigned short)y[m];
                        *reinterpret_cast<unsigned short*>(at + in_block(t + 1, cc >> 3)) = (unsigned short)(y[m] >> 16);
                    }
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
                const Sum ref = sum_at(j * 16 + 15);
                f32x2 ec[2];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    Sum b0, b1;
                    sums_at(j * 16 + 8 * m + 2 * c, b0, b1);
                    ec[m] = pack2(ex2(ref.to(b0)), ex2(ref.to(b1)));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float et = ex2(sum_at(i * 16 + g + 8 * h).to(ref));
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const int at = block_of(i, j) + in_block(g + 8 * h, m) + 4 * c;
                        const f32x2 e = fmul2(ec[m], pack2(et, et));
                        if constexpr (Q) put(terms_p, lay.p(buf), at, fmul2(pair(pp[m], h), e));
                        put(terms_n, lay.n(buf), at, fmul2(pair(nn[m], h), e));
                    }
                }
            }
        }
        bar_arrive(kBarFull + buf, threads);
    }
}

// ---- the warps with columns ---------------------------------------------------------------------------------------------

// Columns of a warp step by step in fp32, two lanes a column: what grows too far for the chunks or is not finite.
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

// The state of sixteen columns, transposed: tile n holds key dimensions 8n + 2c, + 1 of columns g (0, 1) and g + 8 (2, 3).
template <int DKP>
struct State {
    float x[DKP / 8][4];
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
                if (i < dk && j < cols) to[(long long)i * cols + j] = x[n][e];
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
template <int DKP, int N, int NS, int M>
__device__ __forceinline__ void state_times_rows(float (&acc)[NS][2][4], const uint32_t (&op)[M][4], uint32_t tile, int s, const Lane& ln) {
    uint32_t x[NS][4];
#pragma unroll
    for (int i = 0; i < NS; ++i) ldsm(at_b<key_pitch<DKP>()>(ln, tile, i * 16, s * 16), x[i]);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            mma(acc[i][0], op[n], x[i][0], x[i][1]);
            mma(acc[i][1], op[n], x[i][2], x[i][3]);
        }
}
// S += (sixteen tokens' operand) x their rows of a key tile
template <int DKP, int N>
__device__ __forceinline__ void rows_into_state(State<DKP>& S, const uint32_t (&op)[N][4], uint32_t tile, int strip, const Lane& ln) {
    constexpr int KS = DKP / 16, AT = KS % 4 == 0 ? 4 : KS % 2 == 0 ? 2 : 1;   // sixteens of keys at a time
#pragma unroll
    for (int s0 = 0; s0 < KS; s0 += AT) {
        uint32_t y[AT][4];
#pragma unroll
        for (int s = 0; s < AT; ++s) ldsm_trans(at_t<key_pitch<DKP>()>(ln, tile, strip * 16, (s0 + s) * 16), y[s]);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int s = 0; s < AT; ++s) {
                mma(S.x[2 * (s0 + s)], op[n], y[s][0], y[s][1]);
                mma(S.x[2 * (s0 + s) + 1], op[n], y[s][2], y[s][3]);
            }
    }
}
// acc += operand (A terms) x a 16 x 16 block of a token-by-token matrix (B terms, `stride` apart), contracted over its columns, or with TRANS over
// its rows.  Products of terms that are smaller than the last of either are left out.
template <bool TRANS, int A, int B, int M>
__device__ __forceinline__ void times_block(float (&acc)[2][4], const uint32_t (&op)[M][4], uint32_t block, int stride, const Lane& ln) {
    constexpr int kMost = A > B ? A : B;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        uint32_t x[4];
        if constexpr (TRANS) ldsm_trans(block + b * stride + ln.t_block, x);
        else ldsm(block + b * stride + ln.b_block, x);
#pragma unroll
        for (int n = 0; n < A; ++n)
            if (n + b < kMost) {
                mma(acc[0], op[n], x[0], x[1]);
                mma(acc[1], op[n], x[2], x[3]);
            }
    }
}

// How far a column's U (backwards dU) may outgrow what goes into the chunk before it is walked step by step instead.  With beta |k|^2 <= 2 a token's
// transition has norm at most one, which bounds a column's |u| by (129 + dk) beta (|v| + |k| |S|) and its |du| by dk |k| (|A| + 64 |q| |do|), with the chunk's
// largest elements of each.  Beyond, later tokens may take off again what has grown: of the sums' sixteen bits (24 for states) nine are given away here.
constexpr float kGrowth = 512.f;

// One chunk of NS strips forwards.  False where a column of this lane grew too far or is not finite.
template <int DKP, bool EXACT, Way WAY, int NS>
__device__ __forceinline__ bool forward_chunk(State<DKP>& S, const Gdr<bf>& a, const Kept& kept, unsigned char* smem,
                                              const Layout<DKP, EXACT, WAY>& lay, int buf, int cols, long long unit, int n, int chunks, int col0, int lane,
                                              const Lane& ln) {
    using Lay = Layout<DKP, EXACT, WAY>;
    constexpr int KS = DKP / 16, TERMS = Lay::kTerms;
    constexpr bool OUT = WAY == Way::kForward, KEEP = WAY == Way::kKeep;
    const int g = lane >> 2, c = lane & 3;
    const uint32_t base = smem_u32(smem), kt = base + lay.k(buf), qt = base + lay.q(buf), vt = base + cols;
    const float* const gates = reinterpret_cast<const float*>(smem + lay.gates(buf));
    uint32_t vm[2] = {0u, 0u}, sm[2] = {0u, 0u}, vv[NS][4];   // V transposed: strip i, columns g (0, 2), g + 8 (1, 3) of tokens 2c, 2c + 1 (0, 1), + 8 (2, 3)
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        uint32_t x[4];
        ldsm_trans(vt + i * kBlock + ln.t_block, x);
        vv[i][0] = x[0]; vv[i][1] = x[2]; vv[i][2] = x[1]; vv[i][3] = x[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) larger(vm[e & 1], vv[i][e]);
    }
    // products with S, of all strips; then strip by strip, what a strip's U means to the strips behind it as soon as it is there: the next
    // strip's chain (N, the step, the inverse) is what bounds a chunk, all else fills its gaps
    float w[NS][2][4] = {}, o[NS][2][4] = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        uint32_t sa[TERMS][4];
        pack_a<TERMS>(S.x[2 * s], S.x[2 * s + 1], sa);
#pragma unroll
        for (int e = 0; e < 4; ++e) larger(sm[e & 1], sa[0][e]);
        if constexpr (KEEP) kept.keep_state<DKP>(kept.S, kept.state_term, unit * chunks + n, col0, s, sa, g, c, n > 0 || a.state_in);
        state_times_rows<DKP, TERMS, NS>(w, sa, kt, s, ln);
        if constexpr (OUT) state_times_rows<DKP, 2, NS>(o, sa, qt, s, ln);
    }
    S.decay(gates[kEb * kChunk + kChunk - 1]);
    float limit[2];
    {
        const float4 k4 = *reinterpret_cast<const float4*>(gates + kMost * kChunk);
        const float k = fmaxf(fmaxf(k4.x, k4.y), fmaxf(k4.z, k4.w)), step = gates[kMost * kChunk + 8] * kGrowth;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x = fmaf(k, largest_of(sm[h]), largest_of(vm[h]));
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            limit[h] = x * step;
        }
    }
    uint32_t um[2] = {0u, 0u};
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
            const f32x2 beta = gate_pair(gates, kBeta, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 y = ffma2(pair(w[i][m], h), pack2(-1.f, -1.f), widen_bf16(vv[i][2 * m + h]));
                if constexpr (KEEP) set_pair(w[i][m], h, y);
                set_pair(r[m], h, fmul2(beta, y));
            }
        }
        uint32_t ra[TERMS][4], u[TERMS][4];
        pack_a<TERMS>(r[0], r[1], ra);
        times_block<false, TERMS, TERMS>(uu, ra, base + lay.inv(buf) + i * kBlock, Lay::kInv, ln);
        pack_a<TERMS>(uu[0], uu[1], u);
#pragma unroll
        for (int e = 0; e < 4; ++e) see(um[e & 1], u[0][e]);
#pragma unroll
        for (int j = i + 1; j < NS; ++j) times_block<false, TERMS, TERMS>(w[j], u, base + lay.n(buf) + block_of(j, i), Lay::kMat, ln);
        if constexpr (OUT)
#pragma unroll
            for (int j = i; j < NS; ++j) times_block<false, 2, 2>(o[j], u, base + lay.p(buf) + block_of(j, i), Lay::kMat, ln);
        // S += (e^{b_C - b} U)^T K
        uint32_t ud[TERMS][4];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 dl = gate_pair(gates, kDl, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(uu[m], h, fmul2(pair(uu[m], h), dl));
        }
        pack_a<TERMS>(uu[0], uu[1], ud);
        rows_into_state<DKP, TERMS>(S, ud, kt, i, ln);
        if constexpr (!OUT && !KEEP) continue;
        // over the strip's values, and out from there in pieces of sixteen bytes
        constexpr int kOut = OUT ? 1 : 2;
        uint32_t res[2][2][kOut];
        if constexpr (KEEP) {   // W of the strip: what its own block takes off
            float own[2][4] = {};
            times_block<false, 2, 2>(own, u, base + lay.n(buf) + block_of(i, i), Lay::kMat, ln);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) split<kOut>(ffma2(pair(own[m], h), pack2(-1.f, -1.f), pair(w[i][m], h)), res[m][h]);
        } else {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) split<kOut>(pair(o[i][m], h), res[m][h]);
        }
        const int t = n * kChunk + i * 16 + (lane >> 1), e = (lane & 1) * 8;
        const uint4* const piece = reinterpret_cast<const uint4*>(smem + cols + i * kBlock + in_block(lane >> 1, lane & 1));
#pragma unroll
        for (int m = 0; m < kOut; ++m) {
            if (m > 0) __syncwarp();
            stsm_trans(vt + i * kBlock + ln.t_block, res[0][0][m], res[1][0][m], res[0][1][m], res[1][1][m]);
            __syncwarp();
            if constexpr (OUT) {
                if (t < a.L && col0 + e < a.ldv) *reinterpret_cast<uint4*>(a.out + a.row(unit, t) * a.ldv + col0 + e) = *piece;
            } else *reinterpret_cast<uint4*>(kept.w + m * kept.row_term + (unit * chunks * kChunk + t) * kept.dvp + col0 + e) = *piece;
        }
    }
    return within(um[0], limit[0]) && within(um[1], limit[1]);
}

// One chunk of NS strips backwards: S is A, the columns are those of dO.
template <int DKP, bool EXACT, Way WAY, int NS>
__device__ __forceinline__ bool backward_chunk(State<DKP>& A, const Gdr<bf>& a, const Kept& kept, unsigned char* smem,
                                               const Layout<DKP, EXACT, WAY>& lay, int buf, int cols, long long unit, int n, int chunks, int col0,
                                               int lane, const Lane& ln) {
    using Lay = Layout<DKP, EXACT, WAY>;
    constexpr int KS = DKP / 16, TERMS = Lay::kTerms;
    const int g = lane >> 2, c = lane & 3;
    const uint32_t base = smem_u32(smem), kt = base + lay.k(buf), qt = base + lay.q(buf), vt = base + cols;
    const float* const gates = reinterpret_cast<const float*>(smem + lay.gates(buf));
    uint32_t dm[2] = {0u, 0u}, am[2] = {0u, 0u}, dd[NS][1][4];   // dO, an operand as it is
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        uint32_t x[4];
        ldsm_trans(vt + i * kBlock + ln.t_block, x);
        dd[i][0][0] = x[0]; dd[i][0][1] = x[2]; dd[i][0][2] = x[1]; dd[i][0][3] = x[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) larger(dm[e & 1], dd[i][0][e]);
    }
    float r[NS][2][4] = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        uint32_t aa[TERMS][4];
        pack_a<TERMS>(A.x[2 * s], A.x[2 * s + 1], aa);
#pragma unroll
        for (int e = 0; e < 4; ++e) larger(am[e & 1], aa[0][e]);
        if constexpr (WAY == Way::kBack) kept.keep_state<DKP>(kept.A, kept.state_term, unit * chunks + n, col0, s, aa, g, c, n + 1 < chunks || a.d_state_out);
        state_times_rows<DKP, TERMS, NS>(r, aa, kt, s, ln);
    }
    A.decay(gates[kEb * kChunk + kChunk - 1]);
    float limit[2];
    {
        const float4 k4 = *reinterpret_cast<const float4*>(gates + kMost * kChunk), q4 = *reinterpret_cast<const float4*>(gates + kMost * kChunk + 4);
        const float k = fmaxf(fmaxf(k4.x, k4.y), fmaxf(k4.z, k4.w)), q = fmaxf(fmaxf(q4.x, q4.y), fmaxf(q4.z, q4.w));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x = fmaf(64.f * q, largest_of(dm[h]), largest_of(am[h]));
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            limit[h] = x * k * kGrowth;
        }
    }
    uint32_t um[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 dl = gate_pair(gates, kDl, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(r[i][m], h, fmul2(pair(r[i][m], h), dl));
        }
#pragma unroll
    for (int j = NS - 1; j >= 0; --j)
#pragma unroll
        for (int i = j; i >= 0; --i) times_block<true, 1, TERMS>(r[i], dd[j], base + lay.p(buf) + block_of(j, i), Lay::kMat, ln);
#pragma unroll
    for (int i = NS - 1; i >= 0; --i) {
        uint32_t pa[TERMS][4];
        float du[2][4] = {}, x[2][4];
        pack_a<TERMS>(r[i][0], r[i][1], pa);
        times_block<true, TERMS, TERMS>(du, pa, base + lay.inv(buf) + i * kBlock, Lay::kInv, ln);
        uint32_t dv[2][2], dh[2][2][2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 beta = gate_pair(gates, kBeta, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 y = fmul2(pair(du[m], h), beta);
                float p, q;
                unpack2(y, p, q);
                dv[m][h] = pack_bf16(p, q);
                split<2>(pair(du[m], h), dh[m][h]);
                see(um[h], dh[m][h][0]);
                set_pair(x[m], h, fmul2(y, pack2(-1.f, -1.f)));
            }
        }
        uint32_t ra[TERMS][4];   // - R
        pack_a<TERMS>(x[0], x[1], ra);
#pragma unroll
        for (int j = i - 1; j >= 0; --j) times_block<true, TERMS, TERMS>(r[j], ra, base + lay.n(buf) + block_of(i, j), Lay::kMat, ln);
        // A += (e^b dO)^T Q - (e^b R)^T K
        uint32_t pe[TERMS][4];
        float y[2][4];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x2 eb = gate_pair(gates, kEb, i * 16 + 8 * m + 2 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                set_pair(x[m], h, fmul2(pair(x[m], h), eb));
                set_pair(y[m], h, fmul2(widen_bf16(dd[i][0][2 * m + h]), eb));
            }
        }
        pack_a<TERMS>(x[0], x[1], pe);
        rows_into_state<DKP, TERMS>(A, pe, kt, i, ln);
        pack_a<TERMS>(y[0], y[1], pe);
        rows_into_state<DKP, TERMS>(A, pe, qt, i, ln);
        if constexpr (WAY != Way::kBack) continue;
        // out: dv, then the terms of dU, through the strip's rows
        const int t = n * kChunk + i * 16 + (lane >> 1), e = (lane & 1) * 8;
        const uint32_t at = vt + i * kBlock + ln.t_block;
        const uint4* const piece = reinterpret_cast<const uint4*>(smem + cols + i * kBlock + in_block(lane >> 1, lane & 1));
        stsm_trans(at, dv[0][0], dv[1][0], dv[0][1], dv[1][1]);
        __syncwarp();
        if (t < a.L && col0 + e < a.ldv) *reinterpret_cast<uint4*>(a.dv_out + a.row(unit, t) * a.ldv + col0 + e) = *piece;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            __syncwarp();
            stsm_trans(at, dh[0][0][m], dh[1][0][m], dh[0][1][m], dh[1][1][m]);
            __syncwarp();
            *reinterpret_cast<uint4*>(kept.du + m * kept.row_term + (unit * chunks * kChunk + t) * kept.dvp + col0 + e) = *piece;
        }
    }
    return within(um[0], limit[0]) && within(um[1], limit[1]);
}

// Whether two blocks share an SM: their shared memory must.  Each then has 128 registers a thread.  (Unequal shares, 80 to 104 for the preparing
// warps and 176 to 152 for the others: 53 to 47 us for 64 x 12 units of 196 tokens, 32 x 64, against 46, with one term an operand.)
template <int DKP, bool EXACT, Way WAY>
constexpr bool two_blocks() { return 2 * (Layout<DKP, EXACT, WAY>::total(kMostWarps) + 1024) <= 228 * 1024; }

// EXACT: states leave the call in fp32, so that what they are made of is taken with 24 bits (three terms an operand); otherwise only bf16
// results do, and sixteen bits keep a rounding of the loop's own below a hundredth of theirs.
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
            cp_async16(base + cols(buf) + i * kBlock + in_block(lane >> 1, lane & 1), rows + (in ? a.row(unit, n * kChunk + t) * a.ldv + col0 + e : 0), in);
        }
        cp_async_commit();
    };
    const long long plane = (long long)a.dk * a.dv, at = unit * segs.n + seg;
    State<DKP> S;
    bool lost = false;
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
            if constexpr (BACK) lost |= !backward_chunk<DKP, EXACT, WAY, ns>(S, a, kept, smem, lay, buf, cols(buf), unit, n, chunks, col0, lane, ln);
            else lost |= !forward_chunk<DKP, EXACT, WAY, ns>(S, a, kept, smem, lay, buf, cols(buf), unit, n, chunks, col0, lane, ln);
        };
        if (strips == 4) chunk(std::integral_constant<int, 4>());
        else if (strips == 1) chunk(std::integral_constant<int, 1>());
        else if (strips == 2) chunk(std::integral_constant<int, 2>());
        else chunk(std::integral_constant<int, 3>());
        if (it + 2 < count) bar_arrive(kBarEmpty + buf, threads);
        __syncwarp();
    }
    lost = __any_sync(0xffffffffu, lost);
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
        if (WAY == Way::kBack && a.d_state_in && ends) S.store(a.d_state_in + unit * plane, a.dk, a.dv, col0 + g, c);
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
    const int slabs = (sixteens + kMostWarps - 1) / kMostWarps, warps = sixteens / slabs;   // (narrower blocks for few units: 332 -> 414 us for 2 x 16 x 4096, 128 x 128, with one term an operand)
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
// 32 units of 4096 tokens, 24 x 48, 8 segments 49 + 39 us for the two launches, 5 segments, with which the first fits the chip too, 40 + 57, with one term an
// operand.)
int segments(long long units, int L, int dk, int dv) {
    if (dk % 8 || dv % 8) return 1;   // (the states' copies between segments are whole pieces of sixteen bytes: other sizes go without)
    if (dk > kMostSegmentKeys) return 1;   // (one block an SM, and as many columns for the transition as for the state: 2 x 16 units of 4096 tokens, 128 x 128, gain
                                            // nothing; of fewer units than SMs, where segments may well pay, neither side has been measured)
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
    k.row_term = (long long)(units * chunks * kChunk * dvp);
    k.state_term = (long long)(units * chunks * dvp * dkp);
    k.w = (bf*)take(2 * k.row_term * 2);
    k.du = (bf*)take(2 * k.row_term * 2);
    k.S = (bf*)take(2 * k.state_term * 2);
    k.A = (bf*)take(2 * k.state_term * 2);
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
