// The gated delta rule's gradient on the tensor cores (bf16 calls): what is left chunk by chunk once the two walks (gdr_chunk.cu) have W, dU and
// the states S before and A behind every chunk.  With Gam_ts = e^{b_t - b_s}, U = beta W, X = tril(dO U^T . Gam), E = strict_tril(dU U^T . Gam):
//
//   dQ = e^b dO S^T + X K
//   dK = - beta (e^b dU S^T + E K)  +  e^{b_C - b} U A^T + X^T Q - E'^T K          (E'^T: E^T with the beta of its columns)
//   dbeta_t = dU_t . W_t          dlog_alpha_t = e_t + .. + e_C + <S_C, A>,   e = q . dQ - beta dbeta + k . (the first bracket of dK)
//
// (E K's part of dK and e: replacing S by its decayed form shows e_t = q.dq - v.dv, and v = w + what k retrieves.)
// A block takes a chunk, a warp sixteen of its tokens as rows: the blocks of X and E up to the diagonal and those of their transposes from it
// on, five of each for every warp, so that no warp needs another's.  K, Q and dO are bf16 as they come, all else is two bf16 terms an operand (gdr_tile.cuh):
// what the walks kept, and X and E.  Bound by instruction issue and shared memory (two blocks an SM for 32 x 64).
#include <type_traits>

#include "gdr.h"
#include "gdr_tile.cuh"

namespace vig {
namespace {

using namespace gdr;
using bf = __nv_bfloat16;

constexpr int kMostColumns = 128;
template <int DKP>
constexpr int grad_threads() { return DKP > 64 ? 256 : 128; }   // two warps a strip where the key dimensions are many

// Whether A takes the place of S in shared memory once nothing more is read of S: where both do not fit (128 x 128: 255 KB).
template <int DKP>
constexpr bool grad_shares() { return DKP > 96; }

// Per token, arrays of kChunk floats: running sum of log2 alpha (two floats), 2^b, 2^{b_C - b}, beta, and e of a strip's first and second warp.
enum { kB, kBl, kEb, kDl, kBeta, kE, kE2, kRows };

struct GradLayout {   // W, dU, S and A: two terms, row_term and state_term bytes apart
    int kp, vp, row_term, state_term, k, q, d, r, w, s, a, gates, red, total;
    __host__ __device__ GradLayout(int dkp, int dvp, bool shares) {
        kp = dkp * 2 + 16;
        vp = dvp * 2 + 16;
        row_term = kChunk * vp;
        state_term = dvp * kp;
        int at = 0;
        auto take = [&](int bytes) { const int o = at; at += bytes; return o; };
        k = take(kChunk * kp);
        q = take(kChunk * kp);
        d = take(row_term);
        r = take(2 * row_term);
        w = take(2 * row_term);
        s = take(2 * state_term);
        a = shares ? s : take(2 * state_term);
        gates = take(kChunk * kRows * 4);
        red = take(16 * 4);
        total = at;
    }
};

__device__ __forceinline__ void ldsm_a(uint32_t addr, uint32_t (&a)[4]) {
    uint32_t x[4];
    ldsm(addr, x);
    a[0] = x[0]; a[1] = x[2]; a[2] = x[1]; a[3] = x[3];
}
__device__ __forceinline__ float2 row2(const float* gates, int row, int t) { return *reinterpret_cast<const float2*>(gates + row * kChunk + t); }
__device__ __forceinline__ f32x2 row_pair(const float* gates, int row, int t) { return *reinterpret_cast<const f32x2*>(gates + row * kChunk + t); }

// acc += a (A terms) x y (B terms), without the product of second terms.
template <int A, int B>
__device__ __forceinline__ void add_products(float (&acc)[2][4], const uint32_t (&a)[A][4], const uint32_t (&y)[B][4]) {
#pragma unroll
    for (int i = 0; i < A; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (i + j < 2) {
                mma(acc[0], a[i], y[j][0], y[j][1]);
                mma(acc[1], a[i], y[j][2], y[j][3]);
            }
}

// Strip I of the chunk; key dimensions in sixteens s0, s0 + step, ..  (I is a variable and the five blocks' code the same for all warps: with a
// copy for each strip, fetching instructions was what the warps waited for most, 173 us for 64 x 12 units of 196 tokens, 32 x 64.)
// bring_a: called by all threads of the block between the products with S and those with A.
template <int DKP, typename F>
__device__ __forceinline__ void grad_strip(const int I, const Gdr<bf>& a, unsigned char* smem, const GradLayout& lay, int dvp, long long unit, int n,
                                           bool before, bool behind, int s0, int step, int lane, uint32_t& seen, F bring_a) {
    constexpr int KP = DKP * 2 + 16;
    const int g = lane >> 2, c = lane & 3, vp = lay.vp, strips = (min(kChunk, a.L - n * kChunk) + 15) >> 4;
    const Lane ln(lane);
    const uint32_t base = smem_u32(smem), kt = base + lay.k, qt = base + lay.q, dt = base + lay.d, rt = base + lay.r, wt = base + lay.w, st = base + lay.s,
                   at = base + lay.a;
    float* const gates = reinterpret_cast<float*>(smem + lay.gates);
    const int lane_at = ln.b_row * vp + ln.b_col * 2;
    auto b_of = [&](uint32_t tile, int row0, int col0) { return tile + lane_at + row0 * vp + col0 * 2; };
    auto both_a = [&](uint32_t tile, int row0, int col0, uint32_t (&x)[2][4]) {
        ldsm_a(b_of(tile, row0, col0), x[0]);
        ldsm_a(b_of(tile + lay.row_term, row0, col0), x[1]);
    };
    auto both_b = [&](uint32_t tile, int row0, int col0, uint32_t (&x)[2][4]) {
        ldsm(b_of(tile, row0, col0), x[0]);
        ldsm(b_of(tile + lay.row_term, row0, col0), x[1]);
    };
    // Block p: of dO W^T and dU W^T up to the diagonal (p <= I, columns of strip p), of W dO^T and W dU^T from it on (columns of strip p - 1)
    float x[5][2][4] = {}, e[5][2][4] = {};
#pragma unroll 1
    for (int v = I < strips ? 0 : dvp; v < dvp; v += 16) {
        uint32_t da[1][4], ra[2][4], wa[2][4];
        ldsm_a(b_of(dt, I * 16, v), da[0]);
        both_a(rt, I * 16, v, ra);
        both_a(wt, I * 16, v, wa);
#pragma unroll
        for (int p = 0; p < 5; ++p) {
            uint32_t y[2][4];
            if (p <= I) {
                both_b(wt, p * 16, v, y);
                add_products(x[p], da, y);
                add_products(e[p], ra, y);
            } else if (p <= strips) {
                uint32_t z[1][4];
                ldsm(b_of(dt, (p - 1) * 16, v), z[0]);
                add_products(x[p], wa, z);
                both_b(rt, (p - 1) * 16, v, y);
                add_products(e[p], wa, y);
            }
        }
    }
    const int t0 = I * 16 + g;   // rows t0, t0 + 8
    auto sum_at = [&](int t) { return Sum{gates[kB * kChunk + t], gates[kBl * kChunk + t]}; };
    auto sums_at = [&](int t, Sum (&x)[2]) {   // of two neighbours
        const float2 h = row2(gates, kB, t), l = row2(gates, kBl, t);
        x[0] = {h.x, l.x};
        x[1] = {h.y, l.y};
    };
    const Sum bt[2] = {sum_at(t0), sum_at(t0 + 8)}, end = sum_at(I * 16 + 15);
    const float beta[2] = {gates[kBeta * kChunk + t0], gates[kBeta * kChunk + t0 + 8]};
    float db[2] = {0.f, 0.f};
    // to operands of two terms, e^{b_t - b_s} by way of the last token of s' sixteen off the diagonal (both factors are at most one)
    uint32_t xa[5][2][4], ea[5][2][4];
    auto put = [&](uint32_t (&to)[2][4], int i, f32x2 v) {
        uint32_t t[2];
        split<2>(v, t);
        to[0][i] = t[0];
        to[1][i] = t[1];
    };
#pragma unroll
    for (int p = 0; p < 5; ++p) {
        const bool low = p <= I;
        const int j = low ? p : p - 1;
        if (j >= strips) {   // (no tokens there, and nothing in shared memory)
#pragma unroll
            for (int h = 0; h < 4; ++h) xa[p][0][h] = xa[p][1][h] = ea[p][0][h] = ea[p][1][h] = 0u;
        } else if (j != I) {
            const Sum ref = low ? sum_at(j * 16 + 15) : end;
            f32x2 er[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float r = ex2(low ? bt[h].to(ref) : ref.to(bt[h]));
                er[h] = pack2(r, r);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int col = j * 16 + 8 * m + 2 * c;
                Sum bc[2];
                sums_at(col, bc);
                f32x2 fx = pack2(ex2(low ? ref.to(bc[0]) : bc[0].to(ref)), ex2(low ? ref.to(bc[1]) : bc[1].to(ref))), fe = fmul2(fx, row_pair(gates, kBeta, col));
                if (low) fx = fe;                          // columns s: times beta_s
                else fe = fmul2(fe, pack2(-1.f, -1.f));    // columns t: times - beta_t, X as it is
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    put(xa[p], 2 * m + h, fmul2(pair(x[p][m], h), fmul2(fx, er[h])));
                    put(ea[p], 2 * m + h, fmul2(pair(e[p][m], h), fmul2(fe, er[h])));
                }
            }
        } else {
            if (low)   // dbeta: the diagonal of dU W^T, row g + 8 h and the same column: in lane c = g / 2
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float d = g & 1 ? e[p][h][2 * h + 1] : e[p][h][2 * h];
                    db[h] = __shfl_sync(0xffffffffu, d, (lane & 28) | (g >> 1));
                }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int cc = 8 * m + 2 * c, col = I * 16 + cc;
                const float2 be = row2(gates, kBeta, col);
                Sum bc[2];
                sums_at(col, bc);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = g + 8 * h;
                    float xx[2], ee[2];
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const bool in = low ? cc + f <= row : cc + f >= row, strict = in && cc + f != row;
                        const float gam = in ? ex2(low ? bt[h].to(bc[f]) : bc[f].to(bt[h])) : 0.f, step = f ? be.y : be.x;
                        xx[f] = in ? x[p][m][2 * h + f] * gam * (low ? step : 1.f) : 0.f;
                        ee[f] = strict ? e[p][m][2 * h + f] * gam * (low ? step : -step) : 0.f;
                    }
                    put(xa[p], 2 * m + h, pack2(xx[0], xx[1]));
                    put(ea[p], 2 * m + h, pack2(ee[0], ee[1]));
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            see(seen, xa[p][0][h]);
            see(seen, ea[p][0][h]);
        }
    }
    const float eb[2] = {gates[kEb * kChunk + t0], gates[kEb * kChunk + t0 + 8]}, dl[2] = {gates[kDl * kChunk + t0], gates[kDl * kChunk + t0 + 8]};
    float sum[2] = {0.f, 0.f};
    auto state = [&](uint32_t tile, int s, int v, uint32_t (&y)[2][4]) {
        ldsm_trans(at_t<KP>(ln, tile, v, s * 16), y[0]);
        ldsm_trans(at_t<KP>(ln, tile + lay.state_term, v, s * 16), y[1]);
    };
    // sixteen key dimensions of dq, and o: the first bracket of dK (with its sign)
    auto with_s = [&](int s, float (&o)[2][4]) {
        float hq[2][4] = {}, h1[2][4] = {};
        if (before)
#pragma unroll 2
            for (int v = 0; v < dvp; v += 16) {
                uint32_t da[1][4], ra[2][4], y[2][4];
                ldsm_a(b_of(dt, I * 16, v), da[0]);
                both_a(rt, I * 16, v, ra);
                state(st, s, v, y);
                add_products(hq, da, y);
                add_products(h1, ra, y);
            }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                set_pair(hq[m], h, fmul2(pair(hq[m], h), pack2(eb[h], eb[h])));
                set_pair(h1[m], h, fmul2(pair(h1[m], h), pack2(eb[h], eb[h])));
            }
#pragma unroll
        for (int p = 0; p < 4; ++p)
            if (p <= I) {
                uint32_t y[1][4];
                ldsm_trans(at_t<KP>(ln, kt, p * 16, s * 16), y[0]);
                add_products(hq, xa[p], y);
                add_products(h1, ea[p], y);
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = t0 + 8 * h;
            const bool in = n * kChunk + t < a.L;
            const long long r = in ? a.row(unit, n * kChunk + t) * a.ldk : 0;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int col = s * 16 + 8 * m + 2 * c;
                const float2 kk = unpack_bf16(*reinterpret_cast<const uint32_t*>(smem + lay.k + t * KP + col * 2)),
                             qq = unpack_bf16(*reinterpret_cast<const uint32_t*>(smem + lay.q + t * KP + col * 2));
                o[m][2 * h] = -beta[h] * h1[m][2 * h];
                o[m][2 * h + 1] = -beta[h] * h1[m][2 * h + 1];
                sum[h] += qq.x * hq[m][2 * h] + qq.y * hq[m][2 * h + 1] + kk.x * o[m][2 * h] + kk.y * o[m][2 * h + 1];
                if (in && col < a.ldk) *reinterpret_cast<uint32_t*>(a.dq + r + col) = pack_bf16(hq[m][2 * h], hq[m][2 * h + 1]);
            }
        }
    };
    // the other two, and dk
    auto with_a = [&](int s, const float (&o)[2][4]) {
        float h2[2][4] = {};
        if (behind)
#pragma unroll 2
            for (int v = 0; v < dvp; v += 16) {
                uint32_t wa[2][4], y[2][4];
                both_a(wt, I * 16, v, wa);
                state(at, s, v, y);
                add_products(h2, wa, y);
            }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(h2[m], h, fmul2(pair(h2[m], h), pack2(dl[h], dl[h])));
#pragma unroll
        for (int p = 1; p < 5; ++p)
            if (p > I && p <= strips) {
                uint32_t y[1][4];
                ldsm_trans(at_t<KP>(ln, kt, (p - 1) * 16, s * 16), y[0]);
                add_products(h2, ea[p], y);
                ldsm_trans(at_t<KP>(ln, qt, (p - 1) * 16, s * 16), y[0]);
                add_products(h2, xa[p], y);
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = t0 + 8 * h;
            if (n * kChunk + t >= a.L) continue;
            bf* const r = a.dk_out + a.row(unit, n * kChunk + t) * a.ldk;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int col = s * 16 + 8 * m + 2 * c;
                if (col < a.ldk)
                    *reinterpret_cast<uint32_t*>(r + col) = pack_bf16(fmaf(beta[h], h2[m][2 * h], o[m][2 * h]), fmaf(beta[h], h2[m][2 * h + 1], o[m][2 * h + 1]));
            }
        }
    };
    if constexpr (grad_shares<DKP>()) {
        float o[DKP / 32][2][4];   // (two warps a strip)
        if (I < strips)
#pragma unroll
            for (int i = 0; i < DKP / 32; ++i) with_s(s0 + i * step, o[i]);
        bring_a();
        if (I < strips)
#pragma unroll
            for (int i = 0; i < DKP / 32; ++i) with_a(s0 + i * step, o[i]);
    } else {
#pragma unroll 1
        for (int s = s0; s < DKP / 16; s += step) {
            float o[2][4];
            with_s(s, o);
            with_a(s, o);
        }
    }
    if (I >= strips) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
        const int t = t0 + 8 * h;
        if (c == 0) {
            if (s0 == 0) {
                if (n * kChunk + t < a.L) a.dbeta[a.row(unit, n * kChunk + t)] = __float2bfloat16_rn(db[h]);
                sum[h] -= beta[h] * db[h];
            }
            gates[(s0 == 0 ? kE : kE2) * kChunk + t] = sum[h];
        }
    }
}

template <int DKP>
__global__ void __launch_bounds__(grad_threads<DKP>(), DKP <= 32 ? 3 : DKP <= 64 ? 2 : 1) gdr_grad_kernel(Gdr<bf> a, GdrKept kept, int chunks) {
    constexpr int KP = DKP * 2 + 16, kThreads = grad_threads<DKP>();
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, dvp = kept.dvp;
    const GradLayout lay(DKP, dvp, grad_shares<DKP>());
    const long long unit = blockIdx.x / chunks;
    const int n = blockIdx.x % chunks, t0 = n * kChunk, nt = min(kChunk, a.L - t0);
    const long long here = unit * chunks + n, states = unit * (chunks + 1) + n;
    float* const gates = reinterpret_cast<float*>(smem + lay.gates);
    float* const red = reinterpret_cast<float*>(smem + lay.red);
    pdl_wait();
    pdl_launch_dependents();
    // everything comes in by asynchronous copies at once and is an operand as it lies; rows up to the last strip with tokens
    const uint32_t base = smem_u32(smem);
    const int rows = (nt + 15) & ~15;
    const bool before = n > 0 || a.state_in, behind = n + 1 < chunks || a.d_state_out;   // (zeros otherwise, which nothing is read of)
    for (int i = tid; i < rows * (DKP / 8); i += kThreads) {
        const int t = i / (DKP / 8), e = i % (DKP / 8) * 8;
        const bool in = t < nt && e < a.ldk;
        const long long at = in ? a.row(unit, t0 + t) * a.ldk + e : 0;
        cp_async16(base + lay.k + t * KP + e * 2, a.k + at, in);
        cp_async16(base + lay.q + t * KP + e * 2, a.q + at, in);
    }
    const int lg = dvp <= 16 ? 1 : dvp <= 32 ? 2 : dvp <= 64 ? 3 : 4, piece = (tid & ((1 << lg) - 1)) * 8;   // lanes of a row of dv columns, and this one's columns
    if (piece < dvp)
        for (int t = tid >> lg; t < rows; t += kThreads >> lg) {
            const bool in = t < nt;   // (rows behind the last token were not written)
            const uint32_t to = t * lay.vp + piece * 2;
            const long long at = (here * kChunk + t) * dvp + piece;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                cp_async16(base + lay.w + m * lay.row_term + to, kept.w + m * kept.row_term + at, in);
                cp_async16(base + lay.r + m * lay.row_term + to, kept.du + m * kept.row_term + at, in);
            }
            const bool values = in && piece < a.ldv;
            cp_async16(base + lay.d + to, a.d_out + (values ? a.row(unit, t0 + t) * a.ldv + piece : 0), values);
        }
    auto bring_state = [&](int to, const bf* from, long long term, bool there) {   // (nothing is read of one that is not)
        if (there)
            for (int i = tid; i < dvp * (DKP / 8); i += kThreads) {
                const int j = i / (DKP / 8), e = i % (DKP / 8) * 8;
#pragma unroll
                for (int m = 0; m < 2; ++m) cp_async16(base + to + m * lay.state_term + j * KP + e * 2, from + m * term + (long long)i * 8, true);
            }
        cp_async_commit();
    };
    const bf* const A = kept.A + here * dvp * DKP;
    if constexpr (!grad_shares<DKP>()) bring_state(lay.a, A, kept.A_term, behind);
    bring_state(lay.s, kept.S + states * dvp * DKP, kept.S_term, before);
    if (warp == 0) {   // gates, as the walks have them
        float la[2], be[2];
        Sum b[2], all;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = 2 * lane + h;
            la[h] = t < nt ? __bfloat162float(a.la[a.row(unit, t0 + t)]) : 0.f;
            be[h] = t < nt ? __bfloat162float(a.beta[a.row(unit, t0 + t)]) : 0.f;
        }
        gate_sums(la, b, all);
        auto two = [&](int row, float x, float y) { *reinterpret_cast<float2*>(gates + row * kChunk + 2 * lane) = make_float2(x, y); };
        two(kB, b[0].h, b[1].h);
        two(kBl, b[0].l, b[1].l);
        two(kEb, ex2(b[0].h + b[0].l), ex2(b[1].h + b[1].l));
        two(kDl, ex2(all.to(b[0])), ex2(all.to(b[1])));
        two(kBeta, be[0], be[1]);
    }
    cp_async_wait<0>();
    __syncthreads();
    float anchor = 0.f;   // what the next chunk's first gate sees: the product of A with the state behind the chunk
    auto meet = [&]() {
        if (!behind) return;
        for (int i = tid; i < dvp * (DKP / 8); i += kThreads) {
            const int j = i / (DKP / 8), e = i % (DKP / 8) * 8;
            const unsigned char* const x = smem + lay.a + j * KP + e * 2;
            const bf* const y = kept.S + ((states + 1) * dvp + j) * DKP + e;
            const uint4 xh = *reinterpret_cast<const uint4*>(x), xl = *reinterpret_cast<const uint4*>(x + lay.state_term), yh = *reinterpret_cast<const uint4*>(y),
                        yl = *reinterpret_cast<const uint4*>(y + kept.S_term);
            const uint32_t xs[2][4] = {{xh.x, xh.y, xh.z, xh.w}, {xl.x, xl.y, xl.z, xl.w}}, ys[2][4] = {{yh.x, yh.y, yh.z, yh.w}, {yl.x, yl.y, yl.z, yl.w}};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float u0, u1, v0, v1;
                unpack2(fadd2(widen_bf16(xs[0][q]), widen_bf16(xs[1][q])), u0, u1);
                unpack2(fadd2(widen_bf16(ys[0][q]), widen_bf16(ys[1][q])), v0, v1);
                anchor = fmaf(u0, v0, fmaf(u1, v1, anchor));
            }
        }
    };
    if constexpr (!grad_shares<DKP>()) meet();
    uint32_t seen = 0u;
    const int strip = warp & 3, half = warp >> 2, step = kThreads / 128;
    auto bring_a = [&]() {
        __syncthreads();
        bring_state(lay.a, A, kept.A_term, behind);
        cp_async_wait<0>();
        __syncthreads();
        meet();
    };
    if (grad_shares<DKP>() || strip * 16 < nt) grad_strip<DKP>(strip, a, smem, lay, dvp, unit, n, before, behind, half, step, lane, seen, bring_a);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) anchor += __shfl_xor_sync(0xffffffffu, anchor, o);
    if (lane == 0) red[warp] = anchor;
    const int lost = __syncthreads_or(!within(seen, 3.3e38f));
    if (tid == 0) kept.lost_grad[here] = lost;
    // dlog_alpha: sums from the chunk's end; a gate that leaves nothing, or has nothing to scale, has none, and the sums start anew there
    if (warp == 0) {
        float run = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) run += red[w];
        float sum[2];
        bool stop[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = 2 * lane + h;
            sum[h] = t < nt ? gates[kE * kChunk + t] + (kThreads > 128 ? gates[kE2 * kChunk + t] : 0.f) : 0.f;
            stop[h] = t < nt && (expf(__bfloat162float(a.la[a.row(unit, t0 + t)])) == 0.f || (t0 + t == 0 && !a.state_in));
            if (stop[h]) sum[h] = 0.f;
        }
        const float later = suffix_of_pairs(sum, stop, run);
        const float d1 = stop[1] ? 0.f : sum[1] + later, d0 = stop[0] ? 0.f : sum[0] + d1;
        if (2 * lane < nt) a.dla[a.row(unit, t0 + 2 * lane)] = __float2bfloat16_rn(d0);
        if (2 * lane + 1 < nt) a.dla[a.row(unit, t0 + 2 * lane + 1)] = __float2bfloat16_rn(d1);
    }
}

}  // namespace

bool gdr_grad_supported(int dk, int dv) { return dk <= 128 && dv <= kMostColumns; }

cudaError_t launch_gdr_grad(const Gdr<__nv_bfloat16>& a, const GdrKept& kept, cudaStream_t stream) {
    const int chunks = (a.L + kChunk - 1) / kChunk;
    auto launch = [&](auto D) {
        constexpr int dkp = decltype(D)::value;
        const int smem = GradLayout(dkp, kept.dvp, grad_shares<dkp>()).total;
        cudaError_t e = allow_smem<gdr_grad_kernel<dkp>>(GradLayout(dkp, kMostColumns, grad_shares<dkp>()).total);
        if (e != cudaSuccess) return e;
        count_launch();
        return launch_pdl(gdr_grad_kernel<dkp>, dim3((unsigned)(a.units * chunks)), dim3(grad_threads<dkp>()), smem, stream, a, kept, chunks);
    };
    if (a.dk <= 16) return launch(std::integral_constant<int, 16>());
    if (a.dk <= 32) return launch(std::integral_constant<int, 32>());
    if (a.dk <= 48) return launch(std::integral_constant<int, 48>());
    if (a.dk <= 64) return launch(std::integral_constant<int, 64>());
    if (a.dk <= 96) return launch(std::integral_constant<int, 96>());
    return launch(std::integral_constant<int, 128>());
}

}  // namespace vig
