// The gated delta rule's gradient on the tensor cores (bf16 calls): what is left chunk by chunk once the two walks (gdr_chunk.cu) have W, dU and
// the states S before and A behind every chunk.  With Gam_ts = e^{b_t - b_s}, U = beta W, X = tril(dO U^T . Gam), E = strict_tril(dU U^T . Gam):
//
//   dQ = e^b dO S^T + X K
//   dK = - beta (e^b dU S^T + E K)  +  e^{b_C - b} U A^T + X^T Q - E'^T K          (E'^T: E^T with the beta of its columns)
//   dbeta_t = dU_t . W_t
//   dlog_alpha_t = e^{b_C} <S, A> + sum_{r >= t} F_r + sum_{s < t} G_s + sum_{s < t <= r} H_rs
//     F_r = e^{b_r} (q_r . S do_r - beta_r k_r . S du_r)    G_s = e^{b_C - b_s} k_s . A u_s    H_rs = X_rs q_r . k_s - beta_r E_rs k_r . k_s
//
// (The gates' gradient: all that passes through a gate, and nothing to be taken off again; see gdr_walk.cu.)
// A block takes a chunk, a warp sixteen of its tokens as rows: the blocks of X and E up to the diagonal and those of their transposes from it
// on, five of each for every warp, so that no warp needs another's.  K, Q and dO are bf16 as they come, all else is two bf16 terms an operand (gdr_tile.cuh):
// what the walks kept, and X and E.  64 x 12 units of 196 tokens, 32 x 64: 140 us for 150 MB, three blocks an SM, bound by instructions: issue 0.38, and fetching
// them is the second of the stalls.
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

// Per token, arrays of kChunk floats: running sum of log2 alpha (two floats), 2^b, 2^{b_C - b}, beta; for the gates' gradient F, G, H's sums of a row over the
// strips in front of its own (R) and those of a column over the rows of strips 1 to 3 behind its own (C1 ..), of a strip's first and second warp each;
// and H of the pairs within the gate's own strip.
enum { kB, kBl, kEb, kDl, kBeta, kOwn, kF, kG, kR, kC1, kC2, kC3, kRows };
constexpr int kSums = kRows - kF;   // rows that a strip's second warp has too, behind the others

// Rows of key dimensions (K, Q, and S and A by columns) without gaps: pieces of sixteen bytes change places with the row, so that eight rows at one column
// never share a bank.  (With gaps instead 32 x 64 would be two blocks an SM, not three.)
template <int DKP>
struct KeyRows {
    static constexpr int kPitch = DKP * 2, kTurn = DKP % 64 == 0 ? 0 : DKP % 32 == 0 ? 1 : 2;
    __device__ __forceinline__ static int at(int row, int piece) { return row * kPitch + ((piece ^ ((row & 7) >> kTurn)) << 4); }
};

struct GradLayout {   // W, dU, S and A: two terms, row_term and state_term bytes apart
    int vp, row_term, state_term, k, q, d, r, w, s, a, gates, red, total;
    __host__ __device__ GradLayout(int dkp, int dvp, bool shares) {
        vp = dvp * 2 + 16;
        row_term = kChunk * vp;
        state_term = dvp * dkp * 2;
        int at = 0;
        auto take = [&](int bytes) { const int o = at; at += bytes; return o; };
        k = take(kChunk * dkp * 2);
        q = take(kChunk * dkp * 2);
        d = take(row_term);
        r = take(2 * row_term);
        w = take(2 * row_term);
        s = take(2 * state_term);
        a = shares ? s : take(2 * state_term);
        gates = take(kChunk * (kRows + (dkp > 64 ? kSums : 0)) * 4);
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
template <int DKP, typename Bring>
__device__ __forceinline__ void grad_strip(const int I, const Gdr<bf>& a, unsigned char* smem, const GradLayout& lay, int dvp, long long unit, int n,
                                           bool before, bool behind, int s0, int step, int lane, uint32_t& seen, Bring bring_a) {
    using Keys = KeyRows<DKP>;
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
    const Sum bt[2] = {sum_at(t0), sum_at(t0 + 8)};
    const float beta[2] = {gates[kBeta * kChunk + t0], gates[kBeta * kChunk + t0 + 8]};
    float db[2] = {0.f, 0.f};
    float xd[2][4] = {}, ed[2][4] = {};   // X and E of the strip's own block
    // to operands of two terms; one code for the blocks on the diagonal and off it (by way of a border between the two strips off it, with half the
    // exponentials, it is twice the code, and fetching it costs more)
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
            continue;
        }
        if (p == I)   // dbeta: the diagonal of dU W^T, row g + 8 h and the same column: in lane c = g / 2
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float d = g & 1 ? e[p][h][2 * h + 1] : e[p][h][2 * h];
                db[h] = __shfl_sync(0xffffffffu, d, (lane & 28) | (g >> 1));
            }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int col = j * 16 + 8 * m + 2 * c;
            const float2 be = row2(gates, kBeta, col);
            Sum bc[2];
            sums_at(col, bc);
            // columns s of X and E: times beta_s; columns t of their transposes: E times - beta_t, X as it is
            const float fx[2] = {low ? be.x : 1.f, low ? be.y : 1.f}, fe[2] = {low ? be.x : -be.x, low ? be.y : -be.y};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = t0 + 8 * h;
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const bool in = low ? col + f <= row : col + f >= row, strict = in && col + f != row;
                    const float d = bt[h].to(bc[f]), gam = ex2(low ? d : -d);
                    float &xx = x[p][m][2 * h + f], &ee = e[p][m][2 * h + f];
                    xx = in ? xx * (gam * fx[f]) : 0.f;
                    ee = strict ? ee * (gam * fe[f]) : 0.f;
                }
                put(xa[p], 2 * m + h, pair(x[p][m], h));
                put(ea[p], 2 * m + h, pair(e[p][m], h));
            }
        }
        if (p == I)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    xd[m][h] = x[p][m][h];
                    ed[m][h] = e[p][m][h];
                }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            see(seen, xa[p][0][h]);
            see(seen, ea[p][0][h]);
        }
    }
    const float eb[2] = {gates[kEb * kChunk + t0], gates[kEb * kChunk + t0 + 8]}, dl[2] = {gates[kDl * kChunk + t0], gates[kDl * kChunk + t0 + 8]};
    if (s0 == 0 && I < strips) {   // H over s < t <= r within the strip: each row's sums in front of t (its lanes: c), then those of the rows from t on
        float qk[2][4] = {}, kk[2][4] = {}, of_gate[2][2] = {};
#pragma unroll
        for (int s = 0; s < DKP / 16; ++s) {
            uint32_t q[1][4], k[1][4], y[1][4];
            const int own = Keys::at(I * 16 + ln.b_row, 2 * s + (ln.b_col >> 3));
            ldsm_a(qt + own, q[0]);
            ldsm(kt + own, y[0]);
            k[0][0] = y[0][0]; k[0][1] = y[0][2]; k[0][2] = y[0][1]; k[0][3] = y[0][3];
            add_products(qk, q, y);
            add_products(kk, k, y);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float own[2][2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int f = 0; f < 2; ++f) {   // (zeros stay: what is not finite in later keys)
                    const float z = fmaf(xd[m][2 * h + f], qk[m][2 * h + f], -beta[h] * ed[m][2 * h + f] * kk[m][2 * h + f]);
                    own[m][f] = 8 * m + 2 * c + f < g + 8 * h ? z : 0.f;
                }
            float low = own[0][0] + own[0][1], high = own[1][0] + own[1][1];   // columns 2c, 2c + 1 and 8 more
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                const float y = __shfl_up_sync(0xffffffffu, low, o), z = __shfl_up_sync(0xffffffffu, high, o);
                if (c >= o) {
                    low += y;
                    high += z;
                }
            }
            const float all = __shfl_sync(0xffffffffu, low, lane | 3), l1 = __shfl_up_sync(0xffffffffu, low, 1), h1 = __shfl_up_sync(0xffffffffu, high, 1);
            const float run[2] = {c > 0 ? l1 : 0.f, all + (c > 0 ? h1 : 0.f)};
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int t = 8 * m + 2 * c, r = g + 8 * h;
                if (t <= r) of_gate[m][0] += run[m];
                if (t + 1 <= r) of_gate[m][1] += run[m] + own[m][0];
            }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) of_gate[m][f] += __shfl_xor_sync(0xffffffffu, of_gate[m][f], o);
            if (g == 0) *reinterpret_cast<float2*>(gates + kOwn * kChunk + I * 16 + 8 * m + 2 * c) = make_float2(of_gate[m][0], of_gate[m][1]);
        }
    }
    float F[2] = {0.f, 0.f}, G[2] = {0.f, 0.f}, R[2] = {0.f, 0.f}, C[3][2] = {};   // (C: of strips 1 to 3)
    auto row_of = [&](int tile, int t, int col) { return unpack_bf16(*reinterpret_cast<const uint32_t*>(smem + tile + Keys::at(t, col >> 3) + (col & 7) * 2)); };
    auto across = [&](uint32_t tile, int row0, int s) { return tile + Keys::at(row0 + ln.t_row, 2 * s + (ln.t_col >> 3)); };   // for a transposing load
    auto state = [&](uint32_t tile, int s, int v, uint32_t (&y)[2][4]) {
        ldsm_trans(across(tile, v, s), y[0]);
        ldsm_trans(across(tile + lay.state_term, v, s), y[1]);
    };
    // q . x - beta k . y of rows' halves, this lane's part of sixteen dimensions from 16 s on
    auto meet = [&](float (&sum)[2], int s, const float (&x)[2][4], const float (&y)[2][4]) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float2 k = row_of(lay.k, t0 + 8 * h, s * 16 + 8 * m + 2 * c), q = row_of(lay.q, t0 + 8 * h, s * 16 + 8 * m + 2 * c);
                sum[h] += fmaf(q.x, x[m][2 * h], q.y * x[m][2 * h + 1]) - beta[h] * fmaf(k.x, y[m][2 * h], k.y * y[m][2 * h + 1]);
            }
    };
    // beta k . x, with beta k at hand
    auto meet_keys = [&](float (&sum)[2], const float2 (&k)[2][2], const float (&x)[2][4]) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[h] = fmaf(k[m][h].x, x[m][2 * h], fmaf(k[m][h].y, x[m][2 * h + 1], sum[h]));
    };
    auto join = [&](float (&x)[2][4], const float (&y)[2][4]) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(x[m], h, fadd2(pair(x[m], h), pair(y[m], h)));
    };
    auto scale = [&](float (&x)[2][4], const float (&f)[2]) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) set_pair(x[m], h, fmul2(pair(x[m], h), pack2(f[h], f[h])));
    };
    // sixteen key dimensions of dq, and o: the first bracket of dK (with its sign)
    auto with_s = [&](int s, float (&o)[2][4]) {
        float hq[2][4] = {}, h1[2][4] = {}, fq[2][4] = {}, f1[2][4] = {};
        if (before) {
#pragma unroll 2
            for (int v = 0; v < dvp; v += 16) {
                uint32_t da[1][4], ra[2][4], y[2][4];
                ldsm_a(b_of(dt, I * 16, v), da[0]);
                both_a(rt, I * 16, v, ra);
                state(st, s, v, y);
                add_products(hq, da, y);
                add_products(h1, ra, y);
            }
            scale(hq, eb);
            scale(h1, eb);
            meet(F, s, hq, h1);
        }
        if (I > 0) {
#pragma unroll
            for (int p = 0; p < 3; ++p)
                if (p < I) {
                    uint32_t y[1][4];
                    ldsm_trans(across(kt, p * 16, s), y[0]);
                    add_products(fq, xa[p], y);
                    add_products(f1, ea[p], y);
                }
            meet(R, s, fq, f1);
            join(hq, fq);
            join(h1, f1);
        }
#pragma unroll
        for (int p = 0; p < 4; ++p)
            if (p == I) {
                uint32_t y[1][4];
                ldsm_trans(across(kt, p * 16, s), y[0]);
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
                o[m][2 * h] = -beta[h] * h1[m][2 * h];
                o[m][2 * h + 1] = -beta[h] * h1[m][2 * h + 1];
                if (in && col < a.ldk) *reinterpret_cast<uint32_t*>(a.dq + r + col) = pack_bf16(hq[m][2 * h], hq[m][2 * h + 1]);
            }
        }
    };
    // the other two, and dk
    auto with_a = [&](int s, const float (&o)[2][4]) {
        float h2[2][4] = {};
        float2 k[2][2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                k[m][h] = row_of(lay.k, t0 + 8 * h, s * 16 + 8 * m + 2 * c);
                k[m][h].x *= beta[h];
                k[m][h].y *= beta[h];
            }
        if (behind) {
#pragma unroll 2
            for (int v = 0; v < dvp; v += 16) {
                uint32_t wa[2][4], y[2][4];
                both_a(wt, I * 16, v, wa);
                state(at, s, v, y);
                add_products(h2, wa, y);
            }
            scale(h2, dl);
            meet_keys(G, k, h2);
        }
#pragma unroll
        for (int p = 1; p < 5; ++p)
            if (p > I && p <= strips) {
                uint32_t y[1][4];
                float h3[2][4] = {};
                ldsm_trans(across(kt, (p - 1) * 16, s), y[0]);
                add_products(h3, ea[p], y);
                ldsm_trans(across(qt, (p - 1) * 16, s), y[0]);
                add_products(h3, xa[p], y);
                if (p > 1) meet_keys(C[p - 2], k, h3);   // (of the strip's own block, p = I + 1, it is not used)
                join(h2, h3);
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
    float* const sums = gates + (kF + (s0 == 0 ? 0 : kSums)) * kChunk;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = t0 + 8 * h;
        auto put_sum = [&](int row, float x) {
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            if (c == 0) sums[(row - kF) * kChunk + t] = x;
        };
        put_sum(kF, F[h]);
        put_sum(kG, G[h]);
        put_sum(kR, R[h]);
#pragma unroll
        for (int i = 1; i < 4; ++i)
            if (i > I) put_sum(kC1 + i - 1, C[i - 1][h]);
        if (c == 0 && s0 == 0 && n * kChunk + t < a.L) a.dbeta[a.row(unit, n * kChunk + t)] = __float2bfloat16_rn(db[h]);
    }
}

template <int DKP>
__global__ void __launch_bounds__(grad_threads<DKP>(), DKP <= 32 ? 3 : DKP <= 64 ? 2 : 1) gdr_grad_kernel(Gdr<bf> a, GdrKept kept, int chunks) {
    constexpr int kThreads = grad_threads<DKP>();
    using Keys = KeyRows<DKP>;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, dvp = kept.dvp;
    const GradLayout lay(DKP, dvp, grad_shares<DKP>());
    const long long unit = blockIdx.x / chunks;
    const int n = blockIdx.x % chunks, t0 = n * kChunk, nt = min(kChunk, a.L - t0);
    const long long here = unit * chunks + n;
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
        cp_async16(base + lay.k + Keys::at(t, e >> 3), a.k + at, in);
        cp_async16(base + lay.q + Keys::at(t, e >> 3), a.q + at, in);
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
    auto bring_state = [&](int to, const bf* from, bool there) {   // (nothing is read of one that is not)
        if (there)
            for (int i = tid; i < dvp * (DKP / 8); i += kThreads) {
                const int row = Keys::at(i / (DKP / 8), i % (DKP / 8));
#pragma unroll
                for (int m = 0; m < 2; ++m) cp_async16(base + to + m * lay.state_term + row, from + m * kept.state_term + (long long)i * 8, true);
            }
        cp_async_commit();
    };
    const bf *const S = kept.S + here * dvp * DKP, *const A = kept.A + here * dvp * DKP;
    if constexpr (!grad_shares<DKP>()) bring_state(lay.a, A, behind);
    bring_state(lay.s, S, before);
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
    float through = 0.f;   // what passes through all gates of the chunk: <S, A>
    auto meet = [&]() {
        if (!before || !behind) return;
        for (int i = tid; i < dvp * (DKP / 8); i += kThreads) {
            const unsigned char* const x = smem + lay.a + Keys::at(i / (DKP / 8), i % (DKP / 8));
            const bf* const y = S + (long long)i * 8;
            const uint4 xh = *reinterpret_cast<const uint4*>(x), xl = *reinterpret_cast<const uint4*>(x + lay.state_term), yh = *reinterpret_cast<const uint4*>(y),
                        yl = *reinterpret_cast<const uint4*>(y + kept.state_term);
            const uint32_t xs[2][4] = {{xh.x, xh.y, xh.z, xh.w}, {xl.x, xl.y, xl.z, xl.w}}, ys[2][4] = {{yh.x, yh.y, yh.z, yh.w}, {yl.x, yl.y, yl.z, yl.w}};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float u0, u1, v0, v1;
                unpack2(fadd2(widen_bf16(xs[0][q]), widen_bf16(xs[1][q])), u0, u1);
                unpack2(fadd2(widen_bf16(ys[0][q]), widen_bf16(ys[1][q])), v0, v1);
                through = fmaf(u0, v0, fmaf(u1, v1, through));
            }
        }
    };
    if constexpr (!grad_shares<DKP>()) meet();
    uint32_t seen = 0u;
    const int strip = warp & 3, half = warp >> 2, step = kThreads / 128;
    auto bring_a = [&]() {
        __syncthreads();
        bring_state(lay.a, A, behind);
        cp_async_wait<0>();
        __syncthreads();
        meet();
    };
    if (grad_shares<DKP>() || strip * 16 < nt) grad_strip<DKP>(strip, a, smem, lay, dvp, unit, n, before, behind, half, step, lane, seen, bring_a);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) through += __shfl_xor_sync(0xffffffffu, through, o);
    if (lane == 0) red[warp] = through;
    const int lost = __syncthreads_or(!within(seen, 3.3e38f));
    if (tid == 0) kept.lost_grad[here] = lost;
    if (warp == 0) {   // dlog_alpha, two tokens a lane
        float run = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) run += red[w];
        run *= gates[kEb * kChunk + kChunk - 1];
        const int t = 2 * lane, strip = lane >> 3;
        auto pair_at = [&](int row, bool there) {
            float2 x = row2(gates, row, t);
            if constexpr (kThreads > 128)
                if (row >= kF) {
                    const float2 y = row2(gates, row + kSums, t);
                    x = make_float2(x.x + y.x, x.y + y.y);
                }
            return there ? x : make_float2(0.f, 0.f);
        };
        const bool in = t < rows;
        const float2 f = pair_at(kF, in), g = pair_at(kG, in), r = pair_at(kR, in), own = pair_at(kOwn, in);
        // rows from t on: of all strips, and of the own one
        float d1 = run + f.y + behind_pair(f.x, f.y), d0 = d1 + f.x, low = r.x + r.y;
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
            const float y = __shfl_down_sync(0xffffffffu, low, o, 8);
            if ((lane & 7) + o < 8) low += y;
        }
        low = __shfl_down_sync(0xffffffffu, low, 1, 8);
        low = (lane & 7) == 7 ? 0.f : low;
        const float front = before_pair(g.x, g.y);
        d0 += front + own.x + (r.x + r.y + low);
        d1 += front + g.x + own.y + (r.y + low);
#pragma unroll
        for (int i = 1; i < 4; ++i) {   // pairs whose later token is in strip i, behind this one's
            const float2 x = pair_at(kC1 + i - 1, i * 16 < nt && strip < i);
            const float y = before_pair(x.x, x.y);
            if (strip < i) {
                d0 += y;
                d1 += y + x.x;
            }
        }
        if (t < nt) a.dla[a.row(unit, t0 + t)] = __float2bfloat16_rn(d0);
        if (t + 1 < nt) a.dla[a.row(unit, t0 + t + 1)] = __float2bfloat16_rn(d1);
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
