// The gated delta rule's gradient on the tensor cores (bf16 calls): what is left chunk by chunk once the two walks (gdr_chunk.cu) have W, dU and
// the states S before and A behind every chunk.  With Gam_ts = e^{b_t - b_s}, U = beta W, X = tril(dO U^T . Gam), E = strict_tril(dU U^T . Gam):
//
//   dQ = e^b dO S^T + X K
//   dK = - beta (e^b dU S^T + E K)  +  e^{b_C - b} U A^T + X^T Q - E'^T K          (E'^T: E^T with the beta of its columns)
//   dbeta_t = dU_t . W_t          dlog_alpha_t = e_t + .. + e_C + <S_C, A>,   e = q . dQ - beta dbeta + k . (the first bracket of dK)
//
// (E K's part of dK and e: replacing S by its decayed form shows e_t = q.dq - v.dv, and v = w + what k retrieves.)
// A block takes a chunk, a warp sixteen of its tokens as rows: the blocks of X and E up to the diagonal and those of their transposes from it
// on, five of each for every warp, so that no warp needs another's.  Sums over dv run in fp32 over fp16 operands that are scaled by powers of
// two: rows of K, Q and dO by their largest element, columns by what the walks kept them under.  64 x 12 units of 196 tokens, 32 x 64: 91 us for 112 MB, bound by
// instruction issue (3400 a warp, 160 of them products).
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

// Per token, arrays of kChunk floats: running sum of log2 alpha, 2^b, 2^{b_C - b}, beta, scales of the rows of K, Q and dO (2^e, ..), those of dO
// and Q together over their largest, beta 2^e, beta 2^{2e}, and e of a strip's first and second warp.
enum { kB, kEb, kDl, kBeta, kKu, kQu, kH, kHf, kGv, kGn, kE, kE2, kRows };

struct GradLayout {
    int kp, vp, k, q, d, r, w, s, a, gates, cols, total;
    __host__ __device__ GradLayout(int dkp, int dvp) {
        kp = dkp * 2 + 16;
        vp = dvp * 2 + 16;
        int at = 0;
        auto take = [&](int bytes) { const int o = at; at += bytes; return o; };
        k = take(kChunk * kp);
        q = take(kChunk * kp);
        d = take(kChunk * vp);
        r = take(kChunk * vp);
        w = take(kChunk * vp);
        s = take(dvp * kp);
        a = take(dvp * kp);
        gates = take(kChunk * kRows * 4);
        cols = take(dvp * 2 * 4 + 16 * 4);   // per column: y over the largest, and that times z over its largest; then what is reduced
        total = at;
    }
};

__device__ __forceinline__ void ldsm_a(uint32_t addr, uint32_t (&a)[4]) {
    uint32_t x[4];
    ldsm(addr, x);
    a[0] = x[0]; a[1] = x[2]; a[2] = x[1]; a[3] = x[3];
}
__device__ __forceinline__ float2 row2(const float* gates, int row, int t) { return *reinterpret_cast<const float2*>(gates + row * kChunk + t); }
__device__ __forceinline__ uint4 scale_halves(uint4 x, float s) {
    const __half2 f = __float2half2_rn(s);   // a power of two of at most one (zero below 2^-24: nothing is left of such a column beside the largest)
    __half2* h = reinterpret_cast<__half2*>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __hmul2(h[i], f);
    return x;
}

__device__ __forceinline__ f32x2 row_pair(const float* gates, int row, int t) { return *reinterpret_cast<const f32x2*>(gates + row * kChunk + t); }

// Strip I of the chunk; key dimensions in sixteens s0, s0 + step, ..  (I is a variable and the five blocks' code the same for all warps: with a
// copy for each strip, fetching instructions was what the warps waited for most, 173 us for 64 x 12 units of 196 tokens, 32 x 64.)
template <int DKP>
__device__ __forceinline__ void grad_strip(const int I, const Gdr<bf>& a, unsigned char* smem, const GradLayout& lay, int dvp, long long unit, int n, float Y,
                                           float Z, float HF, bool before, bool behind, int s0, int step, int lane, Largest& seen) {
    constexpr int KP = DKP * 2 + 16;
    const int g = lane >> 2, c = lane & 3, vp = lay.vp, strips = (min(kChunk, a.L - n * kChunk) + 15) >> 4;
    const Lane ln(lane);
    const uint32_t base = smem_u32(smem), kt = base + lay.k, qt = base + lay.q, dt = base + lay.d, rt = base + lay.r, wt = base + lay.w, st = base + lay.s,
                   at = base + lay.a;
    float* const gates = reinterpret_cast<float*>(smem + lay.gates);
    const int lane_at = ln.b_row * vp + ln.b_col * 2;
    auto b_of = [&](uint32_t tile, int row0, int col0) { return tile + lane_at + row0 * vp + col0 * 2; };
    // Block p: of dO W^T and dU W^T up to the diagonal (p <= I, columns of strip p), of W dO^T and W dU^T from it on (columns of strip p - 1)
    float x[5][2][4] = {}, e[5][2][4] = {};
#pragma unroll 1
    for (int v = 0; v < dvp; v += 16) {
        uint32_t da[4], ra[4], wa[4];
        ldsm_a(b_of(dt, I * 16, v), da);
        ldsm_a(b_of(rt, I * 16, v), ra);
        ldsm_a(b_of(wt, I * 16, v), wa);
#pragma unroll
        for (int p = 0; p < 5; ++p) {
            uint32_t y[4];
            if (p <= I) {
                ldsm(b_of(wt, p * 16, v), y);
                mma(x[p][0], da, y[0], y[1]);
                mma(x[p][1], da, y[2], y[3]);
                mma(e[p][0], ra, y[0], y[1]);
                mma(e[p][1], ra, y[2], y[3]);
            } else if (p <= strips) {
                ldsm(b_of(dt, (p - 1) * 16, v), y);
                mma(x[p][0], wa, y[0], y[1]);
                mma(x[p][1], wa, y[2], y[3]);
                ldsm(b_of(rt, (p - 1) * 16, v), y);
                mma(e[p][0], wa, y[0], y[1]);
                mma(e[p][1], wa, y[2], y[3]);
            }
        }
    }
    const int t0 = I * 16 + g;   // rows t0, t0 + 8
    const float bt[2] = {gates[kB * kChunk + t0], gates[kB * kChunk + t0 + 8]}, beta[2] = {gates[kBeta * kChunk + t0], gates[kBeta * kChunk + t0 + 8]},
                ku[2] = {gates[kKu * kChunk + t0], gates[kKu * kChunk + t0 + 8]};
    const float end = gates[kB * kChunk + I * 16 + 15];
    float db[2] = {0.f, 0.f};
    // to operands, e^{b_t - b_s} by way of the last token of s' sixteen off the diagonal (both factors are at most one)
    uint32_t xa[5][4], ea[5][4];
#pragma unroll
    for (int p = 0; p < 5; ++p) {
        const bool low = p <= I;
        const int j = low ? p : p - 1;
        if (j >= strips) {   // (no tokens there, and nothing in shared memory)
#pragma unroll
            for (int h = 0; h < 4; ++h) xa[p][h] = ea[p][h] = 0u;
        } else if (j != I) {
            const float ref = low ? gates[kB * kChunk + j * 16 + 15] : end;
            f32x2 er[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float r = ex2(low ? bt[h] - ref : ref - bt[h]);
                er[h] = pack2(r, r);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int col = j * 16 + 8 * m + 2 * c;
                const float2 bc = row2(gates, kB, col);
                f32x2 fx = pack2(ex2(low ? ref - bc.x : bc.x - ref), ex2(low ? ref - bc.y : bc.y - ref)), fe = fx;
                if (low) fe = fx = fmul2(fx, row_pair(gates, kGv, col));   // columns s: times 2^e beta_s
                else {                                                      // columns t: times the scale of dO's and q's rows, or - beta_t 2^{2e}
                    fx = fmul2(fx, row_pair(gates, kHf, col));
                    fe = fmul2(fmul2(fe, row_pair(gates, kGn, col)), pack2(-1.f, -1.f));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    xa[p][2 * m + h] = pack_half(fmul2(pair(x[p][m], h), fmul2(fx, er[h])));
                    ea[p][2 * m + h] = pack_half(fmul2(pair(e[p][m], h), fmul2(fe, er[h])));
                }
            }
        } else {
            if (low)   // dbeta: the diagonal of dU W^T, row g + 8 h and the same column: in lane c = g / 2
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float d = g & 1 ? e[p][h][2 * h + 1] : e[p][h][2 * h];
                    db[h] = __shfl_sync(0xffffffffu, d, (lane & 28) | (g >> 1)) * ku[h] * Y * Z;
                }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int cc = 8 * m + 2 * c, col = I * 16 + cc;
                const float2 bc = row2(gates, kB, col), fx = row2(gates, low ? kGv : kHf, col), fe = row2(gates, low ? kGv : kGn, col);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = g + 8 * h;
                    float xx[2], ee[2];
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const bool in = low ? cc + f <= row : cc + f >= row, strict = in && cc + f != row;
                        const float gam = in ? ex2(low ? bt[h] - (f ? bc.y : bc.x) : (f ? bc.y : bc.x) - bt[h]) : 0.f;
                        xx[f] = in ? x[p][m][2 * h + f] * gam * (f ? fx.y : fx.x) : 0.f;
                        ee[f] = strict ? e[p][m][2 * h + f] * gam * (f ? fe.y : fe.x) * (low ? 1.f : -1.f) : 0.f;
                    }
                    xa[p][2 * m + h] = pack_half(xx[0], xx[1]);
                    ea[p][2 * m + h] = pack_half(ee[0], ee[1]);
                }
            }
        }
        seen.see(xa[p]);
        seen.see(ea[p]);
    }
    const float eb[2] = {gates[kEb * kChunk + t0], gates[kEb * kChunk + t0 + 8]}, dl[2] = {gates[kDl * kChunk + t0], gates[kDl * kChunk + t0 + 8]};
    const float qs[2] = {gates[kH * kChunk + t0] * Y, gates[kH * kChunk + t0 + 8] * Y};
    float sum[2] = {0.f, 0.f};
#pragma unroll 1
    for (int s = s0; s < DKP / 16; s += step) {
        float hq[2][4] = {}, h1[2][4] = {}, h2[2][4] = {}, h3[2][4] = {};
        if (before)
#pragma unroll 2
            for (int v = 0; v < dvp; v += 16) {
                uint32_t da[4], ra[4], y[4];
                ldsm_a(b_of(dt, I * 16, v), da);
                ldsm_a(b_of(rt, I * 16, v), ra);
                ldsm_trans(at_t<KP>(ln, st, v, s * 16), y);
                mma(hq[0], da, y[0], y[1]);
                mma(hq[1], da, y[2], y[3]);
                mma(h1[0], ra, y[0], y[1]);
                mma(h1[1], ra, y[2], y[3]);
            }
        if (behind)
#pragma unroll 2
            for (int v = 0; v < dvp; v += 16) {
                uint32_t wa[4], y[4];
                ldsm_a(b_of(wt, I * 16, v), wa);
                ldsm_trans(at_t<KP>(ln, at, v, s * 16), y);
                mma(h2[0], wa, y[0], y[1]);
                mma(h2[1], wa, y[2], y[3]);
            }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                set_pair(hq[m], h, fmul2(pair(hq[m], h), pack2(eb[h], eb[h])));
                set_pair(h1[m], h, fmul2(pair(h1[m], h), pack2(eb[h], eb[h])));
                set_pair(h2[m], h, fmul2(pair(h2[m], h), pack2(dl[h], dl[h])));
            }
#pragma unroll
        for (int p = 0; p < 5; ++p) {
            uint32_t y[4];
            if (p <= I) {
                ldsm_trans(at_t<KP>(ln, kt, p * 16, s * 16), y);
                mma(hq[0], xa[p], y[0], y[1]);
                mma(hq[1], xa[p], y[2], y[3]);
                mma(h1[0], ea[p], y[0], y[1]);
                mma(h1[1], ea[p], y[2], y[3]);
            } else if (p <= strips) {
                ldsm_trans(at_t<KP>(ln, kt, (p - 1) * 16, s * 16), y);
                mma(h2[0], ea[p], y[0], y[1]);
                mma(h2[1], ea[p], y[2], y[3]);
                ldsm_trans(at_t<KP>(ln, qt, (p - 1) * 16, s * 16), y);
                mma(h3[0], xa[p], y[0], y[1]);
                mma(h3[1], xa[p], y[2], y[3]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = t0 + 8 * h;
            const bool in = n * kChunk + t < a.L;
            const long long r = in ? a.row(unit, n * kChunk + t) * a.ldk : 0;
            const float step1 = -beta[h] * ku[h] * Y, qu = gates[kQu * kChunk + t];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int col = s * 16 + 8 * m + 2 * c;
                const float2 kk = unpack_half(*reinterpret_cast<const uint32_t*>(smem + lay.k + t * KP + col * 2)),
                             qq = unpack_half(*reinterpret_cast<const uint32_t*>(smem + lay.q + t * KP + col * 2));
                const float q0 = qs[h] * hq[m][2 * h], q1 = qs[h] * hq[m][2 * h + 1], o0 = step1 * h1[m][2 * h] * Z, o1 = step1 * h1[m][2 * h + 1] * Z;
                const float k0 = o0 + beta[h] * Y * (h2[m][2 * h] * Z + h3[m][2 * h] * HF), k1 = o1 + beta[h] * Y * (h2[m][2 * h + 1] * Z + h3[m][2 * h + 1] * HF);
                sum[h] += qu * (qq.x * q0 + qq.y * q1) + ku[h] * (kk.x * o0 + kk.y * o1);
                if (in && col < a.ldk) {
                    *reinterpret_cast<uint32_t*>(a.dq + r + col) = pack_bf16(q0, q1);
                    *reinterpret_cast<uint32_t*>(a.dk_out + r + col) = pack_bf16(k0, k1);
                }
            }
        }
    }
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
__global__ void __launch_bounds__(grad_threads<DKP>(), DKP <= 32 ? 4 : DKP <= 64 ? 2 : 1) gdr_grad_kernel(Gdr<bf> a, GdrKept kept, int chunks) {
    constexpr int KP = DKP * 2 + 16, kThreads = grad_threads<DKP>();
    constexpr int kLanes = DKP <= 16 ? 2 : DKP <= 32 ? 4 : DKP <= 64 ? 8 : 16;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, dvp = kept.dvp;
    const GradLayout lay(DKP, dvp);
    const long long unit = blockIdx.x / chunks;
    const int n = blockIdx.x % chunks, t0 = n * kChunk, nt = min(kChunk, a.L - t0);
    const long long here = unit * chunks + n, states = unit * (chunks + 1) + n;
    float* const gates = reinterpret_cast<float*>(smem + lay.gates);
    float *const cy = reinterpret_cast<float*>(smem + lay.cols), *const cyz = cy + dvp, *const red = cyz + dvp;
    pdl_wait();
    pdl_launch_dependents();
    // everything comes in by asynchronous copies at once, and is turned into operands where it lies; rows up to the last strip with tokens
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
            cp_async16(base + lay.w + to, kept.w + at, in);
            cp_async16(base + lay.r + to, kept.du + at, in);
            const bool values = in && piece < a.ldv;
            cp_async16(base + lay.d + to, a.d_out + (values ? a.row(unit, t0 + t) * a.ldv + piece : 0), values);
        }
    for (int i = tid; i < dvp * (DKP / 8); i += kThreads) {
        const int j = i / (DKP / 8), e = i % (DKP / 8) * 8;
        if (before) cp_async16(base + lay.s + j * KP + e * 2, kept.S + (states * dvp + j) * DKP + e, true);
        if (behind) cp_async16(base + lay.a + j * KP + e * 2, kept.A + (here * dvp + j) * DKP + e, true);
    }
    cp_async_commit();
    // the state behind the chunk, for the gradient that the next chunk's first gate sees
    constexpr int kBehind = 128 * (DKP / 8) / kThreads;   // pieces of a thread, at most
    uint4 next[kBehind];
#pragma unroll
    for (int p = 0; p < kBehind; ++p) {
        const int i = tid + p * kThreads;
        if (behind && i < dvp * (DKP / 8)) next[p] = *reinterpret_cast<const uint4*>(kept.S + (states + 1) * dvp * DKP + i * 8);
    }
    // columns: their powers of two over the largest
    float Y = 0.f, Z = 0.f;
    for (int j = lane; j < dvp; j += 32) {
        Y = fmaxf(Y, kept.y[states * dvp + j]);
        Z = fmaxf(Z, kept.z[here * dvp + j]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Y = fmaxf(Y, __shfl_xor_sync(0xffffffffu, Y, o));
        Z = fmaxf(Z, __shfl_xor_sync(0xffffffffu, Z, o));
    }
    for (int j = tid; j < dvp; j += kThreads) {
        const float y = kept.y[states * dvp + j] / Y;
        cy[j] = y;
        cyz[j] = y * (kept.z[here * dvp + j] / Z);
    }
    if (warp == 0) {   // gates, as the walks have them
        float l[2], s[2], be[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = 2 * lane + h;
            const float x = t < nt ? __bfloat162float(a.la[a.row(unit, t0 + t)]) * 1.4426950408889634f : 0.f;
            l[h] = x < -160.f ? -160.f : x;
            be[h] = t < nt ? __bfloat162float(a.beta[a.row(unit, t0 + t)]) : 0.f;
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
    cp_async_wait<0>();
    __syncthreads();
    // K, Q to fp16 under their rows' powers of two
#pragma unroll
    for (int p = 0; p < 2 * kChunk * kLanes / kThreads; ++p) {
        const int i = tid + p * kThreads, r = i / kLanes, e8 = i % kLanes * 8, t = r & (kChunk - 1);
        const bool key = r < kChunk;
        if (p * kThreads / kLanes % kChunk >= rows) continue;   // the first of the pass's rows
        uint4* const at = reinterpret_cast<uint4*>(smem + (key ? lay.k : lay.q) + t * KP + e8 * 2);
        const uint4 x = e8 < DKP && t < rows ? *at : make_uint4(0u, 0u, 0u, 0u);
        uint32_t m = largest_bf16(x);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        float down, up;
        power_of(m >> 7, down, up);
        if (e8 < DKP && t < rows) *at = bf16_to_half(x, down);
        if (e8 == 0) {
            gates[(key ? kKu : kQu) * kChunk + t] = up;
            if (key) {
                const float gv = gates[kBeta * kChunk + t] * up;
                gates[kGv * kChunk + t] = gv;
                gates[kGn * kChunk + t] = gv * up;
            }
        }
    }
    // dO under its rows' and its columns' powers of two, dU under its columns'
    {
        f32x2 fy[4];
        __half2 fz[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            fy[p] = piece < dvp ? *reinterpret_cast<const f32x2*>(cy + piece + 2 * p) : 0ull;
            fz[p] = piece < dvp ? __floats2half2_rn(cyz[piece + 2 * p], cyz[piece + 2 * p + 1]) : __float2half2_rn(0.f);
        }
        // (whole warps: a warp's rows, at most sixteen, are either all there or all not)
        for (int t = tid >> lg; t < rows; t += kThreads >> lg) {
            uint4* const at = reinterpret_cast<uint4*>(smem + lay.d + t * lay.vp + piece * 2);
            const uint4 x = piece < dvp ? *at : make_uint4(0u, 0u, 0u, 0u);
            uint32_t m = largest_bf16(x);
            for (int o = 1; o < 1 << lg; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            float down, up;
            power_of(m >> 7, down, up);
            if (piece < dvp) {
                const f32x2 dn = pack2(down, down);
                *at = make_uint4(pack_half(fmul2(fmul2(widen_bf16(x.x), dn), fy[0])), pack_half(fmul2(fmul2(widen_bf16(x.y), dn), fy[1])),
                                 pack_half(fmul2(fmul2(widen_bf16(x.z), dn), fy[2])), pack_half(fmul2(fmul2(widen_bf16(x.w), dn), fy[3])));
                uint4* const ar = reinterpret_cast<uint4*>(smem + lay.r + t * lay.vp + piece * 2);
                uint4 y = *ar;
                __half2* const h = reinterpret_cast<__half2*>(&y);
#pragma unroll
                for (int p = 0; p < 4; ++p) h[p] = __hmul2(h[p], fz[p]);
                *ar = y;
            }
            if (piece == 0) gates[kH * kChunk + t] = up;
        }
    }
    // A under its columns' powers of two, and its product with the state behind the chunk
    float anchor = 0.f;
#pragma unroll
    for (int p = 0; p < kBehind; ++p) {
        const int i = tid + p * kThreads, j = i / (DKP / 8), e = i % (DKP / 8) * 8;
        if (behind && i < dvp * (DKP / 8)) {
            uint4* const at = reinterpret_cast<uint4*>(smem + lay.a + j * KP + e * 2);
            const uint4 x = *at;
            *at = scale_halves(x, cyz[j]);
            {
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ss[4] = {next[p].x, next[p].y, next[p].z, next[p].w};
                float dot = 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float2 u = unpack_half(xs[q]), v = unpack_half(ss[q]);
                    dot = fmaf(u.x, v.x, fmaf(u.y, v.y, dot));
                }
                anchor = fmaf(dot * kept.y[(states + 1) * dvp + j], kept.z[here * dvp + j], anchor);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) anchor += __shfl_xor_sync(0xffffffffu, anchor, o);
    if (lane == 0) red[warp] = anchor;
    __syncthreads();
    // the scales of dO's and q's rows together, over the largest
    float HF = 0.f;
    {
        const float p = lane < rows ? gates[kH * kChunk + lane] * gates[kQu * kChunk + lane] : 0.f,
                    q = lane + 32 < rows ? gates[kH * kChunk + lane + 32] * gates[kQu * kChunk + lane + 32] : 0.f;
        HF = fmaxf(p, q);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) HF = fmaxf(HF, __shfl_xor_sync(0xffffffffu, HF, o));
        if (warp == 0) {
            gates[kHf * kChunk + lane] = p / HF;
            gates[kHf * kChunk + lane + 32] = q / HF;
        }
    }
    __syncthreads();
    Largest seen;
    const int strip = warp & 3, half = warp >> 2, step = kThreads / 128;
    if (strip * 16 < nt) grad_strip<DKP>(strip, a, smem, lay, dvp, unit, n, Y, Z, HF, before, behind, half, step, lane, seen);
    const int lost = __syncthreads_or(seen.lost());
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
        const int smem = GradLayout(dkp, kept.dvp).total;
        cudaError_t e = allow_smem<gdr_grad_kernel<dkp>>(GradLayout(dkp, kMostColumns).total);
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
