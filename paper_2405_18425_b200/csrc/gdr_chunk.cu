// The gated delta rule's forward pass in chunks of 64 tokens on the tensor cores (bf16 calls).
//
// With b the running sum of log alpha in a chunk, Gam_ts = e^{b_t - b_s}, N = strict_tril(K K^T . Gam), P = tril(Q K^T . Gam):
//   U = beta (V - e^b K S - N U)         O = e^b Q S + P U         S <- e^{b_C} S + (e^{b_C - b} K)^T U
// The triangular system is solved sixteen tokens at a time: what the sixteen before contribute is a product with N, what the sixteen do to
// one another a product with the inverse of 1 + beta N of their own 16 x 16 block, which one warp computes by substitution in fp32.
// e^{b_t - b_s} is taken of the difference, never of its parts, so that no gate is out of range.
//
// A block is a unit's chunk loop for up to 64 columns; its warps share the staging and the token-by-token matrices and own sixteen columns
// each (gdr_tile.cuh).  The next chunk's rows arrive by asynchronous copies meanwhile.
#include <type_traits>

#include "gdr.h"
#include "gdr_tile.cuh"

namespace vig {
namespace {

using namespace gdr;
using bf = __nv_bfloat16;

constexpr int kMostWarps = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMatPitch = kChunk * 2 + 16, kInvPitch = 48;

template <int DKP>
constexpr int key_pitch() { return DKP * 2 + 16; }

// Shared memory, in bytes.
template <int DKP, bool EXACT>
struct Layout {
    static constexpr int kKeys = kChunk * key_pitch<DKP>();
    int k[2], q[2], v[2], n, p, inv, n_lo, inv_lo, x, gates, total;
    __host__ __device__ explicit Layout(int warps) {
        const int vb = kChunk * (warps * 32 + 16);
        int at = 0;
        auto take = [&](int bytes) { const int o = at; at += bytes; return o; };
        for (int i = 0; i < 2; ++i) {
            k[i] = take(kKeys);
            q[i] = take(kKeys);
            v[i] = take(vb);
        }
        n = take(kChunk * kMatPitch);
        p = take(kChunk * kMatPitch);
        inv = take(kChunk * kInvPitch);
        n_lo = EXACT ? take(kChunk * kMatPitch) : 0;
        inv_lo = EXACT ? take(kChunk * kInvPitch) : 0;
        x = take(4 * 16 * 20 * 4);          // the diagonal blocks of beta N, transposed, rows of 20 floats
        gates = take(kChunk * 8 * 4);
        total = at;
    }
};

// Per token of the chunk, in shared memory.
struct Gates {
    float b;      // running sum of log2 alpha
    float eb;     // e^b
    float dl;     // e^{b_C - b}
    float beta;
    float gv;     // beta 2^e: the step from outside
    float gn;     // beta 2^{2e}: what S and U give, times this
    float ku;     // 2^e of the key's row
    float qu;     // 2^e of the query's row
};

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

// EXACT: states leave the call, so that what S is made of is taken with 22 bits (two fp16 an operand); otherwise only bf16 results do, and
// eleven bits keep the error below a quarter of their rounding.
template <int DKP, bool EXACT>
__global__ void __launch_bounds__(32 * kMostWarps) gdr_chunk_kernel(Gdr<bf> a, int slabs, int* status) {
    constexpr int KP = key_pitch<DKP>(), KS = DKP / 16;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5, nth = blockDim.x;
    const int g = lane >> 2, c = lane & 3;
    const Layout<DKP, EXACT> lay(warps);
    const uint32_t base = smem_u32(smem);
    const int vp = warps * 32 + 16;
    Gates* const gates = reinterpret_cast<Gates*>(smem + lay.gates);
    const long long unit = blockIdx.x / slabs;
    const int j0 = blockIdx.x % slabs * warps * 16;
    const int chunks = (a.L + kChunk - 1) / kChunk;
    const Lane ln(lane);

    auto fetch = [&](int n, int buf) {
        const int t0 = n * kChunk, key_pieces = DKP / 8, v_pieces = warps * 2;
        for (int i = tid; i < kChunk * key_pieces; i += nth) {
            const int t = i / key_pieces, e = i % key_pieces * 8;
            const bool in = t0 + t < a.L && e < a.dk;
            const long long src = in ? a.row(unit, t0 + t) * a.dk + e : 0;
            cp_async16(base + lay.k[buf] + t * KP + e * 2, a.k + src, in);
            cp_async16(base + lay.q[buf] + t * KP + e * 2, a.q + src, in);
        }
        for (int i = tid; i < kChunk * v_pieces; i += nth) {
            const int t = i / v_pieces, e = i % v_pieces * 8;
            const bool in = t0 + t < a.L && j0 + e < a.dv;
            cp_async16(base + lay.v[buf] + t * vp + e * 2, a.v + (in ? a.row(unit, t0 + t) * a.dv + j0 + e : 0), in);
        }
        cp_async_commit();
    };

    pdl_wait();
    pdl_launch_dependents();
    fetch(0, 0);

    // this warp's columns of S, transposed: tile n holds key dimensions 8n + 2c, + 1 of columns g (0, 1) and g + 8 (2, 3)
    float S[2 * KS][4];
    const int col = j0 + warp * 16 + g;
    const long long plane = (long long)a.dk * a.dv;
#pragma unroll
    for (int n = 0; n < 2 * KS; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = n * 8 + 2 * c + (e & 1), j = col + (e >> 1) * 8;
            S[n][e] = a.state_in && i < a.dk && j < a.dv ? a.state_in[unit * plane + (long long)i * a.dv + j] : 0.f;
        }
    float scale[2] = {1.f, 1.f};   // S holds the state times this, a power of two per column
    Largest seen;

    for (int n = 0; n < chunks; ++n) {
        const int buf = n & 1, t0 = n * kChunk, nt = min(kChunk, a.L - t0), strips = (nt + 15) >> 4;
        if (n + 1 < chunks) {
            fetch(n + 1, buf ^ 1);
            cp_async_wait<1>();
        } else cp_async_wait<0>();
        // gates: running sum of log2 alpha over the chunk, two tokens a lane
        if (warp == 0) {
            float l[2], s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = 2 * lane + h;
                // (below 2^-150 nothing of the state is left in fp32; the bound keeps sums of such gates exact to 2^-11)
                const float x = t < nt ? __bfloat162float(a.la[a.row(unit, t0 + t)]) * kLog2e : 0.f;
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
            const float before = run - s[1], all = __shfl_sync(0xffffffffu, run, 31);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = 2 * lane + h;
                const float b = before + s[h];
                gates[t].b = b;
                gates[t].eb = ex2(b);
                gates[t].dl = ex2(all - b);
                gates[t].beta = t < nt ? __bfloat162float(a.beta[a.row(unit, t0 + t)]) : 0.f;
            }
        }
        __syncthreads();
        // K and Q to fp16, each row over its largest element's power of two, in place
        {
            constexpr int kLanes = DKP <= 16 ? 2 : DKP <= 32 ? 4 : DKP <= 64 ? 8 : 16;   // of a row
            for (int i = tid; i < 2 * kChunk * kLanes; i += nth) {
                const int r = i / kLanes, e = i % kLanes, t = r & (kChunk - 1);
                const bool key = r < kChunk, in = e * 8 < DKP;
                uint4* const p = reinterpret_cast<uint4*>(smem + (key ? lay.k[buf] : lay.q[buf]) + t * KP + e * 16);
                uint4 x = in ? *p : make_uint4(0u, 0u, 0u, 0u);
                uint32_t m = max(max(max(x.x & 0x7fffu, x.x >> 16 & 0x7fffu), max(x.y & 0x7fffu, x.y >> 16 & 0x7fffu)),
                                 max(max(x.z & 0x7fffu, x.z >> 16 & 0x7fffu), max(x.w & 0x7fffu, x.w >> 16 & 0x7fffu)));
#pragma unroll
                for (int o = 1; o < kLanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                float down, up;
                power_of(m >> 7, down, up);
                auto half2_of = [&](uint32_t y) { return pack_half(__uint_as_float(y << 16) * down, __uint_as_float(y & 0xffff0000u) * down); };
                if (in) *p = make_uint4(half2_of(x.x), half2_of(x.y), half2_of(x.z), half2_of(x.w));
                if (e == 0) {
                    if (key) {
                        const float gv = gates[t].beta * up;
                        gates[t].gv = gv;
                        gates[t].gn = gv * up;
                        gates[t].ku = up;
                    } else gates[t].qu = up;
                }
            }
        }
        __syncthreads();
        // N and P by blocks of sixteen by sixteen; the diagonal ones first, their inverses take longest
        const uint32_t kt = base + lay.k[buf], qt = base + lay.q[buf], vt = base + lay.v[buf];
        for (int w = warp; w < 10; w += warps) {
            // 0 .. 3: the diagonal; then (1,0) (2,0) (2,1) (3,0) (3,1) (3,2)
            const int i = w < 4 ? w : w == 4 ? 1 : w < 7 ? 2 : 3, j = w < 4 ? w : w == 4 ? 0 : w < 7 ? w - 5 : w - 7;
            if (i >= strips) continue;
            float nn[2][4] = {}, pp[2][4] = {};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t kb[4], ka[4], qa[4], x[4];
                ldsm(at_b<KP>(ln, kt, j * 16, s * 16), kb);
                ldsm(at_b<KP>(ln, qt, i * 16, s * 16), x);
                qa[0] = x[0]; qa[1] = x[2]; qa[2] = x[1]; qa[3] = x[3];
                ldsm(at_b<KP>(ln, kt, i * 16, s * 16), x);
                ka[0] = x[0]; ka[1] = x[2]; ka[2] = x[1]; ka[3] = x[3];
                mma(nn[0], ka, kb[0], kb[1]);
                mma(nn[1], ka, kb[2], kb[3]);
                mma(pp[0], qa, kb[0], kb[1]);
                mma(pp[1], qa, kb[2], kb[3]);
            }
            float* const xt = reinterpret_cast<float*>(smem + lay.x) + i * 16 * 20;
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // rows g, g + 8
                const int t = i * 16 + g + 8 * h;
                const float bt = gates[t].b, gn = gates[t].gn;
#pragma unroll
                for (int m = 0; m < 2; ++m) {   // columns 8m + 2c, + 1
                    const int s = j * 16 + 8 * m + 2 * c;
                    const float e0 = s <= t ? ex2(bt - gates[s].b) : 0.f, e1 = s + 1 <= t ? ex2(bt - gates[s + 1].b) : 0.f;
                    const float p0 = s <= t ? pp[m][2 * h] * e0 : 0.f, p1 = s + 1 <= t ? pp[m][2 * h + 1] * e1 : 0.f;
                    *reinterpret_cast<uint32_t*>(smem + lay.p + t * kMatPitch + s * 2) = pack_half(p0, p1);
                    if (i != j) {
                        const float n0 = nn[m][2 * h] * e0, n1 = nn[m][2 * h + 1] * e1;
                        const uint32_t hi = pack_half(n0, n1);
                        *reinterpret_cast<uint32_t*>(smem + lay.n + t * kMatPitch + s * 2) = hi;
                        if constexpr (EXACT) *reinterpret_cast<uint32_t*>(smem + lay.n_lo + t * kMatPitch + s * 2) = rest_half(n0, n1, hi);
                    } else {   // beta N, transposed: row s, column t
                        const int ss = 8 * m + 2 * c, tt = g + 8 * h;
                        xt[ss * 20 + tt] = ss < tt ? nn[m][2 * h] * e0 * gn : 0.f;
                        xt[(ss + 1) * 20 + tt] = ss + 1 < tt ? nn[m][2 * h + 1] * e1 * gn : 0.f;
                    }
                }
            }
            if (i == j) {
                __syncwarp();
                // (1 + beta N)^-1, a column a lane: x_t -= (beta N)_ts x_s as soon as x_s is known
                float x[16];
                const int cc = lane & 15;
#pragma unroll
                for (int t = 0; t < 16; ++t) x[t] = t == cc ? 1.f : 0.f;
#pragma unroll
                for (int s = 0; s < 15; ++s) {
#pragma unroll
                    for (int p = (s + 1) / 4; p < 4; ++p) {
                        const float4 r = *reinterpret_cast<const float4*>(xt + s * 20 + 4 * p);
                        x[4 * p] = fmaf(-r.x, 4 * p > s ? x[s] : 0.f, x[4 * p]);
                        x[4 * p + 1] = fmaf(-r.y, 4 * p + 1 > s ? x[s] : 0.f, x[4 * p + 1]);
                        x[4 * p + 2] = fmaf(-r.z, 4 * p + 2 > s ? x[s] : 0.f, x[4 * p + 2]);
                        x[4 * p + 3] = fmaf(-r.w, 4 * p + 3 > s ? x[s] : 0.f, x[4 * p + 3]);
                    }
                }
                if (lane < 16)
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        const __half hi = __float2half_rn(x[t]);
                        *reinterpret_cast<__half*>(smem + lay.inv + (i * 16 + t) * kInvPitch + cc * 2) = hi;
                        if constexpr (EXACT)
                            *reinterpret_cast<__half*>(smem + lay.inv_lo + (i * 16 + t) * kInvPitch + cc * 2) = __float2half_rn(x[t] - __half2float(hi));
                    }
            }
        }
        __syncthreads();

        // this warp's columns: scale of the chunk
        float gmax = fmaxf(fabsf(gates[lane].gv), fabsf(gates[lane + 32].gv)), smax[2] = {0.f, 0.f}, vmax[2] = {0.f, 0.f};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) gmax = fmaxf(gmax, __shfl_xor_sync(0xffffffffu, gmax, o));
        uint32_t vv[4][4];   // V transposed: strip i, columns g / g + 8 of tokens 2c, 2c + 1 / + 8
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t x[4];
            ldsm_trans(vt + (i * 16 + ln.t_row) * vp + (warp * 16 + ln.t_col) * 2, x);
            vv[i][0] = x[0]; vv[i][1] = x[2]; vv[i][2] = x[1]; vv[i][3] = x[3];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint32_t y = vv[i][2 * m + h];
                    vmax[h] = fmaxf(vmax[h], fmaxf(fabsf(__uint_as_float(y << 16)), fabsf(__uint_as_float(y & 0xffff0000u))));
                }
        }
#pragma unroll
        for (int m = 0; m < 2 * KS; ++m) {
            smax[0] = fmaxf(smax[0], fmaxf(fabsf(S[m][0]), fabsf(S[m][1])));
            smax[1] = fmaxf(smax[1], fmaxf(fabsf(S[m][2]), fabsf(S[m][3])));
        }
        float back[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                smax[h] = fmaxf(smax[h], __shfl_xor_sync(0xffffffffu, smax[h], o));
                vmax[h] = fmaxf(vmax[h], __shfl_xor_sync(0xffffffffu, vmax[h], o));
            }
            const float most = fmaxf(vmax[h] * gmax, smax[h] / scale[h]);   // (a power of two: exact)
            const uint32_t ex = min(max(__float_as_uint(most) >> 23, 4u), 250u);
            const float now = __uint_as_float((256u - ex) << 23);   // the largest to [4, 8)
            back[h] = __uint_as_float((ex - 2u) << 23);
            const float change = now / scale[h];
            scale[h] = now;
#pragma unroll
            for (int m = 0; m < 2 * KS; ++m) {
                S[m][2 * h] *= change;
                S[m][2 * h + 1] *= change;
            }
        }
        uint32_t sa[KS][4], sl[EXACT ? KS : 1][4];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            pack_a(S[2 * s], S[2 * s + 1], sa[s]);
            seen.see(sa[s]);
            if constexpr (EXACT) pack_a_rest(S[2 * s], S[2 * s + 1], sa[s], sl[s]);
        }
        const float all = gates[kChunk - 1].eb;
#pragma unroll
        for (int m = 0; m < 2 * KS; ++m) {
#pragma unroll
            for (int e = 0; e < 4; ++e) S[m][e] *= all;
        }
        uint32_t u[4][4], ul[EXACT ? 4 : 1][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= strips) break;
            float w[2][4] = {}, o[2][4] = {};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t x[4];
                ldsm(at_b<KP>(ln, kt, i * 16, s * 16), x);
                mma(w[0], sa[s], x[0], x[1]);
                mma(w[1], sa[s], x[2], x[3]);
                if constexpr (EXACT) {
                    mma(w[0], sl[s], x[0], x[1]);
                    mma(w[1], sl[s], x[2], x[3]);
                }
                ldsm(at_b<KP>(ln, qt, i * 16, s * 16), x);
                mma(o[0], sa[s], x[0], x[1]);
                mma(o[1], sa[s], x[2], x[3]);
            }
            Gates gt[2][2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    gt[m][e] = gates[i * 16 + 8 * m + 2 * c + e];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        w[m][2 * h + e] *= gt[m][e].eb;
                        o[m][2 * h + e] *= gt[m][e].eb;
                    }
                }
#pragma unroll
            for (int j = 0; j < i; ++j) {
                uint32_t x[4], y[4];
                ldsm(at_b<kMatPitch>(ln, base + lay.n, i * 16, j * 16), x);
                mma(w[0], u[j], x[0], x[1]);
                mma(w[1], u[j], x[2], x[3]);
                if constexpr (EXACT) {
                    mma(w[0], ul[j], x[0], x[1]);
                    mma(w[1], ul[j], x[2], x[3]);
                    ldsm(at_b<kMatPitch>(ln, base + lay.n_lo, i * 16, j * 16), y);
                    mma(w[0], u[j], y[0], y[1]);
                    mma(w[1], u[j], y[2], y[3]);
                }
            }
            // beta 2^e (v - 2^e ..)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t y = vv[i][2 * m + h];
                    w[m][2 * h] = fmaf(__uint_as_float(y << 16) * gt[m][0].gv, scale[h], -gt[m][0].gn * w[m][2 * h]);
                    w[m][2 * h + 1] = fmaf(__uint_as_float(y & 0xffff0000u) * gt[m][1].gv, scale[h], -gt[m][1].gn * w[m][2 * h + 1]);
                }
            uint32_t wa[4], x[4];
            float uu[2][4] = {};
            pack_a(w[0], w[1], wa);
            seen.see(wa);
            ldsm(at_b<kInvPitch>(ln, base + lay.inv, i * 16, 0), x);
            mma(uu[0], wa, x[0], x[1]);
            mma(uu[1], wa, x[2], x[3]);
            if constexpr (EXACT) {
                uint32_t wl[4], y[4];
                pack_a_rest(w[0], w[1], wa, wl);
                mma(uu[0], wl, x[0], x[1]);
                mma(uu[1], wl, x[2], x[3]);
                ldsm(at_b<kInvPitch>(ln, base + lay.inv_lo, i * 16, 0), y);
                mma(uu[0], wa, y[0], y[1]);
                mma(uu[1], wa, y[2], y[3]);
            }
            pack_a(uu[0], uu[1], u[i]);
            if constexpr (EXACT) pack_a_rest(uu[0], uu[1], u[i], ul[i]);
            seen.see(u[i]);
            // S += (e^{b_C - b} U)^T K
            uint32_t ud[4];
            float du[2][4];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) du[m][e] = uu[m][e] * gt[m][e & 1].dl;
            pack_a(du[0], du[1], ud);
            uint32_t udl[4];
            if constexpr (EXACT) pack_a_rest(du[0], du[1], ud, udl);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t y[4];
                ldsm_trans(at_t<KP>(ln, kt, i * 16, s * 16), y);
                mma(S[2 * s], ud, y[0], y[1]);
                mma(S[2 * s + 1], ud, y[2], y[3]);
                if constexpr (EXACT) {
                    mma(S[2 * s], udl, y[0], y[1]);
                    mma(S[2 * s + 1], udl, y[2], y[3]);
                }
            }
            // O, over the strip's values
#pragma unroll
            for (int j = 0; j <= i; ++j) {
                uint32_t y[4];
                ldsm(at_b<kMatPitch>(ln, base + lay.p, i * 16, j * 16), y);
                mma(o[0], u[j], y[0], y[1]);
                mma(o[1], u[j], y[2], y[3]);
            }
            uint32_t r[2][2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    r[m][h] = pack_bf16(o[m][2 * h] * gt[m][0].qu * back[h], o[m][2 * h + 1] * gt[m][1].qu * back[h]);
            stsm_trans(vt + (i * 16 + ln.t_row) * vp + (warp * 16 + ln.t_col) * 2, r[0][0], r[1][0], r[0][1], r[1][1]);
        }
        __syncthreads();
        for (int i = tid; i < nt * warps * 2; i += nth) {
            const int t = i / (warps * 2), e = i % (warps * 2) * 8;
            if (j0 + e < a.dv)
                *reinterpret_cast<uint4*>(a.out + a.row(unit, t0 + t) * a.dv + j0 + e) = *reinterpret_cast<const uint4*>(smem + lay.v[buf] + t * vp + e * 2);
        }
        __syncthreads();
    }
    if (__any_sync(0xffffffffu, seen.lost())) {
        // (the tile stores of this warp's columns above are behind a barrier; these come after them)
        if (lane == 0) atomicAdd(status + 1, 1);
        walk_sixteen<DKP>(a, unit, j0 + warp * 16 + (lane & 15), lane >> 4);
        return;
    }
    if (a.state_out)
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = n * 8 + 2 * c + (e & 1), j = col + (e >> 1) * 8;
                if (i < a.dk && j < a.dv) a.state_out[unit * plane + (long long)i * a.dv + j] = S[n][e] / scale[e >> 1];
            }
}

}  // namespace

bool gdr_chunk_supported(int dk, int dv) { return dk % 8 == 0 && dv % 8 == 0; }

cudaError_t launch_gdr_chunk_fwd(const Gdr<__nv_bfloat16>& a, cudaStream_t stream) {
    int* status = device_status_ptr();
    if (!status) return cudaErrorUnknown;
    const int all = (a.dv + 15) / 16, slabs = (all + kMostWarps - 1) / kMostWarps, warps = (all + slabs - 1) / slabs;
    auto launch = [&](auto D) {
        constexpr int dkp = decltype(D)::value;
        auto go = [&](auto E) {
            constexpr bool exact = decltype(E)::value;
            const int smem = Layout<dkp, exact>(warps).total;
            auto kernel = gdr_chunk_kernel<dkp, exact>;
            cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
            if (e != cudaSuccess) return e;
            count_launch();
            return launch_pdl(kernel, dim3((unsigned)(a.units * slabs)), dim3(32 * warps), smem, stream, a, slabs, status);
        };
        return a.state_out ? go(std::true_type()) : go(std::false_type());
    };
    if (a.dk <= 16) return launch(std::integral_constant<int, 16>());
    if (a.dk <= 32) return launch(std::integral_constant<int, 32>());
    if (a.dk <= 48) return launch(std::integral_constant<int, 48>());
    if (a.dk <= 64) return launch(std::integral_constant<int, 64>());
    if (a.dk <= 96) return launch(std::integral_constant<int, 96>());
    return launch(std::integral_constant<int, 128>());
}

}  // namespace vig
