// Gradient of the selective scan.
//
//   g_t = C_t dy_t + a_{t+1} g_{t+1}  (dy: d_out through the gate; a_t = e^(delta_t A))
//   dC_t = sum_c dy_t h_t;  dB_t = sum_c g_t delta_t x_t;  w_t = g_t a_t h_{t-1}: what passes through a token's decay
//   dx_t = delta_t sum_n g_t B_t + D dy_t;  d delta_t = sum_n w_t A + x_t sum_n g_t B_t;  dA = sum_t w_t delta_t
//
// A block walks forward over its tokens and keeps the state in front of every few of them (scratch of its own: the grid is what runs at a
// time and takes one piece of work after another), then backward: decays and states of those few tokens once more, this time kept on chip
// (states in registers, decays in shared memory), and over them from behind.  64 x 196 x 1152 with 16 states, bf16: 459 us, bound by what it
// issues (570 warp instructions for 32 tokens and channels, an instruction in about 54 % of the cycles).  So the exponentials are computed twice, and
// nothing is divided or taken off again.
// Sums over the states cross four lanes; sums over the channels, two for every state and token, are tensor-core products with a
// matrix of zeros and ones, a quarter of the shuffles' instructions: every product enters as two terms, of bf16 in bf16 calls (error 2^-17; a
// training step of the size above 555 us, 550 with a single term of tf32, 2^-12, which shows where channels cancel), of tf32 in fp32 calls (2^-23).
// What a block has summed over its channels goes through memory to a last launch that adds the blocks in order.
#include "gdr.h"
#include "mma.cuh"
#include "ssm.cuh"

namespace vig {
namespace {

using namespace ssm;

__device__ __forceinline__ uint32_t to_tf32(float x) {
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    return r;
}
// D += A B: A 16 x 8 (rows g and g + 8, columns r and r + 4 of lane 4 g + r), B 8 x 8 (rows r and r + 4, column g), tf32.
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Both of a pair as two bf16 terms each, side by side: the upper half of a number, and what is left, rounded (error 2^-17).
__device__ __forceinline__ void two_terms(f32x2 v, uint32_t& t0, uint32_t& t1) {
    float v0, v1, rest0, rest1;
    unpack2(v, v0, v1);
    const float hi0 = __uint_as_float(__float_as_uint(v0) & 0xffff0000u), hi1 = __uint_as_float(__float_as_uint(v1) & 0xffff0000u);
    unpack2(neg_add2(pack2(hi0, hi1), v), rest0, rest1);
    t0 = pack_bf16(hi0, rest0);
    t1 = pack_bf16(hi1, rest1);
}
// Adds up two pairs of values each over the lanes of equal lane / 4: their first values to column 2 p of rows g, g + 8, their second ones to
// column 2 p + 1.  b0, b1: ones in lanes of lane / 4 == 2 p, 2 p + 1.
template <bool TF32>
__device__ __forceinline__ void add_four(float (&d)[4], f32x2 v, f32x2 w, uint32_t b0, uint32_t b1) {
    if constexpr (TF32) {
        float f[4];
        unpack2(v, f[0], f[1]);
        unpack2(w, f[2], f[3]);
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = to_tf32(f[i]);
            lo[i] = to_tf32(f[i] - __uint_as_float(hi[i]));
        }
        mma_tf32(d, hi[0], hi[2], hi[1], hi[3], b0, b1);
        mma_tf32(d, lo[0], lo[2], lo[1], lo[3], b0, b1);
    } else {
        uint32_t t[4];   // (a register's two terms are neighbouring columns of A)
        two_terms(v, t[0], t[2]);
        two_terms(w, t[1], t[3]);
        wmma16::mma_k16(d, t, b0, b1);
    }
}

template <int NS, int K, int F>
struct Smem {
    static constexpr int NP = 4 * NS, kTile = tile_of(K);
    float step[kTile][kCh][2];        // delta, delta x
    float dy[kTile][kCh];
    float rows_b[kTile * NP], rows_c[kTile * NP];
    float sums[3][kTile][kRow];       // y; sum w A (of A log2 e); sum g B
    float bc[kTile][8 / K][2 * NP];   // sums over a warp's channels
    float slope[kTile][kCh];          // of the step size
    float bias[kCh], skip[kCh];
    float decay[F][K][threads_of(K)][NS];   // a lane's own
};

// F: tokens whose states a lane holds in registers, and whose decays in shared memory.
template <typename T, int NS, int K, int F, int BLOCKS>
__global__ void __launch_bounds__(threads_of(K), BLOCKS) ssm_grad_kernel(Ssm<T> a) {
    constexpr int NP = 4 * NS, P = NS / 2, kThreads = threads_of(K), kTile = tile_of(K), kWarps = 8 / K;
    constexpr bool kTf32 = sizeof(T) == 4;
    constexpr uint32_t kOnes = kTf32 ? 0x3f800000u : 0x3f803f80u;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<NS, K, F>& sm = *reinterpret_cast<Smem<NS, K, F>*>(smem_raw);
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, ch = (warp * 8 + (lane & 7)) * K, quarter = lane >> 3, n0 = quarter * NS;
    const int et = tid / (kCh / 4), ec = (tid % (kCh / 4)) * 4;
    const int per_seg = (a.seg + F - 1) / F;
    float* kept = a.kept + ((long long)blockIdx.x * per_seg * K * kThreads + tid) * NS;
    // products with ones: pair i of columns takes lanes of lane / 4 == 2 i (row r of B) and 2 i + 1 (row r + 4)
    const int lg = lane >> 2, lr = lane & 3;
    uint32_t one0[4], one1[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        one0[i] = lg == 2 * i ? kOnes : 0u;
        one1[i] = lg == 2 * i + 1 ? kOnes : 0u;
    }
    for (long long item = blockIdx.x; item < a.items; item += gridDim.x) {
        const Place at(a, item);
        const bool mine = ec < at.live;
        const int g0 = at.c0 + (mine ? ec : 0);
        const int t0 = at.seg * a.seg, t1 = min(t0 + a.seg, a.L), tiles = (t1 - t0 + kTile - 1) / kTile;
        f32x2 rate[K][P], h[K][P], g[K][P], da[K][P];
        const long long slot = (((long long)at.b * a.segs + at.seg) * a.C + at.c0 + ch) * NP + n0, own = ((long long)at.b * a.C + at.c0 + ch) * a.N;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool live = ch + k < at.live;
            load_states<NS, false>(a.A + (long long)(at.c0 + ch + k) * a.N, live ? a.N : 0, n0, rate[k]);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                rate[k][i] = rate_of2(rate[k][i]);
                h[k][i] = g[k][i] = da[k][i] = 0;
            }
            if (live) {
                if (a.segs > 1) {
                    load_pairs<NS>(a.ends + slot + k * NP, h[k]);
                    load_pairs<NS>(a.adjoint + slot + k * NP, g[k]);
                } else {
                    if (a.state_in) load_states<NS, false>(a.state_in + own + k * a.N, a.N, n0, h[k]);
                    if (a.d_state_out) load_states<NS, false>(a.d_state_out + own + k * a.N, a.N, n0, g[k]);
                }
            }
        }
        f32x2 d_skip[2] = {0, 0}, d_bias[2] = {0, 0};
        for (int i = tid; i < kCh; i += kThreads) {
            sm.bias[i] = a.bias && i < at.live ? a.bias[at.c0 + i] : 0.f;
            sm.skip[i] = a.D && i < at.live ? a.D[at.c0 + i] : 0.f;
        }
        __syncthreads();
        typename Four<T>::Raw rx = {}, rd = {}, rz = {}, ro = {};
        Rows<T, NP, kTile, kThreads, false> rb, rc;
        rb.start(a.Bt, a, a.ldB, at, t0);
        rc.start(a.Ct, a, a.ldC, at, t0);
        rc.move((tiles - 1) * kTile);
        auto load = [&](int t, bool back) {
            if (mine && t + et < t1) {
                const long long r = a.row(at.b, t + et);
                rx = load4(a.x + r * a.ldx + g0);
                rd = load4(a.dt + r * a.lddt + g0);
                if (back) {
                    if (a.z) rz = load4(a.z + r * a.ldz + g0);
                    ro = load4(a.d_out + r * a.ldo + g0);
                }
            }
            rb.load(t, t1, a.N);
            if (back) rc.load(t, t1, a.N);
        };
        // forward: the state in front of every F-th token
        load(t0, false);
        for (int m = 0; m < tiles; ++m) {
            const int t = t0 + m * kTile;
            const bool there = mine && t + et < t1;
            f32x2 x[2], d[2], bias[2];
            widen4(rx, x);
            widen4(rd, d);
            load_pairs<4>(&sm.bias[ec], bias);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f32x2 delta = fadd2(d[j], bias[j]);
                if (a.softplus) delta = softplus2(delta, exp_minus_abs<T>(delta));
                f32x2 in = fmul2(delta, x[j]);
                if (!there) delta = in = 0;
                put_step(&sm.step[et][ec + 2 * j], delta, in);
            }
            rb.put(sm.rows_b);
            __syncthreads();
            if (m + 1 < tiles) {
                rb.move(kTile);
                load(t + kTile, false);
            } else {
                load(t, true);
            }
#pragma unroll 1
            for (int s = 0; s < kTile; s += F) {
                if (t + s >= t1) break;
                float* to = kept + (long long)((m * kTile + s) / F) * K * kThreads * NS;
#pragma unroll
                for (int k = 0; k < K; ++k) store_pairs<NS>(to + k * kThreads * NS, h[k]);
                if (t + s + F >= t1) break;   // (the last few's end is not asked for)
#pragma unroll
                for (int j = 0; j < F; ++j) {
                    f32x2 bt[P];
                    float d2[2 * K];
                    load_floats<2 * K>(&sm.step[s + j][ch][0], d2);
                    load_pairs<NS>(&sm.rows_b[(s + j) * NP + n0], bt);
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int i = 0; i < P; ++i) h[k][i] = ffma2(decay2<T>(fmul2(rate[k][i], both(d2[2 * k]))), h[k][i], fmul2(both(d2[2 * k + 1]), bt[i]));
                }
            }
            __syncthreads();
        }
        // backward
        for (int m = tiles - 1; m >= 0; --m) {
            const int t = t0 + m * kTile;
            const bool there = mine && t + et < t1;
            const typename Four<T>::Raw cx = rx, cz = rz, co = ro;
            {
                f32x2 x[2], z[2], dy[2], delta[2], slope[2], bias[2];
                widen4(cx, x);
                widen4(rd, delta);
                widen4(cz, z);
                widen4(co, dy);
                load_pairs<4>(&sm.bias[ec], bias);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    delta[j] = fadd2(delta[j], bias[j]);
                    slope[j] = both(1.f);
                    if (a.softplus) {
                        const f32x2 u = exp_minus_abs<T>(delta[j]);
                        slope[j] = sigmoid2<T>(delta[j], u);
                        delta[j] = softplus2(delta[j], u);
                    }
                    if (a.z) dy[j] = fmul2(dy[j], fmul2(z[j], sigmoid2<T>(z[j])));
                    f32x2 in = fmul2(delta[j], x[j]);
                    if (!there) delta[j] = dy[j] = in = 0;
                    put_step(&sm.step[et][ec + 2 * j], delta[j], in);
                }
                store4(&sm.dy[et][ec], dy);
                store4(&sm.slope[et][ec], slope);
            }
            rb.put(sm.rows_b);
            rc.put(sm.rows_c);
            __syncthreads();
            if (m > 0) {
                rb.move(-kTile);
                rc.move(-kTile);
                load(t - kTile, true);
            }
#pragma unroll 1
            for (int s = kTile - F; s >= 0; s -= F) {
                if (t + s >= t1) continue;
                f32x2 before[F][K][P];
                float part[2][4][K];
                const float* from = kept + (long long)((m * kTile + s) / F) * K * kThreads * NS;
#pragma unroll
                for (int k = 0; k < K; ++k) load_pairs<NS>(from + k * kThreads * NS, h[k]);
#pragma unroll
                for (int j = 0; j < F; ++j) {
                    f32x2 bt[P], ct[P];
                    float d2[2 * K];
                    load_floats<2 * K>(&sm.step[s + j][ch][0], d2);
                    load_pairs<NS>(&sm.rows_b[(s + j) * NP + n0], bt);
                    if (a.z) load_pairs<NS>(&sm.rows_c[(s + j) * NP + n0], ct);
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        f32x2 y = 0, e[P];
#pragma unroll
                        for (int i = 0; i < P; ++i) {
                            before[j][k][i] = h[k][i];
                            e[i] = decay2<T>(fmul2(rate[k][i], both(d2[2 * k])));
                            h[k][i] = ffma2(e[i], h[k][i], fmul2(both(d2[2 * k + 1]), bt[i]));
                            if (a.z) y = i == 0 ? fmul2(ct[i], h[k][i]) : ffma2(ct[i], h[k][i], y);
                        }
                        store_pairs<NS>(sm.decay[j][k][tid], e);
                        part[0][j % 4][k] = sum2(y);
                    }
                    if (j % 4 == 3 && a.z) {
                        float to[K];
#pragma unroll
                        for (int k = 0; k < K; ++k) to[k] = over_quarters(part[0][0][k], part[0][1][k], part[0][2][k], part[0][3][k], quarter);
                        store_floats<K>(&sm.sums[0][s + j - 3 + quarter][ch], to);
                    }
                }
                float acc[4] = {0.f, 0.f, 0.f, 0.f};
                constexpr int kTogether = 8 / NS;   // tokens whose sums over channels fill a product's eight columns
#pragma unroll
                for (int j = F - 1; j >= 0; --j) {
                    f32x2 bt[P], ct[P], vb[P], vc[P];
                    float d2[2 * K], gy[K];
                    load_floats<2 * K>(&sm.step[s + j][ch][0], d2);
                    load_floats<K>(&sm.dy[s + j][ch], gy);
                    load_pairs<NS>(&sm.rows_b[(s + j) * NP + n0], bt);
                    load_pairs<NS>(&sm.rows_c[(s + j) * NP + n0], ct);
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        f32x2 sw = 0, sb = 0, e[P];
                        load_pairs<NS>(sm.decay[j][k][tid], e);
#pragma unroll
                        for (int i = 0; i < P; ++i) {
                            const f32x2 after = j + 1 < F ? before[j + 1 < F ? j + 1 : j][k][i] : h[k][i];
                            g[k][i] = ffma2(ct[i], both(gy[k]), g[k][i]);
                            vb[i] = k == 0 ? fmul2(g[k][i], both(d2[2 * k + 1])) : ffma2(g[k][i], both(d2[2 * k + 1]), vb[i]);
                            vc[i] = k == 0 ? fmul2(after, both(gy[k])) : ffma2(after, both(gy[k]), vc[i]);
                            sb = i == 0 ? fmul2(g[k][i], bt[i]) : ffma2(g[k][i], bt[i], sb);
                            g[k][i] = fmul2(g[k][i], e[i]);
                            const f32x2 w = fmul2(g[k][i], before[j][k][i]);
                            sw = i == 0 ? fmul2(w, rate[k][i]) : ffma2(w, rate[k][i], sw);
                            da[k][i] = ffma2(w, both(d2[2 * k]), da[k][i]);
                        }
                        part[0][j % 4][k] = sum2(sw);
                        part[1][j % 4][k] = sum2(sb);
                    }
#pragma unroll
                    for (int q = 0; q < NS / 2; ++q) {   // (a lane's values: NS of vb, then NS of vc)
                        const f32x2 v = 2 * q < P ? vb[2 * q % P] : vc[2 * q % P], w = 2 * q + 1 < P ? vb[(2 * q + 1) % P] : vc[(2 * q + 1) % P];
                        add_four<kTf32>(acc, v, w, one0[j % kTogether * (NS / 2) + q], one1[j % kTogether * (NS / 2) + q]);
                    }
                    if (j % kTogether == 0) {
                        // lane 4 g + r: values 4 q .. + 3 of token j + r / (NS / 2), q = r % (NS / 2), of four of the eight lanes' channels; the
                        // other four are the neighbouring g's
                        const bool odd = lg & 1;
                        const float v0 = acc[0], v1 = acc[1], v2 = acc[2], v3 = acc[3];
                        float k0 = odd ? v2 : v0, k1 = odd ? v3 : v1;
                        k0 += __shfl_xor_sync(0xffffffffu, odd ? v0 : v2, 4);
                        k1 += __shfl_xor_sync(0xffffffffu, odd ? v1 : v3, 4);
                        const int value = 4 * (lr % (NS / 2)) + (odd ? 2 : 0), kind = value / NS;
                        *reinterpret_cast<float2*>(&sm.bc[s + j + lr / (NS / 2)][warp][kind * NP + (lg >> 1) * NS + value % NS]) = make_float2(k0, k1);
                        acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
                    }
                    if (j % 4 == 0) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float to[K];
#pragma unroll
                            for (int k = 0; k < K; ++k) to[k] = over_quarters(part[e][0][k], part[e][1][k], part[e][2][k], part[e][3][k], quarter);
                            store_floats<K>(&sm.sums[1 + e][s + j + quarter][ch], to);
                        }
                    }
                }
            }
            __syncthreads();
            if (there) {
                const long long r = a.row(at.b, t + et);
                f32x2 w[2], into[2], x[2], dy[2], slope[2], skip[2];
                widen4(cx, x);
                load_pairs<4>(&sm.sums[1][et][ec], w);
                load_pairs<4>(&sm.sums[2][et][ec], into);
                load_pairs<4>(&sm.dy[et][ec], dy);
                load_pairs<4>(&sm.slope[et][ec], slope);
                load_pairs<4>(&sm.skip[ec], skip);
                f32x2 dx[2], dd[2];
                float d[8];
                load_floats<8>(&sm.step[et][ec][0], d);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    dx[j] = ffma2(pack2(d[4 * j], d[4 * j + 2]), into[j], fmul2(skip[j], dy[j]));
                    dd[j] = fmul2(ffma2(w[j], both(0.69314718055994531f), fmul2(x[j], into[j])), slope[j]);   // (w is of A log2 e)
                    d_skip[j] = ffma2(dy[j], x[j], d_skip[j]);
                    d_bias[j] = fadd2(d_bias[j], dd[j]);
                }
                store4(a.dx + r * a.lddx + g0, dx);
                store4(a.ddt + r * a.ldddt + g0, dd);
                if (a.z && a.dz) {
                    f32x2 z[2], o[2], y[2];
                    widen4(cz, z);
                    widen4(co, o);
                    load_pairs<4>(&sm.sums[0][et][ec], y);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x2 s = sigmoid2<T>(z[j]);
                        y[j] = fmul2(fmul2(o[j], ffma2(skip[j], x[j], y[j])), fmul2(s, ffma2(z[j], neg_add2(s, both(1.f)), both(1.f))));
                    }
                    store4(a.dz + r * a.lddz + g0, y);
                }
            }
            // the block's sums over channels: its warps in order
            const int cb = (int)(item % a.blocks);
            for (int i = tid; i < kTile * 2 * NP; i += kThreads) {
                const int tt = i / (2 * NP), e = i % (2 * NP);
                if (t + tt >= t1) continue;
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) s += sm.bc[tt][w][e];
                a.part_bc[(((long long)cb * a.B * a.L + a.row(at.b, t + tt)) * a.G + at.group) * (2 * NP) + e] = s;
            }
            __syncthreads();   // (sums, bc and step are written again)
        }
        const long long where = (long long)at.b * a.segs + at.seg;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (ch + k >= at.live) break;
            store_pairs<NS>(a.part_a + (where * a.C + at.c0 + ch + k) * NP + n0, da[k]);
            if (a.d_state_in && at.seg == 0) store_states<NS>(a.d_state_in + own + k * a.N, a.N, n0, g[k]);
        }
        // sums over the tokens of what is a channel's: the threads of a tile's tokens hold a part each
        store4(&sm.sums[0][et][ec], d_skip);
        store4(&sm.sums[1][et][ec], d_bias);
        __syncthreads();
        for (int i = tid; i < 2 * kCh; i += kThreads) {
            if (i % kCh >= at.live) continue;
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < kTile; ++e) s += sm.sums[i / kCh][e][i % kCh];
            a.part_c[(where * 2 + i / kCh) * a.C + at.c0 + i % kCh] = s;
        }
        __syncthreads();
    }
}

// The last sums: blocks of a group's channels (dB, dC), and sequences and segments (dA; dD and the bias's), each in order.
template <typename T>
__global__ void __launch_bounds__(256) ssm_grad_sums_kernel(Ssm<T> a, int NP, unsigned row_blocks) {
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x < row_blocks) {
        const long long id = (long long)blockIdx.x * 256 + threadIdx.x, rows = (long long)a.B * a.L * a.G, each = rows * 2 * NP;
        if (id >= each) return;
        const int e = (int)(id % (2 * NP)), kind = e / NP, n = e % NP;
        if (n >= a.N) return;
        float s = 0.f;
        for (int k = 0; k < a.blocks; ++k) s += a.part_bc[k * each + id];
        const long long row = id / (2 * NP), token = row / a.G;
        const int group = (int)(row % a.G);
        from_f32((kind ? a.dC + token * a.lddC : a.dB + token * a.lddB) + group * a.N + n, s);
        return;
    }
    // eight threads take the rows of a column in eight runs
    __shared__ float part[8][33];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const long long columns_a = (long long)a.C * NP, col = (long long)(blockIdx.x - row_blocks) * 32 + lane, columns = columns_a + 2LL * a.C;
    const int rows = a.B * a.segs, per = (rows + 7) / 8, lo = min(run * per, rows), hi = min(lo + per, rows);
    float s = 0.f;
    const float* p = nullptr;
    long long pitch = 0;
    if (col < columns_a) {
        p = a.part_a + col;
        pitch = columns_a;
    } else if (col < columns) {
        p = a.part_c + (col - columns_a);
        pitch = 2LL * a.C;
    }
    if (p)
#pragma unroll 8
        for (int r = lo; r < hi; ++r) s += p[r * pitch];
    part[run][lane] = s;
    __syncthreads();
    if (run != 0 || !p) return;
    for (int i = 1; i < 8; ++i) s += part[i][lane];
    if (col < columns_a) {
        const int c = (int)(col / NP), n = (int)(col % NP);
        if (n < a.N) a.dA[(long long)c * a.N + n] = s;
    } else {
        const int c = (int)(col - columns_a);
        if (c < a.C) {
            if (a.dD) a.dD[c] = s;
        } else if (a.dbias) {
            a.dbias[c - a.C] = s;
        }
    }
}

// How the padded states of a channel are spread: channels of a lane, tokens taken together, blocks an SM.  64 x 196 x 1152, a training step
// (with a single term of tf32): 550 us; one channel, eight tokens, two blocks 615; two, eight, three 608; two, eight, two 594; two, four, three 592.
template <int NS>
struct Form { static constexpr int K = 2, F = kSsmKept, kBlocks = ssm_grad_blocks(4 * NS); };

template <typename F>
auto by_states(int NP, F f) { return NP == 8 ? f(Form<2>{}) : NP == 16 ? f(Form<4>{}) : f(Form<8>{}); }

long long blocks_at_a_time(int per_sm, long long items) { return items < 148LL * per_sm ? items : 148LL * per_sm; }

template <typename T, int NS>
cudaError_t grad(const Ssm<T>& a, cudaStream_t stream) {
    typedef Form<NS> Of;
    constexpr size_t smem = sizeof(Smem<NS, Of::K, Of::F>);
    const cudaError_t e = allow_smem<ssm_grad_kernel<T, NS, Of::K, Of::F, Of::kBlocks>>(smem);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(ssm_grad_kernel<T, NS, Of::K, Of::F, Of::kBlocks>, dim3((unsigned)blocks_at_a_time(Of::kBlocks, a.items)), dim3(threads_of(Of::K)), smem,
                      stream, a);
}

}  // namespace

template <typename T>
size_t ssm_grad_scratch(Ssm<T>& a, char* base) {
    const int NP = ssm_padded(a.N);
    size_t at = 0;
    auto take = [&](float*& p, size_t floats) {
        p = reinterpret_cast<float*>(base ? base + at : nullptr);
        at += (floats * sizeof(float) + 255) / 256 * 256;
    };
    const size_t segs = (size_t)a.B * a.segs;
    take(a.ends, a.segs > 1 ? segs * a.C * NP : 0);
    take(a.adjoint, a.segs > 1 ? segs * a.C * NP : 0);
    take(a.total, a.segs > 1 ? segs * a.C : 0);
    take(a.kept, by_states(NP, [&](auto of) {
             typedef decltype(of) Of;
             return (size_t)blocks_at_a_time(Of::kBlocks, a.items) * ((a.seg + Of::F - 1) / Of::F) * kCh * NP;
         }));
    take(a.part_bc, (size_t)a.blocks * a.B * a.L * a.G * 2 * NP);
    take(a.part_a, segs * a.C * NP);
    take(a.part_c, segs * 2 * a.C);
    return at;
}

template <typename T>
cudaError_t launch_ssm_bwd(const Ssm<T>& a, cudaStream_t stream) {
    const int NP = ssm_padded(a.N);
    cudaError_t e = a.segs > 1 ? launch_ssm_segments<T>(a, true, stream) : cudaSuccess;
    if (e != cudaSuccess) return e;
    e = NP == 8 ? grad<T, 2>(a, stream) : NP == 16 ? grad<T, 4>(a, stream) : grad<T, 8>(a, stream);
    if (e != cudaSuccess) return e;
    const unsigned row_blocks = (unsigned)(((long long)a.B * a.L * a.G * 2 * NP + 255) / 256);
    const unsigned columns = (unsigned)(((long long)a.C * (NP + 2) + 31) / 32);
    count_launch();
    return launch_pdl(ssm_grad_sums_kernel<T>, dim3(row_blocks + columns), dim3(256), 0, stream, a, NP, row_blocks);
}

#define VIG_INSTANCES(T)                                            \
    template size_t ssm_grad_scratch<T>(Ssm<T>&, char*);            \
    template cudaError_t launch_ssm_bwd<T>(const Ssm<T>&, cudaStream_t);
VIG_INSTANCES(__nv_bfloat16)
VIG_INSTANCES(float)

}  // namespace vig
