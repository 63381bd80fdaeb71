// Gradient of the selective scan.
//
//   g_t = C_t dy_t + a_{t+1} g_{t+1}  (dy: d_out through the gate; a_t = e^(delta_t A))
//   dC_t = sum_c dy_t h_t;  dB_t = sum_c g_t delta_t x_t;  w_t = g_t a_t h_{t-1}: what passes through a token's decay
//   dx_t = delta_t sum_n g_t B_t + D dy_t;  d delta_t = sum_n w_t A + x_t sum_n g_t B_t;  dA = sum_t w_t delta_t
//
// A block walks forward over its tokens and keeps the state in front of every few of them (scratch of its own, which stays in L2: the
// grid is what runs at a time and takes one piece of work after another), then backward: decays and states of those few tokens once
// more, this time into registers, and over them from behind.  So the exponentials are computed twice, and nothing is divided or taken off again.
// Sums over the states cross four lanes; sums over the channels, two for every state and token, are tensor-core products with a
// matrix of zeros and ones (tf32 terms, one for bf16 calls, whose results are rounded to eight bits, and two for fp32), a quarter of
// the shuffles' instructions.  What a block has summed over its channels goes through memory to a last launch that adds the blocks in order.
#include "gdr.h"
#include "ssm.cuh"

namespace vig {
namespace {

using namespace ssm;

template <int NS>
struct Few { static constexpr int N = NS <= 4 ? 8 : 4; };   // tokens whose decays and states a lane holds in registers

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
// Adds up four values each over the lanes of equal lane / 4: values 0, 2 to column 2 p of rows g, g + 8, values 1, 3 to column 2 p + 1.
// ones: 1.0f (as tf32) in lanes of lane / 4 == i.
template <bool SPLIT>
__device__ __forceinline__ void add_four(float (&d)[4], float v0, float v1, float v2, float v3, uint32_t b0, uint32_t b1) {
    if constexpr (SPLIT) {
        const float v[4] = {v0, v1, v2, v3};
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = to_tf32(v[i]);
            lo[i] = to_tf32(v[i] - __uint_as_float(hi[i]));
        }
        mma_tf32(d, hi[0], hi[2], hi[1], hi[3], b0, b1);
        mma_tf32(d, lo[0], lo[2], lo[1], lo[3], b0, b1);
    } else {
        mma_tf32(d, to_tf32(v0), to_tf32(v2), to_tf32(v1), to_tf32(v3), b0, b1);
    }
}

template <int NS>
struct Smem {
    static constexpr int NP = 4 * NS;
    float step[kTile][kCh][4];        // delta, delta, delta x, delta x
    float dy[kTile][kCh][2];
    float rows_b[kTile * NP], rows_c[kTile * NP];
    float sums[3][kTile][kRow];       // y; sum w A (of A log2 e); sum g B
    float bc[kTile][8][2 * NP];       // sums over a warp's channels
};

template <typename T, int NS>
__global__ void __launch_bounds__(kThreads, NS <= 4 ? 2 : 1) ssm_grad_kernel(Ssm<T> a) {
    constexpr int NP = 4 * NS, P = NS / 2, F = Few<NS>::N;
    constexpr bool kSplit = sizeof(T) == 4;
    extern __shared__ __align__(16) unsigned char raw[];
    Smem<NS>& sm = *reinterpret_cast<Smem<NS>*>(raw);
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, ch = warp * 8 + (lane & 7), quarter = lane >> 3, n0 = quarter * NS;
    const int et = tid / 16, ec = (tid % 16) * 4;
    const int per_seg = (a.seg + F - 1) / F;
    float* kept = a.kept + (long long)blockIdx.x * per_seg * kThreads * NS + tid * NS;
    // products with ones: pair i of columns takes lanes of lane / 4 == 2 i (row r of B) and 2 i + 1 (row r + 4)
    const int lg = lane >> 2, lr = lane & 3;
    uint32_t one0[4], one1[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        one0[i] = lg == 2 * i ? 0x3f800000u : 0u;
        one1[i] = lg == 2 * i + 1 ? 0x3f800000u : 0u;
    }
    for (long long item = blockIdx.x; item < a.items; item += gridDim.x) {
        const Place at(a, item);
        const bool live = ch < at.live, mine = ec < at.live;
        const int c = at.c0 + (live ? ch : 0), g0 = at.c0 + ec;
        const int t0 = at.seg * a.seg, t1 = min(t0 + a.seg, a.L), tiles = (t1 - t0 + kTile - 1) / kTile;
        f32x2 rate[P], h[P], g[P], da[P];
        load_states<NS>(a.A + (long long)c * a.N, live ? a.N : 0, n0, rate);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            rate[i] = fmul2(rate[i], pack2(kLog2E, kLog2E));
            h[i] = g[i] = da[i] = 0;
        }
        const long long slot = (((long long)at.b * a.segs + at.seg) * a.C + c) * NP + n0, own = ((long long)at.b * a.C + c) * a.N;
        if (live) {
            if (a.segs > 1) {
                load_pairs<NS>(a.ends + slot, h);
                load_pairs<NS>(a.adjoint + slot, g);
            } else {
                if (a.state_in) load_states<NS>(a.state_in + own, a.N, n0, h);
                if (a.d_state_out) load_states<NS>(a.d_state_out + own, a.N, n0, g);
            }
        }
        float bias[4] = {}, skip[4] = {}, d_skip[4] = {}, d_bias[4] = {};
        if (mine) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (a.bias) bias[j] = a.bias[g0 + j];
                if (a.D) skip[j] = a.D[g0 + j];
            }
        }
        typename Four<T>::Raw rx = {}, rd = {}, rz = {}, ro = {};
        Rows<T, NP> rb, rc;
        auto load = [&](int t, bool back) {
            const int tt = t + et;
            if (mine && tt < t1) {
                const long long r = a.row(at.b, tt);
                rx = load4(a.x + r * a.ldx + g0);
                rd = load4(a.dt + r * a.lddt + g0);
                if (back) {
                    if (a.z) rz = load4(a.z + r * a.ldz + g0);
                    ro = load4(a.d_out + r * a.ldo + g0);
                }
            }
            rb.load(a.Bt, a, a.ldB, at, t);
            if (back) rc.load(a.Ct, a, a.ldC, at, t);
        };
        // forward: the state in front of every F-th token
        load(t0, false);
        for (int k = 0; k < tiles; ++k) {
            const int t = t0 + k * kTile;
            float x[4], d[4];
            widen4(rx, x);
            widen4(rd, d);
            const bool there = mine && t + et < t1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = d[j] + bias[j];
                float delta = a.softplus ? softplus_of(v, exp_minus_abs<T>(v)) : v;
                if (!there) delta = 0.f;
                const float in = there ? delta * x[j] : 0.f;
                *reinterpret_cast<float4*>(&sm.step[et][ec + j][0]) = make_float4(delta, delta, in, in);
            }
            rb.put(sm.rows_b);
            __syncthreads();
            if (k + 1 < tiles) load(t + kTile, false);
            else load(t, true);
#pragma unroll 1
            for (int s = 0; s < kTile; s += F) {
                if (t + s >= t1) break;
                store_pairs<NS>(kept + (long long)((k * kTile + s) / F) * kThreads * NS, h);
                if (t + s + F >= t1) break;   // (the last few's end is not asked for)
#pragma unroll
                for (int j = 0; j < F; ++j) {
                    const ulonglong2 dd = *reinterpret_cast<const ulonglong2*>(&sm.step[s + j][ch][0]);
                    f32x2 bt[P];
                    load_pairs<NS>(&sm.rows_b[(s + j) * NP + n0], bt);
#pragma unroll
                    for (int i = 0; i < P; ++i) h[i] = ffma2(exp2_pair(fmul2(rate[i], dd.x)), h[i], fmul2(dd.y, bt[i]));
                }
            }
            __syncthreads();
        }
        // backward
        for (int k = tiles - 1; k >= 0; --k) {
            const int t = t0 + k * kTile;
            float x[4], d[4], z[4], o[4], delta[4], slope[4], dy[4];
            widen4(rx, x);
            widen4(rd, d);
            widen4(rz, z);
            widen4(ro, o);
            const bool there = mine && t + et < t1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = d[j] + bias[j], u = exp_minus_abs<T>(v);
                delta[j] = a.softplus ? softplus_of(v, u) : v;
                slope[j] = a.softplus ? sigmoid_of<T>(v, u) : 1.f;
                dy[j] = o[j];
                if (a.z) dy[j] *= z[j] * sigmoid_of<T>(z[j], exp_minus_abs<T>(z[j]));
                if (!there) delta[j] = dy[j] = x[j] = 0.f;
                const float in = delta[j] * x[j];
                *reinterpret_cast<float4*>(&sm.step[et][ec + j][0]) = make_float4(delta[j], delta[j], in, in);
            }
            *reinterpret_cast<float4*>(&sm.dy[et][ec][0]) = make_float4(dy[0], dy[0], dy[1], dy[1]);
            *reinterpret_cast<float4*>(&sm.dy[et][ec + 2][0]) = make_float4(dy[2], dy[2], dy[3], dy[3]);
            rb.put(sm.rows_b);
            rc.put(sm.rows_c);
            __syncthreads();
            if (k > 0) load(t - kTile, true);
#pragma unroll 1
            for (int s = kTile - F; s >= 0; s -= F) {
                if (t + s >= t1) continue;
                f32x2 decay[F][P], before[F][P];
                float py[F], pw[F], pb[F];
                load_pairs<NS>(kept + (long long)((k * kTile + s) / F) * kThreads * NS, h);
#pragma unroll
                for (int j = 0; j < F; ++j) {
                    const ulonglong2 dd = *reinterpret_cast<const ulonglong2*>(&sm.step[s + j][ch][0]);
                    f32x2 bt[P], ct[P], y = 0;
                    load_pairs<NS>(&sm.rows_b[(s + j) * NP + n0], bt);
                    if (a.z) load_pairs<NS>(&sm.rows_c[(s + j) * NP + n0], ct);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        before[j][i] = h[i];
                        decay[j][i] = exp2_pair(fmul2(rate[i], dd.x));
                        h[i] = ffma2(decay[j][i], h[i], fmul2(dd.y, bt[i]));
                        if (a.z) y = ffma2(ct[i], h[i], y);
                    }
                    py[j] = sum2(y);
                }
                float acc[4] = {0.f, 0.f, 0.f, 0.f};
                constexpr int kTogether = 8 / NS;   // tokens whose sums over channels fill a product's eight columns
#pragma unroll
                for (int j = F - 1; j >= 0; --j) {
                    const ulonglong2 dd = *reinterpret_cast<const ulonglong2*>(&sm.step[s + j][ch][0]);
                    const f32x2 gy = *reinterpret_cast<const f32x2*>(&sm.dy[s + j][ch][0]);
                    f32x2 bt[P], ct[P], sw = 0, sb = 0;
                    float v[2 * NS];
                    load_pairs<NS>(&sm.rows_b[(s + j) * NP + n0], bt);
                    load_pairs<NS>(&sm.rows_c[(s + j) * NP + n0], ct);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        g[i] = ffma2(ct[i], gy, g[i]);
                        const f32x2 after = j + 1 < F ? before[j + 1 < F ? j + 1 : j][i] : h[i];
                        unpack2(fmul2(g[i], dd.y), v[2 * i], v[2 * i + 1]);
                        unpack2(fmul2(gy, after), v[NS + 2 * i], v[NS + 2 * i + 1]);
                        sb = ffma2(g[i], bt[i], sb);
                        g[i] = fmul2(g[i], decay[j][i]);
                        const f32x2 w = fmul2(g[i], before[j][i]);
                        sw = ffma2(w, rate[i], sw);
                        da[i] = ffma2(w, dd.x, da[i]);
                    }
                    pw[j] = sum2(sw);
                    pb[j] = sum2(sb);
#pragma unroll
                    for (int q = 0; q < NS / 2; ++q)
                        add_four<kSplit>(acc, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], one0[j % kTogether * (NS / 2) + q], one1[j % kTogether * (NS / 2) + q]);
                    if (j % kTogether == 0) {
                        // lane 4 g + r: values 4 q .. + 3 of token j + r / (NS / 2), q = r % (NS / 2), of four of the eight channels; the
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
                }
#pragma unroll
                for (int j = 0; j < F; j += 4) {
                    if (a.z) sm.sums[0][s + j + quarter][ch] = over_quarters(py[j], py[j + 1], py[j + 2], py[j + 3], quarter);
                    sm.sums[1][s + j + quarter][ch] = over_quarters(pw[j], pw[j + 1], pw[j + 2], pw[j + 3], quarter);
                    sm.sums[2][s + j + quarter][ch] = over_quarters(pb[j], pb[j + 1], pb[j + 2], pb[j + 3], quarter);
                }
            }
            __syncthreads();
            if (there) {
                const long long r = a.row(at.b, t + et);
                const float4 w4 = *reinterpret_cast<const float4*>(&sm.sums[1][et][ec]), b4 = *reinterpret_cast<const float4*>(&sm.sums[2][et][ec]);
                const float w[4] = {w4.x, w4.y, w4.z, w4.w}, into[4] = {b4.x, b4.y, b4.z, b4.w};
                float dx[4], dd[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dx[j] = fmaf(delta[j], into[j], skip[j] * dy[j]);
                    dd[j] = fmaf(w[j], 0.69314718055994531f, x[j] * into[j]) * slope[j];   // (w is of A log2 e)
                    d_skip[j] = fmaf(dy[j], x[j], d_skip[j]);
                    d_bias[j] += dd[j];
                }
                store4(a.dx + r * a.lddx + g0, dx);
                store4(a.ddt + r * a.ldddt + g0, dd);
                if (a.z && a.dz) {
                    const float4 y4 = *reinterpret_cast<const float4*>(&sm.sums[0][et][ec]);
                    const float y[4] = {y4.x, y4.y, y4.z, y4.w};
                    float dz[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float s = sigmoid_of<T>(z[j], exp_minus_abs<T>(z[j]));
                        dz[j] = o[j] * fmaf(skip[j], x[j], y[j]) * s * fmaf(z[j], 1.f - s, 1.f);
                    }
                    store4(a.dz + r * a.lddz + g0, dz);
                }
            }
            // the block's sums over channels: its warps in order
            const int cb = (int)(item % a.blocks);
            for (int i = tid; i < kTile * 2 * NP; i += kThreads) {
                const int tt = i / (2 * NP), e = i % (2 * NP);
                if (t + tt >= t1) continue;
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < 8; ++w) s += sm.bc[tt][w][e];
                a.part_bc[(((long long)cb * a.B * a.L + a.row(at.b, t + tt)) * a.G + at.group) * (2 * NP) + e] = s;
            }
            __syncthreads();   // (sums, bc and step are written again)
        }
        const long long where = (long long)at.b * a.segs + at.seg;
        if (live) {
            store_pairs<NS>(a.part_a + (where * a.C + c) * NP + n0, da);
            if (a.d_state_in && at.seg == 0) store_states<NS>(a.d_state_in + own, a.N, n0, g);
        }
        // sums over the tokens of what is a channel's: sixteen threads hold a part each
        *reinterpret_cast<float4*>(&sm.sums[0][et][ec]) = make_float4(d_skip[0], d_skip[1], d_skip[2], d_skip[3]);
        *reinterpret_cast<float4*>(&sm.sums[1][et][ec]) = make_float4(d_bias[0], d_bias[1], d_bias[2], d_bias[3]);
        __syncthreads();
        if (tid < 2 * kCh && (tid % kCh) < at.live) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < kTile; ++i) s += sm.sums[tid / kCh][i][tid % kCh];
            a.part_c[(where * 2 + tid / kCh) * a.C + at.c0 + tid % kCh] = s;
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

int blocks_at_a_time(int NS, long long items) {
    const long long most = 148LL * (NS <= 4 ? 2 : 1);
    return (int)(items < most ? items : most);
}

template <typename T, int NS>
cudaError_t grad(const Ssm<T>& a, cudaStream_t stream) {
    const cudaError_t e = allow_smem<ssm_grad_kernel<T, NS>>(sizeof(Smem<NS>));
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(ssm_grad_kernel<T, NS>, dim3(blocks_at_a_time(NS, a.items)), dim3(kThreads), sizeof(Smem<NS>), stream, a);
}

}  // namespace

template <typename T>
size_t ssm_grad_scratch(Ssm<T>& a, char* base) {
    const int NP = ssm_padded(a.N), NS = NP / 4, F = NS <= 4 ? 8 : 4;
    size_t at = 0;
    auto take = [&](float*& p, size_t floats) {
        p = reinterpret_cast<float*>(base ? base + at : nullptr);
        at += (floats * sizeof(float) + 255) / 256 * 256;
    };
    const size_t segs = (size_t)a.B * a.segs;
    take(a.ends, a.segs > 1 ? segs * a.C * NP : 0);
    take(a.adjoint, a.segs > 1 ? segs * a.C * NP : 0);
    take(a.total, a.segs > 1 ? segs * a.C : 0);
    take(a.kept, (size_t)blocks_at_a_time(NS, a.items) * ((a.seg + F - 1) / F) * kThreads * NS);
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
