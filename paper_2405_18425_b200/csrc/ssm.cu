// Selective state space scan: forward pass, the states in front of segments, and the single-token form.
//
//   delta_t = softplus(dt_t + bias);  h_t[n] = e^(delta_t A[c,n]) h_{t-1}[n] + delta_t x_t B_t[n];  y_t = sum_n C_t[n] h_t[n] + D x_t
//   out_t = y_t z_t sigmoid(z_t)
//
// The recurrence has an exponential for every token, channel and state, sixteen a clock and SM from the special-function unit: that bounds
// it, not memory (64 x 196 x 1152 with 16 states, bf16: 96 us; at 1965 MHz the exponentials take 50 of them at least, step sizes and gates 9 more, the
// memory 18).  So a state lives in a register from its first token to its last, pairs of states share an instruction, and everything
// that belongs to a token and channel alone is computed once (ssm.cuh).  Sequences of few channels are cut into segments: a first launch
// gives what each segment adds to the state behind it and the sum of its step sizes (its decay is e^(A sum), so no products are
// kept), a small one carries the states through, and the launch proper starts every segment from its own.
#include "ssm.cuh"

namespace vig {
namespace {

using namespace ssm;

constexpr int kMain = 0, kEnds = 1, kBoth = 2;   // kEnds: a segment's end state; kBoth: and what its outputs' gradients add to the adjoint in front

template <typename T, int NS, int K, int MODE>
__global__ void __launch_bounds__(threads_of(K)) ssm_kernel(Ssm<T> a) {
    constexpr int NP = 4 * NS, P = NS / 2, kThreads = threads_of(K), kTile = tile_of(K);
    __shared__ __align__(16) float step[kTile][kCh][2];   // delta, delta x
    __shared__ __align__(16) float rows_b[kTile * NP], rows_c[MODE == kEnds ? 4 : kTile * NP];
    __shared__ __align__(16) float sums[MODE == kMain ? kTile : 1][4][kRow];   // a quarter's part of y
    __shared__ __align__(16) float grad[MODE == kBoth ? kTile : 1][kCh];       // the gradient of y
    pdl_wait();
    pdl_launch_dependents();
    const Place at(a, blockIdx.x);
    const int lane = threadIdx.x & 31, ch = ((threadIdx.x >> 5) * 8 + (lane & 7)) * K, quarter = lane >> 3, n0 = quarter * NS;
    const int t0 = at.seg * a.seg, t1 = min(t0 + a.seg, a.L);
    f32x2 rate[K][P], h[K][P];
    const long long slot = (((long long)at.b * a.segs + at.seg) * a.C + at.c0 + ch) * NP + n0, own = ((long long)at.b * a.C + at.c0 + ch) * a.N;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool live = ch + k < at.live;
        load_states<NS, MODE == kMain>(a.A + (long long)(at.c0 + ch + k) * a.N, live ? a.N : 0, n0, rate[k]);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            rate[k][i] = rate_of2(rate[k][i]);
            h[k][i] = 0;
        }
        if (MODE == kMain && live) {
            if (a.segs > 1) load_pairs<NS>(a.ends + slot + k * NP, h[k]);
            else if (a.state_in) load_states<NS, true>(a.state_in + own + k * a.N, a.N, n0, h[k]);
        }
    }
    // element-wise: token et of a tile, channels ec .. ec + 3
    const int et = threadIdx.x / (kCh / 4), ec = (threadIdx.x % (kCh / 4)) * 4;
    const bool mine = ec < at.live;
    const int g0 = at.c0 + (mine ? ec : 0);
    f32x2 bias[2], skip[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        bias[j] = a.bias ? pack2(a.bias[g0 + 2 * j], a.bias[g0 + 2 * j + 1]) : 0;
        skip[j] = MODE == kMain && a.D ? pack2(a.D[g0 + 2 * j], a.D[g0 + 2 * j + 1]) : 0;
    }
    const long long r0 = a.row(at.b, t0 + et), way = a.reverse ? -kTile : kTile;
    const T *px = a.x + r0 * a.ldx + g0, *pd = a.dt + r0 * a.lddt + g0, *pz = a.z + r0 * a.ldz + g0, *po = a.d_out + r0 * a.ldo + g0;
    T* out = a.out + r0 * a.ldo + g0;
    typename Four<T>::Raw rx = {}, rd = {}, rz = {}, ro = {};
    Rows<T, NP, kTile, kThreads, MODE == kMain> rb, rc;
    rb.start(a.Bt, a, a.ldB, at, t0);
    rc.start(a.Ct, a, a.ldC, at, t0);
    auto load = [&](int t) {   // a tile, and on to the next one
        if (mine && t + et < t1) {
            rx = load4(px);
            rd = load4(pd);
            if (MODE != kEnds && a.z) rz = load4(pz);
            if (MODE == kBoth) ro = load4(po);
        }
        px += way * a.ldx;
        pd += way * a.lddt;
        if (MODE != kEnds) pz += way * a.ldz;
        if (MODE == kBoth) po += way * a.ldo;
        rb.load(t, t1, a.N);
        rb.move(kTile);
        if (MODE != kEnds) {
            rc.load(t, t1, a.N);
            rc.move(kTile);
        }
    };
    f32x2 decay[K][P], back[K][P];   // kBoth
    float total[K] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i) {
            decay[k][i] = both(1.f);
            back[k][i] = 0;
        }
    load(t0);
    for (int t = t0; t < t1; t += kTile) {
        const typename Four<T>::Raw cx = rx, cz = rz;
        const bool there = mine && t + et < t1;
        {
            f32x2 x[2], z[2], d[2], o[2];
            widen4(rx, x);
            widen4(rd, d);
            widen4(rz, z);
            widen4(ro, o);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f32x2 delta = fadd2(d[j], bias[j]);
                if (a.softplus) delta = softplus2(delta, exp_minus_abs<T>(delta));
                f32x2 in = fmul2(delta, x[j]);
                if (!there) delta = in = 0;   // (decay one, nothing added)
                put_step(&step[et][ec + 2 * j], delta, in);
                if (MODE == kBoth) {
                    if (a.z) o[j] = fmul2(o[j], fmul2(z[j], sigmoid2<T>(z[j])));
                    if (!there) o[j] = 0;
                }
            }
            if (MODE == kBoth) store4(&grad[et][ec], o);
            rb.put(rows_b);
            if (MODE == kMain) rc.put_reduced(rows_c, a.N);
            if (MODE == kBoth) rc.put(rows_c);
        }
        __syncthreads();
        if (t + kTile < t1) load(t + kTile);
#pragma unroll 1
        for (int s = 0; s < kTile && t + s < t1; s += 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f32x2 bt[P], ct[P];
                float d[2 * K], dy[K], part[K];
                load_floats<2 * K>(&step[s + j][ch][0], d);
                load_pairs<NS>(&rows_b[(s + j) * NP + n0], bt);
                if (MODE != kEnds) load_pairs<NS>(&rows_c[(s + j) * NP + n0], ct);
                if (MODE == kBoth) load_floats<K>(&grad[s + j][ch], dy);
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const f32x2 delta = both(d[2 * k]), in = both(d[2 * k + 1]);
                    f32x2 y = 0;
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const f32x2 e = decay2<T>(fmul2(rate[k][i], delta));
                        h[k][i] = ffma2(e, h[k][i], fmul2(in, bt[i]));
                        if (MODE == kMain) y = i == 0 ? fmul2(ct[i], h[k][i]) : ffma2(ct[i], h[k][i], y);
                        if (MODE == kBoth) {
                            decay[k][i] = fmul2(decay[k][i], e);
                            back[k][i] = ffma2(decay[k][i], fmul2(ct[i], both(dy[k])), back[k][i]);
                        }
                    }
                    if (MODE == kMain) part[k] = sum2(y);
                    else total[k] += d[2 * k];
                }
                if (MODE == kMain) store_floats<K>(&sums[s + j][quarter][ch], part);
            }
        }
        __syncthreads();
        if (MODE == kMain) {
            if (there) {
                f32x2 x[2], z[2], y[2], part[2];
                widen4(cx, x);
                widen4(cz, z);
                load_pairs<4>(&sums[et][0][ec], y);
#pragma unroll
                for (int q = 1; q < 4; ++q) {
                    load_pairs<4>(&sums[et][q][ec], part);
                    y[0] = fadd2(y[0], part[0]);
                    y[1] = fadd2(y[1], part[1]);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    y[j] = ffma2(skip[j], x[j], y[j]);
                    if (a.z) y[j] = fmul2(y[j], fmul2(z[j], sigmoid2<T>(z[j])));
                }
                store4(out, y);
            }
            out += way * a.ldo;
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (ch + k >= at.live) break;
        if (MODE == kMain) {
            if (a.state_out && at.seg == a.segs - 1) store_states<NS>(a.state_out + own + k * a.N, a.N, n0, h[k]);
        } else {
            store_pairs<NS>(a.ends + slot + k * NP, h[k]);
            if (MODE == kBoth) store_pairs<NS>(a.adjoint + slot + k * NP, back[k]);
            if (quarter == 0) a.total[((long long)at.b * a.segs + at.seg) * a.C + at.c0 + ch + k] = total[k];
        }
    }
}

// The states in front of the segments from what each adds, and from behind the adjoint's: a thread a state.
template <typename T>
__global__ void __launch_bounds__(128) ssm_carry_kernel(Ssm<T> a, int NP) {
    pdl_wait();
    pdl_launch_dependents();
    const long long id = (long long)blockIdx.x * 128 + threadIdx.x, each = (long long)a.C * NP;
    const int b = (int)(id / each);
    if (b >= a.B) return;
    const int at = (int)(id - b * each), c = at / NP, n = at % NP;
    // behind the last state, the outputs' launch has that one again, and the gradient's zero
    const bool there = n < a.N, gradient = gridDim.y == 2;
    if (!there && !gradient) return;
    const bool last = n == a.N - 1 && n != NP - 1 && !gradient;
    const float rate = there ? rate_of(a.A[(long long)c * a.N + n]) : 0.f;
    const long long own = ((long long)b * a.C + c) * a.N + n;
    float* ends = a.ends + (long long)b * a.segs * each + at;
    const float* total = a.total + (long long)b * a.segs * a.C + c;
    const bool back = blockIdx.y == 1;   // (a grid of two rows in the gradient)
    float* p = back ? a.adjoint + (long long)b * a.segs * each + at : ends;
    const float* first = back ? a.d_state_out : a.state_in;
    float h = there && first ? first[own] : 0.f;
    constexpr int kAhead = 8;
    for (int s = 0; s < a.segs; s += kAhead) {
        float add[kAhead], sum[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = back ? a.segs - 1 - s - i : s + i;
            const bool in = s + i < a.segs;
            add[i] = in && there ? p[k * each] : 0.f;
            sum[i] = in ? total[(long long)k * a.C] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (s + i >= a.segs) break;
            const int k = back ? a.segs - 1 - s - i : s + i;
            p[k * each] = h;
            if (last)
#pragma unroll 1
                for (int more = 1; more < NP - n; ++more) p[k * each + more] = h;
            h = fmaf(decay_of<T>(rate * sum[i]), h, add[i]);
        }
    }
}

// One token: four states a thread, `lanes` threads a channel.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(128) ssm_step_kernel(Ssm<T> a, float* state, int lanes) {
    pdl_wait();
    pdl_launch_dependents();
    const long long id = (long long)blockIdx.x * 128 + threadIdx.x, unit = id / lanes;
    const int sub = (int)(id - unit * lanes), n0 = 4 * sub;
    const bool live = unit < (long long)a.B * a.C;
    const int b = live ? (int)(unit / a.C) : 0, c = live ? (int)(unit - (long long)b * a.C) : 0;
    const int group = c / a.per;
    float h[4], A[4], Bt[4], Ct[4];
    float* s = state + ((long long)b * a.C + c) * a.N + n0;
    const float* rate = a.A + (long long)c * a.N + n0;
    const T *pb = a.Bt + b * a.ldB + group * a.N + n0, *pc = a.Ct + b * a.ldC + group * a.N + n0;
    if (WIDE && n0 < a.N) {
        load_floats<4>(s, h);
        load_floats<4>(rate, A);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool there = n0 + j < a.N;
        if (!WIDE || n0 >= a.N) h[j] = there ? s[j] : 0.f;
        if (!WIDE || n0 >= a.N) A[j] = there ? rate[j] : 0.f;
        Bt[j] = there ? to_f32(pb[j]) : 0.f;
        Ct[j] = there ? to_f32(pc[j]) : 0.f;
    }
    const float x = to_f32(a.x[b * a.ldx + c]), v = to_f32(a.dt[b * a.lddt + c]) + (a.bias ? a.bias[c] : 0.f);
    const float z = a.z ? to_f32(a.z[b * a.ldz + c]) : 0.f, skip = a.D ? a.D[c] : 0.f;
    const float delta = a.softplus ? softplus_of<T>(v) : v, in = delta * x;
    float y = 0.f;
    const bool still = delta == 0.f;   // (keeps the state at any rate, one of minus infinity too)
#pragma unroll
    for (int j = 0; j < 4; ++j) {   // (decays of fp32 calls from the special-function unit too: as arithmetic they take a tenth of the time)
        const float e = ex2(delta * (A[j] * kLog2E));
        h[j] = fmaf(still ? 1.f : e, h[j], in * Bt[j]);
        if (WIDE || n0 + j < a.N) y = fmaf(Ct[j], h[j], y);
    }
    if (WIDE && n0 >= a.N) y = 0.f;   // (where there is no state, an infinite delta x times zero is NaN)
    if (live) {
        if (WIDE && n0 < a.N) *reinterpret_cast<float4*>(s) = make_float4(h[0], h[1], h[2], h[3]);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n0 + j < a.N) s[j] = h[j];
    }
    for (int o = lanes / 2; o > 0; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
    if (!live || sub != 0) return;
    y = fmaf(skip, x, y);
    if (a.z) y *= z * sigmoid_of<T>(z);
    from_f32(a.out + b * a.ldo + c, y);
}

template <typename T, int NS, int K, int MODE>
cudaError_t walk_of(const Ssm<T>& a, cudaStream_t stream) {
    count_launch();
    return launch_pdl(ssm_kernel<T, NS, K, MODE>, dim3((unsigned)a.items), dim3(threads_of(K)), 0, stream, a);
}
template <typename T, int MODE>
cudaError_t walk(const Ssm<T>& a, cudaStream_t stream) {
    switch (ssm_padded(a.N)) {
        case 8: return walk_of<T, 2, 2, MODE>(a, stream);
        case 16: return walk_of<T, 4, 2, MODE>(a, stream);
        default: return walk_of<T, 8, 1, MODE>(a, stream);
    }
}

}  // namespace

// Segments where whole sequences would leave SMs idle: as many as make one round of blocks (five an SM, in the gradient four), of 64 tokens or
// more.  Two passes over the exponentials instead of one, so not where whole sequences fill half a round.  8 x 4096 x 384: 160 us, 176 with
// four fifths of a round and a bit, 192 with four fifths, 167 with six fifths; 1 x 16384 x 768: 157, 189, 188, 163.
// In the gradient segments are no longer than 16 GiB of kept states allow (28336 tokens with more than eight states where a whole round of blocks
// runs), a tenth of the memory, at the price of the second pass: 32 x 16384 x 1152 22.5 ms in segments of 7 Ki, 18.7 whole.
constexpr long long kMostKept = 16LL << 30;
template <typename T>
void ssm_segments(Ssm<T>& a, bool gradient) {
    a.blocks = (a.per + kCh - 1) / kCh;
    const long long whole = (long long)a.B * a.G * a.blocks, want = 148 * (gradient ? 4 : 5);
    long long segs = whole >= want / 2 ? 1 : want / (whole > 0 ? whole : 1);
    const long long most = (a.L + 63LL) / 64;
    if (segs > most) segs = most;
    if (segs < 1) segs = 1;
    if (gradient) {
        // bytes kept for a token by the blocks that run, were every segment long
        const int padded = ssm_padded(a.N);
        const long long each = kSsmChannels * (long long)padded * sizeof(float) / kSsmKept, running = 148LL * ssm_grad_blocks(padded);
        const long long longest = kMostKept / (each * running) / kSsmTile * kSsmTile;
        if (whole * a.L > kMostKept / each && (a.L + segs - 1) / segs > longest) segs = (a.L + longest - 1) / longest;
    }
    long long seg = (a.L + segs - 1) / segs;
    seg = (seg + kSsmTile - 1) / kSsmTile * kSsmTile;
    a.seg = (int)(seg < kSsmTile ? kSsmTile : seg);
    a.segs = (int)((a.L + (long long)a.seg - 1) / a.seg);
    if (a.segs < 1) a.segs = 1;
    a.items = whole * a.segs;
}
size_t ssm_segment_floats(int B, int C, int N, int segs) { return (size_t)B * segs * C * ssm_padded(N); }

template <typename T>
cudaError_t launch_ssm_segments(const Ssm<T>& a, bool gradient, cudaStream_t stream) {
    const cudaError_t e = gradient ? walk<T, kBoth>(a, stream) : walk<T, kEnds>(a, stream);
    if (e != cudaSuccess) return e;
    const int NP = ssm_padded(a.N);
    count_launch();
    return launch_pdl(ssm_carry_kernel<T>, dim3((unsigned)(((long long)a.B * a.C * NP + 127) / 128), gradient ? 2 : 1), dim3(128), 0, stream, a, NP);
}
template <typename T>
cudaError_t launch_ssm_fwd(const Ssm<T>& a, cudaStream_t stream) {
    if (a.segs > 1) {
        const cudaError_t e = launch_ssm_segments<T>(a, false, stream);
        if (e != cudaSuccess) return e;
    }
    return walk<T, kMain>(a, stream);
}
template <typename T>
cudaError_t launch_ssm_step(const Ssm<T>& a, float* state, cudaStream_t stream) {
    int lanes = 1;
    while (4 * lanes < a.N) lanes *= 2;
    const dim3 grid((unsigned)(((long long)a.B * a.C * lanes + 127) / 128));
    count_launch();
    if (a.N % 4 == 0 && (reinterpret_cast<uintptr_t>(a.A) & 15u) == 0) return launch_pdl(ssm_step_kernel<T, true>, grid, dim3(128), 0, stream, a, state, lanes);
    return launch_pdl(ssm_step_kernel<T, false>, grid, dim3(128), 0, stream, a, state, lanes);
}

#define VIG_INSTANCES(T)                                                                      \
    template void ssm_segments<T>(Ssm<T>&, bool);                                             \
    template cudaError_t launch_ssm_segments<T>(const Ssm<T>&, bool, cudaStream_t);           \
    template cudaError_t launch_ssm_fwd<T>(const Ssm<T>&, cudaStream_t);                      \
    template cudaError_t launch_ssm_step<T>(const Ssm<T>&, float*, cudaStream_t);
VIG_INSTANCES(__nv_bfloat16)
VIG_INSTANCES(float)

}  // namespace vig
