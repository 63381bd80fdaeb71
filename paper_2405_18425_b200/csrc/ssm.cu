// Selective state space scan: forward pass, the states in front of segments, and the single-token form.
//
//   delta_t = softplus(dt_t + bias);  h_t[n] = e^(delta_t A[c,n]) h_{t-1}[n] + delta_t x_t B_t[n];  y_t = sum_n C_t[n] h_t[n] + D x_t
//   out_t = y_t z_t sigmoid(z_t)
//
// The recurrence has an exponential for every token, channel and state, sixteen a clock and SM from the special-function unit: that bounds
// it, not memory.  So a state lives in a register from its first token to its last, pairs of states share an instruction, and everything
// that belongs to a token and channel alone is computed once (ssm.cuh).  Sequences of few channels are cut into segments: a first launch
// gives what each segment adds to the state behind it and the sum of its step sizes (its decay is e^(A sum), so no products are
// kept), a small one carries the states through, and the launch proper starts every segment from its own.
#include "ssm.cuh"

namespace vig {
namespace {

using namespace ssm;

constexpr int kMain = 0, kEnds = 1, kBoth = 2;   // kEnds: a segment's end state; kBoth: and what its outputs' gradients add to the adjoint in front

template <typename T, int NS, int MODE>
__global__ void __launch_bounds__(kThreads, NS <= 4 ? 4 : 2) ssm_kernel(Ssm<T> a) {
    constexpr int NP = 4 * NS, P = NS / 2;
    __shared__ __align__(16) float step[kTile][kCh][4];   // delta, delta, delta x, delta x: pairs as the products take them
    __shared__ __align__(16) float rows_b[kTile * NP], rows_c[MODE == kEnds ? 4 : kTile * NP];
    __shared__ __align__(16) float sums[MODE == kEnds ? 1 : kTile][kRow];   // y; kBoth: the gradient of y
    pdl_wait();
    pdl_launch_dependents();
    const Place at(a, blockIdx.x);
    const int lane = threadIdx.x & 31, ch = (threadIdx.x >> 5) * 8 + (lane & 7), quarter = lane >> 3, n0 = quarter * NS;
    const bool live = ch < at.live;
    const int c = at.c0 + (live ? ch : 0);
    const int t0 = at.seg * a.seg, t1 = min(t0 + a.seg, a.L);
    f32x2 rate[P], h[P];
    load_states<NS>(a.A + (long long)c * a.N, live ? a.N : 0, n0, rate);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        rate[i] = fmul2(rate[i], pack2(kLog2E, kLog2E));
        h[i] = 0;
    }
    const long long slot = (((long long)at.b * a.segs + at.seg) * a.C + c) * NP + n0;
    if (MODE == kMain && live) {
        if (a.segs > 1) load_pairs<NS>(a.ends + slot, h);
        else if (a.state_in) load_states<NS>(a.state_in + ((long long)at.b * a.C + c) * a.N, a.N, n0, h);
    }
    // element-wise: token et of a tile, channels ec .. ec + 3
    const int et = threadIdx.x / 16, ec = (threadIdx.x % 16) * 4;
    const bool mine = ec < at.live;
    const int g0 = at.c0 + ec;
    float bias[4] = {}, skip[4] = {};
    if (mine) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (a.bias) bias[j] = a.bias[g0 + j];
            if (MODE == kMain && a.D) skip[j] = a.D[g0 + j];
        }
    }
    typename Four<T>::Raw rx = {}, rd = {}, rz = {}, ro = {};
    Rows<T, NP> rb, rc;
    auto load = [&](int t) {
        const int tt = t + et;
        if (mine && tt < t1) {
            const long long r = a.row(at.b, tt);
            rx = load4(a.x + r * a.ldx + g0);
            rd = load4(a.dt + r * a.lddt + g0);
            if (MODE != kEnds && a.z) rz = load4(a.z + r * a.ldz + g0);
            if (MODE == kBoth) ro = load4(a.d_out + r * a.ldo + g0);
        }
        rb.load(a.Bt, a, a.ldB, at, t);
        if (MODE != kEnds) rc.load(a.Ct, a, a.ldC, at, t);
    };
    f32x2 decay[P], back[P];   // kBoth
#pragma unroll
    for (int i = 0; i < P; ++i) {
        decay[i] = pack2(1.f, 1.f);
        back[i] = 0;
    }
    float total = 0.f;
    load(t0);
    for (int t = t0; t < t1; t += kTile) {
        float x[4], z[4];
        {
            float d[4], o[4];
            widen4(rx, x);
            widen4(rd, d);
            widen4(rz, z);
            widen4(ro, o);
            const bool there = mine && t + et < t1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = d[j] + bias[j];
                float delta = a.softplus ? softplus_of(v, exp_minus_abs<T>(v)) : v;
                if (!there) delta = 0.f;   // (decay one, nothing added)
                const float in = there ? delta * x[j] : 0.f;
                *reinterpret_cast<float4*>(&step[et][ec + j][0]) = make_float4(delta, delta, in, in);
                if (MODE == kBoth) {
                    const float gate = a.z ? z[j] * sigmoid_of<T>(z[j], exp_minus_abs<T>(z[j])) : 1.f;
                    sums[et][ec + j] = there ? o[j] * gate : 0.f;
                }
            }
            rb.put(rows_b);
            if (MODE != kEnds) rc.put(rows_c);
        }
        __syncthreads();
        if (t + kTile < t1) load(t + kTile);
#pragma unroll 1
        for (int s = 0; s < kTile; s += 4) {
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const ulonglong2 d = *reinterpret_cast<const ulonglong2*>(&step[s + j][ch][0]);
                f32x2 bt[P], ct[P], y = 0;
                load_pairs<NS>(&rows_b[(s + j) * NP + n0], bt);
                if (MODE != kEnds) load_pairs<NS>(&rows_c[(s + j) * NP + n0], ct);
                if (MODE == kBoth) y = pack2(sums[s + j][ch], sums[s + j][ch]);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const f32x2 e = exp2_pair(fmul2(rate[i], d.x));
                    h[i] = ffma2(e, h[i], fmul2(d.y, bt[i]));
                    if (MODE == kMain) y = ffma2(ct[i], h[i], y);
                    if (MODE == kBoth) {
                        decay[i] = fmul2(decay[i], e);
                        back[i] = ffma2(decay[i], fmul2(ct[i], y), back[i]);
                    }
                }
                p[j] = sum2(y);
                if (MODE != kMain) {
                    float lo, hi;
                    unpack2(d.x, lo, hi);
                    total += lo;
                }
            }
            if (MODE == kMain) sums[s + quarter][ch] = over_quarters(p[0], p[1], p[2], p[3], quarter);
        }
        __syncthreads();
        if (MODE == kMain && mine && t + et < t1) {
            const float4 s4 = *reinterpret_cast<const float4*>(&sums[et][ec]);
            float y[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = fmaf(skip[j], x[j], y[j]);
                if (a.z) y[j] *= z[j] * sigmoid_of<T>(z[j], exp_minus_abs<T>(z[j]));
            }
            store4(a.out + a.row(at.b, t + et) * a.ldo + g0, y);
        }
    }
    if (!live) return;
    if (MODE == kMain) {
        if (a.state_out && at.seg == a.segs - 1) store_states<NS>(a.state_out + ((long long)at.b * a.C + c) * a.N, a.N, n0, h);
    } else {
        store_pairs<NS>(a.ends + slot, h);
        if (MODE == kBoth) store_pairs<NS>(a.adjoint + slot, back);
        if (quarter == 0) a.total[((long long)at.b * a.segs + at.seg) * a.C + c] = total;
    }
}

// The states in front of the segments from what each adds, and from behind the adjoint's: a thread a state.
template <typename T>
__global__ void __launch_bounds__(128) ssm_carry_kernel(Ssm<T> a, int NP, bool gradient) {
    pdl_wait();
    pdl_launch_dependents();
    const long long id = (long long)blockIdx.x * 128 + threadIdx.x, each = (long long)a.C * NP;
    const int b = (int)(id / each);
    if (b >= a.B) return;
    const int at = (int)(id - b * each), c = at / NP, n = at % NP;
    const bool there = n < a.N;
    const float rate = there ? a.A[(long long)c * a.N + n] * kLog2E : 0.f;
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
            add[i] = in ? p[k * each] : 0.f;
            sum[i] = in ? total[(long long)k * a.C] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (s + i >= a.segs) break;
            const int k = back ? a.segs - 1 - s - i : s + i;
            p[k * each] = h;
            h = fmaf(ex2(rate * sum[i]), h, add[i]);
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
        const float4 u = *reinterpret_cast<const float4*>(s);
        h[0] = u.x; h[1] = u.y; h[2] = u.z; h[3] = u.w;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool there = n0 + j < a.N;
        if (!WIDE || n0 >= a.N) h[j] = there ? s[j] : 0.f;
        A[j] = there ? rate[j] * kLog2E : 0.f;
        Bt[j] = there ? to_f32(pb[j]) : 0.f;
        Ct[j] = there ? to_f32(pc[j]) : 0.f;
    }
    const float x = to_f32(a.x[b * a.ldx + c]), v = to_f32(a.dt[b * a.lddt + c]) + (a.bias ? a.bias[c] : 0.f);
    const float z = a.z ? to_f32(a.z[b * a.ldz + c]) : 0.f, skip = a.D ? a.D[c] : 0.f;
    const float delta = a.softplus ? softplus_of(v, exp_minus_abs<T>(v)) : v, in = delta * x;
    float y = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[j] = fmaf(ex2(delta * A[j]), h[j], in * Bt[j]);
        y = fmaf(Ct[j], h[j], y);
    }
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
    if (a.z) y *= z * sigmoid_of<T>(z, exp_minus_abs<T>(z));
    from_f32(a.out + b * a.ldo + c, y);
}

template <typename T, int MODE>
cudaError_t walk(const Ssm<T>& a, cudaStream_t stream) {
    const dim3 grid((unsigned)a.items);
    count_launch();
    switch (ssm_padded(a.N)) {
        case 8: return launch_pdl(ssm_kernel<T, 2, MODE>, grid, dim3(kThreads), 0, stream, a);
        case 16: return launch_pdl(ssm_kernel<T, 4, MODE>, grid, dim3(kThreads), 0, stream, a);
        default: return launch_pdl(ssm_kernel<T, 8, MODE>, grid, dim3(kThreads), 0, stream, a);
    }
}

}  // namespace

// Segments where whole sequences would leave SMs idle: as many as give every SM four blocks, of 64 tokens or more.
template <typename T>
void ssm_segments(Ssm<T>& a, bool gradient) {
    a.blocks = (a.per + kCh - 1) / kCh;
    const long long whole = (long long)a.B * a.G * a.blocks, want = 148 * (gradient ? 2 : 4);
    long long segs = whole >= want / 2 ? 1 : (want + whole - 1) / (whole > 0 ? whole : 1);
    const long long most = (a.L + 63LL) / 64;
    if (segs > most) segs = most;
    if (segs < 1) segs = 1;
    long long seg = (a.L + segs - 1) / segs;
    seg = (seg + kTile - 1) / kTile * kTile;
    a.seg = (int)(seg < kTile ? kTile : seg);
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
    return launch_pdl(ssm_carry_kernel<T>, dim3((unsigned)(((long long)a.B * a.C * NP + 127) / 128), gradient ? 2 : 1), dim3(128), 0, stream, a, NP, gradient);
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
    if (a.N % 4 == 0) return launch_pdl(ssm_step_kernel<T, true>, grid, dim3(128), 0, stream, a, state, lanes);
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
