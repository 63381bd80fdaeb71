// Depth-wise convolution along the tokens that looks back only, with an optional SiLU, its gradient and its single-token form.
//
//   v_t = bias + sum_{k < K} w_k x_{t - K + 1 + k},  out_t = act(v_t);  x_{-(K-1)} .. x_{-1}: state_in, or zeros
//   gradient:  g_t = d_out_t act'(v_t);  dx_s = sum_j w_{K-1-j} g_{s+j};  dw_k = sum g_t x_{t-K+1+k};  dbias = sum g_t
//
// Memory bounds it: a thread walks over a piece of a sequence with the 16-byte vectors of its channels, the last K values of x (in the
// gradient of g too) in registers, so a value is read once, but for the K - 1 tokens beside a piece.  8 x 4096 x 384 bf16, K 4: 17 us (0.45 of a
// copy's rate); 64 x 196 x 1152: 19 us, its gradient 49 (248 registers, two blocks an SM) and 5 for the filters' last sums.
#include "layers.h"
#include "wide.cuh"

namespace vig {
namespace {

constexpr int kThreads = 128;
constexpr int kAhead = 4;   // tokens whose loads are in flight together

// out = act(v) and act'(v); the bf16 results' sigmoid from the special-function unit.
template <typename T>
__device__ __forceinline__ float sig(float v) { return sizeof(T) == 2 ? sigmoid(v) : 1.f / (1.f + expf(-v)); }

template <typename T, int K>
struct Taps {
    static constexpr int N = Vec<T>::N;
    float w[K][N], b[N];
    __device__ __forceinline__ Taps(const T* weight, const T* bias, int c) {
        uint4 raw[K];   // [N channels][K] is K vectors
#pragma unroll
        for (int i = 0; i < K; ++i) raw[i] = load16(weight + (long long)c * K + i * N);
        float f[K][N];
#pragma unroll
        for (int i = 0; i < K; ++i) widen(raw[i], f[i], (const T*)nullptr);
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][j] = f[(j * K + k) / N][(j * K + k) % N];
        widen(bias ? load16(bias + c) : make_uint4(0, 0, 0, 0), b, (const T*)nullptr);
    }
};

// The vector of a token in walking order, in front of the first one of the state.
template <typename T, int K>
__device__ __forceinline__ uint4 at(const Conv<T>& a, int b, int t, int c) {
    if (t >= 0) return t < a.L ? load16(a.x + a.row(b, t) * a.ldx + c) : make_uint4(0, 0, 0, 0);
    return a.state_in && t >= 1 - K ? load16(a.state_in + ((long long)b * (K - 1) + t + K - 1) * a.C + c) : make_uint4(0, 0, 0, 0);
}

template <typename T, int K, bool SILU>
__global__ void __launch_bounds__(kThreads) conv_kernel(Conv<T> a) {
    constexpr int N = Vec<T>::N;
    pdl_wait();
    pdl_launch_dependents();
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int nv = a.C / N;
    const long long rest = id / nv;
    const int c = (int)(id - rest * nv) * N;
    const int b = (int)(rest / a.pieces), t0 = (int)(rest % a.pieces) * a.piece;
    if (b >= a.B) return;
    const int t1 = min(t0 + a.piece, a.L);
    const Taps<T, K> taps(a.w, a.bias, c);
    uint4 first[K - 1];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) first[k] = at<T, K>(a, b, t0 - K + 1 + k, c);
    if (a.state_out && t0 == 0) {   // by the thread that reads state_in, so that the two may be one
        uint4 last[K - 1];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) last[k] = at<T, K>(a, b, a.L - K + 1 + k, c);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) store16(a.state_out + ((long long)b * (K - 1) + k) * a.C + c, last[k]);
    }
    float x[K][N];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) widen(first[k], x[k + 1], (const T*)nullptr);
    const long long way = a.reverse ? -1 : 1;
    const T* in = a.x + a.row(b, t0) * a.ldx + c;
    T* out = a.out + a.row(b, t0) * a.ldo + c;
    for (int t = t0; t < t1; t += kAhead) {
        uint4 raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = t + i < t1 ? load16(in + way * i * a.ldx) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) x[k][j] = x[k + 1][j];
            widen(raw[i], x[K - 1], (const T*)nullptr);
            float y[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float v = taps.b[j];
#pragma unroll
                for (int k = 0; k < K; ++k) v = fmaf(taps.w[k][j], x[k][j], v);
                y[j] = SILU ? v * sig<T>(v) : v;
            }
            if (t + i < t1) store16(out + way * i * a.ldo, narrow(y, (const T*)nullptr));
        }
        in += way * kAhead * a.ldx;
        out += way * kAhead * a.ldo;
    }
}

// A piece's thread gives dx of its tokens: it walks K - 1 tokens further for their g.  The first piece gives the window in front of the
// sequence too.
template <typename T, int K, bool SILU>
__global__ void __launch_bounds__(kThreads) conv_bwd_kernel(Conv<T> a) {
    constexpr int N = Vec<T>::N;
    pdl_wait();
    pdl_launch_dependents();
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int nv = a.C / N;
    const long long rest = id / nv;
    const int c = (int)(id - rest * nv) * N;
    const int b = (int)(rest / a.pieces), t0 = (int)(rest % a.pieces) * a.piece;
    if (b >= a.B) return;
    const int t1 = min(t0 + a.piece, a.L);
    const Taps<T, K> taps(a.w, a.bias, c);
    float x[K][N], g[K][N], dw[K][N], db[N];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < N; ++j) g[k][j] = dw[k][j] = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) db[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) widen(at<T, K>(a, b, t0 - K + 1 + k, c), x[k + 1], (const T*)nullptr);
    const int from = t0 == 0 ? 1 - K : t0;   // tokens whose dx this thread gives
    for (int t = t0; t < t1 + K - 1; t += kAhead) {
        uint4 raw[kAhead], up[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const bool there = t + i < a.L && t + i < t1 + K - 1;
            raw[i] = there ? load16(a.x + a.row(b, t + i) * a.ldx + c) : make_uint4(0, 0, 0, 0);
            up[i] = there ? load16(a.d_out + a.row(b, t + i) * a.ldo + c) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int tt = t + i;
            if (tt >= t1 + K - 1) break;
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    x[k][j] = x[k + 1][j];
                    g[k][j] = g[k + 1][j];
                }
            widen(raw[i], x[K - 1], (const T*)nullptr);
            float d[N];
            widen(up[i], d, (const T*)nullptr);
            if (tt < a.L) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float slope = 1.f;
                    if (SILU) {
                        float v = taps.b[j];
#pragma unroll
                        for (int k = 0; k < K; ++k) v = fmaf(taps.w[k][j], x[k][j], v);
                        const float s = sig<T>(v);
                        slope = s * fmaf(v, 1.f - s, 1.f);
                    }
                    g[K - 1][j] = d[j] * slope;
                }
                if (tt < t1) {   // (the tokens behind the piece are another thread's)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        db[j] += g[K - 1][j];
#pragma unroll
                        for (int k = 0; k < K; ++k) dw[k][j] = fmaf(g[K - 1][j], x[k][j], dw[k][j]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) g[K - 1][j] = 0.f;
            }
            const int s = tt - K + 1;   // its g: g[0] of token s .. g[K-1] of token s + K - 1
            if (s < from || (s < 0 && !a.d_state_in)) continue;
            float dx[N];
            const int tail = s - (a.L - (K - 1));   // its place in state_out
            widen(tail >= 0 && a.d_state_out ? load16(a.d_state_out + ((long long)b * (K - 1) + tail) * a.C + c) : make_uint4(0, 0, 0, 0), dx,
                  (const T*)nullptr);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) dx[j] = fmaf(taps.w[K - 1 - k][j], g[k][j], dx[j]);
            const uint4 y = narrow(dx, (const T*)nullptr);
            if (s >= 0) store16(a.dx + a.row(b, s) * a.lddx + c, y);
            else store16(a.d_state_in + ((long long)b * (K - 1) + s + K - 1) * a.C + c, y);
        }
    }
    if (!a.part) return;
    float* part = a.part + rest * ((long long)a.C * (K + 1));
    float line[N * K];   // [N channels][K], as the weights lie
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int k = 0; k < K; ++k) line[j * K + k] = dw[k][j];
#pragma unroll
    for (int i = 0; i < N * K; i += 4) *reinterpret_cast<float4*>(part + (long long)c * K + i) = make_float4(line[i], line[i + 1], line[i + 2], line[i + 3]);
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(part + (long long)a.C * K + c + j) = make_float4(db[j], db[j + 1], db[j + 2], db[j + 3]);
}

// One token of each sequence; the window moves on by one.
template <typename T, int K, bool SILU>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(Conv<T> a, T* state) {
    constexpr int N = Vec<T>::N;
    pdl_wait();
    pdl_launch_dependents();
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int nv = a.C / N;
    const long long b = id / nv;
    const int c = (int)(id - b * nv) * N;
    if (b >= a.B) return;
    uint4 raw[K];
    T* s = state + b * (K - 1) * a.C + c;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) raw[k] = load16(s + (long long)k * a.C);
    raw[K - 1] = load16(a.x + b * a.ldx + c);
    const Taps<T, K> taps(a.w, a.bias, c);
    float y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = taps.b[j];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float x[N];
        widen(raw[k], x, (const T*)nullptr);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = fmaf(taps.w[k][j], x[j], y[j]);
        if (k > 0) store16(s + (long long)(k - 1) * a.C, raw[k]);
    }
    if (SILU)
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] *= sig<T>(y[j]);
    store16(a.out + b * a.ldo + c, narrow(y, (const T*)nullptr));
}

template <typename F>
cudaError_t by_width(int K, int act, F f) {
    const bool silu = act == VIG_ACT_SILU;
    count_launch();
    switch (K) {
        case 2: return silu ? f.template operator()<2, true>() : f.template operator()<2, false>();
        case 3: return silu ? f.template operator()<3, true>() : f.template operator()<3, false>();
        default: return silu ? f.template operator()<4, true>() : f.template operator()<4, false>();
    }
}
template <typename T>
dim3 grid_of(const Conv<T>& a) {
    return dim3((unsigned)(((long long)a.B * a.pieces * (a.C / Vec<T>::N) + kThreads - 1) / kThreads));
}

template <typename T>
struct Forward {
    const Conv<T>& a;
    cudaStream_t stream;
    template <int K, bool SILU>
    cudaError_t operator()() const { return launch_pdl(conv_kernel<T, K, SILU>, grid_of(a), dim3(kThreads), 0, stream, a); }
};
template <typename T>
struct Gradient {
    const Conv<T>& a;
    cudaStream_t stream;
    template <int K, bool SILU>
    cudaError_t operator()() const { return launch_pdl(conv_bwd_kernel<T, K, SILU>, grid_of(a), dim3(kThreads), 0, stream, a); }
};
template <typename T>
struct Step {
    const Conv<T>& a;
    T* state;
    cudaStream_t stream;
    template <int K, bool SILU>
    cudaError_t operator()() const { return launch_pdl(conv_step_kernel<T, K, SILU>, grid_of(a), dim3(kThreads), 0, stream, a, state); }
};

}  // namespace

// The longest pieces that still give every SM the threads that its registers hold (640; the gradient, which leaves partial sums of K + 1
// values a channel and piece too, 256, once and a half): the K - 1 tokens beside a piece are read twice.
template <typename T>
void conv_pieces(Conv<T>& a, bool gradient) {
    const long long one = (long long)a.B * (a.C / Vec<T>::N), want = 148 * (gradient ? 384 : 640);
    int piece = 64;
    while (piece > (gradient ? 8 : 4) && one * ((a.L + piece - 1LL) / piece) < want) piece /= 2;
    // as long as one another, and at least K - 1 tokens where there is more than one: only the first reads the state in front
    a.pieces = (int)((a.L + (long long)piece - 1) / piece);
    a.piece = (int)((a.L + (long long)a.pieces - 1) / a.pieces);
    a.pieces = (int)((a.L + (long long)a.piece - 1) / a.piece);
}
template <typename T>
cudaError_t launch_conv(const Conv<T>& a, int K, int act, cudaStream_t stream) { return by_width(K, act, Forward<T>{a, stream}); }
template <typename T>
cudaError_t launch_conv_bwd(const Conv<T>& a, int K, int act, T* dw, T* dbias, cudaStream_t stream) {
    const cudaError_t e = by_width(K, act, Gradient<T>{a, stream});
    if (e != cudaSuccess || !a.part) return e;
    return launch_column_sums<T>({a.part, (long long)a.B * a.pieces, a.C * (K + 1), a.C * K, dw, dbias}, stream);
}
template <typename T>
cudaError_t launch_conv_step(const Conv<T>& a, int K, int act, T* state, cudaStream_t stream) { return by_width(K, act, Step<T>{a, state, stream}); }

#define VIG_INSTANCES(T)                                                                            \
    template void conv_pieces<T>(Conv<T>&, bool);                                                   \
    template cudaError_t launch_conv<T>(const Conv<T>&, int, int, cudaStream_t);                    \
    template cudaError_t launch_conv_bwd<T>(const Conv<T>&, int, int, T*, T*, cudaStream_t);        \
    template cudaError_t launch_conv_step<T>(const Conv<T>&, int, int, T*, cudaStream_t);
VIG_INSTANCES(__nv_bfloat16)
VIG_INSTANCES(float)

}  // namespace vig
