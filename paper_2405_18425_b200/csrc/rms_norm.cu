// RMS norm over rows of C values with the residual's addition, and its gradient.
//
//   s = x + residual;  r = 1 / sqrt(mean(s^2) + eps);  out = s r weight, or e4m3(out / scale) with scale = max |out| / 448
//   gradient:  g = d_out weight;  xhat = s r;  dx = r (g - xhat mean(g xhat)) + d_sum;  dweight = sum over the rows of d_out xhat
//
// Memory bounds all of it: a row stays in the registers of its threads (a warp up to 128 vectors of 16 bytes, four vectors a thread at
// most) between its sum and its use, so every value crosses memory once in and once out.  The sum of squares and the mean of the
// gradient are fp32; the norm is of the sum before it is rounded to the call's type, and the gradient of the sum as it was stored.
// 12544 x 768 bf16 with residual, 8 bits: 14.5 us (0.72 of a copy's rate); 32768 x 192 fp32: 16 us, its gradient 18.
#include "gdr.h"
#include "layers.h"
#include "wide.cuh"

namespace vig {
namespace {

// Threads of a block: several rows of a warp each, or one row (so that what depends on a row's values is the same for a whole block
// wherever the threads meet in it).
constexpr int threads_of_block(int tpr) { return tpr == 32 ? 256 : tpr; }

__device__ __forceinline__ float max_or_nan(float a, float b) {   // (fmaxf would drop a NaN: a block that holds one has it as its scale)
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Sum (or maximum) over the TPR threads of a row, in a fixed order; `red`: 32 floats of shared memory a row of more than one warp.
template <int TPR, bool MAX>
__device__ __forceinline__ float over_row(float v, float* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_or_nan(v, u) : v + u;
    }
    if constexpr (TPR > 32) {
        const int warp = threadIdx.x >> 5;
        __syncthreads();   // (red may still be read for the sum before)
        if ((threadIdx.x & 31) == 0) red[warp] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int i = 1; i < TPR / 32; ++i) v = MAX ? max_or_nan(v, red[i]) : v + red[i];
    }
    return v;
}

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}

// OUT: 0 the call's type, 1 e4m3 with a scale a row, 2 e4m3 with a scale for every 128 values (sixteen or thirty-two neighbouring
// vectors of a row: lanes of one warp).
template <typename T, int V, int TPR, int OUT>
__global__ void __launch_bounds__(threads_of_block(TPR)) rms_norm_kernel(RmsNorm<T> a) {
    constexpr int N = Vec<T>::N, kPer = threads_of_block(TPR) / TPR;
    __shared__ float red[32];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const long long row = (long long)blockIdx.x * kPer + group;
    const bool live = row < a.rows;
    const int nv = a.C / N;
    const long long at = row * a.C;
    uint4 in[V], res[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int v = lane + i * TPR;
        in[i] = res[i] = make_uint4(0, 0, 0, 0);
        if (live && v < nv) {
            in[i] = load16(a.x + at + v * N);
            if (a.residual) res[i] = load16(a.residual + at + v * N);
        }
    }
    float s[V][N], sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int v = lane + i * TPR;
        widen(in[i], s[i], (const T*)nullptr);
        if (a.residual) {
            float r[N];
            widen(res[i], r, (const T*)nullptr);
#pragma unroll
            for (int j = 0; j < N; ++j) s[i][j] += r[j];
        }
        if (a.sum_out && live && v < nv) store16(a.sum_out + at + v * N, narrow(s[i], (const T*)nullptr));
#pragma unroll
        for (int j = 0; j < N; ++j) sum = fmaf(s[i][j], s[i][j], sum);
    }
    sum = over_row<TPR, false>(sum, red);
    float r = __frsqrt_rn(sum * a.inv_C + a.eps), rstd = r;
    // Squares that overflow, or that underflow with no eps beside them: of the row over its largest value or the root of eps, whichever is
    // larger, so that neither the squares nor eps over its square leave the range.  (From an eps of 2^-60 on, squares that underflow
    // are nothing beside it.)
    if (!(sum < 0x1p+120f) || (sum < 0x1p-80f && a.eps < 0x1p-60f)) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(s[i][j]));
        top = over_row<TPR, true>(top, red);
        if (top > 0.f && top < INFINITY && sum == sum) {
            const float unit = fmaxf(top, sqrtf(a.eps));
            const float down = unit > 1.f ? 0x1p-64f : 0x1p+64f;   // (either way twice, so that neither factor leaves the range)
            const float part = 1.f / (unit * down);
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float u = s[i][j] * down * part;
                    sum = fmaf(u, u, sum);
                }
            sum = over_row<TPR, false>(sum, red);
            const float e = a.eps * down * part;   // eps / unit^2 in two steps
            r = __frsqrt_rn(sum * a.inv_C + e * down * part) * part;
            rstd = r * down;
            if (unit > 1.f) {
                r = rstd;
            } else {   // 1 / unit may leave the range, the result not: the row takes the other factor
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) s[i][j] *= down;
            }
        }
    }
    if (a.rstd && live && lane == 0) a.rstd[row] = rstd;
    // In 8 bits rstd's own digits fall out of out / scale: the row is multiplied by its power of two, which is exact, and the rest of it goes to
    // the scale alone, so that a code comes of s w, the largest |s w| and two roundings.
    float by = r, rest = 1.f;
    if (OUT != 0) {
        uint32_t bits = __float_as_uint(r) & 0x7f800000u;   // (infinity of a NaN, which the rest then is)
        if (bits == 0 && r > 0.f) bits = 0x00800000u;
        by = __uint_as_float(bits);
        rest = r * __uint_as_float(0x7f000000u - bits);     // r / by
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int v = lane + i * TPR;
        float w[N];
        widen(v < nv ? load16(a.weight + v * N) : make_uint4(0, 0, 0, 0), w, (const T*)nullptr);
#pragma unroll
        for (int j = 0; j < N; ++j) s[i][j] = s[i][j] * by * w[j];
        if constexpr (OUT == 0) {
            if (live && v < nv) store16(a.out + at + v * N, narrow(s[i], (const T*)nullptr));
        }
    }
    if constexpr (OUT != 0) {
        constexpr int kLanes = 128 / N;   // of a block of 128 values
        const int blocks = OUT == 2 ? (a.C + 127) / 128 : 1;
        float each[V], most = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) m = max_or_nan(m, fabsf(s[i][j]));
            if (lane + i * TPR >= nv) m = 0.f;   // (behind the row: zero times a scale that may be infinite)
            if constexpr (OUT == 2) {
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) m = max_or_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
            }
            each[i] = m;
            most = max_or_nan(most, m);
        }
        if constexpr (OUT == 1) most = over_row<TPR, true>(most, red);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int v = lane + i * TPR;
            // the smallest normal number at least, so that a block of zeros divides by it too
            constexpr float kLeast = 1.17549435e-38f;
            const float m = OUT == 1 ? most : each[i], scale = max_or_nan(__fdiv_rn(m, 448.f) * rest, kLeast);
            const float over = scale == kLeast ? rest * 0x1p126f : __fdiv_rn(448.f, m);   // (of a NaN a NaN)
            if (!live || v >= nv) continue;
            // bf16 calls: and what is left of 448 s w behind q m, exactly, so that middles between two codes, which their few digits meet, stay
            // middles (12544 x 768: 14.5 us instead of 13.8; without it one code in 800 000 was the other of two neighbours)
            float q[N];
            const bool exactly = sizeof(T) == 2 && scale != kLeast && over > 0.f && m < 0x1p+100f;
            const f32x2 quick = pack2(over, over), small = pack2(over * (1.f / 448.f), over * (1.f / 448.f)), most2 = pack2(m, m), less2 = pack2(-m, -m);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const f32x2 t = pack2(s[i][j], s[i][j + 1]);
                f32x2 y = fmul2(t, quick);
                if (exactly) {
                    const f32x2 p = fmul2(y, less2), rounded = ffma2(y, most2, p);
                    y = ffma2(ffma2(rounded, pack2(-1.f, -1.f), ffma2(t, pack2(448.f, 448.f), p)), small, y);
                }
                unpack2(y, q[j], q[j + 1]);
            }
            unsigned char* p = a.q + at + v * N;
            if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(e4m3x4(q[0], q[1], q[2], q[3]), e4m3x4(q[4], q[5], q[6], q[7]));
            else *reinterpret_cast<uint32_t*>(p) = e4m3x4(q[0], q[1], q[2], q[3]);
            if (OUT == 2 && v % kLanes == 0) a.scales[row * blocks + v / kLanes] = scale;
            if (OUT == 1 && v == 0) a.scales[row] = scale;
        }
    }
}

// A group of threads takes every so many-th row and keeps its channels' part of the weight's gradient in registers; a block adds its
// groups' in order and leaves one row of partial sums.
template <typename T, int V, int TPR>
__global__ void __launch_bounds__(threads_of_block(TPR)) rms_norm_bwd_kernel(RmsNormGrad<T> a) {
    constexpr int N = Vec<T>::N, kPer = threads_of_block(TPR) / TPR;
    extern __shared__ float sums[];   // [C], where the weight's gradient is wanted
    __shared__ float red[32];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR, nv = a.C / N;
    float w[V][N], dw[V][N];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int v = lane + i * TPR;
        widen(v < nv ? load16(a.weight + v * N) : make_uint4(0, 0, 0, 0), w[i], (const T*)nullptr);
#pragma unroll
        for (int j = 0; j < N; ++j) dw[i][j] = 0.f;
    }
    const long long step = (long long)gridDim.x * kPer;
    for (long long first = (long long)blockIdx.x * kPer; first < a.rows; first += step) {
        const long long row = first + group, at = row * a.C;
        const bool live = row < a.rows;
        uint4 in[V], go[V], on[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int v = lane + i * TPR;
            in[i] = go[i] = on[i] = make_uint4(0, 0, 0, 0);
            if (live && v < nv) {
                in[i] = load16(a.sum + at + v * N);
                go[i] = load16(a.d_out + at + v * N);
                if (a.d_sum) on[i] = load16(a.d_sum + at + v * N);
            }
        }
        const float r = live ? a.rstd[row] : 0.f;
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float s[N], g[N];
            widen(in[i], s, (const T*)nullptr);
            widen(go[i], g, (const T*)nullptr);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float xhat = s[j] * r;
                dot = fmaf(g[j] * w[i][j], xhat, dot);
                if (live && lane + i * TPR < nv) dw[i][j] = fmaf(g[j], xhat, dw[i][j]);
            }
        }
        dot = over_row<TPR, false>(dot, red) * a.inv_C;
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int v = lane + i * TPR;
            if (v >= nv) continue;
            float s[N], g[N], d[N];
            widen(in[i], s, (const T*)nullptr);
            widen(go[i], g, (const T*)nullptr);
            widen(on[i], d, (const T*)nullptr);
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = fmaf(r, fmaf(-s[j] * r, dot, g[j] * w[i][j]), d[j]);
            store16(a.dx + at + v * N, narrow(d, (const T*)nullptr));
        }
    }
    if (!a.part) return;
    for (int turn = 0; turn < kPer; ++turn) {
        if (turn == group) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int v = lane + i * TPR;
                if (v >= nv) continue;
#pragma unroll
                for (int j = 0; j < N; ++j) sums[v * N + j] = turn == 0 ? dw[i][j] : sums[v * N + j] + dw[i][j];
            }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) a.part[(long long)blockIdx.x * a.C + c] = sums[c];
}

constexpr int kRuns = 32;   // a block is a warp a run
template <typename T>
__global__ void __launch_bounds__(32 * kRuns) column_sums_kernel(ColumnSums<T> a) {
    __shared__ float part[kRuns][33];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    // runs of neighbouring rows, each in order, then the runs in order
    const long long per = (a.rows + kRuns - 1) / kRuns, lo = run * per < a.rows ? run * per : a.rows, hi = lo + per < a.rows ? lo + per : a.rows;
    float s = 0.f;
    if (c < a.columns) {
        long long r = lo;
        for (; r + 8 <= hi; r += 8) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = a.part[(r + i) * a.columns + c];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[i];
        }
        for (; r < hi; ++r) s += a.part[r * a.columns + c];
    }
    part[run][lane] = s;
    __syncthreads();
    if (run != 0 || c >= a.columns) return;
    for (int i = 1; i < kRuns; ++i) s += part[i][lane];
    if (c < a.first) {
        if (a.a) from_f32(a.a + c, s);
    } else if (a.b) {
        from_f32(a.b + (c - a.first), s);
    }
}

// What a row of nv vectors takes: a warp up to 128 of them, then as many threads as hold four each.
int threads_of_row(int nv) { return nv <= 128 ? 32 : nv <= 512 ? 128 : nv <= 1024 ? 256 : nv <= 2048 ? 512 : 1024; }
template <typename T>
constexpr int kMostThreads = kRmsMostC / Vec<T>::N / 4;   // 512 for bf16

template <typename T, int V, int TPR>
cudaError_t norm_of(const RmsNorm<T>& a, int out, cudaStream_t stream) {
    constexpr int threads = threads_of_block(TPR);
    const dim3 grid((unsigned)((a.rows + threads / TPR - 1) / (threads / TPR)));
    count_launch();
    if (out == 0) return launch_pdl(rms_norm_kernel<T, V, TPR, 0>, grid, dim3(threads), 0, stream, a);
    if (out == 1) return launch_pdl(rms_norm_kernel<T, V, TPR, 1>, grid, dim3(threads), 0, stream, a);
    return launch_pdl(rms_norm_kernel<T, V, TPR, 2>, grid, dim3(threads), 0, stream, a);
}
template <typename T, int V, int TPR>
cudaError_t grad_of(const RmsNormGrad<T>& a, int blocks, cudaStream_t stream) {
    constexpr int threads = threads_of_block(TPR);
    const size_t smem = a.part ? a.C * sizeof(float) : 0;
    const cudaError_t e = allow_smem<rms_norm_bwd_kernel<T, V, TPR>>(kRmsMostC * sizeof(float));
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(rms_norm_bwd_kernel<T, V, TPR>, dim3(blocks), dim3(threads), smem, stream, a);
}

#define VIG_BY_VECTORS(CALL)                                                    \
    switch (tpr) {                                                              \
        case 32:                                                                \
            switch ((nv + 31) / 32) {                                           \
                case 1: CALL(1, 32);                                            \
                case 2: CALL(2, 32);                                            \
                case 3: CALL(3, 32);                                            \
                default: CALL(4, 32);                                           \
            }                                                                   \
        case 128:                                                               \
            switch ((nv + 127) / 128) {                                         \
                case 2: CALL(2, 128);                                           \
                case 3: CALL(3, 128);                                           \
                default: CALL(4, 128);                                          \
            }                                                                   \
        case 256: CALL(4, 256);                                                 \
        case 512: CALL(4, 512);                                                 \
        default: CALL(4, kMostThreads<T>);                                      \
    }

}  // namespace

template <typename T>
cudaError_t launch_rms_norm(const RmsNorm<T>& a, int out, cudaStream_t stream) {
    const int nv = a.C / Vec<T>::N, tpr = threads_of_row(nv);
#define VIG_CALL(V, TPR) return norm_of<T, V, TPR>(a, out, stream)
    VIG_BY_VECTORS(VIG_CALL)
#undef VIG_CALL
}

// Blocks of the gradient: enough to fill the GPU, so that partial sums are few (C floats a block).
template <typename T>
int rms_norm_bwd_blocks(long long rows, int C) {
    const int tpr = threads_of_row(C / Vec<T>::N), per = threads_of_block(tpr) / tpr;
    const long long need = (rows + per - 1) / per, most = 148LL * (tpr > 512 ? 1 : tpr > 256 ? 2 : 4);
    return (int)(need < most ? need : most);
}

template <typename T>
cudaError_t launch_rms_norm_bwd(const RmsNormGrad<T>& a, T* dweight, cudaStream_t stream) {
    const int nv = a.C / Vec<T>::N, tpr = threads_of_row(nv), blocks = rms_norm_bwd_blocks<T>(a.rows, a.C);
    const cudaError_t e = [&] {
#define VIG_CALL(V, TPR) return grad_of<T, V, TPR>(a, blocks, stream)
        VIG_BY_VECTORS(VIG_CALL)
#undef VIG_CALL
    }();
    if (e != cudaSuccess || !a.part) return e;
    return launch_column_sums<T>({a.part, blocks, a.C, a.C, dweight, nullptr}, stream);
}

template <typename T>
cudaError_t launch_column_sums(const ColumnSums<T>& a, cudaStream_t stream) {
    count_launch();
    return launch_pdl(column_sums_kernel<T>, dim3((a.columns + 31) / 32), dim3(32 * kRuns), 0, stream, a);
}

#define VIG_INSTANCES(T)                                                                        \
    template cudaError_t launch_rms_norm<T>(const RmsNorm<T>&, int, cudaStream_t);              \
    template int rms_norm_bwd_blocks<T>(long long, int);                                        \
    template cudaError_t launch_rms_norm_bwd<T>(const RmsNormGrad<T>&, T*, cudaStream_t);       \
    template cudaError_t launch_column_sums<T>(const ColumnSums<T>&, cudaStream_t);
VIG_INSTANCES(__nv_bfloat16)
VIG_INSTANCES(float)

}  // namespace vig
