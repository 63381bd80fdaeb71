// The gated delta rule step by step in fp32 on the CUDA cores: fp32 calls; bf16 calls of a handful of tokens, gradients of more than 128 value columns, and
// units that the chunks leave (grown too far, or not finite); and the single token.
//
//   S~_t = alpha_t S_{t-1};  w_t = v_t - S~_t^T k_t;  u_t = beta_t w_t;  S_t = S~_t + k_t u_t^T;  out_t = S_t^T q_t
//
// The columns of S never meet: column j needs v_tj and the vectors k_t, q_t that all columns share.  A column is held in the registers
// of four lanes (eight for vectors of more than 64), the shared vectors come through shared memory, 16 or 32 tokens at a time.  A step's chain bounds
// it (two exchanges between lanes, two passes over the column): 48 units of 196 tokens, 32 x 64 fp32, 35 us, 340 cycles a token.
// The gradient is four such walks and nothing else:
//   columns forwards   w, and S at the end of every 64 tokens but the last ones
//   columns backwards  A = what arrives at S_t from behind;  D = A + q do^T;  du = D^T k;  dv = beta du;  A <- alpha (D - beta k du^T);
//                      and A at the end of every 64 tokens
//   rows forwards      dq = S do,  dk'' = - beta S~ du     (S from w: u = beta w)
//   rows backwards     dk' = D u                           (D from du)
// and what is left per token (finish):  dk = dk' + dk'';  dbeta = du . w;  and the gates' gradient.
#include <type_traits>

#include "gdr.h"
#include "gdr_tile.cuh"
#include "ptx.cuh"

namespace vig {
namespace {

template <int DP>
constexpr int tile_tokens() { return DP <= 64 ? 32 : 16; }   // staged at a time, a tile ahead of the walk
constexpr int kBorder = 64;   // tokens between the states that the gradient keeps

__device__ __forceinline__ float to_f(float x);
__device__ __forceinline__ float to_f(__nv_bfloat16 x);
__device__ __forceinline__ void cp_async4(float* dst, const float* src, bool in) {   // zero where !in
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(float* dst, const float* src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 16 : 0) : "memory");
}
// Rows of a tile to shared memory as fp32: n rows (of kTile) of `cols` values at src(row), part of rows of `ld` values from a multiple of eight on;
// zeros up to `width` and kTile.  fp32 by asynchronous copies, which the walk of the tile before hides; bf16 through registers, four values at a time.
template <typename T, int kTile, typename F>
__device__ __forceinline__ void stage_rows(float* dst, int n, int cols, int ld, int width, F src) {
    const int tid = threadIdx.x, nth = blockDim.x;
    if constexpr (sizeof(T) == 4) {
        const float* const any = (const float*)src(0);
        if (((cols | ld | width) & 3) == 0) {   // (rows then start on sixteen bytes: so do the tensors)
            const int w = width >> 2;
            for (int i = tid; i < kTile * w; i += nth) {
                const int t = i / w, e = (i - t * w) * 4;
                const bool in = t < n && e < cols;
                cp_async16(dst + t * width + e, in ? (const float*)src(t) + e : any, in);
            }
        } else
            for (int i = tid; i < kTile * width; i += nth) {
                const int t = i / width, e = i - t * width;
                const bool in = t < n && e < cols;
                cp_async4(dst + i, in ? (const float*)src(t) + e : any, in);
            }
    } else
        for (int i0 = tid; i0 < kTile * width; i0 += 4 * nth) {
            T x[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int i = i0 + h * nth, t = i / width, e = i - t * width;
                x[h] = i < kTile * width && t < n && e < cols ? src(t)[e] : T(0.f);
            }
#pragma unroll
            for (int h = 0; h < 4; ++h)
                if (i0 + h * nth < kTile * width) dst[i0 + h * nth] = to_f(x[h]);
        }
}
__device__ __forceinline__ void stage_one(float* dst, const float* src) { cp_async4(dst, src, true); }
__device__ __forceinline__ void stage_one(float* dst, const __nv_bfloat16* src) { *dst = to_f(*src); }
__device__ __forceinline__ void staged() { asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

struct Scratch {
    float *w, *du;               // [units][L][dv]
    float *dk1, *dk2, *dq;       // [units][L][dk]; dq: where the call's own is bf16
    float *S, *A;                // [units][borders][dk][dv]
};

__host__ __device__ inline int borders(int L) { return (L + kBorder - 1) / kBorder; }

// One lane's part of a vector of R G elements: quads (m G + l), m = 0 .. R / 4 - 1.
template <int R, int G>
struct Vec {
    f32x2 x[R / 2];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < R / 2; ++i) x[i] = pack2(0.f, 0.f);
    }
    __device__ __forceinline__ void load(const float* row, int l) {   // shared memory, 16-byte aligned
#pragma unroll
        for (int m = 0; m < R / 4; ++m) {
            const ulonglong2 p = *reinterpret_cast<const ulonglong2*>(row + (m * G + l) * 4);
            x[2 * m] = p.x;
            x[2 * m + 1] = p.y;
        }
    }
    __device__ __forceinline__ void scale(float s) {
        const f32x2 ss = pack2(s, s);
#pragma unroll
        for (int i = 0; i < R / 2; ++i) x[i] = fmul2(x[i], ss);
    }
    __device__ __forceinline__ void add(const Vec& v, float s) {
        const f32x2 ss = pack2(s, s);
#pragma unroll
        for (int i = 0; i < R / 2; ++i) x[i] = ffma2(v.x[i], ss, x[i]);
    }
    __device__ __forceinline__ float dot(const Vec& v) const {   // over the whole vector, in all its lanes
        f32x2 a = fmul2(x[0], v.x[0]), b = fmul2(x[1], v.x[1]);
#pragma unroll
        for (int i = 2; i < R / 2; i += 2) {
            a = ffma2(x[i], v.x[i], a);
            b = ffma2(x[i + 1], v.x[i + 1], b);
        }
        float s = sum2(fadd2(a, b));
#pragma unroll
        for (int o = 1; o < G; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        return s;
    }
    template <typename F>
    __device__ __forceinline__ void each(int l, F f) {   // f(element, value)
#pragma unroll
        for (int m = 0; m < R / 4; ++m) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float a, b;
                unpack2(x[2 * m + h], a, b);
                const int e = (m * G + l) * 4 + 2 * h;
                f(e, a);
                f(e + 1, b);
                x[2 * m + h] = pack2(a, b);
            }
        }
    }
};

// Shared memory of a walk, in floats: two buffers of N vectors of kTile tokens, a scalar per owner (column or row) and token, the two
// gates; one buffer of results.
template <int N, int DP>
__host__ __device__ constexpr int buffer_floats(int owners) { return tile_tokens<DP>() * (N * DP + 2 * owners + 2); }
template <int N, int DP>
constexpr size_t walk_smem(int owners) { return (size_t)(2 * buffer_floats<N, DP>(owners) + 2 * tile_tokens<DP>() * owners) * 4; }

// ---- columns: owners are columns of S, vectors of dk ------------------------------------------------------------------
// BACK: the walk of A.  KEEP (the gradient's walks): states at the borders.
template <typename T, int R, int G, bool BACK, bool KEEP>
__device__ void walk_columns(const Gdr<T>& a, const Scratch& s, float* sm, long long unit, int j0, int owners) {
    constexpr int DP = R * G, kTile = tile_tokens<DP>();
    const int tid = threadIdx.x, nth = blockDim.x, l = tid % G, col = tid / G, j = j0 + col;
    const int mine = min(owners, a.dv - j0);
    const bool valid = col < mine;
    const int bf = buffer_floats<2, DP>(owners);
    float* const res = sm + 2 * bf;
    const int tiles = (a.L + kTile - 1) / kTile, lg = 31 - __clz(owners);   // (owners: a power of two)
    const T* const scalar = BACK ? a.d_out : a.v;
    auto stage = [&](int tile, int b) {
        float *kk = sm + b * bf, *qq = kk + kTile * DP, *sc = qq + kTile * DP, *al = sc + 2 * kTile * owners, *be = al + kTile;
        const int t0 = tile * kTile, n = min(kTile, a.L - t0);
        stage_rows<T, kTile>(kk, n, a.dk, a.ldk, DP, [&](int t) { return a.k + a.row(unit, t0 + t) * a.ldk; });
        stage_rows<T, kTile>(qq, n, a.dk, a.ldk, DP, [&](int t) { return a.q + a.row(unit, t0 + t) * a.ldk; });
        stage_rows<T, kTile>(sc, n, mine, a.ldv, owners, [&](int t) { return scalar + a.row(unit, t0 + t) * a.ldv + j0; });
        if (tid < n) {
            const long long r = a.row(unit, t0 + tid);
            stage_one(al + tid, a.la + r);
            stage_one(be + tid, a.beta + r);
        }
    };
    Vec<R, G> x;
    x.zero();
    const float* first = BACK ? a.d_state_out : a.state_in;
    const long long plane = (long long)a.dk * a.dv;
    if (first && valid)
        x.each(l, [&](int e, float& y) {
            if (e < a.dk) y = first[unit * plane + (long long)e * a.dv + j];
        });
    auto keep = [&](float* to, int border) {
        if (valid)
            x.each(l, [&](int e, float& y) {
                if (e < a.dk) to[(unit * borders(a.L) + border) * plane + (long long)e * a.dv + j] = y;
            });
    };
    stage(BACK ? tiles - 1 : 0, 0);
    staged();
    __syncthreads();
    for (int n = 0; n < tiles; ++n) {
        const int tile = BACK ? tiles - 1 - n : n, t0 = tile * kTile, nt = min(kTile, a.L - t0), b = n & 1;
        if (n + 1 < tiles) stage(BACK ? tile - 1 : tile + 1, b ^ 1);
        const float *kk = sm + b * bf, *qq = kk + kTile * DP, *sc = qq + kTile * DP, *al = sc + 2 * kTile * owners, *be = al + kTile;
        if (KEEP && BACK && (t0 + nt) % kBorder == 0 && t0 + nt < a.L) keep(s.A, (t0 + nt - 1) / kBorder);   // (behind the last token: d_state_out)
        // (a token's vectors are read while the one before it is walked)
        Vec<R, G> k, q;
        const int at0 = BACK ? nt - 1 : 0;
        k.load(kk + at0 * DP, l);
        q.load(qq + at0 * DP, l);
        float alpha = expf(al[at0]), beta = be[at0], y = sc[at0 * owners + col];
#pragma unroll 2
        for (int i = 0; i < nt; ++i) {
            const int t = BACK ? nt - 1 - i : i, t1 = i + 1 < nt ? (BACK ? t - 1 : t + 1) : t;
            Vec<R, G> k1, q1;
            k1.load(kk + t1 * DP, l);
            q1.load(qq + t1 * DP, l);
            const float alpha1 = expf(al[t1]), beta1 = be[t1], y1 = sc[t1 * owners + col];
            if (BACK) {
                x.add(q, y);
                const float du = x.dot(k);
                x.add(k, -beta * du);
                x.scale(alpha);
                if (l == 0) res[t * owners + col] = du;
            } else {
                x.scale(alpha);
                const float w = y - x.dot(k);
                x.add(k, beta * w);
                if (KEEP) {
                    if (l == 0) res[t * owners + col] = w;
                } else {
                    const float o = x.dot(q);
                    if (l == 0) res[t * owners + col] = o;
                }
            }
            k = k1;
            q = q1;
            alpha = alpha1;
            beta = beta1;
            y = y1;
        }
        if (KEEP && !BACK && (t0 + nt) % kBorder == 0 && t0 + nt < a.L) keep(s.S, (t0 + nt - 1) / kBorder);
        staged();   // the next tile
        __syncthreads();
        for (int i = tid; i < nt * owners; i += nth) {
            const int t = i >> lg, c = i & (owners - 1);
            if (c >= mine) continue;
            const long long r = a.row(unit, t0 + t), at = r * a.dv + j0 + c;
            if (BACK) {
                s.du[at] = res[i];
                a.dv_out[r * a.ldv + j0 + c] = from_f<T>(be[t] * res[i]);
            } else if (KEEP) s.w[at] = res[i];
            else a.out[r * a.ldv + j0 + c] = from_f<T>(res[i]);
        }
        __syncthreads();
    }
    float* last = BACK ? a.d_state_in : a.state_out;
    if (last && valid)
        x.each(l, [&](int e, float& y) {
            if (e < a.dk) last[unit * plane + (long long)e * a.dv + j] = y;
        });
}

template <typename T, int R, int G>
__global__ void __launch_bounds__(256) gdr_columns_kernel(Gdr<T> a, int owners) {
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_launch_dependents();
    walk_columns<T, R, G, false, false>(a, Scratch{}, sm, blockIdx.x, blockIdx.y * owners, owners);
}
template <typename T, int R, int G>
__global__ void __launch_bounds__(256) gdr_columns_grad_kernel(Gdr<T> a, Scratch s, int owners) {
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.z == 0) walk_columns<T, R, G, false, true>(a, s, sm, blockIdx.x, blockIdx.y * owners, owners);
    else walk_columns<T, R, G, true, true>(a, s, sm, blockIdx.x, blockIdx.y * owners, owners);
}

// ---- rows: owners are rows of S, vectors of dv ---------------------------------------------------------------------------
template <typename T, int R, int G, bool BACK>
__device__ void walk_rows(const Gdr<T>& a, const Scratch& s, float* sm, long long unit, int i0, int owners) {
    constexpr int DP = R * G, kTile = tile_tokens<DP>();
    const int tid = threadIdx.x, nth = blockDim.x, l = tid % G, own = tid / G, row = i0 + own;
    const int mine = min(owners, a.dk - i0);
    const bool valid = own < mine;
    const int bf = buffer_floats<3, DP>(owners);
    float* const res = sm + 2 * bf;
    const int tiles = (a.L + kTile - 1) / kTile, lg = 31 - __clz(owners);   // (owners: a power of two)
    auto stage = [&](int tile, int b) {
        float *uu = sm + b * bf, *dd = uu + kTile * DP, *oo = dd + kTile * DP, *kk = oo + kTile * DP, *qq = kk + kTile * owners,
              *al = qq + kTile * owners, *be = al + kTile;
        const int t0 = tile * kTile, n = min(kTile, a.L - t0);
        stage_rows<float, kTile>(uu, n, a.dv, a.dv, DP, [&](int t) { return s.w + a.row(unit, t0 + t) * a.dv; });
        stage_rows<float, kTile>(dd, n, a.dv, a.dv, DP, [&](int t) { return s.du + a.row(unit, t0 + t) * a.dv; });
        stage_rows<T, kTile>(oo, n, a.dv, a.ldv, DP, [&](int t) { return a.d_out + a.row(unit, t0 + t) * a.ldv; });
        stage_rows<T, kTile>(kk, n, mine, a.ldk, owners, [&](int t) { return a.k + a.row(unit, t0 + t) * a.ldk + i0; });
        stage_rows<T, kTile>(qq, n, mine, a.ldk, owners, [&](int t) { return a.q + a.row(unit, t0 + t) * a.ldk + i0; });
        if (tid < n) {
            const long long r = a.row(unit, t0 + tid);
            stage_one(al + tid, a.la + r);
            stage_one(be + tid, a.beta + r);
        }
    };
    Vec<R, G> x;
    x.zero();
    const float* first = BACK ? a.d_state_out : a.state_in;
    if (first && valid)
        x.each(l, [&](int e, float& y) {
            if (e < a.dv) y = first[(unit * a.dk + row) * a.dv + e];
        });
    stage(BACK ? tiles - 1 : 0, 0);
    staged();
    __syncthreads();
    for (int n = 0; n < tiles; ++n) {
        const int tile = BACK ? tiles - 1 - n : n, t0 = tile * kTile, nt = min(kTile, a.L - t0), b = n & 1;
        if (n + 1 < tiles) stage(BACK ? tile - 1 : tile + 1, b ^ 1);
        const float *uu = sm + b * bf, *dd = uu + kTile * DP, *oo = dd + kTile * DP, *kk = oo + kTile * DP, *qq = kk + kTile * owners,
                    *al = qq + kTile * owners, *be = al + kTile;
        auto token = [&](int t, Vec<R, G>& w, Vec<R, G>& du, Vec<R, G>& dout, float& alpha, float& beta, float& k, float& q) {
            w.load(uu + t * DP, l);
            du.load(dd + t * DP, l);
            dout.load(oo + t * DP, l);
            alpha = expf(al[t]);
            beta = be[t];
            k = kk[t * owners + own];
            q = qq[t * owners + own];
        };
        constexpr bool AHEAD = R <= 16;   // read a token's vectors while the one before it is walked: registers permitting
        Vec<R, G> w, du, dout, w1, du1, dout1;
        float alpha, beta, k, q, alpha1, beta1, k1, q1;
        token(BACK ? nt - 1 : 0, w, du, dout, alpha, beta, k, q);
#pragma unroll 2
        for (int i = 0; i < nt; ++i) {
            const int t = BACK ? nt - 1 - i : i, t1 = i + 1 < nt ? (BACK ? t - 1 : t + 1) : t;
            if (AHEAD) token(t1, w1, du1, dout1, alpha1, beta1, k1, q1);
            if (BACK) {
                x.add(dout, q);
                const float g = beta * x.dot(w);
                x.add(du, -beta * k);
                x.scale(alpha);
                if (l == 0) res[t * owners + own] = g;
            } else {
                x.scale(alpha);
                const float g = -beta * x.dot(du);
                x.add(w, beta * k);
                const float dq = x.dot(dout);
                if (l == 0) {
                    res[t * owners + own] = g;
                    res[(kTile + t) * owners + own] = dq;
                }
            }
            if (AHEAD) {
                w = w1;
                du = du1;
                dout = dout1;
                alpha = alpha1;
                beta = beta1;
                k = k1;
                q = q1;
            } else token(t1, w, du, dout, alpha, beta, k, q);
        }
        staged();   // the next tile
        __syncthreads();
        for (int i = tid; i < nt * owners; i += nth) {
            const int t = i >> lg, c = i & (owners - 1);
            if (c >= mine) continue;
            const long long at = a.row(unit, t0 + t) * a.dk + i0 + c;
            if (BACK) s.dk1[at] = res[i];
            else {
                s.dk2[at] = res[i];
                s.dq[at] = res[kTile * owners + i];
            }
        }
        __syncthreads();
    }
}

template <typename T, int R, int G>
__global__ void __launch_bounds__(256) gdr_rows_grad_kernel(Gdr<T> a, Scratch s, int owners) {
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.z == 0) walk_rows<T, R, G, false>(a, s, sm, blockIdx.x, blockIdx.y * owners, owners);
    else walk_rows<T, R, G, true>(a, s, sm, blockIdx.x, blockIdx.y * owners, owners);
}

// ---- what is left per token: a block of 256 threads per 64 tokens of a unit ---------------------------------------------------
// A gate's gradient <dS~_t, S~_t> is the sum over everything that passes through the gate: with S in front of the 64 tokens, A behind them, b the running sum
// of the log gates in them and Gam_rs = e^{b_r - b_s},
//   dlog_alpha_t = e^{b_64} <S, A> + sum_{r >= t} F_r + sum_{s < t} G_s + sum_{s < t <= r} H_rs
//   F_r = e^{b_r} (q_r . S do_r - beta_r k_r . S du_r)     G_s = e^{b_64 - b_s} k_s . A u_s
//   H_rs = Gam_rs ((q_r . k_s) (do_r . u_s) - beta_r (k_r . k_s) (du_r . u_s))
// Every term has the gate's own factor in it and nothing is subtracted that it does not contain.  (Running sums of q . dq - v . dv, which is the same
// by algebra, are differences of terms without that factor: at log_alpha = -12 nothing but their rounding was left.)
// 64 tokens of 32 x 64 are 0.8 M multiplications, products of 64 x 64 a slice of 32 dimensions at a time, in 256 threads: 48 units
// of 196 tokens 37 us, the multiplications themselves.
constexpr int kSlice = 32, kPitch = kBorder + 4;
struct FinishShared {
    union {
        __align__(16) float stage[4][kSlice][kPitch];   // [dimension][token or column]
        float H[kBorder][kBorder + 1];                  // rows r, columns s
    };
    float bh[kBorder], bl[kBorder], beta[kBorder], F[kBorder], G[kBorder], part[8];
};

// to[dimension][token] of `kSlice` dimensions from e0 on: value(t, e), n tokens of `width` values.
template <typename F>
__device__ __forceinline__ void stage_slice(float (&to)[kSlice][kPitch], int n, int e0, int width, F value) {
    constexpr int kEach = kSlice * kBorder / 256;
    const int e = threadIdx.x % kSlice, t = threadIdx.x / kSlice;
    float x[kEach];
#pragma unroll
    for (int p = 0; p < kEach; ++p) x[p] = value(min(t + p * 8, n - 1), min(e0 + e, width - 1));   // (all of them at once, none behind a branch)
#pragma unroll
    for (int p = 0; p < kEach; ++p) to[e][t + p * 8] = t + p * 8 < n && e0 + e < width ? x[p] : 0.f;
}

// The same of a state [dk][dv] (null: zeros), 64 columns from j0 on.
__device__ __forceinline__ void stage_state(float (&to)[kSlice][kPitch], const float* S, int e0, int j0, int dk, int dv) {
    constexpr int kEach = kSlice * kBorder / 256;
    const int e = threadIdx.x / kBorder, j = threadIdx.x % kBorder;
    float x[kEach];
    if (S)
#pragma unroll
        for (int p = 0; p < kEach; ++p) x[p] = S[(long long)min(e0 + e + p * 4, dk - 1) * dv + min(j0 + j, dv - 1)];
#pragma unroll
    for (int p = 0; p < kEach; ++p) to[e + p * 4][j] = S && e0 + e + p * 4 < dk && j0 + j < dv ? x[p] : 0.f;
}

// RT: rows of a thread, sixteen of them in a column of the block; tokens in front of 16 RT.
template <typename T, int RT>
__device__ void gate_gradient(const Gdr<T>& a, const Scratch& s, FinishShared& m, long long unit, int t0, int nt, const float* S, const float* A) {
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, r0 = ty * RT, s0 = tx * 4;
    auto at = [&](int t) { return a.row(unit, t0 + t); };
    auto sum = [&](int t) { return gdr::Sum{m.bh[t], m.bl[t]}; };
    auto cols = [&](const float (&x)[kSlice][kPitch], int e, f32x2 (&y)[2]) {   // two values an instruction
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&x[e][s0]);
        y[0] = v.x;
        y[1] = v.y;
    };
    auto add = [&](f32x2 (&acc)[RT][2], const float (&x)[RT], const f32x2 (&y)[2]) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const f32x2 xx = pack2(x[r], x[r]);
            acc[r][0] = ffma2(xx, y[0], acc[r][0]);
            acc[r][1] = ffma2(xx, y[1], acc[r][1]);
        }
    };
    auto each = [&](const f32x2 (&acc)[RT][2], float (&y)[RT][4]) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            unpack2(acc[r][0], y[r][0], y[r][1]);
            unpack2(acc[r][1], y[r][2], y[r][3]);
        }
    };
    auto rows = [&](const float (&x)[kSlice][kPitch], int e, float (&y)[RT]) {
        if constexpr (RT == 4) {
            const float4 v = *reinterpret_cast<const float4*>(&x[e][r0]);
            y[0] = v.x; y[1] = v.y; y[2] = v.z; y[3] = v.w;
        } else y[0] = x[e][r0];
    };
    float f[RT] = {}, g[RT] = {};
    for (int j0 = 0; j0 < a.dv && (S || A); j0 += kBorder) {   // q S, k S and k A, 64 columns at a time
        f32x2 qs2[RT][2] = {}, ks2[RT][2] = {}, ka2[RT][2] = {};
        for (int e0 = 0; e0 < a.dk; e0 += kSlice) {
            __syncthreads();
            stage_slice(m.stage[0], nt, e0, a.dk, [&](int t, int e) { return to_f(a.k[at(t) * a.ldk + e]); });
            stage_slice(m.stage[1], nt, e0, a.dk, [&](int t, int e) { return to_f(a.q[at(t) * a.ldk + e]); });
            stage_state(m.stage[2], S, e0, j0, a.dk, a.dv);
            stage_state(m.stage[3], A, e0, j0, a.dk, a.dv);
            __syncthreads();
            if (r0 < nt)
#pragma unroll 2
                for (int i = 0; i < kSlice; ++i) {
                    float k[RT], q[RT];
                    f32x2 c[2], d[2];
                    rows(m.stage[0], i, k);
                    rows(m.stage[1], i, q);
                    cols(m.stage[2], i, c);
                    cols(m.stage[3], i, d);
                    add(qs2, q, c);
                    add(ks2, k, c);
                    add(ka2, k, d);
                }
        }
        float qs[RT][4], ks[RT][4], ka[RT][4];
        each(qs2, qs);
        each(ks2, ks);
        each(ka2, ka);
        if (r0 < nt)
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const long long r = at(min(r0 + i, nt - 1));
                const float beta = m.beta[r0 + i];
                float o[4], d[4], w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = min(j0 + s0 + j, a.dv - 1);
                    o[j] = to_f(a.d_out[r * a.ldv + c]);
                    d[j] = s.du[r * a.dv + c];
                    w[j] = s.w[r * a.dv + c];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = j0 + s0 + j < a.dv;
                    f[i] = in ? fmaf(qs[i][j], o[j], fmaf(-beta * ks[i][j], d[j], f[i])) : f[i];
                    g[i] = in ? fmaf(ka[i][j], beta * w[j], g[i]) : g[i];
                }
            }
    }
    const gdr::Sum end = sum(kBorder - 1);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            f[i] += __shfl_xor_sync(0xffffffffu, f[i], o);
            g[i] += __shfl_xor_sync(0xffffffffu, g[i], o);
        }
        if (tx == 0 && r0 + i < nt) {
            const gdr::Sum b = sum(r0 + i);
            m.F[r0 + i] = ex2(b.h + b.l) * f[i];
            m.G[r0 + i] = ex2(end.to(b)) * g[i];
        }
    }
    float meet = 0.f;
    if (S && A)
#pragma unroll 8
        for (int i = tid; i < a.dk * a.dv; i += 256) meet = fmaf(S[i], A[i], meet);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) meet += __shfl_xor_sync(0xffffffffu, meet, o);
    if ((tid & 31) == 0) m.part[tid >> 5] = meet;
    // H
    const bool mine = r0 < nt && s0 < r0 + RT;
    f32x2 qk2[RT][2] = {}, kk2[RT][2] = {}, x2[RT][2] = {}, e2[RT][2] = {};
    for (int e0 = 0; e0 < a.dk; e0 += kSlice) {
        __syncthreads();
        stage_slice(m.stage[0], nt, e0, a.dk, [&](int t, int e) { return to_f(a.k[at(t) * a.ldk + e]); });
        stage_slice(m.stage[1], nt, e0, a.dk, [&](int t, int e) { return to_f(a.q[at(t) * a.ldk + e]); });
        __syncthreads();
        if (mine)
#pragma unroll 2
            for (int i = 0; i < kSlice; ++i) {
                float k[RT], q[RT];
                f32x2 c[2];
                rows(m.stage[0], i, k);
                rows(m.stage[1], i, q);
                cols(m.stage[0], i, c);
                add(qk2, q, c);
                add(kk2, k, c);
            }
    }
    for (int e0 = 0; e0 < a.dv; e0 += kSlice) {
        __syncthreads();
        stage_slice(m.stage[0], nt, e0, a.dv, [&](int t, int e) { return to_f(a.d_out[at(t) * a.ldv + e]); });
        stage_slice(m.stage[1], nt, e0, a.dv, [&](int t, int e) { return s.du[at(t) * a.dv + e]; });
        stage_slice(m.stage[2], nt, e0, a.dv, [&](int t, int e) { return s.w[at(t) * a.dv + e]; });
        __syncthreads();
        if (mine)
#pragma unroll 2
            for (int i = 0; i < kSlice; ++i) {
                float g[RT], d[RT];
                f32x2 c[2];
                rows(m.stage[0], i, g);
                rows(m.stage[1], i, d);
                cols(m.stage[2], i, c);
                add(x2, g, c);
                add(e2, d, c);
            }
    }
    __syncthreads();
    float qk[RT][4], kk[RT][4], x[RT][4], e[RT][4];
    each(qk2, qk);
    each(kk2, kk);
    each(x2, x);
    each(e2, e);
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = r0 + i, c = s0 + j;
            // (a step of zero has no u, whatever its w)
            m.H[r][c] = c < r && r < nt && m.beta[c] != 0.f ? ex2(sum(r).to(sum(c))) * m.beta[c] * fmaf(x[i][j], qk[i][j], -m.beta[r] * e[i][j] * kk[i][j]) : 0.f;
            if (c == r && r < nt) a.dbeta[at(r)] = from_f<T>(e[i][j]);   // du . w
        }
    __syncthreads();
    if (tid < nt) {   // a row's sums up to each of its columns
        float run = 0.f;
        for (int c = 0; c <= tid; c += 8) {   // (zeros behind the diagonal)
            float h[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = m.H[tid][c + i];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m.H[tid][c + i] = run;
                run += h[i];
            }
        }
    }
    __syncthreads();
    if (tid < nt) {
        float through = 0.f, x = 0.f;
        for (int w = 0; w < 8; ++w) through += m.part[w];
#pragma unroll 8
        for (int c = 0; c < tid; ++c) x += m.G[c];
#pragma unroll 8
        for (int r = tid; r < nt; ++r) x += m.F[r] + m.H[r][tid];
        a.dla[at(tid)] = from_f<T>(fmaf(through, ex2(end.h + end.l), x));
    }
}

template <typename T>
__device__ void finish(const Gdr<T>& a, const Scratch& s, long long unit, int border) {
    __shared__ FinishShared m;
    const int t0 = border * kBorder, nt = min(kBorder, a.L - t0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long plane = (long long)a.dk * a.dv, at = unit * borders(a.L) + border;
    if (warp == 0) {
        float la[2], be[2];
        gdr::Sum b[2], all;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = 2 * lane + h;
            la[h] = t < nt ? to_f(a.la[a.row(unit, t0 + t)]) : 0.f;
            be[h] = t < nt ? to_f(a.beta[a.row(unit, t0 + t)]) : 0.f;
        }
        gdr::gate_sums(la, b, all);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            m.bh[2 * lane + h] = b[h].h;
            m.bl[2 * lane + h] = b[h].l;
            m.beta[2 * lane + h] = be[h];
        }
    }
    // dk = dk' + dk'', and dq where it is not the call's own yet: rows of the block in a row, four values a thread at a time
    const long long first = min(a.row(unit, t0), a.row(unit, t0 + nt - 1));
    for (int i0 = tid; i0 < nt * a.dk; i0 += 4 * 256) {
        float x[4], y[4], q[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const long long i = first * a.dk + min(i0 + p * 256, nt * a.dk - 1);
            x[p] = s.dk1[i];
            y[p] = s.dk2[i];
            if constexpr (sizeof(T) == 2) q[p] = s.dq[i];
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int i = i0 + p * 256, t = i / a.dk;
            if (i >= nt * a.dk) break;
            const long long to = (first + t) * a.ldk + i - t * a.dk;
            a.dk_out[to] = from_f<T>(x[p] + y[p]);
            if constexpr (sizeof(T) == 2) a.dq[to] = from_f<T>(q[p]);
        }
    }
    __syncthreads();
    const float* const front = border > 0 ? s.S + (at - 1) * plane : a.state_in ? a.state_in + unit * plane : nullptr;
    const float* const behind = t0 + nt < a.L ? s.A + at * plane : a.d_state_out ? a.d_state_out + unit * plane : nullptr;
    if (nt <= 16) gate_gradient<T, 1>(a, s, m, unit, t0, nt, front, behind);
    else gate_gradient<T, 4>(a, s, m, unit, t0, nt, front, behind);
}

template <typename T>
__global__ void __launch_bounds__(256, 2) gdr_finish_kernel(Gdr<T> a, Scratch s) {
    pdl_wait();
    pdl_launch_dependents();
    finish<T>(a, s, blockIdx.x / borders(a.L), blockIdx.x % borders(a.L));
}

// Behind the gradient in chunks: units that the loop left to the walks (grown too far, or not finite), whole, a block at a time.  Without any the block ends
// at once.
constexpr int kRepairR = 32, kRepairG = 4, kRepairOwners = 64;
__global__ void __launch_bounds__(256) gdr_repair_kernel(Gdr<__nv_bfloat16> a, Scratch s, const int* first, int per, const int* second, int chunks, int* status) {
    using T = __nv_bfloat16;
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_launch_dependents();
    auto flagged = [&](long long unit, int from, int step) {
        int any = 0;
        for (int i = from; i < per + chunks; i += step) any |= i < per ? first[unit * per + i] : second[unit * chunks + i - per];
        return any;
    };
    int any = 0;
    for (long long unit = blockIdx.x + (long long)(threadIdx.x >> 5) * gridDim.x; unit < a.units; unit += 8LL * gridDim.x) any |= flagged(unit, threadIdx.x & 31, 32);
    if (!__syncthreads_or(any)) return;
    for (long long unit = blockIdx.x; unit < a.units; unit += gridDim.x) {
        if (!__syncthreads_or(flagged(unit, threadIdx.x, 256))) continue;
        if (threadIdx.x == 0) atomicAdd(status + 1, 1);
        // this block's slot, as the walks address it
        const long long v = ((long long)blockIdx.x - unit) * a.L * a.dv, k = ((long long)blockIdx.x - unit) * a.L * a.dk,
                        p = ((long long)blockIdx.x - unit) * borders(a.L) * a.dk * a.dv;
        const Scratch mine = {s.w + v, s.du + v, s.dk1 + k, s.dk2 + k, s.dq + k, s.S + p, s.A + p};
        for (int j = 0; j < a.dv; j += kRepairOwners) {
            walk_columns<T, kRepairR, kRepairG, false, true>(a, mine, sm, unit, j, kRepairOwners);
            __syncthreads();
            walk_columns<T, kRepairR, kRepairG, true, true>(a, mine, sm, unit, j, kRepairOwners);
            __syncthreads();
        }
        for (int i = 0; i < a.dk; i += kRepairOwners) {
            walk_rows<T, kRepairR, kRepairG, false>(a, mine, sm, unit, i, kRepairOwners);
            __syncthreads();
            walk_rows<T, kRepairR, kRepairG, true>(a, mine, sm, unit, i, kRepairOwners);
            __syncthreads();
        }
        for (int b = 0; b < borders(a.L); ++b) {
            finish<T>(a, mine, unit, b);
            __syncthreads();
        }
    }
}

// The same behind the forward pass in segments.
__global__ void __launch_bounds__(256) gdr_repair_fwd_kernel(Gdr<__nv_bfloat16> a, const int* flags, int per, int* status) {
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_launch_dependents();
    for (long long unit = blockIdx.x; unit < a.units; unit += gridDim.x) {
        int any = 0;
        for (int i = threadIdx.x; i < per; i += 256) any |= flags[unit * per + i];
        if (!__syncthreads_or(any)) continue;
        if (threadIdx.x == 0) atomicAdd(status + 1, 1);
        for (int j = 0; j < a.dv; j += kRepairOwners) {
            walk_columns<__nv_bfloat16, kRepairR, kRepairG, false, false>(a, Scratch{}, sm, unit, j, kRepairOwners);
            __syncthreads();
        }
    }
}

// f(R, G) for vectors of d elements: four lanes, eight beyond 64 elements (48 units of 196 tokens, 128 x 128 fp32, a training step 560 -> 497 us; of 32 x 64
// it would be 150 -> 162: a step's chain is what counts there, and it has one more exchange).
template <typename F>
cudaError_t with_vector(int d, F f) {
    if (d <= 16) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
    if (d <= 32) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
    if (d <= 48) return f(std::integral_constant<int, 12>(), std::integral_constant<int, 4>());
    if (d <= 64) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
    if (d <= 96) return f(std::integral_constant<int, 12>(), std::integral_constant<int, 8>());
    if (d <= 128) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
}

// Owners a block holds: whole warps, a power of two, at most 256 threads; fewer where that gives every SM a block (48 units of 196 tokens, 32 x 64
// fp32: one block a unit 47 us).
int owners_of(int n, int G, long long walks) {
    const int most = 256 / G;
    int owners = 32 / G;
    while (owners < most && owners < n && walks * ((n + 2 * owners - 1) / (2 * owners)) >= 148) owners *= 2;
    return owners;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
Scratch cut_scratch(char* base, const Gdr<T>* a, long long units, int L, int dk, int dv, size_t* total) {
    Scratch s = {};
    size_t at = 0;
    auto take = [&](size_t floats) {
        float* p = base ? reinterpret_cast<float*>(base + at) : nullptr;
        at += up(floats * 4);
        return p;
    };
    const size_t rows = (size_t)units * L, states = (size_t)units * borders(L) * dk * dv;
    s.w = take(rows * dv);
    s.du = take(rows * dv);
    s.dk1 = take(rows * dk);
    s.dk2 = take(rows * dk);
    if constexpr (sizeof(T) == 2) s.dq = take(rows * dk);
    else if (a) s.dq = (float*)a->dq;
    s.S = take(states);
    s.A = take(states);
    *total = at;
    return s;
}

}  // namespace

bool gdr_supported(int dk, int dv) { return dk <= 128 && dv <= 256; }

template <typename T>
cudaError_t launch_gdr_walk_fwd(const Gdr<T>& a, cudaStream_t stream) {
    return with_vector(a.dk, [&](auto R, auto G) {
        constexpr int r = decltype(R)::value, g = decltype(G)::value;
        const int owners = owners_of(a.dv, g, a.units);
        const size_t smem = walk_smem<2, r * g>(owners);
        cudaError_t e = allow_smem<gdr_columns_kernel<T, r, g>>(walk_smem<2, r * g>(256 / g));
        if (e != cudaSuccess) return e;
        count_launch();
        return launch_pdl(gdr_columns_kernel<T, r, g>, dim3((unsigned)a.units, (a.dv + owners - 1) / owners), dim3(owners * g), smem, stream, a, owners);
    });
}

template <typename T>
size_t gdr_walk_bwd_scratch_bytes(long long units, int L, int dk, int dv) {
    size_t total;
    cut_scratch<T>(nullptr, nullptr, units, L, dk, dv, &total);
    return total;
}

template <typename T>
cudaError_t launch_gdr_walk_bwd(const Gdr<T>& a, void* scratch, cudaStream_t stream) {
    size_t total;
    const Scratch s = cut_scratch<T>((char*)scratch, &a, a.units, a.L, a.dk, a.dv, &total);
    cudaError_t e = with_vector(a.dk, [&](auto R, auto G) {
        constexpr int r = decltype(R)::value, g = decltype(G)::value;
        const int owners = owners_of(a.dv, g, 2 * a.units);
        const size_t smem = walk_smem<2, r * g>(owners);
        cudaError_t e = allow_smem<gdr_columns_grad_kernel<T, r, g>>(walk_smem<2, r * g>(256 / g));
        if (e != cudaSuccess) return e;
        return launch_pdl(gdr_columns_grad_kernel<T, r, g>, dim3((unsigned)a.units, (a.dv + owners - 1) / owners, 2), dim3(owners * g), smem, stream, a, s, owners);
    });
    if (e != cudaSuccess) return e;
    e = with_vector(a.dv, [&](auto R, auto G) {
        constexpr int r = decltype(R)::value, g = decltype(G)::value;
        const int owners = owners_of(a.dk, g, 2 * a.units);
        const size_t smem = walk_smem<3, r * g>(owners);
        cudaError_t e = allow_smem<gdr_rows_grad_kernel<T, r, g>>(walk_smem<3, r * g>(256 / g));
        if (e != cudaSuccess) return e;
        return launch_pdl(gdr_rows_grad_kernel<T, r, g>, dim3((unsigned)a.units, (a.dk + owners - 1) / owners, 2), dim3(owners * g), smem, stream, a, s, owners);
    });
    if (e != cudaSuccess) return e;
    count_launch(3);
    return launch_pdl(gdr_finish_kernel<T>, dim3((unsigned)(a.units * borders(a.L))), dim3(256), 0, stream, a, s);
}

size_t gdr_repair_slot_bytes(int L, int dk, int dv) { return gdr_walk_bwd_scratch_bytes<__nv_bfloat16>(1, L, dk, dv); }
cudaError_t launch_gdr_repair(const Gdr<__nv_bfloat16>& a, const int* first, int per, const int* second, int chunks, void* scratch, int slots, cudaStream_t stream) {
    int* status = device_status_ptr();
    if (!status) return cudaErrorUnknown;
    size_t total;
    const Scratch s = cut_scratch<__nv_bfloat16>((char*)scratch, &a, slots, a.L, a.dk, a.dv, &total);
    constexpr int DP = kRepairR * kRepairG;
    const size_t smem = walk_smem<3, DP>(kRepairOwners);
    cudaError_t e = allow_smem<gdr_repair_kernel>(smem);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(gdr_repair_kernel, dim3(slots), dim3(kRepairG * kRepairOwners), smem, stream, a, s, first, per, second, chunks, status);
}

cudaError_t launch_gdr_repair_fwd(const Gdr<__nv_bfloat16>& a, const int* flags, int per, cudaStream_t stream) {
    int* status = device_status_ptr();
    if (!status) return cudaErrorUnknown;
    const size_t smem = walk_smem<2, kRepairR * kRepairG>(kRepairOwners);
    cudaError_t e = allow_smem<gdr_repair_fwd_kernel>(smem);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(gdr_repair_fwd_kernel, dim3((unsigned)(a.units < 148 ? a.units : 148)), dim3(kRepairG * kRepairOwners), smem, stream, a, flags, per, status);
}

template cudaError_t launch_gdr_walk_fwd<float>(const Gdr<float>&, cudaStream_t);
template cudaError_t launch_gdr_walk_fwd<__nv_bfloat16>(const Gdr<__nv_bfloat16>&, cudaStream_t);
template size_t gdr_walk_bwd_scratch_bytes<float>(long long, int, int, int);
template size_t gdr_walk_bwd_scratch_bytes<__nv_bfloat16>(long long, int, int, int);
template cudaError_t launch_gdr_walk_bwd<float>(const Gdr<float>&, void*, cudaStream_t);
template cudaError_t launch_gdr_walk_bwd<__nv_bfloat16>(const Gdr<__nv_bfloat16>&, void*, cudaStream_t);

// ---- one token -------------------------------------------------------------------------------------------------------
// A block takes 32 columns of a unit's state: sixteen groups of rows, a thread four columns (or one) of every sixteenth row, all of
// them in registers at once.  Retrieval and read-out are summed in one pass over the state as it was:
//   S^T k and S^T q;   w = v - alpha S^T k;   out = alpha S^T q + (q . k) u;   S <- alpha S + k u^T
// Bound by the state's way in and out: 4096 states of 128 x 128, 541 MB, 92 us, 0.90 of the rate of a copy.  (Blocks of 32 columns: a row's piece is
// one line of 128 bytes, and sixteen blocks fit an SM.)
namespace {

template <typename T, int V>
__global__ void __launch_bounds__(16 * (32 / V)) gdr_step_kernel(const T* q, const T* k, const T* v, const T* la, const T* beta, float* state, T* out,
                                                                int dk, int dv) {
    constexpr int kCols = 32 / V, kRows = 8;   // threads along the columns; rows of a thread (dk <= 128)
    constexpr int kWarps = 16 * kCols / 32;
    __shared__ float sk[128], sq[128], red[2][kWarps][32];
    pdl_wait();
    pdl_launch_dependents();
    const long long unit = blockIdx.x;
    const int tid = threadIdx.x, c = tid % kCols, g = tid / kCols, j = blockIdx.y * 32 + c * V;
    const bool in = j < dv;   // (V = 4: dv is a multiple of four)
    float* const S = state + unit * dk * dv + j;
    float x[kRows][V];
#pragma unroll
    for (int m = 0; m < kRows; ++m) {
        const int i = m * 16 + g;
#pragma unroll
        for (int e = 0; e < V; ++e) x[m][e] = 0.f;
        if (in && i < dk) {
            if constexpr (V == 4) {
                const float4 y = *reinterpret_cast<const float4*>(S + (long long)i * dv);
                x[m][0] = y.x; x[m][1] = y.y; x[m][2] = y.z; x[m][3] = y.w;
            } else x[m][0] = S[(long long)i * dv];
        }
    }
    for (int i = tid; i < 128; i += 16 * kCols) {
        sk[i] = i < dk ? to_f(k[unit * dk + i]) : 0.f;
        sq[i] = i < dk ? to_f(q[unit * dk + i]) : 0.f;
    }
    const float alpha = expf(to_f(la[unit])), b = to_f(beta[unit]);
    __syncthreads();
    float r[V] = {}, o[V] = {}, qk = 0.f;
#pragma unroll
    for (int m = 0; m < kRows; ++m) {
        const float ki = sk[m * 16 + g], qi = sq[m * 16 + g];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            r[e] = fmaf(ki, x[m][e], r[e]);
            o[e] = fmaf(qi, x[m][e], o[e]);
        }
    }
    for (int i = tid & 31; i < 128; i += 32) qk = fmaf(sk[i], sq[i], qk);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) qk += __shfl_xor_sync(0xffffffffu, qk, s);
#pragma unroll
    for (int s = kCols; s < 32; s <<= 1)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            r[e] += __shfl_xor_sync(0xffffffffu, r[e], s);
            o[e] += __shfl_xor_sync(0xffffffffu, o[e], s);
        }
    if ((tid & 31) < kCols)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            red[0][tid >> 5][c * V + e] = r[e];
            red[1][tid >> 5][c * V + e] = o[e];
        }
    __syncthreads();
    if (!in) return;
    float u[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float rr = 0.f, oo = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            rr += red[0][w][c * V + e];
            oo += red[1][w][c * V + e];
        }
        u[e] = b * (to_f(v[unit * dv + j + e]) - alpha * rr);
        if (g == 0) out[unit * dv + j + e] = from_f<T>(fmaf(qk, u[e], alpha * oo));
    }
#pragma unroll
    for (int m = 0; m < kRows; ++m) {
        const int i = m * 16 + g;
        if (i >= dk) break;
        const float ki = sk[i];
#pragma unroll
        for (int e = 0; e < V; ++e) x[m][e] = fmaf(ki, u[e], alpha * x[m][e]);
        if constexpr (V == 4) *reinterpret_cast<float4*>(S + (long long)i * dv) = make_float4(x[m][0], x[m][1], x[m][2], x[m][3]);
        else S[(long long)i * dv] = x[m][0];
    }
}

}  // namespace

template <typename T>
cudaError_t launch_gdr_step(const T* q, const T* k, const T* v, const T* la, const T* beta, float* state, T* out, long long units, int dk, int dv,
                            cudaStream_t stream) {
    const dim3 grid((unsigned)units, (dv + 31) / 32);
    count_launch();
    if (dv % 4 == 0) return launch_pdl(gdr_step_kernel<T, 4>, grid, dim3(128), 0, stream, q, k, v, la, beta, state, out, dk, dv);
    return launch_pdl(gdr_step_kernel<T, 1>, grid, dim3(512), 0, stream, q, k, v, la, beta, state, out, dk, dv);
}
template cudaError_t launch_gdr_step<float>(const float*, const float*, const float*, const float*, const float*, float*, float*, long long, int, int,
                                            cudaStream_t);
template cudaError_t launch_gdr_step<__nv_bfloat16>(const __nv_bfloat16*, const __nv_bfloat16*, const __nv_bfloat16*, const __nv_bfloat16*,
                                                    const __nv_bfloat16*, float*, __nv_bfloat16*, long long, int, int, cudaStream_t);

}  // namespace vig
