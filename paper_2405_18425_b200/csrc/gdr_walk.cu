// The gated delta rule step by step in fp32 on the CUDA cores: fp32 calls, and the head sizes that the tensor-core kernels do not take.
//
//   S~_t = alpha_t S_{t-1};  w_t = v_t - S~_t^T k_t;  u_t = beta_t w_t;  S_t = S~_t + k_t u_t^T;  out_t = S_t^T q_t
//
// The columns of S never meet: column j needs v_tj and the vectors k_t, q_t that all columns share.  A column is held in the registers
// of four lanes (eight for vectors of more than 64), the shared vectors come through shared memory, 16 or 32 tokens at a time.  A step's chain bounds
// it (two exchanges between lanes, two passes over the column): 48 units of 196 tokens, 32 x 64 fp32, 35 us, 340 cycles a token.
// The gradient is four such walks and nothing else:
//   columns forwards   w, and S at the end of every 64 tokens (of the last ones where d_state_out meets it)
//   columns backwards  A = what arrives at S_t from behind;  D = A + q do^T;  du = D^T k;  dv = beta du;  A <- alpha (D - beta k du^T);
//                      and A at the end of every 64 tokens
//   rows forwards      dq = S do,  dk'' = - beta S~ du     (S from w: u = beta w)
//   rows backwards     dk' = D u                           (D from du)
// and what is left per token:  dk = dk' + dk'';  dbeta = du . w;  dlog_alpha_t = E_t + .. + E_c + <S_c, A_c> with E = q . dq - v . dv and c
// the end of the 64 tokens (replacing S by its decayed form shows <S~_t, dS~_t> = E_t + <S_t, A_t>, and <S_t, A_t> is the gradient of the
// next token's gate), so that a long sequence's sums start anew every 64 tokens.
#include <type_traits>

#include "gdr.h"
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
        if (KEEP && !BACK && (t0 + nt == a.L ? a.d_state_out != nullptr : (t0 + nt) % kBorder == 0)) keep(s.S, (t0 + nt - 1) / kBorder);
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

// ---- what is left per token: a block per 64 tokens of a unit -----------------------------------------------------------------
template <typename T>
__device__ void finish(const Gdr<T>& a, const Scratch& s, long long unit, int border) {
    __shared__ float E[kBorder], part[16];
    const int threads = blockDim.x, warps = threads >> 5;
    const int t0 = border * kBorder, nt = min(kBorder, a.L - t0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long plane = (long long)a.dk * a.dv, at = (unit * borders(a.L) + border) * plane;
    float sum = 0.f;
    const bool last = t0 + nt == a.L;
    const float* const behind = last ? a.d_state_out ? a.d_state_out + unit * plane : nullptr : s.A + at;
    if (behind)
#pragma unroll 8
        for (int i = tid; i < plane; i += threads) sum = fmaf(s.S[at + i], behind[i], sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) part[warp] = sum;
#pragma unroll 2
    for (int t = warp; t < nt; t += warps) {
        const long long r = a.row(unit, t0 + t);
        const float beta = to_f(a.beta[r]);
        float e = 0.f, db = 0.f;
        for (int i = lane; i < a.dk; i += 32) {
            const float dq = s.dq[r * a.dk + i];
            e = fmaf(to_f(a.q[r * a.ldk + i]), dq, e);
            if constexpr (sizeof(T) == 2) a.dq[r * a.ldk + i] = from_f<T>(dq);
            a.dk_out[r * a.ldk + i] = from_f<T>(s.dk1[r * a.dk + i] + s.dk2[r * a.dk + i]);
        }
        for (int i = lane; i < a.dv; i += 32) {
            const float du = s.du[r * a.dv + i];
            db = fmaf(du, s.w[r * a.dv + i], db);
            e = fmaf(-beta * du, to_f(a.v[r * a.ldv + i]), e);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            e += __shfl_xor_sync(0xffffffffu, e, o);
            db += __shfl_xor_sync(0xffffffffu, db, o);
        }
        if (lane == 0) {
            E[t] = e;
            a.dbeta[r] = from_f<T>(db);
        }
    }
    __syncthreads();
    // sums from the border; a gate that leaves nothing (what the sums come to there is rounding), or that has nothing to scale (the first of a
    // sequence without an initial state), has none, and they start anew there
    if (warp == 0) {
        float run = 0.f;
        for (int w = 0; w < warps; ++w) run += part[w];
        float mine[2];
        bool stop[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = 2 * lane + h;
            stop[h] = t < nt && (expf(to_f(a.la[a.row(unit, t0 + t)])) == 0.f || (t0 + t == 0 && !a.state_in));
            mine[h] = t < nt && !stop[h] ? E[t] : 0.f;
        }
        run = suffix_of_pairs(mine, stop, run);
        if (2 * lane + 1 < nt) a.dla[a.row(unit, t0 + 2 * lane + 1)] = from_f<T>(run = stop[1] ? 0.f : mine[1] + run);
        if (2 * lane < nt) a.dla[a.row(unit, t0 + 2 * lane)] = from_f<T>(stop[0] ? 0.f : mine[0] + run);
    }
}

template <typename T>
__global__ void __launch_bounds__(512) gdr_finish_kernel(Gdr<T> a, Scratch s) {
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
    return launch_pdl(gdr_finish_kernel<T>, dim3((unsigned)(a.units * borders(a.L))), dim3(512), 0, stream, a, s);
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
