// C-ABI entry points of the selective scan, the causal convolution and the RMS norm: argument validation, dispatch, scratch.
#include <cmath>

#include "ssm.h"
#include "test_hooks.h"

namespace vig {
namespace {

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }   // (NULL is)
template <typename... P>
bool any_null(P... p) { return ((p == nullptr) || ...); }
template <typename... P>
bool all_aligned(size_t to, P... p) { return (aligned(p, to) && ...); }
int status_of(cudaError_t e) { return e == cudaSuccess ? VIG_OK : VIG_ERR_CUDA; }

constexpr int kMostTokens = 0x7fffffff - 0xffff, kMostC = 1 << 20;
constexpr long long kMostPitch = 1LL << 40;

// Pitches as the caller gave them, or dense rows.  A row of `width` values has a pitch of at least that, a multiple of `to` bytes.
struct Pitch {
    int status = VIG_OK;
    const long long* ld;
    size_t elem;
    Pitch(const long long* ld_, size_t elem_) : ld(ld_), elem(elem_) {}
    void set(long long& out, int i, long long width, size_t to, bool used = true) {
        out = ld && used ? ld[i] : width;
        if (status == VIG_OK && (out < width || out > kMostPitch)) status = VIG_ERR_BAD_DIM;
        else if (status == VIG_OK && out * elem % to != 0) status = VIG_ERR_MISALIGNED;
    }
};

// Runs f with scratch of the library's pool.
template <typename F>
int with_scratch(size_t bytes, cudaStream_t stream, F f) {
    void* p = nullptr;
    if (bytes > 0 && pool_alloc(&p, bytes, stream) != cudaSuccess) return VIG_ERR_CUDA;
    int st = status_of(f(static_cast<char*>(p)));
    if (bytes > 0 && cudaFreeAsync(p, stream) != cudaSuccess && st == VIG_OK) st = VIG_ERR_CUDA;
    return st;
}
int clear(void* p, size_t bytes, cudaStream_t stream) { return p ? status_of(cudaMemsetAsync(p, 0, bytes, stream)) : VIG_OK; }
// A call without tokens: what comes out is what went in.
int pass(const void* in, void* out, size_t bytes, cudaStream_t stream) {
    if (!out || out == in || bytes == 0) return VIG_OK;
    return status_of(in ? cudaMemcpyAsync(out, in, bytes, cudaMemcpyDeviceToDevice, stream) : cudaMemsetAsync(out, 0, bytes, stream));
}

// ---- selective scan ----
int check_ssm(int B, int L, int C, int G, int N, int unit) {
    if (N > kSsmMostN || C > kMostC || L > kMostTokens || C % G != 0 || (C / G) % unit != 0) return VIG_ERR_UNSUPPORTED;
    // grids count blocks of channels and pieces of sixteen tokens, or the states
    const long long blocks = (long long)G * ((C / G + kSsmChannels - 1) / kSsmChannels);
    if ((long long)B * L > (1LL << 40) || B * blocks * (L / kSsmTile + 1LL) > 0x7fffffffLL || (long long)B * C > (1LL << 35)) return VIG_ERR_UNSUPPORTED;
    return VIG_OK;
}
bool bad_sizes(int B, int L, int C, int G, int N) { return B < 0 || L < 0 || C < 1 || G < 1 || N < 1; }

template <typename T>
int ssm_fwd_impl(const void* x, const void* dt, const void* A, const void* Bt, const void* Ct, const void* D, const void* z, const void* bias,
                 const void* state_in, void* out, void* state_out, int B, int L, int C, int G, int N, const long long* ld, int softplus, int reverse,
                 cudaStream_t stream) {
    if (any_null(A)) return VIG_ERR_NULL_POINTER;
    if (B != 0 && L != 0 && any_null(x, dt, Bt, Ct, out)) return VIG_ERR_NULL_POINTER;
    if (bad_sizes(B, L, C, G, N)) return VIG_ERR_BAD_DIM;
    Ssm<T> a = {};
    Pitch pitch(ld, sizeof(T));
    pitch.set(a.ldx, 0, C, 16);
    pitch.set(a.lddt, 1, C, 16);
    pitch.set(a.ldz, 2, C, 16, z != nullptr);
    pitch.set(a.ldo, 3, C, 16);
    pitch.set(a.ldB, 4, (long long)G * N, sizeof(T));
    pitch.set(a.ldC, 5, (long long)G * N, sizeof(T));
    if (pitch.status == VIG_ERR_BAD_DIM) return pitch.status;
    if (!all_aligned(16, x, dt, z, out) || !all_aligned(sizeof(T), Bt, Ct) || !all_aligned(4, A, D, bias, state_in, state_out)) return VIG_ERR_MISALIGNED;
    int st = check_ssm(B, L, C, G, N, 16 / sizeof(T));
    if (st == VIG_OK) st = pitch.status;
    if (st != VIG_OK) return st;
    if (B == 0) return VIG_OK;
    if (L == 0) return pass(state_in, state_out, (size_t)B * C * N * sizeof(float), stream);
    a.x = (const T*)x; a.dt = (const T*)dt; a.z = (const T*)z; a.Bt = (const T*)Bt; a.Ct = (const T*)Ct;
    a.A = (const float*)A; a.D = (const float*)D; a.bias = (const float*)bias; a.state_in = (const float*)state_in;
    a.out = (T*)out; a.state_out = (float*)state_out;
    a.B = B; a.L = L; a.C = C; a.G = G; a.N = N; a.per = C / G; a.softplus = softplus != 0; a.reverse = reverse != 0;
    ssm_segments<T>(a, false);
    const size_t states = a.segs > 1 ? ssm_segment_floats(B, C, N, a.segs) : 0, sums = a.segs > 1 ? (size_t)B * a.segs * C : 0;
    return with_scratch((states + sums) * sizeof(float), stream, [&](char* p) {
        a.ends = (float*)p;
        a.total = a.ends + states;
        return launch_ssm_fwd<T>(a, stream);
    });
}

template <typename T>
int ssm_bwd_impl(const void* x, const void* dt, const void* A, const void* Bt, const void* Ct, const void* D, const void* z, const void* bias,
                 const void* state_in, const void* d_out, const void* d_state_out, void* dx, void* ddt, void* dA, void* dB, void* dC, void* dD, void* dz,
                 void* d_bias, void* d_state_in, int B, int L, int C, int G, int N, const long long* ld, int softplus, int reverse, cudaStream_t stream) {
    if (any_null(A) || !dA || (dz && !z)) return VIG_ERR_NULL_POINTER;
    if (B != 0 && L != 0 && (any_null(x, dt, Bt, Ct, d_out) || any_null(dx, ddt, dB, dC))) return VIG_ERR_NULL_POINTER;
    if (bad_sizes(B, L, C, G, N)) return VIG_ERR_BAD_DIM;
    Ssm<T> a = {};
    Pitch pitch(ld, sizeof(T));
    const long long gn = (long long)G * N;
    pitch.set(a.ldx, 0, C, 16);
    pitch.set(a.lddt, 1, C, 16);
    pitch.set(a.ldz, 2, C, 16, z != nullptr);
    pitch.set(a.ldo, 3, C, 16);
    pitch.set(a.ldB, 4, gn, sizeof(T));
    pitch.set(a.ldC, 5, gn, sizeof(T));
    pitch.set(a.lddx, 6, C, 16);
    pitch.set(a.ldddt, 7, C, 16);
    pitch.set(a.lddz, 8, C, 16, dz != nullptr);
    pitch.set(a.lddB, 9, gn, sizeof(T));
    pitch.set(a.lddC, 10, gn, sizeof(T));
    if (pitch.status == VIG_ERR_BAD_DIM) return pitch.status;
    if (!all_aligned(16, x, dt, z, d_out, dx, ddt, dz) || !all_aligned(sizeof(T), Bt, Ct, dB, dC) ||
        !all_aligned(4, A, D, bias, state_in, d_state_out, dA, dD, d_bias, d_state_in))
        return VIG_ERR_MISALIGNED;
    int st = check_ssm(B, L, C, G, N, 16 / sizeof(T));
    if (st == VIG_OK) st = pitch.status;
    // the last launch's grid counts values of dB and dC, and then those of dA
    if (st == VIG_OK && (long long)B * L > (0x3fffffffLL * 128) / ((long long)G * ssm_padded(N))) st = VIG_ERR_UNSUPPORTED;
    if (st != VIG_OK) return st;
    if (B == 0 || L == 0) {
        if ((st = clear(dA, (size_t)C * N * 4, stream)) != VIG_OK || (st = clear(dD, (size_t)C * 4, stream)) != VIG_OK ||
            (st = clear(d_bias, (size_t)C * 4, stream)) != VIG_OK)
            return st;
        return pass(d_state_out, d_state_in, (size_t)B * C * N * sizeof(float), stream);
    }
    a.x = (const T*)x; a.dt = (const T*)dt; a.z = (const T*)z; a.Bt = (const T*)Bt; a.Ct = (const T*)Ct; a.d_out = (const T*)d_out;
    a.A = (const float*)A; a.D = (const float*)D; a.bias = (const float*)bias;
    a.state_in = (const float*)state_in; a.d_state_out = (const float*)d_state_out;
    a.dx = (T*)dx; a.ddt = (T*)ddt; a.dz = (T*)dz; a.dB = (T*)dB; a.dC = (T*)dC;
    a.dA = (float*)dA; a.dD = (float*)dD; a.dbias = (float*)d_bias; a.d_state_in = (float*)d_state_in;
    a.B = B; a.L = L; a.C = C; a.G = G; a.N = N; a.per = C / G; a.softplus = softplus != 0; a.reverse = reverse != 0;
    ssm_segments<T>(a, true);
    return with_scratch(ssm_grad_scratch<T>(a, nullptr), stream, [&](char* p) {
        ssm_grad_scratch<T>(a, p);
        return launch_ssm_bwd<T>(a, stream);
    });
}

template <typename T>
int ssm_step_impl(const void* x, const void* dt, const void* A, const void* Bt, const void* Ct, const void* D, const void* z, const void* bias, void* state,
                  void* out, int B, int C, int G, int N, const long long* ld, int softplus, cudaStream_t stream) {
    if (any_null(A) || (B != 0 && (any_null(x, dt, Bt, Ct) || !state || !out))) return VIG_ERR_NULL_POINTER;
    if (bad_sizes(B, 1, C, G, N)) return VIG_ERR_BAD_DIM;
    Ssm<T> a = {};
    Pitch pitch(ld, sizeof(T));
    pitch.set(a.ldx, 0, C, sizeof(T));
    pitch.set(a.lddt, 1, C, sizeof(T));
    pitch.set(a.ldz, 2, C, sizeof(T), z != nullptr);
    pitch.set(a.ldo, 3, C, sizeof(T));
    pitch.set(a.ldB, 4, (long long)G * N, sizeof(T));
    pitch.set(a.ldC, 5, (long long)G * N, sizeof(T));
    if (pitch.status != VIG_OK) return pitch.status;
    if (!all_aligned(sizeof(T), x, dt, z, out, Bt, Ct) || !all_aligned(4, A, D, bias) || !aligned(state, 16)) return VIG_ERR_MISALIGNED;
    if (N > kSsmMostN || C > kMostC || C % G != 0 || (long long)B * C > (1LL << 34)) return VIG_ERR_UNSUPPORTED;
    if (B == 0) return VIG_OK;
    a.x = (const T*)x; a.dt = (const T*)dt; a.z = (const T*)z; a.Bt = (const T*)Bt; a.Ct = (const T*)Ct;
    a.A = (const float*)A; a.D = (const float*)D; a.bias = (const float*)bias;
    a.out = (T*)out;
    a.B = B; a.L = 1; a.C = C; a.G = G; a.N = N; a.per = C / G; a.softplus = softplus != 0;
    return status_of(launch_ssm_step<T>(a, (float*)state, stream));
}

// ---- causal convolution ----
int check_conv(int B, int L, int C, int K, int act, size_t elem) {
    if (K < 2 || K > 4 || (act != VIG_ACT_NONE && act != VIG_ACT_SILU)) return VIG_ERR_UNSUPPORTED;
    if (C > kMostC || C % (16 / elem) != 0 || L > kMostTokens) return VIG_ERR_UNSUPPORTED;
    // grids count threads: a vector of channels and four tokens each, 128 to a block
    if ((long long)B * (L / 4 + 1LL) > 0x7fffffffLL * 128 / (C / (int)(16 / elem))) return VIG_ERR_UNSUPPORTED;
    return VIG_OK;
}

template <typename T>
int conv_impl(const void* x, const void* w, const void* bias, const void* state_in, void* out, void* state_out, int B, int L, int C, int K,
              const long long* ld, int act, int reverse, cudaStream_t stream) {
    if (any_null(w) || (B != 0 && L != 0 && (any_null(x) || !out))) return VIG_ERR_NULL_POINTER;
    if (B < 0 || L < 0 || C < 1 || K < 1) return VIG_ERR_BAD_DIM;
    Conv<T> a = {};
    Pitch pitch(ld, sizeof(T));
    pitch.set(a.ldx, 0, C, 16);
    pitch.set(a.ldo, 1, C, 16);
    if (pitch.status == VIG_ERR_BAD_DIM) return pitch.status;
    if (!all_aligned(16, x, w, bias, state_in, out, state_out)) return VIG_ERR_MISALIGNED;
    int st = check_conv(B, L, C, K, act, sizeof(T));
    if (st == VIG_OK) st = pitch.status;
    if (st != VIG_OK) return st;
    if (B == 0) return VIG_OK;
    if (L == 0) return pass(state_in, state_out, (size_t)B * (K - 1) * C * sizeof(T), stream);
    a.x = (const T*)x; a.w = (const T*)w; a.bias = (const T*)bias; a.state_in = (const T*)state_in;
    a.out = (T*)out; a.state_out = (T*)state_out;
    a.B = B; a.L = L; a.C = C; a.reverse = reverse != 0;
    conv_pieces<T>(a, false);
    return status_of(launch_conv<T>(a, K, act, stream));
}

template <typename T>
int conv_bwd_impl(const void* x, const void* w, const void* bias, const void* state_in, const void* d_out, const void* d_state_out, void* dx, void* dw,
                  void* dbias, void* d_state_in, int B, int L, int C, int K, const long long* ld, int act, int reverse, cudaStream_t stream) {
    if (any_null(w) || (B != 0 && L != 0 && (any_null(x, d_out) || !dx))) return VIG_ERR_NULL_POINTER;
    if (B < 0 || L < 0 || C < 1 || K < 1) return VIG_ERR_BAD_DIM;
    Conv<T> a = {};
    Pitch pitch(ld, sizeof(T));
    pitch.set(a.ldx, 0, C, 16);
    pitch.set(a.ldo, 1, C, 16);
    pitch.set(a.lddx, 2, C, 16);
    if (pitch.status == VIG_ERR_BAD_DIM) return pitch.status;
    if (!all_aligned(16, x, w, bias, state_in, d_out, d_state_out) || !all_aligned(16, dx, dw, dbias, d_state_in)) return VIG_ERR_MISALIGNED;
    int st = check_conv(B, L, C, K, act, sizeof(T));
    if (st == VIG_OK) st = pitch.status;
    if (st != VIG_OK) return st;
    if (B == 0 || L == 0) {
        if ((st = clear(dw, (size_t)C * K * sizeof(T), stream)) != VIG_OK || (st = clear(dbias, (size_t)C * sizeof(T), stream)) != VIG_OK) return st;
        return pass(d_state_out, d_state_in, (size_t)B * (K - 1) * C * sizeof(T), stream);
    }
    a.x = (const T*)x; a.w = (const T*)w; a.bias = (const T*)bias; a.state_in = (const T*)state_in;
    a.d_out = (const T*)d_out; a.d_state_out = (const T*)d_state_out; a.dx = (T*)dx; a.d_state_in = (T*)d_state_in;
    a.B = B; a.L = L; a.C = C; a.reverse = reverse != 0;
    conv_pieces<T>(a, true);
    const size_t need = dw || dbias ? (size_t)B * a.pieces * C * (K + 1) * sizeof(float) : 0;
    return with_scratch(need, stream, [&](char* p) {
        a.part = (float*)p;
        return launch_conv_bwd<T>(a, K, act, (T*)dw, (T*)dbias, stream);
    });
}

template <typename T>
int conv_step_impl(const void* x, const void* w, const void* bias, void* state, void* out, int B, int C, int K, const long long* ld, int act,
                   cudaStream_t stream) {
    if (any_null(w) || (B != 0 && (any_null(x) || !state || !out))) return VIG_ERR_NULL_POINTER;
    if (B < 0 || C < 1 || K < 1) return VIG_ERR_BAD_DIM;
    Conv<T> a = {};
    Pitch pitch(ld, sizeof(T));
    pitch.set(a.ldx, 0, C, 16);
    pitch.set(a.ldo, 1, C, 16);
    if (pitch.status == VIG_ERR_BAD_DIM) return pitch.status;
    if (!all_aligned(16, x, w, bias, state, out)) return VIG_ERR_MISALIGNED;
    int st = check_conv(B, 1, C, K, act, sizeof(T));
    if (st == VIG_OK) st = pitch.status;
    if (st != VIG_OK) return st;
    if (B == 0) return VIG_OK;
    a.x = (const T*)x; a.w = (const T*)w; a.bias = (const T*)bias; a.out = (T*)out;
    a.B = B; a.L = 1; a.C = C; a.piece = a.pieces = 1;
    return status_of(launch_conv_step<T>(a, K, act, (T*)state, stream));
}

// ---- RMS norm ----
int check_rms(long long rows, int C, size_t elem) {
    if (C > kRmsMostC || C % (16 / elem) != 0 || rows > 0x7fffffffLL) return VIG_ERR_UNSUPPORTED;
    return VIG_OK;
}

template <typename T>
int rms_impl(const void* x, const void* residual, const void* weight, void* out, void* scales, void* sum_out, void* rstd, long long rows, int C, int block,
             bool eight, float eps, cudaStream_t stream) {
    if (any_null(weight) || (rows != 0 && (any_null(x) || !out || (eight && !scales)))) return VIG_ERR_NULL_POINTER;
    if (rows < 0 || C < 1 || !(eps >= 0.f) || !std::isfinite(eps)) return VIG_ERR_BAD_DIM;
    if (!all_aligned(16, x, residual, weight, sum_out) || !aligned(out, eight ? 8 : 16) || !all_aligned(4, rstd, scales)) return VIG_ERR_MISALIGNED;
    int st = check_rms(rows, C, sizeof(T));
    if (st == VIG_OK && eight && block != 0 && block != 128) st = VIG_ERR_UNSUPPORTED;
    if (st != VIG_OK || rows == 0) return st;
    RmsNorm<T> a = {};
    a.x = (const T*)x; a.residual = (const T*)residual; a.weight = (const T*)weight;
    a.out = (T*)out; a.q = (unsigned char*)out; a.sum_out = (T*)sum_out; a.rstd = (float*)rstd; a.scales = (float*)scales;
    a.rows = rows; a.C = C; a.eps = eps; a.inv_C = 1.f / (float)C;
    return status_of(launch_rms_norm<T>(a, !eight ? 0 : block == 0 ? 1 : 2, stream));
}

template <typename T>
int rms_bwd_impl(const void* sum, const void* weight, const void* rstd, const void* d_out, const void* d_sum, void* dx, void* dweight, long long rows, int C,
                 cudaStream_t stream) {
    if (any_null(weight) || (rows != 0 && (any_null(sum, rstd, d_out) || !dx))) return VIG_ERR_NULL_POINTER;
    if (rows < 0 || C < 1) return VIG_ERR_BAD_DIM;
    if (!all_aligned(16, sum, weight, d_out, d_sum) || !all_aligned(16, dx, dweight) || !aligned(rstd, 4)) return VIG_ERR_MISALIGNED;
    const int st = check_rms(rows, C, sizeof(T));
    if (st != VIG_OK) return st;
    if (rows == 0) return clear(dweight, (size_t)C * sizeof(T), stream);
    RmsNormGrad<T> a = {};
    a.sum = (const T*)sum; a.weight = (const T*)weight; a.d_out = (const T*)d_out; a.d_sum = (const T*)d_sum; a.rstd = (const float*)rstd;
    a.dx = (T*)dx; a.rows = rows; a.C = C; a.inv_C = 1.f / (float)C;
    return with_scratch(dweight ? (size_t)rms_norm_bwd_blocks<T>(rows, C) * C * sizeof(float) : 0, stream, [&](char* p) {
        a.part = (float*)p;
        return launch_rms_norm_bwd<T>(a, (T*)dweight, stream);
    });
}

}  // namespace
}  // namespace vig

using namespace vig;

extern "C" {

#define VIG_ROWS(T, NAME)                                                                                                                         \
    int vig_ssm_fwd_##NAME(const void* x, const void* dt, const void* A, const void* Bt, const void* Ct, const void* D, const void* z,             \
                           const void* dt_bias, const void* state_in, void* out, void* state_out, int B, int L, int C, int G, int N,               \
                           const long long* ld, int softplus, int reverse, void* stream) {                                                         \
        return ssm_fwd_impl<T>(x, dt, A, Bt, Ct, D, z, dt_bias, state_in, out, state_out, B, L, C, G, N, ld, softplus, reverse,                    \
                               (cudaStream_t)stream);                                                                                             \
    }                                                                                                                                             \
    int vig_ssm_bwd_##NAME(const void* x, const void* dt, const void* A, const void* Bt, const void* Ct, const void* D, const void* z,             \
                           const void* dt_bias, const void* state_in, const void* d_out, const void* d_state_out, void* dx, void* ddt, void* dA,   \
                           void* dB, void* dC, void* dD, void* dz, void* d_dt_bias, void* d_state_in, int B, int L, int C, int G, int N,           \
                           const long long* ld, int softplus, int reverse, void* stream) {                                                         \
        return ssm_bwd_impl<T>(x, dt, A, Bt, Ct, D, z, dt_bias, state_in, d_out, d_state_out, dx, ddt, dA, dB, dC, dD, dz, d_dt_bias, d_state_in, B, \
                               L, C, G, N, ld, softplus, reverse, (cudaStream_t)stream);                                                           \
    }                                                                                                                                             \
    int vig_ssm_step_##NAME(const void* x, const void* dt, const void* A, const void* Bt, const void* Ct, const void* D, const void* z,            \
                            const void* dt_bias, void* state, void* out, int B, int C, int G, int N, const long long* ld, int softplus,            \
                            void* stream) {                                                                                                       \
        return ssm_step_impl<T>(x, dt, A, Bt, Ct, D, z, dt_bias, state, out, B, C, G, N, ld, softplus, (cudaStream_t)stream);                      \
    }                                                                                                                                             \
    int vig_causal_conv_##NAME(const void* x, const void* w, const void* bias, const void* state_in, void* out, void* state_out, int B, int L,     \
                               int C, int K, const long long* ld, int act, int reverse, void* stream) {                                            \
        return conv_impl<T>(x, w, bias, state_in, out, state_out, B, L, C, K, ld, act, reverse, (cudaStream_t)stream);                             \
    }                                                                                                                                             \
    int vig_causal_conv_bwd_##NAME(const void* x, const void* w, const void* bias, const void* state_in, const void* d_out,                        \
                                   const void* d_state_out, void* dx, void* dw, void* dbias, void* d_state_in, int B, int L, int C, int K,          \
                                   const long long* ld, int act, int reverse, void* stream) {                                                      \
        return conv_bwd_impl<T>(x, w, bias, state_in, d_out, d_state_out, dx, dw, dbias, d_state_in, B, L, C, K, ld, act, reverse,                 \
                                (cudaStream_t)stream);                                                                                            \
    }                                                                                                                                             \
    int vig_causal_conv_step_##NAME(const void* x, const void* w, const void* bias, void* state, void* out, int B, int C, int K,                   \
                                    const long long* ld, int act, void* stream) {                                                                  \
        return conv_step_impl<T>(x, w, bias, state, out, B, C, K, ld, act, (cudaStream_t)stream);                                                  \
    }                                                                                                                                             \
    int vig_rms_norm_##NAME(const void* x, const void* residual, const void* weight, void* out, void* sum_out, void* rstd, long long rows, int C,  \
                            float eps, void* stream) {                                                                                            \
        return rms_impl<T>(x, residual, weight, out, nullptr, sum_out, rstd, rows, C, 0, false, eps, (cudaStream_t)stream);                        \
    }                                                                                                                                             \
    int vig_rms_norm_e4m3_##NAME(const void* x, const void* residual, const void* weight, void* out, void* scales, void* sum_out, long long rows,  \
                                 int C, int block, float eps, void* stream) {                                                                      \
        return rms_impl<T>(x, residual, weight, out, scales, sum_out, nullptr, rows, C, block, true, eps, (cudaStream_t)stream);                   \
    }                                                                                                                                             \
    int vig_rms_norm_bwd_##NAME(const void* sum, const void* weight, const void* rstd, const void* d_out, const void* d_sum, void* dx,             \
                                void* dweight, long long rows, int C, void* stream) {                                                             \
        return rms_bwd_impl<T>(sum, weight, rstd, d_out, d_sum, dx, dweight, rows, C, (cudaStream_t)stream);                                       \
    }

VIG_ROWS(__nv_bfloat16, bf16)
VIG_ROWS(float, f32)

size_t vig_test_ssm_bwd_scratch(int B, int L, int C, int G, int N) {
    Ssm<float> a = {};   // (the same for either type)
    a.B = B; a.L = L; a.C = C; a.G = G; a.N = N; a.per = C / G;
    ssm_segments<float>(a, true);
    return ssm_grad_scratch<float>(a, nullptr);
}

}  // extern "C"
