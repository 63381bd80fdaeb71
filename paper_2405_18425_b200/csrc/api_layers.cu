// C-ABI entry points of the gated delta rule and of the group norm: argument validation, dispatch, scratch.
#include <cmath>

#include "gdr.h"
#include "test_hooks.h"

namespace vig {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }   // (NULL is)

template <typename... P>
bool any_null(P... p) { return ((p == nullptr) || ...); }
template <typename... P>
bool all_aligned(P... p) { return (aligned16(p) && ...); }

int status_of(cudaError_t e) { return e == cudaSuccess ? VIG_OK : VIG_ERR_CUDA; }

// A call without tokens: what comes out is what went in.
int pass_state(const void* in, void* out, long long units, int dk, int dv, cudaStream_t stream) {
    const size_t bytes = (size_t)units * dk * dv * sizeof(float);
    if (!out || out == in || bytes == 0) return VIG_OK;
    return status_of(in ? cudaMemcpyAsync(out, in, bytes, cudaMemcpyDeviceToDevice, stream) : cudaMemsetAsync(out, 0, bytes, stream));
}

constexpr int kMostRows = 0x7fffffff - 0xffff;   // tokens or pixels

int check_sizes(int B, int H, int L, int dk, int dv) {
    if (B < 0 || H < 0 || L < 0 || dk < 1 || dv < 1) return VIG_ERR_BAD_DIM;
    if (!gdr_supported(dk, dv)) return VIG_ERR_UNSUPPORTED;
    // grids count units, or units times pieces of 64 tokens; tokens are counted in 32 bits up to the end of their last piece
    if (L > kMostRows || (long long)B * H * (L / 64 + 1LL) > 0x7fffffffLL) return VIG_ERR_UNSUPPORTED;
    return VIG_OK;
}

// bf16: chunks on the tensor cores, or walks.  A chunk costs its set-up whatever it holds, a walk its tokens: 1500 units of 64 x 64, forward, tiles and walks
// us: 2 tokens 29, 21; 8 tokens 29, 33; 128 x 128: 8 tokens 96, 93, 12 tokens 98, 122; gradient alone of 150 units of 64 x 64: 2 tokens 28, 28; 4 tokens
// 28, 32; of 150 of 128 x 128: 2 tokens 58, 54; 4 tokens 58, 62; of 500 of 64 x 64: 1 token 42, 50.
template <typename T>
bool takes_tiles(long long units, int L, int dk, int dv, bool gradient) {
    if (sizeof(T) != 2 || (gradient && !gdr_grad_supported(dk, dv))) return false;
    const int pref = kernel_preference();
    if (pref == VIG_TEST_KERNEL_SIMT || pref == VIG_TEST_KERNEL_WARP_TILES) return pref == VIG_TEST_KERNEL_WARP_TILES;
    return L > (gradient ? (units <= 300 ? 2 : 0) : 8);
}

// Copies of a call's rows with zeros up to multiples of eight, where the sizes are none.
struct Padded {
    int dk, dv, dk0, dv0;
    size_t keys, values;   // bytes of a copy; 0: no copies
    Padded(int dk_, int dv_, size_t rows) : dk((dk_ + 7) & ~7), dv((dv_ + 7) & ~7), dk0(dk_), dv0(dv_) {
        const bool any = dk != dk0 || dv != dv0;
        keys = any ? (rows * dk * 2 + 255) / 256 * 256 : 0;
        values = any ? (rows * dv * 2 + 255) / 256 * 256 : 0;
    }
    template <typename T>
    void key(const T*& t, RowCopy& c, char*& at) const {
        c = {t, at, dk0, dk};
        t = (const T*)at;
        at += keys;
    }
    template <typename T>
    void value(const T*& t, RowCopy& c, char*& at) const {
        c = {t, at, dv0, dv};
        t = (const T*)at;
        at += values;
    }
};

template <typename T>
int gdr_fwd_impl(const void* q, const void* k, const void* v, const void* la, const void* beta, const void* state_in, void* out, void* state_out, int B,
                 int H, int L, int dk, int dv, int reverse, cudaStream_t stream) {
    if (B != 0 && H != 0 && L != 0 && any_null(q, k, v, la, beta, out)) return VIG_ERR_NULL_POINTER;   // (tensors without elements may have no address)
    if (B < 0 || H < 0 || L < 0 || dk < 1 || dv < 1) return VIG_ERR_BAD_DIM;
    if (!all_aligned(q, k, v, la, beta, state_in, out, state_out)) return VIG_ERR_MISALIGNED;
    const int st = check_sizes(B, H, L, dk, dv);
    if (st != VIG_OK) return st;
    const long long units = (long long)B * H;
    if (units == 0) return VIG_OK;
    if (L == 0) return pass_state(state_in, state_out, units, dk, dv, stream);
    Gdr<T> a = {};
    a.q = (const T*)q; a.k = (const T*)k; a.v = (const T*)v; a.la = (const T*)la; a.beta = (const T*)beta;
    a.state_in = (const float*)state_in; a.out = (T*)out; a.state_out = (float*)state_out;
    a.units = units; a.L = L; a.dk = a.ldk = dk; a.dv = a.ldv = dv; a.reverse = reverse != 0;
    if constexpr (sizeof(T) == 2)
        if (takes_tiles<T>(units, L, dk, dv, false)) {
            const size_t rows = (size_t)units * L;
            const Padded pad(dk, dv, rows);
            const size_t need = (gdr_chunk_scratch_bytes(units, L, dk, dv) + 255) / 256 * 256, copies = 2 * pad.keys + 2 * pad.values;
            // an initial state that the call overwrites is put aside where segments' units that leave the tiles' range start from it again
            const size_t aside = need > 0 && state_in && state_in == state_out ? (size_t)units * dk * dv * sizeof(float) : 0;
            if (need + aside + copies == 0) return status_of(launch_gdr_chunk_fwd(a, nullptr, stream));
            char* ws = nullptr;
            if (pool_alloc((void**)&ws, need + aside + copies, stream) != cudaSuccess) return VIG_ERR_CUDA;
            cudaError_t e = cudaSuccess;
            if (aside) {
                e = cudaMemcpyAsync(ws + need + copies, state_in, aside, cudaMemcpyDeviceToDevice, stream);
                a.state_in = (const float*)(ws + need + copies);
            }
            if (copies && e == cudaSuccess) {
                char* p = ws + need;
                RowCopy in[kRowCopies];
                int n = 0;
                pad.key(a.q, in[n++], p);
                pad.key(a.k, in[n++], p);
                pad.value(a.v, in[n++], p);
                e = launch_copy_rows(in, n, rows, stream);
                a.out = (T*)p;
                a.ldk = pad.dk;
                a.ldv = pad.dv;
            }
            if (e == cudaSuccess) e = launch_gdr_chunk_fwd(a, ws, stream);
            if (copies && e == cudaSuccess) {
                const RowCopy back = {a.out, out, pad.dv, dv};
                e = launch_copy_rows(&back, 1, rows, stream);
            }
            const bool freed = cudaFreeAsync(ws, stream) == cudaSuccess;
            return freed ? status_of(e) : VIG_ERR_CUDA;
        }
    return status_of(launch_gdr_walk_fwd<T>(a, stream));
}

template <typename T>
int gdr_bwd_impl(const void* q, const void* k, const void* v, const void* la, const void* beta, const void* state_in, const void* d_out,
                 const void* d_state_out, void* dq, void* dk_out, void* dv_out, void* dla, void* dbeta, void* d_state_in, int B, int H, int L, int dk,
                 int dv, int reverse, cudaStream_t stream) {
    if (B != 0 && H != 0 && L != 0 && (any_null(q, k, v, la, beta, d_out) || any_null(dq, dk_out, dv_out, dla, dbeta))) return VIG_ERR_NULL_POINTER;
    if (B < 0 || H < 0 || L < 0 || dk < 1 || dv < 1) return VIG_ERR_BAD_DIM;
    if (!all_aligned(q, k, v, la, beta, state_in, d_out, d_state_out) || !all_aligned(dq, dk_out, dv_out, dla, dbeta, d_state_in)) return VIG_ERR_MISALIGNED;
    int st = check_sizes(B, H, L, dk, dv);
    if (st != VIG_OK) return st;
    const long long units = (long long)B * H;
    if (units == 0) return VIG_OK;
    if (L == 0) return pass_state(d_state_out, d_state_in, units, dk, dv, stream);
    Gdr<T> a = {};
    a.q = (const T*)q; a.k = (const T*)k; a.v = (const T*)v; a.la = (const T*)la; a.beta = (const T*)beta; a.d_out = (const T*)d_out;
    a.state_in = (const float*)state_in; a.d_state_out = (const float*)d_state_out;
    a.dq = (T*)dq; a.dk_out = (T*)dk_out; a.dv_out = (T*)dv_out; a.dla = (T*)dla; a.dbeta = (T*)dbeta; a.d_state_in = (float*)d_state_in;
    a.units = units; a.L = L; a.dk = a.ldk = dk; a.dv = a.ldv = dv; a.reverse = reverse != 0;
    size_t need = 0;
    bool chunks = false;
    if constexpr (sizeof(T) == 2) {
        chunks = takes_tiles<T>(units, L, dk, dv, true);
        if (chunks) need = gdr_grad_scratch_bytes(units, L, dk, dv);
    }
    if (!chunks) need = gdr_walk_bwd_scratch_bytes<T>(units, L, dk, dv);
    // a final state's gradient that the call overwrites is put aside: later launches start from it again
    const size_t aside = d_state_in && d_state_in == d_state_out ? (size_t)units * dk * dv * sizeof(float) : 0;
    const size_t rows = (size_t)units * L;
    const Padded pad(dk, dv, rows);
    const size_t copies = chunks ? 4 * pad.keys + 3 * pad.values : 0;
    need = (need + 255) / 256 * 256;
    const size_t put = (aside + 255) / 256 * 256;
    char* ws = nullptr;
    if (pool_alloc((void**)&ws, need + put + copies, stream) != cudaSuccess) return VIG_ERR_CUDA;
    cudaError_t e = cudaSuccess;
    if (aside) {
        e = cudaMemcpyAsync(ws + need, d_state_out, aside, cudaMemcpyDeviceToDevice, stream);
        a.d_state_out = (const float*)(ws + need);
    }
    if constexpr (sizeof(T) == 2)
        if (chunks && e == cudaSuccess) {
            if (copies) {
                char* p = ws + need + put;
                RowCopy in[kRowCopies];
                pad.key(a.q, in[0], p);
                pad.key(a.k, in[1], p);
                pad.value(a.v, in[2], p);
                pad.value(a.d_out, in[3], p);
                e = launch_copy_rows(in, 4, rows, stream);
                a.dq = (T*)p;
                a.dk_out = (T*)(p + pad.keys);
                a.dv_out = (T*)(p + 2 * pad.keys);
                a.ldk = pad.dk;
                a.ldv = pad.dv;
            }
            if (e == cudaSuccess) e = launch_gdr_chunk_bwd(a, ws, stream);
            if (copies && e == cudaSuccess) {
                const RowCopy back[3] = {{a.dq, dq, pad.dk, dk}, {a.dk_out, dk_out, pad.dk, dk}, {a.dv_out, dv_out, pad.dv, dv}};
                e = launch_copy_rows(back, 3, rows, stream);
            }
        }
    if (!chunks && e == cudaSuccess) e = launch_gdr_walk_bwd<T>(a, ws, stream);
    st = status_of(e);
    if (cudaFreeAsync(ws, stream) != cudaSuccess && st == VIG_OK) st = VIG_ERR_CUDA;
    return st;
}

template <typename T>
int gdr_step_impl(const void* q, const void* k, const void* v, const void* la, const void* beta, void* state, void* out, int B, int H, int dk, int dv,
                  cudaStream_t stream) {
    if (B != 0 && H != 0 && any_null(q, k, v, la, beta, state, out)) return VIG_ERR_NULL_POINTER;
    if (B < 0 || H < 0 || dk < 1 || dv < 1) return VIG_ERR_BAD_DIM;
    if (!all_aligned(q, k, v, la, beta, state, out)) return VIG_ERR_MISALIGNED;
    const int st = check_sizes(B, H, 1, dk, dv);
    if (st != VIG_OK) return st;
    if (B == 0 || H == 0) return VIG_OK;
    return status_of(launch_gdr_step<T>((const T*)q, (const T*)k, (const T*)v, (const T*)la, (const T*)beta, (float*)state, (T*)out, (long long)B * H,
                                        dk, dv, stream));
}

int check_norm(int B, int Hh, int Ww, int C, int groups, int act, size_t elem) {
    if (B < 0 || Hh < 0 || Ww < 0 || C < 1 || groups < 1) return VIG_ERR_BAD_DIM;
    if (act != VIG_ACT_NONE && act != VIG_ACT_SILU && act != VIG_ACT_GELU) return VIG_ERR_UNSUPPORTED;
    if ((long long)Hh * Ww > kMostRows || !group_norm_supported(B, Hh * Ww, C, groups, elem)) return VIG_ERR_UNSUPPORTED;
    return VIG_OK;
}

template <typename T>
int group_norm_impl(const void* x, const void* weight, const void* bias, void* out, void* mean, void* rstd, int B, int Hh, int Ww, int C, int groups,
                    float eps, int act, cudaStream_t stream) {
    if (B != 0 && Hh != 0 && Ww != 0 && any_null(x, out)) return VIG_ERR_NULL_POINTER;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return VIG_ERR_BAD_DIM;
    if (B < 0 || Hh < 0 || Ww < 0 || C < 1 || groups < 1) return VIG_ERR_BAD_DIM;
    if (!all_aligned(x, weight, bias, out, mean, rstd)) return VIG_ERR_MISALIGNED;
    int st = check_norm(B, Hh, Ww, C, groups, act, sizeof(T));
    if (st != VIG_OK) return st;
    const int HW = Hh * Ww;
    if (B == 0 || HW == 0) return VIG_OK;
    const size_t need = group_norm_scratch_bytes(B, HW, C, groups, sizeof(T), false);
    void* scratch = nullptr;
    if (need > 0 && pool_alloc(&scratch, need, stream) != cudaSuccess) return VIG_ERR_CUDA;
    st = status_of(launch_group_norm<T>((const T*)x, (const T*)weight, (const T*)bias, (T*)out, (float*)mean, (float*)rstd, B, HW, C, groups, eps, act,
                                        scratch, stream));
    if (need > 0 && cudaFreeAsync(scratch, stream) != cudaSuccess && st == VIG_OK) st = VIG_ERR_CUDA;
    return st;
}

template <typename T>
int group_norm_bwd_impl(const void* x, const void* weight, const void* bias, const void* mean, const void* rstd, const void* d_out, void* dx,
                        void* dweight, void* dbias, int B, int Hh, int Ww, int C, int groups, int act, cudaStream_t stream) {
    if (B != 0 && Hh != 0 && Ww != 0 && (any_null(x, mean, rstd, d_out) || !dx)) return VIG_ERR_NULL_POINTER;
    if (B < 0 || Hh < 0 || Ww < 0 || C < 1 || groups < 1) return VIG_ERR_BAD_DIM;
    if (!all_aligned(x, weight, bias, mean, rstd, d_out) || !all_aligned(dx, dweight, dbias)) return VIG_ERR_MISALIGNED;
    int st = check_norm(B, Hh, Ww, C, groups, act, sizeof(T));
    if (st != VIG_OK) return st;
    const int HW = Hh * Ww;
    if (B == 0 || HW == 0) {
        if (dweight && cudaMemsetAsync(dweight, 0, C * sizeof(T), stream) != cudaSuccess) return VIG_ERR_CUDA;
        if (dbias && cudaMemsetAsync(dbias, 0, C * sizeof(T), stream) != cudaSuccess) return VIG_ERR_CUDA;
        return VIG_OK;
    }
    void* scratch = nullptr;
    if (pool_alloc(&scratch, group_norm_scratch_bytes(B, HW, C, groups, sizeof(T), true), stream) != cudaSuccess) return VIG_ERR_CUDA;
    st = status_of(launch_group_norm_bwd<T>((const T*)x, (const T*)weight, (const T*)bias, (const float*)mean, (const float*)rstd, (const T*)d_out,
                                            (T*)dx, (T*)dweight, (T*)dbias, B, HW, C, groups, act, scratch, stream));
    if (cudaFreeAsync(scratch, stream) != cudaSuccess && st == VIG_OK) st = VIG_ERR_CUDA;
    return st;
}

}  // namespace
}  // namespace vig

using namespace vig;

extern "C" {

#define VIG_LAYERS(T, NAME)                                                                                                                      \
    int vig_gdr_fwd_##NAME(const void* q, const void* k, const void* v, const void* log_alpha, const void* beta, const void* state_in, void* out, \
                           void* state_out, int B, int H, int L, int dk, int dv, int reverse, void* stream) {                                     \
        return gdr_fwd_impl<T>(q, k, v, log_alpha, beta, state_in, out, state_out, B, H, L, dk, dv, reverse, (cudaStream_t)stream);               \
    }                                                                                                                                            \
    int vig_gdr_bwd_##NAME(const void* q, const void* k, const void* v, const void* log_alpha, const void* beta, const void* state_in,            \
                           const void* d_out, const void* d_state_out, void* dq, void* dk_out, void* dv_out, void* dlog_alpha, void* dbeta,       \
                           void* d_state_in, int B, int H, int L, int dk, int dv, int reverse, void* stream) {                                    \
        return gdr_bwd_impl<T>(q, k, v, log_alpha, beta, state_in, d_out, d_state_out, dq, dk_out, dv_out, dlog_alpha, dbeta, d_state_in, B, H, L, \
                               dk, dv, reverse, (cudaStream_t)stream);                                                                           \
    }                                                                                                                                            \
    int vig_gdr_step_##NAME(const void* q, const void* k, const void* v, const void* log_alpha, const void* beta, void* state, void* out, int B,  \
                            int H, int dk, int dv, void* stream) {                                                                               \
        return gdr_step_impl<T>(q, k, v, log_alpha, beta, state, out, B, H, dk, dv, (cudaStream_t)stream);                                        \
    }                                                                                                                                            \
    int vig_group_norm_##NAME(const void* x, const void* weight, const void* bias, void* out, void* mean, void* rstd, int B, int Hh, int Ww,      \
                              int C, int groups, float eps, int act, void* stream) {                                                             \
        return group_norm_impl<T>(x, weight, bias, out, mean, rstd, B, Hh, Ww, C, groups, eps, act, (cudaStream_t)stream);                        \
    }                                                                                                                                            \
    int vig_group_norm_bwd_##NAME(const void* x, const void* weight, const void* bias, const void* mean, const void* rstd, const void* d_out,     \
                                  void* dx, void* dweight, void* dbias, int B, int Hh, int Ww, int C, int groups, int act, void* stream) {        \
        return group_norm_bwd_impl<T>(x, weight, bias, mean, rstd, d_out, dx, dweight, dbias, B, Hh, Ww, C, groups, act, (cudaStream_t)stream);   \
    }

VIG_LAYERS(__nv_bfloat16, bf16)
VIG_LAYERS(float, f32)

}  // extern "C"
