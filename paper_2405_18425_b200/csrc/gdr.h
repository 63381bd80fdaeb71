// Internal declarations of the gated delta rule and of the group norm (not part of the C ABI).
#pragma once
#include "vig_internal.h"

namespace vig {

// A call of the gated delta rule.  Row t of a unit in walking order is token t, or L - 1 - t in a reverse call.  Null pointers:
// state_in, state_out, d_state_out, d_state_in where the caller has none; out in the gradient, d_out and the gradients forward.
template <typename T>
struct Gdr {
    const T *q, *k, *v, *la, *beta, *d_out;
    const float *state_in, *d_state_out;
    T *out, *dq, *dk_out, *dv_out, *dla, *dbeta;
    float *state_out, *d_state_in;
    long long units;
    int L, dk, dv;
    bool reverse;
    __host__ __device__ long long row(long long unit, int t) const { return unit * L + (reverse ? L - 1 - t : t); }
};

bool gdr_supported(int dk, int dv);   // dk <= 128, dv <= 256

// ---- step by step in fp32 on the CUDA cores ----
template <typename T>
cudaError_t launch_gdr_walk_fwd(const Gdr<T>& a, cudaStream_t stream);
template <typename T>
size_t gdr_walk_bwd_scratch_bytes(long long units, int L, int dk, int dv);
template <typename T>
cudaError_t launch_gdr_walk_bwd(const Gdr<T>& a, void* scratch, cudaStream_t stream);

// ---- forward in chunks on the tensor cores: head sizes that are multiples of eight ----
bool gdr_chunk_supported(int dk, int dv);
cudaError_t launch_gdr_chunk_fwd(const Gdr<__nv_bfloat16>& a, cudaStream_t stream);

// ---- one token: state updated in place ----
template <typename T>
cudaError_t launch_gdr_step(const T* q, const T* k, const T* v, const T* la, const T* beta, float* state, T* out, long long units, int dk, int dv,
                            cudaStream_t stream);

// ---- group norm with an activation, channels last ----
bool group_norm_supported(int B, int HW, int C, int groups, size_t elem);
size_t group_norm_scratch_bytes(int B, int HW, int C, int groups, size_t elem, bool gradient);   // 0: the call uses no scratch
template <typename T>
cudaError_t launch_group_norm(const T* x, const T* weight, const T* bias, T* out, float* mean, float* rstd, int B, int HW, int C, int groups,
                              float eps, int act, void* scratch, cudaStream_t stream);
template <typename T>
cudaError_t launch_group_norm_bwd(const T* x, const T* weight, const T* bias, const float* mean, const float* rstd, const T* d_out, T* dx, T* dweight,
                                  T* dbias, int B, int HW, int C, int groups, int act, void* scratch, cudaStream_t stream);

}  // namespace vig
