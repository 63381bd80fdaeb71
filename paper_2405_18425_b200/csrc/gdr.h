// Internal declarations of the gated delta rule and of the group norm (not part of the C ABI).
#pragma once
#include <atomic>

#include "vig_internal.h"

namespace vig {

// Lets a kernel have up to `most` bytes of dynamic shared memory, the largest that any call of it takes: set once per device.  (The limit belongs to the
// process: set to each call's own size, another thread's smaller one could come between it and the launch.)
template <auto Kernel>
cudaError_t allow_smem(size_t most) {
    static std::atomic<bool> done[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (most <= 48 * 1024 || done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    if ((e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most)) != cudaSuccess) return e;
    done[dev].store(true, std::memory_order_release);
    return cudaSuccess;
}

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
    int ldk, ldv;   // values of a row of q, k, dq, dk and of v, d_out, out, dv in memory: dk and dv, or those to a multiple of eight (gdr_pad.cu)
    bool reverse;
    __host__ __device__ long long row(long long unit, int t) const { return unit * L + (reverse ? L - 1 - t : t); }
};

#ifdef __CUDACC__
// Of 64 values, two a lane: what is in front of this lane's pair, and what is behind it.  (Nothing is added and taken off again: a small sum beside large
// values keeps its digits.)
__device__ __forceinline__ float before_pair(float x0, float x1) {
    const int lane = threadIdx.x & 31;
    float run = x0 + x1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float y = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += y;
    }
    run = __shfl_up_sync(0xffffffffu, run, 1);
    return lane == 0 ? 0.f : run;
}
__device__ __forceinline__ float behind_pair(float x0, float x1) {
    const int lane = threadIdx.x & 31;
    float run = x0 + x1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float y = __shfl_down_sync(0xffffffffu, run, o);
        if (lane + o < 32) run += y;
    }
    run = __shfl_down_sync(0xffffffffu, run, 1);
    return lane == 31 ? 0.f : run;
}
#endif

bool gdr_supported(int dk, int dv);   // dk <= 128, dv <= 256

// ---- step by step in fp32 on the CUDA cores ----
template <typename T>
cudaError_t launch_gdr_walk_fwd(const Gdr<T>& a, cudaStream_t stream);
template <typename T>
size_t gdr_walk_bwd_scratch_bytes(long long units, int L, int dk, int dv);
template <typename T>
cudaError_t launch_gdr_walk_bwd(const Gdr<T>& a, void* scratch, cudaStream_t stream);

// ---- rows of other sizes than multiples of eight: laid out again with zeros behind them for the forms that take pieces of sixteen bytes ----
struct RowCopy {
    const void* src;
    void* dst;
    int from, to;   // values of a row there and here
};
constexpr int kRowCopies = 4;
// rows x n copies of bf16 rows; zeros behind the source's values.
cudaError_t launch_copy_rows(const RowCopy* copies, int n, long long rows, cudaStream_t stream);

// ---- forward in chunks on the tensor cores: ldk and ldv multiples of eight ----
size_t gdr_chunk_scratch_bytes(long long units, int L, int dk, int dv);   // 0: the call uses no scratch
cudaError_t launch_gdr_chunk_fwd(const Gdr<__nv_bfloat16>& a, void* scratch, cudaStream_t stream);

// What the two walks of the gradient keep, two bf16 terms each (the second `.._term` values behind the first; sixteen significant bits, at two bytes a
// term what fp32 would take, and ready to be an operand); dvp: dv to sixteen, DKP: dk as the kernels pad it.
struct GdrKept {
    __nv_bfloat16* w;      // [2][units][chunks][64][dvp]: W; rows behind a call's last sixteen are not written
    __nv_bfloat16* du;     // [2][units][chunks][64][dvp]: dU
    __nv_bfloat16 *S, *A;  // transposed, [2][units][chunks][dvp][DKP]: before each chunk, and what arrives behind it
    long long row_term, state_term;
    int* lost_grad;        // [units][chunks]: something is not finite
    int dvp;
    // Sixteen columns and sixteen key dimensions of a state, as packed for an A operand; not `there`: a state of zeros, which nothing is read of.
    template <int DKP, int N>
    __device__ __forceinline__ void keep_state(__nv_bfloat16* to, long long term, long long at, int col0, int s, const uint32_t (&sa)[N][4], int g, int c,
                                               bool there) const {
        if (!there) return;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            __nv_bfloat16* const p = to + m * term + (at * dvp + col0 + g) * DKP + s * 16 + 2 * c;
            *reinterpret_cast<uint32_t*>(p) = sa[m][0];
            *reinterpret_cast<uint32_t*>(p + 8 * DKP) = sa[m][1];
            *reinterpret_cast<uint32_t*>(p + 8) = sa[m][2];
            *reinterpret_cast<uint32_t*>(p + 8 * DKP + 8) = sa[m][3];
        }
    }
};
int gdr_padded_columns(int dv);   // dvp
int gdr_padded_keys(int dk);      // DKP
bool gdr_grad_supported(int dk, int dv);
size_t gdr_grad_scratch_bytes(long long units, int L, int dk, int dv);
// The whole gradient: both walks, the chunks, and the fp32 walks for units that left the range.
cudaError_t launch_gdr_chunk_bwd(const Gdr<__nv_bfloat16>& a, void* scratch, cudaStream_t stream);
cudaError_t launch_gdr_grad(const Gdr<__nv_bfloat16>& a, const GdrKept& kept, cudaStream_t stream);
// Redoes every unit of which a flag is set (first: `per` flags a unit, second: `chunks`) by the fp32 walks, `slots` at a time.
size_t gdr_repair_slot_bytes(int L, int dk, int dv);
cudaError_t launch_gdr_repair(const Gdr<__nv_bfloat16>& a, const int* first, int per, const int* second, int chunks, void* scratch, int slots, cudaStream_t stream);
cudaError_t launch_gdr_repair_fwd(const Gdr<__nv_bfloat16>& a, const int* flags, int per, cudaStream_t stream);

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
