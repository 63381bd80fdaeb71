// Internal declarations of the RMS norm, the causal convolution and the selective scan (not part of the C ABI).
#pragma once
#include "vig_internal.h"

namespace vig {

// ---- sums over the rows of `part` [rows][columns] in a fixed order, to two results side by side: `first` columns to a, the rest to b (either
// may be null) ----
template <typename T>
struct ColumnSums {
    const float* part;
    long long rows;
    int columns, first;
    T *a, *b;
};
template <typename T>
cudaError_t launch_column_sums(const ColumnSums<T>& a, cudaStream_t stream);

// ---- RMS norm ----
constexpr int kRmsMostC = 16384;
template <typename T>
struct RmsNorm {
    const T *x, *residual, *weight;   // residual, sum_out, rstd: null where there is none
    T *out, *sum_out;
    float *rstd, *scales;
    unsigned char* q;
    long long rows;
    int C;
    float eps, inv_C;
};
template <typename T>
struct RmsNormGrad {
    const T *sum, *weight, *d_out, *d_sum;
    const float* rstd;
    T* dx;
    float* part;   // [blocks][C], null: no gradient of the weight
    long long rows;
    int C;
    float inv_C;
};
template <typename T>
cudaError_t launch_rms_norm(const RmsNorm<T>& a, int out, cudaStream_t stream);   // out: 0 T, 1 e4m3 by rows, 2 e4m3 by 128 values
template <typename T>
int rms_norm_bwd_blocks(long long rows, int C);
template <typename T>
cudaError_t launch_rms_norm_bwd(const RmsNormGrad<T>& a, T* dweight, cudaStream_t stream);

// ---- causal convolution along the tokens.  Row t in walking order is token t, or L - 1 - t in a reverse call ----
template <typename T>
struct Conv {
    const T *x, *w, *bias, *state_in, *d_out, *d_state_out;   // null where there is none: bias, the states
    T *out, *state_out, *dx, *d_state_in;
    float* part;   // [B pieces][C K + C]
    long long ldx, ldo, lddx;   // values from row to row of x, of out or d_out, and of dx
    int B, L, C;
    bool reverse;
    int piece, pieces;   // tokens a thread walks over, and how many pieces a sequence has
    __host__ __device__ long long row(int b, int t) const { return (long long)b * L + (reverse ? L - 1 - t : t); }
};
template <typename T>
void conv_pieces(Conv<T>& a, bool gradient);
template <typename T>
cudaError_t launch_conv(const Conv<T>& a, int K, int act, cudaStream_t stream);
template <typename T>
cudaError_t launch_conv_bwd(const Conv<T>& a, int K, int act, T* dw, T* dbias, cudaStream_t stream);
template <typename T>
cudaError_t launch_conv_step(const Conv<T>& a, int K, int act, T* state, cudaStream_t stream);

}  // namespace vig
