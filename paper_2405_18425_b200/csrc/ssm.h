// Internal declarations of the selective scan (not part of the C ABI).
#pragma once
#include "layers.h"

namespace vig {

constexpr int kSsmChannels = 64;   // of a block
constexpr int kSsmTile = 16;       // segments are multiples of it, and it of the tokens that a block takes through its element-wise work together
constexpr int kSsmMostN = 32;
// The gradient's blocks of an SM, and how often they keep a channel's states: in front of every kSsmKept-th token.  A block keeps its segment's.
constexpr int ssm_grad_blocks(int padded) { return padded == 32 ? 2 : 4; }
constexpr int kSsmKept = 4;

// A call of the selective scan.  Row t in walking order is token t, or L - 1 - t in a reverse call.  Null pointers: D, z, bias, the states,
// dD, dz, dbias where the caller has none; what the call does not read or write.
template <typename T>
struct Ssm {
    const T *x, *dt, *z, *Bt, *Ct, *d_out;
    const float *A, *D, *bias, *state_in, *d_state_out;
    T *out, *dx, *ddt, *dz, *dB, *dC;
    float *dA, *dD, *dbias, *state_out, *d_state_in;
    long long ldx, lddt, ldz, ldo, ldB, ldC, lddx, ldddt, lddz, lddB, lddC;   // values from row to row (ldo: of out or d_out)
    int B, L, C, G, N, per;   // per: channels of a group
    bool softplus, reverse;
    int blocks;               // of a group's channels
    // Segments of `seg` tokens (a multiple of the tile) that run side by side.  Scratch where there is more than one, all
    // [B][segs][C][states padded to the lanes']: what a segment adds to the state behind it, afterwards the state in front of it; the
    // same of the adjoint, from behind; [B][segs][C]: the sum of a segment's step sizes.
    int seg, segs;
    float *ends, *adjoint, *total;
    // the gradient's: states of every few tokens of the blocks that run, sums over a block's channels [blocks][B L][G][2][padded N],
    // sums over a segment's tokens [B segs][C padded N], [B segs][2][C]
    float *kept, *part_bc, *part_a, *part_c;
    long long items;
    __host__ __device__ long long row(int b, int t) const { return (long long)b * L + (reverse ? L - 1 - t : t); }
};

inline int ssm_padded(int N) { return N <= 8 ? 8 : N <= 16 ? 16 : 32; }   // four lanes of 2, 4 or 8 states

template <typename T>
void ssm_segments(Ssm<T>& a, bool gradient);             // sets seg and segs
size_t ssm_segment_floats(int B, int C, int N, int segs);   // of ends (and of adjoint)
template <typename T>
cudaError_t launch_ssm_fwd(const Ssm<T>& a, cudaStream_t stream);
// Fills ends and total (and adjoint) and turns them into states; the gradient's first launches.
template <typename T>
cudaError_t launch_ssm_segments(const Ssm<T>& a, bool gradient, cudaStream_t stream);
template <typename T>
size_t ssm_grad_scratch(Ssm<T>& a, char* base);   // bytes; sets the pointers where base is given
template <typename T>
cudaError_t launch_ssm_bwd(const Ssm<T>& a, cudaStream_t stream);
template <typename T>
cudaError_t launch_ssm_step(const Ssm<T>& a, float* state, cudaStream_t stream);

}  // namespace vig
