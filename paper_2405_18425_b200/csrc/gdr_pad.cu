// Rows laid out again: bf16 calls of the gated delta rule whose head sizes are no multiples of eight get copies of their rows with zeros up to the next
// one, so that the kernels' loads stay whole pieces of sixteen bytes (unaligned loads inside them cost calls of every size 5 to 10 %), and the
// results come back the same way.  A few percent of such a call.
#include "gdr.h"
#include "ptx.cuh"

namespace vig {
namespace {

struct Copies {
    RowCopy c[kRowCopies];
};

// A thread eight values of the wider side's row; grid (blocks, copies).
__global__ void __launch_bounds__(256) copy_rows_kernel(Copies all, long long rows) {
    pdl_wait();
    pdl_launch_dependents();
    const RowCopy c = all.c[blockIdx.y];
    const unsigned short* const src = (const unsigned short*)c.src;
    unsigned short* const dst = (unsigned short*)c.dst;
    const int pieces = (max(c.from, c.to) + 7) / 8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (long long)gridDim.x * 256) {
        const long long r = i / pieces;
        const int e = (int)(i - r * pieces) * 8;
        unsigned short x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = e + k < c.from ? src[r * c.from + e + k] : (unsigned short)0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (e + k < c.to) dst[r * c.to + e + k] = x[k];
    }
}

}  // namespace

cudaError_t launch_copy_rows(const RowCopy* copies, int n, long long rows, cudaStream_t stream) {
    Copies all = {};
    int widest = 0;
    for (int i = 0; i < n; ++i) {
        all.c[i] = copies[i];
        widest = max(widest, max(copies[i].from, copies[i].to));
    }
    const long long blocks = (rows * ((widest + 7) / 8) + 255) / 256;
    count_launch();
    return launch_pdl(copy_rows_kernel, dim3((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8), n), dim3(256), 0, stream, all, rows);
}

}  // namespace vig
