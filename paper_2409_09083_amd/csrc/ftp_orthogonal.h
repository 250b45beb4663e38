// What the kernels of orthogonal updates share.
#pragma once
#include "ftp_training.h"
#include "ftp_product.h"

namespace ftp {

// Matrices whose smaller side is at most 64: a launch a step (ftp_orthogonal_small.hip).
inline bool orthogonal_is_small(const ftp_orthogonal_shape& s) { return (s.rows < s.cols ? s.rows : s.cols) <= 64; }
size_t orthogonal_small_workspace(const ftp_orthogonal_shape& s, Parts& t);
bool orthogonal_small_sums(const ftp_orthogonal_shape& s);          // whether it wants the sums
// sums: `parts` parts of each matrix' sum of squares; t: the scratch behind them
void orthogonal_small(const ftp_orthogonal_shape& s, const void* x, void* out, const double* sums, int parts, Parts& t, hipStream_t st);

// 1 / (|x| + eps) of a matrix, for a whole workgroup
__device__ __forceinline__ double inverse_norm(const double* sums, int parts, double eps)
{
    __shared__ double lds[4];
    double s = 0;
    for (int i = threadIdx.x; i < parts; i += 256) s += sums[i];
#pragma unroll
    for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    return 1.0 / (sqrt(lds[0] + lds[1] + lds[2] + lds[3]) + eps);
}

}  // namespace ftp
