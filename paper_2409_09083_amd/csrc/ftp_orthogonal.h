// What the kernels of orthogonal updates share.
#pragma once
#include "ftp_training.h"
#include "ftp_product.h"

namespace ftp {

// Most blocks of 64 columns that one workgroup takes through all steps (fp32, so and with a launch a step: 60 x 50 20, 43 us; 64 x 128 29, 46; 64 x 256 48.6, 48.9; 8 x 256 x 50 42, 61; as three products a step 1 x 64 x 64 76, 1024 x 64 x 256
// 548 where it takes 272).
constexpr int kWhole = 4;
// Matrices of ftp_orthogonal_small.hip: the smaller side is at most 64, and the other one gives at most kWhole blocks, or a launch a step is faster than three products, which go over all CUs and add up S by themselves: where the blocks of all
// matrices are few, and where they are many with a long side, whose X is read once a step and not twice.  Launch a step and three products, us of 5 steps, fp32 | bfloats:
//   blocks                   1 x 64 x 576   9: 57, 96 | 51, 79      16 x 64 x 320    80: 79, 102 | 72, 77   2 x 64 x 3000   94: 101, 111 | 89, 92    1 x 64 x 6144   96: 119, 119 | 103, 94
//   8 x 64 x 2048  256: 153, 122 | 143, 98   64 x 64 x 576 576: 204, 159 | 171, 121  2 x 64 x 32768 1024: 458, 307 | 362, 210  64 x 64 x 2048 2048: 547, 288 | 399, 205  128 x 64 x 2048 4096: 1010, 566 | 689, 369
//   16 x 64 x 12000 3008: 401, 430 | 298, 300  6 x 64 x 32768 3072: 507, 505 | 412, 333  8 x 64 x 32768 4096: 530, 672 | 429, 401  16 x 64 x 32768 8192: 939, 1210 | 557, 707  64 x 64 x 8192 8192: 1073, 1127 | 691, 664
inline bool orthogonal_is_small(const ftp_orthogonal_shape& s)
{
    const long long shorter = s.rows < s.cols ? s.rows : s.cols, longer = s.rows < s.cols ? s.cols : s.rows, blocks = ceil_div(longer, 64), all = blocks * s.count;
    return shorter <= 64 && (blocks <= kWhole || all <= 96 || (all >= 4096 && longer >= 12000));
}
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
