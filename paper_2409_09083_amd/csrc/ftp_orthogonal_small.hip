// Newton-Schulz steps of matrices with a side of at most 64, one launch a step or one for all: a chain of latencies, not of work (which ones: ftp_orthogonal.h).
//
// X lies as m x L, m <= 64 (a tall matrix transposed), in blocks of 64 columns that belong to one workgroup from step to step.  A step's workgroup adds up the parts of S = X X^T that the workgroups of the step before left, makes
// a I + b S + c S^2 of it in LDS (each for itself: 24 matrix instructions a wavefront), multiplies its blocks with that, and takes their part of the next S from the result while it is in LDS.
// 64 x 576, fp32, 5 steps: 134 us as three products a step, 56 so.  Up to 4 blocks stay in one workgroup's LDS, all steps in one launch.
#include "ftp_orthogonal.h"

#include <algorithm>

namespace ftp {
namespace {

constexpr int kSide = 64, kTile = kSide * kSide * 2;           // bytes of a plane of 64 x 64

// 16 bytes (8 columns: chunk) of a row: neither 16 rows of one chunk nor the transposing load's 4 rows x 64 bytes meet on the banks.
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * (kSide * 2) + ((chunk ^ (((row & 2) << 1) | ((row >> 2) & 3))) << 4); }
// operand (index i0 + lane % 32: a row; contraction 16 s + 8 h + j: columns)
__device__ __forceinline__ b16x8 rows_operand(const char* t, int i0, int s)
{
    const int l = threadIdx.x & 63;
    return *(const b16x8*)(t + chunk_at(i0 + (l & 31), 2 * s + (l >> 5)));
}
// operand (index i0 + lane % 32: a column; contraction 16 s + 8 h + j: rows)
__device__ __forceinline__ b16x8 columns_operand(const char* t, int i0, int s)
{
    const int l = threadIdx.x & 63, h = l >> 5, i = l & 15, col = i0 + (l & 16) + (i & 3) * 4;
    s16x4 v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
        v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(t + chunk_at(16 * s + 8 * h + 4 * j + (i >> 2), col >> 3) + (col & 7) * 2));
    return __builtin_bit_cast(b16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

// The products of planes: those of one size have a sum of their own, so that an instruction need not wait for the one before, added up smallest first.
template <int P, class A, class B>
__device__ __forceinline__ f32x16 product(f32x16 acc, A a, B b)
{
    f32x16 sums[P] = {};
    sums[0] = acc;
#pragma unroll
    for (int s = 0; s < kSide / 16; ++s) {
        b16x8 x[P], y[P];
#pragma unroll
        for (int p = 0; p < P; ++p) { x[p] = a(p, s); y[p] = b(p, s); }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int n = P - 1; n >= p; --n) sums[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[n - p], y[p], sums[n], 0, 0, 0);
    }
#pragma unroll
    for (int n = P - 1; n > 0; --n) sums[n - 1] += sums[n];
    return sums[0];
}

struct SmallArgs {
    const void* x; void* out; const double* sums;
    bf16_t* planes;                                 // [matrix][block][plane][64 x 64, as it lies in LDS]
    const float* from; float* to;                   // parts of S: [matrix][workgroup][4][256 threads] of 4
    long long mstride, rstride;
    int m, len, tall, parts, groups, per, blocks;   // groups: workgroups of a matrix, each `per` blocks
    float a, b, c; double eps;
    int last;
};

// Four neighbouring results as planes of a tile: row b, columns a .. a + 3
template <int P>
__device__ __forceinline__ void put4(char* t, int row, int col, float v0, float v1, float v2, float v3)
{
    uint32_t x[P], y[P];
    planes_of<P>(v0, v1, x);
    planes_of<P>(v2, v3, y);
#pragma unroll
    for (int p = 0; p < P; ++p) *(uint2*)(t + p * kTile + chunk_at(row, col >> 3) + (col & 7) * 2) = uint2{x[p], y[p]};
}

// x / (|x| + eps) in planes, and the first parts of S.
template <typename T, int P>
__global__ __launch_bounds__(256) void k_small_start(const SmallArgs a)
{
    __shared__ __align__(16) char t[P * kTile];
    const int matrix = blockIdx.x / a.groups, group = blockIdx.x - matrix * a.groups, tid = threadIdx.x;
    const double inv = inverse_norm(a.sums + (long long)matrix * a.parts, a.parts, a.eps);
    const int wave = tid >> 6, a0 = 32 * (wave & 1), b0 = 32 * (wave >> 1);
    const T* x = (const T*)a.x + matrix * a.mstride;
    f32x16 acc = {};
    for (int block = group * a.per; block < min((group + 1) * a.per, a.blocks); ++block) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            // neighbours in memory on neighbouring lanes, whichever way x lies
            const int e = tid + 256 * k, r = a.tall ? e & 63 : e >> 6, l = a.tall ? e >> 6 : e & 63, at = block * kSide + l;
            float v = 0;
            if (r < a.m && at < a.len) v = (float)(ld(x + (a.tall ? at * a.rstride + r : r * a.rstride + at)) * inv);
            uint32_t q[P];
            planes_of<P>(v, 0.0f, q);
#pragma unroll
            for (int p = 0; p < P; ++p) *(bf16_t*)(t + p * kTile + chunk_at(r, l >> 3) + (l & 7) * 2) = (bf16_t)q[p];
        }
        __syncthreads();
        acc = product<P>(acc, [&](int p, int s) { return rows_operand(t + p * kTile, a0, s); }, [&](int p, int s) { return rows_operand(t + p * kTile, b0, s); });
        uint4* to = (uint4*)(a.planes + ((long long)matrix * a.blocks + block) * (P * kTile / 2));
        for (int u = tid; u < P * kTile / 16; u += 256) to[u] = ((const uint4*)t)[u];
    }
    f32x4* to = (f32x4*)a.to + (long long)blockIdx.x * 1024 + tid;
#pragma unroll
    for (int q = 0; q < 4; ++q) to[256 * q] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
}

template <typename T, int P>
__global__ __launch_bounds__(256) void k_small_step(const SmallArgs a)
{
    __shared__ __align__(16) char ts[P * kTile], tq[P * kTile], tx[P * kTile], tn[P * kTile];
    const int matrix = blockIdx.x / a.groups, group = blockIdx.x - matrix * a.groups, tid = threadIdx.x;
    const int wave = tid >> 6, l = tid & 63, h = l >> 5, a0 = 32 * (wave & 1), b0 = 32 * (wave >> 1), row = b0 + (l & 31);
    // registers 4 q .. 4 q + 3 of a result: row `row`, columns a0 + 8 q + 4 h ..
    const bf16_t* planes = a.planes + (long long)matrix * a.blocks * (P * kTile / 2);
    const int first = group * a.per, end = min(first + a.per, a.blocks);
    uint4 ahead[P * 2];                             // the next block of X on its way
    const auto fetch = [&](int block) __attribute__((always_inline)) {
        const uint4* from = (const uint4*)(planes + (long long)block * (P * kTile / 2));
#pragma unroll
        for (int k = 0; k < P * 2; ++k) ahead[k] = from[tid + 256 * k];
    };
    fetch(first);
    f32x16 s = {};
    const f32x4* part = (const f32x4*)a.from + (long long)matrix * a.groups * 1024 + tid;
#pragma unroll 4
    for (int w = 0; w < a.groups; ++w)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = part[w * 1024 + 256 * q];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * q + e] += v[e];
        }
#pragma unroll
    for (int q = 0; q < 4; ++q) put4<P>(ts, row, a0 + 8 * q + 4 * h, s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]);
    __syncthreads();
    f32x16 acc = product<P>(f32x16{}, [&](int p, int k) { return rows_operand(ts + p * kTile, a0, k); }, [&](int p, int k) { return rows_operand(ts + p * kTile, b0, k); });
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = fmaf(a.c, acc[r], a.b * s[r]) + (a0 + 8 * (r >> 2) + 4 * h + (r & 3) == row ? a.a : 0.0f);
#pragma unroll
    for (int q = 0; q < 4; ++q) put4<P>(tq, row, a0 + 8 * q + 4 * h, acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    f32x16 next = {};
    for (int block = first; block < end; ++block) {
        // (tx and tn have had their last readers before the barrier)
#pragma unroll
        for (int k = 0; k < P * 2; ++k) ((uint4*)tx)[tid + 256 * k] = ahead[k];
        __syncthreads();
        if (block + 1 < end) fetch(block + 1);
        f32x16 v = product<P>(f32x16{}, [&](int p, int k) { return columns_operand(tx + p * kTile, a0, k); }, [&](int p, int k) { return rows_operand(tq + p * kTile, b0, k); });
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = a0 + 8 * q + 4 * h;
            if (a.last) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = block * kSide + col + e;
                    if (row < a.m && at < a.len) st((T*)a.out + (long long)matrix * a.m * a.len + (a.tall ? (long long)at * a.m + row : (long long)row * a.len + at), v[4 * q + e]);
                }
            } else put4<P>(tn, row, col, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
        __syncthreads();
        if (a.last) continue;
        next = product<P>(next, [&](int p, int k) { return rows_operand(tn + p * kTile, a0, k); }, [&](int p, int k) { return rows_operand(tn + p * kTile, b0, k); });
        uint4* to = (uint4*)(a.planes + ((long long)matrix * a.blocks + block) * (P * kTile / 2));
#pragma unroll
        for (int k = 0; k < P * 2; ++k) to[tid + 256 * k] = ((const uint4*)tn)[tid + 256 * k];
    }
    if (a.last) return;
    f32x4* to = (f32x4*)a.to + (long long)blockIdx.x * 1024 + tid;
#pragma unroll
    for (int q = 0; q < 4; ++q) to[256 * q] = f32x4{next[4 * q], next[4 * q + 1], next[4 * q + 2], next[4 * q + 3]};
}

// All steps of a matrix of up to NB blocks by one workgroup, X in its LDS: four wavefronts a block.
template <typename T, int P, int NB>
__global__ __launch_bounds__(256 * NB) void k_small_all(const SmallArgs a, int steps)
{
    constexpr int kJoin = (NB - 1) * kSide * kSide * 4, kWork = kJoin > 2 * P * kTile ? kJoin : 2 * P * kTile;
    __shared__ __align__(16) char work[kWork], tx[NB][P * kTile];
    __shared__ double sums[4 * NB];
    char *const ts = work, *const tq = work + P * kTile;
    const int matrix = blockIdx.x, block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255, wave = tid >> 6, l = tid & 63, h = l >> 5, a0 = 32 * (wave & 1),
              b0 = 32 * (wave >> 1), row = b0 + (l & 31);
    const T* x = (const T*)a.x + matrix * a.mstride;
    char* const mine = tx[block];
    // neighbours in memory on neighbouring lanes, whichever way x lies
    float held[16];
    double square = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int e = tid + 256 * k, r = a.tall ? e & 63 : e >> 6, at = block * kSide + (a.tall ? e >> 6 : e & 63);
        held[k] = r < a.m && at < a.len ? (float)ld(x + (a.tall ? at * a.rstride + r : r * a.rstride + at)) : 0.0f;
        square = fma((double)held[k], (double)held[k], square);
    }
#pragma unroll
    for (int k = 32; k; k >>= 1) square += __shfl_xor(square, k);
    if (l == 0) sums[4 * block + wave] = square;
    __syncthreads();
    square = 0;
#pragma unroll
    for (int k = 0; k < 4 * NB; ++k) square += sums[k];
    const double inv = 1.0 / (sqrt(square) + a.eps);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int e = tid + 256 * k, r = a.tall ? e & 63 : e >> 6, c = a.tall ? e >> 6 : e & 63;
        uint32_t q[P];
        planes_of<P>((float)(held[k] * inv), 0.0f, q);
#pragma unroll
        for (int p = 0; p < P; ++p) *(bf16_t*)(mine + p * kTile + chunk_at(r, c >> 3) + (c & 7) * 2) = (bf16_t)q[p];
    }
    const auto put = [&](char* t, const f32x16& v) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) put4<P>(t, row, a0 + 8 * q + 4 * h, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    };
    for (int step = 0; step < steps; ++step) {
        __syncthreads();
        f32x16 s = product<P>(f32x16{}, [&](int p, int k) { return rows_operand(mine + p * kTile, a0, k); }, [&](int p, int k) { return rows_operand(mine + p * kTile, b0, k); });
        if constexpr (NB > 1) {
            // the blocks' parts of S, added up in their order by the first one's wavefronts
            f32x4* part = (f32x4*)work;
            if (block) {
#pragma unroll
                for (int q = 0; q < 4; ++q) part[((block - 1) * 4 + q) * 256 + tid] = f32x4{s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]};
            }
            __syncthreads();
            if (!block) {
#pragma unroll
                for (int n = 0; n < NB - 1; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 v = part[(n * 4 + q) * 256 + tid];
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[4 * q + e] += v[e];
                    }
            }
            __syncthreads();
        }
        if (!block) put(ts, s);
        __syncthreads();
        if (!block) {
            f32x16 q = product<P>(f32x16{}, [&](int p, int k) { return rows_operand(ts + p * kTile, a0, k); }, [&](int p, int k) { return rows_operand(ts + p * kTile, b0, k); });
#pragma unroll
            for (int r = 0; r < 16; ++r) q[r] = fmaf(a.c, q[r], a.b * s[r]) + (a0 + 8 * (r >> 2) + 4 * h + (r & 3) == row ? a.a : 0.0f);
            put(tq, q);
        }
        __syncthreads();
        const f32x16 v = product<P>(f32x16{}, [&](int p, int k) { return columns_operand(mine + p * kTile, a0, k); }, [&](int p, int k) { return rows_operand(tq + p * kTile, b0, k); });
        __syncthreads();
        if (step + 1 < steps) {
            put(mine, v);
            continue;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int at = block * kSide + a0 + 8 * (r >> 2) + 4 * h + (r & 3);
            if (row < a.m && at < a.len) st((T*)a.out + (long long)matrix * a.m * a.len + (a.tall ? (long long)at * a.m + row : (long long)row * a.len + at), v[r]);
        }
    }
}

// Workgroups of a matrix: one a block up to 32, whose parts of S each of them adds up.
void shape_of(const ftp_orthogonal_shape& s, SmallArgs& a)
{
    a.tall = s.rows > s.cols;
    a.m = std::min(s.rows, s.cols);
    a.len = std::max(s.rows, s.cols);
    a.blocks = (int)ceil_div(a.len, kSide);
    a.per = (int)ceil_div(a.blocks, 32);
    a.groups = (int)ceil_div(a.blocks, a.per);
}

template <typename T, int P>
void run(const ftp_orthogonal_shape& s, SmallArgs& a, float* (&parts)[2], hipStream_t st)
{
    if (a.blocks <= kWhole) {
        if (a.blocks == 1) k_small_all<T, P, 1><<<(unsigned)s.count, 256, 0, st>>>(a, s.steps);
        else if (a.blocks == 2) k_small_all<T, P, 2><<<(unsigned)s.count, 512, 0, st>>>(a, s.steps);
        else k_small_all<T, P, kWhole><<<(unsigned)s.count, 256 * kWhole, 0, st>>>(a, s.steps);
        return;
    }
    const unsigned grid = (unsigned)(s.count * a.groups);
    a.to = parts[0];
    k_small_start<T, P><<<grid, 256, 0, st>>>(a);
    for (int step = 0; step < s.steps; ++step) {
        a.from = parts[step & 1];
        a.to = parts[~step & 1];
        a.last = step + 1 == s.steps;
        k_small_step<T, P><<<grid, 256, 0, st>>>(a);
    }
}

void take(const ftp_orthogonal_shape& s, const SmallArgs& a, Parts& t, bf16_t*& planes, float* (&parts)[2])
{
    planes = t.take<bf16_t>((size_t)s.count * a.blocks * 3 * kSide * kSide);
    for (auto& p : parts) p = t.take<float>((size_t)s.count * a.groups * kSide * kSide);
}

}  // namespace

bool orthogonal_small_sums(const ftp_orthogonal_shape& s)
{
    SmallArgs a = {};
    shape_of(s, a);
    return a.blocks > kWhole;
}

size_t orthogonal_small_workspace(const ftp_orthogonal_shape& s, Parts& t)
{
    SmallArgs a = {};
    bf16_t* planes;
    float* parts[2];
    shape_of(s, a);
    take(s, a, t, planes, parts);
    return t.used;
}

void orthogonal_small(const ftp_orthogonal_shape& s, const void* x, void* out, const double* sums, int parts, Parts& t, hipStream_t st)
{
    SmallArgs a = {};
    float* p[2];
    shape_of(s, a);
    take(s, a, t, a.planes, p);
    a.x = x; a.out = out; a.sums = sums; a.parts = parts; a.mstride = s.matrix_stride; a.rstride = s.row_stride; a.a = s.a; a.b = s.b; a.c = s.c; a.eps = s.eps;
    if (s.dtype == FTP_BF16) run<bf16_t, 2>(s, a, p, st);
    else run<float, 3>(s, a, p, st);
}

}  // namespace ftp
