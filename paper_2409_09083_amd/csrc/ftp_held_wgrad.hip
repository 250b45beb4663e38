// Weight gradient of a linear layer whose input is held in 8 bits: dW[n][k] = sum over rows r of dy[r][n] * q[r][k] * 2^e.
// A held value is exact as a bfloat, so the product runs on the bfloat matrix cores (32x32x16, fp32 sums) without rounding it; fp32 dy goes in as
// three bfloats whose sum it is (three products, about the fp32 instruction's accuracy at five times its rate).
//
// A workgroup is a 128 x 128 block of dW and a share of the rows: 4 wavefronts of 64 x 64.  The contraction runs down the slow axis of both operands, so both are staged in LDS as they
// lie (dy after its split, codes after their conversion) and read through the transposing LDS load: 4 rows x 16 columns a 16 lanes.  A stage is 32 rows, two stages in LDS,
// the next one's loads in flight during the products.  The shares' blocks are added up by a second kernel in a fixed order.
#include "ftp_tokens.h"

#include <algorithm>

namespace ftp {
namespace {

typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct HeldWgradArgs {
    const void* dy; const int8_t* codes; const int8_t* exps; float* dw; float* partial;
    long long rows, dy_stride;
    int N, K, nblocks, lgblock, shares, ntiles, ktiles, vec_dy, vec_codes;
};

constexpr int kStage = 32;                          // rows of a stage
constexpr int kBlk = 128;                           // columns of either operand a workgroup takes

// Byte offset of 8 columns (chunk) of a row of a [row][128] bfloat tile.  The chunk is exchanged so that 4 consecutive rows' equal chunks lie in different quarters of the
// 64 banks (a transposing load reads 4 rows x 64 bytes a half wavefront).
__device__ __forceinline__ int tile_at(int row, int chunk) { return row * 256 + ((chunk ^ (((row & 3) << 2) | ((row >> 2) & 3))) << 4); }

// Operand of 32 columns x 16 rows: lane (column, half h) gets rows 8 h .. 8 h + 7.
__device__ __forceinline__ b16x8 read_t(const char* tile, int row0, int col0)
{
    const int l = threadIdx.x & 63, h = l >> 5, g = (l >> 4) & 1, i = l & 15;
    s16x4 v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = row0 + 8 * h + 4 * j + (i >> 2), col = col0 + 16 * g + (i & 3) * 4;
        v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(tile + tile_at(row, col >> 3) + (col & 7) * 2));
    }
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(b16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

template <typename T>
__global__ __launch_bounds__(256) void k_held_wgrad(const HeldWgradArgs a)
{
    constexpr int P = sizeof(T) == 4 ? 3 : 1;       // bfloats of a dy
    constexpr int kTile = kStage * 256;
    __shared__ __align__(16) char lds[2][(P + 1) * kTile];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int tile = blockIdx.x % (a.ntiles * a.ktiles), share = blockIdx.x / (a.ntiles * a.ktiles);
    const int n0 = (tile % a.ntiles) * kBlk, k0 = (tile / a.ntiles) * kBlk;
    // a share is whole stages
    const long long stages = (a.rows + kStage - 1) / kStage;
    const long long lo = stages * share / a.shares, hi = stages * (share + 1) / a.shares;
    const int wn = (wave & 1) * 64, wk = (wave >> 1) * 64;

    // this thread's part of a stage: of dy 8 columns of rows tid / 16 and tid / 16 + 16, of the codes 16 columns of row tid / 8
    const int drow = tid >> 4, dcol = (tid & 15) * 8, crow = tid >> 3, ccol = (tid & 7) * 16;
    float d[2][8];
    uint32_t c[4];
    float unit = 0;
    const auto fetch = [&](long long stage) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const long long r = stage * kStage + drow + 16 * i;
            const T* p = (const T*)a.dy + r * a.dy_stride + n0 + dcol;
            const int n = r < a.rows ? a.N - n0 - dcol : 0;
            if (a.vec_dy && n >= 8) {
                Pack<T, 8> w;
                w.load(p);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] = w.get(j);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] = j < n ? ld(p + j) : 0.0f;
            }
        }
        const long long r = stage * kStage + crow;
        const int n = r < a.rows ? a.K - k0 - ccol : 0;
        const int8_t* p = a.codes + r * a.K + k0 + ccol;
        if (a.vec_codes && n >= 16) {
            const uint4 w = *(const uint4*)p;
            c[0] = w.x; c[1] = w.y; c[2] = w.z; c[3] = w.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) if (4 * j + b < n) c[j] |= (uint32_t)(uint8_t)p[4 * j + b] << (8 * b);
            }
        }
        unit = n > 0 ? held_scale(a.exps[r * a.nblocks + ((k0 + ccol) >> a.lgblock)]) : 0.0f;
    };
    const auto put = [&](char* t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint4 w[P];
            uint32_t* q = (uint32_t*)w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (P == 1) q[j] = pack_bf16(d[i][2 * j], d[i][2 * j + 1]);
                else split3(d[i][2 * j] * kSplitScale, d[i][2 * j + 1] * kSplitScale, q[j], q[4 + j], q[8 + j]);
            }
#pragma unroll
            for (int s = 0; s < P; ++s) *(uint4*)(t + s * kTile + tile_at(drow + 16 * i, dcol >> 3)) = w[s];
        }
        uint4 w[2];
        uint32_t* q = (uint32_t*)w;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int word = (int)c[j >> 1], sh = (j & 1) * 16;
            q[j] = pack_bf16((float)(int8_t)(word >> sh) * unit, (float)(int8_t)(word >> (sh + 8)) * unit);
        }
        *(uint4*)(t + P * kTile + tile_at(crow, ccol >> 3)) = w[0];
        *(uint4*)(t + P * kTile + tile_at(crow, (ccol >> 3) + 1)) = w[1];
    };

    f32x16 acc[2][2] = {};
    if (lo < hi) {
        fetch(lo);
        put(lds[0]);
        __syncthreads();
        for (long long s = lo; s < hi; ++s) {
            const char* t = lds[(s - lo) & 1];
            if (s + 1 < hi) fetch(s + 1);
#pragma unroll
            for (int r0 = 0; r0 < kStage; r0 += 16) {
                b16x8 b[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) b[j] = read_t(t + P * kTile, r0, wk + 32 * j);
#pragma unroll
                for (int p = P - 1; p >= 0; --p)     // smallest first
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const b16x8 x = read_t(t + p * kTile, r0, wn + 32 * i);
#pragma unroll
                        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, b[j], acc[i][j], 0, 0, 0);
                    }
            }
            if (s + 1 < hi) put(lds[(s + 1 - lo) & 1]);
            __syncthreads();
        }
    }
    // lane: column k = lane % 32 of a 32 x 32 block, rows n = 8 (r / 4) + 4 (lane / 32) + r % 4
    const int l = tid & 63;
    float* out = a.shares == 1 ? a.dw : a.partial + (long long)share * a.N * a.K;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int k = k0 + wk + 32 * j + (l & 31);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = n0 + wn + 32 * i + 8 * (r >> 2) + 4 * (l >> 5) + (r & 3);
                if (n < a.N && k < a.K) out[(long long)n * a.K + k] = P == 3 ? acc[i][j][r] * (1.0f / kSplitScale) : acc[i][j][r];
            }
        }
}

__global__ __launch_bounds__(256) void k_held_wgrad_sum(const float* partial, float* dw, long long n, int shares)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = 0;
#pragma unroll 8
    for (int k = 0; k < shares; ++k) s += partial[k * n + i];
    dw[i] = s;
}

// Shares of the rows: as many as give every CU a workgroup, of at least 8 stages.
int wgrad_shares(long long rows, int n, int k)
{
    const long long tiles = ceil_div(n, kBlk) * ceil_div(k, kBlk);
    return (int)std::max(1ll, std::min<long long>(ceil_div(256, tiles), rows / (8 * kStage)));
}

}  // namespace

size_t held_wgrad_workspace(const ftp_checkpoint_shape& s, int outputs)
{
    const int shares = wgrad_shares(s.rows, outputs, (int)s.cols);
    return shares > 1 ? (size_t)shares * outputs * s.cols * sizeof(float) : 0;
}

void held_wgrad(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exponents, const void* dy, long long dy_stride, int outputs, float* dw,
                float* partial, hipStream_t st)
{
    HeldWgradArgs a = {};
    a.dy = dy; a.codes = codes; a.exps = exponents; a.dw = dw; a.partial = partial;
    a.rows = s.rows; a.dy_stride = dy_stride; a.N = outputs; a.K = (int)s.cols;
    a.nblocks = (int)ceil_div(s.cols, s.block);
    while ((1 << a.lgblock) < s.block) ++a.lgblock;
    a.shares = wgrad_shares(s.rows, a.N, a.K);
    a.ntiles = (int)ceil_div(a.N, kBlk); a.ktiles = (int)ceil_div(a.K, kBlk);
    const bool bf = s.dtype == FTP_BF16;
    a.vec_dy = aligned(dy, 16) && dy_stride % (bf ? 8 : 4) == 0;
    a.vec_codes = aligned(codes, 16) && s.cols % 16 == 0;
    const unsigned grid = (unsigned)(a.ntiles * a.ktiles * a.shares);
    if (bf) k_held_wgrad<bf16_t><<<grid, 256, 0, st>>>(a);
    else k_held_wgrad<float><<<grid, 256, 0, st>>>(a);
    if (a.shares > 1) k_held_wgrad_sum<<<(unsigned)ceil_div((long long)a.N * a.K, 256), 256, 0, st>>>(partial, dw, (long long)a.N * a.K, a.shares);
}

}  // namespace ftp
