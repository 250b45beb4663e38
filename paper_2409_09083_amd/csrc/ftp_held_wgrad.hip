// Weight gradient of a linear layer whose input is held in 8 bits: dW[n][k] = sum over rows r of dy[r][n] * q[r][k] * 2^e.
// A held value is exact as a bfloat, so the product runs on the bfloat matrix cores (32x32x16, fp32 sums) without rounding it; fp32 dy goes in as
// three bfloats whose sum it is (three products, about the fp32 instruction's accuracy at five times its rate).
//
// A workgroup is a 128 x 128 block of dW and a share of the rows: 4 wavefronts of 64 x 64.  The contraction runs down the slow axis of both operands, so both are staged in LDS as they
// lie (dy after its split, codes after their conversion) and read through the transposing LDS load: 4 rows x 16 columns a 16 lanes.  A stage is 64 rows (32 of fp32), two stages in LDS
// and two more on their way in registers: with one, a workgroup waited for HBM most of the time (331 us).  The shares' blocks are added up by a second kernel in a fixed order.
//
// Measured: 46208 rows, 512 -> 1024, bfloats: a pass 86 us among others (48.5 GFLOP, 564 TFLOP/s; a large library product of bfloats reaches 1265), 80 on inputs of the call before; in a trace
// the product 81 and the sum 6.5; fp32 dy 160: matrix cores busy 31 % of the cycles, the codes' conversion and the stores into LDS take the issue slots between them, and 512 workgroups end in one uneven round.  4995 rows, 202 -> 133, fp32: 16.5 us, of which 14 are a workgroup's chain of
// two stages, loads, split, products, store, and the rest the sum of 78 shares.
#include "ftp_tokens.h"
#include "ftp_order.h"

#include <algorithm>
#include <type_traits>

namespace ftp {
namespace {

typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct HeldWgradArgs {
    const void* dy; const int8_t* codes; const int8_t* exps; float* dw; float* partial;
    long long rows, dy_stride;
    int N, K, nblocks, lgblock, shares, ntiles, ktiles, wide;
};

template <typename T> constexpr int kStage = sizeof(T) == 4 ? 32 : 64;       // rows of a stage
constexpr int kBlk = 128;                           // columns of either operand a workgroup takes
// Held values go into the products at a part of their size: 128 * 2^e, which their conversion subtracts, is no finite number at the largest exponents 121 and 122.  (Subtracting
// 128 before the scale needs one instruction a value more: 80 -> 83 us for 46208 rows, 512 -> 1024, bfloats.)  With bfloats a quarter, made good at the end.  fp32 dy is split at
// as many times its size, so that sums are neither larger nor smaller than the result; 2^12 leaves the low bits of numbers down to 2^-122 in their lowest plane (ftp_split.h), and those of held
// values down to 2^-114 (at 2^24, as other kernels split, results above 2^104 would be infinite, or small held values lose as much more).
template <typename T> constexpr float kHeldPart = sizeof(T) == 4 ? 1.0f / 4096.0f : 0.25f;
template <typename T> constexpr float kDyTimes = sizeof(T) == 4 ? 4096.0f : 1.0f;

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
__global__ __launch_bounds__(256, 2) void k_held_wgrad(const HeldWgradArgs a)
{
    constexpr int P = sizeof(T) == 4 ? 3 : 1;       // bfloats of a dy
    constexpr int S = kStage<T>, kTile = S * 256, DR = S / 16, CR = S / 32;
    __shared__ __align__(16) char lds[2][(P + 1) * kTile];
    const int tid = threadIdx.x, wave = tid >> 6;
    // all blocks of a share on one XCD where there are shares for all eight: its L2 serves the rows that they have in common
    int tile, share;
    if (a.shares < 8) {
        share = blockIdx.x / (a.ntiles * a.ktiles);
        tile = blockIdx.x - share * a.ntiles * a.ktiles;
    } else if (!xcd_order((int)blockIdx.x, a.shares, a.ntiles * a.ktiles, share, tile)) return;
    const int n0 = (tile % a.ntiles) * kBlk, k0 = (tile / a.ntiles) * kBlk;
    // a share is whole stages
    const long long stages = (a.rows + S - 1) / S;
    const long long lo = stages * share / a.shares, hi = stages * (share + 1) / a.shares;
    const int wn = (wave & 1) * 64, wk = (wave >> 1) * 64;

    // this thread's part of a stage: of dy 8 columns of rows tid / 16 + 16 i, of the codes 16 columns of rows tid / 8 + 32 i.  Columns past the matrix' edge are
    // read from inside it and not stored; rows past its end are read from its last row and cleared.
    const int drow = tid >> 4, dcol = (tid & 15) * 8, crow = tid >> 3, ccol = (tid & 7) * 16;
    const int dn = n0 + dcol < a.N ? n0 + dcol : 0, cn = k0 + ccol < a.K ? k0 + ccol : 0;
    struct Part { Pack<T, 8> d[DR]; uint4 c[CR]; int e[CR]; };
    const long long last = a.rows - 1;
    const auto fetch_exps = [&](Part& x, long long stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CR; ++i) x.e[i] = a.exps[min(stage * S + crow + 32 * i, last) * a.nblocks + (cn >> a.lgblock)];
    };
    // 8 of dy and 16 codes at once, at any address; past a row's end they come from the next row
    const auto fetch = [&](Part& x, long long stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < DR; ++i) x.d[i].load_any((const T*)a.dy + (stage * S + drow + 16 * i) * a.dy_stride + dn);
#pragma unroll
        for (int i = 0; i < CR; ++i) __builtin_memcpy(&x.c[i], a.codes + (stage * S + crow + 32 * i) * a.K + cn, 16);
        fetch_exps(x, stage);
    };
    // ... one by one, for the last stage, whose last row has no next one, and for rows that are too short
    const auto fetch_each = [&](Part& x, long long stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < DR; ++i) {
            const T* p = (const T*)a.dy + min(stage * S + drow + 16 * i, last) * a.dy_stride;
            T v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[min(dn + j, a.N - 1)];
            __builtin_memcpy(x.d[i].w, v, sizeof(v));
        }
#pragma unroll
        for (int i = 0; i < CR; ++i) {
            const int8_t* p = a.codes + min(stage * S + crow + 32 * i, last) * a.K;
            int8_t v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = p[min(cn + j, a.K - 1)];
            __builtin_memcpy(&x.c[i], v, 16);
        }
        fetch_exps(x, stage);
    };
    // left: rows of the stage that are there
    const auto put = [&](const Part& x, char* t, auto all, int left) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < DR; ++i) {
            const bool there = all || drow + 16 * i < left;
            uint4 w[P];
            uint32_t* q = (uint32_t*)w;
            if constexpr (P == 1) {
                __builtin_memcpy(w, x.d[i].w, 16);
                if (!there) w[0] = uint4{0, 0, 0, 0};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    split3(there ? x.d[i].get(2 * j) * kDyTimes<T> : 0.0f, there ? x.d[i].get(2 * j + 1) * kDyTimes<T> : 0.0f, q[j], q[4 + j], q[8 + j]);
            }
#pragma unroll
            for (int s = 0; s < P; ++s) *(uint4*)(t + s * kTile + tile_at(drow + 16 * i, dcol >> 3)) = w[s];
        }
#pragma unroll
        for (int i = 0; i < CR; ++i) {
            // a part of q * 2^e = (q + 128) * unit - 128 * unit, exact; q + 128 as an unsigned byte takes one conversion from where it lies
            const float unit = all || crow + 32 * i < left ? held_scale(x.e[i]) * kHeldPart<T> : 0.0f, less = -128.0f * unit;
            uint4 w[2];
            uint32_t* q = (uint32_t*)w;
            const uint32_t c[4] = {x.c[i].x ^ 0x80808080u, x.c[i].y ^ 0x80808080u, x.c[i].z ^ 0x80808080u, x.c[i].w ^ 0x80808080u};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t v = c[j >> 1] >> (16 * (j & 1));
                q[j] = pack_bf16(fmaf((float)(v & 0xFFu), unit, less), fmaf((float)((v >> 8) & 0xFFu), unit, less));
            }
            *(uint4*)(t + P * kTile + tile_at(crow + 32 * i, ccol >> 3)) = w[0];
            *(uint4*)(t + P * kTile + tile_at(crow + 32 * i, (ccol >> 3) + 1)) = w[1];
        }
    };

    f32x16 acc[2][2] = {};
    const auto products = [&](const char* now) __attribute__((always_inline)) {
#pragma unroll
        for (int r0 = 0; r0 < S; r0 += 16) {
            b16x8 b[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) b[j] = read_t(now + P * kTile, r0, wk + 32 * j);
#pragma unroll
            for (int p = P - 1; p >= 0; --p)         // smallest first
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const b16x8 x = read_t(now + p * kTile, r0, wn + 32 * i);
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, b[j], acc[i][j], 0, 0, 0);
                }
        }
    };
    const long long full = a.wide ? min(hi, stages - 1) : lo;          // stages below this one go the fast way
    // stage s is in LDS, `next` holds stage s + 1 and takes stage s + 3 once that is in LDS; stage s + 2 is on its way beside it
    const auto step = [&](long long s, const char* now, char* then, Part& next) __attribute__((always_inline)) {
        products(now);
        if (s + 1 < full) put(next, then, std::true_type{}, S);
        if (s + 3 < full) fetch(next, s + 3);
        __syncthreads();
    };
    if (lo < full) {
        Part x, y;
        fetch(x, lo);
        if (lo + 1 < full) fetch(y, lo + 1);
        put(x, lds[0], std::true_type{}, S);
        if (lo + 2 < full) fetch(x, lo + 2);
        __syncthreads();
        for (long long s = lo; s < full; s += 2) {
            step(s, lds[0], lds[1], y);
            if (s + 1 < full) step(s + 1, lds[1], lds[0], x);
        }
    }
    for (long long s = max(lo, full); s < hi; ++s) {
        Part x;
        fetch_each(x, s);
        put(x, lds[0], std::false_type{}, (int)min((long long)S, a.rows - s * S));
        __syncthreads();
        products(lds[0]);
        __syncthreads();
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
                if (n < a.N && k < a.K) out[(long long)n * a.K + k] = acc[i][j][r] * (1.0f / (kDyTimes<T> * kHeldPart<T>));
            }
        }
}

// The shares' sum: 64 elements x 4 groups of shares a workgroup.
__global__ __launch_bounds__(256) void k_held_wgrad_sum(const float* partial, float* dw, long long n, int shares)
{
    __shared__ float lds[4][64];
    const int e = threadIdx.x & 63, grp = threadIdx.x >> 6;
    const long long i = (long long)blockIdx.x * 64 + e;
    float s = 0;
    if (i < n) {
#pragma unroll 8
        for (int k = grp; k < shares; k += 4) s += partial[k * n + i];
    }
    lds[grp][e] = s;
    __syncthreads();
    if (grp == 0 && i < n) dw[i] = (lds[0][e] + lds[1][e]) + (lds[2][e] + lds[3][e]);
}

// Shares of the rows: two workgroups a CU, of at least two stages.
int wgrad_shares(long long rows, int n, int k, int stage)
{
    const long long tiles = ceil_div(n, kBlk) * ceil_div(k, kBlk);
    return (int)std::max(1ll, std::min<long long>(ceil_div(512, tiles), rows / (2 * stage)));
}
int stage_of(const ftp_checkpoint_shape& s) { return s.dtype == FTP_BF16 ? kStage<bf16_t> : kStage<float>; }

}  // namespace

size_t held_wgrad_workspace(const ftp_checkpoint_shape& s, int outputs)
{
    const int shares = wgrad_shares(s.rows, outputs, (int)s.cols, stage_of(s));
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
    a.shares = wgrad_shares(s.rows, a.N, a.K, stage_of(s));
    a.ntiles = (int)ceil_div(a.N, kBlk); a.ktiles = (int)ceil_div(a.K, kBlk);
    const bool bf = s.dtype == FTP_BF16;
    a.wide = dy_stride >= 8 && a.K >= 16;
    const unsigned grid = a.shares < 8 ? (unsigned)(a.ntiles * a.ktiles * a.shares) : xcd_grid(a.shares, a.ntiles * a.ktiles);
    if (bf) k_held_wgrad<bf16_t><<<grid, 256, 0, st>>>(a);
    else k_held_wgrad<float><<<grid, 256, 0, st>>>(a);
    if (a.shares > 1) k_held_wgrad_sum<<<(unsigned)ceil_div((long long)a.N * a.K, 64), 256, 0, st>>>(partial, dw, (long long)a.N * a.K, a.shares);
}

}  // namespace ftp
