// Softmax cross entropy over a vocabulary, from the inputs x and the weight W of the linear layer that makes the logits s = scale W x:
//   loss = log sum_v exp(s_v) - s_label,   G = dloss scale (exp(s - log sum) - [v = label]),   dx = G W,   dW = G^T x.
// No logit is kept.  Forward, a block of logits leaves its registers as one maximum and one sum of powers a row; backward, the logits are computed again and leave as G, rounded to the operands of the
// two products behind it (two bfloats, or three), for a piece of the vocabulary at a time.
//
// Rows without a label have no part in any of it: the others are gathered first (their number stays on the device), so that what the rows left out hold, NaN included, reaches nothing, and costs nothing.
//
// Measured: forward, bfloats, 11552 rows on 16384 x 512 193 us (logits 176: 1.10 PFLOP/s), 4 rows on 32768 x 512 12 (the weight read at 3.8 TB/s); backward, 11552 rows on 32768 x 1024 3.31 to 3.41 ms in three runs (logits 895,
// and with G in two bfloats dx 1346, dweight 1165: 0.87, 1.15 and 1.33 PFLOP/s), fp32, 2997 labelled rows of 4995 on 10007 x 202 369 us.
#include "ftp_training.h"
#include "ftp_product.h"

#include <algorithm>
#include <cmath>

namespace ftp {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Most rows whose labels every workgroup counts by itself, a launch less (forward on 512 x 64, itself and with the launch: 577 rows 14.4, 16.1 us; 2048 15.7, 16.6; 4096 17.6, 17.1; 8192 21.9, 18.8).
constexpr int kCountRows = 4096;
constexpr int kChunk = 64;                          // rows whose labels one wavefront looks at
// From so many rows on W is laid out for the products (forward on 16384 x 512, as it lies and laid out: 577 rows 30, 34 us; 2048 53, 54; 4096 90, 86; 11552 215, 200).
constexpr int kPackRows = 4096;
// Bfloats of G where the tensors are one, at any number of rows.  G's rows add up to 0, and of a weight that has learned its labels its columns nearly do: a part that the rows of W (of x) share goes out of the sums and leaves G's rounding
// behind.  Weights of 1 + a 64th of a random number in 8 of 64 to 320 channels: dx off by 1.2 to 5 % of its norm with one bfloat, by at most 8e-5 with two before its own rounding (dweight 2e-3, 3e-6).  The price, us with one and with two:
// 2048 rows on 16384 x 512 143, 214; 11552 on 8192 x 256 215, 379, on 32768 x 1024 1954, 3310.
constexpr int kGradPlanes = 2;
// Most rows whose statistics one workgroup joins (forward on 32768 x 512: 16 rows 11.0 us, by several and a launch for their mean 12.5; 32 rows 13.7 and 12.5).
constexpr int kJoin = 16;
// Most rows of the logits whose blocks have 32 of them, with W read at the memory's rate (forward on 32768 x 512, blocks of 128 x 32 and of 128 x 128: 4 rows 10.5, 17.7 us; 33 16.4, 19.4; 64 16.6, 19.8; 128 24.6, 20.2).
constexpr int kFew = 64;

template <bool XA, bool XB> using Big = Product<256, 256, 2, 4, XA, XB>;
typedef Product<256, 128, 2, 2, false, false, 32, 3> Two;         // two workgroups a CU: one's powers beside the other's products
template <bool XA, bool XB> using Mid = Product<128, 128, 2, 2, XA, XB>;
typedef Product<128, 32, 4, 1, false, false, 64> Few;

// ---- the labelled rows ---------------------------------------------------------------------------------------------
// How many of each 64 rows have labels.
__global__ __launch_bounds__(256) void k_labelled(const void* ids, int wide, long long rows, int vocab, int* counts)
{
    const long long chunk = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), row = chunk * kChunk + (threadIdx.x & 63);
    const bool there = row < rows && id_of(ids, wide, row, vocab) >= 0;
    const unsigned long long all = __ballot(there);
    if ((threadIdx.x & 63) == 0 && chunk * kChunk < std::max(rows, 1ll)) counts[chunk] = (int)__popcll(all);
}

// 8 neighbours c0 .. c0 + 7 of a row of C as planes, to where they lie; zeros past its end
template <typename T, int P>
__device__ __forceinline__ void copy8(const T* row, int c0, int C, bf16_t* to, long long plane)
{
    Pack<T, 8> v;
    if (c0 + 8 <= C) v.load_any(row + c0);
    else {
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = c0 + j < C ? row[c0 + j] : (T)0;
        __builtin_memcpy(v.w, e, sizeof(e));
    }
    if constexpr (P == 1) __builtin_memcpy(to, v.w, 16);
    else {
        uint32_t q[4][P];
#pragma unroll
        for (int j = 0; j < 4; ++j) planes_of<P>(v.get(2 * j), v.get(2 * j + 1), q[j]);
#pragma unroll
        for (int p = 0; p < P; ++p) *(uint4*)(to + p * plane) = uint4{q[0][p], q[1][p], q[2][p], q[3][p]};
    }
}

struct PrepareArgs {
    const void* ids; const void* x; const int* counts;         // counts null: of so few rows that each workgroup counts them itself
    bf16_t* xc; int* index; int* label; int* place; int* count;
    long long rows, stride, plane, block;           // of xc: as a Matrix lies
    int wide, vocab, C, Cp;
    int gathering;                                  // the first workgroups, four a chunk; the others lay W out
    const void* w; bf16_t* wc; long long wstride, wplane; int Vp;
};

// W as planes, laid out for the products; zeros up to Vp rows of Cp.  `index` of `groups` workgroups.
template <typename T, int P>
__device__ __forceinline__ void lay_out(const PrepareArgs& a, int index, int groups)
{
    // a wavefront has 16 rows x 32 columns, 1 KB where they go
    const int lane = threadIdx.x & 63, across = a.Cp >> 5, c_in = (lane & 3) * 8;
    const long long tiles = (long long)(a.Vp >> 4) * across;
    for (long long t = (long long)index * 4 + (threadIdx.x >> 6); t < tiles; t += 4ll * groups) {
        const int rb = (int)(t / across), cb = (int)(t - (long long)rb * across), r = rb * 16 + (lane >> 2);
        copy8<T, P>((const T*)a.w + r * a.wstride, r < a.vocab ? cb * 32 + c_in : 0, r < a.vocab ? a.C : 0, a.wc + ((long long)cb * a.Vp + r) * 32 + c_in, a.wplane);
    }
}

// The labelled rows one behind the other: row place[r] of xc is row r of x, index and label say which.  Zeros up to the next multiple of 64 rows.  And W.
template <typename T, int P>
__global__ __launch_bounds__(256) void k_prepare(const PrepareArgs a)
{
    if ((int)blockIdx.x >= a.gathering) {
        lay_out<T, P>(a, blockIdx.x - a.gathering, gridDim.x - a.gathering);
        return;
    }
    __shared__ int sums[2][4];
    __shared__ int where[kChunk];
    const long long chunk = blockIdx.x >> 2, row0 = chunk * kChunk, chunks = a.gathering >> 2;
    const int sub = blockIdx.x & 3;                 // which 16 rows of the chunk this workgroup copies
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int before = 0, all = 0;
    if (a.counts) {
        for (long long i = tid; i < chunks; i += 256) {
            const int n = a.counts[i];
            all += n;
            before += i < chunk ? n : 0;
        }
    } else {
#pragma unroll 4
        for (long long r = tid; r < a.rows; r += 256) {
            const int n = id_of(a.ids, a.wide, r, a.vocab) >= 0;
            all += n;
            before += r < row0 ? n : 0;
        }
    }
#pragma unroll
    for (int n = 32; n; n >>= 1) { before += __shfl_xor(before, n); all += __shfl_xor(all, n); }
    if (lane == 0) { sums[0][wave] = before; sums[1][wave] = all; }
    __syncthreads();
    before = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
    all = sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3];
    if (wave == 0) {
        const long long row = row0 + lane;
        const int id = row < a.rows ? id_of(a.ids, a.wide, row, a.vocab) : -1;
        const unsigned long long there = __ballot(id >= 0);
        const int to = before + (int)__popcll(there & ((1ull << lane) - 1));
        where[lane] = id >= 0 ? to : -1;
        if (row < a.rows && sub == 0) a.place[row] = id >= 0 ? to : -1;
        if (id >= 0 && sub == 0) { a.index[to] = (int)row; a.label[to] = id; }
    }
    __syncthreads();
    // a wavefront has 16 rows x 32 columns, 1 KB where they go
    const int r_in = lane >> 2, c_in = (lane & 3) * 8, across = a.Cp >> 5, end = (all + 63) & ~63;
    const int r = sub * 16 + r_in, to = where[r];
    const T* from = (const T*)a.x + (row0 + r) * a.stride;
    if (to >= 0)
#pragma unroll 4
        for (int cb = wave; cb < across; cb += 4) copy8<T, P>(from, cb * 32 + c_in, a.C, a.xc + cb * a.block + to * 32 + c_in, a.plane);
    if (blockIdx.x) return;
    if (tid == 0) *a.count = all;
    for (int row = all + r_in; row < end; row += 16)
        for (int cb = wave; cb < across; cb += 4)
#pragma unroll
            for (int p = 0; p < P; ++p) *(uint4*)(a.xc + p * a.plane + cb * a.block + row * 32 + c_in) = uint4{0, 0, 0, 0};
}

// ---- logits --------------------------------------------------------------------------------------------------------
struct LogitArgs {
    Matrix w, x;                                    // a piece of the vocabulary, the labelled rows
    const int* count;                               // rows of x (null: all)
    const int* label;                               // of them (null: ids)
    const void* ids;
    Terms terms;
    int wide, stages, vocab, ablocks, bblocks;
    int piece0;                                     // the piece's first id
    float c, factor;                                // products become powers of 2 by c, after the factor: 1, or -1 for a negative scale, smaller where c would be too small a number
    float2* part; float* target;                    // forward: [row][ablocks] maximum and sum of a block's powers of 2; the labels' products
    const int* index; const float* lse; const float* dloss;     // backward
    bf16_t* g; long long gblock, gplane;            // G, as a Matrix lies
};

// What a block of logits leaves: STATS, of each row its maximum m (in powers of 2) and the sum of the others' powers above it, and the label's logit; else PLANES of G.
template <class L, int PLANES, bool STATS>
__global__ __launch_bounds__(L::kThreads, 2) void k_logits(const LogitArgs a)
{
    __shared__ __align__(16) typename L::Stage s0, s1, s2;
    __shared__ float2 red[L::WA][L::BB];
    int ia, ib;
    if (!block_of((int)blockIdx.x, a.ablocks, a.bblocks, ia, ib)) return;
    const int a0 = ia * L::BA, b0 = ib * L::BB, rows = a.count ? *a.count : (int)a.x.rows;
    if (b0 >= rows) return;
    f32x16 acc[L::IA][L::IB] = {};
    if constexpr (L::kStages == 3) L::run(acc, a.w, a.x, a0, b0, 0, a.stages, a.terms, s0, s1, s2);
    else {
        __shared__ __align__(16) typename L::Stage s3;
        L::run(acc, a.w, a.x, a0, b0, 0, a.stages, a.terms, s0, s1, s2, s3);
    }
    const int l = threadIdx.x & 63, h = l >> 5, wa = L::wave_a(), wb = L::wave_b();
    if (a.factor != 1.0f)
        L::all(acc, [&](float& v, int) __attribute__((always_inline)) { v *= a.factor; });
    const int left = (int)a.w.rows - a0 - wa;                      // ids of the piece from this wavefront's first one on
    if (left < 32 * L::IA)                                          // (no power of those past its end)
        L::all(acc, [&](float& v, int at) __attribute__((always_inline)) { v = at + 4 * h < left ? v : -INFINITY; });
#pragma unroll
    for (int j = 0; j < L::IB; ++j) {
        const int row = b0 + wb + 32 * j + (l & 31);
        const bool there = row < rows;
        const int id = !there ? -1 : a.label ? a.label[row] : id_of(a.ids, a.wide, row, a.vocab);
        const int mine = id < 0 ? -1 : id - a.piece0 - a0 - wa - 4 * h;         // the label, counted from this lane's first id
        const bool look = __any(mine >= 0 && mine < 32 * L::IA);    // (a wavefront's rows have few labels in its block: most have none)
        if constexpr (STATS) {
            if (look) {
                float t = 0;
#pragma unroll
                for (int i = 0; i < L::IA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) t = mine == 32 * i + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : t;
                if (mine >= 0 && mine < 32 * L::IA && !(mine & 4)) a.target[row] = t;          // (this lane's ids: the others are the other half's)
            }
            float m = -INFINITY, sum = 0;
#pragma unroll
            for (int i = 0; i < L::IA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
            m = fmaxf(m, __shfl_xor(m, 32)) * a.c;
            const float ref = m == -INFINITY ? 0.0f : m;            // (a block of nothing but -infinity sums up to 0)
#pragma unroll
            for (int i = 0; i < L::IA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], a.c, -ref));
            sum += __shfl_xor(sum, 32);
            if (h == 0) red[wa / (L::IA * 32)][wb + 32 * j + l] = float2{m, sum};
        } else {
            float lse2 = INFINITY, weight = 1.0f;                   // (rows behind the last one have powers of 0)
            if (there) {
                const int from = a.index[row];
                lse2 = a.lse[from] * kLog2e;
                if (a.dloss) weight = a.dloss[from];
            }
#pragma unroll
            for (int i = 0; i < L::IA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], a.c, -lse2));
            if (look)
#pragma unroll
                for (int i = 0; i < L::IA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] -= mine == 32 * i + 8 * (r >> 2) + (r & 3) ? 1.0f : 0.0f;
            if (a.dloss)
#pragma unroll
                for (int i = 0; i < L::IA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] *= weight;
        }
    }
    if constexpr (!STATS) {
        const int all = (rows + 63) & ~63;
        const auto to = [&](int i, int j) __attribute__((always_inline)) { return a.g + ((a0 + i) >> 5) * a.gblock + (b0 + j) * 32ll + (i & 31); };
        L::each(acc, [&](int i, int j, const float (&v)[8]) __attribute__((always_inline)) { if (b0 + j < all) store_planes<PLANES>(to(i, j), a.gplane, v); });
    }
    if constexpr (STATS) {
        __syncthreads();
        for (int b = threadIdx.x; b < L::BB; b += L::kThreads) {
            if (b0 + b >= rows) break;
            float2 v = red[0][b];
#pragma unroll
            for (int w = 1; w < L::WA; ++w) {
                const float2 o = red[w][b];
                const float m = fmaxf(v.x, o.x), ref = m == -INFINITY ? 0.0f : m;
                v = float2{m, v.y * __builtin_amdgcn_exp2f(v.x - ref) + o.y * __builtin_amdgcn_exp2f(o.x - ref)};
            }
            a.part[(long long)(b0 + b) * a.ablocks + ia] = v;
        }
    }
}

// The blocks' statistics joined: a wavefront a row, its lanes' blocks in turn; up to 16 rows by one workgroup of 16, which needs no launch for the mean.  Losses and log-sums of all rows (0 where there is no label), and each workgroup's sum of losses and labelled rows.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_loss_join(const float2* part, const float* target, const int* place, const void* ids, int wide, long long rows, int vocab, int blocks, float c, float* loss,
                                                   float* lse, double* sums, float* mean)
{
    __shared__ double total[WAVES];
    __shared__ int known[WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    double sum = 0;
    int n = 0;
    for (long long row = (long long)blockIdx.x * WAVES + wave; row < rows; row += (long long)WAVES * gridDim.x) {
        const long long at = place ? place[row] : id_of(ids, wide, row, vocab) >= 0 ? row : -1;
        float one = 0, two = 0;
        if (at >= 0) {
            const float2* p = part + at * blocks;
            float m = -INFINITY;
            for (int i = lane; i < blocks; i += 64) m = fmaxf(m, p[i].x);
#pragma unroll
            for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
            const float ref = m == -INFINITY ? 0.0f : m;
            float s = 0;
            for (int i = lane; i < blocks; i += 64) s = fmaf(p[i].y, __builtin_amdgcn_exp2f(p[i].x - ref), s);
#pragma unroll
            for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
            two = fmaf(ref, kLn2, logf(s));
            one = fmaf(fmaf(-target[at], c, ref), kLn2, logf(s));
            sum += one;
            ++n;
        }
        if (lane == 0) {
            if (loss) loss[row] = one;
            if (lse) lse[row] = two;
        }
    }
    if (lane == 0) { total[wave] = sum; known[wave] = n; }
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0;
    n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { sum += total[w]; n += known[w]; }
    if (gridDim.x == 1) { if (mean) *mean = n ? (float)(sum / n) : 0.0f; }
    else if (mean) { sums[2 * blockIdx.x] = sum; sums[2 * blockIdx.x + 1] = n; }
}
__global__ __launch_bounds__(256) void k_loss_mean(const double* sums, int n, float* mean)
{
    __shared__ double t[2][4];
    double a = 0, b = 0;
    for (int i = threadIdx.x; i < n; i += 256) { a += sums[2 * i]; b += sums[2 * i + 1]; }
#pragma unroll
    for (int k = 32; k; k >>= 1) { a += __shfl_xor(a, k); b += __shfl_xor(b, k); }
    if ((threadIdx.x & 63) == 0) { t[0][threadIdx.x >> 6] = a; t[1][threadIdx.x >> 6] = b; }
    __syncthreads();
    if (threadIdx.x) return;
    a = t[0][0] + t[0][1] + t[0][2] + t[0][3];
    b = t[1][0] + t[1][1] + t[1][2] + t[1][3];
    *mean = b > 0 ? (float)(a / b) : 0.0f;
}

// ---- gradients -----------------------------------------------------------------------------------------------------
struct GradArgs {
    Matrix a, b;
    const int* count;
    Terms terms;
    int stages, shares, most, ablocks, bblocks, add;           // dx: shares and blocks for all rows; fewer rows have more shares (dx_shares())
    float* part;                                    // sums: [share][block along b][block along a]
    void* out; long long ostride; int C; float scale; int mean;
    int ids;                                        // dw: of the piece
    const int* place; const int* index; int rows, first, summing;          // dx; first, summing: parts of a launch of the sums
};

// The factor of the products' sums, as a number below 1 and a power of 2: in one float, a small scale's share of the rows lost its low bits.
struct Factor {
    float part; int power;
    __device__ __forceinline__ float operator()(float v) const { return ldexpf(v * part, power); }
};
__device__ __forceinline__ Factor gradient_scale(float scale, int mean, const int* count)
{
    int power;
    const float part = (float)frexp(!mean ? (double)scale : *count ? (double)scale / *count : 0.0, &power);
    return Factor{__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(part))), __builtin_amdgcn_readfirstlane(power)};
}

// Shares of the contraction where `rows` of the rows that the launch is made for have labels: as many as the launch has workgroups (all) for, at most `most`.
__device__ __forceinline__ int dx_blocks(int rows, int block) { return max((rows + block - 1) / block, 1); }
__device__ __forceinline__ int dx_shares(int rows, int block, int all, int most) { return min(all / dx_blocks(rows, block), most); }

// dx's block: channels x rows over the piece's ids, added to what the pieces before left
template <class L>
__global__ __launch_bounds__(L::kThreads, 2) void k_loss_dx(const GradArgs a)
{
    __shared__ __align__(16) typename L::Stage s0, s1, s2, s3;
    int ia, ib;
    const int rows = *a.count, bblocks = dx_blocks(rows, L::BB), shares = dx_shares(rows, L::BB, a.bblocks * a.shares, a.most);
    if (rows == 0 || !block_of((int)blockIdx.x, a.ablocks, bblocks * shares, ia, ib)) return;
    const int share = ib / bblocks, a0 = ia * L::BA, b0 = (ib - share * bblocks) * L::BB;
    f32x16 acc[L::IA][L::IB] = {};
    const int lo = (int)((long long)a.stages * share / shares), hi = (int)((long long)a.stages * (share + 1) / shares);
    L::run(acc, a.a, a.b, a0, b0, lo, hi, a.terms, s0, s1, s2, s3);
    L::put(acc, a.part + ((long long)ib * a.ablocks + ia) * L::kSums, a.add);
}

// dW's block: channels x ids over the labelled rows
template <class L, typename T>
__global__ __launch_bounds__(L::kThreads, 2) void k_loss_dw(const GradArgs a)
{
    __shared__ __align__(16) typename L::Stage s0, s1, s2, s3;
    int ia, ib;
    const int blocks = a.bblocks * a.shares;
    if (!block_of((int)blockIdx.x, a.ablocks, blocks, ia, ib)) return;
    const int share = ib / a.bblocks, a0 = ia * L::BA, b0 = (ib - share * a.bblocks) * L::BB, stages = (*a.count + L::KS - 1) / L::KS;
    f32x16 acc[L::IA][L::IB] = {};
    const int lo = (int)((long long)stages * share / a.shares), hi = (int)((long long)stages * (share + 1) / a.shares);
    L::run(acc, a.a, a.b, a0, b0, lo, hi, a.terms, s0, s1, s2, s3);
    const Factor f = gradient_scale(a.scale, a.mean, a.count);
    if (a.shares > 1) {
        L::put(acc, a.part + ((long long)ib * a.ablocks + ia) * L::kSums, false);
        return;
    }
    L::each(acc, [&](int i, int j, const float (&v)[8]) __attribute__((always_inline)) {
        const long long id = b0 + j;
        if (a0 + i >= a.C || id >= a.ids) return;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = f(v[e]);
        store8((T*)a.out + id * a.ostride + a0 + i, a.C - a0 - i, w);
    });
}

// dx from the shares' sums, each in its row's place; rows without a label are zeros (the last launch's workgroups from `summing` on).
template <class L, typename T>
__global__ __launch_bounds__(256) void k_loss_dx_sum(const GradArgs a)
{
    if ((int)blockIdx.x >= a.summing) {
        const int per = (a.C + 7) >> 3;
        const long long n = (long long)a.rows * per, step = (long long)(gridDim.x - a.summing) * 256;
        const float zeros[8] = {};
        for (long long u = (long long)(blockIdx.x - a.summing) * 256 + threadIdx.x; u < n; u += step) {
            const long long r = u / per;
            const int c = (int)(u - r * per) * 8;
            if (a.place[r] < 0) store8((T*)a.out + r * a.ostride + c, a.C - c, zeros);
        }
        return;
    }
    const int rows = *a.count, bblocks = dx_blocks(rows, L::BB), shares = dx_shares(rows, L::BB, a.bblocks * a.shares, a.most);
    const int part = a.first + (int)blockIdx.x, t = part / L::kParts, ib = t / a.ablocks, ia = t - ib * a.ablocks, a0 = ia * L::BA, b0 = ib * L::BB;
    if (b0 >= rows) return;
    const Factor f = gradient_scale(a.scale, a.mean, a.count);
    L::take(a.part + (long long)t * L::kSums, (long long)bblocks * a.ablocks * L::kSums, shares, part - t * L::kParts, [&](int i, int j, float (&v)[8]) __attribute__((always_inline)) {
        if (b0 + j >= rows || a0 + i >= a.C) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f(v[e]);
        store8((T*)a.out + a.index[b0 + j] * a.ostride + a0 + i, a.C - a0 - i, v);
    });
}

template <class L, typename T>
__global__ __launch_bounds__(256) void k_loss_dw_sum(const GradArgs a)
{
    const int t = blockIdx.x / L::kParts, ib = t / a.ablocks, ia = t - ib * a.ablocks, a0 = ia * L::BA, b0 = ib * L::BB;
    const Factor f = gradient_scale(a.scale, a.mean, a.count);
    L::take(a.part + (long long)t * L::kSums, (long long)a.bblocks * a.ablocks * L::kSums, a.shares, blockIdx.x - t * L::kParts, [&](int i, int j, float (&v)[8]) __attribute__((always_inline)) {
        if (b0 + j >= a.ids || a0 + i >= a.C) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f(v[e]);
        store8((T*)a.out + (long long)(b0 + j) * a.ostride + a0 + i, a.C - a0 - i, v);
    });
}

// ---- plans ---------------------------------------------------------------------------------------------------------
int planes_of_type(int dtype) { return dtype == FTP_BF16 ? 1 : 3; }
int padded(int c) { return (c + 63) & ~63; }
long long round_up(long long v, long long to) { return ceil_div(v, to) * to; }

struct Plan {
    int planes, gplanes, Cp, blocks, few;           // bfloats of an input and of an element of G
    long long Np, Vp, chunks, piece;                // rows and ids up to whole blocks of 64; ids of a piece, whole blocks of 256
    Split logits, dx, dw;
    int joins, most;
};
Plan plan_of(const ftp_token_loss_shape& s, bool back)
{
    Plan p = {};
    p.planes = planes_of_type(s.dtype);
    p.Cp = padded(s.channels);
    p.Np = round_up(std::max<long long>(s.rows, 1), 64);
    p.Vp = round_up(s.vocab, 64);
    p.chunks = ceil_div(std::max<long long>(s.rows, 1), kChunk);
    const long long terms = p.planes == 1 ? 1 : 6;
    // whether W, and few rows of x, can be read as they lie (their addresses are looked at by the call: scratch is there for both ways)
    p.few = s.rows <= kFew;
    p.gplanes = p.planes == 1 ? kGradPlanes : p.planes;
    if (!back) {
        p.logits = split_of(s.vocab, s.rows, p.Cp / 32 * terms, 128, 1);
        p.blocks = (int)ceil_div(s.vocab, p.few ? Few::BA : p.logits.block);
        p.joins = (int)std::min<long long>(ceil_div(std::max<long long>(s.rows, 1), 4), s.rows <= kJoin ? 1 : 1024);
        return p;
    }
    // a piece's G in at most 1 GiB and rows of 2^20, whole blocks
    const long long fits = std::min((1024ll << 20) / (2 * p.gplanes * p.Np) / 256 * 256, 1ll << 20), all = round_up(s.vocab, 256);
    const long long pieces = ceil_div(all, std::max(256ll, fits));
    p.piece = round_up(ceil_div(s.vocab, pieces), 256);
    p.logits = split_of(p.piece, s.rows, p.Cp / 32 * terms, 128, 1);
    const long long gterms = p.planes == 1 ? kGradPlanes : 6;
    p.dx = split_of(s.channels, s.rows, p.piece / 32 * gterms, 128, 64);
    p.most = (int)std::max<long long>(p.dx.shares, p.piece / 32 * gterms / 24);
    p.dw = split_of(s.channels, p.piece, p.Np / 32 * gterms, 128, 16);
    return p;
}

struct Buffers {
    int *counts, *index, *label, *place, *count;
    bf16_t *xc, *wc, *g;
    float2* part; float *target, *dx, *dw; double* sums;
    size_t bytes;
};
Buffers buffers_of(const ftp_token_loss_shape& s, const Plan& p, bool back, char* ws)
{
    Buffers b = {};
    Parts t(ws);
    b.counts = t.take<int>(p.chunks);
    b.index = t.take<int>(p.Np);
    b.label = t.take<int>(p.Np);
    b.place = t.take<int>(p.Np);
    b.count = t.take<int>(1);
    b.xc = t.take<bf16_t>(p.planes * p.Np * p.Cp);
    b.wc = t.take<bf16_t>((size_t)p.planes * p.Vp * p.Cp);
    if (!back) {
        b.part = t.take<float2>((size_t)p.Np * p.blocks);
        b.target = t.take<float>(p.Np);
        b.sums = t.take<double>(2 * 1024);
    } else {
        b.g = t.take<bf16_t>((size_t)p.gplanes * p.Np * p.piece);
        b.dx = t.take<float>((size_t)p.dx.shares * round_up(p.Np, p.dx.block) * round_up(p.Cp, p.dx.block));
        b.dw = t.take<float>(p.dw.shares > 1 ? (size_t)p.dw.shares * p.piece * round_up(p.Cp, p.dw.block) : 0);
    }
    b.bytes = t.used;
    return b;
}

unsigned pass_grid(long long n) { return (unsigned)std::min<long long>(std::max<long long>(ceil_div(n, 256), 1), 4096); }

// The labelled rows and W as the products read it: W as it lies where it is read by few rows and allows it, else laid out for them.  rows: whether the rows are wanted.
template <int P>
Matrix prepare(const ftp_token_loss_shape& s, const Plan& p, const Buffers& b, const void* x, const void* w, const void* labels, bool rows, hipStream_t st)
{
    const bool plain = P == 1 && s.rows < kPackRows && s.channels % 64 == 0 && s.w_stride % 8 == 0 && s.w_stride < (1 << 20) && aligned(w, 16);
    PrepareArgs a = {};
    a.ids = labels; a.x = x; a.xc = b.xc; a.index = b.index; a.label = b.label; a.place = b.place; a.count = b.count;
    a.rows = s.rows; a.stride = s.x_stride; a.plane = p.Np * p.Cp; a.block = p.Np * 32; a.wide = s.id_type; a.vocab = s.vocab; a.C = s.channels; a.Cp = p.Cp;
    a.gathering = rows ? (int)p.chunks * 4 : 0;
    a.w = w; a.wc = b.wc; a.wstride = s.w_stride; a.wplane = p.Vp * p.Cp; a.Vp = (int)p.Vp;
    const unsigned grid = (unsigned)a.gathering + (plain ? 0 : (unsigned)std::min<long long>(ceil_div(p.Vp / 16 * (p.Cp / 32), 4), 8192));
    if (rows && s.rows > kCountRows) {
        k_labelled<<<(unsigned)ceil_div(p.chunks, 4), 256, 0, st>>>(labels, s.id_type, s.rows, s.vocab, b.counts);
        a.counts = b.counts;
    }
    if (grid) {
        if constexpr (P == 1) k_prepare<bf16_t, 1><<<grid, 256, 0, st>>>(a);
        else k_prepare<float, 3><<<grid, 256, 0, st>>>(a);
    }
    return plain ? row_major((const bf16_t*)w, s.w_stride, s.vocab, p.Cp) : blocked(b.wc, p.Vp, p.Cp, a.wplane);
}

void set_scale(LogitArgs& a, float scale)
{
    // (c is a normal number and not 0, which times -infinity, ids past the end, would be none)
    const double c = std::fabs((double)scale) * 1.4426950408889634, least = 1e-30;
    a.c = (float)std::max(c, least);
    a.factor = (float)std::copysign(std::min(c / least, 1.0), (double)scale);
}

template <class L, int P, bool STATS>
void logits(LogitArgs& a, long long rows, hipStream_t st)
{
    a.stages = a.w.cols / L::KS;
    a.ablocks = (int)ceil_div(a.w.rows, L::BA);
    a.bblocks = (int)ceil_div(rows, L::BB);
    if (rows) k_logits<L, P, STATS><<<(unsigned)block_grid(a.ablocks, a.bblocks), L::kThreads, 0, st>>>(a);
}

template <int P>
void forward(const ftp_token_loss_shape& s, const void* x, const void* w, const void* labels, float* loss, float* lse, float* mean, char* ws, hipStream_t st)
{
    const Plan p = plan_of(s, false);
    const Buffers b = buffers_of(s, p, false, ws);
    LogitArgs a = {};
    a.terms = terms_of(P); a.wide = s.id_type; a.vocab = s.vocab; set_scale(a, s.scale); a.part = b.part; a.target = b.target; a.ids = labels;
    const long long x_stride = s.rows > 1 ? s.x_stride : s.channels;        // (one row's is no rows' distance: loads of the rows past it would lie on any address)
    const bool plain = p.few && P == 1 && s.channels % 64 == 0 && x_stride % 8 == 0 && x_stride < (1 << 20) && aligned(x, 16);
    a.w = prepare<P>(s, p, b, x, w, labels, !plain, st);
    a.w.rows = s.vocab;
    if (plain) a.x = row_major((const bf16_t*)x, x_stride, s.rows, p.Cp);
    else {
        a.x = blocked(b.xc, p.Np, p.Cp, p.Np * p.Cp);
        a.count = b.count; a.label = b.label;
    }
    if (p.few) logits<Few, P, true>(a, s.rows, st);
    else if (p.logits.block == 256) logits<Two, P, true>(a, s.rows, st);
    else logits<Mid<false, false>, P, true>(a, s.rows, st);
    const auto join = [&](auto kernel, int threads) { kernel<<<p.joins, threads, 0, st>>>(b.part, b.target, plain ? nullptr : b.place, labels, s.id_type, s.rows, s.vocab, a.ablocks, a.c, loss, lse, b.sums, mean); };
    if (s.rows > 4 && p.joins == 1) join(k_loss_join<16>, 1024);
    else join(k_loss_join<4>, 256);
    if (p.joins > 1 && mean) k_loss_mean<<<1, 256, 0, st>>>(b.sums, p.joins, mean);
}

template <class L, typename T>
void dw_pass(GradArgs& a, hipStream_t st)
{
    k_loss_dw<L, T><<<(unsigned)block_grid(a.ablocks, (long long)a.bblocks * a.shares), L::kThreads, 0, st>>>(a);
    if (a.shares > 1) k_loss_dw_sum<L, T><<<(unsigned)(a.ablocks * a.bblocks * L::kParts), 256, 0, st>>>(a);
}
template <class L, typename T>
void dx_sum(GradArgs& a, hipStream_t st)
{
    // a launch has less than 2^32 threads: from 2^34 results on it takes several, the last of which clears the rows without a label
    const unsigned clearing = std::min<unsigned>(pass_grid(a.rows * ceil_div(a.C, 8)), 1024);
    const int all = a.ablocks * a.bblocks * L::kParts, most = (int)(kMostGroups - clearing);
    for (a.first = 0; a.first < all; a.first += a.summing) {
        a.summing = std::min(all - a.first, most);
        k_loss_dx_sum<L, T><<<(unsigned)a.summing + (a.first + a.summing == all ? clearing : 0), 256, 0, st>>>(a);
    }
}
template <class L>
void dx_pass(GradArgs& a, hipStream_t st) { k_loss_dx<L><<<(unsigned)block_grid(a.ablocks, (long long)a.bblocks * a.shares), L::kThreads, 0, st>>>(a); }

template <int P, typename T>
void backward(const ftp_token_loss_shape& s, const void* x, const void* w, const void* labels, const float* lse, const float* dloss, void* dx, void* dw, char* ws, hipStream_t st)
{
    constexpr int G = P == 1 ? kGradPlanes : P;
    const Plan p = plan_of(s, true);
    const Buffers b = buffers_of(s, p, true, ws);
    const Matrix all = prepare<P>(s, p, b, x, w, labels, true, st), xc = blocked(b.xc, p.Np, p.Cp, p.Np * p.Cp), g = blocked(b.g, p.Np, (int)p.piece, p.Np * p.piece);
    for (long long v0 = 0; v0 < s.vocab; v0 += p.piece) {
        const int n = (int)std::min<long long>(p.piece, s.vocab - v0);
        const Matrix wp = rows_of(all, v0, n);
        LogitArgs a = {};
        a.w = wp; a.x = xc; a.count = b.count; a.label = b.label; a.terms = terms_of(P); a.vocab = s.vocab; a.piece0 = (int)v0; set_scale(a, s.scale);
        a.index = b.index; a.lse = lse; a.dloss = dloss; a.g = b.g; a.gblock = g.block; a.gplane = g.plane;
        if (p.few) logits<Few, G, false>(a, s.rows, st);
        else if (p.logits.block == 256) logits<Two, G, false>(a, s.rows, st);
        else logits<Mid<false, false>, G, false>(a, s.rows, st);
        GradArgs k = {};
        k.count = b.count; k.terms = P == 1 ? terms_one_two() : terms_of(P); k.C = s.channels; k.scale = s.scale; k.mean = !dloss;
        if (dx && s.rows) {
            k.a = wp; k.b = g; k.stages = (int)ceil_div(n, 32); k.shares = p.dx.shares; k.most = p.most; k.add = v0 > 0;
            k.ablocks = (int)ceil_div(p.Cp, p.dx.block); k.bblocks = (int)ceil_div(s.rows, p.dx.block);
            k.part = b.dx; k.out = dx; k.ostride = s.dx_stride; k.place = b.place; k.index = b.index; k.rows = (int)s.rows;
            const bool last = v0 + p.piece >= s.vocab;
            if (p.dx.block == 256) {
                dx_pass<Big<true, false>>(k, st);
                if (last) dx_sum<Big<true, false>, T>(k, st);
            } else {
                dx_pass<Mid<true, false>>(k, st);
                if (last) dx_sum<Mid<true, false>, T>(k, st);
            }
        }
        if (dw) {
            k.a = xc; k.b = g; k.shares = p.dw.shares; k.ids = n;
            k.ablocks = (int)ceil_div(p.Cp, p.dw.block); k.bblocks = (int)ceil_div(n, p.dw.block);
            k.part = b.dw; k.out = (T*)dw + v0 * s.dw_stride; k.ostride = s.dw_stride;
            if (p.dw.block == 256) dw_pass<Big<true, true>, T>(k, st);
            else dw_pass<Mid<true, true>, T>(k, st);
        }
    }
}

}  // namespace

bool token_loss_fits(const ftp_token_loss_shape& s)
{
    // rows, ids, blocks and offsets within a stage are 32-bit numbers, and a launch has fewer than 2^32 threads
    return s.rows <= (1ll << 22) && s.vocab <= (1 << 22) && s.channels <= (1 << 14) && ceil_div(s.rows, 256) * ceil_div(s.vocab, 256) < (1 << 21);
}
size_t token_loss_forward_workspace(const ftp_token_loss_shape& s) { return buffers_of(s, plan_of(s, false), false, nullptr).bytes; }
size_t token_loss_backward_workspace(const ftp_token_loss_shape& s) { return buffers_of(s, plan_of(s, true), true, nullptr).bytes; }

void token_loss_forward(const ftp_token_loss_shape& s, const void* x, const void* w, const void* labels, float* loss, float* lse, float* mean, char* ws, hipStream_t st)
{
    if (s.dtype == FTP_BF16) forward<1>(s, x, w, labels, loss, lse, mean, ws, st);
    else forward<3>(s, x, w, labels, loss, lse, mean, ws, st);
}
void token_loss_backward(const ftp_token_loss_shape& s, const void* x, const void* w, const void* labels, const float* lse, const float* dloss, void* dx, void* dw, char* ws,
                         hipStream_t st)
{
    if (s.dtype == FTP_BF16) backward<1, bf16_t>(s, x, w, labels, lse, dloss, dx, dw, ws, st);
    else backward<3, float>(s, x, w, labels, lse, dloss, dx, dw, ws, st);
}

}  // namespace ftp
