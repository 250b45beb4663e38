// Layer norm over channels, forward and backward:
//   mean = sum x / C, var = sum (x - mean)^2 / C, r = (var + eps)^-1/2, h = (x - mean) r, y = h gamma + beta
//   a = dy gamma, dx = r (a - mean(a) - h mean(a h)), dgamma = sum over tokens of dy h, dbeta = sum of dy
// All sums in 32 bits; the variance from the centred values (a second pass over registers or LDS, never E[x^2] - mean^2).  Bound by memory: each pass
// reads its inputs and writes its outputs once.
//
// Tokens whose channels lie side by side (rows) stay in registers: 2^k lanes a row, 16 bytes a load where alignment lets it.  Anything else (NCHW
// maps, map to rows) goes through LDS in tiles of up to 64 tokens x all channels, read along whichever axis is contiguous.
//
// Measured: k_norm_rows 4 tokens of 256 2.3 us (one round trip to memory and the launch); 92416 x 512 bfloats 33 us, 190 MB, 5.7 TB/s (fp32 67); k_norm_back_rows on as many 46.8 us,
// 285 MB, 6.1 TB/s (a large copy: 4.8, but the last-level cache keeps part), 17797 x 250 fp32 from a checkpoint 13.1 us, 40 MB; k_norm_params behind it 4.1 us; k_norm_tiles 16 images of 76 x 76, 128 channels fp32 to rows 27 us, 95 MB, 3.5 TB/s.
#include "ftp_norm_rows.h"
#include "ftp_tokens.h"

#include <algorithm>

namespace ftp {
namespace {

struct RowArgs {
    const void* x; const void* gamma; const void* beta; void* y;
    float* mean; float* rstd;
    const void* dy; void* dx; const int8_t* codes; const int8_t* exps; float* partial;
    long long rows, inner;                          // inner: tokens to an outer step (rows: one step)
    long long xo, xi, yo, yi, go, gi;               // strides: x, y (forward) or dx (backward), dy
    int C, lanes, block, nblocks;
    uint32_t first;                                 // workgroups in earlier launches of the pass
    float eps;
};

__device__ __forceinline__ long long row_offset(long long row, long long inner, long long rows, long long so, long long si)
{
    if (inner == rows) return row * si;
    const long long o = (uint32_t)row / (uint32_t)inner;            // (rows are fewer than 2^31)
    return o * so + (row - o * inner) * si;
}

// Sum over the `lanes` lanes of a row (a power of two); every lane gets it.  Neighbours are exchanged by the vector unit itself (data-parallel primitives, permlane swaps), not
// through the LDS crossbar.  WIDE: the row is the workgroup.
__device__ __forceinline__ float lane_sum(float v, int lanes)
{
    if (lanes > 1) v += quad_xor<1>(v);
    if (lanes > 2) v += quad_xor<2>(v);
    if (lanes > 4) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xF, 0xF, true));      // row_half_mirror: the other quad of 8
    if (lanes > 8) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x140, 0xF, 0xF, true));      // row_mirror: the other half of 16
    if (lanes > 16) { const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false); v = __uint_as_float(r[0]) + __uint_as_float(r[1]); }
    if (lanes > 32) { const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false); v = __uint_as_float(r[0]) + __uint_as_float(r[1]); }
    return v;
}
template <bool WIDE>
__device__ __forceinline__ float row_sum(float v, int lanes, float* lds)
{
    v = lane_sum(v, WIDE ? 64 : lanes);
    if constexpr (WIDE) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
        __syncthreads();
    }
    return v;
}

// Bound by memory: a row is read once and written once.
template <typename T, int VEC, int NV, bool WIDE>
__global__ __launch_bounds__(256) void k_norm_rows(const RowArgs a)
{
    __shared__ float lds[4];
    const int lanes = WIDE ? 256 : a.lanes;
    const int lane = threadIdx.x & (lanes - 1);
    const long long row = (long long)(a.first + blockIdx.x) * (256 / lanes) + (WIDE ? 0 : threadIdx.x / lanes);
    const bool live = row < a.rows;
    Pack<T, VEC> x[NV];
    const T* px = (const T*)a.x + (live ? row_offset(row, a.inner, a.rows, a.xo, a.xi) : 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + lane) * VEC;
        if (live && c < a.C) x[i].load(px + c);
        else x[i].zero();
    }
    float s = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) s += x[i].get(j);
    const float mean = row_sum<WIDE>(s, lanes, lds) / (float)a.C;
    s = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const bool in = (i * lanes + lane) * VEC < a.C;
#pragma unroll
        for (int j = 0; j < VEC; ++j) { const float d = x[i].get(j) - mean; s = in ? fmaf(d, d, s) : s; }
    }
    const float rstd = 1.0f / sqrtf(row_sum<WIDE>(s, lanes, lds) / (float)a.C + a.eps);
    if (!live) return;
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* py = (T*)a.y + row_offset(row, a.inner, a.rows, a.yo, a.yi);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + lane) * VEC;
        if (c >= a.C) continue;
        Pack<T, VEC> g, b;
        if (a.gamma) g.load((const T*)a.gamma + c);
        if (a.beta) b.load((const T*)a.beta + c);
        float v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = fmaf((x[i].get(j) - mean) * rstd, a.gamma ? g.get(j) : 1.0f, a.beta ? b.get(j) : 0.0f);
        x[i].put(v);
        x[i].store(py + c);
    }
}

constexpr int kBackThreads = 512;                   // (twice the wavefronts to a share of dgamma and dbeta than 256)

// A workgroup walks over rows and keeps its part of dgamma and dbeta in registers; the next row's loads are in flight while this one is worked on.
// HELD: x comes from its 8-bit checkpoint.
template <typename T, int VEC, int NV, bool WIDE, bool HELD>
__global__ __launch_bounds__(WIDE ? 256 : kBackThreads) void k_norm_back_rows(const RowArgs a)
{
    constexpr int WAVES = kBackThreads / 64;
    __shared__ float lds[WIDE ? 4 : WAVES * 64 * VEC * NV];
    typedef typename std::conditional<HELD, int8_t, T>::type X;
    const int lanes = WIDE ? 256 : a.lanes;
    const int lane = threadIdx.x & (lanes - 1), per = WIDE ? 1 : kBackThreads / lanes;
    const long long step = (long long)gridDim.x * per;
    Pack<T, VEC> g[NV];
    float dg[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + lane) * VEC;
        float one[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) { one[j] = 1.0f; dg[i][j] = db[i][j] = 0.0f; }
        g[i].put(one);
        if (a.gamma && c < a.C) g[i].load((const T*)a.gamma + c);
    }
    Pack<X, VEC> nx[NV];
    Pack<T, VEC> ny[NV];
    int ne[NV];
    float nmean = 0, nrstd = 0;
    const auto fetch = [&](long long row) {
        const bool live = row < a.rows;
        const X* px;
        if constexpr (HELD) px = a.codes + (live ? row * a.C : 0);
        else px = (const T*)a.x + (live ? row_offset(row, a.inner, a.rows, a.xo, a.xi) : 0);
        const T* py = (const T*)a.dy + (live ? row_offset(row, a.inner, a.rows, a.go, a.gi) : 0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * lanes + lane) * VEC;
            if (live && c < a.C) {
                nx[i].load(px + c);
                ny[i].load(py + c);
                if constexpr (HELD) ne[i] = a.exps[row * a.nblocks + c / a.block];
            } else {
                nx[i].zero();
                ny[i].zero();
                ne[i] = 0;
            }
        }
        nmean = live ? a.mean[row] : 0.0f;
        nrstd = live ? a.rstd[row] : 0.0f;
    };
    // (WIDE: all threads of the workgroup are on one row, so all leave together)
    const long long first = (long long)blockIdx.x * per + (WIDE ? 0 : threadIdx.x / lanes);
    const float inv = 1.0f / (float)a.C;
    fetch(first);
    for (long long base = (long long)blockIdx.x * per, row = first; base < a.rows; base += step, row += step) {
        Pack<T, VEC> y[NV];
        float h[NV][VEC];
        const float mean = nmean, rstd = nrstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            y[i] = ny[i];
            const float unit = HELD ? held_scale(ne[i]) : 1.0f;
            const bool in = (i * lanes + lane) * VEC < a.C;
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[i][j] = in ? ((HELD ? nx[i].get(j) * unit : nx[i].get(j)) - mean) * rstd : 0.0f;
        }
        fetch(row + step);
        float s1 = 0, s2 = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float v = y[i].get(j), w = v * g[i].get(j);
                s1 += w;
                s2 = fmaf(w, h[i][j], s2);
                dg[i][j] = fmaf(v, h[i][j], dg[i][j]);
                db[i][j] += v;
            }
        s1 = row_sum<WIDE>(s1, lanes, lds) * inv;
        s2 = row_sum<WIDE>(s2, lanes, lds) * inv;
        if (row < a.rows) {
            T* p = (T*)a.dx + row_offset(row, a.inner, a.rows, a.yo, a.yi);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * lanes + lane) * VEC;
                if (c >= a.C) continue;
                float v[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[j] = rstd * (fmaf(y[i].get(j), g[i].get(j), -s1) - h[i][j] * s2);
                y[i].put(v);
                y[i].store(p + c);
            }
        }
    }
    if (!a.partial) return;
    // the workgroup's share: rows side by side in a wavefront by lane exchange, wavefronts through LDS, in a fixed order
    float* out = a.partial + (long long)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int which = 0; which < 2; ++which, out += a.C) {
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = (i * 256 + lane) * VEC + j;
                    if (c < a.C) out[c] = which ? db[i][j] : dg[i][j];
                }
        } else {
            __syncthreads();
            const int width = lanes * VEC * NV;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float v = which ? db[i][j] : dg[i][j];
                    for (int m = lanes; m < 64; m <<= 1) v += __shfl_xor(v, m);
                    if ((threadIdx.x & 63) < lanes) lds[(threadIdx.x >> 6) * width + (i * lanes + lane) * VEC + j] = v;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < a.C; c += kBackThreads) {
                float v = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v += lds[w * width + c];
                out[c] = v;
            }
        }
    }
}

// Rows too long for registers: a workgroup a row, elements read again for each step (from the caches).
template <typename T>
__global__ __launch_bounds__(256) void k_norm_long(const RowArgs a)
{
    __shared__ float lds[4];
    const long long row = a.first + blockIdx.x;
    const T* px = (const T*)a.x + row_offset(row, a.inner, a.rows, a.xo, a.xi);
    T* py = (T*)a.y + row_offset(row, a.inner, a.rows, a.yo, a.yi);
    float s = 0;
    for (int c = threadIdx.x; c < a.C; c += 256) s += ld(px + c);
    const float mean = row_sum<true>(s, 256, lds) / (float)a.C;
    s = 0;
    for (int c = threadIdx.x; c < a.C; c += 256) { const float d = ld(px + c) - mean; s = fmaf(d, d, s); }
    const float rstd = 1.0f / sqrtf(row_sum<true>(s, 256, lds) / (float)a.C + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    for (int c = threadIdx.x; c < a.C; c += 256)
        st(py + c, fmaf((ld(px + c) - mean) * rstd, a.gamma ? ld((const T*)a.gamma + c) : 1.0f, a.beta ? ld((const T*)a.beta + c) : 0.0f));
}

template <typename T>
__device__ __forceinline__ float long_x(const RowArgs& a, long long row, long long off, int c)
{
    if (a.codes) return (float)a.codes[row * a.C + c] * held_scale(a.exps[row * a.nblocks + c / a.block]);
    return ld((const T*)a.x + off + c);
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_back_long(const RowArgs a)
{
    __shared__ float lds[4];
    const long long row = a.first + blockIdx.x, off = row_offset(row, a.inner, a.rows, a.xo, a.xi);
    const T* py = (const T*)a.dy + row_offset(row, a.inner, a.rows, a.go, a.gi);
    T* pd = (T*)a.dx + row_offset(row, a.inner, a.rows, a.yo, a.yi);
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0, s2 = 0;
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const float w = ld(py + c) * (a.gamma ? ld((const T*)a.gamma + c) : 1.0f);
        s1 += w;
        s2 = fmaf(w, (long_x<T>(a, row, off, c) - mean) * rstd, s2);
    }
    s1 = row_sum<true>(s1, 256, lds) / (float)a.C;
    s2 = row_sum<true>(s2, 256, lds) / (float)a.C;
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const float h = (long_x<T>(a, row, off, c) - mean) * rstd;
        st(pd + c, rstd * (fmaf(ld(py + c), a.gamma ? ld((const T*)a.gamma + c) : 1.0f, -s1) - h * s2));
    }
}

// ... and their parameter gradients: a thread a channel and a share of the rows.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_long_params(const RowArgs a, int shares)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.C) return;
    const long long lo = a.rows * blockIdx.y / shares, hi = a.rows * (blockIdx.y + 1) / shares;
    float dg = 0, db = 0;
    for (long long row = lo; row < hi; ++row) {
        const float v = ld((const T*)a.dy + row_offset(row, a.inner, a.rows, a.go, a.gi) + c);
        dg = fmaf(v, (long_x<T>(a, row, row_offset(row, a.inner, a.rows, a.xo, a.xi), c) - a.mean[row]) * a.rstd[row], dg);
        db += v;
    }
    a.partial[(long long)blockIdx.y * 2 * a.C + c] = dg;
    a.partial[((long long)blockIdx.y * 2 + 1) * a.C + c] = db;
}

// dgamma and dbeta from the workgroups' shares: 32 columns x 32 groups of shares a workgroup, each thread's loads independent.
__global__ __launch_bounds__(1024) void k_norm_params(const float* partial, int shares, int C, float* dgamma, float* dbeta)
{
    __shared__ float lds[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), grp = threadIdx.x >> 5, width = 2 * C;
    float s = 0;
    if (col < width) {
#pragma unroll 16
        for (int i = grp; i < shares; i += 32) s += partial[(long long)i * width + col];
    }
    lds[grp][threadIdx.x & 31] = s;
    __syncthreads();
    const int c = threadIdx.x >> 5, l = threadIdx.x & 31;            // a half wavefront adds up a column
    s = lds[l][c];
    for (int m = 16; m; m >>= 1) s += __shfl_xor(s, m);
    const int out = blockIdx.x * 32 + c;
    if (l == 0 && out < width) (out < C ? dgamma[out] : dbeta[out - C]) = s;
}

// ---- tiles of tokens through LDS -----------------------------------------------------------------------------------------------------------------------

struct TileArgs {
    const void* x; const void* gamma; const void* beta; void* y;
    float* mean; float* rstd;
    const void* dy; void* dx; float* partial;
    long long outer, inner;
    long long xs[3], ys[3], gs[3];                  // strides: x, y (forward) or dx (backward), dy
    int C, px, shift, tiles;                        // px = 2^shift tokens a tile, `tiles` tiles to an outer step
    uint32_t first;                                 // workgroups in earlier launches of the pass
    int xvec, yvec, gvec;                           // elements of x, y or dx, dy that go together along the tile's contiguous axis (1, or 16 bytes)
    float eps;
};

// LDS tile: [channel][token], a pitch of an odd number of dwords.
template <typename T> __device__ __forceinline__ int tile_pitch(int px) { return px + 4 / (int)sizeof(T); }

template <typename T, int V>
__device__ __forceinline__ void tile_load_v(T* tile, const T* p, const long long (&s)[3], int C, int px, int shift, int n, int pitch)
{
    if (s[2] == 1) {                                // rows: lanes along the channels
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int t = wave; t < px; t += 4)
            for (int c = lane * V; c < C; c += 64 * V) {
                Pack<T, V> v;
                if (t < n) v.load(p + t * s[1] + c);
                else v.zero();
#pragma unroll
                for (int j = 0; j < V; ++j) st(tile + (c + j) * pitch + t, v.get(j));
            }
    } else {                                        // lanes along the tokens (their stride is 1 where V > 1)
        const int units = C * (px / V), lg = shift - (V == 1 ? 0 : V == 4 ? 2 : 3);
#pragma unroll 4
        for (int u = threadIdx.x; u < units; u += 256) {
            const int c = u >> lg, t = (u & ((px / V) - 1)) * V;
            Pack<T, V> v;
            if (t < n) v.load(p + t * s[1] + c * s[2]);
            else v.zero();
#pragma unroll
            for (int j = 0; j < V; ++j) st(tile + c * pitch + t + j, v.get(j));
        }
    }
}

template <typename T>
__device__ __forceinline__ void tile_load(T* tile, const T* p, const long long (&s)[3], int vec, int C, int px, int shift, int n, int pitch)
{
    if (vec == 1) tile_load_v<T, 1>(tile, p, s, C, px, shift, n, pitch);
    else tile_load_v<T, 16 / (int)sizeof(T)>(tile, p, s, C, px, shift, n, pitch);
}

// The parameters as fp32 in LDS (null: `none`).
template <typename T>
__device__ __forceinline__ void param_load(float* to, const void* p, float none, int C)
{
    for (int c = threadIdx.x; c < C; c += 256) to[c] = p ? ld((const T*)p + c) : none;
}

// p[token][channel] = f(channel, token); tokens below n.
template <typename T, int V, class F>
__device__ __forceinline__ void tile_store_v(T* p, const long long (&s)[3], int C, int px, int shift, int n, F f)
{
    if (s[2] == 1) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int c = lane * V; c < C; c += 64 * V)
#pragma unroll 4
            for (int t = wave; t < n; t += 4) {
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = f(c + j, t);
                Pack<T, V> w;
                w.put(v);
                w.store(p + t * s[1] + c);
            }
    } else {
        const int units = C * (px / V), lg = shift - (V == 1 ? 0 : V == 4 ? 2 : 3);
        for (int u = threadIdx.x; u < units; u += 256) {
            const int c = u >> lg, t = (u & ((px / V) - 1)) * V;
            if (t >= n) continue;
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = f(c, t + j);
            Pack<T, V> w;
            w.put(v);
            w.store(p + t * s[1] + c * s[2]);
        }
    }
}

template <typename T, class F>
__device__ __forceinline__ void tile_store(T* p, const long long (&s)[3], int vec, int C, int px, int shift, int n, F f)
{
    if (vec == 1) tile_store_v<T, 1>(p, s, C, px, shift, n, f);
    else tile_store_v<T, 16 / (int)sizeof(T)>(p, s, C, px, shift, n, f);
}

// Sum over the channels of f(channel) for every token of the tile; the sum of token t ends in sums[t].  red: 256 floats.
template <class F>
__device__ __forceinline__ void token_sums(float* sums, float* red, int C, int px, int shift, F f)
{
    const int t = threadIdx.x & (px - 1), part = threadIdx.x >> shift, parts = 256 >> shift;
    float s = 0;
    for (int c = part; c < C; c += parts) s += f(c, t);
    red[threadIdx.x] = s;
    __syncthreads();
    for (int k = parts >> 1; k; k >>= 1) {
        if (part < k) red[threadIdx.x] += red[threadIdx.x + (k << shift)];
        __syncthreads();
    }
    if (part == 0) sums[t] = red[t];
    __syncthreads();
}

// Mean, then variance from LDS, then y: the map is read once.  Bound by the round trips of a workgroup's load, sums and stores; tiles of 128 bytes a channel leave eight workgroups a CU
// (64 tokens a tile, four: 52 us instead of 26).
template <typename T>
__global__ __launch_bounds__(256) void k_norm_tiles(const TileArgs a)
{
    extern __shared__ char smem[];
    float* red = (float*)smem;
    float* mean = red + 256;
    float* rstd = mean + 64;
    float* gamma = rstd + 64;
    float* beta = gamma + a.C;
    T* tile = (T*)(beta + a.C);
    param_load<T>(gamma, a.gamma, 1.0f, a.C);
    param_load<T>(beta, a.beta, 0.0f, a.C);
    const uint32_t block = a.first + blockIdx.x;
    const int o = block / (uint32_t)a.tiles, pitch = tile_pitch<T>(a.px);
    const long long at = (long long)(block - (uint32_t)o * a.tiles) << a.shift;
    const int n = (int)min((long long)a.px, a.inner - at);
    tile_load(tile, (const T*)a.x + o * a.xs[0] + at * a.xs[1], a.xs, a.xvec, a.C, a.px, a.shift, n, pitch);
    __syncthreads();
    token_sums(mean, red, a.C, a.px, a.shift, [&](int c, int t) { return ld(tile + c * pitch + t); });
    if (threadIdx.x < a.px) mean[threadIdx.x] /= (float)a.C;
    __syncthreads();
    token_sums(rstd, red, a.C, a.px, a.shift, [&](int c, int t) { const float d = ld(tile + c * pitch + t) - mean[t]; return d * d; });
    if (threadIdx.x < a.px) {
        const float r = 1.0f / sqrtf(rstd[threadIdx.x] / (float)a.C + a.eps);
        rstd[threadIdx.x] = r;
        if (threadIdx.x < n) {
            if (a.mean) a.mean[o * a.inner + at + threadIdx.x] = mean[threadIdx.x];
            if (a.rstd) a.rstd[o * a.inner + at + threadIdx.x] = r;
        }
    }
    __syncthreads();
    tile_store((T*)a.y + o * a.ys[0] + at * a.ys[1], a.ys, a.yvec, a.C, a.px, a.shift, n, [&](int c, int t) {
        return fmaf((ld(tile + c * pitch + t) - mean[t]) * rstd[t], gamma[c], beta[c]);
    });
}

// A workgroup walks over tiles; channels' sums over a tile's tokens go to LDS, a thread its own channels, and at the end to memory as the workgroup's share.  16 images of 76 x 76, 128
// channels, x a map, dy rows: fp32 75 us (143 MB, 1.9 TB/s), bfloats 72: bound by what follows each other in a workgroup, the load of a tile, two sums, the store, and sums over its tokens by as
// many threads as there are channels.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_back_tiles(const TileArgs a)
{
    extern __shared__ char smem[];
    float* red = (float*)smem;
    float* mean = red + 256;
    float* rstd = mean + 64;
    float* s1 = rstd + 64;
    float* s2 = s1 + 64;
    float* acc = s2 + 64;                           // [2][C], a thread its own channels
    const int pitch = tile_pitch<T>(a.px);
    float* gamma = acc + 2 * a.C;
    T* tx = (T*)(gamma + a.C);
    param_load<T>(gamma, a.gamma, 1.0f, a.C);
    T* ty = tx + (long long)a.C * pitch;
    for (int c = threadIdx.x; c < a.C; c += 256) acc[c] = acc[a.C + c] = 0;
    const float inv = 1.0f / (float)a.C;
    const long long total = a.outer * a.tiles;
    for (long long i = blockIdx.x; i < total; i += gridDim.x) {
        const long long o = i / a.tiles, at = (i - o * a.tiles) << a.shift;
        const int n = (int)min((long long)a.px, a.inner - at);
        __syncthreads();
        if (threadIdx.x < a.px) {
            mean[threadIdx.x] = threadIdx.x < n ? a.mean[o * a.inner + at + threadIdx.x] : 0.0f;
            rstd[threadIdx.x] = threadIdx.x < n ? a.rstd[o * a.inner + at + threadIdx.x] : 0.0f;
        }
        tile_load(tx, (const T*)a.x + o * a.xs[0] + at * a.xs[1], a.xs, a.xvec, a.C, a.px, a.shift, n, pitch);
        tile_load(ty, (const T*)a.dy + o * a.gs[0] + at * a.gs[1], a.gs, a.gvec, a.C, a.px, a.shift, n, pitch);
        __syncthreads();
        const auto h = [&](int c, int t) { return (ld(tx + c * pitch + t) - mean[t]) * rstd[t]; };
        token_sums(s1, red, a.C, a.px, a.shift, [&](int c, int t) { return ld(ty + c * pitch + t) * gamma[c]; });
        token_sums(s2, red, a.C, a.px, a.shift, [&](int c, int t) { return ld(ty + c * pitch + t) * gamma[c] * h(c, t); });
        tile_store((T*)a.dx + o * a.ys[0] + at * a.ys[1], a.ys, a.yvec, a.C, a.px, a.shift, n, [&](int c, int t) {
            return rstd[t] * (fmaf(ld(ty + c * pitch + t), gamma[c], -s1[t] * inv) - h(c, t) * (s2[t] * inv));
        });
        if (a.partial)
            for (int c = threadIdx.x; c < a.C; c += 256) {
                float dg = 0, db = 0;
                for (int t = 0; t < n; ++t) { const float v = ld(ty + c * pitch + t); dg = fmaf(v, h(c, t), dg); db += v; }
                acc[c] += dg;
                acc[a.C + c] += db;
            }
    }
    if (!a.partial) return;
    __syncthreads();
    float* out = a.partial + (long long)blockIdx.x * 2 * a.C;
    for (int c = threadIdx.x; c < 2 * a.C; c += 256) out[c] = acc[c];
}

// ---- which kernel --------------------------------------------------------------------------------------------------------------------------------------

constexpr int kShares = 512;                        // workgroups of a backward pass at most: each leaves 2 C sums

// The strides that a pass uses: x, y and no third, or x (not from a checkpoint), dx and dy.
struct Strides { const int64_t* x; const int64_t* y; const int64_t* g; };
Strides strides_of(const ftp_norm_shape& s, bool back, bool held) { return back ? Strides{held ? s.dy_stride : s.x_stride, s.dx_stride, s.dy_stride} : Strides{s.x_stride, s.y_stride, s.y_stride}; }

bool by_rows(const Strides& t, int channels) { return channels == 1 || (t.x[2] == 1 && t.y[2] == 1 && t.g[2] == 1); }

RowArgs row_args(const ftp_norm_shape& s, const Strides& t)
{
    RowArgs a = {};
    a.rows = s.outer * s.inner;
    a.inner = s.inner;
    a.xo = t.x[0]; a.xi = t.x[1]; a.yo = t.y[0]; a.yi = t.y[1]; a.go = t.g[0]; a.gi = t.g[1];
    if (s.inner == 1) { a.inner = a.rows; a.xi = a.xo; a.yi = a.yo; a.gi = a.go; }
    else if (s.outer == 1 || (a.xo == s.inner * a.xi && a.yo == s.inner * a.yi && a.go == s.inner * a.gi)) a.inner = a.rows;
    if (a.inner == a.rows) a.xo = a.yo = a.go = 0;  // (one step: not used)
    a.C = s.channels; a.eps = s.eps;
    return a;
}

// Largest vector that sizes, strides and addresses allow: 16 bytes down to one element.
int row_vec(const RowArgs& a, int es, const void* const* ptrs, int n, const int8_t* codes)
{
    for (int v = 16 / es; v > 1; v >>= 1) {
        bool ok = a.C % v == 0 && a.xo % v == 0 && a.xi % v == 0 && a.yo % v == 0 && a.yi % v == 0 && a.go % v == 0 && a.gi % v == 0 && aligned(codes, v);
        for (int i = 0; i < n; ++i) ok = ok && aligned(ptrs[i], (size_t)v * es);
        if (ok) return v;
    }
    return 1;
}

template <typename T, int VEC, int NV>
void run_rows(const RowArgs& a, const RowForm& f, bool back, unsigned grid, hipStream_t st)
{
    // (f.wide and NV are what row_form() gives)
    if constexpr (row_built(VEC, NV, true)) {
        if (f.wide) {
            if (!back) k_norm_rows<T, VEC, NV, true><<<grid, 256, 0, st>>>(a);
            else if (a.codes) k_norm_back_rows<T, VEC, NV, true, true><<<grid, 256, 0, st>>>(a);
            else k_norm_back_rows<T, VEC, NV, true, false><<<grid, 256, 0, st>>>(a);
            return;
        }
    }
    if constexpr (row_built(VEC, NV, false)) {
        if (!back) k_norm_rows<T, VEC, NV, false><<<grid, 256, 0, st>>>(a);
        else if (a.codes) k_norm_back_rows<T, VEC, NV, false, true><<<grid, kBackThreads, 0, st>>>(a);
        else k_norm_back_rows<T, VEC, NV, false, false><<<grid, kBackThreads, 0, st>>>(a);
    }
}

template <typename T, int VEC>
void run_rows_v(const RowArgs& a, const RowForm& f, bool back, unsigned grid, hipStream_t st)
{
    switch (f.nv) {
        case 1: run_rows<T, VEC, 1>(a, f, back, grid, st); break;
        case 2: run_rows<T, VEC, 2>(a, f, back, grid, st); break;
        case 4: run_rows<T, VEC, 4>(a, f, back, grid, st); break;
        default: run_rows<T, VEC, 8>(a, f, back, grid, st); break;
    }
}

template <typename T>
void run_rows_t(const RowArgs& a, int vec, const RowForm& f, bool back, unsigned grid, hipStream_t st)
{
    switch (vec) {
        case 8: if constexpr (sizeof(T) == 2) run_rows_v<T, 8>(a, f, back, grid, st); break;
        case 4: run_rows_v<T, 4>(a, f, back, grid, st); break;
        case 2: run_rows_v<T, 2>(a, f, back, grid, st); break;
        default: run_rows_v<T, 1>(a, f, back, grid, st); break;
    }
}

size_t tile_bytes(const ftp_norm_shape& s, int px, bool back)
{
    const size_t es = s.dtype == FTP_BF16 ? 2 : 4;
    return (256 + (back ? 256 : 128)) * 4 + (back ? 3 : 2) * (size_t)s.channels * 4 + (back ? 2 : 1) * (size_t)s.channels * (px + 4 / es) * es;
}
// Tokens a tile: 128 bytes of a map's row; fewer, down to 64 bytes, where a CU would hold less than four workgroups, and fewer still, down to one, above 64 KB (4096 fp32 channels,
// backward: 114 KB of a CU's 160).
int tile_tokens(const ftp_norm_shape& s, bool back)
{
    const int es = s.dtype == FTP_BF16 ? 2 : 4;
    int px = 128 / es;
    while (px * es > 64 && tile_bytes(s, px, back) > 40960) px >>= 1;
    while (px > 1 && tile_bytes(s, px, back) > 65536) px >>= 1;
    while (px > 4 && px / 2 >= s.inner) px >>= 1;
    return px;
}
// A pass of `groups` workgroups of 256 in as many launches as it takes.
template <class Args, class F>
void by_launches(Args a, long long groups, F launch)
{
    for (long long at = 0; at < groups; at += kMostGroups) {
        a.first = (uint32_t)at;
        launch(a, (unsigned)std::min(kMostGroups, groups - at));
    }
}
// Elements that go together along the contiguous axis of one tensor: 16 bytes or one.
int tile_vec(const ftp_norm_shape& s, const int64_t* str, int px, const void* p)
{
    const int v = s.dtype == FTP_BF16 ? 8 : 4;
    if (!aligned(p, 16) || str[0] % v) return 1;
    if (str[2] == 1) return s.channels % v == 0 && str[1] % v == 0 ? v : 1;
    return str[1] == 1 && str[2] % v == 0 && s.inner % v == 0 && px >= v ? v : 1;
}

TileArgs tile_args(const ftp_norm_shape& s, const Strides& t, bool back)
{
    TileArgs a = {};
    a.outer = s.outer; a.inner = s.inner; a.C = s.channels; a.eps = s.eps;
    for (int i = 0; i < 3; ++i) { a.xs[i] = t.x[i]; a.ys[i] = t.y[i]; a.gs[i] = t.g[i]; }
    a.px = tile_tokens(s, back);
    while ((1 << a.shift) < a.px) ++a.shift;
    a.tiles = (int)ceil_div(s.inner, a.px);
    return a;
}

}  // namespace

size_t norm_workspace(const ftp_norm_shape& s) { return (size_t)kShares * 2 * s.channels * sizeof(float); }

void norm_forward(const ftp_norm_shape& s, const void* x, const void* gamma, const void* beta, void* y, float* mean, float* rstd, hipStream_t st)
{
    const bool bf = s.dtype == FTP_BF16;
    const Strides t = strides_of(s, false, false);
    if (!by_rows(t, s.channels)) {
        TileArgs a = tile_args(s, t, false);
        a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd;
        a.xvec = tile_vec(s, t.x, a.px, x); a.yvec = tile_vec(s, t.y, a.px, y);
        by_launches(a, s.outer * a.tiles, [&](const TileArgs& a, unsigned grid) {
            if (bf) k_norm_tiles<bf16_t><<<grid, 256, tile_bytes(s, a.px, false), st>>>(a);
            else k_norm_tiles<float><<<grid, 256, tile_bytes(s, a.px, false), st>>>(a);
        });
        return;
    }
    RowArgs a = row_args(s, t);
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd;
    const void* ptrs[] = {x, gamma, beta, y};
    const int vec = row_vec(a, bf ? 2 : 4, ptrs, 4, nullptr);
    const RowForm f = row_form(a.C, vec);
    a.lanes = f.lanes;
    by_launches(a, ceil_div(a.rows, 256 / f.lanes), [&](const RowArgs& a, unsigned grid) {
        if (f.nv == 0) {
            if (bf) k_norm_long<bf16_t><<<grid, 256, 0, st>>>(a);
            else k_norm_long<float><<<grid, 256, 0, st>>>(a);
        } else if (bf) run_rows_t<bf16_t>(a, vec, f, false, grid, st);
        else run_rows_t<float>(a, vec, f, false, grid, st);
    });
}

void norm_backward(const ftp_norm_shape& s, const void* dy, const void* x, const int8_t* codes, const int8_t* exponents, int block, const void* gamma,
                   const float* mean, const float* rstd, void* dx, float* dgamma, float* dbeta, float* partial, hipStream_t st)
{
    const bool bf = s.dtype == FTP_BF16;
    const Strides t = strides_of(s, true, codes != nullptr);
    int shares = 0;
    if (s.outer == 0 || s.inner == 0) {             // (sums of nothing)
    } else if (!by_rows(t, s.channels)) {
        TileArgs a = tile_args(s, t, true);
        a.x = x; a.gamma = gamma; a.dy = dy; a.dx = dx; a.mean = (float*)mean; a.rstd = (float*)rstd;
        a.partial = dgamma ? partial : nullptr;
        a.xvec = tile_vec(s, t.x, a.px, x); a.yvec = tile_vec(s, t.y, a.px, dx); a.gvec = tile_vec(s, t.g, a.px, dy);
        shares = (int)std::min<long long>(kShares, s.outer * a.tiles);
        if (bf) k_norm_back_tiles<bf16_t><<<shares, 256, tile_bytes(s, a.px, true), st>>>(a);
        else k_norm_back_tiles<float><<<shares, 256, tile_bytes(s, a.px, true), st>>>(a);
    } else {
        RowArgs a = row_args(s, t);
        a.x = x; a.gamma = gamma; a.dy = dy; a.dx = dx; a.mean = (float*)mean; a.rstd = (float*)rstd;
        a.codes = codes; a.exps = exponents;
        if (codes) { a.block = block; a.nblocks = (a.C + block - 1) / block; }
        a.partial = dgamma ? partial : nullptr;
        const void* ptrs[] = {x, gamma, dy, dx};
        const int vec = row_vec(a, bf ? 2 : 4, ptrs, 4, codes);
        const RowForm f = row_form(a.C, vec);
        a.lanes = f.lanes;
        if (f.nv == 0) {
            shares = (int)std::min<long long>(64, a.rows);
            const dim3 grid((a.C + 255) / 256, shares);
            if (a.partial) {                        // (first: dx may overwrite dy)
                if (bf) k_norm_long_params<bf16_t><<<grid, 256, 0, st>>>(a, shares);
                else k_norm_long_params<float><<<grid, 256, 0, st>>>(a, shares);
            }
            by_launches(a, a.rows, [&](const RowArgs& a, unsigned grid) {
                if (bf) k_norm_back_long<bf16_t><<<grid, 256, 0, st>>>(a);
                else k_norm_back_long<float><<<grid, 256, 0, st>>>(a);
            });
        } else {
            shares = (int)std::min<long long>(kShares, ceil_div(a.rows, f.wide ? 1 : kBackThreads / f.lanes));
            if (bf) run_rows_t<bf16_t>(a, vec, f, true, shares, st);
            else run_rows_t<float>(a, vec, f, true, shares, st);
        }
    }
    if (dgamma) k_norm_params<<<(2 * s.channels + 31) / 32, 1024, 0, st>>>(partial, shares, s.channels, dgamma, dbeta);
}

}  // namespace ftp
