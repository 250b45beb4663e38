// Activations held in 8 bits: a block of neighbours of a row has the smallest exponent e >= -126 with max|x| <= 127 * 2^e, a value its code
// q = round(x / 2^e) and stands for q * 2^e.  A scale that is a power of two costs up to one bit of a code against max|x| / 127, and gives: a scale of one byte; codes and values without
// any other rounding (the quotient is exact, and so is q * 2^e as a bfloat), so that a matrix product can take the values as bfloat operands.
// Bound by memory: packing reads a value and writes a byte, the others read a byte (and dy) and write a value.  A lane takes 8 neighbours, 2^k lanes a
// block; no LDS.  Measured at 189 million fp32 values, blocks of 128: packing 187 us (946 MB, 5.1 TB/s), unpacking 170 us (5.6 TB/s; a large copy: 4.8); GELU's derivative of 46208 x 1024 bfloats 45 us
// (237 MB, 5.2 TB/s): its 20 vector instructions and two transcendental ones a value stay below the memory's time.
#include "ftp_tokens.h"

#include <algorithm>

namespace ftp {
namespace {

struct HeldArgs {
    const void* x; void* out; const void* dy;
    int8_t* codes; int8_t* exps;
    long long rows, cols, stride;
    uint32_t units;                                 // lanes' worth of work a row: blocks * block / 8
    uint32_t total;                                 // ... of the launch
    int nblocks, lg;                                // a block is 2^lg lanes
    float slope;
};

// Exponent of a block whose largest magnitude has these bits.
__device__ __forceinline__ int exponent_of(uint32_t bits)
{
    if (bits >= 0x7F800000u) return 127;
    // bits = 1.m * 2^p: 1.m <= 127 / 64 goes with 2^(p - 6); smaller numbers than 2^-120 (zero and denormals too) with the smallest exponent
    const int e = (int)(bits >> 23) - 127 - ((bits & 0x7FFFFFu) <= 0x7E0000u ? 6 : 5);
    return max(e, -126);
}

// The Gauss function's integral and density: Phi(x) by Abramowitz and Stegun's formula 7.1.26 (error of erf below 1.5e-7), whose exponential is the density's.
__device__ __forceinline__ void gauss(float x, float& phi, float& density)
{
    const float z = fabsf(x) * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.0f));
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float e = __builtin_amdgcn_exp2f(z * z * -1.44269504f);
    const float tail = 0.5f * p * e;                // 1 - Phi(|x|)
    phi = x < 0 ? tail : 1.0f - tail;
    density = 0.39894228f * e;
}
__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + __builtin_amdgcn_exp2f(x * -1.44269504f)); }

template <int ACT>
__device__ __forceinline__ float act(float x, float slope)
{
    if constexpr (ACT == FTP_ACT_LEAKY) return leaky(x, slope);
    if constexpr (ACT == FTP_ACT_GELU) { float p, d; gauss(x, p, d); return x * p; }
    if constexpr (ACT == FTP_ACT_SILU) return x * sigmoid(x);
    return x;
}
template <int ACT>
__device__ __forceinline__ float act_derivative(float x, float slope)
{
    if constexpr (ACT == FTP_ACT_LEAKY) return x > 0.0f ? 1.0f : x <= 0.0f ? slope : x;     // (NaN stays NaN)
    if constexpr (ACT == FTP_ACT_GELU) { float p, d; gauss(x, p, d); return fmaf(x, d, p); }
    if constexpr (ACT == FTP_ACT_SILU) { const float s = sigmoid(x); return fmaf(x * s, 1.0f - s, s); }
    return x == x ? 1.0f : x;
}

struct Place { long long row; int col, n; };       // 8 neighbours from col on, n of them inside the row
__device__ __forceinline__ Place place(const HeldArgs& a, uint32_t u)
{
    Place p;
    const uint32_t r = u / a.units;
    p.row = r;
    const long long col = (long long)(u - r * a.units) * 8;
    p.col = (int)col;
    p.n = (int)max(0ll, min(8ll, a.cols - col));
    return p;
}

// 8 neighbours, n of which are there.  VECTOR: sizes and addresses are whole vectors of 16 (codes 8) bytes, all 8 are there or none.  Otherwise 8 go at once where they are there,
// at any address, and the last ones of a row one by one (4000 rows of 5001: 38 us there and back; element by element everywhere 101; 189 million in aligned rows: unpacking 167 us
// with VECTOR, 232 without).
template <typename T, bool VECTOR>
__device__ __forceinline__ void load8(float (&v)[8], const T* p, int n)
{
    Pack<T, 8> w;
    w.zero();
    if constexpr (VECTOR) { if (n > 0) w.load(p); }
    else if (n == 8) w.load_any(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = w.get(i);
    if (VECTOR || n == 8) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        Pack<T, 1> e;
        e.zero();
        if (i < n) e.load(p + i);
        v[i] = e.get(0);
    }
}
template <typename T, bool VECTOR>
__device__ __forceinline__ void store8(const float (&v)[8], T* p, int n)
{
    if (VECTOR || n == 8) {
        Pack<T, 8> w;
        w.put(v);
        if constexpr (VECTOR) w.store(p);
        else w.store_any(p);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) st(p + i, v[i]);
}

template <typename T, bool VECTOR>
__global__ __launch_bounds__(256) void k_held_pack(const HeldArgs a)
{
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    const bool live = u < a.total;
    const Place p = place(a, live ? u : 0);
    const int n = live ? p.n : 0;
    float v[8];
    load8<T, VECTOR>(v, (const T*)a.x + p.row * a.stride + p.col, n);
    // the largest magnitude as bits: NaN and infinities come out above all numbers
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    for (int m = 1; m < (1 << a.lg); m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    const int e = exponent_of(top);
    const float per = e == 127 ? 0.0f : __uint_as_float((uint32_t)(127 - e) << 23), most = e == 122 ? 63.0f : 127.0f;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = e == 127 ? 0.0f : fminf(fmaxf(rintf(v[i] * per), -most), most);
        w[i / 4] |= ((uint32_t)(int)q & 0xFFu) << (8 * (i & 3));
    }
    if (n <= 0) return;
    int8_t* c = a.codes + p.row * a.cols + p.col;
    if (VECTOR || n == 8) {
        Pack<int8_t, 8> o;
        o.w[0] = {w[0], w[1]};
        if constexpr (VECTOR) o.store(c);
        else o.store_any(c);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) c[i] = (int8_t)(w[i / 4] >> (8 * (i & 3)));
    }
    const uint32_t unit = u - (uint32_t)p.row * a.units;
    if ((unit & ((1u << a.lg) - 1)) == 0) a.exps[p.row * a.nblocks + (unit >> a.lg)] = (int8_t)e;
}

// out = act(value), or dy times the derivative there.
template <typename T, bool VECTOR, int ACT, bool BACK>
__global__ __launch_bounds__(256) void k_held_act(const HeldArgs a)
{
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    if (u >= a.total) return;
    const Place p = place(a, u);
    if (p.n <= 0) return;
    float v[8], y[8];
    const int e = a.exps[p.row * a.nblocks + (p.col >> (a.lg + 3))];
    load8<int8_t, VECTOR>(v, (const int8_t*)a.codes + p.row * a.cols + p.col, p.n);
    const float unit = held_scale(e);
    const long long at = p.row * a.stride + p.col;
    if constexpr (BACK) load8<T, VECTOR>(y, (const T*)a.dy + at, p.n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = BACK ? y[i] * act_derivative<ACT>(v[i] * unit, a.slope) : act<ACT>(v[i] * unit, a.slope);
    store8<T, VECTOR>(v, (T*)a.out + at, p.n);
}

HeldArgs held_args(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exps)
{
    HeldArgs a = {};
    a.codes = (int8_t*)codes; a.exps = (int8_t*)exps;
    a.rows = s.rows; a.cols = s.cols; a.stride = s.stride;
    // rows that follow each other and end with a block are one long row (fewer, fuller ones), as far as 32-bit columns go
    if (a.stride == a.cols && a.cols % s.block == 0) {
        while (a.rows % 2 == 0 && a.cols * 2 <= (1ll << 30)) { a.rows /= 2; a.cols *= 2; a.stride *= 2; }
        if (a.cols * a.rows <= (1ll << 30)) { a.cols = a.stride = a.cols * a.rows; a.rows = 1; }
    }
    a.nblocks = (int)ceil_div(a.cols, s.block);
    a.units = (uint32_t)a.nblocks * (uint32_t)(s.block / 8);
    while ((8 << a.lg) < s.block) ++a.lg;
    return a;
}

bool by_vectors(const HeldArgs& a, const void* p, const void* q) { return a.cols % 8 == 0 && a.stride % 8 == 0 && aligned(p, 16) && aligned(q, 16) && aligned(a.codes, 8); }

// One launch for as many rows as 32-bit numbers of lanes allow.
template <class F>
void by_launches(HeldArgs a, int es, F launch)
{
    const long long most = std::max(1ll, (1ll << 31) / a.units);
    for (long long row = 0; row < a.rows; row += most) {
        HeldArgs b = a;
        b.rows = std::min(most, a.rows - row);
        b.total = (uint32_t)(b.rows * a.units);
        b.codes += row * a.cols; b.exps += row * a.nblocks;
        if (b.x) b.x = (const char*)b.x + row * a.stride * es;
        if (b.dy) b.dy = (const char*)b.dy + row * a.stride * es;
        if (b.out) b.out = (char*)b.out + row * a.stride * es;
        launch(b, (b.total + 255u) / 256u);
    }
}

template <typename T, bool BACK, int ACT>
void run_act(const HeldArgs& a, hipStream_t st)
{
    const bool vec = by_vectors(a, BACK ? a.dy : a.out, a.out);
    by_launches(a, sizeof(T), [&](const HeldArgs& b, unsigned grid) {
        if (vec) k_held_act<T, true, ACT, BACK><<<grid, 256, 0, st>>>(b);
        else k_held_act<T, false, ACT, BACK><<<grid, 256, 0, st>>>(b);
    });
}

template <typename T, bool BACK>
void run_acts(const HeldArgs& a, int act, hipStream_t st)
{
    switch (act) {
        case FTP_ACT_LEAKY: run_act<T, BACK, FTP_ACT_LEAKY>(a, st); break;
        case FTP_ACT_GELU: run_act<T, BACK, FTP_ACT_GELU>(a, st); break;
        case FTP_ACT_SILU: run_act<T, BACK, FTP_ACT_SILU>(a, st); break;
        default: run_act<T, BACK, FTP_ACT_NONE>(a, st); break;
    }
}

}  // namespace

void held_pack(const ftp_checkpoint_shape& s, const void* x, int8_t* codes, int8_t* exponents, hipStream_t st)
{
    HeldArgs a = held_args(s, codes, exponents);
    a.x = x;
    const bool vec = by_vectors(a, x, x), bf = s.dtype == FTP_BF16;
    by_launches(a, bf ? 2 : 4, [&](const HeldArgs& b, unsigned grid) {
        if (bf && vec) k_held_pack<bf16_t, true><<<grid, 256, 0, st>>>(b);
        else if (bf) k_held_pack<bf16_t, false><<<grid, 256, 0, st>>>(b);
        else if (vec) k_held_pack<float, true><<<grid, 256, 0, st>>>(b);
        else k_held_pack<float, false><<<grid, 256, 0, st>>>(b);
    });
}

void held_unpack(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exponents, int act, float slope, void* out, hipStream_t st)
{
    HeldArgs a = held_args(s, codes, exponents);
    a.out = out; a.slope = slope;
    if (s.dtype == FTP_BF16) run_acts<bf16_t, false>(a, act, st);
    else run_acts<float, false>(a, act, st);
}

void held_act_backward(const ftp_checkpoint_shape& s, const int8_t* codes, const int8_t* exponents, int act, float slope, const void* dy, void* dx, hipStream_t st)
{
    HeldArgs a = held_args(s, codes, exponents);
    a.dy = dy; a.out = dx; a.slope = slope;
    if (s.dtype == FTP_BF16) run_acts<bf16_t, true>(a, act, st);
    else run_acts<float, true>(a, act, st);
}

}  // namespace ftp
