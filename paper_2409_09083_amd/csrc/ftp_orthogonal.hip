// Newton-Schulz steps towards the orthogonal part of a matrix: X <- a X + (b S + c S^2) X with S = X X^T, or, where X is taller than wide, X <- a X + X (b S + c S^2) with S = X^T X.  Neither needs a transposed copy: a product's
// operand may lie either way (ftp_product.h).
//
// A step is three products.  Errors of X, S and their products meet a factor of up to a (3.4) a step where singular values are small, so numbers go from one product to the next as
// three bfloats (fp32: 24 bits, six products of planes) or two (bfloat: 16 bits, three), and sums are fp32.  S and b S + c S^2 are symmetric: blocks on and below the diagonal are multiplied, the others are mirrored.
// Products with too few blocks for the chip are cut along their contraction, whose shares a second kernel adds up.
#include "ftp_training.h"
#include "ftp_product.h"

#include <algorithm>
#include <cmath>

namespace ftp {
namespace {

template <int B, bool XA, bool XB> struct BlockOf;
template <bool XA, bool XB> struct BlockOf<256, XA, XB> { typedef Product<256, 256, 2, 4, XA, XB> type; };
template <bool XA, bool XB> struct BlockOf<128, XA, XB> { typedef Product<128, 128, 2, 2, XA, XB> type; };
template <bool XA, bool XB> struct BlockOf<64, XA, XB> { typedef Product<64, 64, 2, 2, XA, XB> type; };

// A part of each matrix' sum of squares a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void k_squares(const T* x, long long mstride, long long rstride, int rows, int cols, int parts, double* sums)
{
    __shared__ double lds[4];
    const int matrix = blockIdx.x / parts, part = blockIdx.x - matrix * parts;
    const long long n = (long long)rows * cols, lo = n * part / parts, hi = n * (part + 1) / parts;
    x += matrix * mstride;
    double s = 0;
    for (long long u = lo + threadIdx.x; u < hi; u += 256) {
        const long long r = u / cols;
        const double v = ld(x + r * rstride + (u - r * cols));
        s = fma(v, v, s);
    }
#pragma unroll
    for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) sums[blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}

// x / (|x| + eps) as planes, with zeros up to whole blocks of 64.
template <typename T, int P>
__global__ __launch_bounds__(256) void k_normed(const T* x, long long mstride, long long rstride, int rows, int cols, int parts, const double* sums, double eps, bf16_t* to, int Rp, int Cp, long long plane)
{
    const int matrix = blockIdx.y;
    double total = 0;
    for (int i = 0; i < parts; ++i) total += sums[matrix * parts + i];
    const double inv = 1.0 / (sqrt(total) + eps);
    const int per = Cp >> 3;
    x += matrix * mstride;
    to += (long long)matrix * Rp * Cp;
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < (long long)Rp * per; u += (long long)gridDim.x * 256) {
        const int r = (int)(u / per), c0 = (int)(u - (long long)r * per) * 8;
        uint32_t q[4][P];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = c0 + 2 * j + e;
                v[e] = r < rows && c < cols ? (float)(ld(x + r * rstride + c) * inv) : 0.0f;
            }
            planes_of<P>(v[0], v[1], q[j]);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) *(uint4*)(to + p * plane + ((long long)(c0 >> 5) * Rp + r) * 32 + (c0 & 31)) = uint4{q[0][p], q[1][p], q[2][p], q[3][p]};
    }
}

struct StepArgs {
    Matrix a, b;                                    // of the first matrix
    long long anext, bnext;                         // elements to the next one's
    int planes, stages, shares, count, ablocks, bblocks;
    int symmetric;                                  // blocks below the diagonal are mirrored instead
    // what becomes of the sums v: f0 old + f1 v, old being planes too
    float f0, f1;
    const bf16_t* old; bf16_t* to;
    long long plane, next; int stride, arows, brows;        // (old and to: a Matrix of brows rows and arows columns each) [matrix: next]
    void* out; int orows, ocols;                    // instead of planes: the results, rows along b
    float* part; long long pshare;                  // [share][matrix][index of b][stride]
};

template <int P>
__device__ __forceinline__ f32x4 planes_sum(const bf16_t* p, long long plane)
{
    f32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int k = P - 1; k >= 0; --k) {
        const uint2 w = *(const uint2*)(p + k * plane);
        v += f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u)};
    }
    return v;
}

// Four neighbouring results: (matrix, j: index along b, i: first index along a)
template <typename T, int P>
__device__ __forceinline__ void finish(const StepArgs& a, int matrix, int i, int j, f32x4 v, bool mirror)
{
    const long long block = a.brows * 32ll, at = matrix * a.next + (i >> 5) * block + j * 32 + (i & 31);
    v *= a.f1;
    if (a.f0 != 0) v += a.f0 * planes_sum<P>(a.old + at, a.plane);
    if (a.out) {
        T* p = (T*)a.out + ((long long)matrix * a.orows + j) * a.ocols + i;
        if (j < a.orows)
#pragma unroll
            for (int e = 0; e < 4; ++e) if (i + e < a.ocols) st(p + e, v[e]);
        return;
    }
    uint32_t x[P], y[P];
    planes_of<P>(v[0], v[1], x);
    planes_of<P>(v[2], v[3], y);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        bf16_t* to = a.to + p * a.plane;
        *(uint2*)(to + at) = uint2{x[p], y[p]};
        if (mirror) {
            bf16_t* m = to + matrix * a.next + (j >> 5) * block + i * 32 + (j & 31);
            m[0] = (bf16_t)x[p];
            m[32] = (bf16_t)(x[p] >> 16);
            m[64] = (bf16_t)y[p];
            m[96] = (bf16_t)(y[p] >> 16);
        }
    }
}

template <class L, typename T, int P>
__global__ __launch_bounds__(L::kThreads, 2) void k_step(const StepArgs a)
{
    __shared__ __align__(16) typename L::Stage s0, s1, s2, s3;
    int ia, ib, matrix, share = 0;
    if (a.symmetric) {
        const int per = a.ablocks * (a.ablocks + 1) / 2;
        int t;
        if (!block_of((int)blockIdx.x, per, a.count, t, matrix)) return;
        ib = 0;
        while (t > ib) t -= ++ib;                   // row ib has ib + 1 blocks
        ia = t;
    } else {
        int g;
        if (!block_of((int)blockIdx.x, a.ablocks, a.bblocks * a.shares * a.count, ia, g)) return;
        ib = g % a.bblocks;
        g /= a.bblocks;
        share = g % a.shares;
        matrix = g / a.shares;
    }
    const int a0 = ia * L::BA, b0 = ib * L::BB;
    Matrix x = a.a, y = a.b;
    x.p += matrix * a.anext;
    y.p += matrix * a.bnext;
    f32x16 acc[L::IA][L::IB] = {};
    L::run(acc, x, y, a0, b0, (int)((long long)a.stages * share / a.shares), (int)((long long)a.stages * (share + 1) / a.shares), a.planes, s0, s1, s2, s3);
    L::each(acc, [&](int i, int j, f32x4 v) __attribute__((always_inline)) {
        i += a0;
        j += b0;
        if (i >= a.arows || j >= a.brows) return;
        if (a.shares > 1) *(f32x4*)(a.part + share * a.pshare + matrix * a.next + (long long)j * a.stride + i) = v;
        else finish<T, P>(a, matrix, i, j, v, a.symmetric && ia != ib);
    });
}

template <typename T, int P>
__global__ __launch_bounds__(256) void k_step_sum(const StepArgs a)
{
    const long long n = a.count * a.next / 4;
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < n; u += (long long)gridDim.x * 256) {
        const int matrix = (int)(4 * u / a.next), in = (int)(4 * u - matrix * a.next), j = in / a.stride;
        f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
        for (int s = 0; s < a.shares; ++s) v += *(const f32x4*)(a.part + s * a.pshare + 4 * u);
        finish<T, P>(a, matrix, in - j * a.stride, j, v, false);
    }
}

struct Plan {
    int planes, Rp, Cp, m, mp, parts;
    bool tall;
    Split s, q, x;                                  // of S, its square, X
};
Split symmetric_or_split(int m, long long stages, int count)
{
    // (a symmetric product is not cut as well)
    const Split half = split_of(m, (m + 1) / 2, stages, 64, 1, count), cut = split_of(m, m, stages, 64, 16, count);
    const auto blocks = [&](int b) { const long long n = ceil_div(m, b); return n * (n + 1) / 2 * count; };
    return cut.shares > 1 && blocks(half.block) * 2 < 256 ? cut : Split{half.block, 1};
}
Plan plan_of(const ftp_orthogonal_shape& s)
{
    Plan p = {};
    p.planes = s.dtype == FTP_BF16 ? 2 : 3;
    p.Rp = (s.rows + 63) & ~63;
    p.Cp = (s.cols + 63) & ~63;
    p.tall = s.rows > s.cols;
    p.m = std::min(s.rows, s.cols);
    p.mp = (p.m + 63) & ~63;
    p.parts = (int)std::min<long long>(256, ceil_div((long long)s.rows * s.cols, 4096));
    const long long terms = p.planes == 2 ? 3 : 6, longer = std::max(p.Rp, p.Cp);
    p.s = symmetric_or_split(p.m, longer / 32 * terms, s.count);
    p.q = symmetric_or_split(p.m, p.mp / 32 * terms, s.count);
    p.x = split_of(s.cols, s.rows, p.mp / 32 * terms, 64, 16, s.count);
    return p;
}

struct Buffers { double* sums; bf16_t *x[2], *s, *q; float* part; size_t bytes; };
Buffers buffers_of(const ftp_orthogonal_shape& s, const Plan& p, char* ws)
{
    Buffers b = {};
    Parts t(ws);
    const size_t x = (size_t)s.count * p.Rp * p.Cp, q = (size_t)s.count * p.mp * p.mp;
    b.sums = t.take<double>((size_t)s.count * p.parts);
    for (auto& e : b.x) e = t.take<bf16_t>(p.planes * x);
    b.s = t.take<bf16_t>(p.planes * q);
    b.q = t.take<bf16_t>(p.planes * q);
    const auto shares = [](const Split& k) { return k.shares > 1 ? (size_t)k.shares : 0; };
    b.part = t.take<float>(std::max({shares(p.s) * q, shares(p.q) * q, shares(p.x) * x}));
    b.bytes = t.used;
    return b;
}

template <int B, bool XA, bool XB, typename T, int P>
void launch(StepArgs& a, hipStream_t st)
{
    typedef typename BlockOf<B, XA, XB>::type L;
    a.ablocks = (int)ceil_div(a.arows, B);
    a.bblocks = (int)ceil_div(a.brows, B);
    const long long grid = a.symmetric ? block_grid((long long)a.ablocks * (a.ablocks + 1) / 2, a.count) : block_grid(a.ablocks, (long long)a.bblocks * a.shares * a.count);
    k_step<L, T, P><<<(unsigned)grid, L::kThreads, 0, st>>>(a);
    if (a.shares > 1) k_step_sum<T, P><<<(unsigned)std::min<long long>(ceil_div(a.count * a.next, 1024), 8192), 256, 0, st>>>(a);
}
template <bool XA, bool XB, typename T, int P>
void product(StepArgs& a, const Split& s, hipStream_t st)
{
    a.shares = s.shares;
    a.symmetric = a.symmetric && s.shares == 1;
    if (s.block == 256) launch<256, XA, XB, T, P>(a, st);
    else if (s.block == 128) launch<128, XA, XB, T, P>(a, st);
    else launch<64, XA, XB, T, P>(a, st);
}

template <typename T, int P>
void run(const ftp_orthogonal_shape& s, const T* x, T* out, char* ws, hipStream_t st)
{
    const Plan p = plan_of(s);
    const Buffers b = buffers_of(s, p, ws);
    const long long xnext = (long long)p.Rp * p.Cp, xplane = s.count * xnext, qnext = (long long)p.mp * p.mp, qplane = s.count * qnext;
    k_squares<T><<<(unsigned)(s.count * p.parts), 256, 0, st>>>(x, s.matrix_stride, s.row_stride, s.rows, s.cols, p.parts, b.sums);
    k_normed<T, P><<<dim3((unsigned)std::min<long long>(ceil_div(xnext, 2048), 4096), (unsigned)s.count), 256, 0, st>>>(x, s.matrix_stride, s.row_stride, s.rows, s.cols, p.parts, b.sums, s.eps, b.x[0], p.Rp, p.Cp, xplane);
    const Matrix S = blocked(b.s, p.mp, p.mp, qplane), Q = blocked(b.q, p.mp, p.mp, qplane);
    for (int step = 0; step < s.steps; ++step) {
        const Matrix X = blocked(b.x[step & 1], p.Rp, p.Cp, xplane);
        StepArgs k = {};
        k.planes = P; k.count = s.count; k.part = b.part;
        k.stride = k.arows = k.brows = p.mp; k.next = qnext; k.plane = qplane; k.pshare = qplane;
        // S
        k.a = k.b = X; k.anext = k.bnext = xnext; k.stages = std::max(p.Rp, p.Cp) / 32; k.symmetric = 1; k.f1 = 1; k.to = b.s;
        if (p.tall) product<true, true, T, P>(k, p.s, st);
        else product<false, false, T, P>(k, p.s, st);
        // b S + c S^2
        k.a = k.b = S; k.anext = k.bnext = qnext; k.stages = p.mp / 32; k.symmetric = 1; k.f0 = s.b; k.f1 = s.c; k.old = b.s; k.to = b.q;
        product<false, false, T, P>(k, p.q, st);
        // a X + that times X
        k.symmetric = 0; k.f0 = s.a; k.f1 = 1; k.old = b.x[step & 1]; k.to = b.x[~step & 1];
        k.stride = k.arows = p.Cp; k.brows = p.Rp; k.next = xnext; k.plane = xplane; k.pshare = xplane;
        if (step + 1 == s.steps) { k.out = out; k.orows = s.rows; k.ocols = s.cols; }
        if (p.tall) {
            k.a = Q; k.b = X; k.anext = qnext; k.bnext = xnext;
            product<false, false, T, P>(k, p.x, st);
        } else {
            k.a = X; k.b = Q; k.anext = xnext; k.bnext = qnext;
            product<true, false, T, P>(k, p.x, st);
        }
    }
}

}  // namespace

bool orthogonal_fits(const ftp_orthogonal_shape& s)
{
    if (s.rows > 32768 || s.cols > 32768 || s.steps > 64 || s.count > 65535) return false;
    // launches of fewer than 2^32 threads
    return (double)s.count * (double)ceil_div(s.rows, 64) * (double)ceil_div(s.cols, 64) < (1 << 23);
}
size_t orthogonal_workspace(const ftp_orthogonal_shape& s) { return buffers_of(s, plan_of(s), nullptr).bytes; }
void orthogonal(const ftp_orthogonal_shape& s, const void* x, void* out, char* ws, hipStream_t st)
{
    if (s.dtype == FTP_BF16) run<bf16_t, 2>(s, (const bf16_t*)x, (bf16_t*)out, ws, st);
    else run<float, 3>(s, (const float*)x, (float*)out, ws, st);
}

}  // namespace ftp
