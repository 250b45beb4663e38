// Newton-Schulz steps towards the orthogonal part of a matrix: X <- (a I + b S + c S^2) X with S = X X^T, or, where X is taller than wide, X <- X (a I + b S + c S^2) with S = X^T X.  Neither needs a transposed copy: a product's
// operand may lie either way (ftp_product.h).
//
// A step is three products.  Errors of X, S and their products meet a factor of up to a (3.4) a step where singular values are small, so numbers go from one product to the next as
// three bfloats (fp32: 24 bits, six products of planes) or two (bfloat: 16 bits, three), and sums are fp32.  Of 16 bits nothing is seen behind the result's 8: 4096 x 4096, 1024 x 4096 and 64 x 576 are off by 0.001659, 0.001656 and 0.001670 of
// their norm, as much as the 64-bit result rounded once (1 % of the elements are its neighbours; with 24 bits 0.3 %, in 7.58 ms instead of 3.90).  a goes into the second one's diagonal, so that the third needs no more than its sums.  S and its polynomial are symmetric: blocks on and below the diagonal are multiplied, the others are mirrored.
// Blocks that do not fill a last round of the chip (all, of small products) are cut along their contraction, whose shares a second kernel adds up.
//
// Measured, a step: 4096 x 4096 held in 16 bits S and its polynomial 220 us each (0.96 PFLOP/s of bfloats), X 307 (1.34); 4 x 512 x 2048 fp32 S 29, polynomial 17, X 34; 3 x 707 x 133 fp32 10, 9, 8.
#include "ftp_training.h"
#include "ftp_orthogonal.h"

#include <algorithm>
#include <cmath>

namespace ftp {
namespace {

template <int B, bool XA, bool XB> struct BlockOf;
template <bool XA, bool XB> struct BlockOf<256, XA, XB> { typedef Product<256, 256, 2, 4, XA, XB> type; };
template <bool XA, bool XB> struct BlockOf<128, XA, XB> { typedef Product<128, 128, 2, 2, XA, XB> type; };
template <bool XA, bool XB> struct BlockOf<64, XA, XB> { typedef Product<64, 64, 2, 2, XA, XB, 64> type; };

// A part of each matrix' rows' sum of squares a workgroup: 32 lanes a row.
template <typename T>
__global__ __launch_bounds__(256) void k_squares(const T* x, long long mstride, long long rstride, int rows, int cols, int parts, double* sums)
{
    constexpr int E = 16 / (int)sizeof(T);
    __shared__ double lds[4];
    const int matrix = blockIdx.x / parts, part = blockIdx.x - matrix * parts;
    x += matrix * mstride;
    double s = 0;
    for (int r = part * 8 + (threadIdx.x >> 5); r < rows; r += parts * 8) {
        const T* p = x + r * rstride;
#pragma unroll 4
        for (int c = (threadIdx.x & 31) * E; c < cols; c += 32 * E) {
            if (c + E <= cols) {
                Pack<T, E> v;
                v.load_any(p + c);
#pragma unroll
                for (int e = 0; e < E; ++e) { const double d = v.get(e); s = fma(d, d, s); }
            } else
                for (int e = c; e < cols; ++e) { const double d = ld(p + e); s = fma(d, d, s); }
        }
    }
#pragma unroll
    for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) sums[blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}

// x / (|x| + eps) as planes, laid out for the products, with zeros up to whole blocks of 64: 64 rows x 32 columns at a time.
template <typename T, int P>
__global__ __launch_bounds__(256) void k_normed(const T* x, long long mstride, long long rstride, int rows, int cols, int parts, const double* sums, double eps, bf16_t* to, int Rp, int Cp, long long plane)
{
    const int matrix = blockIdx.y;
    const double inv = inverse_norm(sums + (long long)matrix * parts, parts, eps);
    const int across = Cp >> 5, tiles = across * (Rp >> 6), r_in = threadIdx.x >> 2, c_in = (threadIdx.x & 3) * 8;
    x += matrix * mstride;
    to += (long long)matrix * Rp * Cp;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int rb = t / across, cb = t - rb * across, r = rb * 64 + r_in, c0 = cb * 32 + c_in;
        float v[8] = {};
        if (r < rows) {
            const T* p = x + r * rstride + c0;
            if (c0 + 8 <= cols) {
                Pack<T, 8> w;
                w.load_any(p);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (float)(w.get(e) * inv);
            } else
#pragma unroll
                for (int e = 0; e < 8; ++e) if (c0 + e < cols) v[e] = (float)(ld(p + e) * inv);
        }
        uint32_t q[4][P];
#pragma unroll
        for (int j = 0; j < 4; ++j) planes_of<P>(v[2 * j], v[2 * j + 1], q[j]);
#pragma unroll
        for (int k = 0; k < P; ++k) *(uint4*)(to + k * plane + ((long long)cb * Rp + r) * 32 + c_in) = uint4{q[0][k], q[1][k], q[2][k], q[3][k]};
    }
}

struct StepArgs {
    Matrix a, b;                                    // of the first matrix
    long long anext, bnext;                         // elements to the next one's
    Terms terms;
    int stages, count, ablocks, bblocks;            // stages of 32, an even number
    int blocks, whole, shares;                      // blocks of all matrices; the first `whole` of them by a workgroup each, the others by `shares`
    int groups, grouped;                            // those others: groups (matrices) x blocks
    int symmetric;                                  // blocks above the diagonal are mirrored ones
    // what becomes of the sums v: themselves, or (old not null) diagonal I + f0 old + f1 v, old being planes too
    float f0, f1;
    float diagonal, spare;                          // (three floats in a row had the compiler keep a copy of them in LDS: 4 x 512 x 2048 468 -> 600 us)
    const bf16_t* old; bf16_t* to;
    long long plane, next; int arows, brows;        // (old and to: a Matrix of brows rows and arows columns each) [matrix: next]
    void* out; int orows, ocols;                    // instead of planes: the results, rows along b
    float* part;                                    // sums: [block that is cut][share]
};

// Eight neighbouring results: (matrix, j: index along b, i: first index along a)
template <typename T, int P>
__device__ __forceinline__ void finish(const StepArgs& a, int matrix, int i, int j, float (&v)[8], bool mirror)
{
    const long long block = a.brows * 32ll, at = matrix * a.next + (i >> 5) * block + j * 32 + (i & 31);
    if (a.old) {
        uint4 w[P];
#pragma unroll
        for (int p = 0; p < P; ++p) w[p] = *(const uint4*)(a.old + at + p * a.plane);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float old = 0;
#pragma unroll
            for (int p = P - 1; p >= 0; --p) {
                const uint32_t x = e < 2 ? w[p].x : e < 4 ? w[p].y : e < 6 ? w[p].z : w[p].w;
                old += __uint_as_float(e & 1 ? x & 0xFFFF0000u : x << 16);
            }
            v[e] = fmaf(a.f1, v[e], a.f0 * old) + (i + e == j ? a.diagonal : 0.0f);
        }
    }
    if (a.out) {
        if (j < a.orows) store8((T*)a.out + ((long long)matrix * a.orows + j) * a.ocols + i, a.ocols - i, v);
        return;
    }
    bf16_t* to = a.to + at;
    if (!mirror) {
        store_planes<P>(to, a.plane, v);
        return;
    }
    uint32_t x[4][P];
#pragma unroll
    for (int e = 0; e < 4; ++e) planes_of<P>(v[2 * e], v[2 * e + 1], x[e]);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        *(uint4*)(to + p * a.plane) = uint4{x[0][p], x[1][p], x[2][p], x[3][p]};
        bf16_t* m = a.to + p * a.plane + matrix * a.next + (j >> 5) * block + i * 32 + (j & 31);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[32 * e] = (bf16_t)(x[e >> 1][p] >> (16 * (e & 1)));
    }
}

// Which matrix and block: neighbours in the list share operands.
__device__ __forceinline__ void step_block(const StepArgs& a, int t, int& ia, int& ib, int& matrix)
{
    const int per = a.blocks / a.count;
    matrix = t / per;
    t -= matrix * per;
    if (a.symmetric) {
        ib = 0;
        while (t > ib) t -= ++ib;                   // row ib has ib + 1 blocks
        ia = t;
    } else {
        const int wide = 4 * a.ablocks, band = t / wide, in = t - band * wide, high = min(4, a.bblocks - 4 * band);
        ia = in / high;
        ib = 4 * band + in - ia * high;
    }
}

template <class L, typename T, int P>
__global__ __launch_bounds__(L::kThreads, 2) void k_step(const StepArgs a)
{
    __shared__ __align__(16) typename L::Stage s0, s1, s2, s3;
    // XCD x takes the x-th eighth of the whole blocks; behind them come the shares, in eighths too, those of the same part of a matrix one behind the other
    int t, share = 0, shares = 1, index = (int)blockIdx.x;
    const int per = (a.whole + 7) >> 3;
    if (index < 8 * per) {
        t = (index & 7) * per + (index >> 3);
        if (t >= a.whole) return;
    } else {
        shares = a.shares;
        index -= 8 * per;
        const int all = a.groups * shares * a.grouped, each = (all + 7) >> 3, at = (index & 7) * each + (index >> 3);
        if ((index >> 3) >= each || at >= all) return;
        const int g = at / a.grouped;
        share = g % shares;
        t = a.whole + g / shares * a.grouped + at - g * a.grouped;
    }
    int ia, ib, matrix;
    step_block(a, t, ia, ib, matrix);
    const int a0 = ia * L::BA, b0 = ib * L::BB;
    Matrix x = a.a, y = a.b;
    x.p += matrix * a.anext;
    y.p += matrix * a.bnext;
    f32x16 acc[L::IA][L::IB] = {};
    const int stages = a.stages / (L::KS / 32);
    L::run(acc, x, y, a0, b0, (int)((long long)stages * share / shares), (int)((long long)stages * (share + 1) / shares), a.terms, s0, s1, s2, s3);
    if (shares > 1) L::put(acc, a.part + ((long long)(t - a.whole) * shares + share) * L::kSums, false);
    else
        L::each(acc, [&](int i, int j, float (&v)[8]) __attribute__((always_inline)) {
            if (a0 + i < a.arows && b0 + j < a.brows) finish<T, P>(a, matrix, a0 + i, b0 + j, v, a.symmetric && ia != ib);
        });
}

// The shares' sums, in their order.
template <class L, typename T, int P>
__global__ __launch_bounds__(256) void k_step_sum(const StepArgs a)
{
    const int cut = blockIdx.x / L::kParts;
    int ia, ib, matrix;
    step_block(a, a.whole + cut, ia, ib, matrix);
    L::take(a.part + (long long)cut * a.shares * L::kSums, L::kSums, a.shares, blockIdx.x - cut * L::kParts, [&](int i, int j, float (&v)[8]) __attribute__((always_inline)) {
        i += ia * L::BA;
        j += ib * L::BB;
        if (i < a.arows && j < a.brows) finish<T, P>(a, matrix, i, j, v, a.symmetric && ia != ib);
    });
}

// How a product's blocks go over the chip: their size, how many are whole, and the shares of the others.
struct Cut { int block, blocks, whole, shares; };
Cut cut_of(int a, int b, bool symmetric, long long stages, int count)
{
    Cut best = {};
    double least = 1e300;
    for (int block = 256; block >= 64; block /= 2) {
        const int per_cu = block == 256 ? 1 : 2;
        const long long slots = 256 * per_cu, na = ceil_div(a, block), nb = ceil_div(b, block), n = (symmetric ? na * (na + 1) / 2 : na * nb) * count;
        // microseconds a stage with so many workgroups on a CU; 5 for a workgroup's start and end
        const auto stage = [&](long long beside) { return block == 256 ? 0.92 : block == 128 ? 0.13 + 0.2 * (double)beside : 0.05 + 0.09 * (double)beside; };
        const long long whole = n / slots * slots, left = n - whole;
        const double first = (double)(whole / slots) * ((double)stages * stage(per_cu) + 5);
        for (int s = 1; s <= 32 && (s == 1 || stages / s >= 6); ++s) {
            const double last = left ? (double)ceil_div(left * s, slots) * ((double)ceil_div(stages, s) * stage(std::min<long long>(per_cu, ceil_div(left * s, 256))) + 5) : 0;
            const double sum = left && s > 1 ? 5 + 2e-6 * (double)(left * s) * block * block : 0;
            if (first + last + sum < least) {
                least = first + last + sum;
                best = {block, (int)n, (int)(s > 1 ? whole : n), s};
            }
        }
    }
    return best;
}

struct Plan {
    int planes, Rp, Cp, m, mp, parts;
    bool tall;
    Cut s, q, x;                                    // of S, its square, X
};
// Workgroups of a matrix' sum of squares: of 8 rows and more, fewer than 2^23 in all.
int parts_of(const ftp_orthogonal_shape& s) { return (int)std::min<long long>({1024, ceil_div(s.rows, 8), (1 << 23) / std::max(s.count, 1)}); }
Plan plan_of(const ftp_orthogonal_shape& s)
{
    Plan p = {};
    p.planes = s.dtype == FTP_BF16 ? 2 : 3;
    p.Rp = (s.rows + 63) & ~63;
    p.Cp = (s.cols + 63) & ~63;
    p.tall = s.rows > s.cols;
    p.m = std::min(s.rows, s.cols);
    p.mp = (p.m + 63) & ~63;
    p.parts = parts_of(s);
    const long long terms = p.planes == 2 ? 3 : 6, longer = std::max(p.Rp, p.Cp);
    p.s = cut_of(p.mp, p.mp, true, longer / 32 * terms, s.count);
    p.q = cut_of(p.mp, p.mp, true, p.mp / 32 * terms, s.count);
    p.x = cut_of(p.Cp, p.Rp, false, p.mp / 32 * terms, s.count);
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
    const auto shares = [](const Cut& k) { return (size_t)(k.blocks - k.whole) * k.shares * k.block * k.block; };
    b.part = t.take<float>(std::max({shares(p.s), shares(p.q), shares(p.x)}));
    b.bytes = t.used;
    return b;
}

template <int B, bool XA, bool XB, typename T, int P>
void launch(StepArgs& a, hipStream_t st)
{
    typedef typename BlockOf<B, XA, XB>::type L;
    a.ablocks = (int)ceil_div(a.arows, B);
    a.bblocks = (int)ceil_div(a.brows, B);
    const int cut = a.blocks - a.whole;
    a.groups = a.whole ? 1 : a.count;
    a.grouped = cut / a.groups;
    k_step<L, T, P><<<(unsigned)(ceil_div(a.whole, 8) * 8 + ceil_div((long long)cut * a.shares, 8) * 8), L::kThreads, 0, st>>>(a);
    if (cut) k_step_sum<L, T, P><<<(unsigned)(cut * L::kParts), 256, 0, st>>>(a);
}
template <bool XA, bool XB, typename T, int P>
void product(StepArgs& a, const Cut& c, hipStream_t st)
{
    a.blocks = c.blocks;
    a.whole = c.whole;
    a.shares = c.shares;
    if (c.block == 256) launch<256, XA, XB, T, P>(a, st);
    else if (c.block == 128) launch<128, XA, XB, T, P>(a, st);
    else launch<64, XA, XB, T, P>(a, st);
}

template <typename T, int P>
void run(const ftp_orthogonal_shape& s, const T* x, T* out, char* ws, hipStream_t st)
{
    if (orthogonal_is_small(s)) {
        Parts t(ws);
        const int parts = parts_of(s);
        double* sums = t.take<double>((size_t)s.count * parts);
        if (orthogonal_small_sums(s)) k_squares<T><<<(unsigned)(s.count * parts), 256, 0, st>>>(x, s.matrix_stride, s.row_stride, s.rows, s.cols, parts, sums);
        orthogonal_small(s, x, out, sums, parts, t, st);
        return;
    }
    const Plan p = plan_of(s);
    const Buffers b = buffers_of(s, p, ws);
    const long long xnext = (long long)p.Rp * p.Cp, xplane = s.count * xnext, qnext = (long long)p.mp * p.mp, qplane = s.count * qnext;
    k_squares<T><<<(unsigned)(s.count * p.parts), 256, 0, st>>>(x, s.matrix_stride, s.row_stride, s.rows, s.cols, p.parts, b.sums);
    k_normed<T, P><<<dim3((unsigned)std::min<long long>(xnext / 2048, 2048), (unsigned)s.count), 256, 0, st>>>(x, s.matrix_stride, s.row_stride, s.rows, s.cols, p.parts, b.sums, s.eps, b.x[0], p.Rp, p.Cp, xplane);
    const Matrix S = blocked(b.s, p.mp, p.mp, qplane), Q = blocked(b.q, p.mp, p.mp, qplane);
    for (int step = 0; step < s.steps; ++step) {
        const Matrix X = blocked(b.x[step & 1], p.Rp, p.Cp, xplane);
        StepArgs k = {};
        k.terms = terms_of(P); k.count = s.count; k.part = b.part;
        k.arows = k.brows = p.mp; k.next = qnext; k.plane = qplane;
        // S
        k.a = k.b = X; k.anext = k.bnext = xnext; k.stages = std::max(p.Rp, p.Cp) / 32; k.symmetric = 1; k.to = b.s;
        if (p.tall) product<true, true, T, P>(k, p.s, st);
        else product<false, false, T, P>(k, p.s, st);
        // a I + b S + c S^2
        k.a = k.b = S; k.anext = k.bnext = qnext; k.stages = p.mp / 32; k.symmetric = 1; k.diagonal = s.a; k.f0 = s.b; k.f1 = s.c; k.old = b.s; k.to = b.q;
        product<false, false, T, P>(k, p.q, st);
        // that times X
        k.symmetric = 0; k.old = nullptr; k.to = b.x[~step & 1];
        k.arows = p.Cp; k.brows = p.Rp; k.next = xnext; k.plane = xplane;
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
size_t orthogonal_workspace(const ftp_orthogonal_shape& s)
{
    if (!orthogonal_is_small(s)) return buffers_of(s, plan_of(s), nullptr).bytes;
    Parts t(nullptr);
    t.take<double>((size_t)s.count * parts_of(s));
    return orthogonal_small_workspace(s, t);
}
void orthogonal(const ftp_orthogonal_shape& s, const void* x, void* out, char* ws, hipStream_t st)
{
    if (s.dtype == FTP_BF16) run<bf16_t, 2>(s, (const bf16_t*)x, (bf16_t*)out, ws, st);
    else run<float, 3>(s, (const float*)x, (float*)out, ws, st);
}

}  // namespace ftp
