// Products of bfloat matrices, D[a][b] = sum over k of A(a, k) B(b, k), as the training operators use them: a workgroup's block of D in registers, stages of both operands in LDS.
//
// An operand lies either along the contraction (element (i, k) at i * stride + k) or across it (k * stride + i); the latter is read through the transposing LDS load.  An fp32 matrix is PLANES
// matrices whose sum it is (three hold its 24 bits, two 16), a product of two the sum of the products of planes that are above 2^-24 (2^-16) of it, smallest first: six (three).  So there is one kernel, whose
// contraction is as many times longer.
//
// Stages of 32 (64) are fetched straight into LDS three to four ahead (buffer loads; what is past the end of an operand arrives as zeros), one barrier a stage, loads and reads between the matrix instructions.  A wavefront has 128 x 64 of
// a block of 256 x 256: 8 products of 32 x 32 x 16 to 6 operands of 1 KB.  8192 x 8192 x 2048: 213 to 232 us, 1.18 to 1.29 PFLOP/s (256 x 128 1.13 to 1.14, 128 x 128
// 1.03 to 1.12, 64 x 64 0.63 to 0.66); of zeros, which take less power, 1.76 to 1.80.
#pragma once
#include "ftp_tokens.h"

#include <tuple>
#include <type_traits>
#include <utility>

namespace ftp {

typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// f(0), f(1), .. f(N - 1) with constants
template <class F, int... I>
__device__ __forceinline__ void unrolled(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void unrolled(F f) { unrolled(f, std::make_integer_sequence<int, N>{}); }

// A matrix in bfloats: element (r, c) lies at (c / 32) * block + r * row + c % 32.  So row-major ones (block 32) and those laid out for the products (row 32: 32 columns of all rows one behind the other) go the same way; of
// the latter a stage is one run of memory along and a few across, where rows of 64 bytes each half a cache line were twice the requests to the L2.  16-byte aligned, `row` a multiple of 8; along: cols is a multiple of the
// stages', the part that is none in zeros; across: rows past the end, up to a stage's, are zeros or out of the matrix.
struct Matrix {
    const bf16_t* p;
    long long row, block, plane;                    // elements between rows, between blocks of 32 columns, between planes
    long long rows, size;                           // size: elements from p to the end of a plane
    int cols;
};
inline Matrix blocked(const bf16_t* p, long long rows, int cols, long long plane) { return Matrix{p, 32, rows * 32, plane, rows, rows * cols, cols}; }
inline Matrix row_major(const bf16_t* p, long long stride, long long rows, int cols) { return Matrix{p, stride, 32, 0, rows, (rows - 1) * stride + cols, cols}; }
// rows [r0, r0 + n)
inline Matrix rows_of(Matrix m, long long r0, long long n)
{
    m.p += r0 * m.row;
    m.size -= r0 * m.row;
    m.rows = n;
    return m;
}

// The products of planes that a product is the sum of, smallest first: planes of the two operands, two bits each.
struct Terms { int n; uint32_t a, b; };
inline Terms terms_of(int planes)
{
    // (0, 0);  (1, 0) (0, 1) (0, 0);  (2, 0) (0, 2) (1, 1) (1, 0) (0, 1) (0, 0)
    return planes == 1 ? Terms{1, 0, 0} : planes == 2 ? Terms{3, 0x1, 0x4} : Terms{6, 0x52, 0x118};
}
// ... of one plane with two: (0, 1) (0, 0)
inline Terms terms_one_two() { return Terms{2, 0, 0x1}; }

// A workgroup's block BA x BB by WA x WB wavefronts; XA, XB: the operand lies across.
template <int BA_, int BB_, int WA_, int WB_, bool XA_, bool XB_, int KS_ = 32, int STAGES = 4>
struct Product {
    static constexpr int BA = BA_, BB = BB_, WA = WA_, WB = WB_, kThreads = WA * WB * 64, KS = KS_, kStages = STAGES;
    static constexpr bool XA = XA_, XB = XB_;
    static constexpr int IA = BA / WA / 32, IB = BB / WB / 32;                     // 32 x 32 blocks of a wavefront
    static constexpr int kBytesA = BA * KS * 2, kBytesB = BB * KS * 2;
    static constexpr int kLoadsA = kBytesA / 16 / kThreads, kLoadsB = kBytesB / 16 / kThreads, kLoads = kLoadsA + kLoadsB;
    static_assert(kLoadsA * kThreads * 16 == kBytesA && kLoadsB * kThreads * 16 == kBytesB, "whole loads a thread");
    static_assert(kStages * kLoads < 64, "what vmcnt counts");
    struct Stage { char a[kBytesA], b[kBytesB]; };

    // Which 16 bytes of a row lie where: rows of 64 or 128 bytes (along) so that 16 rows' equal chunks meet no bank twice, longer ones (across) so that 4 rows x 64 bytes do not.
    template <int B, bool X>
    static __device__ __forceinline__ int mix(int row)
    {
        if constexpr (!X) return KS == 32 ? (row >> 2) & 3 : (row >> 1) & 7;
        else return B >= 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 2) << 1) | ((row >> 2) & 3);
    }
    // operand (index i0 + lane % 32; contraction 16 s + 8 h + j)
    template <int B, bool X>
    static __device__ __forceinline__ b16x8 operand(const char* t, int i0, int s)
    {
        const int l = threadIdx.x & 63, h = l >> 5;
        if constexpr (!X) {
            const int row = i0 + (l & 31);
            return *(const b16x8*)(t + row * (KS * 2) + (((2 * s + h) ^ mix<B, X>(row)) << 4));
        } else {
            // each 16 lanes: 4 rows x 16 columns, lane i brings 8 bytes of row i / 4 and takes column i of the four rows
            const int i = l & 15, col = i0 + (l & 16) + (i & 3) * 4;
            s16x4 v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = 16 * s + 8 * h + 4 * j + (i >> 2);
                v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (s16x4 __attribute__((address_space(3)))*)(t + row * (B * 2) + (((col >> 3) ^ mix<B, X>(row)) << 4) + (col & 7) * 2));
            }
            return __builtin_bit_cast(b16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
    // an operand's block on its way to LDS
    template <int B, bool X, int N>
    struct Source {
        const char *first, *base;                   // of plane 0, and of what the resource reaches
        long long plane, all, left;                 // bytes between planes, from the bases to the end
        uint32_t step, off;                         // bytes a stage, from the base to the stage that is being fetched
        __amdgpu_buffer_rsrc_t rsrc;
        int wave;
        int at[N];                                  // this thread's chunks, bytes from the stage
        __device__ __forceinline__ void init(const Matrix& m, long long i0, long long k0)
        {
            const long long o = X ? k0 * m.row + (i0 >> 5) * m.block : i0 * m.row + (k0 >> 5) * m.block;
            first = (const char*)(m.p + o);
            plane = m.plane * 2;
            all = (m.size - o) * 2;
            step = (uint32_t)(X ? KS * m.row * 2 : KS / 32 * m.block * 2);
            wave = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63) * 16;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                constexpr int kRow = X ? B / 8 : KS / 8;                            // chunks of a row
                const int u = threadIdx.x + kThreads * i, row = u / kRow, chunk = (u % kRow) ^ mix<B, X>(row);
                at[i] = (int)((chunk >> 2) * m.block * 2) + (int)(row * m.row * 2) + (chunk & 3) * 16;
            }
        }
        __device__ __forceinline__ void reach()
        {
            off = 0;
            rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, left <= 0 ? 0 : left > 0xFFFFFFF0ll ? (int)0xFFFFFFF0u : (int)(uint32_t)left, 0x00020000);
        }
        __device__ __forceinline__ void start(int p) { base = first + p * plane; left = all; reach(); }
        // (the hardware's check of the range takes the offset with it: num_records - soffset)
        __device__ __forceinline__ void next()
        {
            off += step;
            if (off >= 1u << 30) { base += off; left -= off; reach(); }
        }
        __device__ __forceinline__ void load(char* to, int i) const
        {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(to + wave + kThreads * 16 * i), 16, at[i], (int)off, 0, 0);
        }
    };

    template <int I, class F>
    static __device__ __forceinline__ void rest(int left, F f)
    {
        if constexpr (I + 1 < kStages) {
            if (left <= I) return;
            f(std::integral_constant<int, I>{});
            rest<I + 1>(left, f);
        }
    }

    static __device__ __forceinline__ int wave_a() { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WA) * (IA * 32); }
    static __device__ __forceinline__ int wave_b() { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WA) * (IB * 32); }

    // acc[i][j] += the block at (a0, b0) over the stages [lo, hi) of the contraction, for all terms.  The stages are distinct objects, so that loads into one are no reason to wait for those
    // into another.  At the end all of this wavefront's loads have landed.
    template <class... S>
    static __device__ __forceinline__ void run(f32x16 (&acc)[IA][IB], const Matrix& a, const Matrix& b, long long a0, long long b0, int lo, int hi, Terms terms, S&... stages)
    {
        Source<BA, XA, kLoadsA> fa;
        Source<BB, XB, kLoadsB> fb;
        fa.init(a, a0, (long long)lo * KS);
        fb.init(b, b0, (long long)lo * KS);
        const int wa = wave_a(), wb = wave_b(), per = hi - lo, total = per * terms.n;
        uint32_t pa = terms.a, pb = terms.b;
        if (total == 0) return;
        int k = per, to_come = total;
        fa.start(pa & 3);
        fb.start(pb & 3);
        const auto next_stage = [&]() __attribute__((always_inline)) {
            if (--to_come <= 0) return;             // (past the end the last stage is fetched again, to where nobody reads it)
            fa.next();
            fb.next();
            if (--k == 0) {
                k = per;
                pa >>= 2;
                pb >>= 2;
                fa.start(pa & 3);
                fb.start(pb & 3);
            }
        };
        const auto load = [&](Stage& to, int i) __attribute__((always_inline)) {
            if (i < kLoadsA) fa.load(to.a, i);
            else fb.load(to.b, i - kLoadsA);
        };
        b16x8 x[2][IA], y[2][IB];
        const auto read = [&](int set, const Stage& from, int s, int i) __attribute__((always_inline)) {
            if (i < IA) x[set][i] = operand<BA, XA>(from.a, wa + 32 * i, s);
            else y[set][i - IA] = operand<BB, XB>(from.b, wb + 32 * (i - IA), s);
        };
        // this wavefront's loads of the next stage have landed (n later ones are on their way), its reads of this one too; behind the barrier everybody's
        const auto landed = [&](auto n) __attribute__((always_inline)) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 0x70);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        constexpr int N = KS / 16, NM = IA * IB, NR = IA + IB;
        static_assert(N % 2 == 0, "operands alternate");
        // The products of operands that are there, and between them the reads of the next ones (k part s of `from`) and a part of the loads into `to`.  All at once behind the barrier, loads and reads held the
        // products up (8192 x 8192 x 2048: 240 us, where the loads alone take 92 and the products with their reads 137; so 222, one run each).
        const auto block = [&](int set, const Stage& from, int s, Stage& to, int part) __attribute__((always_inline)) {
            const int l0 = part * kLoads / N, nl = (part + 1) * kLoads / N - l0;
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                acc[m / IB][m % IB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[set][m / IB], y[set][m % IB], acc[m / IB][m % IB], 0, 0, 0);
#pragma unroll
                for (int i = m; i < NR && (i == m || m == NM - 1); ++i) read(set ^ 1, from, s, i);
#pragma unroll
                for (int i = m * nl / NM; i < (m + 1) * nl / NM; ++i) load(to, l0 + i);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // The first operands of a stage are read while the last ones of the stage before are multiplied; that stage's place is free then, and takes the loads of one to come until the next barrier.
        const auto step = [&](Stage& before, Stage& now, Stage& next) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 0; s + 1 < N; ++s) block(s & 1, now, s + 1, before, s + 1);
            landed(std::integral_constant<int, (kStages - 2) * kLoads>{});
            next_stage();
            block(1, next, 0, now, 0);
        };
        static_assert(sizeof...(S) == kStages, "a place a stage");
        const std::tuple<S&...> at(stages...);
        const auto place = [&](auto i) __attribute__((always_inline)) -> Stage& { return std::get<i % kStages>(at); };
        unrolled<kStages>([&](auto i) __attribute__((always_inline)) {
            if constexpr (i > 0) next_stage();
#pragma unroll
            for (int n = 0; n < (i + 1 < kStages ? kLoads : kLoads / N); ++n) load(place(i), n);
        });
        landed(std::integral_constant<int, (kStages - 2) * kLoads + kLoads / N>{});
#pragma unroll
        for (int i = 0; i < NR; ++i) read(0, std::get<0>(at), 0, i);
        const auto steps = [&](auto i) __attribute__((always_inline)) {
            step(place(std::integral_constant<int, i + kStages - 1>{}), place(i), place(std::integral_constant<int, i + 1>{}));
        };
        // (one way through the loop: where ways meet, the compiler waits for all loads)
        for (int s = total / kStages; s; --s) unrolled<kStages>(steps);
        rest<0>(total % kStages, steps);
        __builtin_amdgcn_s_waitcnt(0x70);
        asm volatile("" ::: "memory");
    }

    // f(v, a): every result of this lane, and its index along a counted from the lane's first one
    template <class F>
    static __device__ __forceinline__ void all(f32x16 (&acc)[IA][IB], F f)
    {
#pragma unroll
        for (int i = 0; i < IA; ++i)
#pragma unroll
            for (int j = 0; j < IB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float v = acc[i][j][r];
                    f(v, 32 * i + 8 * (r >> 2) + (r & 3));
                    acc[i][j][r] = v;
                }
    }
    // A share's sums as they lie in the registers, 1 KB a store (as rows of results 32 bytes of each went at once, and 247 MB of them took as long as the products), added to what is there or not.
    static constexpr int kUnits = IA * IB, kSums = BA * BB;
    static __device__ __forceinline__ void put(const f32x16 (&acc)[IA][IB], float* to, bool add)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16& x = acc[u % IA][u / IA];
                f32x4* p = (f32x4*)to + (u * 4 + q) * kThreads + threadIdx.x;
                const f32x4 v = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                *p = add ? *p + v : v;
            }
    }
    // ... added up, `next` floats from one share to the next, by 256 threads: part `index` of kParts, whose four wavefronts take the shares in turn (few blocks have many).  f as for each().
    static constexpr int kParts = kUnits * (kThreads / 64);
    template <class F>
    static __device__ __forceinline__ void take(const float* from, long long next, int shares, int index, F f)
    {
        __shared__ f32x4 sums[4][4][64];
        const int u = index / (kThreads / 64), wave = index % (kThreads / 64), l = threadIdx.x & 63, h = l >> 5, turn = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const f32x4* p = (const f32x4*)(from + turn * next) + u * 4 * kThreads + wave * 64 + l;
        f32x4 s[4] = {};
#pragma unroll 4
        for (int k = turn; k < shares; k += 4, p += next)
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += p[q * kThreads];
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[turn][q][l] = s[q];
        __syncthreads();
        if (turn >= 2) return;
        const int q = 2 * turn;
#pragma unroll
        for (int e = 0; e < 2; ++e) s[e] = (sums[0][q + e][l] + sums[1][q + e][l]) + (sums[2][q + e][l] + sums[3][q + e][l]);
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[0][e]), __float_as_uint(s[1][e]), false, false);
            v[e] = __uint_as_float(x[0]);
            v[4 + e] = __uint_as_float(x[1]);
        }
        f((wave % WA) * (IA * 32) + 32 * (u % IA) + 8 * q + 8 * h, (wave / WA) * (IB * 32) + 32 * (u / IA) + (l & 31), v);
    }

    // f(a, b, v): index of the first of eight neighbours along a, index along b, values; of this wavefront, from the block's corner.  (A lane's registers are four neighbours; the halves exchange every other four: 16 bytes of bfloats a store instead
    // of 8 or less.  32768 x 1024 of them from 11552 rows, G in one bfloat: 712 -> 636 us.)
    template <class F>
    static __device__ __forceinline__ void each(const f32x16 (&acc)[IA][IB], F f)
    {
        const int l = threadIdx.x & 63, h = l >> 5, wa = wave_a(), wb = wave_b();
#pragma unroll
        for (int j = 0; j < IB; ++j)
#pragma unroll
            for (int i = 0; i < IA; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 8) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][r + e]), __float_as_uint(acc[i][j][r + 4 + e]), false, false);
                        v[e] = __uint_as_float(x[0]);
                        v[4 + e] = __uint_as_float(x[1]);
                    }
                    f(wa + 32 * i + 2 * r + 8 * h, wb + 32 * j + (l & 31), v);
                }
    }
};

// The places of a launch's workgroups: XCD x takes the x-th eighth of the blocks in an order where neighbours share operands, four rows of blocks side by side.
__device__ __forceinline__ bool block_of(int index, int ablocks, int bblocks, int& ia, int& ib)
{
    const int total = ablocks * bblocks, per = (total + 7) >> 3, slot = index >> 3, t = (index & 7) * per + slot;
    if (slot >= per || t >= total) return false;
    const int wide = 4 * ablocks, band = t / wide, in = t - band * wide, high = min(4, bblocks - 4 * band);
    ia = in / high;
    ib = 4 * band + in - ia * high;
    return true;
}
inline long long block_grid(long long ablocks, long long bblocks) { return ceil_div(ablocks * bblocks, 8) * 8; }

// Blocks (256, 128 or 64 results squared, not below `least`) and shares of the contraction of a product of a x b results over `stages` stages of 32: the choice that should end first.  A CU holds one
// workgroup of the large blocks, two or four of the others, which then share it.
struct Split { int block, shares; };
inline Split split_of(long long a, long long b, long long stages, int least, int most, long long count = 1)
{
    Split best = {256, 1};
    double time = 1e300;
    for (int block = 256; block >= least; block /= 2) {
        const int per_cu = block == 256 ? 1 : block == 128 ? 2 : 4;
        const double stage = block == 256 ? 1.1 : block == 128 ? 0.31 : 0.12;      // microseconds, of a workgroup by itself
        const long long blocks = ceil_div(a, block) * ceil_div(b, block) * count;
        for (int s = 1; s <= most && (s == 1 || stages / s >= 8); ++s) {
            const long long n = blocks * s, rounds = ceil_div(n, 256 * per_cu), beside = n >= 256 * per_cu ? per_cu : ceil_div(n, 256);
            // start and end of a workgroup; the shares' sum, a launch that reads them
            const double t = (double)rounds * ((double)ceil_div(stages, s) * stage * (double)beside + 4) + (s > 1 ? 4 + 8e-6 * (double)(a * b * count) * s / 4 : 0);
            if (t < time) { time = t; best = {block, s}; }
        }
    }
    return best;
}

// 2 neighbouring numbers as PLANES bfloats each whose sum they are: exactly (3, as split3) or to 16 bits (2; the numbers are known to that only where two planes are used)
template <int PLANES>
__device__ __forceinline__ void planes_of(float a, float b, uint32_t (&w)[PLANES])
{
    if constexpr (PLANES == 3) split3(a, b, w[0], w[1], w[2]);
    else {
        w[0] = pack_bf16(a, b);
        if constexpr (PLANES == 2) w[1] = pack_bf16(a - __uint_as_float(w[0] << 16), b - __uint_as_float(w[0] & 0xFFFF0000u));
    }
}

// 8 neighbours as planes, 16 bytes of each
template <int PLANES>
__device__ __forceinline__ void store_planes(bf16_t* to, long long plane, const float (&v)[8])
{
    uint32_t x[4][PLANES];
#pragma unroll
    for (int e = 0; e < 4; ++e) planes_of<PLANES>(v[2 * e], v[2 * e + 1], x[e]);
#pragma unroll
    for (int p = 0; p < PLANES; ++p) *(uint4*)(to + p * plane) = uint4{x[0][p], x[1][p], x[2][p], x[3][p]};
}
// The first n of 8 neighbours of a row of results, at any address: all eight at once.
template <typename T>
__device__ __forceinline__ void store8(T* to, int n, const float (&v)[8])
{
    if (n >= 8) {
        Pack<T, 8> w;
        w.put(v);
        w.store_any(to);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < n) st(to + e, v[e]);
}

}  // namespace ftp
