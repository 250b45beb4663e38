// What the attention kernels share: operands of the matrix cores from LDS and registers, staging of tiles, which query sees which key.
//
// The queries of the heads that share a key head are rows of one list: row r is query r / group of head r % group of those.  A tile of keys is
// then read once for the whole group, gradients of shared keys need no sum over heads, and one query of a long cache still fills rows.
//
// All products run on 32x32 blocks, 16 deep, on the bfloat matrix cores (v_mfma_f32_32x32x16_bf16).  An fp32 number goes in as three bfloats whose sum it is (ftp_split.h), a product as the
// six of theirs that are above 2^-24 of it: 192 cycles where the fp32 instruction takes 512.  Tiles are split once, on their way into LDS.  A lane holds of
// an operand the 8 values (index lane % 32; contraction 8 h + j, h = lane / 32, j < 8), and of a result column lane % 32 and rows 8 (i / 4) + 4 h + i % 4, i < 16.
// The contraction may run over any order that both operands share.  So a result is the next product's operand as it lies: its registers 8 s .. 8 s + 7 are the operand
// (index lane % 32; contraction 16 s + 8 (j / 4) + 4 h + j % 4), and the other operand is loaded in that order.  No probability passes through LDS.
#pragma once
#include "ftp_tokens.h"
#include "ftp_order.h"

#include <type_traits>
#include <utility>

namespace ftp {

typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Split { b16x8 h, m, l; };                    // 8 fp32 numbers
template <typename T> struct FragOf { typedef b16x8 type; };
template <> struct FragOf<float> { typedef Split type; };

__device__ __forceinline__ f32x16 mma(b16x8 a, b16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(const Split& a, const Split& b, f32x16 c)
{
    c = mma(a.l, b.h, c);                           // smallest first
    c = mma(a.h, b.l, c);
    c = mma(a.m, b.m, c);
    c = mma(a.m, b.h, c);
    c = mma(a.h, b.m, c);
    return mma(a.h, b.h, c);
}

// Operands of pairs of neighbouring registers of a result, as they become known.
__device__ __forceinline__ void set_word(b16x8& f, int j, uint32_t v)
{
    u32x4 w = __builtin_bit_cast(u32x4, f);
    w[j] = v;
    f = __builtin_bit_cast(b16x8, w);
}
template <typename T>
struct Words {
    typename FragOf<T>::type f[2];
    __device__ __forceinline__ void set(int pair, float a, float b)
    {
        if constexpr (sizeof(T) == 4) {
            uint32_t h, m, l;
            split3(a, b, h, m, l);
            Split& x = f[pair >> 2];
            set_word(x.h, pair & 3, h); set_word(x.m, pair & 3, m); set_word(x.l, pair & 3, l);
        } else set_word(f[pair >> 2], pair & 3, pack_bf16(a, b));
    }
};

// Registers 8 s .. 8 s + 7 of a result as an operand: rounded to bfloats where the operands are bfloats (the probabilities and their gradients lose
// what the inputs have lost already; sums stay fp32).
template <typename T>
__device__ __forceinline__ typename FragOf<T>::type operand(const f32x16& v, int s)
{
    Words<T> w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w.set(j, v[8 * s + 2 * j], v[8 * s + 2 * j + 1]);
    return w.f[0];
}

// A tile of ROWS rows of D channels in LDS, in chunks of 8 bfloats (16 bytes); of fp32 numbers three planes of them.  Chunks are exchanged within a row by the row's low bits, so that neither
// 16 rows of one chunk (operand along the channels) nor the transposing load's 4 rows x 64 bytes meet on the 64 banks.
template <typename T, int D, int ROWS>
struct Tile {
    static constexpr int kChunks = D / 8, kRow = D * 2, kPlane = ROWS * kRow, kBytes = kPlane * (sizeof(T) == 4 ? 3 : 1);
    static __device__ __forceinline__ int mix(int row)
    {
        return D == 32 ? (row >> 2) & 3 : D == 64 ? ((row & 2) << 1) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * kRow + ((chunk ^ mix(row)) << 4); }

    template <class F>
    static __device__ __forceinline__ typename FragOf<T>::type planes(F f)
    {
        if constexpr (sizeof(T) == 4) return Split{f(0), f(kPlane), f(2 * kPlane)};
        else return f(0);
    }
    // (mix() goes by a row's low four bits: row0, a multiple of 16, only moves the address)
    // operand (index: row row0 + lane % 32; contraction: channels 16 s + 8 h + j)
    static __device__ __forceinline__ typename FragOf<T>::type along(const char* t, int row0, int s)
    {
        const int l = threadIdx.x & 63;
        const char* p = t + row0 * kRow + at(l & 31, 2 * s + (l >> 5));
        return planes([&](int plane) __attribute__((always_inline)) { return *(const b16x8*)(p + plane); });
    }
    // operand (index: channel d0 + lane % 32; contraction: rows row0 + 8 (j / 4) + 4 h + j % 4)
    static __device__ __forceinline__ typename FragOf<T>::type across(const char* t, int row0, int d0)
    {
        // each 16 lanes: 4 rows x 16 channels, lane i brings 8 bytes of row i / 4 and takes channel i of the four rows
        const int l = threadIdx.x & 63, h = l >> 5, i = l & 15, col = d0 + (l & 16) + (i & 3) * 4;
        return planes([&](int plane) __attribute__((always_inline)) {
            s16x4 v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (s16x4 __attribute__((address_space(3)))*)(t + plane + row0 * kRow + at(8 * j + 4 * h + (i >> 2), col >> 3) + (col & 7) * 2));
            return __builtin_bit_cast(b16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        });
    }
};

// 8 fp32 numbers as an operand
__device__ __forceinline__ Split split8(u32x4 a, u32x4 b)
{
    u32x4 h, m, l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t x, y, z;
        const u32x4& from = j < 2 ? a : b;
        split3(__uint_as_float(from[2 * (j & 1)]), __uint_as_float(from[2 * (j & 1) + 1]), x, y, z);
        h[j] = x; m[j] = y; l[j] = z;
    }
    return Split{__builtin_bit_cast(b16x8, h), __builtin_bit_cast(b16x8, m), __builtin_bit_cast(b16x8, l)};
}

// v of the other half's lane with the same lane % 32, combined with f: both halves get the result.
template <class F>
__device__ __forceinline__ float across_halves(float v, F f)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v) { return across_halves(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float both_max(float v) { return across_halves(v, [](float a, float b) { return fmaxf(a, b); }); }

// The 16 bytes of channels [d0, d0 + 16 / sizeof(T)) of a row; zero past channel d.  vec: addresses allow one load (and d is whole chunks).
template <typename T>
__device__ __forceinline__ u32x4 chunk_of(const T* row, int d0, int d, bool vec)
{
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 r = {0, 0, 0, 0};
    if (vec) {
        if (d0 < d) r = *(const u32x4*)(row + d0);
        return r;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        if (d0 + j >= d) continue;
        if constexpr (sizeof(T) == 4) r[j] = __float_as_uint(row[d0 + j]);
        else r[j >> 1] |= (uint32_t)row[d0 + j] << (16 * (j & 1));
    }
    return r;
}

// Rows of a tile on their way from memory to LDS, for the workgroup's 256 threads.  Bfloats where VEC: straight into LDS (buffer loads whose lanes fill 16 bytes each, one
// after the other; what is out of the resource's range arrives as zeros), landed once wait_tiles() returns.  fp32 numbers, and bfloats whose addresses or head size do not allow
// 16 bytes at once: through registers, written by put().  Where a row lies in its tile is the same for all tiles and is worked out once: offset(r), bytes from
// the tile's base (wavefront-uniform).
template <typename T, int D, int ROWS, bool VEC>
struct Staged {
    typedef Tile<T, D, ROWS> L;
    typedef typename std::conditional<VEC, int, long long>::type Bytes;
    static constexpr bool kDirect = VEC && sizeof(T) == 2;
    static constexpr int kAll = ROWS * L::kChunks, kEach = (kAll + 255) / 256, kNone = -1, kWords = kDirect ? 1 : (int)sizeof(T) / 2;
    static_assert(kAll % 256 == 0 || kEach == 1, "whole chunks a thread");
    Bytes at[kEach];
    u32x4 r[kDirect ? 1 : kEach][kWords];
    int d;
    template <class Offset>
    __device__ __forceinline__ void init(Offset offset, int d_)
    {
        d = d_;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = threadIdx.x + 256 * i, row = u / L::kChunks, chunk = (u % L::kChunks) ^ (kDirect ? L::mix(row) : 0);       // (the chunk that lies here)
            at[i] = (kAll < 256 && u >= kAll) || chunk * 8 >= d ? (Bytes)kNone : offset(row) + chunk * 8 * (int)sizeof(T);
        }
    }
    // `rows`: how many rows there are, the others are zeros, and so are those from `zero0` to `zero1` - 1
    __device__ __forceinline__ void fetch(char* tile, const T* base, int rows, int zero0 = 0, int zero1 = 0)
    {
        const auto is_there = [&](int row) { return row < rows && (row < zero0 || row >= zero1); };
        if constexpr (kDirect) {
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, (int)0x80000000u, 0x00020000);
            if (rows >= ROWS && zero1 <= zero0) {
#pragma unroll
                for (int i = 0; i < kEach; ++i) load(tile, rsrc, i, at[i]);
            } else {
#pragma unroll
                for (int i = 0; i < kEach; ++i) load(tile, rsrc, i, is_there((int)(threadIdx.x + 256 * i) / L::kChunks) ? at[i] : kNone);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int u = threadIdx.x + 256 * i, d0 = (u % L::kChunks) * 8;
                const bool there = is_there(u / L::kChunks) && at[i] >= 0;
                const T* row = (const T*)((const char*)base + (there ? at[i] : 0)) - (there ? d0 : 0);
#pragma unroll
                for (int k = 0; k < kWords; ++k) {
                    r[i][k] = u32x4{0, 0, 0, 0};
                    if (there) r[i][k] = chunk_of(row, d0 + k * (16 / (int)sizeof(T)), d, VEC);
                }
            }
        }
    }
    __device__ __forceinline__ void put(char* tile) const
    {
        if constexpr (!kDirect) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int u = threadIdx.x + 256 * i;
                if (kAll < 256 && u >= kAll) continue;
                char* p = tile + L::at(u / L::kChunks, u % L::kChunks);
                if constexpr (sizeof(T) == 4) {
                    const Split x = split8(r[i][0], r[i][1]);
                    *(b16x8*)p = x.h;
                    *(b16x8*)(p + L::kPlane) = x.m;
                    *(b16x8*)(p + 2 * L::kPlane) = x.l;
                } else *(u32x4*)p = r[i][0];
            }
        }
    }
private:
    static __device__ __forceinline__ void load(char* tile, __amdgpu_buffer_rsrc_t rsrc, int i, int offset)
    {
        const int first = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63) + 256 * i;
        if (kAll < 256 && first >= kAll) return;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(tile + first * 16), 16, offset, 0, 0, 0);
    }
};
// This wavefront's loads have landed (vmcnt(0)); a barrier behind it makes it everybody's.
__device__ __forceinline__ void wait_tiles() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// f(0), f(1), .. f(N - 1) with constants
template <class F, int... I>
__device__ __forceinline__ void unrolled(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void unrolled(F f) { unrolled(f, std::make_integer_sequence<int, N>{}); }

// The work of one unit (32 x 32 pairs) in the order in which it keeps matrix cores and vector units busy at once: NA products of the next unit's scores with the first half of this
// unit's exponentials (valu(0 .. 3), two registers each), NC products of that half's probabilities with the second half of the exponentials, and the other half's products.
// Operands are read from LDS two slots ahead.  The order is fixed (sched_barrier): left to itself the compiler puts all matrix instructions behind each other, where the
// vector unit waits for them.
template <int NA, int NC, class LoadA, class MmaA, class Valu, class LoadC, class MmaC>
__device__ __forceinline__ void overlap(LoadA load_a, MmaA mma_a, Valu valu, LoadC load_c, MmaC mma_c)
{
    constexpr int PA = (NA + 3) / 4, PC = (NC + 3) / 4;
    const auto loads = [&](auto s) __attribute__((always_inline)) {
        if constexpr (s < 4) unrolled<PA>([&](auto i) __attribute__((always_inline)) { if constexpr (s * PA + i < NA) load_a(s * PA + i); });
        else if constexpr (s < 12) unrolled<PC>([&](auto i) __attribute__((always_inline)) { if constexpr ((s & 3) * PC + i < NC) load_c((s - 4) / 4, (s & 3) * PC + i); });
    };
    loads(std::integral_constant<int, 0>{});
    loads(std::integral_constant<int, 1>{});
    __builtin_amdgcn_sched_barrier(0);
    unrolled<12>([&](auto s) __attribute__((always_inline)) {
        loads(std::integral_constant<int, s + 2>{});
        if constexpr (s < 4) unrolled<PA>([&](auto i) __attribute__((always_inline)) { if constexpr (s * PA + i < NA) mma_a(s * PA + i); });
        else unrolled<PC>([&](auto i) __attribute__((always_inline)) { if constexpr ((s & 3) * PC + i < NC) mma_c((s - 4) / 4, (s & 3) * PC + i); });
        if constexpr (s < 8) valu((int)s);
        __builtin_amdgcn_sched_barrier(0);
    });
}

// The score that replaces a hidden pair's, whatever that came out as: its exponential is 0.
constexpr float kHidden = -INFINITY;

// Workgroups a CU that the register budget is set for: two (all sums and operands in 256 registers) where they fit.
template <typename T, int D> constexpr int kPerCu = sizeof(T) == 4 && D == 128 ? 1 : 2;

// Channels 16 s + 8 h .. + 7 of this lane's row, s < D / 16, as they lie in memory; row null: zeros.
template <typename T, int D>
struct RowWords {
    u32x4 w[D / 16][sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* row, int d, bool vec)
    {
        const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                w[s][i] = u32x4{0, 0, 0, 0};
                if (row) w[s][i] = chunk_of(row, 16 * s + 8 * h + 4 * i, d, vec);
            }
    }
    __device__ __forceinline__ float dot(const RowWords& o) const          // of the two lanes of a row
    {
        float v = 0;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t x = w[s][i][j], y = o.w[s][i][j];
                    if constexpr (sizeof(T) == 4) v = fmaf(__uint_as_float(x), __uint_as_float(y), v);
                    else {
                        v = fmaf(__uint_as_float(x << 16), __uint_as_float(y << 16), v);
                        v = fmaf(__uint_as_float(x & 0xFFFF0000u), __uint_as_float(y & 0xFFFF0000u), v);
                    }
                }
        return both_sum(v);
    }
    // operands (index: this lane's row; contraction: channels 16 s + 8 h + j)
    __device__ __forceinline__ void operands(typename FragOf<T>::type (&f)[D / 16], bool negate) const
    {
        const uint32_t sign = !negate ? 0u : sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            if constexpr (sizeof(T) == 4) f[s] = split8(w[s][0] ^ sign, w[s][1] ^ sign);
            else f[s] = __builtin_bit_cast(b16x8, w[s][0] ^ sign);
        }
    }
};
template <typename T, int D>
__device__ __forceinline__ void row_operands(typename FragOf<T>::type (&f)[D / 16], const T* row, int d, bool vec, bool negate)
{
    RowWords<T, D> w;
    w.load(row, d, vec);
    w.operands(f, negate);
}

// Four neighbouring channels d0 .. d0 + 3 of a row, those below d.
template <typename T>
__device__ __forceinline__ void store4(T* row, int d0, int d, bool vec, float a, float b, float c, float e)
{
    if (vec) {
        if (d0 >= d) return;
        if constexpr (sizeof(T) == 4) *(f32x4*)(row + d0) = f32x4{a, b, c, e};
        else *(uint2*)(row + d0) = uint2{pack_bf16(a, b), pack_bf16(c, e)};
        return;
    }
    if (d0 < d) st(row + d0, a);
    if (d0 + 1 < d) st(row + d0 + 1, b);
    if (d0 + 2 < d) st(row + d0 + 2, c);
    if (d0 + 3 < d) st(row + d0 + 3, e);
}

struct AttentionArgs {
    const void* q; const void* k; const void* v; const int* q_lens; const int* kv_lens;
    void* out; float* lse; float* ws;
    const void* dout; void* dq; void* dk; void* dv; float* delta;
    long long qs[3], ks[3], vs[3], os[3], gs[3], dqs[3], dks[3], dvs[3];
    int batch, heads, kv, group, q_len, kv_len, d, causal, vec;
    int blocks, splits, groups, by_xcd;             // workgroups: blocks of rows (keys) x splits of the other axis x (image, key head)
    float scale, c;                                 // c = |scale| * log2(e): exponentials are powers of 2 here
};

// Lengths of an image, and what a row of it sees.
struct Lengths {
    int q, k, off;                                  // off: a causal query i sees keys up to i + off
    __device__ __forceinline__ Lengths(const AttentionArgs& a, int b)
    {
        q = a.q_lens ? min(max(a.q_lens[b], 0), a.q_len) : a.q_len;
        k = a.kv_lens ? min(max(a.kv_lens[b], 0), a.kv_len) : a.kv_len;
        off = k - q;
    }
    // number of keys that query i sees
    __device__ __forceinline__ int seen(const AttentionArgs& a, int i) const { return i >= q ? 0 : a.causal ? min(max(i + off + 1, 0), k) : k; }
};

__device__ __forceinline__ int query_of(const AttentionArgs& a, int row) { return a.group == 1 ? row : (int)((uint32_t)row / (uint32_t)a.group); }

// Which block, split, image and key head a workgroup has; false: none.  Blocks of one (image, key head) read the same keys (queries) and run on one XCD where
// the groups are many enough, and alike enough, to load all eight evenly.  Otherwise the groups' first blocks (of causal calls the longest) come first, a group's blocks on XCDs in turn:
// a few images of their own lengths loaded the XCDs unevenly (prompts, 4 images x 2 key heads, 1550 to 2704 tokens: 69 -> 62 us; 2 x 3 key heads of 4000, causal: 78 -> 63; but
// 6 x 4 key heads of 750 to 1500 113 us by XCDs, 120 in turn).
__device__ __forceinline__ bool place_of(const AttentionArgs& a, int& block, int& split, int& b, int& kvh)
{
    int g;
    const int index = (int)blockIdx.x;
    if (a.by_xcd) {
        if (!xcd_order(index, a.groups, a.blocks, g, block)) return false;
    } else {
        block = index / a.groups;
        g = (index - block * a.groups + block) % a.groups;
    }
    split = g % a.splits;
    g /= a.splits;
    b = g / a.kv;
    kvh = g - b * a.kv;
    return true;
}
// Workgroups of `blocks` blocks each of (image, key head, split) groups.
inline bool by_xcd(long long groups, bool ragged) { return (groups % 8 == 0 && groups >= (ragged ? 24 : 8)) || groups >= 48; }
inline long long place_count(long long groups, long long blocks, bool ragged) { return by_xcd(groups, ragged) ? ceil_div(groups, 8) * 8 * blocks : groups * blocks; }
inline unsigned place_groups(AttentionArgs& a)
{
    const bool ragged = a.q_lens || a.kv_lens;
    a.groups = a.batch * a.kv * a.splits;
    a.by_xcd = by_xcd(a.groups, ragged);
    return (unsigned)place_count(a.groups, a.blocks, ragged);
}

// Hidden keys and rows are multiplied by 0 inside a block, which makes NaN of what is not finite there (only causal calls have hidden values in a block: rows past the lengths are
// zeros).  A workgroup that ends with such results takes a second look if the tiles with hidden pairs do hold such numbers: a row (key) concerned takes those tiles' pairs that are
// seen one after the other, until every channel that came out bad is bad from seen values alone - then the result stands as it is -, and the other tiles are walked over
// once more for the rows left.  So a call on numbers that are not finite takes at most twice the walks and a bounded number of single pairs (4 x 4 heads x 4096 tokens, forward: 74 us, of
// NaN 77; with pairs one by one along whole rows that was 91 ms; a backward pass with one bad row of dout 127 ms -> 1.6).
// v, as if it were not known from before: what is computed from it is computed here
__device__ __forceinline__ int again(int v) { asm volatile("" : "+v"(v)); return v; }
// Channels that are not finite, a bit each.
template <int DT>
__device__ __forceinline__ unsigned long long bad_channels(const f32x16 (&v)[DT])
{
    unsigned long long bad = 0;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad |= (unsigned long long)!(fabsf(v[d][r]) < INFINITY) << (16 * d + r);
    return bad;
}
// Whether `rows` rows of d channels hold what the matrix cores do not take times 0: this thread's share of the workgroup's look.
constexpr float kLargestBfloat = 3.38953139e38f;
template <typename T, class Row>
__device__ __forceinline__ bool find_bad(int rows, int d, Row row)
{
    bool bad = false;
    for (long long u = threadIdx.x; u < (long long)rows * d; u += 256) {
        const int r = (int)(u / d);
        bad = bad || !(fabsf(ld((const T*)row(r) + (u - (long long)r * d))) <= kLargestBfloat);
    }
    return bad;
}
template <typename T>
__device__ __forceinline__ float dot_of(const T* x, const T* y, int d)
{
    float s = 0;
#pragma unroll 4
    for (int c = 0; c < d; ++c) s = fmaf(ld(x + c), ld(y + c), s);
    return s;
}
// v[channel] += f * row[channel] for the channels that this lane holds of a result
template <typename T, int DT>
__device__ __forceinline__ void add_row(f32x16 (&v)[DT], float f, const T* row, int d)
{
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int k = 0; k < DT; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int c = 32 * k + 8 * (r >> 2) + 4 * h + (r & 3);
            if (c < d) v[k][r] = fmaf(f, ld(row + c), v[k][r]);
            __builtin_amdgcn_sched_barrier(0);
        }
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

AttentionArgs attention_args(const ftp_attention_shape& s);
// Wavefronts to a row of 32 in the kernels that walk over the keys: 1 or 2.
int attention_halves(const ftp_attention_shape& s);
// Keys of a workgroup of the key gradients.
inline int attention_key_block(bool wide_fp32) { return wide_fp32 ? 64 : 128; }

// Offsets within a tile (at most 64 such strides) stay below 2^30 bytes.
inline bool near_rows(long long stride) { return stride < (1ll << 21); }

}  // namespace ftp
