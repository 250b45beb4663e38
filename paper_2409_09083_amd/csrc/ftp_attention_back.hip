// Softmax attention, backward: the probabilities are computed again from q, k and the rows' log-sums,
//   p = exp(scale q.k - lse), delta = sum_d dout out, ds = p (dout.v - delta), dv = sum_rows p dout, dq = scale sum_keys ds k, dk = scale sum_rows ds q.
//
// Two kernels, so that every sum stays in one workgroup's registers and in one order: k_attention_dq walks over the keys of 128 rows (as the forward pass does, and leaves
// delta), k_attention_dkv over the rows of 128 keys.  Scores and dout.v are computed in both: seven products of the pairs instead of five, where one kernel would add dq up by
// atomics, in an order that changes.  In dq S^T and dP^T have a row per lane, in dkv S and dP a key per lane, so that P and dS again are operands as they lie
// (ftp_attention.h).  Where 128-row (key) blocks are too few for the CUs, the other axis is split and the parts are added up by a third kernel.
//
// Measured, 64 heads x 5776 tokens of 64, bfloats (1.91 TFLOP in seven products, 1.37 in five): dq 0.78-0.87 ms (940-1050 TFLOP/s of its three products), dk and dv 1.20-1.30 ms (840-910 of their four); a large
// library product reaches 1265 on the same card.  Matrix cores busy 58 and 43-49 % of the cycles, at a clock that the load lowers to 1.9-2.05 GHz; LDS 30-37 %, without bank conflicts; without any load from
// memory the two took 0.78 and 0.99 ms.  577 x 701 tokens of 40, fp32, 3 x 2 key heads: dq 25 us, dk and dv 39, sums of the splits 5 + 5: a workgroup's chain of 4 to 8 tiles.
#include "ftp_attention.h"

#include <algorithm>
#include <cmath>

namespace ftp {
namespace {

template <typename T, int D> constexpr int kKeys = sizeof(T) == 4 ? 32 : 64;       // keys of a tile

// The gradient of a row's scores where it sees one key, from its log-sum, which is that key's score: 0, or NaN where the score is no number.
__device__ __forceinline__ float one_key(float lse) { return lse - lse; }

// A workgroup is 128 rows against tiles of 64 keys (fp32: 32), two tiles in LDS.  The compiler's order of a tile's instructions is kept: by hand as in k_attention_dkv it was slower here (0.80 -> 0.93 ms).
//
// HALVES 2, bfloats: 64 rows, each by two wavefronts that take a unit of every tile and add up their rows through LDS at the end (attention_halves(): 4 x 12 heads x 577 tokens 52.6 -> 45.3 us the pass,
// causal 4 x 8 x 2600 155 -> 144).  fp32 tiles of two units for it would cost the second workgroup of a CU: 16 heads x 1144 of 64 161 -> 207.
template <typename T, int D, bool VEC, int HALVES>
__global__ __launch_bounds__(256, (kPerCu<T, D>)) void k_attention_dq(const AttentionArgs a)
{
    typedef typename FragOf<T>::type Frag;
    constexpr int BN = kKeys<T, D>, UNITS = BN / 32 / HALVES, KS = D / 16, DT = D / 32, ROWS = 128 / HALVES;
    typedef Tile<T, D, BN> L;
    constexpr int kTile = L::kBytes;
    struct Keys { char tile[2][kTile]; };           // a tile of keys and values
    __shared__ __align__(16) Keys even, odd;        // (apart, so that reads of one need not wait for loads of the other)
    int block, split, b, kvh;
    if (!place_of(a, block, split, b, kvh)) return;
    if (a.causal) block = a.blocks - 1 - block;
    const Lengths len(a, b);
    const int rows = a.q_len * a.group;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, h = l >> 5;
    const int half = HALVES == 2 ? wave >> 1 : 0, at0 = (HALVES == 2 ? wave & 1 : wave) * 32, mine0 = 32 * half;         // this wavefront's rows, and its unit's first key of a tile
    const int first = block * ROWS, row = first + at0 + (l & 31);
    const int i = query_of(a, row), head = kvh * a.group + row - i * a.group;
    const bool inside = row < rows;
    const int seen = inside ? len.seen(a, i) : 0;
    const int last = query_of(a, min(first + ROWS, rows) - 1), i0 = query_of(a, first);
    const int end = i0 < len.q ? len.seen(a, min(last, len.q - 1)) : 0, common = len.seen(a, i0);
    const int tiles = (end + BN - 1) / BN, lo = (int)((long long)tiles * split / a.splits), hi = (int)((long long)tiles * (split + 1) / a.splits);
    // this row's operands; delta from the same dout and the row of out
    Frag q[D / 16], g[D / 16];
    float delta;
    {
        RowWords<T, D> o, w;
        o.load(seen ? (const T*)a.out + b * a.os[0] + i * a.os[1] + head * a.os[2] : nullptr, a.d, VEC);
        w.load(seen ? (const T*)a.dout + b * a.gs[0] + i * a.gs[1] + head * a.gs[2] : nullptr, a.d, VEC);
        delta = w.dot(o);
        w.operands(g, false);
    }
    const long long at = (((long long)b * a.kv + kvh) * a.q_len) * a.group + row;
    row_operands<T, D>(q, seen ? (const T*)a.q + b * a.qs[0] + i * a.qs[1] + head * a.qs[2] : nullptr, a.d, VEC, a.scale < 0);
    const float lse = seen ? a.lse[((long long)b * a.heads + head) * a.q_len + i] * kLog2e : INFINITY;     // (a row that sees nothing: p = 0)

    const T* kp = (const T*)a.k + b * a.ks[0] + kvh * a.ks[2];
    const T* vp = (const T*)a.v + b * a.vs[0] + kvh * a.vs[2];
    Staged<T, D, BN, VEC> sk, sv;
    typedef typename Staged<T, D, BN, VEC>::Bytes Bytes;
    sk.init([&](int r) { return r * (Bytes)a.ks[1] * (Bytes)sizeof(T); }, a.d);
    sv.init([&](int r) { return r * (Bytes)a.vs[1] * (Bytes)sizeof(T); }, a.d);
    const auto fetch = [&](int t, Keys& to) __attribute__((always_inline)) {
        sk.fetch(to.tile[0], kp + (long long)t * BN * a.ks[1], len.k - t * BN);
        sv.fetch(to.tile[1], vp + (long long)t * BN * a.vs[1], len.k - t * BN);
    };
    const auto land = [&](Keys& to) __attribute__((always_inline)) {
        sk.put(to.tile[0]);
        sv.put(to.tile[1]);
        wait_tiles();
        __syncthreads();
    };
    f32x16 dq[DT] = {};
    float exact = 0;
    // few: only the row's delta, of p and dP themselves
    const auto step = [&](int t, int to, int seen, Keys& now, Keys& next, auto few) __attribute__((always_inline)) {
        if (t + 1 < to) fetch(t + 1, next);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            f32x16 s = {}, p;
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = few ? 0.0f : -delta;
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                s = mma(L::along(now.tile[0], mine0 + 32 * u, c), q[c], s);
                p = mma(L::along(now.tile[1], mine0 + 32 * u, c), g[c], p);
            }
            if (t * BN + mine0 + 32 * u + 32 > common) {
                const int left = seen - t * BN - mine0 - 32 * u - 4 * h;       // keys of the unit that the row sees, counted from this lane's first
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool hidden = 8 * (r >> 2) + (r & 3) >= left;
                    s[r] = hidden ? kHidden : s[r];
                    p[r] = hidden ? 0.0f : p[r];
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] *= __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -lse));
            if constexpr (few) {
#pragma unroll
                for (int r = 0; r < 16; ++r) exact += p[r];
            } else {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const Frag ds = operand<T>(p, c);
#pragma unroll
                    for (int d = 0; d < DT; ++d) dq[d] = mma(L::across(now.tile[0], mine0 + 32 * u + 16 * c, 32 * d), ds, dq[d]);
                }
            }
        }
        if (t + 1 < to) land(next);
        else if constexpr (few) __syncthreads();    // (the second walk starts with the same tiles)
    };
    const auto walk = [&](int to, int seen, auto few) __attribute__((always_inline)) {
        if (lo < to) {
            fetch(lo, even);
            land(even);
        }
        for (int t = lo; t < to; t += 2) {
            step(t, to, seen, even, odd, few);
            if (t + 1 < to) step(t + 1, to, seen, odd, even, few);
        }
    };
    // Where rows see few keys the rounding of out shows in delta (the products' rounding averages out with the keys, this does not): bfloat rows of up to 256 keys
    // take delta from p and dP, in a walk before (40 tokens: dk and dq 0.0027 -> 0.0024 of their size away, 0.0017 of it the rounding of the results).
    if (sizeof(T) == 2 && a.splits == 1 && tiles * BN <= 256) {
        walk(hi, seen, std::true_type{});
        exact = both_sum(exact);
        if constexpr (HALVES == 2) {
            float* parts = (float*)&odd;            // (odd: the second walk starts with even)
            parts[(wave >> 1) * 128 + at0 * 2 + l] = exact;
            __syncthreads();
            exact = parts[at0 * 2 + l] + parts[128 + at0 * 2 + l];
        }
        delta = exact;
    }
    if (split == 0 && half == 0 && inside && h == 0) a.delta[at] = delta;
    // two wavefronts' rows become the first one's
    const auto join = [&]() __attribute__((always_inline)) {
        if constexpr (HALVES == 2) {
            static_assert((int)sizeof(Keys) >= 2 * DT * 4096, "two wavefronts' rows in a tile's place");
            f32x4* parts = (f32x4*)&even + (at0 / 32) * DT * 4 * 64;
            __syncthreads();                        // (nobody reads tiles any more)
            if (half) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) parts[(d * 4 + r) * 64 + l] = f32x4{dq[d][4 * r], dq[d][4 * r + 1], dq[d][4 * r + 2], dq[d][4 * r + 3]};
            }
            __syncthreads();
            if (half) return;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x4 v = parts[(d * 4 + r) * 64 + l];
#pragma unroll
                    for (int j = 0; j < 4; ++j) dq[d][4 * r + j] += v[j];
                }
        }
    };
    const auto store = [&](int row, int seen) __attribute__((always_inline)) {
        if (a.splits > 1) {
            float* p = a.ws + (((long long)split * a.batch * a.kv * rows) + (((long long)b * a.kv + kvh) * a.q_len) * a.group + row) * D;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(f32x4*)(p + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{dq[d][r], dq[d][r + 1], dq[d][r + 2], dq[d][r + 3]};
            return;
        }
        const int i = query_of(a, row), head = kvh * a.group + row - i * a.group;
        const float zero = seen ? one_key(lse) : 0.0f;
        const f32x4 none = {zero, zero, zero, zero};
        T* p = (T*)a.dq + b * a.dqs[0] + i * a.dqs[1] + head * a.dqs[2];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 v = seen > 1 ? f32x4{dq[d][r], dq[d][r + 1], dq[d][r + 2], dq[d][r + 3]} * a.scale : none;
                store4(p, 32 * d + 8 * (r >> 2) + 4 * h, a.d, a.vec, v[0], v[1], v[2], v[3]);
            }
    };
    walk(hi, seen, std::false_type{});
    join();
    if (!half && inside) store(row, seen);
    if (!a.causal) return;
    // A second look at rows that are not spoiled by their own log-sum or delta.
    {
        const unsigned long long spoiled = bad_channels(dq);
        bool go = !half && inside && fabsf(lse) < INFINITY && fabsf(delta) < INFINITY && both_max(spoiled ? 1.0f : 0.0f) > 0;
        if (!__syncthreads_or(go)) return;
        const int to = min(hi, common / BN), key0 = max(lo, to) * BN, key1 = min(hi * BN, end);
        if (!__syncthreads_or(find_bad<T>(min(hi * BN, len.k) - key0, a.d, [&](int r) { return kp + (key0 + r) * a.ks[1]; }))) return;       // (of whole tiles)
        const int row = again(first + at0 + (l & 31)), i = query_of(a, row), head = kvh * a.group + row - i * a.group;      // (not worth registers before)
        const int seen = row < rows ? len.seen(a, i) : 0;
        const T* qr = (const T*)a.q + b * a.qs[0] + i * a.qs[1] + head * a.qs[2];
        const T* gr = (const T*)a.dout + b * a.gs[0] + i * a.gs[1] + head * a.gs[2];
#pragma unroll
        for (int d = 0; d < DT; ++d) dq[d] = f32x16{};
        for (int key = key0; key < key1 && __any(go); ++key) {
            if (go && key < seen) {
                const T* kr = kp + key * a.ks[1];
                const float s = dot_of(qr, kr, a.d), p = __builtin_amdgcn_exp2f(fmaf(a.scale < 0 ? -s : s, a.c, -lse));
                add_row<T, DT>(dq, p * (dot_of(gr, vp + key * a.vs[1], a.d) - delta), kr, a.d);
            }
            go = go && both_max(spoiled & ~bad_channels(dq) ? 1.0f : 0.0f) > 0;
        }
        if (!__syncthreads_or(go)) return;
        row_operands<T, D>(q, seen ? qr : nullptr, a.d, VEC, a.scale < 0);
        row_operands<T, D>(g, seen ? gr : nullptr, a.d, VEC, false);
        walk(to, seen, std::false_type{});
        join();
        if (go) store(row, seen);
    }
}

template <typename T, int D> constexpr int kKeyHalves = sizeof(T) == 4 && D == 128 ? 2 : 1;        // wavefronts to a key (HALVES below)
template <typename T, int D> constexpr int kRows = sizeof(T) == 4 ? 32 : 64;     // rows of a tile of k_attention_dkv

// Rows that a tile of `most` takes: whole queries of all heads of the group, or for large groups a part of one query's that divides them.
__host__ __device__ inline int rows_of_tile(int group, int most)
{
    if (group <= most) return most - most % group;
    int n = most;
    while (group % n) --n;
    return n;
}

// A workgroup is 128 keys against tiles of 64 rows (fp32: 32), three tiles in LDS in turn with one barrier a tile.  The scores of the next 32 rows are computed beside this unit's exponentials
// (overlap()): 1.28-1.37 -> 1.19 ms against one unit after the other.  fp32 and heads of more than 64 channels need the registers of a whole CU.
//
// HALVES 2, fp32 heads of 128, whose sums and operands one wavefront's registers do not hold (332 spilled): 64 keys, 32 to two wavefronts that take half of the channels each.  Their parts of the
// scores are exchanged through LDS, then each has the gradients of its own channels (4 x 8 heads x 2000, causal: pass 1990 -> 1120 us; 11 x 64 heads on 8 x 15 of 104 70 -> 39; heads of 64 lose,
// 635 -> 1025).
template <typename T, int D, bool VEC, int HALVES>
__global__ __launch_bounds__(256, (D == 128 || sizeof(T) == 4 ? 1 : 2)) void k_attention_dkv(const AttentionArgs a)
{
    typedef typename FragOf<T>::type Frag;
    constexpr int BM = kRows<T, D>, UNITS = BM / 32, MY = D / HALVES, KS = MY / 16, DT = MY / 32, KEYS = 128 / HALVES;
    typedef Tile<T, D, BM> L;
    constexpr int kTile = L::kBytes;
    // a tile of rows: queries, dout; and of its rows the log-sum in powers of 2, -delta, the number of keys seen
    struct Rows { char tile[2][kTile]; float lse[BM], less[BM]; int seen[BM]; };
    __shared__ __align__(16) Rows r0, r1;           // (apart, so that reads of one need not wait for loads of another)
    int block, split, b, kvh;
    if (!place_of(a, block, split, b, kvh)) return;
    const Lengths len(a, b);
    const int rows = len.q * a.group;               // (rows past the lengths see nothing)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, h = l >> 5;
    const int half = HALVES == 2 ? wave >> 1 : 0, c0 = half * MY, my = a.d - c0;      // this wavefront's channels: c0 .. c0 + MY - 1, `my` or fewer of them there
    const int key0 = block * KEYS, mine = key0 + (HALVES == 2 ? wave & 1 : wave) * 32, key = mine + (l & 31);
    const bool inside = key < len.k;
    // rows that see any of the keys: all from the first query that sees key0 on
    const int from = key0 >= len.k ? rows : a.causal ? (int)min((long long)rows, (long long)max(0, key0 - len.off) * a.group) : 0;
    const int each = rows_of_tile(a.group, BM), t0 = from / each, tiles = from < rows ? (rows + each - 1) / each - t0 : 0;
    const int lo = t0 + (int)((long long)tiles * split / a.splits), hi = t0 + (int)((long long)tiles * (split + 1) / a.splits);

    Frag k[KS], v[KS];
    row_operands<T, MY>(k, inside ? (const T*)a.k + b * a.ks[0] + key * a.ks[1] + kvh * a.ks[2] + c0 : nullptr, my, VEC, a.scale < 0);
    row_operands<T, MY>(v, inside ? (const T*)a.v + b * a.vs[0] + key * a.vs[1] + kvh * a.vs[2] + c0 : nullptr, my, VEC, false);
    const T* qp = (const T*)a.q + b * a.qs[0] + kvh * a.group * a.qs[2];
    const T* gp = (const T*)a.dout + b * a.gs[0] + kvh * a.group * a.gs[2];
    const float* lsep = a.lse + ((long long)b * a.heads + kvh * a.group) * a.q_len;
    const float* deltap = a.delta + (((long long)b * a.kv + kvh) * a.q_len) * a.group;
    Staged<T, D, BM, VEC> sq, sg;
    typedef typename Staged<T, D, BM, VEC>::Bytes Bytes;
    float sl = 0, sd = 0;
    int ss = 0;
    // row r of a tile is head j0 + r % group of query i0 + r / group (a tile is `each` rows: whole queries, or a part of one)
    const int tr = threadIdx.x & (BM - 1), ti = a.group <= BM ? query_of(a, tr) : 0, tj = tr - ti * a.group;
    const auto offset = [&](const long long (&str)[3], int r) {
        const int i = a.group <= BM ? query_of(a, r) : 0;
        return (i * (Bytes)str[1] + (r - i * a.group) * (Bytes)str[2]) * (Bytes)sizeof(T);
    };
    sq.init([&](int r) { return offset(a.qs, r); }, a.d);
    sg.init([&](int r) { return offset(a.gs, r); }, a.d);
    // Rows one0 .. one1 - 1 see one key, the first: their probability is 1 and their ds 0, exactly.  They come in with q = 0 and a log-sum of 0 (or NaN).
    const int first_seeing = a.causal ? min(max(0, -len.off), len.q) : 0;
    const int one0 = first_seeing * a.group, one1 = len.k == 1 ? rows : a.causal && len.off <= 0 ? min(one0 + a.group, rows) : one0;
    const int queries = a.group <= BM ? each / a.group : 0;
    const auto first_query = [&](int t) { return queries ? t * queries : t * each / a.group; };
    const auto fetch = [&](int t, Rows& to) __attribute__((always_inline)) {
        const int i0 = first_query(t), j0 = t * each - i0 * a.group, there = min(rows - t * each, each);
        sq.fetch(to.tile[0], qp + i0 * a.qs[1] + j0 * a.qs[2], there, max(one0 - t * each, 0), one1 - t * each);
        sg.fetch(to.tile[1], gp + i0 * a.gs[1] + j0 * a.gs[2], there);
        if (threadIdx.x < BM) {
            ss = tr < there ? len.seen(a, i0 + ti) : 0;
            sl = ss ? lsep[(long long)(j0 + tj) * a.q_len + i0 + ti] : INFINITY;
            sl = ss == 1 ? one_key(sl) : sl * kLog2e;
            sd = ss ? -deltap[t * each + tr] : 0.0f;
        }
    };
    const auto land = [&](Rows& to) __attribute__((always_inline)) {
        sq.put(to.tile[0]);
        sg.put(to.tile[1]);
        if (threadIdx.x < BM) { to.lse[threadIdx.x] = sl; to.less[threadIdx.x] = sd; to.seen[threadIdx.x] = ss; }
        wait_tiles();
        __syncthreads();
    };
    f32x16 dk[DT] = {}, dv[DT] = {};
    // the sums that S and dP - delta of rows u .. u + 31 of a tile start from
    const auto start = [&](const Rows& at, int u, f32x16& s, f32x16& p) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 less = *(const f32x4*)&at.less[u + 8 * (r >> 2) + 4 * h];
#pragma unroll
            for (int j = 0; j < 4; ++j) { s[r + j] = 0; p[r + j] = less[j]; }
        }
    };
    // pairs of those rows with keys that they do not see: probability and gradient 0, whatever the row's log-sum and delta are
    const auto hide = [&](const Rows& at, int u, f32x16& s, f32x16& p, f32x4 (&lse)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const bool hidden = key >= at.seen[u + 8 * (r >> 2) + 4 * h + (r & 3)];
            s[r] = hidden ? kHidden : s[r];
            p[r] = hidden ? 0.0f : p[r];
            lse[r >> 2][r & 3] = hidden ? 0.0f : lse[r >> 2][r & 3];
        }
    };
    // Whether some row of the tile does not see all of the wavefront's keys.  Rows that there are not are zeros, whose product with a key that is not finite is no number: they are hidden from such ones.
    bool odd_keys = false;
    const auto look_at_keys = [&]() __attribute__((always_inline)) {
        if constexpr (sizeof(T) == 2) {             // (a seen infinity of fp32 is NaN anyway)
            uint32_t carry = 0;                     // out of an exponent of all ones
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    carry |= ((__builtin_bit_cast(u32x4, k[s])[j] & 0x7F807F80u) + 0x00800080u) | ((__builtin_bit_cast(u32x4, v[s])[j] & 0x7F807F80u) + 0x00800080u);
            odd_keys = __any((carry & 0x80008000u) != 0);
        }
    };
    const auto hides = [&](int t) { return odd_keys || (a.causal && len.seen(a, first_query(t)) < mine + 32); };       // (a tile's first row sees the fewest keys)
    const auto walk = [&](int begin) __attribute__((always_inline)) {
        if constexpr (HALVES == 2) {
            static_assert(UNITS == 1, "a tile is a unit");
            __shared__ __align__(16) f32x4 parts[4][8][64];         // of S and dP - delta, by wavefront
            const bool any = mine < len.k;
            const auto tile = [&](int t, Rows& now, Rows& next) __attribute__((always_inline)) {
                if (t + 1 < hi) fetch(t + 1, next);
                f32x16 s = {}, p = {};
                if (any) {
                    if (half == 0) start(now, 0, s, p);
#pragma unroll
                    for (int c = 0; c < KS; ++c) {
                        s = mma(L::along(now.tile[0], 0, half * KS + c), k[c], s);
                        p = mma(L::along(now.tile[1], 0, half * KS + c), v[c], p);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        parts[wave][r][l] = f32x4{s[4 * r], s[4 * r + 1], s[4 * r + 2], s[4 * r + 3]};
                        parts[wave][4 + r][l] = f32x4{p[4 * r], p[4 * r + 1], p[4 * r + 2], p[4 * r + 3]};
                    }
                }
                __syncthreads();                        // (and nobody reads the tile before this any more)
                if (any) {
                    f32x4 lse[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 s2 = parts[wave ^ 2][r][l], p2 = parts[wave ^ 2][4 + r][l];
                        lse[r] = *(const f32x4*)&now.lse[8 * r + 4 * h];
#pragma unroll
                        for (int j = 0; j < 4; ++j) { s[4 * r + j] += s2[j]; p[4 * r + j] += p2[j]; }
                    }
                    if (hides(t)) hide(now, 0, s, p, lse);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -lse[r >> 2][r & 3]));
                        p[r] *= s[r];
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const Frag ps = operand<T>(s, c), ds = operand<T>(p, c);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            dv[d] = mma(L::across(now.tile[1], 16 * c, c0 + 32 * d), ps, dv[d]);
                            dk[d] = mma(L::across(now.tile[0], 16 * c, c0 + 32 * d), ds, dk[d]);
                        }
                    }
                }
                if (t + 1 < hi) land(next);
            };
            if (begin < hi) {
                fetch(begin, r0);
                land(r0);
            }
            for (int t = begin; t < hi; t += 2) {
                tile(t, r0, r1);
                if (t + 1 < hi) tile(t + 1, r1, r0);
            }
        } else {
            __shared__ __align__(16) Rows r2;               // (a third)
            // this unit's probabilities and products (rows u .. of `now`), and the scores of the next one (rows w .. of `next`)
            const auto unit = [&](const Rows& now, int u, const Rows& next, int w, bool some_hidden, f32x16& s, f32x16& p, f32x16& s2, f32x16& p2) __attribute__((always_inline)) {
                Frag fa[2 * KS], fc[2][2 * DT];
                Words<T> ws, we;
                f32x4 lse[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) lse[r] = *(const f32x4*)&now.lse[u + 8 * r + 4 * h];
                if (some_hidden) hide(now, u, s, p, lse);
                start(next, w, s2, p2);
                overlap<2 * KS, 2 * DT>(
                    [&](int i) __attribute__((always_inline)) { fa[i] = L::along(next.tile[i & 1], w, i >> 1); },
                    [&](int i) __attribute__((always_inline)) {
                        if (i & 1) p2 = mma(fa[i], v[i >> 1], p2);
                        else s2 = mma(fa[i], k[i >> 1], s2);
                    },
                    [&](int g) __attribute__((always_inline)) {
#pragma unroll
                        for (int r = 2 * g; r < 2 * g + 2; ++r) {
                            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -lse[r >> 2][r & 3]));
                            p[r] *= s[r];
                        }
                        ws.set(g, s[2 * g], s[2 * g + 1]);
                        we.set(g, p[2 * g], p[2 * g + 1]);
                    },
                    [&](int c, int i) __attribute__((always_inline)) { fc[c][i] = L::across(now.tile[1 - (i & 1)], u + 16 * c, 32 * (i >> 1)); },
                    [&](int c, int i) __attribute__((always_inline)) {
                        if (i & 1) dk[i >> 1] = mma(fc[c][i], we.f[c], dk[i >> 1]);
                        else dv[i >> 1] = mma(fc[c][i], ws.f[c], dv[i >> 1]);
                    });
            };
            f32x16 s0, p0, s1, p1;
            const auto tile = [&](int t, Rows& now, Rows& next, Rows& after, auto odd) __attribute__((always_inline)) {
#pragma unroll
                for (int n = 0; n < UNITS; ++n) {
                    const bool end = n == UNITS - 1;
                    if (end) {                              // the next tile has landed, and nobody reads the one before this
                        if (t + 1 < hi) land(next);
                        if (t + 2 < hi) fetch(t + 2, after);
                    }
                    const Rows& then = end ? next : now;
                    const int w = end ? 0 : 32 * (n + 1);
                    const bool some_hidden = hides(t), flip = UNITS == 1 ? odd : n & 1;
                    if (flip) unit(now, 32 * n, then, w, some_hidden, s1, p1, s0, p0);
                    else unit(now, 32 * n, then, w, some_hidden, s0, p0, s1, p1);
                }
            };
            if (begin < hi) {
                fetch(begin, r0);
                land(r0);
                if (begin + 1 < hi) fetch(begin + 1, r1);
                look_at_keys();
                start(r0, 0, s0, p0);
#pragma unroll
                for (int c = 0; c < KS; ++c) {
                    s0 = mma(L::along(r0.tile[0], 0, c), k[c], s0);
                    p0 = mma(L::along(r0.tile[1], 0, c), v[c], p0);
                }
            }
            const std::false_type even;
            const std::true_type odd;
            for (int t = begin; t < hi; t += 3) {
                tile(t, r0, r1, r2, even);
                if (t + 1 < hi) tile(t + 1, r1, r2, r0, odd);
                if (t + 2 < hi) tile(t + 2, r2, r0, r1, even);
                if constexpr (UNITS == 1) {                 // (the scores change places with every unit)
                    t += 3;
                    if (t < hi) tile(t, r0, r1, r2, odd);
                    if (t + 1 < hi) tile(t + 1, r1, r2, r0, even);
                    if (t + 2 < hi) tile(t + 2, r2, r0, r1, odd);
                }
            }
        }
    };
    const auto store = [&](int key) __attribute__((always_inline)) {
        if (a.splits > 1) {
            const long long n = (long long)a.batch * a.kv * a.kv_len;
            const long long at = ((long long)b * a.kv + kvh) * a.kv_len + key;
            float* pk = a.ws + ((2 * split) * n + at) * D + c0;
            float* pv = pk + n * D;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    *(f32x4*)(pk + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{dk[d][r], dk[d][r + 1], dk[d][r + 2], dk[d][r + 3]};
                    *(f32x4*)(pv + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]};
                }
        } else {
            T* pk = (T*)a.dk + b * a.dks[0] + key * a.dks[1] + kvh * a.dks[2] + c0;
            T* pv = (T*)a.dv + b * a.dvs[0] + key * a.dvs[1] + kvh * a.dvs[2] + c0;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 x = inside ? f32x4{dk[d][r], dk[d][r + 1], dk[d][r + 2], dk[d][r + 3]} * a.scale : f32x4{0, 0, 0, 0};
                    const f32x4 y = inside ? f32x4{dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]} : f32x4{0, 0, 0, 0};
                    store4(pk, 32 * d + 8 * (r >> 2) + 4 * h, my, a.vec, x[0], x[1], x[2], x[3]);
                    store4(pv, 32 * d + 8 * (r >> 2) + 4 * h, my, a.vec, y[0], y[1], y[2], y[3]);
                }
        }
    };
    walk(lo);
    if (key < a.kv_len) store(key);
    if (!a.causal) return;
    // A second look: the tiles with hidden pairs are the first ones.
    {
        const unsigned long long spoiled_k = bad_channels(dk), spoiled_v = bad_channels(dv);
        bool go = inside && both_max(spoiled_k | spoiled_v ? 1.0f : 0.0f) > 0;
        if (!__syncthreads_or(go)) return;
        int begin = lo;
        while (begin < hi && len.seen(a, first_query(begin)) < min(key0 + KEYS, len.k)) ++begin;
        const int row0 = lo * each, row1 = (int)min((long long)begin * each, (long long)rows);
        const auto row_of = [&](const T* p, const long long (&str)[3], int row) { const int i = query_of(a, row); return p + i * str[1] + (row - i * a.group) * str[2]; };
        if (!__syncthreads_or(find_bad<T>(row1 - row0, a.d, [&](int r) { return row_of(qp, a.qs, row0 + r); }) ||
                              find_bad<T>(row1 - row0, a.d, [&](int r) { return row_of(gp, a.gs, row0 + r); }))) return;
        const int key = again(mine + (l & 31));         // (not worth registers before)
        const T* kr = (const T*)a.k + b * a.ks[0] + key * a.ks[1] + kvh * a.ks[2];
        const T* vr = (const T*)a.v + b * a.vs[0] + key * a.vs[1] + kvh * a.vs[2];
#pragma unroll
        for (int d = 0; d < DT; ++d) dk[d] = dv[d] = f32x16{};
        for (int row = row0; row < row1 && __any(go); ++row) {
            const int i = query_of(a, row), sees = len.seen(a, i);
            if (go && sees > key) {
                const T* qr = row_of(qp, a.qs, row);
                const T* gr = row_of(gp, a.gs, row);
                const float lse = lsep[(long long)(row - i * a.group) * a.q_len + i];
                if (sees == 1) {
                    add_row<T, DT>(dv, 1.0f + one_key(lse), gr + c0, my);
                    add_row<T, DT>(dk, one_key(lse), qr + c0, my);
                } else {
                    const float s = dot_of(qr, kr, a.d), p = __builtin_amdgcn_exp2f(fmaf(a.scale < 0 ? -s : s, a.c, -lse * kLog2e));
                    add_row<T, DT>(dv, p, gr + c0, my);
                    add_row<T, DT>(dk, p * (dot_of(gr, vr, a.d) - deltap[row]), qr + c0, my);
                }
            }
            go = go && both_max((spoiled_k & ~bad_channels(dk)) | (spoiled_v & ~bad_channels(dv)) ? 1.0f : 0.0f) > 0;
        }
        if (!__syncthreads_or(go)) return;
        row_operands<T, MY>(k, inside ? kr + c0 : nullptr, my, VEC, a.scale < 0);        // (of all keys: another wavefront may need this one's part of the scores)
        row_operands<T, MY>(v, inside ? vr + c0 : nullptr, my, VEC, false);
        walk(begin);
        if (go) store(key);
    }
}

// Sums of the splits, first split first: rows of D floats, `stride` floats from split to split, each to its place.  KEYS: dk (blockIdx.y 0) and dv (1), else dq.
template <typename T, int D, bool KEYS>
__global__ __launch_bounds__(256) void k_attention_add(const AttentionArgs a, long long stride, int splits)
{
    constexpr int LANES = D / 4;
    const int rows = KEYS ? a.kv_len : a.q_len * a.group;
    const long long n = (long long)a.batch * a.kv * rows, at = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (at >= n) return;
    const int d0 = (threadIdx.x % LANES) * 4, row = (int)(at % rows), kvh = (int)(at / rows % a.kv), b = (int)(at / rows / a.kv);
    const float* parts = a.ws + (blockIdx.y * n + at) * D + d0;
    f32x4 v = {0, 0, 0, 0};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) v += *(const f32x4*)(parts + s * stride);
    const Lengths len(a, b);
    T* p;
    bool any;
    float none = 0;
    if constexpr (KEYS) {
        p = blockIdx.y ? (T*)a.dv + b * a.dvs[0] + row * a.dvs[1] + kvh * a.dvs[2] : (T*)a.dk + b * a.dks[0] + row * a.dks[1] + kvh * a.dks[2];
        any = row < len.k;
    } else {
        const int i = query_of(a, row), head = kvh * a.group + row - i * a.group, seen = len.seen(a, i);
        p = (T*)a.dq + b * a.dqs[0] + i * a.dqs[1] + head * a.dqs[2];
        any = seen > 1;
        if (seen == 1) none = one_key(a.lse[((long long)b * a.heads + head) * a.q_len + i]);
    }
    v = any ? v * (blockIdx.y ? 1.0f : a.scale) : f32x4{none, none, none, none};
    store4(p, d0, a.d, a.vec, v[0], v[1], v[2], v[3]);
}

// Splits of the keys (dq) and of the rows (dk, dv): see forward_splits.
struct Splits { int dq, dkv; };
Splits backward_splits(const ftp_attention_shape& s)
{
    const bool bf = s.dtype == FTP_BF16, wide = s.head_dim > 64;
    const long long rows = (long long)s.q_len * (s.heads / s.kv_heads), all = (long long)s.batch * s.kv_heads;
    const long long nq = ceil_div(rows, 128 / attention_halves(s)) * all, nk = ceil_div(s.kv_len, attention_key_block(!bf && wide)) * all;
    // Workgroups that have a CU by themselves (alone) come in rounds of 256: a split costs its tiles and about as long as 6 for its start, a unit too many and its part of the sum
    // (fp32, 13 x 8 heads on 1, 7 x 1172 tokens of 120: 53 us the pass with splits of at least 8 tiles, 47; 4 heads x 300 of 64 59 -> 41; 8 heads x 1000 of 128 171 -> 144).  More than a round
    // of blocks is split for the last one's sake where a tile is long and the blocks are alike (fp32, 16 heads x 1144 of 128: 473 -> 394; split so, causal bfloats of 128 go 95 -> 123).
    const bool rounds = !bf && wide && !s.causal;
    const auto pick = [rounds](long long blocks, long long tiles, bool alone) {
        if (blocks == 0) return 1;
        if (blocks >= 256 && !rounds) return 1;
        if (!alone) return (int)std::max(1ll, std::min({512 / blocks, tiles / 4, 64ll}));
        const auto cost = [&](long long n) { return ceil_div(blocks * n, 256) * (ceil_div(tiles, n) + 6); };
        long long best = 1;
        for (long long n = 2; n <= std::min(64ll, tiles / 2) && blocks * n < 2048; ++n)
            if (cost(n) < cost(best)) best = n;
        return (int)best;
    };
    return {pick(nq, ceil_div(s.kv_len, bf ? 64 : 32), wide && !bf), pick(nk, ceil_div(rows, rows_of_tile(s.heads / s.kv_heads, bf ? 64 : 32)), wide || !bf)};
}

int padded(const ftp_attention_shape& s) { return s.head_dim <= 32 ? 32 : s.head_dim <= 64 ? 64 : 128; }

template <typename T, int D>
void run(AttentionArgs a, const Splits& n, int halves, hipStream_t st)
{
    const long long rows = (long long)a.q_len * a.group, all = (long long)a.batch * a.kv;
    if (rows) {
        a.blocks = (int)ceil_div(rows, 128 / halves);
        a.splits = n.dq;
        const unsigned grid = place_groups(a);
        constexpr int TWO = sizeof(T) == 4 ? 1 : 2;
        if (halves == TWO) {
            if (a.vec) k_attention_dq<T, D, true, TWO><<<grid, 256, 0, st>>>(a);
            else k_attention_dq<T, D, false, TWO><<<grid, 256, 0, st>>>(a);
        } else {
            if (a.vec) k_attention_dq<T, D, true, 1><<<grid, 256, 0, st>>>(a);
            else k_attention_dq<T, D, false, 1><<<grid, 256, 0, st>>>(a);
        }
        if (n.dq > 1) k_attention_add<T, D, false><<<(unsigned)ceil_div(all * rows, 1024 / D), 256, 0, st>>>(a, all * rows * D, n.dq);
    }
    if (a.kv_len) {
        a.blocks = (int)ceil_div(a.kv_len, 128 / kKeyHalves<T, D>);
        a.splits = n.dkv;
        const unsigned grid = place_groups(a);
        if (a.vec) k_attention_dkv<T, D, true, kKeyHalves<T, D>><<<grid, 256, 0, st>>>(a);
        else k_attention_dkv<T, D, false, kKeyHalves<T, D>><<<grid, 256, 0, st>>>(a);
        if (n.dkv > 1) {
            const long long each = all * a.kv_len * D;
            k_attention_add<T, D, true><<<dim3((unsigned)ceil_div(all * a.kv_len, 1024 / D), 2), 256, 0, st>>>(a, 2 * each, n.dkv);
        }
    }
}

}  // namespace

size_t attention_backward_workspace(const ftp_attention_shape& s)
{
    const Splits n = backward_splits(s);
    const size_t rows = (size_t)s.batch * s.heads * s.q_len, keys = (size_t)s.batch * s.kv_heads * s.kv_len, D = padded(s);
    const size_t parts = std::max(n.dq > 1 ? n.dq * rows * D : 0, n.dkv > 1 ? 2 * n.dkv * keys * D : 0);
    return (rows + 3) / 4 * 16 + parts * sizeof(float);            // delta, then the splits' parts (those of dq first, then those of dk and dv)
}

void attention_backward(const ftp_attention_shape& s, const void* dout, const void* q, const void* k, const void* v, const int* q_lens, const int* kv_lens,
                        const void* out, const float* lse, void* dq, void* dk, void* dv, float* ws, hipStream_t st)
{
    AttentionArgs a = attention_args(s);
    a.q = q; a.k = k; a.v = v; a.q_lens = q_lens; a.kv_lens = kv_lens; a.out = (void*)out; a.lse = (float*)lse;
    a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
    const long long rows = (long long)s.batch * s.heads * s.q_len;
    a.delta = ws;
    a.ws = ws + (rows + 3) / 4 * 4;
    const int el = s.dtype == FTP_BF16 ? 8 : 4;
    a.vec = s.head_dim % el == 0;
    for (const void* p : {q, k, v, out, dout, (const void*)dq, (const void*)dk, (const void*)dv}) a.vec = a.vec && aligned(p, 16);
    for (const long long* t : {a.qs, a.ks, a.vs, a.os, a.gs, a.dqs, a.dks, a.dvs})
        for (int i = 0; i < 3; ++i) a.vec = a.vec && t[i] % el == 0;
    for (const long long* t : {a.ks, a.vs, a.qs, a.gs}) a.vec = a.vec && near_rows(t[1]);
    a.vec = a.vec && near_rows(a.qs[2] * a.group / 128) && near_rows(a.gs[2] * a.group / 128);
    const Splits n = backward_splits(s);
    if (s.dtype == FTP_BF16) {
        if (a.d <= 32) run<bf16_t, 32>(a, n, attention_halves(s), st);
        else if (a.d <= 64) run<bf16_t, 64>(a, n, attention_halves(s), st);
        else run<bf16_t, 128>(a, n, attention_halves(s), st);
    } else {
        if (a.d <= 32) run<float, 32>(a, n, attention_halves(s), st);
        else if (a.d <= 64) run<float, 64>(a, n, attention_halves(s), st);
        else run<float, 128>(a, n, attention_halves(s), st);
    }
}

}  // namespace ftp
