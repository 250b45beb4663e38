// Softmax attention, forward: out = softmax(scale q k^T) v over the keys a query sees, one pass over the keys with the running maximum and sum of each row.
//
// A workgroup is 128 rows (32 a wavefront; or 64, two wavefronts to 32) against tiles of keys, staged in LDS with the next tile's loads in flight.  S^T = K Q^T puts a row's scores into one lane pair
// (lane % 32), so maximum, sum and rescaling are per lane; P^T is then the operand of O^T = V^T P^T as it lies (ftp_attention.h).  Few rows (single tokens): the keys are
// split over workgroups, whose unnormalised rows a second kernel joins.
//
// Measured: prompts, 4 images of 1550 to 2704 tokens, 8 heads of 128 on 2, causal, bfloats: 61.5 us, 552 TFLOP/s (bound by the longest workgroups: 42 tiles behind each other on a SIMD shared
// with another such, 28 on average); 64 heads x 5776 tokens of 64: 0.59-0.64 ms, 850-920 TFLOP/s (vector unit 81 % busy, a third of it exponentials; matrix cores 46 %); one token of 8 streams on up to 8192
// keys: 26 us among other calls, 23 with what the call before left in the last-level cache (91 MB, 4.0 TB/s), 4 of them the join.  fp32: prompts 323 us (105 TFLOP/s), one token 106 (1.7 TB/s:
// a CU holds one workgroup).
#include "ftp_attention.h"

#include <algorithm>
#include <cmath>

namespace ftp {
namespace {

template <typename T, int D> constexpr int kKeys = sizeof(T) == 4 ? 32 : 64;       // keys of a tile

// HALVES 1: 128 rows a workgroup, 32 a wavefront.  2: 64 rows, each by two wavefronts that take the tile's 32-key units in turn and join their rows through LDS at the end: half as long
// chains, twice the staging (see attention_halves()).
template <typename T, int D, bool VEC, int HALVES>
__global__ __launch_bounds__(256, (kPerCu<T, D>)) void k_attention(const AttentionArgs a)
{
    typedef typename FragOf<T>::type Frag;
    constexpr int BN = kKeys<T, D>, UNITS = BN / 32 / HALVES, KS = D / 16, DT = D / 32, ROWS = 128 / HALVES;
    typedef Tile<T, D, BN> L;
    constexpr int kTile = L::kBytes;
    struct Keys { char tile[2][kTile]; };           // a tile of keys and values
    __shared__ __align__(16) Keys even, odd;        // (apart, so that reads of one need not wait for loads of the other)
    static_assert(UNITS > 0 && (HALVES == 1 || (int)sizeof(Keys) >= 2 * DT * 4096), "a unit a wavefront; two wavefronts' rows in a tile's place");
    int block, split, b, kvh;
    if (!place_of(a, block, split, b, kvh)) return;
    if (a.causal) block = a.blocks - 1 - block;     // the longest ones first
    const Lengths len(a, b);
    const int rows = a.q_len * a.group;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, h = l >> 5;
    const int half = HALVES == 2 ? wave >> 1 : 0, at0 = (HALVES == 2 ? wave & 1 : wave) * 32, mine0 = 32 * half;         // this wavefront's rows, and its unit's first key of a tile
    const int first = block * ROWS, row = first + at0 + (l & 31);
    const int i = query_of(a, row), head = kvh * a.group + row - i * a.group;
    const bool inside = row < rows;
    const int seen = inside ? len.seen(a, i) : 0;
    // keys that some row of the workgroup sees, and those that all its rows inside the lengths see
    const int last = query_of(a, min(first + ROWS, rows) - 1), i0 = query_of(a, first);
    const int end = i0 < len.q ? len.seen(a, min(last, len.q - 1)) : 0, common = len.seen(a, i0);
    const int tiles = (end + BN - 1) / BN, lo = (int)((long long)tiles * split / a.splits), hi = (int)((long long)tiles * (split + 1) / a.splits);

    Frag q[D / 16];
    row_operands<T, D>(q, seen ? (const T*)a.q + b * a.qs[0] + i * a.qs[1] + head * a.qs[2] : nullptr, a.d, VEC, a.scale < 0);
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

    f32x16 o[DT] = {};
    constexpr float nothing = -3e38f;               // the reference of a row that has seen no key: below all scores, and a number
    float m = nothing, sum = 0;
    const auto step = [&](int t, int to, int seen, Keys& now, Keys& next) __attribute__((always_inline)) {
        if (t + 1 < to) fetch(t + 1, next);
        f32x16 s[UNITS] = {};
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int c = 0; c < KS; ++c) s[u] = mma(L::along(now.tile[0], mine0 + 32 * u, c), q[c], s[u]);
        if ((t + 1) * BN > common) {
            const int left = seen - t * BN - mine0 - 4 * h;            // keys of the tile that the row sees, counted from this lane's first
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = 32 * u + 8 * (r >> 2) + (r & 3) >= left ? kHidden : s[u][r];
        }
        float top = kHidden;
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
        top = both_max(top) * a.c;
        // the reference only has to keep the powers in range: it follows the maximum once that is 2^8 ahead (exact all the same: sums and rows share it), and only then, so
        // that a row's bits do not go by its neighbours'
        if (__any(top > m + 8.0f)) {
            top = top > m + 8.0f ? top : m;
            const float f = __builtin_amdgcn_exp2f(m - top);
            sum *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= f;
            m = top;
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[u][r] = __builtin_amdgcn_exp2f(fmaf(s[u][r], a.c, -m));
                sum += s[u][r];
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const Frag p = operand<T>(s[u], c);
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] = mma(L::across(now.tile[1], mine0 + 32 * u + 16 * c, 32 * d), p, o[d]);
            }
        }
        if (t + 1 < to) land(next);
    };
    const auto walk = [&](int to, int seen) __attribute__((always_inline)) {
        if (lo < to) {
            fetch(lo, even);
            land(even);
        }
        for (int t = lo; t < to; t += 2) {
            step(t, to, seen, even, odd);
            if (t + 1 < to) step(t + 1, to, seen, odd, even);
        }
    };
    // two wavefronts' rows and sums become the first one's
    const auto join = [&]() __attribute__((always_inline)) {
        if constexpr (HALVES == 2) {
            // (the tiles' last readers are behind a barrier: a wavefront leaves the loop's last tile by itself, so one more)
            f32x4* part = (f32x4*)&even + (at0 / 32) * DT * 4 * 64;
            float* stats = (float*)&odd + (at0 / 32) * 128;
            __syncthreads();
            if (half) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) part[(d * 4 + r) * 64 + l] = f32x4{o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]};
                stats[l] = m;
                stats[64 + l] = sum;
            }
            __syncthreads();
            if (half) return;
            const float m2 = stats[l], top = fmaxf(m, m2), f = __builtin_amdgcn_exp2f(m - top), f2 = __builtin_amdgcn_exp2f(m2 - top);
            sum = sum * f + stats[64 + l] * f2;
            m = top;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x4 v = part[(d * 4 + r) * 64 + l];
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[d][4 * r + j] = o[d][4 * r + j] * f + v[j] * f2;
                }
        }
    };
    const auto store = [&](int row, int seen, float sum, bool stats) __attribute__((always_inline)) {
        const int i = query_of(a, row), head = kvh * a.group + row - i * a.group;
        if (a.splits > 1) {
            // [split][image][key head][row][D], and the rows' maxima and sums behind
            const long long at = (((long long)split * a.batch + b) * a.kv + kvh) * rows + row, n = (long long)a.splits * a.batch * a.kv * rows;
            float* p = a.ws + at * D;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(f32x4*)(p + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
            if (h == 0 && stats) { a.ws[n * D + 2 * at] = m; a.ws[n * D + 2 * at + 1] = sum; }
            return;
        }
        const float inv = seen ? 1.0f / sum : 0.0f;
        T* p = (T*)a.out + b * a.os[0] + i * a.os[1] + head * a.os[2];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 v = seen ? f32x4{o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv} : f32x4{0, 0, 0, 0};
                store4(p, 32 * d + 8 * (r >> 2) + 4 * h, a.d, a.vec, v[0], v[1], v[2], v[3]);
            }
        if (h == 0 && a.lse && stats) a.lse[((long long)b * a.heads + head) * a.q_len + i] = seen ? fmaf(m, kLn2, logf(sum)) : -INFINITY;
    };
    walk(hi, seen);
    sum = both_sum(sum);
    join();
    if (!half && inside) store(row, seen, sum, true);
    if (!a.causal) return;
    // A second look at rows whose values, but not their scores, spoiled them: the maxima and sums stand.
    {
        const unsigned long long spoiled = bad_channels(o);
        bool go = !half && inside && sum < INFINITY && both_max(spoiled ? 1.0f : 0.0f) > 0;
        if (!__syncthreads_or(go)) return;
        const int to = min(hi, common / BN), key0 = max(lo, to) * BN, key1 = min(hi * BN, end);
        if (!__syncthreads_or(find_bad<T>(min(hi * BN, len.k) - key0, a.d, [&](int r) { return vp + (key0 + r) * a.vs[1]; }))) return;       // (of whole tiles)
        const int row = again(first + at0 + (l & 31)), i = query_of(a, row), head = kvh * a.group + row - i * a.group;      // (not worth registers before)
        const int seen = row < rows ? len.seen(a, i) : 0;
        const T* qr = (const T*)a.q + b * a.qs[0] + i * a.qs[1] + head * a.qs[2];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x16{};
        for (int key = key0; key < key1 && __any(go); ++key) {
            if (go && key < seen) {
                const float s = dot_of(qr, kp + key * a.ks[1], a.d);
                add_row<T, DT>(o, __builtin_amdgcn_exp2f(fmaf(a.scale < 0 ? -s : s, a.c, -m)), vp + key * a.vs[1], a.d);
            }
            go = go && both_max(spoiled & ~bad_channels(o) ? 1.0f : 0.0f) > 0;
        }
        if (!__syncthreads_or(go)) return;
        const float total = sum;
        row_operands<T, D>(q, seen ? qr : nullptr, a.d, VEC, a.scale < 0);
        walk(to, seen);
        join();
        if (go) store(row, seen, total, false);
    }
}

// Joins the splits of a row: D / 4 lanes with four channels each, GROUPS of them with every GROUPS-th split.  Few rows have a workgroup each, so that all loads are on their way at
// once (128 rows of 16 splits 8.0 -> 3.9 us); many have one group each.
template <typename T, int D, int GROUPS>
__global__ __launch_bounds__(256) void k_attention_join(const AttentionArgs a)
{
    constexpr int LANES = D / 4, ROWS = 256 / (LANES * GROUPS);
    __shared__ f32x4 part[256 / LANES][LANES];
    __shared__ float part_sum[256 / LANES];
    const int rows = a.q_len * a.group, all = a.batch * a.kv * rows, mine = threadIdx.x / LANES;
    const int sub = mine / GROUPS, grp = mine % GROUPS, at = min((int)blockIdx.x * ROWS + sub, all - 1);
    const long long per = all;
    const int lane = threadIdx.x % LANES, d0 = lane * 4;
    const int bk = at / rows, row = at - bk * rows, b = bk / a.kv, kvh = bk - b * a.kv, i = query_of(a, row), head = kvh * a.group + row - i * a.group;
    const float* ms = a.ws + per * a.splits * D;
    float m = -INFINITY;
    for (int s = lane; s < a.splits; s += LANES) m = fmaxf(m, ms[2 * (s * per + at)]);
#pragma unroll
    for (int n = LANES / 2; n; n >>= 1) m = fmaxf(m, __shfl_xor(m, n));
    f32x4 o = {0, 0, 0, 0};
    float sum = 0;
#pragma unroll 4
    for (int s = grp; s < a.splits; s += GROUPS) {
        const long long p = s * per + at;
        const float f = __builtin_amdgcn_exp2f(ms[2 * p] - m);
        o += *(const f32x4*)(a.ws + p * D + d0) * f;
        sum = fmaf(ms[2 * p + 1], f, sum);
    }
    if constexpr (GROUPS > 1) {
        part[mine][lane] = o;
        if (lane == 0) part_sum[mine] = sum;
        __syncthreads();
        if (grp) return;
#pragma unroll
        for (int n = 1; n < GROUPS; ++n) { o += part[mine + n][lane]; sum += part_sum[mine + n]; }
    }
    if ((int)blockIdx.x * ROWS + sub >= all) return;
    const bool any = Lengths(a, b).seen(a, i) > 0;
    o = any ? o * (1.0f / sum) : f32x4{0, 0, 0, 0};
    store4((T*)a.out + b * a.os[0] + i * a.os[1] + head * a.os[2], d0, a.d, a.vec, o[0], o[1], o[2], o[3]);
    if (d0 == 0 && a.lse) a.lse[((long long)b * a.heads + head) * a.q_len + i] = any ? fmaf(m, kLn2, logf(sum)) : -INFINITY;
}

// Splits of the keys: none where the blocks of rows give every CU a workgroup; else as many as do, of at least 4 tiles.
int forward_splits(const ftp_attention_shape& s)
{
    const long long blocks = ceil_div((long long)s.q_len * (s.heads / s.kv_heads), 128 / attention_halves(s)) * s.batch * s.kv_heads;
    const long long tiles = ceil_div(s.kv_len, s.dtype == FTP_BF16 ? 64 : 32);
    if (blocks == 0 || blocks >= 256) return 1;
    return (int)std::max(1ll, std::min({512 / blocks, tiles / 4, 128ll}));
}

template <typename T, int D>
void run(const AttentionArgs& a, bool two, unsigned grid, hipStream_t st)
{
    if (sizeof(T) == 2 && two) {
        if (a.vec) k_attention<T, D, true, sizeof(T) == 2 ? 2 : 1><<<grid, 256, 0, st>>>(a);
        else k_attention<T, D, false, sizeof(T) == 2 ? 2 : 1><<<grid, 256, 0, st>>>(a);
    } else {
        if (a.vec) k_attention<T, D, true, 1><<<grid, 256, 0, st>>>(a);
        else k_attention<T, D, false, 1><<<grid, 256, 0, st>>>(a);
    }
    if (a.splits > 1) {
        const long long rows = (long long)a.batch * a.kv * a.q_len * a.group;
        if (rows <= 2048) k_attention_join<T, D, 1024 / D><<<(unsigned)rows, 256, 0, st>>>(a);
        else k_attention_join<T, D, 1><<<(unsigned)ceil_div(rows, 1024 / D), 256, 0, st>>>(a);
    }
}

}  // namespace

// Wavefronts to a row.  Two (bfloats: an fp32 tile is one unit) where a workgroup has at most 64 rows anyway (256 streams x 8 heads of one token on 200 keys 25.8 -> 23.7 us), and where 128 rows each
// leave the chip few chains of tiles, or uneven ones that causal calls end on (4 x 12 heads x 577 tokens 22.6 -> 13.1 us, 2 x 8 x 2600 52 -> 46, causal 4 x 8 x 2600 62 -> 49); heads of 128 pay
// more for staging twice (causal 2 x 8 x 2600 56 -> 50, all pairs 77 -> 88).  With enough of them 128 rows are better: 8 x 8 x 5776 tokens 597 us, halves 656.
int attention_halves(const ftp_attention_shape& s)
{
    const long long rows = (long long)s.q_len * (s.heads / s.kv_heads), groups = ceil_div(rows, 128) * s.batch * s.kv_heads;
    const bool narrow = s.head_dim <= 64;
    if (s.dtype != FTP_BF16) return 1;
    return rows <= 64 || groups < (narrow && s.causal ? 768 : narrow || s.causal ? 384 : 256) ? 2 : 1;
}

bool attention_fits(const ftp_attention_shape& s)
{
    const long long rows = (long long)s.q_len * (s.heads / s.kv_heads), groups = (long long)s.batch * s.kv_heads;
    const long long blocks = std::max(ceil_div(rows, 128 / attention_halves(s)), ceil_div(s.kv_len, attention_key_block(s.dtype == FTP_F32 && s.head_dim > 64)));
    // (splits come only where there are few; what rounds groups up to eights may come or not, by the lengths)
    return groups <= kMostGroups && blocks <= kMostGroups && std::max(place_count(groups, blocks, true), place_count(groups, blocks, false)) <= kMostGroups;
}

AttentionArgs attention_args(const ftp_attention_shape& s)
{
    AttentionArgs a = {};
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = s.q_stride[i]; a.ks[i] = s.k_stride[i]; a.vs[i] = s.v_stride[i]; a.os[i] = s.out_stride[i];
        a.gs[i] = s.dout_stride[i]; a.dqs[i] = s.dq_stride[i]; a.dks[i] = s.dk_stride[i]; a.dvs[i] = s.dv_stride[i];
    }
    a.batch = s.batch; a.heads = s.heads; a.kv = s.kv_heads; a.group = s.heads / s.kv_heads;
    a.q_len = s.q_len; a.kv_len = s.kv_len; a.d = s.head_dim; a.causal = s.causal && s.q_len > 1;             // (one query sees all keys)
    a.scale = s.scale;
    a.c = std::max(std::fabs(s.scale) * kLog2e, 1e-45f);             // (0 would make NaN of a hidden score, -infinity; this leaves 5e-7 of the largest one)
    return a;
}

size_t attention_forward_workspace(const ftp_attention_shape& s)
{
    const int splits = forward_splits(s), D = s.head_dim <= 32 ? 32 : s.head_dim <= 64 ? 64 : 128;
    return splits > 1 ? (size_t)splits * s.batch * s.heads * s.q_len * (D + 2) * sizeof(float) : 0;
}

void attention_forward(const ftp_attention_shape& s, const void* q, const void* k, const void* v, const int* q_lens, const int* kv_lens, void* out, float* lse,
                       float* ws, hipStream_t st)
{
    AttentionArgs a = attention_args(s);
    a.q = q; a.k = k; a.v = v; a.q_lens = q_lens; a.kv_lens = kv_lens; a.out = out; a.lse = lse; a.ws = ws;
    const int el = s.dtype == FTP_BF16 ? 8 : 4;
    a.vec = s.head_dim % el == 0 && aligned(q, 16) && aligned(k, 16) && aligned(v, 16) && aligned(out, 16);
    for (int i = 0; i < 3; ++i) a.vec = a.vec && a.qs[i] % el == 0 && a.ks[i] % el == 0 && a.vs[i] % el == 0 && a.os[i] % el == 0;
    a.vec = a.vec && near_rows(a.ks[1]) && near_rows(a.vs[1]);
    const bool two = attention_halves(s) == 2;
    a.blocks = (int)ceil_div((long long)a.q_len * a.group, two ? 64 : 128);
    a.splits = forward_splits(s);
    const unsigned grid = place_groups(a);
    if (s.dtype == FTP_BF16) {
        if (a.d <= 32) run<bf16_t, 32>(a, two, grid, st);
        else if (a.d <= 64) run<bf16_t, 64>(a, two, grid, st);
        else run<bf16_t, 128>(a, two, grid, st);
    } else {
        if (a.d <= 32) run<float, 32>(a, two, grid, st);
        else if (a.d <= 64) run<float, 64>(a, two, grid, st);
        else run<float, 128>(a, two, grid, st);
    }
}

}  // namespace ftp
