// Softmax attention, backward: the probabilities are computed again from q, k and the rows' log-sums,
//   p = exp(scale q.k - lse), delta = sum_d dout out, ds = p (dout.v - delta), dv = sum_rows p dout, dq = scale sum_keys ds k, dk = scale sum_rows ds q.
//
// Two kernels, so that every sum stays in one workgroup's registers and in one order: k_attention_dq walks over the keys of 128 rows (as the forward pass does, and leaves
// delta), k_attention_dkv over the rows of 128 keys.  Scores and dout.v are computed in both: seven products of the pairs instead of five, where one kernel would add dq up by
// atomics, in an order that changes.  In dq S^T and dP^T have a row per lane, in dkv S and dP a key per lane, so that P and dS again are operands as they lie
// (ftp_attention.h).  Where 128-row (key) blocks are too few for the CUs, the other axis is split and the parts are added up by a third kernel.
#include "ftp_attention.h"

#include <algorithm>
#include <cmath>

namespace ftp {
namespace {

template <typename T> constexpr int kKeys = sizeof(T) == 4 ? 32 : 64;

template <typename T, int D>
__global__ __launch_bounds__(256) void k_attention_dq(const AttentionArgs a)
{
    typedef Tile<T, D> L;
    typedef typename FragOf<T>::type Frag;
    constexpr int BN = kKeys<T>, SUB = BN / 32, DT = D / 32, kTile = BN * L::kRow;
    __shared__ __align__(16) char lds[2][2][kTile];
    int block, split, b, kvh;
    if (!place_of(a, block, split, b, kvh)) return;
    if (a.causal) block = a.blocks - 1 - block;
    const Lengths len(a, b);
    const int rows = a.q_len * a.group;
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int first = block * 128, row = first + wave * 32 + (l & 31);
    const int i = query_of(a, row), head = kvh * a.group + row - i * a.group;
    const bool inside = row < rows;
    const int seen = inside ? len.seen(a, i) : 0;
    const int last = query_of(a, min(first + 128, rows) - 1), i0 = query_of(a, first);
    const int end = i0 < len.q ? len.seen(a, min(last, len.q - 1)) : 0, common = len.seen(a, i0);
    const int tiles = (end + BN - 1) / BN, lo = (int)((long long)tiles * split / a.splits), hi = (int)((long long)tiles * (split + 1) / a.splits);
    const bool busy = first + wave * 32 < rows;

    // this row's operands; delta from the same dout and the row of out
    Frag q[D / 16], g[D / 16];
    float delta = 0;
    {
        row_operands<T, D>(g, seen ? (const T*)a.out + b * a.os[0] + i * a.os[1] + head * a.os[2] : nullptr, a.d, a.vec, false);
        Frag o[D / 16];
#pragma unroll
        for (int s = 0; s < D / 16; ++s) o[s] = g[s];
        row_operands<T, D>(g, seen ? (const T*)a.dout + b * a.gs[0] + i * a.gs[1] + head * a.gs[2] : nullptr, a.d, a.vec, false);
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta = fmaf((float)o[s][j], (float)g[s][j], delta);
        delta = both_sum(delta);
    }
    const long long at = (((long long)b * a.kv + kvh) * a.q_len) * a.group + row;
    if (split == 0 && inside && h == 0) a.delta[at] = delta;
    row_operands<T, D>(q, seen ? (const T*)a.q + b * a.qs[0] + i * a.qs[1] + head * a.qs[2] : nullptr, a.d, a.vec, a.scale < 0);
    const float lse = seen ? a.lse[((long long)b * a.heads + head) * a.q_len + i] * kLog2e : INFINITY;     // (a row that sees nothing: p = 0)

    const T* kp = (const T*)a.k + b * a.ks[0] + kvh * a.ks[2];
    const T* vp = (const T*)a.v + b * a.vs[0] + kvh * a.vs[2];
    Staged<T, D, BN> sk, sv;
    const auto fetch = [&](int t) {
        sk.fetch([&](int r) { const int key = t * BN + r; return key < len.k ? kp + key * a.ks[1] : nullptr; }, a.d, a.vec);
        sv.fetch([&](int r) { const int key = t * BN + r; return key < len.k ? vp + key * a.vs[1] : nullptr; }, a.d, a.vec);
    };
    f32x16 dq[DT] = {};
    if (lo < hi) {
        fetch(lo);
        sk.put(lds[0][0]);
        sv.put(lds[0][1]);
        __syncthreads();
    }
    for (int t = lo; t < hi; ++t) {
        const char* tk = lds[(t - lo) & 1][0];
        const char* tv = lds[(t - lo) & 1][1];
        if (t + 1 < hi) fetch(t + 1);
        if (busy) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                f32x16 s = {}, p = {};
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    s = mma(L::along(tk, 32 * u, k), q[k], s);
                    p = mma(L::along(tv, 32 * u, k), g[k], p);
                }
                const bool mask = (t + 1) * BN > common;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -lse)) * (p[r] - delta);
                    s[r] = mask && t * BN + 32 * u + 8 * (r >> 2) + 4 * h + (r & 3) >= seen ? 0.0f : e;
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const Frag ds = operand<T>(s, k);
#pragma unroll
                    for (int d = 0; d < DT; ++d) dq[d] = mma(L::across(tk, 32 * u + 16 * k, 32 * d), ds, dq[d]);
                }
            }
        }
        if (t + 1 < hi) {
            sk.put(lds[(t + 1 - lo) & 1][0]);
            sv.put(lds[(t + 1 - lo) & 1][1]);
        }
        __syncthreads();
    }
    if (!inside) return;
    if (a.causal && __any(not_finite(dq))) {
        const T* qr = (const T*)a.q + b * a.qs[0] + i * a.qs[1] + head * a.qs[2];
        const T* gr = (const T*)a.dout + b * a.gs[0] + i * a.gs[1] + head * a.gs[2];
        if (both_max(not_finite(dq) ? 1.0f : 0.0f) > 0) {
#pragma unroll
            for (int d = 0; d < DT; ++d) dq[d] = f32x16{};
            for (int key = lo * BN; key < min(hi * BN, seen); ++key) {
                const T* kr = kp + key * a.ks[1];
                const float s = dot_of(qr, kr, a.d), p = __builtin_amdgcn_exp2f(fmaf(a.scale < 0 ? -s : s, a.c, -lse));
                add_row<T, DT>(dq, p * (dot_of(gr, vp + key * a.vs[1], a.d) - delta), kr, a.d);
            }
        }
    }
    if (a.splits > 1) {
        float* p = a.ws + (((long long)split * a.batch * a.kv * rows) + at) * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(f32x4*)(p + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{dq[d][r], dq[d][r + 1], dq[d][r + 2], dq[d][r + 3]};
        return;
    }
    T* p = (T*)a.dq + b * a.dqs[0] + i * a.dqs[1] + head * a.dqs[2];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 v = seen ? f32x4{dq[d][r], dq[d][r + 1], dq[d][r + 2], dq[d][r + 3]} * a.scale : f32x4{0, 0, 0, 0};
            store4(p, 32 * d + 8 * (r >> 2) + 4 * h, a.d, a.vec, v[0], v[1], v[2], v[3]);
        }
}

constexpr int kRows = 32;                           // rows of a tile of k_attention_dkv

template <typename T, int D>
__global__ __launch_bounds__(256) void k_attention_dkv(const AttentionArgs a)
{
    typedef Tile<T, D> L;
    typedef typename FragOf<T>::type Frag;
    constexpr int DT = D / 32, kTile = kRows * L::kRow;
    __shared__ __align__(16) char lds[2][2][kTile];
    __shared__ float stat[2][2][kRows];             // lse (in powers of 2) and delta of a tile's rows
    __shared__ int seen_by[2][kRows];
    int block, split, b, kvh;
    if (!place_of(a, block, split, b, kvh)) return;
    const Lengths len(a, b);
    const int rows = len.q * a.group;               // (rows past the lengths see nothing)
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int key0 = block * 128, key = key0 + wave * 32 + (l & 31);
    const bool inside = key < len.k;
    // rows that see any of the keys: all from the first query that sees key0 on
    const int from = key0 >= len.k ? rows : a.causal ? min((long long)rows, (long long)max(0, key0 - len.off) * a.group) : 0;
    const int t0 = from / kRows, tiles = from < rows ? (rows + kRows - 1) / kRows - t0 : 0;
    const int lo = t0 + (int)((long long)tiles * split / a.splits), hi = t0 + (int)((long long)tiles * (split + 1) / a.splits);
    const bool busy = key0 + wave * 32 < len.k;

    Frag k[D / 16], v[D / 16];
    row_operands<T, D>(k, inside ? (const T*)a.k + b * a.ks[0] + key * a.ks[1] + kvh * a.ks[2] : nullptr, a.d, a.vec, a.scale < 0);
    row_operands<T, D>(v, inside ? (const T*)a.v + b * a.vs[0] + key * a.vs[1] + kvh * a.vs[2] : nullptr, a.d, a.vec, false);
    const T* qp = (const T*)a.q + b * a.qs[0] + kvh * a.group * a.qs[2];
    const T* gp = (const T*)a.dout + b * a.gs[0] + kvh * a.group * a.gs[2];
    const float* lsep = a.lse + ((long long)b * a.heads + kvh * a.group) * a.q_len;
    const float* deltap = a.delta + (((long long)b * a.kv + kvh) * a.q_len) * a.group;
    Staged<T, D, kRows> sq, sg;
    float sl = 0, sd = 0;
    int ss = 0;
    const auto fetch = [&](int t) {
        const auto address = [&](const T* p, const long long (&str)[3], int r) {
            const int row = t * kRows + r, i = query_of(a, row);
            return row < rows && len.seen(a, i) > 0 ? p + i * str[1] + (row - i * a.group) * str[2] : nullptr;
        };
        sq.fetch([&](int r) { return address(qp, a.qs, r); }, a.d, a.vec);
        sg.fetch([&](int r) { return address(gp, a.gs, r); }, a.d, a.vec);
        if (threadIdx.x < kRows) {
            const int row = t * kRows + threadIdx.x, i = query_of(a, row);
            ss = row < rows ? len.seen(a, i) : 0;
            sl = ss ? lsep[(long long)(row - i * a.group) * a.q_len + i] * kLog2e : INFINITY;
            sd = ss ? deltap[row] : 0.0f;
        }
    };
    const auto put = [&](int buf) {
        sq.put(lds[buf][0]);
        sg.put(lds[buf][1]);
        if (threadIdx.x < kRows) { stat[buf][0][threadIdx.x] = sl; stat[buf][1][threadIdx.x] = sd; seen_by[buf][threadIdx.x] = ss; }
    };
    f32x16 dk[DT] = {}, dv[DT] = {};
    if (lo < hi) {
        fetch(lo);
        put(0);
        __syncthreads();
    }
    for (int t = lo; t < hi; ++t) {
        const int buf = (t - lo) & 1;
        const char* tq = lds[buf][0];
        const char* tg = lds[buf][1];
        if (t + 1 < hi) fetch(t + 1);
        if (busy) {
            f32x16 s = {}, p = {};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                s = mma(L::along(tq, 0, c), k[c], s);
                p = mma(L::along(tg, 0, c), v[c], p);
            }
            // the tile's first row sees the fewest keys
            const bool mask = a.causal && query_of(a, t * kRows) + len.off + 1 < key0 + 128;
            f32x16 e;
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 lse = *(const f32x4*)&stat[buf][0][8 * (r >> 2) + 4 * h], delta = *(const f32x4*)&stat[buf][1][8 * (r >> 2) + 4 * h];
                typedef int i32x4 __attribute__((ext_vector_type(4)));
                const i32x4 seen = *(const i32x4*)&seen_by[buf][8 * (r >> 2) + 4 * h];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(s[r + j], a.c, -lse[j]));
                    const bool hidden = mask && key >= seen[j];
                    e[r + j] = hidden ? 0.0f : w * (p[r + j] - delta[j]);
                    s[r + j] = hidden ? 0.0f : w;
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const Frag fp = operand<T>(s, c), fe = operand<T>(e, c);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    dv[d] = mma(L::across(tg, 16 * c, 32 * d), fp, dv[d]);
                    dk[d] = mma(L::across(tq, 16 * c, 32 * d), fe, dk[d]);
                }
            }
        }
        if (t + 1 < hi) put(buf ^ 1);
        __syncthreads();
    }
    if (key >= a.kv_len) return;
    if (a.causal && __any(not_finite(dk) || not_finite(dv))) {
        if (both_max(not_finite(dk) || not_finite(dv) ? 1.0f : 0.0f) > 0 && inside) {
            const T* kr = (const T*)a.k + b * a.ks[0] + key * a.ks[1] + kvh * a.ks[2];
            const T* vr = (const T*)a.v + b * a.vs[0] + key * a.vs[1] + kvh * a.vs[2];
#pragma unroll
            for (int d = 0; d < DT; ++d) dk[d] = dv[d] = f32x16{};
            for (int row = lo * kRows; row < min(hi * kRows, rows); ++row) {
                const int i = query_of(a, row), j = row - i * a.group;
                if (len.seen(a, i) <= key) continue;
                const T* qr = qp + i * a.qs[1] + j * a.qs[2];
                const T* gr = gp + i * a.gs[1] + j * a.gs[2];
                const float s = dot_of(qr, kr, a.d), p = __builtin_amdgcn_exp2f(fmaf(a.scale < 0 ? -s : s, a.c, -lsep[(long long)j * a.q_len + i] * kLog2e));
                add_row<T, DT>(dv, p, gr, a.d);
                add_row<T, DT>(dk, p * (dot_of(gr, vr, a.d) - deltap[row]), qr, a.d);
            }
        }
    }
    if (a.splits > 1) {
        const long long n = (long long)a.batch * a.kv * a.kv_len;
        const long long at = ((long long)b * a.kv + kvh) * a.kv_len + key;
        float* pk = a.ws + ((2 * split) * n + at) * D;
        float* pv = pk + n * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                *(f32x4*)(pk + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{dk[d][r], dk[d][r + 1], dk[d][r + 2], dk[d][r + 3]};
                *(f32x4*)(pv + 32 * d + 8 * (r >> 2) + 4 * h) = f32x4{dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]};
            }
        return;
    }
    T* pk = (T*)a.dk + b * a.dks[0] + key * a.dks[1] + kvh * a.dks[2];
    T* pv = (T*)a.dv + b * a.dvs[0] + key * a.dvs[1] + kvh * a.dvs[2];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 x = inside ? f32x4{dk[d][r], dk[d][r + 1], dk[d][r + 2], dk[d][r + 3]} * a.scale : f32x4{0, 0, 0, 0};
            const f32x4 y = inside ? f32x4{dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]} : f32x4{0, 0, 0, 0};
            store4(pk, 32 * d + 8 * (r >> 2) + 4 * h, a.d, a.vec, x[0], x[1], x[2], x[3]);
            store4(pv, 32 * d + 8 * (r >> 2) + 4 * h, a.d, a.vec, y[0], y[1], y[2], y[3]);
        }
}

// Sums of the splits, first split first: rows of D floats `stride` floats apart from split to split, each to its place.  WHICH: 0 dq, 1 dk, 2 dv.
template <typename T, int D, int WHICH>
__global__ __launch_bounds__(256) void k_attention_add(const AttentionArgs a, const float* parts, long long stride, int splits)
{
    constexpr int LANES = D / 4;
    const int rows = WHICH ? a.kv_len : a.q_len * a.group;
    const long long at = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (at >= (long long)a.batch * a.kv * rows) return;
    const int d0 = (threadIdx.x % LANES) * 4, row = (int)(at % rows), kvh = (int)(at / rows % a.kv), b = (int)(at / rows / a.kv);
    f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) v += *(const f32x4*)(parts + s * stride + at * D + d0);
    T* p;
    if constexpr (WHICH == 0) {
        const int i = query_of(a, row);
        p = (T*)a.dq + b * a.dqs[0] + i * a.dqs[1] + (kvh * a.group + row - i * a.group) * a.dqs[2];
        v = Lengths(a, b).seen(a, i) ? v * a.scale : f32x4{0, 0, 0, 0};
    } else if constexpr (WHICH == 1) {
        p = (T*)a.dk + b * a.dks[0] + row * a.dks[1] + kvh * a.dks[2];
        v = row < Lengths(a, b).k ? v * a.scale : f32x4{0, 0, 0, 0};
    } else {
        p = (T*)a.dv + b * a.dvs[0] + row * a.dvs[1] + kvh * a.dvs[2];
        v = row < Lengths(a, b).k ? v : f32x4{0, 0, 0, 0};
    }
    store4(p, d0, a.d, a.vec, v[0], v[1], v[2], v[3]);
}

// Splits of the keys (dq) and of the rows (dk, dv): see forward_splits.
struct Splits { int dq, dkv; };
Splits backward_splits(const ftp_attention_shape& s)
{
    const long long rows = (long long)s.q_len * (s.heads / s.kv_heads), all = (long long)s.batch * s.kv_heads;
    const long long nq = ceil_div(rows, 128) * all, nk = ceil_div(s.kv_len, 128) * all;
    const auto pick = [](long long blocks, long long tiles) {
        return blocks >= 256 ? 1 : (int)std::max(1ll, std::min({512 / std::max(blocks, 1ll), tiles / 4, 64ll}));
    };
    return {pick(nq, ceil_div(s.kv_len, s.dtype == FTP_BF16 ? 64 : 32)), pick(nk, ceil_div(rows, kRows))};
}

int padded(const ftp_attention_shape& s) { return s.head_dim <= 32 ? 32 : s.head_dim <= 64 ? 64 : 128; }

template <typename T, int D>
void run(AttentionArgs a, const Splits& n, hipStream_t st)
{
    const long long rows = (long long)a.q_len * a.group, all = (long long)a.batch * a.kv;
    if (rows) {
        a.blocks = (int)ceil_div(rows, 128);
        a.splits = n.dq;
        const unsigned grid = place_groups(a);
        k_attention_dq<T, D><<<grid, 256, 0, st>>>(a);
        if (n.dq > 1) k_attention_add<T, D, 0><<<(unsigned)ceil_div(all * rows, 1024 / D), 256, 0, st>>>(a, a.ws, all * rows * D, n.dq);
    }
    if (a.kv_len) {
        a.blocks = (int)ceil_div(a.kv_len, 128);
        a.splits = n.dkv;
        const unsigned grid = place_groups(a);
        k_attention_dkv<T, D><<<grid, 256, 0, st>>>(a);
        if (n.dkv > 1) {
            const long long each = all * a.kv_len * D;
            const unsigned adds = (unsigned)ceil_div(all * a.kv_len, 1024 / D);
            k_attention_add<T, D, 1><<<adds, 256, 0, st>>>(a, a.ws, 2 * each, n.dkv);
            k_attention_add<T, D, 2><<<adds, 256, 0, st>>>(a, a.ws + each, 2 * each, n.dkv);
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
    const Splits n = backward_splits(s);
    if (s.dtype == FTP_BF16) {
        if (a.d <= 32) run<bf16_t, 32>(a, n, st);
        else if (a.d <= 64) run<bf16_t, 64>(a, n, st);
        else run<bf16_t, 128>(a, n, st);
    } else {
        if (a.d <= 32) run<float, 32>(a, n, st);
        else if (a.d <= 64) run<float, 64>(a, n, st);
        else run<float, 128>(a, n, st);
    }
}

}  // namespace ftp
