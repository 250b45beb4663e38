// Rows of a table looked up by id, and the table's gradient.
//
// Forward: a copy, bound by memory.  Backward: the rows of dy with one id are added up in the order of their rows, whatever the launch: (id, row) pairs are sorted by id (radix sort of up to 8 bits a pass,
// stable), the sorted list is cut into pieces of 32 rows (8 of short lists), and a group of lanes adds up each run of equal ids inside its piece.  Runs that end inside the piece they began in go to the table; parts of longer ones go to scratch,
// where a second kernel joins them in their order.  No atomics on sums; a frequent id is as many pieces as it has rows for.  The table is cleared beside the first pass of the sort, which leaves the memory idle.
//
// Measured: lookup of 46208 rows of 512 fp32 20.4 us (5.5 TB/s with the table in the caches); gradient of 92416 rows of 512 bfloats on 16384 ids 76 us: sort 33, runs 31, joins 7; 4995 rows of 250 fp32 24.
#include "ftp_training.h"

#include <algorithm>

namespace ftp {
namespace {

// Rows of a piece: a group of lanes takes them one after the other, 8 on their way at once; short lists are more of a chain than of work
// (the pass on 16384 ids of 512 bfloats with pieces of 8, of 32: 4995 rows 28, 39 us; 32768 45, 49; 92416 65, 61).
inline int piece_of(long long rows) { return rows <= 32768 ? 8 : 32; }
constexpr int kBins = 256;

struct Pair { int key, row; };

// ---- forward -------------------------------------------------------------------------------------------------------
// 2^lanes lanes a row, each its vectors of E elements one after the other; rows that allow it by whole vectors.
template <typename T>
__global__ __launch_bounds__(256) void k_embed(const void* ids, int wide, const T* table, long long tstride, T* out, long long ostride, long long rows, int vocab, int C, float scale, int lanes)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int per = 1 << lanes, sub = threadIdx.x >> lanes, lane = threadIdx.x & (per - 1), step = 256 >> lanes;
    for (long long r = (long long)blockIdx.x * step + sub; r < rows; r += (long long)gridDim.x * step) {
        const int id = id_of(ids, wide, r, vocab);
        const T* from = table + (long long)std::max(id, 0) * tstride;
        T* to = out + r * ostride;
        for (int c = lane * E; c < C; c += per * E) {
            if (c + E <= C) {
                Pack<T, E> v;
                float f[E];
                if (id >= 0) v.load_any(from + c);
                else v.zero();
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = id >= 0 ? v.get(e) * scale : 0.0f;
                v.put(f);
                v.store_any(to + c);
            } else
                for (int e = c; e < C; ++e) st(to + e, id >= 0 ? ld(from + e) * scale : 0.0f);
        }
    }
}

// ---- sort ----------------------------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSmall = 8192;                        // most keys that one workgroup sorts in its LDS

struct SortArgs {
    const void* ids; const Pair* in; Pair* out; int* hist;
    float* clear; long long cleared;                // elements of the table that the first pass' launch sets to 0
    int wide, vocab, rows, shift, bits, per, blocks;            // per: keys of a workgroup
    int passes, digit;                              // bits of a pass
};

// A key: the id, or `vocab`, behind all others, where there is none.
__device__ __forceinline__ Pair pair_of(const SortArgs& a, int i)
{
    if (a.in) return a.in[i];
    const int id = id_of(a.ids, a.wide, i, a.vocab);
    return Pair{id < 0 ? a.vocab : id, i};
}

// What the workgroups behind the sorting ones do: clear the table.
__device__ __forceinline__ void clear_table(const SortArgs& a, int index, int groups)
{
    const long long step = (long long)groups * kSortThreads * 4;
    for (long long i = ((long long)index * kSortThreads + threadIdx.x) * 4; i < a.cleared; i += step) {
        const float4 zero = {0, 0, 0, 0};
        if (i + 4 <= a.cleared) __builtin_memcpy(a.clear + i, &zero, 16);
        else for (long long e = i; e < a.cleared; ++e) a.clear[e] = 0;
    }
}

// How many keys of each workgroup's share have each digit.  (Counted with global atomics by the pass before instead, frequent ids made that pass 11 -> 70 us.)
__global__ __launch_bounds__(kSortThreads) void k_digits(const SortArgs a)
{
    __shared__ int n[kBins];
    if ((int)blockIdx.x >= a.blocks) {
        clear_table(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    if (threadIdx.x < kBins) n[threadIdx.x] = 0;
    __syncthreads();
    const int lo = blockIdx.x * a.per, hi = min(lo + a.per, a.rows), mask = (1 << a.bits) - 1;
    for (int i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&n[(pair_of(a, i).key >> a.shift) & mask], 1);
    __syncthreads();
    if (threadIdx.x < kBins) a.hist[blockIdx.x * kBins + threadIdx.x] = n[threadIdx.x];
}

// First places of each wavefront's keys of each digit: n holds their numbers; all: the digit's number in the whole list, before: in earlier workgroups (threads 0 .. 255, of a digit each).
__device__ __forceinline__ void first_places(int (&n)[kSortWaves][kBins], int (&wsum)[kBins / 64], int all, int before)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int scan = all;                                 // inclusive, over the digits
    if (tid < kBins) {
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) { const int v = __shfl_up(scan, k); scan += lane >= k ? v : 0; }
        if (lane == 63) wsum[wave] = scan;
    }
    __syncthreads();
    if (tid < kBins) {
        for (int w = 0; w < wave; ++w) scan += wsum[w];
        int base = scan - all + before;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) { const int v = n[w][tid]; n[w][tid] = base; base += v; }
    }
    __syncthreads();
}

constexpr int kHeld = 4;                            // keys that a lane keeps from the count

// A wavefront's keys [lo, hi) to their places, 64 after the other, each behind the lanes of its digit before it.
template <class Get, class Put>
__device__ __forceinline__ void place_keys(int* first, int lo, int hi, int shift, int bits, const Pair (&held)[kHeld], Get get, Put put)
{
    const int lane = threadIdx.x & 63, mask = (1 << bits) - 1;
    volatile int* at = first;
    const auto round = [&](int i0, Pair p) __attribute__((always_inline)) {
        const bool there = i0 + lane < hi;
        if (!there) p = Pair{0, 0};
        const int digit = (p.key >> shift) & mask;
        unsigned long long same = __ballot(there);
        for (int k = 0; k < bits; ++k) {
            const unsigned long long one = __ballot((digit >> k) & 1);
            same &= (digit >> k) & 1 ? one : ~one;
        }
        if (there) {
            const int to = at[digit] + (int)__popcll(same & ((1ull << lane) - 1));
            __builtin_amdgcn_wave_barrier();
            if ((same >> lane) == 1) at[digit] = to + 1;            // the last of its kind
            put(to, p);
        }
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) if (lo + 64 * k < hi) round(lo + 64 * k, held[k]);
    for (int i0 = lo + 64 * kHeld; i0 < hi; i0 += 64) round(i0, i0 + lane < hi ? get(i0 + lane) : Pair{0, 0});
}

// One pass over a list of many workgroups: each key to its place, behind all keys of smaller digits, those of its digit in earlier workgroups, wavefronts and lanes.
__global__ __launch_bounds__(kSortThreads) void k_place(const SortArgs a)
{
    __shared__ int n[kSortWaves][kBins];
    __shared__ int wsum[kBins / 64];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, mask = (1 << a.bits) - 1;
    int before = 0, all = 0;
    if (tid < kBins) {
#pragma unroll 8
        for (int b = 0; b < a.blocks; ++b) {
            const int v = a.hist[b * kBins + tid];
            all += v;
            before += b < (int)blockIdx.x ? v : 0;
        }
    }
    for (int i = tid; i < kSortWaves * kBins; i += kSortThreads) (&n[0][0])[i] = 0;
    __syncthreads();
    const int part = a.per / kSortWaves, lo = blockIdx.x * a.per + wave * part, hi = min(lo + part, a.rows);
    Pair held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        const int i = lo + 64 * k + lane;
        held[k] = i < hi ? pair_of(a, i) : Pair{0, 0};
        if (i < hi) atomicAdd(&n[wave][(held[k].key >> a.shift) & mask], 1);
    }
    for (int i = lo + 64 * kHeld + lane; i < hi; i += 64) atomicAdd(&n[wave][(pair_of(a, i).key >> a.shift) & mask], 1);
    __syncthreads();
    first_places(n, wsum, all, before);
    place_keys(n[wave], lo, hi, a.shift, a.bits, held, [&](int i) { return pair_of(a, i); }, [&](int to, Pair p) { a.out[to] = p; });
}

// All passes over a short list, in one workgroup's LDS (4995 keys of 10 bits: 41 us a backward pass with two launches a pass, 24 so).
__global__ __launch_bounds__(kSortThreads) void k_sort(const SortArgs a)
{
    __shared__ Pair list[2][kSmall];
    __shared__ int n[kSortWaves][kBins];
    __shared__ int wsum[kBins / 64];
    if (blockIdx.x) {
        clear_table(a, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int part = (a.rows + kSortThreads - 1) / kSortThreads * 64, lo = min(wave * part, a.rows), hi = min(lo + part, a.rows);
    for (int i = lo + lane; i < hi; i += 64) list[0][i] = pair_of(a, i);
    int now = 0;
    for (int pass = 0; pass < a.passes; ++pass, now ^= 1) {
        const int shift = pass * a.digit, mask = (1 << a.digit) - 1;
        __syncthreads();
        for (int i = tid; i < kSortWaves * kBins; i += kSortThreads) (&n[0][0])[i] = 0;
        __syncthreads();
        Pair held[kHeld];
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int i = lo + 64 * k + lane;
            held[k] = i < hi ? list[now][i] : Pair{0, 0};
            if (i < hi) atomicAdd(&n[wave][(held[k].key >> shift) & mask], 1);
        }
        for (int i = lo + 64 * kHeld + lane; i < hi; i += 64) atomicAdd(&n[wave][(list[now][i].key >> shift) & mask], 1);
        __syncthreads();
        int all = 0;
        if (tid < kBins)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) all += n[w][tid];
        first_places(n, wsum, all, 0);
        place_keys(n[wave], lo, hi, shift, a.digit, held, [&](int i) { return list[now][i]; }, [&](int to, Pair p) { list[now ^ 1][to] = p; });
    }
    __syncthreads();
    for (int i = tid; i < a.rows; i += kSortThreads) a.out[i] = list[now][i];
}

// ---- sums ----------------------------------------------------------------------------------------------------------
struct SumArgs {
    const Pair* sorted; const void* dy; float* out; float* part;    // part: [piece][2][Cp]: of a run that began before the piece, and of one that goes on behind it
    long long stride;
    int rows, vocab, C, Cp, lanes, pieces, each;    // each: rows of a piece
    float scale;
};

template <int E>
__device__ __forceinline__ void add_out(float* to, int c, int C, const float (&v)[E], float scale)
{
    if (c + E <= C) {
        float w[E];
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = v[e] * scale;
        __builtin_memcpy(to + c, w, sizeof(w));
    } else
#pragma unroll
        for (int e = 0; e < E; ++e) if (c + e < C) to[c + e] = v[e] * scale;
}

// 2^lanes lanes a piece and E * 2^lanes channels (blockIdx.y: which).
template <typename T>
__global__ __launch_bounds__(256) void k_runs(const SumArgs a)
{
    constexpr int E = 16 / (int)sizeof(T), AHEAD = 8;
    const int piece = blockIdx.x * (256 >> a.lanes) + (threadIdx.x >> a.lanes), c = ((int)blockIdx.y * (1 << a.lanes) + (threadIdx.x & ((1 << a.lanes) - 1))) * E;
    if (piece >= a.pieces || c >= a.C) return;
    const int lo = piece * a.each, hi = min(lo + a.each, a.rows);
    int key = a.sorted[lo].key;
    bool began = lo == 0 || a.sorted[lo - 1].key != key;            // in this piece
    float sum[E] = {};
    for (int i0 = lo; i0 < hi && key < a.vocab; i0 += AHEAD) {
        Pair p[AHEAD + 1];
        Pack<T, E> v[AHEAD];
#pragma unroll
        for (int k = 0; k <= AHEAD; ++k) p[k] = i0 + k < a.rows ? a.sorted[i0 + k] : Pair{a.vocab, 0};
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            v[k].zero();
            if (i0 + k >= hi || p[k].key >= a.vocab) continue;
            const T* from = (const T*)a.dy + p[k].row * a.stride;
            if (c + E <= a.C) v[k].load_any(from + c);
            else {
                T e[E];
#pragma unroll
                for (int j = 0; j < E; ++j) e[j] = c + j < a.C ? from[c + j] : (T)0;
                __builtin_memcpy(v[k].w, e, sizeof(e));
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k >= hi || p[k].key >= a.vocab) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += v[k].get(e);
            const bool ends = p[k + 1].key != p[k].key;
            if (ends || i0 + k + 1 == hi) {
                if (ends && began) add_out<E>(a.out + (long long)p[k].key * a.C, c, a.C, sum, a.scale);
                else add_out<E>(a.part + (2ll * piece + began) * a.Cp, c, a.Cp, sum, 1.0f);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = 0;
                began = true;
            }
        }
        key = p[AHEAD].key;
    }
}

// The runs that go over pieces: the piece where one begins adds up its parts, in 8 groups that take them in turn.  A workgroup looks at 8 pieces and 256 channels; a run of up to 8 parts is a wavefront's, a longer one all eight's.
// (All channels by one workgroup, one after the other: 8192 rows of 4096 fp32 with one id 230 us the pass, 104 so; 32768 rows of 2048 bfloats on 300 skewed ids 137, 83.)
__global__ __launch_bounds__(512) void k_join(const SumArgs a)
{
    __shared__ float4 part[8][64];
    __shared__ int ends[8];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, piece = blockIdx.x * 8 + wave;
    const long long lo = (long long)piece * a.each, last = lo + a.each - 1;
    int key = -1, end = 0;                          // the last piece of the run that begins in this one
    if (last + 1 < a.rows) {
        const int k = a.sorted[last].key, after = a.sorted[last + 1].key, before = lo ? a.sorted[lo - 1].key : -1;
        if (k < a.vocab && after == k && before != k) {             // (sorted: the run began before if that one's key is the same)
            key = k;
            end = piece + 1;
            for (;;) {                              // it goes on behind a piece if the next one's first key is the same: 64 of them at once
                const long long first = (end + 1ll + lane) * a.each;
                const unsigned long long same = __ballot(first < a.rows && a.sorted[first].key == k);
                if (same == ~0ull) { end += 64; continue; }
                end += __builtin_ctzll(~same);
                break;
            }
        }
    }
    const bool mine = key >= 0 && end - piece < 8;
    if (lane == 0) ends[wave] = key >= 0 && !mine ? end : -1;
    const auto parts = [&](int p, int q, int c) { return *(const float4*)(a.part + (2ll * q + (q == p)) * a.Cp + c); };
    const auto add = [](float4& s, const float4& v) { s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; };
    const auto out = [&](int k, int c, const float4& s) {
        const float w[4] = {s.x, s.y, s.z, s.w};
        add_out<4>(a.out + (long long)k * a.C, c, a.C, w, a.scale);
    };
    const int c = (int)blockIdx.y * 256 + lane * 4;
    if (mine && c < a.C) {
        float4 v[8];
#pragma unroll
        for (int g = 0; g < 8; ++g) v[g] = piece + g <= end ? parts(piece, piece + g, c) : float4{0, 0, 0, 0};
#pragma unroll
        for (int g = 1; g < 8; ++g) add(v[0], v[g]);
        out(key, c, v[0]);
    }
    __syncthreads();
    for (int w = 0; w < 8; ++w) {
        if (ends[w] < 0) continue;
        const int p = blockIdx.x * 8 + w, e = ends[w], k = a.sorted[(p + 1ll) * a.each - 1].key;
        float4 s = {0, 0, 0, 0};
        if (c < a.Cp)
#pragma unroll 8
            for (int q = p + wave; q <= e; q += 8) add(s, parts(p, q, c));
        part[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < a.C) {
#pragma unroll
            for (int g = 1; g < 8; ++g) add(s, part[g][lane]);
            out(k, c, s);
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void k_clear(float* p, long long n)
{
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) p[i] = 0;
}

struct Buffers { int* hist; Pair *a, *b; float* part; int per, blocks, pieces, Cp; size_t bytes; };
Buffers buffers_of(const ftp_embedding_shape& s, void* ws)
{
    Buffers b = {};
    Parts t(ws);
    b.per = 4096;
    while (ceil_div(s.rows, b.per) > 128) b.per *= 2;
    b.blocks = (int)ceil_div(s.rows, b.per);
    b.pieces = (int)ceil_div(s.rows, piece_of(s.rows));
    b.Cp = (s.channels + 7) & ~7;
    b.hist = t.take<int>((size_t)b.blocks * kBins);
    b.a = t.take<Pair>(s.rows);
    b.b = t.take<Pair>(s.rows);
    b.part = t.take<float>((size_t)b.pieces * 2 * b.Cp);
    b.bytes = t.used;
    return b;
}

// Lanes of a group: the power of two whose vectors cover a row, at most `most`.
int lanes_of(int channels, int vec, int most)
{
    int n = 0;
    while ((1 << n) < most && (vec << n) < channels) ++n;
    return n;
}

}  // namespace

void embedding_forward(const ftp_embedding_shape& s, const void* ids, const void* table, void* out, hipStream_t st)
{
    const int lanes = lanes_of(s.channels, s.dtype == FTP_BF16 ? 8 : 4, 256);
    const unsigned grid = (unsigned)std::min<long long>(ceil_div(s.rows, 256 >> lanes), 16384);
    if (s.dtype == FTP_BF16)
        k_embed<bf16_t><<<grid, 256, 0, st>>>(ids, s.id_type, (const bf16_t*)table, s.table_stride, (bf16_t*)out, s.row_stride, s.rows, s.vocab, s.channels, s.scale, lanes);
    else
        k_embed<float><<<grid, 256, 0, st>>>(ids, s.id_type, (const float*)table, s.table_stride, (float*)out, s.row_stride, s.rows, s.vocab, s.channels, s.scale, lanes);
}

// k_runs has a thread for each vector of 4 numbers (or 8) of a piece of 32 rows: fewer than 2^32 (short lists' pieces of 8 rows stay below that)
bool embedding_backward_fits(const ftp_embedding_shape& s) { return s.rows * s.channels <= 1ll << 38; }
size_t embedding_workspace(const ftp_embedding_shape& s) { return buffers_of(s, nullptr).bytes; }

void embedding_backward(const ftp_embedding_shape& s, const void* ids, const void* dy, float* dtable, void* ws, hipStream_t st)
{
    const long long table = (long long)s.vocab * s.channels;
    const unsigned clearing = (unsigned)std::min<long long>(ceil_div(table, 16384), 1024);
    if (s.rows == 0) {
        k_clear<<<clearing, 256, 0, st>>>(dtable, table);
        return;
    }
    const Buffers b = buffers_of(s, ws);
    SortArgs a = {};
    a.ids = ids; a.hist = b.hist; a.clear = dtable; a.cleared = table; a.wide = s.id_type; a.vocab = s.vocab; a.rows = (int)s.rows; a.per = b.per; a.blocks = b.blocks;
    int bits = 1;
    while ((s.vocab >> bits) > 0) ++bits;           // (keys are up to vocab itself)
    const int passes = (bits + 7) / 8, digit = (bits + passes - 1) / passes;
    a.passes = passes;
    a.digit = digit;
    if (s.rows <= kSmall) {
        a.out = b.a;
        k_sort<<<1 + clearing, kSortThreads, 0, st>>>(a);
        a.in = b.a;
    } else {
        Pair *to = b.a, *other = b.b;
        for (int p = 0; p < passes; ++p) {
            a.shift = p * digit;
            a.bits = std::min(digit, bits - a.shift);
            a.out = to;
            k_digits<<<b.blocks + (p ? 0 : clearing), kSortThreads, 0, st>>>(a);
            k_place<<<b.blocks, kSortThreads, 0, st>>>(a);
            a.in = to;
            std::swap(to, other);
        }
    }
    SumArgs k = {};
    k.sorted = a.in; k.dy = dy; k.out = dtable; k.part = b.part; k.stride = s.row_stride; k.rows = a.rows; k.vocab = s.vocab; k.C = s.channels; k.Cp = b.Cp; k.pieces = b.pieces; k.each = piece_of(s.rows); k.scale = s.scale;
    const int vec = s.dtype == FTP_BF16 ? 8 : 4;
    k.lanes = lanes_of(s.channels, vec, 64);
    const dim3 grid((unsigned)ceil_div(b.pieces, 256 >> k.lanes), (unsigned)ceil_div(s.channels, vec << k.lanes));
    if (s.dtype == FTP_BF16) k_runs<bf16_t><<<grid, 256, 0, st>>>(k);
    else k_runs<float><<<grid, 256, 0, st>>>(k);
    if (b.pieces > 1) k_join<<<dim3((unsigned)ceil_div(b.pieces, 8), (unsigned)ceil_div(s.channels, 256)), 512, 0, st>>>(k);
}

}  // namespace ftp
