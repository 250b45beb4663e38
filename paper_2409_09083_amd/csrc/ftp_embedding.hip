// Rows of a table looked up by id, and the table's gradient.
//
// Forward: a copy, bound by memory.  Backward: the rows of dy with one id are added up in the order of their rows, whatever the launch: (id, row) pairs are sorted by id (radix sort of up to 8 bits a pass,
// stable), the sorted list is cut into pieces of 32 rows, and a group of lanes adds up each run of equal ids inside its piece.  Runs that end inside the piece they began in go to the table; parts of longer ones go to scratch,
// where a second kernel joins them in their order.  No atomics on sums; a frequent id is as many pieces as it has rows for.  The table is cleared beside the first pass of the sort, which leaves the memory idle.
#include "ftp_training.h"

#include <algorithm>

namespace ftp {
namespace {

constexpr int kPiece = 32;                          // rows of a piece
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
struct SortArgs {
    const void* ids; const Pair* in; Pair* out; int* hist;
    float* clear; long long cleared;                // elements of the table that the first pass' launch sets to 0
    int wide, vocab, rows, shift, bits, per, blocks;            // per: keys of a workgroup, a multiple of 256
};

// A key: the id, or `vocab`, behind all others, where there is none.
__device__ __forceinline__ Pair pair_of(const SortArgs& a, int i)
{
    if (a.in) return a.in[i];
    const int id = id_of(a.ids, a.wide, i, a.vocab);
    return Pair{id < 0 ? a.vocab : id, i};
}

// How many keys of each workgroup's share have each digit.
__global__ __launch_bounds__(256) void k_digits(const SortArgs a)
{
    __shared__ int n[kBins];
    if ((int)blockIdx.x >= a.blocks) {              // (the other workgroups clear the table)
        const long long step = (long long)(gridDim.x - a.blocks) * 1024;
        for (long long i = ((long long)(blockIdx.x - a.blocks) * 256 + threadIdx.x) * 4; i < a.cleared; i += step) {
            const float4 zero = {0, 0, 0, 0};
            if (i + 4 <= a.cleared) __builtin_memcpy(a.clear + i, &zero, 16);
            else for (long long e = i; e < a.cleared; ++e) a.clear[e] = 0;
        }
        return;
    }
    n[threadIdx.x] = 0;
    __syncthreads();
    const int lo = blockIdx.x * a.per, hi = min(lo + a.per, a.rows), mask = (1 << a.bits) - 1;
    for (int i = lo + threadIdx.x; i < hi; i += 256) atomicAdd(&n[(pair_of(a, i).key >> a.shift) & mask], 1);
    __syncthreads();
    a.hist[blockIdx.x * kBins + threadIdx.x] = n[threadIdx.x];
}

// Each key to its place: behind all keys of smaller digits, those of its digit in earlier workgroups, wavefronts and lanes.
__global__ __launch_bounds__(256) void k_place(const SortArgs a)
{
    __shared__ int n[4][kBins];
    __shared__ int wsum[4];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, mask = (1 << a.bits) - 1;
    int before = 0, all = 0;
#pragma unroll 8
    for (int b = 0; b < a.blocks; ++b) {
        const int v = a.hist[b * kBins + tid];
        all += v;
        before += b < (int)blockIdx.x ? v : 0;
    }
    int scan = all;                                 // inclusive, over the digits
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) { const int v = __shfl_up(scan, k); scan += lane >= k ? v : 0; }
    if (lane == 63) wsum[wave] = scan;
#pragma unroll
    for (int w = 0; w < 4; ++w) n[w][tid] = 0;
    __syncthreads();
    for (int w = 0; w < wave; ++w) scan += wsum[w];
    int base = scan - all + before;
    // a wavefront's keys are neighbours
    const int part = a.per / 4, lo = blockIdx.x * a.per + wave * part, hi = min(lo + part, a.rows);
    for (int i = lo + lane; i < hi; i += 64) atomicAdd(&n[wave][(pair_of(a, i).key >> a.shift) & mask], 1);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) { const int v = n[w][tid]; n[w][tid] = base; base += v; }
    __syncthreads();
    volatile int* at = n[wave];
    for (int i0 = lo; i0 < hi; i0 += 64) {
        const bool there = i0 + lane < hi;
        Pair p = {0, 0};
        if (there) p = pair_of(a, i0 + lane);
        const int digit = (p.key >> a.shift) & mask;
        unsigned long long same = __ballot(there);
        for (int k = 0; k < a.bits; ++k) {
            const unsigned long long one = __ballot((digit >> k) & 1);
            same &= (digit >> k) & 1 ? one : ~one;
        }
        if (there) {
            const int to = at[digit] + (int)__popcll(same & ((1ull << lane) - 1));
            __builtin_amdgcn_wave_barrier();
            if ((same >> lane) == 1) at[digit] = to + 1;            // the last of its kind
            a.out[to] = p;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- sums ----------------------------------------------------------------------------------------------------------
struct SumArgs {
    const Pair* sorted; const void* dy; float* out; float* part;    // part: [piece][2][Cp]: of a run that began before the piece, and of one that goes on behind it
    long long stride;
    int rows, vocab, C, Cp, lanes, pieces;
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
    const int lo = piece * kPiece, hi = min(lo + kPiece, a.rows);
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

// The runs that go over pieces: the piece where one begins adds up its parts, 8 groups of lanes with parts in turn, joined in LDS.
__global__ __launch_bounds__(512) void k_join(const SumArgs a)
{
    __shared__ float4 part[8][64];
    const int piece = blockIdx.x, lo = piece * kPiece, last = lo + kPiece - 1;
    if (last + 1 >= a.rows) return;
    const int key = a.sorted[last].key;
    if (key >= a.vocab || a.sorted[last + 1].key != key || (lo && a.sorted[lo - 1].key == key)) return;       // (sorted: the run began before if that one's key is the same)
    int from = last + 1, to = a.rows;               // the first that has another key lies in (from, to]
    while (from < to) {
        const int mid = from + (to - from) / 2;
        if (a.sorted[mid].key == key) from = mid + 1;
        else to = mid;
    }
    const int end = (from - 1) / kPiece, grp = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int c0 = 0; c0 < a.Cp; c0 += 256) {
        const int c = c0 + lane * 4;
        float4 s = {0, 0, 0, 0};
        if (c < a.Cp) {
#pragma unroll 4
            for (int q = piece + grp; q <= end; q += 8) {
                const float4 v = *(const float4*)(a.part + (2ll * q + (q == piece)) * a.Cp + c);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
        }
        part[grp][lane] = s;
        __syncthreads();
        if (grp == 0 && c < a.C) {
#pragma unroll
            for (int g = 1; g < 8; ++g) { const float4 v = part[g][lane]; s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; }
            const float w[4] = {s.x, s.y, s.z, s.w};
            add_out<4>(a.out + (long long)key * a.C, c, a.C, w, a.scale);
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
    b.per = 1024;
    while (ceil_div(s.rows, b.per) > 256) b.per *= 2;
    b.blocks = (int)ceil_div(s.rows, b.per);
    b.pieces = (int)ceil_div(s.rows, kPiece);
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

size_t embedding_workspace(const ftp_embedding_shape& s) { return buffers_of(s, nullptr).bytes; }

void embedding_backward(const ftp_embedding_shape& s, const void* ids, const void* dy, float* dtable, void* ws, hipStream_t st)
{
    const long long table = (long long)s.vocab * s.channels;
    const unsigned clearing = (unsigned)std::min<long long>(ceil_div(table, 4096), 4096);
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
    Pair *to = b.a, *other = b.b;
    for (int p = 0; p < passes; ++p) {
        a.shift = p * digit;
        a.bits = std::min(digit, bits - a.shift);
        a.out = to;
        k_digits<<<b.blocks + (p ? 0 : clearing), 256, 0, st>>>(a);
        k_place<<<b.blocks, 256, 0, st>>>(a);
        a.in = to;
        std::swap(to, other);
    }
    SumArgs k = {};
    k.sorted = a.in; k.dy = dy; k.out = dtable; k.part = b.part; k.stride = s.row_stride; k.rows = a.rows; k.vocab = s.vocab; k.C = s.channels; k.Cp = b.Cp; k.pieces = b.pieces; k.scale = s.scale;
    const int vec = s.dtype == FTP_BF16 ? 8 : 4;
    k.lanes = lanes_of(s.channels, vec, 64);
    const dim3 grid((unsigned)ceil_div(b.pieces, 256 >> k.lanes), (unsigned)ceil_div(s.channels, vec << k.lanes));
    if (s.dtype == FTP_BF16) k_runs<bf16_t><<<grid, 256, 0, st>>>(k);
    else k_runs<float><<<grid, 256, 0, st>>>(k);
    if (b.pieces > 1) k_join<<<b.pieces, 512, 0, st>>>(k);
}

}  // namespace ftp
