// Embedding rows of tokens (gwtf_stage_embed) and the table's gradient
// (gwtf_stage_embed_grad).
//
//   out[i] = scale * table[t_i];   grad[v] = scale * sum of dout[i] over t_i = v
//
// Gradient: the tokens are sorted with their positions, so that the rows of
// one token are adjacent and in order; the sorted list is cut into chunks of
// equal length whatever the tokens are, one wave per chunk and slab of 512
// columns.  A wave adds the rows of each run of one token in registers and
// writes a run that lies within its chunk to the table; the parts of a run
// that crosses chunks are added in order by a launch of their own.  No
// floating-point atomics: the same inputs give the same bits.
//
// Bound by memory where tokens or table are many: 16,384 rows of 4096 bf16 into
// 32,000 (396 MB) take 88 us, of which the sums read 134 MB and write 50 in 37
// and the other launches write the rest at about 4.5 TB/s; 2,048 x 1024 into
// 131 MB 27 us.  A short call is bound by its three launches and their reads:
// sort 6.6 us, sums 5, join 5.
#include "stage_device.h"
#include "stage_internal.h"

namespace gwtf {
namespace {

// ---- rows of the table ----

struct EmbedParams {
    gwtf_stage_embed_t a;
    int64_t row0;
    uint32_t units;
    FastDiv steps;
};

// Bound by memory: 16,384 rows of 4096 bf16 29 us (48 with the results kept in
// the caches, where the table's rows now stay); eight rows of 1024 2 us, a launch.
// STREAM: rows written past the caches.
template <class T, bool STREAM>
__global__ __launch_bounds__(256) void embed_kernel(EmbedParams p)
{
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    if (u >= p.units) return;
    const uint32_t r = p.steps.div(u);
    const int64_t row = p.row0 + r, col = int64_t(u - r * p.steps.d) * kVec, n = p.a.hidden - col;
    const int64_t t = load_token(p.a.tokens, p.a.token_type, row);
    float v[8];
    if (t >= 0 && t < p.a.vocab) {
        load8(static_cast<const T *>(p.a.table) + t * p.a.table_stride + col, n, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] *= p.a.scale;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = 0.f;
    }
    store8<T, STREAM>(static_cast<T *>(p.a.out) + row * p.a.out_stride + col, n, v);
}

// ---- zeros for the rows of absent tokens ----
//
// Most of the gradient's bytes are zeros that depend on nothing but which
// tokens are there, so they are written beside the launches that wait for
// their reads rather than for the memory: the sort, the merge, the join, and
// the sums where they are short.  Workgroup g of the fill has the rows g, g +
// groups, .. of the table, a share of them in each launch; in the first one it
// looks through all tokens for its own and keeps what it found as a bit a row.
// (2,048 x 1024 28 us, 16,384 x 4096 86; all zeros beside sort and merge 31 and
// 89, no launch beside another 56 and 157.)

constexpr int kFillRows = 65536;             // most rows of one workgroup
constexpr int64_t kFillTokens = 32768;       // with more tokens a look through them costs more than the sort hides:
                                             // then embed_grad_kernel writes the zeros
constexpr int64_t kShortSums = int64_t(16) << 20; // bytes of dout whose sums wait for reads

struct FillParams {
    void *grad;
    int64_t stride, hidden;
    const void *tokens;
    int64_t N, vocab;
    int32_t token_type, wide; // wide: 32-bit gradient
    FastDiv groups;
    uint32_t *absent; // [groups][words], or NULL: all rows belong to the first launch
    int32_t words;
    int32_t r0, r1;   // this launch's share of a workgroup's rows
    int32_t stream;   // zeros past the caches
};

// In accesses on 16-byte boundaries, and halfwords before the first and after
// the last.
template <bool STREAM>
__device__ __forceinline__ void zero_row(char *g, int64_t bytes)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 z = {0, 0, 0, 0};
    const int lane = threadIdx.x & 63;
    int64_t head = -reinterpret_cast<uintptr_t>(g) & 15;
    if (head > bytes) head = bytes;
    const int64_t end = head + ((bytes - head) & ~int64_t(15));
    if (lane * 2 < head) *reinterpret_cast<uint16_t *>(g + lane * 2) = 0;
    for (int64_t at = head + lane * 16; at < end; at += 64 * 16) {
        if constexpr (STREAM) __builtin_nontemporal_store(z, reinterpret_cast<u32x4 *>(g + at));
        else *reinterpret_cast<u32x4 *>(g + at) = z;
    }
    if (end + lane * 2 < bytes) *reinterpret_cast<uint16_t *>(g + end + lane * 2) = 0;
}

__device__ __forceinline__ void fill_rows(const FillParams &p, int group, const uint32_t *absent, int threads)
{
    const uint32_t groups = p.groups.d;
    const int64_t size = p.wide ? 4 : 2;
    const int rows = int((uint32_t(p.vocab) + groups - 1 - group) / groups), r1 = p.r1 < rows ? p.r1 : rows;
    for (int r = p.r0 + (threadIdx.x >> 6); r < r1; r += threads / 64)
        if (absent[r >> 5] >> (r & 31) & 1) {
            char *row = static_cast<char *>(p.grad) + (group + int64_t(r) * groups) * p.stride * size;
            if (p.stream) zero_row<true>(row, p.hidden * size);
            else zero_row<false>(row, p.hidden * size);
        }
}

// The first launch's part, with kFillRows / 32 words of LDS.
template <int THREADS>
__device__ void fill_first(const FillParams &p, int group, uint32_t *absent)
{
    const uint32_t groups = p.groups.d;
    for (int i = threadIdx.x; i < p.words; i += THREADS) absent[i] = 0xffffffffu;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < p.N; i += 8 * THREADS) {
        int64_t t[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) t[q] = i + q * THREADS < p.N ? load_token(p.tokens, p.token_type, i + q * THREADS) : -1;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (t[q] < 0 || t[q] >= p.vocab) continue;
            const uint32_t own = p.groups.div(uint32_t(t[q]));
            if (uint32_t(t[q]) - own * groups == uint32_t(group)) atomicAnd(&absent[own >> 5], ~(1u << (own & 31)));
        }
    }
    __syncthreads();
    if (p.absent)
        for (int i = threadIdx.x; i < p.words; i += THREADS) p.absent[int64_t(group) * p.words + i] = absent[i];
    fill_rows(p, group, absent, THREADS);
}
__device__ __forceinline__ void fill_later(const FillParams &p, int group, int threads)
{
    fill_rows(p, group, p.absent + int64_t(group) * p.words, threads);
}

// ---- sorting tokens ----
//
// Keys token << 32 | position are all different, so any sort is stable.  One
// workgroup sorts kSortBlock of them (bitonic), two adjacent keys a thread:
// exchanges over up to 64 keys stay within a thread or a wave, only those over
// more, 10 of 66, go through LDS with a barrier (6.6 us a block with 32-bit
// keys, 9 with 64; 15 with all exchanges in LDS).  Up to kMergeWays sorted
// blocks are merged in one launch, where each key finds its place by a binary
// search in every other block.  Workgroups after the sorting ones write zeros.

constexpr int kSortBlock = 2048;
constexpr int kMergeWays = 32;

// The value of lane ^ x.
template <int x>
__device__ __forceinline__ int lane_xor(int v)
{
    if constexpr (x == 1) return __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xf, 0xf, false);      // quad 1 0 3 2
    else if constexpr (x == 2) return __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xf, 0xf, false); // quad 2 3 0 1
    else if constexpr (x == 8) return row_ror<8>(v);
    else return __shfl_xor(v, x);
}
template <int x>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) { return uint32_t(lane_xor<x>(int(v))); }
template <int x>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v)
{
    return (uint64_t(uint32_t(lane_xor<x>(int(v >> 32)))) << 32) | uint32_t(lane_xor<x>(int(uint32_t(v))));
}
template <class K>
__device__ __forceinline__ K lower(K a, K b) { return a < b ? a : b; }
template <class K>
__device__ __forceinline__ K higher(K a, K b) { return a < b ? b : a; }

// Exchange of keys i and i ^ (2 x) between lanes; `up`: the run is ascending.
template <int x, class K>
__device__ __forceinline__ void exchange(K &a, K &b, int lane, bool up)
{
    const K pa = lane_xor<x>(a), pb = lane_xor<x>(b);
    const bool low = ((lane & x) == 0) == up;
    a = low ? lower(pa, a) : higher(pa, a);
    b = low ? lower(pb, b) : higher(pb, b);
}

// K: 32 bits, token << 11 | index in the block, where tokens have at most 21
// bits (the sort is bound by its vector instructions, a third of those for 64
// bits), else 64.
template <class K>
__global__ __launch_bounds__(1024) void sort_block_kernel(const void *tokens, int token_type, int64_t vocab, int64_t N,
                                                          uint64_t *out, uint32_t blocks, FillParams f)
{
    __shared__ K key[2][kSortBlock];
    static_assert(kFillRows / 8 <= sizeof key, "a bit for each row of a workgroup of the fill");
    if (blockIdx.x >= blocks) {
        fill_first<1024>(f, int(blockIdx.x - blocks), reinterpret_cast<uint32_t *>(key));
        return;
    }
    constexpr int kShift = sizeof(K) == 4 ? 11 : 32;
    const int64_t base = int64_t(blockIdx.x) * kSortBlock;
    const int t = threadIdx.x, lane = t & 63;
    K k[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t pos = base + 2 * t + i;
        const int64_t tok = pos < N ? load_token(tokens, token_type, pos) : -1;
        // absent and padding come after all tokens, in order of their position
        k[i] = (K(tok >= 0 && tok < vocab ? tok : vocab) << kShift) | K(2 * t + i);
    }
    int turn = 0;
#pragma unroll
    for (int size = 2; size <= kSortBlock; size <<= 1) {
        const bool up = ((2 * t) & size) == 0;
        // over more than a wave: partner thread t ^ (j / 2); two buffers, so
        // that one barrier is enough
        for (int j = size >> 1; j >= 128; j >>= 1, turn ^= 1) {
            key[turn][2 * t] = k[0];
            key[turn][2 * t + 1] = k[1];
            __syncthreads();
            const int other = 2 * (t ^ (j >> 1));
            const K pa = key[turn][other], pb = key[turn][other + 1];
            const bool low = ((2 * t & j) == 0) == up;
            k[0] = low ? lower(pa, k[0]) : higher(pa, k[0]);
            k[1] = low ? lower(pb, k[1]) : higher(pb, k[1]);
        }
        if (size >= 128) exchange<32>(k[0], k[1], lane, up);
        if (size >= 64) exchange<16>(k[0], k[1], lane, up);
        if (size >= 32) exchange<8>(k[0], k[1], lane, up);
        if (size >= 16) exchange<4>(k[0], k[1], lane, up);
        if (size >= 8) exchange<2>(k[0], k[1], lane, up);
        if (size >= 4) exchange<1>(k[0], k[1], lane, up);
        const K lo = lower(k[0], k[1]), hi = higher(k[0], k[1]);
        k[0] = up ? lo : hi;
        k[1] = up ? hi : lo;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (base + 2 * t + i >= N) continue;
        const int64_t tok = int64_t(k[i] >> kShift);
        out[base + 2 * t + i] = (uint64_t(tok < vocab ? uint32_t(tok) : 0xffffffffu) << 32) |
                                uint32_t(base + int64_t(k[i] & K(kSortBlock - 1)));
    }
}

// Merges groups of kMergeWays sorted blocks of `len` (a power of two) keys.  A
// search is a chain of dependent reads, so every `1 << shift`-th key of the
// group is put into LDS first and only its last steps go to memory (16,384
// tokens: one cache line).  Four lanes share a key, each with up to eight
// searches side by side (eight blocks 8.7 us; one lane a key, all reads from
// memory, 16).
constexpr int kSamples = 4096;
constexpr int kMergeThreads = 1024;
constexpr int kMergeKeys = kMergeThreads / 4;
constexpr int kSearches = kMergeWays / 4;

__global__ __launch_bounds__(kMergeThreads) void merge_kernel(const uint64_t *in, uint32_t N, uint32_t len, int shift,
                                                              uint64_t *out, uint32_t block0, uint32_t blocks, FillParams f)
{
    __shared__ uint64_t sample[kSamples];
    if (blockIdx.x >= blocks) {
        fill_later(f, int(blockIdx.x - blocks), kMergeThreads);
        return;
    }
    // a workgroup's adjacent keys lie within one block, as len is a multiple of
    // their number; offsets below are within the group of blocks
    const uint32_t i0 = (block0 + blockIdx.x) * uint32_t(kMergeKeys), own = i0 / len, group0 = own / kMergeWays * kMergeWays;
    const int64_t start = int64_t(group0) * len;
    const uint64_t *const g = in + start;
    const uint32_t total = uint32_t(N - start < int64_t(len) * kMergeWays ? N - start : int64_t(len) * kMergeWays);
    for (uint32_t q = threadIdx.x; q < total >> shift; q += kMergeThreads) sample[q] = g[((q + 1) << shift) - 1];
    const uint32_t i = uint32_t(i0 + threadIdx.x / 4 - start), part = threadIdx.x & 3;
    const uint64_t k = i < total ? g[i] : 0;
    __syncthreads();
    uint32_t lo[kSearches], end[kSearches];
#pragma unroll
    for (int q = 0; q < kSearches; ++q) {
        const uint32_t b = part + 4 * q, first = b * len;
        lo[q] = first;
        end[q] = b == own - group0 || first >= total ? first : (first + len < total ? first + len : total);
    }
    uint32_t step = len;
    for (; step >= 1u << shift; step >>= 1) {
#pragma unroll
        for (int q = 0; q < kSearches; ++q)
            if (lo[q] + step <= end[q] && sample[((lo[q] + step) >> shift) - 1] < k) lo[q] += step;
    }
    for (; step > 0; step >>= 1) {
        uint64_t v[kSearches];
#pragma unroll
        for (int q = 0; q < kSearches; ++q) v[q] = lo[q] + step <= end[q] ? g[lo[q] + step - 1] : ~uint64_t(0);
#pragma unroll
        for (int q = 0; q < kSearches; ++q)
            if (v[q] < k) lo[q] += step;
    }
    int place = 0;
#pragma unroll
    for (int q = 0; q < kSearches; ++q) place += int(lo[q] - (part + 4 * q) * len);
    place += lane_xor<1>(place);
    place += lane_xor<2>(place);
    if (part == 0 && i < total) out[start + place + (i - (own - group0) * len)] = k;
}

// ---- sums ----

struct EmbedGradParams {
    gwtf_stage_embed_grad_t a;
    const uint64_t *sorted;
    float *partial;           // [chunks][2][H]: of the run that began before the chunk, of the run that goes on after it
    int64_t chunk, chunks;
    int slabs;                // of 512 columns
    int64_t fill_block;       // first workgroup that writes zeros
    bool search;              // it looks its rows up in the sorted list
    FillParams fill;
    bool stream;              // dout is read past the caches
};

constexpr int kSearchRows = 16; // rows of the table a wave looks up for zeros
constexpr int kRowsInFlight = 8;
constexpr int kPartsInFlight = 16; // a run of one token over all chunks: 512 sums, one after another

__device__ __forceinline__ uint32_t key_token(uint64_t k) { return uint32_t(k >> 32); }

template <class G>
__device__ __forceinline__ void write_grad(const gwtf_stage_embed_grad_t &a, int64_t token, int64_t col, int64_t n, float v[8])
{
    G *g = static_cast<G *>(a.grad) + token * a.grad_stride + col;
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] *= a.scale;
    if (a.accumulate) {
        float old[8];
        load8(g, n, old);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] += old[i];
    }
    store8(g, n, v);
}

// One chunk and slab.  Lane l holds the key of entry l of 64; two batches of
// rows are in flight (16,384 rows of one token, 134 MB, 24 us: 5.5 TB/s).
template <class T, class G, bool STREAM>
__device__ __forceinline__ void sum_chunk(const EmbedGradParams &p, int64_t c, int64_t slab_col, int lane)
{
    const gwtf_stage_embed_grad_t &a = p.a;
    constexpr int U = kRowsInFlight * 2 / int(sizeof(T));
    const int64_t N = a.num_tokens, col = slab_col + lane * kVec, n = a.hidden - col;
    const int64_t e0 = c * p.chunk, e1 = e0 + p.chunk < N ? e0 + p.chunk : N;
    const T *dout = static_cast<const T *>(a.dout);
    const bool ends = ends_within(col, a.hidden);
    // tokens just outside the chunk, with the keys of its first entries
    const uint64_t before_key = e0 > 0 ? p.sorted[e0 - 1] : ~uint64_t(0), after_key = e1 < N ? p.sorted[e1] : ~uint64_t(0);
    uint64_t mine = p.sorted[e0 + lane < e1 ? e0 + lane : e1 - 1];
    uint32_t token = __builtin_amdgcn_readfirstlane(key_token(mine));
    if (token == 0xffffffffu) return;
    bool before = __builtin_amdgcn_readfirstlane(key_token(before_key)) == token; // the run began in an earlier chunk
    const uint32_t after_token = __builtin_amdgcn_readfirstlane(key_token(after_key));
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    typename Vec8<T>::type v[U], vn[U];
    for (int64_t eb = e0; eb < e1; eb += 64) {
        if (eb > e0) mine = p.sorted[eb + lane < e1 ? eb + lane : e1 - 1];
        const int count = int(e1 - eb < 64 ? e1 - eb : 64);
        auto fetch = [&](int at, typename Vec8<T>::type (&row)[U]) {
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const uint32_t pos = __builtin_amdgcn_readlane(int(uint32_t(mine)), (at + q) & 63); // entries past the end read the last row
                row[q] = load_columns<T, STREAM>(dout + int64_t(pos) * a.dout_stride, col, a.hidden);
            }
        };
        fetch(0, v);
        for (int at = 0; at < count; at += U) {
            if (at + U < count) fetch(at + U, vn); // the next rows, in flight while these are added
#pragma unroll
            for (int q = 0; q < U; ++q) {
                if (at + q >= count) break;
                const uint32_t t = __builtin_amdgcn_readlane(int(key_token(mine)), at + q);
                if (t != token) {
                    if (before) store8(p.partial + (c * 2) * a.hidden + col, n, acc);
                    else write_grad<G>(a, token, col, n, acc);
                    if (t == 0xffffffffu) return;
                    before = false;
                    token = t;
#pragma unroll
                    for (int i = 0; i < kVec; ++i) acc[i] = 0.f;
                }
                float f[8];
                columns_of<T>(v[q], ends, col, a.hidden, f);
#pragma unroll
                for (int i = 0; i < kVec; ++i) acc[i] += f[i];
            }
#pragma unroll
            for (int q = 0; q < U; ++q) v[q] = vn[q];
        }
    }
    if (before) store8(p.partial + (c * 2) * a.hidden + col, n, acc);
    else if (after_token == token) store8(p.partial + (c * 2 + 1) * a.hidden + col, n, acc);
    else write_grad<G>(a, token, col, n, acc);
}

template <class T, class G>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedGradParams p)
{
    const gwtf_stage_embed_grad_t &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t N = a.num_tokens;
    if (blockIdx.x >= p.fill_block) {
        if (!p.search) {
            fill_later(p.fill, int(blockIdx.x - p.fill_block), 256);
            return;
        }
        const int64_t step = (gridDim.x - p.fill_block) * 4 * kSearchRows;
        for (int64_t v0 = ((blockIdx.x - p.fill_block) * 4 + wave) * kSearchRows; v0 < a.vocab; v0 += step) {
            bool absent = false;
            if (lane < kSearchRows && v0 + lane < a.vocab) {
                const uint64_t k = uint64_t(v0 + lane) << 32;
                int64_t lo = 0, hi = N;
                while (lo < hi) {
                    const int64_t mid = (lo + hi) >> 1;
                    if (p.sorted[mid] < k) lo = mid + 1;
                    else hi = mid;
                }
                absent = lo == N || key_token(p.sorted[lo]) != uint32_t(v0 + lane);
            }
            uint64_t rows = __ballot(absent);
            while (rows) {
                const int r = __builtin_ctzll(rows);
                rows &= rows - 1;
                zero_row<false>(static_cast<char *>(a.grad) + (v0 + r) * a.grad_stride * int64_t(sizeof(G)), a.hidden * int64_t(sizeof(G)));
            }
        }
        return;
    }
    const int64_t item = int64_t(blockIdx.x) * 4 + wave, c = item / p.slabs, slab_col = (item - c * p.slabs) * 512;
    if (c >= p.chunks) return;
    if (p.stream) sum_chunk<T, G, true>(p, c, slab_col, lane);
    else sum_chunk<T, G, false>(p, c, slab_col, lane);
}

// Runs that cross chunks, each by the wave of the chunk in which it begins;
// bound by the reads that follow one another (4.6 us without any run, 46 for one
// run over 512 chunks).
template <class G>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradParams p)
{
    const gwtf_stage_embed_grad_t &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= p.fill_block) {
        fill_later(p.fill, int(blockIdx.x - p.fill_block), 256);
        return;
    }
    const int64_t item = int64_t(blockIdx.x) * 4 + wave;
    const int64_t c = item / p.slabs, N = a.num_tokens;
    const int64_t e0 = c * p.chunk, e1 = e0 + p.chunk;
    if (c >= p.chunks || e1 >= N) return;
    const uint32_t first = key_token(p.sorted[e0]), token = key_token(p.sorted[e1 - 1]), next = key_token(p.sorted[e1]);
    const uint32_t previous = e0 > 0 ? key_token(p.sorted[e0 - 1]) : 0xffffffffu;
    if (token == 0xffffffffu || next != token) return; // no run goes on
    if (first == token && previous == token) return;   // it began earlier
    // chunks after this one that begin with the token, 64 looked at together
    int64_t more = 0;
    for (;;) {
        const int64_t d = c + 1 + more + lane;
        const uint64_t there = __ballot(d < p.chunks && key_token(p.sorted[d * p.chunk]) == token);
        const int run = there == ~uint64_t(0) ? 64 : __builtin_ctzll(~there);
        more += run;
        if (run < 64) break;
    }
    const int64_t slab_col = (item - c * p.slabs) * 512, col = slab_col + lane * kVec, n = a.hidden - col;
    float acc[8];
    load8(p.partial + (c * 2 + 1) * a.hidden + col, n, acc);
    const bool ends = ends_within(col, a.hidden);
    const float *next_part = p.partial + (c + 1) * 2 * a.hidden;
    for (int64_t d = 0; d < more; d += kPartsInFlight) {
        Vec8<float>::type v[kPartsInFlight];
#pragma unroll
        for (int q = 0; q < kPartsInFlight; ++q)
            v[q] = load_columns(next_part + (d + q < more ? d + q : more - 1) * 2 * a.hidden, col, a.hidden);
#pragma unroll
        for (int q = 0; q < kPartsInFlight; ++q) {
            float f[8];
            columns_of<float>(v[q], ends, col, a.hidden, f);
#pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] += d + q < more ? f[i] : 0.f;
        }
    }
    write_grad<G>(a, token, col, n, acc);
}

template <class T>
hipError_t run_embed(const gwtf_stage_embed_t &a, hipStream_t s)
{
    const int64_t steps = (a.hidden + kVec - 1) / kVec, slab = (int64_t(1) << 30) / steps;
    const bool stream = 2 * a.num_tokens * a.hidden * int64_t(sizeof(T)) >= kStreamBytes && on_lines(a.out, a.out_stride, sizeof(T));
    auto kernel = stream ? embed_kernel<T, true> : embed_kernel<T, false>;
    EmbedParams p;
    p.a = a;
    p.steps = FastDiv::make(uint32_t(steps));
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        p.row0 = r;
        p.units = uint32_t(n * steps);
        const hipError_t e = launch(kernel, (p.units + 255) / 256, 256, s, p);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t slabs_of(int64_t H) { return (H + 511) / 512; }

// Entries of a chunk: few enough for kEmbedItems waves, but no fewer than about
// sqrt(N / 32), since the parts of a frequent token's run are added one after
// another (words that come as 1 / rank, 16,384 x 512: chunks of 4 62 us, of 23
// 42; 2,048 x 1024: of 4 31, of 8 30).
int64_t chunk_of(int64_t N, int64_t H)
{
    const int64_t c = (N * slabs_of(H) + kEmbedItems - 1) / kEmbedItems;
    int64_t least = kEmbedMinChunk;
    while (least * least * 32 < N) ++least;
    return c > least ? c : least;
}

template <class T, class G>
hipError_t run_embed_grad(const gwtf_stage_embed_grad_t &a, const StageWorkspace &w, hipStream_t s)
{
    hipError_t e;
    const int64_t N = a.num_tokens;
    EmbedGradParams p;
    p.a = a;
    p.sorted = w.sort_a;
    // zeros past the caches where the table is larger than the L2s together
    // (2,048 x 1024 into 131 MB 27 us, 32 through them; 16,384 x 4096 into 262 MB
    // 89 and 93; 5,000 x 777 f32 into 50,000 rows 47 and 62)
    const bool large_table = a.vocab * a.hidden * int64_t(sizeof(G)) >= kL2Bytes;
    const int64_t bytes = ((a.accumulate ? 0 : a.vocab) * int64_t(sizeof(G)) + N * int64_t(sizeof(T))) * a.hidden;
    p.stream = bytes >= kStreamBytes && on_lines(a.dout, a.dout_stride, sizeof(T));
    p.partial = w.partial;
    p.chunk = chunk_of(N, a.hidden);
    p.chunks = (N + p.chunk - 1) / p.chunk;
    p.slabs = int(slabs_of(a.hidden));
    p.search = !a.accumulate && (N == 0 || N > kFillTokens);
    FillParams &f = p.fill;
    f = FillParams{a.grad, a.grad_stride, a.hidden, a.tokens, N, a.vocab, a.token_type, a.grad_type == GWTF_TYPE_F32,
                   FastDiv::make(1), nullptr, 0, 0, 0, large_table};
    const bool merged = N > kSortBlock, joined = p.chunks > 1, short_sums = N * a.hidden * int64_t(sizeof(T)) < kShortSums;
    uint32_t groups = 0; // of the fill, in every launch that has a share
    int rows = 0, shares = 1, share = 0;
    if (!a.accumulate && !p.search) {
        // with the sorting or merging workgroups, two of 1024 threads on a CU
        const int64_t busy = (N + (merged ? kMergeKeys : kSortBlock) - 1) / (merged ? kMergeKeys : kSortBlock);
        int64_t g = 2 * int64_t(w.cus) - busy;
        if (g < w.cus) g = w.cus;
        if (g > a.vocab) g = a.vocab;
        // whatever the number of CUs, a workgroup's bits fit in its LDS
        if (g < (a.vocab + kFillRows - 1) / kFillRows) g = (a.vocab + kFillRows - 1) / kFillRows;
        if (a.vocab <= kAbsentRows) {
            f.absent = w.absent;
            shares = 1 + merged + short_sums + joined;
        }
        groups = uint32_t(g);
        rows = int((a.vocab + g - 1) / g);
        f.groups = FastDiv::make(groups);
        f.words = (rows + 31) / 32;
    }
    // the next share of the fill: its workgroups
    auto take_share = [&](bool has) -> uint32_t {
        if (!has || share == shares) return 0;
        f.r0 = int(int64_t(rows) * share / shares);
        f.r1 = int(int64_t(rows) * ++share / shares);
        return groups;
    };
    if (N > 0) {
        uint32_t blocks = uint32_t((N + kSortBlock - 1) / kSortBlock);
        uint32_t fill = take_share(true);
        auto sort = a.vocab < int64_t(1) << 21 ? sort_block_kernel<uint32_t> : sort_block_kernel<uint64_t>;
        if ((e = launch(sort, blocks + fill, 1024, s, a.tokens, a.token_type, a.vocab, N, w.sort_a, blocks, f)) != hipSuccess) return e;
        uint64_t *from = w.sort_a, *to = w.sort_b;
        blocks = uint32_t((N + kMergeKeys - 1) / kMergeKeys);
        for (int64_t len = kSortBlock; len < N; len *= kMergeWays) {
            int shift = 4;
            while ((len * kMergeWays) >> shift > kSamples) ++shift;
            fill = groups ? take_share(true) : 0; // one merge at most beside a fill: N <= kSortBlock * kMergeWays
            constexpr uint32_t slab = uint32_t(kLaunchThreads / kMergeThreads);
            for (uint32_t b = 0; b < blocks; b += slab) {
                const uint32_t n = blocks - b < slab ? blocks - b : slab;
                e = launch(merge_kernel, n + fill, kMergeThreads, s, from, uint32_t(N), uint32_t(len), shift, to, b, n, f);
                if (e != hipSuccess) return e;
            }
            uint64_t *t = from;
            from = to;
            to = t;
        }
        p.sorted = from;
    }
    p.fill_block = (p.chunks * p.slabs + 3) / 4;
    int64_t fill = 0;
    if (p.search) {
        fill = (a.vocab + 4 * kSearchRows - 1) / (4 * kSearchRows);
        if (fill > kLaunchThreads / 256 - p.fill_block) fill = kLaunchThreads / 256 - p.fill_block;
    } else {
        fill = take_share(short_sums);
    }
    if (p.fill_block + fill == 0) return hipSuccess;
    if ((e = launch(embed_grad_kernel<T, G>, p.fill_block + fill, 256, s, p)) != hipSuccess || !joined) return e;
    return launch(embed_join_kernel<G>, p.fill_block + take_share(true), 256, s, p);
}

} // namespace

// Chunks times slabs is at most kEmbedItems and a chunk's rounding, and a
// slab has at most 512 columns; short lists have N / kEmbedMinChunk chunks.
int64_t embed_partial_bytes(int64_t max_tokens, int64_t max_hidden)
{
    const int64_t by_items = kEmbedItems * 512 + max_hidden, by_tokens = (max_tokens / kEmbedMinChunk + 1) * max_hidden;
    return (by_items < by_tokens ? by_items : by_tokens) * 2 * int64_t(sizeof(float));
}

// A word more than the bits for each workgroup of the fill, of which there are
// at most two a CU, or kAbsentRows / kFillRows on a device of few.
int64_t embed_absent_bytes(int64_t max_vocab, int cus)
{
    const int64_t rows = max_vocab < kAbsentRows ? max_vocab : kAbsentRows;
    const int64_t few = kAbsentRows / kFillRows, groups = 2 * int64_t(cus) > few ? 2 * int64_t(cus) : few;
    return (rows / 32 + 2 * (groups + 1)) * int64_t(sizeof(uint32_t));
}

hipError_t launch_embed(const gwtf_stage_embed_t &a, hipStream_t s)
{
    switch (a.type) {
    case GWTF_TYPE_F32: return run_embed<float>(a, s);
    case GWTF_TYPE_F16: return run_embed<f16_t>(a, s);
    default: return run_embed<bf16_t>(a, s);
    }
}

hipError_t launch_embed_grad(const gwtf_stage_embed_grad_t &a, const StageWorkspace &w, hipStream_t s)
{
    const bool wide = a.grad_type == GWTF_TYPE_F32;
    switch (a.type) {
    case GWTF_TYPE_F32: return run_embed_grad<float, float>(a, w, s);
    case GWTF_TYPE_F16: return wide ? run_embed_grad<f16_t, float>(a, w, s) : run_embed_grad<f16_t, f16_t>(a, w, s);
    default: return wide ? run_embed_grad<bf16_t, float>(a, w, s) : run_embed_grad<bf16_t, bf16_t>(a, w, s);
    }
}

} // namespace gwtf
