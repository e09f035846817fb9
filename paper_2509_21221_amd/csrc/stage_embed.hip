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

template <class T>
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
    store8(static_cast<T *>(p.a.out) + row * p.a.out_stride + col, n, v);
}

// ---- sorting tokens ----
//
// Keys token << 32 | position are all different, so any sort is stable.  One
// workgroup sorts kSortBlock of them in LDS (bitonic); up to kMergeWays sorted
// blocks are merged in one launch, where each key finds its place by a binary
// search in every other block.

constexpr int kSortBlock = 2048;
constexpr int kMergeWays = 32;

__global__ __launch_bounds__(1024) void sort_block_kernel(const void *tokens, int token_type, int64_t vocab, int64_t N,
                                                          uint64_t *out)
{
    __shared__ uint64_t key[kSortBlock];
    const int64_t base = int64_t(blockIdx.x) * kSortBlock;
    for (int i = threadIdx.x; i < kSortBlock; i += 1024) {
        const int64_t pos = base + i;
        uint64_t k = ~uint64_t(0);
        if (pos < N) {
            const int64_t t = load_token(tokens, token_type, pos);
            k = (uint64_t(t >= 0 && t < vocab ? uint32_t(t) : 0xffffffffu) << 32) | uint32_t(pos);
        }
        key[i] = k;
    }
    __syncthreads();
    for (int size = 2; size <= kSortBlock; size <<= 1) {
        for (int j = size >> 1; j > 0; j >>= 1) {
            const int t = threadIdx.x, i = 2 * t - (t & (j - 1)), l = i + j;
            const uint64_t a = key[i], b = key[l];
            if ((a > b) == ((i & size) == 0)) {
                key[i] = b;
                key[l] = a;
            }
            __syncthreads();
        }
    }
    for (int i = threadIdx.x; i < kSortBlock; i += 1024)
        if (base + i < N) out[base + i] = key[i];
}

// Merges groups of kMergeWays sorted blocks of `len` keys.
__global__ __launch_bounds__(256) void merge_kernel(const uint64_t *in, int64_t N, int64_t len, uint64_t *out)
{
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= N) return;
    const uint64_t k = in[i];
    const int64_t own = i / len, group0 = own / kMergeWays * kMergeWays;
    int64_t place = group0 * len + (i - own * len);
    for (int64_t b = group0; b < group0 + kMergeWays && b * len < N; ++b) {
        if (b == own) continue;
        int64_t lo = b * len, hi = lo + len < N ? lo + len : N;
        const int64_t first = lo;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (in[mid] < k) lo = mid + 1;
            else hi = mid;
        }
        place += lo - first;
    }
    out[place] = k;
}

// ---- sums ----

struct EmbedGradParams {
    gwtf_stage_embed_grad_t a;
    const uint64_t *sorted;
    float *partial;           // [chunks][2][H]: of the run that began before the chunk, of the run that goes on after it
    int64_t chunk, chunks;
    int slabs;                // of 512 columns
    int64_t fill_block;       // first workgroup that writes zeros
};

constexpr int kFillRows = 16; // rows of the table a wave looks at for zeros

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

template <class T, class G>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedGradParams p)
{
    const gwtf_stage_embed_grad_t &a = p.a;
    const int lane = threadIdx.x & 63;
    const int64_t N = a.num_tokens;
    if (blockIdx.x >= p.fill_block) {
        // zeros for the rows whose token is absent
        const int64_t v0 = ((blockIdx.x - p.fill_block) * 4 + (threadIdx.x >> 6)) * int64_t(kFillRows);
        if (v0 >= a.vocab) return;
        bool absent = false;
        if (lane < kFillRows && v0 + lane < a.vocab) {
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
        const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        while (rows) {
            const int r = __builtin_ctzll(rows);
            rows &= rows - 1;
            G *g = static_cast<G *>(a.grad) + (v0 + r) * a.grad_stride;
            for (int64_t col = lane * kVec; col < a.hidden; col += 64 * kVec) store8(g + col, a.hidden - col, zero);
        }
        return;
    }
    const int64_t item = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int64_t c = item / p.slabs;
    if (c >= p.chunks) return;
    const int64_t col = (item - c * p.slabs) * 512 + lane * kVec, n = a.hidden - col;
    const int64_t e0 = c * p.chunk, e1 = e0 + p.chunk < N ? e0 + p.chunk : N;
    const T *dout = static_cast<const T *>(a.dout) + col;
    uint32_t token = key_token(p.sorted[e0]);
    if (token == 0xffffffffu) return;
    bool before = e0 > 0 && key_token(p.sorted[e0 - 1]) == token; // the run began in an earlier chunk
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t e = e0; e < e1; ++e) {
        const uint64_t k = p.sorted[e];
        const uint32_t t = key_token(k);
        if (t != token) {
            if (before) store8(p.partial + (c * 2) * a.hidden + col, n, acc);
            else write_grad<G>(a, token, col, n, acc);
            if (t == 0xffffffffu) return;
            before = false;
            token = t;
#pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] = 0.f;
        }
        float v[8];
        load8(dout + int64_t(uint32_t(k)) * a.dout_stride, n, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] += v[i];
    }
    const bool after = e1 < N && key_token(p.sorted[e1]) == token;
    if (before) store8(p.partial + (c * 2) * a.hidden + col, n, acc);
    else if (after) store8(p.partial + (c * 2 + 1) * a.hidden + col, n, acc);
    else write_grad<G>(a, token, col, n, acc);
}

// Runs that cross chunks, each by the wave of the chunk in which it begins.
template <class G>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradParams p)
{
    const gwtf_stage_embed_grad_t &a = p.a;
    const int lane = threadIdx.x & 63;
    const int64_t item = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int64_t c = item / p.slabs, N = a.num_tokens;
    const int64_t e0 = c * p.chunk, e1 = e0 + p.chunk;
    if (c >= p.chunks || e1 >= N) return;
    const uint32_t token = key_token(p.sorted[e1 - 1]);
    if (token == 0xffffffffu || key_token(p.sorted[e1]) != token) return; // no run goes on
    if (key_token(p.sorted[e0]) == token && e0 > 0 && key_token(p.sorted[e0 - 1]) == token) return; // began earlier
    const int64_t col = (item - c * p.slabs) * 512 + lane * kVec, n = a.hidden - col;
    float acc[8], v[8];
    load8(p.partial + (c * 2 + 1) * a.hidden + col, n, acc);
    for (int64_t d = c + 1; d < p.chunks && key_token(p.sorted[d * p.chunk]) == token; ++d) {
        load8(p.partial + (d * 2) * a.hidden + col, n, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] += v[i];
    }
    write_grad<G>(a, token, col, n, acc);
}

template <class T>
hipError_t run_embed(const gwtf_stage_embed_t &a, hipStream_t s)
{
    const int64_t steps = (a.hidden + kVec - 1) / kVec, slab = (int64_t(1) << 30) / steps;
    EmbedParams p;
    p.a = a;
    p.steps = FastDiv::make(uint32_t(steps));
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        p.row0 = r;
        p.units = uint32_t(n * steps);
        embed_kernel<T><<<dim3((p.units + 255) / 256), dim3(256), 0, s>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t slabs_of(int64_t H) { return (H + 511) / 512; }

int64_t chunk_of(int64_t N, int64_t H)
{
    const int64_t c = (N * slabs_of(H) + kEmbedItems - 1) / kEmbedItems;
    return c > kEmbedMinChunk ? c : kEmbedMinChunk;
}

template <class T, class G>
hipError_t run_embed_grad(const gwtf_stage_embed_grad_t &a, const StageWorkspace &w, hipStream_t s)
{
    hipError_t e;
    const int64_t N = a.num_tokens;
    EmbedGradParams p;
    p.a = a;
    p.sorted = w.sort_a;
    p.partial = w.partial;
    p.chunk = chunk_of(N, a.hidden);
    p.chunks = (N + p.chunk - 1) / p.chunk;
    p.slabs = int(slabs_of(a.hidden));
    if (N > 0) {
        sort_block_kernel<<<dim3(uint32_t((N + kSortBlock - 1) / kSortBlock)), dim3(1024), 0, s>>>(
            a.tokens, a.token_type, a.vocab, N, w.sort_a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        uint64_t *from = w.sort_a, *to = w.sort_b;
        for (int64_t len = kSortBlock; len < N; len *= kMergeWays) {
            merge_kernel<<<dim3(uint32_t((N + 255) / 256)), dim3(256), 0, s>>>(from, N, len, to);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            uint64_t *t = from;
            from = to;
            to = t;
        }
        p.sorted = from;
    }
    p.fill_block = (p.chunks * p.slabs + 3) / 4;
    const int64_t fill = a.accumulate ? 0 : (a.vocab + 4 * kFillRows - 1) / (4 * kFillRows);
    if (p.fill_block + fill == 0) return hipSuccess;
    embed_grad_kernel<T, G><<<dim3(uint32_t(p.fill_block + fill)), dim3(256), 0, s>>>(p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (p.chunks > 1) {
        embed_join_kernel<G><<<dim3(uint32_t(p.fill_block)), dim3(256), 0, s>>>(p);
        e = hipGetLastError();
    }
    return e;
}

} // namespace

// Chunks times slabs is at most kEmbedItems and a chunk's rounding, and a
// slab has at most 512 columns; short lists have N / kEmbedMinChunk chunks.
int64_t embed_partial_bytes(int64_t max_tokens, int64_t max_hidden)
{
    const int64_t by_items = kEmbedItems * 512 + max_hidden, by_tokens = (max_tokens / kEmbedMinChunk + 1) * max_hidden;
    return (by_items < by_tokens ? by_items : by_tokens) * 2 * int64_t(sizeof(float));
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
