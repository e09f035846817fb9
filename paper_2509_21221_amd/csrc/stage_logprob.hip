// Log probabilities of given tokens, entropy and the most likely tokens
// (gwtf_stage_logprob), and the gradient (gwtf_stage_logprob_grad).
//
// One pass over a row with the running maximum m of each lane,
//   s = sum e^(x - m)   and   t = sum e^(x - m) (x - m) / ln 2,
// both rescaled when m grows; parts with different m join the same way.  Then
//   lse = m + ln s,   entropy = ln s - ln 2 * t / s,
// where every term of t has one sign, so nothing cancels.  (x - m) log2 e as
// one fused operation with m log2 e at hand would overflow for masks of the
// type's lowest value.
//
// Alternatives: each wave keeps its largest entries as keys (order of the
// value, then lower index) sorted over its lanes, and looks closer at a step
// only where a lane's largest value passes the last of them.
#include "stage_device.h"
#include "stage_internal.h"

namespace gwtf {
namespace {

constexpr float kLowest = -200.f; // 2^-200 is 0: keeps 0 * -infinity out of t

struct Softmax {
    float m, s, t;
};

__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.f : m; }

__device__ __forceinline__ Softmax join(const Softmax &a, const Softmax &b)
{
    Softmax r;
    r.m = fmaxf(a.m, b.m);
    const float ms = finite_or_zero(r.m);
    const float da = (a.m - ms) * kLog2e, db = (b.m - ms) * kLog2e;
    const float ea = exp2_(da), eb = exp2_(db);
    r.s = a.s * ea + b.s * eb;
    r.t = ea * (a.t + fmaxf(da, kLowest) * a.s) + eb * (b.t + fmaxf(db, kLowest) * b.s);
    return r;
}

template <int n>
__device__ __forceinline__ Softmax row_ror(const Softmax &a)
{
    return {gwtf::row_ror<n>(a.m), gwtf::row_ror<n>(a.s), gwtf::row_ror<n>(a.t)};
}
__device__ __forceinline__ Softmax lane_of(const Softmax &a, int lane)
{
    return {lane_value(a.m, lane), lane_value(a.s, lane), lane_value(a.t, lane)};
}
__device__ __forceinline__ Softmax wave_join(Softmax a)
{
    a = join(a, row_ror<8>(a));
    a = join(a, row_ror<4>(a));
    a = join(a, row_ror<2>(a));
    a = join(a, row_ror<1>(a));
    return join(join(lane_of(a, 0), lane_of(a, 16)), join(lane_of(a, 32), lane_of(a, 48)));
}

// Order of a float as a signed integer; -0 counts as +0.
__device__ __forceinline__ int order_of(float x)
{
    const int b = __float_as_int(x + 0.f);
    return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int order) { return __int_as_float(order ^ ((order >> 31) & 0x7fffffff)); }
// Keys of entries are above 0, which stands for none.
__device__ __forceinline__ uint64_t key_of(int order, uint32_t index)
{
    return (uint64_t(uint32_t(order) ^ 0x80000000u) << 32) | (0xffffffffu - index);
}

__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane)
{
    const uint32_t hi = __builtin_amdgcn_readlane(int(k >> 32), lane), lo = __builtin_amdgcn_readlane(int(uint32_t(k)), lane);
    return (uint64_t(hi) << 32) | lo;
}

// The wave's `top` largest keys, the j-th in lane j, 0 in the other lanes.
// Keys join by rank: every new key is compared with the others and with the
// list in independent steps, where inserting them one after another is a
// chain of some 400 cycles for each (seven rows of 131,072 with eight
// alternatives: 96 us inserting, see the kernel for the present time).
struct TopList {
    uint64_t key, last; // this lane's; the smallest that counts (uniform)
    uint64_t *slots;    // `top` of this wave's, in LDS
    int top;
    __device__ __forceinline__ void start(int k, uint64_t *lds)
    {
        key = last = 0;
        slots = lds;
        top = k;
    }
    __device__ __forceinline__ bool list_empty() const { return lane_key(key, 0) == 0; }
    __device__ __forceinline__ int last_order() const { return int(uint32_t(last >> 32) ^ 0x80000000u); }
    // Takes the keys of the lanes with key > last (`some`, not empty).
    __device__ __forceinline__ void merge(uint64_t k, uint64_t some)
    {
        const int lane = __lane_id();
        int rank = 0, mine = lane;
        if (list_empty()) {
            for (uint64_t m = some; m; m &= m - 1) rank += lane_key(k, __builtin_ctzll(m)) > k;
            mine += __popcll(some);
        } else {
            for (uint64_t m = some; m; m &= m - 1) {
                const uint64_t other = lane_key(k, __builtin_ctzll(m));
                rank += other > k;
                mine += other > key;
            }
            for (int j = 0; j < top; ++j) rank += lane_key(key, j) > k;
        }
        if ((some >> lane & 1) && rank < top) slots[rank] = k;
        if (lane < top && mine < top) slots[mine] = key;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        key = lane < top ? slots[lane] : 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        last = lane_key(key, top - 1);
    }
    __device__ __forceinline__ void offer(uint64_t k)
    {
        const uint64_t some = __ballot(k > last);
        if (some) merge(k, some);
    }
};

struct LogprobParams {
    gwtf_stage_logprob_t a;
    int segments;       // workgroups that share a row
    int64_t width;      // columns of one, a multiple of kStep
    unsigned char *records;
    uint32_t *arrived;  // [rows], 0 between calls
};

constexpr int kLpWaves = 4;
constexpr int kStep = kLpWaves * 64 * kVec * 2; // columns of a workgroup's step

// The values that a row's sums give, from lane 0 of the wave that joined it;
// then its alternatives, from lanes below `top`.
__device__ __forceinline__ float log_prob(float x, float lse)
{
    return x == -__builtin_inff() && lse == lse ? x : x - lse;
}

template <class T>
__device__ __forceinline__ void finish_row(const gwtf_stage_logprob_t &a, int64_t row, const Softmax &r, const TopList &list)
{
    const int lane = threadIdx.x & 63;
    const float ln_s = logf(r.s), lse = finite_or_zero(r.m) + ln_s;
    if (lane == 0) {
        if (a.lse) a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = r.s == 0.f ? 0.f : ln_s - kLn2 * (r.t / r.s);
        if (a.logp) {
            const int64_t t = load_token(a.targets, a.token_type, row);
            float v = 0.f;
            if (t >= 0 && t < a.vocab) v = log_prob(float(static_cast<const T *>(a.logits)[row * a.logits_stride + t]), lse);
            a.logp[row] = v;
        }
    }
    if (lane < a.top) {
        const bool none = list.key == 0;
        const float x = value_of(int(uint32_t(list.key >> 32) ^ 0x80000000u));
        a.top_logp[row * a.top + lane] = none ? __builtin_nanf("") : log_prob(x, lse);
        a.top_ids[row * a.top + lane] = none ? -1 : int32_t(0xffffffffu - uint32_t(list.key));
    }
}

// Words of a record that a workgroup of another XCD reads in the same launch:
// written through to and read from memory, past the caches that the XCDs do
// not share.
__device__ __forceinline__ void put(uint32_t *p, uint32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(uint64_t *p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get_float(const uint32_t *p)
{
    return __uint_as_float(__hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ uint64_t get_key(const uint64_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <class T, bool TOP>
__global__ __launch_bounds__(kLpWaves * 64) void logprob_kernel(LogprobParams p)
{
    __shared__ Softmax parts[kLpWaves];
    __shared__ uint64_t keys[TOP ? kLpWaves * GWTF_STAGE_MAX_TOP : 1];
    __shared__ uint32_t last_one;
    const gwtf_stage_logprob_t &a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / uint32_t(p.segments), segment = blockIdx.x - uint32_t(row) * uint32_t(p.segments);
    const int64_t c0 = segment * p.width, c1 = c0 + p.width < a.vocab ? c0 + p.width : a.vocab;
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_stride;
    Softmax r = {-__builtin_inff(), 0.f, 0.f};
    TopList list;
    list.start(a.top, keys + (TOP ? wave * GWTF_STAGE_MAX_TOP : 0));
    for (int64_t base = c0; base < c1; base += kStep) {
        const int64_t col = base + (wave * 64 + lane) * kVec;
        float v[16];
        load8(x + col, c1 - col, v, -__builtin_inff());
        load8(x + col + kStep / 2, c1 - col - kStep / 2, v + 8, -__builtin_inff());
        float most = v[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, v[i]);
        const float m = fmaxf(r.m, most), ms = finite_or_zero(m);
        const float d0 = (r.m - ms) * kLog2e, e0 = exp2_(d0);
        r.t = e0 * (r.t + fmaxf(d0, kLowest) * r.s);
        r.s *= e0;
        r.m = m;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float d = (v[i] - ms) * kLog2e, e = exp2_(d);
            r.s += e;
            r.t += e * fmaxf(d, kLowest);
        }
        if constexpr (TOP) {
            // A wave goes up through its columns, so what only equals the
            // last of the list in a later step has the higher index.
            if (!__ballot(list.last == 0 || order_of(most) > list.last_order())) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (col + (i < 8 ? 0 : kStep / 2) + (i & 7) >= c1) v[i] = __builtin_nanf("");
            // Each lane offers its largest entry that is left, the lowest
            // index of equal ones, until none is above the list's last.
            for (;;) {
                float best = v[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) best = fmaxf(best, v[i]); // the other one of a NaN
                int slot = -1;
#pragma unroll
                for (int i = 15; i >= 0; --i) slot = v[i] == best ? i : slot;
                const uint32_t at = uint32_t(col) + (slot < 8 ? 0 : kStep / 2) + (slot & 7);
                const uint64_t k = slot < 0 ? 0 : key_of(order_of(best), at);
                const uint64_t some = __ballot(k > list.last);
                if (!some) break;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (slot == i) v[i] = __builtin_nanf("");
                list.merge(k, some);
            }
        }
    }
    r = wave_join(r);
    if (lane == 0) parts[wave] = r;
    if constexpr (TOP) {
        if (lane < a.top) keys[wave * GWTF_STAGE_MAX_TOP + lane] = list.key;
    }
    __syncthreads();
    if (wave == 0) {
        r = join(join(parts[0], parts[1]), join(parts[2], parts[3]));
        if constexpr (TOP) {
            for (int w = 1; w < kLpWaves; ++w) list.offer(lane < a.top ? keys[w * GWTF_STAGE_MAX_TOP + lane] : 0);
        }
    }
    if (p.segments == 1) {
        if (wave == 0) finish_row<T>(a, row, r, list);
        return;
    }
    // The workgroup that arrives last joins the row's records.  Records and
    // counter are words of agent scope; the wait puts a record in memory before
    // its arrival is counted.  (A fence of agent scope would write back and
    // drop the whole L2 of the XCD: 8 us on seven rows of 131,072.)
    unsigned char *record = p.records + int64_t(blockIdx.x) * kLogprobRecord;
    if (wave == 0) {
        if (lane == 0) {
            uint32_t *w = reinterpret_cast<uint32_t *>(record);
            put(w, __float_as_uint(r.m));
            put(w + 1, __float_as_uint(r.s));
            put(w + 2, __float_as_uint(r.t));
        }
        if constexpr (TOP) {
            if (lane < a.top) put(reinterpret_cast<uint64_t *>(record + 16) + lane, list.key);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (lane == 0)
            last_one = __hip_atomic_fetch_add(p.arrived + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                       uint32_t(p.segments - 1);
    }
    __syncthreads();
    if (!last_one) return;
    const unsigned char *first = p.records + row * p.segments * kLogprobRecord;
    if constexpr (TOP) {
        // all waves take parts of the keys, then the first one theirs
        list.start(a.top, keys + wave * GWTF_STAGE_MAX_TOP);
        const int all = p.segments * a.top;
        for (int i0 = wave * 64; i0 < all; i0 += kLpWaves * 64) {
            const int i = i0 + lane, seg = i / a.top;
            list.offer(i < all ? get_key(reinterpret_cast<const uint64_t *>(first + seg * kLogprobRecord + 16) + (i - seg * a.top)) : 0);
        }
        if (lane < a.top) keys[wave * GWTF_STAGE_MAX_TOP + lane] = list.key;
        __syncthreads();
    }
    if (wave != 0) return;
    r = {-__builtin_inff(), 0.f, 0.f};
    for (int i = lane; i < p.segments; i += 64) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(first + i * kLogprobRecord);
        r = join(r, Softmax{get_float(w), get_float(w + 1), get_float(w + 2)});
    }
    r = wave_join(r);
    if constexpr (TOP) {
        for (int w = 1; w < kLpWaves; ++w) list.offer(lane < a.top ? keys[w * GWTF_STAGE_MAX_TOP + lane] : 0);
    }
    finish_row<T>(a, row, r, list);
    if (lane == 0) p.arrived[row] = 0;
}

// ---- gradient ----

struct LogprobGradParams {
    gwtf_stage_logprob_grad_t a;
    int segments;
    int64_t width;
};

constexpr int kGradStep = 256 * kVec;

template <class T>
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobGradParams p)
{
    const gwtf_stage_logprob_grad_t &a = p.a;
    const int64_t row = blockIdx.x / uint32_t(p.segments), segment = blockIdx.x - uint32_t(row) * uint32_t(p.segments);
    const int64_t c0 = segment * p.width, c1 = c0 + p.width < a.vocab ? c0 + p.width : a.vocab;
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_stride;
    T *out = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
    const float lse = a.lse[row], ge = a.dentropy ? a.dentropy[row] : 0.f, entropy = a.dentropy ? a.entropy[row] : 0.f;
    int64_t t = -1;
    float gl = 0.f;
    if (a.dlogp) {
        t = load_token(a.targets, a.token_type, row);
        if (t >= 0 && t < a.vocab) gl = a.dlogp[row];
        else t = -1;
    }
    const bool empty = lse == -__builtin_inff();
    for (int64_t col = c0 + threadIdx.x * kVec; col < c1; col += kGradStep) {
        float v[8];
        load8(x + col, c1 - col, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = v[i] - lse, e = exp2_(d * kLog2e);
            // ln p is -infinity where p is 0
            float g = -e * (gl + ge * (fmaxf(d, kLowest) + entropy));
            if (col + i == t) g += gl;
            v[i] = empty ? 0.f : g;
        }
        store8(out + col, c1 - col, v);
    }
}

// Workgroups that share a row: one where there are rows enough, otherwise
// about four for each CU in all, of one step at least.
template <class P>
void split_rows(P &p, int64_t rows, int64_t vocab, int64_t step, int64_t wanted)
{
    const int64_t steps = (vocab + step - 1) / step;
    int64_t segments = rows >= kLogprobRows ? 1 : (wanted + rows - 1) / rows;
    if (segments > steps) segments = steps;
    const int64_t each = (steps + segments - 1) / segments;
    p.width = each * step;
    p.segments = int((steps + each - 1) / each);
}

template <class T>
hipError_t run_logprob(const gwtf_stage_logprob_t &a, const StageWorkspace &w, hipStream_t s)
{
    LogprobParams p;
    p.records = w.logprob;
    p.arrived = reinterpret_cast<uint32_t *>(w.logprob + int64_t(kLogprobItems) * kLogprobRecord);
    split_rows(p, a.num_tokens, a.vocab, kStep, 1024);
    // a launch's workgroups stay below 2^31
    const int64_t slab = (int64_t(1) << 30) / p.segments;
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        p.a = a;
        if (r > 0) { // only rows that are not split get here
            const size_t e = a.type == GWTF_TYPE_F32 ? 4 : 2;
            p.a.logits = static_cast<const char *>(a.logits) + size_t(r) * size_t(a.logits_stride) * e;
            if (a.targets) p.a.targets = static_cast<const char *>(a.targets) + size_t(r) * (a.token_type ? 8 : 4);
            if (a.logp) p.a.logp += r;
            if (a.entropy) p.a.entropy += r;
            if (a.lse) p.a.lse += r;
            if (a.top) {
                p.a.top_logp += r * a.top;
                p.a.top_ids += r * a.top;
            }
        }
        const dim3 grid(uint32_t(n * p.segments)), block(kLpWaves * 64);
        if (a.top) logprob_kernel<T, true><<<grid, block, 0, s>>>(p);
        else logprob_kernel<T, false><<<grid, block, 0, s>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t run_logprob_grad(const gwtf_stage_logprob_grad_t &a, hipStream_t s)
{
    LogprobGradParams p;
    split_rows(p, a.num_tokens, a.vocab, kGradStep, 2048);
    const int64_t slab = (int64_t(1) << 30) / p.segments;
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        p.a = a;
        const size_t e = a.type == GWTF_TYPE_F32 ? 4 : 2;
        p.a.logits = static_cast<const char *>(a.logits) + size_t(r) * size_t(a.logits_stride) * e;
        p.a.dlogits = static_cast<char *>(a.dlogits) + size_t(r) * size_t(a.dlogits_stride) * e;
        if (a.targets) p.a.targets = static_cast<const char *>(a.targets) + size_t(r) * (a.token_type ? 8 : 4);
        p.a.lse += r;
        if (a.entropy) p.a.entropy += r;
        if (a.dlogp) p.a.dlogp += r;
        if (a.dentropy) p.a.dentropy += r;
        logprob_grad_kernel<T><<<dim3(uint32_t(n * p.segments)), dim3(256), 0, s>>>(p);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

} // namespace

hipError_t launch_logprob(const gwtf_stage_logprob_t &a, const StageWorkspace &w, hipStream_t s)
{
    if (a.num_tokens == 0) return hipSuccess;
    switch (a.type) {
    case GWTF_TYPE_F32: return run_logprob<float>(a, w, s);
    case GWTF_TYPE_F16: return run_logprob<f16_t>(a, w, s);
    default: return run_logprob<bf16_t>(a, w, s);
    }
}

hipError_t launch_logprob_grad(const gwtf_stage_logprob_grad_t &a, const StageWorkspace &, hipStream_t s)
{
    if (a.num_tokens == 0) return hipSuccess;
    switch (a.type) {
    case GWTF_TYPE_F32: return run_logprob_grad<float>(a, s);
    case GWTF_TYPE_F16: return run_logprob_grad<f16_t>(a, s);
    default: return run_logprob_grad<bf16_t>(a, s);
    }
}

} // namespace gwtf
