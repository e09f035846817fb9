// Log probabilities of given tokens, entropy and the most likely tokens
// (gwtf_stage_logprob), and the gradient (gwtf_stage_logprob_grad).
//
// One pass over a row in base 2, y = x log2 e, with the running maximum m of
// each lane's y,
//   s = sum 2^(y - m)   and   t = sum 2^(y - m) (y - m),
// both rescaled when m grows; parts with different m join the same way.  Then
//   lse = ln 2 (m + log2 s),   entropy = ln 2 (log2 s - t / s),
// where every term of t has one sign, so nothing cancels.  The reference m of a
// lane is the rounded product y of its largest x, the same number in y - m, one
// fused operation, and in the result; what the rounding leaves is at most 2^-7
// as long as |m| <= 2^17 (kRange; beyond about 2^31 it would leave the range of
// the exponential).  So m starts at -2^17 and is never below: masked entries,
// -infinity or finite, add what they are worth under that reference, nothing.  A
// row whose largest y is not within (-2^17, 2^17] is gone through again with
// (x - m) log2 e in place of y - m and m the largest x (WIDE); its log
// probabilities are (x - m) - ln s, as lse in 32 bits does not resolve them.
//
// Columns are counted from the 16-byte boundary at or before the row's first
// entry (`off` columns before it), so that all reads but the first are aligned
// whatever the row's address is (4,096 x 131,071 bf16: 226 us without).
//
// Alternatives: a lane reads 16 adjacent columns at a time, a unit, and keeps
// the two units with the largest entries that it has met.  The `top` largest
// of these over the workgroup hold all alternatives, since any other unit has
// `top` entries before its first -- unless both of a lane's units are among
// them and a third might be: then that lane's columns are looked through.  With
// many alternatives, a NaN in the row (a unit may then hold no alternative at all),
// or too few units, it is gone through again with a list that is right for every
// input (list_pass).
// Ties go by index throughout: units are ordered as their columns are.
//
// A long batch is bound by memory with vector issue close behind (4,096 rows of
// 131,072 bf16, four alternatives: 194 us for 1.07 GB, 5.5 TB/s; nine vector
// instructions an entry, one of them the exponential at four times the others'
// issue).  A few rows are shared by workgroups and bound by what follows one
// another: the read, the selection, the record, the arrival (seven rows of
// 131,072, eight alternatives 10.3 us).  The gradient is bound by memory: 2,048 x
// 32,001 bf16 56 us (262 MB, 4.7 TB/s).
#include "stage_device.h"
#include "stage_internal.h"

namespace gwtf {
namespace {

constexpr int kLpWaves = 4;
constexpr int kLpThreads = kLpWaves * 64;
constexpr int kUnit = 16;
constexpr int kStep = kLpThreads * kUnit; // columns of a workgroup's step
// Two of the 24 largest units fall to one of 256 lanes in two rows of three, two
// of 8 in one of nine.
constexpr int kUnitTop = 24;
constexpr float kLowest = -200.f; // 2^-200 is 0: keeps 0 * -infinity out of t
constexpr float kNone = -__builtin_inff();
constexpr float kRange = 0x1p17f; // the largest f16 is below it

struct Softmax {
    float m, s, t;
};

// m as it is subtracted: finite where there is nothing but entries of -infinity.
template <bool WIDE>
__device__ __forceinline__ float reference(float m)
{
    return WIDE && m == kNone ? 0.f : m;
}
template <bool WIDE>
__device__ __forceinline__ Softmax nothing() { return {WIDE ? kNone : -kRange, 0.f, 0.f}; }

template <bool WIDE>
__device__ __forceinline__ Softmax join(const Softmax &a, const Softmax &b)
{
    Softmax r;
    r.m = fmaxf(a.m, b.m);
    const float ms = reference<WIDE>(r.m), f = WIDE ? kLog2e : 1.f;
    const float da = (a.m - ms) * f, db = (b.m - ms) * f;
    const float ea = exp2_(da), eb = exp2_(db);
    r.s = a.s * ea + b.s * eb;
    r.t = ea * (a.t + fmaxf(da, kLowest) * a.s) + eb * (b.t + fmaxf(db, kLowest) * b.s);
    return r;
}

// All lanes' parts, in every lane: each is rescaled once, then they add up.
template <bool WIDE>
__device__ __forceinline__ Softmax wave_join(const Softmax &a)
{
    const float m = wave_fmax(a.m);
    const float d = (a.m - reference<WIDE>(m)) * (WIDE ? kLog2e : 1.f), e = exp2_(d);
    return {m, wave_sum(a.s * e), wave_sum(e * (a.t + fmaxf(d, kLowest) * a.s))};
}

// A lane's 16 columns; `x_max`: their largest with the lane's former ones.
template <bool WIDE>
__device__ __forceinline__ void add_unit(Softmax &r, const float v[kUnit], float x_max)
{
    const float m = WIDE ? x_max : fmaxf(x_max * kLog2e, -kRange), ms = reference<WIDE>(m);
    const float d0 = (r.m - ms) * (WIDE ? kLog2e : 1.f), e0 = exp2_(d0);
    r.t = e0 * (r.t + fmaxf(d0, kLowest) * r.s);
    r.s *= e0;
    r.m = m;
#pragma unroll
    for (int i = 0; i < kUnit; ++i) {
        const float d = WIDE ? (v[i] - ms) * kLog2e : fmaf(v[i], kLog2e, -ms), e = exp2_(d);
        r.s += e;
        r.t = fmaf(e, fmaxf(d, kLowest), r.t);
    }
}
__device__ __forceinline__ float unit_max(const float v[kUnit])
{
    float most = v[0];
#pragma unroll
    for (int i = 1; i < kUnit; ++i) most = fmaxf(most, v[i]); // the other one of a NaN
    return most;
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
__device__ __forceinline__ uint32_t key_order(uint64_t k) { return uint32_t(k >> 32); } // unsigned
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - uint32_t(k); }

__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane)
{
    const uint32_t hi = __builtin_amdgcn_readlane(int(k >> 32), lane), lo = __builtin_amdgcn_readlane(int(uint32_t(k)), lane);
    return (uint64_t(hi) << 32) | lo;
}

// Orders LDS accesses of one wave's lanes.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr int kSlots = GWTF_STAGE_MAX_TOP;

// The wave's `top` largest keys, the j-th in lane j, 0 in the other lanes.
// Keys join by rank: every new key is compared with the others and with the
// list in independent steps, where inserting them one after another is a
// chain of some 400 cycles for each.
struct TopList {
    uint64_t key, last; // this lane's; the smallest that counts (uniform)
    uint64_t *slots;    // kSlots of this wave's, in LDS
    int top;
    __device__ __forceinline__ void start(int k, uint64_t *lds)
    {
        key = last = 0;
        slots = lds;
        top = k;
    }
    // Takes the keys of the lanes with key > last (`some`, not empty).
    __device__ __forceinline__ void merge(uint64_t k, uint64_t some)
    {
        const int lane = __lane_id();
        int rank = 0, mine = lane;
        for (uint64_t m = some; m; m &= m - 1) {
            const uint64_t other = lane_key(k, __builtin_ctzll(m));
            rank += other > k;
            mine += other > key;
        }
        if (lane_key(key, 0)) // not the first keys
            for (int j = 0; j < top; ++j) rank += lane_key(key, j) > k;
        if ((some >> lane & 1) && rank < top) slots[rank] = k;
        if (lane < top && mine < top) slots[mine] = key;
        wave_sync();
        key = lane < top ? slots[lane] : 0;
        wave_sync();
        last = lane_key(key, top - 1);
    }
    __device__ __forceinline__ void offer(uint64_t k)
    {
        const uint64_t some = __ballot(k > last);
        if (some) merge(k, some);
    }
    // A bound that enough of the lanes' words reach: the lanes are dealt out in
    // as many groups as there are keys wanted (or more), and it is the least of
    // the groups' largest words.
    __device__ __forceinline__ uint32_t bound_of(uint32_t w) const
    {
        auto fold = [](uint32_t a, uint32_t b, bool larger) { return (a > b) == larger ? a : b; };
        w = fold(w, uint32_t(__builtin_amdgcn_update_dpp(int(w), int(w), 0xB1, 0xf, 0xf, false)), top <= 32); // quad 1 0 3 2
        w = fold(w, uint32_t(__builtin_amdgcn_update_dpp(int(w), int(w), 0x4E, 0xf, 0xf, false)), top <= 16); // quad 2 3 0 1
        w = fold(w, uint32_t(__builtin_amdgcn_update_dpp(int(w), int(w), 0x141, 0xf, 0xf, false)), top <= 8); // half mirror
        w = fold(w, uint32_t(gwtf::row_ror<8>(int(w))), top <= 4);
        const uint32_t a = fold(__builtin_amdgcn_readlane(w, 0), __builtin_amdgcn_readlane(w, 16), top <= 2);
        const uint32_t b = fold(__builtin_amdgcn_readlane(w, 32), __builtin_amdgcn_readlane(w, 48), top <= 2);
        return fold(a, b, top <= 1);
    }
    // Puts the keys from `least` on into the slots; returns their number.
    template <int M>
    __device__ __forceinline__ int gather(const uint64_t (&k)[M], int m, uint64_t least) const
    {
        int count = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            if (i >= m) break;
            const bool in = k[i] != 0 && k[i] >= least;
            const uint64_t some = __ballot(in);
            const int place = count + __builtin_amdgcn_mbcnt_hi(uint32_t(some >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(some), 0));
            if (in && place < kSlots) slots[place] = k[i];
            count += __popcll(some);
        }
        return count;
    }
    // The largest of the first m of M keys a lane, into an empty list: those
    // that reach a bound, mostly no more than 64, join at once.  Where many
    // share the bound's order, their indices give a second one.
    template <int M>
    __device__ __forceinline__ void select(const uint64_t (&k)[M], int m = M)
    {
        const int lane = __lane_id();
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) best = umax(best, key_order(k[i]));
        const uint32_t order = bound_of(best);
        int count = gather(k, m, uint64_t(order) << 32);
        if (count > kSlots) {
            best = 0;
#pragma unroll
            for (int i = 0; i < M; ++i)
                best = umax(best, key_order(k[i]) > order ? 0xffffffffu : key_order(k[i]) == order ? uint32_t(k[i]) : 0u);
            wave_sync();
            count = gather(k, m, uint64_t(order) << 32 | bound_of(best));
        }
        if (count <= kSlots) {
            wave_sync();
            const uint64_t one = lane < count ? slots[lane] : 0;
            wave_sync();
            int rank = 0;
            for (int j = 0; j < count; j += 4) { // lanes past the last hold 0
#pragma unroll
                for (int q = 0; q < 4; ++q) rank += lane_key(one, j + q) > one;
            }
            if (lane < count && rank < top) slots[rank] = one;
            wave_sync();
            key = lane < top && lane < count ? slots[lane] : 0;
            wave_sync();
            last = lane_key(key, top - 1);
        } else {
#pragma unroll
            for (int i = 0; i < M; ++i) offer(k[i]);
        }
    }
};

struct LogprobParams {
    gwtf_stage_logprob_t a;
    int segments;       // workgroups that share a row
    int64_t width;      // columns of one, a multiple of kStep
    unsigned char *records;
    uint32_t *arrived;  // [rows], 0 between calls
};

// From lse = m + ln s; WIDE: from the parts.
template <bool WIDE>
__device__ __forceinline__ float log_prob(float x, float lse, float m, float ln_s)
{
    return x == kNone && lse == lse ? x : WIDE ? (x - m) - ln_s : x - lse;
}

// The values that a row's sums give, from lane 0 of the wave that joined it;
// then its alternatives, from lanes below `top`.
template <bool WIDE>
__device__ __forceinline__ void finish_row(const gwtf_stage_logprob_t &a, int64_t row, const Softmax &r, const TopList &list,
                                           bool there, float xt, float x_max)
{
    const int lane = __lane_id();
    const float ln_s = logf(r.s), m = reference<WIDE>(r.m);
    // ln 2 in two parts: one product would lose the last bits of m.  What rounding
    // is left may not put lse below the row's largest entry, or entropy below 0.
    float lse = WIDE ? m + ln_s : fmaf(m, kLn2, fmaf(m, kLn2Low, ln_s));
    float entropy = r.s == 0.f ? 0.f : ln_s - kLn2 * (r.t / r.s);
    if (lse < x_max) lse = x_max;
    if (entropy < 0.f) entropy = 0.f;
    if (lane == 0) {
        if (a.lse) a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = entropy;
        if (a.logp) a.logp[row] = there ? log_prob<WIDE>(xt, lse, m, ln_s) : 0.f;
    }
    if (lane < a.top) {
        const bool none = list.key == 0;
        const float x = value_of(int(key_order(list.key) ^ 0x80000000u));
        a.top_logp[row * a.top + lane] = none ? __builtin_nanf("") : log_prob<WIDE>(x, lse, m, ln_s);
        a.top_ids[row * a.top + lane] = none ? -1 : int32_t(key_index(list.key));
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

// The wave's part of the sums over a whole row with (x - m) log2 e.
template <class T>
__device__ __attribute__((noinline)) Softmax wide_pass(const T *x, int64_t vocab)
{
    Softmax r = nothing<true>();
    for (int64_t base = 0; base < vocab; base += kStep) {
        const int64_t col = base + threadIdx.x * kUnit;
        float v[kUnit];
        load8(x + col, vocab - col, v, kNone);
        load8(x + col + kVec, vocab - col - kVec, v + kVec, kNone);
        add_unit<true>(r, v, fmaxf(r.m, unit_max(v)));
    }
    return wave_join<true>(r);
}

// The wave's largest entries of columns [c0, c1) of a row, from all of them:
// each step, a lane offers its largest entry that is left, the lowest index of
// equal ones, until none is above the list's last.
template <class T>
__device__ __attribute__((noinline)) uint64_t list_pass(uint64_t *slots, int top, const T *x, int64_t c0, int64_t c1)
{
    TopList list;
    list.start(top, slots);
    for (int64_t base = c0; base < c1; base += kStep) {
        const int64_t col = base + threadIdx.x * kUnit;
        float v[kUnit];
        load8(x + col, c1 - col, v, __builtin_nanf(""));
        load8(x + col + kVec, c1 - col - kVec, v + kVec, __builtin_nanf(""));
        for (;;) {
            const float best = unit_max(v);
            int slot = -1;
#pragma unroll
            for (int i = kUnit - 1; i >= 0; --i) slot = v[i] == best ? i : slot;
            const uint64_t k = slot < 0 ? 0 : key_of(order_of(best), uint32_t(col + slot));
            const uint64_t some = __ballot(k > list.last);
            if (!some) break;
#pragma unroll
            for (int i = 0; i < kUnit; ++i)
                if (slot == i) v[i] = __builtin_nanf("");
            list.merge(k, some);
        }
    }
    return list.key;
}

// The entries of the units that `units` lists (16 a unit), largest first.
template <class T>
__device__ __forceinline__ void resolve_units(TopList &list, const TopList &units, const T *x, int off, int64_t c0, int64_t c1)
{
    constexpr int kBatch = kUnitTop * kUnit / 64;
    const int lane = __lane_id();
    const uint32_t least = key_order(units.last);
    uint64_t k[kBatch];
    float v[kBatch];
    uint32_t at[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
        const int i = q * 64 + lane;
        v[q] = __builtin_nanf("");
        at[q] = 0;
        if (q * 64 < units.top * kUnit) {
            const uint32_t unit = 0xffffffffu - uint32_t(__shfl(int(uint32_t(units.key)), i / kUnit & 63));
            const int64_t col = c0 + int64_t(unit) * kUnit + i % kUnit;
            at[q] = uint32_t(col - off);
            if (i < units.top * kUnit && col >= off && col < c1) v[q] = float(x[col - off]);
        }
    }
    list.start(units.top, units.slots);
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
        k[q] = v[q] == v[q] ? key_of(order_of(v[q]), at[q]) : 0;
        if (key_order(k[q]) < least) k[q] = 0;
    }
    list.select(k, (units.top * kUnit + 63) / 64);
}

// Offers the entries of every unit of those lanes whose two units are both in
// `units`, but for these two, which are resolved.
template <class T>
__device__ __forceinline__ void resolve_lanes(TopList &list, const TopList &units, const T *x, int off, int64_t c0, int64_t c1)
{
    const int lane = __lane_id();
    const uint32_t unit = key_index(units.key), owner = unit % kLpThreads;
    const int64_t total = (c1 - c0 + kUnit - 1) / kUnit;
    for (int j = 0; j + 1 < units.top; ++j) {
        const uint32_t o = __builtin_amdgcn_readlane(int(owner), j);
        const uint64_t both = __ballot(lane < units.top && owner == o);
        if (__popcll(both) < 2 || __builtin_ctzll(both) != j) continue;
        const uint32_t done0 = __builtin_amdgcn_readlane(int(unit), j);
        const uint32_t done1 = __builtin_amdgcn_readlane(int(unit), 63 - __builtin_clzll(both));
        for (int64_t u0 = o; u0 < total; u0 += 16 * kLpThreads) {
            float v[4];
            int64_t col[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t u = u0 + (q * 4 + lane / kUnit) * kLpThreads;
                col[q] = c0 + u * kUnit + lane % kUnit - off;
                v[q] = u < total && col[q] >= 0 && col[q] + off < c1 && u != done0 && u != done1 ? float(x[col[q]]) : __builtin_nanf("");
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) list.offer(v[q] == v[q] ? key_of(order_of(v[q]), uint32_t(col[q])) : 0);
        }
    }
}

template <class T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void logprob_kernel(LogprobParams p)
{
    __shared__ Softmax parts[kLpWaves];
    __shared__ uint64_t units_of[TOP ? 2 * kLpThreads : 1]; // and each wave's slots
    // two words: a wave may still read the first when another writes the second
    __shared__ uint32_t again_flag, last_flag;
    __shared__ float largest[kLpWaves];
    const gwtf_stage_logprob_t &a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / uint32_t(p.segments), segment = blockIdx.x - uint32_t(row) * uint32_t(p.segments);
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_stride;
    const int off = int(reinterpret_cast<uintptr_t>(x) & 15) / int(sizeof(T));
    const int64_t end = a.vocab + off, c0 = segment * p.width, c1 = c0 + p.width < end ? c0 + p.width : end;
    // The wave that joins the others' results: its work would pile up on one
    // SIMD if it were the same in all workgroups of a CU, which are 256 apart.
    const int chief = blockIdx.x >> 8 & (kLpWaves - 1);
    uint64_t *const slots = units_of + (TOP ? wave * kSlots : 0);
    // the target's entry is needed last and read first: two dependent reads
    int64_t target = -1;
    if (a.logp) target = load_token(a.targets, a.token_type, row);
    const bool there = target >= 0 && target < a.vocab;
    float xt = 0.f;
    if (there) xt = float(x[target]);
    Softmax r = nothing<false>();
    float first = kNone, second = kNone; // the largest entries of the lane's two units
    // The lane's first unit counts whatever it holds, so that rows of masked
    // entries have units too; others of -infinity come after 256 of these.
    int unit = threadIdx.x, unit1 = c0 + unit * kUnit < c1 ? unit : -1, unit2 = -1;
    auto add = [&](const float (&v)[kUnit]) {
        const float most = unit_max(v);
        if constexpr (TOP) {
            const bool above = most > first, between = most > second;
            unit2 = above ? unit1 : between ? unit : unit2;
            second = above ? first : fmaxf(second, most);
            unit1 = above ? unit : unit1;
        }
        first = fmaxf(first, most);
        add_unit<false>(r, v, first);
        unit += kLpThreads;
    };
    // a step that the row begins or ends in
    auto ragged = [&](int64_t base) {
        const int64_t col = base + threadIdx.x * kUnit - off;
        float v[kUnit];
        if (col >= 0) {
            load8(x + col, c1 - off - col, v, kNone);
            load8(x + col + kVec, c1 - off - col - kVec, v + kVec, kNone);
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = col + i >= 0 && col + i < c1 - off ? float(x[col + i]) : kNone;
        }
        add(v);
    };
    // whole steps between, with the next one on its way
    typedef typename Vec8<T>::type Raw;
    int64_t base = c0;
    if (base < off || base + kStep > c1) {
        if (base < c1) ragged(base);
        base += kStep;
    }
    const T *at = x + (base - off) + threadIdx.x * kUnit;
    Raw lo = {}, hi = {};
    if (base + kStep <= c1) {
        lo = *reinterpret_cast<const Raw *>(at);
        hi = *reinterpret_cast<const Raw *>(at + kVec);
    }
    for (; base + kStep <= c1; base += kStep) {
        float v[kUnit];
        widen<T>(lo, v);
        widen<T>(hi, v + kVec);
        at += kStep;
        if (base + 2 * kStep <= c1) {
            lo = *reinterpret_cast<const Raw *>(at);
            hi = *reinterpret_cast<const Raw *>(at + kVec);
        }
        add(v);
    }
    if (base < c1) ragged(base);
    {
        const float x_max = wave_fmax(first);
        const Softmax mine = wave_join<false>(r);
        if (lane == 0) {
            parts[wave] = mine;
            largest[wave] = x_max;
        }
    }
    if constexpr (TOP) {
        units_of[threadIdx.x] = unit1 < 0 ? 0 : key_of(order_of(first), uint32_t(unit1));
        units_of[kLpThreads + threadIdx.x] = unit2 < 0 || unit2 == unit1 ? 0 : key_of(order_of(second), uint32_t(unit2));
    }
    __syncthreads();
    r = wave_join<false>(lane < kLpWaves ? parts[lane] : nothing<false>());
    float x_max = fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3]));
    bool live = x_max > kNone; // an entry that is not masked
    TopList list;
    if constexpr (TOP) {
        // Nothing but masked entries (a NaN would show in s): the first columns.
        const bool masked = !live && r.s == 0.f;
        bool again = !masked && (a.top > kUnitTop || !(r.s == r.s));
        list.start(a.top, slots);
        if (masked) {
            const int64_t col = (c0 > off ? c0 - off : 0) + lane;
            if (lane < a.top && col < c1 - off) list.key = key_of(order_of(kNone), uint32_t(col));
        } else if (!again) {
            if (wave == chief) {
                uint64_t k[2 * kLpWaves];
#pragma unroll
                for (int i = 0; i < 2 * kLpWaves; ++i) k[i] = units_of[i * 64 + lane];
                wave_sync();
                list.select(k, c1 - c0 > kStep ? 2 * kLpWaves : kLpWaves); // one step: no second units
                again = list.last == 0;
                if (!again) {
                    const TopList units = list;
                    resolve_units(list, units, x, off, c0, c1);
                    if (c1 - c0 > 2 * kStep) resolve_lanes(list, units, x, off, c0, c1);
                    again = list.last == 0;
                }
                if (lane == 0) again_flag = again;
            }
            __syncthreads();
            again = again_flag;
        }
        if (again) {
            __syncthreads();
            const uint64_t mine = list_pass(slots, a.top, x, c0 > off ? c0 - off : 0, c1 - off);
            __syncthreads();
            units_of[threadIdx.x] = mine;
            __syncthreads();
            if (wave == chief) {
                uint64_t k[kLpWaves];
#pragma unroll
                for (int i = 0; i < kLpWaves; ++i) k[i] = units_of[i * 64 + lane];
                wave_sync();
                list.start(a.top, slots);
                list.select(k);
            }
        }
    }
    if (p.segments > 1) {
        // The workgroup that arrives last joins the row's records.  Records and
        // counter are words of agent scope; the wait puts a record in memory
        // before its arrival is counted.  (A fence of agent scope would write
        // back and drop the whole L2 of the XCD: 5 us on seven rows of 131,072.)
        if (wave == chief) {
            unsigned char *record = p.records + int64_t(blockIdx.x) * kLogprobRecord;
            if (lane == 0) {
                uint32_t *w = reinterpret_cast<uint32_t *>(record);
                put(w, __float_as_uint(r.m));
                put(w + 1, __float_as_uint(r.s));
                put(w + 2, __float_as_uint(r.t));
                put(w + 3, __float_as_uint(x_max));
            }
            if constexpr (TOP) {
                if (lane < a.top) put(reinterpret_cast<uint64_t *>(record + 16) + lane, list.key);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (lane == 0)
                last_flag = __hip_atomic_fetch_add(p.arrived + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                       uint32_t(p.segments - 1);
        }
        __syncthreads();
        if (!last_flag) return;
        const unsigned char *records = p.records + row * p.segments * kLogprobRecord;
        r = nothing<false>();
        x_max = kNone;
        for (int i = lane; i < p.segments; i += 64) { // in all waves alike
            const uint32_t *w = reinterpret_cast<const uint32_t *>(records + i * kLogprobRecord);
            r = join<false>(r, Softmax{get_float(w), get_float(w + 1), get_float(w + 2)});
            x_max = fmaxf(x_max, get_float(w + 3));
        }
        x_max = wave_fmax(x_max);
        live = x_max > kNone;
        r = wave_join<false>(r);
        if constexpr (TOP) {
            if (wave == chief) {
                constexpr int kBatch = 8; // keys of a lane read side by side
                // of a masked row, the first segment's
                const int all = (!live && r.s == 0.f ? 1 : p.segments) * a.top;
                list.start(a.top, slots);
                for (int i0 = 0; i0 < all; i0 += kBatch * 64) {
                    uint64_t k[kBatch];
#pragma unroll
                    for (int q = 0; q < kBatch; ++q) {
                        const int i = i0 + q * 64 + lane, seg = i / a.top;
                        k[q] = i < all ? get_key(reinterpret_cast<const uint64_t *>(records + seg * kLogprobRecord + 16) + (i - seg * a.top)) : 0;
                    }
                    if (i0 == 0) {
                        list.select(k, (all + 63) / 64);
                    } else {
#pragma unroll
                        for (int q = 0; q < kBatch; ++q) list.offer(k[q]);
                    }
                }
            }
        }
        if (threadIdx.x == 0) p.arrived[row] = 0;
    }
    // r is the row's, in all waves
    if (live && !(r.m > -kRange && r.m <= kRange)) {
        r = wide_pass(x, a.vocab);
        __syncthreads();
        if (lane == 0) parts[wave] = r;
        __syncthreads();
        if (wave != chief) return;
        r = wave_join<true>(lane < kLpWaves ? parts[lane] : nothing<true>());
        finish_row<true>(a, row, r, list, there, xt, x_max);
    } else if (wave == chief) {
        finish_row<false>(a, row, r, list, there, xt, x_max);
    }
}

// ---- gradient ----

struct LogprobGradParams {
    gwtf_stage_logprob_grad_t a;
    int segments;
    int64_t width;
};

constexpr int kGradStep = 256 * kVec;
constexpr int kGradSteps = 2; // with their reads side by side

// STREAM: whole steps past the caches; they lie on lines whatever the rows do.
template <class T, bool STREAM>
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobGradParams p)
{
    const gwtf_stage_logprob_grad_t &a = p.a;
    const uint32_t row32 = blockIdx.x / uint32_t(p.segments), segment = blockIdx.x - row32 * uint32_t(p.segments);
    const int64_t row = row32;
    const T *x = static_cast<const T *>(a.logits) + row * a.logits_stride;
    T *out = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
    // Steps begin where the row of dlogits is aligned to 16 bytes (2,048 x
    // 32,001 bf16: 56 us, 58 without); the columns before belong to the first part.
    int64_t head = (-reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T);
    if (head > a.vocab) head = a.vocab;
    const int64_t c0 = head + segment * p.width, c1 = c0 + p.width < a.vocab ? c0 + p.width : a.vocab;
    float lse = a.lse[row], ge = a.dentropy ? a.dentropy[row] : 0.f, entropy = a.dentropy ? a.entropy[row] : 0.f;
    int64_t t = -1;
    float gl = 0.f;
    if (a.dlogp) {
        t = load_token(a.targets, a.token_type, row);
        if (t >= 0 && t < a.vocab) gl = a.dlogp[row];
        else t = -1;
    }
    if (lse == kNone) { // all masked: nothing reaches them
        lse = ge = gl = 0.f;
        t = -1;
    }
    auto grad = [&](float (&v)[8], int64_t col) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = v[i] - lse, e = exp2_(d * kLog2e);
            // ln p is -infinity where p is 0
            v[i] = -e * (gl + ge * (fmaxf(d, kLowest) + entropy));
        }
        const int64_t mine = t - col;
        if (__ballot(uint64_t(mine) < kVec)) {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (mine == i) v[i] += gl;
        }
    };
    typedef typename Vec8<T>::type Raw;
    int64_t base = c0;
    for (; base + kGradSteps * kGradStep <= c1; base += kGradSteps * kGradStep) {
        const int64_t col = base + threadIdx.x * kVec;
        Raw raw[kGradSteps];
#pragma unroll
        for (int q = 0; q < kGradSteps; ++q) raw[q] = load8_raw<T, STREAM>(x + col + q * kGradStep, kVec);
#pragma unroll
        for (int q = 0; q < kGradSteps; ++q) {
            float v[8];
            widen<T>(raw[q], v);
            grad(v, col + q * kGradStep);
            store8<T, STREAM>(out + col + q * kGradStep, kVec, v);
        }
    }
    for (; base < c1; base += kGradStep) {
        const int64_t col = base + threadIdx.x * kVec;
        float v[8];
        load8(x + col, c1 - col, v);
        grad(v, col);
        store8(out + col, c1 - col, v);
    }
    if (segment == 0 && head > 0 && threadIdx.x < 64) {
        float v[8];
        const int64_t n = threadIdx.x == 0 ? head : 0;
        load8(x, n, v);
        grad(v, threadIdx.x == 0 ? 0 : a.vocab);
        store8(out, n, v);
    }
}

// Workgroups that share a row: one where there are rows enough, otherwise
// about `wanted` in all, of `step` columns at least.  (Log probabilities with
// eight alternatives, two steps of a workgroup at least and one: a row of
// 5,000 6.2 us and 8.8, of 32,000 9.5 and 8.8, seven of 131,072 10.4 and 11.4.)
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
    // columns as the kernel counts them
    const bool aligned = on_lines(a.logits, a.num_tokens > 1 ? a.logits_stride : 0, sizeof(T));
    split_rows(p, a.num_tokens, a.vocab + (aligned ? 0 : 16 / int64_t(sizeof(T)) - 1), 2 * kStep, 1024);
    const int64_t slab = kLaunchThreads / kLpThreads / p.segments;
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
        const hipError_t e = launch(a.top ? logprob_kernel<T, true> : logprob_kernel<T, false>, n * p.segments, kLpThreads, s, p);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t run_logprob_grad(const gwtf_stage_logprob_grad_t &a, hipStream_t s)
{
    LogprobGradParams p;
    split_rows(p, a.num_tokens, a.vocab, kGradStep, 2048);
    const bool stream = 2 * a.num_tokens * a.vocab * int64_t(sizeof(T)) >= kStreamBytes;
    auto kernel = stream ? logprob_grad_kernel<T, true> : logprob_grad_kernel<T, false>;
    const int64_t slab = kLaunchThreads / 256 / p.segments;
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
        const hipError_t err = launch(kernel, n * p.segments, 256, s, p);
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
