// Answers drawn from logits (gwtf_learn_sample).
//
//   w_j = 2^y_j,  y_j = (x_j - max x) log2 e / T,  in 64 bits
//
// A workgroup takes a row.  The tokens that stay are the first n in the order of
// descending logits, so all three filters are cuts in that order: a key (the
// logit's bits in an order of unsigned words) and how many of the entries with
// that key stay, by ascending index.  A cut by number or by sum is found by
// counting keys in equal bins between two bounds (and adding up w, as whole
// numbers, so that the order of the additions does not matter), and again within
// the bin that the cut falls into, until a bin is one key.  The draw needs no
// order: sums of what stays over segments of the row, then a prefix within the
// segment that u falls into.
#include "learn_internal.h"
#include "stage_device.h"

namespace gwtf {
namespace {

constexpr int kStepCols = 64 * kVec; // columns of a wave's step
constexpr uint32_t kNoneKey = 0x007fffffu; // of -infinity
constexpr double kLog2e64 = 1.4426950408889634074;
constexpr double kLn264 = 0.69314718055994530942;

__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f); // -0 is 0
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

// 2^y, y <= 0, to about 1e-15: 2^f by the exponential's series in f ln 2, |f| <= 1/2.
__device__ __forceinline__ double exp2_64(double y)
{
    y = fmax(y, -1100.0);
    const double n = rint(y), z = (y - n) * kLn264;
    double s = 1.0 / 6227020800.0;
    s = fma(s, z, 1.0 / 479001600.0);
    s = fma(s, z, 1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 3628800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, 1.0 / 40320.0);
    s = fma(s, z, 1.0 / 5040.0);
    s = fma(s, z, 1.0 / 720.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, 1.0 / 24.0);
    s = fma(s, z, 1.0 / 6.0);
    s = fma(s, z, 0.5);
    s = fma(s, z, 1.0);
    s = fma(s, z, 1.0);
    return ldexp(s, int(n));
}

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ uint32_t wave_add(uint32_t v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Entries of the order that stay: those with larger keys, and `ties` with this
// one, by ascending index; n of them in all.
struct Cut {
    uint32_t key, ties, n;
};

constexpr int kBins = 2048, kSegs = 1024;

template <int WAVES>
struct Shared {
    uint32_t count[kBins];
    uint64_t mass[kBins];
    double sum[kSegs];    // of a segment's w whose keys are above the cut's
    uint32_t tied[kSegs]; // its entries with the cut's key
    double wsum[WAVES];
    uint32_t wcount[WAVES];
    uint32_t at; // first bin from the top that reaches a target
    struct {
        uint32_t count, above;
        double above_mass;
    } bin;
    struct {
        uint32_t seg, tied;
        double total, before, target;
    } draw;
};

template <class T, int WAVES>
struct Row {
    static constexpr int kThreads = WAVES * 64;
    // keys of a type differ above this bit only
    static constexpr int kRes = sizeof(T) == 4 ? 0 : __is_same(T, bf16_t) ? 16 : 13;
    Shared<WAVES> &sh;
    const T *x;
    int64_t V, steps;
    int lane, wave;
    int per, segs; // steps of a segment, segments
    double top, c; // the largest entry, log2 e / T
    int unit;      // the whole numbers that stand for w are w 2^unit

    // f(first column of this lane's eight, their values) for every step of a segment, done(segment) after them
    template <class F, class D>
    __device__ __forceinline__ void scan(F f, D done)
    {
        for (int seg = wave; seg < segs; seg += WAVES) {
            for (int q = 0; q < per; ++q) {
                const int64_t col = (int64_t(seg) * per + q) * kStepCols + lane * kVec;
                float v[8];
                load8(x + col, V - col, v, -__builtin_inff());
                f(v);
            }
            done(seg);
        }
    }
    __device__ __forceinline__ double weight(float v) const { return exp2_64((double(v) - top) * c); }

    __device__ __forceinline__ uint32_t block_add(uint32_t v)
    {
        v = wave_add(v);
        __syncthreads();
        if (lane == 0) sh.wcount[wave] = v;
        __syncthreads();
        uint32_t s = 0;
        for (int i = 0; i < WAVES; ++i) s += sh.wcount[i];
        return s;
    }
    __device__ __forceinline__ uint32_t block_umax(uint32_t v)
    {
        v = wave_umax(v);
        __syncthreads();
        if (lane == 0) sh.wcount[wave] = v;
        __syncthreads();
        uint32_t s = 0;
        for (int i = 0; i < WAVES; ++i) s = umax(s, sh.wcount[i]);
        return s;
    }

    __device__ __forceinline__ void clear_bins()
    {
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            sh.count[b] = 0;
            sh.mass[b] = 0;
        }
        if (threadIdx.x == 0) sh.at = kBins;
        __syncthreads();
    }
    // The key that bin b of keys from lo on holds, where a bin is one key.
    __device__ __forceinline__ uint32_t bin_key(uint32_t lo, uint32_t b) const
    {
        const uint32_t k = lo + (b << kRes);
        return (k & 0x80000000u) ? k : k | ((1u << kRes) - 1u);
    }
    // The first bin from the top, where entries (or their sum of w) reach the
    // target, with `above` and `above_mass` before all bins; its place is in sh.at,
    // what it holds and what lies above it in sh.bin.  one: a bin is one key.
    __device__ __forceinline__ void find_bin(bool by_mass, uint32_t target, double target_mass, uint32_t above, double above_mass, uint32_t lo, bool one)
    {
        constexpr int kEach = kBins / kThreads;
        __syncthreads();
        uint32_t n[kEach], before = 0;
        double m[kEach], before_mass = 0.0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const int b = kBins - 1 - (int(threadIdx.x) * kEach + q);
            n[q] = sh.count[b];
            m[q] = 0.0;
            if (by_mass && n[q]) m[q] = one ? double(n[q]) * weight(value_of(bin_key(lo, b))) : ldexp(double(sh.mass[b]), -unit);
            before += n[q];
            before_mass += m[q];
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(before, d);
            const double om = __shfl_up(before_mass, d);
            before += lane >= d ? o : 0u;
            before_mass += lane >= d ? om : 0.0;
        }
        if (lane == 63) {
            sh.wcount[wave] = before;
            sh.wsum[wave] = before_mass;
        }
        const uint32_t up = __shfl_up(before, 1);
        const double up_mass = __shfl_up(before_mass, 1);
        before = above;
        before_mass = above_mass;
        __syncthreads();
        for (int i = 0; i < wave; ++i) {
            before += sh.wcount[i];
            before_mass += sh.wsum[i];
        }
        before += lane ? up : 0u;
        before_mass += lane ? up_mass : 0.0;
        uint32_t first = kBins, in = 0, over = 0;
        double over_mass = 0.0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const bool reached = by_mass ? before_mass + m[q] >= target_mass : before + n[q] >= target;
            if (n[q] && reached && first == kBins) {
                first = threadIdx.x * kEach + q;
                in = n[q];
                over = before;
                over_mass = before_mass;
            }
            before += n[q];
            before_mass += m[q];
        }
        if (first < kBins) atomicMin(&sh.at, first);
        __syncthreads();
        if (first < kBins && sh.at == first) {
            sh.bin.count = in;
            sh.bin.above = over;
            sh.bin.above_mass = over_mass;
        }
        __syncthreads();
    }

    // The cut after `target` entries, or after the least number of them whose sum of
    // w reaches `target_mass`; no entry with a key below lo is in question.  none:
    // what holds where rounding lets no sum reach the target.
    __device__ __forceinline__ Cut select(bool by_mass, uint32_t target, double target_mass, uint32_t lo, Cut none)
    {
        uint32_t hi = key_of(float(top)), above = 0;
        double above_mass = 0.0;
        for (;;) {
            lo = lo >> kRes << kRes;
            int shift = kRes;
            while (((hi - lo) >> shift) >= uint32_t(kBins)) ++shift;
            const bool one = shift == kRes, add = by_mass && !one;
            clear_bins();
            scan(
                [&](const float *v) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const uint32_t k = key_of(v[i]);
                        if (k < lo || k > hi || k <= kNoneKey) continue;
                        const uint32_t b = (k - lo) >> shift;
                        atomicAdd(&sh.count[b], 1u);
                        if (add)
                            atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[b]), (unsigned long long)(ldexp(weight(v[i]), unit)));
                    }
                },
                [](int) {});
            find_bin(by_mass, target, target_mass, above, above_mass, lo, one);
            if (sh.at == kBins) return none;
            const uint32_t b = kBins - 1 - sh.at;
            above = sh.bin.above;
            above_mass = sh.bin.above_mass;
            if (one) {
                Cut cut;
                cut.key = bin_key(lo, b);
                if (by_mass) {
                    const double w = weight(value_of(cut.key)), most = double(sh.bin.count);
                    double t = fmin(fmax(ceil((target_mass - above_mass) / w), 1.0), most);
                    // the division may be off by its last bit
                    if (t > 1.0 && above_mass + (t - 1.0) * w >= target_mass) t -= 1.0;
                    if (t < most && above_mass + t * w < target_mass) t += 1.0;
                    cut.ties = uint32_t(t);
                } else {
                    cut.ties = target - above;
                }
                cut.n = above + cut.ties;
                return cut;
            }
            lo += b << shift;
            const uint32_t end = lo + ((1u << shift) - 1u);
            hi = end < hi ? end : hi;
        }
    }

    // Sums of w over what stays, by segment, and over the row (sh.draw.total);
    // then the segment in which the sum passes u times the row's (sh.draw).
    __device__ __forceinline__ void sums(const Cut &cut, double u)
    {
        const float least = value_of(cut.key);
        double s = 0.0;
        uint32_t e = 0;
        __syncthreads();
        scan(
            [&](const float *v) {
                bool any = false;
#pragma unroll
                for (int i = 0; i < kVec; ++i) any = any || v[i] >= least;
                if (!__ballot(any)) return;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    s += v[i] > least ? weight(v[i]) : 0.0;
                    e += v[i] == least ? 1u : 0u;
                }
            },
            [&](int seg) {
                const double all = wave_sum64(s);
                const uint32_t tied = wave_add(e);
                if (lane == 0) {
                    sh.sum[seg] = all;
                    sh.tied[seg] = tied;
                }
                s = 0.0;
                e = 0;
            });
        __syncthreads();
        if (wave == 0) {
            const double wc = cut.ties ? weight(least) : 0.0;
            const int each = (segs + 63) / 64, j0 = lane * each, j1 = j0 + each < segs ? j0 + each : segs;
            uint32_t tied = 0;
            for (int j = j0; j < j1; ++j) tied += sh.tied[j];
            uint32_t before = tied;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t o = __shfl_up(before, d);
                before += lane >= d ? o : 0u;
            }
            before -= tied;
            const uint32_t first_tied = before;
            double mass = 0.0;
            for (int j = j0; j < j1; ++j) {
                mass += sh.sum[j] + double(stay(sh.tied[j], before, cut.ties)) * wc;
                before += sh.tied[j];
            }
            double after = mass;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double o = __shfl_up(after, d);
                after += lane >= d ? o : 0.0;
            }
            const double up = __shfl_up(after, 1), total = __shfl(after, 63), target = u * total;
            double at = lane ? up : 0.0;
            // the first lane whose segments pass the target; where rounding lets none, the last that has a token
            const uint64_t pass = __ballot(after > target && mass > 0.0), some = __ballot(mass > 0.0);
            const int who = pass ? __builtin_ctzll(pass) : 63 - __builtin_clzll(some ? some : 1ull);
            if (lane == who) {
                uint32_t seg = uint32_t(j0), seg_tied = first_tied;
                double seg_at = at;
                before = first_tied;
                for (int j = j0; j < j1; ++j) {
                    const double add = sh.sum[j] + double(stay(sh.tied[j], before, cut.ties)) * wc;
                    if (add > 0.0) {
                        seg = uint32_t(j);
                        seg_tied = before;
                        seg_at = at;
                        if (at + add > target) break;
                    }
                    at += add;
                    before += sh.tied[j];
                }
                sh.draw.seg = seg;
                sh.draw.tied = seg_tied;
                sh.draw.before = seg_at;
                sh.draw.target = target;
                sh.draw.total = total;
            }
        }
        __syncthreads();
    }
    // How many of `tied` entries stay, with `before` of them before.
    static __device__ __forceinline__ uint32_t stay(uint32_t tied, uint32_t before, uint32_t ties)
    {
        const uint32_t left = before < ties ? ties - before : 0u;
        return tied < left ? tied : left;
    }

    // The token within the segment of sh.draw; by one wave.
    __device__ __forceinline__ void draw(const Cut &cut, int32_t *id, float *logp)
    {
        const float least = value_of(cut.key);
        const double target = sh.draw.target;
        double run = sh.draw.before;
        uint32_t tied = sh.draw.tied;
        int64_t found = -1;
        double w_found = 0.0;
        for (int q = 0; q < per; ++q) {
            const int64_t col = (int64_t(sh.draw.seg) * per + q) * kStepCols + lane * kVec;
            float v[8];
            load8(x + col, V - col, v, -__builtin_inff());
            uint32_t e = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) e += v[i] == least && least > -__builtin_inff() ? 1u : 0u;
            uint32_t before = e;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t o = __shfl_up(before, d);
                before += lane >= d ? o : 0u;
            }
            const uint32_t step_tied = __shfl(before, 63);
            before += tied - e;
            tied += step_tied;
            double w[8], mine = 0.0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                bool in = v[i] > least;
                if (v[i] == least && least > -__builtin_inff()) in = before++ < cut.ties;
                w[i] = in ? weight(v[i]) : 0.0;
                mine += w[i];
            }
            double after = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double o = __shfl_up(after, d);
                after += lane >= d ? o : 0.0;
            }
            const double up = __shfl_up(after, 1), end = __shfl(after, 63);
            const uint64_t pass = __ballot(run + after > target && mine > 0.0), some = __ballot(mine > 0.0);
            if (some) { // without a lane that passes, the last token so far is the one if none follows
                const int who = pass ? __builtin_ctzll(pass) : 63 - __builtin_clzll(some);
                double at = run + (lane ? up : 0.0);
                int which = 0;
                bool over = false;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    at += w[i];
                    if (w[i] > 0.0 && !over) {
                        which = i;
                        over = at > target;
                    }
                }
                double w_which = 0.0;
#pragma unroll
                for (int i = 0; i < kVec; ++i) w_which = i == which ? w[i] : w_which;
                found = __shfl(col + which, who);
                w_found = __shfl(w_which, who);
            }
            run += end;
            if (pass) break;
        }
        if (lane == 0) {
            *id = int32_t(found);
            if (logp) *logp = float(log(w_found / sh.draw.total));
        }
    }
};

struct SampleArgs {
    gwtf_learn_sample_t a;
    int64_t row0;
    int32_t steps, per, segs, unit;
};

template <class T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sample_kernel(SampleArgs p)
{
    __shared__ Shared<WAVES> sh;
    const gwtf_learn_sample_t &a = p.a;
    const int64_t i = p.row0 + blockIdx.x;
    Row<T, WAVES> row{sh, static_cast<const T *>(a.logits) + i * a.logits_stride, a.vocab, p.steps, int(threadIdx.x & 63),
                      __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p.per, p.segs, 0.0, 0.0, p.unit};
    const double T_ = a.temperatures ? double(a.temperatures[i]) : a.temperature;
    const double top_p = a.top_ps ? double(a.top_ps[i]) : a.top_p;
    const double min_p = a.min_ps ? double(a.min_ps[i]) : a.min_p;
    const int32_t top_k = a.top_ks ? a.top_ks[i] : a.top_k;
    double u = a.uniform_type == GWTF_UNIFORM_F64 ? static_cast<const double *>(a.u)[i] : double(static_cast<const float *>(a.u)[i]);
    u = u >= 0.0 ? u : 0.0;

    // the largest entry, how many are not masked, whether one is a NaN or +infinity
    float most = -__builtin_inff();
    uint32_t there = 0;
    bool bad = !(T_ >= 0.0 && T_ < __builtin_inf()) || !(top_p >= 0.0) || !(min_p >= 0.0 && min_p <= 1.0);
    row.scan(
        [&](const float *v) {
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                bad = bad || !(v[k] < __builtin_inff());
                most = fmaxf(most, v[k]);
                there += v[k] > -__builtin_inff() ? 1u : 0u;
            }
        },
        [](int) {});
    row.top = double(value_of(row.block_umax(key_of(most))));
    const uint32_t F = row.block_add(there);
    const bool wrong = row.block_add(bad ? 1u : 0u) != 0;
    if (wrong || F == 0) {
        if (threadIdx.x == 0) {
            a.ids[i] = -1;
            if (a.logp) a.logp[i] = wrong ? __builtin_nanf("") : -__builtin_inff();
            if (a.kept) a.kept[i] = 0;
        }
        return;
    }

    Cut cut = {kNoneKey, 0, F};
    bool summed = false;
    row.c = kLog2e64 / (T_ > 1e-300 ? T_ : 1e-300);
    if (T_ == 0.0 || top_k == 1 || top_p == 0.0) {
        cut = {key_of(float(row.top)), 1, 1};
    } else {
        if (top_k > 0 && uint32_t(top_k) < F) cut = row.select(false, uint32_t(top_k), 0.0, kNoneKey + 1, cut);
        if (top_p < 1.0) {
            row.sums(cut, u);
            summed = true;
            // The entry that the sum ends with and those after it are worth more than
            // (1 - p) of the sum: it is above that over their number.
            const double all = sh.draw.total, least = 0.99 * (1.0 - top_p) * all / double(cut.n);
            const uint32_t k = key_of(float(row.top + log2(least) / row.c)), lo = k > kNoneKey + 3 ? k - 2 : kNoneKey + 1;
            const Cut by_mass = row.select(true, 0, top_p * all, lo, cut);
            if (by_mass.n < cut.n) {
                cut = by_mass;
                summed = false;
            }
        }
        if (min_p > 0.0) {
            // the smallest 32-bit number whose w reaches min_p
            const double at = row.top + log2(min_p) / row.c;
            float least = float(at);
            if (double(least) < at) least = value_of(key_of(least) + 1);
            uint32_t n = 0;
            row.scan(
                [&](const float *v) {
#pragma unroll
                    for (int k = 0; k < kVec; ++k) n += v[k] >= least ? 1u : 0u;
                },
                [](int) {});
            n = row.block_add(n);
            if (n < cut.n) {
                cut = {key_of(least), ~0u, n};
                summed = false;
            }
        }
    }
    if (!summed) row.sums(cut, u);
    if (row.wave == 0) row.draw(cut, a.ids + i, a.logp ? a.logp + i : nullptr);
    if (threadIdx.x == 0 && a.kept) a.kept[i] = int32_t(cut.n);
}

template <class T>
hipError_t run(const gwtf_learn_sample_t &a, hipStream_t s)
{
    SampleArgs p;
    p.a = a;
    p.steps = int32_t((a.vocab + kStepCols - 1) / kStepCols);
    p.per = (p.steps + kSegs - 1) / kSegs;
    p.segs = (p.steps + p.per - 1) / p.per;
    p.unit = 62;
    while ((int64_t(1) << (62 - p.unit)) < a.vocab) --p.unit;
    const bool wide = a.vocab > 16384;
    const int threads = wide ? 1024 : 256;
    const int64_t slab = kLaunchThreads / threads;
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        p.row0 = r;
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        const hipError_t e = launch(wide ? sample_kernel<T, 16> : sample_kernel<T, 4>, n, threads, s, p);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace

hipError_t launch_sample(const gwtf_learn_sample_t &a, hipStream_t s)
{
    switch (a.type) {
    case GWTF_TYPE_F32: return run<float>(a, s);
    case GWTF_TYPE_F16: return run<f16_t>(a, s);
    default: return run<bf16_t>(a, s);
    }
}

} // namespace gwtf
