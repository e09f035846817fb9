// Answers drawn from logits (gwtf_learn_sample).
//
//   w_j = 2^y_j,  y_j = (x_j - max x) log2 e / T,  in 64 bits
//
// A workgroup takes a row and keeps it in registers, up to 131,072 columns of 16
// bits or 65,536 of 32, since every filter needs another look at it; a lane also
// keeps the largest of each of its eights, so that looks at few entries pass
// over the others.
//
// The tokens that stay are the first n in the order of descending logits, so all
// three filters are cuts in that order: a key (the logit's bits in an order of
// unsigned words) and how many of the entries with that key stay, by ascending
// index.  A cut by number or by sum is found by counting keys in equal bins
// between two bounds (and adding up w, as whole numbers, so that the order of the
// additions does not matter), and again within the bin that the cut falls into,
// until a bin is one key.  Whole numbers of one unit would lose what is far below the
// largest, so sums of many entries are first taken in bins by distance from it, each in a
// unit of its own.  The draw needs no order: sums of what stays over segments of the row,
// then a prefix within the segment that u falls into.
//
// With top_k up to kFew the k-th largest of the eights' largest entries is a bound
// that about k entries reach; they are ranked by comparison, and one wave does the rest.
// With top_p the entries of one such bin are ranked.  Rows without a filter take one
// reading with 32-bit sums (sample_open_kernel).
//
// Few rows are bound by what follows one another on a row's own compute unit: the
// reading, 64-bit weights at some 20 instructions each, a dozen barriers (7 x
// 131,072 bf16, top_k 50 with top_p and min_p 23 us; 64 x 32,000 f16, top_p 0.95 35; 255 x 50,001 f32,
// each row its own settings 51; 1 x 32,001 f32 without a filter 8).  Many rows without
// a filter: 1,024 x 131,072 bf16 59 us (268 MB, 4.5 TB/s; memory and vector issue alike, eight issue
// slots an entry) and 24 for the rows that are left uncertain.
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

// The largest number below a key's (0 has two keys).
__device__ __forceinline__ float below(uint32_t k) { return value_of(k - (k == 0x80000000u ? 2u : 1u)); }

// 2^y, 0 <= y < 1, by the exponential's series, to about 1e-15.
__device__ __forceinline__ double exp2_series(double y)
{
    const double z = (y - 0.5) * kLn264;
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
    return s * 1.4142135623730950488;
}

// The exponential between two entries of a table of 2^(j / kTable): the series up
// to the fourth power, |f| <= 1 / 2, is off by 4e-14 at most.  The coefficients
// come as arguments of the kernel, to be operands that are the same for all lanes
// (as literals they cost two instructions each).
constexpr int kTable = 64;
struct Series {
    double a1, a2, a3, a4;
    double magic; // added to a number, it leaves the nearest whole one in the low bits
};
constexpr double kZ = kLn264 / kTable;
constexpr Series kSeries = {kZ, kZ * kZ / 2, kZ * kZ * kZ / 6, kZ * kZ * kZ * kZ / 24, 0x1.8p52};

// What is the same for all lanes, to be kept once a wave.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return uint32_t(__builtin_amdgcn_readfirstlane(int(v))); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ double uniform(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, uint64_t(uniform(uint32_t(b >> 32))) << 32 | uniform(uint32_t(b)));
}

__device__ __forceinline__ uint32_t scan_up(uint32_t v, int lane) // sums over lanes 0 .. lane
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(v, d);
        v += lane >= d ? o : 0u;
    }
    return v;
}
__device__ __forceinline__ double scan_up(double v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(v, d);
        v += lane >= d ? o : 0.0;
    }
    return v;
}
// Entries of the order that stay: those with larger keys, and `ties` with this
// one, by ascending index; n of them in all.
struct Cut {
    uint32_t key, ties, n;
};

constexpr int kBins = 2048;
constexpr int kAhead = 4;  // steps that a wave has in flight
constexpr int kFew = 256;  // top_k up to which the entries are ranked (64 x 131,072 bf16, 256 40 us; 300, searched by key, 49)
constexpr int kList = 512; // entries that can be ranked
constexpr int kBySearch = 4096; // top_k up to which its entries' sum is searched by key alone

// SEGS: segments of a row; BINS: kBins, or 1 where nothing is counted or listed.
template <int WAVES, int SEGS, int BINS>
struct Shared {
    double table[kTable]; // 2^(j / kTable)
    uint32_t count[BINS];
    union {
        uint64_t mass[BINS];
        struct {
            uint64_t list[BINS > 1 ? kList : 1], order[BINS > 1 ? kList : 1];
            double w[BINS > 1 ? kFew : 1];
        } few;
    };
    double sum[SEGS];    // of a segment's w whose keys are above the cut's
    uint32_t tied[SEGS]; // its entries with the cut's key
    double wsum[WAVES];
    uint32_t wcount[WAVES], wmost[WAVES], wleast[WAVES];
    uint32_t at; // first bin from the top that reaches a target
    uint32_t listed;
    struct {
        uint32_t count, above;
        double above_mass;
    } bin;
    struct {
        uint32_t seg, tied;
        double total, before, target;
    } draw;
    bool certain;
};

// S: eights that a lane keeps in registers; 0: the row is read at every look.
template <class T, int WAVES, int S, int BINS = kBins>
struct Row {
    static constexpr int kThreads = WAVES * 64;
    static constexpr int kSegs = S ? S * WAVES : 1024;
    // keys of a type differ above this bit only
    static constexpr int kRes = sizeof(T) == 4 ? 0 : __is_same(T, bf16_t) ? 16 : 13;
    Shared<WAVES, kSegs, BINS> &sh;
    const T *x;
    int64_t V;
    int lane, wave;
    int per, segs; // steps of a segment, segments
    int unit;      // the whole numbers that stand for w are w 2^unit
    Series a;
    float top; // the largest entry
    double c;  // kTable log2 e / T
    float zero;    // entries from here down have a w of 0 (2^-1000, but for the rounding of this bound: 2^-600 at most)
    typename Vec8<T>::type raw[S ? S : 1];
    float largest[S ? S : 1]; // of each eight; S = 0: of the lane's

    // first column of this lane's eight
    __device__ __forceinline__ int64_t column(int seg, int q) const { return (int64_t(seg) * per + q) * kStepCols + lane * kVec; }
    __device__ __forceinline__ void read()
    {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int64_t col = column(s * WAVES + wave, 0);
                raw[s] = load8_raw(x + col, V - col, T(-__builtin_inff()));
            }
        }
    }
    // What is worked out of a row's eights at one look is not kept for the next (the
    // compiler would, in memory).
    static __device__ __forceinline__ typename Vec8<T>::type forget(const typename Vec8<T>::type &r)
    {
        typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) * 2)));
        words w = __builtin_bit_cast(words, r);
        asm volatile("" : "+v"(w));
        return __builtin_bit_cast(typename Vec8<T>::type, w);
    }
    // f(eight's number s, first column, eight values) for every eight of this lane, done(segment) at a segment's
    // end.  With `bound` eights are left out where all of a wave's are below; at the first look (S = 0: with a
    // bound of -infinity) none is, eights of nothing but NaN neither.
    template <class F, class D>
    __device__ __forceinline__ void scan(float bound, F f, D done)
    {
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int seg = s * WAVES + wave;
                if (__ballot(largest[s] >= bound)) {
                    float v[8];
                    widen<T>(forget(raw[s]), v);
                    f(s, column(seg, 0), v);
                }
                done(seg);
            }
        } else {
            // steps of this wave's segments, kAhead of them in flight
            const int mine = wave < segs ? (segs - wave + WAVES - 1) / WAVES : 0;
            const int64_t all = int64_t(mine) * per;
            int seg = wave, q = 0, next_seg = wave, next_q = 0;
            typename Vec8<T>::type next[kAhead];
            auto fetch = [&](int slot) {
                const int64_t col = column(next_seg, next_q);
                next[slot] = load8_raw(x + col, next_seg < segs ? V - col : 0, T(-__builtin_inff()));
                if (++next_q == per) {
                    next_q = 0;
                    next_seg += WAVES;
                }
            };
#pragma unroll
            for (int k = 0; k < kAhead; ++k) fetch(k);
            for (int64_t n = 0; n < all; n += kAhead) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (n + k >= all) break; // uniform
                    const int64_t col = column(seg, q);
                    float v[8], most;
                    widen<T>(next[k], v);
                    fetch(k);
                    most = v[0];
#pragma unroll
                    for (int i = 1; i < kVec; ++i) most = fmaxf(most, v[i]);
                    if (__ballot(!(most < bound))) f(0, col, v); // (NaN is not below)
                    if (++q == per) {
                        done(seg);
                        q = 0;
                        seg += WAVES;
                    }
                }
            }
        }
    }
    // Of entries above `zero`.
    __device__ __forceinline__ double weight(float v) const { return power(double(v) - double(top), c); }
    // 2^y, -1020 < y < 1020.
    __device__ __forceinline__ double power(double y) const { return power(y, kTable); }
    // 2^(d c / kTable)
    __device__ __forceinline__ double power(double d, double c) const
    {
        const double k = fma(d, c, a.magic), f = fma(d, c, a.magic - k);
        const uint32_t n = uint32_t(__builtin_bit_cast(uint64_t, k)); // the nearest whole number to d c
        const uint64_t t = __builtin_bit_cast(uint64_t, sh.table[n % kTable]);
        const double r = fma(fma(fma(fma(f, a.a4, a.a3), f, a.a2), f, a.a1), f, 1.0);
        uint32_t high = uint32_t(t >> 32) + ((n & ~uint32_t(kTable - 1)) << 14); // n / kTable in units of the exponent
        asm volatile("" : "+v"(high)); // else the sum is a 64-bit one
        return __builtin_bit_cast(double, uint64_t(high) << 32 | uint32_t(t)) * r;
    }
    // w, or 0 for what is not above `from`; all eight are worked out, side by side.
    __device__ __forceinline__ void weights(const float v[8], float from, double w[8]) const
    {
#pragma unroll
        for (int i = 0; i < kVec; ++i) w[i] = weight(v[i]);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            asm volatile("" : "+v"(w[i])); // else each becomes a branch, with a wait for its own table entry
            w[i] = v[i] > from ? w[i] : 0.0;
        }
    }
    __device__ __forceinline__ double weight_or_0(float v) const { return v > zero ? weight(v) : 0.0; }

    __device__ __forceinline__ uint32_t block_add(uint32_t v)
    {
        v = wave_add(v);
        __syncthreads();
        if (lane == 0) sh.wcount[wave] = v;
        __syncthreads();
        uint32_t s = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) s += sh.wcount[i];
        return s;
    }

    __device__ __forceinline__ void clear_bins(bool masses)
    {
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            sh.count[b] = 0;
            if (masses) sh.mass[b] = 0;
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
    // The first bin from the top, where entries (or their sum of w, mass_of(bin, its entries)) reach the
    // target, with `above` and `above_mass` before all bins; its place is in sh.at,
    // what it holds and what lies above it in sh.bin.
    template <class M>
    __device__ __forceinline__ void find_bin(bool by_mass, uint32_t target, double target_mass, uint32_t above, double above_mass, M mass_of)
    {
        constexpr int kEach = kBins / kThreads;
        __syncthreads();
        uint32_t n[kEach], before = 0;
        double m[kEach], before_mass = 0.0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const int b = kBins - 1 - (int(threadIdx.x) * kEach + q);
            n[q] = sh.count[b];
            m[q] = by_mass && n[q] ? mass_of(b, n[q]) : 0.0;
            before += n[q];
            before_mass += m[q];
        }
        before = scan_up(before, lane);
        if (by_mass) before_mass = scan_up(before_mass, lane);
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

    // w in units of 2^-bits, the nearest whole number, in the low bits of w + magic(bits).
    static __device__ __forceinline__ double magic_of(int bits)
    {
        return __builtin_bit_cast(double, uint64_t(1023 + 52 - bits) << 52 | uint64_t(1) << 51);
    }
    static __device__ __forceinline__ uint64_t whole(double w, double magic)
    {
        return __builtin_bit_cast(uint64_t, w + magic) - __builtin_bit_cast(uint64_t, magic);
    }

    // The least number of entries with this w, of `most`, that reach the target after `above`.
    static __device__ __forceinline__ uint32_t last_of(double target, double above, double w, uint32_t most)
    {
        double t = w > 0.0 ? fmin(fmax(ceil((target - above) / w), 1.0), double(most)) : 1.0;
        // the division may be off by its last bit
        if (t > 1.0 && above + (t - 1.0) * w >= target) t -= 1.0;
        if (t < double(most) && above + t * w < target) t += 1.0;
        return uint32_t(t);
    }

    // The cut after `target` entries, or after the least number of them whose sum of w reaches
    // `target_mass`, which is known to lie among the `inside` entries with keys from lo
    // to hi, with `above` and `above_mass` before them.  Sums are of whole numbers of 2^-bits, at most 2^50 of them a w
    // and 2^62 in all.
    struct Search {
        uint32_t target;
        double target_mass;
        uint32_t lo, hi, inside, above;
        double above_mass;
        int bits;
    };
    __device__ __forceinline__ Cut select(bool by_mass, const Search &q)
    {
        const uint32_t target = q.target;
        const int bits = q.bits;
        const double target_mass = q.target_mass, magic = magic_of(bits);
        uint32_t lo = q.lo, hi = q.hi, inside = q.inside, above = q.above;
        double above_mass = q.above_mass;
        for (;;) {
            lo = lo >> kRes << kRes;
            int shift = kRes;
            while (((hi - lo) >> shift) >= uint32_t(kBins)) ++shift;
            const bool one = shift == kRes, add = by_mass && !one;
            clear_bins(add);
            const float bound = value_of(umax(lo, kNoneKey + 1));
            scan(
                bound,
                [&](int, int64_t, const float *v) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const uint32_t k = key_of(v[i]);
                        if (k < lo || k > hi || k <= kNoneKey) continue;
                        const uint32_t b = (k - lo) >> shift;
                        atomicAdd(&sh.count[b], 1u);
                        if (add)
                            atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[b]), (unsigned long long)(whole(weight_or_0(v[i]), magic)));
                    }
                },
                [](int) {});
            find_bin(by_mass, target, target_mass, above, above_mass, [&](int b, uint32_t n) {
                return one ? double(n) * weight_or_0(value_of(bin_key(lo, b))) : ldexp(double(sh.mass[b]), -bits);
            });
            // a sum that the rounding of its terms keeps below the target ends with the last of them
            const uint32_t at = uniform(sh.at);
            if (at == kBins) return {lo, ~0u, above + inside};
            const uint32_t b = kBins - 1 - at;
            above = uniform(sh.bin.above);
            above_mass = uniform(sh.bin.above_mass);
            inside = uniform(sh.bin.count);
            if (one) {
                Cut cut;
                cut.key = bin_key(lo, b);
                if (by_mass) {
                    cut.ties = last_of(target_mass, above_mass, weight_or_0(value_of(cut.key)), inside);
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

    // The bin of an entry by its distance from the largest: kBins - 1 at the top, 0 at
    // kSpan bits of w and further down.  The smallest temperatures tell entries apart that are next to
    // 0 or not at all: there the distance is taken 2^100 times.  The largest tell entries apart whose
    // distance 32 bits do not hold: there a quarter of it is taken.
    static constexpr int kSpan = 48;
    struct Distance {
        float far, near, from, scale; // far: 1, 2^100 or 2^-2, near: its reciprocal
    };
    __device__ __forceinline__ Distance distance() const
    {
        const double scale = c * (double(kBins) / (kTable * kSpan));
        const bool cold = scale > 1e38 && fabsf(top) < 0x1p20f, hot = scale < 1e-30;
        const float far = cold ? 0x1p100f : hot ? 0.25f : 1.f, near = cold ? 0x1p-100f : hot ? 4.f : 1.f;
        return {far, near, top * far, float(fmin(scale * double(near), 0x1p127))};
    }
    static __device__ __forceinline__ uint32_t bin_of(float v, const Distance &d)
    {
        return uint32_t(kBins - 1) - uint32_t(fminf(fmaf(v, -d.far, d.from) * d.scale, float(kBins - 1)));
    }
    // No w of a bin passes 2^-shift (but by some 1e-5 of it), and but for bin 0 none is much below half of that.
    static __device__ __forceinline__ uint32_t shift_of(uint32_t bin) { return (kBins - 1 - bin) * uint32_t(kSpan / 16) / uint32_t(kBins / 16); }

    // The cut after the least number of entries whose sum of w reaches the target, or (whole_row) top_p
    // times that of the row: w added up in bins of equal widths, then the entries of
    // the bin that the sum is reached in ranked by comparison.  Where they are too many, what is to be
    // searched for among them: returns true.  The cut stays as it is where nothing is cut off.
    //
    // A bin's unit is 2^-unit of its own largest w, so that an entry is off by 2^-unit of
    // itself at most (what lies in bin 0, by 2^-(unit + 47) of the largest): a sum of V entries by V 2^-61.
    // In one unit for all bins a tail of equal entries could be lost: 59,267 of 59,268 tokens
    // of 131,072 with one entry 31 above and a top_p of 1 - 1e-9.
    __device__ __forceinline__ bool nucleus(bool whole_row, double target, double top_p, Cut &cut, Search &search)
    {
        const Distance dist = distance();
        const uint32_t magic = uint32_t(__builtin_bit_cast(uint64_t, magic_of(unit)) >> 32); // (its low word is 0)
        double rest = 0.0;
        uint32_t further = 0;
        clear_bins(true);
        scan(
            value_of(kNoneKey + 1),
            [&](int, int64_t, const float *v) {
                double w[8];
                weights(v, zero, w);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const uint32_t b = bin_of(v[i], dist);
                    if (b) {
                        atomicAdd(&sh.count[b], 1u);
                        const double m = __builtin_bit_cast(double, uint64_t(magic - (shift_of(b) << 20)) << 32);
                        atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[b]), (unsigned long long)(whole(w[i], m)));
                    } else {
                        rest += w[i];
                        further += v[i] > -__builtin_inff() ? 1u : 0u;
                    }
                }
            },
            [](int) {});
        const uint32_t some = wave_add(further);
        rest = wave_sum64(rest);
        if (lane == 0 && some) {
            atomicAdd(&sh.count[0], some);
            atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[0]), (unsigned long long)(ldexp(rest, unit + int(shift_of(0)))));
        }
        auto mass_of = [&](int b, uint32_t) { return ldexp(double(sh.mass[b]), -unit - int(shift_of(b))); };
        if (whole_row) {
            // the row's sum, in an order of its own
            __syncthreads();
            double all = 0.0;
            for (int b = threadIdx.x; b < kBins; b += kThreads) all += mass_of(b, 0);
            all = wave_sum64(all);
            if (lane == 0) sh.wsum[wave] = all;
            __syncthreads();
            all = 0.0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) all += sh.wsum[i];
            target = uniform(top_p * all);
        }
        find_bin(true, 0, target, 0, 0.0, mass_of);
        const uint32_t first = uniform(sh.at);
        if (first == kBins) return false;
        const uint32_t bin = kBins - 1 - first, L = uniform(sh.bin.count), above = uniform(sh.bin.above);
        const double above_mass = uniform(sh.bin.above_mass);
        // nothing of the bin is below this
        const float low = bin ? top - (float(kBins - bin) * 1.0001f + 1.f) / dist.scale * dist.near : -__builtin_inff();
        const float bound = fmaxf(low, value_of(kNoneKey + 1));
        if (L > uint32_t(kList)) {
            // the bin's keys, no entry of another bin among them
            uint32_t high = 0, not_low = 0;
            scan(
                bound,
                [&](int, int64_t, const float *v) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        if (v[i] > -__builtin_inff() && bin_of(v[i], dist) == bin) {
                            const uint32_t k = key_of(v[i]);
                            high = umax(high, k);
                            not_low = umax(not_low, ~k);
                        }
                    }
                },
                [](int) {});
            high = wave_umax(high);
            not_low = wave_umax(not_low);
            if (lane == 0) {
                sh.wmost[wave] = high;
                sh.wleast[wave] = not_low;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                high = umax(high, sh.wmost[i]);
                not_low = umax(not_low, sh.wleast[i]);
            }
            search = {0, target, uniform(~not_low), uniform(high), L, above, above_mass, unit + int(shift_of(bin))};
            return true;
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        scan(
            bound,
            [&](int, int64_t col, const float *v) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    if (v[i] > -__builtin_inff() && bin_of(v[i], dist) == bin) {
                        const uint32_t at = atomicAdd(&sh.listed, 1u);
                        if (at < kList) sh.few.list[at] = uint64_t(key_of(v[i])) << 32 | uint32_t(~uint32_t(col + i));
                    }
                }
            },
            [](int) {});
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < L; j += kThreads) {
            const uint64_t mine = sh.few.list[j];
            uint32_t rank = 0;
            for (uint32_t i = 0; i < L; ++i) rank += sh.few.list[i] > mine ? 1u : 0u;
            sh.few.order[rank] = mine;
        }
        __syncthreads();
        // in every wave alike
        constexpr int kEach = kList / 64;
        const uint32_t j0 = lane * kEach;
        double w[kEach], mass = 0.0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            w[q] = j0 + q < L ? weight_or_0(value_of(uint32_t(sh.few.order[j0 + q] >> 32))) : 0.0;
            mass += w[q];
        }
        double at = scan_up(mass, lane);
        const double up = __shfl_up(at, 1);
        at = above_mass + (lane ? up : 0.0);
        uint32_t under = 0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            at += w[q];
            under += j0 + q < L && at < target ? 1u : 0u;
        }
        under = wave_add(under);
        under = under < L ? under : L - 1;
        const uint32_t key = uint32_t(sh.few.order[under] >> 32);
        uint32_t ties = 0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) ties += j0 + q <= under && uint32_t(sh.few.order[j0 + q] >> 32) == key ? 1u : 0u;
        cut = {key, wave_add(ties), above + under + 1};
        return false;
    }

    // The same of few entries, those of `cut`: all are to be searched for by key, but for equal ones that the cut ends
    // with, of which there may be many more.  K entries are off by K 2^-51 of the largest.  (64 x
    // 131,072 bf16, top_k 1,000, top_p 0.9 94 us, in bins by distance 129; f32 186 and 183.)
    __device__ __forceinline__ bool among_few(double target, Cut &cut, Search &search)
    {
        const double w = weight_or_0(value_of(cut.key)), above = sh.draw.total - double(cut.ties) * w;
        const uint32_t over = cut.n - cut.ties;
        if (over && target <= above) {
            search = {0, target, cut.key + (1u << kRes), key_of(top), over, 0, 0.0, 50};
            return true;
        }
        cut.ties = last_of(target, above, w, cut.ties);
        cut.n = over + cut.ties;
        return false;
    }

    // Sums of w over what stays, by segment, and over the row (sh.draw.total);
    // then the segment in which the sum passes u times the row's (sh.draw).
    __device__ __forceinline__ void sums(const Cut &cut, double u)
    {
        const float least = value_of(cut.key), from = fmaxf(least, zero);
        double s = 0.0;
        uint32_t e = 0;
        bool some = false;
        __syncthreads();
        scan(
            cut.ties ? least : from,
            [&](int, int64_t, const float *v) {
                some = true;
                double w[8];
                weights(v, from, w);
                s += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                if (cut.ties) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) e += v[i] == least ? 1u : 0u;
                }
            },
            [&](int seg) {
                double all = 0.0;
                uint32_t tied = 0;
                if (some) {
                    all = wave_sum64(s);
                    if (cut.ties) tied = wave_add(e);
                }
                if (lane == 0) {
                    sh.sum[seg] = all;
                    sh.tied[seg] = tied;
                }
                s = 0.0;
                e = 0;
                some = false;
            });
        __syncthreads();
        if (wave == 0) pick(cut, u);
        __syncthreads();
    }
    // The segment in which the sum over the segments passes u times the row's; by one wave.
    __device__ __forceinline__ void pick(const Cut &cut, double u)
    {
        const double wc = cut.ties ? weight_or_0(value_of(cut.key)) : 0.0;
        const int each = (segs + 63) / 64, j0 = lane * each, j1 = j0 + each < segs ? j0 + each : segs;
        uint32_t before = 0;
        if (cut.ties) {
            uint32_t tied = 0;
            for (int j = j0; j < j1; ++j) tied += sh.tied[j];
            before = scan_up(tied, lane) - tied;
        }
        const uint32_t first_tied = before;
        // what stays of a segment's tied entries counts too
        auto mass_of = [&](int j) {
            if (!cut.ties) return sh.sum[j];
            const double m = sh.sum[j] + double(stay(sh.tied[j], before, cut.ties)) * wc;
            before += sh.tied[j];
            return m;
        };
        double mass = 0.0;
        for (int j = j0; j < j1; ++j) mass += mass_of(j);
        const double after = scan_up(mass, lane);
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
                const uint32_t tied = before;
                const double add = mass_of(j);
                if (add > 0.0) {
                    seg = uint32_t(j);
                    seg_tied = tied;
                    seg_at = at;
                    if (at + add > target) break;
                }
                at += add;
            }
            sh.draw.seg = seg;
            sh.draw.tied = seg_tied;
            sh.draw.before = seg_at;
            sh.draw.target = target;
            sh.draw.total = total;
        }
    }
    // How many of `tied` entries stay, with `before` of them before.
    static __device__ __forceinline__ uint32_t stay(uint32_t tied, uint32_t before, uint32_t ties)
    {
        const uint32_t left = before < ties ? ties - before : 0u;
        return tied < left ? tied : left;
    }

    // The token within the segment of sh.draw; by the wave that has the segment.
    __device__ __forceinline__ void draw(const Cut &cut, int32_t *id, float *logp)
    {
        const float least = value_of(cut.key);
        const double target = sh.draw.target;
        double run = sh.draw.before;
        uint32_t tied = sh.draw.tied;
        int64_t found = -1;
        double w_found = 0.0;
        const int seg = __builtin_amdgcn_readfirstlane(int(sh.draw.seg));
        typename Vec8<T>::type mine_raw;
        if constexpr (S > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (seg / WAVES == s) mine_raw = raw[s];
        }
        for (int q = 0; q < per; ++q) {
            const int64_t col = column(seg, q);
            if constexpr (S == 0) mine_raw = load8_raw(x + col, V - col, T(-__builtin_inff()));
            float v[8];
            widen<T>(mine_raw, v);
            uint32_t e = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) e += cut.ties && v[i] == least ? 1u : 0u;
            uint32_t before = scan_up(e, lane);
            const uint32_t step_tied = __shfl(before, 63);
            before += tied - e;
            tied += step_tied;
            double w[8], mine = 0.0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                bool in = v[i] > least;
                if (cut.ties && v[i] == least) in = before++ < cut.ties;
                w[i] = in && v[i] > zero ? weight(v[i]) : 0.0;
                mine += w[i];
            }
            const double after = scan_up(mine, lane);
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

    // A key that at least `target` entries reach and not many more: the lower end of
    // the bin of the target-th largest of the eights' largest (S = 0: of the lanes').
    __device__ __forceinline__ uint32_t bound_of(uint32_t target)
    {
        float mine = largest[0];
#pragma unroll
        for (int s = 1; s < S; ++s) mine = fmaxf(mine, largest[s]);
        // no lane's largest is below lo, so that the bins are as narrow as can be
        uint32_t low = key_of(mine);
        low = low <= kNoneKey ? ~0u : low;
        low = ~wave_umax(~low);
        __syncthreads();
        if (lane == 0) sh.wleast[wave] = low;
        clear_bins(false);
#pragma unroll
        for (int i = 0; i < WAVES; ++i) low = low < sh.wleast[i] ? low : sh.wleast[i];
        const uint32_t lo = low >> kRes << kRes, hi = key_of(top);
        int shift = kRes;
        while (((hi - lo) >> shift) >= uint32_t(kBins)) ++shift;
#pragma unroll
        for (int s = 0; s < (S ? S : 1); ++s) {
            const uint32_t k = key_of(largest[s]);
            if (k >= lo && k > kNoneKey) atomicAdd(&sh.count[(k - lo) >> shift], 1u);
        }
        find_bin(false, target, 0.0, 0, 0.0, [](int, uint32_t) { return 0.0; });
        const uint32_t at = sh.at;
        return at == kBins ? kNoneKey + 1 : umax(lo + ((kBins - 1 - at) << shift), kNoneKey + 1);
    }

    // top_k = K <= kFew: the whole rest of the row, if the entries that reach `bound` fit in the list.
    __device__ __forceinline__ bool few(uint32_t K, uint32_t bound, double top_p, double min_p, double u, int32_t *id, float *logp, int32_t *kept)
    {
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        const float least = value_of(bound);
        scan(
            least,
            [&](int, int64_t col, const float *v) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    if (v[i] >= least) {
                        const uint32_t at = atomicAdd(&sh.listed, 1u);
                        // descending: larger keys first, then smaller indices
                        if (at < kList) sh.few.list[at] = uint64_t(key_of(v[i])) << 32 | uint32_t(~uint32_t(col + i));
                    }
                }
            },
            [](int) {});
        __syncthreads();
        const uint32_t L = sh.listed;
        if (L > kList || L < K) return false; // uniform
        for (uint32_t j = threadIdx.x; j < L; j += kThreads) {
            const uint64_t mine = sh.few.list[j];
            uint32_t rank = 0;
            for (uint32_t i = 0; i < L; ++i) rank += sh.few.list[i] > mine ? 1u : 0u;
            if (rank < kFew) sh.few.order[rank] = mine;
        }
        __syncthreads();
        if (wave) return true;
        constexpr int kEach = kFew / 64;
        const uint32_t j0 = lane * kEach;
        uint64_t e[kEach];
        double w[kEach], mass = 0.0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const bool in = j0 + q < K;
            e[q] = in ? sh.few.order[j0 + q] : 0;
            const float v = value_of(uint32_t(e[q] >> 32));
            w[q] = in && v > zero ? weight(v) : 0.0;
            mass += w[q];
        }
        double at = scan_up(mass, lane);
        const double all = __shfl(at, 63);
        const double before = __shfl_up(at, 1);
        at = lane ? before : 0.0;
        uint32_t n_p = 0, n_q = 0;
        const double target = top_p * all;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            at += w[q];
            const bool in = j0 + q < K;
            n_p += in && at < target ? 1u : 0u;
            n_q += in && w[q] >= min_p ? 1u : 0u;
        }
        if (min_p == 1.0) { // a w just below 1 may be 1 in 64 bits
            n_q = 0;
#pragma unroll
            for (int q = 0; q < kEach; ++q) n_q += j0 + q < K && uint32_t(e[q] >> 32) == key_of(top) ? 1u : 0u;
        }
        n_p = top_p < 1.0 ? wave_add(n_p) + 1u : K;
        n_q = wave_add(n_q);
        uint32_t n = n_p < n_q ? n_p : n_q;
        n = n < K ? n : K;
        // by index: a rank among the n, then sums in that order
        uint32_t rank[kEach];
#pragma unroll
        for (int q = 0; q < kEach; ++q) rank[q] = 0;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t other = uint32_t(sh.few.order[i]); // ~index
#pragma unroll
            for (int q = 0; q < kEach; ++q) rank[q] += other > uint32_t(e[q]) ? 1u : 0u;
        }
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            if (j0 + q < n) {
                sh.few.w[rank[q]] = w[q];
                sh.few.list[rank[q]] = e[q];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        mass = 0.0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            w[q] = j0 + q < n ? sh.few.w[j0 + q] : 0.0;
            mass += w[q];
        }
        const double after = scan_up(mass, lane), up = __shfl_up(after, 1), total = __shfl(after, 63), goal = u * total;
        const uint64_t pass = __ballot(after > goal && mass > 0.0), some = __ballot(mass > 0.0);
        const int who = pass ? __builtin_ctzll(pass) : 63 - __builtin_clzll(some);
        at = lane ? up : 0.0;
        uint32_t which = 0;
        double w_which = 0.0;
        bool over = false;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            at += w[q];
            if (w[q] > 0.0 && !over) {
                which = j0 + q;
                w_which = w[q];
                over = at > goal;
            }
        }
        if (lane == who) {
            *id = int32_t(~uint32_t(sh.few.list[which]));
            if (logp) *logp = float(log(w_which / total));
            if (kept) *kept = int32_t(n);
        }
        return true;
    }
};

struct SampleArgs {
    gwtf_learn_sample_t a;
    int64_t row0;
    int32_t per, segs, unit;
    Series series;
    RecheckWorkspace ws;
};

template <class T, int WAVES, int S>
__global__ __launch_bounds__(WAVES * 64) void sample_kernel(SampleArgs p)
{
    using R = Row<T, WAVES, S>;
    __shared__ Shared<WAVES, R::kSegs, kBins> sh;
    const gwtf_learn_sample_t &a = p.a;
    const int64_t i = p.row0 + blockIdx.x;
    R row{sh, static_cast<const T *>(a.logits) + i * a.logits_stride, a.vocab, int(threadIdx.x & 63),
          __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p.per, S ? R::kSegs : p.segs, p.unit, p.series};
    row.read();
    if (threadIdx.x < kTable) sh.table[threadIdx.x] = threadIdx.x ? exp2_series(double(threadIdx.x) / kTable) : 1.0;
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
    if constexpr (S > 0) {
#pragma unroll
        for (int s = 0; s < S; ++s) row.largest[s] = __builtin_inff(); // all are looked at
    }
    row.scan(
        -__builtin_inff(),
        [&](int s, int64_t, const float *v) {
            float m = v[0];
#pragma unroll
            for (int k = 1; k < kVec; ++k) m = fmaxf(m, v[k]);
#pragma unroll
            for (int k = 0; k < kVec; k += 2) bad = bad || __builtin_isunordered(v[k], v[k + 1]);
#pragma unroll
            for (int k = 0; k < kVec; ++k) there += __popcll(__ballot(v[k] > -__builtin_inff()));
            row.largest[s] = m;
            most = fmaxf(most, m);
        },
        [](int) {});
    {
        if constexpr (S == 0) row.largest[0] = most;
        const uint32_t key = wave_umax(key_of(most)), n = there, wrong = __ballot(bad) != 0;
        if (row.lane == 0) {
            sh.wmost[row.wave] = key;
            sh.wcount[row.wave] = n;
            sh.wleast[row.wave] = wrong;
        }
    }
    __syncthreads();
    uint32_t key = 0, F = 0, wrong = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        key = umax(key, sh.wmost[w]);
        F += sh.wcount[w];
        wrong |= sh.wleast[w];
    }
    key = uniform(key);
    F = uniform(F);
    row.top = value_of(key);
    wrong |= row.top == __builtin_inff();
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
    row.c = uniform(kTable * kLog2e64 / (T_ > 1e-300 ? T_ : 1e-300));
    row.zero = uniform(fminf(float(double(row.top) - kTable * 1000.0 / row.c), below(key)));
    if (T_ == 0.0 || top_k == 1 || top_p == 0.0) {
        cut = {key, 1, 1};
    } else {
        if (top_k > 0 && uint32_t(top_k) < F) {
            const uint32_t lo = row.bound_of(uint32_t(top_k));
            if (top_k <= kFew && row.few(uint32_t(top_k), lo, top_p, min_p, u, a.ids + i, a.logp ? a.logp + i : nullptr, a.kept ? a.kept + i : nullptr))
                return;
            cut = row.select(false, {uint32_t(top_k), 0.0, lo, key, F, 0, 0.0, 0});
        }
        if (top_p < 1.0) {
            const bool whole = cut.n == F;
            if (!whole) {
                row.sums(cut, u);
                summed = true;
            }
            typename R::Search search;
            Cut by_mass = cut;
            const double target = top_p * sh.draw.total; // (not of the whole row)
            bool left;
            if (!whole && cut.n <= uint32_t(kBySearch)) left = row.among_few(target, by_mass, search);
            else left = row.nucleus(whole, target, top_p, by_mass, search);
            if (left) by_mass = row.select(true, search);
            if (by_mass.n < cut.n) {
                cut = by_mass;
                summed = false;
            }
        }
        if (min_p > 0.0) {
            // the smallest 32-bit number whose w reaches min_p
            const double at = double(row.top) + kTable * log2(min_p) / row.c;
            float least = float(at);
            if (double(least) < at) least = value_of(key_of(least) + 1);
            uint32_t n = 0;
            row.scan(
                least,
                [&](int, int64_t, const float *v) {
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
    if (row.wave == int(sh.draw.seg % WAVES)) row.draw(cut, a.ids + i, a.logp ? a.logp + i : nullptr);
    if (threadIdx.x == 0 && a.kept) a.kept[i] = int32_t(cut.n);
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Rows of which everything stays (no top_k, top_p or min_p): one reading, with the
// sums of segments in 32 bits, of 2^y, y = x c - r in one fused operation, c = log2 e /
// T in 32 bits and r the product of c and the largest entry that the segment's wave has
// met, or a little less: no y is above kAbove + 1.  Then the one segment that the target
// falls into in 64 bits.
//
// The token is that of 64-bit sums if the target is further from the borders of
// the token than the 32-bit sums can be off.  With A the sum up to a border, B the sum
// after it and W = A + B, the border lies at (1 - u) A - u B from the target.  Of
// A's terms each is off by its y's two roundings (of y, and of c, whose effect at y = 0
// is in the segment's factor), the exponential's 2^-23 and the ten additions': 2^-24 (2 ln
// 2 |y| + 12) relatively.  |y| is at most kAbove + 1 + |log2 w|, w = 2^((x - max x) log2 e /
// T), and the mean of -log2 w under the shares w / A is their entropy less log2 A, log2
// V - log2 A at most.  So A is off by at most A 2^-24 (2 ln 2 (log2 V - log2 A + kAbove +
// 1) + 12), B likewise, and near a border A = u W, B = (1 - u) W.
// Otherwise (one row in twenty of normal logits of deviation 2.5 and 131,072 columns),
// and where the largest x c is beyond kRange, the sums are taken again in 64 bits.  r is
// never below -kRange, so that entries further down, masks of -1e30 among them, add
// nothing.
constexpr float kRange = 0x1p17f;
constexpr float kAbove = 1.f;
constexpr int kOpenPer = 2;                              // steps of a segment
constexpr int64_t kOpenMost = 1024 * kOpenPer * kStepCols; // columns

// The token within the segment of sh.draw, whose sum in 64 bits takes the place of that
// in 32 (by one wave).  Returns whether the token is certain.
template <class R>
__device__ __forceinline__ bool draw_open(const R &row, double u, int32_t *id, float *logp)
{
    const auto &sh = row.sh;
    const int seg = __builtin_amdgcn_readfirstlane(int(sh.draw.seg)), lane = row.lane;
    const double begin = sh.draw.before;
    double w[kOpenPer][8], after[kOpenPer], sum = 0.0;
#pragma unroll
    for (int k = 0; k < kOpenPer; ++k) {
        const int64_t col = row.column(seg, k);
        float v[8];
        load8(row.x + col, row.V - col, v, -__builtin_inff());
        row.weights(v, row.zero, w[k]);
        after[k] = scan_up(((w[k][0] + w[k][1]) + (w[k][2] + w[k][3])) + ((w[k][4] + w[k][5]) + (w[k][6] + w[k][7])), lane) + sum;
        sum = __shfl(after[k], 63); // of the segment so far
    }
    const double W = sh.draw.total - sh.sum[seg] + sum, target = u * W;
    double gap = 0.0, w_found = 0.0;
    int64_t found = -1;
#pragma unroll
    for (int k = 0; k < kOpenPer; ++k) {
        const uint64_t pass = __ballot(begin + after[k] > target);
        if (!pass || found >= 0) continue;
        const int who = __builtin_ctzll(pass);
        const double up = __shfl_up(after[k], 1), before = k ? __shfl(after[k ? k - 1 : 0], 63) : 0.0;
        double at = begin + (lane ? up : before), left = at, right = at, mine = 0.0;
        int which = -1;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const double next = at + w[k][i];
            if (which < 0 && next > target) {
                which = i;
                left = at;
                right = next;
                mine = w[k][i];
            }
            at = next;
        }
        // a sum of nothing is no border
        const double g = which < 0 ? 0.0 : fmin(right - target, left > 0.0 ? target - left : right - target);
        gap = __shfl(g, who);
        w_found = __shfl(mine, who);
        found = __shfl(row.column(seg, k) + which, who);
    }
    if (lane == 0 && found >= 0) {
        *id = int32_t(found);
        if (logp) *logp = float(log(w_found / W));
    }
    const double v = fmin(u, 1.0), A = v * W, B = W - A, span = log2(double(row.V)) + kAbove + 1;
    // (A and B themselves are known to a hundred thousandth)
    const double off_a = A > 0.0 ? 2 * kLn264 * (span - log2(A)) + 12 : 0.0, off_b = B > 0.0 ? 2 * kLn264 * (span - log2(B)) + 12 : 0.0;
    return found >= 0 && gap > 0x1.02p-24 * ((1.0 - v) * A * off_a + v * B * off_b) + 1e-13 * W;
}

// LEAVE: uncertain rows are left to another launch.
template <class T, int WAVES, bool LEAVE>
__global__ __launch_bounds__(WAVES * 64) void sample_open_kernel(SampleArgs p)
{
    using R = Row<T, WAVES, 0, 1>;
    constexpr int kCols = kOpenPer * kStepCols;
    __shared__ Shared<WAVES, R::kSegs, 1> sh;
    __shared__ float2 part[R::kSegs]; // a segment's sum and its r
    const gwtf_learn_sample_t &a = p.a;
    const int64_t i = p.row0 + blockIdx.x;
    R row{sh, static_cast<const T *>(a.logits) + i * a.logits_stride, a.vocab, int(threadIdx.x & 63),
          __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kOpenPer, p.segs, p.unit, p.series};
    const int each = (p.segs + WAVES - 1) / WAVES, first = row.wave * each;
    const int end = first + each < p.segs ? first + each : p.segs, whole = int(a.vocab / kCols); // segments without an end of the row
    typename Vec8<T>::type raw[2][kOpenPer];
    auto fetch = [&](int seg, int slot) {
        if (seg >= end) return;
        const T *from = row.x + int64_t(seg) * kCols + row.lane * kVec;
#pragma unroll
        for (int k = 0; k < kOpenPer; ++k) {
            if (seg < whole) raw[slot][k] = *reinterpret_cast<const typename Vec8<T>::type *>(from + k * kStepCols);
            else raw[slot][k] = load8_raw(from + k * kStepCols, a.vocab - int64_t(seg) * kCols - k * kStepCols - row.lane * kVec, T(-__builtin_inff()));
        }
    };
    fetch(first, 0);
    fetch(first + 1, 1);
    if (threadIdx.x < kTable) sh.table[threadIdx.x] = threadIdx.x ? exp2_series(double(threadIdx.x) / kTable) : 1.0;
    double u = a.uniform_type == GWTF_UNIFORM_F64 ? static_cast<const double *>(a.u)[i] : double(static_cast<const float *>(a.u)[i]);
    u = u >= 0.0 ? u : 0.0;
    row.c = kTable * kLog2e64 / a.temperature;
    const double c = kLog2e64 / a.temperature;
    const float c32 = float(c);

    float most = -__builtin_inff(), ref = -kRange;
    uint32_t there = 0;
    bool bad = false;
    for (int seg = first; seg < end; seg += 2) {
#pragma unroll
        for (int slot = 0; slot < 2; ++slot) {
            if (seg + slot >= end) break; // uniform
            float v[kOpenPer][8], m = -__builtin_inff(), l = __builtin_inff();
#pragma unroll
            for (int k = 0; k < kOpenPer; ++k) {
                widen<T>(raw[slot][k], v[k]);
#pragma unroll
                for (int q = 0; q < kVec; q += 2) {
                    m = max3(m, v[k][q], v[k][q + 1]);
                    l = min3(l, v[k][q], v[k][q + 1]);
                }
            }
            fetch(seg + slot + 2, slot);
            most = fmaxf(most, m);
            if (__ballot(fmaf(m, c32, -ref) > kAbove)) ref = wave_fmax(m) * c32;
            if (__ballot(l == -__builtin_inff())) {
#pragma unroll
                for (int k = 0; k < kOpenPer; ++k) {
#pragma unroll
                    for (int q = 0; q < kVec; ++q) there += __popcll(__ballot(v[k][q] > -__builtin_inff()));
                }
            } else {
                there += kCols;
            }
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kOpenPer; ++k) {
#pragma unroll
                for (int q = 0; q < kVec; ++q) v[k][q] = exp2_(fmaf(v[k][q], c32, -ref));
                s += ((v[k][0] + v[k][1]) + (v[k][2] + v[k][3])) + ((v[k][4] + v[k][5]) + (v[k][6] + v[k][7]));
            }
            s = wave_sum(s);
            bad = bad || s != s; // a NaN, or +infinity less itself
            if (row.lane == 0) part[seg + slot] = {s, ref};
        }
    }
    {
        const uint32_t key = wave_umax(key_of(most));
        if (row.lane == 0) {
            sh.wmost[row.wave] = key;
            sh.wcount[row.wave] = there;
            sh.wleast[row.wave] = bad;
        }
    }
    __syncthreads();
    uint32_t key = 0, F = 0, wrong = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        key = umax(key, sh.wmost[w]);
        F += sh.wcount[w];
        wrong |= sh.wleast[w];
    }
    row.top = value_of(key);
    wrong |= row.top == __builtin_inff();
    if (wrong || F == 0) {
        if (threadIdx.x == 0) {
            a.ids[i] = -1;
            if (a.logp) a.logp[i] = wrong ? __builtin_nanf("") : -__builtin_inff();
            if (a.kept) a.kept[i] = 0;
            if (LEAVE) p.ws.key[i] = 0;
        }
        return;
    }
    row.zero = fminf(float(double(row.top) - kTable * 1000.0 / row.c), below(key));
    const Cut cut = {kNoneKey, 0, F};
    if (threadIdx.x == 0 && a.kept) a.kept[i] = int32_t(F);
    if (row.wave == 0) {
        const double per32 = c / double(c32), highest = double(row.top) * c;
        for (int seg = row.lane; seg < p.segs; seg += 64) {
            const double y = double(part[seg].y) * per32 - highest;
            sh.sum[seg] = y > -1000.0 ? double(part[seg].x) * row.power(y) : 0.0;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        row.pick(cut, u);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        const bool certain = draw_open(row, u, a.ids + i, a.logp ? a.logp + i : nullptr);
        if (row.lane == 0) {
            sh.certain = certain && fabs(highest) < kRange;
            if (LEAVE) p.ws.key[i] = sh.certain ? 0u : key;
        }
    }
    if constexpr (!LEAVE) {
        __syncthreads();
        if (sh.certain) return;
        row.sums(cut, u);
        if (row.wave == 0) row.draw(cut, a.ids + i, a.logp ? a.logp + i : nullptr);
    }
}

// The rows that sample_open_kernel has left, in 64 bits: each shared by kParts workgroups,
// of which the last to arrive draws.  (By the workgroup that finds its row uncertain,
// 20 us after all others have ended: 1,024 rows of 131,072 109 us.)
constexpr int kParts = 8;

template <class T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sample_recheck_kernel(SampleArgs p)
{
    using R = Row<T, WAVES, 0, 1>;
    __shared__ Shared<WAVES, R::kSegs, 1> sh;
    __shared__ uint16_t rows[kRecheckRows];
    const gwtf_learn_sample_t &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the rows that are left, in their order
    constexpr int kEach = kRecheckRows / (WAVES * 64);
    const int r0 = threadIdx.x * kEach, N = int(a.num_tokens);
    static_assert(kEach == 8, "two reads of four rows");
    const uint4 k0 = reinterpret_cast<const uint4 *>(p.ws.key + r0)[0], k1 = reinterpret_cast<const uint4 *>(p.ws.key + r0)[1];
    const uint32_t keys[8] = {k0.x, k0.y, k0.z, k0.w, k1.x, k1.y, k1.z, k1.w}; // (of rows from N on, left by another call)
    uint32_t mine = 0;
#pragma unroll
    for (int q = 0; q < kEach; ++q) mine += r0 + q < N && keys[q] != 0;
    const uint32_t upto = scan_up(mine, lane);
    if (lane == 63) sh.wcount[wave] = upto;
    if (threadIdx.x < kTable) sh.table[threadIdx.x] = threadIdx.x ? exp2_series(double(threadIdx.x) / kTable) : 1.0;
    __syncthreads();
    uint32_t at = upto - mine, left = 0;
    for (int w = 0; w < WAVES; ++w) {
        at += w < wave ? sh.wcount[w] : 0u;
        left += sh.wcount[w];
    }
#pragma unroll
    for (int q = 0; q < kEach; ++q)
        if (r0 + q < N && keys[q] != 0) rows[at++] = uint16_t(r0 + q);
    __syncthreads();
    // the first kRecheckSlots in parts, others whole
    const uint32_t shared = left < uint32_t(kRecheckSlots) ? left : uint32_t(kRecheckSlots), items = shared * kParts + (left - shared);
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const bool whole = item >= shared * kParts;
        const uint32_t slot = whole ? shared + (item - shared * kParts) : item / kParts;
        const int part = whole ? 0 : int(item % kParts);
        const int64_t i = rows[slot];
        R row{sh, static_cast<const T *>(a.logits) + i * a.logits_stride, a.vocab, lane, wave, p.per, p.segs, p.unit, p.series};
        const uint32_t key = p.ws.key[i];
        row.top = value_of(key);
        row.c = kTable * kLog2e64 / a.temperature;
        row.zero = fminf(float(double(row.top) - kTable * 1000.0 / row.c), below(key));
        double u = a.uniform_type == GWTF_UNIFORM_F64 ? static_cast<const double *>(a.u)[i] : double(static_cast<const float *>(a.u)[i]);
        u = u >= 0.0 ? u : 0.0;
        const Cut cut = {kNoneKey, 0, 1};
        if (whole) {
            row.sums(cut, u);
        } else {
            uint64_t *const sums = p.ws.sum + int64_t(slot) * R::kSegs;
            const int each = (p.segs + kParts - 1) / kParts, end = (part + 1) * each < p.segs ? (part + 1) * each : p.segs;
            typename Vec8<T>::type raw[kOpenPer], next[kOpenPer];
            auto fetch = [&](int seg) {
#pragma unroll
                for (int k = 0; k < kOpenPer; ++k) {
                    const int64_t col = row.column(seg, k);
                    next[k] = load8_raw(row.x + col, seg < end ? a.vocab - col : 0, T(-__builtin_inff()));
                }
            };
            fetch(part * each + wave);
            for (int seg = part * each + wave; seg < end; seg += WAVES) {
                double s = 0.0;
#pragma unroll
                for (int k = 0; k < kOpenPer; ++k) raw[k] = next[k];
                fetch(seg + WAVES);
#pragma unroll
                for (int k = 0; k < kOpenPer; ++k) {
                    float v[8];
                    double w[8];
                    widen<T>(raw[k], v);
                    row.weights(v, row.zero, w);
                    s += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                }
                s = wave_sum64(s);
                if (lane == 0) __hip_atomic_store(sums + seg, __builtin_bit_cast(uint64_t, s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            // sums and counter are words of agent scope; the waits put the sums in memory
            // before the arrival is counted
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0)
                sh.certain = __hip_atomic_fetch_add(p.ws.arrived + slot, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == uint32_t(kParts - 1);
            __syncthreads();
            const bool last = sh.certain;
            __syncthreads();
            if (!last) continue;
            for (int seg = threadIdx.x; seg < p.segs; seg += WAVES * 64)
                sh.sum[seg] = __builtin_bit_cast(double, __hip_atomic_load(sums + seg, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            if (threadIdx.x == 0) p.ws.arrived[slot] = 0;
            __syncthreads();
            if (wave == 0) row.pick(cut, u);
            __syncthreads();
        }
        if (wave == 0) row.draw(cut, a.ids + i, a.logp ? a.logp + i : nullptr);
        __syncthreads();
    }
}

template <class T, int WAVES, int S>
hipError_t run(const gwtf_learn_sample_t &a, hipStream_t s)
{
    SampleArgs p;
    p.a = a;
    p.series = kSeries;
    const int64_t steps = (a.vocab + kStepCols - 1) / kStepCols, most = Row<T, WAVES, S>::kSegs;
    p.per = int32_t((steps + most - 1) / most);
    p.segs = int32_t((steps + p.per - 1) / p.per);
    p.unit = 62;
    while ((int64_t(1) << (62 - p.unit)) < a.vocab) --p.unit;
    p.unit = p.unit < 50 ? p.unit : 50;
    const int64_t slab = kLaunchThreads / (WAVES * 64);
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        p.row0 = r;
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        const hipError_t e = launch(sample_kernel<T, WAVES, S>, n, WAVES * 64, s, p);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, int WAVES, bool LEAVE>
hipError_t run_open(const gwtf_learn_sample_t &a, const RecheckWorkspace &ws, hipStream_t s)
{
    SampleArgs p;
    p.a = a;
    p.ws = ws;
    p.series = kSeries;
    p.per = kOpenPer;
    p.segs = int32_t((a.vocab + kOpenPer * kStepCols - 1) / (kOpenPer * kStepCols));
    p.unit = 0;
    const int64_t slab = kLaunchThreads / (WAVES * 64);
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        p.row0 = r;
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        const hipError_t e = launch(sample_open_kernel<T, WAVES, LEAVE>, n, WAVES * 64, s, p);
        if (e != hipSuccess) return e;
    }
    if constexpr (LEAVE) return launch(sample_recheck_kernel<T, 8>, kRecheckGroups, 512, s, p);
    return hipSuccess;
}

// How many waves take a row, and how many eights a lane keeps.  Few waves leave room for other rows on a
// compute unit, many end one row sooner; this way and the other (us, bf16 if nothing else is said):
//   no filter, 4 waves to 16,384 columns: 1,024 rows of 4,096 13.0, of 16,384 21.5 (16 waves 18.4, 24.3; 64 rows
//     10.4 and 9.3); beyond, 64 rows of 32,768 15.4, 1,024 29.6 (4 waves 19.4, 34.5)
//   no filter, 16 waves for no more rows than the card has compute units: 64 rows of 20,000 15.3, 256 16.3 (8 waves
//     16.8, 18.0); from there on 8: 512 rows 21.0, 1,024 26.2 (26.8, 39.8).  At 131,072 columns 8 waves and
//     the second launch would be ahead for few rows too: 64 rows 43, with them 27
//   filters, 4 waves of one eight to 2,048: 1,024 rows of 1,000 with top_p 20.5 (of four eights 32.9)
//   4 waves to 8,192: 1,024 rows of 4,096 with top_p 39, with top_k 50 22 (16 waves 73, 46; 64 rows of 8,192 with top_p
//     24 and 22)
//   16 waves beyond: 64 rows of 16,384 with top_p 27, 1,024 100 (4 waves of eight eights 36, 75)
//   16 eights in registers to 131,072 of 16 bits: 64 rows with top_p 105, of 152,064, read at every look, 132
constexpr int64_t kFewRows = 256;

template <class T>
hipError_t by_width(const gwtf_learn_sample_t &a, const RecheckWorkspace &ws, hipStream_t s)
{
    const int64_t V = a.vocab;
    // 32-bit sums need a temperature whose quotients stay within 32 bits
    const bool open = !a.temperatures && !a.top_ks && !a.top_ps && !a.min_ps && a.top_k <= 0 && a.top_p >= 1.0 && a.min_p == 0.0 &&
                      a.temperature > 1e-30 && a.temperature < 1e30;
    if (open && V <= kOpenMost) {
        if (V <= 16384) return run_open<T, 4, false>(a, ws, s);
        if (a.num_tokens <= kFewRows) return run_open<T, 16, false>(a, ws, s);
        // rows for all of the card: uncertain ones are shared out at the end
        return a.num_tokens <= kRecheckRows ? run_open<T, 8, true>(a, ws, s) : run_open<T, 8, false>(a, ws, s);
    }
    if (V <= 2048) return run<T, 4, 1>(a, s);
    if (V <= 8192) return run<T, 4, 4>(a, s);
    if (V <= 32768) return run<T, 16, 4>(a, s);
    if (V <= 65536) return run<T, 16, 8>(a, s);
    if constexpr (sizeof(T) == 2)
        if (V <= 131072) return run<T, 16, 16>(a, s);
    return run<T, 16, 0>(a, s);
}

} // namespace

hipError_t launch_sample(const gwtf_learn_sample_t &a, const LearnWorkspace &w, hipStream_t s)
{
    switch (a.type) {
    case GWTF_TYPE_F32: return by_width<float>(a, w.recheck, s);
    case GWTF_TYPE_F16: return by_width<f16_t>(a, w.recheck, s);
    default: return by_width<bf16_t>(a, w.recheck, s);
    }
}

} // namespace gwtf
