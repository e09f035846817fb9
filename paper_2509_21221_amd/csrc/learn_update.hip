// Update phase of a node: the norm of its gradients (gwtf_learn_grad_norm) and
// the AdamW step over its parameters (gwtf_learn_adamw).
//
//   g = factor grad, m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2
//   p = p - lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay p)
//
// Tensors come as a table on the device.  A workgroup takes chunks of 2048 values (the
// step one each) and finds a chunk's tensor in two reads that are the same for all
// its lanes: any number of tensors is one launch (301 of odd sizes 27 us; as lists in the
// kernel's arguments, 50 a launch, 70).
//
// Bound by memory: 38 million bf16 weights with 32-bit copies, states and gradients 208 us
// (1.13 GB, 5.5 TB/s), 201 million with 8-bit states 397 us (2.04 GB, 5.1 TB/s), where vector
// issue takes as long: 84 instructions a value, 27 of them the generator's, which
// serves m and v with the same 16 bits.  With divisions and exact roots in place of the
// hardware's 542 us.  The norm of 201 million bf16 70 us (5.8 TB/s).
#include "learn_internal.h"
#include "stage_device.h"

#include <cmath>
#include <new>

namespace gwtf {
namespace {

// ---- Norm ----

constexpr int kNormArrivals = 256;

struct NormArgs {
    int64_t begin, end; // chunks
    double *partial;    // of all launches; this one's from `first` on
    uint32_t *arrived;  // 0 between calls
    int32_t first;
    uint32_t last; // number of the arrival that joins; 0: another launch follows
    double max_norm, scale;
    float *norm, *factor;
};

// partial[first + workgroup] = sum of squares of the chunks begin + blockIdx.x, begin +
// blockIdx.x + gridDim.x, ..; in the last launch the workgroup that arrives last
// joins all of them, in their order.  Sums and counter are words of agent scope, and
// the wait puts a sum in memory before its arrival is counted.  Arrivals follow one another
// 8 ns apart: with more than kNormArrivals workgroups a launch of its own joins (few
// thousand values 6.8 us by arrival, 10.4 by another launch; 201 million 82 and 70).
template <class T>
__global__ __launch_bounds__(256) void norm_kernel(const LearnEntry *__restrict__ entry, const uint32_t *__restrict__ owner, NormArgs a)
{
    __shared__ double red[4];
    __shared__ bool joins;
    double sum = 0.0;
    // one chunk at a time: 201 million bf16 70 us; with two, four and eight in flight 71, 77 and 83
    for (int64_t chunk = a.begin + blockIdx.x; chunk < a.end; chunk += gridDim.x) {
        const LearnEntry &t = entry[owner[chunk]];
        const int64_t i = (chunk - t.first) * kChunk + threadIdx.x * kVec;
        float v[8];
        load8(static_cast<const T *>(t.grad) + i, t.size - i, v);
#pragma unroll
        for (int q = 0; q < kVec; ++q) sum = fma(double(v[q]), double(v[q]), sum);
    }
    sum = wave_sum64(sum);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = (red[0] + red[1]) + (red[2] + red[3]);
        __hip_atomic_store(reinterpret_cast<uint64_t *>(a.partial + a.first + blockIdx.x), __builtin_bit_cast(uint64_t, sum), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        joins = a.last && __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == a.last;
    }
    __syncthreads();
    if (!joins) return;
    const int count = a.first + int(gridDim.x);
    sum = 0.0;
    for (int i = threadIdx.x; i < count; i += 256)
        sum += __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const uint64_t *>(a.partial + i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    sum = wave_sum64(sum);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    *a.arrived = 0;
    const double n = a.scale * sqrt((red[0] + red[1]) + (red[2] + red[3]));
    const float norm = float(n); // infinite where 32 bits do not hold it: no gradient is to be clipped by such
    if (a.norm) *a.norm = norm;
    if (a.factor) *a.factor = norm < __builtin_inff() ? float(n > a.max_norm ? a.scale * (a.max_norm / n) : a.scale) : __builtin_nanf("");
}

__global__ void norm_of_nothing_kernel(float scale, float *norm, float *factor)
{
    if (norm) *norm = 0.f;
    if (factor) *factor = scale;
}

// ---- AdamW ----

struct AdamArgs {
    const LearnEntry *entry;
    const uint32_t *owner;
    int64_t begin; // chunk of the first workgroup
    float lr, beta1, rest1, beta2, rest2, eps, unbias1, unbias2;
    uint32_t k0, k1;
    double log_beta1, log_beta2;
    int64_t step;
    const int64_t *step_at;
    const float *lr_at, *factor;
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(1)));

// Eight 8-bit values as two words, zeros past the end.
__device__ __forceinline__ u32x2 load_f8(const uint8_t *p, int64_t n)
{
    u32x2 w = {0, 0};
    if (n >= kVec) return *reinterpret_cast<const u32x2 *>(p);
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < n) w[i / 4] |= uint32_t(p[i]) << (8 * (i & 3));
    return w;
}
__device__ __forceinline__ void store_f8(uint8_t *p, int64_t n, u32x2 w)
{
    if (n >= kVec) {
        *reinterpret_cast<u32x2 *>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < n) p[i] = uint8_t(w[i / 4] >> (8 * (i & 3)));
}
template <bool E5M2>
__device__ __forceinline__ void widen_f8(u32x2 w, float scale, float v[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8(int(w[i]), false) : __builtin_amdgcn_cvt_pk_f32_fp8(int(w[i]), false);
        const auto hi = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8(int(w[i]), true) : __builtin_amdgcn_cvt_pk_f32_fp8(int(w[i]), true);
        v[4 * i] = lo[0] * scale;
        v[4 * i + 1] = lo[1] * scale;
        v[4 * i + 2] = hi[0] * scale;
        v[4 * i + 3] = hi[1] * scale;
    }
}

// Eight values in 8 bits under the scale of their block of 128 (16 lanes), and
// the scale.  Of a 32-bit value's mantissa CUT bits are left out: adding r there
// carries into what is kept with the probability of the remainder; below the
// smallest normal value the steps are equal.  Of v (E5M2) nothing above 0 becomes 0.
template <bool E5M2>
__device__ __forceinline__ u32x2 narrow_f8(const float x[8], const uint32_t r[8], float &scale)
{
    constexpr int CUT = E5M2 ? 21 : 20, BIAS = E5M2 ? 112 << 2 : 120 << 3, TOP = E5M2 ? 142 : 135;
    constexpr float UNIT = E5M2 ? 0x1p16f : 0x1p9f, NORMAL = E5M2 ? 0x1p-14f : 0x1p-6f;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) most = umax(most, __float_as_uint(x[i]) & 0x7fffffffu);
    most = row_umax(most);
    u32x2 w = {0, 0};
    if (most >= 0x7f800000u) {
        scale = __builtin_nanf("");
        return w;
    }
    // the exponent that puts the largest at or below 1.75 times the code's largest power of two
    const int e = int((most + 0x1fffffu) >> 23) - TOP, at = e > -126 ? e : -126;
    scale = __uint_as_float(uint32_t(at + 127) << 23);
    const float up = __uint_as_float(uint32_t(127 - at) << 23);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float a = __builtin_fabsf(x[i]) * up;
        const uint32_t large = ((__float_as_uint(a) + (r[i] << (CUT - 16)) + (1u << (CUT - 17))) >> CUT) - BIAS;
        uint32_t small = uint32_t(a * UNIT + (float(r[i]) + 0.5f) * 0x1p-16f);
        if (E5M2 && x[i] > 0.f && small == 0) small = 1; // (its magnitude under the scale may be 0 in 32 bits)
        uint32_t c = a >= NORMAL ? large : small;
        if (!E5M2) c |= (__float_as_uint(x[i]) >> 24) & (c ? 0x80u : 0u);
        w[i / 4] |= c << (8 * (i & 3));
    }
    return w;
}

// The root, to its last bit or so; the hardware's knows no values below 2^-126.
__device__ __forceinline__ float root(float x)
{
    const bool small = x < 0x1p-96f;
    const float r = __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x);
    return small ? r * 0x1p-32f : r;
}

template <class T, class G, bool F8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a)
{
    // m and v follow the formula one rounding an operation, so that 8-bit states
    // are the same wherever the step is repeated
#pragma clang fp contract(off)
    const int64_t chunk = a.begin + blockIdx.x;
    const LearnEntry t = a.entry[a.owner[chunk]];
    const float factor = a.factor ? *a.factor : 1.f;
    if (!(__builtin_fabsf(factor) < __builtin_inff())) return;
    const float lr = a.lr_at ? *a.lr_at : a.lr;
    if (!(__builtin_fabsf(lr) < __builtin_inff())) return;
    int64_t step = a.step;
    float unbias1 = a.unbias1, unbias2 = a.unbias2; // 1 / (1 - beta^step)
    if (a.step_at) {
        step = *a.step_at;
        if (step < 1) return;
        unbias1 = float(-1.0 / expm1(double(step) * a.log_beta1));
        unbias2 = float(-1.0 / expm1(double(step) * a.log_beta2));
    }
    const int64_t i = (chunk - t.first) * kChunk + threadIdx.x * kVec, n = t.size - i;
    float g[8], p[8], m[8], v[8];
    load8(static_cast<const G *>(t.grad) + i, n, g);
    if (t.master) load8(t.master + i, n, p);
    else load8(static_cast<const T *>(t.param) + i, n, p);
    if constexpr (F8) {
        const bool in = n > 0;
        widen_f8<false>(load_f8(static_cast<const uint8_t *>(t.m) + i, n), in ? t.m_scale[i / GWTF_STATE_BLOCK] : 0.f, m);
        widen_f8<true>(load_f8(static_cast<const uint8_t *>(t.v) + i, n), in ? t.v_scale[i / GWTF_STATE_BLOCK] : 0.f, v);
    } else {
        load8(static_cast<const float *>(t.m) + i, n, m);
        load8(static_cast<const float *>(t.v) + i, n, v);
    }
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        g[k] = g[k] * factor;
        m[k] = m[k] * a.beta1 + g[k] * a.rest1;
        v[k] = v[k] * a.beta2 + g[k] * g[k] * a.rest2;
        const float den = root(v[k] * unbias2) + a.eps;
        const float d = m[k] * unbias1 * __builtin_amdgcn_rcpf(den < 0x1p-126f ? 0x1p-126f : den);
        p[k] = p[k] - lr * (d + t.decay * p[k]);
    }
    store8(static_cast<T *>(t.param) + i, n, p);
    if (t.master) store8(t.master + i, n, p);
    if constexpr (F8) {
        // values past the end have no part in the scale of the last block
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            m[k] = k < n ? m[k] : 0.f;
            v[k] = k < n ? v[k] : 0.f;
        }
        uint32_t c[4] = {uint32_t(i / kVec), t.site, uint32_t(step), uint32_t(uint64_t(step) >> 32)}, r[8];
        philox4x32(a.k0, a.k1, c);
#pragma unroll
        for (int k = 0; k < kVec; ++k) r[k] = (k & 1) ? c[k / 2] >> 16 : c[k / 2] & 0xffffu;
        float sm, sv;
        const u32x2 wm = narrow_f8<false>(m, r, sm), wv = narrow_f8<true>(v, r, sv);
        store_f8(static_cast<uint8_t *>(t.m) + i, n, wm);
        store_f8(static_cast<uint8_t *>(t.v) + i, n, wv);
        if (n > 0 && i % GWTF_STATE_BLOCK == 0) {
            t.m_scale[i / GWTF_STATE_BLOCK] = sm;
            t.v_scale[i / GWTF_STATE_BLOCK] = sv;
        }
    } else {
        store8(static_cast<float *>(t.m) + i, n, m);
        store8(static_cast<float *>(t.v) + i, n, v);
    }
}

using AdamKernel = void (*)(AdamArgs);
template <bool F8>
AdamKernel adamw_of(int type, int grad_type)
{
    const bool wide = grad_type == GWTF_TYPE_F32;
    switch (type) {
    case GWTF_TYPE_F32: return adamw_kernel<float, float, F8>;
    case GWTF_TYPE_F16: return wide ? adamw_kernel<f16_t, float, F8> : adamw_kernel<f16_t, f16_t, F8>;
    default: return wide ? adamw_kernel<bf16_t, float, F8> : adamw_kernel<bf16_t, bf16_t, F8>;
    }
}

} // namespace

hipError_t build_table(int64_t num, const gwtf_learn_tensor_t *tensors, LearnTable &t)
{
    // classes of types, then the tensors of each in the order of the list
    const int kinds = 9;
    auto kind_of = [&](const gwtf_learn_tensor_t &x) { return t.form == GWTF_STATE_NONE ? x.grad_type : 3 * x.grad_type + x.type; };
    int64_t chunks = 0, used = 0;
    for (int64_t i = 0; i < num; ++i) {
        chunks += (tensors[i].size + kChunk - 1) / kChunk;
        used += tensors[i].size != 0;
    }
    const size_t entries = sizeof(LearnEntry) * size_t(used), bytes = entries + sizeof(uint32_t) * size_t(chunks);
    if (!bytes) return hipSuccess;
    unsigned char *host = new (std::nothrow) unsigned char[bytes];
    if (!host) return hipErrorOutOfMemory;
    LearnEntry *entry = reinterpret_cast<LearnEntry *>(host);
    uint32_t *owner = reinterpret_cast<uint32_t *>(host + entries);
    int64_t at = 0, chunk = 0;
    for (int kind = 0; kind < kinds; ++kind) {
        const int64_t begin = chunk;
        for (int64_t i = 0; i < num; ++i) {
            const gwtf_learn_tensor_t &x = tensors[i];
            if (!x.size || kind_of(x) != kind) continue;
            entry[at] = {x.size, x.grad, x.param, x.master, x.m, x.v, x.m_scale, x.v_scale, chunk, x.weight_decay, x.site};
            for (int64_t q = (x.size + kChunk - 1) / kChunk; q > 0; --q) owner[chunk++] = uint32_t(at);
            ++at;
            t.cls[t.classes] = {x.type, x.grad_type, begin, chunk};
        }
        if (chunk > begin) ++t.classes;
    }
    hipError_t e = hipMalloc(&t.base, bytes);
    if (e == hipSuccess) {
        e = hipMemcpy(t.base, host, bytes, hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            (void)hipFree(t.base);
            t.base = nullptr;
        }
    }
    delete[] host;
    t.entry = static_cast<const LearnEntry *>(t.base);
    t.owner = reinterpret_cast<const uint32_t *>(static_cast<const unsigned char *>(t.base) + entries);
    return e;
}

hipError_t launch_grad_norm(const gwtf_learn_grad_norm_t &a, const LearnTable &t, const LearnWorkspace &w, hipStream_t s)
{
    if (!t.classes) return launch(norm_of_nothing_kernel, 1, 1, s, float(a.scale), a.norm, a.factor);
    NormArgs args = {0, 0, w.partial, w.arrived, 0, 0, a.max_norm, a.scale, a.norm, a.factor};
    for (int c = 0; c < t.classes;) {
        // classes that differ in the parameters' type alone are one here
        int next = c + 1;
        while (next < t.classes && t.cls[next].grad_type == t.cls[c].grad_type) ++next;
        args.begin = t.cls[c].begin;
        args.end = t.cls[next - 1].end;
        const int64_t chunks = args.end - args.begin, groups = chunks < kNormGroups ? chunks : kNormGroups;
        args.last = next == t.classes && groups <= kNormArrivals ? uint32_t(groups) : 0u;
        const int type = t.cls[c].grad_type;
        auto kernel = type == GWTF_TYPE_F32 ? norm_kernel<float> : type == GWTF_TYPE_F16 ? norm_kernel<f16_t> : norm_kernel<bf16_t>;
        const hipError_t e = launch(kernel, groups, 256, s, t.entry, t.owner, args);
        if (e != hipSuccess) return e;
        args.first += int32_t(groups);
        c = next;
    }
    if (args.last) return hipSuccess;
    args.begin = args.end; // a workgroup without a chunk joins
    args.last = 1;
    return launch(norm_kernel<float>, 1, 256, s, t.entry, t.owner, args);
}

hipError_t launch_adamw(const gwtf_learn_adamw_t &a, const LearnTable &t, hipStream_t s)
{
    AdamArgs args;
    args.entry = t.entry;
    args.owner = t.owner;
    args.lr = float(a.lr);
    args.beta1 = float(a.beta1);
    args.rest1 = float(1.0 - a.beta1);
    args.beta2 = float(a.beta2);
    args.rest2 = float(1.0 - a.beta2);
    args.eps = float(a.eps);
    args.log_beta1 = std::log(a.beta1); // -infinity for 0: then expm1 gives -1
    args.log_beta2 = std::log(a.beta2);
    args.unbias1 = a.step_at ? 1.f : float(-1.0 / std::expm1(double(a.step) * args.log_beta1));
    args.unbias2 = a.step_at ? 1.f : float(-1.0 / std::expm1(double(a.step) * args.log_beta2));
    args.k0 = uint32_t(a.seed);
    args.k1 = uint32_t(a.seed >> 32);
    args.step = a.step;
    args.step_at = a.step_at;
    args.lr_at = a.lr_at;
    args.factor = a.factor;
    const int64_t slab = kLaunchThreads / 256;
    for (int c = 0; c < t.classes; ++c) {
        const AdamKernel kernel = t.form == GWTF_STATE_F8 ? adamw_of<true>(t.cls[c].type, t.cls[c].grad_type)
                                                          : adamw_of<false>(t.cls[c].type, t.cls[c].grad_type);
        for (int64_t b = t.cls[c].begin; b < t.cls[c].end; b += slab) {
            args.begin = b;
            const int64_t n = t.cls[c].end - b < slab ? t.cls[c].end - b : slab;
            const hipError_t e = launch(kernel, n, 256, s, args);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

} // namespace gwtf
