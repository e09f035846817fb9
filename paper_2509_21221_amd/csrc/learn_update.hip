// Update phase of a node: the norm of its gradients (gwtf_learn_grad_norm) and
// the AdamW step over its parameters (gwtf_learn_adamw).
//
// Tensors come as a list whose entries travel in the kernel's arguments, as many
// as fit in 4 KB, so that no call copies a table or keeps one between calls; a
// workgroup finds its tensor by a ballot over the entries' first chunks.
#include "learn_internal.h"
#include "stage_device.h"

#include <cmath>

namespace gwtf {
namespace {

// A launch takes fewer chunks than this: below 2^32 threads.
constexpr int64_t kMostChunks = int64_t(1) << 23;

// Which of `count` entries, in order of their first chunks, `chunk` belongs to.
template <int K>
__device__ __forceinline__ int entry_of(const uint32_t (&first)[K], int count, uint32_t chunk)
{
    const int lane = threadIdx.x & 63;
    int at = -1;
#pragma unroll
    for (int base = 0; base < K; base += 64) {
        const int i = base + lane;
        at += __popcll(__ballot(i < count && first[i < K ? i : 0] <= chunk));
    }
    return __builtin_amdgcn_readfirstlane(at);
}

// ---- Norm ----

constexpr int kNormEntries = 160;
constexpr int kNormChunk = 256 * kVec; // values of a workgroup's step

struct NormEntry {
    const void *grad;
    int64_t size;
};
struct NormArgs {
    NormEntry e[kNormEntries];
    uint32_t first[kNormEntries];
    int32_t count;
    uint32_t chunks;
};

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// partial[workgroup] = sum of squares of the chunks blockIdx.x, blockIdx.x + gridDim.x, ..
template <class T>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a, double *partial)
{
    __shared__ double red[4];
    double sum = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const int at = entry_of(a.first, a.count, chunk);
        const T *g = static_cast<const T *>(a.e[at].grad);
        const int64_t i = int64_t(chunk - a.first[at]) * kNormChunk + threadIdx.x * kVec;
        float v[8];
        load8(g + i, a.e[at].size - i, v);
#pragma unroll
        for (int q = 0; q < kVec; ++q) sum = fma(double(v[q]), double(v[q]), sum);
    }
    sum = wave_sum64(sum);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// The sum of `count` partial sums, in a fixed order: to *sum, or as the results.
__global__ __launch_bounds__(256) void norm_join_kernel(const double *partial, int count, double *sum, double max_norm, double scale,
                                                        float *norm, float *factor)
{
    __shared__ double red[4];
    double v = 0.0;
    for (int i = threadIdx.x; i < count; i += 256) v += partial[i];
    v = wave_sum64(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x) return;
    v = (red[0] + red[1]) + (red[2] + red[3]);
    if (sum) {
        *sum = v;
        return;
    }
    const double n = scale * sqrt(v);
    if (norm) *norm = float(n);
    if (factor) *factor = n < __builtin_inf() ? float(n > max_norm ? scale * (max_norm / n) : scale) : __builtin_nanf("");
}

// ---- AdamW ----

constexpr int kAdamEntries = 50;
constexpr int kAdamChunk = 256 * kVec * 2;

struct AdamEntry {
    int64_t size;
    const void *grad;
    void *param;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    float decay;
    uint32_t site;
};
struct AdamArgs {
    AdamEntry e[kAdamEntries];
    uint32_t first[kAdamEntries];
    int32_t count;
    float lr, beta1, rest1, beta2, rest2, eps, unbias1, unbias2;
    uint32_t k0, k1;
    double log_beta1, log_beta2;
    int64_t step;
    const int64_t *step_at;
    const float *lr_at, *factor;
};
static_assert(sizeof(NormArgs) + 8 <= 4096 && sizeof(AdamArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ void philox4x32(uint32_t k0, uint32_t k1, uint32_t c[4])
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = uint64_t(0xD2511F53u) * c[0], b = uint64_t(0xCD9E8D57u) * c[2];
        const uint32_t n0 = __builtin_amdgcn_bitop3_b32(uint32_t(b >> 32), c[1], k0, 0x96);
        const uint32_t n2 = __builtin_amdgcn_bitop3_b32(uint32_t(a >> 32), c[3], k1, 0x96);
        c[1] = uint32_t(b);
        c[3] = uint32_t(a);
        c[0] = n0;
        c[2] = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

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
        if (E5M2 && a > 0.f && small == 0) small = 1;
        uint32_t c = a >= NORMAL ? large : small;
        if (!E5M2) c |= (__float_as_uint(x[i]) >> 24) & (c ? 0x80u : 0u);
        w[i / 4] |= c << (8 * (i & 3));
    }
    return w;
}

template <class T, class G, bool F8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a)
{
#pragma clang fp contract(off)
    const int at = entry_of(a.first, a.count, blockIdx.x);
    const AdamEntry t = a.e[at];
    const float factor = a.factor ? *a.factor : 1.f;
    if (!(__builtin_fabsf(factor) < __builtin_inff())) return;
    const float lr = a.lr_at ? *a.lr_at : a.lr;
    int64_t step = a.step;
    float unbias1 = a.unbias1, unbias2 = a.unbias2;
    if (a.step_at) {
        step = *a.step_at;
        unbias1 = float(-expm1(double(step) * a.log_beta1));
        unbias2 = float(-expm1(double(step) * a.log_beta2));
    }
    const int64_t begin = int64_t(blockIdx.x - a.first[at]) * kAdamChunk;
#pragma unroll
    for (int q = 0; q < kAdamChunk / (256 * kVec); ++q) {
        const int64_t i = begin + (q * 256 + threadIdx.x) * kVec, n = t.size - i;
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
            const float d = (m[k] / unbias1) / (sqrtf(v[k] / unbias2) + a.eps);
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
}

template <class T, class G>
hipError_t run_adamw(const AdamArgs &a, int64_t chunks, bool f8, hipStream_t s)
{
    return launch(f8 ? adamw_kernel<T, G, true> : adamw_kernel<T, G, false>, chunks, 256, s, a);
}

hipError_t flush_adamw(AdamArgs &a, int64_t chunks, int type, int grad_type, bool f8, hipStream_t s)
{
    const bool wide = grad_type == GWTF_TYPE_F32;
    switch (type) {
    case GWTF_TYPE_F32: return run_adamw<float, float>(a, chunks, f8, s);
    case GWTF_TYPE_F16: return wide ? run_adamw<f16_t, float>(a, chunks, f8, s) : run_adamw<f16_t, f16_t>(a, chunks, f8, s);
    default: return wide ? run_adamw<bf16_t, float>(a, chunks, f8, s) : run_adamw<bf16_t, bf16_t>(a, chunks, f8, s);
    }
}

hipError_t flush_norm(const NormArgs &a, int type, int64_t groups, double *partial, hipStream_t s)
{
    switch (type) {
    case GWTF_TYPE_F32: return launch(norm_kernel<float>, groups, 256, s, a, partial);
    case GWTF_TYPE_F16: return launch(norm_kernel<f16_t>, groups, 256, s, a, partial);
    default: return launch(norm_kernel<bf16_t>, groups, 256, s, a, partial);
    }
}

} // namespace

hipError_t launch_grad_norm(const gwtf_learn_grad_norm_t &a, const LearnWorkspace &w, hipStream_t s)
{
    const int64_t most = 8 * int64_t(w.cus);
    NormArgs args;
    int64_t chunks = 0, used = 0;
    args.count = 0;
    int type = 0;
    hipError_t e = hipSuccess;
    auto flush = [&]() {
        if (!args.count) return hipSuccess;
        const int64_t groups = chunks < most ? chunks : most;
        if (used + groups > kNormSlots) { // the sums so far become the first one
            const hipError_t j = launch(norm_join_kernel, 1, 256, s, w.partial, int(used), w.partial, 0.0, 0.0, nullptr, nullptr);
            if (j != hipSuccess) return j;
            used = 1;
        }
        args.chunks = uint32_t(chunks);
        const hipError_t k = flush_norm(args, type, groups, w.partial + used, s);
        used += groups;
        args.count = 0;
        chunks = 0;
        return k;
    };
    for (int64_t i = 0; i < a.num_tensors; ++i) {
        const gwtf_learn_tensor_t &t = a.tensors[i];
        if (!t.size) continue;
        const int64_t more = (t.size + kNormChunk - 1) / kNormChunk;
        if (args.count == kNormEntries || (args.count && (t.grad_type != type || chunks + more > int64_t(1) << 31)))
            if ((e = flush()) != hipSuccess) return e;
        type = t.grad_type;
        args.e[args.count] = {t.grad, t.size};
        args.first[args.count++] = uint32_t(chunks);
        chunks += more;
    }
    if ((e = flush()) != hipSuccess) return e;
    return launch(norm_join_kernel, 1, 256, s, w.partial, int(used), nullptr, a.max_norm, a.scale, a.norm, a.factor);
}

hipError_t launch_adamw(const gwtf_learn_adamw_t &a, hipStream_t s)
{
    const bool f8 = a.form == GWTF_STATE_F8;
    AdamArgs args;
    args.lr = float(a.lr);
    args.beta1 = float(a.beta1);
    args.rest1 = float(1.0 - a.beta1);
    args.beta2 = float(a.beta2);
    args.rest2 = float(1.0 - a.beta2);
    args.eps = float(a.eps);
    args.log_beta1 = std::log(a.beta1); // -infinity for 0: then expm1 gives -1
    args.log_beta2 = std::log(a.beta2);
    args.unbias1 = a.step_at ? 1.f : float(-std::expm1(double(a.step) * args.log_beta1));
    args.unbias2 = a.step_at ? 1.f : float(-std::expm1(double(a.step) * args.log_beta2));
    args.k0 = uint32_t(a.seed);
    args.k1 = uint32_t(a.seed >> 32);
    args.step = a.step;
    args.step_at = a.step_at;
    args.lr_at = a.lr_at;
    args.factor = a.factor;
    args.count = 0;
    int64_t chunks = 0;
    int type = 0, grad_type = 0;
    hipError_t e = hipSuccess;
    for (int64_t i = 0; i < a.num_tensors; ++i) {
        const gwtf_learn_tensor_t &t = a.tensors[i];
        if (!t.size) continue;
        const int64_t more = (t.size + kAdamChunk - 1) / kAdamChunk;
        if (args.count == kAdamEntries ||
            (args.count && (t.type != type || t.grad_type != grad_type || chunks + more > kMostChunks))) {
            if ((e = flush_adamw(args, chunks, type, grad_type, f8, s)) != hipSuccess) return e;
            args.count = 0;
            chunks = 0;
        }
        type = t.type;
        grad_type = t.grad_type;
        args.e[args.count] = {t.size, t.grad, t.param, t.master, t.m, t.v, t.m_scale, t.v_scale, t.weight_decay, t.site};
        args.first[args.count++] = uint32_t(chunks);
        chunks += more;
    }
    return args.count ? flush_adamw(args, chunks, type, grad_type, f8, s) : hipSuccess;
}

} // namespace gwtf
