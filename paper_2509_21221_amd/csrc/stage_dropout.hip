// Dropout whose mask is a function of the seed, the site and the row's
// identity (gwtf_stage_dropout).
//
//   out = residual + (u >= t ? x * 65536 / (65536 - t) : 0)
//
// One call of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011) gives the 16-bit u of eight columns: ten
// rounds of two 32 x 32 -> 64 bit products for 16 bytes of a 16-bit type.
// With 32 bits a value the products, which take four times as long to issue
// as other operations, would cost more than the memory.
//
// Bound by memory: 16,384 x 4096 bf16 with residual 65 us (403 MB, 6.2 TB/s with
// what the memory-side cache still holds), 16,383 x 4095 f16, rows on odd
// addresses, 55 us (268 MB, 4.9 TB/s); 2,048 x 1024 3.6 us.
#include "stage_device.h"
#include "stage_internal.h"

namespace gwtf {
namespace {

struct DropoutParams {
    const void *x, *res;
    void *out;
    const int64_t *rows;
    int64_t xs, rs, os, row0;
    int32_t H;
    uint32_t units; // (rows of this launch) * (steps of eight columns in a row)
    FastDiv steps;
    uint32_t k0, k1, site, limit;
    float keep_scale;
};

// Steps of eight columns a thread takes, with their reads side by side.
constexpr uint32_t kUnits = 2;

template <class T, bool RES, bool STREAM>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutParams p)
{
    const uint32_t u0 = blockIdx.x * (256u * kUnits) + threadIdx.x;
    typename Vec8<T>::type raw[kUnits], rraw[kUnits];
    int64_t row[kUnits];
    uint32_t step[kUnits];
    uint64_t id[kUnits];
#pragma unroll
    for (uint32_t q = 0; q < kUnits; ++q) {
        const uint32_t u = u0 + q * 256u, r = p.steps.div(u < p.units ? u : 0);
        step[q] = (u < p.units ? u : 0) - r * p.steps.d;
        row[q] = p.row0 + r;
        const int64_t col = int64_t(step[q]) * kVec;
        raw[q] = load_columns<T, STREAM>(static_cast<const T *>(p.x) + row[q] * p.xs, col, p.H);
        if constexpr (RES) rraw[q] = load_columns<T, STREAM>(static_cast<const T *>(p.res) + row[q] * p.rs, col, p.H);
        id[q] = p.rows ? uint64_t(p.rows[row[q]]) : uint64_t(row[q]);
    }
#pragma unroll
    for (uint32_t q = 0; q < kUnits; ++q) {
        uint32_t c[4] = {step[q], p.site, uint32_t(id[q]), uint32_t(id[q] >> 32)};
        philox4x32(p.k0, p.k1, c);
        float v[8], res[8];
        const int64_t col = int64_t(step[q]) * kVec;
        const bool ends = ends_within(col, p.H);
        columns_of<T>(raw[q], ends, col, p.H, v);
        if constexpr (RES) columns_of<T>(rraw[q], ends, col, p.H, res);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const uint32_t bits = (i & 1) ? c[i / 2] >> 16 : c[i / 2] & 0xffffu;
            v[i] = bits >= p.limit ? v[i] * p.keep_scale : 0.f;
            if constexpr (RES) v[i] += res[i];
        }
        if (u0 + q * 256u < p.units) store8<T, STREAM>(static_cast<T *>(p.out) + row[q] * p.os + col, p.H - col, v);
    }
}

template <class T>
hipError_t run(const gwtf_stage_dropout_t &a, uint32_t limit, hipStream_t s)
{
    const int64_t steps = (a.hidden + kVec - 1) / kVec;
    // units of one launch stay below 2^30
    const int64_t slab = (int64_t(1) << 30) / steps;
    DropoutParams p;
    p.x = a.x;
    p.res = a.residual;
    p.out = a.out;
    p.rows = a.rows;
    p.xs = a.x_stride;
    p.rs = a.residual_stride;
    p.os = a.out_stride;
    p.H = int32_t(a.hidden);
    p.steps = FastDiv::make(uint32_t(steps));
    p.k0 = uint32_t(a.seed);
    p.k1 = uint32_t(a.seed >> 32);
    p.site = a.site;
    p.limit = limit;
    p.keep_scale = 65536.f / float(65536 - limit);
    const bool stream = a.num_tokens * a.hidden * int64_t(sizeof(T)) * (a.residual ? 3 : 2) >= kStreamBytes &&
                        on_lines(a.x, a.x_stride, sizeof(T)) && on_lines(a.out, a.out_stride, sizeof(T)) &&
                        (!a.residual || on_lines(a.residual, a.residual_stride, sizeof(T)));
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        p.row0 = r;
        p.units = uint32_t(n * steps);
        auto kernel = p.res ? (stream ? dropout_kernel<T, true, true> : dropout_kernel<T, true, false>)
                            : (stream ? dropout_kernel<T, false, true> : dropout_kernel<T, false, false>);
        const hipError_t e = launch(kernel, (p.units + 256 * kUnits - 1) / (256 * kUnits), 256, s, p);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace

hipError_t launch_dropout(const gwtf_stage_dropout_t &a, uint32_t limit, hipStream_t s)
{
    switch (a.type) {
    case GWTF_TYPE_F32: return run<float>(a, limit, s);
    case GWTF_TYPE_F16: return run<f16_t>(a, limit, s);
    default: return run<bf16_t>(a, limit, s);
    }
}

} // namespace gwtf
