// Hand-off between stages: residual added, RMS norm, optional 8-bit values
// (gwtf_stage_norm), and the gradient (gwtf_stage_norm_grad).
//
//   h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h * rstd * weight
//   dx = dh + rstd * (dy * weight - xhat * mean(dy * weight * xhat)), xhat = h * rstd
//   dweight = sum over rows of dy * xhat
//
// A row stays in registers between its reduction and its use, eight columns a
// lane, so that every value is read once: one wave a row up to 1024 columns,
// WAVES waves a row above, 16 columns a lane where that makes fewer waves (eight
// a lane and twice the waves: 4096 columns 87 us in place of 76, 8192 95 and 77).
//
// Bound by memory: 16,384 x 4096 bf16 with residual to 8 bits 75 us (472 MB, 6.3
// TB/s with what the memory-side cache still holds), its gradient 95 us (537 MB,
// 5.7 TB/s); the gradient of 4095 x 1111 f32 17 us (55 MB), 4 of them the second
// launch.  Five rows of 4096 3.8 us: a launch, a read, two barriers.
#include "stage_device.h"
#include "stage_internal.h"

namespace gwtf {
namespace {

constexpr float kF8Max = 448.f;
constexpr float kScaleMin = 0x1p-126f;

// Sum over the waves of a row (one wave: itself), in every lane.
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float *red, int wave)
{
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += red[i];
    }
    return v;
}

__device__ __forceinline__ void store_f8(uint8_t *p, int64_t n, const float v[8])
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    if (n >= kVec) {
        typedef int i32x2 __attribute__((ext_vector_type(2), aligned(1)));
        i32x2 w;
        w[0] = lo;
        w[1] = hi;
        *reinterpret_cast<i32x2 *>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) p[i] = uint8_t((i < 4 ? lo : hi) >> (8 * (i & 3)));
    }
}

// One scale's; `bits`: the largest magnitude's.
__device__ __forceinline__ float scale_of(uint32_t bits)
{
    return bits >= 0x7f800000u ? __builtin_nanf("") : fmaxf(__uint_as_float(bits) / kF8Max, kScaleMin);
}
// The 32-bit quotients y / s: the product with 1 / s and a step along its
// remainder, which makes it the nearest.  (The product alone puts quotients that
// lie half way between two 8-bit values to the wrong one, 0.05 % of all where y
// has few bits.)  Small scales and values are raised first, so that remainders
// keep their bits.
__device__ __forceinline__ void quantise(float y[8], float s)
{
    const float up = s < 0x1p-64f ? 0x1p64f : 1.f, d = s * up, inv = 1.f / d;
    const bool bad = !(s == s);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float a = y[i] * up, p = a * inv, q = fmaf(-fmaf(p, d, -a), inv, p); // in this order -0 stays -0
        const float v = fminf(fmaxf(q, -kF8Max), kF8Max); // the quotient may round past 448
        y[i] = bad ? s : v;
    }
}

template <class T, int K, int WAVES, bool STREAM, bool WIDE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_kernel(gwtf_stage_norm_t p, int64_t row0)
{
    __shared__ float red[WAVES], red_again[WAVES];
    __shared__ uint32_t redmax[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = row0 + (WAVES == 1 ? int64_t(blockIdx.x) * 4 + wave : int64_t(blockIdx.x));
    if (row >= p.num_tokens) return; // WAVES == 1 only: no barrier follows
    const int part = WAVES == 1 ? 0 : wave;
    const T *x = static_cast<const T *>(p.x) + row * p.x_stride;
    const T *res = static_cast<const T *>(p.residual) + row * p.residual_stride;
    const T *weight = static_cast<const T *>(p.weight);
    const int H = int(p.hidden);

    float h[K][8], sq = 0.f;
    typename Vec8<T>::type rx[K], rres[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = ((k * WAVES + part) * 64 + lane) * kVec;
        rx[k] = load_columns<T, STREAM, WIDE>(x, col, H);
        if (p.residual) rres[k] = load_columns<T, STREAM, WIDE>(res, col, H);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = ((k * WAVES + part) * 64 + lane) * kVec;
        const bool ends = ends_within(col, H);
        columns_of<T>(rx[k], ends, col, H, h[k]);
        if (p.residual) {
            float r[8];
            columns_of<T>(rres[k], ends, col, H, r);
#pragma unroll
            for (int i = 0; i < kVec; ++i) h[k][i] += r[i];
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) sq += h[k][i] * h[k][i];
    }
    sq = group_sum<WAVES>(sq, red, part);
    float rstd = 1.f / sqrtf(sq / float(H) + p.eps);
    // The squares' range is half that of the values: where it is left (by values
    // of 2^57 and more, or of 2^-40 and less without an eps), in other units.
    const bool large = !(sq <= 0x1.fffffep127f), small = sq < 0x1p-80f && p.eps < 0x1p-100f;
    if (large || small) {
        const float unit = large ? 0x1p-80f : 0x1p100f;
        sq = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) sq += (h[k][i] * unit) * (h[k][i] * unit);
        }
        sq = group_sum<WAVES>(sq, red_again, part);
        rstd = unit / sqrtf(sq / float(H) + p.eps * unit * unit);
    }
    if (p.rstd && part == 0 && lane == 0) p.rstd[row] = rstd;

    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = ((k * WAVES + part) * 64 + lane) * kVec, n = H - col;
        if (p.h_out) store8<T, STREAM>(static_cast<T *>(p.h_out) + row * p.h_stride + col, n, h[k]);
        float w[8];
        load8(weight + col, n, w);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] = h[k][i] * rstd * w[i];
        if (p.form == GWTF_NORM_PLAIN) {
            store8<T, STREAM>(static_cast<T *>(p.y) + row * p.y_stride + col, n, h[k]);
            continue;
        }
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) m = umax(m, __float_as_uint(h[k][i]) & 0x7fffffffu);
        if (p.form == GWTF_NORM_F8_BLOCK) { // 128 columns are 16 lanes
            const float s = scale_of(row_umax(m));
            quantise(h[k], s);
            store_f8(static_cast<uint8_t *>(p.y) + row * p.y_stride + col, n, h[k]);
            const int blocks = (H + GWTF_NORM_BLOCK - 1) / GWTF_NORM_BLOCK;
            if ((lane & 15) == 0 && n > 0) p.scales[row * blocks + col / GWTF_NORM_BLOCK] = s;
        } else {
            most = umax(most, m);
        }
    }
    if (p.form != GWTF_NORM_F8_ROW) return;
    most = wave_umax(most);
    if constexpr (WAVES > 1) {
        if (lane == 0) redmax[wave] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) most = umax(most, redmax[i]);
    }
    const float s = scale_of(most);
    if (part == 0 && lane == 0) p.scales[row] = s;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = ((k * WAVES + part) * 64 + lane) * kVec;
        quantise(h[k], s);
        store_f8(static_cast<uint8_t *>(p.y) + row * p.y_stride + col, H - col, h[k]);
    }
}

// Every workgroup takes the rows blockIdx.x, blockIdx.x + gridDim.x, .. (four
// at a time with one wave a row) and keeps its sum of dweight in registers.
template <class T, int K, int WAVES, bool STREAM, bool WIDE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_grad_kernel(gwtf_stage_norm_grad_t p, float *partial)
{
    __shared__ float red[2][WAVES];
    __shared__ float sums[WAVES == 1 ? 4 * K * 512 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int part = WAVES == 1 ? 0 : wave, mine = WAVES == 1 ? wave : 0;
    const int64_t rows_at_once = WAVES == 1 ? 4 : 1;
    const int H = int(p.hidden);
    const T *weight = static_cast<const T *>(p.weight);
    float w[K][8], dw[K][8];
    bool ends[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = ((k * WAVES + part) * 64 + lane) * kVec;
        load8(weight + col, H - col, w[k]);
        ends[k] = ends_within(col, H);
#pragma unroll
        for (int i = 0; i < kVec; ++i) dw[k][i] = 0.f;
    }
    // Rows on their way while one is reduced and written: two where a lane has
    // eight columns, one where it has sixteen, none with 16 waves, which spill
    // as it is (33 registers a lane for 32-bit types, 19 for 16-bit ones).
    constexpr bool AHEAD = WAVES < 16;
    constexpr int DEPTH = K == 1 ? 2 : 1;
    typename Vec8<T>::type rdy[DEPTH][K], rh[DEPTH][K], rd[DEPTH][K];
    float rrstd[DEPTH];
    const int64_t stride = int64_t(gridDim.x) * rows_at_once;
    auto fetch = [&](int64_t row, int slot) {
        if (row >= p.num_tokens) return;
        const T *dy = static_cast<const T *>(p.dy) + row * p.dy_stride;
        const T *hp = static_cast<const T *>(p.h) + row * p.h_stride;
        const T *dh = static_cast<const T *>(p.dh) + row * p.dh_stride;
        rrstd[slot] = p.rstd[row];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = ((k * WAVES + part) * 64 + lane) * kVec;
            rdy[slot][k] = load_columns<T, STREAM, WIDE>(dy, col, H);
            rh[slot][k] = load_columns<T, STREAM, WIDE>(hp, col, H);
            if (p.dh) rd[slot][k] = load_columns<T, STREAM, WIDE>(dh, col, H);
        }
    };
    int turn = 0;
    int64_t row = blockIdx.x * rows_at_once + mine;
#pragma unroll
    for (int q = 0; q < (AHEAD ? DEPTH : 0); ++q) fetch(row + q * stride, q);
    for (; row < p.num_tokens; row += stride, turn ^= 1) {
        if constexpr (!AHEAD) fetch(row, 0);
        const float rstd = rrstd[0];
        float g[K][8], xh[K][8], d[K][8], c = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = ((k * WAVES + part) * 64 + lane) * kVec;
            columns_of<T>(rdy[0][k], ends[k], col, H, g[k]);
            columns_of<T>(rh[0][k], ends[k], col, H, xh[k]);
            if (p.dh) {
                columns_of<T>(rd[0][k], ends[k], col, H, d[k]);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) d[k][i] = 0.f;
            }
        }
#pragma unroll
        for (int q = 0; q + 1 < DEPTH; ++q) {
            rrstd[q] = rrstd[q + 1];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                rdy[q][k] = rdy[q + 1][k];
                rh[q][k] = rh[q + 1][k];
                rd[q][k] = rd[q + 1][k];
            }
        }
        if constexpr (AHEAD) fetch(row + DEPTH * stride, DEPTH - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                xh[k][i] *= rstd;
                dw[k][i] += g[k][i] * xh[k][i];
                g[k][i] *= w[k][i];
                c += g[k][i] * xh[k][i];
            }
        }
        // two buffers in turn: a wave may be one row ahead of the slowest reader
        c = group_sum<WAVES>(c, red[turn], part) / float(H);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = ((k * WAVES + part) * 64 + lane) * kVec;
#pragma unroll
            for (int i = 0; i < kVec; ++i) d[k][i] += rstd * (g[k][i] - xh[k][i] * c);
            store8<T, STREAM>(static_cast<T *>(p.dx) + row * p.dx_stride + col, H - col, d[k]);
        }
    }
    if (!partial) return;
    float *out = partial + int64_t(blockIdx.x) * H;
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) sums[(wave * K + k) * 512 + lane * kVec + i] = dw[k][i];
        }
        __syncthreads();
        for (int col = threadIdx.x; col < H; col += 256)
            out[col] = (sums[col] + sums[K * 512 + col]) + (sums[2 * K * 512 + col] + sums[3 * K * 512 + col]);
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = ((k * WAVES + part) * 64 + lane) * kVec;
            store8(out + col, H - col, dw[k]);
        }
    }
}

// dweight from the workgroups' sums: 16 columns a workgroup, 64 threads a
// column, each over adjacent sums in order.
__global__ __launch_bounds__(1024) void dweight_kernel(const float *partial, int groups, int H, float *dweight)
{
    __shared__ float red[64][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    const int each = (groups + 63) / 64, g0 = g * each, g1 = g0 + each < groups ? g0 + each : groups;
    float v = 0.f;
    if (col < H) {
        int i = g0;
        for (; i + 8 <= g1; i += 8) {
            float f[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) f[q] = partial[int64_t(i + q) * H + col];
#pragma unroll
            for (int q = 0; q < 8; ++q) v += f[q];
        }
        for (; i < g1; ++i) v += partial[int64_t(i) * H + col];
    }
    red[g][c] = v;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (g < half) red[g][c] += red[g + half][c];
        __syncthreads();
    }
    if (g == 0 && col < H) dweight[col] = red[0][c];
}

__global__ void zero_kernel(float *p, int64_t n)
{
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) p[i] = 0.f;
}

template <class T, int K, int WAVES>
hipError_t run_norm(const gwtf_stage_norm_t &a, hipStream_t s)
{
    const int64_t rows = WAVES == 1 ? 4 : 1;
    const int64_t values = 1 + (a.residual != nullptr) + (a.h_out != nullptr) + (a.form == GWTF_NORM_PLAIN);
    const int64_t bytes = a.num_tokens * a.hidden * (values * int64_t(sizeof(T)) + (a.form != GWTF_NORM_PLAIN));
    const bool stream = bytes >= kStreamBytes && on_lines(a.x, a.x_stride, sizeof(T)) &&
                        (!a.residual || on_lines(a.residual, a.residual_stride, sizeof(T))) &&
                        (!a.h_out || on_lines(a.h_out, a.h_stride, sizeof(T))) &&
                        (a.form != GWTF_NORM_PLAIN || on_lines(a.y, a.y_stride, sizeof(T)));
    auto kernel = stream ? norm_kernel<T, K, WAVES, true, true> : norm_kernel<T, K, WAVES, false, true>;
    if (K == 1 && WAVES == 1 && a.hidden < kVec) kernel = norm_kernel<T, 1, 1, false, false>;
    constexpr int threads = WAVES == 1 ? 256 : WAVES * 64;
    const int64_t slab = kLaunchThreads / threads * rows;
    for (int64_t r = 0; r < a.num_tokens; r += slab) {
        const int64_t n = a.num_tokens - r < slab ? a.num_tokens - r : slab;
        const hipError_t e = launch(kernel, (n + rows - 1) / rows, threads, s, a, r);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, int K, int WAVES>
hipError_t run_norm_grad(const gwtf_stage_norm_grad_t &a, const StageWorkspace &w, hipStream_t s)
{
    const int64_t rows = WAVES == 1 ? 4 : 1;
    int64_t groups = (a.num_tokens + rows - 1) / rows;
    if (groups > kNormGradGroups) groups = kNormGradGroups;
    const int64_t bytes = a.num_tokens * a.hidden * int64_t(sizeof(T)) * (a.dh ? 4 : 3);
    const bool stream = bytes >= kStreamBytes && on_lines(a.dy, a.dy_stride, sizeof(T)) &&
                        on_lines(a.h, a.h_stride, sizeof(T)) && (!a.dh || on_lines(a.dh, a.dh_stride, sizeof(T))) &&
                        on_lines(a.dx, a.dx_stride, sizeof(T));
    auto kernel = stream ? norm_grad_kernel<T, K, WAVES, true, true> : norm_grad_kernel<T, K, WAVES, false, true>;
    if (K == 1 && WAVES == 1 && a.hidden < kVec) kernel = norm_grad_kernel<T, 1, 1, false, false>;
    const hipError_t e = launch(kernel, groups, WAVES == 1 ? 256 : WAVES * 64, s, a, a.dweight ? w.dweight : nullptr);
    if (e != hipSuccess || !a.dweight) return e;
    return launch(dweight_kernel, (a.hidden + 15) / 16, 1024, s, w.dweight, int(groups), int(a.hidden), a.dweight);
}

// Waves and steps of a row by its width: 512 columns a wave and step.
template <class T, class Fn>
hipError_t by_width(int64_t H, Fn f)
{
    if (H <= 512) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
    if (H <= 1024) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 1>());
    if (H <= 2048) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
    if (H <= 4096) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
    if (H <= 8192) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 2>(), std::integral_constant<int, 16>());
}

template <class T>
hipError_t norm_typed(const gwtf_stage_norm_t &a, hipStream_t s)
{
    return by_width<T>(a.hidden, [&](auto k, auto w) { return run_norm<T, decltype(k)::value, decltype(w)::value>(a, s); });
}
template <class T>
hipError_t norm_grad_typed(const gwtf_stage_norm_grad_t &a, const StageWorkspace &ws, hipStream_t s)
{
    return by_width<T>(a.hidden,
                       [&](auto k, auto w) { return run_norm_grad<T, decltype(k)::value, decltype(w)::value>(a, ws, s); });
}

} // namespace

hipError_t launch_norm(const gwtf_stage_norm_t &a, const StageWorkspace &, hipStream_t s)
{
    if (a.num_tokens == 0) return hipSuccess;
    switch (a.type) {
    case GWTF_TYPE_F32: return norm_typed<float>(a, s);
    case GWTF_TYPE_F16: return norm_typed<f16_t>(a, s);
    default: return norm_typed<bf16_t>(a, s);
    }
}

hipError_t launch_norm_grad(const gwtf_stage_norm_grad_t &a, const StageWorkspace &w, hipStream_t s)
{
    if (a.num_tokens == 0) {
        if (!a.dweight) return hipSuccess;
        return launch(zero_kernel, (a.hidden + 255) / 256, 256, s, a.dweight, a.hidden);
    }
    switch (a.type) {
    case GWTF_TYPE_F32: return norm_grad_typed<float>(a, w, s);
    case GWTF_TYPE_F16: return norm_grad_typed<f16_t>(a, w, s);
    default: return norm_grad_typed<bf16_t>(a, w, s);
    }
}

} // namespace gwtf
