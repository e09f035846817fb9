// What the host sides of the microbatch operators (stage_api.hip) and of the
// learning step's (learn_api.hip) share: the device of a call, and the checks of
// arrays.
#pragma once

#include "gwtf_stage.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace gwtf {

// Makes `device` current for a call; the caller's device comes back after it.
struct DeviceScope {
    int before = -1, device;
    hipError_t e;
    explicit DeviceScope(int d) : device(d)
    {
        e = hipGetDevice(&before);
        if (e == hipSuccess && before != d) e = hipSetDevice(d);
    }
    ~DeviceScope()
    {
        if (before >= 0 && before != device) (void)hipSetDevice(before);
    }
};

inline size_t size_of(int32_t type) { return type == GWTF_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int32_t t) { return t == GWTF_TYPE_F32 || t == GWTF_TYPE_F16 || t == GWTF_TYPE_BF16; }

// A matrix or vector of elements of `size` bytes, `rows` rows of `width`.
inline const char *bad_matrix(const void *p, int64_t stride, int64_t rows, int64_t width, size_t size)
{
    if (rows == 0) return nullptr;
    if (!p) return "a required array is NULL";
    if (reinterpret_cast<uintptr_t>(p) % size) return "an array is not aligned to its element type";
    if (rows > 1 && (stride < width || stride > (int64_t(1) << 40))) return "a row stride is below the width or above 2^40";
    return nullptr;
}
inline const char *bad_vector(const void *p, int64_t n, size_t size) { return bad_matrix(p, n, n ? 1 : 0, n, size); }

} // namespace gwtf
