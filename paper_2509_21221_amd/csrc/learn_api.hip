// Host side of the C ABI declared in include/gwtf_learn.h: argument checks and
// the handle's workspace.
#include "api_checks.h"
#include "learn_internal.h"

#include <cmath>
#include <cstdio>
#include <new>

using namespace gwtf;

struct gwtf_learn {
    int32_t device;
    hipStream_t stream;
    LearnWorkspace ws;
    char err[256];
};

struct gwtf_learn_list {
    int32_t device;
    LearnTable t;
};

namespace {

thread_local char g_learn_err[256];

gwtf_status_t fail(gwtf_learn_t *h, gwtf_status_t code, const char *what, hipError_t e = hipSuccess)
{
    char *to = h ? h->err : g_learn_err;
    if (e != hipSuccess) (void)hipGetLastError(); // it is reported here, not to the thread's next reader
    if (e != hipSuccess) snprintf(to, sizeof g_learn_err, "%s: %s", what, hipGetErrorString(e));
    else snprintf(to, sizeof g_learn_err, "%s", what);
    return code;
}

#define LEARN_BEGIN(name)                                                               \
    if (!h) return fail(nullptr, GWTF_ERR_INVALID_ARG, name ": handle is NULL");        \
    if (!a) return fail(h, GWTF_ERR_INVALID_ARG, name ": arguments are NULL");
#define LEARN_REQUIRE(cond, text) \
    if (!(cond)) return fail(h, GWTF_ERR_INVALID_ARG, text);
#define LEARN_CHECK(expr) \
    if (const char *bad = (expr)) return fail(h, GWTF_ERR_INVALID_ARG, bad);
#define LEARN_LAUNCH(name, expr)                                                        \
    DeviceScope scope(h->device);                                                       \
    if (scope.e != hipSuccess) return fail(h, GWTF_ERR_DEVICE, "hipSetDevice", scope.e); \
    const hipError_t e = (expr);                                                        \
    return e == hipSuccess ? GWTF_OK : fail(h, GWTF_ERR_DEVICE, name " launch", e);

// A number that a kernel takes in 32 bits: finite there too.
bool finite32(double v) { return std::isfinite(v) && std::isfinite(float(v)); }

constexpr int64_t kTensorSize = int64_t(1) << 35, kListSize = int64_t(1) << 42;

// What is wrong with a tensor of a list.
const char *bad_tensor(const gwtf_learn_tensor_t &t, int32_t form)
{
    if (t.size < 0 || t.size >= kTensorSize) return "size outside [0, 2^35)";
    if (!type_ok(t.grad_type)) return "unknown type of grad";
    if (const char *bad = bad_vector(t.grad, t.size, size_of(t.grad_type))) return bad;
    if (form == GWTF_STATE_NONE) return nullptr;
    if (!type_ok(t.type)) return "unknown type";
    if (t.grad_type != t.type && t.grad_type != GWTF_TYPE_F32) return "grad_type must be type or GWTF_TYPE_F32";
    if (!std::isfinite(t.weight_decay)) return "weight_decay must be finite";
    const bool f8 = form == GWTF_STATE_F8;
    const char *bad = bad_vector(t.param, t.size, size_of(t.type));
    if (!bad && t.master) bad = bad_vector(t.master, t.size, 4);
    if (!bad) bad = bad_vector(t.m, t.size, f8 ? 1 : 4);
    if (!bad) bad = bad_vector(t.v, t.size, f8 ? 1 : 4);
    if (!bad && f8) bad = bad_vector(t.m_scale, t.size, 4);
    if (!bad && f8) bad = bad_vector(t.v_scale, t.size, 4);
    return bad;
}

} // namespace

extern "C" gwtf_status_t gwtf_learn_create(int32_t device, void *hip_stream, gwtf_learn_t **out)
{
    if (!out) return fail(nullptr, GWTF_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    if (device < 0) return fail(nullptr, GWTF_ERR_INVALID_ARG, "bad device ordinal");
    int ndev = 0;
    hipError_t e = hipGetDeviceCount(&ndev);
    if (e != hipSuccess) return fail(nullptr, GWTF_ERR_DEVICE, "hipGetDeviceCount", e);
    if (device >= ndev) return fail(nullptr, GWTF_ERR_INVALID_ARG, "bad device ordinal");
    DeviceScope scope(device);
    if (scope.e != hipSuccess) return fail(nullptr, GWTF_ERR_DEVICE, "hipSetDevice", scope.e);
    gwtf_learn_t *h = new (std::nothrow) gwtf_learn_t();
    if (!h) return fail(nullptr, GWTF_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->device = device;
    h->stream = static_cast<hipStream_t>(hip_stream);
    // one allocation, its parts on 256-byte boundaries, the counters first
    LearnWorkspace &w = h->ws;
    size_t total = 0;
    auto take = [&](size_t bytes) {
        const size_t at = total;
        total += (bytes + 255) / 256 * 256;
        return at;
    };
    const size_t arrived = take(sizeof(uint32_t)), rows = take(sizeof(uint32_t) * kRecheckSlots), zeros = total;
    const size_t partial = take(sizeof(double) * kNormSlots), key = take(sizeof(uint32_t) * kRecheckRows);
    const size_t sum = take(sizeof(uint64_t) * kRecheckSlots * kRecheckSegs);
    if ((e = hipMalloc(&w.base, total)) != hipSuccess) {
        delete h;
        return fail(nullptr, GWTF_ERR_OUT_OF_MEMORY, "hipMalloc workspace", e);
    }
    unsigned char *const base = static_cast<unsigned char *>(w.base);
    w.arrived = reinterpret_cast<uint32_t *>(base + arrived);
    w.recheck.arrived = reinterpret_cast<uint32_t *>(base + rows);
    w.partial = reinterpret_cast<double *>(base + partial);
    w.recheck.key = reinterpret_cast<uint32_t *>(base + key);
    w.recheck.sum = reinterpret_cast<uint64_t *>(base + sum);
    if ((e = hipMemsetAsync(base, 0, zeros, h->stream)) != hipSuccess) {
        (void)hipFree(w.base);
        delete h;
        return fail(nullptr, GWTF_ERR_DEVICE, "hipMemsetAsync", e);
    }
    *out = h;
    return GWTF_OK;
}

extern "C" void gwtf_learn_destroy(gwtf_learn_t *h)
{
    if (!h) return;
    DeviceScope scope(h->device);
    if (scope.e == hipSuccess) (void)hipStreamSynchronize(h->stream);
    (void)hipFree(h->ws.base);
    delete h;
}

extern "C" const char *gwtf_learn_last_error(const gwtf_learn_t *h) { return h ? h->err : g_learn_err; }

extern "C" gwtf_status_t gwtf_learn_sample(gwtf_learn_t *h, const gwtf_learn_sample_t *a)
{
    LEARN_BEGIN("gwtf_learn_sample")
    const int64_t N = a->num_tokens, V = a->vocab, top = (int64_t(1) << 31) - 1;
    LEARN_REQUIRE(N >= 0 && N <= top, "num_tokens outside [0, 2^31)")
    LEARN_REQUIRE(V >= 1 && V <= top, "vocab outside [1, 2^31)")
    LEARN_REQUIRE(type_ok(a->type), "unknown type")
    LEARN_REQUIRE(a->uniform_type == GWTF_UNIFORM_F32 || a->uniform_type == GWTF_UNIFORM_F64, "unknown type of u")
    LEARN_REQUIRE(a->temperatures || (a->temperature >= 0 && std::isfinite(a->temperature)), "temperature must be finite and >= 0")
    LEARN_REQUIRE(a->top_ps || a->top_p >= 0, "top_p must be >= 0")
    LEARN_REQUIRE(a->min_ps || (a->min_p >= 0 && a->min_p <= 1), "min_p outside [0, 1]")
    if (N == 0) return GWTF_OK;
    LEARN_CHECK(bad_matrix(a->logits, a->logits_stride, N, V, size_of(a->type)))
    LEARN_CHECK(bad_vector(a->u, N, a->uniform_type == GWTF_UNIFORM_F64 ? 8 : 4))
    LEARN_CHECK(a->temperatures ? bad_vector(a->temperatures, N, 4) : nullptr)
    LEARN_CHECK(a->top_ks ? bad_vector(a->top_ks, N, 4) : nullptr)
    LEARN_CHECK(a->top_ps ? bad_vector(a->top_ps, N, 4) : nullptr)
    LEARN_CHECK(a->min_ps ? bad_vector(a->min_ps, N, 4) : nullptr)
    LEARN_CHECK(bad_vector(a->ids, N, 4))
    LEARN_CHECK(a->logp ? bad_vector(a->logp, N, 4) : nullptr)
    LEARN_CHECK(a->kept ? bad_vector(a->kept, N, 4) : nullptr)
    LEARN_LAUNCH("gwtf_learn_sample", launch_sample(*a, h->ws, h->stream))
}

extern "C" gwtf_status_t gwtf_learn_list_create(gwtf_learn_t *h, int64_t num_tensors, const gwtf_learn_tensor_t *tensors, int32_t form,
                                                gwtf_learn_list_t **out)
{
    if (out) *out = nullptr;
    if (!h) return fail(nullptr, GWTF_ERR_INVALID_ARG, "gwtf_learn_list_create: handle is NULL");
    LEARN_REQUIRE(out, "out is NULL")
    LEARN_REQUIRE(num_tensors >= 0 && num_tensors <= (int64_t(1) << 30), "num_tensors outside [0, 2^30]")
    LEARN_REQUIRE(num_tensors == 0 || tensors, "tensors is NULL")
    LEARN_REQUIRE(form >= GWTF_STATE_F32 && form <= GWTF_STATE_NONE, "unknown form of the states")
    int64_t values = 0;
    for (int64_t i = 0; i < num_tensors; ++i) {
        if (const char *bad = bad_tensor(tensors[i], form)) {
            snprintf(h->err, sizeof h->err, "tensor %lld: %s", static_cast<long long>(i), bad);
            return GWTF_ERR_INVALID_ARG;
        }
        values += tensors[i].size;
        LEARN_REQUIRE(values <= kListSize, "more than 2^42 values")
    }
    gwtf_learn_list_t *list = new (std::nothrow) gwtf_learn_list_t();
    if (!list) return fail(h, GWTF_ERR_OUT_OF_MEMORY, "host allocation failed");
    list->device = h->device;
    list->t.form = form;
    DeviceScope scope(h->device);
    hipError_t e = scope.e;
    if (e == hipSuccess) e = build_table(num_tensors, tensors, list->t);
    if (e != hipSuccess) {
        delete list;
        return fail(h, e == hipErrorOutOfMemory ? GWTF_ERR_OUT_OF_MEMORY : GWTF_ERR_DEVICE, "gwtf_learn_list_create", e);
    }
    *out = list;
    return GWTF_OK;
}

extern "C" void gwtf_learn_list_destroy(gwtf_learn_list_t *list)
{
    if (!list) return;
    DeviceScope scope(list->device);
    if (list->t.base) (void)hipFree(list->t.base); // waits for the device
    delete list;
}

extern "C" gwtf_status_t gwtf_learn_grad_norm(gwtf_learn_t *h, const gwtf_learn_grad_norm_t *a)
{
    LEARN_BEGIN("gwtf_learn_grad_norm")
    LEARN_REQUIRE(a->list, "list is NULL")
    LEARN_REQUIRE(a->list->device == h->device, "the list is on another device")
    LEARN_REQUIRE(a->max_norm >= 0, "max_norm must be >= 0")
    LEARN_REQUIRE(a->scale >= 0 && finite32(a->scale), "scale must be finite in 32 bits and >= 0")
    LEARN_CHECK(a->norm ? bad_vector(a->norm, 1, 4) : nullptr)
    LEARN_CHECK(a->factor ? bad_vector(a->factor, 1, 4) : nullptr)
    if (!a->norm && !a->factor) return GWTF_OK;
    LEARN_LAUNCH("gwtf_learn_grad_norm", launch_grad_norm(*a, a->list->t, h->ws, h->stream))
}

extern "C" gwtf_status_t gwtf_learn_adamw(gwtf_learn_t *h, const gwtf_learn_adamw_t *a)
{
    LEARN_BEGIN("gwtf_learn_adamw")
    LEARN_REQUIRE(a->list, "list is NULL")
    LEARN_REQUIRE(a->list->device == h->device, "the list is on another device")
    LEARN_REQUIRE(a->list->t.form != GWTF_STATE_NONE, "the list has gradients alone")
    LEARN_REQUIRE(a->step_at || a->step >= 1, "step below 1")
    LEARN_REQUIRE(a->lr_at || finite32(a->lr), "lr must be finite in 32 bits")
    LEARN_REQUIRE(a->beta1 >= 0 && float(a->beta1) < 1 && a->beta2 >= 0 && float(a->beta2) < 1, "beta1 or beta2 outside [0, 1)")
    LEARN_REQUIRE(a->eps >= 0 && finite32(a->eps), "eps must be finite in 32 bits and >= 0")
    LEARN_CHECK(a->step_at ? bad_vector(a->step_at, 1, 8) : nullptr)
    LEARN_CHECK(a->lr_at ? bad_vector(a->lr_at, 1, 4) : nullptr)
    LEARN_CHECK(a->factor ? bad_vector(a->factor, 1, 4) : nullptr)
    LEARN_LAUNCH("gwtf_learn_adamw", launch_adamw(*a, a->list->t, h->stream))
}
