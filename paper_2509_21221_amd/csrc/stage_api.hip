// Host side of the C ABI declared in include/gwtf_stage.h: argument checks and
// the handle's workspace.
#include "api_checks.h"
#include "stage_internal.h"

#include <cmath>
#include <cstdio>
#include <new>

using namespace gwtf;

struct gwtf_stage {
    gwtf_stage_shape_t shape;
    hipStream_t stream;
    StageWorkspace ws;
    char err[256];
};

namespace {

thread_local char g_stage_err[256];

gwtf_status_t fail(gwtf_stage_t *h, gwtf_status_t code, const char *what, hipError_t e = hipSuccess)
{
    char *to = h ? h->err : g_stage_err;
    if (e != hipSuccess) (void)hipGetLastError(); // it is reported here, not to the thread's next reader
    if (e != hipSuccess) snprintf(to, sizeof g_stage_err, "%s: %s", what, hipGetErrorString(e));
    else snprintf(to, sizeof g_stage_err, "%s", what);
    return code;
}

bool token_ok(int32_t t) { return t == GWTF_TOKEN_I32 || t == GWTF_TOKEN_I64; }
size_t token_size(int32_t t) { return t == GWTF_TOKEN_I64 ? 8 : 4; }

#define STAGE_BEGIN(name)                                                               \
    if (!h) return fail(nullptr, GWTF_ERR_INVALID_ARG, name ": handle is NULL");        \
    if (!a) return fail(h, GWTF_ERR_INVALID_ARG, name ": arguments are NULL");
#define STAGE_REQUIRE(cond, text) \
    if (!(cond)) return fail(h, GWTF_ERR_INVALID_ARG, text);
#define STAGE_CHECK(expr) \
    if (const char *bad = (expr)) return fail(h, GWTF_ERR_INVALID_ARG, bad);
#define STAGE_LAUNCH(name, expr)                                                        \
    DeviceScope scope(h->shape.device);                                                 \
    if (scope.e != hipSuccess) return fail(h, GWTF_ERR_DEVICE, "hipSetDevice", scope.e); \
    const hipError_t e = (expr);                                                        \
    return e == hipSuccess ? GWTF_OK : fail(h, GWTF_ERR_DEVICE, name " launch", e);

} // namespace

extern "C" gwtf_status_t gwtf_stage_create(const gwtf_stage_shape_t *shape, void *hip_stream, gwtf_stage_t **out)
{
    if (!out) return fail(nullptr, GWTF_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    if (!shape) return fail(nullptr, GWTF_ERR_INVALID_ARG, "shape is NULL");
    const int64_t top = (int64_t(1) << 31) - 1;
    if (shape->max_tokens < 1 || shape->max_tokens > top || shape->max_vocab < 1 || shape->max_vocab > top ||
        shape->max_hidden < 1 || shape->max_hidden > (int64_t(1) << 20))
        return fail(nullptr, GWTF_ERR_INVALID_ARG, "shape values out of range");
    int ndev = 0;
    hipError_t e = hipGetDeviceCount(&ndev);
    if (e != hipSuccess) return fail(nullptr, GWTF_ERR_DEVICE, "hipGetDeviceCount", e);
    if (shape->device < 0 || shape->device >= ndev) return fail(nullptr, GWTF_ERR_INVALID_ARG, "bad device ordinal");
    DeviceScope scope(shape->device);
    if (scope.e != hipSuccess) return fail(nullptr, GWTF_ERR_DEVICE, "hipSetDevice", scope.e);
    gwtf_stage_t *h = new (std::nothrow) gwtf_stage_t();
    if (!h) return fail(nullptr, GWTF_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->shape = *shape;
    h->stream = static_cast<hipStream_t>(hip_stream);
    StageWorkspace &w = h->ws;
    if ((e = hipDeviceGetAttribute(&w.cus, hipDeviceAttributeMultiprocessorCount, shape->device)) != hipSuccess) {
        delete h;
        return fail(nullptr, GWTF_ERR_DEVICE, "hipDeviceGetAttribute", e);
    }
    // one allocation, its parts on 256-byte boundaries
    const size_t lp_records = size_t(kLogprobItems) * kLogprobRecord;
    const int64_t wide = shape->max_hidden < GWTF_STAGE_MAX_HIDDEN ? shape->max_hidden : GWTF_STAGE_MAX_HIDDEN;
    size_t total = 0;
    auto take = [&](size_t bytes) {
        const size_t at = total;
        total += (bytes + 255) / 256 * 256;
        return at;
    };
    const size_t sort_a = take(sizeof(uint64_t) * size_t(shape->max_tokens));
    const size_t sort_b = take(sizeof(uint64_t) * size_t(shape->max_tokens));
    const size_t partial = take(size_t(embed_partial_bytes(shape->max_tokens, shape->max_hidden)));
    const size_t absent = take(size_t(embed_absent_bytes(shape->max_vocab, w.cus)));
    const size_t dweight = take(sizeof(float) * kNormGradGroups * size_t(wide));
    const size_t logprob = take(lp_records + sizeof(uint32_t) * kLogprobRows);
    if ((e = hipMalloc(&w.base, total)) != hipSuccess) {
        delete h;
        return fail(nullptr, GWTF_ERR_OUT_OF_MEMORY, "hipMalloc workspace", e);
    }
    unsigned char *const base = static_cast<unsigned char *>(w.base);
    w.sort_a = reinterpret_cast<uint64_t *>(base + sort_a);
    w.sort_b = reinterpret_cast<uint64_t *>(base + sort_b);
    w.partial = reinterpret_cast<float *>(base + partial);
    w.absent = reinterpret_cast<uint32_t *>(base + absent);
    w.dweight = reinterpret_cast<float *>(base + dweight);
    w.logprob = base + logprob;
    if ((e = hipMemsetAsync(w.logprob + lp_records, 0, sizeof(uint32_t) * kLogprobRows, h->stream)) != hipSuccess) {
        (void)hipFree(w.base);
        delete h;
        return fail(nullptr, GWTF_ERR_DEVICE, "hipMemsetAsync", e);
    }
    *out = h;
    return GWTF_OK;
}

extern "C" void gwtf_stage_destroy(gwtf_stage_t *h)
{
    if (!h) return;
    DeviceScope scope(h->shape.device);
    if (scope.e == hipSuccess) (void)hipStreamSynchronize(h->stream);
    (void)hipFree(h->ws.base);
    delete h;
}

extern "C" const char *gwtf_stage_last_error(const gwtf_stage_t *h) { return h ? h->err : g_stage_err; }

extern "C" gwtf_status_t gwtf_stage_embed(gwtf_stage_t *h, const gwtf_stage_embed_t *a)
{
    STAGE_BEGIN("gwtf_stage_embed")
    const int64_t N = a->num_tokens, H = a->hidden, V = a->vocab;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(H >= 1 && H <= h->shape.max_hidden, "hidden outside [1, max_hidden]")
    STAGE_REQUIRE(V >= 1 && V <= h->shape.max_vocab, "vocab outside [1, max_vocab]")
    STAGE_REQUIRE(type_ok(a->type) && token_ok(a->token_type), "unknown type")
    if (N == 0) return GWTF_OK;
    const size_t z = size_of(a->type);
    STAGE_CHECK(bad_vector(a->tokens, N, token_size(a->token_type)))
    STAGE_CHECK(bad_matrix(a->table, a->table_stride, V, H, z))
    STAGE_CHECK(bad_matrix(a->out, a->out_stride, N, H, z))
    STAGE_LAUNCH("gwtf_stage_embed", launch_embed(*a, h->stream))
}

extern "C" gwtf_status_t gwtf_stage_embed_grad(gwtf_stage_t *h, const gwtf_stage_embed_grad_t *a)
{
    STAGE_BEGIN("gwtf_stage_embed_grad")
    const int64_t N = a->num_tokens, H = a->hidden, V = a->vocab;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(H >= 1 && H <= h->shape.max_hidden, "hidden outside [1, max_hidden]")
    STAGE_REQUIRE(V >= 1 && V <= h->shape.max_vocab, "vocab outside [1, max_vocab]")
    STAGE_REQUIRE(type_ok(a->type) && token_ok(a->token_type), "unknown type")
    STAGE_REQUIRE(a->grad_type == a->type || a->grad_type == GWTF_TYPE_F32, "grad_type must be type or GWTF_TYPE_F32")
    STAGE_CHECK(bad_vector(a->tokens, N, token_size(a->token_type)))
    STAGE_CHECK(bad_matrix(a->dout, a->dout_stride, N, H, size_of(a->type)))
    STAGE_CHECK(bad_matrix(a->grad, a->grad_stride, V, H, size_of(a->grad_type)))
    STAGE_LAUNCH("gwtf_stage_embed_grad", launch_embed_grad(*a, h->ws, h->stream))
}

extern "C" gwtf_status_t gwtf_stage_dropout(gwtf_stage_t *h, const gwtf_stage_dropout_t *a)
{
    STAGE_BEGIN("gwtf_stage_dropout")
    const int64_t N = a->num_tokens, H = a->hidden;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(H >= 1 && H <= h->shape.max_hidden, "hidden outside [1, max_hidden]")
    STAGE_REQUIRE(type_ok(a->type), "unknown type")
    STAGE_REQUIRE(a->p >= 0.0 && a->p < 1.0, "p outside [0, 1)")
    const long limit = std::lrint(a->p * 65536.0);
    STAGE_REQUIRE(limit < 65536, "p rounds to 1 (it is held in 16 bits)")
    if (N == 0) return GWTF_OK;
    const size_t z = size_of(a->type);
    STAGE_CHECK(bad_matrix(a->x, a->x_stride, N, H, z))
    STAGE_CHECK(a->residual ? bad_matrix(a->residual, a->residual_stride, N, H, z) : nullptr)
    STAGE_CHECK(a->rows ? bad_vector(a->rows, N, 8) : nullptr)
    STAGE_CHECK(bad_matrix(a->out, a->out_stride, N, H, z))
    STAGE_LAUNCH("gwtf_stage_dropout", launch_dropout(*a, uint32_t(limit), h->stream))
}

extern "C" gwtf_status_t gwtf_stage_norm(gwtf_stage_t *h, const gwtf_stage_norm_t *a)
{
    STAGE_BEGIN("gwtf_stage_norm")
    const int64_t N = a->num_tokens, H = a->hidden;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(H >= 1 && H <= h->shape.max_hidden && H <= GWTF_STAGE_MAX_HIDDEN,
                  "hidden outside [1, max_hidden] or above GWTF_STAGE_MAX_HIDDEN")
    STAGE_REQUIRE(type_ok(a->type), "unknown type")
    STAGE_REQUIRE(a->form >= GWTF_NORM_PLAIN && a->form <= GWTF_NORM_F8_BLOCK, "unknown form")
    STAGE_REQUIRE(a->eps >= 0.f && a->eps < 1e30f, "eps must be finite and >= 0")
    STAGE_REQUIRE((a->form == GWTF_NORM_PLAIN) == (a->scales == nullptr) || N == 0, "scales must be NULL iff the form is plain")
    if (N == 0) return GWTF_OK;
    const size_t z = size_of(a->type);
    const int64_t groups = a->form == GWTF_NORM_F8_BLOCK ? (H + GWTF_NORM_BLOCK - 1) / GWTF_NORM_BLOCK : 1;
    STAGE_CHECK(bad_matrix(a->x, a->x_stride, N, H, z))
    STAGE_CHECK(a->residual ? bad_matrix(a->residual, a->residual_stride, N, H, z) : nullptr)
    STAGE_CHECK(bad_vector(a->weight, H, z))
    STAGE_CHECK(bad_matrix(a->y, a->y_stride, N, H, a->form == GWTF_NORM_PLAIN ? z : 1))
    STAGE_CHECK(a->h_out ? bad_matrix(a->h_out, a->h_stride, N, H, z) : nullptr)
    STAGE_CHECK(a->scales ? bad_vector(a->scales, N * groups, 4) : nullptr)
    STAGE_CHECK(a->rstd ? bad_vector(a->rstd, N, 4) : nullptr)
    STAGE_LAUNCH("gwtf_stage_norm", launch_norm(*a, h->ws, h->stream))
}

extern "C" gwtf_status_t gwtf_stage_norm_grad(gwtf_stage_t *h, const gwtf_stage_norm_grad_t *a)
{
    STAGE_BEGIN("gwtf_stage_norm_grad")
    const int64_t N = a->num_tokens, H = a->hidden;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(H >= 1 && H <= h->shape.max_hidden && H <= GWTF_STAGE_MAX_HIDDEN,
                  "hidden outside [1, max_hidden] or above GWTF_STAGE_MAX_HIDDEN")
    STAGE_REQUIRE(type_ok(a->type), "unknown type")
    const size_t z = size_of(a->type);
    STAGE_CHECK(bad_matrix(a->dy, a->dy_stride, N, H, z))
    STAGE_CHECK(bad_matrix(a->h, a->h_stride, N, H, z))
    STAGE_CHECK(a->dh ? bad_matrix(a->dh, a->dh_stride, N, H, z) : nullptr)
    STAGE_CHECK(N ? bad_vector(a->weight, H, z) : nullptr)
    STAGE_CHECK(bad_vector(a->rstd, N, 4))
    STAGE_CHECK(bad_matrix(a->dx, a->dx_stride, N, H, z))
    STAGE_CHECK(a->dweight ? bad_vector(a->dweight, H, 4) : nullptr)
    STAGE_LAUNCH("gwtf_stage_norm_grad", launch_norm_grad(*a, h->ws, h->stream))
}

extern "C" gwtf_status_t gwtf_stage_logprob(gwtf_stage_t *h, const gwtf_stage_logprob_t *a)
{
    STAGE_BEGIN("gwtf_stage_logprob")
    const int64_t N = a->num_tokens, V = a->vocab;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(V >= 1 && V <= h->shape.max_vocab, "vocab outside [1, max_vocab]")
    STAGE_REQUIRE(type_ok(a->type) && token_ok(a->token_type), "unknown type")
    STAGE_REQUIRE(a->top >= 0 && a->top <= GWTF_STAGE_MAX_TOP && a->top <= V, "top outside [0, min(vocab, GWTF_STAGE_MAX_TOP)]")
    if (N == 0) return GWTF_OK;
    STAGE_REQUIRE((a->targets == nullptr) == (a->logp == nullptr), "targets must be NULL iff logp is")
    STAGE_REQUIRE((a->top == 0) == (a->top_logp == nullptr) && (a->top == 0) == (a->top_ids == nullptr),
                  "top_logp and top_ids must be NULL iff top is 0")
    STAGE_CHECK(bad_matrix(a->logits, a->logits_stride, N, V, size_of(a->type)))
    STAGE_CHECK(a->targets ? bad_vector(a->targets, N, token_size(a->token_type)) : nullptr)
    STAGE_CHECK(a->logp ? bad_vector(a->logp, N, 4) : nullptr)
    STAGE_CHECK(a->entropy ? bad_vector(a->entropy, N, 4) : nullptr)
    STAGE_CHECK(a->lse ? bad_vector(a->lse, N, 4) : nullptr)
    STAGE_CHECK(a->top ? bad_vector(a->top_logp, N * a->top, 4) : nullptr)
    STAGE_CHECK(a->top ? bad_vector(a->top_ids, N * a->top, 4) : nullptr)
    STAGE_LAUNCH("gwtf_stage_logprob", launch_logprob(*a, h->ws, h->stream))
}

extern "C" gwtf_status_t gwtf_stage_logprob_grad(gwtf_stage_t *h, const gwtf_stage_logprob_grad_t *a)
{
    STAGE_BEGIN("gwtf_stage_logprob_grad")
    const int64_t N = a->num_tokens, V = a->vocab;
    STAGE_REQUIRE(N >= 0 && N <= h->shape.max_tokens, "num_tokens outside [0, max_tokens]")
    STAGE_REQUIRE(V >= 1 && V <= h->shape.max_vocab, "vocab outside [1, max_vocab]")
    STAGE_REQUIRE(type_ok(a->type) && token_ok(a->token_type), "unknown type")
    if (N == 0) return GWTF_OK;
    STAGE_REQUIRE((a->targets == nullptr) == (a->dlogp == nullptr), "targets must be NULL iff dlogp is")
    STAGE_REQUIRE((a->entropy == nullptr) == (a->dentropy == nullptr), "entropy must be NULL iff dentropy is")
    const size_t z = size_of(a->type);
    STAGE_CHECK(bad_matrix(a->logits, a->logits_stride, N, V, z))
    STAGE_CHECK(a->targets ? bad_vector(a->targets, N, token_size(a->token_type)) : nullptr)
    STAGE_CHECK(bad_vector(a->lse, N, 4))
    STAGE_CHECK(a->entropy ? bad_vector(a->entropy, N, 4) : nullptr)
    STAGE_CHECK(a->dlogp ? bad_vector(a->dlogp, N, 4) : nullptr)
    STAGE_CHECK(a->dentropy ? bad_vector(a->dentropy, N, 4) : nullptr)
    STAGE_CHECK(bad_matrix(a->dlogits, a->dlogits_stride, N, V, z))
    STAGE_LAUNCH("gwtf_stage_logprob_grad", launch_logprob_grad(*a, h->ws, h->stream))
}
