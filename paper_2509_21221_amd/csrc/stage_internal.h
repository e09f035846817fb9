// Internal interface between the host API of the microbatch operators
// (stage_api.hip) and their kernels.  Not part of the public C ABI.
#pragma once

#include "gwtf_stage.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

namespace gwtf {

// Device workspace of a handle, used in the order of its stream.
struct StageWorkspace {
    void *base = nullptr;                          // the allocation that holds the parts
    uint64_t *sort_a = nullptr, *sort_b = nullptr; // [max_tokens] each: token << 32 | position
    float *partial = nullptr;                      // embedding gradient: sums of runs that cross chunks
    uint32_t *absent = nullptr;                    // embedding gradient: a bit for each row of the table
    float *dweight = nullptr;                      // norm gradient: [kNormGradGroups][max_hidden]
    unsigned char *logprob = nullptr;              // kLogprobItems records, then kLogprobRows counters (0 between calls)
    int cus = 0;
};

// Embedding gradient: the sorted tokens are dealt out in chunks, one wave per
// chunk and slab of columns, about kEmbedItems of them.
constexpr int64_t kEmbedItems = 4096;
constexpr int kEmbedMinChunk = 4;
int64_t embed_partial_bytes(int64_t max_tokens, int64_t max_hidden);
constexpr int64_t kAbsentRows = int64_t(1) << 22; // tables up to here have their absent rows kept between launches
int64_t embed_absent_bytes(int64_t max_vocab, int cus);

// Norm gradient: most workgroups that sum dweight over their rows.
constexpr int kNormGradGroups = 512;

// Log probabilities: most rows that are split over workgroups, most
// workgroups that then share them, and bytes of one's record.
constexpr int kLogprobRows = 512;
constexpr int kLogprobItems = 2048;
constexpr int kLogprobRecord = 16 + 8 * GWTF_STAGE_MAX_TOP;

// A call that reads and writes this much or more goes past the caches with what
// it touches once, where rows lie on 16-byte boundaries so that no cache line is
// needed twice.  Measured with inputs and results of three calls in turn, bf16,
// through / past: dropout with residual 2,048 x 4096 (50 MB) 9.7 / 10.3 us, 4,096
// (101 MB) 19.1 / 18.6, 8,192 38 / 34, 16,384 72 / 65; norm to 8 bits 12.6 /
// 13.2, 26 / 23, 46 / 41, 84 / 75; its gradient 18.7 / 20.2, 32 / 30, 57 / 52, 104 /
// 95; gradient of log probabilities, 512 x 32,000 (66 MB) 12.8 / 15.1, 2,048 57 /
// 50.  With rows on odd addresses the norm's gradient of 4095 x 1111 f32 takes
// 20 / 28.
constexpr int64_t kStreamBytes = int64_t(96) << 20;
constexpr int64_t kL2Bytes = int64_t(32) << 20; // of all XCDs
// A launch has fewer than 2^32 threads; calls that want more are cut into launches
// of this many at most.
constexpr int64_t kLaunchThreads = int64_t(1) << 31;
inline bool on_lines(const void *p, int64_t stride, size_t size)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * int64_t(size) % 16 == 0;
}

// Enqueues a kernel; the status is the launch's own (that of hipGetLastError may
// be one that an earlier call of the thread, anybody's, has left).
template <class... P>
inline hipError_t launch(void (*kernel)(P...), int64_t groups, int threads, hipStream_t s, std::common_type_t<P>... args)
{
    void *list[] = {&args...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3(uint32_t(groups)), dim3(uint32_t(threads)), list, 0, s);
}

hipError_t launch_embed(const gwtf_stage_embed_t &a, hipStream_t s);
hipError_t launch_embed_grad(const gwtf_stage_embed_grad_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_dropout(const gwtf_stage_dropout_t &a, uint32_t limit, hipStream_t s);
hipError_t launch_norm(const gwtf_stage_norm_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_norm_grad(const gwtf_stage_norm_grad_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_logprob(const gwtf_stage_logprob_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_logprob_grad(const gwtf_stage_logprob_grad_t &a, const StageWorkspace &w, hipStream_t s);

} // namespace gwtf
