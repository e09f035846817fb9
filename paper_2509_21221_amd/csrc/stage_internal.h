// Internal interface between the host API of the microbatch operators
// (stage_api.hip) and their kernels.  Not part of the public C ABI.
#pragma once

#include "gwtf_stage.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

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

// A call that reads and writes more than the cache beside the memory holds
// leaves nothing in it for the next one, and goes past the caches with what it
// touches once, where rows lie on 16-byte boundaries so that no cache line is
// needed twice.  Measured with inputs of three states in turn, kept and past:
// dropout with residual, bf16, 8,192 x 4096 (201 MB) 33 / 34 us, 16,384 x 4096
// (403 MB) 72 / 62; norm 43 / 43 and 96 / 81; its gradient (268, 537 MB) 53 / 49
// and 105 / 90; 4,096 x 4096 norm 22 / 24; its gradient of 4095 x 1111 f32 with
// rows on odd addresses 20 / 28.
constexpr int64_t kMemoryCacheBytes = int64_t(256) << 20;
inline bool on_lines(const void *p, int64_t stride, size_t size)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * int64_t(size) % 16 == 0;
}

hipError_t launch_embed(const gwtf_stage_embed_t &a, hipStream_t s);
hipError_t launch_embed_grad(const gwtf_stage_embed_grad_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_dropout(const gwtf_stage_dropout_t &a, uint32_t limit, hipStream_t s);
hipError_t launch_norm(const gwtf_stage_norm_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_norm_grad(const gwtf_stage_norm_grad_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_logprob(const gwtf_stage_logprob_t &a, const StageWorkspace &w, hipStream_t s);
hipError_t launch_logprob_grad(const gwtf_stage_logprob_grad_t &a, const StageWorkspace &w, hipStream_t s);

} // namespace gwtf
