// Internal interface between the host API of the learning step's operators
// (learn_api.hip) and their kernels.  Not part of the public C ABI.
#pragma once

#include "gwtf_learn.h"
#include "stage_internal.h" // launch(), kLaunchThreads

namespace gwtf {

// Draws of many rows: the rows that are uncertain after 32-bit sums.
constexpr int kRecheckRows = 4096;  // most rows of such a call
constexpr int kRecheckSlots = 256;  // of them shared by workgroups
constexpr int kRecheckSegs = 1024;
constexpr int kRecheckGroups = 512; // workgroups that share them
struct RecheckWorkspace {
    uint32_t *key = nullptr;     // [kRecheckRows] of an uncertain row's largest entry, 0 of others
    uint32_t *arrived = nullptr; // [kRecheckSlots] 0 between calls
    uint64_t *sum = nullptr;     // [kRecheckSlots][kRecheckSegs] sums of segments
};

// Device workspace of a handle, used in the order of its stream.
struct LearnWorkspace {
    void *base = nullptr; // the allocation that holds the parts
    double *partial = nullptr;   // gradient norm: [kNormSlots] sums of workgroups
    uint32_t *arrived = nullptr; // and how many have arrived, 0 between calls
    RecheckWorkspace recheck;
};

constexpr int kNormGroups = 2048; // most workgroups that sum squares of one type
constexpr int kNormSlots = 3 * kNormGroups + 1;

// A list's tensors on the device, those of the same types side by side, and for
// each chunk of values the tensor that it belongs to.
constexpr int kChunk = 2048; // values: 256 threads, eight each
struct LearnEntry {
    int64_t size;
    const void *grad;
    void *param;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t first; // chunk that it begins with
    float decay;
    uint32_t site;
};
struct LearnTable {
    void *base = nullptr; // the allocation: entries, then the chunks' tensors
    int32_t form = GWTF_STATE_NONE;
    int32_t classes = 0;
    // the chunks of entries of one type each (GWTF_STATE_NONE: of one grad_type)
    struct {
        int32_t type, grad_type;
        int64_t begin, end;
    } cls[9];
    const LearnEntry *entry = nullptr;
    const uint32_t *owner = nullptr;
};
hipError_t build_table(int64_t num, const gwtf_learn_tensor_t *tensors, LearnTable &t);

hipError_t launch_sample(const gwtf_learn_sample_t &a, const LearnWorkspace &w, hipStream_t s);
hipError_t launch_grad_norm(const gwtf_learn_grad_norm_t &a, const LearnTable &t, const LearnWorkspace &w, hipStream_t s);
hipError_t launch_adamw(const gwtf_learn_adamw_t &a, const LearnTable &t, hipStream_t s);

} // namespace gwtf
