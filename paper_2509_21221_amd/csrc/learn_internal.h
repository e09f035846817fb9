// Internal interface between the host API of the learning step's operators
// (learn_api.hip) and their kernels.  Not part of the public C ABI.
#pragma once

#include "gwtf_learn.h"
#include "stage_internal.h" // launch(), kLaunchThreads

namespace gwtf {

// Device workspace of a handle, used in the order of its stream.
struct LearnWorkspace {
    double *partial = nullptr; // gradient norm: [kNormSlots] sums of workgroups
    int cus = 0;
};

constexpr int kNormSlots = 1 << 16;

hipError_t launch_sample(const gwtf_learn_sample_t &a, hipStream_t s);
hipError_t launch_grad_norm(const gwtf_learn_grad_norm_t &a, const LearnWorkspace &w, hipStream_t s);
hipError_t launch_adamw(const gwtf_learn_adamw_t &a, hipStream_t s);

} // namespace gwtf
