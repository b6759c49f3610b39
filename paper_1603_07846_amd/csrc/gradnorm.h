// gradnorm.h -- launcher of the global gradient norm and clipping.
#pragma once

#include "internal.h"

namespace singa {

constexpr int NORM_LIST = 112;     // tensors a launch (their list stays below 4 KB of arguments)
constexpr int NORM_PIECES = 4096;  // whole pieces of the largest lists

// One slot per workgroup: at most NORM_PIECES whole pieces and one part of a
// piece per tensor.
inline size_t norm_slots(int count) { return (size_t)NORM_PIECES + count + 1; }

// stat = (norm, scale); outs (may be null): scale * grads.
hipError_t launch_grad_norm(int count, const int* dt, const void* const* grads, void* const* outs, const size_t* sizes,
                            float max_norm, float* stat, double* slots, hipStream_t st);

}  // namespace singa
