// Norms of queries and keys with rotary positions: launchers of mrt_norm_rotary.hip.
#pragma once
#include "mrt_internal.hpp"

namespace mrt {

// Workgroups that leave a part of one tensor's weight gradients, at most (one a head, where every head has weights of its own).
constexpr int kMostNormParts = 1024;

hipError_t launch_norm_rotary(const mrt_rotary& r, float eps, const mrt_norm_tensor* x, int n, const void* const* X,
                              const void* const* dY, void* const* out, float* workspace, hipStream_t s);

}  // namespace mrt
