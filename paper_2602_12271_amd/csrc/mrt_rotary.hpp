// Rotary positions with three axes: launcher of mrt_rotary.hip.
#pragma once
#include "mrt_internal.hpp"

namespace mrt {

hipError_t launch_rotary(const mrt_rotary& r, const mrt_rotary_tensor* x, int n, const void* const* X, void* const* Y,
                         bool inverse, hipStream_t s);

}  // namespace mrt
