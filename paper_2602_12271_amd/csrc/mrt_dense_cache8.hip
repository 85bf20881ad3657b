// Dense softmax attention over a cache of 8 bits.  Calls of many rows run the kernel of bf16 keys (mrt_dense_bf16.hpp),
// which turns codes into bf16 numbers on their way into LDS.
#include "mrt_dense_bf16.hpp"

namespace mrt {

size_t dense_cache8_workspace_bytes(const KParams& kp, int nbh, int group) { return bf16_dense_workspace_bytes(kp, nbh, true); }

template <bool E4M3>
hipError_t launch_dense_cache8(const KParams& kp, int nbh, void* workspace, size_t workspace_bytes, const DenseCache8<E4M3>& cache, hipStream_t s) {
  const DenseShape shape = dense_call_shape(kp, nbh, workspace ? workspace_bytes : 0, true);
  const size_t rows = (size_t)kp.Nq * nbh * shape.parts;
  const bool even = dense_visible(kp, 0) == dense_visible(kp, kp.Nq - 1);
  const DenseParts parts = {(float*)workspace, (float2*)((float*)workspace + rows * kp.d), shape.parts, (unsigned)nbh,
                            even ? 0u : (unsigned)nbh * shape.parts};
  return run_dense_shape(kp, nbh, shape, parts, cache, s);
}
template hipError_t launch_dense_cache8<true>(const KParams&, int, void*, size_t, const DenseCache8<true>&, hipStream_t);
template hipError_t launch_dense_cache8<false>(const KParams&, int, void*, size_t, const DenseCache8<false>&, hipStream_t);

}  // namespace mrt
