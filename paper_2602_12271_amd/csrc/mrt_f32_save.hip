// fp32 path: the dense attention that keeps its row statistics, for calls whose queries fill the chip
// (mrt_dense_fwd_f32.hip has the others, and rows that do not move as quads).  A file of its own, so that these kernels
// compile beside the others.
//
// At 128 features they keep more registers in memory than the kernels without statistics: 73 a lane instead of 35 in
// fp32 storage, 115 instead of 40 under a mask or lengths; 147 instead of 67 and 222 instead of 58 in bf16 storage (none at
// 64 features).  In fp32 storage that shows (us with statistics | without: 12 heads of 4680 tokens 1006 | 954, given
// lengths 1339; 16 heads of 5400 tokens in chunks of 1800 1544 | 1228); in bf16 storage these calls are ahead of those
// without statistics (895 | 1257, 1075 | 1263).
#include "mrt_f32_kernels.hpp"

namespace mrt {

namespace {

template <int D, typename TIn>
hipError_t run(const KParams& kp, dim3 grid, const DenseSave& save, hipStream_t s) {
  if (kp.cc > 0 || save.kv_len) k_f32_dense<D, TIn, true, true><<<grid, 64 * kDenseWaves32, 0, s>>>(kp, save);
  else k_f32_dense<D, TIn, true, false><<<grid, 64 * kDenseWaves32, 0, s>>>(kp, save);
  return hipGetLastError();
}
template <typename TIn>
hipError_t run_t(const KParams& kp, dim3 grid, const DenseSave& save, hipStream_t s) {
  return kp.d <= 64 ? run<64, TIn>(kp, grid, save, s) : run<128, TIn>(kp, grid, save, s);
}

}  // namespace

hipError_t launch_f32_dense_save(const KParams& kp, int dtype, int nbh, const DenseSave& save, hipStream_t s) {
  const dim3 grid((kp.Nq + kDenseQ32 - 1) / kDenseQ32, nbh);
  return dtype == MRT_F32 ? run_t<float>(kp, grid, save, s) : run_t<u16>(kp, grid, save, s);
}

}  // namespace mrt
