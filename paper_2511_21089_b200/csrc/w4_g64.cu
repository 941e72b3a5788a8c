// The 4-bit products with one scale per 64 columns.
#include "w4_wide.cuh"

namespace mlpmoe {

cudaError_t launch_w4_gateup_64(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 64, true>(a, cluster, st); }
cudaError_t launch_w4_down_64(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 64, false>(a, cluster, st); }
cudaError_t launch_w4_wide_gateup_64(const W4WideArgs& a, int chunks, cudaStream_t st) {
  return w4::launch_wide_zero<128 / 64, true>(a, 1, chunks, st);
}
cudaError_t launch_w4_wide_down_64(const W4WideArgs& a, int cluster, int chunks, cudaStream_t st) {
  return w4::launch_wide_zero<128 / 64, false>(a, cluster, chunks, st);
}
cudaError_t launch_w4_digits_64(const W4DigitsArgs& a, cudaStream_t st) { return w4::launch_digits<128 / 64>(a, st); }

}  // namespace mlpmoe
