// The 4-bit products with one scale per 128 columns.
#include "w4_wide.cuh"

namespace mlpmoe {

cudaError_t launch_w4_gateup_128(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 128, true>(a, cluster, st); }
cudaError_t launch_w4_down_128(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 128, false>(a, cluster, st); }
cudaError_t launch_w4_wide_gateup_128(const W4WideArgs& a, int chunks, cudaStream_t st) {
  return w4::launch_wide_zero<128 / 128, true>(a, 1, chunks, st);
}
cudaError_t launch_w4_wide_down_128(const W4WideArgs& a, int cluster, int chunks, cudaStream_t st) {
  return w4::launch_wide_zero<128 / 128, false>(a, cluster, chunks, st);
}
cudaError_t launch_w4_digits_128(const W4DigitsArgs& a, cudaStream_t st) { return w4::launch_digits<128 / 128>(a, st); }

}  // namespace mlpmoe
