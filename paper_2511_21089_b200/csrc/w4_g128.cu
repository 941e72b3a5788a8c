// The 4-bit products with one scale per 128 columns.
#include "w4_kernel.cuh"

namespace mlpmoe {

cudaError_t launch_w4_gateup_128(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 128, true>(a, cluster, st); }
cudaError_t launch_w4_down_128(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 128, false>(a, cluster, st); }

}  // namespace mlpmoe
