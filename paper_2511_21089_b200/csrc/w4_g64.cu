// The 4-bit products with one scale per 64 columns.
#include "w4_kernel.cuh"

namespace mlpmoe {

cudaError_t launch_w4_gateup_64(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 64, true>(a, cluster, st); }
cudaError_t launch_w4_down_64(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 64, false>(a, cluster, st); }

}  // namespace mlpmoe
