// The 4-bit products with one scale per 32 columns.
#include "w4_kernel.cuh"

namespace mlpmoe {

cudaError_t launch_w4_gateup_32(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 32, true>(a, cluster, st); }
cudaError_t launch_w4_down_32(const W4Args& a, int cluster, cudaStream_t st) { return w4::launch_zero<128 / 32, false>(a, cluster, st); }

}  // namespace mlpmoe
