// The 4-bit products on the 5th-generation tensor cores with one scale per 32 columns.
#include "w4_tc.cuh"

namespace mlpmoe {

cudaError_t launch_w4_tc_gateup_32(const W4TcArgs& a, int cluster, cudaStream_t st) { return w4::launch_tc_any<128 / 32, true>(a, cluster, st); }
cudaError_t launch_w4_tc_down_32(const W4TcArgs& a, int cluster, cudaStream_t st) { return w4::launch_tc_any<128 / 32, false>(a, cluster, st); }

}  // namespace mlpmoe
