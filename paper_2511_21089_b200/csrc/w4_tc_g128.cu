// The 4-bit products on the 5th-generation tensor cores with one scale per 128 columns.
#include "w4_tc.cuh"

namespace mlpmoe {

cudaError_t launch_w4_tc_gateup_128(const W4TcArgs& a, int cluster, cudaStream_t st) { return w4::launch_tc_any<128 / 128, true>(a, cluster, st); }
cudaError_t launch_w4_tc_down_128(const W4TcArgs& a, int cluster, cudaStream_t st) { return w4::launch_tc_any<128 / 128, false>(a, cluster, st); }

cudaError_t launch_w4_columns(const W4ColumnsArgs& a, cudaStream_t st) {
  return launch_pdl(w4::w4_columns_kernel, dim3(static_cast<unsigned>(a.n)), dim3(256), 0, st, a);
}

}  // namespace mlpmoe
