// Instantiations of the query-owned kernel of the differential-attention backward.
#include "diff_bwd.hpp"
#include "diff_launch.hpp"

namespace streamkl {

int diff_bwd_dq_waves(int d, int dv) {
  return diff_by_dims(d, dv, [](auto kd, auto kv) { return DiffBwdCfg<kd.value, kv.value>::WAVES_Q; });
}

hipError_t launch_diff_bwd_dq(const DiffArgs& a) {
  return diff_by_dims(a.d, a.dv, [&](auto kd, auto kv) {
    hipLaunchKernelGGL((diff_bwd_dq_kernel<kd.value, kv.value>),
                       dim3((unsigned)((long long)a.B * a.H * diff_row_blocks(a.NQ)), (unsigned)a.q_splits),
                       dim3(kThreads), 0, a.stream, a);
    return hipGetLastError();
  });
}

}  // namespace streamkl
