// Instantiations of the key-owned kernel of the differential-attention
// backward whose registers fit with the MFMA results in the lower half of the
// register file; the others are in diff_bwd_wide_inst.hip.
#include "diff_bwd.hpp"
#include "diff_launch.hpp"

namespace streamkl {

int diff_bwd_dkv_waves(int d, int dv) {
  return diff_by_dims(d, dv, [](auto kd, auto kv) { return DiffBwdCfg<kd.value, kv.value>::WAVES_K; });
}

hipError_t launch_diff_bwd_dkv(const DiffArgs& a) {
  return diff_by_dims(a.d, a.dv, [&](auto kd, auto kv) {
    if constexpr (kDiffWideKeys<kd.value, kv.value>) {
      return launch_diff_bwd_dkv_wide(a);
    } else {
      hipLaunchKernelGGL((diff_bwd_dkv_kernel<kd.value, kv.value, 3>),
                         dim3((unsigned)((long long)a.B * a.HK * diff_row_blocks(a.NK)), (unsigned)a.k_splits),
                         dim3(kThreads), 0, a.stream, a);
      return hipGetLastError();
    }
  });
}

}  // namespace streamkl
