// Instantiations of the key-owned kernel of the differential-attention
// backward for the widest heads. Keys of 128 with values of 256 columns take
// two launches, dK_1 and dK_2, then dV: their accumulators alone fill half of
// the register file, and one kernel for all three spills (d 128/256, 16 heads
// x 4096: 1192 us in one, 842 in two; d 128/192, which fits: 318 and 445).
#include "diff_bwd.hpp"
#include "diff_launch.hpp"

namespace streamkl {

hipError_t launch_diff_bwd_dkv_wide(const DiffArgs& a) {
  return diff_by_dims(a.d, a.dv, [&](auto kd, auto kv) {
    const dim3 grid((unsigned)((long long)a.B * a.HK * diff_row_blocks(a.NK)), (unsigned)a.k_splits);
    if constexpr (kd.value == 128 && kv.value == 256) {
      if (a.dk1 || a.dk2) {
        hipLaunchKernelGGL((diff_bwd_dkv_kernel<kd.value, kv.value, 1>), grid, dim3(kThreads), 0, a.stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
      if (!a.dv_out) return hipSuccess;
      hipLaunchKernelGGL((diff_bwd_dkv_kernel<kd.value, kv.value, 2>), grid, dim3(kThreads), 0, a.stream, a);
      return hipGetLastError();
    } else if constexpr (kDiffWideKeys<kd.value, kv.value>) {
      hipLaunchKernelGGL((diff_bwd_dkv_kernel<kd.value, kv.value, 3>), grid, dim3(kThreads), 0, a.stream, a);
      return hipGetLastError();
    } else {
      return hipErrorInvalidValue;
    }
  });
}

}  // namespace streamkl
