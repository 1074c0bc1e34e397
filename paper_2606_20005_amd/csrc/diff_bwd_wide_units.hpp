// Instantiations of the key-owned kernel of the differential-attention
// backward for one key dim and the values that kDiffWideKeys names.
#pragma once

#include "diff_bwd_units.hpp"

namespace streamkl {

// Head dims that sum to 352 and more take two launches, dK_1 and dK_2, then dV:
// the accumulators and resident rows of one kernel for all three do not fit the
// register file (d 128/256, 16 heads x 4096: 1192 us in one, 842 in two; d 128/192,
// which fits: 318 and 445).
template <int D>
hipError_t launch_diff_bwd_dkv_wide_of(const DiffArgs& a) {
  return diff_by_value_dim(a.dv, [&](auto kv) {
    if constexpr (!kDiffWideKeys<D, kv.value>) {
      return hipErrorInvalidValue;
    } else if constexpr (D + kv.value >= 352) {
      hipError_t e = hipSuccess;
      if (a.dk1 || a.dk2) {
        hipLaunchKernelGGL((diff_bwd_dkv_kernel<D, kv.value, 1>), key_grid(a), dim3(kThreads), 0, a.stream, a);
        e = hipGetLastError();
      }
      if (e == hipSuccess && a.dv_out) {
        hipLaunchKernelGGL((diff_bwd_dkv_kernel<D, kv.value, 2>), key_grid(a), dim3(kThreads), 0, a.stream, a);
        e = hipGetLastError();
      }
      return e;
    } else {
      hipLaunchKernelGGL((diff_bwd_dkv_kernel<D, kv.value, 3>), key_grid(a), dim3(kThreads), 0, a.stream, a);
      return hipGetLastError();
    }
  });
}

}  // namespace streamkl
