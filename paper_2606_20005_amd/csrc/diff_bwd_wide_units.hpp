// Instantiations of the key-owned kernel of the differential-attention
// backward for one key dim and the values that leave room for one wave of 32
// keys per SIMD and for none of 16 twice: 2 d + dv above 384.
//
// Built without MFMA results kept in the lower half of the register file: from
// 160 accumulator registers on (dK_1, dK_2: d, dV: dv / 2) they do not stay
// there beside three logit tiles and their operands, and those moved up and
// down again for every tile are more than the logits that this form spares
// (measured with this kernel at d 128/128, 8 heads x 6007: 653 us kept low, 634 not;
// 128/96, 16 heads x 4096: 437 and 420; 64/160, 144 registers: 373 and 379).
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
    if constexpr (DiffBwdCfg<D, kv.value>::WAVES_K > 1 || kDiffKeys16<D, kv.value>) {
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
