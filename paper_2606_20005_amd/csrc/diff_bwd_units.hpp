// Instantiations of the differential-attention backward for one key dim (one
// unit per kernel and dim, so that they compile side by side). The key-owned
// kernel's widest pairs, one wave of 32 keys per SIMD, are in units of their
// own (diff_bwd_wide_units.hpp), built with other flags (see build.py).
#pragma once

#include "diff_bwd_keys16.hpp"
#include "diff_bwd_rows16.hpp"
#include "diff_launch.hpp"

namespace streamkl {

template <int D>
hipError_t launch_diff_bwd_dkv_wide_of(const DiffArgs& a);

namespace {

inline dim3 key_grid(const DiffArgs& a) {
  return dim3((unsigned)((long long)a.B * a.HK * diff_row_blocks(a.NK)), (unsigned)a.k_splits);
}

}  // namespace

template <int D>
int diff_bwd_dq_waves_of(int dv) {
  return diff_by_value_dim(dv, [](auto kv) { return DiffBwdCfg<D, kv.value>::WAVES_Q; });
}

template <int D>
int diff_bwd_dq_rows_of(int dv) {
  return diff_by_value_dim(dv, [](auto kv) { return kDiffRows16<D, kv.value> ? 64 : 128; });
}

template <int D>
int diff_bwd_dkv_waves_of(int dv) {
  return diff_by_value_dim(dv, [](auto kv) { return DiffBwdCfg<D, kv.value>::WAVES_K; });
}

template <int D>
hipError_t launch_diff_bwd_dq_of(const DiffArgs& a) {
  return diff_by_value_dim(a.dv, [&](auto kv) {
    const dim3 grid((unsigned)((long long)a.B * a.H * a.row_blocks), (unsigned)a.q_splits);
    if constexpr (kDiffRows16<D, kv.value>)
      hipLaunchKernelGGL((diff_bwd_dq16_kernel<D, kv.value>), grid, dim3(kThreads), 0, a.stream, a);
    else
      hipLaunchKernelGGL((diff_bwd_dq_kernel<D, kv.value>), grid, dim3(kThreads), 0, a.stream, a);
    return hipGetLastError();
  });
}

template <int D>
hipError_t launch_diff_bwd_dkv_of(const DiffArgs& a) {
  return diff_by_value_dim(a.dv, [&](auto kv) {
    if constexpr (kDiffKeys16<D, kv.value>) {
      const dim3 grid((unsigned)((long long)a.B * a.HK * ((a.NK + 63LL) / 64)), (unsigned)a.k_splits);
      hipLaunchKernelGGL((diff_bwd_dkv16_kernel<D, kv.value>), grid, dim3(kThreads), 0, a.stream, a);
      return hipGetLastError();
    } else if constexpr (DiffBwdCfg<D, kv.value>::WAVES_K == 1) {
      return launch_diff_bwd_dkv_wide_of<D>(a);
    } else {
      hipLaunchKernelGGL((diff_bwd_dkv_kernel<D, kv.value, 3>), key_grid(a), dim3(kThreads), 0, a.stream, a);
      return hipGetLastError();
    }
  });
}

}  // namespace streamkl
