// Host-side launchers of the differential-attention kernels.
#pragma once

#include <type_traits>

#include "diff_common.hpp"

namespace streamkl {

constexpr int kDiffMaxSplits = 256;

// Head dims that the kernels are built for: keys 64 and 128, values 64, 128,
// 192 and 256. Others run the next one up, with the missing columns read as zeros.
inline bool diff_dims(int d, int dv) {
  return d >= 32 && d <= 128 && d % 32 == 0 && dv >= 32 && dv <= 256 && dv % 32 == 0;
}

// f(key dim, value dim) for the compile-time dims that serve d and dv
template <typename F>
auto diff_by_dims(int d, int dv, F f) {
  auto by_dv = [&](auto kd) {
    switch ((dv + 63) / 64) {
      case 1: return f(kd, std::integral_constant<int, 64>{});
      case 2: return f(kd, std::integral_constant<int, 128>{});
      case 3: return f(kd, std::integral_constant<int, 192>{});
      default: return f(kd, std::integral_constant<int, 256>{});
    }
  };
  return d <= 64 ? by_dv(std::integral_constant<int, 64>{}) : by_dv(std::integral_constant<int, 128>{});
}

// Dims of the key-owned backward kernel that are built without the MFMA
// results kept in the lower half of the register file (see build.py).
template <int D, int DV>
constexpr bool kDiffWideKeys = D + DV > 256;

// Forward: rows per workgroup where a key head serves `rows` packed rows, and a wave's MFMAs per tile.
struct DiffFwdShape {
  int rows, mfmas;
};
DiffFwdShape diff_fwd_shape(int d, int dv, long long rows);
hipError_t launch_diff_fwd(const DiffArgs& a);
hipError_t launch_diff_merge(const DiffArgs& a);

// Backward. Blocks of 128 rows (keys).
constexpr int kDiffMaxGradSplits = 64;
inline int diff_row_blocks(int n) { return (int)((n + 127LL) / 128); }
size_t diff_bwd_stats_floats(int B, int H, int NQ);
size_t diff_bwd_dlam_floats(int B, int H, int NQ, int q_splits);
// waves per SIMD of the two kernels
int diff_bwd_dq_waves(int d, int dv);
int diff_bwd_dkv_waves(int d, int dv);
hipError_t launch_diff_bwd_prep(const DiffArgs& a);
hipError_t launch_diff_bwd_dq(const DiffArgs& a);
hipError_t launch_diff_bwd_dkv(const DiffArgs& a);
hipError_t launch_diff_bwd_dkv_wide(const DiffArgs& a);
hipError_t launch_diff_bwd_join_q(const DiffArgs& a);
hipError_t launch_diff_bwd_join_k(const DiffArgs& a);
hipError_t launch_diff_bwd_dlam(const DiffArgs& a);

}  // namespace streamkl
