// Host-side launchers of the differential-attention kernels.
#pragma once

#include <type_traits>

#include "diff_common.hpp"

namespace streamkl {

constexpr int kDiffMaxSplits = 256;

// Head dims that the kernels are built for: every multiple of 32, keys to 128,
// values to 256.
inline bool diff_dims(int d, int dv) {
  return d >= 32 && d <= 128 && d % 32 == 0 && dv >= 32 && dv <= 256 && dv % 32 == 0;
}

// f(integral constant) for a supported dim
template <typename F>
auto diff_by_key_dim(int d, F f) {
  switch (d / 32) {
    case 1: return f(std::integral_constant<int, 32>{});
    case 2: return f(std::integral_constant<int, 64>{});
    case 3: return f(std::integral_constant<int, 96>{});
    default: return f(std::integral_constant<int, 128>{});
  }
}
template <typename F>
auto diff_by_value_dim(int dv, F f) {
  switch (dv / 32) {
    case 1: return f(std::integral_constant<int, 32>{});
    case 2: return f(std::integral_constant<int, 64>{});
    case 3: return f(std::integral_constant<int, 96>{});
    case 4: return f(std::integral_constant<int, 128>{});
    case 5: return f(std::integral_constant<int, 160>{});
    case 6: return f(std::integral_constant<int, 192>{});
    case 7: return f(std::integral_constant<int, 224>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}

// Forward: rows per workgroup where a key head serves `rows` packed rows, and a wave's MFMAs per tile.
struct DiffFwdShape {
  int rows, mfmas;
};
// Defined in diff_fwd_units.hpp, instantiated for one key dim per unit.
template <int D>
DiffFwdShape diff_fwd_shape_of(int dv, long long rows);
template <int D>
hipError_t launch_diff_fwd_of(const DiffArgs& a);
hipError_t launch_diff_merge(const DiffArgs& a);

// Backward. Blocks of 128 rows (keys), or twice as many of 64.
constexpr int kDiffMaxGradSplits = 64;
inline int diff_row_blocks(int n) { return (int)((n + 127LL) / 128); }
size_t diff_bwd_stats_floats(int B, int H, int NQ);
size_t diff_bwd_dlam_floats(int B, int H, int NQ, int q_splits);
// Defined in diff_bwd_units.hpp, instantiated for one key dim per unit; waves: per SIMD.
template <int D>
int diff_bwd_dq_waves_of(int dv);
template <int D>
int diff_bwd_dq_rows_of(int dv);   // rows of a workgroup
template <int D>
int diff_bwd_dkv_waves_of(int dv);
template <int D>
hipError_t launch_diff_bwd_dq_of(const DiffArgs& a);
template <int D>
hipError_t launch_diff_bwd_dkv_of(const DiffArgs& a);
hipError_t launch_diff_bwd_prep(const DiffArgs& a);
hipError_t launch_diff_bwd_join_q(const DiffArgs& a);
hipError_t launch_diff_bwd_join_k(const DiffArgs& a);
hipError_t launch_diff_bwd_dlam(const DiffArgs& a);

}  // namespace streamkl
