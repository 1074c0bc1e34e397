// Host-side launchers of the differential-attention kernels.
#pragma once

#include "diff_common.hpp"

namespace streamkl {

constexpr int kDiffMaxSplits = 256;

// Head dims that the kernels are built for: keys 64 and 128, values 64, 128
// and 256. Others run the next one up, with the missing columns read as zeros.
inline bool diff_dims(int d, int dv) {
  return d >= 32 && d <= 128 && d % 32 == 0 && dv >= 32 && dv <= 256 && dv % 32 == 0;
}
inline int diff_key_dim(int d) { return d <= 64 ? 64 : 128; }
inline int diff_value_dim(int dv) { return dv <= 64 ? 64 : dv <= 128 ? 128 : 256; }

// Forward: rows per workgroup for NQ rows of G heads, and workgroups resident on the chip.
int diff_fwd_rows(int d, int dv, long long rows);
int diff_fwd_resident(int d, int dv, long long rows);
hipError_t launch_diff_fwd(const DiffArgs& a);
hipError_t launch_diff_merge(const DiffArgs& a);

// Backward.
size_t diff_bwd_stats_floats(int B, int H, int NQ);
size_t diff_bwd_dlam_floats(int B, int H, int NQ);
hipError_t launch_diff_bwd_prep(const DiffArgs& a);
hipError_t launch_diff_bwd_dq(const DiffArgs& a);
hipError_t launch_diff_bwd_dkv(const DiffArgs& a);
hipError_t launch_diff_bwd_dlam(const DiffArgs& a);

}  // namespace streamkl
