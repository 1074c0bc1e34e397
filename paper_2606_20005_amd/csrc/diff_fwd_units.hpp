// Instantiations of the differential-attention forward for one key dim (one
// unit each, so that they compile side by side), and the rule that picks
// among them.
#pragma once

#include "diff_fwd.hpp"
#include "diff_launch.hpp"

namespace streamkl {

namespace {

template <int D, int DV, int RB, int NW>
struct FwdPick {
  using C = DiffFwdCfg<D, DV, RB, NW>;
  static constexpr DiffFwdShape shape() { return {C::ROWS, RB * (D / 16 + DV / 16)}; }
  static hipError_t launch(const DiffArgs& a) {
    const long long R = (long long)a.NQ * (a.H / a.HK);
    const unsigned grid = (unsigned)((long long)a.B * a.HK * ((R + C::ROWS - 1) / C::ROWS));
    hipLaunchKernelGGL((diff_fwd_kernel<D, DV, RB, NW>), dim3(grid, (unsigned)a.splits), dim3(C::NT), 0, a.stream, a);
    return hipGetLastError();
  }
};

// A pair of waves takes two 32-row blocks where its registers then leave room
// for two waves per SIMD, one where they do not (d 128/128, 8 heads x 6007,
// same card: 351 us with one block and two waves per SIMD, 423 with two blocks
// and one). Few rows run in one pair of waves (a whole workgroup would be
// mostly padding, and short ones leave more of them resident).
template <int D, typename F>
auto pick(int dv, long long rows, F f) {
  return diff_by_value_dim(dv, [&](auto kv) {
    constexpr int DV = kv.value;
    constexpr int RB = DiffFwdCfg<D, DV, 2, 4>::WAVES >= 2 ? 2 : 1;
    if (rows <= 32) return f(FwdPick<D, DV, 1, 2>{});
    if constexpr (RB == 2) {
      if (rows <= 64) return f(FwdPick<D, DV, 2, 2>{});
    }
    return f(FwdPick<D, DV, RB, 4>{});
  });
}

}  // namespace

template <int D>
DiffFwdShape diff_fwd_shape_of(int dv, long long rows) {
  return pick<D>(dv, rows, [](auto p) { return p.shape(); });
}

template <int D>
hipError_t launch_diff_fwd_of(const DiffArgs& a) {
  return pick<D>(a.dv, (long long)a.NQ * (a.H / a.HK), [&](auto p) { return p.launch(a); });
}

}  // namespace streamkl

#define STREAMKL_DIFF_FWD_UNIT(D)                                          \
  namespace streamkl {                                                     \
  template DiffFwdShape diff_fwd_shape_of<D>(int dv, long long rows);      \
  template hipError_t launch_diff_fwd_of<D>(const DiffArgs& a);            \
  }
