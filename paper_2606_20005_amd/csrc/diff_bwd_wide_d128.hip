#include "diff_bwd_wide_units.hpp"

namespace streamkl {
template hipError_t launch_diff_bwd_dkv_wide_of<128>(const DiffArgs& a);
}  // namespace streamkl
