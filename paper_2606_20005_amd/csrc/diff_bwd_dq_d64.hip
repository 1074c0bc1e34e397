#include "diff_bwd_units.hpp"

namespace streamkl {
template int diff_bwd_dq_waves_of<64>(int dv);
template int diff_bwd_dq_rows_of<64>(int dv);
template hipError_t launch_diff_bwd_dq_of<64>(const DiffArgs& a);
}  // namespace streamkl
