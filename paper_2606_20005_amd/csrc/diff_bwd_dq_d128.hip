#include "diff_bwd_units.hpp"

namespace streamkl {
template int diff_bwd_dq_waves_of<128>(int dv);
template int diff_bwd_dq_rows_of<128>(int dv);
template hipError_t launch_diff_bwd_dq_of<128>(const DiffArgs& a);
}  // namespace streamkl
