#include "diff_fwd_units.hpp"

STREAMKL_DIFF_FWD_UNIT(128)
