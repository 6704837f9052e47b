#include "attend_wide.hpp"

namespace lagkv {

hipError_t launch_wide_f16(const AttendArgs& a, int row_tile, hipStream_t s) { return launch_wide_of<LAGKV_F16>(a, row_tile, s); }

}  // namespace lagkv
