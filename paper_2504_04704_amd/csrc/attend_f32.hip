#include "attend_pass.hpp"

namespace lagkv {

hipError_t launch_attend_f32(const AttendArgs& a, int row_tile, int waves, hipStream_t s) {
  return launch_attend_of<LAGKV_F32>(a, row_tile, waves, s);
}

}  // namespace lagkv
