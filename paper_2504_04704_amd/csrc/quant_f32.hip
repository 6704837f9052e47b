#include "quant_attend.hpp"

namespace lagkv {

hipError_t launch_quant_f32(const QuantBoth& a, int64_t groups, int code, int row_tile, hipStream_t s) {
  return launch_quant_of<LAGKV_F32>(a, groups, code, row_tile, s);
}

}  // namespace lagkv
