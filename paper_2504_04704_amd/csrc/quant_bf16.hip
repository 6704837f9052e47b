#include "quant_attend.hpp"

namespace lagkv {

hipError_t launch_quant_bf16(const QuantBoth& a, int64_t groups, int code, int row_tile, hipStream_t s) {
  return launch_quant_of<LAGKV_BF16>(a, groups, code, row_tile, s);
}

}  // namespace lagkv
