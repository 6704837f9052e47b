#include "quant_wide.hpp"

namespace lagkv {

hipError_t launch_quant_wide_f16(const QuantBoth& a, int64_t groups, int code, hipStream_t s) {
  return launch_quant_wide_of<LAGKV_F16>(a, groups, code, s);
}

}  // namespace lagkv
