// Products of the layer operators, fp32 operands.
#include "gemm_launch.h"

namespace triaccel {
namespace layers {

hipError_t launch_gemm_fp32(Product kind, const GemmPlan& p, const GemmArgs& g, hipStream_t stream) {
  return launch_any<kFP32>(kind, p, g, stream);
}

hipError_t launch_pair_fp32(bool two_parts, const GemmPlan& px, const GemmPlan& pw, const GemmArgs& x, const GemmArgs& w, hipStream_t stream) {
  return launch_pair_any<kFP32>(two_parts, px, pw, x, w, stream);
}

}  // namespace layers
}  // namespace triaccel
