// Products of the layer operators, bf16 operands.
#include "gemm_launch.h"

namespace triaccel {
namespace layers {

hipError_t launch_gemm_bf16(Product kind, const GemmPlan& p, const GemmArgs& g, hipStream_t stream) {
  return launch_any<kBF16>(kind, p, g, stream);
}

hipError_t launch_pair_bf16(bool two_parts, const GemmPlan& px, const GemmPlan& pw, const GemmArgs& x, const GemmArgs& w, hipStream_t stream) {
  return launch_pair_any<kBF16>(two_parts, px, pw, x, w, stream);
}

}  // namespace layers
}  // namespace triaccel
