// Products of the layer operators, bf16 operands.
#include "gemm_launch.h"

namespace triaccel {
namespace layers {

hipError_t launch_gemm_bf16(Product kind, const GemmPlan& p, const GemmArgs& g, hipStream_t stream) {
  return launch_any<kBF16>(kind, p, g, stream);
}

}  // namespace layers
}  // namespace triaccel
