// Products of the layer operators, fp32 operands.
#include "gemm_launch.h"

namespace triaccel {
namespace layers {

hipError_t launch_gemm_fp32(Product kind, const GemmPlan& p, const GemmArgs& g, hipStream_t stream) {
  return launch_any<kFP32>(kind, p, g, stream);
}

}  // namespace layers
}  // namespace triaccel
