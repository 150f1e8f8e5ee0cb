// Linear layers on fp16 operands, W stored K x N and N x K.
#include "alcop_instantiate_linear.hip.h"
namespace alcop {
void register_linear_f16(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_KERNELS(t, 0, 0)
  ALCOP_LINEAR_KERNELS(t, 0, 1)
}
}  // namespace alcop
