// Linear layers on e4m3 operands, W stored N x K.
#include "alcop_instantiate_linear.hip.h"
namespace alcop {
void register_linear_e4m3(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_KERNELS(t, 2, 1)
}
}  // namespace alcop
