// Products grouped by expert on bf16 operands, W stored K x N and N x K.
#include "alcop_instantiate_grouped.hip.h"
namespace alcop {
void register_grouped_bf16(std::vector<GroupedKernel>& t)
{
  ALCOP_GROUPED_KERNELS(t, 1, 0)
  ALCOP_GROUPED_KERNELS(t, 1, 1)
}
}  // namespace alcop
