// Products grouped by expert on e4m3 operands, widened to bf16 in registers.
#include "alcop_instantiate_grouped.hip.h"
namespace alcop {
void register_grouped_e4m3(std::vector<GroupedKernel>& t) { ALCOP_GROUPED_KERNELS(t, 2, 1) }
}  // namespace alcop
