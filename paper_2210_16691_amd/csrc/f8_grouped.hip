// Products grouped by expert on e4m3 operands that the matrix cores multiply as they are (in libalcop_f8.so, as f8_linear.hip).
#include "alcop_instantiate_grouped.hip.h"
namespace alcop {
void register_grouped_f8(std::vector<GroupedKernel>& t)
{
  ALCOP_GROUPED_F8(t, CLASS_PLAIN)
  ALCOP_GROUPED_F8(t, CLASS_SIGMOID)
  ALCOP_GROUPED_F8(t, CLASS_ERF)
}
}  // namespace alcop
