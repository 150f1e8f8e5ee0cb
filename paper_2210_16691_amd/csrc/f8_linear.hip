// Linear layers on e4m3 operands that the matrix cores multiply as they are.  In a library of its own, libalcop_f8.so: the wait
// states of its matrix instruction are others than those of all kernels of libalcop.so.
#include "alcop_instantiate_linear.hip.h"
namespace alcop {
void register_linear_f8(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_F8(t, CLASS_PLAIN)
  ALCOP_LINEAR_F8(t, CLASS_SIGMOID)
  ALCOP_LINEAR_F8(t, CLASS_ERF)
}
}  // namespace alcop
