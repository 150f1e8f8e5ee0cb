// Gradients of products grouped by expert: the weights' products, activations, the biases' sums.
#include "alcop_instantiate_grouped.hip.h"
namespace alcop {
void register_grouped_grad(std::vector<GroupedGradKernel>& t)
{
  ALCOP_GROUPED_GRAD(t, 0)
  ALCOP_GROUPED_GRAD(t, 1)
}

hipError_t launch_grouped_act_grad(const GroupedActGradArgs& a, int dt, int runs, hipStream_t st)
{
  const dim3 grid((unsigned)((a.a.N + ACT_COLS - 1) / ACT_COLS), (unsigned)runs);
  if (dt)
    alcop_grouped_act_grad<1, Gfx950><<<grid, dim3(256), 4 * ACT_COLS * 4, st>>>(a);
  else
    alcop_grouped_act_grad<0, Gfx950><<<grid, dim3(256), 4 * ACT_COLS * 4, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_grouped_sums(const GroupedSumArgs& a, hipStream_t st)
{
  const dim3 grid((unsigned)((a.s.cols + SUM_COLS - 1) / SUM_COLS), (unsigned)a.l.groups);
  alcop_grouped_sums<Gfx950><<<grid, dim3(GROUP_SUM_THREADS), GROUP_SUM_THREADS * 4, st>>>(a);
  return hipGetLastError();
}

hipError_t prepare_grouped_rows()
{
  hipFuncAttributes at;
  hipError_t rc = hipFuncGetAttributes(&at, (const void*)alcop_grouped_act_grad<0, Gfx950>);
  if (rc == hipSuccess) rc = hipFuncGetAttributes(&at, (const void*)alcop_grouped_act_grad<1, Gfx950>);
  return rc != hipSuccess ? rc : hipFuncGetAttributes(&at, (const void*)alcop_grouped_sums<Gfx950>);
}
}  // namespace alcop
