// Launchers of the row operators: norms and their gradients, rows to 8 bits, activation gradients, column sums.
#include "alcop_gfx950.hip.h"
#include "alcop_linear.h"
namespace alcop {
namespace {
template <class C>
struct Norm {
  static hipError_t go(const NormArgs& a, hipStream_t st)
  {
    alcop_norm_rows<C, Gfx950><<<dim3((unsigned)(((long)a.rows + C::ROWS - 1) / C::ROWS)), dim3(C::NT), ROWS_LDS_BYTES, st>>>(a);
    return hipGetLastError();
  }
};
template <class C>
struct NormGrad {
  static hipError_t go(const NormGradArgs& a, int groups, hipStream_t st)
  {
    alcop_norm_grad<C, Gfx950><<<dim3((unsigned)(groups / C::ROWS)), dim3(C::NT), C::GRAD_LDS_BYTES, st>>>(a, groups);
    return hipGetLastError();
  }
};
template <class C>
struct Load {
  static hipError_t go()
  {
    hipFuncAttributes at;
    const hipError_t rc = hipFuncGetAttributes(&at, (const void*)alcop_norm_rows<C, Gfx950>);
    return rc != hipSuccess ? rc : hipFuncGetAttributes(&at, (const void*)alcop_norm_grad<C, Gfx950>);
  }
};
}  // namespace

hipError_t launch_norm_rows(const NormArgs& a, int dt, bool whole, hipStream_t st)
{
  return dispatch_rows_of<Norm>(dt, whole, a.rows, a.cols, a, st);
}

hipError_t launch_norm_grad(const NormGradArgs& a, int groups, int dt, bool whole, hipStream_t st)
{
  return dispatch_rows_of<NormGrad>(dt, whole, a.rows, a.cols, a, groups, st);
}

hipError_t launch_column_sums(const ColumnSumArgs& a, hipStream_t st)
{
  alcop_column_sums<Gfx950><<<dim3((unsigned)((a.cols + SUM_COLS - 1) / SUM_COLS)), dim3(SUM_THREADS), SUM_THREADS * 4, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_act_grad(const ActGradArgs& a, int dt, hipStream_t st)
{
  const dim3 grid((unsigned)((a.N + ACT_COLS - 1) / ACT_COLS), (unsigned)((a.M + a.rows_per_block - 1) / a.rows_per_block));
  if (dt)
    alcop_act_grad<1, Gfx950><<<grid, dim3(256), 4 * ACT_COLS * 4, st>>>(a);
  else
    alcop_act_grad<0, Gfx950><<<grid, dim3(256), 4 * ACT_COLS * 4, st>>>(a);
  return hipGetLastError();
}

hipError_t prepare_rows()
{
  hipFuncAttributes at;
  hipError_t rc = hipFuncGetAttributes(&at, (const void*)alcop_column_sums<Gfx950>);
  if (rc == hipSuccess) rc = hipFuncGetAttributes(&at, (const void*)alcop_act_grad<0, Gfx950>);
  if (rc == hipSuccess) rc = hipFuncGetAttributes(&at, (const void*)alcop_act_grad<1, Gfx950>);
  if (rc == hipSuccess) rc = each_rows_kernel<Load>();
  return rc;
}

}  // namespace alcop
