// Launchers of the layer norm and its gradients.
#include "alcop_gfx950.hip.h"
#include "alcop_layernorm.h"
namespace alcop {
namespace {
template <class C>
struct Norm {
  static hipError_t go(const LayerNormArgs& a, hipStream_t st)
  {
    alcop_layernorm_rows<C, Gfx950>
        <<<dim3((unsigned)(((long)a.rows + C::ROWS - 1) / C::ROWS)), dim3(C::NT), layernorm_lds<C>(a), st>>>(a);
    return hipGetLastError();
  }
};
template <class C>
struct Grad {
  static hipError_t go(const LayerNormGradArgs& a, int groups, hipStream_t st)
  {
    alcop_layernorm_grad<C, Gfx950><<<dim3((unsigned)(groups / C::ROWS)), dim3(C::NT), layernorm_grad_lds<C>(), st>>>(a, groups);
    return hipGetLastError();
  }
};
template <class C>
struct Load {
  static hipError_t go()
  {
    hipFuncAttributes at;
    const hipError_t rc = hipFuncGetAttributes(&at, (const void*)alcop_layernorm_rows<C, Gfx950>);
    return rc != hipSuccess ? rc : hipFuncGetAttributes(&at, (const void*)alcop_layernorm_grad<C, Gfx950>);
  }
};
}  // namespace

hipError_t launch_layernorm_rows(const LayerNormArgs& a, int dt, bool whole, hipStream_t st)
{
  return dispatch_layernorm<Norm>(dt, whole, a.rows, a.cols, a, st);
}

hipError_t launch_layernorm_grad(const LayerNormGradArgs& a, int groups, int dt, bool whole, hipStream_t st)
{
  return dispatch_layernorm<Grad>(dt, whole, a.rows, a.cols, a, groups, st);
}

hipError_t launch_two_column_sums(const TwoColumnSums& a, int arrays, hipStream_t st)
{
  const dim3 grid((unsigned)((a.of[0].cols + SUM_COLS - 1) / SUM_COLS), (unsigned)arrays);
  alcop_two_column_sums<Gfx950><<<grid, dim3(SUM_THREADS), SUM_THREADS * 4, st>>>(a);
  return hipGetLastError();
}

hipError_t prepare_layernorm()
{
  hipFuncAttributes at;
  const hipError_t rc = hipFuncGetAttributes(&at, (const void*)alcop_two_column_sums<Gfx950>);
  return rc != hipSuccess ? rc : each_layernorm_kernel<Load>();
}

}  // namespace alcop
