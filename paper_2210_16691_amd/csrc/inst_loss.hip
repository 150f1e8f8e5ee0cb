// Kernels of the cross entropy of a vocabulary's product and its gradients.
#include "alcop_instantiate_grouped.hip.h"
#include "alcop_loss.h"
namespace alcop {
namespace {
template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
void add_loss(std::vector<LossKernel>& t)
{
  const alcop_sched s{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0};
  using Strips = LossCfg<false, DT, BM, BN, BK, WM, WN, S, R, F>;
  using Gradient = LossCfg<true, DT, BM, BN, BK, WM, WN, S, R, F>;
  using Dx = DxCfg<DT, BM, BN, BK, WM, WN, S, R, F>;
  using Dw = DwCfg<DT, BM, BN, BK, WM, WN, S, R, F>;
  constexpr auto KS = &alcop_loss_tile<Strips, Gfx950>;
  constexpr auto KG = &alcop_loss_tile<Gradient, Gfx950>;
  constexpr auto KX = &alcop_loss_dx<Dx, Gfx950>;
  constexpr auto KW = &alcop_loss_dw<Dw, Gfx950>;
  t.push_back(LossKernel{LOSS_STRIPS, DT, s, Strips::NT, &launch_kernel<Strips, KS, LossArgs>, nullptr, &prepare_kernel<Strips, KS>});
  t.push_back(LossKernel{LOSS_GRADIENT, DT, s, Gradient::NT, &launch_kernel<Gradient, KG, LossArgs>, nullptr, &prepare_kernel<Gradient, KG>});
  t.push_back(LossKernel{LOSS_DX, DT, s, Dx::NT, nullptr, &launch_kernel<Dx, KX, LossProductArgs>, &prepare_kernel<Dx, KX>});
  t.push_back(LossKernel{LOSS_DW, DT, s, Dw::NT, nullptr, &launch_kernel<Dw, KW, LossProductArgs>, &prepare_kernel<Dw, KW>});
}
}  // namespace

void register_loss(std::vector<LossKernel>& t)
{
  ALCOP_LOSS_KERNELS(t, 0)
  ALCOP_LOSS_KERNELS(t, 1)
}

hipError_t launch_loss_rows(const LossRowsArgs& a, hipStream_t st)
{
  alcop_loss_rows<Gfx950><<<dim3((unsigned)((a.rows + 31L) / 32)), dim3(1024), 1024 * 8, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_loss_scale(const LossScaleArgs& a, hipStream_t st)
{
  alcop_loss_scale<Gfx950><<<dim3(1), dim3(1024), 256, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_round_rows(const RoundArgs& a, hipStream_t st)
{
  alcop_round_rows<Gfx950><<<dim3((unsigned)(((long)a.rows * (a.cols / 8) + 255) / 256)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}
hipError_t prepare_loss_rows()
{
  hipFuncAttributes at;
  hipError_t rc = hipFuncGetAttributes(&at, (const void*)alcop_loss_rows<Gfx950>);
  if (rc == hipSuccess) rc = hipFuncGetAttributes(&at, (const void*)alcop_loss_scale<Gfx950>);
  return rc != hipSuccess ? rc : hipFuncGetAttributes(&at, (const void*)alcop_round_rows<Gfx950>);
}
}  // namespace alcop
