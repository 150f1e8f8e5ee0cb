// The cross entropy of a vocabulary's product on the functional model: its host code (alcop_loss.cpp) linked with launchers that run
// the kernel templates on emu_hw.h.
#include <hip/hip_runtime.h>

#include "emu_hw.h"
#include "alcop_loss.h"

namespace alcop {

namespace {
template <auto KERNEL, class A>
void entry(const void* p)
{
  KERNEL(*(const A*)p);
}
template <class C, auto KERNEL, class A>
hipError_t launch_kernel(const A& a, dim3 grid, hipStream_t)
{
  emu::run_grid(&entry<KERNEL, A>, &a, C::NT, C::LDS_BYTES, grid.x, grid.y, 1);
  return hipSuccess;
}
[[maybe_unused]] hipError_t prepare_none() { return hipSuccess; }

template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
[[maybe_unused]] void add_loss(std::vector<LossKernel>& t)
{
  const alcop_sched s{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0};
  using Strips = LossCfg<false, DT, BM, BN, BK, WM, WN, S, R, F>;
  using Gradient = LossCfg<true, DT, BM, BN, BK, WM, WN, S, R, F>;
  using Dx = DxCfg<DT, BM, BN, BK, WM, WN, S, R, F>;
  using Dw = DwCfg<DT, BM, BN, BK, WM, WN, S, R, F>;
  t.push_back(LossKernel{LOSS_STRIPS, DT, s, Strips::NT, &launch_kernel<Strips, &alcop_loss_tile<Strips, emu::Emu>, LossArgs>,
                         nullptr, &prepare_none});
  t.push_back(LossKernel{LOSS_GRADIENT, DT, s, Gradient::NT, &launch_kernel<Gradient, &alcop_loss_tile<Gradient, emu::Emu>, LossArgs>,
                         nullptr, &prepare_none});
  t.push_back(LossKernel{LOSS_DX, DT, s, Dx::NT, nullptr, &launch_kernel<Dx, &alcop_loss_dx<Dx, emu::Emu>, LossProductArgs>,
                         &prepare_none});
  t.push_back(LossKernel{LOSS_DW, DT, s, Dw::NT, nullptr, &launch_kernel<Dw, &alcop_loss_dw<Dw, emu::Emu>, LossProductArgs>,
                         &prepare_none});
}
}  // namespace

void register_loss_f16(std::vector<LossKernel>&);
void register_loss_bf16(std::vector<LossKernel>&);
#if EMU_PART == 0
void register_loss_f16(std::vector<LossKernel>& t) { ALCOP_LOSS_KERNELS(t, 0) }
#elif EMU_PART == 1
void register_loss_bf16(std::vector<LossKernel>& t) { ALCOP_LOSS_KERNELS(t, 1) }
#else
void register_loss(std::vector<LossKernel>& t)
{
  register_loss_f16(t);
  register_loss_bf16(t);
}
hipError_t launch_loss_rows(const LossRowsArgs& a, hipStream_t)
{
  emu::run_grid(&entry<&alcop_loss_rows<emu::Emu>, LossRowsArgs>, &a, 1024, 1024 * 8, (unsigned)((a.rows + 31L) / 32), 1, 1);
  return hipSuccess;
}
hipError_t launch_loss_scale(const LossScaleArgs& a, hipStream_t)
{
  emu::run_grid(&entry<&alcop_loss_scale<emu::Emu>, LossScaleArgs>, &a, 1024, 256, 1, 1, 1);
  return hipSuccess;
}
hipError_t launch_round_rows(const RoundArgs& a, hipStream_t)
{
  emu::run_grid(&entry<&alcop_round_rows<emu::Emu>, RoundArgs>, &a, 256, 64, (unsigned)(((long)a.rows * (a.cols / 8) + 255) / 256), 1, 1);
  return hipSuccess;
}
hipError_t prepare_loss_rows() { return hipSuccess; }
#endif

}  // namespace alcop
