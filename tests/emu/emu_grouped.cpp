// The products grouped by expert on the functional model: their host code (alcop_grouped.cpp) linked with tables whose launchers
// run the kernel templates on emu_hw.h.
#include <hip/hip_runtime.h>

#include "emu_hw.h"
#include "alcop_grouped.h"

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
  emu::run_grid(&entry<KERNEL, A>, &a, C::NT, C::LDS_BYTES, grid.x, 1, 1);
  return hipSuccess;
}
[[maybe_unused]] hipError_t prepare_none() { return hipSuccess; }

template <int CL, int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F, int BL>
[[maybe_unused]] void add_grouped(std::vector<GroupedKernel>& t)
{
  using C = LCfg<CL, DT, BM, BN, BK, WM, WN, S, R, F, BL>;
  t.push_back(GroupedKernel{CL, DT, BL, alcop_sched{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0}, C::NT, false,
                            &launch_kernel<C, &alcop_grouped_tile<C, emu::Emu>, GroupedArgs>, &prepare_none});
}
template <int CL, int DT, int BM, int BN, int NW, int BL>
[[maybe_unused]] void add_grouped_ksplit(std::vector<GroupedKernel>& t)
{
  using C = LWCfg<CL, DT, BM, BN, NW, 2, BL>;
  t.push_back(GroupedKernel{CL, DT, BL, alcop_sched{BM, BN, 64, BM, BN, 2, 1, 0, 1, 0, 3}, C::NT, false,
                            &launch_kernel<C, &alcop_grouped_ksplit<C, emu::Emu>, GroupedArgs>, &prepare_none});
}
template <int CL, int DT, int BM, int BN, int BK, int WM, int WN, int S, int BL>
[[maybe_unused]] void add_grouped_quarters(std::vector<GroupedKernel>& t)
{
  using C = LCfg<CL, DT, BM, BN, BK, WM, WN, S, 2, 1, BL>;
  using Q = LCfg<CL, DT, BM / 2, BN / 2, 64, WM / 2, WN / 2, 3, 2, 1, BL>;
  static_assert(C::LDS_BYTES >= Q::LDS_BYTES, "what is asked for is what the whole tiles need");
  t.push_back(GroupedKernel{CL, DT, BL, alcop_sched{BM, BN, BK, WM, WN, S, 2, 1, 1, 0, 0}, C::NT, true,
                            &launch_kernel<C, &alcop_grouped_quarters<C, Q, emu::Emu>, GroupedArgs>, &prepare_none});
}
template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
[[maybe_unused]] void add_grouped_grad(std::vector<GroupedGradKernel>& t)
{
  using C = GradCfg<DT, BM, BN, BK, WM, WN, S, R, F>;
  t.push_back(GroupedGradKernel{DT, alcop_sched{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0}, C::NT,
                                &launch_kernel<C, &alcop_grouped_grad<C, emu::Emu>, GroupedGradArgs>, &prepare_none});
}
}  // namespace

#if EMU_PART == 0
void register_grouped_f16(std::vector<GroupedKernel>& t)
{
  ALCOP_GROUPED_KERNELS(t, 0, 0)
  ALCOP_GROUPED_KERNELS(t, 0, 1)
}
#elif EMU_PART == 1
void register_grouped_bf16(std::vector<GroupedKernel>& t)
{
  ALCOP_GROUPED_KERNELS(t, 1, 0)
  ALCOP_GROUPED_KERNELS(t, 1, 1)
}
#elif EMU_PART == 2
void register_grouped_e4m3(std::vector<GroupedKernel>& t) { ALCOP_GROUPED_KERNELS(t, 2, 1) }
#elif EMU_PART == 3
void register_grouped_f8(std::vector<GroupedKernel>& t)
{
  ALCOP_GROUPED_F8(t, CLASS_PLAIN)
  ALCOP_GROUPED_F8(t, CLASS_SIGMOID)
  ALCOP_GROUPED_F8(t, CLASS_ERF)
}
#elif EMU_PART == 4
void register_grouped_grad(std::vector<GroupedGradKernel>& t)
{
  ALCOP_GROUPED_GRAD(t, 0)
  ALCOP_GROUPED_GRAD(t, 1)
}
hipError_t launch_grouped_act_grad(const GroupedActGradArgs& a, int dt, int runs, hipStream_t)
{
  emu::run_grid(dt ? &entry<&alcop_grouped_act_grad<1, emu::Emu>, GroupedActGradArgs>
                   : &entry<&alcop_grouped_act_grad<0, emu::Emu>, GroupedActGradArgs>,
                &a, 256, 4 * ACT_COLS * 4, (unsigned)((a.a.N + ACT_COLS - 1) / ACT_COLS), (unsigned)runs, 1);
  return hipSuccess;
}
hipError_t launch_grouped_sums(const GroupedSumArgs& a, hipStream_t)
{
  emu::run_grid(&entry<&alcop_grouped_sums<emu::Emu>, GroupedSumArgs>, &a, GROUP_SUM_THREADS, GROUP_SUM_THREADS * 4,
                (unsigned)((a.s.cols + SUM_COLS - 1) / SUM_COLS), (unsigned)a.l.groups, 1);
  return hipSuccess;
}
hipError_t prepare_grouped_rows() { return hipSuccess; }
#endif

}  // namespace alcop
