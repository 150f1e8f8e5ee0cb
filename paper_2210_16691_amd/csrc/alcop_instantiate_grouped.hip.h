// Launchers and table helpers of the kernels of products grouped by expert.
#pragma once
#include <mutex>

#include "alcop_gfx950.hip.h"
#include "alcop_grouped.h"

namespace alcop {

// The opt-in to the kernel's LDS size, once per kernel and device.
template <class C, auto KERNEL>
hipError_t prepare_kernel()
{
  constexpr int DEVICES = 64;
  static std::once_flag once[DEVICES];
  static hipError_t rc[DEVICES];
  int dev = 0;
  const hipError_t err = hipGetDevice(&dev);
  if (err != hipSuccess || dev < 0 || dev >= DEVICES) return err != hipSuccess ? err : hipErrorInvalidDevice;
  std::call_once(once[dev], [&] {
    rc[dev] = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES);
  });
  return rc[dev];
}
template <class C, auto KERNEL, class A>
hipError_t launch_kernel(const A& a, dim3 grid, hipStream_t st)
{
  const hipError_t rc = prepare_kernel<C, KERNEL>();
  if (rc != hipSuccess) return rc;
  KERNEL<<<grid, dim3(C::NT), C::LDS_BYTES, st>>>(a);
  return hipGetLastError();
}

template <int CL, int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F, int BL>
void add_grouped(std::vector<GroupedKernel>& t)
{
  using C = LCfg<CL, DT, BM, BN, BK, WM, WN, S, R, F, BL>;
  constexpr auto K = &alcop_grouped_tile<C, Gfx950>;
  t.push_back(GroupedKernel{CL, DT, BL, alcop_sched{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0}, C::NT, false,
                            &launch_kernel<C, K, GroupedArgs>, &prepare_kernel<C, K>});
}
template <int CL, int DT, int BM, int BN, int NW, int BL>
void add_grouped_ksplit(std::vector<GroupedKernel>& t)
{
  using C = LWCfg<CL, DT, BM, BN, NW, 2, BL>;
  constexpr auto K = &alcop_grouped_ksplit<C, Gfx950>;
  t.push_back(GroupedKernel{CL, DT, BL, alcop_sched{BM, BN, 64, BM, BN, 2, 1, 0, 1, 0, 3}, C::NT, false,
                            &launch_kernel<C, K, GroupedArgs>, &prepare_kernel<C, K>});
}
template <int CL, int DT, int BM, int BN, int BK, int WM, int WN, int S, int BL>
void add_grouped_quarters(std::vector<GroupedKernel>& t)
{
  using C = LCfg<CL, DT, BM, BN, BK, WM, WN, S, 2, 1, BL>;
  using Q = LCfg<CL, DT, BM / 2, BN / 2, 64, WM / 2, WN / 2, 3, 2, 1, BL>;
  static_assert(C::LDS_BYTES >= Q::LDS_BYTES, "what is asked for is what the whole tiles need");
  constexpr auto K = &alcop_grouped_quarters<C, Q, Gfx950>;
  t.push_back(GroupedKernel{CL, DT, BL, alcop_sched{BM, BN, BK, WM, WN, S, 2, 1, 1, 0, 0}, C::NT, true,
                            &launch_kernel<C, K, GroupedArgs>, &prepare_kernel<C, K>});
}
template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
void add_grouped_grad(std::vector<GroupedGradKernel>& t)
{
  using C = GradCfg<DT, BM, BN, BK, WM, WN, S, R, F>;
  constexpr auto K = &alcop_grouped_grad<C, Gfx950>;
  t.push_back(GroupedGradKernel{DT, alcop_sched{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0}, C::NT, &launch_kernel<C, K, GroupedGradArgs>,
                                &prepare_kernel<C, K>});
}

}  // namespace alcop
