// Launchers and table helpers of the linear layers' kernels.
#pragma once
#include <mutex>

#include "alcop_gfx950.hip.h"
#include "alcop_linear.h"

namespace alcop {

// The opt-in to the kernel's LDS size, once per kernel and device.
template <class C, void (*KERNEL)(LinearArgs)>
hipError_t prepare_linear()
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

template <class C, void (*KERNEL)(LinearArgs)>
hipError_t launch_linear(const LinearArgs& a, dim3 grid, hipStream_t st)
{
  const hipError_t rc = prepare_linear<C, KERNEL>();
  if (rc != hipSuccess) return rc;
  KERNEL<<<grid, dim3(C::NT), C::LDS_BYTES, st>>>(a);
  return hipGetLastError();
}

template <int CL, int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F, int BL>
void add_linear(std::vector<LinearKernel>& t)
{
  using C = LCfg<CL, DT, BM, BN, BK, WM, WN, S, R, F, BL>;
  constexpr auto K = &alcop_linear_tile<C, Gfx950>;
  t.push_back(LinearKernel{CL, DT, BL, alcop_sched{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0}, C::NT, C::LDS_BYTES,
                           &launch_linear<C, K>, &prepare_linear<C, K>});
}
template <int CL, int DT, int BM, int BN, int NW, int BL>
void add_linear_ksplit(std::vector<LinearKernel>& t)
{
  using C = LWCfg<CL, DT, BM, BN, NW, 2, BL>;
  constexpr auto K = &alcop_linear_ksplit<C, Gfx950>;
  t.push_back(LinearKernel{CL, DT, BL, alcop_sched{BM, BN, 64, BM, BN, 2, 1, 0, 1, 0, 3}, C::NT, C::LDS_BYTES,
                           &launch_linear<C, K>, &prepare_linear<C, K>});
}

}  // namespace alcop
