// Tables and launchers of the cross entropy of a vocabulary's product, between its host code (alcop_loss.cpp) and
// inst_loss.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <vector>

#include "alcop_linear.h"
#include "alcop_loss.hip.h"

namespace alcop {

// what a kernel computes
enum LossStep { LOSS_STRIPS = 0, LOSS_GRADIENT = 1, LOSS_DX = 2, LOSS_DW = 3 };
struct LossKernel {
  int step, dt;
  alcop_sched s;
  int threads;
  hipError_t (*launch)(const LossArgs&, dim3, hipStream_t);                  // the first two steps,
  hipError_t (*launch_product)(const LossProductArgs&, dim3, hipStream_t);   // the others
  hipError_t (*prepare)();
  const LinearCost* cost = nullptr;
};
void register_loss(std::vector<LossKernel>&);

hipError_t launch_loss_rows(const LossRowsArgs& a, hipStream_t st);
hipError_t launch_loss_scale(const LossScaleArgs& a, hipStream_t st);
hipError_t launch_round_rows(const RoundArgs& a, hipStream_t st);
hipError_t prepare_loss_rows();
hipError_t prepare_loss();

template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
using DxCfg = LCfg<CLASS_PLAIN, DT, BM, BN, BK, WM, WN, S, R, F, 0>;
template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
using DwCfg = KCfg<DT, BM, BN, BK, WM, WN, S, R, F, 0, 0, 1>;

}  // namespace alcop

#define ALCOP_LOSS_KERNELS(T, DT)                     \
  add_loss<DT, 64, 64, 64, 32, 32, 3, 2, 1>(T);       \
  add_loss<DT, 128, 64, 64, 64, 32, 3, 2, 1>(T);      \
  add_loss<DT, 128, 128, 64, 64, 64, 2, 2, 1>(T);     \
  add_loss<DT, 256, 128, 64, 128, 64, 3, 2, 1>(T);    \
  add_loss<DT, 256, 256, 32, 128, 64, 3, 2, 1>(T);
