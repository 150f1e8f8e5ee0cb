// Tables and launchers of the products grouped by expert, between their host code (alcop_grouped.cpp) and the shards that hold
// the kernels.
#pragma once
#include "alcop_linear.h"
#include "alcop_grouped.hip.h"

namespace alcop {

struct GroupedKernel {
  int cls, dt, bl;             // as in LCfg
  alcop_sched s;
  int threads;
  bool quarters;               // alcop_grouped_quarters
  hipError_t (*launch)(const GroupedArgs&, dim3, hipStream_t);
  hipError_t (*prepare)();
  const LinearCost* cost = nullptr;
};
struct GroupedGradKernel {
  int dt;
  alcop_sched s;
  int threads;
  hipError_t (*launch)(const GroupedGradArgs&, dim3, hipStream_t);
  hipError_t (*prepare)();
  const LinearCost* cost = nullptr;
};
void register_grouped_f16(std::vector<GroupedKernel>&);
void register_grouped_bf16(std::vector<GroupedKernel>&);
void register_grouped_e4m3(std::vector<GroupedKernel>&);
void register_grouped_f8(std::vector<GroupedKernel>&);        // in libalcop_f8.so
void register_grouped_grad(std::vector<GroupedGradKernel>&);

hipError_t launch_grouped_act_grad(const GroupedActGradArgs& a, int dt, int runs, hipStream_t st);
hipError_t launch_grouped_sums(const GroupedSumArgs& a, hipStream_t st);
hipError_t prepare_grouped_rows();
hipError_t prepare_grouped();

}  // namespace alcop

// The kernels of one operand type and layout, each per class of activation: those of a linear layer but for 64x64 tiles of four waves that
// split K and the deeper 128x128, which are for few tiles.
#define ALCOP_GROUPED_CLASS(T, CL, DT, BL)                  \
  add_grouped_ksplit<CL, DT, 16, 16, 8, BL>(T);             \
  add_grouped_ksplit<CL, DT, 16, 32, 8, BL>(T);             \
  add_grouped_ksplit<CL, DT, 32, 32, 8, BL>(T);             \
  add_grouped_ksplit<CL, DT, 32, 64, 4, BL>(T);             \
  add_grouped<CL, DT, 64, 64, 64, 32, 32, 3, 2, 1, BL>(T);  \
  add_grouped<CL, DT, 128, 64, 64, 64, 32, 3, 2, 1, BL>(T); \
  add_grouped<CL, DT, 128, 128, 64, 64, 64, 2, 2, 1, BL>(T); \
  add_grouped_quarters<CL, DT, 256, 128, 64, 128, 64, 3, BL>(T); \
  add_grouped_quarters<CL, DT, 256, 256, 32, 128, 64, 3, BL>(T);
#define ALCOP_GROUPED_KERNELS(T, DT, BL)        \
  ALCOP_GROUPED_CLASS(T, CLASS_PLAIN, DT, BL)   \
  ALCOP_GROUPED_CLASS(T, CLASS_SIGMOID, DT, BL) \
  ALCOP_GROUPED_CLASS(T, CLASS_ERF, DT, BL)
// The kernels that multiply e4m3 as they are.
#define ALCOP_GROUPED_F8(T, CL)                              \
  add_grouped<CL, 3, 64, 64, 64, 32, 32, 3, 2, 1, 1>(T);     \
  add_grouped<CL, 3, 128, 64, 64, 64, 32, 3, 2, 1, 1>(T);    \
  add_grouped<CL, 3, 128, 128, 64, 64, 64, 2, 2, 1, 1>(T);   \
  add_grouped_quarters<CL, 3, 256, 128, 64, 128, 64, 3, 1>(T);  \
  add_grouped_quarters<CL, 3, 256, 256, 64, 128, 64, 2, 1>(T);
#define ALCOP_GROUPED_GRAD(T, DT)                              \
  add_grouped_grad<DT, 64, 64, 64, 32, 32, 3, 2, 1>(T);        \
  add_grouped_grad<DT, 128, 64, 64, 64, 32, 3, 2, 1>(T);       \
  add_grouped_grad<DT, 128, 128, 64, 64, 64, 2, 2, 1>(T);      \
  add_grouped_grad<DT, 256, 128, 64, 128, 64, 3, 2, 1>(T);     \
  add_grouped_grad<DT, 256, 256, 32, 128, 64, 3, 2, 1>(T);
