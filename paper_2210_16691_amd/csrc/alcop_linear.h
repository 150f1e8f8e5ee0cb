// Tables and launchers of the linear layers and the row operators, between their host code (alcop_linear.cpp) and
// the shards that hold the kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <vector>

#include "../../include/alcop.h"
#include "alcop_rows.hip.h"

namespace alcop {

struct LinearCost;
struct LinearKernel {
  int cls, dt, bl;             // as in LCfg
  alcop_sched s;               // tile and pipelining
  int threads, lds_bytes;
  hipError_t (*launch)(const LinearArgs&, dim3, hipStream_t);
  hipError_t (*prepare)();
  const LinearCost* cost = nullptr;     // alcop_linear_cost.h
};
void register_linear_f16(std::vector<LinearKernel>&);
void register_linear_bf16(std::vector<LinearKernel>&);
void register_linear_e4m3(std::vector<LinearKernel>&);
void register_linear_f8(std::vector<LinearKernel>&);      // in libalcop_f8.so

hipError_t launch_norm_rows(const NormArgs& a, int dt, bool whole, hipStream_t st);
hipError_t launch_norm_grad(const NormGradArgs& a, int groups, int dt, bool whole, hipStream_t st);
hipError_t launch_column_sums(const ColumnSumArgs& a, hipStream_t st);
hipError_t launch_act_grad(const ActGradArgs& a, int dt, hipStream_t st);
hipError_t prepare_rows();

// Threads that share a row, and their chunks of eight elements: a wave, or a block of 256 or 1024.
constexpr int ROWS_MAX_COLS = 32768;
// Whether a wave has a row: up to 1024 columns, and up to 2048 where there are rows enough to fill the card.  1600 columns of
// bf16 with a block for each row and with a wave, us: to 8 bits 512 rows 3.5 and 3.7, 2048 rows 5.1 and 5.3, 32768 rows 43.1 and 31.6;
// norms 3.8 and 4.2, 5.5 and 5.6, 53.9 and 53.9; the norm's gradients 7.8 and 9.1, 12.3 and 10.6, 62.0 and 66.5.
inline bool wave_rows(int rows, int cols) { return cols <= 1024 || (cols <= 2048 && rows >= 1536); }
template <int DT, bool WHOLE, template <class> class LAUNCH, class... A>
hipError_t dispatch_rows(int rows, int cols, const A&... a)
{
  if (cols <= 512) return LAUNCH<RowCfg<DT, 64, 1, WHOLE>>::go(a...);
  if (cols <= 1024) return LAUNCH<RowCfg<DT, 64, 2, WHOLE>>::go(a...);
  if (cols <= 2048 && wave_rows(rows, cols)) return LAUNCH<RowCfg<DT, 64, 4, WHOLE>>::go(a...);
  if (cols <= 2048) return LAUNCH<RowCfg<DT, 256, 1, WHOLE>>::go(a...);
  if (cols <= 4096) return LAUNCH<RowCfg<DT, 256, 2, WHOLE>>::go(a...);
  if (cols <= 8192) return LAUNCH<RowCfg<DT, 256, 4, WHOLE>>::go(a...);
  if (cols <= 16384) return LAUNCH<RowCfg<DT, 1024, 2, WHOLE>>::go(a...);
  return LAUNCH<RowCfg<DT, 1024, 4, WHOLE>>::go(a...);
}
inline int rows_per_block(int rows, int cols) { return wave_rows(rows, cols) ? 4 : 1; }
template <template <class> class LAUNCH, class... A>
hipError_t dispatch_rows_of(int dt, bool whole, int rows, int cols, const A&... a)
{
  if (dt == 0) return whole ? dispatch_rows<0, true, LAUNCH>(rows, cols, a...) : dispatch_rows<0, false, LAUNCH>(rows, cols, a...);
  if (dt == 1) return whole ? dispatch_rows<1, true, LAUNCH>(rows, cols, a...) : dispatch_rows<1, false, LAUNCH>(rows, cols, a...);
  return whole ? dispatch_rows<2, true, LAUNCH>(rows, cols, a...) : dispatch_rows<2, false, LAUNCH>(rows, cols, a...);
}
// All of them: rows and columns that between them reach every line of dispatch_rows.
template <template <class> class LAUNCH, class... A>
hipError_t each_rows_kernel(const A&... a)
{
  static const int sizes[][2] = {{1, 512}, {1, 1024}, {1, 2048}, {1536, 2048}, {1, 4096}, {1, 8192}, {1, 16384}, {1, 32768}};
  hipError_t rc = hipSuccess;
  for (int dt = 0; dt < 3; dt++)
    for (int whole = 0; whole < 2; whole++)
      for (const auto& s : sizes)
        if (rc == hipSuccess) rc = dispatch_rows_of<LAUNCH>(dt, whole, s[0], s[1], a...);
  return rc;
}

// What the first calls of these operators would do besides launching.
hipError_t prepare_layers();

// dW[M,N] = alpha * A^T . B with A stored K x M and B stored K x N, as alcop_gemm computes it, for any K
// (alcop_api.cpp): rows past K lie outside both descriptors.
// Its sum is split over blocks where that pays and the workspace (16-byte aligned) has the room that
// gradient_workspace names.
int gradient_product(const void* A, const void* B, void* C, int M, int N, int K, long lda, long ldb, long ldc,
                     alcop_dtype in, alcop_dtype out, float alpha, void* workspace, size_t workspace_bytes, void* stream);
size_t gradient_workspace(int M, int N, int K);
// What alcop_gemm would answer, without a launch.
int product_check(const void* A, const void* B, const void* C, int M, int N, int K, long lda, long ldb, long ldc, int transA,
                  int transB, alcop_dtype in, alcop_dtype out);

}  // namespace alcop

// The kernels of one operand type and layout, each per class of activation.
#define ALCOP_LINEAR_CLASS(T, CL, DT, BL)                      \
  add_linear_ksplit<CL, DT, 16, 16, 8, BL>(T);                 \
  add_linear_ksplit<CL, DT, 16, 32, 8, BL>(T);                 \
  add_linear_ksplit<CL, DT, 32, 32, 8, BL>(T);                 \
  add_linear_ksplit<CL, DT, 32, 64, 4, BL>(T);                 \
  add_linear_ksplit<CL, DT, 64, 64, 4, BL>(T);                 \
  add_linear<CL, DT, 64, 64, 64, 32, 32, 3, 2, 1, BL>(T);      \
  add_linear<CL, DT, 128, 64, 64, 64, 32, 3, 2, 1, BL>(T);     \
  add_linear<CL, DT, 128, 128, 64, 64, 64, 2, 2, 1, BL>(T);    \
  add_linear<CL, DT, 128, 128, 64, 64, 64, 4, 2, 1, BL>(T);    \
  add_linear<CL, DT, 256, 128, 64, 128, 64, 3, 2, 1, BL>(T);   \
  add_linear<CL, DT, 256, 256, 32, 128, 64, 3, 2, 1, BL>(T);
#define ALCOP_LINEAR_KERNELS(T, DT, BL)     \
  ALCOP_LINEAR_CLASS(T, CLASS_PLAIN, DT, BL)   \
  ALCOP_LINEAR_CLASS(T, CLASS_SIGMOID, DT, BL) \
  ALCOP_LINEAR_CLASS(T, CLASS_ERF, DT, BL)
// The kernels that multiply e4m3 as they are.
#define ALCOP_LINEAR_F8(T, CL)                              \
  add_linear<CL, 3, 64, 64, 64, 32, 32, 3, 2, 1, 1>(T);     \
  add_linear<CL, 3, 128, 64, 64, 64, 32, 3, 2, 1, 1>(T);    \
  add_linear<CL, 3, 128, 128, 64, 64, 64, 2, 2, 1, 1>(T);   \
  add_linear<CL, 3, 128, 128, 64, 64, 64, 4, 2, 1, 1>(T);   \
  add_linear<CL, 3, 256, 128, 64, 128, 64, 3, 2, 1, 1>(T);  \
  add_linear<CL, 3, 256, 256, 64, 128, 64, 2, 2, 1, 1>(T);
