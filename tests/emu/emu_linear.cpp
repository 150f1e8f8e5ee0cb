// The linear layers and the row operators on the functional model: their host code (alcop_linear.cpp) linked with
// tables whose launchers run the kernel templates on emu_hw.h.
#include <hip/hip_runtime.h>

#include <set>

#include "emu_hw.h"
#include "alcop_linear.h"

namespace alcop {

template <class C>
static void tile_entry(const void* p)
{
  alcop_linear_tile<C, emu::Emu>(*(const LinearArgs*)p);
}
template <class C>
static void ksplit_entry(const void* p)
{
  alcop_linear_ksplit<C, emu::Emu>(*(const LinearArgs*)p);
}
template <class C, void (*ENTRY)(const void*)>
static hipError_t launch_linear(const LinearArgs& a, dim3 grid, hipStream_t)
{
  emu::run_grid(ENTRY, &a, C::NT, C::LDS_BYTES, grid.x, 1, 1);
  return hipSuccess;
}
static hipError_t prepare_none() { return hipSuccess; }

template <int CL, int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F, int BL>
void add_linear(std::vector<LinearKernel>& t)
{
  using C = LCfg<CL, DT, BM, BN, BK, WM, WN, S, R, F, BL>;
  t.push_back(LinearKernel{CL, DT, BL, alcop_sched{BM, BN, BK, WM, WN, S, R, F, 1, 0, 0}, C::NT, C::LDS_BYTES,
                           &launch_linear<C, &tile_entry<C>>, &prepare_none});
}
template <int CL, int DT, int BM, int BN, int NW, int BL>
void add_linear_ksplit(std::vector<LinearKernel>& t)
{
  using C = LWCfg<CL, DT, BM, BN, NW, 2, BL>;
  t.push_back(LinearKernel{CL, DT, BL, alcop_sched{BM, BN, 64, BM, BN, 2, 1, 0, 1, 0, 3}, C::NT, C::LDS_BYTES,
                           &launch_linear<C, &ksplit_entry<C>>, &prepare_none});
}

#if EMU_PART == 0
void register_linear_f16(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_KERNELS(t, 0, 0)
  ALCOP_LINEAR_KERNELS(t, 0, 1)
}
#elif EMU_PART == 1
void register_linear_bf16(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_KERNELS(t, 1, 0)
  ALCOP_LINEAR_KERNELS(t, 1, 1)
}
#elif EMU_PART == 2
void register_linear_e4m3(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_KERNELS(t, 2, 1)
}
#elif EMU_PART == 4
void register_linear_f8(std::vector<LinearKernel>& t)
{
  ALCOP_LINEAR_F8(t, CLASS_PLAIN)
  ALCOP_LINEAR_F8(t, CLASS_SIGMOID)
  ALCOP_LINEAR_F8(t, CLASS_ERF)
}
#elif EMU_PART == 3
template <class C>
struct Norm {
  static void entry(const void* p) { alcop_norm_rows<C, emu::Emu>(*(const NormArgs*)p); }
  static hipError_t go(const NormArgs& a, hipStream_t)
  {
    emu::run_grid(&entry, &a, C::NT, ROWS_LDS_BYTES, (unsigned)((a.rows + C::ROWS - 1) / C::ROWS), 1, 1);
    return hipSuccess;
  }
};
template <class C>
struct NormGrad {
  struct Both {
    NormGradArgs a;
    int groups;
  };
  static void entry(const void* p) { alcop_norm_grad<C, emu::Emu>(((const Both*)p)->a, ((const Both*)p)->groups); }
  static hipError_t go(const NormGradArgs& a, int groups, hipStream_t)
  {
    const Both b{a, groups};
    emu::run_grid(&entry, &b, C::NT, C::GRAD_LDS_BYTES, (unsigned)(groups / C::ROWS), 1, 1);
    return hipSuccess;
  }
};
hipError_t launch_norm_rows(const NormArgs& a, int dt, bool whole, hipStream_t st)
{
  return dispatch_rows_of<Norm>(dt, whole, a.rows, a.cols, a, st);
}
hipError_t launch_norm_grad(const NormGradArgs& a, int groups, int dt, bool whole, hipStream_t st)
{
  return dispatch_rows_of<NormGrad>(dt, whole, a.rows, a.cols, a, groups, st);
}
static void sums_entry(const void* p) { alcop_column_sums<emu::Emu>(*(const ColumnSumArgs*)p); }
hipError_t launch_column_sums(const ColumnSumArgs& a, hipStream_t)
{
  emu::run_grid(&sums_entry, &a, SUM_THREADS, SUM_THREADS * 4, (unsigned)((a.cols + SUM_COLS - 1) / SUM_COLS), 1, 1);
  return hipSuccess;
}
template <int DT>
static void act_entry(const void* p)
{
  alcop_act_grad<DT, emu::Emu>(*(const ActGradArgs*)p);
}
hipError_t launch_act_grad(const ActGradArgs& a, int dt, hipStream_t)
{
  emu::run_grid(dt ? &act_entry<1> : &act_entry<0>, &a, 256, 4 * ACT_COLS * 4, (unsigned)((a.N + ACT_COLS - 1) / ACT_COLS),
                (unsigned)((a.M + a.rows_per_block - 1) / a.rows_per_block), 1);
  return hipSuccess;
}
hipError_t prepare_rows() { return hipSuccess; }

// the kernels that calls of these sizes launch, and those that are loaded ahead
static std::set<const void*> reached;
template <class C>
struct Reach {
  static hipError_t go()
  {
    reached.insert((const void*)&Norm<C>::entry);
    return hipSuccess;
  }
};
#endif

}  // namespace alcop

#if EMU_PART == 3
// Kernels that are loaded ahead; those that `n` rows and columns reach; those of the latter that are not among the former.
extern "C" void emu_rows_kernels(const int* sizes, int n, int* out)
{
  using namespace alcop;
  reached.clear();
  (void)each_rows_kernel<Reach>();
  const std::set<const void*> loaded = reached;
  reached.clear();
  for (int i = 0; i < n; i++)
    for (int dt = 0; dt < 3; dt++)
      for (int whole = 0; whole < 2; whole++) (void)dispatch_rows_of<Reach>(dt, whole, sizes[2 * i], sizes[2 * i + 1]);
  out[0] = (int)loaded.size();
  out[1] = (int)reached.size();
  out[2] = 0;
  for (const void* k : reached) out[2] += !loaded.count(k);
}

// One thread's 16-byte stores of each kind to `ptr`, for the test of what the model reports.
namespace {
struct Stores {
  void* ptr;
  int kind;
};
void stores_entry(const void* p)
{
  const Stores& s = *(const Stores*)p;
  const alcop::u32x4 v = {1, 2, 3, 4};
  if (emu::Emu::lane_id() != 0) return;
  if (s.kind == 0) emu::Emu::global_store16(s.ptr, v);
  if (s.kind == 1) emu::Emu::global_store16_through(s.ptr, v);
  if (s.kind == 2) emu::Emu::global_store16_keep(s.ptr, v);
  if (s.kind == 3) emu::Emu::global_store16_any(s.ptr, v);
  if (s.kind == 4) emu::Emu::global_store16_through_any(s.ptr, v);
}
}  // namespace
extern "C" void emu_store16(void* ptr, int kind)
{
  const Stores s{ptr, kind};
  emu::run_grid(&stores_entry, &s, 64, 1024, 1, 1, 1);
}
// the model's conversions of 8-bit numbers, so that a test can pin them
extern "C" uint8_t emu_f32_to_e4m3(float v) { return emu::float_to_e4m3(v); }
extern "C" float emu_e4m3_to_f32(uint8_t b) { return emu::e4m3_to_float(b); }
#endif
