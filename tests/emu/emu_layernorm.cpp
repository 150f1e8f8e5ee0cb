// The layer norm on the functional model: its host code (alcop_layernorm.cpp) linked with launchers that run the kernel templates
// on emu_hw.h.
#include <hip/hip_runtime.h>

#include "emu_hw.h"
#include "alcop_layernorm.h"

namespace alcop {

namespace {
template <class C>
struct Norm {
  static void entry(const void* p) { alcop_layernorm_rows<C, emu::Emu>(*(const LayerNormArgs*)p); }
  static hipError_t go(const LayerNormArgs& a, hipStream_t)
  {
    emu::run_grid(&entry, &a, C::NT, LAYERNORM_LDS_BYTES, (unsigned)(((long)a.rows + C::ROWS - 1) / C::ROWS), 1, 1);
    return hipSuccess;
  }
};
template <class C>
struct Grad {
  struct Both {
    LayerNormGradArgs a;
    int groups;
  };
  static void entry(const void* p) { alcop_layernorm_grad<C, emu::Emu>(((const Both*)p)->a, ((const Both*)p)->groups); }
  static hipError_t go(const LayerNormGradArgs& a, int groups, hipStream_t)
  {
    const Both b{a, groups};
    emu::run_grid(&entry, &b, C::NT, layernorm_grad_lds<C>(), (unsigned)(groups / C::ROWS), 1, 1);
    return hipSuccess;
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
static void sums_entry(const void* p) { alcop_two_column_sums<emu::Emu>(*(const TwoColumnSums*)p); }
hipError_t launch_two_column_sums(const TwoColumnSums& a, int arrays, hipStream_t)
{
  emu::run_grid(&sums_entry, &a, SUM_THREADS, SUM_THREADS * 4, (unsigned)((a.of[0].cols + SUM_COLS - 1) / SUM_COLS),
                (unsigned)arrays, 1);
  return hipSuccess;
}
hipError_t prepare_layernorm() { return hipSuccess; }

}  // namespace alcop
