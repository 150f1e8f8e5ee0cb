// Launchers of the layer norm, between its host code (alcop_layernorm.cpp) and inst_layernorm.hip.
#pragma once
#include "alcop_linear.h"
#include "alcop_layernorm.hip.h"

namespace alcop {

// Rows of up to 256 columns, which leave most of a wave without a chunk, are four to a wave (alcop_rows.hip.h has the others).  us with
// a wave to a row and so, bf16 with a residual: norms of 128 columns, 16 rows 4.2 and 4.8, 4096 rows 4.9 and 4.4, 16384 9.5 and 4.8,
// 65536 28.7 and 12.4; of 256 4.7 and 4.5, 4.9 and 4.7, 10.0 and 6.7, 30.8 and 21.4; gradients of 128 columns, 16 rows 7.3 and 4.6, 1024
// 7.3 and 7.6, 16384 13.2 and 9.4, 65536 33.2 and 18.4; of 256 7.9 and 4.8, 7.9 and 8.4, 14.3 and 12.5, 38.9 and 29.9.
constexpr int SHORT_COLS = 256;
inline int layernorm_rows_per_block(int rows, int cols) { return cols <= SHORT_COLS ? 16 : rows_per_block(rows, cols); }
template <int DT, bool WHOLE, template <class> class LAUNCH, class... A>
hipError_t dispatch_short_rows(int cols, const A&... a)
{
  return cols <= SHORT_COLS / 2 ? LAUNCH<RowCfg<DT, 16, 1, WHOLE>>::go(a...) : LAUNCH<RowCfg<DT, 16, 2, WHOLE>>::go(a...);
}
template <template <class> class LAUNCH, class... A>
hipError_t dispatch_layernorm(int dt, bool whole, int rows, int cols, const A&... a)
{
  if (cols > SHORT_COLS) return dispatch_rows_of<LAUNCH>(dt, whole, rows, cols, a...);
  if (dt == 0) return whole ? dispatch_short_rows<0, true, LAUNCH>(cols, a...) : dispatch_short_rows<0, false, LAUNCH>(cols, a...);
  if (dt == 1) return whole ? dispatch_short_rows<1, true, LAUNCH>(cols, a...) : dispatch_short_rows<1, false, LAUNCH>(cols, a...);
  return whole ? dispatch_short_rows<2, true, LAUNCH>(cols, a...) : dispatch_short_rows<2, false, LAUNCH>(cols, a...);
}
// All of them.
template <template <class> class LAUNCH>
hipError_t each_layernorm_kernel()
{
  hipError_t rc = each_rows_kernel<LAUNCH>();
  for (int dt = 0; dt < 3; dt++)
    for (int whole = 0; whole < 2; whole++)
      for (int cols : {SHORT_COLS / 2, SHORT_COLS})
        if (rc == hipSuccess) rc = dispatch_layernorm<LAUNCH>(dt, whole, 1, cols);
  return rc;
}

hipError_t launch_layernorm_rows(const LayerNormArgs& a, int dt, bool whole, hipStream_t st);
hipError_t launch_layernorm_grad(const LayerNormGradArgs& a, int groups, int dt, bool whole, hipStream_t st);
hipError_t launch_two_column_sums(const TwoColumnSums& a, int arrays, hipStream_t st);
hipError_t prepare_layernorm();

}  // namespace alcop
