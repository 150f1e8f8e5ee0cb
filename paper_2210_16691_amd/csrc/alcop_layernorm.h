// Launchers of the layer norm, between its host code (alcop_layernorm.cpp) and inst_layernorm.hip.
#pragma once
#include "alcop_linear.h"
#include "alcop_layernorm.hip.h"

namespace alcop {

hipError_t launch_layernorm_rows(const LayerNormArgs& a, int dt, bool whole, hipStream_t st);
hipError_t launch_layernorm_grad(const LayerNormGradArgs& a, int groups, int dt, bool whole, hipStream_t st);
hipError_t launch_two_column_sums(const TwoColumnSums& a, int arrays, hipStream_t st);
hipError_t prepare_layernorm();

}  // namespace alcop
