// Which kernel a linear layer gets: measured costs, as alcop_dispatch.h has them for the plain products.
//
//     us = a + b * turns * k-tiles + c * turns + d * (bytes of A, W, C, residual and pre at 5.1 TB/s)
//            + e * (flops at 1.4 PFLOP/s) + f * turns2 * k-tiles
// with turns = ceil(tiles / 256) and, for kernels of which two blocks share a compute unit, turns2 = 2 ceil(tiles / 512).
// An e4m3 problem counts as one of half its K on 16 bits, which moves as many bytes.  Fitted (least squares of the
// relative error, no negative coefficient) on 920 layers of each kind with a bias and a residual: 1 to 8192 rows, 64 to
// 8192 columns and K, up to 550 GFLOP, operands and results cycled through three buffers, launches replayed from
// a graph.  On them the pick takes 1.01 times the best kernel's time in the mean, 1.00 to 1.01 at the 90th percentile, 1.16 to
// 1.3 at worst (but for one of the e4m3 layers).  None were held out.  A kernel is here if leaving it out costs anything in
// the mean: 0.02 % (128 x 64, e4m3) to 10 % (16 x 16).  The widened tiles of 64 x 64 and more serve e4m3 layers with an
// fp32 result.
#pragma once
#include "../../include/alcop.h"

namespace alcop {

struct LinearCost {
  alcop_sched s;
  int dt, bl;          // as in LCfg; 16-bit types have one set of costs
  int waves_k;         // waves a tile's k-tiles are divided among
  int blocks;          // blocks that share a compute unit
  double a, b, c, d, e, f;
};

inline const LinearCost kLinearCost[] = {
    // 16-bit operands, W stored K x N
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 2.372, 0.121, 0.590, 0.591, 9.910, 0.121},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 1.743, 0.356, 1.374, 0.553, 5.487, 0.054},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 1.563, 0.365, 1.855, 0.406, 4.037, 0.125},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 1, 0, 4, 2, 0.999, 0.198, 2.897, 0.316, 2.276, 0.154},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 2.518, 0.094, 0.816, 0.518, 0.769, 0.058},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 2.438, 0.078, 1.485, 0.557, 1.028, 0.084},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 4.286, 0.000, 0.046, 1.179, 0.491, 0.265},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 1.535, 0.290, 3.559, 0.730, 0.541, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 3.350, 0.491, 2.798, 1.625, 0.235, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 4.313, 0.470, 2.193, 1.471, 0.111, 0.000},
    // 16-bit operands, W stored N x K
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 2.418, 0.077, 0.723, 0.334, 4.721, 0.068},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 1.862, 0.341, 1.432, 0.390, 3.479, 0.000},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 1.566, 0.173, 2.057, 0.314, 3.145, 0.146},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 1, 1, 4, 2, 1.185, 0.211, 2.681, 0.416, 1.960, 0.102},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 2.586, 0.054, 0.894, 0.438, 0.849, 0.074},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 2.500, 0.070, 1.478, 0.583, 0.962, 0.084},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 4.122, 0.000, 0.224, 1.141, 0.500, 0.268},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 1.816, 0.312, 3.145, 0.881, 0.447, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 3.619, 0.506, 2.576, 1.678, 0.200, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 4.350, 0.568, 1.854, 1.462, 0.081, 0.000},
    // e4m3 widened to bf16
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 2.461, 0.108, 0.708, 0.285, 5.135, 0.062},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 1.957, 0.410, 1.337, 0.344, 4.513, 0.000},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 1.651, 0.257, 1.914, 0.294, 3.712, 0.152},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 2, 1, 4, 2, 1.101, 0.270, 2.837, 0.344, 2.183, 0.153},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 2.589, 0.113, 1.085, 0.294, 0.421, 0.111},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 2.450, 0.146, 1.702, 0.611, 0.684, 0.146},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 4.317, 0.200, 0.237, 1.132, 0.554, 0.297},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 1.731, 0.636, 3.382, 1.059, 0.186, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 4.000, 1.010, 2.167, 1.848, 0.132, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 4.138, 0.944, 2.574, 1.515, 0.164, 0.000},
    // e4m3 as they are
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 2.693, 0.035, 0.757, 0.628, 1.224, 0.062},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 2.843, 0.018, 1.181, 0.793, 1.191, 0.099},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 4.381, 0.000, 0.064, 1.140, 0.493, 0.283},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 2.319, 0.328, 2.637, 1.052, 0.419, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 4.733, 0.589, 1.295, 1.865, 0.044, 0.000},
    {{256, 256, 64, 128, 64, 2, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 5.987, 1.309, 0.312, 1.455, 0.000, 0.000},
};

// K in 16-bit units; bytes: of everything read and written.
inline double linear_us(const LinearCost& m, int M, int N, int K, double bytes)
{
  auto up = [](double x, double y) { return (double)(long)((x + y - 1) / y); };
  const double tiles = up(M, m.s.bm) * up(N, m.s.bn);
  const double turns = up(tiles, 256), kt = up(up(K, m.s.bk), m.waves_k);
  const double turns2 = m.blocks == 2 ? 2.0 * up(tiles, 512) : 0.0;
  return m.a + m.b * turns * kt + m.c * turns + m.d * bytes / 5.1e6 + m.e * 2.0 * M * N * (double)K / 1.4e9 +
         m.f * turns2 * kt;
}

// The kernels whose waves split K are compared only while 64 x 64 tiles leave compute units idle.
inline bool linear_applies(const LinearCost& m, int M, int N)
{
  return m.s.variant != 3 || (double)((M + 63L) / 64) * ((N + 63L) / 64) <= 256;
}

}  // namespace alcop
