// Which kernel a linear layer gets: measured costs, as alcop_dispatch.h has them for the plain products.
//
//     us = a + b * turns * k-tiles + c * turns + d * (bytes of A, W, C, residual and pre at 5.1 TB/s)
//            + e * (flops at 1.4 PFLOP/s) + f * turns2 * k-tiles
// with turns = ceil(tiles / 256) and, for kernels of which two blocks share a compute unit, turns2 = 2 ceil(tiles / 512).
// An e4m3 problem counts as one of half its K on 16 bits, which moves as many bytes.  Fitted (least squares of the
// relative error, no negative coefficient) on 800 layers of each kind with a bias and a residual: 1 to 8192 rows, 64 to
// 8192 columns and K, up to 137 GFLOP, operands and results cycled through three buffers, launches replayed from
// a graph.  On them the pick takes 1.01 times the best kernel's time in the mean, 1.00 to 1.04 at the 90th percentile, 1.3 at
// worst.  None were held out.  A kernel stays in the table if some products are slower without it: leaving out any
// of them but the 256 x 128 tile of 32-deep k-tiles, which is gone, costs 0.1 to 10 % in the mean.
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
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 2.369, 0.117, 0.587, 0.581, 9.846, 0.127},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 1.750, 0.359, 1.364, 0.546, 5.402, 0.056},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 1.619, 0.390, 1.807, 0.398, 3.927, 0.116},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 1, 0, 4, 2, 1.123, 0.209, 2.772, 0.287, 2.372, 0.149},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 2.758, 0.083, 0.593, 0.481, 0.934, 0.058},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 2.386, 0.077, 1.423, 0.425, 1.123, 0.087},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 4.315, 0.000, 0.000, 1.113, 0.565, 0.260},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 0.991, 0.290, 4.064, 0.596, 0.742, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 0.679, 0.486, 5.257, 1.447, 0.353, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 0.000, 0.498, 6.260, 1.236, 0.146, 0.000},
    // 16-bit operands, W stored N x K
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 2.433, 0.079, 0.722, 0.321, 4.704, 0.068},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 1.876, 0.343, 1.421, 0.383, 3.408, 0.000},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 1.619, 0.193, 2.006, 0.301, 3.080, 0.137},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 1, 1, 4, 2, 1.321, 0.230, 2.555, 0.369, 2.141, 0.093},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 2.784, 0.043, 0.681, 0.375, 1.036, 0.076},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 2.377, 0.066, 1.463, 0.428, 1.081, 0.090},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 4.235, 0.000, 0.088, 1.083, 0.596, 0.259},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 1.356, 0.305, 3.589, 0.762, 0.632, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 0.714, 0.502, 5.206, 1.459, 0.308, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 0.000, 0.605, 5.835, 1.230, 0.079, 0.000},
    // e4m3 widened to bf16
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 2.467, 0.110, 0.705, 0.264, 5.059, 0.063},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 1.969, 0.412, 1.332, 0.328, 4.406, 0.000},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 1.686, 0.279, 1.880, 0.270, 3.692, 0.143},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 2, 1, 4, 2, 1.220, 0.322, 2.736, 0.269, 2.424, 0.128},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 2.834, 0.124, 0.842, 0.250, 0.518, 0.107},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 2.459, 0.161, 1.577, 0.448, 0.823, 0.139},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 3.989, 0.103, 0.594, 0.990, 0.845, 0.330},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 1.744, 0.619, 3.365, 0.946, 0.310, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 1.611, 1.063, 4.355, 1.634, 0.043, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 0.000, 1.055, 6.098, 1.227, 0.000, 0.000},
    // e4m3 as they are
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 2.895, 0.022, 0.588, 0.509, 1.496, 0.069},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 2.710, 0.000, 1.180, 0.554, 1.505, 0.109},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 4.463, 0.000, 0.000, 1.056, 0.580, 0.275},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 1.986, 0.316, 3.036, 0.901, 0.620, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 1.751, 0.587, 4.029, 1.619, 0.151, 0.000},
    {{256, 256, 64, 128, 64, 2, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 0.000, 1.445, 5.876, 1.169, 0.000, 0.000},
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
