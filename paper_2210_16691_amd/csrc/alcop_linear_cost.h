// Which kernel a linear layer gets: measured costs, as alcop_dispatch.h has them for the plain products.
//
//     us = a + b * turns * k-tiles + c * turns + d * (bytes of A, W, C, residual and pre at 5.1 TB/s)
//            + e * (flops at 1.4 PFLOP/s) + f * turns2 * k-tiles
// with turns = ceil(tiles / 256) and, for kernels of which two blocks share a compute unit, turns2 = 2 ceil(tiles / 512).
// An e4m3 problem counts as one of half its K on 16 bits, which moves as many bytes.  Fitted (least squares of the
// relative error, no negative coefficient) on 1200 layers of each kind with a bias and a residual: 1 to 8192 rows, 64 to
// 8192 columns and K up to 137 GFLOP, 100 of 34 to 550, 300 of up to 512 rows with up to 16384 columns and K; operands and
// results cycled through three buffers, launches replayed from a graph; times within 2.5 (e4m3 4) times the best one's.  On them the pick takes 1.01 times the best kernel's
// time in the mean, 1.01 (e4m3 1.04) at the 90th percentile, 1.2 to 1.3 at worst.  On 135 others with a bias and a residual (45 of
// each table below, two in five of them 17 to 506 rows with up to 16384 columns and K) 1.010, 1.002 and 1.009 in the mean, 1.02, 1.01 and 1.02
// at the 90th percentile, 1.16 (948 x 2504 x 64), 1.02 and 1.20 (64 x 13616 x 576) at worst.  What leaving a
// kernel out costs in the mean: 0.1 (four waves of 64 x 64, which saves a quarter to a third where 128 to 512 rows meet a K of ten
// thousand) to 9 % (16 x 16).  The widened tiles of 64 x 64 and more serve e4m3 layers with an fp32 result.
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
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 2.353, 0.280, 0.488, 0.605, 7.611, 0.074},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 1.733, 0.510, 1.255, 0.549, 4.295, 0.013},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 1, 0, 8, 2, 1.722, 0.674, 1.594, 0.449, 2.949, 0.000},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 1, 0, 4, 2, 1.308, 0.399, 2.543, 0.372, 1.826, 0.057},
    {{64, 64, 64, 64, 64, 2, 1, 0, 1, 0, 3}, 1, 0, 4, 1, 0.820, 0.661, 4.157, 0.318, 1.150, 0.000},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 2.382, 0.099, 0.891, 0.425, 0.727, 0.059},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 2.075, 0.085, 1.825, 0.359, 1.057, 0.085},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 1, 0, 1, 2, 3.091, 0.000, 1.243, 0.894, 0.533, 0.276},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 0.445, 0.300, 4.681, 0.394, 0.712, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 0.000, 0.430, 6.720, 0.796, 0.655, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 0, 1, 1, 3.864, 0.407, 2.883, 1.420, 0.301, 0.000},
    // 16-bit operands, W stored N x K
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 2.463, 0.201, 0.631, 0.415, 3.233, 0.008},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 1.836, 0.352, 1.384, 0.483, 3.077, 0.000},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 1, 1, 8, 2, 1.795, 0.471, 1.777, 0.417, 2.199, 0.000},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 1, 1, 4, 2, 1.534, 0.361, 2.303, 0.474, 1.640, 0.025},
    {{64, 64, 64, 64, 64, 2, 1, 0, 1, 0, 3}, 1, 1, 4, 1, 0.767, 0.642, 4.235, 0.377, 0.936, 0.000},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 2.502, 0.053, 0.901, 0.453, 0.835, 0.077},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 2.162, 0.092, 1.768, 0.432, 0.926, 0.079},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 1, 1, 1, 2, 3.289, 0.000, 1.034, 0.947, 0.524, 0.278},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 0.525, 0.321, 4.465, 0.498, 0.606, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 0.000, 0.433, 6.765, 0.890, 0.614, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 1, 1, 1, 1, 4.293, 0.544, 2.008, 1.488, 0.137, 0.000},
    // e4m3 widened to bf16
    {{16, 16, 64, 16, 16, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 2.455, 0.198, 0.664, 0.381, 3.727, 0.019},
    {{16, 32, 64, 16, 32, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 1.928, 0.410, 1.360, 0.427, 3.830, 0.000},
    {{32, 32, 64, 32, 32, 2, 1, 0, 1, 0, 3}, 2, 1, 8, 2, 1.834, 0.553, 1.745, 0.405, 2.102, 0.000},
    {{32, 64, 64, 32, 64, 2, 1, 0, 1, 0, 3}, 2, 1, 4, 2, 1.225, 0.435, 2.740, 0.364, 1.500, 0.068},
    {{64, 64, 64, 64, 64, 2, 1, 0, 1, 0, 3}, 2, 1, 4, 1, 0.449, 0.772, 4.525, 0.283, 1.055, 0.000},
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 2.385, 0.152, 1.222, 0.136, 0.063, 0.109},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 1.545, 0.206, 2.643, 0.083, 0.464, 0.148},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 2, 1, 1, 2, 2.603, 0.212, 1.873, 0.712, 0.362, 0.369},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 0.000, 0.674, 5.511, 0.283, 0.426, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 0.447, 1.028, 8.056, 0.869, 0.390, 0.000},
    {{256, 256, 32, 128, 64, 3, 2, 1, 1, 0, 0}, 2, 1, 1, 1, 4.545, 0.986, 4.394, 1.292, 0.145, 0.000},
    // e4m3 as they are
    {{64, 64, 64, 32, 32, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 2.539, 0.034, 0.842, 0.558, 1.177, 0.068},
    {{128, 64, 64, 64, 32, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 2.168, 0.018, 1.821, 0.444, 1.200, 0.112},
    {{128, 128, 64, 64, 64, 2, 2, 1, 1, 0, 0}, 3, 1, 1, 2, 3.302, 0.000, 1.072, 0.882, 0.448, 0.316},
    {{128, 128, 64, 64, 64, 4, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 0.508, 0.370, 4.549, 0.436, 0.555, 0.000},
    {{256, 128, 64, 128, 64, 3, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 0.000, 0.585, 7.990, 0.588, 0.487, 0.000},
    {{256, 256, 64, 128, 64, 2, 2, 1, 1, 0, 0}, 3, 1, 1, 1, 5.552, 1.314, 2.420, 1.276, 0.000, 0.000},
};

// K in 16-bit units; bytes: of everything read and written.  tiles: of C; products: M N
inline double linear_us(const LinearCost& m, double tiles, double products, int K, double bytes)
{
  auto up = [](double x, double y) { return (double)(long)((x + y - 1) / y); };
  const double turns = up(tiles, 256), kt = up(up(K, m.s.bk), m.waves_k);
  const double turns2 = m.blocks == 2 ? 2.0 * up(tiles, 512) : 0.0;
  return m.a + m.b * turns * kt + m.c * turns + m.d * bytes / 5.1e6 + m.e * 2.0 * products * (double)K / 1.4e9 +
         m.f * turns2 * kt;
}
inline double linear_us(const LinearCost& m, int M, int N, int K, double bytes)
{
  return linear_us(m, (double)(((long)M + m.s.bm - 1) / m.s.bm) * (((long)N + m.s.bn - 1) / m.s.bn), (double)M * N, K, bytes);
}

// The kernels whose waves split K are compared only while 64 x 64 tiles leave compute units idle, those of such tiles up to
// two turns of the card.
inline bool linear_applies(const LinearCost& m, int M, int N)
{
  return m.s.variant != 3 || (double)((M + 63L) / 64) * ((N + 63L) / 64) <= (m.s.bm == 64 ? 512 : 256);
}

}  // namespace alcop
