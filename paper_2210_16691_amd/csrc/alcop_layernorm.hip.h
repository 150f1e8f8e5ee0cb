// Layer norm of rows and its gradients.
//
//   norm      h = x + residual;  mean, var of h over the row;  rstd = 1 / sqrt(var + eps);  y = (h - mean) rstd gain + shift
//   gradient  with xh = (total - mean) rstd, t = gain dy:  dx = dtotal + rstd (t - mean(t) - xh mean(t xh)),
//             dgain = sum over rows of dy xh,  dshift = sum over rows of dy
//
// As the root-mean-square norm (alcop_rows.hip.h), whose layout of a row this takes over: bound by memory, a row loaded once,
// held in fp32 registers and stored once, past the caches.
//
// The mean is found in two steps.  sum(h) / n is off by some 2^-24 of |h|'s mean, which where rows lie far from 0 is not small
// beside their spread; so it only gives a point m near the mean, and the second turn sums d = h - m and d^2 together: mean = m + sum(d) / n,
// var = mean(d^2) - mean(d)^2.  m is a multiple of 2^-12 of |h|'s mean (down to its power of two): h - m is then exact but for
// fp32 rows, where a rounding that all of a row's numbers share would not average out of their sum.  mean(d) is up to 2^-13 of |h|'s mean:
// its square costs no digits while that is below the spread, and where it is not (a spread of 1 about 10^4 and more) a third turn sums
// about m + mean(d).  No sum of squares of h itself is formed, and any other row needs two turns of the block, as many as the plain two-pass form.
// The gradient's two means share a turn.
//
// A block of the norm has one row (one of its waves up to 1024 columns, sixteen of its lanes up to 256): 16384 x 4096 bf16 94 us; blocks
// that walk over several rows, the next one loaded ahead of the sums, 97 to 107 where this took 95.5.  The gradient's blocks walk, for the
// sums over rows that they keep, and load ahead: 8192 x 4096 bf16 with dtotal 52 us.
#pragma once
#include "alcop_rows.hip.h"

namespace alcop {

struct LayerNormArgs {
  const void *x, *residual;
  const float *gain, *shift;
  void *total, *y;
  float *scale, *mean, *rstd;
  long ldx, ldr, ldt, ldy;
  int rows, cols;
  float eps;
  int out;                     // type of y (3: e4m3)
};

struct LayerNormGradArgs {
  const void *dy, *total, *dtotal;
  const float *gain, *mean, *rstd;
  void* dx;
  float *dgain, *dshift;       // sums of the rows of each block, a row of them per block, or null
  long lddy, ldt, lddt, lddx;
  int rows, cols;
};

// gain (1) and shift (0): `none` where there is no vector or no column
template <class C, class HW>
__device__ __forceinline__ void load_columns(const float* from, float none, int me, int cols, float (&g)[C::NV][8])
{
  if (from != nullptr) {
    load_gain<C, HW>(from, me, cols, g);
    return;
  }
#pragma unroll
  for (int i = 0; i < C::NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) g[i][e] = none;
}

constexpr int LAYERNORM_LDS_BYTES = 512;      // two floats per wave and reduction, two reductions, twice

template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_layernorm_rows(const LayerNormArgs p)
{
  constexpr int NV = C::NV, DT = C::DT;
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int me = tid % C::TPR;
  const long first = (long)HW::block_x() * C::ROWS + HW::wave_id() * 64 / C::TPR;
  if (first >= p.rows) return;                     // a whole wave, where a wave has rows; else never
  // where a wave has four rows, lanes past the last row have the last one once more, and store nothing
  const long mine = first + HW::lane_id() / C::TPR, row = C::TPR < 64 && mine >= p.rows ? p.rows - 1 : mine;
  const int cols = row == mine ? p.cols : 0;       // to be stored
  // ahead of the sums that they do not depend on, where there are registers for them
  constexpr bool AHEAD = C::TPR < 1024 && NV < 4;
  const float n = (float)p.cols;
  float g[NV][8], b[NV][8];

  Raw<C> x = load_raw<C, HW>(row_at<DT>(p.x, row, p.ldx), me, p.cols), r = {};
  if (p.residual != nullptr) r = load_raw<C, HW>(row_at<DT>(p.residual, row, p.ldr), me, p.cols);
  if (AHEAD) {
    load_columns<C, HW>(p.gain, 1.0f, me, p.cols, g);
    load_columns<C, HW>(p.shift, 0.0f, me, p.cols, b);
  }
  finish<C>(x, me, p.cols);
  if (p.residual != nullptr) finish<C>(r, me, p.cols);
  float h[NV][8];
  float s = 0.f, size = 0.f;
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) h[i][e] = value<C, HW>(x, i, e);
  if (p.residual != nullptr) {
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) h[i][e] += value<C, HW>(r, i, e);
  }
  if (p.total != nullptr) store_values<C, DT, HW>((void*)row_at<DT>(p.total, row, p.ldt), me, cols, h);
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) {
      s += h[i][e];
      size += __builtin_fabsf(h[i][e]);
    }
  row_sums<C::TPR, HW>(s, size, lds);
  // the nearest multiple of 2^-12 of a power of two: what is left when 3 / 2 of 2^23 of them are added and taken away
  const float many = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, size / n) & 0x7f800000u) * 0x1.8p11f;
  float m = (s / n + many) - many;
  float sd = 0.f, sdd = 0.f;
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) {
      // columns past the end hold 0, which is not their part of a sum over h - m
      const bool there = C::WHOLE ? chunk_at<C>(me, i) < p.cols : chunk_at<C>(me, i) + e < p.cols;
      h[i][e] = there ? h[i][e] - m : 0.f;
      sd += h[i][e];
      sdd += h[i][e] * h[i][e];
    }
  row_sums<C::TPR, HW>(sd, sdd, lds + 128);
  float off = sd / n, var = sdd / n - off * off;
  // a row that lies so far away that m is further from the mean than its spread: the square took the digits, and the row moves once more
  const bool far = off * off > var;
  if (HW::ballot(far)) {
    const float by = far ? off : 0.f;              // the other rows of the wave stay as they are
    m += by;
    sd = sdd = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const bool there = C::WHOLE ? chunk_at<C>(me, i) < p.cols : chunk_at<C>(me, i) + e < p.cols;
        h[i][e] -= by;
        const float d = there ? h[i][e] : 0.f;
        sd += d;
        sdd += d * d;
      }
    row_sums<C::TPR, HW>(sd, sdd, lds);            // where the first two were
    if (far) {
      off = sd / n;
      var = sdd / n - off * off;
    }
  }
  const float rstd = 1.0f / HW::sqrt((var < 0.f ? 0.f : var) + p.eps);       // NaN stays
  if (me == 0 && cols) {
    if (p.mean != nullptr) HW::global_store_u32(p.mean + row, __builtin_bit_cast(uint32_t, m + off));
    if (p.rstd != nullptr) HW::global_store_u32(p.rstd + row, __builtin_bit_cast(uint32_t, rstd));
  }
  if (!AHEAD) load_columns<C, HW>(p.gain, 1.0f, me, p.cols, g);
  if (!AHEAD) load_columns<C, HW>(p.shift, 0.0f, me, p.cols, b);
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) h[i][e] = HW::fma((h[i][e] - off) * rstd, g[i][e], b[i][e]);
  store_result<C, HW>(h, p.y, p.ldy, p.out, p.scale, row, me, cols, lds + 256);
}

// A group of TPR threads takes rows g, g + groups, ... and keeps the sums of dgain and dshift for its columns in registers; the
// groups of a block add theirs, alcop_column_sums adds the blocks'.  Where a wave has four rows, its lanes walk as long as the first of them, and
// past the last row do the last row once more without adding or storing it.
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_layernorm_grad(const LayerNormGradArgs p, int groups)
{
  constexpr int NV = C::NV, DT = C::DT;
  // rows of more elements than the registers have room for are read again behind the sums
  constexpr bool HOLD = NV * C::TPR <= 2048;
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int me = tid % C::TPR;
  const int group = (int)HW::block_x() * C::ROWS + HW::wave_id() * 64 / C::TPR, part = HW::lane_id() / C::TPR;
  auto clamped = [&](long row) __attribute__((always_inline)) {
    if constexpr (C::TPR >= 64)
      return row;
    else
      return row + part < p.rows ? row + part : (long)p.rows - 1;
  };
  float dg[NV][8], ds[NV][8];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) dg[i][e] = ds[i][e] = 0.f;
  constexpr bool GAIN_HELD = NV <= 2 && C::TPR < 1024;      // as far as the registers go
  float g[NV][8];
  if (GAIN_HELD) load_columns<C, HW>(p.gain, 1.0f, me, p.cols, g);
  const float n = (float)p.cols;
  int turn = 0;
  // the next row ahead of the sums of the one at hand, where there are registers for it
  constexpr bool NEXT = HOLD && NV * C::TPR <= 1024;
  Raw<C> dy2 = {}, h2 = {}, dt2 = {};
  float mean2 = 0.f, rstd2 = 0.f;
  auto load_next = [&](long row) __attribute__((always_inline)) {
    dy2 = load_raw<C, HW>(row_at<DT>(p.dy, row, p.lddy), me, p.cols);
    h2 = load_raw<C, HW>(row_at<DT>(p.total, row, p.ldt), me, p.cols);
    if (p.dtotal != nullptr) dt2 = load_raw<C, HW>(row_at<DT>(p.dtotal, row, p.lddt), me, p.cols);
    mean2 = __builtin_bit_cast(float, HW::global_load_u32(p.mean + row));
    rstd2 = __builtin_bit_cast(float, HW::global_load_u32(p.rstd + row));
  };
  if (NEXT && group < p.rows) load_next(clamped(group));
  for (long first = group; first < p.rows; first += groups, turn ^= 1) {
    const long row = clamped(first);
    const int cols = C::TPR >= 64 || first + part < p.rows ? p.cols : 0;
    Raw<C> dy, h, dt = {};
    float mean, rstd;
    if constexpr (NEXT) {
      dy = dy2, h = h2, dt = dt2, mean = mean2, rstd = rstd2;
      if (first + groups < p.rows) load_next(clamped(first + groups));
    } else {
      dy = load_raw<C, HW>(row_at<DT>(p.dy, row, p.lddy), me, p.cols);
      h = load_raw<C, HW>(row_at<DT>(p.total, row, p.ldt), me, p.cols);
      mean = __builtin_bit_cast(float, HW::global_load_u32(p.mean + row));
      rstd = __builtin_bit_cast(float, HW::global_load_u32(p.rstd + row));
    }
    if (!GAIN_HELD) load_columns<C, HW>(p.gain, 1.0f, me, p.cols, g);
    finish<C>(dy, me, p.cols);
    finish<C>(h, me, p.cols);
    float st = 0.f, stx = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        // past the end dy is 0 (the mean may be infinite, which 0 times is not 0)
        const bool there = C::WHOLE ? chunk_at<C>(me, i) < cols : chunk_at<C>(me, i) + e < cols;
        const float d = C::TPR >= 64 || there ? value<C, HW>(dy, i, e) : 0.f, xh = there ? (value<C, HW>(h, i, e) - mean) * rstd : 0.f;
        st += d * g[i][e];
        stx += d * g[i][e] * xh;
        dg[i][e] += d * xh;
        ds[i][e] += d;
      }
    row_sums<C::TPR, HW>(st, stx, lds + 128 * turn);
    st /= n;
    stx /= n;
    if constexpr (!HOLD) {
      dy = load_raw<C, HW>(row_at<DT>(p.dy, row, p.lddy), me, p.cols);
      h = load_raw<C, HW>(row_at<DT>(p.total, row, p.ldt), me, p.cols);
      load_columns<C, HW>(p.gain, 1.0f, me, p.cols, g);
      finish<C>(dy, me, p.cols);
      finish<C>(h, me, p.cols);
    }
    float dx[NV][8];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++)
        dx[i][e] = rstd * (value<C, HW>(dy, i, e) * g[i][e] - st - (value<C, HW>(h, i, e) - mean) * rstd * stx);
    if (p.dtotal != nullptr) {
      if (!NEXT) dt = load_raw<C, HW>(row_at<DT>(p.dtotal, row, p.lddt), me, p.cols);
      finish<C>(dt, me, p.cols);
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) dx[i][e] += value<C, HW>(dt, i, e);
    }
    store_values<C, DT, HW>((void*)row_at<DT>(p.dx, row, p.lddx), me, cols, dx);
  }
  // the sums of a block: of dgain, then in the same LDS of dshift
  auto leave = [&](float(&v)[NV][8], float* to, bool again) __attribute__((always_inline)) {
    if (to == nullptr) return;
    if constexpr (C::TPR < 64) {
      // the four parts of a wave, which from here on add and store the same
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
          v[i][e] += __builtin_bit_cast(float, HW::xor_lanes(__builtin_bit_cast(uint32_t, v[i][e]), 16));
          v[i][e] += __builtin_bit_cast(float, HW::xor_lanes(__builtin_bit_cast(uint32_t, v[i][e]), 32));
        }
    }
    if constexpr (C::ROWS > 1) {
      constexpr uint32_t ROW = C::TPR * 4;
      const uint32_t at = lds + LAYERNORM_LDS_BYTES + (uint32_t)me * 4;
      const int wave = HW::wave_id();
      if (again) HW::block_barrier();
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < 8; e++)
          HW::lds_write1(at + (uint32_t)((wave * NV + i) * 8 + e) * ROW, __builtin_bit_cast(uint32_t, v[i][e]));
      HW::wait_lds();
      HW::block_barrier();
      if (wave == 0) {
#pragma unroll
        for (int w = 1; w < C::NT / 64; w++)
#pragma unroll
          for (int i = 0; i < NV; i++)
#pragma unroll
            for (int e = 0; e < 8; e++)
              v[i][e] += __builtin_bit_cast(float, HW::lds_read4(at + (uint32_t)((w * NV + i) * 8 + e) * ROW));
      }
      HW::wait_lds();
      if (wave > 0) return;
    }
    store_values<C, 2, HW>(to + (long)HW::block_x() * p.cols, me, p.cols, v);
  };
  leave(dg, p.dgain, false);
  leave(ds, p.dshift, p.dgain != nullptr);
}

// the sums of both gradients in one launch (blocks y = 0 and 1)
struct TwoColumnSums {
  ColumnSumArgs of[2];
};
template <class HW>
__global__ void __launch_bounds__(SUM_THREADS) alcop_two_column_sums(const TwoColumnSums p)
{
  column_sums<HW>(HW::block_y() ? p.of[1] : p.of[0]);
}

// LDS that the norm asks for: more than it needs where fewer blocks on a compute unit are better, as 64 KB of rows (three blocks at least)
// are enough on their way, and more are read in a worse order.  us with all blocks that the registers allow, and so: 16384 x 4096
// with a residual, bf16 103 and 95.6, fp32 202 and 188; 8192 x 8192 bf16 95.3 and 93.6; 65536 x 1024 91.8 and 90.3; without
// a residual 16384 x 4096, 8 KB a block, 64.0 either way.
template <class C>
int layernorm_lds(const LayerNormArgs& a)
{
  const long block = (long)C::ROWS * a.cols * (C::DT == 2 ? 4 : 2) * (a.residual != nullptr ? 2 : 1);
  const long blocks = 65536 / block < 3 ? 3 : 65536 / block;
  return blocks >= 8 || C::TPR == 1024 ? LAYERNORM_LDS_BYTES : (int)(163840 / blocks / 512 * 512);
}

template <class C>
constexpr int layernorm_grad_lds()
{
  return LAYERNORM_LDS_BYTES + (C::ROWS > 1 ? C::NT / 64 * C::NV * 8 * C::TPR * 4 : 0);
}

}  // namespace alcop
