// Operators on rows around the products of a transformer block: root-mean-square norm with the residual's addition
// and its gradients, rows to 8 bits with a scale each, the gradient of an activation with the bias's.
//
//   norm      h = x + residual;  rstd = 1 / sqrt(mean(h^2) + eps);  y = h rstd gain
//   8 bits    scale = max(max |y| / 448, 2^-126);  q = e4m3(y / scale)            (448: the largest e4m3 number)
//   gradient  with xh = h rstd, t = gain dy:  dx = dtotal + rstd (t - xh mean(t xh)),  dgain = sum over rows of dy xh
//
// All of them are bound by memory: a row is loaded once, held in registers in fp32 while its sum and its maximum are
// found, and stored once, past the caches (kept in the memory-side cache, a norm and the layer that reads it take 3 to 11 % less with
// 256 rows, 0 to 7 with 1024, but 3 to 4 % more with one to sixteen rows of 768 and up to 3 with 256 of 4096).  Sums are fp32 in a fixed order; nothing is atomic, so results do not change between runs.
//
// A row belongs to TPR threads (a wave, a whole block, or sixteen lanes of a wave), each holding NV chunks of eight elements, moved sixteen bytes a load at
// whatever address they lie (a global access may start at any element).  Where the length is no multiple of eight (!WHOLE)
// the last chunk is loaded as the row's last eight elements and stored element by element.
//
// Measured: norm of 16384 x 4096 bf16 with residual and sum 90.6 us = 5.9 TB/s, 8192 x 4096 bf16 to 8 bits 17.2 us, the norm's
// gradients of 8192 x 4096 51.4 us = 5.2 TB/s and 6 for the sums of the gain's, dZ of 4096 x 4096 20 us = 5.0 TB/s (a copy of
// 512 MiB 5.4 TB/s); one row of 4096 3.6 us, two sums over a block one after the other.
#pragma once
#include "alcop_linear.hip.h"

namespace alcop {

constexpr int ROWS_LDS_BYTES = 256;      // a float per wave and reduction, two reductions, twice

struct NormArgs {
  const void *x, *residual;
  const float* gain;
  void *total, *y;
  float *scale, *rstd;
  long ldx, ldr, ldt, ldy;
  int rows, cols;
  float eps;
  int flags;                   // type of y (3: e4m3) | the rows are normalised << 2
};

struct NormGradArgs {
  const void *dy, *total, *dtotal;
  const float *gain, *rstd;
  void* dx;
  float* partial;              // dgain's sums of the rows of each block, or null
  long lddy, ldt, lddt, lddx;
  int rows, cols;
};

struct ActGradArgs {
  const void *dc, *pre;
  void* dz;                    // null: only the sums
  float* partial;              // dbias's sums of the rows of each block, or null
  long lddc, ldp, ldz;
  int M, N, rows_per_block, act, lanes;
};

struct ColumnSumArgs {
  const float* partial;
  float* out;
  int count, cols;
};

// ---- sums and maxima over the threads of a row -------------------------------------------------------------
template <class HW>
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __builtin_bit_cast(float, HW::xor_lanes(__builtin_bit_cast(uint32_t, v), m));
  return v;
}
// of magnitudes, as bit patterns: those of NaN are above all others, so that one NaN makes the result NaN
template <int LANES, class HW>
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
  for (int m = LANES / 2; m >= 1; m >>= 1) {
    const uint32_t o = HW::xor_lanes(v, m);
    v = o > v ? o : v;
  }
  return v;
}
// over a row's TPR threads; `at`: LDS of this reduction, 4 bytes a wave, not used by the one before
template <int TPR, class HW>
__device__ __forceinline__ float row_sum(float v, uint32_t at)
{
  v = wave_sum<HW>(v);
  if constexpr (TPR > 64) {
    HW::lds_write1(at + 4 * HW::wave_id(), __builtin_bit_cast(uint32_t, v));
    HW::wait_lds();
    HW::block_barrier();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; w++) v += __builtin_bit_cast(float, HW::lds_read4(at + 4 * w));
  }
  return v;
}
// two sums for one turn of the block; `at`: 8 bytes a wave
template <int TPR, class HW>
__device__ __forceinline__ void row_sums(float& a, float& b, uint32_t at)
{
  if constexpr (TPR == 16) {
    a = HW::sum_sixteen(a);
    b = HW::sum_sixteen(b);
    return;
  }
  a = HW::sum_lanes(a);
  b = HW::sum_lanes(b);
  if constexpr (TPR > 64) {
    HW::lds_write(at + 8 * HW::wave_id(), u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)});
    HW::wait_lds();
    HW::block_barrier();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; w++) {
      const u32x2 t = HW::lds_read8(at + 8 * w);
      const uint32_t ta = t[0], tb = t[1];         // a cast of t[1] itself takes t[0]
      a += __builtin_bit_cast(float, ta);
      b += __builtin_bit_cast(float, tb);
    }
  }
}
template <int TPR, class HW>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t at)
{
  v = wave_max<(TPR < 64 ? TPR : 64), HW>(v);
  if constexpr (TPR > 64) {
    HW::lds_write1(at + 4 * HW::wave_id(), v);
    HW::wait_lds();
    HW::block_barrier();
    v = 0;
#pragma unroll
    for (int w = 0; w < TPR / 64; w++) {
      const uint32_t o = HW::lds_read4(at + 4 * w);
      v = o > v ? o : v;
    }
  }
  return v;
}

// ---- a thread's part of a row ----------------------------------------------------------------------------------
// Chunk i of a thread is columns (i TPR + me) 8 ..+7.
template <int DT_, int TPR_, int NV_, bool WHOLE_>
struct RowCfg {
  static constexpr int DT = DT_, TPR = TPR_, NV = NV_, NT = TPR_ < 256 ? 256 : TPR_;
  static constexpr bool WHOLE = WHOLE_;
  static constexpr int ROWS = NT / TPR;            // rows of a block
  // the norm's gradient: where a wave has a row, the block's waves add their sums for the gain
  static constexpr int GRAD_LDS_BYTES = ROWS_LDS_BYTES + (ROWS > 1 ? ROWS * NV * 8 * 64 * 4 : 0);
};

template <class C>
__device__ __forceinline__ int chunk_at(int me, int i)
{
  return (i * C::TPR + me) * 8;
}
// whole(n) for a chunk that the row has all of, part(n, e) for each element of its last one
template <class C, class F, class G>
__device__ __forceinline__ void by_chunk(int me, int i, int cols, F&& whole, G&& part)
{
  const int n = chunk_at<C>(me, i);
  if (n + 8 <= cols) {
    whole(n);
  } else if constexpr (!C::WHOLE) {
    if (n < cols) {
#pragma unroll
      for (int e = 0; e < 7; e++)
        if (n + e < cols) part(n, e);
    }
  }
}

// The chunks of a row as they lie in memory; columns past the end are 0, but for what finish() below is there for.
template <class C>
struct Raw {
  RawRow<8, C::DT> c[C::NV];
};
// Where a row of cols elements, 8 or more, is not made of chunks, its last chunk is loaded as the eight elements that the row ends with,
// and chunks past it alike, so that no load waits for a branch; finish() shifts out what is not theirs, once the loads of all
// matrices are on their way.  end_of_row: the last 8 - k elements in front, zeros behind (1 <= k <= 8).  Element by element it took longer:
// gradients of the layer norm of 1531 x 1111 fp16 16.5 us, 12.8 so, norm of 8000 x 1111 bf16 42 and 27.8.
template <int DT>
__device__ __forceinline__ RawRow<8, DT> end_of_row(RawRow<8, DT> r, int k)
{
  constexpr int WORDS = DT == 2 ? 8 : 4;
#pragma unroll
  for (int step = WORDS / 2; step >= 1; step /= 2) {
    const bool by = (k & (DT == 2 ? step : 2 * step)) != 0;
#pragma unroll
    for (int i = 0; i < WORDS; i++) r.w[i] = by ? (i + step < WORDS ? r.w[i + step < WORDS ? i + step : 0] : 0u) : r.w[i];
  }
  if constexpr (DT != 2) {
#pragma unroll
    for (int i = 0; i < WORDS; i++)
      r.w[i] = k & 1 ? r.w[i] >> 16 | (i + 1 < WORDS ? r.w[i + 1 < WORDS ? i + 1 : 0] << 16 : 0u) : r.w[i];
  }
#pragma unroll
  for (int i = 0; i < WORDS; i++) r.w[i] = k >= 8 ? 0u : r.w[i];
  return r;
}
template <class C, class HW>
__device__ __forceinline__ Raw<C> load_raw(const void* row, int me, int cols)
{
  constexpr int DT = C::DT;
  Raw<C> r;
#pragma unroll
  for (int i = 0; i < C::NV; i++) {
    r.c[i] = {};
    if (!C::WHOLE && cols >= 8) {
      const int n = chunk_at<C>(me, i);
      r.c[i] = load_chunk<8, DT, HW>(element_at<DT>(row, n + 8 <= cols ? n : cols - 8));
      continue;
    }
    if (C::WHOLE || i == 0)          // the others lie past a row shorter than a chunk
      by_chunk<C>(
          me, i, cols, [&](int n) __attribute__((always_inline)) { r.c[i] = load_chunk<8, DT, HW>(element_at<DT>(row, n)); },
          [&](int n, int e) __attribute__((always_inline)) {
            const char* at = element_at<DT>(row, n + e);
            if constexpr (DT == 2)
              r.c[i].w[e] = HW::global_load_u32(at);
            else
              r.c[i].w[e / 2] |= (uint32_t)HW::global_load_u16(at) << (e & 1 ? 16 : 0);
          });
  }
  return r;
}
template <class C>
__device__ __forceinline__ void finish(Raw<C>& r, int me, int cols)
{
  if constexpr (!C::WHOLE) {
#pragma unroll
    for (int i = 0; i < C::NV; i++) {
      const int k = chunk_at<C>(me, i) + 8 - cols;
      if (k > 0 && cols >= 8) r.c[i] = end_of_row<C::DT>(r.c[i], k < 8 ? k : 8);
    }
  }
}
template <class C, class HW>
__device__ __forceinline__ float value(const Raw<C>& r, int i, int e)
{
  return element<8, C::DT, HW>(r.c[i], e);
}

// v[NV][8] to a row of type DT (0, 1, 2; 3: e4m3).  The last chunk of a row that is not made of them is picked out first and then stored
// element by element: unrolled for every chunk that might be the last, that takes more than twice the registers.
template <class C, int DT, class HW>
__device__ __forceinline__ void store_values(void* row, int me, int cols, const float (&v)[C::NV][8])
{
  constexpr int WORDS = DT == 2 ? 8 : DT == 3 ? 2 : 4;
  uint32_t last[WORDS] = {};
  int n1 = cols;               // where the row's last chunk starts, if it is this thread's
#pragma unroll
  for (int i = 0; i < C::NV; i++) {
    const int n = chunk_at<C>(me, i);
    const bool whole = n + 8 <= cols;
    if (whole) {
      if constexpr (DT == 3) {
        const uint32_t lo = HW::cvt_e4m3(v[i][0], v[i][1]) | HW::cvt_e4m3(v[i][2], v[i][3]) << 16;
        const uint32_t hi = HW::cvt_e4m3(v[i][4], v[i][5]) | HW::cvt_e4m3(v[i][6], v[i][7]) << 16;
        HW::global_store8_byte((char*)row + n, u32x2{lo, hi});
      } else {
        store_row<8, DT, HW, false>(element_at<DT>(row, n), v[i]);
      }
    }
    if constexpr (!C::WHOLE) {
      const bool mine = !whole && n < cols;
      n1 = mine ? n : n1;
#pragma unroll
      for (int e = 0; e < WORDS; e++) {
        uint32_t w;
        if constexpr (DT == 2)
          w = __builtin_bit_cast(uint32_t, v[i][e]);
        else if constexpr (DT == 3)
          w = HW::cvt_e4m3(v[i][4 * e], v[i][4 * e + 1]) | HW::cvt_e4m3(v[i][4 * e + 2], v[i][4 * e + 3]) << 16;
        else
          w = float_to_half<DT, HW>(v[i][2 * e]) | float_to_half<DT, HW>(v[i][2 * e + 1]) << 16;
        const uint32_t before = last[e];
        last[e] = mine ? w : before;
      }
    }
  }
  if constexpr (!C::WHOLE) {
    char* at = (char*)row + (long)n1 * (DT == 2 ? 4 : DT == 3 ? 1 : 2);
#pragma unroll
    for (int e = 0; e < 7; e++) {
      if (n1 + e < cols) {
        if constexpr (DT == 2)
          HW::global_store_u32(at + 4 * e, last[e]);
        else if constexpr (DT == 3)
          HW::global_store_u8(at + e, (uint8_t)(last[e / 4] >> 8 * (e % 4)));
        else
          HW::global_store_u16(at + 2 * e, (uint16_t)(last[e / 2] >> 16 * (e % 2)));
      }
    }
  }
}

template <class C, class HW>
__device__ __forceinline__ void load_gain(const float* gain, int me, int cols, float (&g)[C::NV][8])
{
#pragma unroll
  for (int i = 0; i < C::NV; i++) {
#pragma unroll
    for (int e = 0; e < 8; e++) g[i][e] = 1.0f;
    if (gain == nullptr) continue;
    if (!C::WHOLE && cols >= 8) {
      const int n = chunk_at<C>(me, i), k = n + 8 - cols;
      RawRow<8, 2> t = load_chunk<8, 2, HW>((const char*)(gain + (k <= 0 ? n : cols - 8)));
      if (k > 0) t = end_of_row<2>(t, k < 8 ? k : 8);
#pragma unroll
      for (int e = 0; e < 8; e++) g[i][e] = element<8, 2, HW>(t, e);
      continue;
    }
    if (C::WHOLE || i == 0)
      by_chunk<C>(
          me, i, cols,
          [&](int n) __attribute__((always_inline)) {
            const RawRow<8, 2> t = load_chunk<8, 2, HW>((const char*)(gain + n));
#pragma unroll
            for (int e = 0; e < 8; e++) g[i][e] = element<8, 2, HW>(t, e);
          },
          [&](int n, int e) __attribute__((always_inline)) { g[i][e] = load_element<2, HW>(gain, n + e); });
  }
}

template <int DT>
__device__ __forceinline__ const char* row_at(const void* base, long row, long ld)
{
  return (const char*)base + row * ld * (DT == 2 ? 4 : 2);
}

// v / scale, each rounded once to fp32, scale >= 2^-126.  The quotient decides on which side of a tie of e4m3 a number lies, and
// the product with 1 / scale, rounded twice, is off at one element in two thousand.  A division is some ten instructions an
// element, this four: the product with the reciprocal in two parts is within one step of the quotient, and such a q, corrected
// by the rest v - q scale (exact in one fma) times the reciprocal, is the quotient rounded to nearest (Markstein, Computation of
// elementary functions on the IBM RISC System/6000 processor, 1990).  Rests of tiny rows need numbers below the fp32 range: rows of
// scales below 2^-64 are multiplied by 2^64 first.  8192 x 4096 bf16 17.2 us, 16.75 with the product alone.
template <class HW, int NV>
__device__ __forceinline__ void divide_row(float (&v)[NV][8], float scale)
{
  if (scale < 0x1p-64f) {
    scale *= 0x1p64f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) v[i][e] *= 0x1p64f;
  }
  // head + low is the reciprocal, low >= 0, and the rest is taken with its sign turned, so that -0 stays -0
  const float inv = 1.0f / scale;
  const float head = HW::fma(-scale, inv, 1.0f) < 0.f ? __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, inv) - 1) : inv;
  // of an infinite row nothing is corrected
  const bool finite = scale < __builtin_inff();
  const float low = finite ? HW::fma(-scale, head, 1.0f) * inv : 0.f, by = finite ? scale : 0.f;
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float q = HW::fma(v[i][e], head, v[i][e] * low);
      v[i][e] = HW::fma(-HW::fma(q, by, -v[i][e]), inv, q);
    }
}

// ---- norm, 8 bits ------------------------------------------------------------------------------------------------
// A row h of the result, in type `out` (3: e4m3, whose scale goes to scale[row]); `at`: LDS of the row's maximum; no cols: nothing is stored.
template <class C, class HW>
__device__ __forceinline__ void store_result(float (&h)[C::NV][8], void* base, long ld, int out, float* scale_of, long row, int me,
                                             int cols, uint32_t at)
{
  constexpr int NV = C::NV;
  if (out == 3) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const uint32_t b = __builtin_bit_cast(uint32_t, h[i][e]) & 0x7fffffffu;
        // a thread past the row's end holds zeros, which a gain of its own must not turn into NaN
        if (chunk_at<C>(me, i) + e < cols) top = b > top ? b : top;
      }
    top = row_max<C::TPR, HW>(top, at);
    const float peak = __builtin_bit_cast(float, top) / 448.0f;
    const float scale = peak < 1.17549435e-38f ? 1.17549435e-38f : peak;     // NaN stays
    if (me == 0 && cols > 0) HW::global_store_u32(scale_of + row, __builtin_bit_cast(uint32_t, scale));
    divide_row<HW>(h, scale);
  }
  char* y = (char*)base + row * ld * (out == 3 ? 1 : out == 2 ? 4 : 2);
  if (out == 3)
    store_values<C, 3, HW>(y, me, cols, h);
  else
    by_type(out, [&](auto t) __attribute__((always_inline)) { store_values<C, decltype(t)::value, HW>(y, me, cols, h); });
}

template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_norm_rows(const NormArgs p)
{
  constexpr int NV = C::NV, DT = C::DT;
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int me = tid % C::TPR;
  const long row = (long)HW::block_x() * C::ROWS + tid / C::TPR;
  if (row >= p.rows) return;                       // a whole wave, where a wave has a row; else never
  const bool norm = (p.flags & 4) != 0;
  const int out = p.flags & 3;

  Raw<C> x = load_raw<C, HW>(row_at<DT>(p.x, row, p.ldx), me, p.cols), r = {};
  // ahead of everything else where the row's end takes a while to be cut; else that costs rows without a residual registers (8192 x 4096
  // bf16 to 8 bits 18.4 us and 17.3)
  constexpr bool R_AHEAD = !C::WHOLE;
  if (R_AHEAD && p.residual != nullptr) r = load_raw<C, HW>(row_at<DT>(p.residual, row, p.ldr), me, p.cols);
  // ahead of the sum that it does not depend on, where there are registers for it
  constexpr bool GAIN_AHEAD = C::TPR < 1024 || NV < 4;
  float g[NV][8];
  if (GAIN_AHEAD && norm) load_gain<C, HW>(p.gain, me, p.cols, g);
  float h[NV][8];
  finish<C>(x, me, p.cols);
  if (p.residual != nullptr) {
    if (!R_AHEAD) r = load_raw<C, HW>(row_at<DT>(p.residual, row, p.ldr), me, p.cols);
    finish<C>(r, me, p.cols);
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) h[i][e] = value<C, HW>(x, i, e) + value<C, HW>(r, i, e);
  } else {
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) h[i][e] = value<C, HW>(x, i, e);
  }
  if (p.total != nullptr)
    store_values<C, DT, HW>((void*)row_at<DT>(p.total, row, p.ldt), me, p.cols, h);
  if (norm) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) s += h[i][e] * h[i][e];
    s = row_sum<C::TPR, HW>(s, lds);
    const float rstd = 1.0f / HW::sqrt(s / (float)p.cols + p.eps);
    if (!GAIN_AHEAD) load_gain<C, HW>(p.gain, me, p.cols, g);
    if (p.rstd != nullptr && me == 0) HW::global_store_u32(p.rstd + row, __builtin_bit_cast(uint32_t, rstd));
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) h[i][e] = h[i][e] * rstd * g[i][e];
  }
  store_result<C, HW>(h, p.y, p.ldy, out, p.scale, row, me, p.cols, lds + 64);
}

// ---- gradients of the norm ------------------------------------------------------------------------------------------
// A group of TPR threads takes rows g, g + groups, ... and keeps the sums of dgain for its columns in registers; the waves of a
// block add theirs where each has a row, alcop_column_sums adds the blocks'.
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_norm_grad(const NormGradArgs p, int groups)
{
  constexpr int NV = C::NV, DT = C::DT;
  // rows of more elements than the registers have room for are read again behind the sum
  constexpr bool HOLD = NV * C::TPR <= 2048;
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int me = tid % C::TPR;
  const int group = (int)HW::block_x() * C::ROWS + tid / C::TPR;
  float dg[NV][8];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) dg[i][e] = 0.f;
  constexpr bool GAIN_HELD = NV <= 2 && C::TPR < 1024;      // as far as the registers go
  float g[NV][8];
  if (GAIN_HELD) load_gain<C, HW>(p.gain, me, p.cols, g);
  int turn = 0;
  for (long row = group; row < p.rows; row += groups, turn ^= 1) {
    const char *dy_row = row_at<DT>(p.dy, row, p.lddy), *h_row = row_at<DT>(p.total, row, p.ldt);
    Raw<C> dy = load_raw<C, HW>(dy_row, me, p.cols);
    Raw<C> h = load_raw<C, HW>(h_row, me, p.cols);
    const char* dt_row = row_at<DT>(p.dtotal, row, p.lddt);
    Raw<C> dt = {};
    constexpr bool AHEAD = NV * C::TPR <= 1024;    // of the sum, where there are registers for it
    if (AHEAD && p.dtotal != nullptr) dt = load_raw<C, HW>(dt_row, me, p.cols);
    const float rstd = __builtin_bit_cast(float, HW::global_load_u32(p.rstd + row));
    if (!GAIN_HELD) load_gain<C, HW>(p.gain, me, p.cols, g);
    finish<C>(dy, me, p.cols);
    finish<C>(h, me, p.cols);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float d = value<C, HW>(dy, i, e), xh = value<C, HW>(h, i, e) * rstd;
        s += d * g[i][e] * xh;
        dg[i][e] += d * xh;
      }
    const float mean = row_sum<C::TPR, HW>(s, lds + 64 * turn) / (float)p.cols;
    if constexpr (!HOLD) {
      dy = load_raw<C, HW>(dy_row, me, p.cols);
      h = load_raw<C, HW>(h_row, me, p.cols);
      load_gain<C, HW>(p.gain, me, p.cols, g);
      finish<C>(dy, me, p.cols);
      finish<C>(h, me, p.cols);
    }
    float dx[NV][8];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++)
        dx[i][e] = rstd * (value<C, HW>(dy, i, e) * g[i][e] - value<C, HW>(h, i, e) * rstd * mean);
    if (p.dtotal != nullptr) {
      if (!AHEAD) dt = load_raw<C, HW>(dt_row, me, p.cols);
      finish<C>(dt, me, p.cols);
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) dx[i][e] += value<C, HW>(dt, i, e);
    }
    store_values<C, DT, HW>((void*)row_at<DT>(p.dx, row, p.lddx), me, p.cols, dx);
  }
  if (p.partial == nullptr) return;
  if constexpr (C::ROWS > 1) {
    const uint32_t at = lds + ROWS_LDS_BYTES + (uint32_t)me * 4;
    const int wave = HW::wave_id();
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int e = 0; e < 8; e++)
        HW::lds_write1(at + (uint32_t)((wave * NV + i) * 8 + e) * 256, __builtin_bit_cast(uint32_t, dg[i][e]));
    HW::wait_lds();
    HW::block_barrier();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < C::ROWS; w++)
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) dg[i][e] += __builtin_bit_cast(float, HW::lds_read4(at + (uint32_t)((w * NV + i) * 8 + e) * 256));
  }
  store_values<C, 2, HW>(p.partial + (long)HW::block_x() * p.cols, me, p.cols, dg);
}

// ---- column sums ------------------------------------------------------------------------------------------------------
// out[j] = sum over i of partial[i][j], in a fixed order: 32 columns a block, 32 runs of rows, then the runs.
constexpr int SUM_THREADS = 1024, SUM_COLS = 32;
template <class HW, int THREADS = SUM_THREADS>
__device__ __forceinline__ void column_sums(const ColumnSumArgs& p)
{
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int c = tid % SUM_COLS, run = tid / SUM_COLS;
  const int j = (int)HW::block_x() * SUM_COLS + c;
  float s = 0.f;
  if (j < p.cols) {
#pragma unroll 8
    for (int i = run; i < p.count; i += THREADS / SUM_COLS)
      s += __builtin_bit_cast(float, HW::global_load_u32(p.partial + (long)i * p.cols + j));
  }
  HW::lds_write1(lds + 4 * (run * SUM_COLS + c), __builtin_bit_cast(uint32_t, s));
  HW::wait_lds();
  HW::block_barrier();
  if (tid >= 64) return;
  float t = 0.f;
#pragma unroll 4
  for (int i = 0; i < THREADS / SUM_COLS; i++) t += __builtin_bit_cast(float, HW::lds_read4(lds + 4 * (i * SUM_COLS + c)));
  if (tid < SUM_COLS && j < p.cols) HW::global_store_u32(p.out + j, __builtin_bit_cast(uint32_t, t));
}
template <class HW>
__global__ void __launch_bounds__(SUM_THREADS) alcop_column_sums(const ColumnSumArgs p)
{
  column_sums<HW>(p);
}

// ---- gradient of an activation, sums for the bias ----------------------------------------------------------------------
// dZ = dC act'(Z), rounded to the operands' type: it is an operand of the two products that follow, which take
// 16 bits.  A block has 512 columns (or all, where there are fewer) and a run of rows; of 64 lanes `p.lanes` share a row,
// so that a wave has 64 / lanes rows at a time; 16-byte chunks.
constexpr int ACT_COLS = 512;
// Rows r0 .. r1 - 1 of it, whose sums go to row `part` of the partial ones.
template <int DT, class HW>
__device__ __forceinline__ void act_grad(const ActGradArgs& p, long r0, long r1, long part)
{
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int mine = tid & (p.lanes - 1), rows = 256 / p.lanes;     // lanes: a power of two
  const int n = (int)HW::block_x() * ACT_COLS + mine * 8;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; e++) sum[e] = 0.f;
  if (n < p.N) {
    for (long m = r0 + tid / p.lanes; m < r1; m += rows) {
      const RawRow<8, DT> dc = load_chunk<8, DT, HW>(element_at<DT>(p.dc, m * p.lddc + n));
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = element<8, DT, HW>(dc, e);
      if (p.act != ACT_NONE) {
        const RawRow<8, DT> z = load_chunk<8, DT, HW>(element_at<DT>(p.pre, m * p.ldp + n));
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] *= slope<HW>(element<8, DT, HW>(z, e), p.act);
      }
      if (p.dz != nullptr) store_row<8, DT, HW, true>(element_at<DT>(p.dz, m * p.ldz + n), v);
#pragma unroll
      for (int e = 0; e < 8; e++) sum[e] += v[e];
    }
  }
  if (p.partial == nullptr) return;
  // sums of the block's `rows` groups of lanes: [group][8 lanes columns], 2048 values; then column by column
  HW::lds_write(lds + (uint32_t)tid * 32, f32x4{sum[0], sum[1], sum[2], sum[3]});
  HW::lds_write(lds + (uint32_t)tid * 32 + 16, f32x4{sum[4], sum[5], sum[6], sum[7]});
  HW::wait_lds();
  HW::block_barrier();
  const int width = p.lanes * 8;
#pragma unroll 1
  for (int c0 = 0; c0 < width; c0 += 256) {
    const int c = c0 + tid, j = (int)HW::block_x() * ACT_COLS + c;
    float t = 0.f;
#pragma unroll 4
    for (int g = 0; g < rows; g++) t += __builtin_bit_cast(float, HW::lds_read4(lds + (uint32_t)(g * width + (c < width ? c : 0)) * 4));
    if (c < width && j < p.N) HW::global_store_u32(p.partial + part * p.N + j, __builtin_bit_cast(uint32_t, t));
  }
}
template <int DT, class HW>
__global__ void __launch_bounds__(256) alcop_act_grad(const ActGradArgs p)
{
  const long r0 = (long)HW::block_y() * p.rows_per_block;
  act_grad<DT, HW>(p, r0, r0 + p.rows_per_block < p.M ? r0 + p.rows_per_block : p.M, (long)HW::block_y());
}

}  // namespace alcop
