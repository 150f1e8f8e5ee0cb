// Cross entropy of rows against the product with a vocabulary's vectors, without keeping the logits, and its gradients.
//
//     z[t][v] = alpha sum_k X(t,k) W(v,k);   lse[t] = log sum_v exp z[t][v];   loss[t] = lse[t] - z[t][label[t]]
//     G[t][v] = dloss[t] (exp(z[t][v] - lse[t]) - [v = label[t]]);   dX = alpha G W;   dW = alpha G^T X
//
// Forward: the product's loop (alcop_kernel.hip.h) with an epilogue that leaves of every tile, for each of its rows, the largest logit and
// the sum of exp over the tile's columns relative to it: 8 bytes in place of a tile's row.  In the accumulators a lane holds
// half of a row's columns, so both come out of registers and one exchange of two lanes; the waves side by side meet in LDS.  A second
// kernel merges the strips, in a fixed order.
//
// Backward: the logits are computed again, a piece of the vocabulary at a time, and leave as G in 16 bits (the two products
// behind it take such operands); dW of the piece is whole, dX is added up over the pieces in fp32.  That is four products in all, of
// which none reads or writes rows x vocabulary numbers beyond one piece.
//
// G in fp16: its numbers are as small as dloss / vocabulary, which fp16 does not reach.  They are multiplied by a power of two S
// that takes the largest |dloss| of the rows that count to 2^14 .. 2^15 (G is at most that), and the products by 1 / S.  bf16 has
// fp32's range, S = 1.
//
// What bounds them: the matrix cores.  8192 rows, 65536 x 2048 bf16: 1.83 to 1.94 ms by card = 1.20 to 1.13 PFLOP/s (the cores 67 % busy
// at the 1.7 GHz that power leaves), 6 us for the strips.  Gradients of 4096 rows: four pieces of 248 to 256 us for the logits and G (1.11
// to 1.08 PFLOP/s), 220 to 226 for dX and 207 to 215 for dW, 15 in the end to round dX.  509 x 30011 x 768 fp16, one turn of the card: 31 us, in which 46 MB of new vectors are read, and 5.
//
// Exponents are of 2: u = z log2 e, exp2(u - shift) with u - shift in one fma from the accumulator.
#pragma once
#include "alcop_rows.hip.h"

namespace alcop {

constexpr float LOG2_E = 1.44269504089f, LN_2 = 0.69314718056f;

// (shift, sum) stands for sum 2^shift; (-infinity, 0) for nothing.  A strip's shift is finite; one whose logits are all -infinity
// has the sum 0 and must not move the shift.  The smaller one's factor is 2^-126 at least: beside the other's sum of some 1 that is nothing,
// and a sum that an infinite logit made infinite (its strip has the shift 0) stays so, where 0 would make it NaN.  No branch: the strips of
// a row are a chain of such steps (5 rows of 34328 x 528
// bf16 23.4 us with a second factor of exp2(0) and a branch for sums of 0, 16.3 so).
template <class HW>
__device__ __forceinline__ void add_strip(float& shift, float& sum, float shift2, float sum2)
{
  shift2 = sum2 == 0.f ? -__builtin_inff() : shift2;
  const bool up = shift2 > shift;
  const float d = up ? shift - shift2 : shift2 - shift;              // NaN where both are nothing, which is taken as -126
  const float f = HW::exp2(__builtin_fmaxf(d, -126.f));
  sum = up ? HW::fma(sum, f, sum2) : HW::fma(sum2, f, sum);
  shift = up ? shift2 : shift;
}

struct LossArgs {
  const void *X, *W;
  const void* labels;          // 64-bit numbers
  void* out;                   // forward: pairs (shift, sum), [strip][row]; backward: G
  float* hit;                  // forward: the label's logit, as accumulated (without alpha)
  const float *lse, *dloss, *scale;      // backward; scale: S, or null = `s`
  int M, N, K, lda, ldw, ldg;
  int v0, vocab;               // the piece's first column, and all columns
  float alpha, s;
};

struct LossParams : Params {
  const char* labels;
  float* hit;
  const float *lse, *dloss, *scale;
  int v0, vocab;
  float s;
};
template <class C>
__device__ __forceinline__ LossParams expand_loss(const LossArgs& a)
{
  LossParams p = {};
  p.A = a.X;
  p.B = a.W;
  p.C = a.out;
  p.M = p.Mv = a.M;
  p.N = p.Nv = a.N;
  p.K = a.K;
  p.lda = a.lda;
  p.ldb = a.ldw;
  p.ldc = a.ldg;
  p.alpha = a.alpha;
  p.raster = 1;
  p.ntm = (p.M + C::BM - 1) / C::BM;
  p.ntn = (p.N + C::BN - 1) / C::BN;
  p.group_m = p.ntm < 8 ? p.ntm : 8;
  p.labels = (const char*)a.labels;
  p.hit = a.hit;
  p.lse = a.lse;
  p.dloss = a.dloss;
  p.scale = a.scale;
  p.v0 = a.v0;
  p.vocab = a.vocab;
  p.s = a.s;
  return p;
}

// What a lane needs of its rows m0 + 32 j + lane % 32, fetched ahead of the main loop: the label's column in the piece (-1: not
// there), and backward lse in exponents of 2, dloss S, and whether the row counts.
template <class C>
struct LossAhead {
  int at[C::TM];
  float lse2[C::TM], weight[C::TM];
  bool counts[C::TM];
  template <class HW>
  __device__ __forceinline__ void load(const LossParams& p, int m0, int, int lane)
  {
#pragma unroll
    for (int j = 0; j < C::TM; j++) {
      const int m = m0 + 32 * j + (lane & 31), row = m < p.M ? m : 0;
      const char* label = p.labels + (long)row * 8;
      // a label is a column of the vocabulary, below 2^31; negative ones have bits above
      const uint32_t lo = HW::global_load_u32(label), hi = HW::global_load_u32(label + 4);
      counts[j] = hi == 0 && lo < (uint32_t)p.vocab;
      const int col = (int)lo - p.v0;
      at[j] = counts[j] && m < p.M && col >= 0 && col < p.N ? col : -1;
      if constexpr (C::BACKWARD) {
        const float s = p.scale != nullptr ? __builtin_bit_cast(float, HW::global_load_u32(p.scale)) : p.s;
        const float d = p.dloss != nullptr ? __builtin_bit_cast(float, HW::global_load_u32(p.dloss + row)) : 1.0f;
        lse2[j] = __builtin_bit_cast(float, HW::global_load_u32(p.lse + row)) * LOG2_E;
        weight[j] = d * s;
      }
    }
  }
  template <class HW>
  __device__ __forceinline__ void load_late(const LossParams&, int, int, int)
  {
  }
};

// Element v of sub-tile i is column 32 i + 8 (v / 4) + 4 (lane / 32) + v % 4 of the wave's tile.
__device__ __forceinline__ int column_of(int i, int v, int lane) { return 32 * i + 8 * (v / 4) + 4 * (lane >> 5) + v % 4; }

// Forward: (shift, sum) of the block's rows over its columns, and the label's accumulator where it is among them.
template <class C, class HW>
__device__ __forceinline__ void loss_strip(const LossParams& p, LossAhead<C>& ahead, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, int lane)
{
  constexpr int TN = C::TN, TM = C::TM;
  const uint32_t lds = HW::lds_base();
  const int wave_n = n0 % C::BN / C::WN, row0 = m0 % C::BM + (lane & 31);
  const float a2 = p.alpha * LOG2_E;
  const bool edge = n0 + C::WN > p.N;
#pragma unroll
  for (int j = 0; j < TM; j++) {
    if (edge) {
#pragma unroll
      for (int i = 0; i < TN; i++)
#pragma unroll
        for (int v = 0; v < 16; v++)
          if (n0 + column_of(i, v, lane) >= p.N) acc[i][j][v] = -__builtin_inff();
    }
    const int y = ahead.at[j] - n0;            // negative where there is none
    if (HW::ballot(y >= 0 && y < C::WN)) {
      float hit = 0.f;
      bool here = false;
#pragma unroll
      for (int i = 0; i < TN; i++)
#pragma unroll
        for (int v = 0; v < 16; v++)
          if (column_of(i, v, lane) == y) {
            hit = acc[i][j][v];
            here = true;
          }
      if (here) HW::global_store_u32(p.hit + m0 + 32 * j + (lane & 31), __builtin_bit_cast(uint32_t, hit));
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int v = 0; v < 16; v++) top = acc[i][j][v] > top ? acc[i][j][v] : top;
    const float other = __builtin_bit_cast(float, HW::xor_lanes(__builtin_bit_cast(uint32_t, top), 32));
    top = (other > top ? other : top) * a2;
    // an infinite logit is itself what comes out, of a row without any the sum is 0
    const float shift = __builtin_fabsf(top) < __builtin_inff() ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int v = 0; v < 16; v++) sum += HW::exp2(HW::fma(acc[i][j][v], a2, -shift));
    sum += __builtin_bit_cast(float, HW::xor_lanes(__builtin_bit_cast(uint32_t, sum), 32));
    HW::lds_write(lds + (uint32_t)((wave_n * C::BM + row0 + 32 * j) * 8),
                  u32x2{__builtin_bit_cast(uint32_t, shift), __builtin_bit_cast(uint32_t, sum)});
  }
  HW::wait_lds();
  HW::block_barrier();
  const int row = HW::wave_id() * 64 + lane;
  const long m = m0 / C::BM * (long)C::BM + row;
  if (row >= C::BM) return;
  float shift = -__builtin_inff(), sum = 0.f;
#pragma unroll
  for (int w = 0; w < C::WAVES_N; w++) {
    const u32x2 t = HW::lds_read8(lds + (uint32_t)((w * C::BM + row) * 8));
    const uint32_t t0 = t[0], t1 = t[1];
    add_strip<HW>(shift, sum, __builtin_bit_cast(float, t0), __builtin_bit_cast(float, t1));
  }
  if (m < p.M)
    HW::global_store8_any((char*)p.C + ((long)(n0 / C::BN) * p.M + m) * 8,
                          u32x2{__builtin_bit_cast(uint32_t, shift), __builtin_bit_cast(uint32_t, sum)});
}

// Backward: G of the wave's tile in 16 bits, columns from N up to the next multiple of 8 as 0.
template <class C, class HW>
__device__ __forceinline__ void loss_gradient(const LossParams& p, LossAhead<C>& ahead, f32x16 (&acc)[C::TN][C::TM], int m0, int n0,
                                              uint32_t ebase, int lane)
{
  constexpr int TN = C::TN, TM = C::TM, RS = C::WN * 2 + 16, LPR = C::WN / 8, RPI = 64 / LPR;
  const float a2 = p.alpha * LOG2_E;
  const bool edge = n0 + C::WN > p.N;
#pragma unroll
  for (int j = 0; j < TM; j++) {
    const int y = ahead.at[j] - n0;            // negative where there is none
    const bool hit = HW::ballot(y >= 0 && y < C::WN) != 0;
    const uint32_t row = ebase + (lane & 31) * RS + 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int vq = 0; vq < 4; vq++) {
        float g[4];
#pragma unroll
        for (int e = 0; e < 4; e++) g[e] = HW::exp2(HW::fma(acc[i][j][4 * vq + e], a2, -ahead.lse2[j]));
        if (hit) {
#pragma unroll
          for (int e = 0; e < 4; e++) g[e] -= column_of(i, 4 * vq + e, lane) == y ? 1.0f : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const bool there = ahead.counts[j] && !(edge && n0 + column_of(i, 4 * vq + e, lane) >= p.N);
          g[e] = there ? g[e] * ahead.weight[j] : 0.f;
        }
        HW::lds_write(row + (i * 32 + 8 * vq) * 2,
                      u32x2{float_to_half<C::DT, HW>(g[0]) | float_to_half<C::DT, HW>(g[1]) << 16,
                            float_to_half<C::DT, HW>(g[2]) | float_to_half<C::DT, HW>(g[3]) << 16});
      }
#pragma unroll
    for (int t = 0; t < 32 / RPI; t++) {
      const int r = t * RPI + lane / LPR, c8 = lane % LPR * 8, m = m0 + 32 * j + r, n = n0 + c8;
      const u32x4 v = HW::lds_read16(ebase + r * RS + c8 * 2);
      if ((m < p.M) & (n < p.N)) HW::global_store16_through((char*)p.C + ((long)m * p.ldc + n) * 2, v);
    }
  }
}

// what linear_tile (alcop_linear.hip.h) calls with these parameters; out_dtype is 0
template <class C, int DT, class HW>
__device__ __forceinline__ void linear_bands(const LossParams& p, LossAhead<C>& ahead, f32x16 (&acc)[C::TN][C::TM], int m0, int n0,
                                             uint32_t ebase, int lane)
{
  if constexpr (DT != 0)
    return;
  else if constexpr (C::BACKWARD)
    loss_gradient<C, HW>(p, ahead, acc, m0, n0, ebase, lane);
  else
    loss_strip<C, HW>(p, ahead, acc, m0, n0, lane);
}

template <bool BACKWARD_, int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
struct LossCfg : KCfg<DT, BM, BN, BK, WM, WN, S, R, F, 1, 0> {
  static constexpr bool LINEAR = true, BACKWARD = BACKWARD_;
  using Ahead = LossAhead<LossCfg>;
};
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_loss_tile(const LossArgs a)
{
  mainloop_body<C, HW>(expand_loss<C>(a));
}

// ---- the strips of a row: lse and the loss ---------------------------------------------------------------------
// 32 rows a block, 32 runs of strips, then the runs.
struct LossRowsArgs {
  const char* strips;
  const void* labels;
  const float* hit;
  float *loss, *lse;
  int rows, count, vocab;
  float alpha;
};
template <class HW>
__global__ void __launch_bounds__(1024) alcop_loss_rows(const LossRowsArgs p)
{
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  const int c = tid & 31, run = tid >> 5;
  const long row = (long)HW::block_x() * 32 + c;
  float shift = -__builtin_inff(), sum = 0.f;
  if (row < p.rows) {
#pragma unroll 4
    for (int i = run; i < p.count; i += 32) {
      const u32x2 t = HW::global_load8_any(p.strips + ((long)i * p.rows + row) * 8);
      const uint32_t t0 = t[0], t1 = t[1];
      add_strip<HW>(shift, sum, __builtin_bit_cast(float, t0), __builtin_bit_cast(float, t1));
    }
  }
  HW::lds_write(lds + (uint32_t)tid * 8, u32x2{__builtin_bit_cast(uint32_t, shift), __builtin_bit_cast(uint32_t, sum)});
  HW::wait_lds();
  HW::block_barrier();
  if (tid >= 64) return;
  shift = -__builtin_inff();
  sum = 0.f;
#pragma unroll 4
  for (int i = 0; i < 32; i++) {
    const u32x2 t = HW::lds_read8(lds + (uint32_t)(i * 32 + c) * 8);
    const uint32_t t0 = t[0], t1 = t[1];
    add_strip<HW>(shift, sum, __builtin_bit_cast(float, t0), __builtin_bit_cast(float, t1));
  }
  if (tid >= 32 || row >= p.rows) return;
  const float bits = __builtin_log2f(sum), lse = LN_2 * (shift + bits);
  if (p.lse != nullptr) HW::global_store_u32(p.lse + row, __builtin_bit_cast(uint32_t, lse));
  const char* label = (const char*)p.labels + row * 8;
  const bool counts = HW::global_load_u32(label + 4) == 0 && HW::global_load_u32(label) < (uint32_t)p.vocab;
  float loss = 0.f;
  if (counts) {
    // not lse - z: both are rounded where they are, which of a row that is predicted well leaves nothing.  The label's exponent is
    // taken relative to the shift by the same fma as in the sum, so that where it is the largest the two agree but for exp2 and log2
    // (label logits of 15 to 60, loss 0: off by up to 3.8e-6 before, one in ten negative)
    const float d = HW::fma(__builtin_bit_cast(float, HW::global_load_u32(p.hit + row)), p.alpha * LOG2_E, -shift);
    loss = LN_2 * (bits - d);
    loss = loss < 0.f ? 0.f : loss;          // NaN stays
  }
  HW::global_store_u32(p.loss + row, __builtin_bit_cast(uint32_t, loss));
}

// ---- S: the power of two that takes the largest |dloss| to 2^14 .. 2^15, and 1 / S ---------------------------------
// Of the rows that count, and of finite ones: what a masked row holds there, or a row that is lost anyway, must not shrink the others.
struct LossScaleArgs {
  const float* dloss;
  const void* labels;
  float* scale;
  int rows, vocab;
};
template <class HW>
__global__ void __launch_bounds__(1024) alcop_loss_scale(const LossScaleArgs p)
{
  const uint32_t lds = HW::lds_base();
  const int tid = HW::wave_id() * 64 + HW::lane_id();
  uint32_t top = 0;
#pragma unroll 4
  for (int i = tid; i < p.rows; i += 1024) {
    const uint32_t b = HW::global_load_u32(p.dloss + i) & 0x7fffffffu;
    const char* label = (const char*)p.labels + (long)i * 8;
    const bool counts = HW::global_load_u32(label + 4) == 0 && HW::global_load_u32(label) < (uint32_t)p.vocab;
    top = counts && b < 0x7f800000u && b > top ? b : top;
  }
  top = row_max<1024, HW>(top, lds);
  int e = 14 - ((int)(top >> 23) - 127);
  e = e > 126 ? 126 : e;                   // -113 at least; S and 1 / S are normal numbers
  if (tid == 0) {
    HW::global_store_u32(p.scale, (uint32_t)(127 + e) << 23);
    HW::global_store_u32(p.scale + 1, (uint32_t)(127 - e) << 23);
  }
}

// ---- dX += alpha / S G W, dW = alpha / S G^T X -----------------------------------------------------------------------
struct LossProductArgs {
  LinearArgs l;                // dX: A = G, W = the piece's vectors.  dW: A = G, W = X
  const float* inverse;        // 1 / S, or null = 1
  int depth;                   // dX: the piece's columns, of which K is the next multiple of 8.  dW: its rows, M likewise
  int slice;                   // dX: columns that blocks y have each, a multiple of 64, or K
  long next;                   // dX: elements from the sums of one slice to the next one's
};
struct DepthParams : LinearParams {
  int depth;
};
__device__ __forceinline__ int depth_of_b(const DepthParams& p, int) { return p.depth; }

template <class HW>
__device__ __forceinline__ float with_inverse(float alpha, const float* inverse)
{
  return inverse != nullptr ? alpha * __builtin_bit_cast(float, HW::read_lane(HW::global_load_u32(inverse), 0)) : alpha;
}
// G's columns past the piece are 0, the vectors' rows there lie beyond the descriptor.  The piece is a long axis: where dX has too few tiles
// to fill the card, blocks y add up a slice of it each, in sums of their own.
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_loss_dx(const LossProductArgs a)
{
  DepthParams p = {};
  (LinearParams&)p = expand_linear<C>(a.l);
  p.alpha = with_inverse<HW>(p.alpha, a.inverse);
  const int y = (int)HW::block_y(), k0 = y * a.slice;
  p.K = p.K - k0 < a.slice ? p.K - k0 : a.slice;
  p.depth = a.depth - k0 < p.K ? a.depth - k0 : p.K;
  p.A = (const char*)p.A + (long)k0 * 2;
  p.B = (const char*)p.B + (long)k0 * p.ldb * 2;
  if (y) {
    p.C = (float*)p.C + y * a.next;
    if (p.residual != nullptr) p.residual = (const float*)p.residual + y * a.next;
  }
  mainloop_body<C, HW>(p);
}
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_loss_dw(const LossProductArgs a)
{
  Params p = expand_linear<C>(a.l);
  p.alpha = with_inverse<HW>(p.alpha, a.inverse);
  p.Mv = a.depth;
  p.keep = 0;
  mainloop_body<C, HW>(p);
}

// ---- dX after the last piece: the slices' sums, rounded ------------------------------------------------------------------
struct RoundArgs {
  const float* from;
  void* to;
  long ld;                     // of `to`; `from` has none
  int rows, cols, out;         // cols: a multiple of 8
  int slices;
};
template <class HW>
__global__ void __launch_bounds__(256) alcop_round_rows(const RoundArgs p)
{
  const int per_row = p.cols / 8;
  const long i = (long)HW::block_x() * 256 + HW::wave_id() * 64 + HW::lane_id(), row = i / per_row;
  if (row >= p.rows) return;
  const int n = (int)(i - row * per_row) * 8;
  const RawRow<8, 2> r = load_chunk<8, 2, HW, true>((const char*)(p.from + row * p.cols + n));
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = element<8, 2, HW>(r, e);
  for (int z = 1; z < p.slices; z++) {
    const RawRow<8, 2> t = load_chunk<8, 2, HW, true>((const char*)(p.from + (z * (long)p.rows + row) * p.cols + n));
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] += element<8, 2, HW>(t, e);
  }
  by_type(p.out, [&](auto t) __attribute__((always_inline)) {
    store_row<8, decltype(t)::value, HW, false>(element_at<decltype(t)::value>(p.to, row * p.ld + n), v);
  });
}

}  // namespace alcop
