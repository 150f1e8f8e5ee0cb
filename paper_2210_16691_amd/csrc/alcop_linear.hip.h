// Linear layers: a product with everything that stands between it and the next operator in its epilogue.
//
//     Z[i][j] = alpha * sa[i] * sw[j] * sum_k A(i,k) W(k,j) + bias[j]        (kept as `pre` if asked for)
//     C[i][j] = act(Z[i][j]) + residual[i][j]
//
// on fp16, bf16 or e4m3 operands (sa, sw: the scales of 8-bit rows and output channels), all in fp32 on the
// accumulators and rounded once to the output type; what is kept as `pre` is Z rounded, the activation sees Z.
//
// The loops are those of alcop_kernel.hip.h and alcop_ksplit.hip.h.  An e4m3 operand is to them one of 16-bit
// elements, two e4m3 each: K and the pitches count pairs, and a fragment's 16 bytes are sixteen k in place of eight, for
// two matrix instructions.  Which k a lane holds differs from the 16-bit layouts, but equally for both operands, and a
// sum over k does not ask for their order.  They are widened to bf16 in registers, or (large products whose result is
// rounded to 16 bits) multiplied as they are, at twice the rate: alcop_gfx950.hip.h says what that costs a sum.
//
// Epilogue of a tile (linear_tile): as in alcop_kernel.hip.h a wave parks 32 rows of its accumulators in LDS, here
// in fp32, and reads them back along the rows, eight columns a lane, so that residual, pre and C move in 16-byte
// accesses (at any element) that cover whole lines.  A lane's columns are the same in every row: bias and column scales
// are fetched once per tile.
//
// What bounds it.  The loop of a large layer runs at 1.26 PFLOP/s on bf16 and 2.7 on e4m3 (power, as for the plain products);
// the epilogue stands beside it, as all compute units write at once: 8192 x 8192 x 2048 bf16 with GELU and pre 265 us, of which
// 218 are left if every block stops behind its loop, 8192 x 8192 x 4096 e4m3 with a residual 262, of which 202 are.  While decoding it is the weights' bytes:
// 16 x 4096 x 4096 on e4m3 5.2 us, bf16 8.1.  A single token's call, 768 x 768, takes what a launch takes, 3.0 us in a graph.
#pragma once
#include "alcop_ksplit.hip.h"

namespace alcop {

template <int V>
struct TypeOf {
  static constexpr int value = V;
};

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

// The arguments of a launch.  K and the pitches of A and W in 16-bit units.
struct LinearArgs {
  const void *A, *W;
  void* C;
  const void* residual;
  void* pre;
  const float *bias, *sa, *sw;
  int M, N, K, lda, ldw, ldc, ldr, ldp;
  float alpha;
  int flags;                   // output type | activation << 2 | C is kept in the caches << 5
};

struct LinearParams : Params {
  const void* residual;
  void* pre;
  const float *sa, *sw;
  int ldr, ldp;
};

template <class C>
__device__ __forceinline__ LinearParams expand_linear(const LinearArgs& a)
{
  LinearParams p = {};
  p.A = a.A;
  p.B = a.W;
  p.C = a.C;
  p.M = p.Mv = a.M;
  p.N = p.Nv = a.N;
  p.K = a.K;
  p.lda = a.lda;
  p.ldb = a.ldw;
  p.ldc = a.ldc;
  p.bias = a.bias;
  p.alpha = a.alpha;
  p.out_dtype = a.flags & 3;
  p.act = (a.flags >> 2) & 7;
  p.keep = (short)(a.flags >> 5 & 1);
  p.raster = 1;
  p.ntm = (p.M + C::BM - 1) / C::BM;
  p.ntn = (p.N + C::BN - 1) / C::BN;
  p.group_m = p.ntm < 8 ? p.ntm : 8;
  p.residual = a.residual;
  p.pre = a.pre;
  p.sa = a.sa;
  p.sw = a.sw;
  p.ldr = a.ldr;
  p.ldp = a.ldp;
  return p;
}

// ---- activations ---------------------------------------------------------------------------------------
// SiLU and the tanh form of GELU are z * sigmoid(u) with u = z (a + b z^2): 0.5 (1 + tanh(t)) = sigmoid(2 t).
struct Sigmoid {
  float a, b;
  __device__ static __forceinline__ Sigmoid of(int act)
  {
    // 2 sqrt(2 / pi) and 0.044715 of it
    return act == ACT_SILU ? Sigmoid{1.0f, 0.0f} : Sigmoid{1.5957691216f, 0.0713548163f};
  }
  template <class HW>
  __device__ __forceinline__ float at(float z) const
  {
    const float zz = z * z;
    const float u = z * (a + b * (zz < 1e30f ? zz : 1e30f));       // b may be 0, z^2 infinite
    return HW::rcp(1.0f + HW::exp2(-1.44269504089f * u));
  }
};

// Kernels exist per class of activation: their epilogues are unrolled, and with all five in each the code of one tile
// would be several times the instruction cache.
enum { CLASS_PLAIN = 0, CLASS_SIGMOID = 1, CLASS_ERF = 2 };
inline int class_of(int act) { return act == ACT_GELU ? CLASS_ERF : act >= ACT_GELU_TANH ? CLASS_SIGMOID : CLASS_PLAIN; }

// erfc(|z| / sqrt 2) / 2, what the normal distribution leaves beyond |z|, and gauss = exp(-z^2 / 2): gauss times a polynomial of
// t = 1 / (1 + 0.36 |z|), which is finite and smooth from 0 to infinity as the quotient of the two is.  Its coefficients are a
// least-squares fit of the relative error with the weights moved to the largest errors until they are level: 7.9e-7 up to |z| = 13.5,
// where gauss leaves the fp32 range.  In fp32 the relative error is at most (40 + 1.5 z^2) 2^-24, z^2 from the exponent's roundings:
// GELU far left of 0 is this number times z, and one that is only absolutely near (1e-7) is off by half a step of fp16 at z = -4.
// As many instructions as a degree of 5 in erfc's own argument and factor took: 8192 x 8192 x 2048 with `pre` 292 -> 294.5 us,
// 507 x 2072 x 1000 11.07 -> 11.02; the library's erff, with a branch of its own on either side of 1, some 25 more.
template <class HW>
__device__ __forceinline__ float half_erfc(float z, float& gauss)
{
  const float t = HW::rcp(1.0f + 0.36f * __builtin_fabsf(z));
  gauss = HW::exp2(-0.72134752044f * (z * z));
  return gauss * (t * (0.143717438f + t * (0.141710728f + t * (0.140057132f + t * (0.0256246459f +
                  t * (0.18229638f + t * (-0.180750787f + t * 0.0473443195f)))))));
}

template <int CLASS, class HW, int W>
__device__ __forceinline__ void activate(float (&v)[W], int act)
{
  if constexpr (CLASS == CLASS_PLAIN) {
    if (act == ACT_RELU) {
#pragma unroll
      for (int e = 0; e < W; e++) v[e] = v[e] < 0.f ? 0.f : v[e];
    }
  } else if constexpr (CLASS == CLASS_ERF) {
#pragma unroll
    for (int e = 0; e < W; e++) {
      float gauss;
      const float q = half_erfc<HW>(v[e], gauss), half = q == 0.f ? 0.f : v[e] * q;      // v may be infinite
      v[e] = v[e] < 0.f ? half : v[e] - half;
    }
  } else {
    const Sigmoid s = Sigmoid::of(act);
#pragma unroll
    for (int e = 0; e < W; e++) v[e] *= s.at<HW>(v[e]);
  }
}

// act'(z).  Far out, where the second term's first factor is 0 and its others may be infinite, it is 0.
template <class HW>
__device__ __forceinline__ float slope(float z, int act)
{
  if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == ACT_GELU) {
    float gauss;                                                  // exp(-z^2 / 2)
    const float half = half_erfc<HW>(z, gauss);
    return (z < 0.f ? half : 1.0f - half) + (gauss == 0.f ? 0.f : z * gauss * 0.39894228040f);
  }
  if (act >= ACT_GELU_TANH) {
    const Sigmoid g = Sigmoid::of(act);
    const float s = g.at<HW>(z), t = s * (1.0f - s);
    return s + (t == 0.f ? 0.f : z * t * (g.a + 3.0f * g.b * (z * z)));
  }
  return 1.f;
}

// ---- elements of the three output types (DT: 0 fp16, 1 bf16, 2 fp32) -----------------------------------------
template <int DT, class HW>
__device__ __forceinline__ float half_to_float(uint32_t bits)
{
  return DT == 0 ? HW::f16_bits((uint16_t)bits) : __builtin_bit_cast(float, bits << 16);
}
template <int DT, class HW>
__device__ __forceinline__ uint32_t float_to_half(float v)
{
  return DT == 0 ? (uint32_t)__builtin_bit_cast(uint16_t, HW::template cvt<_Float16>(v))
                 : (uint32_t)__builtin_bit_cast(uint16_t, HW::template cvt<__bf16>(v));
}
template <int DT>
__device__ __forceinline__ const char* element_at(const void* base, long at)
{
  return (const char*)base + at * (DT == 2 ? 4 : 2);
}

// W consecutive elements of a row as they lie in memory, at any element.
template <int W, int DT>
struct RawRow {
  uint32_t w[DT == 2 ? W : W / 2];
};
// ONCE: the caches need not keep the lines
template <int W, int DT, class HW, bool ONCE = false>
__device__ __forceinline__ RawRow<W, DT> load_chunk(const char* ptr)
{
  constexpr int WORDS = DT == 2 ? W : W / 2;
  RawRow<W, DT> r;
  if constexpr (WORDS % 4 == 0) {
#pragma unroll
    for (int i = 0; i < WORDS / 4; i++) {
      const u32x4 t = ONCE ? HW::global_load16_once(ptr + 16 * i) : HW::global_load16_any(ptr + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; e++) r.w[4 * i + e] = t[e];
    }
  } else {
    const u32x2 t = HW::global_load8_any(ptr);
    r.w[0] = t[0];
    r.w[1] = t[1];
  }
  return r;
}
template <int W, int DT, class HW>
__device__ __forceinline__ float element(const RawRow<W, DT>& r, int e)
{
  if constexpr (DT == 2)
    return __builtin_bit_cast(float, r.w[e]);
  else
    return half_to_float<DT, HW>((e & 1) ? r.w[e / 2] >> 16 : r.w[e / 2] & 0xffffu);
}
// KEEP: the line stays in the memory-side cache, as the next operator reads it (store_chunk in alcop_kernel.hip.h); 16-byte stores
// only, eight bytes pass the caches (no gain from keeping them: alcop_linear)
template <int W, int DT, class HW, bool KEEP>
__device__ __forceinline__ void store_row(const char* at, const float (&v)[W])
{
  char* ptr = const_cast<char*>(at);
  auto put16 = [&](char* dst, u32x4 t) __attribute__((always_inline)) {
    if constexpr (KEEP)
      HW::global_store16_through_any(dst, t);
    else
      HW::global_store16_any(dst, t);
  };
  if constexpr (DT == 2) {
#pragma unroll
    for (int i = 0; i < W / 4; i++)
      put16(ptr + 16 * i, __builtin_bit_cast(u32x4, f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]}));
  } else {
    uint32_t w[W / 2];
#pragma unroll
    for (int e = 0; e < W / 2; e++) w[e] = float_to_half<DT, HW>(v[2 * e]) | float_to_half<DT, HW>(v[2 * e + 1]) << 16;
    if constexpr (W == 8)
      put16(ptr, u32x4{w[0], w[1], w[2], w[3]});
    else
      HW::global_store8_any(ptr, u32x2{w[0], w[1]});
  }
}
template <int DT, class HW>
__device__ __forceinline__ float load_element(const void* base, long at)
{
  const char* ptr = element_at<DT>(base, at);
  if constexpr (DT == 2)
    return __builtin_bit_cast(float, HW::global_load_u32(ptr));
  else
    return half_to_float<DT, HW>(HW::global_load_u16(ptr));
}
template <int DT, class HW>
__device__ __forceinline__ void store_element(void* base, long at, float v)
{
  char* ptr = const_cast<char*>(element_at<DT>(base, at));
  if constexpr (DT == 2)
    HW::global_store_u32(ptr, __builtin_bit_cast(uint32_t, v));
  else
    HW::global_store_u16(ptr, (uint16_t)float_to_half<DT, HW>(v));
}
// f(integral constant of the type)
template <class F>
__device__ __forceinline__ void by_type(int dt, F&& f)
{
  if (dt == 2)
    f(TypeOf<2>{});
  else if (dt == 0)
    f(TypeOf<0>{});
  else
    f(TypeOf<1>{});
}

// ---- the epilogue ------------------------------------------------------------------------------------------
// What W consecutive columns from n on, all of which exist, have in common over all rows.
template <int W>
struct LinearColumns {
  float scale[W], bias[W];
};
template <int W, class HW>
__device__ __forceinline__ void load_floats(const float* from, float none, float (&to)[W])
{
#pragma unroll
  for (int e = 0; e < W; e++) to[e] = none;
  if (from == nullptr) return;
  if constexpr (W == 1) {
    to[0] = __builtin_bit_cast(float, HW::global_load_u32(from));
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; i++) {
      const f32x4 t = __builtin_bit_cast(f32x4, HW::global_load16_any(from + 4 * i));
#pragma unroll
      for (int e = 0; e < 4; e++) to[4 * i + e] = t[e];
    }
  }
}
template <int W, class HW>
__device__ __forceinline__ LinearColumns<W> linear_columns(const LinearParams& p, int n)
{
  LinearColumns<W> c;
  load_floats<W, HW>(p.bias ? p.bias + n : nullptr, 0.f, c.bias);
  load_floats<W, HW>(p.sw ? p.sw + n : nullptr, 1.f, c.scale);
#pragma unroll
  for (int e = 0; e < W; e++) c.scale[e] *= p.alpha;
  return c;
}
template <class HW>
__device__ __forceinline__ float row_scale(const LinearParams& p, int m)
{
  return p.sa != nullptr ? __builtin_bit_cast(float, HW::global_load_u32(p.sa + m)) : 1.0f;
}

// W columns of a row, of which v holds the sums and `res` the residual's; at_c, at_p: their place in C and pre.
template <int W, int DT, int CLASS, class HW>
__device__ __forceinline__ void linear_row(const LinearParams& p, const LinearColumns<W>& c, const char* at_c, const char* at_p,
                                           float (&v)[W], float sa, const RawRow<W, DT>& res)
{
  // branches that all lanes take alike: an epilogue's vector instructions are not covered by anything
  if (p.sa != nullptr) {
#pragma unroll
    for (int e = 0; e < W; e++) v[e] = v[e] * (c.scale[e] * sa) + c.bias[e];
  } else {
#pragma unroll
    for (int e = 0; e < W; e++) v[e] = v[e] * c.scale[e] + c.bias[e];
  }
  if (p.pre != nullptr) store_row<W, DT, HW, false>(at_p, v);
  activate<CLASS, HW>(v, p.act);
  if (p.residual != nullptr) {
#pragma unroll
    for (int e = 0; e < W; e++) v[e] += element<W, DT, HW>(res, e);
  }
  if (p.keep)
    store_row<W, DT, HW, true>(at_c, v);
  else
    store_row<W, DT, HW, false>(at_c, v);
}
// A single element, the last of a row that are no whole chunk.
template <int DT, int CLASS, class HW>
__device__ __forceinline__ void linear_element(const LinearParams& p, int m, int n, float sum)
{
  const LinearColumns<1> c = linear_columns<1, HW>(p, n);
  float v[1] = {sum * (c.scale[0] * row_scale<HW>(p, m)) + c.bias[0]};
  if (p.pre != nullptr) store_element<DT, HW>(p.pre, (long)m * p.ldp + n, v[0]);
  activate<CLASS, HW>(v, p.act);
  if (p.residual != nullptr) v[0] += load_element<DT, HW>(p.residual, (long)m * p.ldr + n);
  store_element<DT, HW>(p.C, (long)m * p.ldc + n, v[0]);
}

// A lane's place in a matrix of results, read or written band by band: the address of row `row` (the same for all lanes)
// and column n0, and the bytes from there to the lane's row and column, less than 2^31.
struct LanePlace {
  const char* tile;
  long pitch;
  uint32_t lane;
  __device__ __forceinline__ const char* at(int row) const { return tile + (long)row * pitch + lane; }
};
template <int DT>
__device__ __forceinline__ LanePlace lane_place(const void* base, int ld, int m0, int n0, int row, int col)
{
  constexpr int SIZE = DT == 2 ? 4 : 2;
  return LanePlace{element_at<DT>(base, (long)m0 * ld + n0), (long)ld * SIZE, (uint32_t)row * (uint32_t)ld * SIZE + (uint32_t)col * SIZE};
}

// What a wave's lanes need for the epilogue of their tile: columns' bias and scale, rows' scales, the residual
// (16-bit types).  Tiles of up to eight reads fetch all of it ahead of the main loop, so that its latency is not the
// epilogue's; larger ones, which have no registers for that, fetch the columns' values and a band behind the loop and
// every other band while the one before it is worked on.
//   The residual is fetched past the caches (ONCE): 8192 x 8192 x 4096 on e4m3, operands fresh from memory, takes 263 us so,
// 298 with ordinary loads, 251 without a residual; its 134 MB evict the panels of A and W that other compute units are about
// to read again.  Bringing its lines into L2 during the last k-tiles is no faster than ordinary loads.
template <class C>
struct LinearAhead {
  static constexpr int LPR = C::WN / 8;            // lanes per row when reading a band back
  static constexpr int RPI = 64 / LPR;             // rows per read
  static constexpr int NIT = 32 / RPI;
  static constexpr int TM = C::TM;
  static constexpr bool EARLY = TM * NIT <= 8;
  static constexpr int BANDS = EARLY ? TM : 2;
  static_assert(64 % LPR == 0 && 32 % RPI == 0, "a wave reads whole rows");
  LinearColumns<8> cols;
  float sa[BANDS][NIT];
  RawRow<8, 0> res[BANDS][NIT];

  static __device__ __forceinline__ int row_of(int m0, int lane, int j, int t) { return m0 + j * 32 + t * RPI + lane / LPR; }
  // whether read t of band j is part of C for this lane, as a whole chunk
  static __device__ __forceinline__ bool there(const LinearParams& p, int m0, int n0, int lane, int j, int t)
  {
    return (n0 + lane % LPR * 8 + 8 <= p.N) & (row_of(m0, lane, j, t) < p.M);
  }
  template <class HW>
  __device__ __forceinline__ void load_columns(const LinearParams& p, int n0, int lane)
  {
    const int n = n0 + lane % LPR * 8;
    cols = {};
    if (p.N >= 8) cols = linear_columns<8, HW>(p, n + 8 <= p.N ? n : 0);
  }
  template <class HW>
  __device__ __forceinline__ void load_band(const LinearParams& p, int m0, int n0, int lane, int j)
  {
#pragma unroll
    for (int t = 0; t < NIT; t++) {
      sa[j % BANDS][t] = 1.0f;
      res[j % BANDS][t] = {};
    }
    if (p.sa != nullptr) {
#pragma unroll
      for (int t = 0; t < NIT; t++) {
        const int m = row_of(m0, lane, j, t);
        sa[j % BANDS][t] = row_scale<HW>(p, m < p.M ? m : 0);
      }
    }
    if (p.residual != nullptr && p.out_dtype != 2) {
      const LanePlace r = lane_place<0>(p.residual, p.ldr, m0, n0, lane / LPR, lane % LPR * 8);
#pragma unroll
      for (int t = 0; t < NIT; t++)
        if (there(p, m0, n0, lane, j, t)) res[j % BANDS][t] = load_chunk<8, 0, HW, true>(r.at(j * 32 + t * RPI));
    }
  }
  template <class HW>
  __device__ __forceinline__ void load(const LinearParams& p, int m0, int n0, int lane)
  {
    if constexpr (EARLY) {
      load_columns<HW>(p, n0, lane);
#pragma unroll
      for (int j = 0; j < BANDS; j++) load_band<HW>(p, m0, n0, lane, j);
    }
  }
  template <class HW>
  __device__ __forceinline__ void load_late(const LinearParams& p, int m0, int n0, int lane)
  {
    if constexpr (!EARLY) {
      load_columns<HW>(p, n0, lane);
      load_band<HW>(p, m0, n0, lane, 0);
    }
  }
};

// A wave's tile, rows m0.., columns n0..; `ebase`: the wave's band in LDS.
template <class C, int DT, class HW>
__device__ __forceinline__ void linear_bands(const LinearParams& p, LinearAhead<C>& ahead, f32x16 (&acc)[C::TN][C::TM], int m0,
                                             int n0, uint32_t ebase, int lane)
{
  using L = LinearAhead<C>;
  constexpr int TN = C::TN, TM = C::TM, NIT = L::NIT;
  constexpr int RS = C::WN * 4 + 16;               // LDS row stride of the band
  constexpr int PART = L::EARLY ? NIT : 2;         // reads in registers at a time
  const int r0 = lane / L::LPR, c8 = lane % L::LPR * 8;
  const LanePlace c_at = lane_place<DT>(p.C, p.ldc, m0, n0, r0, c8), p_at = lane_place<DT>(p.pre, p.ldp, m0, n0, r0, c8);
  const LanePlace r_at = lane_place<DT>(p.residual, p.ldr, m0, n0, r0, c8);
  const bool tail_here = (p.N & 7) != 0 && (p.N & ~7) >= n0 && (p.N & ~7) < n0 + C::WN;
  LinearColumns<1> last = {};
  if (tail_here && (p.N & ~7) + (lane & 7) < p.N) last = linear_columns<1, HW>(p, (p.N & ~7) + (lane & 7));
#pragma unroll
  for (int j = 0; j < TM; j++) {
    if (!L::EARLY && j + 1 < TM) ahead.template load_band<HW>(p, m0, n0, lane, j + 1);
    const uint32_t row = ebase + (lane & 31) * RS + 16 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int vq = 0; vq < 4; vq++)
        HW::lds_write(row + (i * 32 + 8 * vq) * 4, f32x4{acc[i][j][4 * vq], acc[i][j][4 * vq + 1], acc[i][j][4 * vq + 2],
                                                        acc[i][j][4 * vq + 3]});
#pragma unroll
    for (int t0 = 0; t0 < NIT; t0 += PART) {
      RawRow<8, DT> res[PART];
      float v[PART][8];
#pragma unroll
      for (int q = 0; q < PART; q++) {
        const int t = t0 + q;
        if constexpr (DT == 2) {
          res[q] = {};
          if (p.residual != nullptr && L::there(p, m0, n0, lane, j, t)) res[q] = load_chunk<8, DT, HW, true>(r_at.at(j * 32 + t * L::RPI));
        } else {
#pragma unroll
          for (int e = 0; e < 4; e++) res[q].w[e] = ahead.res[j % L::BANDS][t].w[e];
        }
        const uint32_t at = ebase + (t * L::RPI + r0) * RS + c8 * 4;
        const f32x4 lo = __builtin_bit_cast(f32x4, HW::lds_read16(at)), hi = __builtin_bit_cast(f32x4, HW::lds_read16(at + 16));
#pragma unroll
        for (int e = 0; e < 4; e++) {
          v[q][e] = lo[e];
          v[q][4 + e] = hi[e];
        }
      }
#pragma unroll
      for (int q = 0; q < PART; q++) {
        const int t = t0 + q;
        if (L::there(p, m0, n0, lane, j, t))
          linear_row<8, DT, C::CLASS, HW>(p, ahead.cols, c_at.at(j * 32 + t * L::RPI), p_at.at(j * 32 + t * L::RPI), v[q],
                                          ahead.sa[j % L::BANDS][t], res[q]);
      }
    }
    // columns behind the last whole chunk, at most seven: eight rows of them at a time, element by element
    if (tail_here) {
      const int c = lane & 7, n1 = (p.N & ~7) + c;
      float r1[4], s1[4];
      bool in[4];
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int m = m0 + j * 32 + q * 8 + (lane >> 3);
        in[q] = (n1 < p.N) & (m < p.M);
        r1[q] = 0.f;
        s1[q] = 1.f;
        if (in[q]) {
          if (p.residual != nullptr) r1[q] = load_element<DT, HW>(p.residual, (long)m * p.ldr + n1);
          s1[q] = row_scale<HW>(p, m);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int r = q * 8 + (lane >> 3), m = m0 + j * 32 + r;
        const uint32_t bits = HW::lds_read4(ebase + r * RS + ((p.N & ~7) - n0 + c) * 4);
        if (in[q]) {
          float v[1] = {__builtin_bit_cast(float, bits) * (last.scale[0] * s1[q]) + last.bias[0]};
          if (p.pre != nullptr) store_element<DT, HW>(p.pre, (long)m * p.ldp + n1, v[0]);
          activate<C::CLASS, HW>(v, p.act);
          store_element<DT, HW>(p.C, (long)m * p.ldc + n1, v[0] + r1[q]);
        }
      }
    }
  }
}
template <class C, class HW, class P>
__device__ __forceinline__ void linear_tile(const P& p, typename C::Ahead& ahead, f32x16 (&acc)[C::TN][C::TM], int m0, int n0,
                                            uint32_t ebase, int lane)
{
  by_type(p.out_dtype, [&](auto t) __attribute__((always_inline)) {
    linear_bands<C, decltype(t)::value, HW>(p, ahead, acc, m0, n0, ebase, lane);
  });
}

// The same for the kernels whose waves split K, where a thread ends up with groups of four columns of a row (group
// `turn` NT + thread of the tile).
template <class C>
struct LinearGroups {
  static constexpr int GPR = C::BN / 4, GROUPS = C::BM * GPR, TURNS = (GROUPS + C::NT - 1) / C::NT;
  LinearColumns<4> cols[TURNS];
  float sa[TURNS];
  RawRow<4, 0> res[TURNS];
  template <class HW>
  __device__ __forceinline__ void load(const LinearParams& p, int m0, int n0, int thread)
  {
#pragma unroll
    for (int i = 0; i < TURNS; i++) {
      const int g = i * C::NT + thread, m = m0 + g / GPR, n = n0 + g % GPR * 4;
      cols[i] = {};
      sa[i] = 1.0f;
      res[i] = {};
      if ((g < GROUPS) & (m < p.M) & (n + 4 <= p.N)) {
        cols[i] = linear_columns<4, HW>(p, n);
        sa[i] = row_scale<HW>(p, m);
        if (p.residual != nullptr && p.out_dtype != 2) res[i] = load_chunk<4, 0, HW>(element_at<0>(p.residual, (long)m * p.ldr + n));
      }
    }
  }
};

template <class C, class HW, class P>
__device__ __forceinline__ void linear_group(const P& p, const typename C::Ahead& ahead, int turn, int m, int n, const f32x4& sum)
{
  if ((m >= p.M) | (n >= p.N)) return;
  by_type(p.out_dtype, [&](auto t) __attribute__((always_inline)) {
    constexpr int DT = decltype(t)::value;
    if (n + 4 <= p.N) {
      RawRow<4, DT> res = {};
      if constexpr (DT == 2) {
        if (p.residual != nullptr) res = load_chunk<4, DT, HW>(element_at<DT>(p.residual, (long)m * p.ldr + n));
      } else {
        res.w[0] = ahead.res[turn].w[0];
        res.w[1] = ahead.res[turn].w[1];
      }
      float v[4] = {sum[0], sum[1], sum[2], sum[3]};
      linear_row<4, DT, C::CLASS, HW>(p, ahead.cols[turn], element_at<DT>(p.C, (long)m * p.ldc + n),
                                      element_at<DT>(p.pre, (long)m * p.ldp + n), v, ahead.sa[turn], res);
    } else {
#pragma unroll
      for (int e = 0; e < 3; e++)
        if (n + e < p.N) linear_element<DT, C::CLASS, HW>(p, m, n + e, sum[e]);
    }
  });
}

// ---- the kernels -------------------------------------------------------------------------------------------
// DT: 0 fp16, 1 bf16, 2 pairs of e4m3 widened to bf16, 3 pairs of e4m3 as they are; BL: 0 W stored K x N, 1 N x K.
template <int CLASS_, int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int FUSE, int BL>
struct LCfg : KCfg<DT, BM, BN, BK, WM, WN, S, R, FUSE, BL, 0> {
  static constexpr bool LINEAR = true;
  using Ahead = LinearAhead<LCfg>;
  static constexpr int CLASS = CLASS_;
  static_assert(DT < 2 || BL == 1, "the transposing read moves 16-bit elements");
};
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_linear_tile(const LinearArgs a)
{
  mainloop_body<C, HW>(expand_linear<C>(a));
}

template <int CLASS_, int DT, int BM, int BN, int NW, int S, int BL>
struct LWCfg : WCfg<DT, BM, BN, NW, S, BL, 0> {
  static constexpr bool LINEAR = true;
  using Ahead = LinearGroups<LWCfg>;
  static constexpr int CLASS = CLASS_;
  static_assert(DT != 2 || BL == 1, "the transposing read moves 16-bit elements");
};
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_linear_ksplit(const LinearArgs a)
{
  ksplit_body<C, HW>(expand_linear<C>(a));
}

}  // namespace alcop
