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
// sum over k does not ask for their order.  They are widened to bf16 in registers (alcop_gfx950.hip.h says why).
//
// Epilogue of a tile (linear_tile): as in alcop_kernel.hip.h a wave parks 32 rows of its accumulators in LDS, here
// in fp32, and reads them back along the rows, eight columns a lane, so that residual, pre and C move in 16-byte
// accesses that cover whole lines.  A lane's columns are the same in every row: bias and column scales are
// fetched once per tile.
#pragma once
#include "alcop_ksplit.hip.h"

namespace alcop {

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
  int flags;                   // output type | activation << 2 | rows of C, residual and pre made of 16-byte chunks << 5
};

struct LinearParams : Params {
  const void* residual;
  void* pre;
  const float *sa, *sw;
  int ldr, ldp;
  bool chunks;
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
  p.chunks = (a.flags & 32) != 0;
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

template <class HW, int W>
__device__ __forceinline__ void activate(float (&v)[W], int act)
{
  if (act == ACT_RELU) {
#pragma unroll
    for (int e = 0; e < W; e++) v[e] = v[e] < 0.f ? 0.f : v[e];
  } else if (act == ACT_GELU) {
#pragma unroll
    for (int e = 0; e < W; e++) v[e] = 0.5f * v[e] * (1.0f + HW::erf(v[e] * 0.70710678119f));
  } else if (act >= ACT_GELU_TANH) {
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
    const float e = HW::exp2(-0.72134752044f * (z * z));          // exp(-z^2 / 2)
    return 0.5f * (1.0f + HW::erf(z * 0.70710678119f)) + (e == 0.f ? 0.f : z * e * 0.39894228040f);
  }
  if (act >= ACT_GELU_TANH) {
    const Sigmoid g = Sigmoid::of(act);
    const float s = g.at<HW>(z), t = s * (1.0f - s);
    return s + (t == 0.f ? 0.f : z * t * (g.a + 3.0f * g.b * (z * z)));
  }
  return 1.f;
}

// ---- elements of the three output types ------------------------------------------------------------------
template <class HW>
__device__ __forceinline__ float half_to_float(uint32_t bits, int dt)
{
  return dt == 0 ? HW::f16_bits((uint16_t)bits) : __builtin_bit_cast(float, bits << 16);
}
template <class HW>
__device__ __forceinline__ uint32_t float_to_half(float v, int dt)
{
  return dt == 0 ? (uint32_t)__builtin_bit_cast(uint16_t, HW::template cvt<_Float16>(v))
                 : (uint32_t)__builtin_bit_cast(uint16_t, HW::template cvt<__bf16>(v));
}

// W consecutive elements of a row as they lie in memory: 16-bit ones in the first W / 2 words.
template <int W>
struct RawRow {
  uint32_t w[W];
};
template <int W, class HW>
__device__ __forceinline__ RawRow<W> load_chunk(const void* base, long at, int dt)
{
  RawRow<W> r;
  const char* ptr = (const char*)base + at * (dt == 2 ? 4 : 2);
  if (dt == 2) {
#pragma unroll
    for (int i = 0; i < W / 4; i++) {
      const u32x4 t = HW::global_load16_any(ptr + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; e++) r.w[4 * i + e] = t[e];
    }
  } else if constexpr (W == 8) {
    const u32x4 t = HW::global_load16_any(ptr);
#pragma unroll
    for (int e = 0; e < 4; e++) r.w[e] = t[e];
  } else {
    const u32x2 t = HW::global_load8(ptr);
    r.w[0] = t[0];
    r.w[1] = t[1];
  }
  return r;
}
template <int W, class HW>
__device__ __forceinline__ float element(const RawRow<W>& r, int e, int dt)
{
  if (dt == 2) return __builtin_bit_cast(float, r.w[e]);
  const uint32_t h = (e & 1) ? r.w[e / 2] >> 16 : r.w[e / 2] & 0xffffu;
  return half_to_float<HW>(h, dt);
}
// KEEP: the line stays in the memory-side cache, as the next operator reads it (store_chunk in alcop_kernel.hip.h)
template <int W, class HW, bool KEEP>
__device__ __forceinline__ void store_row(void* base, long at, int dt, const float (&v)[W])
{
  char* ptr = (char*)base + at * (dt == 2 ? 4 : 2);
  auto put16 = [&](char* dst, u32x4 t) {
    if constexpr (KEEP)
      HW::global_store16_through(dst, t);
    else
      HW::global_store16(dst, t);
  };
  if (dt == 2) {
#pragma unroll
    for (int i = 0; i < W / 4; i++)
      put16(ptr + 16 * i, __builtin_bit_cast(u32x4, f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]}));
    return;
  }
  uint32_t w[W / 2];
#pragma unroll
  for (int e = 0; e < W / 2; e++) w[e] = float_to_half<HW>(v[2 * e], dt) | float_to_half<HW>(v[2 * e + 1], dt) << 16;
  if constexpr (W == 8)
    put16(ptr, u32x4{w[0], w[1], w[2], w[3]});
  else
    HW::template global_store<u32x2>(ptr, u32x2{w[0], w[1]});
}
template <class HW>
__device__ __forceinline__ float load_element(const void* base, long at, int dt)
{
  if (dt == 2) return __builtin_bit_cast(float, HW::global_load_u32((const char*)base + at * 4));
  return half_to_float<HW>(HW::global_load_u16((const char*)base + at * 2), dt);
}
template <class HW>
__device__ __forceinline__ void store_element(void* base, long at, int dt, float v)
{
  if (dt == 2)
    HW::global_store_u32((char*)base + at * 4, __builtin_bit_cast(uint32_t, v));
  else
    HW::global_store_u16((char*)base + at * 2, (uint16_t)float_to_half<HW>(v, dt));
}

// ---- the epilogue ------------------------------------------------------------------------------------------
// What W consecutive columns from n < N on have in common over all rows.  W > 1: all of them exist.
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
      const f32x4 t = HW::global_load_f32x4(from + 4 * i);
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

// Row m's W columns from n on, of which v holds the sums.  W > 1: C, pre and the residual's chunk `res` are aligned.
template <int W, class HW>
__device__ __forceinline__ void linear_row(const LinearParams& p, const LinearColumns<W>& c, int m, int n, float (&v)[W],
                                           float sa, const RawRow<W>& res)
{
#pragma unroll
  for (int e = 0; e < W; e++) v[e] = v[e] * (c.scale[e] * sa) + c.bias[e];
  const long at = (long)m * p.ldc + n, at_p = (long)m * p.ldp + n;
  if (p.pre != nullptr) {
    if constexpr (W == 1)
      store_element<HW>(p.pre, at_p, p.out_dtype, v[0]);
    else
      store_row<W, HW, false>(p.pre, at_p, p.out_dtype, v);
  }
  activate<HW>(v, p.act);
  if (p.residual != nullptr) {
    if constexpr (W == 1) {
      v[0] += load_element<HW>(p.residual, (long)m * p.ldr + n, p.out_dtype);
    } else {
#pragma unroll
      for (int e = 0; e < W; e++) v[e] += element<W, HW>(res, e, p.out_dtype);
    }
  }
  if constexpr (W == 1)
    store_element<HW>(p.C, at, p.out_dtype, v[0]);
  else
    store_row<W, HW, true>(p.C, at, p.out_dtype, v);
}
template <class HW>
__device__ __forceinline__ float row_scale(const LinearParams& p, int m)
{
  return p.sa != nullptr ? __builtin_bit_cast(float, HW::global_load_u32(p.sa + m)) : 1.0f;
}

// A wave's tile, rows m0.., columns n0..; `ebase`: the wave's band in LDS.
template <class C, class HW, class P>
__device__ __forceinline__ void linear_tile(const P& p, f32x16 (&acc)[C::TN][C::TM], int m0, int n0, uint32_t ebase, int lane)
{
  constexpr int TN = C::TN, TM = C::TM;
  constexpr int RS = C::WN * 4 + 16;               // LDS row stride of the band
  constexpr int LPR = C::WN / 8;                   // lanes per row when reading back
  constexpr int RPI = 64 / LPR;                    // rows per read; 96 columns: five, and four lanes idle
  constexpr int NIT = (32 + RPI - 1) / RPI;
  const int r0 = lane / LPR, n = n0 + lane % LPR * 8;
  const bool lane_ok = r0 < RPI && n < p.N;
  LinearColumns<8> cols;
  if (p.chunks) cols = linear_columns<8, HW>(p, lane_ok ? n : 0);
  // this lane's row in read t of band j; its part of the residual there
  auto row_of = [&](int j, int t) __attribute__((always_inline)) { return m0 + j * 32 + t * RPI + r0; };
  auto there = [&](int j, int t) __attribute__((always_inline)) {
    return lane_ok & (t * RPI + r0 < 32) & (row_of(j, t) < p.M);
  };
  auto fetch = [&](int j, int t) __attribute__((always_inline)) {
    RawRow<8> r = {};
    if (p.residual != nullptr && there(j, t)) r = load_chunk<8, HW>(p.residual, (long)row_of(j, t) * p.ldr + n, p.out_dtype);
    return r;
  };
#pragma unroll
  for (int j = 0; j < TM; j++) {
    RawRow<8> res = {};
    if (p.chunks) res = fetch(j, 0);
    const uint32_t row = ebase + (lane & 31) * RS + 16 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int vq = 0; vq < 4; vq++)
        HW::lds_write(row + (i * 32 + 8 * vq) * 4, f32x4{acc[i][j][4 * vq], acc[i][j][4 * vq + 1], acc[i][j][4 * vq + 2],
                                                        acc[i][j][4 * vq + 3]});
    if (p.chunks) {
#pragma unroll 1
      for (int t = 0; t < NIT; t++) {
        const RawRow<8> next = fetch(j, t + 1);
        const int r = t * RPI + r0;
        const uint32_t at = ebase + (r < 32 ? r : 0) * RS + lane % LPR * 32;     // every lane takes part in the read
        const f32x4 lo = __builtin_bit_cast(f32x4, HW::lds_read16(at)), hi = __builtin_bit_cast(f32x4, HW::lds_read16(at + 16));
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (there(j, t)) {
          const int m = row_of(j, t);
          linear_row<8, HW>(p, cols, m, n, v, row_scale<HW>(p, m), res);
        }
        res = next;
      }
    } else {
      // rows that are not made of chunks: element by element, lane next to lane
#pragma unroll 1
      for (int t = lane; t < 32 * C::WN; t += 64) {
        const int r = t / C::WN, c = t % C::WN;
        float v[1] = {__builtin_bit_cast(float, HW::lds_read4(ebase + r * RS + c * 4))};
        const int m = m0 + j * 32 + r;
        if ((m < p.M) & (n0 + c < p.N))
          linear_row<1, HW>(p, linear_columns<1, HW>(p, n0 + c), m, n0 + c, v, row_scale<HW>(p, m), RawRow<1>{});
      }
    }
  }
}

// Four columns of a row, from the kernels whose waves split K.
template <class HW, class P>
__device__ __forceinline__ void linear_group(const P& p, int m, int n, const f32x4& sum)
{
  if (p.chunks) {
    if ((m >= p.M) | (n >= p.N)) return;
    const LinearColumns<4> cols = linear_columns<4, HW>(p, n);
    RawRow<4> res = {};
    if (p.residual != nullptr) res = load_chunk<4, HW>(p.residual, (long)m * p.ldr + n, p.out_dtype);
    float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    linear_row<4, HW>(p, cols, m, n, v, row_scale<HW>(p, m), res);
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      float v[1] = {sum[e]};
      if ((m < p.M) & (n + e < p.N))
        linear_row<1, HW>(p, linear_columns<1, HW>(p, n + e), m, n + e, v, row_scale<HW>(p, m), RawRow<1>{});
    }
  }
}

// ---- the kernels -------------------------------------------------------------------------------------------
// DT: 0 fp16, 1 bf16, 2 pairs of e4m3; BL: 0 W stored K x N, 1 N x K.
template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int FUSE, int BL>
struct LCfg : KCfg<DT, BM, BN, BK, WM, WN, S, R, FUSE, BL, 0> {
  static constexpr bool LINEAR = true;
  static_assert(DT != 2 || BL == 1, "the transposing read moves 16-bit elements");
};
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_linear_tile(const LinearArgs a)
{
  mainloop_body<C, HW>(expand_linear<C>(a));
}

template <int DT, int BM, int BN, int NW, int S, int BL>
struct LWCfg : WCfg<DT, BM, BN, NW, S, BL, 0> {
  static constexpr bool LINEAR = true;
  static_assert(DT != 2 || BL == 1, "the transposing read moves 16-bit elements");
};
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_linear_ksplit(const LinearArgs a)
{
  ksplit_body<C, HW>(expand_linear<C>(a));
}

}  // namespace alcop
