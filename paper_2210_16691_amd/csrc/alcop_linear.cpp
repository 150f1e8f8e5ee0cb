// Host code of the linear layers and the row operators: argument checks, choice of the kernel, launches.
// Declarations and argument contracts are in include/alcop.h.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "alcop_linear.h"
#include "alcop_linear_cost.h"

namespace alcop {
namespace {

// All kernels, and those of one class of activation, operand type (of a call: e4m3 as 2) and layout.
struct LinearTable {
  std::vector<LinearKernel> all;
  std::vector<const LinearKernel*> of[3][3][2];
  LinearTable()
  {
    register_linear_f16(all);
    register_linear_bf16(all);
    register_linear_e4m3(all);
    register_linear_f8(all);
    for (LinearKernel& k : all) {
      for (const LinearCost& m : kLinearCost)
        if (m.dt == (k.dt == 0 ? 1 : k.dt) && m.bl == k.bl && std::memcmp(&m.s, &k.s, sizeof(k.s)) == 0) k.cost = &m;
      of[k.cls][std::min(k.dt, 2)][k.bl].push_back(&k);
    }
  }
};
const LinearTable& linear_table()
{
  static const LinearTable t;
  return t;
}

int size_of(alcop_dtype t) { return t == ALCOP_F32 ? 4 : t == ALCOP_E4M3 ? 1 : 2; }
bool is_half(alcop_dtype t) { return t == ALCOP_F16 || t == ALCOP_BF16; }
bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

// A matrix in memory, in bytes.
struct Span {
  const char* p;
  double rows, row, pitch;
  Span(const void* ptr, int rows_, int cols, long ld, int size)
      : p((const char*)ptr), rows(rows_), row((double)cols * size), pitch((double)ld * size)
  {
  }
};
// Whether two matrices share bytes.  Column ranges of one buffer, rows equally far apart, do not.
bool meet(const Span& a, const Span& b)
{
  if (!a.p || !b.p) return false;
  const double ea = (a.rows - 1) * a.pitch + a.row, eb = (b.rows - 1) * b.pitch + b.row;
  if (!(a.p < b.p + (size_t)eb && b.p < a.p + (size_t)ea)) return false;
  if (a.pitch != b.pitch || a.rows < 2 || b.rows < 2) return true;
  const long pitch = (long)a.pitch;
  const long d = (long)((((b.p - a.p) % pitch) + pitch) % pitch);      // b's columns start d bytes behind a's
  return !(d >= (long)a.row && d + (long)b.row <= pitch);
}
bool same(const Span& a, const Span& b) { return a.p == b.p && (a.rows < 2 || a.pitch == b.pitch) && a.row == b.row; }

// The kernel of the lowest measured cost.  fine: sums are to be fp32, which those of the 8-bit matrix instruction are not
// (8192 x 8192 x 4096 without a residual 228 us, 412 on widened operands): asked for, or a result in fp32, which is worth it.
const LinearKernel* pick(int cls, int dt, int bl, bool fine, int M, int N, int K, double bytes)
{
  const LinearKernel* best = nullptr;
  double best_us = 0;
  const char* env = std::getenv("ALCOP_LINEAR_KERNEL");       // a tuning and test knob: its number among those of the layout
  int nr = 0;
  for (const LinearKernel* e : linear_table().of[cls][dt][bl]) {
    const LinearKernel& k = *e;
    if (k.dt == 3 && fine) continue;
    if (env && *env) {
      if (nr++ == std::atoi(env)) return &k;
      continue;
    }
    if (!k.cost || !linear_applies(*k.cost, M, N)) continue;
    const double us = linear_us(*k.cost, M, N, K, bytes);
    if (!best || us < best_us) {
      best = &k;
      best_us = us;
    }
  }
  return best;
}

size_t r256(double bytes) { return ((size_t)bytes + 255) & ~(size_t)255; }

// Lanes that share a row in alcop_act_grad.
int act_grad_lanes(int N)
{
  int lanes = 1;
  while (lanes < 64 && lanes * 8 < N) lanes *= 2;
  return lanes;
}

// Blocks of rows whose sums of the bias's gradient are added by a second kernel, and their rows: enough blocks to fill
// the card (2048 with 512 columns each), at most 256 sums to a column.
int act_grad_rows(int M, int N)
{
  const int strips = (N + ACT_COLS - 1) / ACT_COLS, at_once = 256 / act_grad_lanes(N);
  const int want = std::max(1, std::min(256, 2048 / strips));
  return std::max(at_once, (int)(((long)M + want - 1) / want));
}

// Blocks that walk the rows of a norm's gradient, each leaving a row of sums for dgain.  A single block writes dgain
// itself: a second turn of it takes 1.8 us, a second launch 2.8.
int norm_blocks(int rows, int cols)
{
  const long blocks = ((long)rows + rows_per_block(rows, cols) - 1) / rows_per_block(rows, cols);
  return blocks <= 2 ? 1 : (int)std::min(blocks, 1024L);
}

// The workspace of a layer's gradients: dZ, the bias's partial sums from here on, dW's behind them.
size_t backward_sums(int M, int N) { return r256(2.0 * M * N); }

}  // namespace

hipError_t prepare_layers()
{
  for (const LinearKernel& k : linear_table().all) {
    const hipError_t rc = k.prepare();
    if (rc != hipSuccess) return rc;
  }
  return prepare_rows();
}

}  // namespace alcop

using namespace alcop;

extern "C" {

int alcop_linear(const void* A, const void* W, void* C, int M, int N, int K, long lda, long ldw, long ldc, int transB,
                 alcop_dtype in, alcop_dtype out, const alcop_linear_tail* tail, void* hip_stream)
{
  alcop_linear_tail t;
  std::memset(&t, 0, sizeof(t));
  t.alpha = 1.0f;
  if (tail) t = *tail;
  const bool fine = out == ALCOP_F32 || (t.act & ALCOP_FP32_SUMS);
  t.act &= ~ALCOP_FP32_SUMS;
  transB = transB ? 1 : 0;
  if (!A || !W || !C) return ALCOP_ERR_NULL;
  if (!is_half(in) && in != ALCOP_E4M3) return ALCOP_ERR_DTYPE;
  if (!is_half(out) && out != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if (t.act < 0 || t.act > 4 || (in == ALCOP_E4M3 && !transB)) return ALCOP_ERR_UNSUPPORTED;
  const int esz = size_of(in), osz = size_of(out), unit = 16 / esz;
  if (M <= 0 || N <= 0 || K <= 0 || K % unit || (!transB && N % unit)) return ALCOP_ERR_SHAPE;
  if (lda < K || ldw < (transB ? K : N) || ldc < N || (t.residual && t.ldr < N) || (t.pre && t.ldp < N)) return ALCOP_ERR_SHAPE;
  if (!aligned(A, 16) || !aligned(W, 16) || lda % unit || ldw % unit) return ALCOP_ERR_ALIGN;
  if (!aligned(C, osz) || !aligned(t.residual, osz) || !aligned(t.pre, osz)) return ALCOP_ERR_ALIGN;
  if (!aligned(t.bias, 16) || !aligned(t.scale_w, 16) || !aligned(t.scale_a, 4)) return ALCOP_ERR_ALIGN;
  const long far = 1L << 30;
  if (lda >= far || ldw >= far || ldc >= far || t.ldr >= far || t.ldp >= far) return ALCOP_ERR_SIZE;
  if (std::max(M, N) > 0x7ffff000) return ALCOP_ERR_SIZE;     // rows and columns rounded up to tiles

  const int K16 = in == ALCOP_E4M3 ? K / 2 : K;              // in units of 16 bits
  const double c_bytes = (double)osz * M * N;
  const double bytes = 2.0 * K16 * ((double)M + N) + c_bytes * (1 + (t.residual ? 1 : 0) + (t.pre ? 1 : 0));
  const LinearKernel* k = pick(class_of(t.act), in == ALCOP_E4M3 ? 2 : in == ALCOP_BF16 ? 1 : 0, transB, fine, M, N, K16, bytes);
  if (!k) return ALCOP_ERR_SCHED;
  // 32-bit byte offsets from a tile's origin, rows past the end of a partial k-tile included
  const double rows = std::min(k->s.bm, M), cols = std::min(k->s.bn, N);
  const double kceil = (double)((K16 + k->s.bk - 1) / k->s.bk) * k->s.bk;
  if (esz * (rows * (double)lda) >= 2147483648.0 || (transB ? esz * (cols * (double)ldw) : 2.0 * kceil * ldw) >= 2147483648.0)
    return ALCOP_ERR_SIZE;
  if (osz * rows * (double)std::max(ldc, std::max(t.residual ? t.ldr : 0, t.pre ? t.ldp : 0)) >= 2147483648.0) return ALCOP_ERR_SIZE;
  const long ntm = ((long)M + k->s.bm - 1) / k->s.bm, ntn = ((long)N + k->s.bn - 1) / k->s.bn;
  if (ntm * ntn >= (1L << 32) / k->threads) return ALCOP_ERR_SHAPE;      // threads of a launch are counted in 32 bits

  const Span c(C, M, N, ldc, osz), r(t.residual, M, N, t.ldr, osz), z(t.pre, M, N, t.ldp, osz);
  const Span read[] = {Span(A, M, K, lda, esz), Span(W, transB ? N : K, transB ? K : N, ldw, esz), Span(t.bias, 1, N, N, 4),
                       Span(t.scale_a, 1, M, M, 4), Span(t.scale_w, 1, N, N, 4)};
  for (const Span& s : read)
    if (meet(c, s) || meet(z, s)) return ALCOP_ERR_UNSUPPORTED;
  if (meet(c, z) || meet(r, z) || (meet(c, r) && !same(c, r))) return ALCOP_ERR_UNSUPPORTED;

  // C stays in the memory-side cache, for the operator that reads it next, unless it is too large for that: two layers in a
  // row (hidden results of 4 to 34 MB) are 4 to 10 % faster kept, from 67 MB on 1 to 2.5 % slower; what nothing reads
  // costs 1 to 6 % more to keep.  The kernels whose waves split K keep results in fp32 only: their 16-bit groups of eight bytes,
  // kept, change pairs of layers with 1 to 256 rows by less than 1.5 % either way
  const bool keep = c_bytes <= 48e6;
  LinearArgs a;
  a.A = A;
  a.W = W;
  a.C = C;
  a.residual = t.residual;
  a.pre = t.pre;
  a.bias = (const float*)t.bias;
  a.sa = (const float*)t.scale_a;
  a.sw = (const float*)t.scale_w;
  a.M = M;
  a.N = N;
  a.K = K16;
  a.lda = (int)(in == ALCOP_E4M3 ? lda / 2 : lda);
  a.ldw = (int)(in == ALCOP_E4M3 ? ldw / 2 : ldw);
  a.ldc = (int)ldc;
  a.ldr = t.residual ? (int)t.ldr : 0;
  a.ldp = t.pre ? (int)t.ldp : 0;
  a.alpha = t.alpha;
  a.flags = (int)out | t.act << 2 | (keep ? 32 : 0);
  if (std::getenv("ALCOP_LOG"))
    std::fprintf(stderr, "alcop: linear M %d N %d K %d in %d -> tile %dx%dx%d waves %dx%d S%d R%d F%d variant %d grid %ld\n", M,
                 N, K, (int)in, k->s.bm, k->s.bn, k->s.bk, k->s.wm, k->s.wn, k->s.stages, k->s.reg_stages, k->s.fuse_inner,
                 k->s.variant, ntm * ntn);
  return k->launch(a, dim3((unsigned)(ntm * ntn)), (hipStream_t)hip_stream) == hipSuccess ? ALCOP_OK : ALCOP_ERR_LAUNCH;
}

size_t alcop_linear_backward_workspace_bytes(int M, int N, int K)
{
  if (M <= 0 || N <= 0 || K <= 0 || N % 8 || K % 8) return 0;
  const size_t split = std::max(gradient_workspace(N, K, M), gradient_workspace(K, N, M));
  return backward_sums(M, N) + r256(4.0 * N * ((M + (double)act_grad_rows(M, N) - 1) / act_grad_rows(M, N))) + split;
}

int alcop_linear_backward(const void* dC, const void* A, const void* W, const void* pre, void* dA, void* dW, void* dbias,
                          int M, int N, int K, long lddc, long lda, long ldw, long ldp, long ldda, long lddw, int transB,
                          alcop_dtype in, alcop_dtype out, float alpha, int act, void* workspace, size_t workspace_bytes,
                          void* hip_stream)
{
  transB = transB ? 1 : 0;
  if (!dC || (!dA && !dW && !dbias) || (dA && !W) || (dW && !A)) return ALCOP_ERR_NULL;
  if (!is_half(in) || (out != in && out != ALCOP_F32)) return ALCOP_ERR_DTYPE;
  if (act < 0 || act > 4) return ALCOP_ERR_UNSUPPORTED;
  if (act && !pre) return ALCOP_ERR_NULL;
  if ((act || dbias) && !workspace) return ALCOP_ERR_NULL;
  if (M <= 0 || N <= 0 || K <= 0 || N % 8 || K % 8) return ALCOP_ERR_SHAPE;
  if (std::max(M, std::max(N, K)) > 0x7ffff000) return ALCOP_ERR_SIZE;
  const int w_rows = transB ? N : K, w_cols = transB ? K : N;
  if (lddc < N || (dW && lda < K) || (dA && ldw < w_cols) || (act && ldp < N) || (dA && ldda < K) || (dW && lddw < w_cols))
    return ALCOP_ERR_SHAPE;
  if (!aligned(dC, 16) || !aligned(workspace, 16) || !aligned(dbias, 4) || lddc % 8) return ALCOP_ERR_ALIGN;
  if (act && (!aligned(pre, 16) || ldp % 8)) return ALCOP_ERR_ALIGN;
  if (dA && (!aligned(dA, 16) || !aligned(W, 16) || ldda % 8 || ldw % 8)) return ALCOP_ERR_ALIGN;
  if (dW && (!aligned(dW, 16) || !aligned(A, 16) || lddw % 8 || lda % 8)) return ALCOP_ERR_ALIGN;
  const long far = 1L << 30;
  if (lddc >= far || (act && ldp >= far) || (dA && (ldda >= far || ldw >= far)) || (dW && (lddw >= far || lda >= far)))
    return ALCOP_ERR_SIZE;
  if ((act || dbias) && workspace_bytes < alcop_linear_backward_workspace_bytes(M, N, K)) return ALCOP_ERR_SIZE;

  // outputs overlap nothing that is read, nor each other
  const int osz = size_of(out);
  const Span outs[] = {Span(dA, M, K, ldda, osz), Span(dW, w_rows, w_cols, lddw, osz), Span(dbias, 1, N, N, 4),
                       Span(workspace, 1, 1, 1, 1)};
  const Span ins[] = {Span(dC, M, N, lddc, 2), Span(dW ? A : nullptr, M, K, lda, 2), Span(dA ? W : nullptr, w_rows, w_cols, ldw, 2),
                      Span(act ? pre : nullptr, M, N, ldp, 2)};
  for (int i = 0; i < 4; i++) {
    Span o = outs[i];
    if (i == 3) o.row = o.pitch = (double)workspace_bytes;
    for (const Span& s : ins)
      if (meet(o, s)) return ALCOP_ERR_UNSUPPORTED;
    for (int j = 0; j < i; j++)
      if (meet(o, outs[j])) return ALCOP_ERR_UNSUPPORTED;
  }

  const bool own_dz = act && (dA || dW);
  const void* dZ = own_dz ? workspace : dC;
  const long lddz = own_dz ? N : lddc;
  // a product that refuses its operands does so before anything is launched
  if (dA) {
    const int rc = product_check(dZ, W, dA, M, K, N, lddz, ldw, ldda, 0, transB ? 0 : 1, in, out);
    if (rc) return rc;
  }
  if (dW) {
    const int Mr = (M + 7) & ~7;                   // as gradient_product rounds it; M is below 2^31 - 4096
    const int rc = transB ? product_check(dZ, A, dW, N, K, Mr, lddz, lda, lddw, 1, 0, in, out)
                          : product_check(A, dZ, dW, K, N, Mr, lda, lddz, lddw, 1, 0, in, out);
    if (rc) return rc;
  }

  hipStream_t st = (hipStream_t)hip_stream;
  if (act || dbias) {
    ActGradArgs g;
    std::memset(&g, 0, sizeof(g));
    g.rows_per_block = act_grad_rows(M, N);
    const int blocks = (int)(((long)M + g.rows_per_block - 1) / g.rows_per_block);
    g.dc = dC;
    g.pre = act ? pre : nullptr;
    g.M = M;
    g.N = N;
    g.lddc = lddc;
    g.ldp = ldp;
    g.act = act;
    g.lanes = act_grad_lanes(N);
    if (own_dz) {
      g.dz = workspace;
      g.ldz = N;
    }
    float* sums = (float*)((char*)workspace + backward_sums(M, N));
    if (dbias) g.partial = blocks == 1 ? (float*)dbias : sums;
    if (launch_act_grad(g, in == ALCOP_BF16, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    if (dbias && blocks > 1) {
      const ColumnSumArgs s{sums, (float*)dbias, blocks, N};
      if (launch_column_sums(s, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    }
  }
  if (dA) {
    const alcop_epilogue e{alpha, nullptr, 0};
    const int rc = alcop_gemm_fused(dZ, W, dA, M, K, N, lddz, ldw, ldda, 0, transB ? 0 : 1, in, out, &e, nullptr, st);
    if (rc) return rc;
  }
  if (dW) {
    // what is left of the workspace behind dZ and the partial sums
    const size_t split = std::max(gradient_workspace(N, K, M), gradient_workspace(K, N, M));
    const size_t all = alcop_linear_backward_workspace_bytes(M, N, K);
    void* ws = workspace && workspace_bytes >= all ? (char*)workspace + (all - split) : nullptr;
    const int rc = transB ? gradient_product(dZ, A, dW, N, K, M, lddz, lda, lddw, in, out, alpha, ws, split, st)
                          : gradient_product(A, dZ, dW, K, N, M, lda, lddz, lddw, in, out, alpha, ws, split, st);
    if (rc) return rc;
  }
  return ALCOP_OK;
}

static int norm_rows(const void* x, const void* residual, const void* gain, void* total, void* y, void* scale, void* rstd,
                     int rows, int cols, long ldx, long ldr, long ldt, long ldy, float eps, bool norm, alcop_dtype in,
                     alcop_dtype out, void* hip_stream)
{
  if (!x || !y || (out == ALCOP_E4M3 && !scale)) return ALCOP_ERR_NULL;
  if (!is_half(in) && in != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if (!is_half(out) && out != ALCOP_F32 && out != ALCOP_E4M3) return ALCOP_ERR_DTYPE;
  if (rows <= 0 || cols <= 0) return ALCOP_ERR_SHAPE;
  if (ldx < cols || ldy < cols || (residual && ldr < cols) || (total && ldt < cols)) return ALCOP_ERR_SHAPE;
  if (cols > ROWS_MAX_COLS) return ALCOP_ERR_SIZE;
  if (rows / rows_per_block(rows, cols) >= (1 << 22) - 1) return ALCOP_ERR_SIZE;    // threads of a launch: 32 bits, 1024 a block
  const int isz = size_of(in), osz = size_of(out);
  if (!aligned(x, isz) || !aligned(residual, isz) || !aligned(total, isz) || !aligned(y, osz) || !aligned(gain, 4) ||
      !aligned(scale, 4) || !aligned(rstd, 4))
    return ALCOP_ERR_ALIGN;
  if (out != ALCOP_E4M3) scale = nullptr;
  // a row is read whole before anything of y is stored, element by element before the sum is
  const Span sx(x, rows, cols, ldx, isz), sr(residual, rows, cols, ldr, isz), st(total, rows, cols, ldt, isz),
      sy(y, rows, cols, ldy, osz), sg(gain, 1, cols, cols, 4), ss(scale, 1, rows, rows, 4), sd(rstd, 1, rows, rows, 4);
  if ((meet(sy, sx) && !(same(sy, sx) && in == out)) || (meet(sy, sr) && !(same(sy, sr) && in == out)) || meet(sy, st))
    return ALCOP_ERR_UNSUPPORTED;
  if ((meet(st, sx) && !same(st, sx)) || (meet(st, sr) && !same(st, sr))) return ALCOP_ERR_UNSUPPORTED;
  for (const Span& o : {sy, st, ss, sd})
    if (meet(o, sg)) return ALCOP_ERR_UNSUPPORTED;
  for (const Span& s : {sx, sr, st, sy})
    if (meet(s, ss) || meet(s, sd)) return ALCOP_ERR_UNSUPPORTED;
  if (meet(ss, sd)) return ALCOP_ERR_UNSUPPORTED;

  NormArgs a;
  a.x = x;
  a.residual = residual;
  a.gain = (const float*)gain;
  a.total = total;
  a.y = y;
  a.scale = (float*)scale;
  a.rstd = (float*)rstd;
  a.ldx = ldx;
  a.ldr = residual ? ldr : 0;
  a.ldt = total ? ldt : 0;
  a.ldy = ldy;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  a.flags = (int)out | (norm ? 4 : 0);
  return launch_norm_rows(a, (int)in, cols % 8 == 0, (hipStream_t)hip_stream) == hipSuccess ? ALCOP_OK : ALCOP_ERR_LAUNCH;
}

int alcop_rmsnorm(const void* x, const void* residual, const void* gain, void* total, void* y, void* scale, void* rstd,
                  int rows, int cols, long ldx, long ldr, long ldt, long ldy, float eps, alcop_dtype in, alcop_dtype out,
                  void* hip_stream)
{
  return norm_rows(x, residual, gain, total, y, scale, rstd, rows, cols, ldx, ldr, ldt, ldy, eps, true, in, out, hip_stream);
}

int alcop_quantize_rows(const void* x, void* y, void* scale, int rows, int cols, long ldx, long ldy, alcop_dtype in,
                        void* hip_stream)
{
  return norm_rows(x, nullptr, nullptr, nullptr, y, scale, nullptr, rows, cols, ldx, 0, 0, ldy, 0.0f, false, in, ALCOP_E4M3,
                   hip_stream);
}

size_t alcop_rmsnorm_backward_workspace_bytes(int rows, int cols)
{
  if (rows <= 0 || cols <= 0 || cols > ROWS_MAX_COLS) return 0;
  return r256(4.0 * norm_blocks(rows, cols) * cols);
}

int alcop_rmsnorm_backward(const void* dy, const void* total, const void* gain, const void* rstd, const void* dtotal,
                           void* dx, void* dgain, int rows, int cols, long lddy, long ldt, long lddt, long lddx,
                           alcop_dtype in, void* workspace, size_t workspace_bytes, void* hip_stream)
{
  if (!dy || !total || !rstd || !dx || (dgain && !workspace)) return ALCOP_ERR_NULL;
  if (!is_half(in) && in != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if (rows <= 0 || cols <= 0) return ALCOP_ERR_SHAPE;
  if (lddy < cols || ldt < cols || lddx < cols || (dtotal && lddt < cols)) return ALCOP_ERR_SHAPE;
  if (cols > ROWS_MAX_COLS) return ALCOP_ERR_SIZE;
  const int isz = size_of(in);
  if (!aligned(dy, isz) || !aligned(total, isz) || !aligned(dtotal, isz) || !aligned(dx, isz) || !aligned(gain, 4) ||
      !aligned(rstd, 4) || !aligned(dgain, 4) || !aligned(workspace, 16))
    return ALCOP_ERR_ALIGN;
  const size_t need = alcop_rmsnorm_backward_workspace_bytes(rows, cols);
  if (dgain && workspace_bytes < need) return ALCOP_ERR_SIZE;
  // dx may be dy or dtotal, whose elements its own threads have read by then
  const Span sdy(dy, rows, cols, lddy, isz), sh(total, rows, cols, ldt, isz), sdt(dtotal, rows, cols, lddt, isz),
      sdx(dx, rows, cols, lddx, isz), sg(gain, 1, cols, cols, 4), sr(rstd, 1, rows, rows, 4), sdg(dgain, 1, cols, cols, 4);
  if ((meet(sdx, sdy) && !(same(sdx, sdy))) || (meet(sdx, sdt) && !same(sdx, sdt)) || meet(sdx, sh) || meet(sdx, sg) ||
      meet(sdx, sr) || meet(sdx, sdg))
    return ALCOP_ERR_UNSUPPORTED;
  Span sw(dgain ? workspace : nullptr, 1, 1, 1, 1);
  sw.row = sw.pitch = (double)need;
  for (const Span& s : {sdy, sh, sdt, sg, sr})
    if (meet(s, sdg) || meet(s, sw)) return ALCOP_ERR_UNSUPPORTED;
  if (meet(sw, sdx) || meet(sw, sdg)) return ALCOP_ERR_UNSUPPORTED;

  NormGradArgs a;
  a.dy = dy;
  a.total = total;
  a.dtotal = dtotal;
  a.gain = (const float*)gain;
  a.rstd = (const float*)rstd;
  a.dx = dx;
  a.partial = dgain ? (float*)workspace : nullptr;
  a.lddy = lddy;
  a.ldt = ldt;
  a.lddt = dtotal ? lddt : 0;
  a.lddx = lddx;
  a.rows = rows;
  a.cols = cols;
  const int blocks = norm_blocks(rows, cols);
  if (dgain && blocks == 1) a.partial = (float*)dgain;
  hipStream_t st = (hipStream_t)hip_stream;
  if (launch_norm_grad(a, blocks * rows_per_block(rows, cols), (int)in, cols % 8 == 0, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  if (dgain && blocks > 1) {
    const ColumnSumArgs s{(const float*)workspace, (float*)dgain, blocks, cols};
    if (launch_column_sums(s, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  }
  return ALCOP_OK;
}

}  // extern "C"
