// Host code of the products grouped by expert: argument checks, choice of the kernel, launches.  Declarations and argument
// contracts are in include/alcop.h.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "alcop_checks.h"
#include "alcop_grouped.h"
#include "alcop_linear_cost.h"

namespace alcop {
namespace {

const LinearCost* cost_of(int dt, int bl, const alcop_sched& s)
{
  for (const LinearCost& m : kLinearCost)
    if (m.dt == (dt == 0 ? 1 : dt) && m.bl == bl && std::memcmp(&m.s, &s, sizeof(s)) == 0) return &m;
  return nullptr;
}

struct GroupedTable {
  std::vector<GroupedKernel> all;
  std::vector<const GroupedKernel*> of[3][3][2];      // class of activation, operand type of a call (e4m3 as 2), layout
  std::vector<GroupedGradKernel> grad;
  GroupedTable()
  {
    register_grouped_f16(all);
    register_grouped_bf16(all);
    register_grouped_e4m3(all);
    register_grouped_f8(all);
    register_grouped_grad(grad);
    for (GroupedKernel& k : all) {
      k.cost = cost_of(k.dt, k.bl, k.s);
      of[k.cls][std::min(k.dt, 2)][k.bl].push_back(&k);
    }
    for (GroupedGradKernel& k : grad) k.cost = cost_of(k.dt, 0, k.s);
  }
};
const GroupedTable& grouped_table()
{
  static const GroupedTable t;
  return t;
}

// Tiles of bm rows that `rows` rows of `groups` groups make at most.
long most_tiles(long rows, long groups, long bm)
{
  const long g = std::min(groups, rows);
  return (rows + g * (bm - 1)) / bm;
}
// Microseconds by the costs of the linear layers (alcop_linear_cost.h) where the groups' sizes are not known: as many full tiles as
// even groups have, a half more each for the one that is not full, and turns of the card that need not be whole.
double grouped_us(const LinearCost& m, long rows, long groups, int N, int K, double bytes)
{
  const double live = (double)std::min(groups, rows), per = (double)rows / live;
  const double tiles = live * std::max(1.0, per / m.s.bm + 0.5) * (double)((N + (long)m.s.bn - 1) / m.s.bn);
  const double turns = std::max(1.0, tiles / 256), turns2 = m.blocks == 2 ? 2 * std::max(1.0, tiles / 512) : 0.0;
  const double kt = (double)((K + m.s.bk - 1) / m.s.bk + m.waves_k - 1) / m.waves_k;
  const double us = m.a + m.b * turns * kt + m.c * turns + m.d * bytes / 5.1e6 + m.e * 2.0 * rows * N * (double)K / 1.4e9 + m.f * turns2 * kt;
  // The costs are those of one product; groups' tiles end at other rows than its, and the two large ones are quartered.  What three tiles
  // take beside their costs, with the other tiles of the same products (us, bf16, measured for the cost):
  //   256x256  16384 x 4096 x 2048 in 16 groups 336 for 373, in one 267 for 282; 2500 rows in 5 66 (256x128 71); 8192 x 2048 x 2048 in
  //            16 groups, gradients, 202 (256x128 206, 128x128 224)
  //   256x128  the first in 16 groups 343 for 411, in one 286 for 348 (128x128 382 for 387, 295 for 331)
  //   128x64   1531 x 1048 x 520 in 12 groups, fp16, 12.3 for 9.2 (64x64 11.0 for 9.3); 1150 x 2048 x 1024 in 4 14.2 (64x64 13.7)
  const double side = m.s.bm == 256 ? (m.s.bn == 128 ? 0.86 : 0.88) : m.s.bm == 128 && m.s.bn == 64 ? 1.08 : 1.0;
  return side * us;
}

// The kernel of the lowest cost.
const GroupedKernel* pick(int cls, int dt, int bl, bool fine, int rows, int groups, int N, int K, double bytes)
{
  const GroupedKernel* best = nullptr;
  double best_us = 0;
  const char* env = std::getenv("ALCOP_LINEAR_KERNEL");       // a tuning and test knob: its number among those of the layout
  int nr = 0;
  for (const GroupedKernel* e : grouped_table().of[cls][dt][bl]) {
    const GroupedKernel& k = *e;
    if (k.dt == 3 && fine) continue;
    if (env && *env) {
      if (nr++ == std::atoi(env)) return &k;
      continue;
    }
    if (!k.cost) continue;
    const double us = grouped_us(*k.cost, rows, groups, N, K, bytes);
    if (!best || us < best_us) {
      best = &k;
      best_us = us;
    }
  }
  return best;
}

// Rows of a block of alcop_grouped_act_grad, as a power of two: enough blocks to fill the card, which finds room for 2048 at a time (1024 with
// 512 columns each; 8192 rows of 2048 in 16 groups, us of the whole backward pass: 234, 230, 232, 229, 245 and 275 with 4 to 128
// rows), each with all its waves at work, and at most 1024 sums to a column beside a group's last.
int act_shift(int rows, int N)
{
  const int strips = (N + ACT_COLS - 1) / ACT_COLS;
  int lanes = 1, shift = 2;
  while (lanes < 64 && lanes * 8 < N) lanes *= 2;
  while ((1 << shift) < 256 / lanes) shift++;
  while (shift < 30 && (((long)rows >> shift) * strips > 1024 || ((long)rows >> shift) > 1024)) shift++;
  return shift;
}

struct GradPlan {
  size_t dz, sums, all;        // where the partial sums start, and the end
  int shift;
  long runs;
};
GradPlan plan_of(int rows, int groups, int N)
{
  GradPlan p;
  p.shift = act_shift(rows, N);
  p.runs = most_tiles(rows, groups, 1l << p.shift);
  p.dz = r256(2.0 * rows * N);
  p.sums = r256(4.0 * p.runs * N);
  p.all = p.dz + p.sums;
  return p;
}

// One matrix per group: rows x cols, `ld` apart, the groups `stride`.
Span group_span(const void* p, int groups, int rows, int cols, long ld, long stride, int size)
{
  Span s(p, groups, 1, stride, size);
  s.row = ((double)(rows - 1) * ld + cols) * size;
  return s;
}

// The kernel and the grid of a product whose arguments are in order.
int plan_product(const GroupedArgs& a, int cls, int dt, int bl, bool fine, int osz, double bytes, const GroupedKernel** kernel, dim3* grid)
{
  const LinearArgs& l = a.l;
  const GroupedKernel* k = pick(cls, dt, bl, fine, l.M, a.groups, l.N, l.K, bytes);
  if (!k) return ALCOP_ERR_SCHED;
  // 32-bit byte offsets from a tile's origin, rows past the end of a partial k-tile included
  const double rows = std::min(k->s.bm, l.M), cols = std::min(k->s.bn, l.N);
  const double kceil = (double)((l.K + k->s.bk - 1) / k->s.bk) * k->s.bk;
  if (2.0 * rows * l.lda >= 2147483648.0 || (bl ? 2.0 * cols * l.ldw : 2.0 * kceil * l.ldw) >= 2147483648.0) return ALCOP_ERR_SIZE;
  if (osz * rows * (double)std::max(l.ldc, l.ldp) >= 2147483648.0) return ALCOP_ERR_SIZE;
  const long strips = ((long)l.N + k->s.bn - 1) / k->s.bn, tiles = most_tiles(l.M, a.groups, k->s.bm);
  const long blocks = tiles * strips + (k->quarters ? 3L * (CARD / 2) : 0);      // tiles and strips are below 2^32
  if (blocks >= (1L << 32) / k->threads) return ALCOP_ERR_SHAPE;                 // threads are counted in 32 bits
  if (std::getenv("ALCOP_LOG"))
    std::fprintf(stderr, "alcop: grouped linear rows %d groups %d N %d K %d in %d -> tile %dx%dx%d waves %dx%d S%d R%d F%d variant %d grid %ld\n",
                 l.M, a.groups, l.N, l.K, dt, k->s.bm, k->s.bn, k->s.bk, k->s.wm, k->s.wn, k->s.stages, k->s.reg_stages,
                 k->s.fuse_inner, k->s.variant, blocks);
  *kernel = k;
  *grid = dim3((unsigned)blocks);
  return ALCOP_OK;
}

}  // namespace

hipError_t prepare_grouped()
{
  for (const GroupedKernel& k : grouped_table().all) {
    const hipError_t rc = k.prepare();
    if (rc != hipSuccess) return rc;
  }
  for (const GroupedGradKernel& k : grouped_table().grad) {
    const hipError_t rc = k.prepare();
    if (rc != hipSuccess) return rc;
  }
  return prepare_grouped_rows();
}

}  // namespace alcop

using namespace alcop;

extern "C" {

int alcop_grouped_linear(const void* A, const void* W, const void* offsets, void* C, int rows, int groups, int N, int K, long lda,
                         long ldw, long strideW, long ldc, int transB, alcop_dtype in, alcop_dtype out,
                         const alcop_linear_tail* tail, void* hip_stream)
{
  alcop_linear_tail t;
  std::memset(&t, 0, sizeof(t));
  t.alpha = 1.0f;
  if (tail) t = *tail;
  const bool fine = out == ALCOP_F32 || (t.act & ALCOP_FP32_SUMS);
  t.act &= ~ALCOP_FP32_SUMS;
  transB = transB ? 1 : 0;
  if (!A || !W || !offsets || !C) return ALCOP_ERR_NULL;
  if (!is_half(in) && in != ALCOP_E4M3) return ALCOP_ERR_DTYPE;
  if (!is_half(out) && out != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if (t.act < 0 || t.act > 4 || (in == ALCOP_E4M3 && !transB) || t.residual) return ALCOP_ERR_UNSUPPORTED;
  const int esz = size_of(in), osz = size_of(out), unit = 16 / esz;
  if (rows <= 0 || groups <= 0 || N <= 0 || K <= 0 || K % unit || (!transB && N % unit)) return ALCOP_ERR_SHAPE;
  const int w_rows = transB ? N : K, w_cols = transB ? K : N;
  if (lda < K || ldw < w_cols || ldc < N || (t.pre && t.ldp < N) || strideW < 0) return ALCOP_ERR_SHAPE;
  if (!aligned(A, 16) || !aligned(W, 16) || lda % unit || ldw % unit || strideW % unit) return ALCOP_ERR_ALIGN;
  if (!aligned(C, osz) || !aligned(t.pre, osz)) return ALCOP_ERR_ALIGN;
  for (const void* p : {offsets, t.bias, t.scale_w, t.scale_a})
    if (!aligned(p, 4)) return ALCOP_ERR_ALIGN;
  const long far = 1L << 30;
  if (lda >= far || ldw >= far || ldc >= far || t.ldp >= far) return ALCOP_ERR_SIZE;
  if (std::max(rows, N) > 0x7ffff000 || groups >= (1 << 24)) return ALCOP_ERR_SIZE;

  const Span c(C, rows, N, ldc, osz), z(t.pre, rows, N, t.ldp, osz);
  Span bias(t.bias, groups, N, N, 4), sw(t.scale_w, groups, N, N, 4);
  const Span read[] = {Span(A, rows, K, lda, esz), group_span(W, groups, w_rows, w_cols, ldw, strideW, esz), bias, sw,
                       Span(t.scale_a, 1, rows, rows, 4), Span(offsets, 1, groups + 1, groups + 1, 4)};
  for (const Span& s : read)
    if (meet(c, s) || meet(z, s)) return ALCOP_ERR_UNSUPPORTED;
  if (meet(c, z)) return ALCOP_ERR_UNSUPPORTED;

  const int K16 = in == ALCOP_E4M3 ? K / 2 : K;              // in units of 16 bits
  const double c_bytes = (double)osz * rows * N;
  const double bytes = 2.0 * K16 * ((double)rows + (double)std::min(groups, rows) * N) + c_bytes * (1 + (t.pre ? 1 : 0));
  GroupedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.l.A = A;
  a.l.W = W;
  a.l.C = C;
  a.l.pre = t.pre;
  a.l.bias = (const float*)t.bias;
  a.l.sa = (const float*)t.scale_a;
  a.l.sw = (const float*)t.scale_w;
  a.l.M = rows;
  a.l.N = N;
  a.l.K = K16;
  a.l.lda = (int)(in == ALCOP_E4M3 ? lda / 2 : lda);
  a.l.ldw = (int)(in == ALCOP_E4M3 ? ldw / 2 : ldw);
  a.l.ldc = (int)ldc;
  a.l.ldp = t.pre ? (int)t.ldp : 0;
  a.l.alpha = t.alpha;
  a.l.flags = (int)out | t.act << 2 | (c_bytes <= 48e6 ? 32 : 0);      // C kept in the memory-side cache, as alcop_linear does
  a.offsets = (const int*)offsets;
  a.groups = groups;
  a.strideW = in == ALCOP_E4M3 ? strideW / 2 : strideW;
  const GroupedKernel* k = nullptr;
  dim3 grid;
  const int rc = plan_product(a, class_of(t.act), in == ALCOP_E4M3 ? 2 : in == ALCOP_BF16 ? 1 : 0, transB, fine, osz, bytes, &k, &grid);
  if (rc) return rc;
  return k->launch(a, grid, (hipStream_t)hip_stream) == hipSuccess ? ALCOP_OK : ALCOP_ERR_LAUNCH;
}

size_t alcop_grouped_linear_backward_workspace_bytes(int rows, int groups, int N, int K)
{
  if (rows <= 0 || groups <= 0 || N <= 0 || K <= 0 || N % 8 || K % 8) return 0;
  return plan_of(rows, groups, N).all;
}

int alcop_grouped_linear_backward(const void* dC, const void* A, const void* W, const void* pre, const void* offsets, void* dA,
                                  void* dW, void* dbias, int rows, int groups, int N, int K, long lddc, long lda, long ldw,
                                  long strideW, long ldp, long ldda, long lddw, long stridedW, int transB, alcop_dtype in,
                                  alcop_dtype out, float alpha, int act, void* workspace, size_t workspace_bytes, void* hip_stream)
{
  transB = transB ? 1 : 0;
  if (!dC || !offsets || (!dA && !dW && !dbias) || (dA && !W) || (dW && !A)) return ALCOP_ERR_NULL;
  if (!is_half(in) || (out != in && out != ALCOP_F32)) return ALCOP_ERR_DTYPE;
  if (act < 0 || act > 4) return ALCOP_ERR_UNSUPPORTED;
  if (act && !pre) return ALCOP_ERR_NULL;
  if ((act || dbias) && !workspace) return ALCOP_ERR_NULL;
  if (rows <= 0 || groups <= 0 || N <= 0 || K <= 0 || N % 8 || K % 8) return ALCOP_ERR_SHAPE;
  if (std::max(rows, std::max(N, K)) > 0x7ffff000 || groups > 64000) return ALCOP_ERR_SIZE;
  // (64000 groups and the full runs of alcop_grouped_act_grad are fewer than 65536 blocks)
  const int w_rows = transB ? N : K, w_cols = transB ? K : N;
  if (lddc < N || (dW && lda < K) || (dA && (ldw < w_cols || strideW < 0)) || (act && ldp < N) || (dA && ldda < K)) return ALCOP_ERR_SHAPE;
  if (dW && (lddw < w_cols || (groups > 1 && stridedW < (long)(w_rows - 1) * lddw + w_cols))) return ALCOP_ERR_SHAPE;
  if (!aligned(dC, 16) || !aligned(workspace, 16) || !aligned(dbias, 4) || !aligned(offsets, 4) || lddc % 8) return ALCOP_ERR_ALIGN;
  if (act && (!aligned(pre, 16) || ldp % 8)) return ALCOP_ERR_ALIGN;
  if (dA && (!aligned(dA, 16) || !aligned(W, 16) || ldda % 8 || ldw % 8 || strideW % 8)) return ALCOP_ERR_ALIGN;
  if (dW && (!aligned(dW, 16) || !aligned(A, 16) || lddw % 8 || lda % 8 || stridedW % 8)) return ALCOP_ERR_ALIGN;
  const long far = 1L << 30;
  if (lddc >= far || (act && ldp >= far) || (dA && (ldda >= far || ldw >= far)) || (dW && (lddw >= far || lda >= far)))
    return ALCOP_ERR_SIZE;
  const GradPlan plan = plan_of(rows, groups, N);
  if ((act || dbias) && workspace_bytes < plan.all) return ALCOP_ERR_SIZE;
  if (dbias && ((long)N + SUM_COLS - 1) / SUM_COLS * GROUP_SUM_THREADS >= 1L << 32) return ALCOP_ERR_SIZE;      // threads of a launch

  const int osz = size_of(out);
  const Span outs[] = {Span(dA, rows, K, ldda, osz), group_span(dW, groups, w_rows, w_cols, lddw, stridedW, osz),
                       Span(dbias, groups, N, N, 4), Span(act || dbias ? workspace : nullptr, 1, 1, 1, 1)};
  const Span ins[] = {Span(dC, rows, N, lddc, 2), Span(dW ? A : nullptr, rows, K, lda, 2),
                      group_span(dA ? W : nullptr, groups, w_rows, w_cols, ldw, strideW, 2), Span(act ? pre : nullptr, rows, N, ldp, 2),
                      Span(offsets, 1, groups + 1, groups + 1, 4)};
  for (int i = 0; i < 4; i++) {
    Span o = outs[i];
    if (i == 3) o.row = o.pitch = (double)plan.all;
    for (const Span& s : ins)
      if (meet(o, s)) return ALCOP_ERR_UNSUPPORTED;
    for (int j = 0; j < i; j++)
      if (meet(o, outs[j])) return ALCOP_ERR_UNSUPPORTED;
  }

  const bool own_dz = act && (dA || dW);
  const void* dZ = own_dz ? workspace : dC;
  const long lddz = own_dz ? N : lddc;
  // dW: a group's rows are walked by 32-bit offsets, up to a k-tile past its last row
  if (dW && ((double)rows + 128) * 2.0 * std::max(lddz, lda) >= 2147483648.0) return ALCOP_ERR_SIZE;

  // what is refused is refused before anything is launched
  GroupedArgs ga;
  GroupedGradArgs gg;
  std::memset(&ga, 0, sizeof(ga));
  std::memset(&gg, 0, sizeof(gg));
  const GroupedKernel* ak = nullptr;
  const GroupedGradKernel* wk = nullptr;
  dim3 a_grid, w_grid;
  if (dA) {
    ga.l.A = dZ;
    ga.l.W = W;
    ga.l.C = dA;
    ga.l.M = rows;
    ga.l.N = K;
    ga.l.K = N;
    ga.l.lda = (int)lddz;
    ga.l.ldw = (int)ldw;
    ga.l.ldc = (int)ldda;
    ga.l.alpha = alpha;
    ga.l.flags = (int)out;
    ga.offsets = (const int*)offsets;
    ga.groups = groups;
    ga.strideW = strideW;
    const double bytes = 2.0 * N * ((double)rows + (double)std::min(groups, rows) * K) + (double)osz * rows * K;
    const int rc = plan_product(ga, CLASS_PLAIN, in == ALCOP_BF16, transB ? 0 : 1, true, osz, bytes, &ak, &a_grid);
    if (rc) return rc;
  }
  if (dW) {
    gg.P = transB ? dZ : A;
    gg.Q = transB ? A : dZ;
    gg.ldp = (int)(transB ? lddz : lda);
    gg.ldq = (int)(transB ? lda : lddz);
    gg.M = w_rows;
    gg.N = w_cols;
    gg.dW = dW;
    gg.ldw = (int)lddw;
    gg.strideW = stridedW;
    gg.offsets = (const int*)offsets;
    gg.groups = groups;
    gg.rows = rows;
    gg.alpha = alpha;
    gg.out = (int)out;
    if (osz * 256.0 * lddw >= 2147483648.0) return ALCOP_ERR_SIZE;
    const double depth = std::max(8.0, (double)rows / std::min(groups, rows));
    const double bytes = 2.0 * rows * ((double)N + K) + (double)osz * groups * N * K;
    double best_us = 0;
    const char* env = std::getenv("ALCOP_GRADIENT_KERNEL");       // a tuning and test knob: its number among those of the type
    int nr = 0;
    for (const GroupedGradKernel& k : grouped_table().grad) {
      if (k.dt != (in == ALCOP_BF16)) continue;
      const double tiles = (double)groups * ((w_rows + (long)k.s.bm - 1) / k.s.bm) * ((w_cols + (long)k.s.bn - 1) / k.s.bn);
      if (tiles >= 2147483648.0 || tiles * k.threads >= 4294967296.0) continue;
      const bool named = env && *env;
      if (named ? nr++ != std::atoi(env) : !k.cost) continue;
      // 256x256 tiles are a tenth below their costs: 2000 rows in 16 groups, 5000 x 4096, us of the whole backward pass 385 for 420 with 128x128,
      // 500 rows in 60 groups, 4096 x 4096, 779 for 880; 12000 in 30, 4096 x 512, 228 and 243
      const double side = k.s.bn == 256 ? 0.9 : 1.0;
      const double us = named ? 0.0 : side * linear_us(*k.cost, tiles, (double)groups * N * K, (int)depth, bytes);
      if (!wk || us < best_us) {
        wk = &k;
        best_us = us;
        w_grid = dim3((unsigned)tiles);
      }
    }
    if (!wk) return ALCOP_ERR_SHAPE;
  }

  hipStream_t st = (hipStream_t)hip_stream;
  if (own_dz || dbias) {
    GroupedActGradArgs g;
    std::memset(&g, 0, sizeof(g));
    g.a.dc = dC;
    g.a.pre = act ? pre : nullptr;
    g.a.M = rows;
    g.a.N = N;
    g.a.lddc = lddc;
    g.a.ldp = ldp;
    g.a.act = act;
    g.a.lanes = 1;
    while (g.a.lanes < 64 && g.a.lanes * 8 < N) g.a.lanes *= 2;
    if (own_dz) {
      g.a.dz = workspace;
      g.a.ldz = N;
    }
    float* sums = (float*)((char*)workspace + plan.dz);
    g.a.partial = dbias ? sums : nullptr;
    g.l = GroupList{(const int*)offsets, groups, rows};
    g.shift = plan.shift;
    if (launch_grouped_act_grad(g, in == ALCOP_BF16, (int)plan.runs, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    if (dbias) {
      const GroupedSumArgs s{ColumnSumArgs{sums, (float*)dbias, (int)plan.runs, N}, g.l, plan.shift};
      if (launch_grouped_sums(s, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    }
  }
  if (dA && ak->launch(ga, a_grid, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  if (dW && wk->launch(gg, w_grid, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  return ALCOP_OK;
}

}  // extern "C"
