// Host code of the cross entropy of a vocabulary's product: argument checks, the pieces, launches.  Declarations and argument
// contracts are in include/alcop.h.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "alcop_checks.h"
#include "alcop_linear_cost.h"
#include "alcop_loss.h"

namespace alcop {
namespace {

struct LossTable {
  std::vector<LossKernel> all;
  LossTable()
  {
    register_loss(all);
    for (LossKernel& k : all)
      for (const LinearCost& m : kLinearCost)
        if (m.dt == 1 && m.bl == (k.step == LOSS_STRIPS || k.step == LOSS_GRADIENT ? 1 : 0) && std::memcmp(&m.s, &k.s, sizeof(k.s)) == 0)
          k.cost = &m;
  }
};
const LossTable& loss_table()
{
  static const LossTable t;
  return t;
}

// Strips leave next to nothing of a tile, where the costs of a layer count its store, and few rows leave most of a large tile's loads out.  us
// of 64x64, 128x64, 128x128, 256x128 and 256x256 tiles, and (in brackets) what the costs alone would have picked of them, bf16:
//   128 x 65536 x 2048  92.7 [79.1] 73.2 78.2 75.8     256 rows  143 121 97.1 [84.8] 79.5     100 x 50257 x 1600  59.1 [55.7] 45.1 54.8 51.4
//   200 x 128256 x 1024 135 118 [96.7] 93.4 80.7       64 rows   [69.1] 73.8 72.8 76.3 79.6   400 x 10007 x 128  11.6 12.4 [11.5] 13.4 13.8
// On 24 products that the factors were not fitted on (100 to 600 rows, 5000 to 40000 columns, K of 2000 to 8000) the pick of the strips took 1.04 of
// the best kernel's time on average, 1.19 at worst (139 x 14496 x 4784: 82.0 us with 256x128, 69.1 with 128x64).
// dX in slices of a long vocabulary in 256x256 tiles, us of the whole backward pass and [what the costs alone would have picked]:
//   700 x 50257 x 768  303 [311] 309 307 280     2000 x 100000 x 512  976 940 927 [911] 844     300 x 30000 x 1024  118 [125] 125 129 145
double side(LossStep step, const alcop_sched& s)
{
  if (step == LOSS_DX) return s.bn == 256 ? 0.85 : 1.0;
  if (step != LOSS_STRIPS) return 1.0;
  return s.bm == 256 ? (s.bn == 256 ? 0.70 : 0.75) : s.bm == 128 && s.bn == 128 ? 0.86 : 1.0;
}

// The kernel of a step of the lowest cost, as alcop_linear has it; slices: as many such products in one launch.
const LossKernel* pick(LossStep step, int dt, int M, int N, int K, double bytes, int slices = 1)
{
  const LossKernel* best = nullptr;
  double best_us = 0;
  const char* env = std::getenv("ALCOP_LINEAR_KERNEL");       // a tuning and test knob: its number among those of a step
  int nr = 0;
  for (const LossKernel& k : loss_table().all) {
    if (k.step != step || k.dt != dt) continue;
    if (env && *env) {
      if (nr++ == std::atoi(env)) return &k;
      continue;
    }
    if (!k.cost) continue;
    const double tiles = (double)(((long)M + k.s.bm - 1) / k.s.bm) * (((long)N + k.s.bn - 1) / k.s.bn) * slices;
    const double us = linear_us(*k.cost, tiles, (double)M * N * slices, K, bytes) * side(step, k.s);
    if (!best || us < best_us) {
      best = &k;
      best_us = us;
    }
  }
  return best;
}

// Whether a product's tiles can be addressed and counted; its grid.
int grid_of(const LossKernel* k, int M, int N, long lda, long ldb, dim3* grid)
{
  if (!k) return ALCOP_ERR_SCHED;
  const double rows = std::min(k->s.bm, M), cols = std::min(k->s.bn, N);
  if (2.0 * rows * lda >= 2147483648.0 || 2.0 * cols * ldb >= 2147483648.0) return ALCOP_ERR_SIZE;
  const long ntm = ((long)M + k->s.bm - 1) / k->s.bm, ntn = ((long)N + k->s.bn - 1) / k->s.bn;
  if (ntm * ntn >= (1L << 32) / k->threads) return ALCOP_ERR_SHAPE;      // threads of a launch are counted in 32 bits
  *grid = dim3((unsigned)(ntm * ntn));
  return ALCOP_OK;
}

constexpr int STRIP = 64;      // columns of the narrowest strip

// The pieces of the vocabulary, and what the workspace holds: G, the fp32 sums of dX, S.
struct Pieces {
  int width;                   // columns, a multiple of 256 where there are several pieces
  int pitch;                   // of G
  int count;
  int slices, slice;           // of a piece's columns, for dX
  bool sums;                   // whether dX is added up in the workspace
  size_t dx, scale, all;       // where they start, and the end
};
Pieces pieces_of(int rows, int vocab, int K)
{
  // G of a piece: 128 MiB, which with what the products read stays in the memory-side cache (4096 rows, 65536 x 2048 bf16, pieces of
  // 64 to 512 MiB: 2878, 2762, 2896 and 2970 us, of 32 MiB 3200), or 256 columns of so many rows that it is more
  const char* env = std::getenv("ALCOP_LOSS_PIECE");          // a test knob: columns of a piece, a multiple of 256
  long most = env && std::atoi(env) > 0 ? (std::atoi(env) + 255) / 256 * 256 : std::max(256L, (1L << 26) / rows / 256 * 256);
  // dX walks the vectors of a slice by 32-bit offsets, up to 128 past the last: 1 GiB of them at most, so that pitches of up to 2 K reach
  const long reach = std::max(256L, ((1L << 29) / K - 128) / 256 * 256);
  const double tiles = (double)((rows + 255L) / 256) * ((K + 255L) / 256);
  Pieces p;
  for (;; most = std::min(most - 256, reach * p.slices)) {
    p.width = (int)std::min((long)vocab, most);
    p.count = (int)(((long)vocab + p.width - 1) / p.width);
    if (p.count > 1) {
      // equal pieces
      const long even = ((long)vocab + p.count - 1) / p.count;
      p.width = (int)((even + 255) / 256 * 256);
      p.count = (int)(((long)vocab + p.width - 1) / p.width);
    }
    p.pitch = (p.width + 7) & ~7;
    // dX: slices of the piece while its largest tiles leave compute units idle, each 2048 columns or more
    p.slices = 1;
    while (p.slices < 16 && tiles * p.slices * 2 <= 256 && p.pitch / (p.slices * 2) >= 2048) p.slices *= 2;
    p.slice = p.slices > 1 ? (p.pitch / p.slices + 255) / 256 * 256 : p.pitch;
    p.slices = (p.pitch + p.slice - 1) / p.slice;
    if (p.slice <= reach) break;          // at 256 columns at the latest
  }
  p.sums = p.count > 1 || p.slices > 1;
  p.dx = r256(2.0 * rows * p.pitch);
  p.scale = p.dx + (p.sums ? r256(4.0 * rows * K * p.slices) : 0);
  p.all = p.scale + 256;
  return p;
}

int check_operands(const void* X, const void* W, const void* labels, int rows, int vocab, int K, long ldx, long ldw, float alpha,
                   alcop_dtype in)
{
  if (!X || !W || !labels) return ALCOP_ERR_NULL;
  if (!is_half(in)) return ALCOP_ERR_DTYPE;
  if (rows <= 0 || vocab <= 0 || K <= 0 || K % 8) return ALCOP_ERR_SHAPE;
  if (ldx < K || ldw < K) return ALCOP_ERR_SHAPE;
  if (!aligned(X, 16) || !aligned(W, 16) || ldx % 8 || ldw % 8 || !aligned(labels, 8)) return ALCOP_ERR_ALIGN;
  if (!(alpha > 0.f) || alpha > 2e38f) return ALCOP_ERR_UNSUPPORTED;       // alpha log2(e) is finite
  if (ldx >= (1L << 30) || ldw >= (1L << 30) || std::max(rows, std::max(vocab, K)) > 0x7ffff000) return ALCOP_ERR_SIZE;
  return ALCOP_OK;
}

}  // namespace

hipError_t prepare_loss()
{
  for (const LossKernel& k : loss_table().all) {
    const hipError_t rc = k.prepare();
    if (rc != hipSuccess) return rc;
  }
  return prepare_loss_rows();
}

}  // namespace alcop

using namespace alcop;

extern "C" {

size_t alcop_linear_cross_entropy_workspace_bytes(int rows, int vocab, int K)
{
  if (rows <= 0 || vocab <= 0 || K <= 0 || K % 8) return 0;
  return r256(4.0 * rows) + r256(8.0 * rows * (((double)vocab + STRIP - 1) / STRIP));
}

int alcop_linear_cross_entropy(const void* X, const void* W, const void* labels, void* loss, void* lse, int rows, int vocab, int K,
                               long ldx, long ldw, float alpha, alcop_dtype in, void* workspace, size_t workspace_bytes,
                               void* hip_stream)
{
  if (!loss || !workspace) return ALCOP_ERR_NULL;
  int rc = check_operands(X, W, labels, rows, vocab, K, ldx, ldw, alpha, in);
  if (rc) return rc;
  if (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(workspace, 16)) return ALCOP_ERR_ALIGN;
  const size_t need = alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K);
  if (workspace_bytes < need || (rows + 31L) / 32 * 1024 >= 1L << 32) return ALCOP_ERR_SIZE;      // threads of the second launch
  Span sw(workspace, 1, 1, 1, 1);
  sw.row = sw.pitch = (double)need;
  const Span outs[] = {Span(loss, 1, rows, rows, 4), Span(lse, 1, rows, rows, 4), sw};
  const Span ins[] = {Span(X, rows, K, ldx, 2), Span(W, vocab, K, ldw, 2), Span(labels, 1, rows, rows, 8)};
  for (int i = 0; i < 3; i++) {
    for (const Span& s : ins)
      if (meet(outs[i], s)) return ALCOP_ERR_UNSUPPORTED;
    for (int j = 0; j < i; j++)
      if (meet(outs[i], outs[j])) return ALCOP_ERR_UNSUPPORTED;
  }
  const LossKernel* k = pick(LOSS_STRIPS, in == ALCOP_BF16, rows, vocab, K, 2.0 * K * ((double)rows + vocab));
  dim3 grid;
  rc = grid_of(k, rows, vocab, ldx, ldw, &grid);
  if (rc) return rc;

  LossArgs a;
  std::memset(&a, 0, sizeof(a));
  a.X = X;
  a.W = W;
  a.labels = labels;
  a.hit = (float*)workspace;
  a.out = (char*)workspace + r256(4.0 * rows);
  a.M = rows;
  a.N = a.vocab = vocab;
  a.K = K;
  a.lda = (int)ldx;
  a.ldw = (int)ldw;
  a.alpha = alpha;
  hipStream_t st = (hipStream_t)hip_stream;
  if (std::getenv("ALCOP_LOG"))
    std::fprintf(stderr, "alcop: linear cross entropy rows %d vocabulary %d K %d -> tile %dx%dx%d grid %u\n", rows, vocab, K, k->s.bm,
                 k->s.bn, k->s.bk, grid.x);
  if (k->launch(a, grid, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  LossRowsArgs r;
  r.strips = (const char*)a.out;
  r.labels = labels;
  r.hit = a.hit;
  r.loss = (float*)loss;
  r.lse = (float*)lse;
  r.rows = rows;
  r.count = (int)(((long)vocab + k->s.bn - 1) / k->s.bn);
  r.vocab = vocab;
  r.alpha = alpha;
  return launch_loss_rows(r, st) == hipSuccess ? ALCOP_OK : ALCOP_ERR_LAUNCH;
}

size_t alcop_linear_cross_entropy_backward_workspace_bytes(int rows, int vocab, int K)
{
  if (rows <= 0 || vocab <= 0 || K <= 0 || K % 8) return 0;
  return pieces_of(rows, vocab, K).all;
}

int alcop_linear_cross_entropy_backward(const void* X, const void* W, const void* labels, const void* lse, const void* dloss,
                                        void* dX, void* dW, int rows, int vocab, int K, long ldx, long ldw, long lddx, long lddw,
                                        float alpha, alcop_dtype in, alcop_dtype out, void* workspace, size_t workspace_bytes,
                                        void* hip_stream)
{
  if (!lse || (!dX && !dW) || !workspace) return ALCOP_ERR_NULL;
  int rc = check_operands(X, W, labels, rows, vocab, K, ldx, ldw, alpha, in);
  if (rc) return rc;
  if (out != in && out != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if ((dX && lddx < K) || (dW && lddw < K)) return ALCOP_ERR_SHAPE;
  if (!aligned(lse, 4) || !aligned(dloss, 4) || !aligned(workspace, 16)) return ALCOP_ERR_ALIGN;
  if ((dX && (!aligned(dX, 16) || lddx % 8)) || (dW && (!aligned(dW, 16) || lddw % 8))) return ALCOP_ERR_ALIGN;
  if ((dX && lddx >= (1L << 30)) || (dW && lddw >= (1L << 30))) return ALCOP_ERR_SIZE;
  const Pieces pc = pieces_of(rows, vocab, K);
  if (workspace_bytes < pc.all) return ALCOP_ERR_SIZE;
  const int osz = size_of(out), dt = in == ALCOP_BF16;
  Span sw(workspace, 1, 1, 1, 1);
  sw.row = sw.pitch = (double)pc.all;
  const Span outs[] = {Span(dX, rows, K, lddx, osz), Span(dW, vocab, K, lddw, osz), sw};
  const Span ins[] = {Span(X, rows, K, ldx, 2), Span(W, vocab, K, ldw, 2), Span(labels, 1, rows, rows, 8), Span(lse, 1, rows, rows, 4),
                      Span(dloss, 1, rows, rows, 4)};
  for (int i = 0; i < 3; i++) {
    for (const Span& s : ins)
      if (meet(outs[i], s)) return ALCOP_ERR_UNSUPPORTED;
    for (int j = 0; j < i; j++)
      if (meet(outs[i], outs[j])) return ALCOP_ERR_UNSUPPORTED;
  }

  // dX is added up in fp32: where it is to be, or in the workspace
  const bool direct = !pc.sums || (out == ALCOP_F32 && pc.slices == 1);
  if (dX && !direct && (long)rows * (K / 8) > (1L << 32) - 256) return ALCOP_ERR_SIZE;             // threads of the last launch
  // every piece's products, the widest and the last, before anything is launched
  const int last = vocab - (pc.count - 1) * pc.width;
  const LossKernel *kg[2], *kx[2] = {nullptr, nullptr}, *kw[2] = {nullptr, nullptr};
  dim3 gg[2], gx[2], gw[2];
  for (int i = 0; i < 2; i++) {
    const int n = i ? last : pc.width, n8 = (n + 7) & ~7;
    const double g_bytes = 2.0 * rows * n8;
    kg[i] = pick(LOSS_GRADIENT, dt, rows, n, K, 2.0 * K * ((double)rows + n) + g_bytes);
    rc = grid_of(kg[i], rows, n, ldx, ldw, &gg[i]);
    if (rc) return rc;
    if (dX) {
      const int slices = (n8 + pc.slice - 1) / pc.slice;
      kx[i] = pick(LOSS_DX, dt, rows, K, std::min(n8, pc.slice), (g_bytes + 2.0 * n * (double)K) + 8.0 * rows * K * slices, slices);
      rc = grid_of(kx[i], rows, K, pc.pitch, 8, &gx[i]);
      if (rc) return rc;
      gx[i].y = (unsigned)slices;
      if (2.0 * (std::min(n8, pc.slice) + 128.0) * ldw >= 2147483648.0 || 4.0 * 256 * lddx >= 2147483648.0) return ALCOP_ERR_SIZE;
    }
    if (dW) {
      kw[i] = pick(LOSS_DW, dt, n8, K, rows, g_bytes + 2.0 * rows * (double)K + (double)osz * n * K);
      rc = grid_of(kw[i], n8, K, 8, 8, &gw[i]);
      if (rc) return rc;
      // rows are walked by 32-bit offsets, up to a k-tile past the last
      if (2.0 * (rows + 128.0) * std::max((long)pc.pitch, ldx) >= 2147483648.0 || 4.0 * 256 * lddw >= 2147483648.0) return ALCOP_ERR_SIZE;
    }
  }

  hipStream_t st = (hipStream_t)hip_stream;
  float *sums = (float*)((char*)workspace + pc.dx), *scale = (float*)((char*)workspace + pc.scale);
  const bool scaled = in == ALCOP_F16;
  if (scaled && dloss) {
    const LossScaleArgs s{(const float*)dloss, labels, scale, rows, vocab};
    if (launch_loss_scale(s, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  }
  const float fixed = scaled && !dloss ? 16384.0f : 1.0f;        // S where |dloss| is 1
  const float* inverse = scaled && dloss ? scale + 1 : nullptr;
  for (int i = 0; i < pc.count; i++) {
    const int end = i == pc.count - 1, v0 = i * pc.width, n = end ? last : pc.width, n8 = (n + 7) & ~7;
    LossArgs a;
    std::memset(&a, 0, sizeof(a));
    a.X = X;
    a.W = (const char*)W + 2 * (long)v0 * ldw;
    a.labels = labels;
    a.out = workspace;
    a.lse = (const float*)lse;
    a.dloss = (const float*)dloss;
    a.scale = scaled && dloss ? scale : nullptr;
    a.s = fixed;
    a.M = rows;
    a.N = n;
    a.K = K;
    a.lda = (int)ldx;
    a.ldw = (int)ldw;
    a.ldg = pc.pitch;
    a.v0 = v0;
    a.vocab = vocab;
    a.alpha = alpha;
    if (kg[end]->launch(a, gg[end], st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    LossProductArgs p;
    if (dX) {
      std::memset(&p, 0, sizeof(p));
      p.l.A = workspace;
      p.l.W = a.W;
      p.l.C = direct ? dX : sums;
      p.l.ldc = direct ? (int)lddx : K;
      p.l.residual = i ? p.l.C : nullptr;          // the last piece may have fewer slices: theirs are the first
      p.l.ldr = p.l.ldc;
      p.l.M = rows;
      p.l.N = K;
      p.l.K = n8;
      p.l.lda = pc.pitch;
      p.l.ldw = (int)ldw;
      p.l.alpha = alpha / fixed;
      p.l.flags = (int)(direct ? out : ALCOP_F32);
      p.inverse = inverse;
      p.depth = n;
      p.slice = std::min(n8, pc.slice);
      p.next = (long)rows * K;
      if (kx[end]->launch_product(p, gx[end], st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    }
    if (dW) {
      std::memset(&p, 0, sizeof(p));
      p.l.A = workspace;
      p.l.W = X;
      p.l.C = (char*)dW + (long)v0 * lddw * osz;
      p.l.ldc = (int)lddw;
      p.l.M = n8;
      p.l.N = K;
      p.l.K = rows;
      p.l.lda = pc.pitch;
      p.l.ldw = (int)ldx;
      p.l.alpha = alpha / fixed;
      p.l.flags = (int)out;
      p.inverse = inverse;
      p.depth = n;
      if (kw[end]->launch_product(p, gw[end], st) != hipSuccess) return ALCOP_ERR_LAUNCH;
    }
  }
  if (dX && !direct) {
    const RoundArgs r{sums, dX, lddx, rows, K, (int)out, pc.slices};
    if (launch_round_rows(r, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  }
  return ALCOP_OK;
}

}  // extern "C"
