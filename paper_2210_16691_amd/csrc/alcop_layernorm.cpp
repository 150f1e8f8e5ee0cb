// Host code of the layer norm: argument checks and launches.  Declarations and argument contracts are in include/alcop.h.
#include <algorithm>
#include <cstring>

#include "alcop_checks.h"
#include "alcop_layernorm.h"

namespace alcop {
namespace {

// Blocks that walk the rows of the gradients, each leaving a row of sums for dgain and one for dshift; as for the
// root-mean-square norm, a single block writes them itself.  One block a compute unit, two where its rows are short: more of them leave
// more sums, which are read again.  us with 256 and 512 blocks: 8192 x 4096 bf16 54.5 and 55.4 (1024: 70), 3000 x 16384 89 and 106, 2000 x
// 2048 13.6 and 19.4, 20000 x 1024 34.3 and 35.7; 1531 x 1111 fp16 14.2 and 13.0, 4750 x 318 12.7 and 11.8.
int grad_blocks(int rows, int cols, int size)
{
  const long blocks = ((long)rows + layernorm_rows_per_block(rows, cols) - 1) / layernorm_rows_per_block(rows, cols);
  const long most = (long)layernorm_rows_per_block(rows, cols) * cols * size >= 4096 ? 256 : 512;
  return blocks <= 2 ? 1 : (int)std::min(blocks, most);
}

}  // namespace
}  // namespace alcop

using namespace alcop;

extern "C" {

int alcop_layernorm(const void* x, const void* residual, const void* gain, const void* shift, void* total, void* y, void* scale,
                    void* mean, void* rstd, int rows, int cols, long ldx, long ldr, long ldt, long ldy, float eps, alcop_dtype in,
                    alcop_dtype out, void* hip_stream)
{
  if (!x || !y || (out == ALCOP_E4M3 && !scale)) return ALCOP_ERR_NULL;
  if (!is_half(in) && in != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if (!is_half(out) && out != ALCOP_F32 && out != ALCOP_E4M3) return ALCOP_ERR_DTYPE;
  if (rows <= 0 || cols <= 0) return ALCOP_ERR_SHAPE;
  if (ldx < cols || ldy < cols || (residual && ldr < cols) || (total && ldt < cols)) return ALCOP_ERR_SHAPE;
  if (cols > ROWS_MAX_COLS) return ALCOP_ERR_SIZE;
  if (rows / rows_per_block(rows, cols) >= (1 << 22) - 1) return ALCOP_ERR_SIZE;    // threads of a launch: 32 bits, 1024 a block; as alcop_rmsnorm
  const int isz = size_of(in), osz = size_of(out);
  if (!aligned(x, isz) || !aligned(residual, isz) || !aligned(total, isz) || !aligned(y, osz)) return ALCOP_ERR_ALIGN;
  for (const void* p : {gain, shift, (const void*)scale, (const void*)mean, (const void*)rstd})
    if (!aligned(p, 4)) return ALCOP_ERR_ALIGN;
  if (out != ALCOP_E4M3) scale = nullptr;
  // a row is read whole before anything of y is stored, element by element before the sum is
  const Span sx(x, rows, cols, ldx, isz), sr(residual, rows, cols, ldr, isz), st(total, rows, cols, ldt, isz),
      sy(y, rows, cols, ldy, osz), sg(gain, 1, cols, cols, 4), sb(shift, 1, cols, cols, 4);
  const Span per_row[] = {Span(scale, 1, rows, rows, 4), Span(mean, 1, rows, rows, 4), Span(rstd, 1, rows, rows, 4)};
  if ((meet(sy, sx) && !(same(sy, sx) && in == out)) || (meet(sy, sr) && !(same(sy, sr) && in == out)) || meet(sy, st))
    return ALCOP_ERR_UNSUPPORTED;
  if ((meet(st, sx) && !same(st, sx)) || (meet(st, sr) && !same(st, sr))) return ALCOP_ERR_UNSUPPORTED;
  for (const Span& v : {sg, sb}) {
    if (meet(v, st) || meet(v, sy)) return ALCOP_ERR_UNSUPPORTED;
    for (const Span& o : per_row)
      if (meet(v, o)) return ALCOP_ERR_UNSUPPORTED;
  }
  for (int i = 0; i < 3; i++) {
    for (const Span& s : {sx, sr, st, sy})
      if (meet(s, per_row[i])) return ALCOP_ERR_UNSUPPORTED;
    for (int j = 0; j < i; j++)
      if (meet(per_row[i], per_row[j])) return ALCOP_ERR_UNSUPPORTED;
  }

  LayerNormArgs a;
  a.x = x;
  a.residual = residual;
  a.gain = (const float*)gain;
  a.shift = (const float*)shift;
  a.total = total;
  a.y = y;
  a.scale = (float*)scale;
  a.mean = (float*)mean;
  a.rstd = (float*)rstd;
  a.ldx = ldx;
  a.ldr = residual ? ldr : 0;
  a.ldt = total ? ldt : 0;
  a.ldy = ldy;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  a.out = (int)out;
  return launch_layernorm_rows(a, (int)in, cols % 8 == 0, (hipStream_t)hip_stream) == hipSuccess ? ALCOP_OK : ALCOP_ERR_LAUNCH;
}

size_t alcop_layernorm_backward_workspace_bytes(int rows, int cols)
{
  if (rows <= 0 || cols <= 0 || cols > ROWS_MAX_COLS) return 0;
  return 2 * r256(4.0 * grad_blocks(rows, cols, 2) * cols);      // 32-bit rows need no more
}

int alcop_layernorm_backward(const void* dy, const void* total, const void* gain, const void* mean, const void* rstd,
                             const void* dtotal, void* dx, void* dgain, void* dshift, int rows, int cols, long lddy, long ldt,
                             long lddt, long lddx, alcop_dtype in, void* workspace, size_t workspace_bytes, void* hip_stream)
{
  if (!dy || !total || !mean || !rstd || !dx || ((dgain || dshift) && !workspace)) return ALCOP_ERR_NULL;
  if (!is_half(in) && in != ALCOP_F32) return ALCOP_ERR_DTYPE;
  if (rows <= 0 || cols <= 0) return ALCOP_ERR_SHAPE;
  if (lddy < cols || ldt < cols || lddx < cols || (dtotal && lddt < cols)) return ALCOP_ERR_SHAPE;
  if (cols > ROWS_MAX_COLS) return ALCOP_ERR_SIZE;
  const int isz = size_of(in);
  if (!aligned(dy, isz) || !aligned(total, isz) || !aligned(dtotal, isz) || !aligned(dx, isz) || !aligned(workspace, 16))
    return ALCOP_ERR_ALIGN;
  for (const void* p : {gain, mean, rstd, (const void*)dgain, (const void*)dshift})
    if (!aligned(p, 4)) return ALCOP_ERR_ALIGN;
  const size_t need = alcop_layernorm_backward_workspace_bytes(rows, cols);
  const bool sums = dgain || dshift;
  if (sums && workspace_bytes < need) return ALCOP_ERR_SIZE;
  // dx may be dy or dtotal, whose elements its own threads have read by then
  const Span sdy(dy, rows, cols, lddy, isz), sh(total, rows, cols, ldt, isz), sdt(dtotal, rows, cols, lddt, isz),
      sdx(dx, rows, cols, lddx, isz), sg(gain, 1, cols, cols, 4), sm(mean, 1, rows, rows, 4), sr(rstd, 1, rows, rows, 4),
      sdg(dgain, 1, cols, cols, 4), sds(dshift, 1, cols, cols, 4);
  Span sw(sums ? workspace : nullptr, 1, 1, 1, 1);
  sw.row = sw.pitch = (double)need;
  if ((meet(sdx, sdy) && !same(sdx, sdy)) || (meet(sdx, sdt) && !same(sdx, sdt))) return ALCOP_ERR_UNSUPPORTED;
  for (const Span& s : {sh, sg, sm, sr, sdg, sds, sw})
    if (meet(sdx, s)) return ALCOP_ERR_UNSUPPORTED;
  for (const Span& s : {sdy, sh, sdt, sg, sm, sr})
    if (meet(s, sdg) || meet(s, sds) || meet(s, sw)) return ALCOP_ERR_UNSUPPORTED;
  if (meet(sdg, sds) || meet(sdg, sw) || meet(sds, sw)) return ALCOP_ERR_UNSUPPORTED;

  LayerNormGradArgs a;
  a.dy = dy;
  a.total = total;
  a.dtotal = dtotal;
  a.gain = (const float*)gain;
  a.mean = (const float*)mean;
  a.rstd = (const float*)rstd;
  a.dx = dx;
  a.lddy = lddy;
  a.ldt = ldt;
  a.lddt = dtotal ? lddt : 0;
  a.lddx = lddx;
  a.rows = rows;
  a.cols = cols;
  const int blocks = grad_blocks(rows, cols, isz);
  float *sums_g = (float*)workspace, *sums_s = sums ? (float*)((char*)workspace + need / 2) : nullptr;
  a.dgain = !dgain ? nullptr : blocks == 1 ? (float*)dgain : sums_g;
  a.dshift = !dshift ? nullptr : blocks == 1 ? (float*)dshift : sums_s;
  hipStream_t st = (hipStream_t)hip_stream;
  if (launch_layernorm_grad(a, blocks * layernorm_rows_per_block(rows, cols), (int)in, cols % 8 == 0, st) != hipSuccess)
    return ALCOP_ERR_LAUNCH;
  if (sums && blocks > 1) {
    TwoColumnSums s;
    int n = 0;
    if (dgain) s.of[n++] = ColumnSumArgs{sums_g, (float*)dgain, blocks, cols};
    if (dshift) s.of[n++] = ColumnSumArgs{sums_s, (float*)dshift, blocks, cols};
    if (n == 1) s.of[1] = s.of[0];
    if (launch_two_column_sums(s, n, st) != hipSuccess) return ALCOP_ERR_LAUNCH;
  }
  return ALCOP_OK;
}

}  // extern "C"
