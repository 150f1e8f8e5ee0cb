// Products grouped by expert: rows sorted by group, each group's rows times weights of its own, and the gradients.
//
//     rows offsets[g] .. offsets[g + 1] - 1:   Z = alpha sa sw A W_g + bias_g,  C = act(Z)
//     dA = alpha dZ W_g^T,   dW_g = alpha A_g^T dZ_g,   dbias_g = sum over the group's rows of dZ
//
// How many rows a group has is known on the device only.  A launch has as many blocks as the rows could make tiles
// (a partial tile for each group at most), and every wave finds its own tile: a lane per group reads two offsets, the groups' tiles are
// summed up across the lanes, and the lane whose group holds the block's tile passes it on, all ahead of the first load; a kernel that
// writes a table would be a launch more.  Blocks beyond the last tile leave at once.  Tiles of a group are neighbours, and the eight
// XCDs get equal runs of them, so that a group's weights are read into one or two L2s (tiles that their groups do not fill put last, to even
// out the end, read the weights again: 54 groups of 300 rows, 4096 x 2048, 532 us in place of 436).
// From there on a tile is that of a product of its own: the loops and the epilogue are those of the linear layers.
//
// What bounds them.  16384 rows in one group, 4096 x 2048 bf16 with SiLU and pre, take 267 us as the linear layer does (1.03
// PFLOP/s); in 16 even groups 293, as 268 MB of weights come from memory in place of 17; in 16 uneven ones 336: tiles that their groups
// do not fill, and the turn of the card that the last ones begin.  32 rows over 32 groups, 2048 x 1024: the weights' bytes, 11 us.
//
// Offsets are clamped to 0 .. rows and to rising order where they are read: what they hold decides what is computed, never
// whether an access is in bounds.
#pragma once
#include "alcop_rows.hip.h"

namespace alcop {

template <class B>
struct Placed : B {
  int tile_m, tile_n;
};
template <class B>
__device__ __forceinline__ void tile_of_block(const Placed<B>& p, int, int& tm, int& tn)
{
  tm = p.tile_m;
  tn = p.tile_n;
}

struct GroupList {
  const int* offsets;          // groups + 1 numbers
  int groups, rows;
};

// ---- the tile of a block ---------------------------------------------------------------------------------
// The rows of group 64 c + lane; its tiles of 2^shift rows, the last one maybe not full, times `width`; those of the lanes before it and
// of all lanes.
struct GroupLane {
  int first, rows, tiles, before, total;
};
template <class HW>
__device__ __forceinline__ GroupLane group_lane(const GroupList& l, int c, int shift, int width)
{
  const int lane = HW::lane_id(), g = c * 64 + lane;
  GroupLane r = {0, 0, 0, 0, 0};
  if (g < l.groups) {
    const int a = (int)HW::global_load_u32(l.offsets + g), b = (int)HW::global_load_u32(l.offsets + g + 1);
    r.first = a < 0 ? 0 : a > l.rows ? l.rows : a;
    const int end = b > l.rows ? l.rows : b;
    r.rows = end > r.first ? end - r.first : 0;
    r.tiles = (int)(((uint32_t)r.rows + (1u << shift) - 1) >> shift) * width;
  }
  const int upto = (int)HW::scan_lanes((uint32_t)r.tiles);
  r.before = upto - r.tiles;
  r.total = (int)HW::read_lane((uint32_t)upto, 63);
  return r;
}

struct GroupTile {
  int group, first, rows, tile;      // tile: among the group's own
};
template <class HW>
__device__ __forceinline__ void take_lane(const GroupLane& g, int c, int lane, GroupTile& t)
{
  t.group = c * 64 + lane;
  t.first = (int)HW::read_lane((uint32_t)g.first, lane);
  t.rows = (int)HW::read_lane((uint32_t)g.rows, lane);
}

// Run `lid` of all groups' runs of 2^shift rows, the last of each shorter.  False if there are not so many.
template <class HW>
__device__ __forceinline__ bool group_run(const GroupList& l, int shift, int lid, GroupTile& t)
{
  const int chunks = (l.groups + 63) / 64;
  for (int c = 0; c < chunks; c++) {
    const GroupLane g = group_lane<HW>(l, c, shift, 1);
    const uint64_t mine = HW::ballot(lid >= g.before && lid - g.before < g.tiles);
    if (mine) {
      const int lane = __builtin_ctzll(mine);
      take_lane<HW>(g, c, lane, t);
      t.tile = lid - (int)HW::read_lane((uint32_t)g.before, lane);
      return true;
    }
    lid -= g.total;
  }
  return false;
}
// The rows of a group, its runs (returned) and those ahead of it (in t.tile).
template <class HW>
__device__ __forceinline__ int group_runs(const GroupList& l, int shift, int group, GroupTile& t)
{
  int ahead = 0, c = 0;
  GroupLane g = group_lane<HW>(l, 0, shift, 1);
  for (; c < group / 64; c++) {
    ahead += g.total;
    g = group_lane<HW>(l, c + 1, shift, 1);
  }
  const int lane = group - c * 64;
  take_lane<HW>(g, c, lane, t);
  t.tile = ahead + (int)HW::read_lane((uint32_t)g.before, lane);
  return (int)HW::read_lane((uint32_t)g.tiles, lane);
}

// Item `lid` of `all` that are dealt to the XCDs in equal runs (blocks go to the XCDs in turn).
__device__ __forceinline__ int spread_out(int lid, int all)
{
  const int x = lid & 7, rem8 = all & 7;
  return x * (all >> 3) + (x < rem8 ? x : rem8) + (lid >> 3);
}

// The tile of block `lid` among those of `width` strips of columns: the tiles of a group are neighbours, also the ones that it does not
// fill, so that its weights are read once.  False if there are not so many.
// quarter: what is left behind the last whole turn of the card, up to QUARTERED tiles, is dealt out in quarters of a tile, 0 .. 3; -1: a
// whole one.
constexpr int CARD = 256;            // compute units, of which each has one of the large tiles at a time
template <int QUARTERED, class HW>
__device__ __forceinline__ bool group_tile(const GroupList& l, int shift, int width, int lid, GroupTile& t, int& quarter)
{
  const int chunks = (l.groups + 63) / 64;
  GroupLane g = group_lane<HW>(l, 0, shift, width);
  int all = g.total;
  for (int c = 1; c < chunks; c++) {
    // a launch has fewer than 2^24 blocks, 64 groups so fewer than 2^30 tiles; all could be more where offsets do not rise
    const int more = group_lane<HW>(l, c, shift, width).total, most = 1 << 30;
    all = all > most - more ? most : all + more;
  }
  quarter = -1;
  const int whole = all % CARD <= QUARTERED ? all / CARD * CARD : all;
  if (lid < whole) {
    lid = spread_out(lid, whole);
  } else {
    if (lid - whole >= 4 * (all - whole)) return false;
    lid = spread_out(lid - whole, 4 * (all - whole));
    quarter = lid & 3;
    lid = whole + (lid >> 2);
  }
  for (int c = 0; c < chunks; c++) {
    if (c) g = group_lane<HW>(l, c, shift, width);
    const uint64_t mine = HW::ballot(lid >= g.before && lid - g.before < g.tiles);
    if (mine) {
      const int lane = __builtin_ctzll(mine);
      take_lane<HW>(g, c, lane, t);
      t.tile = lid - (int)HW::read_lane((uint32_t)g.before, lane);
      return true;
    }
    lid -= g.total;
  }
  return false;
}

constexpr int log2_of(int v)
{
  int s = 0;
  while ((1 << s) < v) s++;
  return s;
}

// ---- C = act(alpha sa sw A W_g + bias_g) ---------------------------------------------------------------------
struct GroupedArgs {
  LinearArgs l;                // M: all rows
  const int* offsets;
  int groups;
  long strideW;                // between the weights of two groups, 16-bit units
};

template <class C, int QUARTERED, class HW>
__device__ __forceinline__ bool place_group(const GroupedArgs& a, Placed<LinearParams>& p, int& quarter)
{
  (LinearParams&)p = expand_linear<C>(a.l);
  GroupTile t;
  if (!group_tile<QUARTERED, HW>(GroupList{a.offsets, a.groups, a.l.M}, log2_of(C::BM), p.ntn, (int)HW::block_x(), t, quarter)) return false;
  const int osz = p.out_dtype == 2 ? 4 : 2;
  p.M = p.Mv = t.rows;
  p.ntm = (t.rows + C::BM - 1) / C::BM;
  p.group_m = p.ntm < 8 ? p.ntm : 8;
  tile_in_bands(p, t.tile, p.tile_m, p.tile_n);
  p.A = (const char*)p.A + (long)t.first * p.lda * 2;
  p.B = (const char*)p.B + (long)t.group * a.strideW * 2;
  p.C = (char*)p.C + (long)t.first * p.ldc * osz;
  if (p.pre) p.pre = (char*)p.pre + (long)t.first * p.ldp * osz;
  if (p.bias) p.bias += (long)t.group * p.N;
  if (p.sw) p.sw += (long)t.group * p.N;
  if (p.sa) p.sa += t.first;
  return true;
}

template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_grouped_tile(const GroupedArgs a)
{
  Placed<LinearParams> p;
  int quarter;
  if (place_group<C, 0, HW>(a, p, quarter)) mainloop_body<C, HW>(p);
}
template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_grouped_ksplit(const GroupedArgs a)
{
  Placed<LinearParams> p;
  int quarter;
  if (place_group<C, 0, HW>(a, p, quarter)) ksplit_body<C, HW>(p);
}
// Large tiles C, of which a compute unit has one at a time, and quarters Q of them behind the last whole turn of the card: how many
// tiles uneven groups make is as good as never a multiple of its units, and a turn that a few tiles begin takes as long as one of all.
// Of 256x256 tiles up to 128 are quartered (two turns of quarters), of 256x128, whose quarters load more for each product, up to 64 (one turn).
// us, bf16, with none, 64, 128, 192 and all quartered:
//   256x256  16384 x 4096 x 2048 in 16 groups 344, 345, 336, 336, 336; 4000 rows in 2 96.8, 78.7, 77.6, 78.4, 78.1; 2500 in 5 66.1,
//            65.7, 65.7, 72.9, 80.3; 8192 x 2048 x 2048 in 16 groups, gradients, 223, 213, 208, 207, 207, of 5000 in 7 137, 138, 137, 145, 145
//   256x128  the first 344, 343, 341, 342, 341; 4000 rows in 2 91.9, 82.8, 83.2, 83.1, 82.9; 2500 in 5 70.5, 71.0, 73.9, 81.6, 82.0;
//            the gradients 210, 210, 212, 226, 224
template <class C>
constexpr int quartered()
{
  return C::BN >= 256 ? CARD / 2 : CARD / 4;
}
template <class C, class Q, class HW>
__global__ void __launch_bounds__(C::NT) alcop_grouped_quarters(const GroupedArgs a)
{
  static_assert(C::NT == Q::NT && 2 * Q::BM == C::BM && 2 * Q::BN == C::BN, "a quarter of the tile, as many waves");
  Placed<LinearParams> p;
  int quarter;
  if (!place_group<C, quartered<C>(), HW>(a, p, quarter)) return;
  if (quarter < 0) {
    mainloop_body<C, HW>(p);
    return;
  }
  p.tile_m = 2 * p.tile_m + (quarter & 1);
  p.tile_n = 2 * p.tile_n + (quarter >> 1);
  if (p.tile_m * Q::BM < p.M && p.tile_n * Q::BN < p.N) mainloop_body<Q, HW>(p);
}

// ---- dW_g = alpha P_g^T Q_g, P and Q stored with the rows' axis first ------------------------------------------
struct GroupedGradArgs {
  const void *P, *Q;
  void* dW;
  const int* offsets;
  int groups, rows, M, N, ldp, ldq, ldw;
  long strideW;                // elements of dW
  float alpha;
  int out;
};

template <class C, class HW>
__global__ void __launch_bounds__(C::NT) alcop_grouped_grad(const GroupedGradArgs a)
{
  Placed<Params> p = {};
  p.M = p.Mv = a.M;
  p.N = p.Nv = a.N;
  p.lda = a.ldp;
  p.ldb = a.ldq;
  p.ldc = a.ldw;
  p.alpha = a.alpha;
  p.out_dtype = a.out;
  p.ntm = (p.M + C::BM - 1) / C::BM;
  p.ntn = (p.N + C::BN - 1) / C::BN;
  p.group_m = p.ntm < 4 ? p.ntm : 4;
  // all groups have as many tiles, which take as long as the group has rows: every XCD gets a run of each group's, not groups of its own
  // (8192 rows in 16 uneven groups, 2048 x 2048, the whole backward pass: 227 us with two groups to an XCD, 218 so, 212 with bands of four
  // rows of tiles, of which a run needs fewer panels; in 14 groups of 600 rows 202, 211 and 211)
  const int per = p.ntm * p.ntn, group = (int)HW::block_x() / per, r = group * per + spread_out((int)HW::block_x() - group * per, per);
  tile_in_bands(p, r - group * per, p.tile_m, p.tile_n);
  GroupTile t;
  t.first = (int)HW::read_lane(HW::global_load_u32(a.offsets + group), 0);
  int end = (int)HW::read_lane(HW::global_load_u32(a.offsets + group + 1), 0);
  t.first = t.first < 0 ? 0 : t.first > a.rows ? a.rows : t.first;
  end = end > a.rows ? a.rows : end;
  const int osz = a.out == 2 ? 4 : 2;
  p.C = (char*)a.dW + (long)group * a.strideW * osz;
  if (end <= t.first) {
    // no rows: the gradient is 0
    const int per_row = C::BN / 8, tid = HW::wave_id() * 64 + HW::lane_id();
#pragma unroll 1
    for (int i = tid; i < C::BM * per_row; i += C::NT) {
      const int m = p.tile_m * C::BM + i / per_row, n = p.tile_n * C::BN + i % per_row * 8;
      if (m < p.M && n < p.N) {
        char* at = (char*)p.C + ((long)m * p.ldc + n) * osz;
        HW::global_store16(at, u32x4{0, 0, 0, 0});
        if (osz == 4) HW::global_store16(at + 16, u32x4{0, 0, 0, 0});
      }
    }
    return;
  }
  p.K = end - t.first;                      // rows past it lie beyond both descriptors
  p.A = (const char*)a.P + (long)t.first * p.lda * 2;
  p.B = (const char*)a.Q + (long)t.first * p.ldb * 2;
  mainloop_body<C, HW>(p);
}

// ---- dZ = dC act'(Z) and its sums by group -------------------------------------------------------------------
// Blocks y have up to 2^shift rows of one group; the sums of a group's blocks are neighbours.
struct GroupedActGradArgs {
  ActGradArgs a;
  GroupList l;
  int shift;
};
template <int DT, class HW>
__global__ void __launch_bounds__(256) alcop_grouped_act_grad(const GroupedActGradArgs p)
{
  GroupTile t;
  if (!group_run<HW>(p.l, p.shift, (int)HW::block_y(), t)) return;
  const long r0 = t.first + ((long)t.tile << p.shift), r1 = r0 + (1l << p.shift), end = (long)t.first + t.rows;
  act_grad<DT, HW>(p.a, r0, r1 < end ? r1 : end, (long)HW::block_y());
}
// out[g][j]: the sum over the partial sums of group g
struct GroupedSumArgs {
  ColumnSumArgs s;
  GroupList l;
  int shift;
};
constexpr int GROUP_SUM_THREADS = 256;      // a group has few of them
template <class HW>
__global__ void __launch_bounds__(GROUP_SUM_THREADS) alcop_grouped_sums(const GroupedSumArgs p)
{
  const int group = (int)HW::block_y();
  GroupTile t;
  ColumnSumArgs s = p.s;
  const int count = group_runs<HW>(p.l, p.shift, group, t);
  // offsets that do not rise could count more blocks than there are
  s.count = t.tile + count <= p.s.count ? count : t.tile < p.s.count ? p.s.count - t.tile : 0;
  s.partial += (long)t.tile * s.cols;
  s.out += (long)group * s.cols;
  column_sums<HW, GROUP_SUM_THREADS>(s);
}

// the tiles of dW
template <int DT, int BM, int BN, int BK, int WM, int WN, int S, int R, int F>
using GradCfg = KCfg<DT, BM, BN, BK, WM, WN, S, R, F, 0, 0, 1>;

}  // namespace alcop
