// Rows sorted by group, as kernels take them (gcn_gemm_grouped).
//
// The groups' sizes are known on the device only. So a launch covers every tile
// that any offsets could need, and a workgroup finds its own: with R rows per
// tile, the tiles of group g take the slots from offsets[g] / R + g on. Its rows
// need at most offsets[g + 1] / R - offsets[g] / R + 1 tiles, so the next group
// begins behind them, all groups end before rows / R + n_groups, and the group of
// a slot is found by comparing, without sums over the groups before it.
#pragma once

#include "element.h"
#include "scratch.h"

namespace gcn {

struct Groups {
  int n;
  const int64_t* offsets;  // [n + 1]
  int64_t rows;
};

inline int64_t group_slots(const Groups& g, int64_t R) { return g.rows / R + g.n; }

// The grouped products on the bf16 matrix cores with three-part operands
// (gemm_split.hip). C [rows x N] = A [rows x K] op(B_g), B_g of group g at
// B + g stride_w; takes: whether sizes and strides fit the kernel.
bool gemm_split_grouped_takes(int op, int64_t N, int64_t K, int64_t lda, int64_t ldb, int64_t ldc);
gcn_status gemm_split_grouped(int op, const Groups& g, int64_t N, int64_t K, const float* A,
                              int64_t lda, const float* B, int64_t ldb, int64_t stride_w, float* C,
                              int64_t ldc, hipStream_t stream);
// C_g [K x N] = A_g^T B_g, C_g at C + g stride_w.
gcn_status gemm_split_tn_grouped(const Groups& g, int64_t N, int64_t K, const float* A, int64_t lda,
                                 const float* B, int64_t ldb, float* C, int64_t ldc,
                                 int64_t stride_w, Scratch* scratch, hipStream_t stream);
// bf16 products (gemm_grouped.hip): C = A op(B_g), or C_g = A_g^T B_g, C bf16 or fp32.
bool gemm_grouped_bf16_takes(int64_t N, int64_t K, int64_t lda, int64_t ldb);
gcn_status gemm_grouped_bf16(int op, const Groups& g, int64_t N, int64_t K, const void* A,
                             int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc,
                             bool c_bf16, int64_t stride_w, Scratch* scratch, hipStream_t stream);
// C_g += the partial sums of the chunks behind the first one of group g, in their
// order; chunks of `split` rows, that of slot s at part + (s - g - 1) K N.
gcn_status sum_group_partials(const Groups& g, int64_t split, int64_t K, int64_t N,
                              const float* part, float* C, int64_t ldc, int64_t stride_w,
                              hipStream_t stream);

#ifdef __HIPCC__
// An offset, inside [0, rows] whatever the array holds.
__device__ inline int64_t group_offset(const Groups& a, int g) {
  const int64_t o = a.offsets[g];
  return o < 0 ? 0 : (o > a.rows ? a.rows : o);
}

// Tiles of R rows that a group of so many rows has, at least `least`.
__device__ inline int tiles_of(int64_t rows, int R, int least) {
  const int tiles = rows > 0 ? (int)((rows + R - 1) / R) : 0;
  return tiles > least ? tiles : least;
}

// With up to this many groups a workgroup counts the tiles before its own, so that no
// slots are empty and the tiles divide evenly among the XCDs (32,768 x 4096 x 2048, one
// group: 129 slots for 128 tiles, 537 us in runs of slots, 496 so); of more groups the
// slots' search reads less.
constexpr int kCountedGroups = 1024;

// Sums over the lanes up to each one (register moves: within rows of 16, then the last lane of a
// row to the next row, of two rows to the next two).
__device__ inline int wave_inclusive(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 to rows 2 and 3
  return v;
}

__device__ inline int64_t lane_value(int64_t v, int lane) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, lane) |
         (int64_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32;
}

__device__ inline int64_t uniform(int64_t v) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) |
         (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
}

// A tile's group and rows; beg >= end: nothing (first: the group's first tile).
struct GroupTile {
  int g;
  int64_t beg, end, first;  // the tile's first row, the group's end, the group's first row
};

// The last group that begins (begins(g, its offset), true up to some group) and its rows, beg = first:
// every lane of the wavefront asks for one group of the range left.
template <class Begins>
__device__ inline GroupTile group_tile_from(const Groups& a, Begins begins) {
  int lo = 0, len = a.n;
  while (len > 1) {
    const int step = (len + 63) / 64;
    const int g = lo + (int)(threadIdx.x & 63) * step;
    const uint64_t hit = __ballot(g < lo + len && begins(g, group_offset(a, g)));
    const int last = hit ? 63 - __clzll((long long)hit) : 0;
    len = min(step, len - last * step);
    lo += last * step;
  }
  GroupTile t;
  t.g = __builtin_amdgcn_readfirstlane(lo);
  t.beg = t.first = group_offset(a, t.g);
  t.end = group_offset(a, t.g + 1);
  return t;
}

// The tile of a slot.
__device__ inline GroupTile group_tile(const Groups& a, int64_t slot, int R) {
  GroupTile t = group_tile_from(a, [&](int g, int64_t o) { return o / R + g <= slot; });
  const int64_t tile = slot - (t.first / R + t.g);
  t.beg = tile < 0 ? t.end : t.first + tile * R;
  return t;
}

// The tiles of all groups, counted by a wavefront; each lane has a.n / 64 groups, rounded up.
struct TileCount {
  int total, before;   // of the groups before the lane's own
  int64_t first, end;  // the lane's group, where it has one
};

__device__ inline TileCount count_tiles(const Groups& a, int R, int least) {
  const int per = (a.n + 63) / 64, lane = threadIdx.x & 63;
  TileCount c{0, 0, 0, 0};
  int mine = 0;
  for (int i = 0; i < per; ++i)
    if (lane * per + i < a.n) {
      c.first = group_offset(a, lane * per + i);
      c.end = group_offset(a, lane * per + i + 1);
      mine += tiles_of(c.end - c.first, R, least);
    }
  // All groups' tiles are fewer than 2^24 + n (R >= 128, or few rows); of offsets that decrease, whose
  // groups overlap, no more are counted than an int holds.
  mine = min(mine, (1 << 25) - 1);
  const int upto = wave_inclusive(mine);
  c.before = upto - mine;
  c.total = __builtin_amdgcn_readlane(upto, 63);
  return c;
}

// Tile t of the counted ones.
__device__ inline GroupTile counted_tile(const Groups& a, const TileCount& c, int t, int R,
                                         int least) {
  const int per = (a.n + 63) / 64, lane = threadIdx.x & 63;
  // the last lane whose groups begin at or before t (those of the lanes behind it begin later)
  const uint64_t at = __ballot(lane * per < a.n && c.before <= t);
  const int l = 63 - __clzll((long long)at);
  t -= __builtin_amdgcn_readlane(c.before, l);
  GroupTile r;
  if (per == 1) {
    r.g = l;
    r.first = lane_value(c.first, l);
    r.end = lane_value(c.end, l);
  } else {
    const int g = l * per;
    int mine = 0;
    if (lane < per && g + lane < a.n)
      mine = tiles_of(group_offset(a, g + lane + 1) - group_offset(a, g + lane), R, least);
    const int first = wave_inclusive(mine) - mine;
    const uint64_t in = __ballot(mine > 0 && first <= t);
    const int j = in ? 63 - __clzll((long long)in) : 0;
    t -= __builtin_amdgcn_readlane(first, j);
    r.g = __builtin_amdgcn_readfirstlane(g + j);
    r.first = uniform(group_offset(a, r.g));
    r.end = uniform(group_offset(a, r.g + 1));
  }
  r.beg = r.first + (int64_t)t * R;
  return r;
}
#endif

}  // namespace gcn
