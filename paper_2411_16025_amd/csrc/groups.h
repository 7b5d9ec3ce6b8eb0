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
                                 int64_t stride_w, hipStream_t stream);
// bf16 products (gemm_grouped.hip): C = A op(B_g), or C_g = A_g^T B_g, C bf16 or fp32.
bool gemm_grouped_bf16_takes(int64_t N, int64_t K, int64_t lda, int64_t ldb);
gcn_status gemm_grouped_bf16(int op, const Groups& g, int64_t N, int64_t K, const void* A,
                             int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc,
                             bool c_bf16, int64_t stride_w, hipStream_t stream);
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

// Tiles of R rows of all groups, counted (each group at least `least` tiles). The whole wavefront.
__device__ inline int group_tiles_of(const Groups& a, int g, int R, int least) {
  const int64_t rows = group_offset(a, g + 1) - group_offset(a, g);
  const int tiles = rows > 0 ? (int)((rows + R - 1) / R) : 0;
  return tiles > least ? tiles : least;
}

// With up to this many groups a workgroup counts the tiles before its own, so that no
// slots are empty and the tiles divide evenly among the XCDs (32,768 x 4096 x 2048, one
// group: 129 slots for 128 tiles, 537 us in runs of slots, 496 so); of more groups the
// slots' search reads less.
constexpr int kCountedGroups = 1024;

__device__ inline int wave_inclusive(int v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int u = __shfl_up(v, off, 64);
    if ((int)(threadIdx.x & 63) >= off) v += u;
  }
  return v;
}

// A tile's group and rows; beg >= end: nothing (first: the group's first tile).
struct GroupTile {
  int g;
  int64_t beg, end, first;  // the tile's first row, the group's end, the group's first row
};

// The last group that begins (begins(g), true up to some group) and its rows, beg = first:
// every lane of the wavefront asks for one group of the range left.
template <class Begins>
__device__ inline GroupTile group_tile_from(const Groups& a, Begins begins) {
  int lo = 0, len = a.n;
  while (len > 1) {
    const int step = (len + 63) / 64;
    const int g = lo + (int)(threadIdx.x & 63) * step;
    const uint64_t hit = __ballot(g < lo + len && begins(g));
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
  GroupTile t = group_tile_from(a, [&](int g) { return group_offset(a, g) / R + g <= slot; });
  const int64_t tile = slot - (t.first / R + t.g);
  t.beg = tile < 0 ? t.end : t.first + tile * R;
  return t;
}

// The number of tiles; before: of the groups before this lane's (a.n / 64 of them, rounded up).
__device__ inline int group_tiles(const Groups& a, int R, int least, int* before) {
  const int per = (a.n + 63) / 64, lane = threadIdx.x & 63;
  int mine = 0;
  for (int i = 0; i < per; ++i)
    if (lane * per + i < a.n) mine += group_tiles_of(a, lane * per + i, R, least);
  const int upto = wave_inclusive(mine);
  *before = upto - mine;
  return __builtin_amdgcn_readlane(upto, 63);
}

// Tile t of the counted ones.
__device__ inline GroupTile counted_tile(const Groups& a, int t, int R, int least, int before) {
  const int per = (a.n + 63) / 64, lane = threadIdx.x & 63;
  // the last lane whose groups begin at or before t (those of the lanes behind it begin later)
  const uint64_t at = __ballot(lane * per < a.n && before <= t);
  const int l = 63 - __clzll((long long)at);
  t -= __builtin_amdgcn_readlane(before, l);
  int g = l * per;
  if (per > 1) {
    const int mine = lane < per && g + lane < a.n ? group_tiles_of(a, g + lane, R, least) : 0;
    const int first = wave_inclusive(mine) - mine;
    const uint64_t in = __ballot(mine > 0 && first <= t);
    const int j = in ? 63 - __clzll((long long)in) : 0;
    t -= __builtin_amdgcn_readlane(first, j);
    g += j;
  }
  GroupTile r;
  r.g = __builtin_amdgcn_readfirstlane(g);
  r.first = group_offset(a, r.g);
  r.end = group_offset(a, r.g + 1);
  r.beg = r.first + (int64_t)t * R;
  return r;
}
#endif

}  // namespace gcn
