// Rows as pieces of eight elements, spread over the threads of a launch.
#pragma once

#include <algorithm>

#include "element.h"

namespace gcn {

// Eight elements, as they lie in memory.
template <class T>
struct Raw8 {
  static constexpr int kParts = 8 / kPiece<T>;
  u4 part[kParts];
};

// Those at column f of a row of F (any alignment); zeros behind its end, and nothing read where
// F is at most f.
template <class T>
__device__ inline Raw8<T> load8(const T* row, int f, int F) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < Raw8<T>::kParts; ++i) r.part[i] = load_piece(row, f + i * kPiece<T>, F);
  return r;
}

template <class T>
__device__ inline void unpack8(const Raw8<T>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < Raw8<T>::kParts; ++i) {
    float p[kPiece<T>];
    unpack<T>(r.part[i], p);
#pragma unroll
    for (int e = 0; e < kPiece<T>; ++e) v[i * kPiece<T> + e] = p[e];
  }
}

// The part inside the row, each value rounded to nearest even.
template <class T>
__device__ inline void store8(T* row, int f, int F, const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < Raw8<T>::kParts; ++i) {
    float p[kPiece<T>];
#pragma unroll
    for (int e = 0; e < kPiece<T>; ++e) p[e] = v[i * kPiece<T> + e];
    if (f + i * kPiece<T> < F) store_piece<T>(row, f + i * kPiece<T>, F, p);
  }
}

// n rows of so many pieces, `tile` of them to a workgroup: a run of whole rows, or a part of a long
// one. A thread finds its piece's row by a multiplication.
struct RowTiles {
  uint32_t n, pieces;    // pieces of a row
  uint32_t rows, parts;  // rows of a workgroup, workgroups of a row
  uint32_t magic;        // ceil(2^32 / pieces): t magic / 2^32 = t / pieces for pieces > 1, t < 2^15
  int64_t blocks() const { return ((int64_t)n + rows - 1) / rows * parts; }
};

inline RowTiles row_tiles(int64_t n, int64_t pieces, int64_t tile) {
  RowTiles t;
  t.n = (uint32_t)n;
  t.pieces = (uint32_t)pieces;
  t.rows = (uint32_t)std::max<int64_t>(1, tile / pieces);
  t.parts = (uint32_t)ceil_div(pieces, tile);
  t.magic = (uint32_t)std::min<int64_t>(ceil_div(int64_t(1) << 32, pieces), 0xFFFFFFFF);
  return t;
}

// Piece t of the workgroup's tile; whether there is one.
__device__ inline bool locate(const RowTiles& a, uint32_t tile, uint32_t t, uint32_t* row,
                              uint32_t* piece) {
  const uint32_t r = a.pieces == 1 ? t : (a.rows > 1 ? (uint32_t)((uint64_t)t * a.magic >> 32) : 0);
  *row = blockIdx.x / a.parts * a.rows + r;
  *piece = blockIdx.x % a.parts * tile + t - r * a.pieces;
  return r < a.rows && *row < a.n && *piece < a.pieces;
}

}  // namespace gcn
