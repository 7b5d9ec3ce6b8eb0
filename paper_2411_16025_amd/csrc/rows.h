// Rows as pieces of four or eight elements, spread over the threads of a launch.
#pragma once

#include <algorithm>

#include "element.h"

namespace gcn {

// N elements (4 or 8), as they lie in memory.
template <class T, int N>
struct Raw {
  static constexpr int kBytes = N * (int)sizeof(T);  // 8, 16 or 32
  u4 part[(kBytes + 15) / 16];
};

// Those at column f of a row of F (any alignment); zeros behind its end, and nothing read where
// F is at most f.
template <class T, int N>
__device__ inline Raw<T, N> load_raw(const T* row, int f, int F) {
  Raw<T, N> r;
  if constexpr (Raw<T, N>::kBytes == 8) {
    typedef uint32_t half __attribute__((ext_vector_type(2), aligned(2)));
    r.part[0] = u4{0, 0, 0, 0};
    if (f + 4 <= F) {
      const half h = *reinterpret_cast<const half*>(row + f);
      r.part[0][0] = h[0];
      r.part[0][1] = h[1];
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (f + e < F)
          r.part[0][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[f + e] << (16 * (e & 1));
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / kPiece<T>; ++i) r.part[i] = load_piece(row, f + i * kPiece<T>, F);
  }
  return r;
}

template <class T, int N>
__device__ inline void unpack_raw(const Raw<T, N>& r, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < (N + kPiece<T> - 1) / kPiece<T>; ++i) {
    float p[kPiece<T>];
    unpack<T>(r.part[i], p);
#pragma unroll
    for (int e = 0; e < kPiece<T>; ++e)
      if (i * kPiece<T> + e < N) v[i * kPiece<T> + e] = p[e];
  }
}

// The part inside the row, each value rounded to nearest even; N elements are 16 or 32 bytes.
template <class T, int N>
__device__ inline void store_raw(T* row, int f, int F, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / kPiece<T>; ++i) {
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
