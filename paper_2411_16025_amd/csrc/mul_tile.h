// Operand tiles in LDS for the bf16 matrix instruction, and how they get there (gemm_grouped.hip,
// gemm_q8.hip).
#pragma once

#include <algorithm>

#include "element.h"

namespace gcn {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u2a __attribute__((ext_vector_type(2), aligned(2)));  // 8 bytes at any element
typedef Unaligned<bf16>::type u4u;  // 16 bytes at any element

#define GCN_GLOBAL __attribute__((address_space(1)))
#define GCN_LDS __attribute__((address_space(3)))

__device__ const u4 g_zeros = {0, 0, 0, 0};

// One operand's part of a stage: BK of the inner size by X rows of A (columns of B). KC: the
// inner size is contiguous in memory (A of NN and NT, B of NT): X lines of BK
// elements; else BK lines of X. A line is stored in 16-byte pieces, piece c at c ^ swz(line),
// so that the reads of neighbouring lines fall on different banks.
template <bool KC, int X, int BK>
struct Tile {
  static constexpr int kPieces = X * BK / 8;
  static constexpr int kPerLine = (KC ? BK : X) / 8;
  static constexpr int kBytes = kPieces * 16;
  __device__ static inline int swz(int line) {
    if constexpr (KC) return BK == 64 ? (line >> 1) & 7 : (line >> 2) & 3;
    return X >= 128 ? 4 * (line & 3) : (X == 64 ? 4 * ((line >> 1) & 1) : 0);
  }
  // What the lane reads of block blk (32 of X) and step (16 of BK): the 8 of the
  // inner size of operand row (lane % 32).
  __device__ static inline bf8 read(const char* base, int blk, int step, int lane) {
    if constexpr (KC) {
      const int line = lane & 31;
      const int at = line * (BK * 2) + (((lane >> 5) ^ swz(line)) * 16 ^ 32 * step);
      return *reinterpret_cast<const bf8*>(base + at + blk * 32 * BK * 2);
    } else {
      // the transposing read: of 16 lanes, lane i names 4 elements of line i / 4 and gets
      // element i of each of the 4 lines
      const int i = lane & 15, line = 8 * (lane >> 5) + (i >> 2);
      const int piece = 4 * blk + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
      const int at = line * (X * 2) + (piece ^ swz(line)) * 16 + (i & 1) * 8 + 16 * step * X * 2;
      const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (GCN_LDS s4*)(base + at));
      const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (GCN_LDS s4*)(base + at + 4 * X * 2));
      const s8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf8, v);
    }
  }
};

// The pieces of an operand that a thread brings to LDS: their offsets in memory from the
// operand's first element of a stage. DIRECT: rows start on 16 bytes and hold whole
// pieces, and the loads go to LDS themselves. Else through registers, without a branch between
// the loads: a piece that reaches over a row's end is read from 8 elements before the end
// on (rows have 8) and moved down when it is stored.
template <bool KC, int X, int BK, int NT, bool DIRECT>
struct Loader {
  using T = Tile<KC, X, BK>;
  static constexpr int kCount = T::kPieces / NT;
  static_assert(T::kPieces % NT == 0, "every thread has as many pieces");
  const bf16* base;   // the operand's element (first of X, inner 0)
  int64_t ld;
  int have;           // of X inside the matrix
  int64_t had;        // of the inner size, in the stage whose pieces are in v
  uint32_t off[kCount];
  u4 v[DIRECT ? 1 : kCount];

  __device__ static inline int line_of(int p) { return (int)(threadIdx.x + p * NT) / T::kPerLine; }
  __device__ static inline int element_of(int p) {  // of its line, a multiple of 8
    return 8 * (((int)(threadIdx.x + p * NT) % T::kPerLine) ^ T::swz(line_of(p)));
  }
  __device__ inline void init(const bf16* b, int64_t ld_, int have_) {
    base = b;
    ld = ld_;
    have = have_;
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      const int line = line_of(p), e = element_of(p);
      if constexpr (KC)
        off[p] = 2 * ((line < have ? line : have - 1) * (uint32_t)ld + e);
      else if constexpr (DIRECT)
        off[p] = 2 * (line * (uint32_t)ld + (e < have ? e : 0));
      else  // (from the first of X - 8, which may lie before the tile)
        off[p] = 2 * (line * (uint32_t)ld + (uint32_t)(std::min(e, have - 8) + 8));
    }
  }
  // Pieces of the stage whose inner range begins at k0 and has `left` elements.
  __device__ inline void load(char* lds, int64_t k0, int64_t left) {
    const char* at = reinterpret_cast<const char*>(KC ? base + k0 : base + k0 * ld);
    if constexpr (DIRECT) {
      const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int p = 0; p < kCount; ++p) {
        const char* q = at + off[p];
        if (left < BK && (KC ? element_of(p) : line_of(p)) >= left)
          q = reinterpret_cast<const char*>(&g_zeros);
        __builtin_amdgcn_global_load_lds((const GCN_GLOBAL void*)q,
                                         (GCN_LDS void*)(lds + (w * 64 + p * NT) * 16), 16, 0, 0);
      }
    } else {
      had = left;
      if (left <= 0) return;  // past the last stage
      if (!KC) at -= 16;
      if (left >= BK) {
#pragma unroll
        for (int p = 0; p < kCount; ++p)
          v[p] = *reinterpret_cast<const u4u*>(at + off[p]);
      } else {
#pragma unroll
        for (int p = 0; p < kCount; ++p) {
          const int over = KC ? element_of(p) - (int)left + 8 : line_of(p) - (int)left + 1;
          const char* q = at + off[p];
          if (over > 0) q -= KC ? 2 * (int64_t)over : 2 * over * ld;
          v[p] = *reinterpret_cast<const u4u*>(q);
        }
      }
    }
  }
  __device__ inline void store(char* lds) {
    if constexpr (!DIRECT) {
      const bool whole = had >= BK && (KC || have >= X);
#pragma unroll
      for (int p = 0; p < kCount; ++p) {
        u4 x = v[p];
        if (!whole) {
          const int64_t over = (KC ? element_of(p) - had : (int64_t)element_of(p) - have) + 8;
          x = move_down<bf16>(x, (int)std::min<int64_t>(8, std::max<int64_t>(0, over)));
          if (!KC && line_of(p) >= had) x = u4{0, 0, 0, 0};
        }
        *reinterpret_cast<u4*>(lds + (threadIdx.x + p * NT) * 16) = x;
      }
    }
  }
};

// The loads to LDS are done, but for the last N of a thread, for all wavefronts.
template <int N = 0>
__device__ inline void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4 << 14));  // vector memory
  __syncthreads();
}

}  // namespace
}  // namespace gcn
