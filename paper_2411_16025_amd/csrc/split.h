// fp32 numbers as three bf16 parts, and tiles of sums that are not finite (gemm_split.hip, gemm_q8.hip).
#pragma once

#include "common.h"

namespace gcn {
namespace {

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));  // 4-byte aligned 16-byte load
typedef float f16 __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr float kUp = 0x1p24f, kDown = 0x1p-48f;  // of an operand, of a sum (gemm_split.hip)

// The parts of two neighbouring values, each pair packed in 32 bits.
__device__ inline void split2(float x0, float x1, uint32_t& h, uint32_t& m, uint32_t& l) {
  const f2 x = {x0, x1};
  h = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf2));
  const f2 r = {x0 - __uint_as_float(h << 16), x1 - __uint_as_float(h & 0xFFFF0000u)};
  m = __builtin_bit_cast(uint32_t, __builtin_convertvector(r, bf2));
  const f2 q = {r.x - __uint_as_float(m << 16), r.y - __uint_as_float(m & 0xFFFF0000u)};
  l = __builtin_bit_cast(uint32_t, __builtin_convertvector(q, bf2));
}

__device__ inline void split8(const float* x, u4* out) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t h, m, l;
    split2(x[2 * j], x[2 * j + 1], h, m, l);
    out[0][j] = h;
    out[1][j] = m;
    out[2][j] = l;
  }
}

// Operand layout of the instruction: lane l holds A[l % 32][8 (l / 32) + j]
// and B[8 (l / 32) + j][l % 32], j = 0 .. 7; result element e of lane l is
// C[(e % 4) + 8 (e / 4) + 4 (l / 32)][l % 32].
__device__ inline int result_row(int e, int lane) {
  return (e & 3) + 8 * (e >> 2) + 4 * (lane >> 5);
}

// Whether a sum of the wavefront is not finite.
template <int RBW, int NBW>
__device__ inline bool not_finite(const f16 (*acc)[NBW]) {
  float bad = 0.f;  // NaN once a sum is not finite
#pragma unroll
  for (int i = 0; i < RBW; ++i)
#pragma unroll
    for (int j = 0; j < NBW; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) bad = __builtin_fmaf(acc[i][j][e], 0.f, bad);
  return __any(bad != bad);
}

// The wavefront's sums over [k0, k1) again on the fp32 matrix instruction, the
// operands from global memory. Lane l holds A[l % 32][k] and B[k][l % 32], k the
// same for both in each half of the wavefront: four k of each half are fetched
// at a time by load(k, a, b), zeros from k1 on. (Element by element, a product of
// 32,768 x 256 x 516 whose operands are NaN took 8.8 ms; 0.32 here, 0.09 with
// finite ones.)
template <int RBW, int NBW, class Load>
__device__ inline void mul_again(int64_t k0, int64_t k1, Load load, f16 (*acc)[NBW]) {
#pragma unroll
  for (int i = 0; i < RBW; ++i)
#pragma unroll
    for (int j = 0; j < NBW; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
#pragma unroll 1
  for (int64_t k = k0; k < k1; k += 8) {
    float x[RBW][4], y[NBW][4];
    load(k + 4 * ((threadIdx.x >> 5) & 1), x, y);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < RBW; ++i)
#pragma unroll
        for (int j = 0; j < NBW; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i][q], y[j][q], acc[i][j], 0, 0, 0);
  }
}

}  // namespace
}  // namespace gcn
