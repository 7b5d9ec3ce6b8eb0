// Sums over the lanes that hold a row, and 1 / sqrt in double.
#pragma once

#include "common.h"

namespace gcn {

// A slot is the G neighbouring lanes that hold one row. Its butterfly pairs
// lanes within the slot: the partner at distance 1 and 2 comes from a quad permutation, at 4 and 8 from the mirror of the
// half row and of the row (after the earlier steps every lane of a quad,
// then of a half row, holds the same value, so the mirror partner carries
// the same operand as lane ^ 4 or lane ^ 8), further ones from a wavefront
// shuffle. The DPP moves need no LDS round trip; the sums are those of the
// xor butterfly, bit for bit.
template <int CTRL>
__device__ inline int dpp_mov(int x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xF, 0xF, false);
}

template <int OFF>
__device__ inline int slot_partner(int x) {
  if constexpr (OFF == 1) return dpp_mov<0xB1>(x);   // quad_perm [1, 0, 3, 2]
  if constexpr (OFF == 2) return dpp_mov<0x4E>(x);   // quad_perm [2, 3, 0, 1]
  if constexpr (OFF == 4) return dpp_mov<0x141>(x);  // row_half_mirror
  if constexpr (OFF == 8) return dpp_mov<0x140>(x);  // row_mirror
  return __shfl_xor(x, OFF, 64);
}

template <int OFF>
__device__ inline float slot_partner(float v) {
  return __int_as_float(slot_partner<OFF>(__float_as_int(v)));
}

template <int OFF>
__device__ inline double slot_partner(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = slot_partner<OFF>((int)b);
  const int hi = slot_partner<OFF>((int)(b >> 32));
  return __longlong_as_double((long long)(((unsigned long long)(unsigned)hi << 32) | (unsigned)lo));
}

template <int G, int OFF = 1, class V>
__device__ inline V slot_sum(V v) {
  if constexpr (OFF < G) {
    v += slot_partner<OFF>(v);
    return slot_sum<G, 2 * OFF>(v);
  } else {
    return v;
  }
}

template <int G, int OFF = 1>
__device__ inline void slot_minmax(float& mn, float& mx) {
  if constexpr (OFF < G) {
    mn = fminf(mn, slot_partner<OFF>(mn));
    mx = fmaxf(mx, slot_partner<OFF>(mx));
    slot_minmax<G, 2 * OFF>(mn, mx);
  }
}

// 1 / sqrt(x) for finite x > 0: the hardware estimate refined by two Newton
// steps on the residual e = 1 - x r^2 (r += r e / 2; each step squares the
// relative error), a few ulps of double from the quotient of the correctly
// rounded square root. The normalized values are rounded to fp32 afterwards,
// so such an ulp decides a value only when its exact product lies within
// about 2^-50 of a rounding boundary of fp32.
__device__ inline double inv_sqrt(double x) {
  double r = __builtin_amdgcn_rsq(x);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const double e = __builtin_fma(-x * r, r, 1.0);
    r = __builtin_fma(0.5 * r, e, r);
  }
  return r;
}

}  // namespace gcn
