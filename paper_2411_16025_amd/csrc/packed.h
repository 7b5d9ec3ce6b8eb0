// Rows in 8 bits: int8 codes, and for each 32 columns of a row a scale byte (gcn_pack8).
#pragma once

#include "element.h"

namespace gcn {

typedef uint32_t u2b __attribute__((ext_vector_type(2), aligned(1)));  // 8 bytes anywhere

constexpr uint32_t kNoScale = 255;  // of 32 columns with an infinity or NaN

// The scale byte of 32 columns whose largest magnitude has these bits: e + 127, e the least of
// [-126, 121] with top <= 127 2^e. 127 is 1.984375 2^6: the exponent less 6, and one more where
// the mantissa is above that.
__device__ inline uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return kNoScale;
  const int b = (int)(top >> 23) - 6 + ((top & 0x7FFFFFu) > 0x7E0000u);
  return (uint32_t)min(max(b, 1), 248);
}

// What a code of 1 stands for: 2^(b - 127); 255: infinity, whose product with the code 0 is NaN.
__device__ inline float scale_of(uint32_t b) { return __uint_as_float(b << 23); }

// The eight codes at column f of a row of F; zeros behind its end.
__device__ inline u2b load_codes(const int8_t* row, int f, int F) {
  if (f + 8 <= F) return *reinterpret_cast<const u2b*>(row + f);
  u2b r = {0, 0};
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (f + e < F) r[e / 4] |= (uint32_t)(uint8_t)row[f + e] << (8 * (e & 3));
  return r;
}

// The part inside the row.
__device__ inline void store_codes(int8_t* row, int f, int F, const uint32_t (&c)[2]) {
  if (f + 8 <= F) {
    *reinterpret_cast<u2b*>(row + f) = u2b{c[0], c[1]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (f + e < F) row[f + e] = (int8_t)(c[e / 4] >> (8 * (e & 3)));
}

}  // namespace gcn
