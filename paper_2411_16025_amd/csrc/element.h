// Element types of the calls that take a dtype.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "common.h"

namespace gcn {

typedef __bf16 bf16;

template <class T>
__device__ inline float to_float(T v) {
  return (float)v;
}

// Rounded to nearest even.
template <class T>
__device__ inline T from_float(float v) {
  return (T)v;
}

// Pieces of 16 bytes, at any element.
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
template <class T>
constexpr int kPiece = 16 / (int)sizeof(T);

template <class T>
struct Unaligned {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Unaligned<bf16> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};

// The piece at column f of a row of F; zeros behind its end.
template <class T>
__device__ inline u4 load_piece(const T* row, int f, int F) {
  if (f + kPiece<T> <= F) return *reinterpret_cast<const typename Unaligned<T>::type*>(row + f);
  u4 r = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < kPiece<T> - 1; ++e)
    if (f + e < F) {
      if constexpr (sizeof(T) == 4)
        r[e] = reinterpret_cast<const uint32_t*>(row)[f + e];
      else
        r[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[f + e] << (16 * (e & 1));
    }
  return r;
}

// A piece's elements moved down by n (at least 0), zeros behind them.
template <class T>
__device__ inline u4 move_down(u4 v, int n) {
  const uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
  constexpr int kHalf = kPiece<T> / 2;
  const int bits = 8 * (int)sizeof(T) * (n & (kHalf - 1));
  const uint64_t a = n & kHalf ? hi : lo, b = n & kHalf ? 0 : hi;
  uint64_t x = a >> bits | (bits ? b << (64 - bits) : 0), y = b >> bits;
  if (n >= kPiece<T>) x = y = 0;
  return u4{(uint32_t)x, (uint32_t)(x >> 32), (uint32_t)y, (uint32_t)(y >> 32)};
}

template <class T>
__device__ inline void unpack(u4 r, float (&v)[kPiece<T>]) {
#pragma unroll
  for (int e = 0; e < kPiece<T>; ++e) {
    if constexpr (sizeof(T) == 4)
      v[e] = __uint_as_float(r[e]);
    else
      v[e] = __uint_as_float(e & 1 ? r[e / 2] & 0xFFFF0000u : r[e / 2] << 16);
  }
}

// The part inside the row; each value rounded to nearest even.
template <class T>
__device__ inline void store_piece(T* row, int f, int F, const float (&v)[kPiece<T>]) {
  u4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 4) {
      r[e] = __float_as_uint(v[e]);
    } else {
      typedef float f2 __attribute__((ext_vector_type(2)));
      typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
      r[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{v[2 * e], v[2 * e + 1]}), bf2));
    }
  }
  if (f + kPiece<T> <= F) {
    *reinterpret_cast<typename Unaligned<T>::type*>(row + f) = r;
    return;
  }
#pragma unroll
  for (int e = 0; e < kPiece<T> - 1; ++e)
    if (f + e < F) {
      if constexpr (sizeof(T) == 4)
        reinterpret_cast<uint32_t*>(row)[f + e] = r[e];
      else
        reinterpret_cast<uint16_t*>(row)[f + e] = (uint16_t)(r[e / 2] >> (16 * (e & 1)));
    }
}

// A launch has fewer than 2^32 threads along an axis.
inline gcn_status launch_fits(int64_t blocks, int64_t threads) {
  if (blocks < (int64_t(1) << 32) / threads) return GCN_OK;
  set_error("more tiles than one launch takes");
  return GCN_ERANGE;
}

// Rows of so many bytes, `stride` bytes apart, or one array.
struct Span {
  const void* p;
  int64_t rows, stride, bytes;
};
inline Span array_of(const void* p, int64_t bytes) { return Span{p, 1, bytes, bytes}; }
inline Span rows_of(const void* p, int64_t n, int64_t ld, int64_t F, int64_t size) {
  return Span{p, n, ld * size, F * size};
}
inline int64_t size_of(int dtype) { return dtype == GCN_DT_BF16 ? 2 : 4; }

// Whether they share a byte; rows may lie between the other's.
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
  if (p > q) return overlap(b, a);
  if (!p || a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
  const uint64_t end = (uint64_t)(a.rows - 1) * a.stride + a.bytes;
  // (rows of the same stride all lie as the first one does; of others the ways to lie repeat)
  const int64_t ways = a.stride == b.stride ? 1 : std::min(b.rows, a.stride);
  uint64_t at = q - p;
  for (int64_t i = 0; i < ways && at < end; ++i, at += b.stride) {
    if (a.rows == 1) return true;
    const uint64_t in = at % (uint64_t)a.stride;
    if (in < (uint64_t)a.bytes || in + b.bytes > (uint64_t)a.stride) return true;
  }
  return false;
}

// Outputs apart from the inputs and from each other.
inline gcn_status check_apart(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
  for (const Span* a = outputs.begin(); a != outputs.end(); ++a) {
    bool bad = false;
    for (const Span& b : inputs) bad = bad || overlap(*a, b);
    for (const Span* b = outputs.begin(); b != a; ++b) bad = bad || overlap(*a, *b);
    if (!bad) continue;
    set_error("an output may not overlap an input or another output");
    return GCN_EINVAL;
  }
  return GCN_OK;
}

// n rows of F columns of a known type.
inline gcn_status check_rows(int64_t n, int64_t F, int dtype) {
  if (n < 0 || F <= 0 || F > (int64_t(1) << 30) ||
      (dtype != GCN_DT_F32 && dtype != GCN_DT_BF16)) {
    set_error("need n >= 0, F in [1, 2^30] and a known dtype");
    return GCN_EINVAL;
  }
  if (n >= (int64_t(1) << 31)) {
    set_error("need n < 2^31");
    return GCN_ERANGE;
  }
  return GCN_OK;
}

}  // namespace gcn
