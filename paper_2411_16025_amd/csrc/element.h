// Element types of the calls that take a dtype.
#pragma once

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

// n rows of F columns of a known type.
inline gcn_status check_rows(int64_t n, int64_t F, int dtype) {
  if (n < 0 || F <= 0 || F >= (int64_t(1) << 31) ||
      (dtype != GCN_DT_F32 && dtype != GCN_DT_BF16)) {
    set_error("need n >= 0, F in [1, 2^31) and a known dtype");
    return GCN_EINVAL;
  }
  if (n >= (int64_t(1) << 31)) {
    set_error("need n < 2^31");
    return GCN_ERANGE;
  }
  return GCN_OK;
}

}  // namespace gcn
