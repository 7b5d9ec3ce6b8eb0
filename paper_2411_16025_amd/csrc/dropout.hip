// Dropout whose mask is never stored (dropout.h).

#include "dropout.h"

#include <algorithm>

#include "element.h"

namespace gcn {

gcn_status make_drop(const gcn_dropout_spec* spec, int64_t n, Drop* out) {
  *out = Drop{0, 1.f, 0, 0, 0, nullptr, 0};
  if (!spec) return GCN_OK;
  if (!(spec->p >= 0.0 && spec->p < 1.0) || spec->row0 < 0) {
    set_error("dropout needs 0 <= p < 1 and row0 >= 0");
    return GCN_EINVAL;
  }
  if (spec->row0 > (int64_t(1) << 32) - n) {
    set_error("dropout needs row0 + n <= 2^32");
    return GCN_ERANGE;
  }
  out->least = (uint32_t)(spec->p * 4294967296.0);
  out->scale = (float)(1.0 / (1.0 - spec->p));
  out->k0 = (uint32_t)spec->seed;
  out->k1 = (uint32_t)(spec->seed >> 32);
  out->call = spec->call;
  out->step = spec->step;
  out->row0 = (uint32_t)spec->row0;
  return GCN_OK;
}

namespace {

constexpr int kThreads = 256;

// One thread per block of four columns.
template <class T>
__global__ __launch_bounds__(kThreads) void k_dropout(int64_t n, int64_t F, const T* x, int64_t ldx,
                                                      T* y, int64_t ldy, Drop d) {
  const int64_t per = (F + 3) / 4;
  const uint64_t call = drop_call(d);
  for (int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x; t < n * per;
       t += (int64_t)gridDim.x * kThreads) {
    const int64_t i = t / per, b = t % per;
    uint32_t w[4];
    drop_words(d, call, (uint32_t)i, (uint32_t)b, w);
    for (int e = 0; e < 4 && 4 * b + e < F; ++e) {
      const float v = to_float(x[i * ldx + 4 * b + e]);
      y[i * ldy + 4 * b + e] = from_float<T>(w[e] >= d.least ? v * d.scale : 0.f);
    }
  }
}

template <class T>
gcn_status dropout(int64_t n, int64_t F, const void* X, int64_t ldx, const Drop& d, void* Y,
                   int64_t ldy, hipStream_t s) {
  ProfScope ps("dropout", s);
  const int64_t blocks = ceil_div(n * ((F + 3) / 4), (int64_t)kThreads);
  hipLaunchKernelGGL(k_dropout<T>, dim3((unsigned)std::min<int64_t>(blocks, 16384)),
                     dim3(kThreads), 0, s, n, F, static_cast<const T*>(X), ldx,
                     static_cast<T*>(Y), ldy, d);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_dropout(int64_t n, int64_t F, const void* X, int64_t ldx, int dtype,
                                  const gcn_dropout_spec* drop, void* Y, int64_t ldy,
                                  void* stream) {
  clear_error();
  GCN_CHECK(check_rows(n, F, dtype));
  if (!drop) {
    set_error("drop must be non-NULL");
    return GCN_EINVAL;
  }
  Drop d;
  GCN_CHECK(make_drop(drop, n, &d));
  if (n == 0) return GCN_OK;
  if (!X || !Y || ldx < F || ldy < F || (X == Y && ldx != ldy)) {
    set_error("X and Y must be non-NULL with ldx, ldy >= F (and one stride where Y is X)");
    return GCN_EINVAL;
  }
  hipStream_t s = (hipStream_t)stream;
  return dtype == GCN_DT_F32 ? dropout<float>(n, F, X, ldx, d, Y, ldy, s)
                             : dropout<bf16>(n, F, X, ldx, d, Y, ldy, s);
}
