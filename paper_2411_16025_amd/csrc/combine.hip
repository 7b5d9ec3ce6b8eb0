// Rows from the groups' order back to their tokens, weighted, and the gradients
// (gcn_combine_fwd, gcn_combine_bwd).

#include "lanes.h"
#include "rows.h"

namespace gcn {
namespace {

constexpr int kThreads = 256;

struct CombineArgs {
  RowTiles tiles;
  int64_t n;
  int k;
  uint32_t F, rows;
  const void* z;
  int64_t ldz;
  const int32_t* slot;
  const float* w;
  void* y;         // forward
  const void* dy;  // backward
  int64_t ldy;
  void* dz;
  int64_t lddz;
  float* dw;
};

// A thread has a piece of a token's row; the pieces of kAhead choices are on their way together. Bytes
// bound it (16,384 tokens, 8 rows of 1024 bf16 each: 58 us, 5.2 TB/s).
template <class T>
__global__ __launch_bounds__(kThreads) void k_combine(CombineArgs a) {
  constexpr int kAhead = 4;
  uint32_t t, piece;
  if (!locate(a.tiles, kThreads, threadIdx.x, &t, &piece)) return;
  const int f = (int)(8 * piece);
  const int32_t* slot = a.slot + (int64_t)t * a.k;
  const float* w = a.w + (a.w ? (int64_t)t * a.k : 0);
  float v[8] = {};
  for (int i = 0; i < a.k; i += kAhead) {
    uint32_t at[kAhead];
    float by[kAhead];
    Raw<T, 8> raw[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      at[j] = i + j < a.k ? (uint32_t)slot[i + j] : 0xFFFFFFFFu;
      by[j] = a.w && i + j < a.k ? w[i + j] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const bool in = at[j] < a.rows;
      raw[j] = load_raw<T, 8>(static_cast<const T*>(a.z) + (in ? at[j] : 0) * a.ldz, f, in ? (int)a.F : 0);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (at[j] >= a.rows) continue;
      float x[8];
      unpack_raw(raw[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(by[j], x[e], v[e]);
    }
  }
  store_raw(static_cast<T*>(a.y) + (int64_t)t * a.ldy, f, (int)a.F, v);
}

// G lanes have a token, so that the choices' weights' gradients are sums within a wavefront: dY's row is
// read from the caches for the second choice on. Bytes bound it (32,768 tokens, 2 rows of 2048 bf16
// each: 142 us, 4.7 TB/s).
template <class T, int G>
__global__ __launch_bounds__(kThreads) void k_combine_bwd(CombineArgs a) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const int in = threadIdx.x % G;
  if (t >= a.n) return;
  const T* dy = static_cast<const T*>(a.dy) + t * a.ldy;
  for (int i = 0; i < a.k; ++i) {
    const uint32_t at = (uint32_t)a.slot[t * a.k + i];
    const bool real = at < a.rows;
    const float w = a.w ? a.w[t * a.k + i] : 1.f;
    float dot = 0.f;
    if (real)
      for (int64_t f = 8 * in; f < a.F; f += 8 * G) {
        float g[8], x[8];
        unpack_raw(load_raw<T, 8>(dy, (int)f, (int)a.F), g);
        if (a.dw) {
          unpack_raw(load_raw<T, 8>(static_cast<const T*>(a.z) + at * a.ldz, (int)f, (int)a.F), x);
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(g[e], x[e], dot);
        }
        if (a.dz) {
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] *= w;
          store_raw(static_cast<T*>(a.dz) + at * a.lddz, (int)f, (int)a.F, g);
        }
      }
    if (a.dw) {
      dot = slot_sum<G>(dot);
      if (in == 0) a.dw[t * a.k + i] = dot;
    }
  }
}

template <class T>
gcn_status combine(CombineArgs a, hipStream_t s) {
  ProfScope ps("combine_fwd", s);
  a.tiles = row_tiles(a.n, ceil_div((int64_t)a.F, (int64_t)8), kThreads);
  GCN_CHECK(launch_fits(a.tiles.blocks(), kThreads));
  hipLaunchKernelGGL(k_combine<T>, dim3((unsigned)a.tiles.blocks()), dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <class T>
gcn_status combine_bwd(const CombineArgs& a, hipStream_t s) {
  ProfScope ps("combine_bwd", s);
  const int64_t pieces = ceil_div((int64_t)a.F, (int64_t)8);
  const int lanes = pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
  const int64_t blocks = ceil_div(a.n, (int64_t)(kThreads / lanes));
  GCN_CHECK(launch_fits(blocks, kThreads));
  const dim3 grid((unsigned)blocks);
  switch (lanes) {
    case 8: hipLaunchKernelGGL((k_combine_bwd<T, 8>), grid, dim3(kThreads), 0, s, a); break;
    case 16: hipLaunchKernelGGL((k_combine_bwd<T, 16>), grid, dim3(kThreads), 0, s, a); break;
    case 32: hipLaunchKernelGGL((k_combine_bwd<T, 32>), grid, dim3(kThreads), 0, s, a); break;
    default: hipLaunchKernelGGL((k_combine_bwd<T, 64>), grid, dim3(kThreads), 0, s, a);
  }
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

gcn_status check_combine(int64_t n, int64_t k, int64_t F, int64_t rows, int dtype) {
  GCN_CHECK(check_rows(n, F, dtype));
  GCN_CHECK(check_rows(rows, F, dtype));
  if (k < 1 || k > 65536) {
    set_error("need k in [1, 2^16]");
    return GCN_EINVAL;
  }
  return GCN_OK;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_combine_fwd(int64_t n, int64_t k, int64_t F, const void* Z, int64_t rows,
                                      int64_t ldz, int dtype, const int32_t* slot,
                                      const float* weights, void* Y, int64_t ldy, void* stream) {
  clear_error();
  GCN_CHECK(check_combine(n, k, F, rows, dtype));
  if (n == 0) return GCN_OK;
  if ((rows > 0 && (!Z || ldz < F)) || !slot || !Y || Y == Z || ldy < F) {
    set_error("Z, slot and Y must be non-NULL, Y and Z apart, with ldz, ldy >= F");
    return GCN_EINVAL;
  }
  GCN_CHECK(check_apart({rows_of(Y, n, ldy, F, size_of(dtype))},
                        {rows_of(Z, rows, ldz, F, size_of(dtype)), array_of(slot, 4 * n * k),
                         array_of(weights, 4 * n * k)}));
  CombineArgs a{};
  a.n = n;
  a.k = (int)k;
  a.F = (uint32_t)F;
  a.rows = (uint32_t)rows;
  a.z = Z;
  a.ldz = ldz;
  a.slot = slot;
  a.w = weights;
  a.y = Y;
  a.ldy = ldy;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GCN_DT_F32 ? combine<float>(a, s) : combine<bf16>(a, s);
}

extern "C" gcn_status gcn_combine_bwd(int64_t n, int64_t k, int64_t F, const void* Z, int64_t rows,
                                      int64_t ldz, int dtype, const int32_t* slot,
                                      const float* weights, const void* dY, int64_t lddy, void* dZ,
                                      int64_t lddz, float* dweights, void* stream) {
  clear_error();
  GCN_CHECK(check_combine(n, k, F, rows, dtype));
  if (!dZ && !dweights) {
    set_error("at least one of dZ and dweights must be non-NULL");
    return GCN_EINVAL;
  }
  if (n == 0) return GCN_OK;
  if (!slot || !dY || lddy < F || dY == dZ || dY == Z ||
      (rows > 0 && ((dweights && (!Z || ldz < F)) || (dZ && (lddz < F || (dZ == Z && lddz != ldz)))))) {
    set_error("slot, dY and, for dweights, Z must be non-NULL, dY apart from Z and dZ, with row "
              "strides >= F (and one stride where dZ is Z)");
    return GCN_EINVAL;
  }
  // (dweights in the weights' place: each one is read before its gradient is written)
  const Span none{}, z = rows_of(dweights ? Z : nullptr, rows, ldz, F, size_of(dtype));
  const Span dy = rows_of(dY, n, lddy, F, size_of(dtype)), at = array_of(slot, 4 * n * k);
  const Span w = array_of(weights, 4 * n * k), dw = array_of(dweights, 4 * n * k);
  GCN_CHECK(check_apart({rows_of(dZ, rows, lddz, F, size_of(dtype)), dw},
                        {dZ == Z ? none : z, dy, at, weights == dweights ? none : w}));
  GCN_CHECK(check_apart({dw}, {z}));
  CombineArgs a{};
  a.n = n;
  a.k = (int)k;
  a.F = (uint32_t)F;
  a.rows = (uint32_t)rows;
  a.z = Z;
  a.ldz = ldz;
  a.slot = slot;
  a.w = weights;
  a.dy = dY;
  a.ldy = lddy;
  a.dz = dZ;
  a.lddz = lddz;
  a.dw = dweights;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GCN_DT_F32 ? combine_bwd<float>(a, s) : combine_bwd<bf16>(a, s);
}
