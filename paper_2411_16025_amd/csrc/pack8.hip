// Rows kept in 8 bits: 32 columns under one power of two (gcn_pack8, gcn_unpack8).

#include "lanes.h"
#include "packed.h"
#include "rows.h"

namespace gcn {
namespace {

constexpr int kThreads = 256;

struct PackArgs {
  RowTiles tiles;  // pieces of eight columns, four to a scale byte
  uint32_t F;
  const void* x;
  int64_t ldx;
  int8_t* q;
  int64_t ldq;
  uint8_t* s;
  int64_t lds;
  void* y;
  int64_t ldy;
};

// Four neighbouring lanes have the 32 columns of a scale byte (rows have whole ones: so many
// pieces are counted). The largest magnitude is taken as a whole number, of which infinities and
// NaN are larger than all others. Bytes bound it and k_unpack (2,449,029 x 256 fp32: 577 and 580 us, 5.5
// and 5.4 TB/s).
template <class T>
__global__ __launch_bounds__(kThreads) void k_pack(PackArgs a) {
  uint32_t row, piece;
  const bool in = locate(a.tiles, kThreads, threadIdx.x, &row, &piece);
  const int f = (int)(8 * piece);
  float v[8];
  unpack_raw(load_raw<T, 8>(static_cast<const T*>(a.x) + (in ? (int64_t)row * a.ldx : 0), f, in ? (int)a.F : 0), v);
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)slot_partner<1>((int)top));
  top = max(top, (uint32_t)slot_partner<2>((int)top));
  if (!in) return;
  const uint32_t b = scale_byte(top);
  uint32_t c[2] = {0, 0};
  if (b != kNoScale) {
    const float inverse = __uint_as_float((254 - b) << 23);  // 2^-(b - 127)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int code = (int)fminf(fmaxf(rintf(v[e] * inverse), -127.f), 127.f);
      c[e / 4] |= (uint32_t)(code & 255) << (8 * (e & 3));
    }
  }
  store_codes(a.q + (int64_t)row * a.ldq, f, (int)a.F, c);
  if ((piece & 3) == 0) a.s[(int64_t)row * a.lds + piece / 4] = (uint8_t)b;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_unpack(PackArgs a) {
  uint32_t row, piece;
  if (!locate(a.tiles, kThreads, threadIdx.x, &row, &piece)) return;
  const int f = (int)(8 * piece);
  const u2b c = load_codes(a.q + (int64_t)row * a.ldq, f, (int)a.F);
  const float unit = scale_of(a.s[(int64_t)row * a.lds + piece / 4]);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = unit * (float)((int32_t)(c[e / 4] << (24 - 8 * (e & 3))) >> 24);
  store_raw(static_cast<T*>(a.y) + (int64_t)row * a.ldy, f, (int)a.F, v);
}

gcn_status check_pack(int64_t n, int64_t F, int dtype, const void* x, int64_t ldx, const int8_t* Q,
                      int64_t ldq, const uint8_t* S, int64_t lds) {
  GCN_CHECK(check_rows(n, F, dtype));
  if (n > 0 && (!x || !Q || !S || ldx < F || ldq < F || lds < ceil_div(F, (int64_t)32))) {
    set_error("rows, Q and S must be non-NULL, with row strides >= F (S: (F + 31) / 32)");
    return GCN_EINVAL;
  }
  return GCN_OK;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_pack8(int64_t n, int64_t F, const void* X, int64_t ldx, int dtype,
                                int8_t* Q, int64_t ldq, uint8_t* S, int64_t lds, void* stream) {
  clear_error();
  GCN_CHECK(check_pack(n, F, dtype, X, ldx, Q, ldq, S, lds));
  if (n == 0) return GCN_OK;
  GCN_CHECK(check_apart({rows_of(Q, n, ldq, F, 1), rows_of(S, n, lds, ceil_div(F, (int64_t)32), 1)},
                        {rows_of(X, n, ldx, F, size_of(dtype))}));
  // (whole scale bytes, in each workgroup too)
  PackArgs a{row_tiles(n, ceil_div(F, (int64_t)32) * 4, kThreads), (uint32_t)F, X, ldx, Q, ldq, S,
             lds, nullptr, 0};
  GCN_CHECK(launch_fits(a.tiles.blocks(), kThreads));
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps("pack8", s);
  const dim3 grid((unsigned)a.tiles.blocks());
  if (dtype == GCN_DT_F32)
    hipLaunchKernelGGL(k_pack<float>, grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(k_pack<bf16>, grid, dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

extern "C" gcn_status gcn_unpack8(int64_t n, int64_t F, const int8_t* Q, int64_t ldq,
                                  const uint8_t* S, int64_t lds, void* Y, int64_t ldy, int dtype,
                                  void* stream) {
  clear_error();
  GCN_CHECK(check_pack(n, F, dtype, Y, ldy, Q, ldq, S, lds));
  if (n == 0) return GCN_OK;
  GCN_CHECK(check_apart({rows_of(Y, n, ldy, F, size_of(dtype))},
                        {rows_of(Q, n, ldq, F, 1), rows_of(S, n, lds, ceil_div(F, (int64_t)32), 1)}));
  PackArgs a{row_tiles(n, ceil_div(F, (int64_t)8), kThreads), (uint32_t)F, nullptr, 0,
             const_cast<int8_t*>(Q), ldq, const_cast<uint8_t*>(S), lds, Y, ldy};
  GCN_CHECK(launch_fits(a.tiles.blocks(), kThreads));
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps("unpack8", s);
  const dim3 grid((unsigned)a.tiles.blocks());
  if (dtype == GCN_DT_F32)
    hipLaunchKernelGGL(k_unpack<float>, grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(k_unpack<bf16>, grid, dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}
