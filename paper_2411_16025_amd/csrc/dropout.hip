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

// Pieces of 16 bytes, eight to a thread, so that a thread's loads are all on their way
// before its first mask; a workgroup has a run of whole rows (or a part of a long one), and a
// thread finds its piece's row by a multiplication. Reading and writing bound it, also at
// 2 bytes an element: seven rounds are 14 wide multiplications for 4 elements.
constexpr int kThreads = 256, kPer = 8, kTile = kThreads * kPer;

struct DropArgs {
  uint32_t n, F, pieces;   // pieces of a row
  uint32_t rows, parts;    // rows of a workgroup, workgroups of a row
  uint32_t magic;          // ceil(2^32 / pieces): t magic / 2^32 = t / pieces for pieces > 1, t < 2^16
  const void* x;
  int64_t ldx;
  void* y;
  int64_t ldy;
  Drop drop;
};

template <class T>
__global__ __launch_bounds__(kThreads) void k_dropout(DropArgs a) {
  const uint32_t row0 = blockIdx.x / a.parts * a.rows, piece0 = blockIdx.x % a.parts * kTile;
  const uint64_t call = drop_call(a.drop);
  uint32_t row[kPer], f[kPer];
  u4 raw[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const uint32_t t = threadIdx.x + k * kThreads;
    const uint32_t r =
        a.pieces == 1 ? t : (a.rows > 1 ? (uint32_t)((uint64_t)t * a.magic >> 32) : 0);
    const uint32_t piece = piece0 + t - r * a.pieces;
    row[k] = row0 + r;
    f[k] = piece * kPiece<T>;
    if (r >= a.rows || row[k] >= a.n || piece >= a.pieces) f[k] = a.F;
    raw[k] = load_piece(static_cast<const T*>(a.x) + row[k] * a.ldx, (int)f[k],
                        f[k] < a.F ? (int)a.F : 0);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (f[k] >= a.F) continue;
    float v[kPiece<T>];
    unpack<T>(raw[k], v);
    drop_piece<kPiece<T>>(a.drop, call, row[k], (int)f[k], v);
    store_piece<T>(static_cast<T*>(a.y) + row[k] * a.ldy, (int)f[k], (int)a.F, v);
  }
}

template <class T>
gcn_status dropout(int64_t n, int64_t F, const void* X, int64_t ldx, const Drop& d, void* Y,
                   int64_t ldy, hipStream_t s) {
  ProfScope ps("dropout", s);
  const int64_t pieces = ceil_div(F, (int64_t)kPiece<T>);
  const int64_t rows = std::max<int64_t>(1, kTile / pieces), parts = ceil_div(pieces, (int64_t)kTile);
  DropArgs a{(uint32_t)n, (uint32_t)F, (uint32_t)pieces, (uint32_t)rows, (uint32_t)parts,
             (uint32_t)std::min<int64_t>(ceil_div(int64_t(1) << 32, pieces), 0xFFFFFFFF),
             X, ldx, Y, ldy, d};
  const int64_t blocks = ceil_div(n, rows) * parts;
  GCN_CHECK(launch_fits(blocks, kThreads));
  hipLaunchKernelGGL(k_dropout<T>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
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
