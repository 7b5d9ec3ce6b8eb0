// Rows of a learned table and the table's gradient by sorted ids (gcn_embed_fwd, gcn_embed_bwd).

#include <cmath>

#include "groups.h"
#include "rows.h"

namespace gcn {
namespace {

constexpr int kThreads = 256;

// ---- the rows --------------------------------------------------------------------

struct TakeArgs {
  RowTiles tiles;
  uint32_t F, V, per;
  const int32_t* ids;
  const void* t;
  int64_t ldt;
  float scale;
  void* y;
  int64_t ldy;
};

// A thread has PER pieces of 16 bytes of Y, whose ids, then whose rows, are on their way together.
template <class T, class TY, int PER>
__global__ __launch_bounds__(kThreads) void k_take(TakeArgs a) {
  constexpr int N = kPiece<TY>;
  uint32_t row[PER], piece[PER], from[PER];
  bool real[PER];
  Raw<T, N> raw[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (!locate(a.tiles, kThreads * PER, threadIdx.x + k * kThreads, &row[k], &piece[k])) {
      piece[k] = a.tiles.pieces;
      row[k] = 0;
    }
    from[k] = (uint32_t)a.ids[row[k]];
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    real[k] = (int32_t)from[k] >= 0;
    if (a.per != 1) from[k] /= a.per;
    real[k] = real[k] && from[k] < a.V && piece[k] < a.tiles.pieces;
    raw[k] = load_raw<T, N>(static_cast<const T*>(a.t) + (real[k] ? from[k] : 0) * a.ldt,
                   (int)(N * piece[k]), real[k] ? (int)a.F : 0);
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (piece[k] >= a.tiles.pieces) continue;
    float v[N];
    unpack_raw(raw[k], v);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = real[k] ? a.scale * v[e] : 0.f;
    store_raw(static_cast<TY*>(a.y) + row[k] * a.ldy, (int)(N * piece[k]), (int)a.F, v);
  }
}

template <class T, class TY>
gcn_status take(TakeArgs a, int64_t n, int64_t F, hipStream_t s) {
  ProfScope ps("embed_fwd", s);
  const int64_t pieces = ceil_div(F, (int64_t)kPiece<TY>);
  const bool few = n * pieces < 512 * 4 * kThreads;
  a.tiles = row_tiles(n, pieces, kThreads * (few ? 1 : 4));
  GCN_CHECK(launch_fits(a.tiles.blocks(), kThreads));
  if (few)
    hipLaunchKernelGGL((k_take<T, TY, 1>), dim3((unsigned)a.tiles.blocks()), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_take<T, TY, 4>), dim3((unsigned)a.tiles.blocks()), dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

// ---- the gradient ----------------------------------------------------------------
//
// Rows of the table with up to `chunk` places are summed by the threads that own their pieces.
// Longer ones in chunks: a workgroup per chunk behind a row's first one writes its sum, and those
// workgroups then share the row's columns, each adding the first chunk's rows and the sums. Two
// long rows never begin in one run of `chunk` places, so the sum of chunk i of a row that begins at
// place b has the number b / chunk + i - 1 (groups.h counts the partial sums of products so).

struct SumArgs {
  RowTiles tiles;
  Groups by;            // the table's rows; by.rows places
  int32_t n;            // rows of dY
  uint32_t F;
  int chunk;
  const int32_t* order;
  const void* dy;
  int64_t lddy;
  float scale;
  void* dt;
  int64_t lddt;
  bool add;
  float* part;          // [places / chunk][F]
  int64_t ldp;
};

// v += the rows at places [beg, end), in their order.
template <class T, int N>
__device__ inline void add_rows(const SumArgs& a, int64_t beg, int64_t end, int f, float (&v)[N]) {
  constexpr int kAhead = 4;
  for (int64_t j = beg; j < end; j += kAhead) {
    int32_t at[kAhead];
    Raw<T, N> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) at[i] = j + i < end ? a.order[j + i] : -1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool in = at[i] >= 0 && at[i] < a.n;
      raw[i] = load_raw<T, N>(static_cast<const T*>(a.dy) + (in ? at[i] : 0) * a.lddy, f, in ? (int)a.F : 0);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      float x[N];
      unpack_raw(raw[i], x);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] += x[e];
    }
  }
}

// Scaled, added to the row's piece where wanted, and stored.
template <class TT, int N>
__device__ inline void write_piece(const SumArgs& a, int64_t row, int f, float (&v)[N]) {
  TT* to = static_cast<TT*>(a.dt) + row * a.lddt;
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] *= a.scale;
  if (a.add) {
    float old[N];
    unpack_raw(load_raw<TT, N>(to, f, (int)a.F), old);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += old[e];
  }
  store_raw(to, f, (int)a.F, v);
}

// PER pieces of 16 bytes of dT to a thread: most rows of a large table have no place, and what
// bounds the pass then is writing their zeros.
template <class T, class TT, int PER>
__global__ __launch_bounds__(kThreads) void k_sum_rows(SumArgs a) {
  constexpr int N = kPiece<TT>;
  uint32_t row[PER], piece[PER];
  int64_t beg[PER], end[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const bool in =
        locate(a.tiles, kThreads * PER, threadIdx.x + k * kThreads, &row[k], &piece[k]);
    if (!in) row[k] = 0;
    beg[k] = group_offset(a.by, (int)row[k]);
    end[k] = group_offset(a.by, (int)row[k] + 1);
    if (!in) end[k] = beg[k] + a.chunk + 1;  // not here
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (end[k] - beg[k] > a.chunk || (a.add && end[k] <= beg[k])) continue;
    const int f = (int)(N * piece[k]);
    float v[N] = {};
    add_rows<T>(a, beg[k], end[k], f, v);
    write_piece<TT>(a, row[k], f, v);
  }
}

// The long row that partial sum p belongs to: whether there is one.
__device__ inline bool long_row(const SumArgs& a, int64_t p, GroupTile* t, int64_t* p0,
                                int64_t* more) {
  *t = group_tile_from(a.by, [&](int, int64_t o) { return o / a.chunk <= p; });
  *p0 = t->first / a.chunk;
  *more = (t->end - t->first + a.chunk - 1) / a.chunk - 1;
  return p >= *p0 && p < *p0 + *more;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_sum_chunks(SumArgs a, int64_t p) {
  p += blockIdx.y;
  GroupTile t;
  int64_t p0, more;
  if (!long_row(a, p, &t, &p0, &more)) return;
  const int64_t beg = t.first + (p - p0 + 1) * a.chunk, end = min(beg + a.chunk, t.end);
  const uint32_t piece = blockIdx.x * kThreads + threadIdx.x;
  if (8 * piece >= a.F) return;
  float v[8] = {};
  add_rows<T>(a, beg, end, (int)(8 * piece), v);
  store_raw(a.part + p * a.ldp, (int)(8 * piece), (int)a.F, v);
}

// The pieces of a long row, shared by the workgroups of its partial sums.
template <class T, class TT>
__global__ __launch_bounds__(kThreads) void k_join_chunks(SumArgs a, int64_t p) {
  p += blockIdx.y;
  GroupTile t;
  int64_t p0, more;
  if (!long_row(a, p, &t, &p0, &more)) return;
  for (int64_t piece = ((p - p0) * gridDim.x + blockIdx.x) * kThreads + threadIdx.x;
       8 * piece < a.F; piece += more * gridDim.x * kThreads) {
    const int f = (int)(8 * piece);
    float v[8] = {};
    add_rows<T>(a, t.first, t.first + a.chunk, f, v);
    double s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = (double)v[e];
    for (int64_t q = p0; q < p0 + more; ++q) {
      float x[8];
      unpack_raw(load_raw<float, 8>(a.part + q * a.ldp, f, (int)a.F), x);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += (double)x[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)s[e];
    write_piece<TT>(a, t.g, f, v);
  }
}

template <class T, class TT>
gcn_status embed_bwd(SumArgs a, Scratch* scratch, hipStream_t s) {
  const int64_t pieces = ceil_div((int64_t)a.F, (int64_t)kPiece<TT>);
  const bool few = a.by.n * pieces < 2048 * kThreads;
  a.tiles = row_tiles(a.by.n, pieces, kThreads * (few ? 1 : 4));
  a.chunk = 32;
  GCN_CHECK(launch_fits(a.tiles.blocks(), kThreads));
  const int64_t parts = a.by.rows / a.chunk;
  a.ldp = ceil_div((int64_t)a.F, (int64_t)8) * 8;
  if (parts > 0) GCN_CHECK(scratch->alloc(&a.part, parts * a.ldp, "sums of repeated ids"));
  if (scratch->asked()) return GCN_OK;
  ProfScope ps("embed_bwd", s);
  const dim3 rows((unsigned)a.tiles.blocks());
  if (few)
    hipLaunchKernelGGL((k_sum_rows<T, TT, 1>), rows, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_sum_rows<T, TT, 4>), rows, dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  const unsigned wide = (unsigned)ceil_div(a.ldp, (int64_t)8 * kThreads);
  for (int64_t p = 0; p < parts; p += 65535) {  // (a grid's second axis)
    const dim3 grid(wide, (unsigned)std::min<int64_t>(parts - p, 65535));
    hipLaunchKernelGGL(k_sum_chunks<T>, grid, dim3(kThreads), 0, s, a, p);
    GCN_HIP(hipGetLastError());
  }
  for (int64_t p = 0; p < parts; p += 65535) {
    const dim3 grid(wide, (unsigned)std::min<int64_t>(parts - p, 65535));
    hipLaunchKernelGGL((k_join_chunks<T, TT>), grid, dim3(kThreads), 0, s, a, p);
    GCN_HIP(hipGetLastError());
  }
  return GCN_OK;
}

bool known(int dtype) { return dtype == GCN_DT_F32 || dtype == GCN_DT_BF16; }

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_embed_fwd(int64_t n, int64_t F, int64_t V, const int32_t* ids,
                                    int64_t per, const void* T, int64_t ldt, int dtype,
                                    double scale, void* Y, int64_t ldy, int dtype_y, void* stream) {
  clear_error();
  GCN_CHECK(check_rows(n, F, dtype));
  GCN_CHECK(check_rows(V, F, dtype_y));
  if (V < 1 || per < 1 || per >= (int64_t(1) << 31) || !std::isfinite((float)scale)) {
    set_error("need V >= 1, per in [1, 2^31) and a finite scale");
    return GCN_EINVAL;
  }
  if (n == 0) return GCN_OK;
  if (!ids || !T || !Y || T == Y || ldt < F || ldy < F) {
    set_error("ids, T and Y must be non-NULL, T and Y apart, with ldt, ldy >= F");
    return GCN_EINVAL;
  }
  const TakeArgs a{{}, (uint32_t)F, (uint32_t)V, (uint32_t)per, ids, T, ldt, (float)scale, Y, ldy};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == GCN_DT_F32)
    return dtype_y == GCN_DT_F32 ? take<float, float>(a, n, F, s) : take<float, bf16>(a, n, F, s);
  return dtype_y == GCN_DT_F32 ? take<bf16, float>(a, n, F, s) : take<bf16, bf16>(a, n, F, s);
}

extern "C" gcn_status gcn_embed_bwd(int64_t n, int64_t F, int64_t V, const int64_t* offsets,
                                    const int32_t* order, const void* dY, int64_t lddy, int dtype,
                                    double scale, void* dT, int64_t lddt, int dtype_t,
                                    uint32_t flags, void* work, int64_t* work_bytes, void* stream) {
  clear_error();
  CallScope scope(stream);
  GCN_CHECK(check_rows(n, F, dtype));
  if (V < 1 || !known(dtype_t) || !std::isfinite((float)scale) || (flags & ~GCN_ACCUMULATE)) {
    set_error("need V >= 1, known dtypes and flags and a finite scale");
    return GCN_EINVAL;
  }
  if (V > (int64_t(1) << 30)) {
    set_error("need V <= 2^30");
    return GCN_ERANGE;
  }
  GCN_CHECK(check_work(work, work_bytes));
  hipStream_t s = (hipStream_t)stream;
  Scratch scratch(work, work_bytes, s);
  if (n == 0 && (flags & GCN_ACCUMULATE)) return GCN_OK;
  if (!offsets || !dT || lddt < F || (n > 0 && (!order || !dY || lddy < F || dY == dT))) {
    set_error("offsets, order, dY and dT must be non-NULL, dY and dT apart, with lddy, lddt >= F");
    return GCN_EINVAL;
  }
  SumArgs a{};
  a.by = Groups{(int)V, offsets, n};
  a.n = (int32_t)n;
  a.F = (uint32_t)F;
  a.order = order;
  a.dy = dY;
  a.lddy = lddy;
  a.scale = (float)scale;
  a.dt = dT;
  a.lddt = lddt;
  a.add = flags & GCN_ACCUMULATE;
  if (dtype == GCN_DT_F32)
    return dtype_t == GCN_DT_F32 ? embed_bwd<float, float>(a, &scratch, s)
                                 : embed_bwd<float, bf16>(a, &scratch, s);
  return dtype_t == GCN_DT_F32 ? embed_bwd<bf16, float>(a, &scratch, s)
                               : embed_bwd<bf16, bf16>(a, &scratch, s);
}
