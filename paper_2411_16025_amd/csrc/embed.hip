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

// A thread has PER pieces of 16 bytes of Y, whose ids, then whose rows, are on their way together. Bytes
// bound it (65,536 rows of 2048 bf16: 88 us, 4.6 TB/s); of few rows the latency of the two loads, so
// that each thread then has one piece (24 rows: 2.7 us).
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
// Longer ones in chunks: the sum of each chunk behind the first is a partial sum, and the row's
// pieces are then shared by the workgroups of those, which add the first chunk's rows and the partial
// sums. Two long rows never begin in one run of `chunk` places, so the sum of chunk i of a row that
// begins at place b has the number b / chunk + i - 1 (groups.h counts the partial sums of products
// so). The pass over the rows writes a number's row beside it; whoever has a number takes that row
// only if its offsets say so too, so numbers of no long row need no value there.

struct SumArgs {
  RowTiles tiles;
  Groups by;            // the table's rows; by.rows places
  int32_t n;            // rows of dY
  uint32_t F;
  int shift;            // chunk = 1 << shift
  const int32_t* order;
  const void* dy;
  int64_t lddy;
  float scale;
  void* dt;
  int64_t lddt;
  bool add;
  bool zeroed;          // dT is 0
  uint32_t parts;       // places / chunk
  int32_t* owner;       // [parts]
  float* part;          // [parts][ldp]
  int64_t ldp;
};

// v += the rows at places [beg, end), in their order.
template <class T, int N, int kAhead = 4>
__device__ inline void add_rows(const SumArgs& a, int64_t beg, int64_t end, int f, float (&v)[N]) {
  for (int64_t j = beg; j < end; j += kAhead) {
    int32_t at[kAhead];
    Raw<T, N> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) at[i] = j + i < end ? a.order[j + i] : -1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool in = at[i] >= 0 && at[i] < a.n;
      raw[i] = load_raw<T, N>(static_cast<const T*>(a.dy) + (in ? at[i] : 0) * a.lddy, f,
                              in ? (int)a.F : 0);
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

// Zeros over `bytes` bytes from an element's address on: in pieces of 16 bytes where memory has them.
constexpr int kZeroEach = 8;
__global__ __launch_bounds__(kThreads) void k_zero(char* p, int64_t bytes) {
  const int64_t head = std::min<int64_t>(-(int64_t)reinterpret_cast<uintptr_t>(p) & 15, bytes);
  const int64_t pieces = (bytes - head) / 16, tail = head + 16 * pieces;
  const int64_t at = (int64_t)blockIdx.x * (kThreads * kZeroEach) + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kZeroEach; ++i)
    if (at + i * kThreads < pieces)
      reinterpret_cast<u4*>(p + head)[at + i * kThreads] = u4{0, 0, 0, 0};
  if (blockIdx.x == 0 && threadIdx.x < 16) {  // (elements: 2 or 4 bytes)
    if (2 * (int)threadIdx.x < head) *reinterpret_cast<uint16_t*>(p + 2 * threadIdx.x) = 0;
    if (tail + 2 * threadIdx.x < bytes) *reinterpret_cast<uint16_t*>(p + tail + 2 * threadIdx.x) = 0;
  }
}

// A workgroup has up to kRows rows, or a part of a long one, in pieces of 16 bytes of dT. Rows without
// a place, most of a large table's, are zeros, which bound the pass; those that have some are listed, so
// that all lanes gather (2,449,029 x 100 fp32, 250,000 places: 318 us where each piece looked for its
// row's places, 245 with the zeros of a workgroup's rows written first; 282 with zeros past the caches; all these without the
// sort).
// A table with a place for fewer than every 32nd row, whose rows lie beside each other, is zeroed by a
// launch before, which knows nothing of rows and writes at 6.8 TB/s (25,000 places: 244 and 204 us;
// 250,000 places at 128 columns: 274 and 305, so not there). Rows that are no whole pieces cost the pass
// more, which then is for every 8th (245,000 places at 47 columns: 217 and 149, at 101: 300 and 284;
// 490,000 at 101: 338 and 348; 408,000 at 47, in the pass by this rule: 239 and 173). bf16 outputs go by it too, a place for
// every 6th, 24th and 48th row in the pass and zeroed before: 47 columns 178 and 116, 117 and 60, 114 and 54; 48 columns 97
// and 93, 61 and 59, 45 and 52; 128 columns 178 and 212, 139 and 147, 130 and 137.
constexpr int kRows = 1024;

template <class T, class TT, int kRowTile>
__global__ __launch_bounds__(kThreads) void k_sum_rows(SumArgs a) {
  constexpr int N = kPiece<TT>;
  __shared__ int32_t first[kRows + 1];  // the rows' first places
  __shared__ uint16_t list[kRows];      // rows of 1 .. chunk places, and from the end on those of more
  __shared__ uint32_t listed, longs;
  const RowTiles& t = a.tiles;
  const uint32_t row0 = blockIdx.x / t.parts * t.rows, rows = min(t.rows, t.n - row0);
  const uint32_t piece0 = blockIdx.x % t.parts * kRowTile;
  const uint32_t pieces = min(t.pieces - piece0, t.parts > 1 ? (uint32_t)kRowTile : t.pieces);  // of a row, here
  for (uint32_t r = threadIdx.x; r <= rows; r += kThreads)
    first[r] = (int32_t)group_offset(a.by, (int)(row0 + r));
  __syncthreads();
  const int32_t chunk = 1 << a.shift;
  // the first wavefront lists the rows, in their order
  if (threadIdx.x < 64) {
    uint32_t n = 0, l = 0;
    for (uint32_t r0 = 0; r0 < rows; r0 += 64) {
      const uint32_t r = r0 + threadIdx.x;
      const int32_t len = r < rows ? first[r + 1] - first[r] : 0;
      const uint64_t some = __ballot(len > 0 && len <= chunk), more = __ballot(len > chunk);
      const uint64_t below = (1ull << threadIdx.x) - 1;
      if (len > chunk)
        list[kRows - 1 - l - (uint32_t)__popcll(more & below)] = (uint16_t)r;
      else if (len > 0)
        list[n + (uint32_t)__popcll(some & below)] = (uint16_t)r;
      n += (uint32_t)__popcll(some);
      l += (uint32_t)__popcll(more);
    }
    if (threadIdx.x == 0) {
      listed = n;
      longs = l;
    }
  }
  if (!a.add && !a.zeroed) {
    const float zero[N] = {};
    for (uint32_t q = threadIdx.x; q < rows * pieces; q += kThreads) {
      const uint32_t r = pieces == 1 ? q : (rows > 1 ? (uint32_t)((uint64_t)q * t.magic >> 32) : 0);
      if (first[r + 1] <= first[r])
        store_raw(static_cast<TT*>(a.dt) + (int64_t)(row0 + r) * a.lddt,
                  (int)(N * (piece0 + q - r * pieces)), (int)a.F, zero);
    }
  }
  __syncthreads();
  // the numbers of long rows' partial sums
  if (blockIdx.x % t.parts == 0)
    for (uint32_t i = 0; i < longs; ++i) {
      const uint32_t r = list[kRows - 1 - i], p0 = (uint32_t)first[r] >> a.shift;
      const uint32_t more = (uint32_t)(first[r + 1] - first[r] - 1) >> a.shift;
      for (uint32_t p = threadIdx.x; p < more; p += kThreads) a.owner[p0 + p] = (int32_t)(row0 + r);
    }
  for (uint32_t q = threadIdx.x; q < listed * pieces; q += kThreads) {
    const uint32_t i = pieces == 1 ? q : (rows > 1 ? (uint32_t)((uint64_t)q * t.magic >> 32) : 0);
    const uint32_t r = list[i];
    const int f = (int)(N * (piece0 + q - i * pieces));
    float v[N] = {};
    add_rows<T>(a, first[r], first[r + 1], f, v);
    write_piece<TT>(a, row0 + r, f, v);
  }
}

// The long row that partial sum p belongs to.
struct LongRow {
  bool any;
  int v;
  int64_t first, end;
  uint32_t p0, more;  // its partial sums
};
__device__ inline LongRow long_row(const SumArgs& a, uint32_t p) {
  LongRow r{};
  if (p >= a.parts) return r;
  r.v = a.owner[p];
  if (r.v < 0 || r.v >= a.by.n) return r;
  r.first = group_offset(a.by, r.v);
  r.end = group_offset(a.by, r.v + 1);
  const int64_t len = r.end - r.first;
  r.p0 = (uint32_t)(r.first >> a.shift);
  r.more = len > (1 << a.shift) ? (uint32_t)((len - 1) >> a.shift) : 0;
  r.any = p >= r.p0 && p - r.p0 < r.more;
  return r;
}

// A thread has a piece of a chunk's sum.
template <class T>
__global__ __launch_bounds__(kThreads) void k_sum_chunks(SumArgs a, RowTiles tiles) {
  constexpr int N = kPiece<T>;
  uint32_t p, piece;
  if (!locate(tiles, kThreads, threadIdx.x, &p, &piece)) return;
  const LongRow r = long_row(a, p);
  if (!r.any) return;
  const int64_t beg = r.first + ((int64_t)(p - r.p0 + 1) << a.shift);
  float v[N] = {};
  add_rows<T, N, 8>(a, beg, min(beg + (1 << a.shift), r.end), (int)(N * piece), v);
  store_raw(a.part + p * a.ldp, (int)(N * piece), (int)a.F, v);
}

// A share of a long row's pieces: the threads divide the first chunk's rows and the partial sums
// among them, and the sums of a piece meet in LDS. kInTurn numbers to a workgroup, as most are of no
// long row.
constexpr int kInTurn = 2;

template <class T, class TT>
__global__ __launch_bounds__(kThreads) void k_join_chunks(SumArgs a) {
  __shared__ double sums[kThreads][9];  // (9: the rows fall on different banks)
  const int64_t pieces = ((int64_t)a.F + 7) / 8;
  for (int i = 0; i < kInTurn; ++i) {
    const uint32_t p = blockIdx.x * kInTurn + i;
    const LongRow r = long_row(a, p);  // (the same for all threads)
    if (!r.any) continue;
    int share = 8;  // pieces of a workgroup
    while (share < kThreads && (int64_t)share * r.more < pieces) share *= 2;
    const int groups = kThreads / share, g = threadIdx.x / share;
    const int part = max(1, (1 << a.shift) / groups);  // of the first chunk's places
    for (int64_t s0 = (int64_t)(p - r.p0) * share; s0 < pieces; s0 += (int64_t)r.more * share) {
      const int64_t piece = s0 + threadIdx.x % share;
      const int f = (int)(8 * piece);
      double s[8] = {};
      float v[8] = {};
      if (piece < pieces) {
        if (g * part < (1 << a.shift))
          add_rows<T>(a, r.first + g * part, r.first + (g + 1) * part, f, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = (double)v[e];
        constexpr int kAhead = 4;
        for (uint32_t q = r.p0 + g; q < r.p0 + r.more; q += kAhead * groups) {
          Raw<float, 8> raw[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            raw[j] = load_raw<float, 8>(a.part + min(q + j * groups, r.p0 + r.more - 1) * a.ldp, f,
                                        (int)a.F);
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            float x[8];
            unpack_raw(raw[j], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += q + j * groups < r.p0 + r.more ? (double)x[e] : 0.0;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[threadIdx.x][e] = s[e];
      __syncthreads();
      if (g == 0 && piece < pieces) {
        for (int o = 1; o < groups; ++o)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e] += sums[threadIdx.x + o * share][e];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)s[e];
        write_piece<TT>(a, r.v, f, v);
      }
      __syncthreads();
    }
  }
}

template <class T, class TT>
gcn_status embed_bwd(SumArgs a, Scratch* scratch, hipStream_t s) {
  // small tiles where many rows have places to gather (131,072 places of 50,000 rows of 1024 bf16: 182 us
  // in tiles of 4096 pieces, 85 in 1024; 16,384 of 32,000 x 4096: 134 and 50)
  const bool sparse = a.by.n > 4 * a.by.rows;
  a.tiles = row_tiles(a.by.n, ceil_div((int64_t)a.F, (int64_t)kPiece<TT>), sparse ? 4096 : 1024);
  a.tiles.rows = std::min<uint32_t>(a.tiles.rows, kRows);
  const bool whole = a.lddt % kPiece<TT> == 0;
  a.zeroed = a.by.n > (whole ? 32 : 8) * a.by.rows && !a.add && a.lddt == a.F;
  if (a.zeroed && a.tiles.parts == 1)  // more rows, of which few are listed
    a.tiles.rows = std::min(512u, std::max(1u, 16384 / a.tiles.pieces));
  a.shift = a.by.rows <= (1 << 18) ? 5 : 7;
  GCN_CHECK(launch_fits(a.tiles.blocks(), kThreads));
  a.parts = (uint32_t)(a.by.rows >> a.shift);
  a.ldp = ceil_div((int64_t)a.F, (int64_t)8) * 8;
  if (a.parts > 0) {
    GCN_CHECK(scratch->alloc(&a.part, a.parts * a.ldp, "sums of repeated ids"));
    GCN_CHECK(scratch->alloc(&a.owner, a.parts, "rows of repeated ids"));
  }
  if (scratch->asked()) return GCN_OK;
  ProfScope ps("embed_bwd", s);
  const dim3 rows((unsigned)a.tiles.blocks());
  const int64_t bytes = (int64_t)a.by.n * a.F * (int64_t)sizeof(TT);
  if (a.zeroed) {
    const int64_t blocks = ceil_div(bytes, (int64_t)16 * kThreads * kZeroEach);
    GCN_CHECK(launch_fits(blocks, kThreads));
    hipLaunchKernelGGL(k_zero, dim3((unsigned)blocks), dim3(kThreads), 0, s, static_cast<char*>(a.dt),
                       bytes);
    GCN_HIP(hipGetLastError());
  }
  if (sparse)
    hipLaunchKernelGGL((k_sum_rows<T, TT, 4096>), rows, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_sum_rows<T, TT, 1024>), rows, dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  if (a.parts == 0) return GCN_OK;
  const RowTiles chunks = row_tiles(a.parts, ceil_div((int64_t)a.F, (int64_t)kPiece<T>), kThreads);
  GCN_CHECK(launch_fits(chunks.blocks(), kThreads));
  hipLaunchKernelGGL(k_sum_chunks<T>, dim3((unsigned)chunks.blocks()), dim3(kThreads), 0, s, a, chunks);
  GCN_HIP(hipGetLastError());
  hipLaunchKernelGGL((k_join_chunks<T, TT>), dim3((unsigned)ceil_div(a.parts, (int64_t)kInTurn)),
                     dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
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
  GCN_CHECK(check_apart({rows_of(Y, n, ldy, F, size_of(dtype_y))},
                        {rows_of(T, V, ldt, F, size_of(dtype)), array_of(ids, 4 * n)}));
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
  if (!scratch.asked())
    GCN_CHECK(check_apart({rows_of(dT, V, lddt, F, size_of(dtype_t))},
                          {rows_of(dY, n, lddy, F, size_of(dtype)), array_of(offsets, 8 * (V + 1)),
                           array_of(order, 4 * n)}));
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
