// Products of rows sorted by group with one matrix per group (gcn_gemm_grouped).

#include <algorithm>
#include <type_traits>

#include "element.h"
#include "groups.h"

namespace gcn {
namespace {

constexpr int kThreads = 256;

struct GroupArgs {
  Groups by;
  int N, K;  // columns of C; of A
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb;
  void* C;
  int64_t ldc;
  int64_t stride_w;
  int64_t split = 0;      // TN: rows of a chunk (groups.h), the sums of a group's first one in C,
  float* part = nullptr;  // of the others here
};

// The general kernel: one 64 x 64 tile of C per workgroup, fp32 products, any
// type, size and alignment. The tiles lie along the grid's first axis, which alone takes all that a
// launch does. TN: a group's rows in chunks, so that a narrow C has workgroups (bf16, 500,000 rows of 4
// groups, 256 x 4: 17.4 ms in one chunk each, 0.39 so).
constexpr int kTile = 64, kDepth = 16;

template <class T, class TC, int OP>
__global__ __launch_bounds__(kThreads) void k_grouped(GroupArgs a) {
  __shared__ float as[kDepth][kTile + 4], bs[kDepth][kTile + 4];
  const T* A = static_cast<const T*>(a.A);
  const T* B = static_cast<const T*>(a.B);
  TC* C = static_cast<TC*>(a.C);
  const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
  const uint32_t col_tiles = (a.N + kTile - 1) / kTile;
  const uint32_t tile = blockIdx.x / col_tiles;
  const int n0 = (int)(blockIdx.x % col_tiles) * kTile;
  int64_t i0 = 0;  // first row of C
  int64_t m_end, k0 = 0, k1 = a.K;
  if constexpr (OP == GCN_GEMM_TN) {
    const uint32_t row_tiles = (a.K + kTile - 1) / kTile;
    const int64_t slot = tile / row_tiles;
    const GroupTile gt = group_tile(a.by, slot, (int)a.split);
    if (gt.beg >= gt.end && gt.beg != gt.first) return;  // an empty group's first chunk: zeros
    k0 = gt.beg;
    k1 = std::min(gt.beg + a.split, gt.end);
    i0 = (int64_t)(tile % row_tiles) * kTile;
    m_end = a.K;
    if (gt.beg == gt.first) {
      C += gt.g * a.stride_w;
    } else {
      C = reinterpret_cast<TC*>(a.part) + (slot - gt.g - 1) * a.K * a.N;
      a.ldc = a.N;
    }
  } else {
    const GroupTile gt = group_tile(a.by, tile, kTile);
    i0 = gt.beg;
    m_end = gt.end;
    if (i0 >= m_end) return;
    B += gt.g * a.stride_w;
  }
  float acc[4][4] = {};
  for (int64_t kk = k0; kk < k1; kk += kDepth) {
    for (int e = t; e < kDepth * kTile; e += kThreads) {
      // neighbouring threads read neighbouring elements of a row
      const int kf = e % kDepth, rf = e / kDepth, kt = e / kTile, rt = e % kTile;
      if constexpr (OP == GCN_GEMM_TN) {
        const bool in = kk + kt < k1;
        as[kt][rt] = in && i0 + rt < m_end ? to_float(A[(kk + kt) * a.lda + i0 + rt]) : 0.f;
        bs[kt][rt] = in && n0 + rt < a.N ? to_float(B[(kk + kt) * a.ldb + n0 + rt]) : 0.f;
      } else {
        as[kf][rf] = kk + kf < k1 && i0 + rf < m_end ? to_float(A[(i0 + rf) * a.lda + kk + kf]) : 0.f;
        if constexpr (OP == GCN_GEMM_NN)
          bs[kt][rt] = kk + kt < k1 && n0 + rt < a.N ? to_float(B[(kk + kt) * a.ldb + n0 + rt]) : 0.f;
        else
          bs[kf][rf] = kk + kf < k1 && n0 + rf < a.N ? to_float(B[(n0 + rf) * a.ldb + kk + kf]) : 0.f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_fmaf(as[k][4 * ty + i], bs[k][4 * tx + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t r = i0 + 4 * ty + i;
      const int c = n0 + 4 * tx + j;
      if (r < m_end && c < a.N) C[r * a.ldc + c] = from_float<TC>(acc[i][j]);
    }
}

// ---- few rows per group ----------------------------------------------------------
//
// With a few rows to a group the matrices' bytes bound the product (24 rows over 13 of
// 16 groups, 2048 x 1024 bf16: 54.5 MB). So a workgroup has 16 or 32 rows and 64 columns of C, its
// eight wavefronts share the inner size in units of 64 (bf16) or 32 (fp32), and B comes from
// memory straight into the registers of the matrix instruction, the next unit's on its way while
// one is multiplied; the wavefronts' sums meet in LDS. bf16: v_mfma_f32_16x16x32_bf16, lane l holds
// row (column) l % 16 and 8 of the inner size from 8 (l / 16); fp32: v_mfma_f32_16x16x4_f32,
// one of the inner size, at 4 (l / 16) + s in step s. Both sides may take the inner size in any
// order as long as it is the same one.
constexpr int kFewCols = 64;

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u2a __attribute__((ext_vector_type(2), aligned(2)));

// 4 values at column f of a row of N; zeros behind its end.
__device__ inline u2 load4(const bf16* row, int f, int N) {
  if (f + 4 <= N) return *reinterpret_cast<const u2a*>(row + f);
  u2 r = {0, 0};
  const uint16_t* h = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (f + e < N) r[e / 2] |= (uint32_t)h[f + e] << (16 * (e & 1));
  return r;
}

// A piece without its first `cut` elements (zeros).
template <class T>
__device__ inline u4 cut_piece(u4 v, int cut) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4)
      v[i] = i < cut ? 0 : v[i];
    else
      v[i] = 2 * i + 1 < cut ? 0 : (2 * i < cut ? v[i] & 0xFFFF0000u : v[i]);
  }
  return v;
}

// What a wavefront holds of B for a unit, and the product with R blocks of 16 rows of A. cut():
// the unit's first `skip` of the inner size do not count.
// acc[r][j]: rows 4 (l / 16) + e of block r; column: see few_column.
template <class T, int OP, int R>
struct Unit;

template <int OP, int R>
struct Unit<bf16, OP, R> {
  static constexpr int K = 64;
  u4 a[2][R], b[2][4];  // NN: b[h][j] = lines 8 (l / 16) + 2 j, + 1 of columns 4 (l % 16) ..
  __device__ inline void load(const bf16* A, int64_t lda, const int (&row)[R], const bf16* B,
                              int64_t ldb, int n0, int N, int k0, int K) {
    const int l = threadIdx.x & 63, c = l & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + 32 * h + 8 * (l >> 4);
#pragma unroll
      for (int r = 0; r < R; ++r) a[h][r] = load_piece(A + row[r] * lda, k, K);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (OP == GCN_GEMM_NT) {
          const int n = n0 + 16 * j + c;
          b[h][j] = load_piece(B + (int64_t)n * ldb, k, n < N ? K : 0);
        } else {
          const int f = n0 + 4 * c;
          const u2 p = load4(B + (k + 2 * j) * ldb, f, k + 2 * j < K ? N : 0);
          const u2 q = load4(B + (k + 2 * j + 1) * ldb, f, k + 2 * j + 1 < K ? N : 0);
          b[h][j] = u4{p[0], p[1], q[0], q[1]};
        }
      }
    }
  }
  __device__ inline void cut(int skip) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = skip - 32 * h - 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
      for (int r = 0; r < R; ++r) a[h][r] = cut_piece<bf16>(a[h][r], first);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (OP == GCN_GEMM_NT)
          b[h][j] = cut_piece<bf16>(b[h][j], first);
        else  // whole lines
#pragma unroll
          for (int i = 0; i < 4; ++i) b[h][j][i] = 2 * j + i / 2 < first ? 0 : b[h][j][i];
      }
    }
  }
  __device__ inline void multiply(f4 (&acc)[R][4]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u4 v = b[h][j];
        if constexpr (OP == GCN_GEMM_NN)  // column 4 (l % 16) + j of the 8 lines
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = __builtin_amdgcn_perm(b[h][i][2 + j / 2], b[h][i][j / 2],
                                         j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int r = 0; r < R; ++r)
          acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf8, a[h][r]), __builtin_bit_cast(bf8, v), acc[r][j], 0, 0, 0);
      }
  }
};

template <int OP, int R>
struct Unit<float, OP, R> {
  static constexpr int K = 32;
  u4 a[2][R], b[2][4];  // NN: b[h][s] = line 4 (l / 16) + s, columns 4 (l % 16) ..; NT: b[h][j] = 4 lines
  __device__ inline void load(const float* A, int64_t lda, const int (&row)[R], const float* B,
                              int64_t ldb, int n0, int N, int k0, int K) {
    const int l = threadIdx.x & 63, c = l & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + 16 * h + 4 * (l >> 4);
#pragma unroll
      for (int r = 0; r < R; ++r) a[h][r] = load_piece(A + row[r] * lda, k, K);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (OP == GCN_GEMM_NT) {
          const int n = n0 + 16 * j + c;
          b[h][j] = load_piece(B + (int64_t)n * ldb, k, n < N ? K : 0);
        } else {
          b[h][j] = load_piece(B + (k + j) * ldb, n0 + 4 * c, k + j < K ? N : 0);
        }
      }
    }
  }
  __device__ inline void cut(int skip) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = skip - 16 * h - 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
      for (int r = 0; r < R; ++r) a[h][r] = cut_piece<float>(a[h][r], first);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        b[h][j] = OP == GCN_GEMM_NT ? cut_piece<float>(b[h][j], first)
                                    : (j < first ? u4{0, 0, 0, 0} : b[h][j]);
    }
  }
  __device__ inline void multiply(f4 (&acc)[R][4]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < R; ++r)
            acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                __uint_as_float(a[h][r][s]),
                __uint_as_float(OP == GCN_GEMM_NN ? b[h][s][j] : b[h][j][s]), acc[r][j], 0, 0, 0);
  }
};

template <class T, class TC, int OP, int R, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void k_few(GroupArgs a) {
  constexpr int kRows = 16 * R;
  __shared__ float sums[kWaves][kRows][kFewCols];
  const int col_tiles = (a.N + kFewCols - 1) / kFewCols;
  const uint32_t tile = blockIdx.x / col_tiles;
  // the last columns' tile ends with the matrix and computes some of its neighbour's again, so
  // that only narrow matrices have guarded columns (53 rows, 3032 x 2825 fp32: 35 us, 67 with guards)
  const int n0 = max(0, min((int)(blockIdx.x % col_tiles) * kFewCols, a.N - kFewCols));
  GroupTile gt;
  if (a.by.n <= kCountedGroups) {
    const TileCount count = count_tiles(a.by, kRows, 0);
    if (tile >= (uint32_t)count.total) return;
    gt = counted_tile(a.by, count, (int)tile, kRows, 0);
  } else {
    gt = group_tile(a.by, tile, kRows);
  }
  if (gt.beg >= gt.end) return;
  const int rows = (int)std::min<int64_t>(gt.end - gt.beg, kRows);
  const T* A = static_cast<const T*>(a.A) + gt.beg * a.lda;
  const T* B = static_cast<const T*>(a.B) + gt.g * a.stride_w;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int row[R];
#pragma unroll
  for (int r = 0; r < R; ++r) row[r] = std::min(16 * r + (l & 15), rows - 1);
  f4 acc[R][4] = {};
  using U = Unit<T, OP, R>;
  U u[2];
  const int step = kWaves * U::K;
  int k = w * U::K;
  // The last unit is whole, too, where the inner size has one: it begins earlier, without what the
  // unit before it has (24 rows of 16 groups, 2047 x 1023 bf16 NT: 30 us, 34 with guards).
  const int last = max(0, a.K - U::K);
  auto load = [&](U& to, int at) {
    to.load(A, a.lda, row, B, a.ldb, n0, a.N, min(at, last), a.K);
  };
  auto multiply = [&](U& of, int at) {
    if (at > last) of.cut(at - last);
    of.multiply(acc);
  };
  if (k < a.K) load(u[0], k);
  for (; k < a.K; k += 2 * step) {
    if (k + step < a.K) load(u[1], k + step);
    multiply(u[0], k);
    if (k + step >= a.K) break;
    if (k + 2 * step < a.K) load(u[0], k + 2 * step);
    multiply(u[1], k + step);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sums[w][16 * r + 4 * (l >> 4) + e][OP == GCN_GEMM_NN ? 4 * (l & 15) + j
                                                             : 16 * j + (l & 15)] = acc[r][j][e];
  __syncthreads();
  TC* C = static_cast<TC*>(a.C) + gt.beg * a.ldc;
  for (int t = threadIdx.x; t < rows * kFewCols; t += 64 * kWaves) {
    const int i = t / kFewCols, c = t % kFewCols;
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < kWaves; ++q) s += sums[q][i][c];
    if (n0 + c < a.N) C[i * a.ldc + n0 + c] = from_float<TC>(s);
  }
}

// Few rows to a group on average: of 16 groups, 2048 x 1024, bf16, 600 rows take 22.7 us here and
// 27.5 in tiles, 1024 rows 31.8 and 28.3; fp32 1024 rows 90 and 122, 2048 rows 147 and 123. And rows
// that are few large tiles, which would leave most CUs without work (4 groups of 433 rows,
// 1712 x 256: fp32 18 us and 81, bf16 9 and 18; 2,500 rows of 2, 1024 x 512: 48 and 53, 21 and 30;
// 6,865 rows of 4, 3728 x 59 fp32: 79 and 135; but 4,000 rows, 512 x 512, in 132 tiles: 36 and 31,
// 19 and 15; and more rows would read B more often: 13,080 rows of 2, 3568 x 40: 145 and 122, bf16
// 83 and 45).
bool few_takes(const Groups& g, int64_t N, int dtype) {
  const int64_t tiles = group_slots(g, 128) * ceil_div(N, (int64_t)128);
  return g.rows <= (dtype == GCN_DT_F32 ? 96 : 48) * (int64_t)g.n ||
         (tiles < 110 && g.rows <= (dtype == GCN_DT_F32 ? 8192 : 4096));
}

template <class T, class TC, int R, int W>
gcn_status few(int op, const GroupArgs& a, hipStream_t s) {
  const int64_t blocks = group_slots(a.by, 16 * R) * ceil_div((int64_t)a.N, (int64_t)kFewCols);
  GCN_CHECK(launch_fits(blocks, 64 * W));
  if (op == GCN_GEMM_NN)
    hipLaunchKernelGGL((k_few<T, TC, GCN_GEMM_NN, R, W>), dim3((unsigned)blocks), dim3(64 * W), 0,
                       s, a);
  else
    hipLaunchKernelGGL((k_few<T, TC, GCN_GEMM_NT, R, W>), dim3((unsigned)blocks), dim3(64 * W), 0,
                       s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <class T, class TC>
gcn_status few(int op, const GroupArgs& a, hipStream_t s) {
  ProfScope ps(op == GCN_GEMM_NN ? "grouped_nn_few" : "grouped_nt_few", s);
  // 16 rows to a workgroup where 32 would leave CUs without work (53 rows, 3032 x 2816 fp32: 31 us
  // and 48; 433 rows of 4 groups, 1712 x 256: 18 and 28)
  const bool one = a.by.rows <= 16 * a.by.n ||
                   group_slots(a.by, 32) * ceil_div((int64_t)a.N, (int64_t)kFewCols) < 256;
  // two wavefronts where a short inner size leaves the others none (232 rows of 100 groups, 48 x 3208:
  // fp32 21 us and 56, bf16 24 and 95)
  if (a.K <= 4 * Unit<T, GCN_GEMM_NN, 1>::K)
    return one ? few<T, TC, 1, 2>(op, a, s) : few<T, TC, 2, 2>(op, a, s);
  return one ? few<T, TC, 1, 8>(op, a, s) : few<T, TC, 2, 8>(op, a, s);
}

template <class T, class TC>
gcn_status grouped(int op, GroupArgs a, Scratch* scratch, hipStream_t s) {
  const bool tn = op == GCN_GEMM_TN;
  int64_t tiles = ceil_div((int64_t)a.N, (int64_t)kTile), slots, parts = 0;
  if (tn) {
    // four workgroups to a CU, chunks of 128 to 4096 rows (4096 where the groups' tiles are enough, longer
    // for more than a launch would take); partial sums as in the other kernels
    tiles *= ceil_div((int64_t)a.K, (int64_t)kTile);
    GCN_CHECK(launch_fits(tiles, kThreads));
    const int64_t even = ceil_div(ceil_div(a.by.rows * tiles, (int64_t)1024), (int64_t)kDepth) * kDepth;
    a.split = std::max(a.by.n * tiles >= 512
                           ? 4096
                           : std::min<int64_t>(4096, std::max<int64_t>(128, even)),
                       std::min(a.by.rows, ceil_div(a.by.rows * tiles, int64_t(1) << 22)));
    slots = group_slots(a.by, a.split);
    parts = a.by.rows / a.split;
  } else {
    slots = group_slots(a.by, kTile);
  }
  const int64_t blocks = tiles * slots;
  GCN_CHECK(launch_fits(blocks, kThreads));
  if (parts > 0)
    GCN_CHECK(scratch->alloc(&a.part, parts * a.K * a.N, "grouped GEMM partials"));
  if (scratch->asked()) return GCN_OK;
  const dim3 grid((unsigned)blocks);
  ProfScope ps(tn ? "grouped_tn" : op == GCN_GEMM_NN ? "grouped_nn" : "grouped_nt", s);
  if (tn)
    hipLaunchKernelGGL((k_grouped<T, TC, GCN_GEMM_TN>), grid, dim3(kThreads), 0, s, a);
  else if (op == GCN_GEMM_NN)
    hipLaunchKernelGGL((k_grouped<T, TC, GCN_GEMM_NN>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_grouped<T, TC, GCN_GEMM_NT>), grid, dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return parts > 0 ? sum_group_partials(a.by, a.split, a.K, a.N, a.part, static_cast<float*>(a.C),
                                        a.ldc, a.stride_w, s)
                   : GCN_OK;
}

// Partial sum p (blockIdx.y) belongs to the last group that begins in chunk p of all rows or
// before it, if that has so many: a group of several chunks reaches the next multiple of
// `split`. The workgroups of a group's partial sums share its elements, each element
// the sum of all of them in an order that their number decides: sixteen at a time (and fewer at
// the end) by pairs, those sums in double. (2,449,029 x 256 x 96: 9.3e-7 from 64 bits where 1276
// partial sums were one fp32 chain, 4.7e-7 so and in shorter chunks. 113,045 rows of 22 groups, 1024 x 256:
// 45 us, 58 with one load at a time.)
__global__ __launch_bounds__(kThreads) void k_group_sums(Groups by, int64_t split, int64_t K,
                                                         int64_t N, int64_t p, const float* part, float* C,
                                                         int64_t ldc, int64_t stride_w) {
  p += blockIdx.y;
  const GroupTile gt = group_tile_from(by, [&](int, int64_t o) { return o / split <= p; });
  const int64_t p0 = gt.first / split, more = (gt.end - gt.first + split - 1) / split - 1;
  if (p < p0 || p >= p0 + more) return;
  part += p0 * K * N;
  C += gt.g * stride_w;
  for (int64_t t = ((p - p0) * gridDim.x + blockIdx.x) * kThreads + threadIdx.x; t < K * N;
       t += more * gridDim.x * kThreads) {
    float* c = C + t / N * ldc + t % N;
    const float first = *c;  // (not waited for before the loads of the others)
    double s = 0.0;
    const float* q = part + t;
    int64_t left = more;
    auto add = [&](auto ahead) {  // so many, pairs first, their loads on their way at a time
      constexpr int n = decltype(ahead)::value;
      float v[n];
#pragma unroll
      for (int i = 0; i < n; ++i) v[i] = q[i * K * N];
#pragma unroll
      for (int h = n / 2; h > 0; h /= 2)
#pragma unroll
        for (int i = 0; i < h; ++i) v[i] += v[i + h];
      s += (double)v[0];
      q += n * K * N;
      left -= n;
    };
    while (left >= 16) add(std::integral_constant<int, 16>());
    if (left >= 8) add(std::integral_constant<int, 8>());
    if (left >= 4) add(std::integral_constant<int, 4>());
    if (left >= 2) add(std::integral_constant<int, 2>());
    if (left >= 1) add(std::integral_constant<int, 1>());
    *c = (float)(s + (double)first);
  }
}

}  // namespace

gcn_status sum_group_partials(const Groups& g, int64_t split, int64_t K, int64_t N,
                              const float* part, float* C, int64_t ldc, int64_t stride_w,
                              hipStream_t stream) {
  const int64_t parts = g.rows / split;
  const int64_t blocks = std::min(ceil_div(K * N, (int64_t)kThreads),
                                  std::max<int64_t>(16, ceil_div(1024, parts)));
  for (int64_t p = 0; p < parts; p += 65535) {  // (a grid's second axis)
    hipLaunchKernelGGL(k_group_sums, dim3((unsigned)blocks, (unsigned)std::min<int64_t>(parts - p, 65535)),
                       dim3(kThreads), 0, stream, g, split, K, N, p, part, C, ldc, stride_w);
    GCN_HIP(hipGetLastError());
  }
  return GCN_OK;
}

}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_gemm_grouped(int op, int64_t n_groups, const int64_t* offsets,
                                       int64_t rows, int64_t N, int64_t K, const void* A,
                                       int64_t lda, const void* B, int64_t ldb, int dtype, void* C,
                                       int64_t ldc, int dtype_c, int64_t stride_w, void* work,
                                       int64_t* work_bytes, void* stream) {
  clear_error();
  CallScope scope(stream);
  const bool tn = op == GCN_GEMM_TN;
  if ((op != GCN_GEMM_NN && op != GCN_GEMM_NT && !tn) || n_groups < 1 || n_groups >= 65536 ||
      rows < 0 || N < 1 || K < 1 || N >= (1 << 24) || K >= (1 << 24)) {
    set_error("need a known op, n_groups in [1, 65536), rows >= 0 and N, K in [1, 2^24)");
    return GCN_EINVAL;
  }
  if (rows >= (int64_t(1) << 31)) {
    set_error("need rows < 2^31");
    return GCN_ERANGE;
  }
  if ((dtype != GCN_DT_F32 && dtype != GCN_DT_BF16) ||
      (dtype_c != GCN_DT_F32 && (tn || dtype_c != dtype))) {
    set_error("need a known dtype, and dtype_c fp32 or (NN, NT) the operands'");
    return GCN_EINVAL;
  }
  GCN_CHECK(check_work(work, work_bytes));
  hipStream_t s = (hipStream_t)stream;
  Scratch scratch(work, work_bytes, s);
  if (rows == 0 && !tn) return GCN_OK;
  const int64_t big = int64_t(1) << 40;
  if (!offsets || !C || (rows > 0 && (!A || !B)) || lda < K || ldc < N ||
      ldb < (op == GCN_GEMM_NT ? K : N) || lda > big || ldb > big || ldc > big || stride_w < 0 ||
      (tn && n_groups > 1 && stride_w < (K - 1) * ldc + N)) {
    set_error("offsets, A, B, C must be non-NULL, row strides at least the rows' lengths, and "
              "stride_w >= 0 (TN: at least a matrix of C)");
    return GCN_EINVAL;
  }
  const Groups by{(int)n_groups, offsets, rows};
  const GroupArgs a{by, (int)N, (int)K, A, lda, B, ldb, C, ldc, stride_w};
  if (!tn && few_takes(by, N, dtype)) {
    if (scratch.asked()) return GCN_OK;
    if (dtype == GCN_DT_F32) return few<float, float>(op, a, s);
    return dtype_c == GCN_DT_F32 ? few<bf16, float>(op, a, s) : few<bf16, bf16>(op, a, s);
  }
  if (dtype == GCN_DT_F32 && gemm_split_grouped_takes(op, N, K, lda, ldb, ldc)) {
    ProfScope ps(tn ? "grouped_tn" : op == GCN_GEMM_NN ? "grouped_nn" : "grouped_nt", s);
    const float *fa = static_cast<const float*>(A), *fb = static_cast<const float*>(B);
    float* fc = static_cast<float*>(C);
    return tn ? gemm_split_tn_grouped(by, N, K, fa, lda, fb, ldb, fc, ldc, stride_w, &scratch, s)
              : scratch.asked() ? GCN_OK
              : gemm_split_grouped(op, by, N, K, fa, lda, fb, ldb, stride_w, fc, ldc, s);
  }
  if (dtype == GCN_DT_BF16 && gemm_grouped_bf16_takes(N, K, lda, ldb)) {
    ProfScope ps(tn ? "grouped_tn" : op == GCN_GEMM_NN ? "grouped_nn" : "grouped_nt", s);
    return gemm_grouped_bf16(op, by, N, K, A, lda, B, ldb, C, ldc, dtype_c == GCN_DT_BF16, stride_w,
                             &scratch, s);
  }
  if (dtype == GCN_DT_F32) return grouped<float, float>(op, a, &scratch, s);
  return dtype_c == GCN_DT_F32 ? grouped<bf16, float>(op, a, &scratch, s)
                               : grouped<bf16, bf16>(op, a, &scratch, s);
}
