// Weight gradients from rows kept in 8 bits: C_g = X_g^T B_g (gcn_gemm_grouped_q8).

#include <algorithm>

#include "groups.h"
#include "packed.h"

namespace gcn {
namespace {

struct Q8Args {
  Groups by;
  int N, K;  // columns of B, of X
  const int8_t* q;
  int64_t ldq;
  const uint8_t* s;
  int64_t lds;
  const void* b;
  int64_t ldb;
  float* c;
  int64_t ldc, stride_c;
  int64_t split;  // rows of a chunk (groups.h): the sums of a group's first one in C,
  float* part;    // of the others here
};

// The general kernel: 64 x 64 of C per workgroup, fp32 products, any size.
constexpr int kThreads = 256, kTile = 64, kDepth = 16;

template <class T>
__global__ __launch_bounds__(kThreads) void k_q8(Q8Args a) {
  __shared__ float as[kDepth][kTile + 4], bs[kDepth][kTile + 4];
  const T* B = static_cast<const T*>(a.b);
  const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
  const uint32_t col_tiles = (a.N + kTile - 1) / kTile, row_tiles = (a.K + kTile - 1) / kTile;
  const uint32_t tile = blockIdx.x / col_tiles;
  const int n0 = (int)(blockIdx.x % col_tiles) * kTile, i0 = (int)(tile % row_tiles) * kTile;
  const int64_t slot = tile / row_tiles;
  const GroupTile gt = group_tile(a.by, slot, (int)a.split);
  if (gt.beg >= gt.end && gt.beg != gt.first) return;  // an empty group's first chunk: zeros
  const int64_t k1 = std::min(gt.beg + a.split, gt.end);
  float* C = a.c + gt.g * a.stride_c;
  int64_t ldc = a.ldc;
  if (gt.beg != gt.first) {
    C = a.part + (slot - gt.g - 1) * a.K * a.N;
    ldc = a.N;
  }
  float acc[4][4] = {};
  for (int64_t kk = gt.beg; kk < k1; kk += kDepth) {
    for (int e = t; e < kDepth * kTile; e += kThreads) {
      const int kt = e / kTile, rt = e % kTile, i = i0 + rt;
      const int64_t row = kk + kt;
      const bool in = row < k1;
      as[kt][rt] = in && i < a.K ? scale_of(a.s[row * a.lds + i / 32]) * (float)a.q[row * a.ldq + i]
                                 : 0.f;
      bs[kt][rt] = in && n0 + rt < a.N ? to_float(B[row * a.ldb + n0 + rt]) : 0.f;
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
      const int r = i0 + 4 * ty + i, c = n0 + 4 * tx + j;
      if (r < a.K && c < a.N) C[r * ldc + c] = acc[i][j];
    }
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_gemm_grouped_q8(int64_t n_groups, const int64_t* offsets, int64_t rows,
                                          int64_t N, int64_t K, const int8_t* Q, int64_t ldq,
                                          const uint8_t* S, int64_t lds, const void* B, int64_t ldb,
                                          int dtype, float* C, int64_t ldc, int64_t stride_w,
                                          void* work, int64_t* work_bytes, void* stream) {
  clear_error();
  CallScope scope(stream);
  if (n_groups < 1 || n_groups >= 65536 || rows < 0 || N < 1 || K < 1 || N >= (1 << 24) ||
      K >= (1 << 24) || (dtype != GCN_DT_F32 && dtype != GCN_DT_BF16)) {
    set_error("need n_groups in [1, 65536), rows >= 0, N and K in [1, 2^24) and a known dtype");
    return GCN_EINVAL;
  }
  if (rows >= (int64_t(1) << 31)) {
    set_error("need rows < 2^31");
    return GCN_ERANGE;
  }
  GCN_CHECK(check_work(work, work_bytes));
  hipStream_t s = (hipStream_t)stream;
  Scratch scratch(work, work_bytes, s);
  const int64_t big = int64_t(1) << 40;
  if (!offsets || !C || ldc < N || ldc > big || (n_groups > 1 && stride_w < (K - 1) * ldc + N) ||
      stride_w < 0 ||
      (rows > 0 && (!Q || !S || !B || ldq < K || lds < ceil_div(K, (int64_t)32) || ldb < N ||
                    ldq > big || lds > big || ldb > big))) {
    set_error("offsets, Q, S, B, C must be non-NULL, row strides at least the rows' lengths, and "
              "stride_w at least a matrix of C");
    return GCN_EINVAL;
  }
  Q8Args a{Groups{(int)n_groups, offsets, rows}, (int)N, (int)K, Q, ldq, S, lds, B, ldb, C, ldc,
           stride_w, 0, nullptr};
  // four workgroups to a CU, chunks of 128 to 4096 rows (4096 where the groups' tiles are enough, longer
  // for more than a launch would take)
  const int64_t tiles = ceil_div(N, (int64_t)kTile) * ceil_div(K, (int64_t)kTile);
  GCN_CHECK(launch_fits(tiles, kThreads));
  const int64_t even = ceil_div(ceil_div(rows * tiles, (int64_t)1024), (int64_t)kDepth) * kDepth;
  a.split = std::max(n_groups * tiles >= 512
                         ? 4096
                         : std::min<int64_t>(4096, std::max<int64_t>(128, even)),
                     std::min(rows, ceil_div(rows * tiles, int64_t(1) << 22)));
  const int64_t blocks = tiles * group_slots(a.by, a.split), parts = rows / a.split;
  GCN_CHECK(launch_fits(blocks, kThreads));
  if (parts > 0) GCN_CHECK(scratch.alloc(&a.part, parts * K * N, "grouped GEMM partials"));
  if (scratch.asked()) return GCN_OK;
  ProfScope ps("grouped_q8", s);
  if (dtype == GCN_DT_F32)
    hipLaunchKernelGGL(k_q8<float>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(k_q8<bf16>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return parts > 0 ? sum_group_partials(a.by, a.split, K, N, a.part, C, ldc, stride_w, s) : GCN_OK;
}
