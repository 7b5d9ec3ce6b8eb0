// Weight gradients from rows kept in 8 bits: C_g = X_g^T B_g (gcn_gemm_grouped_q8).

#include <algorithm>
#include <cmath>

#include "groups.h"
#include "mul_tile.h"
#include "packed.h"
#include "split.h"

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
  int col_tiles, row_tiles;
  uint32_t slots;
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

// ---- on the matrix cores ----------------------------------------------------------

typedef uint32_t u4b __attribute__((ext_vector_type(4), aligned(1)));  // 16 bytes anywhere

// The sixteen bytes of v moved down by n (at least 0), zeros behind them.
__device__ inline u4 bytes_down(u4 v, int n) {
  const uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
  const int bits = 8 * (n & 7);
  const uint64_t a = n & 8 ? hi : lo, b = n & 8 ? 0 : hi;
  uint64_t x = a >> bits | (bits ? b << (64 - bits) : 0), y = b >> bits;
  if (n >= 16) x = y = 0;
  return u4{(uint32_t)x, (uint32_t)(x >> 32), (uint32_t)y, (uint32_t)(y >> 32)};
}

// The values of eight codes, exact in bf16: codes + 128 are bytes, which fp32 takes in one
// instruction, and u unit - 128 unit is exact.
__device__ inline u4 decode8(uint32_t c0, uint32_t c1, float unit) {
  const float off = -128.f * unit;
  u4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t u = (i ? c1 : c0) ^ 0x80808080u;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf((float)(u >> (8 * e) & 255), unit, off);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      r[2 * i + e] = __builtin_amdgcn_perm(__float_as_uint(v[2 * e + 1]), __float_as_uint(v[2 * e]),
                                           0x07060302u);
  }
  return r;
}

// BK rows of X columns of the codes: units of 16, which are decoded into two 16-byte pieces
// of the tile. A unit that reaches over a row's end is read from 16 codes before the end on (rows have
// 16) and moved down; one past the last row is the last row's with a unit of 0.
template <int X, int BK, int NT>
struct CodeLoader {
  using T = Tile<false, X, BK>;
  static constexpr int kUnits = X * BK / 16, kPerLine = X / 16;
  static constexpr int kCount = (kUnits + NT - 1) / NT;
  static constexpr bool kFull = kUnits % NT == 0;
  const int8_t* q;
  const uint8_t* s;
  int64_t ldq, lds;
  int have;      // columns inside the matrix
  int64_t had;   // rows of the stage whose units are in v
  u4 v[kCount];
  uint32_t scale[kCount];

  __device__ static inline int line_of(int p) { return (int)(threadIdx.x + p * NT) / kPerLine; }
  __device__ static inline int element_of(int p) { return 16 * ((int)(threadIdx.x + p * NT) % kPerLine); }
  __device__ static inline bool mine(int p) { return kFull || (int)threadIdx.x + p * NT < kUnits; }
  __device__ inline void init(const int8_t* q_, int64_t ldq_, const uint8_t* s_, int64_t lds_, int have_) {
    q = q_;
    s = s_;
    ldq = ldq_;
    lds = lds_;
    have = have_;
  }
  __device__ inline void load(int64_t k0, int64_t left) {
    had = left;
    if (left <= 0) return;  // past the last stage
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      if (!mine(p)) continue;
      const int64_t row = k0 + std::min<int64_t>(line_of(p), left - 1);
      v[p] = *reinterpret_cast<const u4b*>(q + row * ldq + std::min(element_of(p), have - 16));
      scale[p] = s[row * lds + std::min(element_of(p), have - 1) / 32];
    }
  }
  __device__ inline void store(char* lds_to, uint32_t sign) {
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      if (!mine(p)) continue;
      const int line = line_of(p), e = element_of(p);
      u4 x = v[p];
      if (have < X) x = bytes_down(x, std::min(16, std::max(0, e + 16 - have)));
      if (line >= had) x = u4{0, 0, 0, 0};
      const float unit = line < had ? __uint_as_float(scale[p] << 23 ^ sign) : 0.f;
      char* to = lds_to + line * (X * 2) + ((e / 8) ^ T::swz(line)) * 16;
      *reinterpret_cast<u4*>(to) = decode8(x[0], x[1], unit);
      *reinterpret_cast<u4*>(to + 16) = decode8(x[2], x[3], unit);
    }
  }
};

// BK rows of X columns of fp32, split into three tiles: pieces of 8, read as two of 4 (as
// Loader's: from before a row's end, and moved down).
template <int X, int BK, int NT>
struct PartLoader {
  using T = Tile<false, X, BK>;
  static constexpr int kCount = T::kPieces / NT, kPerLine = T::kPerLine;
  static_assert(T::kPieces % NT == 0, "every thread has as many pieces");
  const float* base;
  int64_t ld;
  int have;
  int64_t had;
  u4 v[kCount][2];

  __device__ static inline int line_of(int p) { return (int)(threadIdx.x + p * NT) / kPerLine; }
  __device__ static inline int element_of(int p) { return 8 * ((int)(threadIdx.x + p * NT) % kPerLine); }
  __device__ inline void init(const float* b, int64_t ld_, int have_) {
    base = b;
    ld = ld_;
    have = have_;
  }
  __device__ inline void load(char*, int64_t k0, int64_t left) {
    had = left;
    if (left <= 0) return;  // past the last stage
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      const float* row = base + (k0 + std::min<int64_t>(line_of(p), left - 1)) * ld;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        v[p][i] = *reinterpret_cast<const Unaligned<float>::type*>(
            row + std::min(element_of(p) + 4 * i, have - 4));
    }
  }
  __device__ inline void store(char* lds_to) {
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      const int line = line_of(p), e = element_of(p);
      float x[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u4 r = v[p][i];
        if (have < X) r = move_down<float>(r, std::min(4, std::max(0, e + 4 * i + 4 - have)));
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = line < had ? __uint_as_float(r[j]) * kUp : 0.f;
      }
      u4 parts[3];
      split8(x, parts);
      char* to = lds_to + line * (X * 2) + ((e / 8) ^ T::swz(line)) * 16;
#pragma unroll
      for (int i = 0; i < 3; ++i) *reinterpret_cast<u4*>(to + i * T::kBytes) = parts[i];
    }
  }
};

// bf16 rows: as in gemm_grouped.hip.
template <class TB, int X, int BK, int NT, bool DIRECT>
struct RowLoader : Loader<false, X, BK, NT, DIRECT> {
  static constexpr int kParts = 1;
};
template <int X, int BK, int NT, bool DIRECT>
struct RowLoader<float, X, BK, NT, DIRECT> : PartLoader<X, BK, NT> {
  static constexpr int kParts = 3;
};

// A workgroup of WR x WC wavefronts, RB x CB blocks of 32 x 32 of C each. DIRECT: bf16 rows
// that direct loads take to LDS.
template <class TB, bool DIRECT, int BK, int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_mul8(Q8Args a) {
  constexpr int NT = 64 * WR * WC, BM = 32 * WR * RB, BN = 32 * WC * CB;
  using LA = CodeLoader<BM, BK, NT>;
  using LB = RowLoader<TB, BN, BK, NT, DIRECT>;
  using TA = Tile<false, BM, BK>;
  using TN = Tile<false, BN, BK>;
  constexpr int NP = LB::kParts;
  __shared__ __align__(16) char a0[TA::kBytes], a1[TA::kBytes], b0[NP * TN::kBytes],
      b1[NP * TN::kBytes];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  // the chunks' tiles divide evenly among the XCDs, those of a chunk beside each other
  const int R = (int)a.split;
  const bool counted = a.by.n <= kCountedGroups;
  TileCount count{};
  if (counted) count = count_tiles(a.by, R, 1);
  const uint32_t rows = counted ? count.total : a.slots;
  const uint32_t per = a.col_tiles * a.row_tiles, units = rows * per, xcd = blockIdx.x & 7;
  const uint32_t u = (uint32_t)((uint64_t)units * xcd / 8) + (blockIdx.x >> 3);
  if (u >= (uint32_t)((uint64_t)units * (xcd + 1) / 8)) return;
  const uint32_t slot = u / per;
  const int m0 = (int)(u % per) / a.col_tiles * BM, n0 = (int)(u % per) % a.col_tiles * BN;
  const GroupTile gt = counted ? counted_tile(a.by, count, (int)slot, R, 1)
                               : group_tile(a.by, slot, R);
  if (gt.beg >= gt.end && gt.beg != gt.first) return;  // an empty group's first chunk: zeros
  const int64_t k_beg = gt.beg, k_end = std::max(gt.beg, std::min(gt.beg + a.split, gt.end));
  const int64_t chunk = (gt.beg - gt.first) / a.split;
  LA la;
  LB lb;
  la.init(a.q + m0, a.ldq, a.s + m0 / 32, a.lds, a.K - m0);
  lb.init(static_cast<const TB*>(a.b) + n0, a.ldb, a.N - n0);
  // (the matrix core's rounding has one sign: every other chunk's sums are of negated products)
  const uint32_t sign = chunk & 1 ? 0x80000000u : 0;

  f16 acc[RB][CB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Fragments of a step are read while the step before it is multiplied, the first ones of the next
  // stage too (gemm_grouped.hip).
  constexpr int STEPS = BK / 16;
  static_assert(STEPS % 2 == 0, "the fragments' buffers alternate over the stages");
  bf8 fa[2][RB], fb[2][CB][NP];
  auto read = [&](int to, int step, const char* ca, const char* cb) {
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[to][i] = TA::read(ca, wr * RB + i, step, lane);
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int p = 0; p < NP; ++p)
        fb[to][j][p] = TN::read(cb + p * TN::kBytes, wc * CB + j, step, lane);
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int p = NP - 1; p >= 0; --p)  // the small parts first
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[from][i], fb[from][j][p],
                                                              acc[i][j], 0, 0, 0);
  };
  const int64_t stages = (k_end - k_beg + BK - 1) / BK;
  auto load = [&](int64_t s, char* to) {
    const int64_t k = k_beg + s * BK;
    la.load(k, k_end - k);
    lb.load(to, k, k_end - k);
  };
  auto pass_on = [&](int64_t s, char* cb, char* na, char* nb) {
    la.store(na, sign);
    lb.store(nb);
    wait_loads();
    load(s + 2, cb);
  };
  auto stage = [&](int64_t s, char* ca, char* cb, char* na, char* nb) {
#pragma unroll
    for (int st = 0; st + 1 < STEPS; ++st) {
      read((st + 1) & 1, st + 1, ca, cb);
      multiply(st & 1);
    }
    pass_on(s, cb, na, nb);
    read(0, 0, na, nb);
    multiply((STEPS - 1) & 1);
  };
  if (stages > 0) {
    load(0, b0);
    la.store(a0, sign);
    lb.store(b0);
    load(1, b1);
    wait_loads<DIRECT ? TN::kPieces / NT : 63>();  // stage 0's; the direct loads of stage 1 are the last ones
    read(0, 0, a0, b0);
    for (int64_t s = 0; s < stages; s += 2) {
      stage(s, a0, b0, a1, b1);
      if (s + 1 >= stages) break;
      stage(s + 1, a1, b1, a0, b0);
    }
    wait_loads();  // those past the last stage
  }

  float* C = a.c + gt.g * a.stride_c;
  int64_t ldc = a.ldc;
  if (chunk > 0) {
    C = a.part + (gt.first / a.split + chunk - 1) * a.K * a.N;
    ldc = a.N;
  }
  float down = NP == 3 ? 1.f / kUp : 1.f;
  if (chunk & 1) down = -down;
  if constexpr (NP == 3) {
    if (not_finite<RB, CB>(acc)) {
      down = 1.f;
      auto again = [&](int64_t k, float (*x)[4], float (*y)[4]) {
#pragma unroll
        for (int i = 0; i < RB; ++i) {
          const int m = std::min(m0 + (wr * RB + i) * 32 + (lane & 31), a.K - 1);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[i][j] = k + j < k_end ? scale_of(a.s[(k + j) * a.lds + m / 32]) *
                                          (float)a.q[(k + j) * a.ldq + m]
                                    : 0.f;
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
          const int n = std::min(n0 + (wc * CB + i) * 32 + (lane & 31), a.N - 1);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            y[i][j] = k + j < k_end ? static_cast<const float*>(a.b)[(k + j) * a.ldb + n] : 0.f;
        }
      };
      mul_again<RB, CB>(k_beg, k_end, again, acc);
    }
  }
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int r0 = m0 + (wr * RB + i) * 32 + 4 * (lane >> 5);
      const int c = n0 + (wc * CB + j) * 32 + (lane & 31);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = r0 + (e & 3) + 8 * (e >> 2);
        if (r < a.K && c < a.N) C[r * ldc + c] = __builtin_fmaf(acc[i][j][e], down, 0.f);
      }
    }
}

template <class TB, bool DIRECT, int BK, int WR, int WC, int RB, int CB>
gcn_status launch(Q8Args a, hipStream_t s) {
  constexpr int BM = 32 * WR * RB, BN = 32 * WC * CB;
  a.col_tiles = (int)ceil_div((int64_t)a.N, (int64_t)BN);
  a.row_tiles = (int)ceil_div((int64_t)a.K, (int64_t)BM);
  const int64_t slots = group_slots(a.by, a.split);
  const int64_t blocks = ceil_div(slots * a.col_tiles * a.row_tiles, (int64_t)8) * 8;
  GCN_CHECK(launch_fits(blocks, 64 * WR * WC));
  a.slots = (uint32_t)slots;
  hipLaunchKernelGGL((k_mul8<TB, DIRECT, BK, WR, WC, RB, CB>), dim3((unsigned)blocks),
                     dim3(64 * WR * WC), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

// Rows of sixteen codes, and strides whose offsets over a stage's rows are 32 bits.
bool mul8_takes(const Q8Args& a) {
  return a.N >= 8 && a.K >= 16 && a.ldb < (int64_t(1) << 22);
}

gcn_status mul8(Q8Args a, int dtype, Scratch* scratch, hipStream_t s) {
  const int64_t N = a.N, K = a.K, rows = a.by.rows;
  // chunks as gemm_grouped.hip's
  const bool direct = dtype == GCN_DT_BF16 && reinterpret_cast<uintptr_t>(a.b) % 16 == 0 &&
                      a.ldb % 8 == 0 && N % 8 == 0;
  const bool wide = N > 128 && K > 128 && rows / a.by.n >= 192 && direct;
  const int64_t tm = wide ? 256 : 128, tn = wide ? 256 : dtype == GCN_DT_F32 && N > 128 ? 256 : 128;
  const int64_t tiles = ceil_div(K, tm) * ceil_div(N, tn);
  const int64_t want = wide || tn == 256 ? 240 : 480;
  const double even = (double)rows * (double)tiles / (double)want;
  const double sums = std::sqrt(2e-4 * (double)rows * (double)K * (double)N);
  const double chunk = std::min(
      65536.0, std::max({256.0, sums, a.by.n * tiles < want ? std::min(even, 4096.0) : 4096.0}));
  a.split = ceil_div((int64_t)chunk, (int64_t)64) * 64;
  const int64_t parts = rows / a.split;
  if (parts > 0) GCN_CHECK(scratch->alloc(&a.part, parts * K * N, "grouped GEMM partials"));
  if (scratch->asked()) return GCN_OK;
  ProfScope ps("grouped_q8", s);
  if (dtype == GCN_DT_F32)
    GCN_CHECK((tn == 256 ? launch<float, false, 32, 2, 4, 2, 2>(a, s)
                         : launch<float, false, 32, 2, 2, 2, 2>(a, s)));
  else if (wide)
    GCN_CHECK((launch<bf16, true, 64, 4, 2, 2, 4>(a, s)));
  else
    GCN_CHECK((direct ? launch<bf16, true, 64, 2, 2, 2, 2>(a, s)
                      : launch<bf16, false, 64, 2, 2, 2, 2>(a, s)));
  return parts > 0 ? sum_group_partials(a.by, a.split, K, N, a.part, a.c, a.ldc, a.stride_c, s)
                   : GCN_OK;
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
           stride_w, 0, nullptr, 0, 0, 0};
  if (mul8_takes(a)) return mul8(a, dtype, &scratch, s);
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
