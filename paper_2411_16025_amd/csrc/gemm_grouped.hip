// bf16 products of rows sorted by group, on the matrix cores (gcn_gemm_grouped).

#include <algorithm>

#include "element.h"
#include "groups.h"

namespace gcn {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4u __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any element

#define GCN_GLOBAL __attribute__((address_space(1)))
#define GCN_LDS __attribute__((address_space(3)))

struct MulArgs {
  Groups by;
  int M, N, K;  // TN: C_g is M x N; else C is rows x N, K the inner size
  const bf16* A;
  int64_t lda;
  const bf16* B;
  int64_t ldb, stride_b;
  void* C;
  int64_t ldc, stride_c;
  int col_tiles, row_tiles;  // tiles along N, and (TN) along M
  int64_t slots, split;      // groups.h; TN: rows of a chunk
  float* part;               // TN: sums of the chunks behind the first ones
};

__device__ const u4 g_zeros = {0, 0, 0, 0};

// One operand's part of a stage: BK of the inner size by X rows of A (columns of B). KC: the
// inner size is contiguous in memory (A of NN and NT, B of NT): X lines of BK
// elements; else BK lines of X. A line is stored in 16-byte pieces, piece c at c ^ swz(line),
// so that the reads of neighbouring lines fall on different banks.
template <bool KC, int X, int BK>
struct Tile {
  static constexpr int kPieces = X * BK / 8;
  static constexpr int kPerLine = (KC ? BK : X) / 8;
  static constexpr int kBytes = kPieces * 16;
  __device__ static inline int swz(int line) {
    if constexpr (KC) return BK == 64 ? (line >> 1) & 7 : (line >> 2) & 3;
    return X >= 128 ? 4 * (line & 3) : (X == 64 ? 4 * ((line >> 1) & 1) : 0);
  }
  // What the lane reads of block blk (32 of X) and step (16 of BK): the 8 of the
  // inner size of operand row (lane % 32).
  __device__ static inline bf8 read(const char* base, int blk, int step, int lane) {
    if constexpr (KC) {
      const int line = lane & 31;
      const int at = line * (BK * 2) + (((lane >> 5) ^ swz(line)) * 16 ^ 32 * step);
      return *reinterpret_cast<const bf8*>(base + at + blk * 32 * BK * 2);
    } else {
      // the transposing read: of 16 lanes, lane i names 4 elements of line i / 4 and gets
      // element i of each of the 4 lines
      const int i = lane & 15, line = 8 * (lane >> 5) + (i >> 2);
      const int piece = 4 * blk + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
      const int at = line * (X * 2) + (piece ^ swz(line)) * 16 + (i & 1) * 8 + 16 * step * X * 2;
      const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (GCN_LDS s4*)(base + at));
      const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (GCN_LDS s4*)(base + at + 4 * X * 2));
      const s8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf8, v);
    }
  }
};

// The pieces of an operand that a thread brings to LDS: their offsets in memory from the
// operand's first element of a stage, and whether the stage's inner range has them.
// DIRECT: rows start on 16 bytes and hold whole pieces, and the loads go to LDS
// themselves; else through registers, element by element where a piece is not whole.
template <bool KC, int X, int BK, int NT, bool DIRECT>
struct Loader {
  using T = Tile<KC, X, BK>;
  static constexpr int kCount = (T::kPieces + NT - 1) / NT;
  const bf16* base;   // the operand's element (first of X, inner 0)
  int64_t ld;
  int have;           // of X inside the matrix
  uint32_t off[kCount];
  u4 v[DIRECT ? 1 : kCount];

  __device__ static inline bool mine(int p) {
    return T::kPieces % NT == 0 || (int)threadIdx.x + p * NT < T::kPieces;
  }
  __device__ inline void init(const bf16* b, int64_t ld_, int have_) {
    base = b;
    ld = ld_;
    have = have_;
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      const int s = threadIdx.x + p * NT, line = s / T::kPerLine;
      const int e = 8 * ((s % T::kPerLine) ^ T::swz(line));
      if constexpr (KC)
        off[p] = 2 * (uint32_t)((line < have ? line : have - 1) * (uint32_t)ld + e);
      else
        off[p] = 2 * (uint32_t)(line * (uint32_t)ld + (e < have || !DIRECT ? e : 0));
    }
  }
  // Pieces of the stage whose inner range begins at k0 and has `left` elements.
  __device__ inline void load(char* lds, int64_t k0, int64_t left) {
    const char* at = reinterpret_cast<const char*>(KC ? base + k0 : base + k0 * ld);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      if (!mine(p)) continue;
      const int s = threadIdx.x + p * NT, line = s / T::kPerLine;
      const int e = 8 * ((s % T::kPerLine) ^ T::swz(line));
      if constexpr (DIRECT) {
        const char* q = at + off[p];
        if (left < BK && (KC ? e : line) >= left) q = reinterpret_cast<const char*>(&g_zeros);
        __builtin_amdgcn_global_load_lds((const GCN_GLOBAL void*)q,
                                         (GCN_LDS void*)(lds + (w * 64 + p * NT) * 16), 16, 0, 0);
      } else {
        const bf16* q = reinterpret_cast<const bf16*>(at + off[p]);
        const int in = KC ? (int)std::min<int64_t>(left - e, 8)
                          : (line < left ? std::min(have - e, 8) : 0);
        u4 x = {0, 0, 0, 0};
        if (in >= 8) {
          x = *reinterpret_cast<const u4u*>(q);
        } else {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < in) x[j / 2] |= (uint32_t)h[j] << (16 * (j & 1));
        }
        v[p] = x;
      }
    }
  }
  __device__ inline void store(char* lds) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int p = 0; p < kCount; ++p)
        if (mine(p)) *reinterpret_cast<u4*>(lds + (threadIdx.x + p * NT) * 16) = v[p];
    }
  }
};

__device__ inline void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vector memory, that is the loads to LDS
  __syncthreads();
}

// A workgroup of WR x WC wavefronts, RB x CB blocks of 32 x 32 of C each.
template <int OP, class TC, bool DIRECT, int BK, int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_mul(MulArgs a) {
  constexpr bool AK = OP != GCN_GEMM_TN, BKC = OP == GCN_GEMM_NT;
  constexpr int NT = 64 * WR * WC, BM = 32 * WR * RB, BN = 32 * WC * CB;
  using TA = Tile<AK, BM, BK>;
  using TB = Tile<BKC, BN, BK>;
  __shared__ __align__(16) char a0[TA::kBytes], a1[TA::kBytes], b0[TB::kBytes], b1[TB::kBytes];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  // Each XCD takes a run of row slots, four of them beside each other over the columns:
  // the workgroups that run at a time share rows of A and columns of B in its L2.
  const int64_t per_xcd = (a.slots + 7) / 8, idx = blockIdx.x >> 3;
  int64_t slot;
  int ct, rt = 0;
  if constexpr (OP == GCN_GEMM_TN) {
    const int tiles = a.col_tiles * a.row_tiles;
    slot = (blockIdx.x & 7) * per_xcd + idx / tiles;
    rt = (int)(idx % tiles) / a.col_tiles;
    ct = (int)(idx % tiles) % a.col_tiles;
    if (idx / tiles >= per_xcd) return;
  } else {
    const int64_t band = idx / (4 * a.col_tiles), in = idx - band * 4 * a.col_tiles;
    const int64_t of = std::min<int64_t>(4, per_xcd - 4 * band);  // slots of the band
    if (of <= 0) return;
    if (in >= of * a.col_tiles) return;
    slot = (blockIdx.x & 7) * per_xcd + 4 * band + in % of;
    ct = (int)(in / of);
  }
  if (slot >= a.slots) return;
  const GroupTile gt = group_tile(a.by, slot, OP == GCN_GEMM_TN ? (int)a.split : BM);
  int64_t k_beg = 0, k_end = a.K;
  Loader<AK, BM, BK, NT, DIRECT> la;
  Loader<BKC, BN, BK, NT, DIRECT> lb;
  const int n0 = ct * BN;
  int64_t m0;     // first row of C, and the row behind the last one
  int64_t m_end;
  const bf16* B = a.B;
  if constexpr (OP == GCN_GEMM_TN) {
    if (gt.beg >= gt.end && gt.beg != gt.first) return;  // an empty group's first chunk: zeros
    k_beg = gt.beg;
    k_end = std::max(gt.beg, std::min(gt.beg + a.split, gt.end));
    m0 = rt * BM;
    m_end = a.M;
    la.init(a.A + m0, a.lda, (int)(m_end - m0));
  } else {
    m0 = gt.beg;
    m_end = gt.end;
    if (m0 >= m_end) return;
    B += gt.g * a.stride_b;
    la.init(a.A + m0 * a.lda, a.lda, (int)std::min<int64_t>(m_end - m0, BM));
  }
  if constexpr (BKC)
    lb.init(B + n0 * a.ldb, a.ldb, a.N - n0);
  else
    lb.init(B + n0, a.ldb, a.N - n0);

  f16 acc[RB][CB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  auto stage = [&](int64_t k, const char* ca, const char* cb, char* na, char* nb) {
    const bool more = k + BK < k_end;
    if (more) {
      la.load(na, k + BK, k_end - k - BK);
      lb.load(nb, k + BK, k_end - k - BK);
    }
#pragma unroll
    for (int st = 0; st < BK / 16; ++st) {
      bf8 fa[RB], fb[CB];
#pragma unroll
      for (int i = 0; i < RB; ++i) fa[i] = TA::read(ca, wr * RB + i, st, lane);
#pragma unroll
      for (int j = 0; j < CB; ++j) fb[j] = TB::read(cb, wc * CB + j, st, lane);
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
    if (more) {
      la.store(na);
      lb.store(nb);
    }
    wait_loads();
  };
  if (k_beg < k_end) {
    la.load(a0, k_beg, k_end - k_beg);
    lb.load(b0, k_beg, k_end - k_beg);
    la.store(a0);
    lb.store(b0);
    wait_loads();
  }
  for (int64_t k = k_beg; k < k_end; k += 2 * BK) {
    stage(k, a0, b0, a1, b1);
    if (k + BK < k_end) stage(k + BK, a1, b1, a0, b0);
  }

  TC* C = static_cast<TC*>(a.C);
  int64_t ldc = a.ldc;
  if constexpr (OP == GCN_GEMM_TN) {
    if (gt.beg != gt.first) {
      C = reinterpret_cast<TC*>(a.part) + (slot - gt.g - 1) * a.M * a.N;
      ldc = a.N;
    } else {
      C += gt.g * a.stride_c;
    }
  }
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t r = m0 + (wr * RB + i) * 32 + (e & 3) + 8 * (e >> 2) + 4 * (lane >> 5);
      TC* q = C + r * ldc;
#pragma unroll
      for (int j = 0; j < CB; ++j) {
        const int c = n0 + (wc * CB + j) * 32 + (lane & 31);
        if (r < m_end && c < a.N) q[c] = from_float<TC>(acc[i][j][e]);
      }
    }
}

template <int OP, class TC, bool DIRECT, int BK, int WR, int WC, int RB, int CB>
gcn_status launch(MulArgs a, hipStream_t s) {
  constexpr int BM = 32 * WR * RB, BN = 32 * WC * CB;
  a.col_tiles = (int)ceil_div((int64_t)a.N, (int64_t)BN);
  a.row_tiles = OP == GCN_GEMM_TN ? (int)ceil_div((int64_t)a.M, (int64_t)BM) : 1;
  a.slots = group_slots(a.by, OP == GCN_GEMM_TN ? a.split : BM);
  const int64_t blocks = ceil_div(a.slots, (int64_t)8) * 8 * a.col_tiles * a.row_tiles;
  GCN_CHECK(launch_fits(blocks, 64 * WR * WC));
  hipLaunchKernelGGL((k_mul<OP, TC, DIRECT, BK, WR, WC, RB, CB>), dim3((unsigned)blocks),
                     dim3(64 * WR * WC), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <int OP, class TC, bool DIRECT>
gcn_status mul(const MulArgs& a, hipStream_t s) {
  if (a.N > 128 && a.by.rows / a.by.n >= 192)
    return launch<OP, TC, DIRECT, 64, 2, 4, 4, 2>(a, s);
  return launch<OP, TC, DIRECT, 64, 2, 2, 2, 2>(a, s);
}

bool aligned16(const void* p, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0;
}

}  // namespace

bool gemm_grouped_bf16_takes(int64_t lda, int64_t ldb) {
  return lda < (int64_t(1) << 22) && ldb < (int64_t(1) << 22);
}

gcn_status gemm_grouped_bf16(int op, const Groups& g, int64_t N, int64_t K, const void* A,
                             int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc,
                             bool c_bf16, int64_t stride_w, hipStream_t s) {
  MulArgs a{};
  a.by = g;
  a.A = static_cast<const bf16*>(A);
  a.lda = lda;
  a.B = static_cast<const bf16*>(B);
  a.ldb = ldb;
  a.C = C;
  a.ldc = ldc;
  a.N = (int)N;
  const bool rows_ok = aligned16(A, lda) && aligned16(B, ldb);
  if (op == GCN_GEMM_TN) {
    a.M = (int)K;
    a.stride_c = stride_w;
    a.split = 2048;
    TempScope temps(s);
    const int64_t parts = g.rows / a.split;
    if (parts > 0) GCN_CHECK(temps.alloc(&a.part, parts * K * N, "grouped GEMM partials"));
    GCN_CHECK(rows_ok && K % 8 == 0 && N % 8 == 0 ? (mul<GCN_GEMM_TN, float, true>(a, s))
                                                  : (mul<GCN_GEMM_TN, float, false>(a, s)));
    return parts > 0 ? sum_group_partials(g, a.split, K, N, a.part, static_cast<float*>(C), ldc,
                                          stride_w, s)
                     : GCN_OK;
  }
  a.K = (int)K;
  a.stride_b = stride_w;
  const bool direct = rows_ok && K % 8 == 0 && stride_w % 8 == 0 &&
                      (op == GCN_GEMM_NT || N % 8 == 0);
  auto go = [&](auto kernel_nn, auto kernel_nt) {
    return op == GCN_GEMM_NN ? kernel_nn(a, s) : kernel_nt(a, s);
  };
  if (direct)
    return c_bf16 ? go(mul<GCN_GEMM_NN, bf16, true>, mul<GCN_GEMM_NT, bf16, true>)
                  : go(mul<GCN_GEMM_NN, float, true>, mul<GCN_GEMM_NT, float, true>);
  return c_bf16 ? go(mul<GCN_GEMM_NN, bf16, false>, mul<GCN_GEMM_NT, bf16, false>)
                : go(mul<GCN_GEMM_NN, float, false>, mul<GCN_GEMM_NT, float, false>);
}

}  // namespace gcn
