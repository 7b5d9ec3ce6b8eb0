// bf16 products of rows sorted by group, on the matrix cores (gcn_gemm_grouped).
//
// C = A B_g, A B_g^T or (TN) C_g = A_g^T B_g, products exact, sums in fp32, one rounding. The
// matrix cores bound it where the inner size is long: a wavefront has 64 x 128 of C, so that a
// step's 6 fragments feed 8 instructions, and eight of them share 256 x 256 x 64 in LDS, which
// direct loads fill (through registers 430 TFLOP/s instead of 900). The operand whose inner size
// is not contiguous is transposed by the reads from LDS. 8192^3 in one group: 1250 to 1300
// TFLOP/s, a library product 1380; 32,768 rows of 16 ragged groups, 2048 x 4096: 925 to 985 (the
// tiles of rows that do not fill them, and the last round of tiles). Few steps, or short groups:
// the bytes of B and C (16,384 rows of 64 groups, 1024 x 512: 49 us for dX, 58 for dW; 38 and 43
// with the operands in the last cache).

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "element.h"
#include "groups.h"

namespace gcn {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u2a __attribute__((ext_vector_type(2), aligned(2)));  // 8 bytes at any element
typedef Unaligned<bf16>::type u4u;  // 16 bytes at any element

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
  uint32_t slots;            // groups.h
  int64_t split;             // TN: rows of a chunk
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
// operand's first element of a stage. DIRECT: rows start on 16 bytes and hold whole
// pieces, and the loads go to LDS themselves. Else through registers, without a branch between
// the loads: a piece that reaches over a row's end is read from 8 elements before the end
// on (rows have 8) and moved down when it is stored.
template <bool KC, int X, int BK, int NT, bool DIRECT>
struct Loader {
  using T = Tile<KC, X, BK>;
  static constexpr int kCount = T::kPieces / NT;
  static_assert(T::kPieces % NT == 0, "every thread has as many pieces");
  const bf16* base;   // the operand's element (first of X, inner 0)
  int64_t ld;
  int have;           // of X inside the matrix
  int64_t had;        // of the inner size, in the stage whose pieces are in v
  uint32_t off[kCount];
  u4 v[DIRECT ? 1 : kCount];

  __device__ static inline int line_of(int p) { return (int)(threadIdx.x + p * NT) / T::kPerLine; }
  __device__ static inline int element_of(int p) {  // of its line, a multiple of 8
    return 8 * (((int)(threadIdx.x + p * NT) % T::kPerLine) ^ T::swz(line_of(p)));
  }
  __device__ inline void init(const bf16* b, int64_t ld_, int have_) {
    base = b;
    ld = ld_;
    have = have_;
#pragma unroll
    for (int p = 0; p < kCount; ++p) {
      const int line = line_of(p), e = element_of(p);
      if constexpr (KC)
        off[p] = 2 * ((line < have ? line : have - 1) * (uint32_t)ld + e);
      else if constexpr (DIRECT)
        off[p] = 2 * (line * (uint32_t)ld + (e < have ? e : 0));
      else  // (from the first of X - 8, which may lie before the tile)
        off[p] = 2 * (line * (uint32_t)ld + (uint32_t)(std::min(e, have - 8) + 8));
    }
  }
  // Pieces of the stage whose inner range begins at k0 and has `left` elements.
  __device__ inline void load(char* lds, int64_t k0, int64_t left) {
    const char* at = reinterpret_cast<const char*>(KC ? base + k0 : base + k0 * ld);
    if constexpr (DIRECT) {
      const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int p = 0; p < kCount; ++p) {
        const char* q = at + off[p];
        if (left < BK && (KC ? element_of(p) : line_of(p)) >= left)
          q = reinterpret_cast<const char*>(&g_zeros);
        __builtin_amdgcn_global_load_lds((const GCN_GLOBAL void*)q,
                                         (GCN_LDS void*)(lds + (w * 64 + p * NT) * 16), 16, 0, 0);
      }
    } else {
      had = left;
      if (left <= 0) return;  // past the last stage
      if (!KC) at -= 16;
      if (left >= BK) {
#pragma unroll
        for (int p = 0; p < kCount; ++p)
          v[p] = *reinterpret_cast<const u4u*>(at + off[p]);
      } else {
#pragma unroll
        for (int p = 0; p < kCount; ++p) {
          const int over = KC ? element_of(p) - (int)left + 8 : line_of(p) - (int)left + 1;
          const char* q = at + off[p];
          if (over > 0) q -= KC ? 2 * (int64_t)over : 2 * over * ld;
          v[p] = *reinterpret_cast<const u4u*>(q);
        }
      }
    }
  }
  __device__ inline void store(char* lds) {
    if constexpr (!DIRECT) {
      const bool whole = had >= BK && (KC || have >= X);
#pragma unroll
      for (int p = 0; p < kCount; ++p) {
        u4 x = v[p];
        if (!whole) {
          const int64_t over = (KC ? element_of(p) - had : (int64_t)element_of(p) - have) + 8;
          x = move_down<bf16>(x, (int)std::min<int64_t>(8, std::max<int64_t>(0, over)));
          if (!KC && line_of(p) >= had) x = u4{0, 0, 0, 0};
        }
        *reinterpret_cast<u4*>(lds + (threadIdx.x + p * NT) * 16) = x;
      }
    }
  }
};

// The loads to LDS are done, but for the last N of a thread, for all wavefronts.
template <int N = 0>
__device__ inline void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4 << 14));  // vector memory
  __syncthreads();
}

// Lane l of 4 has four rows' values of column l; it gets the four columns of row l as bf16.
__device__ inline u2 quad_rows(float r0, float r1, float r2, float r3) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  const uint32_t p0 = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{r0, r1}), bf2));
  const uint32_t p1 = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{r2, r3}), bf2));
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
  // with lane l ^ 1: rows 0, 2 (even lanes) or 1, 3 of two columns
  const uint32_t q0 = __builtin_amdgcn_mov_dpp(p0, 0xB1, 0xF, 0xF, false);
  const uint32_t q1 = __builtin_amdgcn_mov_dpp(p1, 0xB1, 0xF, 0xF, false);
  const uint32_t sel = odd ? 0x03020706u : 0x05040100u;
  const uint32_t w0 = __builtin_amdgcn_perm(q0, p0, sel), w1 = __builtin_amdgcn_perm(q1, p1, sel);
  // with lane l ^ 2: row 0 or 1 (lower lanes) or 2 or 3 of four columns
  const uint32_t t = __builtin_amdgcn_mov_dpp(high ? w0 : w1, 0x4E, 0xF, 0xF, false);
  return high ? u2{t, w1} : u2{w0, t};
}

// A workgroup of WR x WC wavefronts, RB x CB blocks of 32 x 32 of C each.
template <int OP, class TC, bool DIRECT, int BK, int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, RB * CB > 8 ? 1 : 2) void k_mul(MulArgs a) {
  constexpr bool AK = OP != GCN_GEMM_TN, BKC = OP == GCN_GEMM_NT;
  constexpr int NT = 64 * WR * WC, BM = 32 * WR * RB, BN = 32 * WC * CB;
  using TA = Tile<AK, BM, BK>;
  using TB = Tile<BKC, BN, BK>;
  // an array per buffer: the compiler then knows that reads of one need not wait for the
  // loads to another
  __shared__ __align__(16) char a0[TA::kBytes], a1[TA::kBytes], b0[TB::kBytes], b1[TB::kBytes];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  // The tiles, chunk by chunk (TN) or in bands of four row tiles beside each other over the
  // columns, divide evenly among the XCDs: the workgroups that run at a time on one share
  // rows of A and columns of B in its L2.
  constexpr int LEAST = OP == GCN_GEMM_TN ? 1 : 0;  // an empty group's C is zero
  const int R = OP == GCN_GEMM_TN ? (int)a.split : BM;
  const bool counted = a.by.n <= kCountedGroups;
  TileCount count{};
  if (counted) count = count_tiles(a.by, R, LEAST);
  const uint32_t rows = counted ? count.total : a.slots;
  const uint32_t per_row = a.col_tiles * a.row_tiles, units = rows * per_row, xcd = blockIdx.x & 7;
  const uint32_t u = (uint32_t)((uint64_t)units * xcd / 8) + (blockIdx.x >> 3);
  if (u >= (uint32_t)((uint64_t)units * (xcd + 1) / 8)) return;
  uint32_t slot;
  int ct, rt = 0;
  if constexpr (OP == GCN_GEMM_TN) {
    slot = u / per_row;
    rt = (int)(u % per_row) / a.col_tiles;
    ct = (int)(u % per_row) % a.col_tiles;
  } else {
    const uint32_t band = u / (4 * per_row), in = u - band * 4 * per_row;
    const uint32_t of = std::min(4u, rows - 4 * band);  // row tiles of the band
    slot = 4 * band + in % of;
    ct = (int)(in / of);
  }
  const GroupTile gt = counted ? counted_tile(a.by, count, (int)slot, R, LEAST)
                               : group_tile(a.by, slot, R);
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

  // Fragments of a step are read while the step before it is multiplied; the first ones of
  // the next stage too, so the one barrier of a stage stands before its last step: all
  // have read the stage's last fragments then, and the next stage is in LDS.
  constexpr int STEPS = BK / 16;
  static_assert(STEPS % 2 == 0, "the fragments' buffers alternate over the stages");
  bf8 fa[2][RB], fb[2][CB];
  auto read = [&](int to, int step, const char* ca, const char* cb) {
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[to][i] = TA::read(ca, wr * RB + i, step, lane);
#pragma unroll
    for (int j = 0; j < CB; ++j) fb[to][j] = TB::read(cb, wc * CB + j, step, lane);
  };
  // One or two LDS reads between two products.
  constexpr int READS = (AK ? 1 : 2) * RB + (BKC ? 1 : 2) * CB;
  auto multiply = [&](int from) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
        acc[i][j] =
            __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[from][i], fb[from][j], acc[i][j], 0, 0, 0);
#pragma unroll
    for (int p = 0; p < RB * CB; ++p) {
      __builtin_amdgcn_sched_group_barrier(0x100, (READS + RB * CB - 1) / (RB * CB), 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    }
  };
  const int64_t stages = (k_end - k_beg + BK - 1) / BK;
  auto load = [&](int64_t s, char* la_to, char* lb_to) {
    const int64_t k = k_beg + s * BK;
    la.load(la_to, k, k_end - k);
    lb.load(lb_to, k, k_end - k);
  };
  // stage s has been read from (ca, cb): stage s + 1, in (na, nb) or on its way there, is waited
  // for, and stage s + 2 goes to (ca, cb) (past the last one, zeros)
  auto pass_on = [&](int64_t s, char* ca, char* cb, char* na, char* nb) {
    la.store(na);
    lb.store(nb);
    wait_loads();
    load(s + 2, ca, cb);
  };
  auto stage = [&](int64_t s, char* ca, char* cb, char* na, char* nb) {
#pragma unroll
    for (int st = 0; st + 1 < STEPS; ++st) {
      read((st + 1) & 1, st + 1, ca, cb);
      multiply(st & 1);
    }
    pass_on(s, ca, cb, na, nb);
    read(0, 0, na, nb);
    multiply((STEPS - 1) & 1);
  };
  if (stages > 0) {
    load(0, a0, b0);
    la.store(a0);
    lb.store(b0);
    load(1, a1, b1);
    wait_loads<DIRECT ? decltype(la)::kCount + decltype(lb)::kCount : 63>();
    if (m0 + wr * RB * 32 >= m_end) {  // no rows for this wavefront: it brings its part only
      for (int64_t s = 0; s < stages; s += 2) {
        pass_on(s, a0, b0, a1, b1);
        if (s + 1 < stages) pass_on(s + 1, a1, b1, a0, b0);
      }
      wait_loads();
      return;
    }
    read(0, 0, a0, b0);
    for (int64_t s = 0; s < stages; s += 2) {
      stage(s, a0, b0, a1, b1);
      if (s + 1 >= stages) break;
      stage(s + 1, a1, b1, a0, b0);
    }
    wait_loads();  // those past the last stage
  }

  TC* C = static_cast<TC*>(a.C);
  int64_t ldc = a.ldc;
  if constexpr (OP == GCN_GEMM_TN) {
    if (gt.beg != gt.first) {
      C = reinterpret_cast<TC*>(a.part) +
          (gt.first / a.split + (gt.beg - gt.first) / a.split - 1) * a.M * a.N;
      ldc = a.N;
    } else {
      C += gt.g * a.stride_c;
    }
  }
  auto write = [&](auto past) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j) {
        const int64_t r0 = m0 + (wr * RB + i) * 32 + 4 * (lane >> 5);
        const int c0 = n0 + (wc * CB + j) * 32;
        if constexpr (sizeof(TC) == 4) {
          const int c = c0 + (lane & 31);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int64_t r = r0 + (e & 3) + 8 * (e >> 2);
            float* q = reinterpret_cast<float*>(C) + r * ldc + c;
            if (r >= m_end || c >= a.N) continue;
            if constexpr (decltype(past)::value)
              __builtin_nontemporal_store(acc[i][j][e], q);
            else
              *q = acc[i][j][e];
          }
        } else {
          // 4 x 4 values of 4 lanes change places, so that a lane has 4 columns of a row (one
          // 8-byte store instead of 4 of 2 bytes)
          const int c = c0 + (lane & 28);
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const int64_t r = r0 + (lane & 3) + 2 * e;
            const u2 v = quad_rows(acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]);
            if (r >= m_end) continue;
            uint16_t* q = reinterpret_cast<uint16_t*>(C) + r * ldc + c;
            if (c + 4 <= a.N) {
              if constexpr (decltype(past)::value)
                __builtin_nontemporal_store(v, reinterpret_cast<u2a*>(q));
              else
                *reinterpret_cast<u2a*>(q) = v;
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (c + k < a.N) q[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
            }
          }
        }
      }
  };
  // C past the caches, which hold A and B for the workgroups that still read them (32,768 x 4096 x
  // 2048, one group: 521 us, 490 so), but only where its rows fill whole lines: parts of lines
  // wait in the caches for the rest (300,000 rows of 4 groups, 48 x 252: 122 us past them, 43).
  if (((reinterpret_cast<uintptr_t>(C) | (uintptr_t)(ldc * (int64_t)sizeof(TC))) & 127) == 0)
    write(std::true_type{});
  else
    write(std::false_type{});
}

template <int OP, class TC, bool DIRECT, int BK, int WR, int WC, int RB, int CB>
gcn_status launch(MulArgs a, hipStream_t s) {
  constexpr int BM = 32 * WR * RB, BN = 32 * WC * CB;
  a.col_tiles = (int)ceil_div((int64_t)a.N, (int64_t)BN);
  a.row_tiles = OP == GCN_GEMM_TN ? (int)ceil_div((int64_t)a.M, (int64_t)BM) : 1;
  const int64_t slots = group_slots(a.by, OP == GCN_GEMM_TN ? a.split : BM);
  const int64_t blocks = ceil_div(slots * a.col_tiles * a.row_tiles, (int64_t)8) * 8;
  GCN_CHECK(launch_fits(blocks, 64 * WR * WC));
  a.slots = (uint32_t)slots;
  hipLaunchKernelGGL((k_mul<OP, TC, DIRECT, BK, WR, WC, RB, CB>), dim3((unsigned)blocks),
                     dim3(64 * WR * WC), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

// Columns for more than one 128-wide tile, and rows to a group that fill a 256-high one mostly.
// Operands that are brought through registers have none left for tiles of 256 x 256.
inline bool wide_tiles(const Groups& g, int64_t N) { return N > 128 && g.rows / g.n >= 192; }

// The shape of a workgroup's tile: 256 x 256 of wide products, else 128 x 128. With a short inner
// size smaller tiles, several to a CU, whose stores the others' products hide: 128 x
// 256 (100,000 rows of 4 groups, 512 x 1024: 148 us, 128 x 128 152; 256 x 256 12 more; but 32,768
// rows of 16 groups, 2048 x 4096: 616 us and 593 in 256 x 256), and 128 x 128 where it is
// shorter still or groups end inside many tiles (100,000 rows, 256 x 256: 31 us and 34; 16,384 rows of
// 64 groups, 512 x 1024: 38 and 40).
template <int OP, class TC, bool DIRECT>
gcn_status mul(const MulArgs& a, hipStream_t s) {
  const bool wide = wide_tiles(a.by, a.N);
  if constexpr (OP != GCN_GEMM_TN)
    if (wide && a.K < 1024) {
      if (a.K < 512 || a.by.rows / a.by.n < 1024)
        return launch<OP, TC, DIRECT, 32, 2, 2, 2, 2>(a, s);
      return launch<OP, TC, DIRECT, 32, 2, 2, 2, 4>(a, s);
    }
  if constexpr (DIRECT)
    if (wide) return launch<OP, TC, true, 64, 4, 2, 2, 4>(a, s);
  return launch<OP, TC, DIRECT, 64, 2, 2, 2, 2>(a, s);
}

// Rows of 8-element pieces that start on 16 bytes.
struct Operand {
  const bf16* p;
  int64_t ld, stride;   // of rows, of the groups' matrices
  int64_t groups, rows, cols;
  bool direct() const {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 &&
           (groups == 1 || stride % 8 == 0);
  }
  int64_t pieces() const { return groups * rows * ((cols + 7) / 8); }
};

__global__ __launch_bounds__(256) void k_pad(Operand o, u4* out) {
  const uint32_t per = (uint32_t)((o.cols + 7) / 8);
  const uint32_t t = blockIdx.x * 256 + threadIdx.x;
  if (t >= o.groups * o.rows * per) return;
  const uint32_t line = t / per, f = 8 * (t % per), g = line / (uint32_t)o.rows;
  out[t] = load_piece(o.p + g * o.stride + (line - g * o.rows) * o.ld, (int)f, (int)o.cols);
}

// Whether both operands can be loaded directly, after copies of those that cannot, with rows
// padded with zeros to whole pieces, where the product is large against them: of odd sizes a
// product runs at about 430 TFLOP/s through registers and 900 directly, and a copy moves 32
// bytes a piece (32,768 rows of 16 groups, 2047 x 4093: 766 us, 1290 without). Without memory for
// the copies it stays with the registers; meant: whether the sizes alone call for direct loads, so
// that what decides the order of the sums does not depend on the memory.
gcn_status make_direct(Operand* a, Operand* b, double work, Scratch* scratch, bool* direct,
                       bool* meant, hipStream_t s) {
  int64_t pieces = 0;
  for (Operand* o : {a, b})
    if (!o->direct()) pieces += o->pieces();
  *direct = *meant = pieces == 0;
  if (*direct || work < 0x1p34 || work / 2048 < (double)pieces || pieces >= (int64_t(1) << 31))
    return GCN_OK;
  *meant = true;
  u4* to = nullptr;
  if (scratch->alloc(&to, pieces, "aligned copies of operands") != GCN_OK) {
    clear_error();
    return GCN_OK;
  }
  *direct = true;
  if (scratch->asked()) return GCN_OK;
  for (Operand* o : {a, b}) {
    if (o->direct()) continue;
    hipLaunchKernelGGL(k_pad, dim3((unsigned)ceil_div(o->pieces(), (int64_t)256)), dim3(256), 0, s,
                       *o, to);
    GCN_HIP(hipGetLastError());
    const bf16* copy = reinterpret_cast<const bf16*>(to);
    to += o->pieces();
    o->p = copy;
    o->ld = (o->cols + 7) / 8 * 8;
    o->stride = o->rows * o->ld;
  }
  return GCN_OK;
}

}  // namespace

bool gemm_grouped_bf16_takes(int64_t N, int64_t K, int64_t lda, int64_t ldb) {
  return N >= 8 && K >= 8 && lda < (int64_t(1) << 22) && ldb < (int64_t(1) << 22);
}

gcn_status gemm_grouped_bf16(int op, const Groups& g, int64_t N, int64_t K, const void* A,
                             int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc,
                             bool c_bf16, int64_t stride_w, Scratch* scratch, hipStream_t s) {
  const bool tn = op == GCN_GEMM_TN;
  Operand oa{static_cast<const bf16*>(A), lda, 0, 1, g.rows, K}, ob = oa;
  ob.p = static_cast<const bf16*>(B);
  ob.ld = ldb;
  ob.cols = op == GCN_GEMM_NT ? K : N;
  if (!tn) {
    ob.stride = stride_w;
    ob.groups = stride_w == 0 ? 1 : g.n;
    ob.rows = op == GCN_GEMM_NT ? N : K;
  }
  bool direct = false, meant = false;
  GCN_CHECK(make_direct(&oa, &ob, (double)g.rows * (double)N * (double)K, scratch, &direct, &meant, s));
  MulArgs a{};
  a.by = g;
  a.A = oa.p;
  a.lda = oa.ld;
  a.B = ob.p;
  a.ldb = ob.ld;
  a.stride_b = stride_w == 0 ? 0 : ob.stride;
  a.C = C;
  a.ldc = ldc;
  a.N = (int)N;
  if (tn) {
    a.M = (int)K;
    a.stride_c = stride_w;
    // Chunks of rows for one workgroup of 256 x 256 of C to a CU or two of 128 x 128, up to 4096
    // (500,000 rows of 4 groups, 256 x 256: 122 us, with two to a CU and twice the partial sums
    // 172); where the groups' tiles are enough by themselves, 4096 bound the work of one
    // (16,384 rows of 64 groups, 512 x 512: 26 us, 76 in chunks of 320). But a chunk costs time by
    // its rows, and the partial sums by K N to each: their sum is least at a root of rows K N
    // (65,536 rows of 64 groups, 256 x 256: 44 us, 53 without that bound; 32,768 of 8, 1024 x
    // 1024: 107 and 152; 65,536 of 8, 2048 x 4096: 1.35 ms and 1.57; but 500,000 of 4, 512 x 512:
    // 345 us and 320). 65536 rows bound the sums' chains.
    const int64_t tile = meant && wide_tiles(g, N) ? 256 : 128, want = tile == 256 ? 240 : 480;
    const int64_t tiles = ceil_div(K, tile) * ceil_div(N, tile);
    const double even = (double)g.rows * (double)tiles / (double)want;  // a chunk to each
    const double sums = std::sqrt(2e-4 * (double)g.rows * (double)K * (double)N);
    const double chunk = std::min(
        65536.0, std::max({256.0, sums, g.n * tiles < want ? std::min(even, 4096.0) : 4096.0}));
    a.split = ceil_div((int64_t)chunk, (int64_t)64) * 64;
    const int64_t parts = g.rows / a.split;
    if (parts > 0) GCN_CHECK(scratch->alloc(&a.part, parts * K * N, "grouped GEMM partials"));
    if (scratch->asked()) return GCN_OK;
    GCN_CHECK(direct ? (mul<GCN_GEMM_TN, float, true>(a, s))
                     : (mul<GCN_GEMM_TN, float, false>(a, s)));
    return parts > 0 ? sum_group_partials(g, a.split, K, N, a.part, static_cast<float*>(C), ldc,
                                          stride_w, s)
                     : GCN_OK;
  }
  if (scratch->asked()) return GCN_OK;
  a.K = (int)K;
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
