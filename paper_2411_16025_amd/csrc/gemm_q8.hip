// Weight gradients from rows kept in 8 bits: C_g = X_g^T B_g (gcn_gemm_grouped_q8).
//
// The codes' values are exact in bf16, so they are decoded on their way to LDS, and the product is that
// of bf16 rows (gemm_grouped.hip), or of one bf16 operand with the three parts of an fp32 one
// (gemm_split.hip). Decoding takes 2.5 instructions an element of X for every 256 columns of B;
// between the products it costs little. bf16, 32,768 rows of 16 ragged groups, 2048 x 4096: 595 to 637 us,
// 41% of the cycles in the matrix cores; in one group 918 TFLOP/s. fp32, 500,000 rows of
// 4 groups, 100 x 256: 143 to 150 us, bound by its bytes (3.9 to 4.2 TB/s).

#include <algorithm>
#include <cmath>
#include <type_traits>

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
  bool by_chunk;  // each chunk's tiles on one XCD; else every XCD has a rectangle of them,
  int across;     // so many beside each other, of rect_rows x rect_cols (across 0: an eighth of them in a row)
  int rect_rows, rect_cols;
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

// The values of eight codes, exact in bf16: a signed byte becomes fp32 in one instruction, its product with
// the unit is another. (Unsigned bytes less an offset of 128 units would take as many, but at the largest unit,
// 2^121, that offset is no fp32 number. With 0 added: of plain products the compiler forms a stage's early and
// spills 27 registers of the 256 x 256 tile, 790 us for the 607 of the ragged groups above; signed bytes
// as unsigned ones less 128, times the unit: 635.)
__device__ inline u4 decode8(uint32_t c0, uint32_t c1, float unit) {
  u4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t c = i ? c1 : c0;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf((float)(int8_t)(c >> (8 * e)), unit, 0.f);
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

// A workgroup's part of C and its chunk of a group's rows.
struct Place {
  bool any, whole;  // whether there is one; whether the chunk is the whole group
  int m0, n0, g;
  int64_t first, beg, end, chunk;
};

// Chunk `slot` of at most 64 groups, the long groups first: lane l has group l's chunks, those of
// the groups before it are counted by their sizes.
__device__ inline GroupTile long_first(const Groups& by, const TileCount& c, int slot, int R) {
  const int lane = threadIdx.x & 63;
  const int size = lane < by.n ? (int)std::max<int64_t>(0, c.end - c.first) : -1;
  const int mine = lane < by.n ? tiles_of(size, R, 1) : 0;
  int before = 0;
  for (int o = 0; o < by.n; ++o) {
    const int so = __builtin_amdgcn_readlane(size, o), to = __builtin_amdgcn_readlane(mine, o);
    before += so > size || (so == size && o < lane) ? to : 0;
  }
  const uint64_t at = __ballot(lane < by.n && before <= slot && slot < before + mine);
  const int l = at ? 63 - __clzll((long long)at) : 0;
  GroupTile r;
  r.g = l;
  r.first = lane_value(c.first, l);
  r.end = lane_value(c.end, l);
  r.beg = r.first + (int64_t)(slot - __builtin_amdgcn_readlane(before, l)) * R;
  return r;
}

// Of few chunks the XCDs share every one's tiles, of many (or with fewer than eight tiles) each has
// whole chunks, which it reads once; long groups come first. 16 groups of 100 to 5,000 rows, 2048 x 4096:
// 1128 us where each XCD had an eighth of all tiles in the groups' order, the XCDs of the long ones the
// most work.
__device__ inline Place place(const Q8Args& a, int BM, int BN) {
  Place r{};
  const int R = (int)a.split;
  const bool counted = a.by.n <= kCountedGroups;
  TileCount count{};
  if (counted) count = count_tiles(a.by, R, 1);
  const uint32_t slots = counted ? count.total : a.slots;
  const uint32_t per = a.col_tiles * a.row_tiles, share = (per + 7) / 8, xcd = blockIdx.x & 7;
  uint32_t slot, t;
  if (!a.by_chunk) {
    slot = (blockIdx.x >> 3) / share;
    const uint32_t x = (xcd + slot) & 7;  // (which XCD has one tile less than others changes)
    const uint32_t in = (blockIdx.x >> 3) % share;
    if (a.across > 0) {
      const int row = (int)x / a.across * a.rect_rows + (int)in / a.rect_cols;
      const int col = (int)x % a.across * a.rect_cols + (int)in % a.rect_cols;
      if (row >= a.row_tiles || col >= a.col_tiles) return r;
      t = row * a.col_tiles + col;
    } else {
      t = per * x / 8 + in;
      if (t >= per * (x + 1) / 8) return r;
    }
  } else {
    const uint32_t turn = blockIdx.x / (8 * per);  // there and back, as the chunks get shorter
    slot = turn * 8 + (turn & 1 ? 7 - xcd : xcd);
    t = (blockIdx.x >> 3) % per;
  }
  if (slot >= slots) return r;
  const GroupTile gt = a.by.n <= 64 ? long_first(a.by, count, (int)slot, R)
                       : counted    ? counted_tile(a.by, count, (int)slot, R, 1)
                                    : group_tile(a.by, slot, R);
  if (gt.beg >= gt.end && gt.beg != gt.first) return r;  // an empty group's first chunk: zeros
  r.any = true;
  r.whole = gt.end - gt.first <= R;
  r.m0 = (int)t / a.col_tiles * BM;
  r.n0 = (int)t % a.col_tiles * BN;
  r.g = gt.g;
  r.first = gt.first;
  r.beg = gt.beg;
  r.end = std::max(gt.beg, std::min(gt.beg + a.split, gt.end));
  r.chunk = (gt.beg - gt.first) / a.split;
  return r;
}

// A wavefront's sums, times `down`, to C or to the chunk's partial sums (with 0 added to the
// product: -0 becomes +0).
template <int RB, int CB>
__device__ inline void write_sums(const Q8Args& a, const Place& pl, int m0, int n0,
                                  const f16 (*acc)[CB], float down) {
  float* C = a.c + pl.g * a.stride_c;
  int64_t ldc = a.ldc;
  if (pl.chunk > 0) {
    C = a.part + (pl.first / a.split + pl.chunk - 1) * a.K * a.N;
    ldc = a.N;
  }
  const int lane = threadIdx.x & 63;
  // (addresses: a uniform row, and the lane's part in 32 bits)
  const uint32_t lane_at = (uint32_t)(4 * (lane >> 5)) * (uint32_t)ldc + (lane & 31);
  auto write = [&](auto past) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = m0 + i * 32 + (e & 3) + 8 * (e >> 2);
        float* row = C + r * ldc + n0;
        if (r + 4 * (lane >> 5) >= a.K) continue;
#pragma unroll
        for (int j = 0; j < CB; ++j) {
          if (n0 + j * 32 + (lane & 31) >= a.N) continue;
          const float v = __builtin_fmaf(acc[i][j][e], down, 0.f);
          if constexpr (decltype(past)::value)
            __builtin_nontemporal_store(v, row + lane_at + j * 32);
          else
            row[lane_at + j * 32] = v;
        }
      }
  };
  // past the caches where rows are whole lines, as in gemm_grouped.hip, and no partial sums are added
  // (32,768 rows of 8 groups in 16 chunks, 1024 x 1024: 139 us with those past the caches, 128)
  if (pl.whole && ((reinterpret_cast<uintptr_t>(C) | (uintptr_t)(4 * ldc)) & 127) == 0)
    write(std::true_type{});
  else
    write(std::false_type{});
}

// A workgroup of WR x WC wavefronts, RB x CB blocks of 32 x 32 of C each.
// bf16 rows of any alignment.
template <int BK, int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_mul8(Q8Args a) {
  constexpr int NT = 64 * WR * WC, BM = 32 * WR * RB, BN = 32 * WC * CB;
  using LA = CodeLoader<BM, BK, NT>;
  using LB = Loader<false, BN, BK, NT, false>;
  using TA = Tile<false, BM, BK>;
  using TN = Tile<false, BN, BK>;
  __shared__ __align__(16) char a0[TA::kBytes], a1[TA::kBytes], b0[TN::kBytes], b1[TN::kBytes];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  const Place pl = place(a, BM, BN);
  if (!pl.any) return;
  const int m0 = pl.m0, n0 = pl.n0;
  const int64_t k_beg = pl.beg, k_end = pl.end;
  LA la;
  LB lb;
  la.init(a.q + m0, a.ldq, a.s + m0 / 32, a.lds, a.K - m0);
  lb.init(static_cast<const bf16*>(a.b) + n0, a.ldb, a.N - n0);
  // (the matrix core's rounding has one sign: every other chunk's sums are of negated products)
  const uint32_t sign = pl.chunk & 1 ? 0x80000000u : 0;

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
  bf8 fa[2][RB], fb[2][CB];
  auto read = [&](int to, int step, const char* ca, const char* cb) {
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[to][i] = TA::read(ca, wr * RB + i, step, lane);
#pragma unroll
    for (int j = 0; j < CB; ++j) fb[to][j] = TN::read(cb, wc * CB + j, step, lane);
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
        acc[i][j] =
            __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[from][i], fb[from][j], acc[i][j], 0, 0, 0);
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
    wait_loads<63>();
    read(0, 0, a0, b0);
    for (int64_t s = 0; s < stages; s += 2) {
      stage(s, a0, b0, a1, b1);
      if (s + 1 >= stages) break;
      stage(s + 1, a1, b1, a0, b0);
    }
    wait_loads();  // those past the last stage
  }

  write_sums<RB, CB>(a, pl, m0 + wr * RB * 32, n0 + wc * CB * 32, acc, pl.chunk & 1 ? -1.f : 1.f);
}

// bf16 rows that start on 16 bytes and hold whole pieces. The codes' way to LDS is through
// registers, three stages long, so that decoding them (20 vector instructions for 8) stands between
// the products of the stage before theirs: their loads are issued with the direct loads of the
// other operand, waited for with them one stage later, and decoded during the next one. No branch
// divides a stage: past the last one its loads are repeated, rows past the chunk's end have a unit of
// 0 and a piece of zeros. ODD: rows of codes that do not end with a unit of 16.
template <bool ODD, int BK, int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_mul8_direct(Q8Args a) {
  constexpr int NT = 64 * WR * WC, BM = 32 * WR * RB, BN = 32 * WC * CB;
  using TA = Tile<false, BM, BK>;
  using TN = Tile<false, BN, BK>;
  constexpr int UA = BM * BK / 16 / NT, PB = TN::kPieces / NT;  // units, pieces of a thread
  static_assert(BM * BK / 16 % NT == 0 && TN::kPieces % NT == 0, "every thread has as many");
  __shared__ __align__(16) char a0[TA::kBytes], a1[TA::kBytes], b0[TN::kBytes], b1[TN::kBytes];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  const Place pl = place(a, BM, BN);
  if (!pl.any) return;
  const int m0 = pl.m0, n0 = pl.n0;

  // Where a thread's first unit and piece are in memory, from the stage's first row on, and in LDS.
  // Its others are whole rows further on, in the same columns.
  constexpr int LA = NT / (BM / 16), LB = NT / (BN / 8);  // rows between them
  static_assert(NT % (BM / 16) == 0 && NT % (BN / 8) == 0 && LA % 4 == 0 && LB % 4 == 0,
                "the same columns and places in their lines");
  const int line_a = threadIdx.x / (BM / 16), line_b = threadIdx.x / (BN / 8);
  const int e_a = 16 * (threadIdx.x % (BM / 16)), have = a.K - m0;
  const uint32_t qo = line_a * (uint32_t)a.ldq + (uint32_t)(std::min(e_a, have - 16) + 16);
  const uint32_t so = line_a * (uint32_t)a.lds + (uint32_t)std::min(e_a, have - 1) / 32;
  const uint32_t ao = line_a * (BM * 2) + ((e_a / 8) ^ TA::swz(line_a)) * 16;
  const int down_a = std::min(16, std::max(0, e_a + 16 - have));
  const int e_b = 8 * ((threadIdx.x % (BN / 8)) ^ TN::swz(line_b));
  const uint32_t bo = 2 * (line_b * (uint32_t)a.ldb + (e_b < a.N - n0 ? e_b : 0));
  // (from 16 codes before the tile on, where a unit at a row's end may begin)
  const int8_t* q = a.q + pl.beg * a.ldq + m0 - 16;
  const uint8_t* sc = a.s + pl.beg * a.lds + m0 / 32;
  const bf16* b = static_cast<const bf16*>(a.b) + pl.beg * a.ldb + n0;
  const int rows = (int)(pl.end - pl.beg), stages = (rows + BK - 1) / BK;
  const uint32_t sign = pl.chunk & 1 ? 0x80000000u : 0;

  f16 acc[RB][CB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  struct Raw {
    u4 v[UA];
    uint32_t scale[UA];
  } r0, r1;
  // the codes of a stage (in the last one of the rows that there are)
  auto load_a = [&](Raw& r, int s) {
    s = std::min(s, stages - 1);
    const int8_t* qs = q + (int64_t)(s * BK) * a.ldq;
    const uint8_t* ss = sc + (int64_t)(s * BK) * a.lds;
    const int over = s * BK + BK - rows;  // rows past the chunk's end
#pragma unroll
    for (int p = 0; p < UA; ++p) {
      const uint32_t on = p * LA - std::max(0, line_a + p * LA + over - (BK - 1));
      r.v[p] = *reinterpret_cast<const u4b*>(qs + (uint32_t)(qo + on * (uint32_t)a.ldq));
      r.scale[p] = ss[(uint32_t)(so + on * (uint32_t)a.lds)];
    }
  };
  auto decode = [&](char* to, const Raw& r, int s, int piece) {  // piece: of the thread's 2 UA
    const int p = piece / 2, h = piece & 1;
    u4 x = r.v[p];
    if constexpr (ODD) x = bytes_down(x, down_a);
    const float unit =
        line_a + p * LA + s * BK < rows ? __uint_as_float(r.scale[p] << 23 ^ sign) : 0.f;
    *reinterpret_cast<u4*>(to + (ao + p * LA * BM * 2 + 16 * h)) =
        decode8(x[2 * h], x[2 * h + 1], unit);
  };
  auto load_b = [&](char* to, int s) {
    s = std::min(s, stages - 1);
    const char* bs = reinterpret_cast<const char*>(b + (int64_t)(s * BK) * a.ldb);
    const int left = rows - s * BK;
#pragma unroll
    for (int p = 0; p < PB; ++p) {
      const char* at = bs + 2 * p * LB * a.ldb + bo;
      if (line_b + p * LB >= left) at = reinterpret_cast<const char*>(&g_zeros);
      __builtin_amdgcn_global_load_lds((const GCN_GLOBAL void*)at,
                                       (GCN_LDS void*)(to + (w * 64 + p * NT) * 16), 16, 0, 0);
    }
  };
  constexpr int STEPS = BK / 16;
  static_assert(STEPS % 2 == 0, "the fragments' buffers alternate over the stages");
  bf8 fa[2][RB], fb[2][CB];
  auto read = [&](int to, int step, const char* ca, const char* cb) {
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[to][i] = TA::read(ca, wr * RB + i, step, lane);
#pragma unroll
    for (int j = 0; j < CB; ++j) fb[to][j] = TN::read(cb, wc * CB + j, step, lane);
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
        acc[i][j] =
            __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[from][i], fb[from][j], acc[i][j], 0, 0, 0);
  };
  // Between two products: one or two LDS reads, and some of the decoding.
  constexpr int READS = 2 * (RB + CB), MULS = RB * CB;
  auto order = [&](bool decodes) {
#pragma unroll
    for (int p = 0; p < MULS; ++p) {
      __builtin_amdgcn_sched_group_barrier(0x100, (READS + MULS - 1) / MULS, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      if (decodes) __builtin_amdgcn_sched_group_barrier(0x2, 6, 0);
    }
  };
  // Stage s, in (ca, cb): the codes of stage s + 1 go from r to na, then those of stage s + 3 to r.
  auto stage = [&](int s, char* ca, char* cb, char* na, char* nb, Raw& r) {
    constexpr int PER = (2 * UA + STEPS - 2) / (STEPS - 1);  // pieces to decode in a step
#pragma unroll
    for (int st = 0; st + 1 < STEPS; ++st) {
      read((st + 1) & 1, st + 1, ca, cb);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (st * PER + i < 2 * UA) decode(na, r, s + 1, st * PER + i);
      multiply(st & 1);
      order(true);
    }
    wait_loads();
    load_b(cb, s + 2);
    load_a(r, s + 3);
    read(0, 0, na, nb);
    multiply((STEPS - 1) & 1);
    order(false);
  };
  if (stages > 0) {
    load_b(b0, 0);
    load_a(r0, 0);
    load_a(r1, 1);
    load_b(b1, 1);
#pragma unroll
    for (int i = 0; i < 2 * UA; ++i) decode(a0, r0, 0, i);
    load_a(r0, 2);
    wait_loads();
    read(0, 0, a0, b0);
    for (int s = 0; s < stages; s += 2) {
      stage(s, a0, b0, a1, b1, r1);
      if (s + 1 >= stages) break;
      stage(s + 1, a1, b1, a0, b0, r0);
    }
    wait_loads();  // those past the last stage
  }
  write_sums<RB, CB>(a, pl, m0 + wr * RB * 32, n0 + wc * CB * 32, acc, pl.chunk & 1 ? -1.f : 1.f);
}

// fp32 rows, split into three parts on their way to LDS (8 to 9 vector instructions an element), three
// products of a code's value and a part. Rows of 32 a stage; the codes and rows of stage s + 1 are in
// registers when stage s begins, are decoded and split between its products, and the loads of
// stage s + 3 follow in the same registers. ODD: rows that do not end with a unit of 8 codes, or with 4
// columns.
template <bool ODD, int WR, int WC, int RB, int CB>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_mul8_parts(Q8Args a) {
  constexpr int BK = 32, NT = 64 * WR * WC, BM = 32 * WR * RB, BN = 32 * WC * CB;
  using TA = Tile<false, BM, BK>;
  using TN = Tile<false, BN, BK>;
  constexpr int UA = BM * BK / 8 / NT, PB = BN * BK / 8 / NT;  // units of 8 codes, pieces of 8 columns
  constexpr int LA = NT / (BM / 8), LB = NT / (BN / 8);        // rows between a thread's
  static_assert(BM * BK / 8 % NT == 0 && BN * BK / 8 % NT == 0 && LA % 4 == 0 && LB % 4 == 0,
                "every thread has as many, in the same columns and places in their lines");
  __shared__ __align__(16) char a0[TA::kBytes], a1[TA::kBytes], b0[3 * TN::kBytes], b1[3 * TN::kBytes];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  const Place pl = place(a, BM, BN);
  if (!pl.any) return;
  const int m0 = pl.m0, n0 = pl.n0;

  const int line_a = threadIdx.x / (BM / 8), line_b = threadIdx.x / (BN / 8);
  const int e_a = 8 * (threadIdx.x % (BM / 8)), have_a = a.K - m0;
  const int e_b = 8 * (threadIdx.x % (BN / 8)), have_b = a.N - n0;
  // (from 8 codes, or 4 columns, before the tile on, where one at a row's end may begin)
  const uint32_t qo = line_a * (uint32_t)a.ldq + (uint32_t)(std::min(e_a, have_a - 8) + 8);
  const uint32_t so = line_a * (uint32_t)a.lds + (uint32_t)std::min(e_a, have_a - 1) / 32;
  const uint32_t bo0 = 4 * (line_b * (uint32_t)a.ldb + (uint32_t)(std::min(e_b, have_b - 4) + 4));
  const uint32_t bo1 = 4 * (line_b * (uint32_t)a.ldb + (uint32_t)(std::min(e_b + 4, have_b - 4) + 4));
  const uint32_t ao = line_a * (BM * 2) + ((e_a / 8) ^ TA::swz(line_a)) * 16;
  const uint32_t to_b = line_b * (BN * 2) + ((e_b / 8) ^ TN::swz(line_b)) * 16;
  const int down_a = std::min(8, std::max(0, e_a + 8 - have_a));
  const int8_t* q = a.q + pl.beg * a.ldq + m0 - 8;
  const uint8_t* sc = a.s + pl.beg * a.lds + m0 / 32;
  const float* b = static_cast<const float*>(a.b) + pl.beg * a.ldb + n0 - 4;
  const int rows = (int)(pl.end - pl.beg), stages = (rows + BK - 1) / BK;
  const uint32_t sign = pl.chunk & 1 ? 0x80000000u : 0;

  f16 acc[RB][CB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  struct Raw {
    u2b code[UA];
    uint32_t scale[UA];
    u4 v[PB][2];
  } r0, r1;
  // unit or piece p of a stage (in the last one of the rows that there are)
  auto load_a = [&](Raw& r, int s, int p) {
    s = std::min(s, stages - 1);
    const int over = s * BK + BK - rows;  // rows past the chunk's end
    const uint32_t on = p * LA - std::max(0, line_a + p * LA + over - (BK - 1));
    const int8_t* qs = q + (int64_t)(s * BK) * a.ldq;
    const uint8_t* ss = sc + (int64_t)(s * BK) * a.lds;
    r.code[p] = *reinterpret_cast<const u2b*>(qs + (uint32_t)(qo + on * (uint32_t)a.ldq));
    r.scale[p] = ss[(uint32_t)(so + on * (uint32_t)a.lds)];
  };
  auto load_b = [&](Raw& r, int s, int p) {
    s = std::min(s, stages - 1);
    const int over = s * BK + BK - rows;
    const uint32_t on = 4 * (p * LB - std::max(0, line_b + p * LB + over - (BK - 1))) * (uint32_t)a.ldb;
    const char* bs = reinterpret_cast<const char*>(b + (int64_t)(s * BK) * a.ldb);
    r.v[p][0] = *reinterpret_cast<const Unaligned<float>::type*>(bs + (uint32_t)(bo0 + on));
    r.v[p][1] = *reinterpret_cast<const Unaligned<float>::type*>(bs + (uint32_t)(bo1 + on));
  };
  auto decode = [&](char* to, const Raw& r, int s, int p) {
    uint64_t c = r.code[p][0] | (uint64_t)r.code[p][1] << 32;
    if constexpr (ODD) c = down_a < 8 ? c >> 8 * down_a : 0;
    const float unit =
        line_a + p * LA + s * BK < rows ? __uint_as_float(r.scale[p] << 23 ^ sign) : 0.f;
    *reinterpret_cast<u4*>(to + (ao + p * LA * BM * 2)) =
        decode8((uint32_t)c, (uint32_t)(c >> 32), unit);
  };
  auto split = [&](char* to, const Raw& r, int s, int p) {
    const bool in = line_b + p * LB + s * BK < rows;
    float x[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u4 v = r.v[p][i];
      if constexpr (ODD) v = move_down<float>(v, std::min(4, std::max(0, e_b + 4 * i + 4 - have_b)));
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = in ? __uint_as_float(v[j]) * kUp : 0.f;
    }
    u4 parts[3];
    split8(x, parts);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      *reinterpret_cast<u4*>(to + (to_b + p * LB * BN * 2 + i * TN::kBytes)) = parts[i];
  };
  bf8 fa[2][RB], fb[2][CB][3];
  auto read = [&](int step, const char* ca, const char* cb) {
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[step][i] = TA::read(ca, wr * RB + i, step, lane);
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int p = 0; p < 3; ++p)
        fb[step][j][p] = TN::read(cb + p * TN::kBytes, wc * CB + j, step, lane);
  };
  auto multiply = [&](int step) {
#pragma unroll
    for (int p = 2; p >= 0; --p)  // the small parts first
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[step][i], fb[step][j][p],
                                                              acc[i][j], 0, 0, 0);
  };
  // Stage s, whose first fragments are read, in (ca, cb): stage s + 1 goes from r to (na, nb).
  constexpr int MULS = 3 * RB * CB;
  auto stage = [&](int s, char* ca, char* cb, char* na, char* nb, Raw& r) {
    read(1, ca, cb);
#pragma unroll
    for (int p = 0; p < UA; ++p) {
      decode(na, r, s + 1, p);
      load_a(r, s + 3, p);
    }
#pragma unroll
    for (int p = 0; p < PB; ++p) {
      split(nb, r, s + 1, p);
      load_b(r, s + 3, p);
    }
    multiply(0);
    multiply(1);
#pragma unroll
    for (int p = 0; p < 2 * MULS; ++p) {
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 8, 0);
    }
    __syncthreads();
    read(0, na, nb);
  };
  if (stages > 0) {
    auto load = [&](Raw& r, int s) {
#pragma unroll
      for (int p = 0; p < UA; ++p) load_a(r, s, p);
#pragma unroll
      for (int p = 0; p < PB; ++p) load_b(r, s, p);
    };
    load(r0, 0);
    load(r1, 1);
#pragma unroll
    for (int p = 0; p < UA; ++p) decode(a0, r0, 0, p);
#pragma unroll
    for (int p = 0; p < PB; ++p) split(b0, r0, 0, p);
    load(r0, 2);
    __syncthreads();
    read(0, a0, b0);
    for (int s = 0; s < stages; s += 2) {
      stage(s, a0, b0, a1, b1, r1);
      if (s + 1 >= stages) break;
      stage(s + 1, a1, b1, a0, b0, r0);
    }
  }

  const int wm = m0 + wr * RB * 32, wn = n0 + wc * CB * 32;
  float down = pl.chunk & 1 ? -1.f / kUp : 1.f / kUp;
  if (not_finite<RB, CB>(acc)) {
    down = 1.f;
    auto again = [&](int64_t k, float (*x)[4], float (*y)[4]) {
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int m = std::min(wm + i * 32 + (lane & 31), a.K - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[i][j] = k + j < pl.end ? scale_of(a.s[(k + j) * a.lds + m / 32]) *
                                         (float)a.q[(k + j) * a.ldq + m]
                                   : 0.f;
      }
#pragma unroll
      for (int i = 0; i < CB; ++i) {
        const int n = std::min(wn + i * 32 + (lane & 31), a.N - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          y[i][j] = k + j < pl.end ? static_cast<const float*>(a.b)[(k + j) * a.ldb + n] : 0.f;
      }
    };
    mul_again<RB, CB>(pl.beg, pl.end, again, acc);
  }
  write_sums<RB, CB>(a, pl, wm, wn, acc, down);
}

template <int WR, int WC, int RB, int CB, class Kernel>
gcn_status launch(Kernel kernel, Q8Args a, int b_bytes, hipStream_t s) {
  constexpr int BM = 32 * WR * RB, BN = 32 * WC * CB;
  a.col_tiles = (int)ceil_div((int64_t)a.N, (int64_t)BN);
  a.row_tiles = (int)ceil_div((int64_t)a.K, (int64_t)BM);
  const int64_t slots = group_slots(a.by, a.split);
  const int64_t per = (int64_t)a.col_tiles * a.row_tiles;
  a.by_chunk = per < 8 || slots >= 32;
  // rectangles of which the XCDs read the fewest bytes, where they divide the tiles as evenly
  int64_t least = 0;
  for (int across = 1; across <= 8; across *= 2) {
    const int64_t rr = ceil_div(a.row_tiles, 8 / across), rc = ceil_div(a.col_tiles, across);
    const int64_t bytes = rr * BM + rc * BN * b_bytes;
    if (rr * rc > ceil_div(per, (int64_t)8) || (a.across > 0 && bytes >= least)) continue;
    least = bytes;
    a.across = across;
    a.rect_rows = (int)rr;
    a.rect_cols = (int)rc;
  }
  const int64_t blocks =
      8 * (a.by_chunk ? ceil_div(slots, (int64_t)8) * per : slots * ceil_div(per, (int64_t)8));
  GCN_CHECK(launch_fits(blocks, 64 * WR * WC));
  a.slots = (uint32_t)slots;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * WR * WC), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

// C_g apart from what the product reads.
gcn_status apart(const Q8Args& a, int dtype) {
  const int64_t rows = a.by.rows, K = a.K, N = a.N;
  const Span in[4] = {array_of(a.by.offsets, 8 * ((int64_t)a.by.n + 1)), rows_of(a.q, rows, a.ldq, K, 1),
                      rows_of(a.s, rows, a.lds, ceil_div(K, (int64_t)32), 1),
                      rows_of(a.b, rows, a.ldb, N, size_of(dtype))};
  // (matrices as long rows first: most lie nowhere near)
  for (const Span& x : in)
    if (overlap(rows_of(a.c, a.by.n, a.by.n > 1 ? a.stride_c : 1, (K - 1) * a.ldc + N, 4), x))
      for (int g = 0; g < a.by.n; ++g)
        GCN_CHECK(check_apart({rows_of(a.c + g * a.stride_c, K, a.ldc, N, 4)}, {x}));
  return GCN_OK;
}

// Rows of sixteen codes, and strides whose offsets over a stage's rows are 32 bits.
bool mul8_takes(const Q8Args& a) {
  return a.N >= 8 && a.K >= 16 && a.ldb < (int64_t(1) << 22) && a.ldq < (int64_t(1) << 24) &&
         a.lds < (int64_t(1) << 24) && a.ldc < (int64_t(1) << 26);
}

gcn_status mul8(Q8Args a, int dtype, Scratch* scratch, hipStream_t s) {
  const int64_t N = a.N, K = a.K, rows = a.by.rows;
  // chunks as gemm_grouped.hip's, but shorter where few groups leave units idle: there a chunk's time
  // weighs more than its sums (32,768 rows of 16 groups, 2048 x 4096 bf16: 673 us, 857 with the few's
  // 1e-4; 200,000 of 8, 256 x 512: 95 so, 114 with the others' 2e-4)
  const bool direct = dtype == GCN_DT_BF16 && reinterpret_cast<uintptr_t>(a.b) % 16 == 0 &&
                      a.ldb % 8 == 0 && N % 8 == 0;
  const bool f32 = dtype == GCN_DT_F32;
  // tiles of 256 x 256 from 192 rows of a group on: 170 groups of 192, 1024 x 1024: 182 us, 227 in tiles of
  // 128; 208 of 192, 256 x 256: 24 and 28. (Large matrices gain from fewer rows on, 341 groups of 96, 1024 x 1024: 317 and
  // 419, small ones do not, 312 of 128, 256 x 256: 37 and 35; and where few groups have few tiles, tiles of 128
  // fill more units: four of 2048, 2048 x 1024: 88 and 50.)
  const bool wide = N > 128 && K > 128 && rows / a.by.n >= 192 && direct;
  const int64_t tm = wide ? 256 : f32 && K <= 64 ? 64 : 128;
  const int64_t tn = wide ? 256 : !f32 ? 128 : N <= 64 ? 64 : tm == 64 ? 128 : (N - 1) % 256 < 128 ? 128 : 256;
  const int64_t tiles = ceil_div(K, tm) * ceil_div(N, tn);
  const int64_t want = tn == 256 ? 240 : 480;
  const bool few = a.by.n * tiles < want;
  const double even = (double)rows * (double)tiles / (double)want;
  const double sums = std::sqrt((few ? 1e-4 : 2e-4) * (double)rows * (double)K * (double)N);
  const double chunk =
      std::min(65536.0, std::max({256.0, sums, few ? std::min(even, 4096.0) : 4096.0}));
  a.split = ceil_div((int64_t)chunk, (int64_t)64) * 64;
  const int64_t parts = rows / a.split;
  if (parts > 0) GCN_CHECK(scratch->alloc(&a.part, parts * K * N, "grouped GEMM partials"));
  if (scratch->asked()) return GCN_OK;
  GCN_CHECK(apart(a, dtype));
  ProfScope ps("grouped_q8", s);
  const bool odd = K % (f32 ? 8 : 16) != 0 || (f32 && N % 4 != 0);
  auto parts_of = [&](auto waves_r, auto waves_c, auto blocks_r, auto blocks_c) {
    constexpr int WR = decltype(waves_r)::value, WC = decltype(waves_c)::value;
    constexpr int RB = decltype(blocks_r)::value, CB = decltype(blocks_c)::value;
    return odd ? launch<WR, WC, RB, CB>(k_mul8_parts<true, WR, WC, RB, CB>, a, 4, s)
               : launch<WR, WC, RB, CB>(k_mul8_parts<false, WR, WC, RB, CB>, a, 4, s);
  };
  std::integral_constant<int, 1> n1;
  std::integral_constant<int, 2> n2;
  std::integral_constant<int, 4> n4;
  if (f32)
    GCN_CHECK(tm == 64 ? (tn == 64 ? parts_of(n2, n2, n1, n1) : parts_of(n2, n2, n1, n2))
              : tn == 64 ? parts_of(n2, n2, n2, n1)
              : tn == 128 ? parts_of(n2, n2, n2, n2)
                          : parts_of(n2, n4, n2, n2));
  else if (wide)
    GCN_CHECK((odd ? launch<4, 2, 2, 4>(k_mul8_direct<true, 64, 4, 2, 2, 4>, a, 2, s)
                   : launch<4, 2, 2, 4>(k_mul8_direct<false, 64, 4, 2, 2, 4>, a, 2, s)));
  else if (direct)
    GCN_CHECK((odd ? launch<2, 2, 2, 2>(k_mul8_direct<true, 64, 2, 2, 2, 2>, a, 2, s)
                   : launch<2, 2, 2, 2>(k_mul8_direct<false, 64, 2, 2, 2, 2>, a, 2, s)));
  else
    GCN_CHECK((launch<2, 2, 2, 2>(k_mul8<64, 2, 2, 2, 2>, a, 2, s)));
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
           stride_w, 0, nullptr, 0, 0, 0, false, 0, 0, 0};
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
  GCN_CHECK(apart(a, dtype));
  ProfScope ps("grouped_q8", s);
  if (dtype == GCN_DT_F32)
    hipLaunchKernelGGL(k_q8<float>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(k_q8<bf16>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  GCN_HIP(hipGetLastError());
  return parts > 0 ? sum_group_partials(a.by, a.split, K, N, a.part, C, ldc, stride_w, s) : GCN_OK;
}
