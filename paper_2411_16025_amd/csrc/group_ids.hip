// Positions sorted by group (gcn_group_ids): a stable radix sort of the ids that ends in the sorted
// positions, their places and the groups' offsets.
//
// Digits of up to 11 bits, as even as the ids' bits allow: up to 2047 groups take one pass, 2^22
// two. A pass has three launches: every tile counts its digits, the counts are summed down the
// tiles digit by digit, and every tile places its ids. A wavefront ranks 64 consecutive ids at a
// time: ballots, bit by bit, give the lanes of the same digit; a counter of the wavefront's own in
// LDS those before them. No atomics but the tiles' counts (whole numbers), so the order is the one
// stable order. Ids outside of the groups are sorted as the group behind the last one.

#include <algorithm>

#include "element.h"
#include "scratch.h"

namespace gcn {
namespace {

constexpr int kMaxBits = 11, kMaxDigits = 1 << kMaxBits;

struct SortArgs {
  uint32_t n, groups;
  int shift, bits;      // of the pass
  uint32_t digits;      // 2^bits, or in a single pass the groups and one more
  const int32_t* ids;   // first pass
  const uint64_t* in;   // later ones: key << 32 | position
  uint64_t* out;        // but in the last
  uint32_t* hist;       // [tiles][digits]: counts, then those of the tiles before
  uint32_t* total;      // [digits]
  uint32_t tiles;
  int32_t* order;
  int32_t* slot;
  uint32_t* sorted;     // the keys in order (last of several passes)
  int64_t* offsets;     // (single pass)
};

template <bool FIRST>
__device__ inline uint64_t load_key(const SortArgs& a, uint32_t i) {
  if constexpr (FIRST) {
    const uint32_t id = (uint32_t)a.ids[i];
    return (uint64_t)(id < a.groups ? id : a.groups) << 32 | i;
  } else {
    return a.in[i];
  }
}

__device__ inline uint32_t digit(const SortArgs& a, uint64_t key) {
  return (uint32_t)(key >> (32 + a.shift)) & ((1u << a.bits) - 1);
}

template <bool FIRST, int NT, int ITEMS>
__global__ __launch_bounds__(NT) void k_count(SortArgs a) {
  __shared__ uint32_t cnt[kMaxDigits];
  for (uint32_t d = threadIdx.x; d < a.digits; d += NT) cnt[d] = 0;
  __syncthreads();
  const uint32_t base = blockIdx.x * (NT * ITEMS);
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const uint32_t i = base + j * NT + threadIdx.x;
    if (i < a.n) atomicAdd(&cnt[digit(a, load_key<FIRST>(a, i))], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < a.digits; d += NT)
    a.hist[(uint64_t)blockIdx.x * a.digits + d] = cnt[d];
}

// 64 digits to a workgroup; its sixteen wavefronts share the tiles, eight at a time.
__global__ __launch_bounds__(1024) void k_sum_tiles(SortArgs a) {
  __shared__ uint32_t sums[16][64];
  const uint32_t lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
  const uint32_t per = (a.tiles + 15) / 16, beg = min(w * per, a.tiles), end = min(beg + per, a.tiles);
  const bool in = d < a.digits;
  uint32_t* h = a.hist + (in ? d : 0);
  uint32_t v[8], s = 0;
  auto load = [&](uint32_t t) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      v[i] = in && t + i < end ? h[(uint64_t)(t + i) * a.digits] : 0;
  };
  for (uint32_t t = beg; t < end; t += 8) {
    load(t);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i];
  }
  sums[w][lane] = s;
  __syncthreads();
  uint32_t run = 0, all = 0;
#pragma unroll
  for (uint32_t q = 0; q < 16; ++q) {
    run += q < w ? sums[q][lane] : 0;
    all += sums[q][lane];
  }
  if (!in) return;
  if (w == 0) a.total[d] = all;
  for (uint32_t t = beg; t < end; t += 8) {
    if (per > 8) load(t);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (t + i < end) {
        h[(uint64_t)(t + i) * a.digits] = run;
        run += v[i];
      }
  }
}

// A wavefront's ITEMS times 64 keys from `base` (the lane's first) on.
template <bool FIRST, int ITEMS>
__device__ inline void load_keys(const SortArgs& a, uint32_t base, uint64_t (&key)[ITEMS]) {
#pragma unroll
  for (int j = 0; j < ITEMS; ++j)
    key[j] = base + j * 64 < a.n ? load_key<FIRST>(a, base + j * 64) : ~0ull;
}

// Each one's number among the wavefront's of its digit, whose counts cnt [digits], all 0 before, then
// holds.
template <int ITEMS>
__device__ inline void rank_keys(const SortArgs& a, uint32_t base, uint32_t* cnt,
                                 const uint64_t (&key)[ITEMS], uint32_t (&rank)[ITEMS]) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const bool valid = base + j * 64 < a.n;
    const uint32_t d = digit(a, key[j]);
    uint64_t peers = __ballot(valid);
    for (int bit = 0; bit < a.bits; ++bit) {
      const bool b = (d >> bit) & 1u;
      const uint64_t m = __ballot(b);
      peers &= b ? m : ~m;
    }
    const uint32_t before = (uint32_t)__popcll(peers & below);
    const uint32_t have = valid ? cnt[d] : 0;
    // (LDS operations of one wavefront take effect in order; the fence keeps
    // the compiler from moving the store before the other lanes' loads)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (valid && before == 0) cnt[d] = have + (uint32_t)__popcll(peers);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    rank[j] = have + before;
  }
}

// The sum of v over the threads before this one; sums [threads / 64] in LDS.
__device__ inline uint32_t before_thread(uint32_t v, uint32_t* sums) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t upto = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(upto, off, 64);
    if (lane >= off) upto += o;
  }
  if (lane == 63) sums[w] = upto;
  __syncthreads();
  uint32_t run = upto - v;
  for (int q = 0; q < w; ++q) run += sums[q];
  return run;
}

__device__ inline void put(const SortArgs& a, uint64_t key, uint32_t place) {
  const uint32_t at = (uint32_t)key;
  const bool in = (uint32_t)(key >> 32) < a.groups;
  if (a.order) a.order[place] = in ? (int32_t)at : -1;
  if (a.slot) a.slot[at] = in ? (int32_t)place : -1;
}

template <bool FIRST, bool LAST, int NT, int ITEMS>
__global__ __launch_bounds__(NT) void k_place(SortArgs a) {
  constexpr int kWaves = NT / 64;
  __shared__ uint32_t first[kMaxDigits];        // the place of the tile's first id of a digit
  __shared__ uint32_t cnt[kWaves][kMaxDigits];  // ids of a wavefront, then of those before it
  __shared__ uint32_t sums[kWaves];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  uint64_t key[ITEMS];
  uint32_t rank[ITEMS];
  const uint32_t base = blockIdx.x * (NT * ITEMS) + w * (64 * ITEMS) + lane;
  load_keys<FIRST>(a, base, key);
#pragma unroll
  for (int q = 0; q < kWaves; ++q)
    for (uint32_t d = t; d < a.digits; d += NT) cnt[q][d] = 0;
  // each thread has a run of digits
  constexpr int kRun = kMaxDigits / NT;
  const uint32_t per = (a.digits + NT - 1) / NT;
  uint32_t total[kRun], here[kRun], mine = 0;
#pragma unroll
  for (uint32_t i = 0; i < kRun; ++i) {
    const uint32_t d = t * per + i;
    const bool in = i < per && d < a.digits;
    total[i] = in ? a.total[d] : 0;
    here[i] = in ? a.hist[(uint64_t)blockIdx.x * a.digits + d] : 0;
  }
#pragma unroll
  for (int i = 0; i < kRun; ++i) mine += total[i];
  uint32_t run = before_thread(mine, sums);
#pragma unroll
  for (uint32_t i = 0; i < kRun; ++i) {
    const uint32_t d = t * per + i;
    if (i >= per || d >= a.digits) break;
    if (FIRST && LAST && blockIdx.x == 0) a.offsets[d] = run;
    first[d] = run + here[i];
    run += total[i];
  }
  rank_keys(a, base, cnt[w], key, rank);
  __syncthreads();
  for (uint32_t d = t; d < a.digits; d += NT) {
    uint32_t s = first[d];
#pragma unroll
    for (int q = 0; q < kWaves; ++q) {
      const uint32_t c = cnt[q][d];
      cnt[q][d] = s;
      s += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    if (base + j * 64 >= a.n) continue;
    const uint32_t place = cnt[w][digit(a, key[j])] + rank[j];
    if constexpr (LAST) {
      put(a, key[j], place);
      if constexpr (!FIRST) a.sorted[place] = (uint32_t)(key[j] >> 32);
    } else {
      a.out[place] = key[j];
    }
  }
}

// Few ids and groups: all of it by one workgroup, in one launch (4096 ids of 64 groups: 9 us a
// call of the binding; 65,536 in three launches 13).
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kOneItems = 4, kOneMost = kThreads * kOneItems;
constexpr uint32_t kOneDigits = kThreads;

__global__ __launch_bounds__(kThreads) void k_sort_one(SortArgs a) {
  __shared__ uint32_t cnt[kWaves][kOneDigits];
  __shared__ uint32_t sums[kWaves];
  const uint32_t t = threadIdx.x, w = t >> 6;
  uint64_t key[kOneItems];
  uint32_t rank[kOneItems];
  const uint32_t base = w * (64 * kOneItems) + (t & 63);
  load_keys<true>(a, base, key);
  if (t < a.digits)
#pragma unroll
    for (int q = 0; q < kWaves; ++q) cnt[q][t] = 0;
  __syncthreads();
  rank_keys(a, base, cnt[w], key, rank);
  __syncthreads();
  uint32_t mine = 0;
  if (t < a.digits)
#pragma unroll
    for (int q = 0; q < kWaves; ++q) mine += cnt[q][t];
  uint32_t run = before_thread(mine, sums);
  if (t < a.digits) {
    a.offsets[t] = run;
#pragma unroll
    for (int q = 0; q < kWaves; ++q) {
      const uint32_t c = cnt[q][t];
      cnt[q][t] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kOneItems; ++j)
    if (base + j * 64 < a.n) put(a, key[j], cnt[w][digit(a, key[j])] + rank[j]);
}

// The first place of a key that is at least v: the wavefront's lanes look at 64 places at a time.
__device__ inline uint32_t wave_lower_bound(const uint32_t* keys, uint32_t n, uint32_t v) {
  uint32_t lo = 0, len = n;  // the keys before lo are below v, the one at lo + len is not
  while (len > 0) {
    const uint32_t step = (len + 63) / 64, at = lo + (threadIdx.x & 63) * step + step - 1;
    const bool below = at < lo + len && keys[at] < v;
    const uint32_t steps = (uint32_t)__popcll(__ballot(below));
    const uint32_t end = lo + len;
    lo += steps * step;
    len = lo < end ? min(step - 1, end - lo) : 0;
  }
  return lo;
}

// Offsets from the sorted keys, 1024 groups to a workgroup: the keys between its ends are found by
// two wavefronts; all of them, or every some, are brought to LDS, where most of a search is.
constexpr uint32_t kFinders = 256, kEach = 4, kPerBlock = kFinders * kEach, kStaged = 2048;
__global__ __launch_bounds__(kFinders) void k_offsets(const uint32_t* sorted, uint32_t n,
                                                      uint32_t groups, int64_t* offsets) {
  __shared__ uint32_t ends[2], keys[kStaged];
  const uint32_t v0 = blockIdx.x * kPerBlock, w = threadIdx.x >> 6;
  if (w < 2) {
    const uint32_t p = wave_lower_bound(sorted, n, w == 0 ? v0 : min(v0 + kPerBlock, groups));
    if ((threadIdx.x & 63) == 0) ends[w] = p;
  }
  __syncthreads();
  const uint32_t lo = ends[0], len = ends[1] - lo, step = len / kStaged + 1;
  const uint32_t staged = len / step;  // the last key of every `step`
  for (uint32_t i = threadIdx.x; i < staged; i += kFinders) keys[i] = sorted[lo + i * step + step - 1];
  __syncthreads();
  // a thread's searches go on together
  uint32_t at[kEach] = {}, left = staged;
  auto halve = [&](uint32_t& left, auto key) {  // of `left` keys from at on, half are known to be below or not
    const uint32_t mid = left / 2;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
      at[i] += key(at[i] + mid) < v0 + threadIdx.x + i * kFinders ? left - mid : 0;
    left = mid;
  };
  while (left > 0) halve(left, [&](uint32_t i) { return keys[min(i, staged - 1)]; });
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) at[i] *= step;
  for (left = step - 1; left > 0;)
    halve(left, [&](uint32_t i) { return i < len ? sorted[lo + i] : 0xFFFFFFFFu; });
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) {
    const uint32_t v = v0 + threadIdx.x + i * kFinders;
    if (v <= groups) offsets[v] = lo + min(at[i], len);
  }
}

__global__ __launch_bounds__(kThreads) void k_zero_offsets(int64_t* offsets, int64_t count) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < count) offsets[i] = 0;
}

template <bool FIRST, bool LAST, int NT, int ITEMS>
gcn_status pass(const SortArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_count<FIRST, NT, ITEMS>), dim3(a.tiles), dim3(NT), 0, s, a);
  GCN_HIP(hipGetLastError());
  hipLaunchKernelGGL(k_sum_tiles, dim3((a.digits + 63) / 64), dim3(1024), 0, s, a);
  GCN_HIP(hipGetLastError());
  hipLaunchKernelGGL((k_place<FIRST, LAST, NT, ITEMS>), dim3(a.tiles), dim3(NT), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <int NT, int ITEMS>
gcn_status sort_ids(SortArgs a, int bits, int passes, uint64_t* pairs[2], hipStream_t s) {
  if (passes == 1) return pass<true, true, NT, ITEMS>(a, s);
  for (int p = 0; p < passes; ++p) {
    a.shift = bits * p / passes;
    a.bits = bits * (p + 1) / passes - a.shift;
    a.digits = 1u << a.bits;
    a.in = pairs[(p + 1) & 1];
    a.out = pairs[p & 1];
    GCN_CHECK((p == 0            ? pass<true, false, NT, ITEMS>(a, s)
               : p + 1 == passes ? pass<false, true, NT, ITEMS>(a, s)
                                 : pass<false, false, NT, ITEMS>(a, s)));
  }
  hipLaunchKernelGGL(k_offsets, dim3((unsigned)ceil_div((int64_t)a.groups + 1, (int64_t)kPerBlock)),
                     dim3(kFinders), 0, s, a.sorted, a.n, a.groups, a.offsets);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

// Ids of a tile: small ones while those are not enough for the CUs (131,072 ids of 50,000 groups: 36 us in
// tiles of 1024, 42 of 4096; 1,000,000 of 64: 25 and 20), 16 to a thread where there are many.
int tile_of(int64_t n) { return n <= (1 << 18) ? 1024 : n <= (1 << 20) ? 4096 : 16384; }

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_group_ids(int64_t n, const int32_t* ids, int64_t n_groups,
                                    int64_t* offsets, int32_t* order, int32_t* slot, void* work,
                                    int64_t* work_bytes, void* stream) {
  clear_error();
  CallScope scope(stream);
  if (n < 0 || n_groups < 1 || !offsets || (n > 0 && (!ids || order == ids || slot == ids))) {
    set_error("need n >= 0, n_groups >= 1, non-NULL ids and offsets, and order and slot apart from ids");
    return GCN_EINVAL;
  }
  if (n >= (int64_t(1) << 31) || n_groups > (int64_t(1) << 30)) {
    set_error("need n < 2^31 and n_groups <= 2^30");
    return GCN_ERANGE;
  }
  GCN_CHECK(check_work(work, work_bytes));
  hipStream_t s = (hipStream_t)stream;
  Scratch scratch(work, work_bytes, s);
  const int64_t zero_blocks = ceil_div(n_groups + 1, (int64_t)kThreads);
  if (!scratch.asked())
    GCN_CHECK(check_apart({array_of(offsets, 8 * (n_groups + 1)), array_of(order, 4 * n), array_of(slot, 4 * n)},
                          {array_of(ids, 4 * n)}));
  if (n == 0) {
    if (scratch.asked()) return GCN_OK;
    ProfScope ps("group_ids", s);
    hipLaunchKernelGGL(k_zero_offsets, dim3((unsigned)zero_blocks), dim3(kThreads), 0, s, offsets,
                       n_groups + 1);
    GCN_HIP(hipGetLastError());
    return GCN_OK;
  }
  const int bits = bits_for((uint64_t)n_groups);
  const int passes = std::max(1, (bits + kMaxBits - 1) / kMaxBits);
  SortArgs a{};
  a.n = (uint32_t)n;
  a.groups = (uint32_t)n_groups;
  a.ids = ids;
  a.order = order;
  a.slot = slot;
  a.offsets = offsets;
  a.bits = bits;
  a.digits = (uint32_t)n_groups + 1;
  if (n <= kOneMost && a.digits <= kOneDigits) {
    if (scratch.asked()) return GCN_OK;
    ProfScope ps("group_ids", s);
    hipLaunchKernelGGL(k_sort_one, dim3(1), dim3(kThreads), 0, s, a);
    GCN_HIP(hipGetLastError());
    return GCN_OK;
  }
  a.tiles = (uint32_t)ceil_div(n, (int64_t)tile_of(n));
  const int64_t digits = passes == 1 ? n_groups + 1 : int64_t(1) << ((bits + passes - 1) / passes);
  GCN_CHECK(scratch.alloc(&a.hist, (int64_t)a.tiles * digits, "digit counts"));
  GCN_CHECK(scratch.alloc(&a.total, digits, "digit totals"));
  uint64_t* pairs[2] = {nullptr, nullptr};
  if (passes > 1) {
    GCN_CHECK(scratch.alloc(&pairs[0], n, "sorted ids"));
    if (passes > 2) GCN_CHECK(scratch.alloc(&pairs[1], n, "sorted ids"));
    GCN_CHECK(scratch.alloc(&a.sorted, n, "sorted ids"));
  }
  if (scratch.asked()) return GCN_OK;
  ProfScope ps("group_ids", s);
  switch (tile_of(n)) {
    case 1024: return sort_ids<256, 4>(a, bits, passes, pairs, s);
    case 4096: return sort_ids<1024, 4>(a, bits, passes, pairs, s);
    default: return sort_ids<1024, 16>(a, bits, passes, pairs, s);
  }
}
