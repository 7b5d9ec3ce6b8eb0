// A router's choice, the balance loss and their gradient (gcn_route_fwd, gcn_route_bwd).
//
// G neighbouring lanes hold a row, V logits each in registers, so it is read once: the largest
// logit, the exponentials and their sum, then k times the largest of those left, whose index lane
// i % G keeps. Ties go to the lowest index. What each lane adds up of p over its rows, and the
// choices counted in LDS, are a workgroup's sums, which a second launch adds. 131,072 rows of 64 bf16
// logits, 8 chosen: 18.5 us, 5.4 in the sums' launch (traced; 21.4 for both among other calls); its bytes would take
// 4. Vector instructions take 57% of the cycles; the rest is latency: each workgroup has two turns,
// and the second one's logits are loaded after the first one's choices.

#include <cmath>
#include <type_traits>

#include "groups.h"
#include "lanes.h"
#include "rows.h"

namespace gcn {
namespace {

constexpr int kMaxExperts = 1024;
// Workgroups of 16 wavefronts for many rows: two to a CU keep it busy, and their sums are few.
constexpr int kFew = 256, kMany = 1024;

struct RouteArgs {
  int64_t n;
  int E, k;
  const void* z;
  int64_t ldz;
  bool normalize;
  const uint8_t* mask;
  float* weights;
  int32_t* experts;
  // [blocks][E + 1]: choices and sums of p of the workgroups (the last: rows with a choice)
  struct Part {
    uint32_t count;
    float p;
  };
  Part* part;
  double* part_loss;  // three sums of each workgroup of k_finish
  uint32_t* ticket;
  int blocks;
  double coef;
  int64_t* counts;
  float* loss;
  // backward
  const int32_t* chosen;
  const float* w;
  const int64_t* all_counts;
  const float* dw;
  const float* dloss;
  void* dz;
  int64_t ldd;
};

template <int G, int OFF = 1>
__device__ inline float slot_max(float v) {
  if constexpr (OFF < G) return slot_max<G, 2 * OFF>(fmaxf(v, slot_partner<OFF>(v)));
  return v;
}
template <int G, int OFF = 1>
__device__ inline uint32_t slot_max(uint32_t v) {
  if constexpr (OFF < G) return slot_max<G, 2 * OFF>(max(v, (uint32_t)slot_partner<OFF>((int)v)));
  return v;
}
template <int G, int OFF = 1>
__device__ inline int slot_min(int v) {
  if constexpr (OFF < G) return slot_min<G, 2 * OFF>(min(v, slot_partner<OFF>(v)));
  return v;
}

// The V logits of a lane, -inf behind the row's end.
template <class T, int V>
__device__ inline void load_logits(const T* row, int f, int E, float (&z)[V]) {
#pragma unroll
  for (int i = 0; i < V; i += 8) {
    float v[8];
    unpack_raw(load_raw<T, 8>(row, f + i, E), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[i + e] = f + i + e < E ? v[e] : -INFINITY;
  }
}

// e^x = 2^(x log2 e), log2 e in two parts (at x = -80 the rounding of the product alone would be
// 80 of the result's; the second part and the rest of the first product make it one), the rest's
// factor 2^r = 1 + r ln 2. Results below 2^-126 are 0.
__device__ inline float exp_of(float x) {
  const float t = x * 0x1.715476p0f;
  const float r = __builtin_fmaf(x, 0x1.4ae0cp-26f, __builtin_fmaf(x, 0x1.715476p0f, -t));
  const float y = __builtin_amdgcn_exp2f(t);
  return x < -104.f ? 0.f : __builtin_fmaf(y * r, 0x1.62e43p-1f, y);
}

// p of the row: e / sum. A row of -inf alone: zeros, and false.
template <int G, int V>
__device__ inline bool softmax(const float (&z)[V], float (&p)[V], float* top, float* inverse) {
  float m = -INFINITY, s = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) m = fmaxf(m, z[i]);
  m = slot_max<G>(m);
  *top = m;
  const bool any = m > -INFINITY;
  const float from = any ? m : 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    p[i] = exp_of(z[i] - from);
    s += p[i];
  }
  s = slot_sum<G>(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
  *inverse = inv;
#pragma unroll
  for (int i = 0; i < V; ++i) p[i] *= inv;
  return any;
}

// What next() gives: index() is that of a logit, or -1, value() the logit.
struct Choice {
  uint32_t key;
  float v;
};

// The logits that are left to choose from. fp32: the largest one, then the least index that has it.
template <class T, int G, int V>
struct Left {
  float z[V];
  __device__ inline Left(const float (&v)[V], int) {
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = v[e];
  }
  __device__ inline Choice next(int f) {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < V; ++e) m = fmaxf(m, z[e]);
    m = slot_max<G>(m);
    int i = G * V;
#pragma unroll
    for (int e = V - 1; e >= 0; --e) i = z[e] == m ? f + e : i;
    i = slot_min<G>(i);
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] = f + e == i ? -INFINITY : z[e];
    return Choice{(uint32_t)i, m};
  }
  __device__ static inline int index(const Choice& c) { return c.v > -INFINITY ? (int)c.key : -1; }
  __device__ static inline float value(const Choice& c) { return c.v; }
};

// bf16: value and index in one whole number, the value's bits in an order that grows with it (-0 as
// +0), below them the index from the end; 0 for a logit that cannot be chosen. A lane's are sorted
// once (Batcher's odd-even merge), so that the next one is its first, or another lane's
// (131,072 rows of 64, 8 chosen: 30 us with a search of the eight each time, 19 so and with exp2).
template <int G, int V>
struct Left<bf16, G, V> {
  uint32_t key[V];
  __device__ inline Left(const float (&v)[V], int f) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const uint32_t b = __float_as_uint(v[e] + 0.f);
      const uint32_t up = (b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) & 0xFFFF0000u;
      key[e] = v[e] > -INFINITY ? up | (0xFFFFu - (uint32_t)(f + e)) : 0;
    }
#pragma unroll
    for (int p = 1; p < V; p *= 2)
#pragma unroll
      for (int q = p; q >= 1; q /= 2)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int l = j + q;
          if (l < V && j >= q % p && ((j - q % p) / q) % 2 == 0 && j / (2 * p) == l / (2 * p)) {
            const uint32_t hi = max(key[j], key[l]), lo = min(key[j], key[l]);
            key[j] = hi;
            key[l] = lo;
          }
        }
  }
  __device__ inline Choice next(int) {
    const uint32_t m = slot_max<G>(key[0]);
    const bool mine = key[0] == m;
#pragma unroll
    for (int e = 0; e < V; ++e) key[e] = mine ? (e + 1 < V ? key[e + 1] : 0) : key[e];
    return Choice{m, 0.f};
  }
  __device__ static inline int index(const Choice& c) {
    return c.key ? (int)(0xFFFFu - (c.key & 0xFFFFu)) : -1;
  }
  __device__ static inline float value(const Choice& c) {
    const uint32_t b = c.key & 0xFFFF0000u;
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b & 0xFFFF0000u);
  }
};

// Sums over the threads of a workgroup, which thread 0 gets.
template <int NT>
__device__ inline void block_sums(double (&v)[3]) {
  __shared__ double sums[3][NT / 64];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    v[i] = slot_sum<64>(v[i]);
    if ((threadIdx.x & 63) == 0) sums[i][threadIdx.x >> 6] = v[i];
  }
  __syncthreads();
  if (threadIdx.x == 0)
    for (int q = 1; q < NT / 64; ++q)
#pragma unroll
      for (int i = 0; i < 3; ++i) v[i] += sums[i][q];
}

// The loss from sum_e c_e P_e, sum_e c_e and the rows with a choice (without one p is 0 or, of rows
// that hold a NaN alone, NaN).
__device__ inline void write_loss(const RouteArgs& a, const double (&v)[3]) {
  const double all = v[1] * v[2];
  *a.loss = (float)(a.coef * a.E * (all > 0.0 ? v[0] / all : v[0]));
}

// counts, their number of rows and the loss from the workgroups' sums. A workgroup has 16 experts;
// its threads add the sums of every 32nd workgroup, sixteen loads at a time (they come from the
// other XCDs). The last one to end adds up the loss, in the experts' order: the ticket that tells it
// was set to 0 by the kernel before (by one workgroup alone, 131,072 rows of 64: 9 us).
constexpr int kCols = 16, kFinish = 512;
__global__ __launch_bounds__(kFinish) void k_finish(RouteArgs a) {
  constexpr int kGroups = kFinish / kCols;
  __shared__ uint32_t part_c[kFinish];
  __shared__ double part_p[kFinish];
  const int t = threadIdx.x, e = blockIdx.x * kCols + t % kCols, g = t / kCols;
  uint32_t n = 0;
  double p = 0.0;
  if (e <= a.E)
    for (int b = g; b < a.blocks; b += 16 * kGroups) {
      RouteArgs::Part v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        v[i] = a.part[(int64_t)min(b + i * kGroups, a.blocks - 1) * (a.E + 1) + e];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (b + i * kGroups < a.blocks) {
          n += v[i].count;
          p += (double)v[i].p;
        }
    }
  part_c[t] = n;
  part_p[t] = p;
  __syncthreads();
  double v[3] = {0.0, 0.0, 0.0};
  if (t < kCols && e <= a.E) {
    for (int q = 1; q < kGroups; ++q) {
      n += part_c[t + q * kCols];
      p += part_p[t + q * kCols];
    }
    a.counts[e] = n;
    if (e < a.E) {
      v[0] = (double)n * p;
      v[1] = (double)n;
    } else {
      v[2] = (double)n;
    }
  }
  if (!a.loss) return;
  block_sums<kFinish>(v);
  if (t > 0) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) a.part_loss[3 * blockIdx.x + i] = v[i];
  __threadfence();
  if (atomicAdd(a.ticket, 1u) != gridDim.x - 1) return;
  __threadfence();
  v[0] = v[1] = v[2] = 0.0;
  for (uint32_t b = 0; b < gridDim.x; ++b)
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] += a.part_loss[3 * b + i];
  write_loss(a, v);
}

// KEPT: choices that a lane keeps, at least k / G.
template <class T, int NT, int G, int V, int KEPT>
__global__ __launch_bounds__(NT, NT == kMany && V == 8 ? 8 : 1) void k_route(RouteArgs a) {
  constexpr int kSlots = NT / G;  // rows at a time
  __shared__ uint32_t cnt[kMaxExperts + 1];
  __shared__ float sums[NT / 64][G * V];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, in = threadIdx.x % G, f = in * V;
  for (int e = threadIdx.x; e <= a.E; e += NT) cnt[e] = 0;
  __syncthreads();
  float acc[V] = {};
  for (int64_t t0 = (int64_t)blockIdx.x * kSlots; t0 < a.n; t0 += (int64_t)gridDim.x * kSlots) {
    const int64_t t = t0 + threadIdx.x / G;
    const bool row = t < a.n && (!a.mask || a.mask[t] != 0);
    float z[V], p[V], top, inv;
    load_logits(static_cast<const T*>(a.z) + (row ? t : 0) * a.ldz, f, row ? a.E : 0, z);
    const bool any = softmax<G>(z, p, &top, &inv);
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] += p[i];
    if (any && in == 0) atomicAdd(&cnt[a.E], 1u);
    Left<T, G, V> left(z, f);
    int at[KEPT];
    float weight[KEPT], sum = 0.f;
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
      Choice kept{0, -INFINITY};
      for (int i = 0; i < min(a.k - c * G, G); ++i) {
        const Choice next = left.next(f);
        if (i == in) kept = next;
      }
      at[c] = left.index(kept);
      weight[c] = at[c] >= 0 ? exp_of(left.value(kept) - top) * inv : 0.f;
      sum += weight[c];
    }
    if (a.normalize) sum = slot_sum<G>(sum);
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
      const int i = c * G + in;
      if (t >= a.n || i >= a.k) continue;
      a.experts[t * a.k + i] = at[c];
      a.weights[t * a.k + i] = a.normalize && at[c] >= 0 ? weight[c] / sum : weight[c];
      if (at[c] >= 0) atomicAdd(&cnt[at[c]], 1u);
    }
  }
  if (a.loss) {
    // the slots of a wavefront, then the wavefronts, in their order
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int off = G; off < 64; off *= 2) acc[i] += __shfl_xor(acc[i], off, 64);
      if (lane < G) sums[w][f + i] = acc[i];
    }
  }
  __syncthreads();
  const bool only = NT == kFew && gridDim.x == 1;  // no other workgroup: its sums are all
  if (!only && a.loss && blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
  double v[3] = {0.0, 0.0, 0.0};
  for (int e = threadIdx.x; e <= a.E; e += NT) {
    float s = 0.f;
    if (a.loss && e < a.E)
#pragma unroll
      for (int q = 0; q < NT / 64; ++q) s += sums[q][e];
    if (only) {
      a.counts[e] = cnt[e];
      v[0] += e < a.E ? (double)cnt[e] * (double)s : 0.0;
      v[1] += e < a.E ? (double)cnt[e] : 0.0;
    } else {
      a.part[(int64_t)blockIdx.x * (a.E + 1) + e] = RouteArgs::Part{cnt[e], s};
    }
  }
  if constexpr (NT == kFew)
    if (only && a.loss) {
      block_sums<NT>(v);
      v[2] = (double)cnt[a.E];
      if (threadIdx.x == 0) write_loss(a, v);
    }
}

template <class T, int NT, int G, int V>
__global__ __launch_bounds__(NT) void k_route_bwd(RouteArgs a) {
  constexpr int kSlots = NT / G;
  const int in = threadIdx.x % G, f = in * V;
  // a_e of the balance loss
  float bal[V] = {};
  if (a.coef != 0.0) {
    double c[V], all = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      c[i] = f + i < a.E ? (double)a.all_counts[f + i] : 0.0;
      all += c[i];
    }
    all = slot_sum<G>(all) * (double)a.all_counts[a.E];
    const double s = all > 0.0 ? a.coef * a.E * (a.dloss ? (double)*a.dloss : 1.0) / all : 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) bal[i] = (float)(s * c[i]);
  }
  for (int64_t t0 = (int64_t)blockIdx.x * kSlots; t0 < a.n; t0 += (int64_t)gridDim.x * kSlots) {
    const int64_t t = t0 + threadIdx.x / G;
    const bool in_rows = t < a.n;
    const bool row = in_rows && a.chosen[t * a.k] >= 0;
    float z[V], p[V], d[V] = {}, top, inv;
    load_logits(static_cast<const T*>(a.z) + (row ? t : 0) * a.ldz, f, row ? a.E : 0, z);
    softmax<G>(z, p, &top, &inv);
    // the chosen ones, four at a time; all lanes of the slot load them
    float inner = 0.f;  // sum of g w over them
    int at[4];
    float g[4], cw[4];
    auto chosen = [&](int i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t q = t * a.k + min(i + j, a.k - 1);
        at[j] = a.chosen[q];
        g[j] = a.dw[q];
        cw[j] = a.w[q];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j >= a.k || at[j] < 0 || at[j] >= a.E) at[j] = -1;
    };
    if (row && a.dw) {
      for (int i = 0; i < a.k; i += 4) {
        chosen(i);
#pragma unroll
        for (int j = 0; j < 4; ++j) inner += at[j] >= 0 ? g[j] * cw[j] : 0.f;
      }
      for (int i = 0; i < a.k; i += 4) {
        if (a.k > 4) chosen(i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = at[j] >= 0 ? cw[j] * (a.normalize ? g[j] - inner : g[j]) : 0.f;
#pragma unroll
          for (int e = 0; e < V; ++e) d[e] += f + e == at[j] ? x : 0.f;
        }
      }
    }
    float mean = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) mean += bal[i] * p[i];
    mean = slot_sum<G>(mean) + (a.normalize ? 0.f : inner);
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] += p[i] * (bal[i] - mean);
    if (in_rows)
#pragma unroll
      for (int i = 0; i < V; i += 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row ? d[i + e] : 0.f;
        store_raw(static_cast<T*>(a.dz) + t * a.ldd, f + i, a.E, v);
      }
  }
}

inline int route_lanes(int64_t E) {
  int g = 1;
  while (g < 64 && g * 8 < E) g *= 2;
  return g;
}

bool many_rows(int64_t n, int64_t E) { return n > 256 * (int64_t)(kFew / route_lanes(E)); }
int route_blocks(int64_t n, int64_t E, int64_t most) {
  return (int)std::min<int64_t>(
      most, ceil_div(n, (int64_t)((many_rows(n, E) ? kMany : kFew) / route_lanes(E))));
}

template <class T, int NT, bool BWD>
gcn_status launch(const RouteArgs& a, int blocks, hipStream_t s) {
  auto go = [&](auto lanes, auto values) {
    constexpr int G = decltype(lanes)::value, V = decltype(values)::value;
    if constexpr (BWD)
      hipLaunchKernelGGL((k_route_bwd<T, NT, G, V>), dim3(blocks), dim3(NT), 0, s, a);
    else if (a.k <= G)
      hipLaunchKernelGGL((k_route<T, NT, G, V, 1>), dim3(blocks), dim3(NT), 0, s, a);
    else if constexpr (G < 64)  // (k is at most 64, and 8 G)
      hipLaunchKernelGGL((k_route<T, NT, G, V, (G <= 8 ? 8 : 64 / G)>), dim3(blocks), dim3(NT), 0, s, a);
  };
  std::integral_constant<int, 8> v8;
  switch (route_lanes(a.E)) {
    case 1: go(std::integral_constant<int, 1>(), v8); break;
    case 2: go(std::integral_constant<int, 2>(), v8); break;
    case 4: go(std::integral_constant<int, 4>(), v8); break;
    case 8: go(std::integral_constant<int, 8>(), v8); break;
    case 16: go(std::integral_constant<int, 16>(), v8); break;
    case 32: go(std::integral_constant<int, 32>(), v8); break;
    default:
      if (a.E <= 512)
        go(std::integral_constant<int, 64>(), v8);
      else
        go(std::integral_constant<int, 64>(), std::integral_constant<int, 16>());
  }
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <bool BWD>
gcn_status launch(const RouteArgs& a, int dtype, int blocks, hipStream_t s) {
  if constexpr (!BWD)
    if (many_rows(a.n, a.E))
      return dtype == GCN_DT_F32 ? launch<float, kMany, BWD>(a, blocks, s)
                                 : launch<bf16, kMany, BWD>(a, blocks, s);
  return dtype == GCN_DT_F32 ? launch<float, kFew, BWD>(a, blocks, s)
                             : launch<bf16, kFew, BWD>(a, blocks, s);
}

gcn_status check_route(int64_t n, int64_t E, int dtype, int64_t k, uint32_t flags, double coef) {
  GCN_CHECK(check_rows(n, std::max<int64_t>(E, 0), dtype));
  if (E > kMaxExperts || k < 1 || k > std::min<int64_t>(E, 64) || (flags & ~GCN_ROUTE_NORMALIZE) ||
      !std::isfinite(coef)) {
    set_error("need E in [1, 1024], k in [1, min(E, 64)], known flags and a finite coef");
    return GCN_EINVAL;
  }
  if (n * k >= (int64_t(1) << 31)) {
    set_error("need n k < 2^31");
    return GCN_ERANGE;
  }
  return GCN_OK;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_route_fwd(int64_t n, int64_t E, const void* logits, int64_t ldz,
                                    int dtype, int64_t k, uint32_t flags, const uint8_t* mask,
                                    double coef, int32_t* experts, float* weights, int64_t* counts,
                                    float* loss, void* work, int64_t* work_bytes, void* stream) {
  clear_error();
  CallScope scope(stream);
  GCN_CHECK(check_route(n, E, dtype, k, flags, coef));
  GCN_CHECK(check_work(work, work_bytes));
  hipStream_t s = (hipStream_t)stream;
  Scratch scratch(work, work_bytes, s);
  if (!counts || (n > 0 && (!logits || !experts || !weights || ldz < E))) {
    set_error("logits, experts, weights and counts must be non-NULL with ldz >= E");
    return GCN_EINVAL;
  }
  if (!scratch.asked())
    GCN_CHECK(check_apart({array_of(experts, 4 * n * k), array_of(weights, 4 * n * k),
                           array_of(counts, 8 * (E + 1)), array_of(loss, 4)},
                          {rows_of(logits, n, ldz, E, size_of(dtype)), array_of(mask, n)}));
  RouteArgs a{};
  a.n = n;
  a.E = (int)E;
  a.k = (int)k;
  a.z = logits;
  a.ldz = ldz;
  a.normalize = flags & GCN_ROUTE_NORMALIZE;
  a.mask = mask;
  a.weights = weights;
  a.experts = experts;
  a.coef = coef;
  a.counts = counts;
  a.loss = loss;
  a.blocks = std::max(1, route_blocks(n, E, 512));  // (no rows: zeros)
  const int64_t finish = ceil_div(E + 1, (int64_t)kCols);
  if (a.blocks > 1) {
    GCN_CHECK(scratch.alloc(&a.part, a.blocks * (E + 1), "sums of workgroups"));
    GCN_CHECK(scratch.alloc(&a.part_loss, 3 * finish, "sums of the loss"));
    GCN_CHECK(scratch.alloc(&a.ticket, 1, "a ticket"));
  }
  if (scratch.asked()) return GCN_OK;
  ProfScope ps("route_fwd", s);
  GCN_CHECK(launch<false>(a, dtype, a.blocks, s));
  if (a.blocks == 1) return GCN_OK;
  hipLaunchKernelGGL(k_finish, dim3((unsigned)finish), dim3(kFinish), 0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

extern "C" gcn_status gcn_route_bwd(int64_t n, int64_t E, const void* logits, int64_t ldz,
                                    int dtype, int64_t k, uint32_t flags, const int32_t* experts,
                                    const float* weights, const int64_t* counts, double coef,
                                    const float* dweights, const float* dloss, void* dlogits,
                                    int64_t ldd, void* stream) {
  clear_error();
  GCN_CHECK(check_route(n, E, dtype, k, flags, coef));
  if (n == 0) return GCN_OK;
  if (!logits || !experts || (dweights && !weights) || (coef != 0.0 && !counts) || !dlogits ||
      ldz < E || ldd < E || (logits == dlogits && ldz != ldd)) {
    set_error("logits, experts, dlogits, the weights of dweights and the counts of coef must be "
              "non-NULL, with ldz, ldd >= E (and one stride where dlogits are the logits)");
    return GCN_EINVAL;
  }
  const Span none{}, z = rows_of(logits, n, ldz, E, size_of(dtype));
  GCN_CHECK(check_apart({rows_of(dlogits, n, ldd, E, size_of(dtype))},
                        {logits == dlogits ? none : z, array_of(experts, 4 * n * k), array_of(weights, 4 * n * k),
                         array_of(counts, 8 * (E + 1)), array_of(dweights, 4 * n * k), array_of(dloss, 4)}));
  RouteArgs a{};
  a.n = n;
  a.E = (int)E;
  a.k = (int)k;
  a.z = logits;
  a.ldz = ldz;
  a.normalize = flags & GCN_ROUTE_NORMALIZE;
  a.coef = coef;
  a.chosen = experts;
  a.w = weights;
  a.all_counts = counts;
  a.dw = dweights;
  a.dloss = dloss;
  a.dz = dlogits;
  a.ldd = ldd;
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps("route_bwd", s);
  const int blocks = (int)std::min<int64_t>(1024, ceil_div(n, (int64_t)(kFew / route_lanes(E))));
  return launch<true>(a, dtype, blocks, s);
}
