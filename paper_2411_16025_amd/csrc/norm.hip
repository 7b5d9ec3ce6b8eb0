// Row LayerNorm with weights and the dropout behind it, forward and backward.

#include <algorithm>
#include <type_traits>

#include "dropout.h"
#include "element.h"
#include "lanes.h"
#include "scratch.h"

namespace gcn {
namespace {

struct NormArgs {
  int64_t n;
  int F;
  const void* x;
  int64_t ldx;
  const float *gamma, *beta;
  double eps;
  Drop drop;
  const void* dy;
  int64_t lddy;
  void* out;  // Y or dX
  int64_t ldo;
  float *dgamma, *dbeta;  // of a single workgroup; else part [workgroups][2][F]
  float* part;
};

// The mean as the sum of two floats: d = (x - hi) - lo loses nothing where the mean is far from 0.
struct Mean {
  float hi, lo;
  __device__ inline explicit Mean(double mean)
      : hi((float)mean), lo((float)(mean - (double)(float)mean)) {}
  __device__ inline float from(float x) const { return (x - hi) - lo; }
};

// ---- rows in registers -----------------------------------------------------------
//
// G lanes hold a row (a part of a wavefront, or a workgroup of G threads), each NV
// pieces of 16 bytes, piece j of lane l at column (l + j G) V, V elements to a piece;
// memory is read once and written once. A workgroup walks its rows, the next one's
// pieces in flight while it works on one, and keeps the weights (and, backward, its
// sums of their gradients) in registers meanwhile. Sums of the statistics in double:
// they cost two operations per element more than fp32 and have the whole range of x^2.

constexpr int threads_of(int G) { return G > 256 ? G : 256; }  // of a workgroup

// FULL: the row's length is that of its lanes' registers, so nothing is guarded (at 16,384 x 4096
// bf16 the guards were 184 branches of a row's backward pass). Otherwise what lies behind
// the row is 0 in the registers.
template <class T, int G, int NV, bool FULL>
struct Rows {
  static constexpr int V = kPiece<T>, NT = threads_of(G), kSlots = NT / G;
  static constexpr int kWaves = NT / 64;

  // Sum over the row's lanes (every lane gets it). `red`: LDS that the sum two before this one
  // used, so that one barrier is enough.
  template <class S>
  __device__ static inline S sum(S v, S* red) {
    if constexpr (G <= 64) {
      return slot_sum<G>(v);
    } else {
      v = slot_sum<64>(v);
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      v = red[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += red[w];
      return v;
    }
  }
  __device__ static inline int column(int j) { return ((int)(threadIdx.x % G) + j * G) * V; }
  // Row i; zeros from row n on. Without a branch, so that the loads stay on their way: a piece
  // that reaches over the row's end is read from V elements before the end on (rows have V, but
  // the shortest), and what lies behind the row is taken off when it is used (36,429 x 4747 bf16
  // forward 280 us, 429 by elements at once). 1024 lanes have no registers for that (8,000 x
  // 16001 fp32: 289 us, 206 at once).
  static constexpr bool LATE = G < 1024;
  __device__ static inline void load(u4 (&r)[NV], const void* x, int64_t ld, int64_t i, int64_t n,
                                     int F) {
    if (i >= n) {
#pragma unroll
      for (int j = 0; j < NV; ++j) r[j] = u4{0, 0, 0, 0};
      return;
    }
    const T* row = static_cast<const T*>(x) + i * ld;
    typedef typename Unaligned<T>::type piece;
    if (FULL || (LATE && F >= V)) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        r[j] = *reinterpret_cast<const piece*>(row + (FULL ? column(j) : min(column(j), F - V)));
    } else if (!LATE && F % V == 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        r[j] = *reinterpret_cast<const piece*>(row + (column(j) < F ? column(j) : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) r[j][e] = column(j) < F ? r[j][e] : 0;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) r[j] = load_piece(row, column(j), F);
    }
  }
  __device__ static inline void values(float (&v)[NV][V], const u4 (&r)[NV], int F) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      u4 p = r[j];
      if (!FULL && LATE && F >= V) {
        if (F % V == 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = column(j) < F ? p[e] : 0;
        } else {
          p = move_down<T>(p, max(0, column(j) + V - F));
        }
      }
      unpack<T>(p, v[j]);
    }
  }
  __device__ static inline void store(T* row, int j, int F, const float (&v)[V]) {
    store_piece<T>(row, column(j), FULL ? column(j) + V : F, v);
  }
  __device__ static inline void weights(float (&w)[NV][V], const float* from, float none, int F) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const int f = column(j) + e;
        const u4 r = from ? load_piece(from, f, FULL ? f + 4 : F) : u4(__float_as_uint(none));
#pragma unroll
        for (int k = 0; k < 4; ++k) w[j][e + k] = __uint_as_float(r[k]);
      }
  }
  // x becomes x - mean (0 behind the row); 1 / sqrt(var + eps).
  __device__ static inline float center(float (&x)[NV][V], int F, double eps,
                                        double (&red)[2][kWaves]) {
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) s += (double)x[j][e];
    const Mean mean(sum(s, red[0]) / (double)F);
    double q = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float d = mean.from(x[j][e]);
        if (!FULL) {
          asm volatile("" : "+v"(d));  // (chosen, not branched over)
          d = column(j) + e < F ? d : 0.f;
        }
        x[j][e] = d;
        q = __builtin_fma((double)d, (double)d, q);
      }
    return (float)inv_sqrt(sum(q, red[1]) / (double)F + eps);
  }
};

template <class T, int G, int NV, bool DROP, bool FULL>
__global__ __launch_bounds__(threads_of(G)) void k_norm_fwd(NormArgs a) {
  using R = Rows<T, G, NV, FULL>;
  constexpr int V = R::V;
  __shared__ double red[2][R::kWaves];
  const uint64_t call = DROP ? drop_call(a.drop) : 0;
  float gamma[NV][V], beta[NV][V];
  R::weights(gamma, a.gamma, 1.f, a.F);
  R::weights(beta, a.beta, 0.f, a.F);
  const int64_t step = (int64_t)gridDim.x * R::kSlots;
  int64_t i = (int64_t)blockIdx.x * R::kSlots + threadIdx.x / G;
  u4 raw[NV];
  R::load(raw, a.x, a.ldx, i, a.n, a.F);
  // rows [first, + kSlots) of the workgroup: all its threads stay while one has a row
  for (int64_t first = (int64_t)blockIdx.x * R::kSlots; first < a.n; first += step, i += step) {
    float x[NV][V];
    R::values(x, raw, a.F);
    R::load(raw, a.x, a.ldx, i + step, a.n, a.F);
    const float rstd = R::center(x, a.F, a.eps, red);
    if (i >= a.n) continue;
    T* y = static_cast<T*>(a.out) + i * a.ldo;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int e = 0; e < V; ++e)
        x[j][e] = __builtin_fmaf(x[j][e] * rstd, gamma[j][e], beta[j][e]);
      if (DROP) drop_piece<V>(a.drop, call, (uint32_t)i, R::column(j), x[j]);
      R::store(y, j, a.F, x[j]);
    }
  }
}

// dX where a.out is given, and the sums for dgamma and dbeta where a place for them is.
template <class T, int G, int NV, bool DROP, bool FULL>
__global__ __launch_bounds__(threads_of(G)) void k_norm_bwd(NormArgs a) {
  using R = Rows<T, G, NV, FULL>;
  constexpr int V = R::V;
  // 1024 threads have no registers for the weights over the rows and the next row's pieces
  constexpr bool KEEP = G < 1024;
  __shared__ double red[2][R::kWaves];
  __shared__ float2 red2[R::kWaves];
  const uint64_t call = DROP ? drop_call(a.drop) : 0;
  float gamma[NV][V], sg[NV][V] = {}, sb[NV][V] = {};
  if (KEEP) R::weights(gamma, a.gamma, 1.f, a.F);
  const int64_t step = (int64_t)gridDim.x * R::kSlots;
  int64_t i = (int64_t)blockIdx.x * R::kSlots + threadIdx.x / G;
  u4 rx[NV], rg[NV];
  auto load = [&](int64_t row) {
    R::load(rx, a.x, a.ldx, row, a.n, a.F);
    R::load(rg, a.dy, a.lddy, row, a.n, a.F);
  };
  if (KEEP) load(i);
  for (int64_t first = (int64_t)blockIdx.x * R::kSlots; first < a.n; first += step, i += step) {
    float x[NV][V], g[NV][V];
    if (!KEEP) load(i);
    R::values(x, rx, a.F);
    R::values(g, rg, a.F);
    if (KEEP) load(i + step);
    float rstd = R::center(x, a.F, a.eps, red);
    // a slot without a row has zeros, no deviation and with eps = 0 no root: nothing of it counts
    if (R::kSlots > 1) rstd = i < a.n ? rstd : 0.f;
    if (!KEEP) R::weights(gamma, a.gamma, 1.f, a.F);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (DROP) drop_piece<V>(a.drop, call, (uint32_t)i, R::column(j), g[j]);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[j][e] *= rstd;  // H; G and H are 0 behind the rows, G behind the row
        sg[j][e] = __builtin_fmaf(g[j][e], x[j][e], sg[j][e]);
        sb[j][e] += g[j][e];
        g[j][e] *= gamma[j][e];  // T
        s1 += g[j][e];
        s2 = __builtin_fmaf(g[j][e], x[j][e], s2);
      }
    }
    if (!a.out) continue;
    float m1, m2;
    if constexpr (G <= 64) {
      m1 = slot_sum<G>(s1) / (float)a.F;
      m2 = slot_sum<G>(s2) / (float)a.F;
    } else {
      s1 = slot_sum<64>(s1);
      s2 = slot_sum<64>(s2);
      if ((threadIdx.x & 63) == 0) red2[threadIdx.x >> 6] = make_float2(s1, s2);
      __syncthreads();  // (the next row's sums have barriers before red2 is written again)
      s1 = s2 = 0.f;
#pragma unroll
      for (int w = 0; w < R::kWaves; ++w) {
        s1 += red2[w].x;
        s2 += red2[w].y;
      }
      m1 = s1 / (float)a.F;
      m2 = s2 / (float)a.F;
    }
    if (i >= a.n) continue;
    T* dx = static_cast<T*>(a.out) + i * a.ldo;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int e = 0; e < V; ++e) g[j][e] = rstd * (g[j][e] - m1 - x[j][e] * m2);
      R::store(dx, j, a.F, g[j]);
    }
  }
  // the workgroup's sums: over the slots of a wavefront, then over the wavefronts
  float* out_g = a.part ? a.part + (int64_t)blockIdx.x * 2 * a.F : a.dgamma;
  float* out_b = a.part ? out_g + a.F : a.dbeta;
  if (!out_g && !out_b) return;
  constexpr int L = G < 64 ? 64 : G, W = R::NT / L;  // lanes that hold a sum each, lines of them
  __shared__ float sums[W > 1 ? W - 1 : 1][G * NV * V];
  auto finish = [&](float (&s)[NV][V], float* out) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int off = G; off < 64; off *= 2) s[j][e] += __shfl_xor(s[j][e], off, 64);
      }
    const int w = (int)threadIdx.x / L;
    const bool mine = (int)threadIdx.x % L < G;
    if constexpr (W > 1) {
      __syncthreads();
      if (w > 0 && mine)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) sums[w - 1][R::column(j) + e] = s[j][e];
      __syncthreads();
    }
    if (w > 0 || !mine || !out) return;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int f = R::column(j) + e;
        float v = s[j][e];
        if constexpr (W > 1)
#pragma unroll
          for (int k = 0; k < W - 1; ++k) v += sums[k][f];
        if (f < a.F) out[f] = v;
      }
  };
  finish(sg, out_g);
  finish(sb, out_b);
}

// ---- rows of any length ------------------------------------------------------------
//
// A workgroup walks the row, three times forward (the second and third time from the
// caches) and four times backward.

constexpr int kThreads = 256;

template <class V>
__device__ inline V block_sum(V v) {
  __shared__ V part[kThreads / 64];
  v = slot_sum<64>(v);
  __syncthreads();  // the values of the sum before have been read
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < kThreads / 64; ++w) v += part[w];
  return v;
}

// The row's mean and 1 / sqrt(var + eps).
struct Stats {
  Mean mean;
  float rstd;
  __device__ inline float norm(float x) const { return mean.from(x) * rstd; }
};

template <class T>
__device__ inline Stats row_stats(const T* x, int F, double eps) {
  double s = 0.0;
  for (int f = threadIdx.x; f < F; f += kThreads) s += (double)to_float(x[f]);
  const Mean mean(block_sum(s) / (double)F);
  double q = 0.0;
  for (int f = threadIdx.x; f < F; f += kThreads) {
    const double d = (double)mean.from(to_float(x[f]));
    q = __builtin_fma(d, d, q);
  }
  return Stats{mean, (float)inv_sqrt(block_sum(q) / (double)F + eps)};
}

__device__ inline bool kept(const Drop& d, uint64_t call, int64_t i, int f) {
  uint32_t w[4];
  drop_words(d, call, (uint32_t)i, (uint32_t)f >> 2, w);
  return w[f & 3] >= d.least;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_fwd_long(NormArgs a) {
  const uint64_t call = drop_call(a.drop);
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + i * a.ldx;
    T* y = static_cast<T*>(a.out) + i * a.ldo;
    const Stats st = row_stats(x, a.F, a.eps);
    for (int f = threadIdx.x; f < a.F; f += kThreads) {
      float v = st.norm(to_float(x[f]));
      v = __builtin_fmaf(v, a.gamma ? a.gamma[f] : 1.f, a.beta ? a.beta[f] : 0.f);
      y[f] = from_float<T>(kept(a.drop, call, i, f) ? v * a.drop.scale : 0.f);
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_long(NormArgs a) {
  const uint64_t call = drop_call(a.drop);
  float* pg = a.part + (int64_t)blockIdx.x * 2 * a.F;
  float* pb = pg + a.F;
  if (a.part)
    for (int f = threadIdx.x; f < a.F; f += kThreads) pg[f] = pb[f] = 0.f;
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + i * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + i * a.lddy;
    T* dx = static_cast<T*>(a.out) + i * a.ldo;
    const Stats st = row_stats(x, a.F, a.eps);
    auto g_at = [&](int f) {
      return kept(a.drop, call, i, f) ? to_float(dy[f]) * a.drop.scale : 0.f;
    };
    float s1 = 0.f, s2 = 0.f;
    for (int f = threadIdx.x; f < a.F; f += kThreads) {
      const float g = g_at(f), h = st.norm(to_float(x[f])), t = a.gamma ? g * a.gamma[f] : g;
      s1 += t;
      s2 = __builtin_fmaf(t, h, s2);
      if (a.part) {
        pg[f] = __builtin_fmaf(g, h, pg[f]);
        pb[f] += g;
      }
    }
    const float m1 = block_sum(s1) / (float)a.F, m2 = block_sum(s2) / (float)a.F;
    if (!a.out) continue;
    for (int f = threadIdx.x; f < a.F; f += kThreads) {
      const float g = g_at(f), h = st.norm(to_float(x[f])), t = a.gamma ? g * a.gamma[f] : g;
      dx[f] = from_float<T>(st.rstd * (t - m1 - h * m2));
    }
  }
}

// dgamma and dbeta from the workgroups' rows of sums: 16 columns by 64 lines of threads, each
// of which adds every 64th row in double, then the 64 sums in turn.
__global__ __launch_bounds__(1024) void k_norm_sums(int64_t blocks, int F, const float* part,
                                                    float* dgamma, float* dbeta) {
  __shared__ double sums[64][16];
  const int l = threadIdx.x & 15, w = threadIdx.x >> 4;
  const int64_t c = (int64_t)blockIdx.x * 16 + l;
  double s = 0.0;
  if (c < 2 * (int64_t)F)
#pragma unroll 8
    for (int64_t b = w; b < blocks; b += 64) s += (double)part[b * 2 * F + c];
  sums[w][l] = s;
  __syncthreads();
  if (w > 0 || c >= 2 * (int64_t)F) return;
#pragma unroll 8
  for (int k = 1; k < 64; ++k) s += sums[k][l];
  float* out = c < F ? dgamma : dbeta;
  if (out) out[c < F ? c : c - F] = (float)s;
}

// ---- launch ----------------------------------------------------------------------

constexpr int kLongest = 16384;  // longer rows do not fit the registers of 1024 threads

// The shape for rows of F elements: lanes that hold a row in 4 to 16 elements of each.
template <class T, class Do>
gcn_status with_shape(int F, Do go) {
  constexpr int P = 16 / kPiece<T>;  // pieces of 16 elements
  using std::integral_constant;
  if (F <= 8 * kPiece<T>) return go(integral_constant<int, 8>(), integral_constant<int, 1>());
  if (F <= 64) return go(integral_constant<int, 8>(), integral_constant<int, P / 2>());
  if (F <= 128) return go(integral_constant<int, 16>(), integral_constant<int, P / 2>());
  if (F <= 256) return go(integral_constant<int, 16>(), integral_constant<int, P>());
  if (F <= 512) return go(integral_constant<int, 32>(), integral_constant<int, P>());
  if (F <= 1024) return go(integral_constant<int, 64>(), integral_constant<int, P>());
  if (F <= 2048) return go(integral_constant<int, 256>(), integral_constant<int, P / 2>());
  if (F <= 4096) return go(integral_constant<int, 256>(), integral_constant<int, P>());
  if (F <= 8192) return go(integral_constant<int, 512>(), integral_constant<int, P>());
  return go(integral_constant<int, 1024>(), integral_constant<int, P>());
}

template <class Do>
void with_flags(bool first, bool second, Do go) {
  if (first)
    second ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
  else
    second ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
}

// Workgroups of a kernel that the device holds at a time: as many walk the rows (2,449,029 x 256
// fp32 forward 945 us, with twice as many 1004; 16,384 x 4096 bf16 backward 116 and 129, whose
// sums each cost a row of partial sums).
template <class Kernel>
int64_t resident(Kernel kernel, int threads) {
  int dev = 0, cus = 256, per_cu = 2;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, threads, 0) != hipSuccess)
    (void)hipGetLastError();
  return (int64_t)std::max(1, cus) * std::max(1, per_cu);
}

template <class T>
gcn_status norm_fwd(const NormArgs& a, bool drop, hipStream_t s) {
  ProfScope ps("layernorm_affine_fwd", s);
  if (a.F > kLongest) {
    hipLaunchKernelGGL(k_norm_fwd_long<T>, dim3((unsigned)std::min<int64_t>(a.n, 4096)),
                       dim3(kThreads), 0, s, a);
    GCN_HIP(hipGetLastError());
    return GCN_OK;
  }
  return with_shape<T>(a.F, [&](auto g, auto nv) {
    constexpr int G = decltype(g)::value, NV = decltype(nv)::value;
    constexpr int slots = threads_of(G) / G;
    with_flags(drop, a.F == G * NV * kPiece<T>, [&](auto d, auto full) {
      auto kernel = k_norm_fwd<T, G, NV, decltype(d)::value, decltype(full)::value>;
      static const int64_t fit = resident(kernel, threads_of(G));
      const int64_t blocks = std::min(ceil_div(a.n, (int64_t)slots), fit);
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads_of(G)), 0, s, a);
    });
    GCN_HIP(hipGetLastError());
    return GCN_OK;
  });
}

gcn_status norm_sums(const NormArgs& a, int64_t blocks, hipStream_t s) {
  hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)ceil_div(2 * (int64_t)a.F, (int64_t)16)),
                     dim3(1024), 0, s, blocks, a.F, (const float*)a.part, a.dgamma, a.dbeta);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <class T>
gcn_status norm_bwd(NormArgs a, bool drop, Scratch* scratch, hipStream_t s) {
  ProfScope ps("layernorm_affine_bwd", s);
  const bool want_w = a.dgamma || a.dbeta;
  if (a.n == 0) return want_w && !scratch->asked() ? norm_sums(a, 0, s) : GCN_OK;
  if (a.F > kLongest) {
    const int64_t blocks = std::min<int64_t>(a.n, 512);
    if (want_w) GCN_CHECK(scratch->alloc(&a.part, blocks * 2 * a.F, "sums of the weights' gradients"));
    if (scratch->asked()) return GCN_OK;
    hipLaunchKernelGGL(k_norm_bwd_long<T>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
    GCN_HIP(hipGetLastError());
    return want_w ? norm_sums(a, blocks, s) : GCN_OK;
  }
  return with_shape<T>(a.F, [&](auto g, auto nv) {
    constexpr int G = decltype(g)::value, NV = decltype(nv)::value;
    constexpr int slots = threads_of(G) / G;
    int64_t blocks = 0;
    gcn_status st = GCN_OK;
    with_flags(drop, a.F == G * NV * kPiece<T>, [&](auto d, auto full) {
      auto kernel = k_norm_bwd<T, G, NV, decltype(d)::value, decltype(full)::value>;
      // four rows and more to a slot: with one workgroup the sums are the results
      static const int64_t fit = resident(kernel, threads_of(G));
      blocks = std::min(ceil_div(a.n, (int64_t)4 * slots), fit);
      if (want_w && blocks > 1)
        st = scratch->alloc(&a.part, blocks * 2 * a.F, "sums of the weights' gradients");
      if (st == GCN_OK && !scratch->asked())
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads_of(G)), 0, s, a);
    });
    GCN_CHECK(st);
    GCN_HIP(hipGetLastError());
    return want_w && blocks > 1 && !scratch->asked() ? norm_sums(a, blocks, s) : GCN_OK;
  });
}

gcn_status check_eps(double eps) {
  if (eps >= 0.0) return GCN_OK;
  set_error("need eps >= 0");
  return GCN_EINVAL;
}

}  // namespace
}  // namespace gcn

using namespace gcn;

extern "C" gcn_status gcn_layernorm_affine_fwd(int64_t n, int64_t F, const void* X, int64_t ldx,
                                               int dtype, const float* gamma, const float* beta,
                                               double eps, const gcn_dropout_spec* drop, void* Y,
                                               int64_t ldy, void* stream) {
  clear_error();
  GCN_CHECK(check_rows(n, F, dtype));
  GCN_CHECK(check_eps(eps));
  NormArgs a{n, (int)F, X, ldx, gamma, beta, eps, {}, nullptr, 0, Y, ldy, nullptr, nullptr, nullptr};
  GCN_CHECK(make_drop(drop, n, &a.drop));
  if (n == 0) return GCN_OK;
  if (!X || !Y || ldx < F || ldy < F || (X == Y && ldx != ldy)) {
    set_error("X and Y must be non-NULL with ldx, ldy >= F (and one stride where Y is X)");
    return GCN_EINVAL;
  }
  hipStream_t s = (hipStream_t)stream;
  const bool on = a.drop.least > 0;
  return dtype == GCN_DT_F32 ? norm_fwd<float>(a, on, s) : norm_fwd<bf16>(a, on, s);
}

extern "C" gcn_status gcn_layernorm_affine_bwd(int64_t n, int64_t F, const void* X, int64_t ldx,
                                               int dtype, const float* gamma, double eps,
                                               const gcn_dropout_spec* drop, const void* dY,
                                               int64_t lddy, void* dX, int64_t lddx, float* dgamma,
                                               float* dbeta, void* work, int64_t* work_bytes,
                                               void* stream) {
  clear_error();
  CallScope scope(stream);
  GCN_CHECK(check_rows(n, F, dtype));
  GCN_CHECK(check_eps(eps));
  NormArgs a{n, (int)F, X, ldx, gamma, nullptr, eps, {}, dY, lddy, dX, lddx, dgamma, dbeta, nullptr};
  GCN_CHECK(make_drop(drop, n, &a.drop));
  if (n > 0 && (!X || !dY || ldx < F || lddy < F || (dX && lddx < F) ||
                (dX == X && lddx != ldx) || (dX == dY && lddx != lddy))) {
    set_error("X and dY must be non-NULL with leading dimensions >= F (and one stride where dX is "
              "one of them)");
    return GCN_EINVAL;
  }
  if (!dX && !dgamma && !dbeta) {
    set_error("at least one of dX, dgamma and dbeta must be non-NULL");
    return GCN_EINVAL;
  }
  GCN_CHECK(check_work(work, work_bytes));
  hipStream_t s = (hipStream_t)stream;
  Scratch scratch(work, work_bytes, s);
  const bool on = a.drop.least > 0;
  return dtype == GCN_DT_F32 ? norm_bwd<float>(a, on, &scratch, s)
                             : norm_bwd<bf16>(a, on, &scratch, s);
}
