// Row LayerNorm with weights and the dropout behind it, forward and backward.

#include <algorithm>

#include "dropout.h"
#include "element.h"

namespace gcn {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

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
};

// Sum over the workgroup (every thread gets it).
template <class V>
__device__ inline V block_sum(V v) {
  __shared__ V part[kWaves];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();  // the values of the sum before have been read
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < kWaves; ++w) v += part[w];
  return v;
}

// mean as the sum of two floats (h = ((x - hi) - lo) rstd loses nothing where the
// mean is far from 0), and 1 / sqrt(var + eps).
struct Stats {
  float hi, lo, rstd;
  __device__ inline float norm(float x) const { return ((x - hi) - lo) * rstd; }
};

template <class T>
__device__ inline Stats row_stats(const T* x, int F, double eps) {
  double s = 0.0;
  for (int f = threadIdx.x; f < F; f += kThreads) s += (double)to_float(x[f]);
  const double mean = block_sum(s) / (double)F;
  double q = 0.0;
  for (int f = threadIdx.x; f < F; f += kThreads) {
    const double d = (double)to_float(x[f]) - mean;
    q += d * d;
  }
  const double var = block_sum(q) / (double)F;
  const float hi = (float)mean;
  return Stats{hi, (float)(mean - (double)hi), (float)(1.0 / sqrt(var + eps))};
}

// The factor of element (i, f): scale where it is kept, else 0.
__device__ inline bool kept(const Drop& d, uint64_t call, int64_t i, int f) {
  uint32_t w[4];
  drop_words(d, call, (uint32_t)i, (uint32_t)f >> 2, w);
  return w[f & 3] >= d.least;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_fwd(NormArgs a) {
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

// A workgroup's rows: i = blockIdx.x, + gridDim.x, ...; part [gridDim.x][2][F]
// gets its sums of G H and G.
template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(NormArgs a, float* part) {
  const uint64_t call = drop_call(a.drop);
  float* pg = part + (int64_t)blockIdx.x * 2 * a.F;
  float* pb = pg + a.F;
  if (part)
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
      s2 += t * h;
      if (part) {
        pg[f] += g * h;
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

// dgamma and dbeta: the sums of the workgroups' partial rows, in their order.
__global__ __launch_bounds__(kThreads) void k_norm_sums(int64_t blocks, int F, const float* part,
                                                        float* dgamma, float* dbeta) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= 2 * (int64_t)F) return;
  float* out = c < F ? dgamma : dbeta;
  if (!out) return;
  double s = 0.0;
  for (int64_t b = 0; b < blocks; ++b) s += (double)part[b * 2 * F + c];
  out[c < F ? c : c - F] = (float)s;
}

constexpr int64_t kRowBlocks = 2048;

template <class T>
gcn_status norm_fwd(const NormArgs& a, hipStream_t s) {
  ProfScope ps("layernorm_affine_fwd", s);
  hipLaunchKernelGGL(k_norm_fwd<T>, dim3((unsigned)std::min(a.n, 8 * kRowBlocks)), dim3(kThreads),
                     0, s, a);
  GCN_HIP(hipGetLastError());
  return GCN_OK;
}

template <class T>
gcn_status norm_bwd(const NormArgs& a, float* dgamma, float* dbeta, hipStream_t s) {
  ProfScope ps("layernorm_affine_bwd", s);
  TempScope temps(s);
  const int64_t blocks = std::min(a.n, kRowBlocks);
  float* part = nullptr;
  if ((dgamma || dbeta) && blocks > 0)
    GCN_CHECK(temps.alloc(&part, blocks * 2 * a.F, "sums of the weights' gradients"));
  if (blocks > 0) {
    hipLaunchKernelGGL(k_norm_bwd<T>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, part);
    GCN_HIP(hipGetLastError());
  }
  if (dgamma || dbeta) {
    hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)ceil_div(2 * (int64_t)a.F, (int64_t)kThreads)),
                       dim3(kThreads), 0, s, blocks, a.F, (const float*)part, dgamma, dbeta);
    GCN_HIP(hipGetLastError());
  }
  return GCN_OK;
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
  NormArgs a{n, (int)F, X, ldx, gamma, beta, eps, {}, nullptr, 0, Y, ldy};
  GCN_CHECK(make_drop(drop, n, &a.drop));
  if (n == 0) return GCN_OK;
  if (!X || !Y || ldx < F || ldy < F || (X == Y && ldx != ldy)) {
    set_error("X and Y must be non-NULL with ldx, ldy >= F (and one stride where Y is X)");
    return GCN_EINVAL;
  }
  hipStream_t s = (hipStream_t)stream;
  return dtype == GCN_DT_F32 ? norm_fwd<float>(a, s) : norm_fwd<bf16>(a, s);
}

extern "C" gcn_status gcn_layernorm_affine_bwd(int64_t n, int64_t F, const void* X, int64_t ldx,
                                               int dtype, const float* gamma, double eps,
                                               const gcn_dropout_spec* drop, const void* dY,
                                               int64_t lddy, void* dX, int64_t lddx, float* dgamma,
                                               float* dbeta, void* stream) {
  clear_error();
  CallScope scope(stream);
  GCN_CHECK(check_rows(n, F, dtype));
  GCN_CHECK(check_eps(eps));
  NormArgs a{n, (int)F, X, ldx, gamma, nullptr, eps, {}, dY, lddy, dX, lddx};
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
  hipStream_t s = (hipStream_t)stream;
  return dtype == GCN_DT_F32 ? norm_bwd<float>(a, dgamma, dbeta, s)
                             : norm_bwd<bf16>(a, dgamma, dbeta, s);
}
