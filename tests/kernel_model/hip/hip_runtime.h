// A model of what the typed layers' kernels use of HIP, for a build on the CPU: every thread of a
// workgroup is a fiber, the lanes of a wavefront meet where they exchange values, all of them at
// barriers. Device memory lies between pages that nothing may touch (model.cpp).
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstring>

#define __device__
#define __global__
#define __host__
#define __shared__ static
#define __launch_bounds__(...)
#define __align__(n) __attribute__((aligned(n)))

enum hipError_t { hipSuccess = 0, hipErrorOutOfMemory = 2 };
enum hipDeviceAttribute_t { hipDeviceAttributeMultiprocessorCount = 1 };
typedef struct ModelStream* hipStream_t;
typedef struct ModelEvent* hipEvent_t;
inline hipError_t hipGetLastError() { return hipSuccess; }
inline hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
inline hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) {
  return *v = 256, hipSuccess;
}
template <class K>
hipError_t hipOccupancyMaxActiveBlocksPerMultiprocessor(int* v, K, int, size_t) {
  return *v = 2, hipSuccess;
}

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
struct float2 {
  float x, y;
};
inline float2 make_float2(float x, float y) { return {x, y}; }
extern dim3 threadIdx, blockIdx, gridDim;
using std::max;
using std::min;

namespace model {
// The values that the lanes of a wavefront gave: 64 slots of 64 bytes, and which lanes did.
struct Given {
  char v[64][64];
  uint64_t lanes;
  template <class T>
  T of(int lane) const {
    T t;
    memcpy(&t, v[lane & 63], sizeof(T));
    return t;
  }
};
const Given& give(const char* what, const void* v, size_t n);
void barrier();
void run(dim3 grid, dim3 block, void (*go)(void*), void* self);
template <class F>
void launch(dim3 grid, dim3 block, F f) {
  run(grid, block, [](void* p) { (*static_cast<F*>(p))(); }, &f);
}
inline int lane() { return threadIdx.x & 63; }
template <class T>
T from_lane(const char* what, T v, int l) {
  return give(what, &v, sizeof v).template of<T>(l);
}
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
}  // namespace model

#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) \
  model::launch((grid), (block), [&] { (kernel)(__VA_ARGS__); })

inline void __syncthreads() { model::barrier(); }
inline uint32_t __float_as_uint(float v) { return __builtin_bit_cast(uint32_t, v); }
inline float __uint_as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
inline int __float_as_int(float v) { return __builtin_bit_cast(int, v); }
inline float __int_as_float(int v) { return __builtin_bit_cast(float, v); }
inline long long __double_as_longlong(double v) { return __builtin_bit_cast(long long, v); }
inline double __longlong_as_double(long long v) { return __builtin_bit_cast(double, v); }
inline int __clzll(long long v) { return v ? __builtin_clzll((unsigned long long)v) : 64; }

inline int __popcll(unsigned long long v) { return __builtin_popcountll(v); }
template <class T>
T atomicAdd(T* p, T v) {  // (workgroups run in processes that share the arrays)
  return __atomic_fetch_add(p, v, __ATOMIC_SEQ_CST);
}
inline void __threadfence() { __atomic_thread_fence(__ATOMIC_SEQ_CST); }
// the lanes of a wavefront do what stands before it before any does what stands behind it
inline void __builtin_amdgcn_fence(int, const char*) {
  const char c = 0;
  model::give("fence", &c, 1);
}

inline uint64_t __ballot(bool p) {
  const model::Given& g = model::give("ballot", &p, sizeof p);
  uint64_t m = 0;
  for (int l = 0; l < 64; ++l)
    if (g.lanes >> l & 1 && g.of<bool>(l)) m |= 1ull << l;
  return m;
}
inline bool __any(bool p) { return __ballot(p) != 0; }
template <class T>
T __shfl_xor(T v, int off, int) {
  return model::from_lane("shfl_xor", v, model::lane() ^ off);
}
template <class T>
T __shfl_up(T v, unsigned off, int) {
  const int from = model::lane() - (int)off;
  return model::from_lane("shfl_up", v, from < 0 ? model::lane() : from);
}
inline int __builtin_amdgcn_readlane(int v, int l) { return model::from_lane("readlane", v, l); }
inline int __builtin_amdgcn_readfirstlane(int v) {
  const model::Given& g = model::give("readfirstlane", &v, sizeof v);
  return g.of<int>(__builtin_ctzll(g.lanes));
}
inline int __builtin_amdgcn_update_dpp(int old, int v, int ctrl, int rows, int, bool) {
  const model::Given& g = model::give("dpp", &v, sizeof v);
  const int l = model::lane(), row = l / 16;
  int from = -1;
  if (ctrl < 0x100) from = (l & ~3) | (ctrl >> 2 * (l & 3) & 3);                          // quad_perm
  if (ctrl > 0x110 && ctrl < 0x120) from = l % 16 >= ctrl - 0x110 ? l - (ctrl - 0x110) : -1;  // row_shr
  if (ctrl == 0x140) from = l ^ 15;                     // row_mirror
  if (ctrl == 0x141) from = l ^ 7;                      // row_half_mirror
  if (ctrl == 0x142) from = row > 0 ? 16 * row - 1 : -1;  // row_bcast:15
  if (ctrl == 0x143) from = row > 1 ? 31 : -1;            // row_bcast:31
  return rows >> row & 1 && from >= 0 ? g.of<int>(from) : old;
}
inline int __builtin_amdgcn_mov_dpp(int v, int ctrl, int rows, int banks, bool b) {
  return __builtin_amdgcn_update_dpp(0, v, ctrl, rows, banks, b);
}
inline uint32_t __builtin_amdgcn_perm(uint32_t hi, uint32_t lo, uint32_t sel) {
  const uint64_t v = (uint64_t)hi << 32 | lo;
  uint32_t r = 0;
  for (int i = 0; i < 4; ++i) r |= (uint32_t)(v >> 8 * (sel >> 8 * i & 7) & 255) << 8 * i;
  return r;
}
inline float __builtin_amdgcn_exp2f(float v) { return std::exp2(v); }
inline double __builtin_amdgcn_rsq(double v) { return 1.0 / std::sqrt(v); }
inline void __builtin_amdgcn_s_waitcnt(int) {}
inline void __builtin_amdgcn_sched_group_barrier(int, int, int) {}
// 16 bytes of each lane to LDS, one lane's behind the other's
inline void __builtin_amdgcn_global_load_lds(const __attribute__((address_space(1))) void* from,
                                             __attribute__((address_space(3))) void* to, int size,
                                             int, int) {
  memcpy((char*)to + model::lane() * size, (const char*)from, size);
}
// of 16 lanes, lane i names 4 elements of line i / 4 and gets element i of each of the 4 lines
inline model::s4 __builtin_amdgcn_ds_read_tr16_b64_v4i16(__attribute__((address_space(3))) model::s4* p) {
  const model::s4 v = *(model::s4*)p;
  const model::Given& g = model::give("ds_read_tr16", &v, sizeof v);
  const int l = model::lane(), i = l & 15;
  model::s4 r;
  for (int q = 0; q < 4; ++q) r[q] = g.of<model::s4>((l & 48) + 4 * q + i / 4)[i % 4];
  return r;
}
// Operands as the instructions hold them: lane l has row (column) l % rows and the inner size
// from each * (l / rows) on.
template <int ROWS, int EACH, class V>
struct ModelOperands {
  float a[EACH], b[EACH];
  ModelOperands(V x, V y) {
    for (int i = 0; i < EACH; ++i) {
      if constexpr (EACH == 1)
        a[i] = x, b[i] = y;
      else
        a[i] = (float)x[i], b[i] = (float)y[i];
    }
  }
  // the product of a row and the lane's own column
  static float row(const model::Given& g, int r) {
    const int c = model::lane() % ROWS;
    float s = 0.f;
    for (int l = 0; l < 64; l += ROWS) {
      const float* x = reinterpret_cast<const float*>(g.v[l + r]);
      const float* y = reinterpret_cast<const float*>(g.v[l + c]) + EACH;
      for (int i = 0; i < EACH; ++i) s += x[i] * y[i];
    }
    return s;
  }
};
inline model::f16 __builtin_amdgcn_mfma_f32_32x32x16_bf16(model::bf8 a, model::bf8 b, model::f16 c, int,
                                                          int, int) {
  typedef ModelOperands<32, 8, model::bf8> O;
  const O o(a, b);
  const model::Given& g = model::give("mfma_32x32x16", &o, sizeof o);
  for (int e = 0; e < 16; ++e) c[e] += O::row(g, (e & 3) + 8 * (e >> 2) + 4 * (model::lane() >> 5));
  return c;
}
inline model::f16 __builtin_amdgcn_mfma_f32_32x32x2f32(float a, float b, model::f16 c, int, int, int) {
  typedef ModelOperands<32, 1, float> O;
  const O o(a, b);
  const model::Given& g = model::give("mfma_32x32x2", &o, sizeof o);
  for (int e = 0; e < 16; ++e) c[e] += O::row(g, (e & 3) + 8 * (e >> 2) + 4 * (model::lane() >> 5));
  return c;
}
inline model::f4 __builtin_amdgcn_mfma_f32_16x16x32_bf16(model::bf8 a, model::bf8 b, model::f4 c, int, int,
                                                         int) {
  typedef ModelOperands<16, 8, model::bf8> O;
  const O o(a, b);
  const model::Given& g = model::give("mfma_16x16x32", &o, sizeof o);
  for (int e = 0; e < 4; ++e) c[e] += O::row(g, 4 * (model::lane() >> 4) + e);
  return c;
}
inline model::f4 __builtin_amdgcn_mfma_f32_16x16x4f32(float a, float b, model::f4 c, int, int, int) {
  typedef ModelOperands<16, 1, float> O;
  const O o(a, b);
  const model::Given& g = model::give("mfma_16x16x4", &o, sizeof o);
  for (int e = 0; e < 4; ++e) c[e] += O::row(g, 4 * (model::lane() >> 4) + e);
  return c;
}
