// The dropout mask: Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011, whose tests it passes from 7
// rounds on) over counters that name the element, so that the backward pass
// forms the same mask from the same numbers (include/gcnagg.h has the layout).
#pragma once

#include "common.h"

namespace gcn {

// A gcn_dropout_spec as kernels take it.
struct Drop {
  uint32_t least;  // words below it are dropped
  float scale;     // 1 / (1 - p)
  uint32_t k0, k1;
  uint64_t call;
  const uint64_t* step;
  uint32_t row0;
};

// Checks a spec for n rows; GCN_OK and no dropout (least = 0, scale = 1) without one.
gcn_status make_drop(const gcn_dropout_spec* spec, int64_t n, Drop* out);

#ifdef __HIPCC__
// The words of columns 4 block .. 4 block + 3 of a row; call: of the spec, with
// its step added.
__device__ inline void drop_words(const Drop& d, uint64_t call, uint32_t row, uint32_t block,
                                  uint32_t (&w)[4]) {
  uint32_t c0 = block, c1 = d.row0 + row, c2 = (uint32_t)call, c3 = (uint32_t)(call >> 32);
  uint32_t k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    c0 = n0;
    c2 = n2;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0;
  w[1] = c1;
  w[2] = c2;
  w[3] = c3;
}

// Columns f .. f + N - 1 of a row (f and N multiples of 4).
template <int N>
__device__ inline void drop_piece(const Drop& d, uint64_t call, uint32_t row, int f, float (&v)[N]) {
#pragma unroll
  for (int b = 0; b < N; b += 4) {
    uint32_t w[4];
    drop_words(d, call, row, (uint32_t)(f + b) / 4, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[b + e] = w[e] >= d.least ? v[b + e] * d.scale : 0.f;
  }
}

__device__ inline uint64_t drop_call(const Drop& d) { return d.call + (d.step ? *d.step : 0); }
#endif

}  // namespace gcn
