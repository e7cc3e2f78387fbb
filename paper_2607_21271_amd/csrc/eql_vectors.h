// eql_vectors.h -- rows in vectors of 16 or 8 bytes, whatever their length and alignment.
//   kWhole: every vector is aligned and full.  kLoose: a row's last vector ends where the row does, its first `skip`
// elements are those of the one before, which owns them; all are read at the elements' own alignment, which the memory
// takes (a convolution of four taps over 1275 f16 columns: 3.1 TB/s, with single elements 1.3).  kTiny: rows shorter than
// a vector, n elements one by one.
#pragma once
#include "eql_common.h"
#include "eql_config.h"
#include "eql_recurrent.h"

namespace eqk {

typedef uint32_t u32x4_loose __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_loose __attribute__((ext_vector_type(2), aligned(2)));
template <int W, int MODE>
struct VectorOf {
  using T = u32x4_loose;
};
template <>
struct VectorOf<4, kWhole> {
  using T = u32x4;
};
template <>
struct VectorOf<2, kWhole> {
  using T = u32x2;
};
template <>
struct VectorOf<2, kLoose> {
  using T = u32x2_loose;
};

// a vector as raw words; kTiny: n elements, 0 behind them
template <int DT, int VEC, int MODE>
__device__ __forceinline__ void load_vector(const void* p, int n, uint32_t* w) {
  constexpr int EB = Elem<DT>::bytes, W = VEC * EB / 4;
  if constexpr (MODE != kTiny) {
    const auto v = *reinterpret_cast<const typename VectorOf<W, MODE>::T*>(p);
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = v[i];
  } else if constexpr (EB == 4) {
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[i] = i < n ? q[i] : 0u;
  } else {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t lo = 2 * i < n ? q[2 * i] : 0u, hi = 2 * i + 1 < n ? q[2 * i + 1] : 0u;
      w[i] = lo | hi << 16;
    }
  }
}
// its elements from `skip` on (kLoose) or before n (kTiny)
template <int DT, int VEC, int MODE>
__device__ __forceinline__ void store_vector(void* p, int skip, int n, const float* f) {
  using E = typename Elem<DT>::T;
  constexpr int EB = Elem<DT>::bytes, W = VEC * EB / 4;
  if (MODE == kWhole || (MODE == kLoose && skip == 0)) {
    typename VectorOf<W, MODE>::T v;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = pack2<DT>(f[i * (4 / EB)], f[i * (4 / EB) + (EB == 2)]);
    *reinterpret_cast<typename VectorOf<W, MODE>::T*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (MODE == kLoose ? i >= skip : i < n) reinterpret_cast<E*>(p)[i] = (E)f[i];
  }
}

}  // namespace eqk
