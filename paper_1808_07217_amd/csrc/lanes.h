// A value of each lane combined over rows of 16 lanes or the whole wavefront, the result in every
// lane: by rotations within a row (by 8, 4, 2, 1) and exchanges between rows, which take a few cycles
// where a permutation by way of LDS takes a hundred. Lanes combine the same pairs in the same
// order up to the order within a pair: with a commutative `f` all end with the same bits.
#pragma once
#include "kernels.h"

namespace lsgd {

template <int N>
__device__ __forceinline__ uint32_t rotated(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, false);
}
template <int N, class V>
__device__ __forceinline__ V row_rotated(V v) {
  if constexpr (sizeof(V) == 8) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, (uint64_t)rotated<N>((uint32_t)(b >> 32)) << 32 |
                                     rotated<N>((uint32_t)b));
  } else {
    return __builtin_bit_cast(V, rotated<N>(__builtin_bit_cast(uint32_t, v)));
  }
}
// rows 2 i and 2 i + 1 (HALVES: the halves of the wavefront) side by side in both
template <bool HALVES, class V>
__device__ __forceinline__ void paired(V v, V& a, V& b) {
  auto swap = [](uint32_t w) __attribute__((always_inline)) {
    if constexpr (HALVES)
      return __builtin_amdgcn_permlane32_swap(w, w, false, false);
    else
      return __builtin_amdgcn_permlane16_swap(w, w, false, false);
  };
  if constexpr (sizeof(V) == 8) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const auto lo = swap((uint32_t)w), hi = swap((uint32_t)(w >> 32));
    a = __builtin_bit_cast(V, (uint64_t)hi[0] << 32 | lo[0]);
    b = __builtin_bit_cast(V, (uint64_t)hi[1] << 32 | lo[1]);
  } else {
    const auto p = swap(__builtin_bit_cast(uint32_t, v));
    a = __builtin_bit_cast(V, (uint32_t)p[0]);
    b = __builtin_bit_cast(V, (uint32_t)p[1]);
  }
}
// lanes l ^ 1 (N = 1) or l ^ 2 of each four
template <int N, class V>
__device__ __forceinline__ V quad_swapped(V v) {
  auto swap = [](uint32_t w) __attribute__((always_inline)) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, w, N == 1 ? 0xB1 : 0x4E, 0xf, 0xf, false);
  };
  if constexpr (sizeof(V) == 8) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, (uint64_t)swap((uint32_t)(b >> 32)) << 32 | swap((uint32_t)b));
  } else {
    return __builtin_bit_cast(V, swap(__builtin_bit_cast(uint32_t, v)));
  }
}
template <class V, class F>
__device__ __forceinline__ V over_rows(V v, F f) {
  V a, b;
  paired<false>(v, a, b);
  v = f(a, b);
  paired<true>(v, a, b);
  return f(a, b);
}
// each T neighbouring lanes by themselves: 1, 4, 16 or 64
template <int T, class V, class F>
__device__ __forceinline__ V over_lanes(V v, F f) {
  static_assert(T == 1 || T == 4 || T == 16 || T == 64, "lanes, fours, rows of 16 or a wavefront");
  if constexpr (T == 4) {
    v = f(v, quad_swapped<2>(v));
    v = f(v, quad_swapped<1>(v));
  } else if constexpr (T >= 16) {
    v = f(v, row_rotated<8>(v));
    v = f(v, row_rotated<4>(v));
    v = f(v, row_rotated<2>(v));
    v = f(v, row_rotated<1>(v));
    if constexpr (T == 64) v = over_rows(v, f);
  }
  return v;
}
template <int T, class V>
__device__ __forceinline__ V lanes_sum(V v) {
  return over_lanes<T>(v, [](V a, V b) __attribute__((always_inline)) { return a + b; });
}
// the other way: lanes l, l + T, l + 2 T, ... of the wavefront
template <int T, class V>
__device__ __forceinline__ V strided_sum(V v) {
  static_assert(T == 1 || T == 4 || T == 16 || T == 64, "");
  if constexpr (T <= 4) {
    v += row_rotated<8>(v);
    v += row_rotated<4>(v);
  }
  if constexpr (T == 1) {
    v += row_rotated<2>(v);
    v += row_rotated<1>(v);
  }
  if constexpr (T <= 16)
    v = over_rows(v, [](V a, V b) __attribute__((always_inline)) { return a + b; });
  return v;
}

}  // namespace lsgd
