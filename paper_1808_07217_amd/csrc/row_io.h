// Eight neighbours of a row of floats or bfloat16, at any element's alignment.
#pragma once
#include "kernels.h"

namespace lsgd {

typedef uint32_t row_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t row_u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t row_u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t row_u32_any __attribute__((aligned(2)));

// As they lie in memory: four dwords of bfloat16 or eight of floats.
template <bool BF>
struct Raw8 {
  static constexpr int kDwords = BF ? 4 : 8;
  uint32_t w[kDwords];
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (BF)
      return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else
      return __uint_as_float(w[i]);
  }
  __device__ __forceinline__ void put(const float (&v)[8]) {
    if constexpr (BF) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = f32_to_bf16(v[2 * i]) | (uint32_t)f32_to_bf16(v[2 * i + 1]) << 16;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
    }
  }
  // the first S values leave, zeros follow the last (S a power of two)
  template <int S>
  __device__ __forceinline__ void drop() {
    constexpr int s = BF ? S / 2 : S;
#pragma unroll
    for (int i = 0; i < kDwords; ++i) {
      if constexpr (BF && S == 1)
        w[i] = w[i] >> 16 | (i + 1 < kDwords ? w[i + 1] << 16 : 0u);
      else
        w[i] = i + s < kDwords ? w[i + s] : 0u;
    }
  }
};

// The columns n .. n + 7 of the row of N values that starts at element `row`, zeros past the
// last: fetch8, and settle8 once they are needed. The vector that the row ends in is the row's last
// eight, which settle8 moves: one load whatever N, where a row has eight values (SMALL: it may
// have fewer), and none that waits for another.
template <bool BF, bool SMALL = false>
__device__ __forceinline__ void fetch8(const void* X, long long row, int n, int N, Raw8<BF>& v) {
#pragma unroll
  for (int i = 0; i < Raw8<BF>::kDwords; ++i) v.w[i] = 0;
  if constexpr (SMALL) {
    if (N < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (n + i < N) {
          if constexpr (BF)
            v.w[i / 2] |= (uint32_t)((const bf16_t*)X)[row + n + i] << 16 * (i % 2);
          else
            v.w[i] = ((const uint32_t*)X)[row + n + i];
        }
      return;
    }
  }
  if (n >= N) return;
  const int first = min(n, N - 8);
  if constexpr (BF) {
    const row_u32x4 a = *(const row_u32x4_any*)((const bf16_t*)X + row + first);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = a[i];
  } else {
    const row_u32x4 a = *(const row_u32x4_any*)((const float*)X + row + first);
    const row_u32x4 b = *(const row_u32x4_any*)((const float*)X + row + first + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) v.w[i] = i < 4 ? a[i] : b[i - 4];
  }
}
template <bool BF, bool SMALL = false>
__device__ __forceinline__ void settle8(int n, int N, Raw8<BF>& v) {
  const int left = N - n;
  if (left >= 8 || left <= 0 || (SMALL && N < 8)) return;
  const int k = 8 - left;
  if (k & 4) v.template drop<4>();
  if (k & 2) v.template drop<2>();
  if (k & 1) v.template drop<1>();
}
template <bool BF, bool SMALL = false>
__device__ __forceinline__ void load8(const void* X, long long row, int n, int N, float (&v)[8]) {
  Raw8<BF> r;
  fetch8<BF, SMALL>(X, row, n, N, r);
  settle8<BF, SMALL>(n, N, r);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = r[i];
}

template <bool BF>
__device__ __forceinline__ void store8(void* Y, long long row, int n, int N, Raw8<BF> r) {
  const int left = N - n;
  if (left <= 0) return;
  if constexpr (BF) {
    bf16_t* y = (bf16_t*)Y + row + n;
    if (left >= 8) {
      *(row_u32x4_any*)y = row_u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
      return;
    }
    if (left & 4) {
      *(row_u32x2_any*)y = row_u32x2_any{r.w[0], r.w[1]};
      r.template drop<4>();
      y += 4;
    }
    if (left & 2) {
      *(row_u32_any*)y = r.w[0];
      r.template drop<2>();
      y += 2;
    }
    if (left & 1) *y = (bf16_t)r.w[0];
  } else {
    uint32_t* y = (uint32_t*)Y + row + n;
    if (left >= 4) *(row_u32x4_any*)y = row_u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
    if (left >= 8) {
      *(row_u32x4_any*)(y + 4) = row_u32x4{r.w[4], r.w[5], r.w[6], r.w[7]};
      return;
    }
    if (left & 4) {
      r.template drop<4>();
      y += 4;
    }
    if (left & 2) {
      *(row_u32x2_any*)y = row_u32x2_any{r.w[0], r.w[1]};
      r.template drop<2>();
      y += 2;
    }
    if (left & 1) *y = r.w[0];
  }
}
template <bool BF>
__device__ __forceinline__ void store8(void* Y, long long row, int n, int N, const float (&v)[8]) {
  Raw8<BF> r;
  r.put(v);
  store8<BF>(Y, row, n, N, r);
}

}  // namespace lsgd
