// Eight neighbours of a row of floats or bfloat16, at any element's alignment.
#pragma once
#include "kernels.h"

namespace lsgd {

typedef uint32_t row_u32x4 __attribute__((ext_vector_type(4)));
typedef float row_v4f __attribute__((ext_vector_type(4)));
typedef float row_v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t row_u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// From element `at` on, `left` of them (zeros past those).
template <bool BF>
__device__ __forceinline__ void load8(const void* X, long long at, int left, float (&v)[8]) {
  if (left >= 8) {
    if constexpr (BF) {
      const row_u32x4 w = *(const row_u32x4_any*)((const bf16_t*)X + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
      const row_v4f lo = *(const row_v4f_any*)((const float*)X + at);
      const row_v4f hi = *(const row_v4f_any*)((const float*)X + at + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = lo[i];
        v[4 + i] = hi[i];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (i < left) v[i] = BF ? bf16_to_f32(((const bf16_t*)X)[at + i]) : ((const float*)X)[at + i];
    }
  }
}
template <bool BF>
__device__ __forceinline__ void store8(void* Y, long long at, int left, const float (&v)[8]) {
  if (left >= 8) {
    if constexpr (BF) {
      row_u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = f32_to_bf16(v[2 * i]) | (uint32_t)f32_to_bf16(v[2 * i + 1]) << 16;
      *(row_u32x4_any*)((bf16_t*)Y + at) = w;
    } else {
      *(row_v4f_any*)((float*)Y + at) = row_v4f{v[0], v[1], v[2], v[3]};
      *(row_v4f_any*)((float*)Y + at + 4) = row_v4f{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) {
        if constexpr (BF)
          ((bf16_t*)Y)[at + i] = f32_to_bf16(v[i]);
        else
          ((float*)Y)[at + i] = v[i];
      }
  }
}

}  // namespace lsgd
