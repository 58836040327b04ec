// Tensors in 8 bits with a power-of-two scale for each block of 128 values along
// a row, and the grouped product of two of them.
//
// A block's scale is 2^e, e the smallest exponent in [-127, 127] with
// max |x| <= 2^e F, F the format's largest value (e4m3: 448 = 1.75 2^8, e5m2:
// 57344 = 1.75 2^15; both 1.75 times a power of two, so that e follows from the
// bits of max |x|). A power of two costs an 8-bit float no precision, only up to
// one binade of its range; x 2^-e is exact in fp32 for whatever rounds to a
// non-zero value, so each element is rounded once. Infinities and NaN stay
// out of the maximum and are stored as the format has them (e4m3 holds no
// infinity: NaN), so that every product that reads one shows it.
#include "device_common.h"
#include "kernels.h"

namespace lsgd {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// vectors at any element's alignment
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kThreads = 256;

// ---------------------------------------------------------------- quantise
// |x| as an integer that orders like it; 0 for infinities and NaN.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// The biased exponent byte e + 127 of a block with max |x| = amax (its bits).
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  constexpr int kTop = FMT == kFmtE4M3 ? 8 : 15;
  if (amax == 0) return 127u;
  const int e = (int)(amax >> 23) - kTop + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 0);
}
// 2^-e of a scale byte (e <= 120, so it is a normal number)
__device__ __forceinline__ float inv_scale(uint32_t byte) {
  return __uint_as_float((254u - byte) << 23);
}
// four values as 8-bit floats, round to nearest even (no overflow: see the top)
template <int FMT>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int v = 0;
  if constexpr (FMT == kFmtE4M3) {
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  } else {
    v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
  }
  return (uint32_t)v;
}

// A tile of 16 RP rows and 128 columns: thread t holds RP rows from RP (t / 16) and
// 8 columns from 8 (t % 16), all in registers. BOTH (RP = 8: a square tile): the
// transposed tensor as well, whose blocks run down the tile's columns, its bytes
// turned in LDS so that each row leaves as a whole 128-byte line.
constexpr int kTurnPitch = 144;  // bytes; 16-byte aligned, not a multiple of the banks' 256
template <bool BF, int FMT, int RP, bool BOTH>
__global__ __launch_bounds__(kThreads) void k_quantise(QuantArgs a, int tm, int tn, int total) {
  static_assert(!BOTH || RP == 8, "the transposed blocks need 128 rows");
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int g = id / (tm * tn), mt = id % (tm * tn) / tn, nt = id % tn;
  const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4;
  const int n0 = nt * 128, m0 = mt * 16 * RP;
  const int n = n0 + c * 8, r0 = m0 + rg * RP;
  float v[RP][8];
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    const int m = r0 + p;
    const long long at = (long long)g * a.sX + (long long)m * a.ldx + n;
    if (m < a.M && n + 8 <= a.N) {
      if constexpr (BF) {
        const u32x4 w = *(const u32x4_any*)((const bf16_t*)a.X + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[p][2 * i] = __uint_as_float(w[i] << 16);
          v[p][2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      } else {
        const v4f lo = *(const v4f_any*)((const float*)a.X + at);
        const v4f hi = *(const v4f_any*)((const float*)a.X + at + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[p][i] = lo[i];
          v[p][4 + i] = hi[i];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[p][i] = 0.f;
        if (m < a.M && n + i < a.N)
          v[p][i] = BF ? bf16_to_f32(((const bf16_t*)a.X)[at + i]) : ((const float*)a.X)[at + i];
      }
    }
  }
  const int ldq = (a.N + 127) / 128 * 128, nb = ldq / 128, lds = (nb + 3) / 4 * 4;
  if (a.Q) {
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = max(amax, finite_bits(v[p][i]));
#pragma unroll
      for (int s = 1; s < 16; s *= 2) amax = max(amax, (uint32_t)__shfl_xor((int)amax, s));
      const uint32_t byte = scale_byte<FMT>(amax);
      const float f = inv_scale(byte);
      const int m = r0 + p;
      if (m >= a.M) continue;
      const long long row = (long long)g * a.M + m;
      u32x2 q;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        q[h] = pack4<FMT>(v[p][4 * h] * f, v[p][4 * h + 1] * f, v[p][4 * h + 2] * f,
                          v[p][4 * h + 3] * f);
      *(u32x2*)(a.Q + row * ldq + n) = q;
      // the block's scale, and behind a row's last block the padding
      if (c == 0) a.S[row * lds + nt] = (uint8_t)byte;
      else if (nt + 1 == nb && nt + c < lds) a.S[row * lds + nt + c] = 127;
    }
  }
  if constexpr (BOTH) {
    __shared__ uint32_t cmax[4][128];
    __shared__ __align__(16) uint8_t turn[128 * kTurnPitch];
    const int wave = tid >> 6, lane = tid & 63;
    uint32_t am[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      am[i] = 0;
#pragma unroll
      for (int p = 0; p < RP; ++p) am[i] = max(am[i], finite_bits(v[p][i]));
      am[i] = max(am[i], (uint32_t)__shfl_xor((int)am[i], 16));
      am[i] = max(am[i], (uint32_t)__shfl_xor((int)am[i], 32));
    }
    if (lane < 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) cmax[wave][c * 8 + i] = am[i];
    }
    __syncthreads();
    const int ldt = (a.M + 127) / 128 * 128, mb = ldt / 128, ldst = (mb + 3) / 4 * 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = c * 8 + i;
      const uint32_t amax = max(max(cmax[0][j], cmax[1][j]), max(cmax[2][j], cmax[3][j]));
      const uint32_t byte = scale_byte<FMT>(amax);
      const float f = inv_scale(byte);
      u32x2 q;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        q[h] = pack4<FMT>(v[4 * h][i] * f, v[4 * h + 1][i] * f, v[4 * h + 2][i] * f,
                          v[4 * h + 3][i] * f);
      *(u32x2*)(turn + j * kTurnPitch + rg * 8) = q;
      if (n + i < a.N) {
        uint8_t* st = a.St + ((long long)g * a.N + n + i) * ldst + mt;
        if (rg == 0) *st = (uint8_t)byte;
        else if (mt + 1 == mb && mt + rg < ldst) st[rg] = 127;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = i * kThreads + tid, j = at >> 3, k = (at & 7) * 16;
      if (n0 + j < a.N)
        *(u32x4*)(a.Qt + ((long long)g * a.N + n0 + j) * ldt + m0 + k) =
            *(const u32x4*)(turn + j * kTurnPitch + k);
    }
  }
}

template <bool BF, int FMT>
hipError_t quantise(const QuantArgs& a, hipStream_t s) {
  const long long tn = (a.N + 127LL) / 128;
  // a tile of 128 rows where the columns' blocks need it, 16 otherwise
  const int rows = a.Qt ? 128 : 16;
  const long long tm = ((long long)a.M + rows - 1) / rows;
  if (tm * tn > 0x7fffffffLL / a.G) return hipErrorInvalidValue;
  const long long total = tm * tn * a.G;
  if (a.Qt)
    hipLaunchKernelGGL((k_quantise<BF, FMT, 8, true>), grid_of(total), dim3(kThreads), 0, s, a,
                       (int)tm, (int)tn, (int)total);
  else
    hipLaunchKernelGGL((k_quantise<BF, FMT, 1, false>), grid_of(total), dim3(kThreads), 0, s, a,
                       (int)tm, (int)tn, (int)total);
  return hipGetLastError();
}

// ------------------------------------------------------------------ product
// Two precisions, by the type of C. bf16: v_mfma_scale_f32_16x16x128_f8f6f4, whose
// scale operands are the blocks' bytes. It sums eight neighbouring products at a
// time with 13 bits below the largest of them (probed: 2^10 + 2^-3 is exact, 2^10 +
// 2^-4 is 2^10) and those sums in fp32: an error of 2^-10 sum |a b| at worst and about
// 2^-15 of it on normal data, well below bf16's own 2^-9. That is too coarse for a
// result in fp32, which instead widens the values, scale and all, to bf16 (exact: 4
// bits of a value, and 2^e is in bf16's range) as they reach the registers and takes
// v_mfma_f32_16x16x32_bf16, half as fast: exact products, fp32 sums.
// Lane l holds 32 of a block's 128 k for row l % 16; which 32 is free, the scale being
// one for all: two vectors of 16 bytes, 64 apart. The first operand is B's rows, so that a
// lane's four results are neighbours in a row of C.
template <int FMT>
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale) {
  bf16x2 p[4];
  if constexpr (FMT == kFmtE4M3) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
  }
  return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// 4 wavefronts, each 32 x 32 of a 64 x 64 tile.
template <int FA, int FB, bool OUTBF>
__global__ __launch_bounds__(kThreads) void k_gemm_blocks(BlockGemmArgs a, int tm, int tn,
                                                          int total) {
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int g = id / (tm * tn), mt = id % (tm * tn) / tn, nt = id % tn;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const int m0 = mt * 64 + (wave >> 1) * 32, n0 = nt * 64 + (wave & 1) * 32;
  const int nb = (a.Kd + 127) / 128;
  const long long ld = nb * 128LL, lds = (nb + 3) / 4 * 4;
  const uint8_t *pa[2], *pb[2], *qa[2], *qb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = min(m0 + i * 16 + lr, a.M - 1), n = min(n0 + i * 16 + lr, a.N - 1);
    pa[i] = a.A + (long long)g * a.sA + m * ld + lq * 16;
    pb[i] = a.B + (long long)g * a.sB + n * ld + lq * 16;
    qa[i] = a.SA + (long long)g * a.sSA + m * lds;
    qb[i] = a.SB + (long long)g * a.sSB + n * lds;
  }
  v4f acc[2][2] = {};
  for (int kb = 0; kb < nb; ++kb) {
    v8i va[2], vb[2];
    int fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const v4i a0 = *(const v4i*)(pa[i] + kb * 128LL), a1 = *(const v4i*)(pa[i] + kb * 128LL + 64);
      const v4i b0 = *(const v4i*)(pb[i] + kb * 128LL), b1 = *(const v4i*)(pb[i] + kb * 128LL + 64);
      va[i] = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
      vb[i] = __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7);
      fa[i] = qa[i][kb];
      fb[i] = qb[i][kb];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (OUTBF) {
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              vb[j], va[i], acc[i][j], FB, FA, 0, fb[j], 0, fa[i]);
        } else {
#pragma unroll
          for (int h = 0; h < 8; h += 2)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                widen<FB>(vb[j][h], vb[j][h + 1], __uint_as_float((unsigned)fb[j] << 23)),
                widen<FA>(va[i][h], va[i][h + 1], __uint_as_float((unsigned)fa[i] << 23)),
                acc[i][j], 0, 0, 0);
        }
      }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int m = m0 + i * 16 + lr, n = n0 + j * 16 + lq * 4;
      if (m >= a.M) continue;
      const long long at = (long long)g * a.sC + (long long)m * a.ldc + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) {
          if constexpr (OUTBF)
            ((bf16_t*)a.C)[at + e] = f32_to_bf16(acc[i][j][e]);
          else
            ((float*)a.C)[at + e] = acc[i][j][e];
        }
    }
}

template <int FA, int FB>
hipError_t gemm_blocks(const BlockGemmArgs& a, hipStream_t s) {
  const long long tm = (a.M + 63LL) / 64, tn = (a.N + 63LL) / 64;
  if (tm * tn > 0x7fffffffLL / a.G) return hipErrorInvalidValue;
  const long long total = tm * tn * a.G;
  if (a.out_bf16)
    hipLaunchKernelGGL((k_gemm_blocks<FA, FB, true>), grid_of(total), dim3(kThreads), 0, s, a,
                       (int)tm, (int)tn, (int)total);
  else
    hipLaunchKernelGGL((k_gemm_blocks<FA, FB, false>), grid_of(total), dim3(kThreads), 0, s, a,
                       (int)tm, (int)tn, (int)total);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantise(int bf16, int fmt, const QuantArgs& a, hipStream_t s) {
  if (fmt == kFmtE4M3)
    return bf16 ? quantise<true, kFmtE4M3>(a, s) : quantise<false, kFmtE4M3>(a, s);
  return bf16 ? quantise<true, kFmtE5M2>(a, s) : quantise<false, kFmtE5M2>(a, s);
}

size_t gemm_blocks_workspace_bytes(int, int, int, int) { return 0; }

hipError_t launch_gemm_blocks(int fmt_a, int fmt_b, const BlockGemmArgs& a, hipStream_t s) {
  if (fmt_a == kFmtE4M3)
    return fmt_b == kFmtE4M3 ? gemm_blocks<kFmtE4M3, kFmtE4M3>(a, s)
                             : gemm_blocks<kFmtE4M3, kFmtE5M2>(a, s);
  return fmt_b == kFmtE4M3 ? gemm_blocks<kFmtE5M2, kFmtE4M3>(a, s)
                           : gemm_blocks<kFmtE5M2, kFmtE5M2>(a, s);
}

}  // namespace lsgd
