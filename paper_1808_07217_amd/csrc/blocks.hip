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
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "tile_loop.h"

namespace lsgd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// vectors at any element's alignment
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kThreads = 256;

// ---------------------------------------------------------------- quantise
// The larger of two magnitudes; a NaN counts for nothing.
__device__ __forceinline__ float larger(float m, float x) { return fmaxf(m, fabsf(x)); }
// 0 in place of an infinity or a NaN
__device__ __forceinline__ float finite(float x) {
  return fabsf(x) <= 3.402823466e38f ? x : 0.f;
}
// The largest of a row of 16 lanes, in all of them: max with the row rotated by 8, 4, 2, 1.
__device__ __forceinline__ float row_max(float m) {
#define LSGD_ROTATED(n) \
  __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(m), 0x120 + n, 0xf, 0xf, false))
  m = fmaxf(m, LSGD_ROTATED(8));
  m = fmaxf(m, LSGD_ROTATED(4));
  m = fmaxf(m, LSGD_ROTATED(2));
  return fmaxf(m, LSGD_ROTATED(1));
#undef LSGD_ROTATED
}
// The largest of a wavefront's four lanes l, l + 16, l + 32, l + 48, in all of them.
__device__ __forceinline__ float column_max(float m) {
  const uint32_t b = __float_as_uint(m);
  const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  const uint32_t c = __float_as_uint(fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const auto q = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
// The biased exponent byte e + 127 of a block whose largest finite magnitude is `max`.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(float max) {
  constexpr int kTop = FMT == kFmtE4M3 ? 8 : 15;
  const uint32_t amax = __float_as_uint(max);
  if (amax == 0) return 127u;
  const int e = (int)(amax >> 23) - kTop + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)(e > 0 ? e : 0);
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
// (rows of 128 bytes; piece k of 16 lies in slot k ^ (row / 8 % 8), which spreads the rows,
// eight apart, that a wavefront writes at once over the banks)
__device__ __forceinline__ int turned(int row, int byte) {
  return row * 128 + (byte ^ (row / 8 % 8 * 16));
}
template <bool BF, int FMT, int RP, bool BOTH, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_quantise(QuantArgs a, int tm, int tn, int total) {
  static_assert(!BOTH || RP == 8, "the transposed blocks need 128 rows");
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int l = xcd_order(id, total);
  const int g = l / (tm * tn), mt = l % (tm * tn) / tn, nt = l % tn;
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
  // past the caches where they could not hold the tensors anyway
  auto put = [&](auto value, auto* to) __attribute__((always_inline)) {
    if constexpr (STREAM)
      __builtin_nontemporal_store(value, to);
    else
      *to = value;
  };
  // Largest magnitudes of the rows and of the columns. With an infinity among them (rare, and
  // looked for only here) once more over the finite values.
  float rm[RP], cm[8];
  auto maxima = [&](auto value) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      rm[p] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) rm[p] = larger(rm[p], value(v[p][i]));
    }
    if constexpr (BOTH) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        cm[i] = 0.f;
#pragma unroll
        for (int p = 0; p < RP; ++p) cm[i] = larger(cm[i], value(v[p][i]));
      }
    }
  };
  maxima([](float x) { return x; });
  float most = 0.f;
#pragma unroll
  for (int p = 0; p < RP; ++p) most = fmaxf(most, rm[p]);
  if (most == __builtin_inff()) maxima([](float x) { return finite(x); });
  const int ldq = (a.N + 127) / 128 * 128, nb = ldq / 128, lds = (nb + 3) / 4 * 4;
  if (a.Q) {
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      const uint32_t byte = scale_byte<FMT>(row_max(rm[p]));
      const float f = inv_scale(byte);
      const int m = r0 + p;
      if (m >= a.M) continue;
      const long long row = (long long)g * a.M + m;
      u32x2 q;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        q[h] = pack4<FMT>(v[p][4 * h] * f, v[p][4 * h + 1] * f, v[p][4 * h + 2] * f,
                          v[p][4 * h + 3] * f);
      put(q, (u32x2*)(a.Q + row * ldq + n));
      // the block's scale, and behind a row's last block the padding
      if (c == 0) a.S[row * lds + nt] = (uint8_t)byte;
      else if (nt + 1 == nb && nt + c < lds) a.S[row * lds + nt + c] = 127;
    }
  }
  if constexpr (BOTH) {
    __shared__ float cmax[4][128];
    __shared__ uint8_t bytes[128];
    __shared__ __align__(16) uint8_t turn[128 * 128];
    const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
    for (int i = 0; i < 8; ++i) cm[i] = column_max(cm[i]);
    if (lane < 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) cmax[wave][c * 8 + i] = cm[i];
    }
    __syncthreads();
    const int ldt = (a.M + 127) / 128 * 128, mb = ldt / 128, ldst = (mb + 3) / 4 * 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = c * 8 + i;
      const uint32_t byte = scale_byte<FMT>(
          fmaxf(fmaxf(cmax[0][j], cmax[1][j]), fmaxf(cmax[2][j], cmax[3][j])));
      const float f = inv_scale(byte);
      u32x2 q;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        q[h] = pack4<FMT>(v[4 * h][i] * f, v[4 * h + 1][i] * f, v[4 * h + 2][i] * f,
                          v[4 * h + 3][i] * f);
      *(u32x2*)(turn + turned(j, rg * 8)) = q;
      if (rg == 0) bytes[j] = (uint8_t)byte;
    }
    __syncthreads();
    if (tid < 128 && n0 + tid < a.N) {
      uint8_t* st = a.St + ((long long)g * a.N + n0 + tid) * ldst + mt;
      *st = bytes[tid];
      for (int k = 1; mt + 1 == mb && mt + k < ldst; ++k) st[k] = 127;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = i * kThreads + tid, j = at >> 3, k = (at & 7) * 16;
      if (n0 + j < a.N)
        put(*(const u32x4*)(turn + turned(j, k)),
            (u32x4*)(a.Qt + ((long long)g * a.N + n0 + j) * ldt + m0 + k));
    }
  }
}

// From kNtBytesCaller of input and output on the values are streamed: 16384 x 8192 in bf16
// both ways (537 MB), repeated on one input, 156 -> 119 us; with 268 MB (8192^2) the call
// itself gains as much, but the product that reads the values next loses more (506 -> 519 us
// together).
template <bool BF, int FMT>
hipError_t quantise(const QuantArgs& a, hipStream_t s) {
  const double bytes = (double)a.M * a.N * a.G *
                       ((BF ? 2 : 4) + (a.Q != nullptr) + (a.Qt != nullptr));
  const bool stream = bytes >= (double)kNtBytesCaller;
  const long long tn = (a.N + 127LL) / 128;
  // a tile of 128 rows where the columns' blocks need it, 16 otherwise
  const int rows = a.Qt ? 128 : 16;
  const long long tm = ((long long)a.M + rows - 1) / rows;
  if (tm * tn > 0x7fffffffLL / a.G) return hipErrorInvalidValue;
  const long long total = tm * tn * a.G;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid_of(total), dim3(kThreads), 0, s, a, (int)tm, (int)tn,
                       (int)total);
    return hipGetLastError();
  };
  if (a.Qt)
    return stream ? launch(k_quantise<BF, FMT, 8, true, true>)
                  : launch(k_quantise<BF, FMT, 8, true, false>);
  return stream ? launch(k_quantise<BF, FMT, 1, false, true>)
                : launch(k_quantise<BF, FMT, 1, false, false>);
}

// ------------------------------------------------------------------ product
// Two precisions, by the type of C. bf16: v_mfma_scale_f32_16x16x128_f8f6f4, whose
// scale operands are the blocks' bytes. It sums eight neighbouring products at a
// time with 13 bits below the largest of them (probed: 2^10 + 2^-3 is exact, 2^10 +
// 2^-4 is 2^10) and those sums in fp32: an error of 2^-10 sum |a b| at worst and about
// 2^-15 of it on normal data, well below bf16's own 2^-8. That is too coarse for a
// result in fp32, which instead widens the values, scale and all, to bf16 (exact: 4
// bits of a value, and 2^e is in bf16's range; only a value below 2^-126 becomes a
// multiple of bf16's 2^-133, and 2^128, to which only fp32's last values round, an infinity) as they reach the registers and takes
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

// The scales of a tile's rows, for two steps at the end of an even step's stage: for each
// row the dword with the bytes of four steps (what a load to LDS moves), of which a lane
// reads the two (read byte by byte for every step they cost 15% of the 8192^3 product's
// time).
template <int BP, int BQ, int FP, int FQ>
struct Scales {
  struct Next {
    uint32_t p[FP], q[FQ];  // an even step's byte and the odd one's
  };
  static constexpr int kEvenLoads = 1, kLoads = (BP + BQ) / 64, kAt = (BP + BQ) * 128;
  const uint8_t *P, *Q;
  int leftp, leftq, wave, row, rp, rq;
  Next s;
  // (arguments as TileLoop::init's; wp, wq: the wavefront's place in the tile;
  // k0: the first step, a multiple of four)
  __device__ __forceinline__ void init(const uint8_t* p, const uint8_t* q, int pitch, int np,
                                       int nq, int wp, int wq, int k0) {
    const int lane = threadIdx.x & 63;
    // (a tile of fewer rows than threads loads them more than once)
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kLoads;
    P = p + k0;
    Q = q + k0;
    leftp = min(np, BP) * pitch - k0;
    leftq = min(nq, BQ) * pitch - k0;
    row = ((wave < BP / 64 ? wave : wave - BP / 64) * 64 + lane) * pitch;
    rp = kAt + 4 * (wp + (lane & 15));
    rq = kAt + 4 * (BP + wq + (lane & 15));
  }
  __device__ __forceinline__ void load(uint8_t* stage, int k, bool want) {
    const bool isp = wave < BP / 64;
    const int at = k & ~3, left = (isp ? leftp : leftq) - at;
    const __amdgpu_buffer_rsrc_t b = __builtin_amdgcn_make_buffer_rsrc(
        (void*)((isp ? P : Q) + at), 0, want ? left : 0, kRsrcRaw);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        b, (__attribute__((address_space(3))) void*)(stage + kAt + wave * 256), 4, row, 0, 0, 0);
  }
  __device__ __forceinline__ void begin(const uint8_t* stage, int k, Next& up) const {
#pragma unroll
    for (int i = 0; i < FP; ++i) up.p[i] = *(const uint16_t*)(stage + rp + (k & 2) + i * 64);
#pragma unroll
    for (int j = 0; j < FQ; ++j) up.q[j] = *(const uint16_t*)(stage + rq + (k & 2) + j * 64);
  }
  __device__ __forceinline__ void take(const Next& up) { s = up; }
  __device__ __forceinline__ void last(bool odd) {
#pragma unroll
    for (int i = 0; i < FP; ++i) s.p[i] >>= odd ? 8 : 0;
#pragma unroll
    for (int j = 0; j < FQ; ++j) s.q[j] >>= odd ? 8 : 0;
  }
};

// The 8-bit matrix instruction.
template <int FA, int FB, int BP, int BQ, int FP, int FQ>
struct MacBlocks : Scales<BP, BQ, FP, FQ> {
  typedef Frag P;
  typedef Frag Q;
  typedef v4f Acc;
  using Next = typename Scales<BP, BQ, FP, FQ>::Next;
  template <int PH>
  __device__ __forceinline__ P p(const Frag& f, int) const { return f; }
  template <int PH>
  __device__ __forceinline__ Q q(const Frag& f, int, const Next&) const { return f; }
  template <int PH>
  __device__ __forceinline__ void mac(v4f& c, const P& p, int i, const Q& q, int j) const {
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, c, FB, FA, PH, this->s.p[i], PH,
                                                         this->s.q[j]);
  }
};

// The values widened to bf16.
struct Wide {
  bf16x8 v[4];
};
template <int FA, int FB, int BP, int BQ, int FP, int FQ>
struct MacWide : Scales<BP, BQ, FP, FQ> {
  typedef Wide P;
  typedef Wide Q;
  typedef v4f Acc;
  using Next = typename Scales<BP, BQ, FP, FQ>::Next;
  template <int FMT>
  static __device__ __forceinline__ Wide wide(const Frag& f, uint32_t byte) {
    const float scale = __uint_as_float((byte & 255u) << 23);
    Wide w;
#pragma unroll
    for (int h = 0; h < 4; ++h) w.v[h] = widen<FMT>(f[2 * h], f[2 * h + 1], scale);
    return w;
  }
  template <int PH>
  __device__ __forceinline__ P p(const Frag& f, int i) const {
    return wide<FB>(f, this->s.p[i] >> 8 * PH);
  }
  template <int PH>
  __device__ __forceinline__ Q q(const Frag& f, int j, const Next& up) const {
    return wide<FA>(f, PH == 0 ? up.q[j] : this->s.q[j] >> 8);
  }
  template <int PH>
  __device__ __forceinline__ void mac(v4f& c, const P& p, int, const Q& q, int) const {
#pragma unroll
    for (int h = 0; h < 4; ++h)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p.v[h], q.v[h], c, 0, 0, 0);
  }
};

// Eight neighbours of a row of C from LDS, n of them.
template <bool BF>
__device__ __forceinline__ void store8(void* C, long long at, const uint8_t* from, int n) {
  if constexpr (BF) {
    bf16_t* c = (bf16_t*)C + at;
    if (n >= 8) {
      *(u32x4_any*)c = *(const u32x4*)from;
    } else {
      for (int e = 0; e < n; ++e) c[e] = ((const bf16_t*)from)[e];
    }
  } else {
    float* c = (float*)C + at;
    if (n >= 8) {
      *(v4f_any*)c = *(const v4f*)from;
      *(v4f_any*)(c + 4) = *(const v4f*)(from + 16);
    } else {
      for (int e = 0; e < n; ++e) c[e] = ((const float*)from)[e];
    }
  }
}

// Tiles of C by way of LDS, in C's type, so that whole rows of a tile leave at once (the
// halves of its rows in two of the stages; a pitch of 16 bytes more than a row spreads the
// sixteen rows that a wavefront writes at once over the banks).
template <bool BF, int THREADS, class T>
__device__ __forceinline__ void tile_out(const T& t, const v4f (&acc)[T::FP][T::FQ], uint8_t* s0,
                                         uint8_t* s1, void* C, long long row0, long long ldc,
                                         int np, int nq) {
  constexpr int kSize = BF ? 2 : 4, kPitch = T::kP * kSize + 16, kHalf = T::kQ / 2;
  static_assert(kHalf * kPitch <= T::kStage, "half a tile fits a stage");
  auto at = [&](int q, int p) __attribute__((always_inline)) {
    return (q < kHalf ? s0 : s1) + q % kHalf * kPitch + p * kSize;
  };
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int j = 0; j < T::FQ; ++j)
#pragma unroll
    for (int i = 0; i < T::FP; ++i) {
      uint8_t* to = at(t.wq + j * 16 + (t.lane & 15), t.wp + i * 16 + (t.lane >> 4) * 4);
      const v4f v = acc[i][j];
      if constexpr (BF)
        *(u32x2*)to = u32x2{f32_to_bf16(v[0]) | (uint32_t)f32_to_bf16(v[1]) << 16,
                            f32_to_bf16(v[2]) | (uint32_t)f32_to_bf16(v[3]) << 16};
      else
        *(v4f*)to = v;
    }
  __syncthreads();
#pragma unroll 2
  for (int u = threadIdx.x; u < T::kP * T::kQ / 8; u += THREADS) {
    const int q = u / (T::kP / 8), p = u % (T::kP / 8) * 8;
    if (q < nq && p < np) store8<BF>(C, row0 + (long long)q * ldc + p, at(q, p), np - p);
  }
}

// The tile of BP rows of B and BQ rows of A, over one of `splits` ranges of the inner
// dimension (chunk steps each, a multiple of four); a split's sums go to `part`.
template <int FA, int FB, bool OUTBF, int BP, int BQ, int WP, int WQ, int S>
__global__ __launch_bounds__((64 * (BP / WP) * (BQ / WQ)), 2) void k_gemm_tile(BlockGemmArgs a,
                                                                               int tp, int tq,
                                                                               int total) {
  using T = TileLoop<BP, BQ, WP, WQ, S, (BP + BQ) * 4>;
  LSGD_TILE_STAGES(st, S, T::kStage);
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  int l = xcd_order(id, total);
  const int sg = l / (tp * tq), g = sg % a.G, split = sg / a.G;
  int pt, qt;
  band_order(l % (tp * tq), tp, tq, pt, qt);
  const int p0 = pt * BP, q0 = qt * BQ;
  const int nb = (a.Kd + 127) / 128, ld = nb * 128, lds = (nb + 3) / 4 * 4;
  const int k0 = split * a.chunk, steps = min(a.chunk, nb - k0);
  T t;
  t.init(a.B + (long long)g * a.sB + (long long)p0 * ld, a.A + (long long)g * a.sA + (long long)q0 * ld,
         ld, a.N - p0, a.M - q0);
  t.skip(k0);
  std::conditional_t<OUTBF, MacBlocks<FA, FB, BP, BQ, T::FP, T::FQ>,
                     MacWide<FA, FB, BP, BQ, T::FP, T::FQ>> mac;
  mac.init(a.SB + (long long)g * a.sSB + (long long)p0 * lds,
           a.SA + (long long)g * a.sSA + (long long)q0 * lds, lds, a.N - p0, a.M - q0, t.wp,
           t.wq, k0);
  v4f acc[T::FP][T::FQ] = {};
  t.run(st, steps, mac, acc);
  if constexpr (BP == 64) {  // the only tiles that are split
    if (a.splits > 1) {
      tile_out<false, T::kThreads>(t, acc, st[0], st[1], a.part,
                                   ((long long)sg * a.M + q0) * a.N + p0, a.N, a.N - p0, a.M - q0);
      return;
    }
  }
  tile_out<OUTBF, T::kThreads>(t, acc, st[0], st[1], a.C,
                               (long long)g * a.sC + (long long)q0 * a.ldc + p0, a.ldc, a.N - p0,
                               a.M - q0);
}

// C = the splits' sums in ascending order, four neighbours a thread.
template <bool OUTBF>
__global__ __launch_bounds__(kThreads) void k_gemm_join(BlockGemmArgs a, int quads,
                                                        long long total) {
  const long long i = (long long)workgroup_id() * kThreads + threadIdx.x;
  if (i >= total) return;
  const long long row = i / quads;  // of G M
  const int n = (int)(i % quads) * 4, left = a.N - n;
  const long long each = (long long)a.G * a.M * a.N;
  const float* p = a.part + row * a.N + n;
  v4f v = {};
  for (int s = 0; s < a.splits; ++s, p += each) {
    if (left >= 4) {
      v += *(const v4f_any*)p;
    } else {
      for (int e = 0; e < left; ++e) v[e] += p[e];
    }
  }
  const long long at = row / a.M * a.sC + row % a.M * a.ldc + n;
  for (int e = 0; e < 4 && e < left; ++e) {
    if constexpr (OUTBF)
      ((bf16_t*)a.C)[at + e] = f32_to_bf16(v[e]);
    else
      ((float*)a.C)[at + e] = v[e];
  }
}

// ------------------------------------------------------------------ launches
constexpr int kCus = 256;
long long tiles_of(int G, int M, int N, long long b) {
  return (N + b - 1) / b * ((M + b - 1) / b) * G;
}

// Ranges the inner dimension is cut into: as many as leave the least estimated time where
// 64 x 64 tiles leave compute units idle. A workgroup alone on its unit takes 0.18 us a
// step (0.39 to fp32), all of them together cannot beat 5 TB/s, and a second launch
// joins the sums (4 us, and their bytes). Measured in us, cut in 1 / 2 / 4 / 8: 512 x 512 x
// 8192 to bf16 17 / 12 / 11 / 15, 512 x 512 x 65536 126 / 71 / 46 / 44, 128 x 4096 x 4096 to bf16
// 8.8 / 10.5 / 15 / 20, 1 x 8192 x 8192 to fp32 28 / 20 / 19 / 23.
int splits_of(bool bf16, int G, int M, int N, int Kd) {
  const long long tiles = tiles_of(G, M, N, 64), nb = (Kd + 127) / 128;
  const double step = bf16 ? 0.18 : 0.39;
  const double bytes = (double)G * ((double)M + N) * nb * 128 / 5e6;
  const double sums = 2.0 * G * M * N * sizeof(float) / 4e6;  // written and read, a range
  int best = 1;
  double least = std::max(step * nb, bytes);
  for (int s = 2; s <= 64 && tiles * s <= 2 * kCus && nb >= 4 * s; s *= 2) {
    const double t = std::max(step * nb / s, bytes) + 4 + sums * s;
    if (t < least) {
      best = s;
      least = t;
    }
  }
  // whole groups of four steps: fewer ranges may do
  const long long chunk = (nb + 4 * best - 1) / (4 * best) * 4;
  return (int)((nb + chunk - 1) / chunk);
}

// Tile sizes and stages, by estimated time: see ortho.hip's for what the numbers mean;
// these are from 4096^3 and 8192^3 (us, repeated on one input, to bf16 112 / 82 / 73 / 62 and
// 886 / 597 / 492 / 404; to fp32 170 / 147 / 125 and 1294 / 1031 / 889; under the kernel trace,
// whose pauses let the clock change, 117 / 79 / 68 / 57 and 1027 / 688 / 614 / 490, 194 / 155 /
// 130 and 1351 / 1125 / 979).
struct BlockCut {
  int tile, stages;
};
BlockCut block_cut(bool bf16, int G, int M, int N, int splits) {
  if (splits > 1) return BlockCut{64, 4};
  const BlockCut cuts[4] = {{64, 4}, {128, 4}, {128, 2}, {256, 2}};
  const int per_cu[4] = {2, 1, 2, 1};
  const double each[2][4] = {{1.6, 5.3, 4.5, 0.0}, {1.6, 4.5, 3.8, 12.6}};
  int at = 0;
  double least = 0;
  for (int i = 0; i < (bf16 ? 4 : 3); ++i) {
    const double rounds =
        std::ceil((double)tiles_of(G, M, N, cuts[i].tile) / (kCus * per_cu[i]));
    const double t = rounds * per_cu[i] * each[bf16][i];
    if (i == 0 || t < least) {
      at = i;
      least = t;
    }
  }
  return cuts[at];
}

template <int FA, int FB, bool OUTBF, int B, int W, int S>
hipError_t launch_tile(const BlockGemmArgs& a, hipStream_t s) {
  constexpr int WP = B == 256 ? 128 : B / 2;
  const long long tp = (a.N + B - 1LL) / B, tq = (a.M + B - 1LL) / B;
  if (tp * tq > 0x7fffffffLL / a.G / a.splits) return hipErrorInvalidValue;
  const long long total = tp * tq * a.G * a.splits;
  hipLaunchKernelGGL((k_gemm_tile<FA, FB, OUTBF, B, B, WP, W, S>), grid_of(total),
                     dim3(64 * (B / WP) * (B / W)), 0, s, a, (int)tp, (int)tq, (int)total);
  return hipGetLastError();
}
template <int FA, int FB, bool OUTBF>
hipError_t gemm_blocks(BlockGemmArgs a, hipStream_t s) {
  a.splits = splits_of(OUTBF, a.G, a.M, a.N, a.Kd);
  const int nb = (a.Kd + 127) / 128;
  a.chunk = (nb + 4 * a.splits - 1) / (4 * a.splits) * 4;
  const BlockCut c = block_cut(OUTBF, a.G, a.M, a.N, a.splits);
  hipError_t e;
  if (c.tile == 64)
    e = launch_tile<FA, FB, OUTBF, 64, 32, 4>(a, s);
  else if (c.tile == 128 && c.stages == 4)
    e = launch_tile<FA, FB, OUTBF, 128, 32, 4>(a, s);
  else if (c.tile == 128)
    e = launch_tile<FA, FB, OUTBF, 128, 64, 2>(a, s);
  else  // (to bf16 only)
    e = launch_tile<FA, FB, true, 256, 64, 2>(a, s);
  if (e != hipSuccess || a.splits == 1) return e;
  const int quads = (a.N + 3) / 4;
  const long long total = (long long)a.G * a.M * quads;
  hipLaunchKernelGGL((k_gemm_join<OUTBF>), grid_of((total + kThreads - 1) / kThreads),
                     dim3(kThreads), 0, s, a, quads, total);
  return hipGetLastError();
}
template <int FA, int FB>
hipError_t gemm_blocks(const BlockGemmArgs& a, hipStream_t s) {
  return a.out_bf16 ? gemm_blocks<FA, FB, true>(a, s) : gemm_blocks<FA, FB, false>(a, s);
}

}  // namespace

hipError_t launch_quantise(int bf16, int fmt, const QuantArgs& a, hipStream_t s) {
  if (fmt == kFmtE4M3)
    return bf16 ? quantise<true, kFmtE4M3>(a, s) : quantise<false, kFmtE4M3>(a, s);
  return bf16 ? quantise<true, kFmtE5M2>(a, s) : quantise<false, kFmtE5M2>(a, s);
}

size_t gemm_blocks_workspace_bytes(int bf16, int G, int M, int N, int Kd) {
  const int s = splits_of(bf16, G, M, N, Kd);
  return s == 1 ? 0 : (size_t)s * G * M * N * sizeof(float);
}

void gemm_blocks_cut(int bf16, int G, int M, int N, int Kd, int cut[3]) {
  cut[2] = splits_of(bf16, G, M, N, Kd);
  const BlockCut c = block_cut(bf16, G, M, N, cut[2]);
  cut[0] = c.tile;
  cut[1] = c.stages;
}

hipError_t launch_gemm_blocks(int fmt_a, int fmt_b, const BlockGemmArgs& a, hipStream_t s) {
  if (fmt_a == kFmtE4M3)
    return fmt_b == kFmtE4M3 ? gemm_blocks<kFmtE4M3, kFmtE4M3>(a, s)
                             : gemm_blocks<kFmtE4M3, kFmtE5M2>(a, s);
  return fmt_b == kFmtE4M3 ? gemm_blocks<kFmtE5M2, kFmtE4M3>(a, s)
                           : gemm_blocks<kFmtE5M2, kFmtE5M2>(a, s);
}

}  // namespace lsgd
