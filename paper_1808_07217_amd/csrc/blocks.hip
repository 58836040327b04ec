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
  // (arguments as TileLoop::init's; wp, wq: the wavefront's place in the tile)
  __device__ __forceinline__ void init(const uint8_t* p, const uint8_t* q, int pitch, int np,
                                       int nq, int wp, int wq) {
    const int lane = threadIdx.x & 63;
    // (a tile of fewer rows than threads loads them more than once)
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kLoads;
    P = p;
    Q = q;
    leftp = min(np, BP) * pitch;
    leftq = min(nq, BQ) * pitch;
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

// Four neighbours of a row of C.
template <bool OUTBF>
__device__ __forceinline__ void store4(void* C, long long at, const v4f& v, int n) {
  if constexpr (OUTBF) {
    bf16_t* c = (bf16_t*)C + at;
    uint32_t h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = f32_to_bf16(v[e]);
    if (n >= 4) {
      *(u32x2_any*)c = u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n) c[e] = (bf16_t)h[e];
    }
  } else {
    float* c = (float*)C + at;
    if (n >= 4) {
      *(v4f_any*)c = v;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n) c[e] = v[e];
    }
  }
}

template <int FA, int FB, bool OUTBF, int BP, int BQ, int WP, int WQ, int S>
__global__ __launch_bounds__(64 * (BP / WP) * (BQ / WQ), 2) void k_gemm_tile(BlockGemmArgs a,
                                                                             int tp, int tq,
                                                                             int total) {
  using T = TileLoop<BP, BQ, WP, WQ, S, (BP + BQ) * 4>;
  LSGD_TILE_STAGES(st, S, T::kStage);
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int l = xcd_order(id, total), g = l / (tp * tq);
  int pt, qt;
  band_order(l % (tp * tq), tp, tq, pt, qt);
  const int p0 = pt * BP, q0 = qt * BQ;
  const int nb = (a.Kd + 127) / 128, ld = nb * 128, lds = (nb + 3) / 4 * 4;
  T t;
  t.init(a.B + (long long)g * a.sB + (long long)p0 * ld,
         a.A + (long long)g * a.sA + (long long)q0 * ld, ld, a.N - p0, a.M - q0);
  std::conditional_t<OUTBF, MacBlocks<FA, FB, BP, BQ, T::FP, T::FQ>,
                     MacWide<FA, FB, BP, BQ, T::FP, T::FQ>> mac;
  mac.init(a.SB + (long long)g * a.sSB + (long long)p0 * lds,
           a.SA + (long long)g * a.sSA + (long long)q0 * lds, lds, a.N - p0, a.M - q0, t.wp,
           t.wq);
  v4f acc[T::FP][T::FQ] = {};
  t.run(st, nb, mac, acc);
  const int lr = t.lane & 15, lq = t.lane >> 4;
#pragma unroll
  for (int j = 0; j < T::FQ; ++j) {
    const int m = q0 + t.wq + j * 16 + lr;
    if (m >= a.M) continue;
#pragma unroll
    for (int i = 0; i < T::FP; ++i) {
      const int n = p0 + t.wp + i * 16 + lq * 4;
      store4<OUTBF>(a.C, (long long)g * a.sC + (long long)m * a.ldc + n, acc[i][j], a.N - n);
    }
  }
}

template <int FA, int FB, bool OUTBF, int BP, int BQ, int WP, int WQ, int S = 2>
hipError_t launch_tile(const BlockGemmArgs& a, hipStream_t s) {
  const long long tp = (a.N + BP - 1LL) / BP, tq = (a.M + BQ - 1LL) / BQ;
  if (tp * tq > 0x7fffffffLL / a.G) return hipErrorInvalidValue;
  const long long total = tp * tq * a.G;
  hipLaunchKernelGGL((k_gemm_tile<FA, FB, OUTBF, BP, BQ, WP, WQ, S>), grid_of(total),
                     dim3(64 * (BP / WP) * (BQ / WQ)), 0, s, a, (int)tp, (int)tq, (int)total);
  return hipGetLastError();
}

template <int FA, int FB>
hipError_t gemm_blocks(const BlockGemmArgs& a, hipStream_t s) {
  auto tiles = [&](int b) {
    return ((a.N + b - 1LL) / b) * ((a.M + b - 1LL) / b) * a.G;
  };
  if (a.out_bf16) {
    if (tiles(256) >= 256) return launch_tile<FA, FB, true, 256, 256, 128, 64>(a, s);
    if (tiles(128) >= 256) return launch_tile<FA, FB, true, 128, 128, 64, 64>(a, s);
    return launch_tile<FA, FB, true, 64, 64, 32, 32, 4>(a, s);
  }
  if (tiles(128) >= 256) return launch_tile<FA, FB, false, 128, 128, 64, 64>(a, s);
  return launch_tile<FA, FB, false, 64, 64, 32, 32, 4>(a, s);
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
