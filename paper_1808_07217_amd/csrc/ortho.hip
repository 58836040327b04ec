// Orthogonalised momentum: X = U S V^T taken towards U V^T by Newton-Schulz steps
//   A = X X^T,  B = b A + c A A,  X := a X + B X,
// from X / (|X|_F + eps), so that every singular value s of X runs through
// s (a + b s^2 + c s^4).
//
// The products run on v_mfma_f32_16x16x32_f16. Singular values stay below a bound
// known from the coefficients, so every entry has one too, and a power of two puts
// each matrix where fp16 is exact enough: a value is held as two fp16 pieces,
// x = x1 + x2 (22 to 24 significant bits), and fp32 products are x1 y1 + x1 y2 + x2 y1,
// each exact in fp32; what is left out is 2^-24 |x y| at worst. In the bf16 form
// the products of matrices of kOnePieceFrom rows and more take the first piece alone
// (2^-11 at worst, an eighth of bf16's own rounding; see kOnePieceFrom). X keeps both
// pieces there too, because a X passes on the small singular directions, which the steps
// amplify by a each time: rounding X itself to 11 bits loses them (error 1.8e-2 instead of
// 1.7e-3 for matrices of low rank in noise).
//
// A and B are symmetric: only their tiles on and below the diagonal are computed,
// and each is stored on both sides. All three products are tiles of tile_loop.h.
// A matrix whose norm is small against eps starts that much below 1 and grows by at
// most a known factor a step; X of step t is held 2^k(t) higher, k(t) = max(0,
// k(0) - t * grow), so that it too has all of its bits: k(0) takes the norm r, 0 < r < 1,
// to 1 <= 2^k(0) r < 2, which the scale of X leaves room for (r = 1 - 1e-7, nearly every
// matrix's, to almost 2).
// The steps work on m = min(M, N) rows. X lies in memory both ways, [m][n] for X X^T
// and [n][m] for B X, rows padded with zeros to a multiple of 64 so that no product
// has a tail; a zero row or column stays zero through the steps. In fp32 precision the two
// pieces of 32 neighbours share a line of 128 bytes, first pieces, then second ones; in
// the bf16 form each piece is a matrix of its own, and only the first is multiplied.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "tile_loop.h"

namespace lsgd {
namespace {

// vectors at any element's alignment
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

// ------------------------------------------------------------- the first step
// Up to four neighbours (n of them; the others 0) of a row.
__device__ __forceinline__ v4f load4(const float* p, int n) {
  v4f v = {};
  if (n >= 4) {
    v = *(const v4f_any*)p;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) v[e] = p[e];
  }
  return v;
}
__device__ __forceinline__ v4f load4(const bf16_t* p, int n) {
  v4f v = {};
  if (n >= 4) {
    const u32x2_any w = *(const u32x2_any*)p;
    v = v4f{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u),
            __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) v[e] = bf16_to_f32(p[e]);
  }
  return v;
}

// n neighbours, from (r, c) on, of the matrix to orthogonalise: X's, or of an update
// d = g + m u or u; fetch() loads them, take() makes d of them. STEP: takes the momentum
// step u = m u + g first and stores it.
struct Fetched {
  v4f x, u;
};
template <bool STEP>
__device__ __forceinline__ Fetched fetch(const OrthoArgs& a, int g, int r, int c, int n) {
  const long long x = (long long)g * a.sX + (long long)r * a.ldx + c;
  Fetched f{};
  if (!a.U) {
    f.x = a.x_bf16 ? load4((const bf16_t*)a.X + x, n) : load4((const float*)a.X + x, n);
  } else {
    f.u = load4(a.U + (long long)g * a.sU + (long long)r * a.ldu + c, n);
    if (STEP || a.nesterov) f.x = load4((const float*)a.X + x, n);
  }
  return f;
}
template <bool STEP>
__device__ __forceinline__ v4f take(const OrthoArgs& a, int g, int r, int c, int n,
                                    const Fetched& f) {
  if (!a.U) return f.x;
  v4f u = f.u;
  if constexpr (STEP) {
    float* pu = a.U + (long long)g * a.sU + (long long)r * a.ldu + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __builtin_fmaf(a.mom, u[e], f.x[e]);
    if (n >= 4) {
      *(v4f_any*)pu = u;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n) pu[e] = u[e];
    }
  }
  if (a.nesterov) {
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __builtin_fmaf(a.mom, u[e], f.x[e]);
  }
  return u;
}

// The sum of red[0 .. 255] in a fixed tree, by all 256 threads.
__device__ __forceinline__ double tree_sum(double* red) {
  __syncthreads();
#pragma unroll
  for (int w = kThreads / 2; w; w /= 2) {
    if (threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  return red[0];
}

// Partial sums of squares in 64 bits, [G][chunks] (no overflow for any fp32 input),
// and an update's momentum step. A row is taken in fours, its last one short.
__global__ __launch_bounds__(kThreads) void k_ortho_norm(OrthoArgs a, int chunks) {
  const unsigned id = workgroup_id();
  if (id >= (unsigned)chunks * a.G) return;
  const int g = id / chunks, ch = id % chunks, quads = (a.N + 3) / 4;
  // four fours at a time: their loads wait for none of the stores
  const int by = chunks * kThreads, dr = by / quads, dc = by % quads;
  const int first = ch * kThreads + threadIdx.x;
  int r = first / quads, c = first % quads;
  double s = 0;
  while (r < a.M) {
    constexpr int kAtOnce = 4;
    Fetched f[kAtOnce];
    int fr[kAtOnce], fc[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      fr[i] = r;
      fc[i] = c * 4;
      if (r < a.M) f[i] = fetch<true>(a, g, r, c * 4, a.N - c * 4);
      r += dr;
      c += dc;
      if (c >= quads) {
        c -= quads;
        ++r;
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (fr[i] < a.M) {
        const v4f d = take<true>(a, g, fr[i], fc[i], a.N - fc[i], f[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s += (double)d[e] * (double)d[e];
      }
    }
  }
  __shared__ double red[kThreads];
  red[threadIdx.x] = s;
  s = tree_sum(red);
  if (threadIdx.x == 0) a.part[(long long)g * chunks + ch] = s;
}

__device__ __forceinline__ void split2(float x, _Float16& h, _Float16& l) {
  h = (_Float16)x;
  l = (_Float16)(x - (float)h);
}
// Where the first piece of element (r, k) lies in a matrix of rows of K, and how far
// behind it the second does (P: see the top; plane: elements of a matrix).
template <int P>
__device__ __forceinline__ long long at(int r, int k, int K) {
  return P == 2 ? (long long)r * 2 * K + (k >> 5) * 64 + (k & 31) : (long long)r * K + k;
}
template <int P>
__device__ __forceinline__ long long second(long long plane) {
  return P == 2 ? 32 : plane;
}

// k(t) of matrix g: see the top.
__device__ __forceinline__ int raise(const OrthoArgs& a, int g, int t) {
  return max(0, a.kexp[g] - t * a.grow);
}

// X / (|X|_F + eps) times the scale, in pieces, both ways; zeros in the padding.
template <int P>
__global__ __launch_bounds__(kThreads) void k_ortho_split(OrthoArgs a, int chunks, int tm, int tn) {
  const unsigned id = workgroup_id();
  if (id >= (unsigned)tm * tn * a.G) return;
  const int g = id / (tm * tn), p0 = id % (tm * tn) / tn * 64, q0 = id % tn * 64;
  __shared__ float tile[64][65];
  __shared__ double red[kThreads];
  // the loads run along the matrix's own rows
  const int r0 = a.flip ? q0 : p0, c0 = a.flip ? p0 : q0;
  Fetched f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int u = i * kThreads + threadIdx.x, y = u >> 4, x = (u & 15) * 4;
    if (r0 + y < a.M) f[i] = fetch<false>(a, g, r0 + y, c0 + x, a.N - c0 - x);
  }
  double s = 0;
  for (int i = threadIdx.x; i < chunks; i += kThreads) s += a.part[(long long)g * chunks + i];
  red[threadIdx.x] = s;
  s = tree_sum(red);
  const double norm = sqrt(s), r = norm / (norm + (double)a.eps);
  const int k = r > 0 ? min(100, -ilogb(r)) : 0;  // 0 for an infinite or NaN norm
  if (id % (tm * tn) == 0 && threadIdx.x == 0) a.kexp[g] = max(k, 0);
  const double inv = ldexp((double)a.scale_x, max(k, 0)) / (norm + (double)a.eps);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int u = i * kThreads + threadIdx.x, y = u >> 4, x = (u & 15) * 4;
    v4f v = {};
    if (r0 + y < a.M) v = take<false>(a, g, r0 + y, c0 + x, a.N - c0 - x, f[i]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float w = (float)((double)v[e] * inv);
      if (a.flip)
        tile[x + e][y] = w;
      else
        tile[y][x + e] = w;
    }
  }
  __syncthreads();
  const long long plane = (long long)a.mp * a.np;
  _Float16* X = a.Xr + (long long)g * P * plane;
  _Float16* T = a.Xt[0] + (long long)g * 2 * plane;
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    const int u = i * kThreads + threadIdx.x, y = u >> 3, x = (u & 7) * 8;
    f16x8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 s0, s1;
      split2(tile[y][x + e], s0, s1);
      h[e] = s0;
      l[e] = s1;
    }
    const long long o = at<P>(p0 + y, q0 + x, a.np);
    *(f16x8*)(X + o) = h;
    if constexpr (P == 2) *(f16x8*)(X + o + 32) = l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 s0, s1;
      split2(tile[x + e][y], s0, s1);
      h[e] = s0;
      l[e] = s1;
    }
    const long long t = at<P>(q0 + y, p0 + x, a.mp);
    *(f16x8*)(T + t) = h;
    *(f16x8*)(T + t + second<P>(plane)) = l;
  }
}

// ------------------------------------------------------------------ products
// A fragment is 32 k of both pieces (P == 2) or 64 of the first. TWO: x1 y1 has sums of
// its own, so that they round once in 32 k, not three times; it keeps long products (X X^T
// of few long rows: 40 x 3000 off by 2.0e-6 without) as exact as sums in fp32 are.
struct TwoSums {
  v4f a, b;
};
template <int P_, bool TWO>
struct MacHalf {
  typedef Frag P;
  typedef Frag Q;
  typedef std::conditional_t<TWO, TwoSums, v4f> Acc;
  static __device__ __forceinline__ v4f sum(const v4f& c) { return c; }
  static __device__ __forceinline__ v4f sum(const TwoSums& c) { return c.a + c.b; }
  struct Next {};
  static constexpr int kEvenLoads = 0;
  __device__ __forceinline__ void load(uint8_t*, int, bool) const {}
  __device__ __forceinline__ void begin(const uint8_t*, int, Next&) const {}
  __device__ __forceinline__ void take(const Next&) const {}
  __device__ __forceinline__ void last(bool) const {}
  template <int PH>
  __device__ __forceinline__ P p(const Frag& f, int) const { return f; }
  template <int PH>
  __device__ __forceinline__ Q q(const Frag& f, int, const Next&) const { return f; }
  template <int PH>
  __device__ __forceinline__ void mac(Acc& c, const P& p, int, const Q& q, int) const {
    mac(c, half<0>(p), half<4>(p), half<0>(q), half<4>(q));
  }
  static __device__ __forceinline__ void mac(Acc& c, const f16x8& p0, const f16x8& p1,
                                             const f16x8& q0, const f16x8& q1) {
    if constexpr (TWO) {
      static_assert(P_ == 2, "of two pieces");
      c.b = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, q0, c.b, 0, 0, 0);
      c.b = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q1, c.b, 0, 0, 0);
      c.a = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q0, c.a, 0, 0, 0);
    } else if constexpr (P_ == 2) {
      c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, q0, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q1, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q0, c, 0, 0, 0);
    } else {
      c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q0, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, q1, c, 0, 0, 0);
    }
  }
  template <int O>
  static __device__ __forceinline__ f16x8 half(const Frag& f) {
    return __builtin_bit_cast(f16x8, __builtin_shufflevector(f, f, O, O + 1, O + 2, O + 3));
  }
};

// Tile t of the lower triangle: row p holds p + 1 of them.
__device__ __forceinline__ void triangle(int t, int& p, int& q) {
  p = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
  while (p * (p + 1) / 2 > t) --p;
  while ((p + 1) * (p + 2) / 2 <= t) ++p;
  q = t - p * (p + 1) / 2;
}

__device__ __forceinline__ f16x4 first_of(const float (&v)[4]) {
  return f16x4{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
}
__device__ __forceinline__ f16x4 second_of(const float (&v)[4], const f16x4& h) {
  return f16x4{(_Float16)(v[0] - (float)h[0]), (_Float16)(v[1] - (float)h[1]),
               (_Float16)(v[2] - (float)h[2]), (_Float16)(v[3] - (float)h[3])};
}

// The n (at most 4; none for n <= 0) neighbours from element (r, c) of the result on; x: the
// weights an update finds there.
__device__ __forceinline__ void result(const OrthoArgs& a, int g, int r, int c, int n,
                                       const float (&v)[4], const v4f& x) {
  if (a.W) {
    float* w = a.W + (long long)g * a.sW + (long long)r * a.ldw + c;
    v4f y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __builtin_fmaf(a.keep, x[e], a.step * v[e]);
    if (n >= 4) {
      *(v4f_any*)w = y;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n) w[e] = y[e];
    }
  } else if (a.x_bf16) {
    bf16_t* y = (bf16_t*)a.Y + (long long)g * a.sY + (long long)r * a.ldy + c;
    if (n >= 4) {
      *(u32x2_any*)y = u32x2_any{f32_to_bf16(v[0]) | (uint32_t)f32_to_bf16(v[1]) << 16,
                                 f32_to_bf16(v[2]) | (uint32_t)f32_to_bf16(v[3]) << 16};
    } else {
      for (int e = 0; e < n; ++e) y[e] = f32_to_bf16(v[e]);
    }
  } else {
    float* y = (float*)a.Y + (long long)g * a.sY + (long long)r * a.ldy + c;
    if (n >= 4) {
      *(v4f_any*)y = v4f_any{v[0], v[1], v[2], v[3]};
    } else {
      for (int e = 0; e < n; ++e) y[e] = v[e];
    }
  }
}

// The square tiles: 256 x 256 and 192 x 192 with eight wavefronts, two by four; 128 x 128
// with four of a quarter each, or, with four stages and so alone on a compute unit, eight of
// 64 x 32; 64 x 64 with four.
template <int T, int S>
struct Shape {
  static constexpr bool kEight = T >= 192 || (T == 128 && S == 4);
  static constexpr int kWq = T / (kEight ? 4 : 2), kThreads = kEight ? 512 : 256;
};

// A tile's results leave both ways, [q][p] and [p][q], by way of LDS: first as columns,
// when each thread adds what belongs to its eight neighbours, then as rows, in vectors of
// 16 bytes. Everything after the sums' way to LDS is a rolled loop: instructions that a
// workgroup runs once are fetched from far away, and the same work written out over the
// accumulators took 10.5 to 14.5 us for a 256 x 256 product of 128 x 128 tiles where this
// takes 8.8 to 10.7.
// The halves of the tile's rows go through two of the stages, kRows of them at a time. The
// pitch of T + 4 words keeps the rows that a wavefront touches at once in different
// banks, but for pairs of columns' pieces.
template <int T, int THREADS>
struct Turn {
  static constexpr int kPasses = T == 256 ? 2 : 1, kRows = T / 2 / kPasses;
  static constexpr int kPitch = T + 4, kBytes = kRows * kPitch * 4;
  static constexpr int kExtra = kBytes > 2 * T * 128 ? kBytes - 2 * T * 128 : 0;
  static constexpr int kUnits = 2 * kRows * T / 8 / THREADS;  // eights a thread and pass
  float* half[2];
  __device__ __forceinline__ Turn(uint8_t* s0, uint8_t* s1) : half{(float*)s0, (float*)s1} {}
  // (a wavefront's rows all lie in one half)
  __device__ __forceinline__ float* at(int p, int q) const {
    return half[p >= T / 2] + p % kRows * kPitch + q;
  }
  // row r of the 2 kRows that a pass holds
  static __device__ __forceinline__ int row(int pass, int r) {
    return r / kRows * (T / 2) + pass * kRows + r % kRows;
  }
  // A pass's sums, times f, when every wavefront is done with what LDS held and
  // nothing is on its way there.
  template <class M, class L>
  __device__ __forceinline__ void fill(int pass, const L& t,
                                       const typename M::Acc (&acc)[L::FP][L::FQ], float f) const {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    constexpr int n = L::FP / kPasses;
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int j = 0; j < L::FQ; ++j) {
        const v4f v = M::sum(acc[pass * n + i][j]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *at(t.wp + (pass * n + i) * 16 + (t.lane >> 4) * 4 + e,
              t.wq + j * 16 + (t.lane & 15)) = v[e] * f;
      }
    __syncthreads();
  }
  // Unit u of a thread: as columns, four lanes share 32 p of a column (a line of pieces).
  static __device__ __forceinline__ void column(int pass, int u, int& p, int& q) {
    const int x = u * THREADS + (int)threadIdx.x;
    q = (x >> 2) % T;
    p = row(pass, ((x >> 2) / T * 4 + (x & 3)) * 8);
  }
  static __device__ __forceinline__ void across(int pass, int u, int& p, int& q) {
    const int x = u * THREADS + (int)threadIdx.x;
    p = row(pass, x / (T / 8));
    q = x % (T / 8) * 8;
  }
};

// Eight values in pieces.
__device__ __forceinline__ void to_pieces(const float (&v)[8], f16x8& h, f16x8& l) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    _Float16 a, b;
    split2(v[e], a, b);
    h[e] = a;
    l[e] = b;
  }
}

// The symmetric products: A = X X^T (SECOND = false) and B = b A + c A A, tiles on and
// below the diagonal.
template <int P, bool SECOND, int BT, int S>
__global__ __launch_bounds__((Shape<BT, S>::kThreads), 2) void k_ortho_gram(OrthoArgs a, int step,
                                                                       int tm, int total) {
  using Out = Turn<BT, Shape<BT, S>::kThreads>;
  using T = TileLoop<BT, BT, BT / 2, Shape<BT, S>::kWq, S, Out::kExtra>;
  LSGD_TILE_STAGES(st, S, T::kStage);
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int tri = tm * (tm + 1) / 2, l = xcd_order(id, total), g = l / tri;
  int pt, qt;
  triangle(l % tri, pt, qt);
  const int p0 = pt * BT, q0 = qt * BT, K = SECOND ? a.mp : a.np;
  const long long pm = (long long)a.mp * a.mp;
  const _Float16* src = SECOND ? a.A + g * P * pm : a.Xr + (long long)g * P * a.mp * a.np;
  _Float16* dst = (SECOND ? a.B : a.A) + g * P * pm;
  const float f = SECOND ? a.f_aa : ldexpf(a.f_xx, -2 * raise(a, g, step));
  T t;
  const int ld = K * P * 2;
  t.init((const uint8_t*)src + (long long)p0 * ld, (const uint8_t*)src + (long long)q0 * ld, ld,
         a.mp - p0, a.mp - q0);
  // (256 x 256 tiles have no room for two: see x_cut)
  using Mac = MacHalf<P, P == 2 && !SECOND && BT <= 192>;
  Mac mac;
  typename Mac::Acc acc[T::FP][T::FQ] = {};
  t.run(st, ld / 128, mac, acc);
  const Out out(st[0], st[1]);
#pragma unroll 1
  for (int pass = 0; pass < Out::kPasses; ++pass) {
    if (pass == 0)
      out.template fill<Mac>(0, t, acc, f);
    else
      out.template fill<Mac>(Out::kPasses - 1, t, acc, f);
#pragma unroll
    for (int u = 0; u < Out::kUnits; ++u) {
      int p, q;
      Out::column(pass, u, p, q);
      if (q0 + q >= a.mp || p0 + p >= a.mp) continue;
      const long long o = at<P>(q0 + q, p0 + p, a.mp);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = *out.at(p + e, q);
      if constexpr (SECOND) {  // A's own values: its mirror image's, which lie side by side
        const f16x8 xh = *(const f16x8*)(src + o);
        f16x8 xl = {};
        if constexpr (P == 2) xl = *(const f16x8*)(src + o + 32);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = __builtin_fmaf(a.f_a, (float)xh[e] + (float)xl[e], v[e]);
          *out.at(p + e, q) = v[e];
        }
      }
      f16x8 h, w;
      to_pieces(v, h, w);
      *(f16x8*)(dst + o) = h;
      if constexpr (P == 2) *(f16x8*)(dst + o + 32) = w;
    }
    // (a tile on the diagonal is its own mirror image)
    if (pt != qt) {
      if constexpr (SECOND) __syncthreads();
#pragma unroll 1
      for (int u = 0; u < Out::kUnits; ++u) {
        int p, q;
        Out::across(pass, u, p, q);
        if (q0 + q >= a.mp || p0 + p >= a.mp) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = out.at(p, q)[e];
        f16x8 h, w;
        to_pieces(v, h, w);
        _Float16* o = dst + at<P>(p0 + p, q0 + q, a.mp);
        *(f16x8*)o = h;
        if constexpr (P == 2) *(f16x8*)(o + 32) = w;
      }
    }
  }
}

// X := a X + B X; on the last step what the caller asked for.
template <int P, bool LAST, int BT, int S>
__global__ __launch_bounds__((Shape<BT, S>::kThreads), 2) void k_ortho_apply(OrthoArgs a, int step,
                                                                        int tp, int tq,
                                                                        int total) {
  using Out = Turn<BT, Shape<BT, S>::kThreads>;
  using T = TileLoop<BT, BT, BT / 2, Shape<BT, S>::kWq, S, Out::kExtra>;
  LSGD_TILE_STAGES(st, S, T::kStage);
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int l = xcd_order(id, total), g = l / (tp * tq);
  int pt, qt;
  band_order(l % (tp * tq), tp, tq, pt, qt);
  const int p0 = pt * BT, q0 = qt * BT, from = step & 1;
  const long long px = (long long)a.mp * a.np, pm = (long long)a.mp * a.mp;
  const _Float16* X = a.Xt[from] + g * 2 * px;
  T t;
  const int ld = a.mp * P * 2;
  t.init((const uint8_t*)(a.B + g * P * pm) + (long long)p0 * ld,
         (const uint8_t*)X + (long long)q0 * ld, ld, a.mp - p0, a.np - q0);
  const int k = raise(a, g, step);
  const int shift = LAST ? -k : raise(a, g, step + 1) - k;
  const float fb = ldexpf(LAST ? a.f_out : a.f_bx, shift);
  const float fx = ldexpf(LAST ? a.f_x / a.scale_x : a.f_x, shift);
  using Mac = MacHalf<P, false>;
  Mac mac;
  typename Mac::Acc acc[T::FP][T::FQ] = {};
  t.run(st, ld / 128, mac, acc);
  const Out out(st[0], st[1]);
#pragma unroll 1
  for (int pass = 0; pass < Out::kPasses; ++pass) {
    if (pass == 0)
      out.template fill<Mac>(0, t, acc, fb);
    else
      out.template fill<Mac>(Out::kPasses - 1, t, acc, fb);
#pragma unroll 4
    for (int u = 0; u < Out::kUnits; ++u) {
      int p, q;
      Out::column(pass, u, p, q);
      if (q0 + q >= a.np || p0 + p >= a.mp) continue;
      const long long o = at<P>(q0 + q, p0 + p, a.mp);
      const f16x8 xh = *(const f16x8*)(X + o), xl = *(const f16x8*)(X + o + second<P>(px));
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = __builtin_fmaf(fx, (float)xh[e] + (float)xl[e], *out.at(p + e, q));
        *out.at(p + e, q) = v[e];
      }
      if constexpr (!LAST) {
        f16x8 h, w;
        to_pieces(v, h, w);
        _Float16* to = a.Xt[1 - from] + g * 2 * px + o;
        *(f16x8*)to = h;
        *(f16x8*)(to + second<P>(px)) = w;
      }
    }
    __syncthreads();
    // rows of [p][q], or in the end of the result
#pragma unroll 1
    for (int u = 0; u < Out::kUnits; ++u) {
      int p, q;
      float v[8];
      if (LAST && a.flip) {
        Out::column(pass, u, p, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = *out.at(p + e, q);
      } else {
        Out::across(pass, u, p, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = out.at(p, q)[e];
      }
      if constexpr (LAST) {
        const int r = a.flip ? q0 + q : p0 + p, c = a.flip ? p0 + p : q0 + q;
        const int left = r < a.M ? a.N - c : 0;
        const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
        v4f wl = {}, wh = {};
        if (a.W) {
          const float* w = a.W + (long long)g * a.sW + (long long)r * a.ldw + c;
          wl = load4(w, left);
          wh = load4(w + 4, left - 4);
        }
        result(a, g, r, c, left, lo, wl);
        result(a, g, r, c + 4, left - 4, hi, wh);
      } else {
        if (q0 + q >= a.np || p0 + p >= a.mp) continue;
        f16x8 h, w;
        to_pieces(v, h, w);
        _Float16* o = a.Xr + g * P * px + at<P>(p0 + p, q0 + q, a.np);
        *(f16x8*)o = h;
        if constexpr (P == 2) *(f16x8*)(o + 32) = w;
      }
    }
  }
}

// -------------------------------------------------------------- small matrices
// A whole matrix in one workgroup's LDS, all steps in one launch (as launches of their own
// the steps of 64 x 64 matrices took 72 us, nearly all of it between kernels). X lies
// there once, its two pieces as rows of np + 8 (fragment reads of eight rows fall into
// different banks); B X takes its columns with ds_read_b64_tr_b16, which gives each lane of
// 16 its column's four k from a 4 x 16 block. A and B share a place: B replaces A when
// all of A A is in registers, as X' replaces X. Both precisions take two pieces
// here: the products are not what such a matrix waits for. Rows and columns are padded
// with zeros to multiples of 32, a wavefront works on 32 x 32 blocks.
constexpr int kSmallThreads = 512, kSmallWaves = kSmallThreads / 64, kSmallMost = 128;
constexpr int kSmallBlocks = 5;  // of X a wavefront
constexpr int kSmallFours = 20;  // of X a thread (LDS holds fewer than 20 * 512 * 4 values)
constexpr size_t kSmallLds = 160 * 1024;
__host__ __device__ constexpr int pitch(int n) { return n + 8; }
constexpr size_t small_lds(int mp, int np) {
  return 4 * (size_t)mp * (pitch(np) + pitch(mp));
}

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
struct Place {  // of a row's four neighbours
  int r, c;
  __device__ __forceinline__ void next(int dr, int dc, int quads) {
    r += dr;
    c += dc;
    if (c >= quads) {
      c -= quads;
      ++r;
    }
  }
};
struct Plane2 {  // a matrix's two pieces in LDS
  _Float16* p[2];
  int ld;
};
// acc += F S^T over K: F's rows from r0 (COLS: its columns, K the slow index) and S's
// rows from c0 on.
template <bool COLS, class Mac>
__device__ __forceinline__ void block_product(const Plane2& F, int r0, const Plane2& S, int c0,
                                              int K, int lr, int lq,
                                              typename Mac::Acc (&acc)[2][2]) {
  struct Frags {
    f16x8 f[2][2], g[2][2];
  };
  auto read = [&](int k) __attribute__((always_inline)) {
    Frags x;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if constexpr (COLS) {
          typedef short s16x4 __attribute__((ext_vector_type(4)));
          typedef short s16x8 __attribute__((ext_vector_type(8)));
          using L = __attribute__((address_space(3))) s16x4;
          const _Float16* b =
              F.p[w] + (k + 8 * lq + (lr >> 2)) * F.ld + r0 + i * 16 + 4 * (lr & 3);
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)b);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(b + 4 * F.ld));
          x.f[i][w] = __builtin_bit_cast(
              f16x8, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        } else {
          x.f[i][w] = *(const f16x8*)(F.p[w] + (r0 + i * 16 + lr) * F.ld + k + 8 * lq);
        }
        x.g[i][w] = *(const f16x8*)(S.p[w] + (c0 + i * 16 + lr) * S.ld + k + 8 * lq);
      }
    return x;
  };
  auto mac = [&](const Frags& x) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        Mac::mac(acc[i][j], x.f[i][0], x.f[i][1], x.g[j][0], x.g[j][1]);
  };
  Frags x = read(0);  // the next fragments are on their way while these are multiplied
#pragma unroll 1
  for (int k = 32; k < K; k += 32) {
    const Frags next = read(k);
    mac(x);
    x = next;
  }
  mac(x);
}

__global__ __launch_bounds__(kSmallThreads) void k_ortho_small(OrthoArgs a, int mp, int np) {
  extern __shared__ __align__(16) uint8_t small[];
  const int g = workgroup_id();
  if (g >= a.G) return;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Plane2 X, A;
  X.ld = pitch(np);
  A.ld = pitch(mp);
  X.p[0] = (_Float16*)small;
  X.p[1] = X.p[0] + mp * X.ld;
  A.p[0] = X.p[1] + mp * X.ld;
  A.p[1] = A.p[0] + mp * A.ld;

  // the whole matrix into registers, all loads at once, an update's momentum step with it
  const int quads = (a.N + 3) / 4, total = a.M * quads;
  const int dr = kSmallThreads / quads, dc = kSmallThreads % quads;
  v4f d[kSmallFours];
  Place at{tid / quads, tid % quads};
#pragma unroll
  for (int i = 0; i < kSmallFours; i += 4)
    if (i * kSmallThreads < total) {
      Fetched f[4];
      Place was[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        was[h] = at;
        if (at.r < a.M) f[h] = fetch<true>(a, g, at.r, at.c * 4, a.N - at.c * 4);
        at.next(dr, dc, quads);
      }
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        d[i + h] = v4f{};
        if (was[h].r < a.M)
          d[i + h] = take<true>(a, g, was[h].r, was[h].c * 4, a.N - was[h].c * 4, f[h]);
      }
    }
  // the norm, in the place of A
  double* red = (double*)A.p[0];
  double s = 0;
#pragma unroll
  for (int i = 0; i < kSmallFours; ++i)
    if (i * kSmallThreads < total) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s += (double)d[i][e] * (double)d[i][e];
    }
  red[tid] = s;
  for (int w = kSmallThreads / 2; w; w /= 2) {
    __syncthreads();
    if (tid < w) red[tid] += red[tid + w];
  }
  __syncthreads();
  const double norm = sqrt(red[0]), ratio = norm / (norm + (double)a.eps);
  const int k0 = ratio > 0 ? max(0, min(100, -ilogb(ratio))) : 0;  // see k_ortho_split
  const double inv = ldexp((double)a.scale_x, k0) / (norm + (double)a.eps);
  const int rows = a.flip ? np : mp, cols = (a.flip ? mp : np) / 4;
  at = Place{tid / quads, tid % quads};
#pragma unroll
  for (int i = 0; i < kSmallFours; ++i) {
    if (i * kSmallThreads < total && at.r < a.M) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = at.r, c = at.c * 4 + e, o = a.flip ? c * X.ld + r : r * X.ld + c;
        split2((float)((double)d[i][e] * inv), X.p[0][o], X.p[1][o]);
      }
    }
    at.next(dr, dc, quads);
  }
  // zeros behind the last row and behind each row's last four
  for (int u = tid; u < rows * cols; u += kSmallThreads) {
    const int r = u / cols, c = u % cols * 4;
    if (r < a.M && c < a.N) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int o = a.flip ? (c + e) * X.ld + r : r * X.ld + c + e;
      X.p[0][o] = X.p[1][o] = (_Float16)0.f;
    }
  }
  __syncthreads();

  const int bm = mp / 32, blocks = bm * bm, xblocks = bm * (np / 32);
  auto put = [&](const Plane2& to, int r, int c, const float (&v)[4]) __attribute__((always_inline)) {
    const f16x4 h = first_of(v), l = second_of(v, h);
    *(f16x4*)(to.p[0] + r * to.ld + c) = h;
    *(f16x4*)(to.p[1] + r * to.ld + c) = l;
  };
  auto get = [&](const Plane2& from, int r, int c) __attribute__((always_inline)) {
    const f16x4 h = *(const f16x4*)(from.p[0] + r * from.ld + c);
    const f16x4 l = *(const f16x4*)(from.p[1] + r * from.ld + c);
    return v4f{(float)h[0] + (float)l[0], (float)h[1] + (float)l[1], (float)h[2] + (float)l[2],
               (float)h[3] + (float)l[3]};
  };
#pragma unroll 1
  for (int t = 0; t < a.steps; ++t) {
    const int k = max(0, k0 - t * a.grow), kn = max(0, k0 - (t + 1) * a.grow);
    const bool last = t + 1 == a.steps;
    // A = X X^T; symmetric, so a lane's four results go to one row (all blocks: half of
    // them would leave wavefronts idle)
    const float fxx = ldexpf(a.f_xx, -2 * k);
#pragma unroll 1
    for (int b = wave; b < blocks; b += kSmallWaves) {
      const int p0 = b / bm * 32, q0 = b % bm * 32;
      using Mac = MacHalf<2, true>;
      typename Mac::Acc sums[2][2] = {};
      block_product<false, Mac>(X, p0, X, q0, np, lr, lq, sums);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const v4f x = Mac::sum(sums[i][j]) * fxx;
          const float v[4] = {x[0], x[1], x[2], x[3]};
          put(A, q0 + j * 16 + lr, p0 + i * 16 + lq * 4, v);
        }
    }
    __syncthreads();
    // B = b A + c A A
    {
      constexpr int kEach = (kSmallMost / 32) * (kSmallMost / 32) / kSmallWaves;
      v4f acc[kEach][2][2] = {};
#pragma unroll
      for (int n = 0; n < kEach; ++n) {
        const int b = wave + n * kSmallWaves;
        if (b < blocks)
          block_product<false, MacHalf<2, false>>(A, b / bm * 32, A, b % bm * 32, mp, lr, lq, acc[n]);
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < kEach; ++n) {
        const int b = wave + n * kSmallWaves;
        if (b >= blocks) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = b % bm * 32 + j * 16 + lr, c = b / bm * 32 + i * 16 + lq * 4;
            const v4f x = get(A, r, c);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = __builtin_fmaf(a.f_a, x[e], acc[n][i][j][e] * a.f_aa);
            put(A, r, c, v);
          }
      }
    }
    __syncthreads();
    // X = a X + B X: X's columns as the first operand, so that a lane's results lie in a row
    const int shift = last ? -k : kn - k;
    const float fb = ldexpf(last ? a.f_out : a.f_bx, shift);
    const float fx = ldexpf(last ? a.f_x / a.scale_x : a.f_x, shift);
    v4f acc[kSmallBlocks][2][2] = {};
#pragma unroll
    for (int n = 0; n < kSmallBlocks; ++n) {
      const int b = wave + n * kSmallWaves;
      if (b < xblocks)
        block_product<true, MacHalf<2, false>>(X, b / bm * 32, A, b % bm * 32, mp, lr, lq, acc[n]);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kSmallBlocks; ++n) {
      const int b = wave + n * kSmallWaves;
      if (b >= xblocks) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = b % bm * 32 + j * 16 + lr, c = b / bm * 32 + i * 16 + lq * 4;
          const v4f x = get(X, r, c);
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = __builtin_fmaf(fx, x[e], acc[n][i][j][e] * fb);
          if (!last) {
            put(X, r, c, v);
          } else {  // the fp32 result, its two halves in the pieces' places
            u16x4 h, l;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              h[e] = (uint16_t)(__float_as_uint(v[e]) >> 16);
              l[e] = (uint16_t)__float_as_uint(v[e]);
            }
            *(u16x4*)(X.p[0] + r * X.ld + c) = h;
            *(u16x4*)(X.p[1] + r * X.ld + c) = l;
          }
        }
    }
    __syncthreads();
  }
  // (an update's weights four fours at a time, as above)
  at = Place{tid / quads, tid % quads};
  while (at.r < a.M) {
    v4f w[4];
    Place was[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      was[h] = at;
      if (a.W && at.r < a.M)
        w[h] = load4(a.W + (long long)g * a.sW + (long long)at.r * a.ldw + at.c * 4,
                     a.N - at.c * 4);
      at.next(dr, dc, quads);
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int r = was[h].r, c = was[h].c * 4;
      if (r < a.M) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int o = a.flip ? (c + e) * X.ld + r : r * X.ld + c + e;
          v[e] = __uint_as_float((uint32_t)((const uint16_t*)X.p[0])[o] << 16 |
                                 ((const uint16_t*)X.p[1])[o]);
        }
        result(a, g, r, c, a.N - c, v, w[h]);
      }
    }
  }
}

// More than 64 KB of LDS has to be asked for once on each device.
hipError_t allow_small_lds() {
  static std::atomic<bool> done[64] = {};
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (done[dev].load(std::memory_order_acquire)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(
      (const void*)k_ortho_small, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallLds);
  if (e == hipSuccess) done[dev].store(true, std::memory_order_release);
  return e;
}

// ------------------------------------------------------------------ launches
// How a product is cut into tiles: their size, and how many stages of loads are in flight.
struct Cut {
  int tile, stages;
};
// The cut of least estimated time; tiles(T): how many tiles of T there are. A compute unit
// takes per_cu workgroups at once (LDS), a round of them costs per_cu times `each`, and the
// last round as much as a full one. `each` is the cost of one tile relative to the others,
// fitted to products with one cut forced for all of them. Measured since, B X in fp32
// precision, us for one tile on each unit and an inner range of 2048, in the order of `cuts`:
//   4096^2:     14, 14, 42, 43, 87, 145      8 x 2048^2:   18, 18, 56, 55, 107, 181
// and the whole products, of which the table picks the fastest each time:
//   4096^2, X X^T:   333, 322, 221, 231, 172, 224      B X:   454, 449, 335, 342, 348, 291
//   8 x 2048^2:      312, 309, 243, 243, 260, 269             576, 574, 452, 443, 429, 362
// The 192 x 192 tiles are for what 256 x 256 ones leave half of the units without: the
// triangles of 4096 x 8192 in bf16 172 + 97 -> 150 + 78 us a step, 4 x 1500^2 1137 -> 993 us
// in all. At the other end, with one workgroup to a unit, a product waits for loads and
// launches: 512^2 takes 125 us in 64 x 64 tiles of four stages, 136 of three, 213 / 282 in
// 128 x 128 tiles of four / two, 609 in 256 x 256 ones.
constexpr int kCus = 256;
constexpr int kCuts = 6;
template <class F>
Cut best_cut(F tiles, int n = kCuts) {
  const Cut cuts[kCuts] = {{64, 4}, {64, 3}, {128, 4}, {128, 2}, {192, 2}, {256, 2}};
  const int per_cu[kCuts] = {2, 3, 1, 2, 1, 1};
  const double each[kCuts] = {1.6, 1.55, 4.3, 3.8, 8.4, 12.6};
  int at = 0;
  double least = 0;
  for (int i = 0; i < n; ++i) {
    const double rounds = std::ceil((double)tiles(cuts[i].tile) / (kCus * per_cu[i]));
    const double t = rounds * per_cu[i] * each[i];
    if (i == 0 || t < least) {
      at = i;
      least = t;
    }
  }
  return cuts[at];
}

template <int P, bool SECOND, int T, int S>
void launch_gram(const OrthoArgs& a, int step, hipStream_t s) {
  const int tm = (a.mp + T - 1) / T, total = tm * (tm + 1) / 2 * a.G;
  hipLaunchKernelGGL((k_ortho_gram<P, SECOND, T, S>), grid_of(total), dim3((Shape<T, S>::kThreads)), 0,
                     s, a, step, tm, total);
}
template <int P, bool SECOND>
void gram(Cut c, const OrthoArgs& a, int step, hipStream_t s) {
  if (c.tile == 256) return launch_gram<P, SECOND, 256, 2>(a, step, s);
  if (c.tile == 192) return launch_gram<P, SECOND, 192, 2>(a, step, s);
  if (c.tile == 128 && c.stages == 2) return launch_gram<P, SECOND, 128, 2>(a, step, s);
  if (c.tile == 128) return launch_gram<P, SECOND, 128, 4>(a, step, s);
  if (c.stages == 3) return launch_gram<P, SECOND, 64, 3>(a, step, s);
  return launch_gram<P, SECOND, 64, 4>(a, step, s);
}
template <int P, bool LAST, int T, int S>
void launch_apply(const OrthoArgs& a, int step, hipStream_t s) {
  const int tp = (a.mp + T - 1) / T, tq = (a.np + T - 1) / T, total = tp * tq * a.G;
  hipLaunchKernelGGL((k_ortho_apply<P, LAST, T, S>), grid_of(total), dim3((Shape<T, S>::kThreads)), 0,
                     s, a, step, tp, tq, total);
}
template <int P, bool LAST>
void apply(Cut c, const OrthoArgs& a, int step, hipStream_t s) {
  if (c.tile == 256) return launch_apply<P, LAST, 256, 2>(a, step, s);
  if (c.tile == 192) return launch_apply<P, LAST, 192, 2>(a, step, s);
  if (c.tile == 128 && c.stages == 2) return launch_apply<P, LAST, 128, 2>(a, step, s);
  if (c.tile == 128) return launch_apply<P, LAST, 128, 4>(a, step, s);
  // (of matrices of kOnePieceFrom rows and more, whose 64 x 64 tiles are three times as many as
  // their 128 x 128 ones, no count makes three stages of the small ones the cheapest)
  if constexpr (P == 2)
    if (c.stages == 3) return launch_apply<P, LAST, 64, 3>(a, step, s);
  return launch_apply<P, LAST, 64, 4>(a, step, s);
}

constexpr size_t kOrthoAlign = 256;
size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }
// Workgroups a matrix's norm takes: eight fours a thread, or more where that makes over
// 1024 partial sums.
int norm_chunks(int M, int N) {
  const long long c = ((long long)M * ((N + 3) / 4) + 8 * kThreads - 1) / (8 * kThreads);
  return (int)(c > 1024 ? 1024 : c);
}

// From this many rows on the bf16 form multiplies first pieces alone. The fewer rows, the less
// their errors average out: the bf16 result of that many rows is off by (1e-3; 1.66 is its
// rounding alone, and all there is with two pieces)
//   130 to 160: 2.3 to 2.5, 256: 2.3 to 2.4, 384: 2.2 to 2.4, 448 and 512: 2.1 to 2.3, 2048: 2.0
// and the two pieces' time is, with the single ones' in brackets, for eight matrices in us
//   256 x 256: 106 (89), 256 x 1000: 143 (112), 384 x 384: 132 (99), 384 x 1000: 177 (129),
//   448 x 1000: 185 (143).
// There is no step in either: small matrices keep their precision, where it costs 20 to 40 us,
// large ones, which wait for the matrix cores, do not.
constexpr int kOnePieceFrom = 385;

struct OrthoPlan {
  bool small;
  int pieces;
  int mp, np, chunks;
  size_t part, kexp, xr, xt[2], A, B, total;
};
OrthoPlan ortho_plan(bool bf16, int G, int M, int N) {
  OrthoPlan p{};
  p.pieces = bf16 && (M < N ? M : N) >= kOnePieceFrom ? 1 : 2;
  p.mp = (int)up(M < N ? M : N, 32);
  p.np = (int)up(M < N ? N : M, 32);
  p.small = p.mp <= kSmallMost && small_lds(p.mp, p.np) <= kSmallLds;
  if (p.small) return p;
  p.mp = (int)up(M < N ? M : N, 64);
  p.np = (int)up(M < N ? N : M, 64);
  p.chunks = norm_chunks(M, N);
  size_t t = 0;
  auto take = [&](size_t bytes) {
    const size_t at = t;
    t = up(t + bytes, kOrthoAlign);
    return at;
  };
  const size_t x = (size_t)G * p.mp * p.np * 2, s = (size_t)G * p.pieces * p.mp * p.mp * 2;
  p.part = take((size_t)G * p.chunks * 8);
  p.kexp = take((size_t)G * 4);
  p.xr = take(x * p.pieces);
  p.xt[0] = take(x * 2);
  p.xt[1] = take(x * 2);
  p.A = take(s);
  p.B = take(s);
  p.total = t;
  return p;
}

Cut gram_cut(const OrthoPlan& p, int G, int n = kCuts) {
  return best_cut([&](int T) {
    const long long r = (p.mp + T - 1) / T;
    return r * (r + 1) / 2 * G;
  }, n);
}
// X X^T of few rows takes no 256 x 256 tiles, the last of the cuts, which keep its sums in one:
// 256 of 256 x 4096 off by 3.8e-6 in those and 2.6e-6 in others at the same speed (6566 and
// 6498 us in all; 256 x 512 1161 and 1217 us, 1.8e-6 and 1.7e-6). From 512 rows on the other
// products' errors are as large (80 of 512 x 8192 2.2e-6 and 1.8e-6) and the tiles gain 1 to 7%.
Cut x_cut(const OrthoPlan& p, int G) {
  return gram_cut(p, G, p.mp < kOnePieceFrom ? kCuts - 1 : kCuts);
}
Cut apply_cut(const OrthoPlan& p, int G) {
  return best_cut([&](int T) {
    return (long long)((p.mp + T - 1) / T) * ((p.np + T - 1) / T) * G;
  });
}

template <int P>
hipError_t ortho(const OrthoArgs& a, const OrthoPlan& p, hipStream_t s) {
  // (64 x 64 tiles are the most there are of anything)
  const long long tiles = (long long)(p.mp / 64) * (p.np / 64);
  if (tiles * a.G > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_ortho_norm, grid_of((long long)p.chunks * a.G), dim3(kThreads), 0, s, a,
                     p.chunks);
  hipLaunchKernelGGL(k_ortho_split<P>, grid_of(tiles * a.G), dim3(kThreads), 0, s, a, p.chunks,
                     p.mp / 64, p.np / 64);
  const Cut cx = x_cut(p, a.G), cg = gram_cut(p, a.G), ca = apply_cut(p, a.G);
  for (int t = 0; t < a.steps; ++t) {
    gram<P, false>(cx, a, t, s);
    gram<P, true>(cg, a, t, s);
    if (t + 1 < a.steps)
      apply<P, false>(ca, a, t, s);
    else
      apply<P, true>(ca, a, t, s);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t ortho_workspace_bytes(int bf16, int G, int M, int N) {
  return ortho_plan(bf16, G, M, N).total;
}

void ortho_cut(int bf16, int G, int M, int N, int cut[7]) {
  const OrthoPlan p = ortho_plan(bf16, G, M, N);
  std::fill(cut, cut + 7, 0);
  if (p.small) return;
  const Cut x = x_cut(p, G), g = gram_cut(p, G), a = apply_cut(p, G);
  const int v[7] = {p.pieces, x.tile, x.stages, g.tile, g.stages, a.tile, a.stages};
  std::copy(v, v + 7, cut);
}

hipError_t launch_ortho(int bf16, OrthoArgs a, void* ws, hipStream_t s) {
  const OrthoPlan p = ortho_plan(bf16, a.G, a.M, a.N);
  char* w = (char*)ws;
  a.part = (double*)(w + p.part);
  a.kexp = (int*)(w + p.kexp);
  a.Xr = (_Float16*)(w + p.xr);
  a.Xt[0] = (_Float16*)(w + p.xt[0]);
  a.Xt[1] = (_Float16*)(w + p.xt[1]);
  a.A = (_Float16*)(w + p.A);
  a.B = (_Float16*)(w + p.B);
  a.flip = a.M > a.N;
  a.mp = p.mp;
  a.np = p.np;
  if (p.small) {
    const size_t lds = small_lds(p.mp, p.np);
    if (hipError_t e = allow_small_lds()) return e;
    hipLaunchKernelGGL(k_ortho_small, grid_of(a.G), dim3(kSmallThreads), lds, s, a, p.mp, p.np);
    return hipGetLastError();
  }
  return p.pieces == 2 ? ortho<2>(a, p, s) : ortho<1>(a, p, s);
}

}  // namespace lsgd
