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
// the products take the first piece alone (2^-12), an eighth of bf16's own
// rounding; X keeps both pieces there too, because a X passes on the small
// singular directions, which the steps amplify by a each time: rounding X itself to
// 11 bits loses them (error 1.8e-2 instead of 1.7e-3 for matrices of low rank in noise).
//
// A and B are symmetric: only their tiles on and below the diagonal are computed,
// and each is stored on both sides. All three products are tiles of tile_loop.h.
// A matrix whose norm is small against eps starts that much below 1 and grows by at
// most a known factor a step; X of step t is held 2^k(t) higher, k(t) = max(0,
// k(0) - t * grow), so that it too has all of its bits.
// The steps work on m = min(M, N) rows. X lies in memory both ways, [m][n] for X X^T
// and [n][m] for B X, rows padded with zeros to a multiple of 64 so that no product
// has a tail; a zero row or column stays zero through the steps. In fp32 precision the two
// pieces of 32 neighbours share a line of 128 bytes, first pieces, then second ones; in
// the bf16 form each piece is a matrix of its own, and only the first is multiplied.
#include "kernels.h"
#include "tile_loop.h"

namespace lsgd {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

// ------------------------------------------------------------- the first step
__device__ __forceinline__ float load_elem(const void* p, int bf16, long long i) {
  return bf16 ? bf16_to_f32(((const bf16_t*)p)[i]) : ((const float*)p)[i];
}

// An element of the matrix to orthogonalise: X's, or of an update d = g + m u or u.
// STEP: takes the momentum step u = m u + g first and stores it.
template <bool STEP>
__device__ __forceinline__ float direction(const OrthoArgs& a, int g, int r, int c) {
  if (!a.U) return load_elem(a.X, a.x_bf16, (long long)g * a.sX + (long long)r * a.ldx + c);
  float* pu = a.U + (long long)g * a.sU + (long long)r * a.ldu + c;
  const float gr = ((const float*)a.X)[(long long)g * a.sX + (long long)r * a.ldx + c];
  float u = *pu;
  if constexpr (STEP) {
    u = __builtin_fmaf(a.mom, u, gr);
    *pu = u;
  }
  return a.nesterov ? __builtin_fmaf(a.mom, u, gr) : u;
}

// Partial sums of squares in 64 bits, [G][chunks] (no overflow for any fp32 input),
// and an update's momentum step.
__global__ __launch_bounds__(kThreads) void k_ortho_norm(OrthoArgs a, int chunks) {
  const unsigned id = workgroup_id();
  if (id >= (unsigned)chunks * a.G) return;
  const int g = id / chunks, ch = id % chunks;
  const int by = chunks * kThreads, dr = by / a.N, dc = by % a.N;
  const int first = ch * kThreads + threadIdx.x;
  int r = first / a.N, c = first % a.N;
  double s = 0;
  while (r < a.M) {
    const double d = direction<true>(a, g, r, c);
    s += d * d;
    r += dr;
    c += dc;
    if (c >= a.N) {
      c -= a.N;
      ++r;
    }
  }
  __shared__ double red[kThreads];
  red[threadIdx.x] = s;
  __syncthreads();
  for (int w = kThreads / 2; w; w /= 2) {
    if (threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.part[(long long)g * chunks + ch] = red[0];
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
  double s = 0;
  for (int i = 0; i < chunks; ++i) s += a.part[(long long)g * chunks + i];
  const double norm = sqrt(s), r = norm / (norm + (double)a.eps);
  const int k = r > 0 ? min(100, -ilogb(r)) : 0;  // 0 for an infinite or NaN norm
  if (id % (tm * tn) == 0 && threadIdx.x == 0) a.kexp[g] = max(k, 0);
  const double inv = ldexp((double)a.scale_x, max(k, 0)) / (norm + (double)a.eps);
  const int m = a.flip ? a.N : a.M, n = a.flip ? a.M : a.N;
  for (int i = threadIdx.x; i < 4096; i += kThreads) {
    // the loads run along the matrix's own rows
    const int y = i >> 6, x = i & 63, p = a.flip ? p0 + x : p0 + y, q = a.flip ? q0 + y : q0 + x;
    float v = 0.f;
    if (p < m && q < n)
      v = (float)((double)direction<false>(a, g, a.flip ? q : p, a.flip ? p : q) * inv);
    tile[p - p0][q - q0] = v;
  }
  __syncthreads();
  const long long plane = (long long)a.mp * a.np;
  _Float16* X = a.Xr + (long long)g * P * plane;
  _Float16* T = a.Xt[0] + (long long)g * 2 * plane;
  for (int i = threadIdx.x; i < 4096; i += kThreads) {
    const int y = i >> 6, x = i & 63;
    _Float16 h, l;
    split2(tile[y][x], h, l);
    const long long o = at<P>(p0 + y, q0 + x, a.np);
    X[o] = h;
    if constexpr (P == 2) X[o + 32] = l;
    split2(tile[x][y], h, l);
    const long long t = at<P>(q0 + y, p0 + x, a.mp);
    T[t] = h;
    T[t + second<P>(plane)] = l;
  }
}

// ------------------------------------------------------------------ products
// A fragment is 32 k of both pieces (P == 2) or 64 of the first.
template <int P_>
struct MacHalf {
  typedef Frag P;
  typedef Frag Q;
  __device__ __forceinline__ void load(uint8_t*, int, bool) const {}
  __device__ __forceinline__ void begin(const uint8_t*, int) const {}
  __device__ __forceinline__ P p(const Frag& f, int) const { return f; }
  __device__ __forceinline__ Q q(const Frag& f, int) const { return f; }
  __device__ __forceinline__ void mac(v4f& c, const P& p, int, const Q& q, int) const {
    const f16x8 p0 = half<0>(p), p1 = half<4>(p), q0 = half<0>(q), q1 = half<4>(q);
    if constexpr (P_ == 2) {
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

// The symmetric products: A = X X^T (SECOND = false) and B = b A + c A A, tiles on and
// below the diagonal.
template <int P, bool SECOND, int BT, int WP, int WQ>
__global__ __launch_bounds__(64 * (BT / WP) * (BT / WQ), 2) void k_ortho_gram(OrthoArgs a,
                                                                              int step, int tm,
                                                                              int total) {
  using T = TileLoop<BT, BT, WP, WQ>;
  __shared__ __align__(16) uint8_t s0[T::kStage];
  __shared__ __align__(16) uint8_t s1[T::kStage];
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
  MacHalf<P> mac;
  v4f acc[T::FP][T::FQ] = {};
  t.run(s0, s1, ld / 128, mac, acc);
  const int lr = t.lane & 15, lq = t.lane >> 4;
#pragma unroll
  for (int j = 0; j < T::FQ; ++j) {
    const int q = q0 + t.wq + j * 16 + lr;
    if (q >= a.mp) continue;
#pragma unroll
    for (int i = 0; i < T::FP; ++i) {
      const int p = p0 + t.wp + i * 16 + lq * 4;
      if (p >= a.mp) continue;
      const long long mirror = at<P>(q, p, a.mp);
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e] * f;
      if constexpr (SECOND) {
        const f16x4 x = *(const f16x4*)(src + mirror);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float s = (float)x[e];
          if constexpr (P == 2) s += (float)src[mirror + 32 + e];
          v[e] = __builtin_fmaf(a.f_a, s, v[e]);
        }
      }
      const f16x4 h = first_of(v), w = second_of(v, h);
      *(f16x4*)(dst + mirror) = h;
      if constexpr (P == 2) *(f16x4*)(dst + mirror + 32) = w;
      if (pt != qt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const long long o = at<P>(p + e, q, a.mp);
          dst[o] = h[e];
          if constexpr (P == 2) dst[o + 32] = w[e];
        }
      }
    }
  }
}

// X := a X + B X; on the last step what the caller asked for.
template <int P, bool LAST, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(64 * (BP / WP) * (BQ / WQ), 2) void k_ortho_apply(
    OrthoArgs a, int step, int tp, int tq, int total) {
  using T = TileLoop<BP, BQ, WP, WQ>;
  __shared__ __align__(16) uint8_t s0[T::kStage];
  __shared__ __align__(16) uint8_t s1[T::kStage];
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int l = xcd_order(id, total), g = l / (tp * tq);
  int pt, qt;
  band_order(l % (tp * tq), tp, tq, pt, qt);
  const int p0 = pt * BP, q0 = qt * BQ, from = step & 1;
  const long long px = (long long)a.mp * a.np, pm = (long long)a.mp * a.mp;
  const _Float16* X = a.Xt[from] + g * 2 * px;
  T t;
  const int ld = a.mp * P * 2;
  t.init((const uint8_t*)(a.B + g * P * pm) + (long long)p0 * ld,
         (const uint8_t*)X + (long long)q0 * ld, ld, a.mp - p0, a.np - q0);
  MacHalf<P> mac;
  v4f acc[T::FP][T::FQ] = {};
  t.run(s0, s1, ld / 128, mac, acc);
  const int k = raise(a, g, step);
  const int shift = LAST ? -k : raise(a, g, step + 1) - k;
  const float fb = ldexpf(LAST ? a.f_out : a.f_bx, shift);
  const float fx = ldexpf(LAST ? a.f_x / a.scale_x : a.f_x, shift);
  const int lr = t.lane & 15, lq = t.lane >> 4;
  const int m = a.flip ? a.N : a.M, n = a.flip ? a.M : a.N;
#pragma unroll
  for (int j = 0; j < T::FQ; ++j) {
    const int q = q0 + t.wq + j * 16 + lr;
    if (q >= a.np) continue;
#pragma unroll
    for (int i = 0; i < T::FP; ++i) {
      const int p = p0 + t.wp + i * 16 + lq * 4;
      if (p >= a.mp) continue;
      const long long turned = at<P>(q, p, a.mp);
      const f16x4 xh = *(const f16x4*)(X + turned), xl = *(const f16x4*)(X + turned + second<P>(px));
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = __builtin_fmaf(fx, (float)xh[e] + (float)xl[e], acc[i][j][e] * fb);
      if constexpr (LAST) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (p + e >= m || q >= n) continue;
          const int r = a.flip ? q : p + e, c = a.flip ? p + e : q;
          if (a.W) {
            float* w = a.W + (long long)g * a.sW + (long long)r * a.ldw + c;
            *w = __builtin_fmaf(a.keep, *w, a.step * v[e]);
          } else {
            const long long o = (long long)g * a.sY + (long long)r * a.ldy + c;
            if (a.x_bf16)
              ((bf16_t*)a.Y)[o] = f32_to_bf16(v[e]);
            else
              ((float*)a.Y)[o] = v[e];
          }
        }
      } else {
        const f16x4 h = first_of(v), w = second_of(v, h);
        _Float16* O = a.Xt[1 - from] + g * 2 * px;
        _Float16* R = a.Xr + g * P * px;
        *(f16x4*)(O + turned) = h;
        *(f16x4*)(O + turned + second<P>(px)) = w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const long long o = at<P>(p + e, q, a.np);
          R[o] = h[e];
          if constexpr (P == 2) R[o + 32] = w[e];
        }
      }
    }
  }
}

// The launches of the steps with square tiles of BT.
template <int P, int BT, int WP, int WQ>
hipError_t steps(const OrthoArgs& a, hipStream_t s) {
  const int tm = (a.mp + BT - 1) / BT, tn = (a.np + BT - 1) / BT;
  const long long tri = (long long)tm * (tm + 1) / 2 * a.G, full = (long long)tm * tn * a.G;
  if (tri > 0x7fffffffLL || full > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 block(64 * (BT / WP) * (BT / WQ));
  for (int t = 0; t < a.steps; ++t) {
    hipLaunchKernelGGL((k_ortho_gram<P, false, BT, WP, WQ>), grid_of(tri), block, 0, s, a, t, tm,
                       (int)tri);
    hipLaunchKernelGGL((k_ortho_gram<P, true, BT, WP, WQ>), grid_of(tri), block, 0, s, a, t, tm,
                       (int)tri);
    if (t + 1 < a.steps)
      hipLaunchKernelGGL((k_ortho_apply<P, false, BT, BT, WP, WQ>), grid_of(full), block, 0, s, a,
                         t, tm, tn, (int)full);
    else
      hipLaunchKernelGGL((k_ortho_apply<P, true, BT, BT, WP, WQ>), grid_of(full), block, 0, s, a,
                         t, tm, tn, (int)full);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

constexpr size_t kOrthoAlign = 256;
size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }
int norm_chunks(long long n) {
  const long long c = (n + 16383) / 16384;
  return (int)(c < 1 ? 1 : c > 256 ? 256 : c);
}

struct OrthoPlan {
  int mp, np, chunks;
  size_t part, kexp, xr, xt[2], A, B, total;
};
OrthoPlan ortho_plan(int pieces, int G, int M, int N) {
  OrthoPlan p;
  p.mp = (int)up(M < N ? M : N, 64);
  p.np = (int)up(M < N ? N : M, 64);
  p.chunks = norm_chunks((long long)M * N);
  size_t t = 0;
  auto take = [&](size_t bytes) {
    const size_t at = t;
    t = up(t + bytes, kOrthoAlign);
    return at;
  };
  const size_t x = (size_t)G * p.mp * p.np * 2, s = (size_t)G * pieces * p.mp * p.mp * 2;
  p.part = take((size_t)G * p.chunks * 8);
  p.kexp = take((size_t)G * 4);
  p.xr = take(x * pieces);
  p.xt[0] = take(x * 2);
  p.xt[1] = take(x * 2);
  p.A = take(s);
  p.B = take(s);
  p.total = t;
  return p;
}

template <int P>
hipError_t ortho(const OrthoArgs& a, const OrthoPlan& p, hipStream_t s) {
  const long long tiles = (long long)(p.mp / 64) * (p.np / 64);
  if (tiles * a.G > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_ortho_norm, grid_of((long long)p.chunks * a.G), dim3(kThreads), 0, s, a,
                     p.chunks);
  hipLaunchKernelGGL(k_ortho_split<P>, grid_of(tiles * a.G), dim3(kThreads), 0, s, a, p.chunks,
                     p.mp / 64, p.np / 64);
  if (hipError_t e = hipGetLastError()) return e;
  auto count = [&](long long b) {
    const long long tm = (p.mp + b - 1) / b;
    return tm * (tm + 1) / 2 * a.G;
  };
  if (count(256) >= 128) return steps<P, 256, 128, 64>(a, s);
  if (count(128) >= 128) return steps<P, 128, 64, 64>(a, s);
  return steps<P, 64, 32, 32>(a, s);
}

}  // namespace

size_t ortho_workspace_bytes(int pieces, int G, int M, int N) {
  return ortho_plan(pieces, G, M, N).total;
}

hipError_t launch_ortho(int pieces, OrthoArgs a, void* ws, hipStream_t s) {
  const OrthoPlan p = ortho_plan(pieces, a.G, a.M, a.N);
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
  return pieces == 2 ? ortho<2>(a, p, s) : ortho<1>(a, p, s);
}

}  // namespace lsgd
