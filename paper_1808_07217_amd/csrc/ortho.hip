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
// and each is stored on both sides.
// A matrix whose norm is small against eps starts that much below 1 and grows by at
// most a known factor a step; X of step t is held 2^k(t) higher, k(t) = max(0,
// k(0) - t * grow), so that it too has all of its bits.
// The steps work on m = min(M, N) rows. X lies in memory both ways, [m][n] for X X^T
// and [n][m] for B X, rows padded with zeros to a multiple of 64 so that no product
// has a tail; a zero row or column stays zero through the steps.
#include "device_common.h"
#include "kernels.h"

namespace lsgd {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

__device__ __forceinline__ float load_elem(const void* p, int bf16, long long i) {
  return bf16 ? bf16_to_f32(((const bf16_t*)p)[i]) : ((const float*)p)[i];
}

// Element i of the matrix to orthogonalise: X's, or of an update d = g + m u or u.
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
  const long long n = (long long)a.M * a.N;
  double s = 0;
  for (long long i = (long long)ch * kThreads + threadIdx.x; i < n; i += (long long)chunks * kThreads) {
    const double d = direction<true>(a, g, (int)(i / a.N), (int)(i % a.N));
    s += d * d;
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

// k(t) of matrix g: see the top.
__device__ __forceinline__ int raise(const OrthoArgs& a, int g, int t) {
  return max(0, a.kexp[g] - t * a.grow);
}

// X / (|X|_F + eps) times the scale, in pieces, both ways; zeros in the padding.
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
  _Float16* X = a.Xr + (long long)g * 2 * plane;
  _Float16* T = a.Xt[0] + (long long)g * 2 * plane;
  for (int i = threadIdx.x; i < 4096; i += kThreads) {
    const int y = i >> 6, x = i & 63;
    _Float16 h, l;
    split2(tile[y][x], h, l);
    X[(long long)(p0 + y) * a.np + q0 + x] = h;
    X[plane + (long long)(p0 + y) * a.np + q0 + x] = l;
    split2(tile[x][y], h, l);
    T[(long long)(q0 + y) * a.mp + p0 + x] = h;
    T[plane + (long long)(q0 + y) * a.mp + p0 + x] = l;
  }
}

// A product of two matrices with the contracted index contiguous, in P pieces:
// 4 wavefronts, each 32 x 32 of a 64 x 64 tile. Lane l takes 8 k from 8 (l / 16) of row
// l % 16 of either operand; result e of lane l is at row 4 (l / 16) + e of the first
// and row l % 16 of the second.
template <int P>
__device__ __forceinline__ void tile_product(const _Float16* A, long long planeA,
                                             const _Float16* B, long long planeB, int ld, int K,
                                             int p0, int q0, int rows_a, int rows_b,
                                             v4f (&acc)[2][2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const _Float16 *pa[2], *pb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    pa[i] = A + (long long)min(p0 + (wave >> 1) * 32 + i * 16 + lr, rows_a - 1) * ld + lq * 8;
    pb[i] = B + (long long)min(q0 + (wave & 1) * 32 + i * 16 + lr, rows_b - 1) * ld + lq * 8;
  }
  for (int k = 0; k < K; k += 32) {
    f16x8 a[2][P], b[2][P];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        a[i][p] = *(const f16x8*)(pa[i] + p * planeA + k);
        b[i][p] = *(const f16x8*)(pb[i] + p * planeB + k);
      }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (P == 2) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][1], b[j][0], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][0], b[j][1], acc[i][j], 0, 0, 0);
        }
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][0], b[j][0], acc[i][j], 0, 0, 0);
      }
  }
}

// The symmetric products: A = X X^T (SECOND = false) and B = b A + c A A, tiles on and
// below the diagonal.
template <int P, bool SECOND>
__global__ __launch_bounds__(kThreads) void k_ortho_gram(OrthoArgs a, int step, int tm) {
  const int tri = tm * (tm + 1) / 2;
  const unsigned id = workgroup_id();
  if (id >= (unsigned)tri * a.G) return;
  const int g = id / tri;
  int t = id % tri, pt = 0;
  while (t > pt) t -= ++pt;  // row pt holds pt + 1 tiles
  const int p0 = pt * 64, q0 = t * 64;
  const long long px = (long long)a.mp * a.np, pm = (long long)a.mp * a.mp;
  const _Float16* src = SECOND ? a.A + (long long)g * P * pm : a.Xr + (long long)g * 2 * px;
  _Float16* dst = (SECOND ? a.B : a.A) + (long long)g * P * pm;
  const float f = SECOND ? a.f_aa : ldexpf(a.f_xx, -2 * raise(a, g, step));
  v4f acc[2][2] = {};
  if constexpr (SECOND)
    tile_product<P>(src, pm, src, pm, a.mp, a.mp, p0, q0, a.mp, a.mp, acc);
  else
    tile_product<P>(src, px, src, px, a.np, a.np, p0, q0, a.mp, a.mp, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int p = p0 + (wave >> 1) * 32 + i * 16 + lq * 4 + e;
        const int q = q0 + (wave & 1) * 32 + j * 16 + lr;
        const long long at = (long long)p * a.mp + q, mirror = (long long)q * a.mp + p;
        float v = acc[i][j][e] * f;
        if constexpr (SECOND) {
          float s = (float)src[at];
          if constexpr (P == 2) s += (float)src[pm + at];
          v = __builtin_fmaf(a.f_a, s, v);
        }
        _Float16 h, l;
        split2(v, h, l);
        dst[at] = h;
        if constexpr (P == 2) dst[pm + at] = l;
        if (pt != t) {
          dst[mirror] = h;
          if constexpr (P == 2) dst[pm + mirror] = l;
        }
      }
}

// X := a X + B X; on the last step what the caller asked for.
template <int P, bool LAST>
__global__ __launch_bounds__(kThreads) void k_ortho_apply(OrthoArgs a, int step, int tm, int tn) {
  const unsigned id = workgroup_id();
  if (id >= (unsigned)tm * tn * a.G) return;
  const int g = id / (tm * tn), p0 = id % (tm * tn) / tn * 64, q0 = id % tn * 64;
  const long long px = (long long)a.mp * a.np, pm = (long long)a.mp * a.mp;
  const int from = step & 1, k = raise(a, g, step);
  const int shift = LAST ? -k : raise(a, g, step + 1) - k;
  const float fb = ldexpf(LAST ? a.f_out : a.f_bx, shift);
  const float fx = ldexpf(LAST ? a.f_x / a.scale_x : a.f_x, shift);
  const _Float16* T = a.Xt[from] + (long long)g * 2 * px;
  v4f acc[2][2] = {};
  tile_product<P>(a.B + (long long)g * P * pm, pm, T, px, a.mp, a.mp, p0, q0, a.mp, a.np, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const int m = a.flip ? a.N : a.M, n = a.flip ? a.M : a.N;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int p = p0 + (wave >> 1) * 32 + i * 16 + lq * 4 + e;
        const int q = q0 + (wave & 1) * 32 + j * 16 + lr;
        const long long at = (long long)p * a.np + q, turned = (long long)q * a.mp + p;
        const float x = (float)T[turned] + (float)T[px + turned];
        float v = __builtin_fmaf(fx, x, acc[i][j][e] * fb);
        if constexpr (LAST) {
          if (p >= m || q >= n) continue;
          const int r = a.flip ? q : p, c = a.flip ? p : q;
          if (a.W) {
            float* w = a.W + (long long)g * a.sW + (long long)r * a.ldw + c;
            *w = __builtin_fmaf(a.keep, *w, a.step * v);
          } else {
            const long long o = (long long)g * a.sY + (long long)r * a.ldy + c;
            if (a.x_bf16)
              ((bf16_t*)a.Y)[o] = f32_to_bf16(v);
            else
              ((float*)a.Y)[o] = v;
          }
        } else {
          _Float16 h, l;
          split2(v, h, l);
          _Float16* X = a.Xr + (long long)g * 2 * px;
          _Float16* O = a.Xt[1 - from] + (long long)g * 2 * px;
          X[at] = h;
          X[px + at] = l;
          O[turned] = h;
          O[px + turned] = l;
        }
      }
}

template <int P>
hipError_t steps(const OrthoArgs& a, hipStream_t s) {
  const int tm = a.mp / 64, tn = a.np / 64;
  const long long tri = (long long)tm * (tm + 1) / 2 * a.G, full = (long long)tm * tn * a.G;
  if (tri > 0x7fffffffLL || full > 0x7fffffffLL) return hipErrorInvalidValue;
  for (int t = 0; t < a.steps; ++t) {
    hipLaunchKernelGGL((k_ortho_gram<P, false>), grid_of(tri), dim3(kThreads), 0, s, a, t, tm);
    hipLaunchKernelGGL((k_ortho_gram<P, true>), grid_of(tri), dim3(kThreads), 0, s, a, t, tm);
    if (t + 1 < a.steps)
      hipLaunchKernelGGL((k_ortho_apply<P, false>), grid_of(full), dim3(kThreads), 0, s, a, t, tm,
                         tn);
    else
      hipLaunchKernelGGL((k_ortho_apply<P, true>), grid_of(full), dim3(kThreads), 0, s, a, t, tm,
                         tn);
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
  const size_t x = (size_t)G * 2 * p.mp * p.np * 2, s = (size_t)G * pieces * p.mp * p.mp * 2;
  p.part = take((size_t)G * p.chunks * 8);
  p.kexp = take((size_t)G * 4);
  p.xr = take(x);
  p.xt[0] = take(x);
  p.xt[1] = take(x);
  p.A = take(s);
  p.B = take(s);
  p.total = t;
  return p;
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
  const long long tiles = (long long)(p.mp / 64) * (p.np / 64);
  if (tiles * a.G > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_ortho_norm, grid_of((long long)p.chunks * a.G), dim3(kThreads), 0, s, a,
                     p.chunks);
  hipLaunchKernelGGL(k_ortho_split, grid_of(tiles * a.G), dim3(kThreads), 0, s, a, p.chunks,
                     p.mp / 64, p.np / 64);
  if (hipError_t e = hipGetLastError()) return e;
  return pieces == 2 ? steps<2>(a, s) : steps<1>(a, s);
}

}  // namespace lsgd
