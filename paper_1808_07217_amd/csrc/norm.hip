// Layer norm of the rows of G matrices and its gradients.
//
// Forward: mean = sum x / N, d = x - mean, rstd = (sum d^2 / N + eps)^-1/2, y = d rstd w + b.
// Both sums are held in fp64, and the mean in two floats: rows far from zero and
// finite values of any size come out as exactly as others.
// Backward, from the mean and rstd that the forward pass wrote: n = (x - mean) rstd, e = dy w,
// dx = rstd (e - sum e / N - n sum (e n) / N), dw = sum over rows of dy n, db of dy. The mean is a
// float there: of rows far from zero it is found again from x.
//
// Bound by HBM (each tensor is read or written once: 16384 x 8192 in bf16 107 us, 5.0 TB/s, forward, 168 us,
// 4.8, backward; a copy of 4 GB 4.8), small ones by a launch and a load's latency (3 x 1537 x 771 in fp32
// 10 us). A row lies in the registers of as few threads as hold it, sums go over lanes by rotations
// (by way of LDS 127 -> 119 us, 185 -> 167 backward), and the next row is on its way meanwhile.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "lanes.h"
#include "row_io.h"

namespace lsgd {
namespace {

constexpr int kThreads = 256;

// The sums over T threads of a row (T a power of two; wavefronts of a row's own from 64
// on), in all of them; `room`: a wavefront's sums each, another room than the last call's (whose
// sums may still be read by some). From T = 128 on every thread of the workgroup calls it.
template <int T, int K, class A>
__device__ __forceinline__ void row_sums(A (&v)[K], A (*room)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = lanes_sum<(T < 64 ? T : 64)>(v[k]);
  if constexpr (T > 64) {
    const int wave = threadIdx.x >> 6, first = wave / (T / 64) * (T / 64);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) room[wave][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = room[first][k];
#pragma unroll
      for (int w = 1; w < T / 64; ++w) v[k] += room[first + w][k];
    }
  }
}
// Which of a workgroup's rows a thread works on (the same in a whole wavefront from T = 64 on).
template <int T>
__device__ __forceinline__ int slot_of() {
  return T < 64 ? threadIdx.x / T : __builtin_amdgcn_readfirstlane(threadIdx.x / T);
}

// Where |mean| is below it, no distance of an x from it leaves fp32's range.
constexpr float kLarge = 0x1p100f;
// The mean in two floats. A large one is taken by a sixteenth, as is x then.
struct Mean {
  float hi, by, at, lo;
  __device__ __forceinline__ explicit Mean(double mean) {
    hi = (float)mean;
    by = fabsf(hi) >= kLarge ? 0x1p-4f : 1.f;
    at = -hi * by;
    lo = (float)(mean - hi) * by;
  }
  // (x - mean) by
  __device__ __forceinline__ float operator()(float x) const {
    return __builtin_fmaf(x, by, at) - lo;
  }
  // 1 / deviation, from the sum of those distances' squares. A distance becomes its deviations
  // through first and factor, the second no subnormal number (of which bits are lost).
  __device__ __forceinline__ float inverse_root(double squares, int N, float eps, float& factor,
                                                float& first) const {
    const bool large = by != 1.f;
    if (large) squares *= 0x1p8;
    const double rstd = 1.0 / sqrt(squares / N + eps);
    factor = (float)rstd;
    first = 1.f;
    if (large || factor < 0x1p-120f) {
      const double f = large ? rstd * 0x1p4 : rstd;
      if (f < 0x1p-120) first = 0x1p-8f;
      factor = (float)(f / first);
    }
    return (float)rstd;
  }
};

// A strip of rows a workgroup, T threads a row, V vectors of eight values each, in registers;
// the next row is on its way while one is summed. w and b stay in registers over the strip: from
// the cache for every row they would be four times a bf16 row's own bytes.
template <bool XBF, bool YBF, int T, int V, int B>
__global__ __launch_bounds__(B) void k_norm(NormArgs a, int strips, long long total) {
  constexpr int kBlock = B, kRows = kBlock / T;
  __shared__ double room[2][kBlock / 64][1];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int g = id / strips, m0 = (id - g * strips) * a.strip;
  const int t = threadIdx.x % T, slot = slot_of<T>(), end = min(a.M, m0 + a.strip);
  Raw8<XBF> raw[V];
  auto fetch = [&](int m) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int n = (t + i * T) * 8;
      fetch8<XBF, T == 1>(a.X, g * a.sX + m * a.ldx, n, m < end ? a.N : 0, raw[i]);
    }
  };
  fetch(m0 + slot);
  float w[V][8], b[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int n = (t + i * T) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[i][e] = 1.f, b[i][e] = 0.f;
    if (a.w) load8<false, T == 1>(a.w, g * a.sw, n, a.N, w[i]);
    if (a.b) load8<false, T == 1>(a.b, g * a.sb, n, a.N, b[i]);
  }
  for (int r = m0; r < end; r += kRows) {
    const int m = r + slot;
    float x[V][8];
    double s[1] = {0.0};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      settle8<XBF, T == 1>((t + i * T) * 8, a.N, raw[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[i][e] = raw[i][e];
        s[0] += x[i][e];
      }
    }
    if (r + kRows < end) fetch(m + kRows);
    row_sums<T>(s, room[0]);
    const Mean mean(s[0] / a.N);
    s[0] = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int n = (t + i * T) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[i][e] = n + e < a.N ? mean(x[i][e]) : 0.f;
        s[0] += (double)x[i][e] * x[i][e];
      }
    }
    row_sums<T>(s, room[1]);
    float factor, first;
    const float rstd = mean.inverse_root(s[0], a.N, a.eps, factor, first);
    if (first != 1.f) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] *= first;
    }
    if (m < end) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int n = (t + i * T) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = __builtin_fmaf(x[i][e] * factor, w[i][e], b[i][e]);
        store8<YBF>(a.Y, g * a.sY + m * a.ldy, n, a.N, x[i]);
      }
      if (t == 0) {
        a.mean[(long long)g * a.M + m] = mean.hi;
        a.rstd[(long long)g * a.M + m] = rstd;
      }
    }
  }
}

// Rows of any length: three passes over a row, which a compute unit's share of the L2 holds up to
// some 30K values.
constexpr int kLong = 1024;
template <bool XBF, bool YBF>
__global__ __launch_bounds__(kLong) void k_norm_long(NormArgs a, long long total) {
  __shared__ double room[2][kLong / 64][1];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int g = id / a.M, m = id - g * a.M;
  const long long x0 = g * a.sX + m * a.ldx;
  float x[8];
  double s[1] = {0.0};
  for (int n = threadIdx.x * 8; n < a.N; n += kLong * 8) {
    load8<XBF>(a.X, x0, n, a.N, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[0] += x[e];
  }
  row_sums<kLong>(s, room[0]);
  const Mean mean(s[0] / a.N);
  s[0] = 0.0;
  for (int n = threadIdx.x * 8; n < a.N; n += kLong * 8) {
    load8<XBF>(a.X, x0, n, a.N, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = n + e < a.N ? mean(x[e]) : 0.f;
      s[0] += (double)d * d;
    }
  }
  row_sums<kLong>(s, room[1]);
  float factor, first;
  const float rstd = mean.inverse_root(s[0], a.N, a.eps, factor, first);
  for (int n = threadIdx.x * 8; n < a.N; n += kLong * 8) {
    float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, b[8] = {};
    load8<XBF>(a.X, x0, n, a.N, x);
    if (a.w) load8<false>(a.w, g * a.sw, n, a.N, w);
    if (a.b) load8<false>(a.b, g * a.sb, n, a.N, b);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      x[e] = __builtin_fmaf(mean(x[e]) * first * factor, w[e], b[e]);
    store8<YBF>(a.Y, g * a.sY + m * a.ldy, n, a.N, x);
  }
  if (threadIdx.x == 0) {
    a.mean[(long long)g * a.M + m] = mean.hi;
    a.rstd[(long long)g * a.M + m] = rstd;
  }
}

// ---------------------------------------------------------------- backward
// (x - mean) rstd of a row, from the mean as it was written. `far`: its rounding to fp32 moves that by
// up to 2^-13 and more. What is left is then the mean of the results, and taken off; and in columns past
// the last, which hold zeros, it may leave fp32's range. (Below, the mean is what the caller gave: of two
// columns, whose dx is 10^-5 of dy, the difference shows.)
constexpr float kFar = 2048.f;
template <class A>
struct Row {
  A by, at, rstd;
  bool far;
  __device__ __forceinline__ Row(float mean, float rs) {
    const bool large = fabsf(mean) >= kLarge;
    by = large ? 0x1p-4f : 1.f;
    at = -(A)mean * by;
    rstd = (A)rs * (large ? 0x1p4f : 1.f);
    far = !(fabsf(mean) * rs < kFar);
  }
  // (a large mean by a sixteenth, as above)
  __device__ __forceinline__ A operator()(float x) const {
    if constexpr (sizeof(A) == 8)
      return __builtin_fma((double)x, by, at) * rstd;
    else
      return __builtin_fmaf(x, by, at) * rstd;
  }
};

// A strip of rows a workgroup; a thread keeps the sums of its columns over them. A: the
// arithmetic of a row. Of rows of few columns little is left beside the two directions that are
// taken out (of two columns eps / variance of e): those of up to eight, a thread's each, in fp64.
// A column's sum is fp32 over kChain rows of a thread, and fp64 over those; of three vectors and more,
// which leave no registers for that, fp32 over the strip, of kFewSums rows a thread at most. (us, of 16 x
// 128 x 512: fp64 at every row 15.5, over four 14.6, fp32 alone 14.7. Of 20000 x 10000 in bf16: strips of
// 32 rows 275, of 79 253.)
constexpr int kChain = 4;
template <bool XBF, bool YBF, int T, int V, int B, class A>
__global__ __launch_bounds__(B) void k_norm_back(NormBackArgs a, long long total) {
  constexpr int kBlock = B, kRows = kBlock / T, kCols = T * V * 8;
  constexpr bool kWide = V <= 2;
  __shared__ A room[2][kBlock / 64][2], off[2][kBlock / 64];
  // the columns' sums of several rows at work at one time: a wavefront's, or its rows' each
  constexpr int kSlots = T < 64 ? kBlock / 64 : kRows;
  __shared__ float slots[kSlots > 1 ? kSlots * kCols : 1];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int g = id / a.strips, strip = id - g * a.strips, m0 = strip * a.strip;
  const int t = threadIdx.x % T, slot = slot_of<T>(), end = min(a.M, m0 + a.strip);
  // a row as it was read, and the next one on its way (which four vectors leave no registers for)
  constexpr bool kAhead = V < 4;
  Raw8<XBF> xr[V], xn[V];
  Raw8<YBF> dr[V], dn[V];
  float mean_next = 0.f, rstd_next = 0.f;
  auto fetch = [&](int m) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int n = (t + i * T) * 8, N = m < end ? a.N : 0;
      fetch8<XBF, T == 1>(a.X, g * a.sX + m * a.ldx, n, N, xn[i]);
      fetch8<YBF, T == 1>(a.dY, g * a.sg + m * a.ldg, n, N, dn[i]);
    }
    mean_next = m < end ? a.mean[(long long)g * a.M + m] : 0.f;
    rstd_next = m < end ? a.rstd[(long long)g * a.M + m] : 0.f;
  };
  if (kAhead) fetch(m0 + slot);
  float w[V][8], dw[V][8], db[V][8];
  double wide_w[kWide ? V : 1][8] = {}, wide_b[kWide ? V : 1][8] = {};
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int n = (t + i * T) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[i][e] = 1.f, dw[i][e] = db[i][e] = 0.f;
    if (a.w) load8<false, T == 1>(a.w, g * a.sw, n, a.N, w[i]);
  }
  int odd = 0, chain = 0;
  for (int r = m0; r < end; r += kRows, odd ^= 1) {
    const int m = r + slot;
    A s[2] = {0, 0};
    if (!kAhead) fetch(m);
    const float mean = mean_next, rstd = rstd_next;
    const Row<A> row(mean, rstd);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      xr[i] = xn[i];
      dr[i] = dn[i];
      settle8<XBF, T == 1>((t + i * T) * 8, a.N, xr[i]);
      settle8<YBF, T == 1>((t + i * T) * 8, a.N, dr[i]);
    }
    if (kAhead && r + kRows < end) fetch(m + kRows);
    if (kWide || !row.far) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const A x = row(xr[i][e]), dy = (A)dr[i][e] * w[i][e];
          s[0] += dy;
          s[1] += dy * x;
        }
      }
    }
    A shift = 0;
    if (row.far) {
      double f[3] = {0.0, 0.0, 0.0};
      const auto add = [&](bool in, float x, float dy, float w) __attribute__((always_inline)) {
        const A n = in ? row(x) : (A)0, e = (A)dy * w;
        f[0] += e;
        f[1] += (double)e * n;
        f[2] += n;
      };
      if constexpr (kWide) {
        int left = a.N - t * 8;
        asm volatile("" : "+v"(left));  // (or the comparisons are kept over the rows, two registers each)
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
          for (int e = 0; e < 8; ++e) add(i * T * 8 + e < left, xr[i][e], dr[i][e], w[i][e]);
        }
      } else {  // (read again: kept in registers up to here it takes them from every row)
#pragma unroll 1
        for (int i = 0; i < V; ++i) {
          const int n = (t + i * T) * 8;
          float xs[8], ds[8], ws[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
          load8<XBF>(a.X, g * a.sX + m * a.ldx, n, a.N, xs);
          load8<YBF>(a.dY, g * a.sg + m * a.ldg, n, a.N, ds);
          if (a.w) load8<false>(a.w, g * a.sw, n, a.N, ws);
#pragma unroll
          for (int e = 0; e < 8; ++e) add(n + e < a.N, xs[e], ds[e], ws[e]);
        }
      }
      s[0] = (A)f[0];
      s[1] = (A)f[1];
      shift = lanes_sum<(T < 64 ? T : 64)>((A)f[2]);
      if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) off[odd][threadIdx.x >> 6] = shift;
      }
    }
    row_sums<T>(s, room[odd]);
    if (row.far) {
      if constexpr (T > 64) {
        const int first = (threadIdx.x >> 6) / (T / 64) * (T / 64);
        shift = off[odd][first];
#pragma unroll
        for (int k = 1; k < T / 64; ++k) shift += off[odd][first + k];
      }
      shift /= a.N;
      s[1] -= shift * s[0];
    }
    const A c1 = s[0] / a.N, c2 = s[1] / a.N;
    if (m < end) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int n = (t + i * T) * 8;
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const A x = row(xr[i][e]) - shift, dy = (A)dr[i][e] * w[i][e];
          d[e] = (float)(rstd * (dy - c1 - x * c2));  // (zero where dy is c1: of one column)
          dw[i][e] += dr[i][e] * (float)x;
          db[i][e] += dr[i][e];
        }
        store8<XBF>(a.dX, g * a.sd + m * a.ldd, n, a.N, d);
      }
    }
    if constexpr (kWide) {
      if (++chain == kChain && r + kRows < end) {
        chain = 0;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            wide_w[i][e] += dw[i][e];
            wide_b[i][e] += db[i][e];
            dw[i][e] = db[i][e] = 0.f;
          }
      }
    }
  }
  if (!a.dw) return;
  const auto column = [&](int h, int i, int e) __attribute__((always_inline)) {
    double v = h ? db[i][e] : dw[i][e];
    if constexpr (kWide) v += h ? wide_b[i][e] : wide_w[i][e];
    return v;
  };
  // joined in order; one strip is the result itself
  float* to_w = a.strips == 1 ? a.dw + g * a.sdw : a.part + (long long)id * 2 * a.N;
  float* to_b = a.strips == 1 ? a.db + g * a.sdb : a.part + ((long long)id * 2 + 1) * a.N;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float* to = h ? to_b : to_w;
    if constexpr (kSlots == 1) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = (float)column(h, i, e);
        store8<false>(to, 0, (t + i * T) * 8, a.N, sum);
      }
    } else {
      const int mine = T < 64 ? threadIdx.x >> 6 : slot;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = (float)strided_sum<(T < 64 ? T : 64)>(column(h, i, e));
          if (T >= 64 || (threadIdx.x & 63) < T) slots[mine * kCols + (t + i * T) * 8 + e] = v;
        }
      __syncthreads();
      for (int n = threadIdx.x; n < a.N; n += kBlock) {
        double sum = slots[n];
#pragma unroll
        for (int k = 1; k < kSlots; ++k) sum += slots[k * kCols + n];
        to[n] = (float)sum;
      }
    }
  }
}

// dw, db = the strips' sums in order: 64 columns a workgroup, a sixteenth of the strips a
// wavefront. Columns g, (dw then db), n.
constexpr int kJoin = 1024;
__global__ __launch_bounds__(kJoin) void k_norm_join(NormBackArgs a, int tiles, long long total) {
  constexpr int kWaves = kJoin / 64;
  __shared__ double room[kWaves][64];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int gh = id / tiles, g = gh / 2, h = gh & 1, n = (id - gh * tiles) * 64 + lane;
  const int each = (a.strips + kWaves - 1) / kWaves;
  const int k0 = wave * each, k1 = min(a.strips, k0 + each);
  double sum = 0.0;
  if (n < a.N) {
    const float* p = a.part + (((long long)g * a.strips + k0) * 2 + h) * a.N + n;
#pragma unroll 8
    for (int k = k0; k < k1; ++k, p += 2LL * a.N) sum += *p;
  }
  room[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && n < a.N) {
#pragma unroll
    for (int k = 1; k < kWaves; ++k) sum += room[k][lane];
    (h ? a.db + g * a.sdb : a.dw + g * a.sdw)[n] = (float)sum;
  }
}

// Rows of any length: dx in two passes over a row, dw and db from a third, by columns (2048 x 40000
// in bf16 229 us, 2.1 TB/s of what has to move).
template <bool XBF, bool YBF>
__global__ __launch_bounds__(kLong) void k_norm_back_long(NormBackArgs a, long long total) {
  __shared__ double room[kLong / 64][3];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int g = id / a.M, m = id - g * a.M;
  const long long x0 = g * a.sX + m * a.ldx, d0 = g * a.sg + m * a.ldg;
  const float mean = a.mean[id], rstd = a.rstd[id];
  const Row<float> row(mean, rstd);
  double s[3] = {0.0, 0.0, 0.0};
  float x[8], dy[8];
  auto take = [&](int n) __attribute__((always_inline)) {
    float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    load8<XBF>(a.X, x0, n, a.N, x);
    load8<YBF>(a.dY, d0, n, a.N, dy);
    if (a.w) load8<false>(a.w, g * a.sw, n, a.N, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = row(x[e]);
      dy[e] *= w[e];
    }
  };
  for (int n = threadIdx.x * 8; n < a.N; n += kLong * 8) {
    take(n);
    if (row.far) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (n + e >= a.N) x[e] = 0.f;  // (it may have left fp32's range)
        s[2] += x[e];
      }
    }
    float f[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[0] += dy[e];
      f[1] += dy[e] * x[e];
    }
    s[0] += f[0];
    s[1] += f[1];
  }
  row_sums<kLong>(s, room);
  const double off = s[2] / a.N;  // (none but of far rows)
  const float c1 = (float)(s[0] / a.N), shift = (float)off, c2 = (float)((s[1] - off * s[0]) / a.N);
  if (a.dw && threadIdx.x == 0) a.shift[id] = shift;
  for (int n = threadIdx.x * 8; n < a.N; n += kLong * 8) {
    take(n);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = rstd * (dy[e] - c1 - (x[e] - shift) * c2);
    store8<XBF>(a.dX, g * a.sd + m * a.ldd, n, a.N, x);
  }
}
// 512 columns of a strip a workgroup, every fourth row a wavefront.
template <bool XBF, bool YBF>
__global__ __launch_bounds__(kThreads) void k_norm_params(NormBackArgs a, int tiles, long long total) {
  __shared__ float room[2][4][512];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int gs = id / tiles, g = gs / a.strips, m0 = (gs - g * a.strips) * a.strip;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, end = min(a.M, m0 + a.strip);
  const int n0 = (id - gs * tiles) * 512, n = n0 + lane * 8;
  double dw[8] = {}, db[8] = {};
  float w8[8] = {}, b8[8] = {};
  int chain = 0;
  const auto flush = [&]() __attribute__((always_inline)) {
    chain = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] += w8[e];
      db[e] += b8[e];
      w8[e] = b8[e] = 0.f;
    }
  };
  for (int m = m0 + wave; m < end; m += 4) {
    const long long at = (long long)g * a.M + m;
    const Row<float> row(a.mean[at], a.rstd[at]);
    const float shift = a.shift[at];
    float x[8], dy[8];
    load8<XBF>(a.X, g * a.sX + m * a.ldx, n, a.N, x);
    load8<YBF>(a.dY, g * a.sg + m * a.ldg, n, a.N, dy);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w8[e] += dy[e] * (row(x[e]) - shift);
      b8[e] += dy[e];
    }
    if (++chain == kChain) flush();
  }
  flush();
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    room[0][wave][lane * 8 + e] = (float)dw[e];
    room[1][wave][lane * 8 + e] = (float)db[e];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float* to = a.strips == 1 ? (h ? a.db + g * a.sdb : a.dw + g * a.sdw)
                              : a.part + ((long long)gs * 2 + h) * a.N;
    for (int c = threadIdx.x; c < 512 && n0 + c < a.N; c += kThreads)
      to[n0 + c] = (float)(((double)room[h][0][c] + room[h][1][c]) +
                           ((double)room[h][2][c] + room[h][3][c]));
  }
}

// ------------------------------------------------------------------ launches
// Threads and vectors a row of N values takes, and threads of a workgroup; T == 0: any length. Few
// threads, two to four vectors each: the sums over lanes and the statistics cost a row's threads as
// much as some ten values each. (us in bf16, so and by one vector a thread: 500000 x 64 26 and 51,
// 250000 x 256 48 and 103, 131072 x 512 53 and 66, 32768 x 2048 51 and 62. Threads without values
// wait all the same: of three vectors and, as for the next longer rows, two or four 18678 x 2063 48
// and 58, 6000 x 9000 53 and 77, 100000 x 384 31 and 36. Four vectors against two: 16384 x 8192 107
// and 115, 4096 x 16384 70 and 72, but 16384 x 4096 54 and 51.)
template <int T_, int V_, int B_>
struct Shape {
  static constexpr int T = T_, V = V_, B = B_;
};
template <class F>
auto with_shape(int N, F f) {
  if (N <= 8) return f(Shape<1, 1, 256>{});
  if (N <= 16) return f(Shape<1, 2, 256>{});
  if (N <= 32) return f(Shape<1, 4, 256>{});
  if (N <= 64) return f(Shape<4, 2, 256>{});
  if (N <= 128) return f(Shape<4, 4, 256>{});
  if (N <= 256) return f(Shape<16, 2, 256>{});
  if (N <= 16 * 3 * 8) return f(Shape<16, 3, 256>{});
  if (N <= 512) return f(Shape<16, 4, 256>{});
  if (N <= 1024) return f(Shape<64, 2, 256>{});
  if (N <= 64 * 3 * 8) return f(Shape<64, 3, 256>{});
  if (N <= 2048) return f(Shape<64, 4, 256>{});
  if (N <= 128 * 3 * 8) return f(Shape<128, 3, 256>{});
  if (N <= 4096) return f(Shape<256, 2, 256>{});
  if (N <= 256 * 3 * 8) return f(Shape<256, 3, 256>{});
  if (N <= 8192) return f(Shape<256, 4, 256>{});
  if (N <= 512 * 3 * 8) return f(Shape<512, 3, 512>{});
  if (N <= 16384) return f(Shape<512, 4, 512>{});
  return f(Shape<0, 0, 0>{});
}
// Backward, where sums of the columns stay in registers too, and few strips leave few of them to
// add: large workgroups, one or two a compute unit. (With column sums in fp32 throughout: 16 x 128 x 512 in
// workgroups of 256 and two launches 19.4 us, of 1024 and one 13.7; in bf16 by two vectors a thread and by one 500000 x 64 44 and 50, 250000 x 256
// 81 and 92, 4 x 9777 x 1134 73 and 83; by three and by two or four 4 x 9777 x 1134 61 and 73, 18678 x
// 2063 60 and 80, 6000 x 9000 76 and 85; 4096 x 16384 by 1024 threads, which spill, 278, by 512 without
// a row ahead 98.)
constexpr int kHeld = 16384;  // columns of the longest
template <class F>
auto with_back_shape(int N, F f) {
  if (N <= 8) return f(Shape<1, 1, 256>{});
  if (N <= 32) return f(Shape<4, 1, 1024>{});
  if (N <= 64) return f(Shape<4, 2, 512>{});
  if (N <= 128) return f(Shape<16, 1, 1024>{});
  if (N <= 256) return f(Shape<16, 2, 512>{});
  if (N <= 512) return f(Shape<64, 1, 1024>{});
  if (N <= 1024) return f(Shape<64, 2, 512>{});
  if (N <= 64 * 3 * 8) return f(Shape<64, 3, 512>{});
  if (N <= 2048) return f(Shape<128, 2, 512>{});
  if (N <= 128 * 3 * 8) return f(Shape<128, 3, 512>{});
  if (N <= 4096) return f(Shape<256, 2, 512>{});
  if (N <= 256 * 3 * 8) return f(Shape<256, 3, 512>{});
  if (N <= 8192) return f(Shape<512, 2, 512>{});
  if (N <= 512 * 3 * 8) return f(Shape<512, 3, 512>{});
  if (N <= kHeld) return f(Shape<512, 4, 512>{});
  return f(Shape<0, 0, 0>{});
}
// Rows of a strip: about `strips` strips in all, of whole sets of `each` rows at work at one time.
int strip_rows(long long strips, int each, int G, int M) {
  strips = std::max(1LL, strips / G);
  const long long rows = (M + strips - 1) / strips;
  return (int)((rows + each - 1) / each * each);
}
// Four sets of rows a strip, for which w and b are read once; but five workgroups a compute unit, and
// no more than 4096. (us, of sets a strip: 16384 x 8192 in bf16 4 106, 8 109, 16 114; 32768 x 2048 2 52, 4 50,
// 8 51.5; 131072 x 512 1 58, 2 51, 4 49, 8 52; 4000 x 12000 in fp32 1 102, 2 86, 4 79, 8 80; 3000 x 3500 2 17.3,
// 3 16.5.) Of 512 threads 1024 strips (16384 x 16384 in 1024, 2048, 4096 strips 236, 243, 256).
int norm_strip_rows(int each, bool large, int G, int M) {
  const long long sets = ((long long)M + each - 1) / each * G;
  return strip_rows(large ? 1024 : std::min(4096LL, std::max(1280LL, sets / 4)), each, G, M);
}

template <bool XBF, bool YBF>
hipError_t norm(NormArgs a, hipStream_t s) {
  return with_shape(a.N, [&](auto z) {
    constexpr int T = decltype(z)::T, V = decltype(z)::V, B = decltype(z)::B;
    if constexpr (T == 0) {
      const long long total = (long long)a.G * a.M;
      if (total > 0x7fffffffLL) return hipErrorInvalidValue;
      hipLaunchKernelGGL((k_norm_long<XBF, YBF>), grid_of(total), dim3(kLong), 0, s, a, total);
    } else {
      a.strip = norm_strip_rows(B / T, B > 256, a.G, a.M);
      const int strips = (int)((a.M + (long long)a.strip - 1) / a.strip);
      const long long total = (long long)strips * a.G;
      hipLaunchKernelGGL((k_norm<XBF, YBF, T, V, B>), grid_of(total), dim3(B), 0, s, a, strips, total);
    }
    return hipGetLastError();
  });
}

// One strip, and no second launch, where each of a workgroup's places for rows gets few; else 256
// (16384 x 8192 in bf16 in 256, 512, 1024 strips 186, 194, 206 us, when the sums still went by LDS).
constexpr int kFewRows = 8, kFewSums = 32;
constexpr long long kBackStrips = 256, kNarrowStrips = 1024;
int back_strip_rows(int G, int M, int N) {
  return with_back_shape(N, [&](auto z) {
    constexpr int T = decltype(z)::T, B = decltype(z)::B;
    constexpr int each = T == 0 ? 4 : B / (T == 0 ? 1 : T);
    if (M <= kFewRows * each) return (M + each - 1) / each * each;
    const int rows = strip_rows(T == 1 ? kNarrowStrips : kBackStrips, each, G, M);
    return decltype(z)::V <= 2 ? rows : std::min(rows, kFewSums * each);
  });
}

template <bool XBF, bool YBF>
hipError_t norm_back(NormBackArgs a, void* ws, hipStream_t s) {
  a.strip = back_strip_rows(a.G, a.M, a.N);
  a.strips = (int)((a.M + (long long)a.strip - 1) / a.strip);
  a.part = (float*)ws;
  a.shift = (float*)ws + (a.strips == 1 ? 0 : (size_t)a.G * a.strips * 2 * a.N);
  const long long strips = (long long)a.strips * a.G;
  hipError_t e = with_back_shape(a.N, [&](auto z) {
    constexpr int T = decltype(z)::T, V = decltype(z)::V, B = decltype(z)::B;
    if constexpr (T == 0) {
      const long long total = (long long)a.G * a.M, tiles = (a.N + 511LL) / 512;
      if (total > 0x7fffffffLL || tiles * strips > 0x7fffffffLL) return hipErrorInvalidValue;
      hipLaunchKernelGGL((k_norm_back_long<XBF, YBF>), grid_of(total), dim3(kLong), 0, s, a, total);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess || !a.dw) return e;
      hipLaunchKernelGGL((k_norm_params<XBF, YBF>), grid_of(tiles * strips), dim3(kThreads), 0, s, a,
                         (int)tiles, tiles * strips);
    } else {
      typedef std::conditional_t<T == 1, double, float> A;
      hipLaunchKernelGGL((k_norm_back<XBF, YBF, T, V, B, A>), grid_of(strips), dim3(B), 0, s, a,
                         strips);
    }
    return hipGetLastError();
  });
  if (e != hipSuccess || !a.dw || a.strips == 1) return e;
  const long long tiles = (a.N + 63LL) / 64, total = tiles * 2 * a.G;
  if (total > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_norm_join, grid_of(total), dim3(kJoin), 0, s, a, (int)tiles, total);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(int x_bf16, int y_bf16, const NormArgs& a, hipStream_t s) {
  if (x_bf16) return y_bf16 ? norm<true, true>(a, s) : norm<true, false>(a, s);
  return y_bf16 ? norm<false, true>(a, s) : norm<false, false>(a, s);
}

size_t norm_back_workspace_bytes(int G, int M, int N) {
  const long long strip = back_strip_rows(G, M, N), strips = (M + strip - 1) / strip;
  const size_t sums = strips == 1 ? 0 : (size_t)G * strips * 2 * N;
  // (of rows past what registers hold: how far each is off its mean as it was written)
  return (sums + (N > kHeld ? (size_t)G * M : 0)) * sizeof(float);
}

hipError_t launch_norm_back(int x_bf16, int y_bf16, const NormBackArgs& a, void* ws, hipStream_t s) {
  if (x_bf16) return y_bf16 ? norm_back<true, true>(a, ws, s) : norm_back<true, false>(a, ws, s);
  return y_bf16 ? norm_back<false, true>(a, ws, s) : norm_back<false, false>(a, ws, s);
}

}  // namespace lsgd
