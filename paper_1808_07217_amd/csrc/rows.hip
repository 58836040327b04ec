// Tensors in 8-bit integers with an fp32 scale for each row, and the grouped product
// of two of them.
//
// A row's scale s is max |x| / 127, rounded to fp32, at least 2^-126 (then 1 / s and
// s / 2 are exact enough to work with), 1 for a row of zeros, and a NaN for a row that
// holds an infinity or a NaN, whose integers are zeros: every product that reads the
// row shows it. An element is the integer nearest to x / s, ties to even.
//
// Rows alone take one read of X, a row in registers meanwhile (16384 x 8192 in bf16 73 us, 5.5
// TB/s). A column's scale needs all rows first: both ways take two reads, the second in part from
// the last-level cache (137 us: the maxima 53, at 5.1 TB/s, the integers 86). The product is bound by the
// matrix cores where it is large (8192^3 to bf16 431 us, 2.55 POPS: busy in 60% of the cycles, at a clock
// of 1.95 of 2.4 GHz; operands of zeros, which leave the clock up, 339), by the weights' bytes
// for a token (1 x 8192 x 8192 14.0 us, 4.8 TB/s).
#include <algorithm>
#include <cmath>

#include "lanes.h"
#include "row_io.h"
#include "tile_loop.h"

namespace lsgd {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// vectors at any element's alignment
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kThreads = 256;
constexpr uint32_t kInf = 0x7f800000u;

// ---------------------------------------------------------------- quantise
// Magnitudes are compared as the bits of |x|: infinities and NaN are then the largest. Of
// bfloat16 two in a dword, of floats one.
template <bool BF>
struct Most8 {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  static constexpr uint32_t kMask = BF ? 0x7fff7fffu : 0x7fffffffu;
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (BF)
      return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                    __builtin_bit_cast(u16x2, b)));
    else
      return max(a, b);
  }
  // the magnitude in a dword's half (BF), as a float's bits
  static __device__ __forceinline__ uint32_t bits(uint32_t w, int half) {
    return BF ? (half ? w & 0xffff0000u : w << 16) : w;
  }
  static __device__ __forceinline__ uint32_t most(uint32_t w) {
    return BF ? max(bits(w, 0), bits(w, 1)) : w;
  }
};
// The largest magnitude of eight values, and each of them kept if larger than a column's.
template <bool BF, bool COLS>
__device__ __forceinline__ uint32_t most8(const Raw8<BF>& v, uint32_t (&cols)[Raw8<BF>::kDwords]) {
  typedef Most8<BF> L;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < Raw8<BF>::kDwords; ++i) {
    const uint32_t w = v.w[i] & L::kMask;
    top = L::larger(top, w);
    if constexpr (COLS) cols[i] = L::larger(cols[i], w);
  }
  return L::most(top);
}
__device__ __forceinline__ float scale_of(uint32_t most) {
  if (most == 0) return 1.f;
  if (most >= kInf) return __uint_as_float(0x7fc00000u);
  return fmaxf(__uint_as_float(most) / 127.f, 0x1p-126f);
}
// The integers nearest to v / s. x (1 / s) + 1.5 2^23 rounds to a float whose last byte is the
// integer. The product is off by less than 2^-15, so that it rounds to the wrong neighbour only
// next to the middle between two, and there the remainder x - q s, which is exact in fp32
// (|x| and s below 2^128, at most 24 bits between its first and last), is at least s / 2:
// then, rarely, the tie or the neighbour is settled. Zeros for a NaN in place of s.
__device__ __forceinline__ u32x2 pack8(const float (&v)[8], float s, float r) {
  constexpr float kShift = 12582912.f;
  float q[8], far = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    q[i] = __builtin_fmaf(v[i], r, kShift);
    far = fmaxf(far, fabsf(__builtin_fmaf(kShift - q[i], s, v[i])));
  }
  if (far >= 0.5f * s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float rest = __builtin_fmaf(kShift - q[i], s, v[i]);
      const bool odd = (__float_as_uint(q[i]) & 1) != 0;
      if (fabsf(rest) > 0.5f * s || (fabsf(rest) == 0.5f * s && odd)) q[i] += rest > 0.f ? 1.f : -1.f;
    }
  }
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(q[4 * h + 1]),
                                              __float_as_uint(q[4 * h]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(q[4 * h + 3]),
                                              __float_as_uint(q[4 * h + 2]), 0x0c0c0400u);
    w[h] = s == s ? lo | hi << 16 : 0u;
  }
  return w;
}
template <bool BF>
__device__ __forceinline__ u32x2 pack8(const Raw8<BF>& raw, float s, float r) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = raw[i];
  return pack8(v, s, r);
}

template <int T>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m) {
  return over_lanes<T>(m, [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return max(a, b); });
}

// Rows alone: T threads a row, V vectors of eight values each, all in registers, or
// (V == 0) in two passes of any length.
template <bool BF, int T, int V>
__global__ __launch_bounds__(T < kThreads ? kThreads : T) void k_rows(RowQuantArgs a,
                                                                      long long rows) {
  constexpr int kBlock = T < kThreads ? kThreads : T, kRows = kBlock / T, kWaves = kBlock / 64;
  constexpr bool kSmall = T == 16 && V == 1;
  __shared__ uint32_t most[T > 64 ? kWaves : 1];
  const int t = threadIdx.x % T;
  const long long row = (long long)workgroup_id() * kRows + threadIdx.x / T;
  if (T >= 64 && row >= rows) return;  // (whole wavefronts, and all of a row's)
  const long long g = row / a.M, m = row - g * a.M;
  const long long x = g * a.sX + m * a.ldx;
  const int vecs = (a.N + 127) / 128 * 16;  // of eight
  const bool in = row < rows;
  uint32_t top = 0, none[Raw8<BF>::kDwords];
  Raw8<BF> v[V ? V : 1];
  if constexpr (V > 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) fetch8<BF, kSmall>(a.X, x, (t + i * T) * 8, in ? a.N : 0, v[i]);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      settle8<BF, kSmall>((t + i * T) * 8, a.N, v[i]);
      top = max(top, most8<BF, false>(v[i], none));
    }
  } else {
    for (int k = t; k < vecs; k += T) {
      fetch8<BF>(a.X, x, k * 8, a.N, v[0]);
      settle8<BF>(k * 8, a.N, v[0]);
      top = max(top, most8<BF, false>(v[0], none));
    }
  }
  top = lanes_max<(T < 64 ? T : 64)>(top);
  if constexpr (T > 64) {
    if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = max(top, most[i]);
  }
  const float s = scale_of(top), r = 1.f / s;
  if (!in) return;
  u32x2* q = (u32x2*)(a.Q + row * (vecs * 8LL));
  if constexpr (V > 0) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (t + i * T < vecs) q[t + i * T] = pack8<BF>(v[i], s, r);
  } else {
    for (int k = t; k < vecs; k += T) {
      fetch8<BF>(a.X, x, k * 8, a.N, v[0]);
      settle8<BF>(k * 8, a.N, v[0]);
      q[k] = pack8<BF>(v[0], s, r);
    }
  }
  if (t == 0) a.S[row] = s;
}

// Both ways, in two launches: the largest magnitudes of strips of rows by 512 columns (of up to 128
// columns: by all of them), and from those and a second read of X the scales and the integers of 128 x
// 128 tiles, from the last tile to the first: what the first launch read last is in the last-level
// cache still.
constexpr int kMostThreads = 1024, kMostWaves = kMostThreads / 64;
constexpr int kMostRows = 8;  // of a lane in flight
constexpr int most_lanes(int N) { return N <= 128 ? 16 : 64; }  // a row

// L lanes a row, each eight columns; a wavefront's rows lie side by side, the wavefronts' after each
// other.
template <bool BF, bool SMALL, int L>
__global__ __launch_bounds__(kMostThreads) void k_rows_most(RowQuantArgs a, int tm, int tn,
                                                            int total) {
  typedef Most8<BF> Most;
  constexpr int kCols = 8 * L, kEach = 64 / L;  // rows of a wavefront at one time
  __shared__ uint32_t most[kMostWaves][kCols];
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int g = id / (tm * tn), mt = id % (tm * tn) / tn, nt = id % tn;
  const int lane = threadIdx.x % L, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = nt * kCols + lane * 8, m0 = mt * a.strip, end = min(a.M, m0 + a.strip);
  uint32_t cm[Raw8<BF>::kDwords] = {};
  for (int r = m0 + wave * kEach; r < end; r += kMostWaves * kEach * kMostRows) {
    const int m = L == 64 ? r : r + (threadIdx.x & 63) / L;
    Raw8<BF> v[kMostRows];
#pragma unroll
    for (int k = 0; k < kMostRows; ++k) {
      const int mk = m + k * kMostWaves * kEach;
      fetch8<BF, SMALL>(a.X, g * a.sX + mk * a.ldx, n, mk < end ? a.N : 0, v[k]);
    }
#pragma unroll
    for (int k = 0; k < kMostRows; ++k) {
      const int mk = m + k * kMostWaves * kEach;
      settle8<BF, SMALL>(n, a.N, v[k]);
      const uint32_t rm = lanes_max<L>(most8<BF, true>(v[k], cm));
      if (lane == 0 && mk < end) a.rowmost[((long long)g * tn + nt) * a.M + mk] = rm;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t c = Most::bits(cm[BF ? i / 2 : i], i % 2);
    if constexpr (L == 16)
      c = over_rows(c, [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return max(a, b); });
    if ((threadIdx.x & 63) < L) most[wave][lane * 8 + i] = c;
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c < kCols && nt * kCols + c < a.N) {
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < kMostWaves; ++w) top = max(top, most[w][c]);
    a.colmost[((long long)g * tm + mt) * a.N + nt * kCols + c] = top;
  }
}

// Rows of 128 bytes; piece k of 16 lies in slot k ^ (row / 8 % 8), which spreads the rows,
// eight apart, that a wavefront writes at once over the banks. (The integers of 16384 x 8192 move 537
// MB in 86 us; values past the caches from kNtBytesCaller on, as in blocks.hip.)
__device__ __forceinline__ int turned(int row, int byte) {
  return row * 128 + (byte ^ (row / 8 % 8 * 16));
}
// A tile of 128 x 128: thread t holds eight rows from 8 (t / 16) and eight columns from
// 8 (t % 16); the transpose's bytes are turned in LDS, so that each of its rows leaves
// as a whole line. Thread t < 128 finds the scale of the tile's row t, the others a column's,
// from the strips' maxima; ONE: matrices of a single tile, from its own.
template <bool BF, bool SMALL, bool STREAM, bool ONE>
__global__ __launch_bounds__(kThreads) void k_rows_both(RowQuantArgs a, int tm, int tn, int sm,
                                                        int sn, int total) {
  __shared__ __align__(16) uint8_t turn[128 * 128];
  __shared__ __align__(16) float scale[256], inverse[256];
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  const int l = total - 1 - (int)id;
  const int g = l / (tm * tn), mt = l % (tm * tn) / tn, nt = l % tn;
  const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4;
  const int n0 = nt * 128, m0 = mt * 128, n = n0 + c * 8, r0 = m0 + rg * 8;
  // the strips' maxima first: the scales are found while X is on its way
  constexpr int kAhead = 16;
  const bool row = tid < 128;
  const int at = row ? m0 + tid : n0 + tid - 128, each = row ? a.M : a.N, parts = row ? sn : sm;
  uint32_t tops[kAhead], top = 0;
  auto larger = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) top = max(top, tops[k]);
  };
  if constexpr (!ONE) {
    const uint32_t* part = (row ? a.rowmost : a.colmost) + (long long)g * parts * each + at;
    auto ahead = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        tops[k] = 0;
        if (k0 + k < parts && at < each) tops[k] = part[(long long)(k0 + k) * each];
      }
    };
    ahead(0);
    for (int k0 = kAhead; k0 < parts; k0 += kAhead) {
      larger();
      ahead(k0);
    }
  }
  Raw8<BF> v[8];
#pragma unroll
  for (int p = 0; p < 8; ++p)
    fetch8<BF, SMALL>(a.X, g * a.sX + (r0 + p) * a.ldx, n, r0 + p < a.M ? a.N : 0, v[p]);
#pragma unroll
  for (int p = 0; p < 8; ++p) settle8<BF, SMALL>(n, a.N, v[p]);
  if constexpr (ONE) {
    __shared__ uint32_t rows[128], cols[4][128];
    uint32_t cm[Raw8<BF>::kDwords] = {};
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const uint32_t m = lanes_max<16>(most8<BF, true>(v[p], cm));
      if (c == 0) rows[rg * 8 + p] = m;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = over_rows(Most8<BF>::bits(cm[BF ? i / 2 : i], i % 2),
                                   [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return max(a, b); });
      if ((tid & 63) < 16) cols[tid >> 6][c * 8 + i] = m;
    }
    __syncthreads();
    const int k = tid & 127;
    top = row ? rows[k] : max(max(cols[0][k], cols[1][k]), max(cols[2][k], cols[3][k]));
  } else {
    larger();
  }
  {
    const float s = scale_of(top);
    scale[tid] = s;
    inverse[tid] = 1.f / s;
    if (at < each && (row ? nt : mt) == 0) (row ? a.S : a.St)[(long long)g * each + at] = s;
  }
  __syncthreads();
  auto put = [&](auto value, auto* to) __attribute__((always_inline)) {
    if constexpr (STREAM)
      __builtin_nontemporal_store(value, to);
    else
      *to = value;
  };
  const long long ldq = (a.N + 127) / 128 * 128, ldt = (a.M + 127) / 128 * 128;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    if (r0 + p >= a.M) continue;
    const long long to = (long long)g * a.M + r0 + p;
    put(pack8<BF>(v[p], scale[rg * 8 + p], inverse[rg * 8 + p]), (u32x2*)(a.Q + to * ldq + n));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float w[8] = {v[0][i], v[1][i], v[2][i], v[3][i], v[4][i], v[5][i], v[6][i], v[7][i]};
    *(u32x2*)(turn + turned(c * 8 + i, rg * 8)) =
        pack8(w, scale[128 + c * 8 + i], inverse[128 + c * 8 + i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = i * kThreads + tid, j = at >> 3, k = (at & 7) * 16;
    if (n0 + j < a.N)
      put(*(const u32x4*)(turn + turned(j, k)),
          (u32x4*)(a.Qt + ((long long)g * a.N + n0 + j) * ldt + m0 + k));
  }
}

// Rows of a strip, whole sets of what a workgroup has in flight: few strips leave few column
// maxima to read again, and a workgroup a compute unit is enough where all start at once.
// (16384 x 8192 in bf16, in 256, 512, 1024 strips: both launches 139, 163, 203 us.)
int strip_rows(int G, int M, int N) {
  const int L = most_lanes(N), set = kMostWaves * kMostRows * (64 / L);
  const long long across = ((long long)N + 8 * L - 1) / (8 * L) * G;
  const long long strips = (across <= 64 ? 256 + across - 1 : 1024 + across - 1) / across;
  const long long rows = ((M + strips - 1) / strips + set - 1) / set * set;
  return (int)rows;
}

bool one_tile(int M, int N) { return M <= 128 && N <= 128; }

template <bool BF, bool SMALL, bool STREAM>
hipError_t quantise_both(RowQuantArgs a, void* ws, hipStream_t s) {
  a.strip = strip_rows(a.G, a.M, a.N);
  const long long tm = ((long long)a.M + a.strip - 1) / a.strip;
  const int L = most_lanes(a.N);
  const long long tn = (a.N + 8LL * L - 1) / (8 * L);
  const long long bm = (a.M + 127LL) / 128, bn = (a.N + 127LL) / 128;
  if (one_tile(a.M, a.N)) {
    if constexpr (!STREAM)
      hipLaunchKernelGGL((k_rows_both<BF, SMALL, false, true>), dim3(a.G), dim3(kThreads), 0, s, a, 1,
                         1, 0, 0, a.G);
    return hipGetLastError();
  }
  if (bm * bn > 0x7fffffffLL / a.G) return hipErrorInvalidValue;
  a.rowmost = (uint32_t*)ws;
  a.colmost = a.rowmost + a.G * tn * a.M;
  if (L == 16) {
    hipLaunchKernelGGL((k_rows_most<BF, SMALL, 16>), grid_of(tm * tn * a.G), dim3(kMostThreads), 0, s,
                       a, (int)tm, (int)tn, (int)(tm * tn * a.G));
  } else if constexpr (!SMALL) {
    hipLaunchKernelGGL((k_rows_most<BF, false, 64>), grid_of(tm * tn * a.G), dim3(kMostThreads), 0, s,
                       a, (int)tm, (int)tn, (int)(tm * tn * a.G));
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_rows_both<BF, SMALL, STREAM, false>), grid_of(bm * bn * a.G), dim3(kThreads), 0, s,
                     a, (int)bm, (int)bn, (int)tm, (int)tn, (int)(bm * bn * a.G));
  return hipGetLastError();
}

template <bool BF>
hipError_t quantise(const RowQuantArgs& a, void* ws, hipStream_t s) {
  if (a.Qt) {
    const double bytes = (double)a.M * a.N * a.G * ((BF ? 2 : 4) + 2);
    if (bytes >= (double)kNtBytesCaller && !one_tile(a.M, a.N))
      return a.N < 8 ? quantise_both<BF, true, true>(a, ws, s) : quantise_both<BF, false, true>(a, ws, s);
    return a.N < 8 ? quantise_both<BF, true, false>(a, ws, s) : quantise_both<BF, false, false>(a, ws, s);
  }
  const long long rows = (long long)a.G * a.M;
  auto launch = [&](auto kernel, int per, int threads) {
    const long long n = (rows + per - 1) / per;
    if (n > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, grid_of(n), dim3(threads), 0, s, a, rows);
    return hipGetLastError();
  };
  // (us in bf16 by 16 threads a row and by 64: 250000 x 256 34 and 61, 131072 x 512 34 and 40; by three or six
  // vectors a thread and by twice the threads or by four: 18678 x 2063 21 and 26, 6000 x 9000 27 and 37)
  if (a.N <= 128) return launch(k_rows<BF, 16, 1>, 16, 256);
  if (a.N <= 256) return launch(k_rows<BF, 16, 2>, 16, 256);
  if (a.N <= 512) return launch(k_rows<BF, 16, 4>, 16, 256);
  if (a.N <= 1024) return launch(k_rows<BF, 64, 2>, 4, 256);
  if (a.N <= 64 * 3 * 8) return launch(k_rows<BF, 64, 3>, 4, 256);
  if (a.N <= 2048) return launch(k_rows<BF, 64, 4>, 4, 256);
  if (a.N <= 64 * 6 * 8) return launch(k_rows<BF, 64, 6>, 4, 256);
  if (a.N <= 4096) return launch(k_rows<BF, 256, 2>, 1, 256);
  if (a.N <= 256 * 3 * 8) return launch(k_rows<BF, 256, 3>, 1, 256);
  if (a.N <= 8192) return launch(k_rows<BF, 256, 4>, 1, 256);
  if (a.N <= 512 * 3 * 8) return launch(k_rows<BF, 512, 3>, 1, 512);
  if (a.N <= 16384) return launch(k_rows<BF, 1024, 2>, 1, 1024);
  return launch(k_rows<BF, 1024, 0>, 1, 1024);
}

// ------------------------------------------------------------------ product
// v_mfma_i32_16x16x64_i8 twice a step of 128 (32 x 32 blocks leave fewer places between their
// instructions for the next step's reads: 8192^3 463 us): exact sums in 32 bits. |q| <= 128, so a sum of
// 2^17 - 1 products fits; a longer inner dimension is cut into ranges whose sums are joined in
// 64 bits. Lane l holds 16 of a step half's 64 k for row l % 16, the same ones of both operands. The
// first operand is B's rows, so that a lane's four results are neighbours in a row of C.
constexpr int kMostSteps = 1020;  // of 128: below 2^17, a multiple of four

struct MacRows {
  struct Next {};
  typedef Frag P;
  typedef Frag Q;
  typedef v4i Acc;
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
  __device__ __forceinline__ void mac(v4i& c, const P& p, int, const Q& q, int) const {
    c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_shufflevector(p, p, 0, 1, 2, 3),
                                              __builtin_shufflevector(q, q, 0, 1, 2, 3), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_shufflevector(p, p, 4, 5, 6, 7),
                                              __builtin_shufflevector(q, q, 4, 5, 6, 7), c, 0, 0, 0);
  }
};

// sum sa sb + bias. The smaller scale comes first: a sum of integers times it stays in
// range wherever the result does. (Both scales are taken once, a NaN among them too.)
__device__ __forceinline__ float scaled(float sum, float sa, float sb, float bias) {
  const float lo = sa < sb ? sa : sb, hi = sa < sb ? sb : sa;
  return __builtin_fmaf(sum * lo, hi, bias);
}

// Eight neighbours of a row of C from LDS (`second`: from the fifth on), n of them.
template <int SIZE>
__device__ __forceinline__ void copy8(void* C, long long at, const uint8_t* from,
                                      const uint8_t* second, int n) {
  if constexpr (SIZE == 2) {
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
      *(v4f_any*)(c + 4) = *(const v4f*)second;
    } else {
      for (int e = 0; e < n; ++e) c[e] = ((const float*)(e < 4 ? from : second))[e % 4];
    }
  }
}

enum { kOutFp32 = 0, kOutBf16 = 1, kOutSums = 2 };

// Tiles of C by way of LDS, so that whole rows of a tile leave at once: a group of each
// wavefront's columns at a time, half of their rows in each of two stages. Piece k of 16 bytes of
// row r lies in slot k ^ (r % 16) (or as many as a row has), which spreads the rows that a wavefront
// writes at once over the banks.
// `ends`: the scales of B's rows, their biases, the scales of A's rows.
template <int OUT, int THREADS, class T>
__device__ __forceinline__ void tile_out(const T& t, const v4i (&acc)[T::FP][T::FQ],
                                         const float* ends, uint8_t* s0, uint8_t* s1, void* C,
                                         long long row0, long long ldc, int np, int nq) {
  constexpr int kSize = OUT == kOutBf16 ? 2 : 4, kPitch = T::kP * kSize;
  constexpr int kSpread = (kPitch < 256 ? kPitch : 256) - 16;
  constexpr int kAcross = T::kQ / (T::FQ * 16);  // wavefronts along A's rows
  constexpr int kFit = T::kStage / kPitch * 2 / (kAcross * 16);
  constexpr int kGroup = kFit >= T::FQ ? T::FQ : (kFit >= 2 ? 2 : 1);  // columns of blocks at a time
  constexpr int kRows = kAcross * kGroup * 16, kHalf = kRows / 2;
  static_assert(kHalf * kPitch <= T::kStage && T::FQ % kGroup == 0, "half a group fits a stage");
  auto at = [&](int r, int p) __attribute__((always_inline)) {
    return (r < kHalf ? s0 : s1) + r % kHalf * kPitch + (p * kSize ^ (r * 16 & kSpread));
  };
  const int lane = t.lane, p0 = t.wp + (lane >> 4) * 4, side = t.wq / (T::FQ * 16);
#pragma unroll
  for (int j0 = 0; j0 < T::FQ; j0 += kGroup) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int j = j0; j < j0 + kGroup; ++j) {
      const float sa = ends[2 * T::kP + t.wq + j * 16 + (lane & 15)];
#pragma unroll
      for (int i = 0; i < T::FP; ++i) {
        uint8_t* to = at((side * kGroup + j - j0) * 16 + (lane & 15), p0 + i * 16);
        const v4i v = acc[i][j];
        if constexpr (OUT == kOutSums) {
          *(v4i*)to = v;
        } else {
          const v4f sb = *(const v4f*)(ends + p0 + i * 16);
          const v4f b = *(const v4f*)(ends + T::kP + p0 + i * 16);
          v4f f;
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = scaled((float)v[e], sa, sb[e], b[e]);
          if constexpr (OUT == kOutBf16)
            *(u32x2*)to = u32x2{f32_to_bf16(f[0]) | (uint32_t)f32_to_bf16(f[1]) << 16,
                                f32_to_bf16(f[2]) | (uint32_t)f32_to_bf16(f[3]) << 16};
          else
            *(v4f*)to = f;
        }
      }
    }
    __syncthreads();
#pragma unroll 2
    for (int u = threadIdx.x; u < T::kP * kRows / 8; u += THREADS) {
      const int r = u / (T::kP / 8), p = u % (T::kP / 8) * 8;
      const int q = r / (kGroup * 16) * T::FQ * 16 + j0 * 16 + r % (kGroup * 16);
      if (q < nq && p < np) copy8<kSize>(C, row0 + (long long)q * ldc + p, at(r, p), at(r, p + 4), np - p);
    }
  }
}

// The tile of BP rows of B and BQ rows of A, over one of `splits` ranges of the inner
// dimension (chunk steps each); OUT == kOutSums: a range's sums go to `part`.
template <int OUT, int BP, int BQ, int WP, int WQ, int S>
__global__ __launch_bounds__((64 * (BP / WP) * (BQ / WQ)), 2) void k_rows_tile(RowGemmArgs a, int tp,
                                                                               int tq, int total) {
  using T = TileLoop<BP, BQ, WP, WQ, S>;
  LSGD_TILE_STAGES(st, S, T::kStage);
  __shared__ __align__(16) float ends[2 * BP + BQ];
  const unsigned id = workgroup_id();
  if (id >= (unsigned)total) return;
  int l = xcd_order(id, total);
  const int sg = l / (tp * tq), g = sg % a.G, split = sg / a.G;
  int pt, qt;
  band_order(l % (tp * tq), tp, tq, pt, qt);
  const int p0 = pt * BP, q0 = qt * BQ;
  const int nb = (a.Kd + 127) / 128, ld = nb * 128;
  const int k0 = split * a.chunk, steps = min(a.chunk, nb - k0);
  T t;
  t.init(a.B + (long long)g * a.sB + (long long)p0 * ld, a.A + (long long)g * a.sA + (long long)q0 * ld,
         ld, a.N - p0, a.M - q0);
  t.skip(k0);
  if constexpr (OUT != kOutSums) {
    // scales and biases straight to LDS, ahead of the tiles (loads return in order); zeros
    // past the last row, and for no bias
    constexpr int kParts = (2 * BP + BQ) / 64;
#pragma unroll
    for (int i = 0; i < (kParts + T::kWaves - 1) / T::kWaves; ++i) {
      const int part = t.wave + i * T::kWaves;
      if (part < kParts) {
        const int at = part * 64;
        const float* from = at < BP ? a.SB + g * a.sSB + p0
                                    : (at < 2 * BP ? a.bias + g * a.sbias + p0 : a.SA + g * a.sSA + q0);
        const int skip = at < BP ? at : (at < 2 * BP ? at - BP : at - 2 * BP);
        int left = (at < 2 * BP ? min(a.N - p0, BP) : min(a.M - q0, BQ)) - skip;
        if (at >= BP && at < 2 * BP && !a.bias) left = 0;
        const __amdgpu_buffer_rsrc_t b = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(from + skip), 0, max(left, 0) * 4, kRsrcRaw);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            b, (__attribute__((address_space(3))) void*)(ends + at), 4, t.lane * 4, 0, 0, 0);
      }
    }
  }
  MacRows mac;
  v4i acc[T::FP][T::FQ] = {};
  t.run(st, steps, mac, acc);
  if constexpr (OUT == kOutSums)
    tile_out<OUT, T::kThreads>(t, acc, ends, st[0], st[1], a.part,
                               ((long long)sg * a.M + q0) * a.N + p0, a.N, a.N - p0, a.M - q0);
  else
    tile_out<OUT, T::kThreads>(t, acc, ends, st[0], st[1], a.C,
                               (long long)g * a.sC + (long long)q0 * a.ldc + p0, a.ldc, a.N - p0,
                               a.M - q0);
}

// C = the ranges' sums, four neighbours by P lanes that take every P-th range each, four of them on
// their way at a time (one after the other 64 ranges took 31 us): integers add up to the same bits
// in any order.
template <bool OUTBF, int P>
__global__ __launch_bounds__(kThreads) void k_rows_join(RowGemmArgs a, int quads, long long total) {
  const long long i = ((long long)workgroup_id() * kThreads + threadIdx.x) / P;
  if (i >= total) return;
  const long long row = i / quads, g = row / a.M, m = row - g * a.M;
  const int n = (int)(i - row * quads) * 4, left = min(4, a.N - n);
  const long long each = (long long)a.G * a.M * a.N;
  const int* p = (const int*)a.part + row * a.N + n;
  constexpr int kAhead = 4;
  long long sum[4] = {};
  for (int s = threadIdx.x % P; s < a.splits; s += kAhead * P) {
    int v[kAhead][4];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[u][e] = p[min(s + u * P, a.splits - 1) * each + min(e, left - 1)];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += s + u * P < a.splits ? v[u][e] : 0;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] = lanes_sum<P>(sum[e]);
  if (threadIdx.x % P) return;
  const float sa = a.SA[g * a.sSA + m];
  const long long at = g * a.sC + m * a.ldc + n;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e >= left) break;
    const float f = scaled((float)sum[e], sa, a.SB[g * a.sSB + n + e],
                           a.bias ? a.bias[g * a.sbias + n + e] : 0.f);
    if constexpr (OUTBF)
      ((bf16_t*)a.C)[at + e] = f32_to_bf16(f);
    else
      ((float*)a.C)[at + e] = f;
  }
}

// ------------------------------------------------------------------ launches
constexpr int kCus = 256;
long long tiles_of(int G, int M, int N, long long b) {
  return (N + b - 1) / b * ((M + b - 1) / b) * G;
}

// The tile, its stages, and the ranges of the inner dimension, by estimated time in us: a workgroup
// alone on its unit takes 0.18 a step, all of them together cannot beat 5 TB/s, and a
// second launch joins the ranges' sums (4, and their bytes); 64 x 64 tiles are split where they leave
// units idle. Whole products by the rounds of the 256 compute units and a tile's relative time, from
// (us, to bf16, tiles of 64, 128 with four stages and with two, 256) 4096^3 99 / 80 / 68 / 58,
// 2048 x 2048 x 8192 50 / 36 / 48 / 82, 8192 x 1024 x 1024 23 / 18 / 16 / 22, 16 x 128 x 512 x 512
// 10.8 / 11.0 / 10.8 / 14.1. Where the inner dimension is so long that 64 x 64 tiles, two a unit, take
// 0.45 a step, tiles of 128 in ranges, which take 0.7, can be faster: 1024 x 1024 x 65536 141 -> 93.
struct RowCut {
  int tile, stages, splits, chunk;
};
RowCut row_cut(int G, int M, int N, int Kd) {
  const int nb = (Kd + 127) / 128;
  RowCut c{0, 0, 1, nb};
  const long long tiles = tiles_of(G, M, N, 64), large = tiles_of(G, M, N, 128);
  const double bytes = (double)G * ((double)M + N) * nb * 128 / 5e6;
  const double sums = 2.0 * G * M * N * sizeof(int) / 4e6;
  auto joined = [&](int s) { return s > 1 ? 4 + sums * s : 0.0; };
  double least = std::max(0.18 * nb, bytes);
  for (int s = 2; s <= 64 && tiles * s <= 2 * kCus && nb >= 4 * s; s *= 2) {
    const double t = std::max(0.18 * nb / s, bytes) + joined(s);
    if (t < least) {
      c.splits = s;
      least = t;
    }
  }
  int wide = 0;  // ranges of tiles of 128
  least = 0.9 * (nb * (tiles * c.splits > kCus ? 0.45 : 0.25) / c.splits + joined(c.splits));
  for (int s = 2; s <= 64 && large * s <= kCus && nb >= 64 * s && tiles * c.splits <= 2 * kCus; s *= 2) {
    const double t = 0.7 * nb / s + joined(s);
    if (t < least) {
      wide = s;
      least = t;
    }
  }
  const bool few = c.splits > 1;
  c.splits = std::max(wide ? wide : c.splits, (nb + kMostSteps - 1) / kMostSteps);
  c.chunk = (nb + c.splits - 1) / c.splits;
  c.splits = (nb + c.chunk - 1) / c.chunk;
  const RowCut cuts[4] = {{64, 4}, {128, 4}, {128, 2}, {256, 2}};
  const int per_cu[4] = {2, 1, 2, 1};
  const double each[4] = {1.6, 4.5, 3.8, 12.6};
  int at = wide ? 1 : 0;
  for (int i = 0; i < (few || wide ? 0 : 4); ++i) {
    const double rounds = std::ceil((double)tiles_of(G, M, N, cuts[i].tile) * c.splits /
                                    (kCus * per_cu[i]));
    const double t = rounds * per_cu[i] * each[i];
    if (i == 0 || t < least) {
      at = i;
      least = t;
    }
  }
  c.tile = cuts[at].tile;
  c.stages = cuts[at].stages;
  return c;
}

template <int OUT, int B, int W, int S>
hipError_t launch_tile(const RowGemmArgs& a, hipStream_t s) {
  constexpr int WP = B == 256 ? 128 : B / 2;
  const long long tp = (a.N + B - 1LL) / B, tq = (a.M + B - 1LL) / B;
  if (tp * tq > 0x7fffffffLL / a.G / a.splits) return hipErrorInvalidValue;
  const long long total = tp * tq * a.G * a.splits;
  hipLaunchKernelGGL((k_rows_tile<OUT, B, B, WP, W, S>), grid_of(total),
                     dim3(64 * (B / WP) * (B / W)), 0, s, a, (int)tp, (int)tq, (int)total);
  return hipGetLastError();
}
template <int OUT>
hipError_t gemm_tiles(const RowGemmArgs& a, const RowCut& c, hipStream_t s) {
  if (c.tile == 64) return launch_tile<OUT, 64, 32, 4>(a, s);
  if (c.tile == 128 && c.stages == 4) return launch_tile<OUT, 128, 32, 4>(a, s);
  if (c.tile == 128) return launch_tile<OUT, 128, 64, 2>(a, s);
  return launch_tile<OUT, 256, 64, 2>(a, s);
}

}  // namespace

size_t rows_quantise_workspace_bytes(int G, int M, int N) {
  if (one_tile(M, N)) return 0;
  const size_t strip = strip_rows(G, M, N), tm = ((size_t)M + strip - 1) / strip;
  const size_t L = most_lanes(N), tn = (N + 8 * L - 1) / (8 * L);
  return ((size_t)G * tn * M + (size_t)G * tm * N) * sizeof(uint32_t);
}

hipError_t launch_quantise_rows(int bf16, const RowQuantArgs& a, void* ws, hipStream_t s) {
  return bf16 ? quantise<true>(a, ws, s) : quantise<false>(a, ws, s);
}

size_t gemm_rows_workspace_bytes(int G, int M, int N, int Kd) {
  const RowCut c = row_cut(G, M, N, Kd);
  return c.splits == 1 ? 0 : (size_t)c.splits * G * M * N * sizeof(int);
}

void gemm_rows_cut(int G, int M, int N, int Kd, int cut[3]) {
  const RowCut c = row_cut(G, M, N, Kd);
  cut[0] = c.tile;
  cut[1] = c.stages;
  cut[2] = c.splits;
}

hipError_t launch_gemm_rows(RowGemmArgs a, hipStream_t s) {
  const RowCut c = row_cut(a.G, a.M, a.N, a.Kd);
  a.splits = c.splits;
  a.chunk = c.chunk;
  if (a.splits == 1)
    return a.out_bf16 ? gemm_tiles<kOutBf16>(a, c, s) : gemm_tiles<kOutFp32>(a, c, s);
  const hipError_t e = gemm_tiles<kOutSums>(a, c, s);
  if (e != hipSuccess) return e;
  const int quads = (a.N + 3) / 4;
  const long long total = (long long)a.G * a.M * quads;
  auto join = [&](auto p) {
    constexpr int P = decltype(p)::value;
    const long long groups = (total * P + kThreads - 1) / kThreads;
    if (groups > 0x7fffffffLL) return hipErrorInvalidValue;
    if (a.out_bf16)
      hipLaunchKernelGGL((k_rows_join<true, P>), grid_of(groups), dim3(kThreads), 0, s, a, quads, total);
    else
      hipLaunchKernelGGL((k_rows_join<false, P>), grid_of(groups), dim3(kThreads), 0, s, a, quads, total);
    return hipGetLastError();
  };
  // by four lanes where there are few (us by one and by four: 3 x 18 x 60 of 31 ranges 9.6 and 4.7,
  // 300 x 301 of 8 5.4 and 4.4, 700 x 512 of 4 5.0 and 5.3, 1024 x 1024 of 4 8.4 and 12.1)
  return total <= 65536 ? join(std::integral_constant<int, 4>{}) : join(std::integral_constant<int, 1>{});
}

}  // namespace lsgd
