// The norm of each replica's gradients over all its tensors, and clipping by it.
//
// norm[k]^2 = sum of x^2 over the tensors of replica k, squared and added in fp64: nothing
// overflows or vanishes, and the order of the additions is the cut's alone. Each
// replica's values, tensor after tensor, are cut into chunks, a workgroup each; a second
// launch adds a replica's sums and, where the norm is above the bound, multiplies its
// chunks by bound / norm in fp64, one rounding a value.
//
// Bound by HBM: two reads and a write (2 x 402M values in fp32 1810 us, 5.3 TB/s; the fp64 products
// cost 1%). What the caches hold is read once (16 x 530K values, 34 MB: 8.0 and 11.1 us).
#include <algorithm>
#include <cmath>

#include "device_common.h"
#include "lanes.h"
#include "row_io.h"

namespace lsgd {
namespace {

constexpr int kThreads = 256;
// Tensors a launch takes, by value: 64 of them are 3 KB of its arguments.
constexpr int kBatch = 64;
struct ClipArgs {
  ClipTensor t[kBatch];
  int count, chunks, base, all;  // of the launch; before it; of all launches (a replica's)
  long long each;                // values a chunk
  double most;
  double* part;                  // [K][all]
  double* wide;                  // [K]: the norms; nullptr: found by who needs them
  float* norm;
};

// The sum over a workgroup's WAVES wavefronts, in a fixed order, in every thread.
template <int WAVES>
__device__ __forceinline__ double block_sum(double v, double (&room)[WAVES]) {
  v = lanes_sum<64>(v);
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
  __syncthreads();
  v = room[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v += room[w];
  return v;
}

// Whether a replica's values lie side by side; else its rows are taken in eights, the last of a row
// not whole.
__host__ __device__ inline bool flat(const ClipTensor& t) { return t.M == 1 || t.ld == t.N; }
__host__ __device__ inline long long eights_values(const ClipTensor& t) {
  return flat(t) ? t.M * t.N : t.M * ((t.N + 7) / 8) * 8;
}

// The bits of a value of bfloat16 or fp32 nearest to p. (By way of a float p would be rounded to
// bfloat16 twice; the compiler makes one of it, but need not.)
template <bool BF>
__device__ __forceinline__ uint32_t nearest(double p) {
  if constexpr (BF)
    return __builtin_bit_cast(bf16_t, (__bf16)p);
  else
    return __float_as_uint((float)p);
}

// The values of a chunk of one replica's tensor as T threads take them, `tid` of them this
// one: eights, U of a thread in flight. run(f): f(value) for every one, from a set that start() has on
// its way (of values side by side); WRITE: the value becomes f's (a double), rounded once.
constexpr int kFlight = 4;
template <bool BF, int T>
struct Chunk {
  static constexpr int U = kFlight;
  const ClipTensor& t;
  long long x, e0;  // the replica's first value; the chunk's first, of the replica's
  int values, tid;
  Raw8<BF> v[U];
  __device__ __forceinline__ Chunk(const ClipTensor& t, long long k, long long c, long long each,
                                   int tid)
      : t(t), x(k * t.s), e0(c * each), tid(tid) {
    values = (int)min(eights_values(t) - e0, each);
  }
  __device__ __forceinline__ void fetch(int e) {
    const int whole = values / 8 * 8;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (e + u * T * 8 < whole) fetch8<BF>(t.p, x + e0 + e + u * T * 8, 0, 8, v[u]);
  }
  __device__ __forceinline__ void start() {
    if (flat(t)) fetch(tid * 8);
  }
  template <bool WRITE, class F>
  __device__ __forceinline__ void eight(int u, long long row, int n, int N, F f) {
    if constexpr (WRITE) {
      Raw8<BF> w;
#pragma unroll
      for (int i = 0; i < Raw8<BF>::kDwords; ++i) {
        if constexpr (BF)
          w.w[i] = nearest<BF>(f(v[u][2 * i])) | nearest<BF>(f(v[u][2 * i + 1])) << 16;
        else
          w.w[i] = nearest<BF>(f(v[u][i]));
      }
      store8<BF>(t.p, row, n, N, w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f(v[u][i]);
    }
  }
  template <bool WRITE, class F>
  __device__ __forceinline__ void run(F f) {
    if (flat(t)) {
      const int whole = values / 8 * 8;
      for (int e = tid * 8; e < whole; e += T * 8 * U) {
        if (e != tid * 8) fetch(e);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (e + u * T * 8 < whole) eight<WRITE>(u, x + e0 + e + u * T * 8, 0, 8, f);
      }
      if (tid < values - whole) {
        const long long at = x + e0 + whole + tid;
        const float x = BF ? bf16_to_f32(((const bf16_t*)t.p)[at]) : ((const float*)t.p)[at];
        if constexpr (!WRITE)
          f(x);
        else if constexpr (BF)
          ((bf16_t*)t.p)[at] = (bf16_t)nearest<BF>(f(x));
        else
          ((uint32_t*)t.p)[at] = nearest<BF>(f(x));
      }
    } else {
      // (zeros past a row's last value add nothing to a sum)
      const int N = (int)t.N, across = (N + 7) / 8, dm = T / across, dj = T - dm * across;
      const long long first = e0 / 8 + tid;
      long long m = first / across;
      int j = (int)(first - m * across);
      for (int e = tid * 8; e < values;) {
        constexpr int W = 2;  // (in flight: four take the registers of every fourth workgroup)
        long long row[W];
        int n[W];
#pragma unroll
        for (int u = 0; u < W; ++u) {
          row[u] = x + m * t.ld;
          n[u] = e < values ? j * 8 : N;
          fetch8<BF, true>(t.p, row[u], n[u], N, v[u]);
          e += T * 8;
          m += dm;
          j += dj;
          if (j >= across) {
            j -= across;
            ++m;
          }
        }
#pragma unroll
        for (int u = 0; u < W; ++u) {
          settle8<BF, true>(n[u], N, v[u]);
          if (n[u] < N) eight<WRITE>(u, row[u], n[u], N, f);
        }
      }
    }
  }
};
// Which of the launch's tensors holds a replica's chunk c: one comparison a lane.
__device__ __forceinline__ int tensor_of(const ClipArgs& a, int c) {
  static_assert(kBatch == 64, "a tensor a lane");
  const int lane = threadIdx.x & 63;
  const bool starts = lane < a.count && a.t[lane].first <= c;
  return __popcll(__ballot(starts)) - 1;
}
// body(chunk) for the chunk c of replica k.
template <int T, class B>
__device__ __forceinline__ void with_chunk(const ClipArgs& a, int k, int c, int tid, B body) {
  const ClipTensor& t = a.t[tensor_of(a, c)];
  if (t.bf16) {
    Chunk<true, T> chunk(t, k, c - t.first, a.each, tid);
    body(chunk);
  } else {
    Chunk<false, T> chunk(t, k, c - t.first, a.each, tid);
    body(chunk);
  }
}
struct Squares {
  double sum = 0.0;
  __device__ __forceinline__ void operator()(float v) {
    sum = __builtin_fma((double)v, (double)v, sum);
  }
};
template <class C>
__device__ __forceinline__ double squares_of(C& chunk) {
  Squares q;
  chunk.start();
  chunk.template run<false>([&](float v) __attribute__((always_inline)) { q(v); });
  return q.sum;
}

__global__ __launch_bounds__(kThreads) void k_clip_sums(ClipArgs a, long long total) {
  __shared__ double room[kThreads / 64];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int k = id / a.chunks, c = id - k * a.chunks;
  double sum = 0.0;
  with_chunk<kThreads>(a, k, c, threadIdx.x, [&](auto& chunk) { sum = squares_of(chunk); });
  sum = block_sum(sum, room);
  if (threadIdx.x == 0) a.part[(long long)k * a.all + a.base + c] = sum;
}

// Few values: a workgroup a replica, a chunk a wavefront, all in one launch (4 x 650 values 3.7 us, the
// call 8.6; in two launches 15.3).
constexpr int kOneThreads = 1024, kOneChunk = 512;
constexpr long long kOneValues = 16384;
__global__ __launch_bounds__(kOneThreads) void k_clip_one(ClipArgs a, int scale) {
  __shared__ double room[kOneThreads / 64];
  const int k = workgroup_id(), lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double sum = 0.0;
  for (int c = wave; c < a.chunks; c += kOneThreads / 64)
    with_chunk<64>(a, k, c, lane, [&](auto& chunk) { sum += squares_of(chunk); });
  const double norm = sqrt(block_sum(sum, room));
  if (threadIdx.x == 0) a.norm[k] = (float)norm;
  if (!scale || !(norm > a.most) || norm == __builtin_inf()) return;
  const double f = a.most / norm;
  for (int c = wave; c < a.chunks; c += kOneThreads / 64)
    with_chunk<64>(a, k, c, lane, [&](auto& chunk) {
      chunk.start();
      chunk.template run<true>([&](float v) { return v * f; });
    });
}

template <int T>
__device__ __forceinline__ double norm_of(const ClipArgs& a, int k, double (&room)[T / 64]) {
  double sum = 0.0;
  const double* p = a.part + (long long)k * a.all;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.all; i += T) sum += p[i];
  return sqrt(block_sum(sum, room));
}

constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void k_clip_norm(ClipArgs a) {
  __shared__ double room[kNormThreads / 64];
  const unsigned k = workgroup_id();
  const double norm = norm_of<kNormThreads>(a, k, room);
  if (threadIdx.x != 0) return;
  a.norm[k] = (float)norm;
  if (a.wide) a.wide[k] = norm;
}

// The chunks from the last to the first, eight by eight: what the launch before read last is in
// the caches still, a chunk's in that of the XCD that both launches give it to.
__global__ __launch_bounds__(kThreads) void k_clip_scale(ClipArgs a, long long total) {
  __shared__ double room[kThreads / 64];
  const unsigned first = workgroup_id(), eights = (unsigned)((total + kXcds - 1) / kXcds);
  if (first >= eights * kXcds) return;
  const unsigned id = (eights - 1 - first / kXcds) * kXcds + first % kXcds;
  if (id >= total) return;
  const int k = id / a.chunks, c = id - k * a.chunks;
  with_chunk<kThreads>(a, k, c, threadIdx.x, [&](auto& chunk) {
    chunk.start();  // on its way while the norm is found
    const double norm = a.wide ? a.wide[k] : norm_of<kThreads>(a, k, room);
    if (!a.wide && a.base + c == 0 && threadIdx.x == 0) a.norm[k] = (float)norm;
    // (a norm that is infinite or no number leaves the values as they are)
    if (!(norm > a.most) || norm == __builtin_inf()) return;
    const double f = a.most / norm;
    chunk.template run<true>([&](float v) { return v * f; });
  });
}

// The cut: values a chunk, for about kChunks chunks in all and at least kLeast values; and a
// replica's chunks. (2 x 402M values in 2048, 8192, 16384 chunks 1945, 1837, 1810 us; 16 x 530K in chunks of
// 4096, 6144, 8192 values 19.8, 18.6, 19.5.) From kWide of them on their sums are added by a launch of
// its own (4.8 us for 8200), not by every workgroup.
constexpr long long kChunks = 16384, kLeast = 6144, kStep = 2048;
constexpr int kWide = 512;
double values_of(int count, const ClipTensor* t) {
  double values = 0;
  for (int i = 0; i < count; ++i) values += (double)eights_values(t[i]);
  return values;
}
bool in_one(int count, const ClipTensor* t) {
  return count <= kBatch && values_of(count, t) <= (double)kOneValues;
}
long long chunk_values(int K, int count, const ClipTensor* t) {
  if (in_one(count, t)) return kOneChunk;
  const double each = values_of(count, t) * K / kChunks;
  return std::min(std::max(((long long)(each / kStep) + 1) * kStep, kLeast), 1LL << 30);
}
long long chunks_of(const ClipTensor& t, long long each) {
  return (eights_values(t) + each - 1) / each;
}

}  // namespace

size_t clip_workspace_bytes(int K, int count, const ClipTensor* t) {
  if (in_one(count, t)) return 0;
  const long long each = chunk_values(K, count, t);
  size_t all = 0;
  for (int i = 0; i < count; ++i) all += chunks_of(t[i], each);
  return (all + 1) * K * sizeof(double);
}

hipError_t launch_clip(int K, int count, const ClipTensor* t, bool scale, double most, float* norm,
                       void* ws, hipStream_t s) {
  ClipArgs a;
  a.each = chunk_values(K, count, t);
  a.most = most;
  a.part = (double*)ws;
  a.norm = norm;
  // (below 2^30 chunks of kMostClipped's values, and one more for each of a launch's kBatch tensors of
  // 2^16 replicas: a launch's chunks, and a replica's, number below 2^31; all replicas' need not)
  long long all = 0;
  for (int i = 0; i < count; ++i) all += chunks_of(t[i], a.each);
  a.all = (int)all;
  if (in_one(count, t)) {
    a.count = count;
    a.base = 0;
    a.chunks = 0;
    for (int i = 0; i < count; ++i) {
      a.t[i] = t[i];
      a.t[i].first = a.chunks;
      a.chunks += (int)chunks_of(t[i], a.each);
    }
    hipLaunchKernelGGL(k_clip_one, dim3(K), dim3(kOneThreads), 0, s, a, (int)scale);
    return hipGetLastError();
  }
  a.wide = scale && all >= kWide ? a.part + (size_t)all * K : nullptr;
  // the tensors in batches, in the second pass from the last to the first
  const int batches = (count + kBatch - 1) / kBatch;
  auto pass = [&](auto launch, bool reverse) {
    for (int n = 0; n < batches; ++n) {
      const int from = (reverse ? batches - 1 - n : n) * kBatch;
      a.count = std::min(kBatch, count - from);
      long long base = 0, chunks = 0;
      for (int i = 0; i < from; ++i) base += chunks_of(t[i], a.each);
      for (int i = 0; i < a.count; ++i) {
        a.t[i] = t[from + i];
        a.t[i].first = (int)chunks;
        chunks += chunks_of(t[from + i], a.each);
      }
      a.base = (int)base;
      a.chunks = (int)chunks;
      launch(chunks * K);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  hipError_t e = pass([&](long long total) {
    hipLaunchKernelGGL(k_clip_sums, grid_of(total), dim3(kThreads), 0, s, a, total);
  }, false);
  if (e != hipSuccess) return e;
  if (!scale || a.wide) {
    hipLaunchKernelGGL(k_clip_norm, dim3(K), dim3(kNormThreads), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess || !scale) return e;
  }
  return pass([&](long long total) {
    hipLaunchKernelGGL(k_clip_scale, grid_of((total + kXcds - 1) / kXcds * kXcds), dim3(kThreads), 0,
                       s, a, total);
  }, true);
}

}  // namespace lsgd
