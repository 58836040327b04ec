// The norm of each replica's gradients over all its tensors, and clipping by it.
//
// norm[k]^2 = sum of x^2 over the tensors of replica k, squared and added in fp64: nothing
// overflows or vanishes, and the order of the additions is the cut's alone. Each
// replica's values, tensor after tensor, are cut into chunks, a workgroup each; a second
// launch adds a replica's sums and, where the norm is above the bound, multiplies its
// chunks by bound / norm in fp64, one rounding a value. It takes the chunks from the
// last to the first: what the first launch read last is in the caches still.
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

// f(value) of every value of chunk c of replica k by T threads, `tid` of them this one; WRITE: the
// value becomes f's. Eights, U of a thread in flight, where rows lie side by side, one by one
// otherwise.
template <bool BF, bool WRITE, int T, class F>
__device__ __forceinline__ void each_value(const ClipTensor& t, long long k, long long c,
                                           long long each, int tid, F f) {
  constexpr int U = 4;
  const long long n = t.M * t.N, e0 = c * each, e1 = min(n, e0 + each);
  if (t.M == 1 || t.ld == t.N) {
    const long long x = k * t.s + e0;
    const int values = (int)(e1 - e0), whole = values / 8 * 8;
    for (int e = tid * 8; e < whole; e += T * 8 * U) {
      Raw8<BF> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (e + u * T * 8 < whole) fetch8<BF>(t.p, x + e + u * T * 8, 0, 8, v[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (e + u * T * 8 < whole) {
          float w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = f(v[u][i]);
          if constexpr (WRITE) store8<BF>(t.p, x + e + u * T * 8, 0, 8, w);
        }
    }
    if (tid < values - whole) {
      const long long at = x + whole + tid;
      const float w = f(BF ? bf16_to_f32(((const bf16_t*)t.p)[at]) : ((const float*)t.p)[at]);
      if constexpr (WRITE) {
        if constexpr (BF)
          ((bf16_t*)t.p)[at] = f32_to_bf16(w);
        else
          ((float*)t.p)[at] = w;
      }
    }
  } else {
    const long long dm = T / t.N, dn = T - dm * t.N;
    long long m = (e0 + tid) / t.N, j = e0 + tid - m * t.N;
    for (long long e = e0 + tid; e < e1; e += T) {
      const long long at = k * t.s + m * t.ld + j;
      const float w = f(BF ? bf16_to_f32(((const bf16_t*)t.p)[at]) : ((const float*)t.p)[at]);
      if constexpr (WRITE) {
        if constexpr (BF)
          ((bf16_t*)t.p)[at] = f32_to_bf16(w);
        else
          ((float*)t.p)[at] = w;
      }
      m += dm;
      j += dn;
      if (j >= t.N) {
        j -= t.N;
        ++m;
      }
    }
  }
}
template <bool WRITE, int T, class F>
__device__ __forceinline__ void each_of(const ClipArgs& a, int k, int c, int tid, F f) {
  int i = 0;
  for (int step = kBatch / 2; step; step /= 2)  // the last tensor that starts at c or before
    if (i + step < a.count && a.t[i + step].first <= c) i += step;
  const ClipTensor& t = a.t[i];
  if (t.bf16)
    each_value<true, WRITE, T>(t, k, c - t.first, a.each, tid, f);
  else
    each_value<false, WRITE, T>(t, k, c - t.first, a.each, tid, f);
}

__global__ __launch_bounds__(kThreads) void k_clip_sums(ClipArgs a, long long total) {
  __shared__ double room[kThreads / 64];
  const unsigned id = workgroup_id();
  if (id >= total) return;
  const int k = id / a.chunks, c = id - k * a.chunks;
  double sum = 0.0;
  each_of<false, kThreads>(a, k, c, threadIdx.x, [&](float v) {
    sum = __builtin_fma((double)v, (double)v, sum);
    return v;
  });
  sum = block_sum(sum, room);
  if (threadIdx.x == 0) a.part[(long long)k * a.all + a.base + c] = sum;
}

// Few values: a workgroup a replica, a chunk a wavefront, all in one launch.
constexpr int kOneThreads = 1024, kOneChunk = 512;
constexpr long long kOneValues = 16384;
__global__ __launch_bounds__(kOneThreads) void k_clip_one(ClipArgs a, int scale) {
  __shared__ double room[kOneThreads / 64];
  const int k = workgroup_id(), lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double sum = 0.0;
  for (int c = wave; c < a.chunks; c += kOneThreads / 64)
    each_of<false, 64>(a, k, c, lane, [&](float v) {
      sum = __builtin_fma((double)v, (double)v, sum);
      return v;
    });
  const double norm = sqrt(block_sum(sum, room));
  if (threadIdx.x == 0) a.norm[k] = (float)norm;
  if (!scale || !(norm > a.most) || norm == __builtin_inf()) return;
  const double f = a.most / norm;
  for (int c = wave; c < a.chunks; c += kOneThreads / 64)
    each_of<true, 64>(a, k, c, lane, [&](float v) { return (float)(v * f); });
}

__device__ __forceinline__ double norm_of(const ClipArgs& a, int k,
                                          double (&room)[kThreads / 64]) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.all; i += kThreads) sum += a.part[(long long)k * a.all + i];
  return sqrt(block_sum(sum, room));
}

__global__ __launch_bounds__(kThreads) void k_clip_norm(ClipArgs a) {
  __shared__ double room[kThreads / 64];
  const unsigned k = workgroup_id();
  const double norm = norm_of(a, k, room);
  if (threadIdx.x == 0) a.norm[k] = (float)norm;
}

__global__ __launch_bounds__(kThreads) void k_clip_scale(ClipArgs a, long long total) {
  __shared__ double room[kThreads / 64];
  const unsigned first = workgroup_id();
  if (first >= total) return;
  const unsigned id = (unsigned)(total - 1 - first);
  const int k = id / a.chunks, c = id - k * a.chunks;
  const double norm = norm_of(a, k, room);
  if (a.base + c == 0 && threadIdx.x == 0) a.norm[k] = (float)norm;
  // (a norm that is infinite or no number leaves the values as they are)
  if (!(norm > a.most) || norm == __builtin_inf()) return;
  const double f = a.most / norm;
  each_of<true, kThreads>(a, k, c, threadIdx.x, [&](float v) { return (float)(v * f); });
}

// The cut: values a chunk (about kChunks chunks in all), and a replica's chunks.
constexpr long long kChunks = 2048, kLeast = 4096;
double values_of(int count, const ClipTensor* t) {
  double values = 0;
  for (int i = 0; i < count; ++i) values += (double)t[i].M * t[i].N;
  return values;
}
bool in_one(int count, const ClipTensor* t) {
  return count <= kBatch && values_of(count, t) <= (double)kOneValues;
}
long long chunk_values(int K, int count, const ClipTensor* t) {
  if (in_one(count, t)) return kOneChunk;
  const double each = values_of(count, t) * K / kChunks;
  return std::min(((long long)(each / kLeast) + 1) * kLeast, 1LL << 30);
}
long long chunks_of(const ClipTensor& t, long long each) { return (t.M * t.N + each - 1) / each; }

}  // namespace

size_t clip_workspace_bytes(int K, int count, const ClipTensor* t) {
  if (in_one(count, t)) return 0;
  const long long each = chunk_values(K, count, t);
  size_t all = 0;
  for (int i = 0; i < count; ++i) all += chunks_of(t[i], each);
  return all * K * sizeof(double);
}

hipError_t launch_clip(int K, int count, const ClipTensor* t, bool scale, double most, float* norm,
                       void* ws, hipStream_t s) {
  ClipArgs a;
  a.each = chunk_values(K, count, t);
  a.most = most;
  a.part = (double*)ws;
  a.norm = norm;
  long long all = 0;
  for (int i = 0; i < count; ++i) all += chunks_of(t[i], a.each);
  if (all > 0x7fffffffLL / K) return hipErrorInvalidValue;
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
  // the tensors in batches, in the second pass from the last to the first
  const int batches = (count + kBatch - 1) / kBatch;
  for (int pass = 0; pass < (scale ? 2 : 1); ++pass)
    for (int n = 0; n < batches; ++n) {
      const int from = (pass ? batches - 1 - n : n) * kBatch;
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
      const long long total = chunks * K;
      if (pass)
        hipLaunchKernelGGL(k_clip_scale, grid_of(total), dim3(kThreads), 0, s, a, total);
      else
        hipLaunchKernelGGL(k_clip_sums, grid_of(total), dim3(kThreads), 0, s, a, total);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  if (!scale) {
    hipLaunchKernelGGL(k_clip_norm, dim3(K), dim3(kThreads), 0, s, a);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace lsgd
