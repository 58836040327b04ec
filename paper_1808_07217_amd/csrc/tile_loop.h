// The inner loop shared by the products whose two operands both have the contracted
// index contiguous: tiles of rows of 128 bytes a step, whatever the element type.
//
// A workgroup computes BP x BQ results of P Q^T, its wavefronts WP x WQ each, as
// 16 x 16 blocks: lane l holds two vectors of 16 bytes of row l % 16 of a fragment, the
// 16-byte pieces l / 16 and l / 16 + 4 of the row's 128 bytes, and result e of lane l is at
// row 4 (l / 16) + e of P and row l % 16 of Q.
//
// Operands go from memory straight to LDS (16 bytes a lane), into S stages: two, or
// more where a step is too short to cover a load. LDS holds rows of 128 bytes without padding; piece c of row r lies in slot c ^ (r % 8),
// so that eight rows' pieces c fall into different banks. The lanes fetch the
// pieces in that order, each row still one whole 128-byte line.
// One barrier a step, before its last row of fragments: every wavefront has then
// read the stage (it may be overwritten) and its own loads of the next one have
// landed (loads return in order: as many may be outstanding as the later stages have).
// The stages are arrays of their own and the loop is unrolled over them, so that the
// compiler can tell a stage being read from one being loaded and adds no waits. What remains of the step's matrix instructions runs while the next step's
// first fragments are read.
#pragma once
#include "device_common.h"

namespace lsgd {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));

typedef int v8i __attribute__((ext_vector_type(8)));

using Frag = v8i;  // pieces l / 16 and l / 16 + 4

// The tile a workgroup of a launch of `total` works on. The hardware deals
// consecutive ids round-robin to the XCDs, each with an L2 of its own: every XCD
// takes a contiguous range, and walks it in bands of kBand tile rows, so that the
// tiles at work at one time share few rows and columns.
constexpr int kBand = 8;
__device__ __forceinline__ int xcd_order(int p, int total) {
  const int x = p % kXcds, each = total / kXcds, rest = total % kXcds;
  return x * each + min(x, rest) + p / kXcds;
}
__device__ __forceinline__ void band_order(int l, int tp, int tq, int& p, int& q) {
  const int band = l / (kBand * tq), in = l - band * kBand * tq;
  const int rows = min(kBand, tp - band * kBand);
  p = band * kBand + in % rows;
  q = in / rows;
}

// The last word of a buffer descriptor: plain bytes, bounds checked against its size.
constexpr int kRsrcRaw = 0x00027000;

// The S stages of a kernel, `BYTES` each, as TileLoop::run takes them.
constexpr int kMostStages = 4;
#define LSGD_TILE_STAGES(st, S, BYTES)                                \
  __shared__ __align__(16) uint8_t st##0[BYTES];                      \
  __shared__ __align__(16) uint8_t st##1[BYTES];                      \
  __shared__ __align__(16) uint8_t st##2[(S) > 2 ? (BYTES) : 16];     \
  __shared__ __align__(16) uint8_t st##3[(S) > 3 ? (BYTES) : 16];     \
  uint8_t* const st[kMostStages] = {st##0, st##1, st##2, st##3}

// Policy M: types M::P and M::Q (what a fragment becomes once read, by m.p<PH>(frag, i) and
// m.q<PH>(frag, j, up)), M::Acc (a block's sums) and m.mac<PH>(acc, p, i, q, j), PH the step's
// parity. What comes
// once for two steps: m.load(stage, k, want) starts it (by M::kEvenLoads loads), for an
// even step k, on its way to the kExtra bytes at the end of the stage; m.begin(stage, k, up) reads it into an
// M::Next, while the step before still needs its own, and m.take(up) replaces that;
// q<0> takes it from `up`. m.last(odd): one step is left, of that parity, and calls p and
// mac with PH = 0.
template <int BP, int BQ, int WP, int WQ, int S = 2, int kExtra = 0>
struct TileLoop {
  static constexpr int kP = BP, kQ = BQ, kWaves = (BP / WP) * (BQ / WQ), kThreads = 64 * kWaves;
  static constexpr int FP = WP / 16, FQ = WQ / 16;
  static constexpr int kStage = (BP + BQ) * 128 + kExtra;  // bytes
  static constexpr int kLoads = (BP + BQ) / 8 / kWaves;   // a wavefront's, of 8 rows
  static_assert(BP / 8 % kWaves == 0 && BQ / 8 % kWaves == 0 && FP % 2 == 0, "tile shape");
  static_assert(S >= 2 && S <= kMostStages, "stages");

  using Rsrc = __amdgpu_buffer_rsrc_t;
  const uint8_t *P, *Q;  // the tiles' first rows, at the step to be loaded next
  int leftp, leftq;      // bytes from there to the end of the last row
  int off, every;        // the lane's place in a load's 8 rows; 8 kWaves rows
  int lane, wave, wp, wq;
  uint32_t rp, rq;       // LDS offset of the lane's first piece

  // ld: the row pitch in bytes, 256 ld < 2^31; np, nq: the rows from the tile's first
  // on that exist. The buffer descriptors end behind the last of them, so that nothing
  // past it is read; what LDS then holds in its place reaches only results that are
  // not stored.
  __device__ __forceinline__ void init(const uint8_t* p, const uint8_t* q, int ld, int np, int nq) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    P = p;
    Q = q;
    leftp = min(np, BP) * ld;
    leftq = min(nq, BQ) * ld;
    off = (lane >> 3) * ld + ((lane & 7) ^ (lane >> 3)) * 16;
    every = 8 * ld;
    wp = wave / (BQ / WQ) * WP;
    wq = wave % (BQ / WQ) * WQ;
    const int lr = lane & 15, slot = (lane >> 4) ^ (lr & 7);
    rp = (uint32_t)((wp + lr) * 128 + slot * 16);
    rq = (uint32_t)((BP + wq + lr) * 128 + slot * 16);
  }
  // (before the first load) the first n steps are left out
  __device__ __forceinline__ void skip(int n) {
    P += 128LL * n;
    Q += 128LL * n;
    leftp -= 128 * n;
    leftq -= 128 * n;
  }
  // one step into a stage; !want: nothing is read (no branch: the matrix instructions
  // before one would be moved past it)
  __device__ __forceinline__ void load(uint8_t* stage, bool want = true) {
    const Rsrc bp = __builtin_amdgcn_make_buffer_rsrc((void*)P, 0, want ? leftp : 0, kRsrcRaw);
    const Rsrc bq = __builtin_amdgcn_make_buffer_rsrc((void*)Q, 0, want ? leftq : 0, kRsrcRaw);
#pragma unroll
    for (int t = 0; t < kLoads; ++t) {
      const int at = wave + t * kWaves;  // the load's eighth of the tile's rows
      // (a load's wavefronts all fetch P or all Q)
      if (t < BP / 8 / kWaves)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            bp, (__attribute__((address_space(3))) void*)(stage + at * 1024), 16,
            off + at * every, 0, 0, 0);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            bq, (__attribute__((address_space(3))) void*)(stage + at * 1024), 16,
            off + (at - BP / 8) * every, 0, 0, 0);
    }
    P += 128;
    Q += 128;
    leftp -= 128;
    leftq -= 128;
  }
  __device__ __forceinline__ Frag read(const uint8_t* stage, uint32_t at, int i) const {
    const v4i lo = *(const v4i*)(stage + at + i * 2048);
    const v4i hi = *(const v4i*)(stage + (at ^ 64) + i * 2048);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }

  // until at most the loads of n steps, e of them even, are outstanding, then everyone
  template <class M, int n, int e>
  static __device__ __forceinline__ void wait() {
    static_assert(n * kLoads + e * M::kEvenLoads < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(n * kLoads + e * M::kEvenLoads) : "memory");
    __builtin_amdgcn_s_barrier();
  }

  // Step k (of parity PH), from stage `cur`; the loads of steps k + 1 .. k + S - 1 are on
  // their way, those of step k + 1 to `nxt`.
  template <int PH, class M>
  __device__ __forceinline__ void step(uint8_t* cur, uint8_t* nxt, int k, int n, M& m,
                                       typename M::P (&p)[2], typename M::Q (&q)[FQ],
                                       typename M::Acc (&acc)[FP][FQ]) {
#pragma unroll
    for (int i = 0; i + 1 < FP; ++i) {
      p[(i + 1) & 1] = m.template p<PH>(read(cur, rp, i + 1), i + 1);
#pragma unroll
      for (int j = 0; j < FQ; ++j) m.template mac<PH>(acc[i][j], p[i & 1], i, q[j], j);
      __builtin_amdgcn_sched_barrier(0);  // no fragment is read earlier than that
    }
    // the next stage is whole, and this one read by everyone (of the steps k + 2 ..
    // k + S - 1 every second is even, the first if this one is)
    wait<M, S - 2, (S - 2 + 1 - PH) / 2>();
    // the next step's fragments between the last row's instructions, each into the
    // registers that one of them frees, then the loads (first, they cost 3%)
    const Frag next = read(nxt, rp, 0);
    typename M::Next up;
    if constexpr (PH == 1) m.begin(nxt, k + 1, up);
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
      m.template mac<PH>(acc[FP - 1][j], p[1], FP - 1, q[j], j);
      __builtin_amdgcn_sched_barrier(0);
      q[j] = m.template q<1 - PH>(read(nxt, rq, j), j, up);
    }
    if constexpr (PH == 1) m.take(up);
    p[0] = m.template p<1 - PH>(next, 0);
    __builtin_amdgcn_sched_barrier(0);
    load(cur, k + S < n);
    if constexpr (((PH + S) & 1) == 0) m.load(cur, k + S, k + S < n);
  }

  // The steps 0 .. n - 1 (n >= 1) are multiplied into acc; st: the stages.
  template <class M>
  __device__ __forceinline__ void run(uint8_t* const (&st)[kMostStages], int n, M& m,
                                      typename M::Acc (&acc)[FP][FQ]) {
    constexpr int U = S % 2 ? 2 * S : S;  // steps until stage and parity repeat
#pragma unroll
    for (int i = 0; i < S; ++i) {
      load(st[i], i < n);
      if (i % 2 == 0) m.load(st[i], i, i < n);
    }
    wait<M, S - 1, (S - 1) / 2>();
    typename M::Next up;
    m.begin(st[0], 0, up);
    m.take(up);
    typename M::Q q[FQ];
    typename M::P p[2];
#pragma unroll
    for (int j = 0; j < FQ; ++j) q[j] = m.template q<0>(read(st[0], rq, j), j, up);
    p[0] = m.template p<0>(read(st[0], rp, 0), 0);
    int k = 0;
    for (; k + U < n; k += U) {
#pragma unroll
      for (int i = 0; i < U; i += 2) {
        step<0>(st[i % S], st[(i + 1) % S], k + i, n, m, p, q, acc);
        step<1>(st[(i + 1) % S], st[(i + 2) % S], k + i + 1, n, m, p, q, acc);
      }
    }
    // one to U steps are left, the last without a next one
    const int rest = n - k;
    const uint8_t* cur = st[0];
#pragma unroll
    for (int i = 0; i + 1 < U; ++i)
      if (rest > i + 1) {
        if (i % 2 == 0)
          step<0>(st[i % S], st[(i + 1) % S], k + i, n, m, p, q, acc);
        else
          step<1>(st[i % S], st[(i + 1) % S], k + i, n, m, p, q, acc);
        cur = st[(i + 1) % S];
      }
    m.last(rest % 2 == 0);
#pragma unroll
    for (int i = 0; i < FP; ++i) {
      if (i + 1 < FP) p[(i + 1) & 1] = m.template p<0>(read(cur, rp, i + 1), i + 1);
#pragma unroll
      for (int j = 0; j < FQ; ++j) m.template mac<0>(acc[i][j], p[i & 1], i, q[j], j);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

}  // namespace lsgd
