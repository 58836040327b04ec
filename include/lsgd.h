/*
 * lsgd.h -- C ABI of the MI355X (gfx950) local-SGD hot path.
 *
 * Method: local SGD and post-local SGD of Lin, Stich, Patel, Jaggi, "Don't Use
 * Large Mini-Batches, Use Local SGD" (ICLR 2020). K workers each run H
 * sequential mini-batch SGD steps of batch B_loc on their own model copy, then
 * the K models are replaced by their mean (eq. 2; Algorithm 1). Post-local SGD
 * runs rounds with H = 1 first (eq. "post-local SGD", Algorithm 2); that
 * schedule is a sequence of run_round calls.
 *
 * On one GPU the K workers are K model replicas resident in device memory.
 *
 * Conventions for every call:
 *  - Pointers prefixed d_ are device pointers, h_ host pointers. The caller owns
 *    all memory; the library never allocates device memory. Device buffers
 *    handed to lsgd_init_replicas (dataset, labels, workspace) must stay alive
 *    and unmodified by the caller until lsgd_destroy.
 *  - Work is enqueued asynchronously on the stream given at init (a
 *    hipStream_t passed as void*, NULL = the null stream). Results are valid
 *    once that stream has been synchronised (lsgd_sync does it). Inside a
 *    ResNet-20 local step, work that feeds nothing else at that point may run
 *    on an internal stream of default priority; it is joined back into the
 *    given stream before the step's last command, so stream order on the
 *    given stream still covers all of the step's work.
 *  - Every call returns a status. Argument errors return LSGD_E_INVALID and
 *    change nothing. A failed HIP call returns LSGD_E_HIP and latches: from
 *    then on every call on that context returns LSGD_E_STATE until destroy.
 *  - One context must not be used from two host threads at once. Distinct
 *    contexts are independent.
 *  - Failure detection: every local step checks on the device, with no host
 *    synchronisation, that each replica's mean mini-batch loss is finite; a
 *    non-finite one sets a flag in the workspace that lsgd_sync reports as
 *    LSGD_E_NONFINITE. The flag stays set (the context remains usable)
 *    until lsgd_write_state restores a state or the context is destroyed.
 *    A loss is taken at the pre-update weights, so a step whose update makes
 *    a parameter non-finite shows up at the next step's loss; a non-finite
 *    hidden pre-activation that a ReLU maps to 0 does not reach it.
 *
 * Flat parameter layout of one replica ([P] fp32): for each layer l = 1..L in
 * order, W_l row-major [d_{l-1}][d_l] (element (i, j) maps input i to output
 * j), then the bias b_l [d_l].
 */
#ifndef LSGD_H
#define LSGD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lsgd_ctx lsgd_ctx; /* opaque, host-side */

typedef enum lsgd_status {
  LSGD_OK = 0,
  LSGD_E_INVALID = 1,     /* bad argument; no state was changed */
  LSGD_E_WORKSPACE = 2,   /* workspace smaller than lsgd_workspace_bytes */
  LSGD_E_HIP = 3,         /* a HIP runtime call or launch failed (latched) */
  LSGD_E_STATE = 4,       /* context unusable after an earlier HIP error */
  LSGD_E_UNSUPPORTED = 5, /* valid request the library does not implement */
  LSGD_E_NONFINITE = 6    /* a local step's loss was not finite (sticky; see
                             lsgd_sync) */
} lsgd_status;

/* LSGD_MODEL_MLP: ReLU MLP with widths d_0 .. d_L (L = 1 is softmax
 * regression). LSGD_MODEL_RESNET20: the CIFAR ResNet-20 of the paper's Table 5
 * on 32x32x3 NHWC images (widths[0] = 3072, widths[1] = classes <= 32,
 * n_layers = 1, fp32, B_loc < 131072): a 3x3 stem convolution to 16 channels, three stages of
 * three basic blocks at 16/32/64 channels (stride 2 entering stages 2 and 3,
 * option-A shortcuts: subsample and zero-pad channels), batch normalisation
 * with per-replica batch statistics after every convolution (no weight decay
 * on its scale and shift), global average pooling and a 64 -> classes
 * classifier. Parameter layout: per convolution in order its weight
 * [3][3][c_in][c_out], BN scale [c_out], BN shift [c_out]; then the
 * classifier weight [64][classes] and bias [classes]. Each replica also keeps
 * BN running statistics (they do not enter the training loss): R = 1376
 * values, the running means of the 19 BN layers in convolution order, then
 * their running variances; they start at 0 and 1, follow every local step as
 * r = 0.9 r + 0.1 s (s the batch mean, or the unbiased batch variance
 * var * n / (n - 1) over the n values per channel), and take the plain mean
 * over the replicas at every synchronisation (over the block at a block
 * synchronisation), whatever the scheme. They are read and written through
 * the state blob. */
enum { LSGD_MODEL_MLP = 0, LSGD_MODEL_RESNET20 = 1 };
enum { LSGD_FP32 = 0, LSGD_BF16 = 1 };
/* Local-step / synchronisation scheme (the appendix on compression):
 * LSGD_SCHEME_LOCAL   plain local steps, plain mean (eq. 2);
 * LSGD_SCHEME_SIGN    Algorithm 3: local steps move by sign(d) (d the update
 *                     direction after weight decay and momentum, sign(0) =
 *                     0); the synchronisation sends each worker's model
 *                     difference Delta^k = w_s - w^k as sign(Delta^k) *
 *                     ||Delta^k||_1 / P and sets every replica to
 *                     w_s - (1/K) sum_k of those messages;
 * LSGD_SCHEME_EF_SIGN Algorithm 4: plain local steps; the synchronisation
 *                     compresses Delta^k + e^k the same way and keeps the
 *                     error memory e^k = Delta^k + e^k - message (e^k = 0 at
 *                     init, per worker, never averaged).
 * w_s is the model of the previous synchronisation (w0 at init). */
enum { LSGD_SCHEME_LOCAL = 0, LSGD_SCHEME_SIGN = 1, LSGD_SCHEME_EF_SIGN = 2 };
/* Index sampler. With n_k = floor((k+1)N/K) - floor(kN/K) rows in worker
 * k's slice [floor(kN/K), floor((k+1)N/K)):
 * LSGD_SAMPLER_IID    every local step draws B_loc rows i.i.d. with
 *                     replacement from the worker's fixed slice (eq. 1's
 *                     sampling from the local data): Philox4x32-10, key
 *                     (seed lo, seed hi), counter (j / 4, s lo, k, s hi),
 *                     slot j takes word j mod 4, u -> lo + floor(u n_k / 2^32);
 * LSGD_SAMPLER_EPOCH  the data is repartitioned by a fresh global permutation
 *                     every epoch (the CIFAR training procedure): with
 *                     S = floor(floor(N / K) / B_loc) batches per epoch
 *                     (must be >= 1), step s is batch j = s mod S of epoch
 *                     e = s / S and takes rows pi_e(lo_k + j B_loc + b),
 *                     b < B_loc. pi_e is a 4-round balanced Feistel network on
 *                     2m-bit words (m the smallest >= 1 with 4^m >= N; left
 *                     half the high m bits; round r maps (L, R) to
 *                     (R, L xor (F_r(R) & (2^m - 1)))), F_r(R) word 0 of
 *                     Philox4x32-10 at counter (R, r, e, 0x5348464C) with the
 *                     same key, restricted to [0, N) by cycle walking. */
enum { LSGD_SAMPLER_IID = 0, LSGD_SAMPLER_EPOCH = 1 };
#define LSGD_MAX_LAYERS 8

/*
 * Problem statement, after the REQUIRE list of Algorithms 1 and 2: model,
 * mini-batch size per worker, number of workers, momentum, plus the sampler
 * key. The step size and H are per call (run_round), so schedules such as
 * post-local SGD stay on the host.
 */
typedef struct lsgd_config {
  int32_t model;                          /* LSGD_MODEL_MLP / _RESNET20 */
  int32_t n_layers;                       /* L, 1..LSGD_MAX_LAYERS */
  int32_t widths[LSGD_MAX_LAYERS + 1];    /* d_0 (features) .. d_L (classes) */
  int32_t K;                              /* workers = replicas, >= 1 */
  int32_t B_loc;                          /* local mini-batch, >= 1 */
  int32_t gemm_dtype;                     /* LSGD_FP32 or LSGD_BF16 */
  int32_t nesterov;                       /* 0 heavy ball, 1 Nesterov */
  float momentum;                         /* m in [0, 1) */
  float weight_decay;                     /* coupled L2 on weights and biases */
  float global_momentum;                  /* m_g in [0, 1) at the global
                                             synchronisation; 0: plain mean */
  int32_t scheme;                         /* LSGD_SCHEME_*; a sign scheme
                                             needs global_momentum == 0 */
  int32_t sampler;                        /* LSGD_SAMPLER_* */
  uint64_t seed;                          /* Philox4x32-10 key for sampling */
  int64_t N;                              /* dataset rows, >= K */
} lsgd_config;

/* Number of parameters P of one replica. */
lsgd_status lsgd_param_count(const lsgd_config* cfg, int64_t* P);

/* Bytes of device workspace lsgd_init_replicas needs (replicas, momentum
 * buffers, activations, indices, and for bf16 the operand copies). */
lsgd_status lsgd_workspace_bytes(const lsgd_config* cfg, size_t* bytes);

/*
 * Create a context and synchronise all replicas to w0 (first line of
 * Algorithm 1: w^k_(0) := w_(0)); momentum buffers are zeroed and the local
 * step counter s is set to 0.
 *  d_X   fp32 [N][d_0] row-major dataset, d_y int32 [N] labels in [0, d_L).
 *  d_w0  fp32 [P], copied (stream-ordered); may be freed after the stream
 *        has passed this call.
 *  d_ws  workspace of ws_bytes >= lsgd_workspace_bytes, 256-byte aligned.
 * For LSGD_BF16 the dataset is converted once to a bf16 copy in the
 * workspace (round to nearest even).
 */
lsgd_status lsgd_init_replicas(const lsgd_config* cfg, const float* d_X,
                               const int32_t* d_y, const float* d_w0,
                               void* d_ws, size_t ws_bytes, void* stream,
                               lsgd_ctx** out);

/*
 * One local step on every replica (inner loop of Algorithm 1, local update
 * of eq. 2 with per-replica momentum): sample B_loc indices per worker from
 * its shard, forward, softmax cross-entropy, backward, and
 *   g = grad + wd * w;  u = m u + g;  d = nesterov ? g + m u : u;
 *   w = w - lr * d.
 * d_loss: fp32 [K] receives each replica's mean mini-batch loss at the
 * pre-update weights, or NULL. Increments s.
 */
lsgd_status lsgd_local_step(lsgd_ctx* ctx, float lr, float* d_loss);

/* Synchronisation of eq. 2: every replica becomes (1/K) sum_k w^k, summed in
 * a fixed pairwise tree over k. Momentum buffers are left as they are.
 * LSGD_E_INVALID when the configuration sets a global momentum factor or a
 * sign scheme (those synchronise through lsgd_synchronise). */
lsgd_status lsgd_average(lsgd_ctx* ctx);

/*
 * The form of the plain average (lsgd_average, and the synchronisation of
 * lsgd_run_round without global momentum or a sign scheme). enable = 0 (the
 * default): the mean is written back into all K replicas (K P floats read
 * and K P written). enable = 1, the lazy form that eq. 2 allows since every
 * replica holds the same w after it: the mean is written once (P floats,
 * plus its bf16 copy for LSGD_BF16); the next local step reads that copy as
 * every replica's weights and writes each replica's stepped model. Results
 * are bit for bit those of the default form: every call that reads the
 * replicas (read_params, read_state, block averages, the single-launch
 * softmax round, write_params of one replica) first writes the pending mean
 * into them. MLP models under LSGD_SCHEME_LOCAL without global momentum
 * only, else LSGD_E_UNSUPPORTED; enable outside {0, 1}: LSGD_E_INVALID.
 * Switching it off writes a pending mean out.
 */
lsgd_status lsgd_set_lazy_average(lsgd_ctx* ctx, int32_t enable);

/*
 * The end-of-round synchronisation. With a sign scheme it is the
 * sign-compressed synchronisation of Algorithm 3 or 4 (lr unused; see
 * LSGD_SCHEME_*). With global_momentum == 0 it is lsgd_average (lr unused). Otherwise it is local SGD with global momentum
 * (the momentum appendix's paragraph on global momentum; with local
 * momentum also on, its hybrid scheme): with w_s the model of the previous
 * synchronisation (w0 at init) and u the global buffer (0 at init),
 *   mean = (1/K) sum_k w^k  (the tree of lsgd_average),
 *   u = m_g u + (w_s - mean) / lr,   w_s = w_s - lr u,   every w^k := w_s.
 * The paper's (1/K) sum_k (w_s - w^k) is computed as w_s - mean. lr is the
 * step size of the round's local steps; lr must be finite, and non-zero
 * when m_g != 0, else LSGD_E_INVALID.
 */
lsgd_status lsgd_synchronise(lsgd_ctx* ctx, float lr);

/* H local steps with step sizes h_lr[0..H-1] (host array), then
 * lsgd_synchronise(ctx, h_lr[H-1]) (lsgd_average without global momentum).
 * d_loss: fp32 [H][K] or NULL. With global momentum, H == 0 or a zero last
 * step size is LSGD_E_INVALID.
 * A one-layer fp32 model (softmax regression) under the plain local scheme
 * without global momentum, with 1 <= H <= 64, at most 32 classes and all
 * replicas and buffers within one workgroup's LDS, runs the whole round as a
 * single launch. Its products sum in a different fixed order than the
 * step-by-step path, so the two agree to fp32 rounding, not bit for bit;
 * each is deterministic. */
lsgd_status lsgd_run_round(lsgd_ctx* ctx, int32_t H, const float* h_lr,
                           float* d_loss);

/*
 * Block synchronisation of hierarchical local SGD (Appendix D, the
 * hierarchical local SGD equation; the inner all-reduce of Algorithm 5):
 * replicas 0..K-1 form K/Kb blocks of Kb consecutive replicas and each
 * replica becomes the mean of its block, summed in the same fixed tree as
 * lsgd_average (within the block). Momentum buffers are left as they are.
 * Kb must divide K, else LSGD_E_INVALID; Kb == K is lsgd_average (bit for
 * bit), Kb == 1 changes nothing.
 */
lsgd_status lsgd_average_blocks(lsgd_ctx* ctx, int32_t Kb);

/*
 * One outer round of hierarchical local SGD (Algorithm 5): Hb times, run H
 * local steps then the block synchronisation over blocks of Kb replicas;
 * the last block synchronisation is replaced by the global synchronisation
 * (lsgd_synchronise with the last step size; lsgd_average without global
 * momentum), which the plain block mean would not change in exact
 * arithmetic. h_lr: host
 * array of H * Hb step sizes in step order. d_loss: fp32 [Hb * H][K] or
 * NULL. Kb must divide K; H >= 0, Hb >= 1, else LSGD_E_INVALID. Hb == 1 is
 * lsgd_run_round; Kb == K runs Hb plain rounds of period H.
 */
lsgd_status lsgd_run_hierarchical_round(lsgd_ctx* ctx, int32_t H, int32_t Hb,
                                        int32_t Kb, const float* h_lr,
                                        float* d_loss);

/* Copy replica `replica`'s parameters (or, for replica == -1, their mean by
 * the same tree as lsgd_average, without changing state) to d_dst fp32 [P]. */
lsgd_status lsgd_read_params(lsgd_ctx* ctx, int32_t replica, float* d_dst);

/* Copy replica `replica`'s momentum buffer to d_dst fp32 [P] / overwrite it
 * from d_src fp32 [P] (checkpoint and resume). replica outside [0, K):
 * LSGD_E_INVALID. */
lsgd_status lsgd_read_momentum(lsgd_ctx* ctx, int32_t replica, float* d_dst);
lsgd_status lsgd_write_momentum(lsgd_ctx* ctx, int32_t replica,
                                const float* d_src);

/* Copy the global momentum buffer u to d_dst fp32 [P] / overwrite it from
 * d_src fp32 [P] (checkpoint and resume; the synchronised model w_s is set
 * by lsgd_write_params with replica == -1). LSGD_E_INVALID without global
 * momentum. */
lsgd_status lsgd_read_global_momentum(lsgd_ctx* ctx, float* d_dst);
lsgd_status lsgd_write_global_momentum(lsgd_ctx* ctx, const float* d_src);

/* Copy replica `replica`'s error memory e^k (LSGD_SCHEME_EF_SIGN) to d_dst
 * fp32 [P] / overwrite it from d_src fp32 [P]. LSGD_E_INVALID for other
 * schemes or a replica outside [0, K). */
lsgd_status lsgd_read_error_memory(lsgd_ctx* ctx, int32_t replica, float* d_dst);
lsgd_status lsgd_write_error_memory(lsgd_ctx* ctx, int32_t replica,
                                    const float* d_src);

/* Overwrite replica `replica` (or all replicas for -1) with d_src fp32 [P]
 * (and the bf16 operand copy). For checkpoint restore and tests. With global
 * momentum, replica == -1 also sets the synchronised model w_s. */
lsgd_status lsgd_write_params(lsgd_ctx* ctx, int32_t replica,
                              const float* d_src);

/* Local step counter s (the sampler counter of the next local step). */
lsgd_status lsgd_get_step(lsgd_ctx* ctx, int64_t* step);
lsgd_status lsgd_set_step(lsgd_ctx* ctx, int64_t step);

/* The indices the configured sampler (LSGD_SAMPLER_*) draws at local step
 * `step`: int32 [K][B_loc] into d_idx. */
lsgd_status lsgd_sample_indices(lsgd_ctx* ctx, int64_t step, int32_t* d_idx);

/* Synchronise the context's stream; returns the latched status, else
 * LSGD_E_NONFINITE when a local step since init (or the last
 * lsgd_write_state) had a non-finite loss, else LSGD_OK. */
lsgd_status lsgd_sync(lsgd_ctx* ctx);

/*
 * Checkpoint and resume: the whole training state of a context as one
 * device blob -- what the paper's post-local runs restart from (they switch
 * to local SGD from a mini-batch SGD checkpoint). Layout (all little-endian):
 *   bytes 0..255: header, eight uint64 words: magic 0x3154535F4447534C
 *     ("LSGD_ST1"), a digest of the layout (model, widths, K, P, R and the
 *     section mask, FNV-1a), K, P, R (BN running statistics per replica; 0
 *     for the MLP), the local step counter s, the section mask, the blob's
 *     total bytes; the rest of the 256 bytes is unused;
 *   then, each at the next 256-byte aligned offset and present when its mask
 *   bit is set: bit 0 the replicas fp32 [K][P], bit 1 the momentum buffers
 *   [K][P] (always present), bit 2 the BN running statistics [K][R]
 *   (ResNet-20), bit 3 the synchronised model w_s [P] (global momentum and
 *   the sign schemes), bit 4 the global momentum buffer [P] (global
 *   momentum), bit 5 the error memories [K][P] (LSGD_SCHEME_EF_SIGN).
 * lsgd_state_bytes gives the size for a configuration (no device needed).
 * lsgd_read_state writes the blob to d_dst (stream-ordered, no host sync).
 * lsgd_write_state restores it from d_src: it synchronises the stream to
 * read the header, returns LSGD_E_INVALID without changing anything unless
 * the header matches this context's configuration (magic, digest, K, P, R,
 * mask, size), then overwrites every section (and the bf16 operand copy),
 * sets s and clears the non-finite flag. d_dst / d_src: caller-owned device
 * memory of lsgd_state_bytes bytes, 256-byte aligned, else LSGD_E_INVALID.
 * A context resumed from a blob continues bit for bit as the one that wrote
 * it (same configuration, dataset and step sizes).
 */
lsgd_status lsgd_state_bytes(const lsgd_config* cfg, size_t* bytes);
lsgd_status lsgd_read_state(lsgd_ctx* ctx, void* d_dst);
lsgd_status lsgd_write_state(lsgd_ctx* ctx, const void* d_src);

/* Release the host context (device memory stays with the caller). */
lsgd_status lsgd_destroy(lsgd_ctx* ctx);

/* Static description of a status; never NULL. */
const char* lsgd_status_string(lsgd_status s);

/* Text of the last error recorded on ctx ("" if none); never NULL. */
const char* lsgd_last_error(const lsgd_ctx* ctx);

/* Per-launch timing (a measurement aid, off by default): while enabled,
 * every kernel the context launches is bracketed by two HIP events on its
 * stream, tagged by launch site (sample, fwd<l>, head_fwd, xent, dgrad<l>,
 * wgrad_update for every layer's update, head_wgrad, average ...; a split-K
 * GEMM's tag covers both of its kernels). */
lsgd_status lsgd_profile_enable(lsgd_ctx* ctx, int32_t enable);

/* Restrict the bracketing to launches tagged `tag` (host string, at most 64
 * characters, copied; NULL or "" selects every launch again), and of those
 * to the 1st, (every+1)-th, (2 every+1)-th ... counted from this call, so
 * that one kernel can be timed inside a run at a sampling rate that leaves
 * the run's own speed nearly undisturbed (each bracket costs some
 * microseconds of stream time). LSGD_E_INVALID for a longer tag or
 * every < 1. */
lsgd_status lsgd_profile_select(lsgd_ctx* ctx, const char* tag, int32_t every);

/* Synchronise, then write one line "tag launches total_ms" per tag into the
 * host buffer h_buf (NUL-terminated; LSGD_E_INVALID if len is too small) and
 * clear the records. */
lsgd_status lsgd_profile_report(lsgd_ctx* ctx, char* h_buf, size_t len);

/*
 * Building blocks, exposed for kernel-level tests and bandwidth sweeps.
 */

/* Grouped GEMM over G independent problems (the per-replica layer
 * contractions of the gradient in eq. 2):
 *   C_g[M][N] = opA(A_g)[M][Kd] * opB(B_g)[Kd][N]   (fp32 accumulation)
 * trans_a = 0: A_g is [M][Kd] row-major with leading dimension lda;
 *         = 1: A_g is [Kd][M] row-major (lda >= M).
 * trans_b = 0: B_g is [Kd][N] (ldb >= N); = 1: B_g is [N][Kd] (ldb >= Kd).
 * dtype LSGD_FP32: A, B are float; LSGD_BF16: A, B are bfloat16 bit patterns
 * (uint16). C is fp32 [G][M][N] with leading dimension N, group stride M*N.
 * Group strides sA, sB are in elements. splits in {2, 3, 4, 8} splits K into
 * that many ranges whose fp32 partial sums go to d_part ([splits][G][M][N],
 * caller owned) and are then added in ascending order; splits == 1 needs no
 * d_part; other counts return LSGD_E_INVALID.
 */
lsgd_status lsgd_grouped_gemm(int32_t dtype, int32_t trans_a, int32_t trans_b,
                              int32_t G, int32_t M, int32_t N, int32_t Kd,
                              const void* d_A, int64_t lda, int64_t sA,
                              const void* d_B, int64_t ldb, int64_t sB,
                              float* d_C, int32_t splits, float* d_part,
                              void* stream);

/* In-place K-way replica average of d_W fp32 [K][P] (the kernel behind
 * lsgd_average). */
lsgd_status lsgd_replica_average(float* d_W, int32_t K, int64_t P,
                                 void* stream);

/* The global-momentum synchronisation of lsgd_synchronise on plain arrays:
 * d_W fp32 [K][P] replicas (all set to the new model), d_wsync fp32 [P] the
 * previous synchronised model and d_ug fp32 [P] the global buffer, both
 * updated in place. m_global in [0, 1), lr finite and non-zero, else
 * LSGD_E_INVALID. */
lsgd_status lsgd_replica_average_global_momentum(float* d_W, int32_t K,
                                                 int64_t P, float* d_wsync,
                                                 float* d_ug, float m_global,
                                                 float lr, void* stream);

/* Scratch bytes lsgd_replica_sign_sync needs for K rows of P elements
 * (P % 4 == 0, else LSGD_E_INVALID). */
lsgd_status lsgd_sign_sync_scratch_bytes(int32_t K, int64_t P, size_t* bytes);

/* The sign-compressed synchronisation of lsgd_synchronise on plain arrays:
 * d_W fp32 [K][P] replicas (all set to the new model), d_wsync fp32 [P] the
 * previous synchronised model (updated), d_E fp32 [K][P] the error memories
 * (updated; Algorithm 4) or NULL (Algorithm 3). d_scratch: caller-owned
 * device memory of lsgd_sign_sync_scratch_bytes (LSGD_E_WORKSPACE if
 * smaller). Pointers 16-byte aligned and P % 4 == 0, else LSGD_E_INVALID.
 * Summation orders: each |delta| partial in fp64 over fixed chunks of 8192
 * elements, chunks added in a fixed order; messages added over k in
 * ascending order in fp32. */
lsgd_status lsgd_replica_sign_sync(float* d_W, int32_t K, int64_t P,
                                   float* d_wsync, float* d_E, void* d_scratch,
                                   size_t scratch_bytes, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * lsgd_replica_sign_sync with its scratch taken from a static device array
 * of LSGD_SIGN_SYNC_STATIC_BYTES that the library holds on each GPU it runs
 * on until the process ends, so the call allocates nothing (the caller
 * still passes d_W, d_wsync and d_E). Same arguments, kernels and results as
 * lsgd_replica_sign_sync, bit for bit. Problems needing more scratch than
 * the array holds (lsgd_sign_sync_scratch_bytes(K, P) > 16 MiB, i.e.
 * about K * P > 6.7e7 elements) return LSGD_E_WORKSPACE and launch nothing.
 * Every call on one GPU shares the array: calls that overlap on one GPU
 * (different streams or host threads) race and must be ordered by the
 * caller. The array keeps the last call's contents; nothing in it needs to
 * start at zero.
 */
#define LSGD_SIGN_SYNC_STATIC_BYTES (16u << 20)
lsgd_status lsgd_replica_sign_sync_static(float* d_W, int32_t K, int64_t P,
                                          float* d_wsync, float* d_E,
                                          void* stream);

/* In-place block average of d_W fp32 [K][P]: each of the K/Kb groups of Kb
 * consecutive rows is replaced by its mean (the kernel behind
 * lsgd_average_blocks). Kb must divide K, else LSGD_E_INVALID. */
lsgd_status lsgd_replica_average_blocks(float* d_W, int32_t K, int32_t Kb,
                                        int64_t P, void* stream);

/* Fused update over n elements (the kernel behind the parameter update of
 * lsgd_local_step): g = d_G + wd * w; u = m u + g; d = (nesterov & 1) ?
 * g + m u : u; with nesterov & 2, d = sign(d) (the sign step); w -= lr * d.
 * d_W, d_U updated in place. nesterov outside [0, 3]: LSGD_E_INVALID. */
lsgd_status lsgd_sgd_update(float* d_W, float* d_U, const float* d_G,
                            int64_t n, float lr, float momentum,
                            float weight_decay, int32_t nesterov,
                            void* stream);

/*
 * Matrices in 8 bits with a scale for each block of 128 values of a row: the
 * operands of lsgd_grouped_gemm_blocks. Format LSGD_E4M3 (four exponent bits,
 * largest value 448, no infinity) or LSGD_E5M2 (five, 57344). A row of n
 * values takes up(n, 128) bytes, zeros past the n-th, and
 * up(ceil(n / 128), 4) scale bytes, 127 past the last block's; up(v, m) is v
 * rounded up to a multiple of m. A block's scale 2^e has the smallest
 * -127 <= e <= 127 with max |x| <= 2^e F (F the format's largest value, the
 * maximum over the block's finite values; e = 0 where that is 0) and is held
 * as the byte e + 127. A value x is held as x 2^-e rounded to nearest, ties to
 * even, so nothing finite overflows; a NaN as a NaN, an infinity as the format's
 * (LSGD_E4M3: as a NaN).
 */
enum { LSGD_E4M3 = 0, LSGD_E5M2 = 1 };

/*
 * Writes G matrices X_g [M][N] (dtype LSGD_FP32 or LSGD_BF16, row pitch
 * ldx >= N, group stride sX >= 0 in elements) in blocks: d_Q [G][M][up(N, 128)]
 * with d_S [G][M][up(ceil(N / 128), 4)], blocks along N; and with d_Qt, the
 * transposes, d_Qt [G][N][up(M, 128)] with d_St [G][N][up(ceil(M / 128), 4)],
 * blocks along M. Either pair may be NULL (both pointers), not both pairs; one
 * call reads X once for the two. All padding is written. M, N <= 2^30, d_Q and
 * d_Qt 16-byte aligned, X aligned to its elements, else LSGD_E_INVALID. What is
 * written must not overlap X.
 */
lsgd_status lsgd_quantise_blocks(int32_t dtype, int32_t format, int32_t G,
                                 int32_t M, int32_t N, const void* d_X,
                                 int64_t ldx, int64_t sX, uint8_t* d_Q,
                                 uint8_t* d_S, uint8_t* d_Qt, uint8_t* d_St,
                                 void* stream);

/*
 * Grouped product of matrices in blocks along the contracted dimension:
 *   C_g[M][N] = A_g[M][Kd] * B_g[N][Kd]^T
 * with the precision of C: to LSGD_FP32 every product is exact and summed in
 * fp32 (values below 2^-126 are taken as multiples of 2^-133, one of 2^128, to which
 * 1.9375 2^127 and more rounds in LSGD_E4M3, 1.875 2^127 in LSGD_E5M2, as an infinity,
 * and results below fp32's normal range may come out as zeros); to LSGD_BF16 the 8-bit matrix instruction, which sums eight
 * neighbouring products at a time with 13 bits below the largest of them (an
 * error of about 2^-15 of sum |a b|, 2^-10 at worst) and those sums in fp32, and
 * one rounding at the end. A_g is M rows, B_g N rows of Kd values in the layout above (format_a,
 * format_b may differ): the forward product y = x w takes x and the transpose of
 * w, the input gradient dy w^T takes dy and w, the weight gradient x^T dy the
 * transposes of both. sA, sB (bytes, multiples of 16) and sSA, sSB (scale bytes,
 * multiples of 4) are the group strides; 0 shares one matrix among the groups.
 * d_A, d_B 16-byte, d_SA, d_SB 4-byte aligned. The bytes past Kd of a row
 * must be zeros, as lsgd_quantise_blocks leaves them, and its scale bytes
 * below 255. M, N <= 2^30, Kd <= 2^22. C is out_dtype LSGD_FP32 or LSGD_BF16 (rounded once), row pitch
 * ldc >= N, and its groups must not overlap: sC at least a group's extent (M - 1) ldc + N,
 * or rows of at least G groups side by side (any value for G == 1); nothing between
 * its rows is written. C must not overlap A, B or their scales. d_ws: workspace of
 * lsgd_grouped_gemm_blocks_workspace_bytes (for the same sizes; which may be 0; then NULL is
 * allowed), 16-byte aligned, LSGD_E_WORKSPACE if smaller. A result does not
 * depend on what the workspace held.
 */
lsgd_status lsgd_grouped_gemm_blocks_workspace_bytes(int32_t out_dtype,
                                                     int32_t G, int32_t M,
                                                     int32_t N, int32_t Kd,
                                                     size_t* bytes);
/* How that product is cut, for tests and profiles: cut[0] the tile's rows and columns,
 * cut[1] the stages of loads, cut[2] the ranges of the inner dimension. */
lsgd_status lsgd_grouped_gemm_blocks_cut(int32_t out_dtype, int32_t G, int32_t M, int32_t N,
                                         int32_t Kd, int32_t cut[3]);
lsgd_status lsgd_grouped_gemm_blocks(int32_t format_a, int32_t format_b,
                                     int32_t out_dtype, int32_t G, int32_t M,
                                     int32_t N, int32_t Kd, const uint8_t* d_A,
                                     int64_t sA, const uint8_t* d_SA,
                                     int64_t sSA, const uint8_t* d_B,
                                     int64_t sB, const uint8_t* d_SB,
                                     int64_t sSB, void* d_C, int64_t ldc,
                                     int64_t sC, void* d_ws, size_t ws_bytes,
                                     void* stream);

/*
 * Orthogonalised momentum. O(X) takes X = U S V^T towards U V^T: from
 * X / (||X||_F + eps), `steps` Newton-Schulz steps
 *   A = X X^T,  B = b A + c A A,  X := a X + B X
 * (on X^T where M > N), h_coefficients = {a, b, c} (host). The products
 * take fp32 precision for dtype LSGD_FP32 (two fp16 pieces of each operand on
 * the matrix cores); for LSGD_BF16 operands of 11 significant bits do where
 * min(M, N) > 384 (X itself is held in two pieces all the same): a result off by 2.0e-3 to
 * 2.3e-3 of its norm, where rounding it to bf16 alone takes 1.7e-3. A zero matrix stays zero; an
 * infinity or a NaN makes the whole result NaN.
 *
 * Arguments, else LSGD_E_INVALID: 1 <= G <= 65535, 1 <= M, N <= 2^20 with
 * up(M, 64) up(N, 64) <= 2^30, 1 <= steps <= 64, finite coefficients under
 * which no singular value in [0, 1] grows past 32 on the way, eps finite and
 * > 0. Row pitches are at least N; the groups of a matrix that is written
 * must not overlap (group stride >= the group's extent, or rows of at least G
 * groups side by side). Workspace: caller-owned device memory of
 * lsgd_orthogonalise_workspace_bytes for the dtype (0 for small matrices; then
 * NULL is allowed), 256-byte aligned (LSGD_E_WORKSPACE if smaller); one
 * workspace serves one call at a time.
 */
lsgd_status lsgd_orthogonalise_workspace_bytes(int32_t dtype, int32_t G,
                                               int32_t M, int32_t N,
                                               size_t* bytes);

/* How the steps of such matrices are cut, for tests and profiles: cut[0] the pieces of an
 * operand, 0 where one launch does all steps (the rest is 0 then); cut[1], cut[2] the tile's
 * rows and columns and the stages of loads of X X^T, cut[3], cut[4] those of A A, cut[5],
 * cut[6] those of B X. */
lsgd_status lsgd_orthogonalise_cut(int32_t dtype, int32_t G, int32_t M, int32_t N,
                                   int32_t cut[7]);

/* Y_g = O(X_g) for G matrices, X and Y of `dtype` (pitches and strides in
 * elements). Y may be X itself (same pitch and stride); else
 * they must not overlap. */
lsgd_status lsgd_orthogonalise(int32_t dtype, int32_t G, int32_t M, int32_t N,
                               const void* d_X, int64_t ldx, int64_t sX,
                               void* d_Y, int64_t ldy, int64_t sY,
                               int32_t steps, const float* h_coefficients,
                               float eps, void* d_ws, size_t ws_bytes,
                               void* stream);

/* The update by the orthogonalised momentum, in place on fp32 W and U:
 *   u = m u + g;  d = nesterov ? g + m u : u;
 *   w = (1 - lr wd) w - lr scale O(d).
 * gemm_dtype: the precision of O's products (as dtype above). Pointers may point into
 * the replicas' flat rows (a layer's W of every replica: sW the row length). lr,
 * weight_decay and scale and their products finite in fp32, 0 <= momentum < 1, nesterov 0 or 1. W, U and G must
 * not overlap. */
lsgd_status lsgd_orthogonal_update(int32_t gemm_dtype, int32_t G, int32_t M,
                                   int32_t N, float* d_W, int64_t ldw,
                                   int64_t sW, float* d_U, int64_t ldu,
                                   int64_t sU, const float* d_G, int64_t ldg,
                                   int64_t sG, float lr, float momentum,
                                   float weight_decay, int32_t nesterov,
                                   float scale, int32_t steps,
                                   const float* h_coefficients, float eps,
                                   void* d_ws, size_t ws_bytes, void* stream);

/*
 * Matrices in 8-bit integers with an fp32 scale for each row: the operands of
 * lsgd_grouped_gemm_rows. A row of n values takes up(n, 128) bytes, zeros past the
 * n-th, and one scale s: max |x| / 127 rounded to fp32, at least 2^-126; 1 for a row of
 * zeros; a NaN for a row that holds an infinity or a NaN, whose integers are zeros. A value x
 * is held as the integer nearest to x / s, ties to even, |q| <= 127.
 */

/*
 * Writes G matrices X_g [M][N] (dtype LSGD_FP32 or LSGD_BF16, row pitch
 * ldx >= N, group stride sX >= 0 in elements) in rows: d_Q [G][M][up(N, 128)]
 * with d_S [G][M]; and with d_Qt and d_St (NULL: not wanted) the transposes, a scale for
 * each column of X: d_Qt [G][N][up(M, 128)] with d_St [G][N]. All padding is written.
 * G <= 65535, M, N <= 2^30, d_Q and d_Qt 16-byte aligned, the rest aligned to its
 * elements, else LSGD_E_INVALID. With the transposes: a workspace of
 * lsgd_quantise_rows_workspace_bytes, 4-byte aligned (LSGD_E_WORKSPACE if smaller; 0 for
 * small matrices), one call's at a time; without them, or for 0, NULL is allowed. What is written must not overlap
 * X, the workspace or another result.
 */
lsgd_status lsgd_quantise_rows_workspace_bytes(int32_t G, int32_t M, int32_t N,
                                               size_t* bytes);
lsgd_status lsgd_quantise_rows(int32_t dtype, int32_t G, int32_t M, int32_t N,
                               const void* d_X, int64_t ldx, int64_t sX,
                               int8_t* d_Q, float* d_S, int8_t* d_Qt,
                               float* d_St, void* d_ws, size_t ws_bytes,
                               void* stream);

/*
 * Grouped product of matrices in rows along the contracted dimension:
 *   C_g[m][n] = S_A[m] S_B[n] sum_k A_g[m][k] B_g[n][k] + bias_g[n]
 * The sum of integers is exact; it is rounded to fp32, as are its two products with the
 * scales (the last together with the bias), and once more to LSGD_BF16 (out_dtype). A_g is
 * M rows, B_g N rows of Kd integers in the layout above: the forward product y = x w + b
 * takes x and the transpose of w, the input gradient dy w^T takes dy and w, the weight
 * gradient x^T dy the transposes of both. Group strides sA, sB (bytes, multiples
 * of 16), sSA, sSB and sbias (elements) may be 0: a matrix shared among the groups. d_A, d_B
 * 16-byte aligned; the bytes past Kd of a row must be zeros, as lsgd_quantise_rows
 * leaves them; any integer from -128 to 127 and any positive scale will do. d_bias fp32
 * [G][N] or NULL. G <= 65535, M, N <= 2^30, Kd <= 2^22. C's pitch and group stride and the workspace (of
 * lsgd_grouped_gemm_rows_workspace_bytes, 16-byte aligned) as lsgd_grouped_gemm_blocks
 * has them. C must not overlap anything that is read.
 */
lsgd_status lsgd_grouped_gemm_rows_workspace_bytes(int32_t out_dtype, int32_t G,
                                                   int32_t M, int32_t N,
                                                   int32_t Kd, size_t* bytes);
/* How that product is cut, for tests and profiles: cut[0] the tile's rows and columns,
 * cut[1] the stages of loads, cut[2] the ranges of the inner dimension. */
lsgd_status lsgd_grouped_gemm_rows_cut(int32_t out_dtype, int32_t G, int32_t M,
                                       int32_t N, int32_t Kd, int32_t cut[3]);
lsgd_status lsgd_grouped_gemm_rows(int32_t out_dtype, int32_t G, int32_t M,
                                   int32_t N, int32_t Kd, const int8_t* d_A,
                                   int64_t sA, const float* d_SA, int64_t sSA,
                                   const int8_t* d_B, int64_t sB,
                                   const float* d_SB, int64_t sSB,
                                   const float* d_bias, int64_t sbias,
                                   void* d_C, int64_t ldc, int64_t sC,
                                   void* d_ws, size_t ws_bytes, void* stream);

/*
 * Layer norm of the rows of G matrices X_g [M][N] (dtype), each with a weight and a bias
 * of its own (fp32 [G][N], group strides sw, sb >= 0; NULL: ones, zeros):
 *   mean = sum x / N, rstd = (sum (x - mean)^2 / N + eps)^-1/2,
 *   Y = (x - mean) rstd w + b (in fp32, then rounded to out_dtype), d_mean, d_rstd fp32 [G][M].
 * The sums are held in fp64. A NaN or an infinity in a row makes the row NaN, finite values of
 * any size do not (a d_rstd below 2^-126 holds fewer bits). X's pitch
 * ldx >= N and stride sX >= 0 in elements; Y's groups must not overlap (as C of
 * lsgd_grouped_gemm_blocks). eps finite and > 0. G <= 65535, M, N <= 2^30, else
 * LSGD_E_INVALID. Results must not overlap anything that is read.
 */
lsgd_status lsgd_layer_norm(int32_t dtype, int32_t out_dtype, int32_t G,
                            int32_t M, int32_t N, const void* d_X, int64_t ldx,
                            int64_t sX, const float* d_w, int64_t sw,
                            const float* d_b, int64_t sb, float eps, void* d_Y,
                            int64_t ldy, int64_t sY, float* d_mean,
                            float* d_rstd, void* stream);

/*
 * Its gradients, from dY (out_dtype), X (dtype) and the mean and rstd that
 * lsgd_layer_norm wrote: with n = (x - mean) rstd and e = dy w,
 *   dX = rstd (e - sum e / N - n sum (e n) / N) (dtype),
 *   dw = sum over the group's rows of dy n, db = sum of dy (fp32 [G][N], group strides sdw,
 *   sdb >= N; both NULL: not wanted).
 * The fp32 mean is off the row's own by up to 2^-24 |mean|, and n by that times rstd: of rows
 * of |mean| rstd >= 2048 the row's own mean is found again from X and d_mean and used instead.
 * A row's sums of e and e n are held in fp32 (in fp64 from 16385 columns on and up to 8), whose range
 * they must not leave. A column's sum takes fp32 steps over at most 32 rows, fp64 ones over those.
 * The sums over rows are added in an order that the sizes alone decide. Workspace
 * (not without dw and db): lsgd_layer_norm_backward_workspace_bytes, 16-byte aligned (LSGD_E_WORKSPACE
 * if smaller; may be 0; then NULL is allowed), one call's at a time. Limits as
 * above. Results must not overlap each other or anything that is read.
 */
lsgd_status lsgd_layer_norm_backward_workspace_bytes(int32_t G, int32_t M,
                                                     int32_t N, size_t* bytes);
lsgd_status lsgd_layer_norm_backward(int32_t dtype, int32_t out_dtype, int32_t G,
                                     int32_t M, int32_t N, const void* d_dY,
                                     int64_t ldg, int64_t sG, const void* d_X,
                                     int64_t ldx, int64_t sX,
                                     const float* d_mean, const float* d_rstd,
                                     const float* d_w, int64_t sw, void* d_dX,
                                     int64_t ldd, int64_t sD, float* d_dw,
                                     int64_t sdw, float* d_db, int64_t sdb,
                                     void* d_ws, size_t ws_bytes, void* stream);

/*
 * The gradients of K replicas: `count` tensors, of each replica a matrix [M][N] (dtype
 * LSGD_FP32 or LSGD_BF16, row pitch ld >= N, replica stride s >= 0 in elements; a
 * replica's flat row holds one at an offset, s the row length). The array is read
 * before the call returns.
 */
typedef struct lsgd_tensor {
  void* d_data;
  int64_t M, N, ld, s;
  int32_t dtype;
  int32_t reserved; /* 0 */
} lsgd_tensor;
#define LSGD_MAX_TENSORS 65536

/*
 * lsgd_gradient_norm: d_norm[k] (fp32 [K]) = the root of the sum of squares over all values of
 * replica k's tensors, squares and sum in fp64, in an order that the sizes alone decide (a tensor
 * listed twice counts twice). lsgd_clip_gradients also multiplies the values of each replica
 * whose norm is above max_norm (finite, > 0) by max_norm / norm, the factor and the product in
 * fp64, rounded once; the others' stay as they are, as do those of a replica that holds an infinity or a
 * NaN. d_norm holds the norms before clipping (past fp32's range an infinity, but clipped by the
 * fp64 norm all the same). K <= 65535, count <= LSGD_MAX_TENSORS, M and N at
 * least 1, M N, M ld, s <= 2^44, N <= 2^30 where M > 1 and ld > N, no more than 2^60 values in all (a
 * shared one for each replica, rows of a pitch rounded up to eights), else LSGD_E_INVALID. Clipped tensors' replicas must not overlap
 * (s >= (M - 1) ld + N, or rows of all K side by side), nor two tensors (lsgd_tensors_apart says
 * whether they do, or where that would take over 2^24 runs of values, may), else LSGD_E_INVALID;
 * nor d_norm or the workspace a tensor. Workspace of
 * lsgd_gradient_norm_workspace_bytes, 8-byte aligned (LSGD_E_WORKSPACE if smaller; 0 for few
 * values; then NULL is allowed), one call's at a time.
 */
lsgd_status lsgd_gradient_norm_workspace_bytes(int32_t K, int32_t count,
                                               const lsgd_tensor* h_tensors,
                                               size_t* bytes);
lsgd_status lsgd_tensors_apart(int32_t K, int32_t count,
                               const lsgd_tensor* h_tensors, int32_t* apart);
lsgd_status lsgd_gradient_norm(int32_t K, int32_t count,
                               const lsgd_tensor* h_tensors, float* d_norm,
                               void* d_ws, size_t ws_bytes, void* stream);
lsgd_status lsgd_clip_gradients(int32_t K, int32_t count,
                                const lsgd_tensor* h_tensors, double max_norm,
                                float* d_norm, void* d_ws, size_t ws_bytes,
                                void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LSGD_H */
