/*
 * uad.h -- C ABI of the Urgency-Aware Denoising (UAD) library for GB300 (sm_103a).
 *
 * The library runs the denoising loop of a flow-matching action expert on one GPU:
 * per-action Euler steps with per-action flow times (Sec. 3, Eqs. 1-2; Sec. 4.2, Eqs. 4-5),
 * Urgency-Aware Early Release of actions whose budget ends before N* (Sec. 4.2),
 * Trajectory Reconciliation of released actions with zero extra evaluations (Sec. 4.3,
 * Eqs. 6-7), ghost actions, and Ghost Action Correction of the executable tail (Sec. 4.4,
 * Eqs. 8-9). Releases are handed to the host while the tail keeps refining on the GPU
 * (App. C.1, "Asynchronous Execution").
 *
 * Conventions
 *   - Every call returns an int: UAD_OK (0) or a negative code below. uad_last_error()
 *     gives a message for the last failure on a context.
 *   - Pointers marked "host or device" may point to either; the library inspects them.
 *   - The caller owns every buffer it passes and may reuse it as soon as the call returns
 *     (the library copies what it keeps). The library owns its weights, state, scratch and
 *     the pinned release buffer, all freed by uad_destroy.
 *   - All arguments are validated on the host before anything is launched.
 *   - No call waits on the GPU without a deadline; no call traps the GPU.
 *   - A context is used by one host thread at a time.
 */
#ifndef UAD_H
#define UAD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define UAD_OK 0
#define UAD_EINVAL (-22)     /* invalid argument or configuration */
#define UAD_ESTATE (-1)      /* call out of order (e.g. finish without denoise) */
#define UAD_ENOMEM (-12)     /* device or pinned allocation failed */
#define UAD_ECUDA (-5)       /* a CUDA runtime call failed; see uad_last_error */
#define UAD_ETIMEDOUT (-110) /* the deadline passed before the GPU finished */
#define UAD_ENONFINITE (-33) /* a velocity was NaN or Inf; outputs are still written */

#define UAD_KIND_ADARMS 0    /* joint attention over prefix KV + chunk, adaptive RMSNorm */
#define UAD_KIND_DIT 1       /* chunk self-attention + cross-attention, adaLN-zero */
#define UAD_KIND_CONCAT 2    /* joint attention as ADARMS with plain RMSNorm; each token's time
                                embedding joins its action embedding in the input MLP (App. C.1,
                                the SmolVLA variant) */

#define UAD_DTYPE_F32 0
#define UAD_DTYPE_BF16 1

#define UAD_MAX_STEPS 64     /* largest step budget N_i */

/* Shape of the action expert F_theta (Sec. 3, Eq. 1). */
typedef struct uad_arch {
  int32_t kind;          /* UAD_KIND_ADARMS, UAD_KIND_DIT or UAD_KIND_CONCAT */
  int32_t dtype;         /* UAD_DTYPE_F32: fp32 everywhere; UAD_DTYPE_BF16: bf16 weights and
                            GEMM/attention operands, fp32 accumulation, state and velocities */
  int32_t n_layers;
  int32_t width;         /* W */
  int32_t n_heads;       /* query heads */
  int32_t n_kv_heads;    /* key/value heads (divides n_heads; DiT: == n_heads) */
  int32_t head_dim;
  int32_t mlp_dim;
  int32_t action_dim;    /* D */
  int32_t chunk_len;     /* H, actions per chunk (Sec. 3) */
  int32_t prefix_len;    /* P, observation prefix tokens */
  int32_t prefix_width;  /* DiT: width of the prefix tokens (cross-attention input) */
  int32_t rope;          /* ADARMS: RoPE on chunk queries/keys at positions P + i */
  int32_t max_batch;     /* robots per call, >= 1 */
} uad_arch;

/* The urgency schedule of one call (Sec. 4.2, Eq. 4, generalised to per-action budgets). */
typedef struct uad_schedule {
  const int32_t* budgets;  /* host, [batch][chunk_len], N_i >= 1; N* = max over a robot's row */
  int32_t batch;           /* robots in this call, 1..max_batch */
  int32_t n_exec;          /* S, actions executed before replanning; 0 means chunk_len */
  int32_t tr;              /* Trajectory Reconciliation on (1) or off (0, UAER-only ablation:
                              released actions are fed back frozen at flow time 1) */
  int32_t gac;             /* Ghost Action Correction on/off; needs tr unless chunk_relative */
  int32_t chunk_relative;  /* actions relative to the chunk start: GAC is skipped (Sec. 4.4) */
  const uint8_t* gac_mask; /* host [action_dim], 1 = additive dimension corrected by Eq. 9,
                              0 = left unchanged (rotation / gripper); NULL = all additive */
  int32_t rot_dim;         /* first of three dimensions holding a rotation vector (axis times
                              angle, radians) that GAC corrects by composition on SO(3)
                              (App. C.1): E_R = F_U ... F_2 F_1 with F_i = R(ghost_i)
                              R(released_i)^T over the early actions in token order (each applied
                              after the previous ones); every tail action
                              R <- exp(log(E_R)/|tail|) R.
                              These dimensions are never additive; -1 = no rotation dimensions.
                              Must be -1 or in 0..action_dim-3 (else UAD_EINVAL). */
} uad_schedule;

typedef struct uad_stats {
  int32_t evals;           /* velocity-network evaluations of the chunk (= N*; TR adds none) */
  int32_t n_star;          /* max step budget of the call */
  int32_t nonfinite;       /* count of non-finite velocity entries */
  int32_t tr_extra_evals;  /* evaluations spent on reconciliation: always 0 */
} uad_stats;

typedef struct uad_ctx uad_ctx;

/* Create a context on the current CUDA device.
 * weights: host or device fp32 blob of n_floats values, tensors in this order (linear
 *   weights [in][out], y = x W + b):
 *     t_w1[W][W] t_b1[W] t_w2[W][W] t_b2[W] in_w[D][W] in_b[W]
 *     per layer, ADARMS: mod1_w[W][3W] mod1_b[3W] wq[W][Hq*dh] wk[W][Hkv*dh] wv[W][Hkv*dh]
 *                        wo[Hq*dh][W] mod2_w[W][3W] mod2_b[3W] wg[W][F] wu[W][F] wd[F][W]
 *                DiT:    mod_w[W][6W] mod_b[6W] wq wk wv[W][Hq*dh] wo[Hq*dh][W]
 *                        wqc[W][Hq*dh] wkc wvc[Pw][Hq*dh] woc[Hq*dh][W]
 *                        w1[W][F] b1[F] w2[F][W] b2[W]
 *     modf_w[W][2W] modf_b[2W] out_w[W][D] out_b[D]
 *   CONCAT instead: in_w[D][W] in_b[W] ti_wa[W][W] ti_wt[W][W] ti_b[W] to_w[W][W] to_b[W],
 *     per layer wq wk wv wo wg wu wd (shapes as ADARMS), out_w[W][D] out_b[D]; the input is
 *     h = SiLU((u in_w + in_b) ti_wa + e(tau) ti_wt + ti_b) to_w + to_b with e the token's
 *     sinusoidal time embedding, every norm is RMSNorm without modulation and residuals are
 *     ungated.
 *   Modulation vectors are (scale, shift, gate) for ADARMS and (shift1, scale1, gate1,
 *   shift2, scale2, gate2) for DiT; the final one is (scale, shift) / (shift, scale).
 *   For bf16 architectures every weight is rounded to bf16 (nearest, ties to even).
 * The weights are copied into the library's own layout; the blob may be freed afterwards.
 * Errors: UAD_EINVAL (shape, n_floats), UAD_ENOMEM, UAD_ECUDA. */
int uad_init(const uad_arch* arch, const float* weights, size_t n_floats, uad_ctx** out);

/* Bind robot `robot`'s observation context (the cached vision-language prefix, Sec. 3).
 * ADARMS: k, v = per-layer prefix keys and values [L][P][Hkv][dh] (keys already carry
 *         their own position encoding).
 * DiT:    k = prefix tokens [P][prefix_width], v = NULL; the per-layer cross-attention K/V
 *         are projected here, once per observation.
 * dtype: UAD_DTYPE_F32 or UAD_DTYPE_BF16 element type of the given buffers (host or device);
 * they are copied (converted to the arch dtype). prefix_len must equal arch.prefix_len.
 * Errors: UAD_EINVAL, UAD_ESTATE (a chunk is in flight), UAD_ECUDA. Synchronous. */
int uad_set_prefix_kv(uad_ctx* ctx, int32_t robot, const void* k, const void* v,
                      int32_t prefix_len, int32_t dtype);

/* Precompute the per-action time conditioning for every flow time j/n, 1 <= n <= max_budget,
 * plus 1 (App. C.1). Optional: uad_denoise computes missing times itself. Synchronous. */
int uad_prepare_times(uad_ctx* ctx, int32_t max_budget);

/* Start denoising one chunk for sched->batch robots (robots 0..batch-1) on `stream`
 * (a cudaStream_t; NULL = legacy default stream). Asynchronous: returns once the work is
 * enqueued. noise: host or device fp32 [batch][H][D], the initial state x_0 (Sec. 3).
 * n_star: 0, or the largest budget of the call (checked). Every robot must have a prefix.
 * Early actions are released into pinned host memory after their last step (UAER); the
 * tail continues on the stream. Errors: UAD_EINVAL, UAD_ESTATE (previous chunk not
 * finished), UAD_ECUDA. */
int uad_denoise(uad_ctx* ctx, const float* noise, const uad_schedule* sched, int32_t n_star,
                void* stream);

/* Host-side hand-off of released actions (App. C.1: urgent actions go to the execution
 * queue while the tail refines). Waits until at least `min_ready` of robot `robot`'s
 * actions are available, or until timeout_us passes (0: do not wait).
 * out [H][D] (host): rows of ready actions are written (others untouched);
 * ready [H] (host, may be NULL): 1 if available; release_step [H] (may be NULL): the step
 * after which the action became available (N_i for early actions, N* for the tail, whose
 * rows already include GAC). Released actions never change afterwards (Sec. 4.4).
 * Returns the number of ready actions (>= min_ready), UAD_ETIMEDOUT, or an error (UAD_EINVAL
 * for min_ready > H). */
int uad_poll_released(uad_ctx* ctx, int32_t robot, int32_t min_ready, int64_t timeout_us,
                      float* out, int32_t* ready, int32_t* release_step);

/* Wait (at most timeout_us; < 0 = no limit) for the chunk to complete and read it back.
 * final [batch][H][D]: released actions for early actions, x_{N*} plus GAC (Eq. 9) for the
 *   executable tail, x_{N*} for the rest;
 * ghost [batch][H][D]: reconciled end states x'_{N*} (ghost actions, Sec. 4.3) for early
 *   actions, x_{N*} (before GAC) for the others;
 * gac_error [batch][D]: E of Eq. 8 (zeros where GAC did not run).
 * Any output may be NULL; each may be host or device memory.
 * Returns UAD_OK, UAD_ENONFINITE (outputs written), UAD_ETIMEDOUT (the chunk stays in
 * flight; call again), UAD_ESTATE, UAD_ECUDA. UAD_ECUDA after a bounded device-side wait ran
 * out: if the chunk ran on the persistent evaluation kernel (whose grid barriers need all of
 * its CTAs resident at once, which a shared or partitioned GPU may not grant), the context runs
 * every later chunk on the per-operation kernels (uad_set_wait_limit tries the persistent
 * kernel again). */
int uad_finish(uad_ctx* ctx, float* final_actions, float* ghost, float* gac_error,
               uad_stats* stats, int64_t timeout_us);

/* Device timestamps of the last finished chunk: ms[k-1] = time from the chunk's first
 * kernel to the end of step k (k = 1..n_star), from the GPU's global timer. Returns the
 * number of entries written. */
int uad_step_times(const uad_ctx* ctx, double* ms, int32_t max_entries);

/* Kernel launches the library enqueues per uad_denoise of the given batch and N*
 * (excluding one-time time-conditioning fills). */
int uad_launches_per_chunk(const uad_ctx* ctx, int32_t batch, int32_t n_star);

/* Per-kernel profile of one chunk (measurement support, not part of the method). */
typedef struct uad_kernel_stat {
  char name[32];          /* kernel class, e.g. "gate_up_proj", "attention", "euler_tr_gac" */
  int32_t launches;       /* launches of this class in the chunk */
  int32_t pad;
  double total_ms;        /* sum of CUDA-event durations of those launches */
  double bytes;           /* algorithmic HBM bytes of those launches (operands read once) */
  double flops;           /* algorithmic flops of those launches */
} uad_kernel_stat;

/* Run one chunk like uad_denoise + uad_finish, but launched eagerly (no graph) on the
 * library's worker stream with a CUDA event pair around every kernel, and return per-class
 * totals in out[0..n). Returns n, or an error. Synchronous; results are discarded. */
int uad_profile_chunk(uad_ctx* ctx, const float* noise, const uad_schedule* sched,
                      uad_kernel_stat* out, int32_t max_stats, int64_t timeout_us);

/* Testing aid for the bounded waits (not part of the method). Every wait inside the persistent
 * evaluation kernel gives up after wait_ns nanoseconds (> 0; the default is 2 s), records an
 * error code on the device and lets the launch wind down; the next uad_finish then returns
 * UAD_ECUDA, and the context stays usable. unreachable > 0 makes the first completion count of
 * every evaluation wait for that many arrivals more than the kernel ever makes, so that the
 * wait is sure to run out (0 restores normal operation). Applies to chunks started afterwards
 * (cached graphs are rebuilt), and re-enables the persistent kernel after a fall-back (see
 * uad_finish). Returns UAD_OK, UAD_EINVAL or UAD_ESTATE (chunk in flight). */
int uad_set_wait_limit(uad_ctx* ctx, int64_t wait_ns, int32_t unreachable);

/* Testing aid (not part of the method): the fp32 rotations that Ghost Action Correction applies
 * on SO(3) (App. C.1; Sec. 4.4, Eqs. 8-9), run on the GPU for n rotation vectors w[n][3] (host
 * memory, axis times angle in radians): log_exp[i] = log(exp(w_i)) and
 * log_comp[i] = log(exp(w_i) exp(w_{(i+1) mod n})^T), log giving the principal vector (angle in
 * [0, pi]). Synchronous; allocates its own device memory. Returns UAD_OK, UAD_EINVAL (null
 * pointer, n < 1 or n > 2^20) or UAD_ECUDA. */
int uad_so3_check(const float* w, int32_t n, float* log_exp, float* log_comp);

void uad_destroy(uad_ctx* ctx);
const char* uad_last_error(const uad_ctx* ctx);

/* ---- Host-only helpers (no GPU needed) ------------------------------------------------ */

/* Plan of step k (1-based) for one robot with budgets[H] (Sec. 4.2, Eqs. 4-5; Sec. 4.3, Eq. 7):
 * flags[i] bit 0 = active (k <= N_i: own Euler step 1/N_i), bit 1 = ghost input (early action
 * past its release, fed its reconciled state), bit 2 = released after this step, bit 3 =
 * early (N_i < N*: a TR running sum is kept), bit 4 = frozen input (TR off);
 * tau = tau_num[i] / tau_den[i] (reduced fraction), the flow time fed to the network.
 * Returns N* or UAD_EINVAL. */
int uad_plan_step(const int32_t* budgets, int32_t H, int32_t k, int32_t tr, int32_t* flags,
                  int32_t* tau_num, int32_t* tau_den);

/* Library version string. */
const char* uad_version(void);

/* ---- Kernel-level op: the step loop's tensor-core projection on caller buffers ------------ */

/* Re-lay out one linear weight for the tensor-core projection kernel (host only, no GPU).
 * w: host fp32 [K][N] (y = x w); out: host bf16 bit patterns, N * K values, as 128 x 64 blocks:
 * block (n / 128, k / 64) starts at element ((n / 128) * (K / 64) + k / 64) * 8192; inside it,
 * row n % 128 holds 64 values (128 bytes) whose eight 16-byte groups are permuted by
 * group ^ (n % 8) -- the 128-byte-swizzled K-major shared-memory layout the tensor cores read.
 * Values are rounded to bf16 (nearest, ties to even). Needs N % 128 == 0 and K % 64 == 0.
 * Returns UAD_OK or UAD_EINVAL. */
int uad_tile_weight(const float* w, int32_t K, int32_t N, uint16_t* out);

/* out[M][N] = x[M][K] w + bias on the tensor cores (tcgen05, bf16 operands, fp32 accumulation):
 * the projection kernel of every velocity-network layer (Sec. 3, Eq. 1).
 * x: device bf16 [M][K]; w_tiled: device, the layout of uad_tile_weight; bias: device fp32 [N]
 * or NULL; out: device fp32 [M][N]. Needs N % 128 == 0, K % 64 == 0, M >= 1.
 * 4 KiB of error words are allocated by the library with cudaMalloc on the first call on each device and
 * kept until exit; K splits are combined on the chip, so calls on different streams may overlap.
 * Asynchronous on `stream` (a cudaStream_t, NULL = legacy stream) and in its order: x, w_tiled and bias may
 * be written by work queued on it before the call. Returns UAD_OK, UAD_EINVAL,
 * UAD_ENOMEM or UAD_ECUDA. */
int uad_linear(const void* x, const void* w_tiled, const float* bias, float* out, int32_t M,
               int32_t N, int32_t K, void* stream);

/* Whether the finished projections of the current device (uad_linear, uad_linear_static_scratch) are complete.
 * Every wait inside their kernels is bounded (2 s). One that runs out ends its call, whose output is then
 * incomplete, and no other call, before, after or beside it. Returns UAD_ECUDA if one ran out in the last
 * 1024 calls of the process since the last query (and forgets it), UAD_OK otherwise. Synchronous on the
 * legacy stream: synchronise the calls' streams first; not while a stream is being captured. */
int uad_linear_status(void);

/* Testing aid for those waits (not part of the method): uad_linear as if one of its waits had just run out, so that
 * every other that is not over within microseconds gives up and its part of the output is not computed. */
int uad_linear_check(const void* x, const void* w_tiled, const float* bias, float* out, int32_t M,
                     int32_t N, int32_t K, void* stream);

/* ---- The same projection op for callers that cannot allocate device memory ---------------
 * The paper has no counterpart: this serves deployments rather than the method. A real-time
 * controller that has finished start-up must not block on cudaMalloc (it can take unbounded
 * time and synchronize the device, stalling the control loop), and a host framework whose
 * caching allocator already holds the GPU's memory cannot take a stray allocation. This entry
 * point computes exactly what uad_linear computes but allocates nothing: no cudaMalloc,
 * cudaFree or allocating library call. It needs no scratch beyond error words (4 KiB) inside the
 * library's device image.
 *   - Limits: M * N <= UAD_LINEAR_STATIC_MAX_ELEMS and (N / 128) * ceil(M / 64) <=
 *     UAD_LINEAR_STATIC_MAX_TILES; larger calls return UAD_ETOOBIG and launch nothing.
 *   - The first call on a device looks up their device address (cudaGetSymbolAddress,
 *     which may load the library's device code: with lazy module loading, the CUDA default,
 *     the driver reserves its memory only then). Make one warm-up call per device during
 *     start-up, before any stream capture begins and before the control loop runs, so that
 *     the device code is resident when "allocates nothing" matters.
 * Arguments, layout and other errors are those of uad_linear. */
#define UAD_ETOOBIG (-7)
#define UAD_LINEAR_STATIC_MAX_ELEMS (1 << 20)
#define UAD_LINEAR_STATIC_MAX_TILES 4096
int uad_linear_static_scratch(const void* x, const void* w_tiled, const float* bias, float* out,
                              int32_t M, int32_t N, int32_t K, void* stream);

/* ---- A paged key-value cache on caller buffers: append, attention ---------------------------
 * The paper has no counterpart: its prefix is one cached buffer a robot (App. D). A program that runs the
 * vision-language model on the same GPU keeps that model's keys and values in pages shared by all robots, extends
 * them by the tokens of an instruction, an answer or a draft, and binds them to the expert (uad_set_prefix_paged).
 * The calls below do so for one layer and a batch of sequences of different lengths. They are asynchronous on
 * `stream` (a cudaStream_t, NULL = legacy stream) and in its order, allocate nothing, keep nothing between calls,
 * and may be captured into CUDA graphs: what changes from step to step (tables, lengths, rows) is read on the
 * device when the graph runs. All pointers in the structures are device memory of the current device.
 *
 * Page p, slot s, head h, dimension d of the keys is at k + p * page_stride + s * slot_stride + h * head_stride + d
 * (in elements), of the values at the same place of v: pages of [slot][head][dim], [head][slot][dim] or of keys and
 * values in turn. */
typedef struct uad_kv_pages {
  void *k, *v;           /* 16-byte aligned */
  int64_t page_stride, slot_stride, head_stride;   /* > 0, multiples of 16 bytes */
  int32_t dtype;         /* UAD_DTYPE_F32 or UAD_DTYPE_BF16 */
  int32_t n_pages;       /* >= 1 */
  int32_t page_size;     /* tokens of a page, 1..65536, any number */
  int32_t n_kv_heads;    /* 1..1024 */
  int32_t head_dim;      /* 64, 128 or 256 */
  int32_t pad;
} uad_kv_pages;

/* A batch of sequences. Token i of sequence b is in page table[b * table_stride + i / page_size], slot i % page_size.
 * Rows start[b] .. start[b + 1] - 1 of the token tensors are its newest tokens, in order: row t is the token at position
 * len[b] - (start[b + 1] - t). Rows from start[n_seqs] on belong to nobody and are neither read nor written. A page may
 * stand in the tables of several sequences (a shared prefix); no two rows of one append may name the same slot. */
typedef struct uad_kv_seqs {
  const int32_t* table;  /* [n_seqs][table_stride], the first table_width entries of a row; entries past a sequence's last
                            token, or before what its window sees, are not looked at */
  const int32_t* len;    /* [n_seqs] tokens in the cache, the new ones included; 0 is allowed */
  const int32_t* start;  /* [n_seqs + 1], ascending from 0 or more; NULL: row b is the one new token of sequence b */
  int64_t table_stride;
  int32_t n_seqs;        /* 0..65535 */
  int32_t table_width;   /* >= 1; table_width * page_size <= 2^31 - 2^17 */
  int32_t max_new;       /* at least the largest number of new tokens of a sequence, >= 1 */
  int32_t max_len;       /* attention: about the longest len, from which the work is split (0: table_width * page_size). A
                            longer sequence is served too, less evenly */
} uad_kv_seqs;

/* What the kernels find wrong on the device is added to the caller's status word (a device int32 that the caller
 * clears; NULL: not reported), and never followed: */
#define UAD_KV_BAD_PAGE 1 /* a page outside 0..n_pages-1 where a token is written or seen: it is left out */
#define UAD_KV_BAD_SEQ 2  /* len outside 0..table_width * page_size, fewer tokens than new ones, more new ones than max_new, or
                             start not ascending within the rows: the sequence is left out, its rows stay as they were */

/* Rotation of a head's first `dim` dimensions by its token's position: pair (i, i + dim / 2) by the angle
 * position * theta^(-2 i / dim). The frequencies are kept as 64-bit fractions of a turn, so that far positions
 * lose nothing. Plain memory of the caller, set by uad_rope_init (host only). */
typedef struct uad_rope {
  int32_t dim, pad;
  uint64_t turn[128];
} uad_rope;
/* dim: a multiple of 16, 16..256; theta > 0, finite. Returns UAD_OK or UAD_EINVAL. */
int uad_rope_init(double theta, int32_t dim, uad_rope* out);

/* The new tokens' rows of an append. Head h of row t of q is at q + t * q_stride + h * head_dim, and so on: the three may
 * be parts of one fused projection. Strides in elements; addresses and strides are multiples of 16 bytes. */
typedef struct uad_kv_rows {
  const void *q, *k, *v; /* q: NULL = no queries; k, v: both or NULL = only queries are rotated */
  int64_t q_stride, k_stride, v_stride;
  void* q_out;           /* rotated queries in the cache's type, head h of row t at t * q_out_stride + h * head_dim. May be q where rows
                            and cache are of one type and the strides are the same; otherwise it must not overlap q, k or v */
  int64_t q_out_stride;
  int32_t dtype;         /* type of q, k and v: UAD_DTYPE_F32 (such as uad_linear's output) or UAD_DTYPE_BF16 */
  int32_t n_heads;       /* query heads; 0 without q */
  int32_t n_rows;        /* rows that the tensors hold; start stays within them */
  int32_t pad;
} uad_kv_rows;

/* Rotate the new tokens' queries and keys (rope NULL: no rotation) and write keys and values into their pages, in fp32
 * arithmetic rounded once to the cache's type. Values are not rotated. Slots of other tokens stay as they were.
 * Errors: UAD_EINVAL (arguments), UAD_ECUDA. */
int uad_kv_append(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_kv_rows* rows, const uad_rope* rope,
                  int32_t* status, void* stream);

/* Attention of the new tokens over their sequences' pages. Query head h reads key/value head h / (n_heads / n_kv_heads).
 * A token at position p sees the keys j < len with j <= p (causal), j > p - window (window > 0) and
 * key_mask[b * mask_stride + j] != 0 (key_mask != NULL): out = softmax(scale q k) v over them. What it does not see has no
 * influence, whatever it holds. Where it sees nothing, out is 0 and lse is -infinity. Products and softmax in fp32
 * (bf16 caches: exact products of bf16 keys and queries, probabilities as the sum of two bf16), rounded once to the
 * cache's type. Meant for one to a few new tokens a sequence: each 8 to 32 rows (n_heads / n_kv_heads times new tokens)
 * read the keys once. */
typedef struct uad_attn {
  const void* q;         /* cache's type, head h of row t at t * q_stride + h * head_dim, 16-byte aligned */
  void* out;             /* the same with out_stride; must not overlap q */
  float* lse;            /* [n_rows][n_heads] natural logarithm of the softmax's denominator; NULL: not wanted */
  const uint8_t* key_mask;   /* rows of table_width * page_size bytes, mask_stride apart */
  int64_t q_stride, out_stride, mask_stride;
  float scale;           /* 0: 1 / sqrt(head_dim). For a softmax of zeros, fp32's least number above 0 */
  int32_t n_heads;       /* a multiple of n_kv_heads, at most 64 times it */
  int32_t n_rows;
  int32_t causal;        /* 0 or 1 */
  int32_t window;        /* 0: no limit */
  int32_t pad;
} uad_attn;

/* Bytes of device memory that uad_paged_attention needs for these arguments (0 is possible): host only, the same for
 * the same sizes. What a call without a window needs is enough for every window; another number of sequences, rows or heads, another
 * max_new, max_len or table_width may need more or less. table, len and start may be NULL here. Returns UAD_EINVAL (negative) for bad
 * arguments. */
int64_t uad_paged_attention_workspace(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn);

/* workspace: 16-byte aligned, in use until the call's work is done: calls that may run at the same time (other streams,
 * graphs) need one each. It needs no preparation and carries nothing from call to call.
 * Errors: UAD_EINVAL (arguments, workspace too small), UAD_ECUDA. */
int uad_paged_attention(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn, void* workspace,
                        size_t workspace_bytes, int32_t* status, void* stream);

/* Bind robot `robot`'s prefix from pages: uad_set_prefix_kv of the first arch.prefix_len tokens of a sequence whose keys and
 * values a vision-language model has appended layer by layer. layers: the caches of the arch's n_layers layers, of one type and
 * page size, with the arch's n_kv_heads and head_dim (experts of kind DIT take tokens, not keys: UAD_EINVAL), on the context's
 * device, which has to be the current one. table: host or device, the pages of those tokens (table_len entries, at least as
 * many), one table for all layers. Synchronous, and behind the legacy default stream; pages or a device table that another stream
 * writes have to be finished first.
 * Errors: UAD_EINVAL (also a page outside 0..n_pages-1), UAD_ESTATE (a chunk is in flight), UAD_ENOMEM, UAD_ECUDA. */
int uad_set_prefix_paged(uad_ctx* ctx, int32_t robot, const uad_kv_pages* layers, int32_t n_layers, const int32_t* table,
                         int32_t table_len);

/* ---- The projection of few tokens with 4-bit weights ------------------------------------------------------
 * out[M][N] = x[M][K] w^T + bias with w[n][k] = (q[n][k] - zero[n][k / group]) * scale[n][k / group]: for the tokens of a
 * decoding step, whose time is that of reading the weights. x: device bf16; q: device [N][K / 2], k even in the low
 * four bits of byte k / 2; scale: device bf16 [N][K / group]; zero: device uint8 [N][K / group], 0..15 (only the low four bits are
 * read), or NULL: 8; bias: device fp32 [N] or NULL; out: device fp32 [M][N]. Sums are in fp32: of the exact x (q - zero) over a group
 * first, which has to stay within fp32 by itself, and then scaled. A row of x with infinities gives infinities or NaN. x and q
 * 16-byte aligned. 1 <= M <= UAD_W4_MAX_ROWS, N >= 1, K % group == 0,
 * group 32, 64 or 128, K <= 2^30, N * K <= 2^35. Asynchronous on `stream` and in its order; allocates nothing; may be captured.
 * Errors: UAD_EINVAL, UAD_ETOOBIG (M: give the rows to several calls), UAD_ECUDA. */
#define UAD_W4_MAX_ROWS 64
int uad_linear_w4(const void* x, const uint8_t* q, const uint16_t* scale, const uint8_t* zero, const float* bias,
                  float* out, int32_t M, int32_t N, int32_t K, int32_t group, void* stream);

/* Round a linear weight to that form (host only). w: host fp32 [K][N] (y = x w), finite; q, scale (bf16 bits) and zero
 * as above, host. zero NULL: symmetric, scale = max |w| / 7, values -7..7 (stored plus 8); else over [min(w, 0), max(w, 0)].
 * scale is rounded to bf16 first and q to the nearest for it. Returns UAD_OK or UAD_EINVAL. */
int uad_quantize_w4(const float* w, int32_t K, int32_t N, int32_t group, uint8_t* q, uint16_t* scale, uint8_t* zero);

#ifdef __cplusplus
}
#endif
#endif /* UAD_H */
