/*
 * dppo.h — C ABI of libdppo: the hot path of DPPO's pruned GRPO training step on one B200.
 *
 * DPPO ("Unbiased Dynamic Pruning for Efficient Group-Based Policy Optimization") prunes prompts
 * and completions of a GRPO batch at random, reweights what is retained by importance-sampling
 * factors so that the gradient stays unbiased, packs the retained sequences densely and trains on
 * them.  This library does, per batch:  group advantages -> candidate sets, pruning masks and
 * rescaling factors -> Dense Prompt Packing -> one sweep over the LM-head logits that yields the
 * loss and dlogits; for the frozen policies of that loss, the scoring of the sampled tokens (8-bit LM-head
 * product, log-probs with entropy and alternatives); and, with a second policy beside the trained one, distillation
 * from its alternatives, verification of tokens that it drafted, and its LM-head in block-scaled 8-bit floating point.
 *
 * Conventions (all entry points)
 *  - Return value: 0 (DPPO_OK) or a negative dppo_error.  Nothing throws, aborts or prints.
 *    dppo_last_error() gives the message of the calling thread's last failure.
 *  - Unless a parameter says "host", array pointers are DEVICE pointers owned by the caller.  The
 *    library allocates no memory and keeps no state between calls; scratch comes from a caller
 *    workspace sized by the matching *_workspace_bytes() (a pure host function).  The one exception is
 *    dppo_pack_prompts_static, whose scratch is an array inside the library that all its calls on a device
 *    share (see there).
 *  - Work is enqueued on `stream` (a cudaStream_t passed as void*); there is no host
 *    synchronisation inside.  Outputs are valid once the stream reaches that point.
 *  - Host-visible arguments are validated before anything is launched.  Problems only the device
 *    can see (a unit longer than a row, a target id outside the vocabulary, a wait that ran out)
 *    are recorded in the caller's `status` word (device int32, first error wins, caller zeroes it)
 *    as a positive dppo_status; the kernel then finishes without trapping.
 *  - Every output is a deterministic function of the inputs (no floating-point atomics).
 *  - Each entry point that enqueues work opens an NVTX range of its own name around its host side, so
 *    its launches are grouped under it in a timeline profiler.
 */
#ifndef DPPO_H_
#define DPPO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DPPO_OK = 0,
    DPPO_ERR_INVALID_ARG = -1,          /* NULL where data is required, negative size, bad enum       */
    DPPO_ERR_BAD_SHAPE = -2,            /* sizes inconsistent with each other or above a stated limit */
    DPPO_ERR_MISALIGNED = -3,           /* base pointer or row stride not a multiple of 16 bytes      */
    DPPO_ERR_WORKSPACE_TOO_SMALL = -4,
    DPPO_ERR_UNSUPPORTED = -5,          /* dtype / option this build does not implement               */
    DPPO_ERR_CUDA = -6                  /* a CUDA runtime call failed (message has the CUDA error)    */
} dppo_error;

typedef enum {                          /* values of the device status word */
    DPPO_STATUS_OK = 0,
    DPPO_STATUS_BAD_LENGTH = 1,         /* pack: a retained unit has length < 1 or > L_row            */
    DPPO_STATUS_BAD_TARGET = 2,         /* loss: a target id outside [0, V)                           */
    DPPO_STATUS_TIMEOUT = 3,            /* a bounded device-side wait ran out                         */
    DPPO_STATUS_BAD_SEGMENTS = 4,       /* loss: cu_seqlens does not cover a token                    */
    DPPO_STATUS_BAD_INDEX = 5,          /* history: a prompt id outside the table                     */
    DPPO_STATUS_RANGE = 6               /* fused LM-head backward: a sampled token whose log-prob under the
                                           current policy is below about -66 (see dppo_lmhead_grpo_loss)  */
} dppo_status;

int dppo_version(void);                 /* major*10000 + minor*100 + patch */
const char* dppo_last_error(void);      /* host string, valid until the thread's next failing call */

/* ------------------------------------------------------------------------------------------------
 * Group-relative advantages — Eq. 2 (A_i = (r_i - mean)/std over the G completions of a prompt) and
 * the per-prompt threshold of Eq. 14 (Abar = mean_i |A_i|).
 *   rewards       f32 [P*G], row-major by prompt
 *   std_ddof      0 population std (default reading of "std"), 1 sample std
 *   std_eps       added to std before dividing (1e-6 by default; 0 allowed)
 *   adv           f32 [P*G] out;  mean_abs_adv f32 [P] out
 * A group whose rewards are all bitwise equal gets A = 0.  Arithmetic is binary64, one rounded
 * operation at a time in ascending i, rounded once to f32 — results are reproducible bit for bit.
 * Errors: INVALID_ARG (NULL, P<0, G<1, ddof not 0/1, eps<0).  P == 0 is a no-op.
 */
int dppo_group_advantages(const float* rewards, int P, int G, int std_ddof, double std_eps,
                          float* adv, float* mean_abs_adv, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Candidate sets, dynamic pruning masks, importance rescaling, history update —
 * Eq. 15 (completion policy), Eq. 17 (prompt policy), Eq. 18 (discrete rescaling), Eq. 16 (history).
 */
typedef struct {
    int32_t P, G;
    double r_q, r_o;        /* pruning probabilities in [0,1): a candidate is pruned when u < r      */
    int32_t mode;           /* 0: independent Bernoulli draws (Eq. 15, 17).
                               1: fixed fraction (Appendix A / Algorithm 1): prune the floor(r*|C|)
                                  candidates with the smallest u, ties to the lower index           */
    int32_t reverse;        /* 0: low-|A| completions / low-H prompts are the candidates (the paper's
                               rule); 1: the opposite sets (the ablation of Table 5)                 */
    uint64_t seed, step;    /* Philox4x32-10 key / counter words when u_q,u_o are NULL:
                               key=(seed lo,hi), counter=(index, domain, step lo, step hi),
                               domain 1 prompts (index k), 2 completions (index k*G+i);
                               u = ((out0 | out1<<32) >> 11) * 2^-53                                 */
} dppo_prune_params;

/*   adv, mean_abs_adv   outputs of dppo_group_advantages
 *   H_prev   f32 [P] history scores H_{t-1}(q_k); NULL in the first epoch: no prompt is a candidate
 *   u_q      f64 [P],  u_o f64 [P*G]: explicit draws in [0,1) replacing the generator (NULL: generate)
 *   cand_q   u8 [P]    the floor(P/2) prompts with the lowest H_prev (ties: lower index)
 *   cand_o   u8 [P*G]  |A_i| <= Abar_k, taken as G*|A_i| <= (sum_j |A_j|)*(1+1e-12) in binary64
 *   keep_q   u8 [P];  keep_o u8 [P*G] (all 0 for a pruned prompt)
 *   n_keep_q i32 [1] = |S^q|;  n_keep_o i32 [P] = |S^o(q_k)|
 *   gamma_q  f32 [P]   (|S^q|/P)/(1-P^q);  gamma_o f32 [P*G] (|S^o_k|/G)/(1-P^o); 0 where pruned
 *   w_seq    f32 [P*G] weight of a completion in the pruned objective read as the mean over retained
 *                      prompts of gamma_q x mean over retained completions of gamma_o x term:
 *                      1/(P*G*(1-P^q)*(1-P^o)); 0 where pruned
 *   H_next   f32 [P]   Abar_k if the prompt was retained (or H_prev is NULL), else H_prev[k]
 * In mode 1, P^q and P^o in these formulas are the realised fractions floor(r|C|)/|C| (the true
 * inclusion probabilities), so the weights stay unbiased.
 * Errors: INVALID_ARG (NULL outputs, r outside [0,1), bad mode), BAD_SHAPE (P*G >= 2^31).
 */
int dppo_prune_and_rescale(const dppo_prune_params* p, const float* adv, const float* mean_abs_adv,
                           const float* H_prev, const double* u_q, const double* u_o,
                           uint8_t* cand_q, uint8_t* cand_o, uint8_t* keep_q, uint8_t* keep_o,
                           int32_t* n_keep_q, int32_t* n_keep_o, float* gamma_q, float* gamma_o,
                           float* w_seq, float* H_next, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * History scores across epochs — Eq. 16 keeps one score H_t(q) per DATASET prompt; Algorithm 1 starts
 * from H_0 = 0 and skips prompt pruning in the first epoch.  A batch gathers the scores of its prompts
 * before dppo_prune_and_rescale (H_prev) and scatters H_next back afterwards: retained prompts get
 * their fresh mean |A|, pruned ones keep their old score (the carry-forward).
 *   H_table     f32 [N] one score per dataset prompt (caller zero-initialises it)
 *   prompt_ids  i32 [P] dataset index of each prompt of the batch (distinct within a batch)
 *   H_batch     f32 [P] out of gather;  H_next f32 [P] in to scatter
 * An id outside [0, N) sets status DPPO_STATUS_BAD_INDEX (gather returns 0 for it, scatter skips it).
 */
int dppo_history_gather(const float* H_table, int N, const int32_t* prompt_ids, int P, float* H_batch,
                        int32_t* status, void* stream);
int dppo_history_scatter(float* H_table, int N, const int32_t* prompt_ids, int P, const float* H_next,
                         int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Dense Prompt Packing — Section 4.3 (window-based greedy selection from a candidate pool W of
 * size N_win, refilled from the stream, into rows of capacity L_row).
 */
typedef struct {
    int32_t n_max;          /* units offered (retained or not)                                       */
    int32_t L_row;          /* row capacity in tokens                                                */
    int32_t N_win;          /* pool size, >= 1                                                       */
    int32_t policy;         /* 0 first unit in pool order that fits; 1 longest that fits (ties: oldest) */
} dppo_pack_params;

size_t dppo_pack_workspace_bytes(const dppo_pack_params* p);

/*   len        i32 [n_max] tokens of each unit (prompt + response)
 *   keep       u8  [n_max] or NULL: units with keep == 0 are not in the stream
 *   loss_len   i32 [n_max] or NULL: loss (response) tokens of each unit; NULL: = len
 *   order      i32 [n_max] out: order[p] = unit placed p-th, for p < n_units; -1 beyond
 *   row_of, off_in_row  i32 [n_max] out, indexed by unit; -1 for units not in the stream
 *   row_fill   i32 [n_max] out: tokens used in row r, for r < n_rows; 0 beyond
 *   cu_seqlens i32 [n_max+1] out: exclusive scan of loss_len in placement order; entries past
 *              n_units repeat the total, so the array is non-decreasing over its whole length
 *   counts     i32 [4] out: n_units, n_rows, total tokens, total loss tokens
 * A retained unit with length < 1 or > L_row sets status DPPO_STATUS_BAD_LENGTH and packs nothing
 * (counts = 0); so does a stream whose tokens add up to 2^31 or more (the counts are i32).  The limit is
 * n_max <= 2,097,152 units (a dataset-sized stream, packed once at set-up; one warp places about a million units
 * per second).  Errors: INVALID_ARG, BAD_SHAPE (n_max above the limit: the workspace query reports 0 bytes),
 * WORKSPACE_TOO_SMALL.
 */
int dppo_pack_prompts(const dppo_pack_params* p, const int32_t* len, const uint8_t* keep,
                      const int32_t* loss_len, int32_t* order, int32_t* row_of, int32_t* off_in_row,
                      int32_t* row_fill, int32_t* cu_seqlens, int32_t* counts,
                      void* workspace, size_t workspace_bytes, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Packing without a caller workspace.  (The paper has no counterpart: this entry point exists for the
 * sake of callers, not of the method.)
 *
 * Same operation, same arguments and same results as dppo_pack_prompts, minus `workspace`: the
 * scratch is a fixed 32 KB array inside the library's device image.  It is meant for callers that
 * have no way to hand over device scratch at the point of the call: host code that is given only
 * its input and output buffers by a framework and owns no allocator, or a training loop whose
 * device memory is entirely reserved by a pool, where a cudaMalloc would fail or would stall every
 * stream while it runs.  The call itself allocates nothing (no cudaMalloc / cudaFree, no library
 * allocation).
 *
 *  - Limit: n_max <= dppo_pack_static_max_units() (8192 units); larger requests return
 *    DPPO_ERR_BAD_SHAPE and launch nothing.  Every GPU that loads the library holds the 32 KB until
 *    the process ends, used or not.
 *  - The first call on each device looks up the array's device address (cudaGetSymbolAddress, with
 *    that device current) and caches it; make that first call before starting any stream capture.
 *    The cached address belongs to the device's context at that time: after cudaDeviceReset (or any
 *    other way of replacing that context) this entry point must not be used again in the process.
 *  - All calls on a device share the one array.  It keeps whatever the previous call left there;
 *    the kernel never reads a slot before writing it, so nothing needs clearing.  Two calls whose
 *    kernels can overlap on the GPU (different streams, no ordering between them) race on it:
 *    keep calls on one stream or order them yourself.
 */
int dppo_pack_static_max_units(void);
int dppo_pack_prompts_static(const dppo_pack_params* p, const int32_t* len, const uint8_t* keep,
                             const int32_t* loss_len, int32_t* order, int32_t* row_of,
                             int32_t* off_in_row, int32_t* row_fill, int32_t* cu_seqlens,
                             int32_t* counts, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Fused loss sweep over the logits — Eq. 1 (clipped surrogate minus beta x KL, 1/|o_i| per sequence,
 * KL estimator rho_hat - log rho_hat - 1) with the sequence weights of dppo_prune_and_rescale, and
 * its gradient with respect to the logits.
 *
 * For token t of sequence s (cu_seqlens[s] <= t < cu_seqlens[s+1]), target y, A = adv[s], W =
 * w[s]/|o_s|:  z = logits[t,:]/temperature;  lse = log sum_v exp z_v;  logp = z_y - lse;
 * rho = exp(logp - logp_old);  d = logp_ref - logp;  kl = e^d - d - 1;
 * surr = min(rho A, clip(rho, 1-eps_lo, 1+eps_hi) A);  loss = -sum_t W (surr - beta kl);
 * g = dloss/dlogp = -W (A rho [clipped branch not strictly smaller] + beta (e^d - 1));
 * dlogits[t,v] = g ([v == y] - exp(z_v - lse)) / temperature.
 */
typedef enum { DPPO_F32 = 0, DPPO_BF16 = 1 } dppo_dtype;

typedef struct {
    int64_t T_max;          /* rows of logits / upper bound of loss tokens                           */
    int32_t V;              /* vocabulary size                                                       */
    int32_t dtype;          /* dppo_dtype of logits and dlogits                                      */
    int64_t row_stride;     /* elements between consecutive rows (>= V; bytes a multiple of 16)      */
    int32_t S_max;          /* cu_seqlens has S_max+1 entries, non-decreasing, last >= true T        */
    int32_t variant;        /* 0: the library picks the kernel.  Tuning aid: 1 forces the general two-pass
                               kernel, 2 the warp-per-row kernel (rows up to 8 KB), 3 the streaming kernel (forward-only
                               calls), 4 the tile kernel (dense rows of up to 32 KB),
                               C*10000+threads the shared-memory kernel with C = 1, 2, 4 or 8
                               CTAs per row and 128 / 256 / 512 / 1024 threads per CTA.
                               Self-test of the bounded waits: 1000000 + (0, 3, 4 or a C*10000+threads code) runs
                               the shared-memory, streaming or tile kernel with a barrier expecting a few bytes
                               more than are ever sent and a wait limit of 1 ms: every row then ends as a
                               timed-out row does (status DPPO_STATUS_TIMEOUT; the row's dlogits, logp_out,
                               lse_out and loss terms are zero) and nothing hangs                    */
    double eps_lo, eps_hi;  /* clip range 1-eps_lo .. 1+eps_hi (the paper: both 0.2)                 */
    double beta;            /* KL coefficient                                                        */
    double temperature;     /* > 0 (the paper: 1)                                                    */
    /* Variants for the other objectives the paper combines the method with (Section 5.2); zero / NULL
       give Eq. 1 as printed. */
    int32_t no_length_norm; /* 1: W = w[s] instead of w[s]/|o_s| (a token-level mean is then up to the w
                               the caller passes)                                                    */
    int32_t reserved2;      /* 0                                                                     */
    const float* seq_log_ratio; /* device f32 [S_max] or NULL.  Given: every token of sequence s uses the
                               sequence-level ratio rho = exp(seq_log_ratio[s]) (from
                               dppo_sequence_log_ratio on the current log-probs, i.e. after a forward-only
                               call) in place of exp(logp - logp_old); requires no_length_norm == 0     */
} dppo_loss_params;

size_t dppo_grpo_loss_workspace_bytes(const dppo_loss_params* p);

/*   logits       [T_max x row_stride] of dtype, read-only unless dlogits aliases it
 *   target       i32 [T_max] sampled token ids
 *   logp_old, logp_ref  f32 [T_max] log-probs of the target under the old / reference policy
 *   cu_seqlens   i32 [S_max+1]
 *   n_tokens_dev i32 [1] true number of tokens T <= T_max on the device, or NULL (T = T_max);
 *                rows >= T are neither read nor written
 *   adv, w       f32: advantage and sequence weight of each sequence, read at index seg_map[s]
 *                when seg_map (i32 [S_max], e.g. the packer's `order`) is given, else at index s
 *   dlogits      same dtype/stride as logits; may alias logits (in place); NULL: forward only
 *   logp_out, lse_out   f32 [T_max] or NULL
 *   loss_out     f32 [5]: loss, policy-gradient part -sum W surr, sum W kl, clipped fraction, T
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED (logits/dlogits base or row stride), UNSUPPORTED
 * (dtype), WORKSPACE_TOO_SMALL.  Device status: BAD_TARGET, BAD_SEGMENTS (a row below T that cu_seqlens does not
 * cover): such a row's dlogits are zero, its logp_out is 0 (its lse_out is still the row's log-sum-exp) and it adds
 * nothing to the loss; the other rows are not affected.
 */
int dppo_grpo_loss_fwd_bwd(const dppo_loss_params* p, const void* logits, const int32_t* target,
                           const float* logp_old, const float* logp_ref, const int32_t* cu_seqlens,
                           const int32_t* n_tokens_dev, const float* adv, const float* w,
                           const int32_t* seg_map, void* dlogits, float* logp_out, float* lse_out,
                           float* loss_out, void* workspace, size_t workspace_bytes,
                           int32_t* status, void* stream);

/* Which kernel a dppo_grpo_loss_fwd_bwd call with these parameters runs on the current device (a host-side query:
 * it makes the same choice and the same device checks as the call and launches nothing).  Dense rows (V a whole
 * number of 16-byte vectors) of up to 16 KB go to the tile kernel.  Other rows of
 * up to 8 KB go to the warp-per-row kernel, rows that fit eight shared-memory slices to the shared-memory
 * kernel, longer ones to the general two-pass kernel; a forward-only call (forward_only != 0: the call will pass
 * dlogits = NULL) on rows of 128 KB and more goes to the streaming kernel.  fell_back = 1 says that the device refused the kernel the
 * row length asked for (its shared memory or cluster size) and the slower general kernel runs instead.
 * Errors: INVALID_ARG; UNSUPPORTED when params.variant forces a kernel that cannot take the shape.
 */
typedef enum { DPPO_KERNEL_GENERAL = 0, DPPO_KERNEL_WARP = 1, DPPO_KERNEL_SHARED = 2, DPPO_KERNEL_STREAM = 3, DPPO_KERNEL_TILE = 4 } dppo_loss_kernel;
typedef struct {
    int32_t kernel;         /* dppo_loss_kernel                                                      */
    int32_t ctas_per_row;   /* cluster size of the shared-memory kernel, else 1                      */
    int32_t threads;        /* threads that work on one row at a time in each CTA                    */
    int32_t fell_back;      /* 1: general kernel in place of the one the row length asked for        */
} dppo_loss_kernel_choice;
int dppo_grpo_loss_kernel_choice(const dppo_loss_params* p, int forward_only, dppo_loss_kernel_choice* out);

/* Mean token log-ratio of each sequence, out[s] = mean_t (logp[t] - logp_old[t]) over cu_seqlens[s] <= t <
 * cu_seqlens[s+1] (0 for an empty sequence): the log of the length-normalised sequence-level likelihood
 * ratio of sequence-level objectives (Section 5.2).  logp, logp_old f32 [T]; out f32 [S_max].  Binary64
 * accumulation in a fixed order.  Errors: INVALID_ARG.
 */
int dppo_sequence_log_ratio(const float* logp, const float* logp_old, const int32_t* cu_seqlens, int S_max,
                            float* out, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Fused LM-head + loss: the same loss as dppo_grpo_loss_fwd_bwd with the logits z = hidden W^T
 * produced on the fly by the tensor cores; the [T x V] logits of the batch are never written to memory
 * (Eq. 1's pi_theta is the log-softmax of exactly these logits).
 *
 *   loss     the loss parameters; dtype must be DPPO_BF16; row_stride and variant are ignored
 *   H        hidden width, a multiple of 64
 *   hidden   bf16 [T_max x H] row-major, one row per loss token in packed order
 *   W        bf16 [V x H] row-major LM-head weight
 *   backward 0: forward only (loss_out, logp_out, lse_out; dhidden and dW must be NULL).
 *            1: also the gradients, dhidden = D W and dW = D^T hidden with D = dlogits.  The tokens are taken 9472
 *            at a time.  A chunk's exponentials are kept in workspace scratch as bf16, relative to each row's own
 *            reference, the sampled token's logit (never the full [T x V], and never the logits themselves); D is
 *            that scratch times one factor per row, so the two contractions read the scratch directly and no
 *            dlogits array is formed.  The reference bounds the representable rows: a sampled token whose log-prob
 *            under the current policy is below about -66 sets status DPPO_STATUS_RANGE; that row adds nothing to
 *            the loss and its gradient is zero
 *   dhidden  bf16 [T_max x H] out (rows at or past the true token count are zero)
 *   dW       [V x H] out, f32 or (params.dW_dtype = DPPO_BF16) bf16; overwritten, or added to when
 *            params.accumulate_dW = 1.  It is summed over the chunks in f32 either way (for bf16 in a workspace
 *            buffer, rounded once at the end).  Each element receives one add per chunk, in stream order: the
 *            result does not vary from run to run
 *   other arguments as in dppo_grpo_loss_fwd_bwd.  The workspace (dppo_lmhead_workspace_bytes, which
 *   depends on `backward`) must be 1024-byte aligned.
 * Errors: INVALID_ARG, BAD_SHAPE (H not a multiple of 64), MISALIGNED, UNSUPPORTED, WORKSPACE_TOO_SMALL,
 * CUDA (tensor-map creation).  Device status: BAD_TARGET, BAD_SEGMENTS, RANGE, TIMEOUT.
 */
typedef struct {
    dppo_loss_params loss;
    int32_t H;
    int32_t backward;
    int32_t variant;        /* 0: CTA pairs (cta_group::2) share each B tile; 1: one CTA per tile (tuning aid).
                               100 / 101: the same two with the self-test of the bounded waits: the first pipeline
                               stage of every CTA expects 16 bytes more than are ever copied and the wait limit
                               is 1 ms, so every CTA gives up, frees its tensor memory and returns; the call
                               reports DPPO_STATUS_TIMEOUT and its other outputs are unspecified    */
    int32_t dW_dtype;       /* DPPO_F32 (0) or DPPO_BF16: element type of dW */
    int32_t accumulate_dW;  /* 0: dW is overwritten; 1: the gradient is added to what dW holds (micro-batches) */
    int32_t reserved;       /* 0 */
} dppo_lmhead_params;

size_t dppo_lmhead_workspace_bytes(const dppo_lmhead_params* p);

int dppo_lmhead_grpo_loss(const dppo_lmhead_params* p, const void* hidden, const void* W,
                          const int32_t* target, const float* logp_old, const float* logp_ref,
                          const int32_t* cu_seqlens, const int32_t* n_tokens_dev, const float* adv,
                          const float* w, const int32_t* seg_map, void* dhidden, void* dW,
                          float* logp_out, float* lse_out, float* loss_out, void* workspace,
                          size_t workspace_bytes, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Scoring: log-probs of GIVEN tokens, with the entropy of their distribution and its top alternatives.
 * This is where the loss's logp_old and logp_ref come from (pi_theta_old and pi_ref of Eq. 1 at the sampled
 * tokens), and what a training loop reports beside them.
 *
 * Row t, tau = temperature, m = max_v z_v, l = ln sum_v exp((z_v - m)/tau), p_v = exp((z_v - m)/tau - l):
 *   lse = m/tau + l;   logp = (z_y - m)/tau - l;   entropy = l - sum_v p_v (z_v - m)/tau   (p ln p = 0 at p = 0)
 *   alternatives: the top_k largest z_v in descending order, ties to the lower index, with their log-probs.
 * Entries at -inf are masked: probability 0, never an alternative (a row with fewer than top_k others is filled
 * up with id -1, log-prob -inf).  A row that its mask leaves empty has lse = logp = -inf, entropy 0.  A row with a
 * NaN or +inf has NaN for all of these and ids -1.
 */
typedef struct {
    int64_t T_max;          /* rows of logits / upper bound of tokens                                */
    int32_t V;              /* vocabulary size, up to 2^30                                           */
    int32_t dtype;          /* dppo_dtype of logits and dlogits                                      */
    int64_t row_stride;     /* elements between consecutive rows (>= V; bytes a multiple of 16)      */
    int32_t top_k;          /* alternatives per row, 0..32 (the backward ignores it)                 */
    int32_t variant;        /* 0: the library picks the launch shape.  Tuning aid of the forward:
                               C*10000 + threads: C = 1, 2, 4 or 8 CTAs per row with 128, 256 or 512
                               threads each; 32: one warp per row                                    */
    double temperature;     /* 1e-6 .. 1e6                                                           */
} dppo_logprob_params;

/*   logits       [T_max x row_stride] of dtype
 *   target       i32 [T_max] token ids, or NULL (then logp_out is NULL)
 *   n_tokens_dev i32 [1] true number of tokens T <= T_max on the device, or NULL (T = T_max);
 *                rows >= T are neither read nor written, in any array
 *   logp_out, entropy_out, lse_out   f32 [T_max] or NULL
 *   top_ids      i32 [T_max x top_k], top_logp f32 [T_max x top_k]; NULL if and only if top_k = 0
 *   stats        f32 [T_max x 4] or NULL: {m, l, entropy, 0} of each row for the backward call (m = -inf for a
 *                row that its mask leaves empty)
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED (logits base or row stride, stats base), UNSUPPORTED (dtype, variant).
 * Device status: BAD_TARGET (the row's logp is 0; its other outputs are not affected).
 */
int dppo_token_logprobs(const dppo_logprob_params* p, const void* logits, const int32_t* target,
                        const int32_t* n_tokens_dev, float* logp_out, float* entropy_out, float* lse_out,
                        int32_t* top_ids, float* top_logp, float* stats, int32_t* status, void* stream);

/* Gradient of the scoring call with respect to the logits, for a = dL/dlogp and b = dL/dentropy of each row:
 *   dlogits[t, v] = (a ([v == y] - p_v) - b p_v (ln p_v + entropy)) / tau
 * The probabilities are recomputed from the logits and the forward's stats: one read and one write of the rows.
 * One below 2^-126 counts as 0.
 *   dlogp, dentropy  f32 [T_max], either may be NULL (that term is absent); dlogp needs target
 *   dlogits      same dtype / stride as logits; may alias logits (in place).  Columns at or past V are not written.
 * A row that its mask leaves empty has a zero gradient.
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED, UNSUPPORTED (dtype).  Device status: BAD_TARGET (the row is zero).
 */
int dppo_token_logprobs_backward(const dppo_logprob_params* p, const void* logits, const int32_t* target,
                                 const int32_t* n_tokens_dev, const float* stats, const float* dlogp,
                                 const float* dentropy, void* dlogits, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Matrix product in 8-bit integers with one scale per token and one per output channel: the LM-head (or any
 * projection) of a frozen policy whose log-probs are only scored.
 *
 * Quantisation of rows, symmetric: s = fl32(max_k |x_k| fl32(1/127)), q_k = clamp(rint(fl32(x_k / s)), -127, 127)
 * (ties to even); s = 0 gives q = 0.  A row with a NaN or an infinity gets s = NaN, q = 0, so that products with it are NaN.
 */
typedef struct {
    int64_t rows_max;       /* rows of x (below 2^31)                                                */
    int32_t K;              /* columns, up to 2^30                                                   */
    int32_t dtype;          /* dppo_dtype of x                                                       */
    int64_t x_stride;       /* elements between rows of x (>= K; bytes a multiple of 16)             */
    int64_t q_stride;       /* bytes between rows of q (>= K; a multiple of 16)                      */
} dppo_quantize_params;

/*   x   [rows_max x x_stride] of dtype;  q  i8 [rows_max x q_stride] out (columns at or past K are not written);
 *   scale  f32 [rows_max] out;  n_rows_dev  i32 [1] true number of rows or NULL; rows past it are not touched
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED, UNSUPPORTED (dtype).
 */
int dppo_quantize_rows_i8(const dppo_quantize_params* p, const void* x, int8_t* q, float* scale,
                          const int32_t* n_rows_dev, int32_t* status, void* stream);

/*   out[t, n] = fl32(fl32(x_scale[t] w_scale[n]) fl32(sum_k x[t, k] w[n, k])), rounded once more to a bf16 out.
 * The sum is an exact 32-bit integer (K <= 131,071), so the result does not depend on the order of its terms. */
typedef struct {
    int64_t M_max;          /* rows of x / upper bound of tokens (below 2^31)                        */
    int32_t N, K;           /* output channels; contraction length                                   */
    int64_t x_stride, w_stride;   /* bytes between rows of x and of w (>= K; multiples of 16)        */
    int64_t out_stride;     /* elements between rows of out (>= N)                                   */
    int32_t out_dtype;      /* dppo_dtype of out                                                     */
    int32_t variant;        /* 0: the library picks the kernel; 1 forces the CTA-pair tile kernel, 2 the
                               kernel for few tokens (tuning aid).  101 / 102: the same two with the
                               self-test of the bounded waits (see dppo_lmhead_params.variant): the call
                               reports DPPO_STATUS_TIMEOUT, its output is unspecified                */
} dppo_linear_i8_params;

/*   x   i8 [M_max x x_stride], x_scale f32 [M_max];  w  i8 [N x w_stride], w_scale f32 [N]
 *   out [M_max x out_stride] of out_dtype (no alignment beyond its element's)
 *   n_rows_dev  i32 [1] true number of tokens on the device, or NULL; rows of out past it are not written
 * Codes of -128 are allowed.  Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED (x, w: base or stride), UNSUPPORTED,
 * CUDA (tensor-map creation).  Device status: TIMEOUT.
 */
int dppo_linear_i8(const dppo_linear_i8_params* p, const int8_t* x, const float* x_scale, const int8_t* w,
                   const float* w_scale, void* out, const int32_t* n_rows_dev, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Distillation from a teacher's top log-probs (what dppo_token_logprobs returns for another policy: top_ids, top_logp).
 *
 * Row t lists top_k tokens i_j with the teacher's log-probs; an id of -1 is no entry.  p_j = exp(top_logp_j), s = softmax(z / tau)
 * of the student's logits z, sigma = the sum of s over the tokens that are not listed.
 *   loss = sum_j p_j (ln p_j - ln s_{i_j})          p ln p = 0 at p = 0
 *   mode GIVEN: as it stands;  NORMALIZED: with p_j / sum_j p_j in place of p_j;
 *   REST: plus r (ln r - ln sigma) for the teacher's remainder r = 1 - sum_j p_j; an r up to 2^-16 counts as 0 (that is the
 *         rounding of f32 log-probs)
 *   dloss/dz_v = (G s_v - sum_{j: i_j = v} p_j - [v not listed] s_v r / sigma) / tau,   G = sum_j p_j + r  (r = 0 but in REST)
 * A token listed twice counts with both log-probs, and once in sigma.  A row without entries has loss 0 and a zero gradient.
 * Logits at -inf are masked: probability 0; a listed one with p > 0 makes the loss +inf (its gradient stays finite).  A row that
 * its mask leaves empty has lse = -inf, loss +inf (0 if all p are 0) and a zero gradient.  A row with a NaN or +inf has NaN for
 * all of these.  sigma is summed from its own terms, not taken as 1 minus the others.
 */
typedef enum { DPPO_DISTILL_GIVEN = 0, DPPO_DISTILL_NORMALIZED = 1, DPPO_DISTILL_REST = 2 } dppo_distill_mode;

typedef struct {
    int64_t T_max;          /* rows of logits / upper bound of tokens                                */
    int32_t V;              /* vocabulary size, up to 2^20                                           */
    int32_t dtype;          /* dppo_dtype of logits and dlogits                                      */
    int64_t row_stride;     /* elements between consecutive rows (>= V; bytes a multiple of 16)      */
    int32_t top_k;          /* teacher entries per row, 1..128                                       */
    int32_t mode;           /* dppo_distill_mode                                                     */
    double temperature;     /* of the student, 1e-6 .. 1e6; the teacher's log-probs are taken as they are */
} dppo_distill_params;

/*   logits       [T_max x row_stride] of dtype: the student's
 *   top_ids      i32 [T_max x top_k], top_logp f32 [T_max x top_k]
 *   n_tokens_dev i32 [1] true number of tokens T <= T_max on the device, or NULL (T = T_max);
 *                rows >= T are neither read nor written, in any array
 *   weight       f32 [T_max] or NULL (1): dL/dloss of each row, for dlogits; the loss is written without it
 *   loss_out, lse_out   f32 [T_max] or NULL
 *   stats        f32 [T_max x 4]: {m, S, G, r / sigma} of each row for the backward call (m the largest logit, S = sum_v
 *                exp((z_v - m) / tau); -log2(r / sigma - G) in place of r / sigma where r / sigma - G is above 16); may be NULL without
 *                dlogits
 *   dlogits      NULL (loss alone), or the gradient in the same call: same dtype / stride as logits; may alias logits (in
 *                place).  Columns at or past V are not written.
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED (logits, dlogits, stats: base or row stride), UNSUPPORTED (dtype).
 * Device status: BAD_TARGET (an id below -1 or at or past V: the row's loss is 0 and its gradient zero).
 */
int dppo_distill_topk(const dppo_distill_params* p, const void* logits, const int32_t* top_ids, const float* top_logp,
                      const int32_t* n_tokens_dev, const float* weight, float* loss_out, float* lse_out, float* stats,
                      void* dlogits, int32_t* status, void* stream);

/* The gradient alone, for dloss = dL/dloss of each row (f32 [T_max], NULL: 1) and the stats of a dppo_distill_topk call with the
 * same arguments: one read and one write of the rows.  dlogits may alias logits.  Errors and status as above.
 */
int dppo_distill_topk_backward(const dppo_distill_params* p, const void* logits, const int32_t* top_ids, const float* top_logp,
                               const int32_t* n_tokens_dev, const float* stats, const float* dloss, void* dlogits,
                               int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Verification of drafted tokens (an earlier completion, a smaller model's proposal) against the target policy, from given random
 * numbers: the accepted tokens and the one after them are distributed as the target's own samples.
 *
 * Sequence b has the drafts y_j, j < n, n = cu_drafts[b + 1] - cu_drafts[b], at cu_drafts[b] + j; rows of the target (and of its outputs)
 * lie at cu_drafts[b] + b + j, j = 0 .. n: one more than drafts.  p_j = softmax(target row / temperature); q_j = softmax(draft row /
 * draft_temperature), or, without draft logits, 1 at y_j (drafts copied from somewhere).
 *   y_j is accepted while u_j q_j(y_j) < p_j(y_j).
 *   After a first rejection at j the next token is argmax_v max(p_j(v) - q_j(v), 0) / e_b(v) (if p_j <= q_j everywhere:
 *   argmax_v p_j(v) / e_b(v)), after n acceptances argmax_v p_n(v) / e_b(v); ties to the lower index.  With independent u uniform
 *   in [0, 1) and e exponential that is a sample.  Softmax sums are f32 (about 1e-6 off); all else is decided as in 64 bits.
 *   tokens_out: the accepted drafts, the next token, then -1;  logp_out: their log-probs under the target, then 0.
 * Logits at -inf are masked.  A draft row that its mask leaves empty has q = 0.  At a row with a NaN or +inf, the target's or the draft's,
 * the sequence ends: next token -1, log-prob NaN.  A target row that its mask leaves empty: next token -1, log-prob -inf.
 */
typedef struct {
    int64_t T_max;          /* drafts of all sequences, upper bound                                  */
    int32_t n_seqs;
    int32_t V;              /* vocabulary size, up to 2^30                                           */
    int32_t dtype;          /* dppo_dtype of both policies' logits                                   */
    int64_t target_stride, draft_stride;  /* elements between rows (>= V; bytes a multiple of 16)    */
    int64_t noise_stride;   /* elements between rows of noise (>= V; a multiple of 4)                */
    double temperature, draft_temperature;      /* 1e-6 .. 1e6                                       */
} dppo_verify_params;

size_t dppo_verify_drafts_workspace_bytes(const dppo_verify_params* p);

/*   target_logits [(T_max + n_seqs) x target_stride], draft_logits [T_max x draft_stride] or NULL, of dtype
 *   drafts        i32 [T_max];  cu_drafts i32 [n_seqs + 1], non-decreasing from 0, the last at most T_max; rows past the last
 *                 sequence are neither read nor written
 *   uniforms      f32 [T_max] in [0, 1);  noise f32 [n_seqs x noise_stride], positive, of any size (entries whose noise is outside
 *                 [2^-64, 2^13] are compared in 64 bits, which takes longer)
 *   n_accepted    i32 [n_seqs] out;  tokens_out i32, logp_out f32 [T_max + n_seqs] out
 *   workspace     at least dppo_verify_drafts_workspace_bytes, 16-byte aligned
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED, UNSUPPORTED (dtype), WORKSPACE_TOO_SMALL.
 * Device status: BAD_TARGET (a drafted id outside [0, V) is rejected), BAD_SEGMENTS (cu_drafts decreases, or ends past T_max: such a
 * sequence has n_accepted 0 and no other output).
 */
int dppo_verify_drafts(const dppo_verify_params* p, const void* target_logits, const void* draft_logits, const int32_t* drafts,
                       const int32_t* cu_drafts, const float* uniforms, const float* noise, int32_t* n_accepted, int32_t* tokens_out,
                       float* logp_out, void* workspace, size_t workspace_bytes, int32_t* status, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Matrix product in 8-bit floating point (e4m3) with a scale for each block of 128 of the contraction: the LM-head (or any projection)
 * of a frozen policy or teacher.  Finer scales than dppo_linear_i8's: a channel far larger than the others costs only its own
 * block digits.
 *
 * Quantisation of a block (block_rows = 1: 128 columns of a row; 128: 128 rows x 128 columns; less at the edges):
 * s = max(fl32(max |x| fl32(1/448)), 2^-126), q = e4m3(fl32(x / s)) (nearest, ties to even, held at +-448).  A block with a NaN or an
 * infinity gets s = NaN, q = 0, so that products with it are NaN.
 */
typedef struct {
    int64_t rows_max;       /* rows of x (below 2^31)                                                */
    int32_t K;              /* columns, up to 2^30                                                   */
    int32_t dtype;          /* dppo_dtype of x                                                       */
    int64_t x_stride;       /* elements between rows of x (>= K; bytes a multiple of 16)             */
    int64_t q_stride;       /* bytes between rows of q (>= K; a multiple of 16)                      */
    int64_t scale_stride;   /* block_rows = 1: elements between the scales of consecutive blocks of columns (>= rows_max);
                               128: between those of consecutive blocks of rows (>= ceil(K / 128))   */
    int32_t block_rows;     /* 1 or 128                                                              */
} dppo_quantize_f8_params;

/*   x   [rows_max x x_stride] of dtype;  q  e4m3 [rows_max x q_stride] out (columns at or past K are not written)
 *   scale  f32 out, block_rows = 1: [ceil(K / 128) x scale_stride], the scales of a block of columns side by side for the rows;
 *          128: [ceil(rows_max / 128) x scale_stride]
 *   n_rows_dev  i32 [1] true number of rows or NULL; rows (and blocks) past it are not touched
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED, UNSUPPORTED (dtype, block_rows).
 */
int dppo_quantize_f8(const dppo_quantize_f8_params* p, const void* x, uint8_t* q, float* scale, const int32_t* n_rows_dev,
                     int32_t* status, void* stream);

/*   out[t, n] = sum_B x_scale[B, t] w_scale[n / 128, B] sum_{k in block B} x[t, k] w[n, k], the blocks' sums and their sum in f32,
 * rounded once more to a bf16 out.  The order of the sums is a function of the sizes (M_max, not the true count), of variant, of out's type and of
 * whether its base and rows lie on 16 bytes. */
typedef struct {
    int64_t M_max;          /* rows of x / upper bound of tokens (below 2^31)                        */
    int32_t N, K;           /* output channels; contraction length                                   */
    int64_t x_stride, w_stride;   /* bytes between rows of x and of w (>= K; multiples of 16)        */
    int64_t out_stride;     /* elements between rows of out (>= N)                                   */
    int64_t x_scale_stride; /* elements between rows of x_scale (>= M_max; a multiple of 4)          */
    int64_t w_scale_stride; /* elements between rows of w_scale (>= ceil(K / 128))                   */
    int32_t out_dtype;      /* dppo_dtype of out                                                     */
    int32_t variant;        /* 0: the library picks the kernel; 1 forces the CTA-pair tile kernel, 2 the
                               kernel for few tokens (tuning aid).  101 / 102: the same two with the
                               self-test of the bounded waits (see dppo_lmhead_params.variant): the call
                               reports DPPO_STATUS_TIMEOUT, its output is unspecified                */
} dppo_linear_f8_params;

/*   x   e4m3 [M_max x x_stride], x_scale f32 [ceil(K / 128) x x_scale_stride];  w  e4m3 [N x w_stride], w_scale f32
 *   [ceil(N / 128) x w_scale_stride]: as dppo_quantize_f8 leaves them
 *   out [M_max x out_stride] of out_dtype (no alignment beyond its element's)
 *   n_rows_dev  i32 [1] true number of tokens on the device, or NULL; rows of out past it are not written
 * Errors: INVALID_ARG, BAD_SHAPE, MISALIGNED (x, w, x_scale: base or stride), UNSUPPORTED, CUDA (tensor-map creation).  Device status:
 * TIMEOUT.
 */
int dppo_linear_f8(const dppo_linear_f8_params* p, const uint8_t* x, const float* x_scale, const uint8_t* w, const float* w_scale,
                   void* out, const int32_t* n_rows_dev, int32_t* status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DPPO_H_ */
