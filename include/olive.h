/*
 * olive.h -- C ABI of libolive.so, the GB300 (sm_103a) implementation of the
 * per-token scoring path of OLIVE ("Learning from Teacher Continuations at
 * Student States").
 *
 * The path: a student prefix (prompt x and student tokens y_{1:k}) is cut at a
 * student state and followed by a teacher continuation y~_{1:l}; the student
 * is trained with the masked cross-entropy of Eq. (osd-ce) (Section 3.1) on the
 * continuation tokens only.  The OPD baseline (Section 1) scores tokens with a
 * per-token reverse KL against the teacher instead.  Four calls cover it:
 *
 *   olive_splice_pack        packs the spliced sequences and builds the loss mask
 *   olive_token_logprob_fwd  LM-head projection + online log-sum-exp + masked
 *                            target log-prob and loss (the [T,V] logits are
 *                            never stored)
 *   olive_token_loss_bwd     d loss / d hidden and d loss / d W
 *   olive_token_divergence   full-vocabulary per-token KL (+ d KL / d h_s)
 *
 * and these extend it:
 *
 *   olive_token_loss_fwd_bwd the forward and backward of a training step in
 *                            one call, G formed and consumed on chip
 *   olive_token_loss_fwd_bwd_slab  the same step through an HBM slab of G
 *                            (no logit recomputation)
 *   olive_splice_pack_masked multi-turn packing, loss only on teacher actions
 *                            (Section 3.2)
 *   olive_token_topk_fwd     per-token entropy and top-K log-probs
 *   olive_topk_compare       student/teacher top-K overlap and top-K KL
 *   olive_topk_kl_bwd        gradient of the top-K KL
 *   olive_topk_kl_fwd_bwd    the student's top-K lists, the top-K KL and its
 *                            gradient from one sweep of the student's logits
 *   olive_opd_token_stats    OPD's per-token KL, entropy, top-K lists, overlap
 *                            and top-K KL from one sweep with both heads
 *   olive_token_logprob_fwd_noalloc  the forward without a workspace
 *
 * The hidden rows come out of a decoder layer and the gradients go into an
 * optimiser.  The parts of that way which meet the packed batch have calls too
 * (the paper trains such students, Appendix A, and prints none of them):
 *
 *   olive_packed_positions   position of every packed token in its sequence
 *   olive_qk_norm_rope_fwd, olive_qk_norm_rope_bwd
 *                            RMS norm of each query and key head and rotation
 *                            by position, in one pass
 *   olive_gated_mlp_fwd, olive_gated_mlp_bwd
 *                            gated feed-forward block with its residual
 *   olive_grad_clip          global norm of a list of gradients, and clipping
 *   olive_grad_clip_apart    whether such a list may be scaled (a host check)
 *   olive_embedding_fwd, olive_embedding_bwd
 *                            rows of the embedding by packed ids, and its
 *                            gradient by sorted tokens
 *   olive_packed_attention_fwd, olive_packed_attention_bwd
 *                            attention of packed tokens to their own sequence
 *   olive_row_norm_fwd, olive_row_norm_bwd
 *                            layer norm or RMS norm of the rows, with the
 *                            residual's sum on the way
 *
 * Conventions shared by every call
 *   - Every pointer argument is a DEVICE pointer unless stated otherwise.  The
 *     caller owns every buffer; no call allocates device memory.  Scratch
 *     memory comes from the caller's `workspace` (size from
 *     olive_workspace_size, 256-byte aligned).  Three things outlive a call:
 *     the OLIVE_NOALLOC_SCRATCH_BYTES array that olive_token_logprob_fwd_noalloc
 *     uses (compiled into the library, held by every GPU that loads it); the
 *     per-device kernel attributes (shared-memory limits), set on the first
 *     call on each device so that later calls issue no attribute call and can
 *     be captured in a CUDA graph (the on-chip training step also checks
 *     there, once, that the device holds its whole grid of CTA pairs at
 *     once); and two environment variables, read at each call:
 *     OLIVE_WAIT_LIMIT_MS (wall-clock limit of every internal wait, default
 *     1000; on expiry the call sets OLIVE_ERR_TIMEOUT) and OLIVE_SLAB_ROWS
 *     (lowers the slab of the slab forms, see olive_slab_rows).
 *   - `stream` is a cudaStream_t (NULL = legacy default stream).  All calls
 *     are asynchronous on it; none synchronises the host.
 *   - The returned olive_status covers what the host can check before any
 *     launch (null pointers, shapes, alignment, device).  On any non-OK
 *     return nothing was launched.
 *   - Errors in device data (a token id outside [0,V), offsets that do not
 *     describe the batch, an internal wait that ran out of time) are OR-ed
 *     into *dev_status as bits (1u << code), code from olive_status.  The
 *     caller zeroes *dev_status and reads it whenever it synchronises.
 *   - Row counts such as N_mask stay on the device (`n_rows`), so the three
 *     compute calls can follow olive_splice_pack without a host round trip;
 *     grids are sized from the host-side upper bound T.
 *   - Tensors are row-major and contiguous.  bf16 is IEEE bfloat16.  Base
 *     pointers of hidden, W, d_hidden and d_W must be 16-byte aligned, and
 *     d (every hidden width) must be a multiple of 8.
 *   - The library runs only on compute capability 10.3 (sm_103a).
 */
#ifndef OLIVE_H_
#define OLIVE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define OLIVE_API __attribute__((visibility("default")))
#else
#define OLIVE_API
#endif

#define OLIVE_ABI_VERSION 1

typedef enum {
  OLIVE_OK = 0,
  OLIVE_ERR_INVALID_ARG = 1,       /* null pointer, bad enum value            */
  OLIVE_ERR_SHAPE = 2,             /* non-positive or too large size          */
  OLIVE_ERR_ALIGNMENT = 3,         /* pointer or width breaks the 16-B rule   */
  OLIVE_ERR_TOKEN_RANGE = 4,       /* (device) an id or target outside [0,V)  */
  OLIVE_ERR_OFFSETS = 5,           /* (device) offsets / row list malformed   */
  OLIVE_ERR_TIMEOUT = 6,           /* (device) an internal wait ran out       */
  OLIVE_ERR_UNSUPPORTED_DEVICE = 7,/* current device is not sm_103           */
  OLIVE_ERR_CUDA = 8,              /* a CUDA runtime/driver call failed       */
  OLIVE_ERR_WORKSPACE = 9,         /* workspace null, misaligned or too small */
  OLIVE_ERR_BOUNDS = 10            /* (device, OLIVE_DEBUG builds only) an index
                                      check failed; the access was skipped      */
} olive_status;

enum { OLIVE_REDUCE_SUM = 0, OLIVE_REDUCE_MEAN = 1 };
enum { OLIVE_KL_REVERSE = 0, OLIVE_KL_FORWARD = 1 };
enum { OLIVE_DTYPE_BF16 = 0, OLIVE_DTYPE_F32 = 1 };
enum { OLIVE_ACT_SILU = 0, OLIVE_ACT_GELU_TANH = 1 };
enum { OLIVE_NORM_LAYER = 0, OLIVE_NORM_RMS = 1 };
enum { OLIVE_OP_LOGPROB_FWD = 0, OLIVE_OP_LOSS_BWD = 1, OLIVE_OP_DIVERGENCE = 2,
       OLIVE_OP_TOPK_FWD = 3, OLIVE_OP_SPLICE_MASKED = 4, OLIVE_OP_TOPK_KL_BWD = 5,
       OLIVE_OP_LOSS_FWD_BWD = 6, OLIVE_OP_OPD_STATS = 7, OLIVE_OP_TOPK_KL_FWD_BWD = 8,
       OLIVE_OP_LOSS_FWD_BWD_SLAB = 9, OLIVE_OP_GATED_MLP_FWD = 10,
       OLIVE_OP_GATED_MLP_BWD = 11, OLIVE_OP_QK_NORM_ROPE_BWD = 12, OLIVE_OP_GRAD_CLIP = 13,
       OLIVE_OP_ROW_NORM_BWD = 14, OLIVE_OP_EMBEDDING_BWD = 15,
       OLIVE_OP_PACKED_ATTENTION_BWD = 16 };

/*
 * Rows of the G slab that the slab forms (olive_token_loss_fwd_bwd_slab,
 * olive_topk_kl_bwd, olive_topk_kl_fwd_bwd) hold at a time for T packed rows
 * and V vocabulary
 * entries: about 5.6 GB of bf16 G in whole 128-row tiles, at most 32768 rows
 * and at most T rounded up to 128, lowered by OLIVE_SLAB_ROWS (a multiple of
 * 128).  A call on more masked rows runs ceil(N_mask / rows) slabs.  Returns 0
 * for T < 1 or V < 1.  The paper has no counterpart.
 */
OLIVE_API int32_t olive_slab_rows(int32_t T, int32_t V);

/* ABI version of the loaded library (OLIVE_ABI_VERSION). */
OLIVE_API int olive_abi_version(void);

/* Static text for a status code. Never NULL. */
OLIVE_API const char* olive_status_string(olive_status s);

/* Zeroes a device status word on `stream` (asynchronous). */
OLIVE_API olive_status olive_status_clear(int32_t* dev_status, void* stream);

/*
 * Workspace bytes a compute call needs for host-side upper bound T rows.
 *   op  OLIVE_OP_LOGPROB_FWD / OLIVE_OP_LOSS_BWD: d = hidden width, d_t ignored.
 *   op  OLIVE_OP_DIVERGENCE: d = student width d_s, d_t = teacher width.
 *   op  OLIVE_OP_TOPK_FWD: d = hidden width, d_t ignored.
 *   op  OLIVE_OP_SPLICE_MASKED: T = T_cap; d, d_t, V ignored.
 *   op  OLIVE_OP_OPD_STATS: d = student width d_s, d_t = teacher width.
 *   op  OLIVE_OP_TOPK_KL_BWD, OLIVE_OP_LOSS_FWD_BWD,
 *       OLIVE_OP_TOPK_KL_FWD_BWD: d = (student) hidden width, grad_dtype as
 *       for OLIVE_OP_LOSS_BWD, d_t ignored.
 *   op  OLIVE_OP_GATED_MLP_FWD / OLIVE_OP_GATED_MLP_BWD: d = hidden width,
 *       V = inner width f, d_t ignored.
 *   op  OLIVE_OP_QK_NORM_ROPE_BWD: d = head width; the rest ignored.
 *   op  OLIVE_OP_GRAD_CLIP: T = number of tensors; the rest ignored.
 *   op  OLIVE_OP_ROW_NORM_BWD: d = width; the rest ignored.
 *   op  OLIVE_OP_EMBEDDING_BWD: T, d = width, V; the rest ignored.
 *   op  OLIVE_OP_PACKED_ATTENTION_BWD: T, d = head width, d_t = key heads, V = query
 *       heads; the rest ignored.
 *   `grad` (bwd / divergence): non-zero when gradients are requested
 *   (OLIVE_OP_LOSS_BWD always computes them); `grad_dtype` is the dtype of
 *   d_W for OLIVE_OP_LOSS_BWD (bf16 output needs an fp32 accumulator).
 * Returns 0 for invalid arguments.
 */
OLIVE_API size_t olive_workspace_size(int op, int32_t T, int32_t d, int32_t d_t, int32_t V,
                            int grad, int grad_dtype);

/*
 * olive_splice_pack -- builds the packed student-update batch of Section 3.1:
 * for each sequence s the spliced sequence (x, y_{1:k}, y~_{1:l}) =
 * prefix_s || continuation_s, laid back to back, with the loss of Eq. (osd-ce)
 * on the continuation tokens only ("the prompt and student prefix remain in
 * the conditioning context but are masked out of the loss").
 *
 * Inputs (device, int32):
 *   prefix_ids  all prefixes (prompt + student prefix) back to back;
 *   prefix_off  [S+1] CSR offsets, prefix_off[0] = 0, non-decreasing;
 *               every prefix holds >= 1 id;
 *   cont_ids    all continuations (already in student tokens) back to back;
 *   cont_off    [S+1] CSR offsets, cont_off[0] = 0, non-decreasing (a
 *               continuation may be empty);
 *   S >= 1 sequences, V >= 1 vocabulary size, T_cap >= 1 capacity of the
 *   packed outputs.
 * Outputs (device), with T = sum_s (P_s + C_s) packed tokens:
 *   ids[T_cap]        packed ids; positions >= T are set to 0;
 *   targets[T_cap]    ids[t+1] when t+1 belongs to the same sequence, else -1
 *                     (row t of the hidden states predicts token t+1);
 *   loss_mask[T_cap]  1 where targets[t] is a continuation token y~_j, else 0;
 *   cu_seqlens[S+1]   packed start of every sequence, cu_seqlens[S] = T;
 *   cut_offsets[S]    packed index of y~_1 (= cu_seqlens[s] + P_s);
 *   rows[T_cap]       the masked rows in ascending order (first n_rows valid);
 *   n_rows[1]         N_mask = sum_s C_s.
 * Device errors: OFFSETS (malformed offsets, empty prefix, T > T_cap: then
 * n_rows = 0 and the outputs are cleared), TOKEN_RANGE (an id outside [0,V);
 * the ids are still copied).
 */
OLIVE_API olive_status olive_splice_pack(const int32_t* prefix_ids, const int32_t* prefix_off,
                               const int32_t* cont_ids, const int32_t* cont_off,
                               int32_t S, int32_t V, int32_t T_cap,
                               int32_t* ids, int32_t* targets, uint8_t* loss_mask,
                               int32_t* cu_seqlens, int32_t* cut_offsets,
                               int32_t* rows, int32_t* n_rows,
                               int32_t* dev_status, void* stream);

/*
 * olive_splice_pack_masked -- olive_splice_pack for multi-turn OLIVE
 * (Section 3.2): the whole interaction (student turns, environment
 * observations, teacher turns) is kept as context, and the loss applies only
 * to the teacher's actions.  cont_loss (device, uint8, one flag per
 * continuation id, same CSR as cont_ids) marks the continuation tokens that
 * are teacher actions; row t is masked when targets[t] is such a token.
 * Outputs and device errors as in olive_splice_pack, with
 * n_rows = number of flagged continuation tokens and rows ascending.
 * workspace: olive_workspace_size(OLIVE_OP_SPLICE_MASKED, T_cap, ...) bytes.
 */
OLIVE_API olive_status olive_splice_pack_masked(const int32_t* prefix_ids,
                                                const int32_t* prefix_off, const int32_t* cont_ids,
                                                const int32_t* cont_off, const uint8_t* cont_loss,
                                                int32_t S, int32_t V, int32_t T_cap, int32_t* ids,
                                                int32_t* targets, uint8_t* loss_mask,
                                                int32_t* cu_seqlens, int32_t* cut_offsets,
                                                int32_t* rows, int32_t* n_rows, void* workspace,
                                                size_t ws_bytes, int32_t* dev_status,
                                                void* stream);

/*
 * olive_token_logprob_fwd -- Eq. (osd-ce): for every masked row r (t = rows[r],
 * r < *n_rows) with target y = targets[t],
 *   z_v    = inv_tau * <hidden[t,:], W[v,:]>          (v = 0..V-1, fp32 accumulate)
 *   lse[t] = log sum_v exp(z_v)
 *   logp[t]= z_y - lse[t]
 *   loss   = -sum_r logp[rows[r]]            (OLIVE_REDUCE_SUM, Eq. (osd-ce))
 *          = that / N_mask                   (OLIVE_REDUCE_MEAN; 0 if N_mask = 0)
 * inv_tau is the inverse sampling temperature (1.0 in Appendix A).
 *   hidden  bf16 [T, d]     W bf16 [V, d]     targets int32 [T]
 *   rows    int32 [>= *n_rows] ascending or not, each in [0,T)
 *   logp, lse  fp32 [T]: written on every row, 0 on rows not in `rows`
 *   loss    fp32 [1]
 * The [T,V] logits are never stored: vocabulary tiles are reduced on chip.
 * Device errors: TOKEN_RANGE (target outside [0,V); that row's logp is NaN),
 * OFFSETS (*n_rows > T or a row outside [0,T)), TIMEOUT.
 */
OLIVE_API olive_status olive_token_logprob_fwd(const void* hidden, const void* W,
                                     const int32_t* targets, const int32_t* rows,
                                     const int32_t* n_rows, int32_t T, int32_t d, int32_t V,
                                     float inv_tau, int reduction,
                                     float* logp, float* lse, float* loss,
                                     void* workspace, size_t ws_bytes,
                                     int32_t* dev_status, void* stream);

/*
 * olive_token_topk_fwd -- per-token entropy and the K largest log-probs of
 * the student, from the same LM-head sweep as olive_token_logprob_fwd.  OPD
 * consumes the student's top-16 log-probs per token (Appendix A, Table
 * opd-config, "LogProb top-K 16"); the entropy is -sum_v p_v log p_v.  On
 * every masked row r (t = rows[r], r < *n_rows), with z = inv_tau h[t] W^T:
 *   lse[t]           = log sum_v exp(z_v)
 *   entropy[t]       = lse[t] - sum_v p_v z_v
 *   topk_logp[t, j]  = z_(j) - lse[t], the j-th largest, j = 0..K-1
 *   topk_ids[t, j]   = its vocabulary id (equal log-probs: smaller id first)
 * 1 <= K <= 16.  Rows not in `rows` get 0 (ids -1).  lse, entropy fp32 [T];
 * topk_logp fp32 [T, K]; topk_ids int32 [T, K].  The logits are not stored.
 */
OLIVE_API olive_status olive_token_topk_fwd(const void* hidden, const void* W,
                                            const int32_t* rows, const int32_t* n_rows,
                                            int32_t T, int32_t d, int32_t V, float inv_tau,
                                            int32_t K, float* lse, float* entropy,
                                            float* topk_logp, int32_t* topk_ids,
                                            void* workspace, size_t ws_bytes,
                                            int32_t* dev_status, void* stream);

/*
 * olive_topk_compare -- student/teacher agreement on each masked row's top-K
 * tokens, from two olive_token_topk_fwd outputs (student: s_ids, s_logp;
 * teacher: t_ids, t_lse) and the teacher's LM head (h_t [T, d_t], W_t
 * [V, d_t], bf16):
 *   overlap[t] = |top_K(p_s) intersect top_K(p_t)| / K  (the top-K overlap
 *                ratio tracked during OPD, Section 4.1)
 *   kl_topk[t] = sum_{j<K} p_s(v_j) (log p_s(v_j) - log p_t(v_j)) over the
 *                student's top-K ids v_j, with log p_t(v) = inv_tau
 *                h_t[t] . W_t[v] - t_lse[t]: the reverse KL of Section 1
 *                truncated to the student's K most probable tokens (the
 *                paper's "top-16 KL approximation" is not printed in full;
 *                this is the reading implemented, no renormalisation).
 *   t_logp_s[t, j] = log p_t(v_j), the teacher's log-prob at the student's
 *                j-th id (optional: NULL skips it; the input of
 *                olive_topk_kl_bwd)
 * 1 <= K <= 16; s_ids, t_ids int32 [T, K]; s_logp fp32 [T, K]; t_lse fp32
 * [T]; overlap, kl_topk fp32 [T], t_logp_s fp32 [T, K] (0 on rows not in
 * `rows`).  An id outside [0, V) gives NaN and OLIVE_ERR_TOKEN_RANGE.
 */
OLIVE_API olive_status olive_topk_compare(const void* h_t, const void* W_t, int32_t d_t,
                                          const int32_t* rows, const int32_t* n_rows, int32_t T,
                                          int32_t V, float inv_tau, int32_t K,
                                          const int32_t* s_ids, const float* s_logp,
                                          const int32_t* t_ids, const float* t_lse,
                                          float* overlap, float* kl_topk, float* t_logp_s,
                                          int32_t* dev_status, void* stream);

/*
 * olive_opd_token_stats -- everything OPD reads per token from one sweep over
 * the vocabulary with the student (h_s [T, d_s], W_s [V, d_s]) and teacher
 * (h_t [T, d_t], W_t [V, d_t]) heads, bf16 (Section 1, the per-token KL;
 * Appendix A, Table opd-config, top-16 log-probs; Section 4.1, the top-K
 * overlap ratio).  On every masked row t (z = inv_tau h W^T for each head):
 *   kl[t]               full-vocabulary KL, direction as in
 *                       olive_token_divergence
 *   s_lse[t], t_lse[t]  log sum_v exp(z_v) of each head
 *   s_entropy[t]        -sum_v p_s log p_s
 *   s_topk_logp[t, j], s_topk_ids[t, j]
 *                       the student's K most probable tokens (as
 *                       olive_token_topk_fwd: equal logits, smaller id first)
 *   t_logp_s[t, j]      log p_t at s_topk_ids[t, j]
 *   overlap[t], kl_topk[t]
 *                       as olive_topk_compare (kl_topk: the reverse KL
 *                       truncated to the student's K tokens)
 * Every output pointer may be NULL (not written) but not all of them; fp32
 * [T] or [T, K], ids int32 [T, K]; 0 (ids -1) on rows not in `rows`.
 * 1 <= K <= 16.  The outputs feed olive_topk_kl_bwd directly.  workspace:
 * olive_workspace_size(OLIVE_OP_OPD_STATS, T, d_s, d_t, V, 0, 0) bytes.
 */
OLIVE_API olive_status olive_opd_token_stats(const void* h_s, const void* W_s, int32_t d_s,
                                             const void* h_t, const void* W_t, int32_t d_t,
                                             const int32_t* rows, const int32_t* n_rows,
                                             int32_t T, int32_t V, float inv_tau, int direction,
                                             int32_t K, float* kl, float* s_lse, float* t_lse,
                                             float* s_entropy, float* s_topk_logp,
                                             int32_t* s_topk_ids, float* t_logp_s,
                                             float* overlap, float* kl_topk, void* workspace,
                                             size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * olive_topk_kl_bwd -- gradient of sum_t g_t kl_topk[t] (the truncated
 * reverse KL of olive_topk_compare) with respect to the student's hidden rows
 * and LM head, the student's top-K set S_t held fixed (it is selected, not
 * differentiated).  With l = log p_s, q = log p_t at the ids of S_t,
 * P_S = sum_{v in S_t} p_s(v) and KL_K = kl_topk[t]:
 *   G[t, u]  = g_t inv_tau p_s(u) ([u in S_t] (l_u - q_u + 1) - KL_K - P_S)
 *   d_h_s[t] = sum_u G[t, u] W_s[u]     (0 on rows not in `rows`)
 *   d_W_s[u] = sum_t G[t, u] h_s[t]
 * Inputs: h_s [T, d], W_s [V, d] bf16; s_lse fp32 [T], s_ids int32 [T, K],
 * s_logp fp32 [T, K] from olive_token_topk_fwd on the student; t_logp_s
 * fp32 [T, K] and kl_topk fp32 [T] from olive_topk_compare (or all five from
 * olive_opd_token_stats); grad_kl fp32 [T]
 * the weights g_t.  d_h_s [T, d] and d_W_s [V, d] of grad_dtype as in
 * olive_token_loss_bwd.  The softmax term is recomputed tile by tile as in
 * that backward; the K entries of S_t per row are written over it.  1 <= K
 * <= 16; an id outside [0, V) sets OLIVE_ERR_TOKEN_RANGE.  workspace:
 * olive_workspace_size(OLIVE_OP_TOPK_KL_BWD, T, d, 0, V, 1, grad_dtype) bytes.
 */
OLIVE_API olive_status olive_topk_kl_bwd(const void* h_s, const void* W_s, const int32_t* rows,
                                         const int32_t* n_rows, int32_t T, int32_t d, int32_t V,
                                         float inv_tau, int32_t K, const float* s_lse,
                                         const int32_t* s_ids, const float* s_logp,
                                         const float* t_logp_s, const float* kl_topk,
                                         const float* grad_kl, void* d_h_s, void* d_W_s,
                                         int grad_dtype, void* workspace, size_t ws_bytes,
                                         int32_t* dev_status, void* stream);

/*
 * olive_token_loss_bwd -- gradients of the Eq. (osd-ce) loss through the LM
 * head (the sampled sequences are fixed, Section 3.1, so ids get none):
 *   G[r,v]    = g * inv_tau * (exp(z_v - lse[t]) - [v == y])
 *               with g = *grad_loss, divided by N_mask for OLIVE_REDUCE_MEAN
 *   d_hidden[t,:] = sum_v G[r,v] W[v,:]   on masked rows, 0 on all other rows
 *   d_W[v,:]      = sum_r G[r,v] hidden[t,:]
 * Arguments as in olive_token_logprob_fwd; lse fp32 [T] is the forward's
 * output; grad_loss fp32 [1] (device); d_hidden [T,d] and d_W [V,d] of
 * grad_dtype (OLIVE_DTYPE_BF16: fp32 accumulation, round-to-nearest-even
 * store; OLIVE_DTYPE_F32).  The logits are recomputed tile by tile and G is
 * formed and consumed on chip: groups of ceil(d / 256) CTAs each hold a
 * 128 x 256 column block of the d_hidden (then d_W) accumulator in tensor
 * memory and pass 128 x 256 bf16 tiles of G to one another through a ring of
 * fixed size in the workspace (3 ceil(d/256) tiles of 64 KB per group, tens
 * of MB in all, independent of T and V); no [rows, V] array is stored.  The
 * bf16 tile carries one rounding of G (relative 2^-9).  workspace:
 * olive_workspace_size(OLIVE_OP_LOSS_BWD, T, d, 0, V, 1, grad_dtype) bytes.
 */
OLIVE_API olive_status olive_token_loss_bwd(const void* hidden, const void* W,
                                  const int32_t* targets, const int32_t* rows,
                                  const int32_t* n_rows, int32_t T, int32_t d, int32_t V,
                                  float inv_tau, int reduction,
                                  const float* lse, const float* grad_loss,
                                  void* d_hidden, void* d_W, int grad_dtype,
                                  void* workspace, size_t ws_bytes,
                                  int32_t* dev_status, void* stream);

/*
 * olive_token_loss_fwd_bwd -- olive_token_logprob_fwd and olive_token_loss_bwd
 * of one training step in a single call, for callers that know the loss
 * gradient before the forward runs (*grad_loss is read on the device, e.g. 1
 * for a loss that is the objective itself).  Outputs and arguments as in
 * those two calls: logp, lse fp32 [T], loss fp32 [1], d_hidden [T, d] and
 * d_W [V, d] of grad_dtype.  Nothing of size [rows, V] is stored: the first
 * pass walks each 128-row tile across the vocabulary, forms P = exp(z - R)
 * against a per-row reference R (the maximum of the row's first vocabulary
 * tile) in bf16 tiles that a group of CTAs shares through a fixed-size ring
 * (see olive_token_loss_bwd), and accumulates P . W and the row sums, from
 * which lse, logp and d_hidden = g inv_tau (exp(R - lse) P.W - W[y]) follow;
 * the second pass walks each 128-row vocabulary tile across the masked rows,
 * recomputes the logits and accumulates d_W = G^T hidden with G formed on
 * chip from that lse.  A row whose maximum logit exceeds R by more than 64
 * log2 units has its row tile recomputed with R = its maximum (exact, only
 * slower).  The training step executes four products of 2 N_mask d V flops
 * for the three it needs.  workspace: olive_workspace_size(
 * OLIVE_OP_LOSS_FWD_BWD, T, d, 0, V, 1, grad_dtype) bytes.
 */
OLIVE_API olive_status olive_token_loss_fwd_bwd(const void* hidden, const void* W,
                                                const int32_t* targets, const int32_t* rows,
                                                const int32_t* n_rows, int32_t T, int32_t d,
                                                int32_t V, float inv_tau, int reduction,
                                                const float* grad_loss, float* logp, float* lse,
                                                float* loss, void* d_hidden, void* d_W,
                                                int grad_dtype, void* workspace, size_t ws_bytes,
                                                int32_t* dev_status, void* stream);

/*
 * olive_token_loss_fwd_bwd_slab -- the same step, arguments and outputs as
 * olive_token_loss_fwd_bwd, computing each logit tile once instead of twice
 * by keeping it in HBM: the forward product stores e' = 2^(x - R) in bf16
 * (R = the row's maximum over its first vocabulary tile) in a slab of the
 * workspace of at most min(T, 32768, ~5.6 GB / (2 V)) rows -- at the
 * 8 x 4096-token, V = 151936 batch that slab holds every masked row, about
 * 5 GB -- a per-row pass merges the tile partials into lse and writes logp,
 * the target entry of G and the row scale lam = g inv_tau 2^(R - lse2), and
 * the d_hidden and d_W products read the slab (d_hidden = lam (e' . W) with
 * lam in the epilogue; d_W = e'^T . (lam hidden)).  Faster where HBM capacity
 * allows (three products instead of four) but the G of up to 32768 rows is
 * materialised; olive_token_loss_fwd_bwd is the on-chip form.  The paper has
 * no counterpart (an implementation alternative).  workspace:
 * olive_workspace_size(OLIVE_OP_LOSS_FWD_BWD_SLAB, T, d, 0, V, 1, grad_dtype)
 * bytes.
 */
OLIVE_API olive_status olive_token_loss_fwd_bwd_slab(const void* hidden, const void* W,
                                                     const int32_t* targets, const int32_t* rows,
                                                     const int32_t* n_rows, int32_t T, int32_t d,
                                                     int32_t V, float inv_tau, int reduction,
                                                     const float* grad_loss, float* logp,
                                                     float* lse, float* loss, void* d_hidden,
                                                     void* d_W, int grad_dtype, void* workspace,
                                                     size_t ws_bytes, int32_t* dev_status,
                                                     void* stream);

/*
 * olive_topk_kl_fwd_bwd -- olive_token_topk_fwd on the student,
 * olive_topk_compare and olive_topk_kl_bwd of one OPD training step in a
 * single call, for callers that know the weights g_t = grad_kl[t] before the
 * forward runs and have the teacher's lse (and top-K ids) from
 * olive_token_topk_fwd on the teacher.  Each student logit tile is computed
 * once: the forward product stores e = exp(z - tile max) in bf16 in the G
 * slab of the workspace; per masked row the C = min(K + 8, 24) largest
 * entries of e (read only in the 128-column blocks whose maximum can hold
 * one) are the candidates whose logits are recomputed exactly (fp32 dot
 * products), S_t is the K largest of those, and the teacher's log-probs at
 * S_t come from h_t . W_t[v] - t_lse[t]; a bandwidth-bound pass writes G
 * (the formula of olive_topk_kl_bwd) and the dH and dW products follow.
 * Inputs: h_s [T, d_s], W_s [V, d_s], h_t [T, d_t], W_t [V, d_t] bf16 (d_s,
 * d_t multiples of 8); t_lse fp32 [T]; t_ids int32 [T, K] (nullable: no
 * overlap); grad_kl fp32 [T].  Outputs: s_lse fp32 [T]; s_ids int32 [T, K] and
 * s_logp fp32 [T, K] (S_t by decreasing log-prob, ties by id); t_logp_s fp32
 * [T, K]; kl_topk fp32 [T]; overlap fp32 [T] (written when t_ids is given;
 * may be NULL otherwise); d_h_s [T, d_s] and d_W_s [V, d_s] of grad_dtype.
 * Rows not in `rows` get 0 (ids -1).  S_t differs from the exact top-K only
 * where C - K or more logits lie within bf16 resolution (~2^-8 relative of
 * exp) below the K-th largest.  1 <= K <= min(16, V).  workspace:
 * olive_workspace_size(OLIVE_OP_TOPK_KL_FWD_BWD, T, d_s, 0, V, 1, grad_dtype)
 * bytes.
 */
OLIVE_API olive_status olive_topk_kl_fwd_bwd(const void* h_s, const void* W_s, int32_t d_s,
                                             const void* h_t, const void* W_t, int32_t d_t,
                                             const int32_t* rows, const int32_t* n_rows,
                                             int32_t T, int32_t V, float inv_tau, int32_t K,
                                             const float* t_lse, const int32_t* t_ids,
                                             const float* grad_kl, float* s_lse, int32_t* s_ids,
                                             float* s_logp, float* t_logp_s, float* kl_topk,
                                             float* overlap, void* d_h_s, void* d_W_s,
                                             int grad_dtype, void* workspace, size_t ws_bytes,
                                             int32_t* dev_status, void* stream);

/*
 * olive_scale -- y[i] = x[i] * (*scale) for i < n, x and y of `dtype`
 * (OLIVE_DTYPE_BF16: fp32 product, round to nearest even; OLIVE_DTYPE_F32),
 * x == y allowed, both 16-byte aligned; scale fp32 [1] on the device.  The
 * paper has no counterpart: this lets a caller that learns the loss gradient
 * g only after olive_token_loss_fwd_bwd (an autograd backward) run that call
 * with *grad_loss = 1 and scale d_hidden and d_W by g afterwards.
 */
OLIVE_API olive_status olive_scale(const void* x, void* y, size_t n, int dtype,
                                   const float* scale, void* stream);

/*
 * olive_token_divergence -- OPD's per-token divergence between the student
 * pi_theta and the teacher pi_T over the full vocabulary (Section 1; the
 * paper's top-16 approximation is not used): on masked row t,
 *   p_s = softmax(inv_tau * h_s[t] W_s^T)   (width d_s)
 *   p_t = softmax(inv_tau * h_t[t] W_t^T)   (width d_t, same V)
 *   OLIVE_KL_REVERSE: kl[t] = sum_v p_s (log p_s - log p_t)
 *   OLIVE_KL_FORWARD: kl[t] = sum_v p_t (log p_t - log p_s)
 * kl fp32 [T] (0 on rows not in `rows`).  If grad_kl (fp32 [T], weights g_t)
 * and d_h_s ([T, d_s] of grad_dtype) are both non-NULL, also writes the
 * gradient of sum_t g_t kl[t] with respect to h_s:
 *   reverse: d_h_s[t] = g_t inv_tau sum_v p_s (log p_s - log p_t - kl[t]) W_s[v]
 *   forward: d_h_s[t] = g_t inv_tau sum_v (p_s - p_t) W_s[v]
 * (0 on rows not in `rows`; the teacher receives no gradient).
 * With the gradient the call makes two sweeps over the vocabulary: the first
 * gives kl[t] and both log-sum-exps, the second recomputes both heads' logits
 * tile by tile and contracts G against W_s on chip (G is never written to
 * device memory); its counters and exchange ring are in the workspace.
 */
OLIVE_API olive_status olive_token_divergence(const void* h_s, const void* W_s, int32_t d_s,
                                    const void* h_t, const void* W_t, int32_t d_t,
                                    const int32_t* rows, const int32_t* n_rows,
                                    int32_t T, int32_t V, float inv_tau, int direction,
                                    float* kl, const float* grad_kl, void* d_h_s,
                                    int grad_dtype, void* workspace, size_t ws_bytes,
                                    int32_t* dev_status, void* stream);

/*
 * olive_token_logprob_fwd_noalloc -- the same computation, arguments and
 * outputs as olive_token_logprob_fwd, for callers that cannot provide a
 * workspace: code hosted by another framework whose allocator owns all
 * device memory and lends none, or code that must not call cudaMalloc (it
 * can synchronise the device).  The paper has no counterpart; this is a
 * deployment convenience of this library.
 *
 * Scratch comes from one array of OLIVE_NOALLOC_SCRATCH_BYTES compiled into
 * the library, which every GPU that loads the library keeps until the process
 * exits.  Limit: the call is rejected with OLIVE_ERR_SHAPE, before any
 * launch, when olive_workspace_size(OLIVE_OP_LOGPROB_FWD, T, d, 0, V, 0, 0)
 * exceeds that size (for example T = 2048 rows at d = 4096 fit, T = 4096 rows
 * at d = 4096 do not).  The first call on each device looks up the array's
 * device address; make that first call before any stream capture.  Every
 * call shares the array: calls whose work may overlap on the GPU (other
 * streams, other host threads) race on it, so the caller must serialise
 * them.  The call allocates no device or host memory.
 */
#define OLIVE_NOALLOC_SCRATCH_BYTES (32u * 1024u * 1024u)
OLIVE_API olive_status olive_token_logprob_fwd_noalloc(const void* hidden, const void* W,
                                                       const int32_t* targets, const int32_t* rows,
                                                       const int32_t* n_rows, int32_t T, int32_t d,
                                                       int32_t V, float inv_tau, int reduction,
                                                       float* logp, float* lse, float* loss,
                                                       int32_t* dev_status, void* stream);

/*
 * olive_packed_positions -- position of every packed token inside its own
 * sequence, from olive_splice_pack's cu_seqlens [S+1]:
 *   positions[t] = t - cu_seqlens[s]  for cu_seqlens[s] <= t < cu_seqlens[s+1]
 * and 0 for cu_seqlens[S] <= t < T_cap.  positions int32 [T_cap], T_cap >= 1,
 * S >= 1.
 */
OLIVE_API olive_status olive_packed_positions(const int32_t* cu_seqlens, int32_t S, int32_t T_cap,
                                              int32_t* positions, void* stream);

/*
 * olive_qk_norm_rope_fwd -- for every token t and every head of q (Hq heads)
 * and of k (Hk heads), x the head's D values, w = w_q or w_k [D]:
 *   n = w x / sqrt(mean(x^2) + eps)                                  (fp32)
 *   (out[i], out[i']) = (n[i] c - n[i'] s, n[i'] c + n[i] s)
 *     with c = cos_table[p, j], s = sin_table[p, j], p = positions[t], for the
 *     pairs j < R/2: (i, i') = (j, j + R/2), or (2 j, 2 j + 1) if `interleaved`
 *   out[i] = n[i] for R <= i < D
 * rounded once to `dtype` (OLIVE_DTYPE_BF16 or OLIVE_DTYPE_F32), the type of
 * q, k, w_q, w_k and the outputs.  Any scaling of the angles for long contexts
 * is in the tables: cos_table, sin_table fp32 [P, R/2].
 *   Head h of token t starts at q + t q_token_stride + h q_head_stride
 *   (elements), so q and k can be views of one fused projection; its D values
 *   are contiguous.  The outputs have strides of their own; an output may be
 *   its own input (same pointer and strides).  Heads of an output must not share
 *   memory (OLIVE_ERR_SHAPE); those of an input may (a stride of 0).
 *   D a multiple of 8, 8 <= D <= 256; R a multiple of 8, 0 <= R <= D; 0 <=
 *   Hq, Hk <= 4096, not both 0 (the pointers of a side without heads are ignored);
 *   T >= 0; strides multiples of 8, base pointers 16-byte aligned; eps >= 0.
 * A position outside [0, P) gives NaN for its token and OLIVE_ERR_TOKEN_RANGE;
 * dev_status may be NULL (nothing is reported then).
 */
OLIVE_API olive_status olive_qk_norm_rope_fwd(
    const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k,
    int64_t k_token_stride, int64_t k_head_stride, int32_t Hq, int32_t Hk, const void* w_q,
    const void* w_k, float eps, const float* cos_table, const float* sin_table,
    const int32_t* positions, int32_t P, int32_t T, int32_t D, int32_t R, int interleaved,
    void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void* k_out,
    int64_t k_out_token_stride, int64_t k_out_head_stride, int dtype, int32_t* dev_status,
    void* stream);

/*
 * olive_qk_norm_rope_bwd -- gradients of olive_qk_norm_rope_fwd for its inputs
 * q, k (as they went in) and the gradients g_q, g_k of its outputs: with dn the
 * rotation of g by the opposite angle and r = 1 / sqrt(mean(x^2) + eps),
 *   dx = r (dn w - x r^2 mean(dn w x)),     dw = sum over tokens and heads of dn x r
 * d_q, d_k have the type of q and strides of their own (d_q may be g_q, with its
 * strides); dw_q, dw_k fp32 [D] are both written (0 for a side without heads)
 * and summed in a fixed order, in fp32 within a block of threads and fp64 across.
 * workspace: olive_workspace_size(OLIVE_OP_QK_NORM_ROPE_BWD, 1, D, 0, 1, 0, 0) bytes.
 */
OLIVE_API olive_status olive_qk_norm_rope_bwd(
    const void* g_q, int64_t g_q_token_stride, int64_t g_q_head_stride, const void* g_k,
    int64_t g_k_token_stride, int64_t g_k_head_stride, const void* q, int64_t q_token_stride,
    int64_t q_head_stride, const void* k, int64_t k_token_stride, int64_t k_head_stride,
    int32_t Hq, int32_t Hk, const void* w_q, const void* w_k, float eps, const float* cos_table,
    const float* sin_table, const int32_t* positions, int32_t P, int32_t T, int32_t D, int32_t R,
    int interleaved, void* d_q, int64_t d_q_token_stride, int64_t d_q_head_stride, void* d_k,
    int64_t d_k_token_stride, int64_t d_k_head_stride, float* dw_q, float* dw_k, int dtype,
    void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * olive_gated_mlp_fwd -- the gated feed-forward block on T rows:
 *   g = x W_gate^T, u = x W_up^T           [T, f], fp32 accumulation
 *   h = act(g) u                           bf16 (the operand of the next product)
 *   y = h W_down^T (+ residual)            [T, d], rounded once to bf16
 * act: OLIVE_ACT_SILU, g / (1 + exp(-g)), or OLIVE_ACT_GELU_TANH,
 * g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))).  bf16: x [T, d], W_gate and
 * W_up [f, d], W_down [d, f], residual [T, d] or NULL (y may be residual), y
 * [T, d].  `saved`, if not NULL, takes g and u for olive_gated_mlp_bwd: 4 T f
 * bytes, 16-byte aligned, to be passed on as they are.  (16 bits each: a sign,
 * 6 exponent and 9 fraction bits, 2^-10 relative.  bf16's 2^-8 would put as
 * large an error on the gradients as rounding them to bf16 operands does.
 * Magnitudes below 2^-30 are held in steps of 2^-39; what is larger than
 * 2^33 - 2^24 is held as that, infinities and NaN become NaN.)
 * 0 <= T <= 2^30 (0: nothing happens), d and f multiples of 8.  dev_status may be NULL.
 * workspace: olive_workspace_size(OLIVE_OP_GATED_MLP_FWD, T, d, 0, f, 0, 0) bytes.
 */
OLIVE_API olive_status olive_gated_mlp_fwd(const void* x, const void* W_gate, const void* W_up,
                                           const void* W_down, const void* residual, int32_t T,
                                           int32_t d, int32_t f, int activation, void* y,
                                           void* saved, void* workspace, size_t ws_bytes,
                                           int32_t* dev_status, void* stream);

/*
 * olive_gated_mlp_bwd -- gradients of olive_gated_mlp_fwd (the residual's is dy
 * itself), with g, u from `saved`:
 *   dh = dy W_down,  dg = dh u act'(g),  du = dh act(g)     (dg, du bf16 operands)
 *   dx = dg W_gate + du W_up
 *   dW_gate = dg^T x,  dW_up = du^T x,  dW_down = dy^T h    (h formed again)
 * dy, x bf16 [T, d]; dx [T, d] and the weights' gradients (shaped as the
 * weights) of grad_dtype.  dx may be NULL, and so may the three weights'
 * gradients together: what is NULL is not computed (not everything may be).
 * 0 <= T <= 2^30 (0: the weights' gradients are zeroed).  workspace:
 * olive_workspace_size(OLIVE_OP_GATED_MLP_BWD, T, d, 0, f, 1, grad_dtype) bytes.
 */
OLIVE_API olive_status olive_gated_mlp_bwd(const void* dy, const void* x, const void* W_gate,
                                           const void* W_up, const void* W_down, const void* saved,
                                           int32_t T, int32_t d, int32_t f, int activation,
                                           void* dx, void* dW_gate, void* dW_up, void* dW_down,
                                           int grad_dtype, void* workspace, size_t ws_bytes,
                                           int32_t* dev_status, void* stream);

/*
 * olive_grad_clip -- the 2-norm over all elements of n tensors together, and
 * the tensors scaled so that it is at most max_norm:
 *   norm[0] = sqrt(sum over all tensors of g^2)
 *   dst[i]  = src[i] min(1, max_norm / (norm + 1e-6))
 * src, dst, numel and dtype are HOST arrays of n entries (read before the call
 * returns): device pointers, element counts (0 allowed: the pointers are then
 * ignored) and OLIVE_DTYPE_BF16 or OLIVE_DTYPE_F32, tensor by tensor.  dst[i]
 * may be src[i] (a factor of exactly 1 then writes nothing) but must not overlap
 * it otherwise, nor another tensor (olive_grad_clip_apart tells; this call does
 * not look); dst NULL: only the norm.  Any alignment of
 * whole elements; 16-byte aligned pointers are read and written in 16-byte
 * pieces, others one by one, which takes five to ten times as long.  The squares are
 * summed in fp32 by 32s (fp32 tensors: by 16s; of values scaled by a power of two
 * where their squares would leave fp32's range) and in fp64 beyond; values outside
 * whole 16-byte pieces are squared and summed in fp64.  The order is fixed.
 * A norm that is infinite or NaN goes into the factor as it is (0 or NaN).
 * norm fp32 [1] (device); n >= 0 (0: the norm is 0); max_norm > 0.
 * workspace: olive_workspace_size(OLIVE_OP_GRAD_CLIP, max(n, 1), 0, 0, 1, 0, 0) bytes.
 */
OLIVE_API olive_status olive_grad_clip(const void* const* src, void* const* dst,
                                       const int64_t* numel, const int32_t* dtype, int32_t n,
                                       float max_norm, float* norm, void* workspace,
                                       size_t ws_bytes, void* stream);

/*
 * olive_grad_clip_apart -- whether the tensors of a call to olive_grad_clip are
 * apart as they must be: OLIVE_OK, or OLIVE_ERR_INVALID_ARG where what is written
 * (dst) shares memory with another dst, with another tensor's src, or with its own
 * src without being it.  Host arrays as there; nothing is launched and no device is
 * needed.  (A list that names a tied parameter's gradient twice is such a case:
 * two blocks would scale it at once.)  OLIVE_ERR_WORKSPACE: no host memory to sort in.
 */
OLIVE_API olive_status olive_grad_clip_apart(const void* const* src, void* const* dst,
                                             const int64_t* numel, const int32_t* dtype,
                                             int32_t n);

/*
 * olive_embedding_fwd -- rows of the embedding W [V, d] for packed ids:
 *   out[t] = scale W[ids[t]]   rounded once to `dtype` (OLIVE_DTYPE_BF16 or
 * OLIVE_DTYPE_F32), the type of W and out [T, d].  n_ids (device, int32 [1]) may
 * be NULL: all T rows are looked up; else rows t >= *n_ids are zeroed (what is
 * below 0 or above T counts as 0 or T), e.g. cu_seqlens + S of olive_splice_pack.
 * T >= 0, V >= 1, d a multiple of 8.  An id outside [0, V) gives NaN in its row and
 * OLIVE_ERR_TOKEN_RANGE; dev_status may be NULL (nothing is reported then).
 */
OLIVE_API olive_status olive_embedding_fwd(const void* W, const int32_t* ids, const int32_t* n_ids,
                                           int32_t T, int32_t V, int32_t d, float scale, void* out,
                                           int dtype, int32_t* dev_status, void* stream);

/*
 * olive_embedding_bwd -- the gradient of olive_embedding_fwd's W for the
 * gradient dy [T, d] (of `dtype`) of its output:
 *   dW[v] = scale sum over t with ids[t] = v of dy[t]      (0 where there is none)
 * or, with `accumulate` (1), dW[v] += that, for a W whose gradient holds the LM
 * head's already: only rows that a token names are then read and written.  dW
 * [V, d] of grad_dtype, rounded once (with what it held in the same sum).
 * Tokens are sorted by id and summed in their order in fp32 (runs of more than 32
 * tokens, beyond 65536 tokens 128, in pieces of that size, whose sums are added with
 * a running compensation), so results are the same bits from call to call.  Rows t >= *n_ids and ids outside
 * [0, V) (OLIVE_ERR_TOKEN_RANGE) count nowhere.  T = 0: dW is zeroed, or left.
 * workspace: olive_workspace_size(OLIVE_OP_EMBEDDING_BWD, T, d, 0, V, 0, 0) bytes.
 */
OLIVE_API olive_status olive_embedding_bwd(const void* dy, const int32_t* ids,
                                           const int32_t* n_ids, int32_t T, int32_t V, int32_t d,
                                           float scale, void* dW, int dtype, int grad_dtype,
                                           int accumulate, void* workspace, size_t ws_bytes,
                                           int32_t* dev_status, void* stream);

/*
 * olive_row_norm_fwd -- norm of every row of x [T, d], weights w [d], bias b [d] or
 * NULL, all of `dtype` (OLIVE_DTYPE_BF16 or OLIVE_DTYPE_F32):
 *   h = x, or with a residual [T, d]: h = x + residual, rounded, stored to `sum`
 *   m = mean(h)  (OLIVE_NORM_LAYER; 0 for OLIVE_NORM_RMS)
 *   r = 1 / sqrt(mean((h - m)^2) + eps)
 *   y = (h - m) r w + b     in fp32, rounded once
 * `stats` (fp32 [2, T], NULL: not kept) takes the rows' m, then their r, for
 * olive_row_norm_bwd.  residual and sum are both given or both NULL; y may be x, sum
 * may be x or residual (the same pointer), y and sum differ.  T >= 0, d a multiple of
 * 8 up to 16384, eps >= 0, pointers 16-byte aligned.
 */
OLIVE_API olive_status olive_row_norm_fwd(const void* x, const void* residual, const void* w,
                                          const void* b, int32_t T, int32_t d, float eps, int kind,
                                          void* y, void* sum, float* stats, int dtype,
                                          void* stream);

/*
 * olive_row_norm_bwd -- gradients of olive_row_norm_fwd for the rows h it normed
 * (its x, or its sum), from the gradient dy of y, and g_sum, that of the sum by
 * other ways (NULL: none): with n = (h - m) r and a = dy w,
 *   dx = r (a - mean(a) - n mean(a n)) + g_sum   (mean(a): OLIVE_NORM_LAYER only)
 *   dw = sum over rows of dy n,   db = sum over rows of dy    fp32 [d]
 * dx is the gradient of x and of the residual; it may be dy or g_sum.  db may be
 * NULL.  Sums over rows are fp32 and have a fixed order: T / groups rows in turn by each
 * of up to 1024 groups (widths above 4096: one an SM), up to 32 groups' sums in turn, then
 * a tree.  T = 0: dw and db are zeroed.
 * workspace: olive_workspace_size(OLIVE_OP_ROW_NORM_BWD, 1, d, 0, 1, 0, 0) bytes.
 */
OLIVE_API olive_status olive_row_norm_bwd(const void* dy, const void* h, const void* w,
                                          const float* stats, const void* g_sum, int32_t T,
                                          int32_t d, int kind, void* dx, float* dw, float* db,
                                          int dtype, void* workspace, size_t ws_bytes,
                                          void* stream);

/*
 * olive_packed_attention_fwd -- attention of every packed token to tokens of its own
 * sequence.  Token cu_seqlens[s] + i is row i of sequence s (n_s rows); query head h
 * goes with key head h / (Hq / Hk).  Row i sees key j < n_s where not `causal` or
 * j <= i or j < prefix_end[s] - cu_seqlens[s] (int32 [S], e.g. olive_splice_pack's
 * cut_offsets: prompt and prefix are then seen by all rows; an end before the sequence
 * counts as its beginning, one behind it as its end; NULL: no such keys):
 *   s_ij = z_ij, or cap tanh(z_ij / cap) if cap > 0,  with z_ij = scale <q_i, k_j>
 *          - slopes[h] |i - j|                 (slopes fp32 [Hq], NULL: none)
 *   lse_i = log sum over seen j of exp(s_ij)                      fp32 [Hq, T]
 *   o_i = sum over seen j of exp(s_ij - lse_i) v_j                bf16 [T, Hq, D]
 * Rows behind the last sequence (t >= cu_seqlens[S]) get o = 0, lse = -inf.  q, k, v, o
 * bf16, D values of a head contiguous; token and head strides as in
 * olive_qk_norm_rope_fwd, so q, k, v may be views of one projection (the token stride is
 * not 0 where T > 1).  lse may be NULL.  Scores, maxima and sums are fp32; the weights
 * exp(s - reference) are rounded to bf16 as operands of the second product (2^-8
 * relative each at most).  What the cap itself adds to a score's error is at most 2^-15
 * up to a cap of 64, and 2^-20 of the score above.  A value that is not finite in a row of
 * k or v reaches rows of its own sequence only (it may reach earlier ones of its 128-row
 * tile).
 *   D a multiple of 8, 8 <= D <= 128; Hq a multiple of Hk, 1 <= Hk <= Hq <= 4096;
 *   S >= 1; 0 <= T <= 2^30; scale > 0; cap >= 0; strides multiples of 8, base pointers
 *   16-byte aligned; the heads of o must not share memory, nor with q, k, v.
 * Device errors (dev_status may be NULL): OFFSETS (cu_seqlens does not begin with 0,
 * falls, or exceeds T: rows of the sequences concerned are then undefined, nothing
 * outside the arrays is touched), TIMEOUT.
 */
OLIVE_API olive_status olive_packed_attention_fwd(
    const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k,
    int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
    int64_t v_head_stride, int32_t Hq, int32_t Hk, const int32_t* cu_seqlens, int32_t S, int32_t T,
    int32_t D, float scale, int causal, const int32_t* prefix_end, float cap, const float* slopes,
    void* o, int64_t o_token_stride, int64_t o_head_stride, float* lse, int32_t* dev_status,
    void* stream);

/*
 * olive_packed_attention_bwd -- gradients of olive_packed_attention_fwd for its inputs,
 * its outputs o and lse, and the gradient d_o of o (lse's is taken as 0): with p_ij =
 * exp(s_ij - lse_i) and delta_i = <d_o_i, o_i> (for rows that see up to 16 keys the sum
 * over them of p_ij <d_o_i, v_j>, which o's rounding does not enter),
 *   dv_j = sum p_ij d_o_i,   dz_ij = p_ij (<d_o_i, v_j> - delta_i) (1 - (t_ij)^2),
 *   dq_i = scale sum dz_ij k_j,   dk_j = scale sum dz_ij q_i
 * t_ij = tanh(z_ij / cap), 0 without a cap; dk and dv summed over the query heads of a
 * key head.  p and dz are rounded to bf16 as operands, sums are fp32 in a fixed order.
 * Rows behind the last sequence get 0.  What is not finite in a row reaches its own
 * sequence only.  All views bf16 with strides of their own, as in
 * the forward; the heads of dq, dk and dv must not share memory, nor those with the inputs.
 * workspace: olive_workspace_size(OLIVE_OP_PACKED_ATTENTION_BWD, T, D, Hk, Hq, 0, 0) bytes.
 */
OLIVE_API olive_status olive_packed_attention_bwd(
    const void* d_o, int64_t d_o_token_stride, int64_t d_o_head_stride, const void* q,
    int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
    int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride,
    const void* o, int64_t o_token_stride, int64_t o_head_stride, const float* lse, int32_t Hq,
    int32_t Hk, const int32_t* cu_seqlens, int32_t S, int32_t T, int32_t D, float scale, int causal,
    const int32_t* prefix_end, float cap, const float* slopes, void* dq, int64_t dq_token_stride,
    int64_t dq_head_stride, void* dk, int64_t dk_token_stride, int64_t dk_head_stride, void* dv,
    int64_t dv_token_stride, int64_t dv_head_stride, void* workspace, size_t ws_bytes,
    int32_t* dev_status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* OLIVE_H_ */
