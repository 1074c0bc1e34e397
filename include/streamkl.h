/*
 * streamkl.h -- C ABI of the fused attention-distillation KL primitive for
 * AMD Instinct MI355X (gfx950).
 *
 * The operation (paper Sec. 2.1, "KL Divergence"): for every batch b, head h
 * and query row i,
 *
 *     S1 = s1 * Q1[b,h,i] K1[b,h]^T,   S2 = s2 * Q2[b,h,i] K2[b,h]^T,
 *     P_t = softmax(S_t) over the keys row i may attend,
 *     L[b,h,i] = KL(P1 || P2) = sum_j P1_j (log P1_j - log P2_j)   (eq:kl-def)
 *
 * computed in one online pass over key tiles (eq:kl-final, Algorithm 1) that
 * never materialises P1 or P2, and its gradients (eq:kl-case1, eq:kl-case2,
 * Algorithms 2 and 3) recomputed tile by tile from the saved row statistics.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - All tensor pointers are DEVICE pointers owned by the caller. The library
 *   never allocates, frees or retains device memory, keeps no per-call state,
 *   and never writes its inputs.
 * - Q1, K1, Q2, K2 are bf16, contiguous, row-major:
 *       Q1 [B, H, N_Q, d1]   K1 [B, H, N_K, d1]
 *       Q2 [B, H, N_Q, d2]   K2 [B, H, N_K, d2]
 *   and must be 16-byte aligned. Row statistics and gradients are fp32,
 *   contiguous, 4-byte aligned: kl, lse1, lse2, dkl are [B, H, N_Q];
 *   dQ1 [B,H,N_Q,d1], dQ2 [B,H,N_Q,d2], dK1 [B,H,N_K,d1], dK2 [B,H,N_K,d2].
 * - s1, s2 are the logit scales (the paper leaves the sqrt(d) factor out of
 *   its formulas; the usual choice is 1/sqrt(d_t)). They must be finite and > 0.
 * - causal = 1 masks with bottom-right alignment: query row i sits at
 *   absolute position N_K - N_Q + i and attends keys j <= that position
 *   (j <= i when N_Q = N_K). Rows left with no key (only when N_Q > N_K)
 *   give KL = 0, LSE = -inf and zero gradients.
 * - direction = STREAMKL_KL_FWD evaluates KL(P1 || P2) (the paper's
 *   objective); STREAMKL_KL_REV evaluates KL(P2 || P1). lse1/lse2 always
 *   belong to (Q1,K1,s1) / (Q2,K2,s2).
 * - Supported head dims: d1, d2 in {32, 64, 96, ..., 256} (multiples of 32).
 *   The kernels are built for multiples of 64; 32, 96, 160 and 224 run those
 *   of the next multiple of 64 with the missing columns read as zeros, so
 *   their matrix work is that of the wider head.
 * - B, H, N_Q, N_K >= 0; a zero extent is a valid call that launches
 *   nothing (N_K = 0 with N_Q > 0 makes every row empty). One head's rows
 *   of any tensor must span less than 4 GiB as fp32 (N * max(d1, d2) * 4 <
 *   2^32), else STREAMKL_ERR_UNSUPPORTED.
 * - Inputs are expected finite, with every raw dot product q.k below 1e29
 *   in magnitude (the kernels stand in -1e30 for the logit of a key a row
 *   may not see, so that a forward with such keys, masked or past the end of
 *   a 32-key tile, needs scales between 1e-24 and 1e8; the backward takes any).
 *   Non-finite values are not detected or reported. Where
 *   they reach: the forward outputs (kl, lse1, lse2) of a query row are
 *   non-finite if the row holds one or attends a key row that does, and
 *   are otherwise bit for bit those of finite inputs. The backward adds a
 *   second route: a row's masked (zero) logit gradients still multiply the
 *   key rows of the 32-key tiles the row's block streams (a block is the 32
 *   or 64 rows of a wave), so a non-finite
 *   entry in column c of key row j can make column c of dQ non-finite for
 *   rows of the same head that do not attend key j (0 x inf), and likewise
 *   column c of dK from a query row. Other heads are never affected.
 * - Work is enqueued on `stream` (NULL = the default stream) and the call
 *   returns before it completes. Asynchronous faults surface at the caller's
 *   next synchronisation, as usual for HIP.
 * - Arguments are checked before anything is enqueued; on a non-zero return
 *   nothing was launched (except STREAMKL_ERR_HIP, see below). No C++
 *   exception crosses this interface. Calls on different streams are
 *   independent and thread-safe.
 */
#ifndef STREAMKL_H
#define STREAMKL_H

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  STREAMKL_OK = 0,
  STREAMKL_ERR_INVALID_ARG = 1, /* NULL pointer, negative extent, bad flag, scale, alignment */
  STREAMKL_ERR_UNSUPPORTED = 2, /* head dim not in {32, 64, ..., 256}, extent too large     */
  STREAMKL_ERR_HIP = 3,         /* a kernel launch was rejected by the HIP runtime          */
  STREAMKL_ERR_SCRATCH_LIMIT = 4 /* streamkl_fwd_split_noalloc: partials exceed its scratch */
} streamkl_status;

typedef enum {
  STREAMKL_KL_FWD = 0, /* L = KL(P1 || P2), eq:kl-def                */
  STREAMKL_KL_REV = 1  /* L = KL(P2 || P1), the two roles swapped    */
} streamkl_direction;

/* Attention-score activations (Sec. 3.1, "Generalizability beyond Softmax"). */
typedef enum {
  STREAMKL_ACT_SOFTMAX = 0, /* P_t = softmax(S_t); L = KL(P1 || P2), eq:kl-def                  */
  STREAMKL_ACT_SIGMOID = 1  /* A_t = sigmoid(S_t), not normalised; L = generalized KL (below)  */
} streamkl_activation;

/* Backward kernel strategies of Sec. 4.2 ("GPU Kernel Design"). */
typedef enum {
  STREAMKL_BWD_AUTO = 0,     /* adaptive selection (streamkl_bwd_choose)          */
  STREAMKL_BWD_SEPARATE = 1, /* query-owned dQ kernel + key-owned dK kernel        */
  STREAMKL_BWD_FUSED = 2     /* one key-owned kernel, dQ added with fp32 atomics   */
} streamkl_bwd_strategy;

/* Gradient request bits of streamkl_bwd_choose. */
enum {
  STREAMKL_GRAD_DQ1 = 1,
  STREAMKL_GRAD_DK1 = 2,
  STREAMKL_GRAD_DQ2 = 4,
  STREAMKL_GRAD_DK2 = 8
};

/*
 * Forward pass (Algorithm 1, Sec. 3.2; eq:kl-final): one tiled pass over the
 * keys per block of query rows keeping the five running row scalars
 * (m1, l1, m2, l2, acc). Writes, for every row,
 *   kl   = L as defined by `direction`,
 *   lse1 = natural-log log-sum-exp of the scaled, masked logits S1,
 *   lse2 = the same for S2
 * and nothing else (the saved state of Sec. 3.2, "Saved state for backward").
 * Required: Q1, K1, Q2, K2, kl, lse1, lse2 (unless the extent is zero).
 */
int streamkl_fwd(const void* Q1, const void* K1, const void* Q2, const void* K2,
                 int B, int H, int N_Q, int N_K, int d1, int d2,
                 float s1, float s2, int causal, int direction,
                 float* kl, float* lse1, float* lse2,
                 hipStream_t stream);

/*
 * Backward pass (Algorithms 2 and 3, Sec. 4): recomputes S1, S2 and
 * P_t = exp(S_t - LSE_t) tile by tile from kl/lse1/lse2 of streamkl_fwd (same
 * inputs, scales, causal flag and direction) and returns the gradients of
 * sum_{b,h,i} dkl[b,h,i] * L[b,h,i]:
 *   FWD: dS2 = g (P2 - P1)                                   (eq:kl-case1)
 *        dS1 = g P1 (r - L), r = (S1 - S2) - (LSE1 - LSE2)   (eq:kl-case2, eq:stable-r)
 *   REV: dS1 = g (P1 - P2),  dS2 = g P2 (r' - L), r' = -r
 *   dQ_t = s_t dS_t K_t,  dK_t = s_t dS_t^T Q_t.
 * dkl: per-row upstream gradient g; NULL means g = 1 for every row.
 * dQ1, dK1, dQ2, dK2: each NULL (not computed) or written in full
 * (overwritten, never accumulated into). At least one must be non-NULL.
 * The outputs must not overlap each other or the inputs. When a dK and a dQ
 * are both requested, the call first writes the dK kernel's per-row
 * statistics into one of the dQ outputs, which the dQ kernel then
 * overwrites: work ordered after the call on `stream` sees only the final
 * dQ, but other streams must not read a dQ output before the call completes.
 * dQ tiles are owned by query blocks and dK tiles by key blocks, so no
 * atomics are used and results are bitwise reproducible run to run (the
 * separate-kernel strategy of Sec. 4.2; streamkl_bwd_ex offers the fused one).
 * Both gradient pairs of a call are formed by one set of kernels while
 * d1 + d2 < 448 (head dims rounded up to multiples of 64); from there on by
 * the second-slot kernels followed by the first-slot ones, each recomputing
 * the logits (one kernel holding both pairs would not fit the registers).
 */
int streamkl_bwd(const void* Q1, const void* K1, const void* Q2, const void* K2,
                 int B, int H, int N_Q, int N_K, int d1, int d2,
                 float s1, float s2, int causal, int direction,
                 const float* kl, const float* lse1, const float* lse2,
                 const float* dkl,
                 float* dQ1, float* dK1, float* dQ2, float* dK2,
                 hipStream_t stream);

/*
 * Backward pass with a choice of kernel strategy (Sec. 4.2, "Separate dQ/dK
 * Kernels", "Fused Backward Kernel", "Adaptive Strategy Selection").
 * Arguments, outputs and errors are those of streamkl_bwd, plus `strategy`:
 *   STREAMKL_BWD_SEPARATE  exactly streamkl_bwd (bitwise reproducible).
 *   STREAMKL_BWD_FUSED     one kernel over (batch*head, 128-key blocks): each
 *                          workgroup recomputes its key block against every
 *                          query tile once, writes dK for its keys and adds
 *                          its share of dQ with fp32 atomic adds. dQ is first
 *                          zeroed on `stream`. The summation order of dQ is
 *                          not fixed, so dQ may differ between runs in the
 *                          last bits (dK does not). Returns
 *                          STREAMKL_ERR_UNSUPPORTED when a dQ is requested
 *                          and the fused kernel's working set does not fit
 *                          in LDS for these head dims (only when gradients
 *                          of both distributions are requested and
 *                          d1 + d2 > 320), or when a head dim is not a
 *                          multiple of 64.
 *   STREAMKL_BWD_AUTO      the strategy streamkl_bwd_choose returns.
 * With no dQ requested every strategy runs the dK kernel alone.
 */
int streamkl_bwd_ex(const void* Q1, const void* K1, const void* Q2, const void* K2,
                    int B, int H, int N_Q, int N_K, int d1, int d2,
                    float s1, float s2, int causal, int direction,
                    const float* kl, const float* lse1, const float* lse2,
                    const float* dkl,
                    float* dQ1, float* dK1, float* dQ2, float* dK2,
                    int strategy, hipStream_t stream);

/*
 * Adaptive strategy selection (Sec. 4.2): with T_Q and T_K the numbers of
 * 128-row query and key tiles per head, returns STREAMKL_BWD_FUSED when
 * T_Q * C <= T_K (dQ small next to dK, so its atomics stay cheap) with C = 8,
 * T_Q <= 4, and the fused kernel exists for the request (head dims that
 * are multiples of 64, working set within LDS); else
 * STREAMKL_BWD_SEPARATE. The constants were measured on MI355X: there the
 * fused kernel loses beyond 512 query rows at any N_K. `grads` is an OR of
 * STREAMKL_GRAD_* bits. Returns 0 for invalid or unsupported arguments.
 */
int streamkl_bwd_choose(int B, int H, int N_Q, int N_K, int d1, int d2,
                        int causal, int direction, int grads);

/*
 * Forward with a choice of score activation (Sec. 3.1, "Generalizability
 * beyond Softmax": activations without softmax's global normalisation need
 * no normalisers). The paper defines neither the scores nor the divergence
 * for that case; this library reads it as:
 *   STREAMKL_ACT_SOFTMAX  exactly streamkl_fwd (stat1, stat2 = lse1, lse2).
 *   STREAMKL_ACT_SIGMOID  A_t[j] = sigmoid(S_t[j]) with no normalisation and
 *       L = sum_j [A1 log(A1 / A2) - A1 + A2] over the keys the row may
 *       attend (the generalized KL divergence of the two score rows: >= 0,
 *       0 iff A1 = A2, eq:kl-def when both rows sum to 1); REV swaps the
 *       roles. stat1, stat2 receive the row masses sum_j A1[j], sum_j A2[j]
 *       (each may be NULL). A row with no visible key gives L = 0. ReLU and
 *       tanh scores are not offered: under this divergence L is infinite
 *       where A2 = 0 < A1 (ReLU) and undefined for negative scores (tanh).
 * Single pass only (no split-K); other arguments, layouts and errors as for
 * streamkl_fwd. An activation outside the enum is STREAMKL_ERR_INVALID_ARG.
 */
int streamkl_fwd_act(const void* Q1, const void* K1, const void* Q2, const void* K2,
                     int B, int H, int N_Q, int N_K, int d1, int d2,
                     float s1, float s2, int causal, int direction, int activation,
                     float* kl, float* stat1, float* stat2,
                     hipStream_t stream);

/*
 * Backward for streamkl_fwd_act's objective sum_{b,h,i} dkl L (separate
 * query- and key-owned kernels; bitwise reproducible).
 *   STREAMKL_ACT_SOFTMAX  exactly streamkl_bwd (kl, stat1, stat2 = kl, lse1,
 *                         lse2 of the forward).
 *   STREAMKL_ACT_SIGMOID  FWD: dS2 = g (A2 - A1)(1 - A2),
 *                              dS1 = g A1 (1 - A1)(log A1 - log A2);
 *                         REV: the roles swapped. No saved statistic is
 *                         needed: kl, stat1, stat2 are not read (may be NULL).
 * dQ_t = s_t dS_t K_t, dK_t = s_t dS_t^T Q_t; other arguments as streamkl_bwd.
 */
int streamkl_bwd_act(const void* Q1, const void* K1, const void* Q2, const void* K2,
                     int B, int H, int N_Q, int N_K, int d1, int d2,
                     float s1, float s2, int causal, int direction, int activation,
                     const float* kl, const float* stat1, const float* stat2,
                     const float* dkl,
                     float* dQ1, float* dK1, float* dQ2, float* dK2,
                     hipStream_t stream);

/*
 * Backward pass with a choice of the gradients' storage type, for callers
 * that hand the gradients on in the inputs' bf16 (a training framework whose
 * parameters are bf16): streamkl_bwd_ex / streamkl_bwd_act with
 *   bf16_grads  OR of STREAMKL_GRAD_* bits: the gradients stored as bf16
 *               (contiguous [B,H,N,d], 4-byte aligned). Sums are float32 as
 *               ever and each value is rounded once, to nearest even, when it
 *               is written. Gradients without a bit are float32. Bits of
 *               gradients that are not requested are ignored.
 * The fused strategy adds into a float32 dQ: with a bf16 dQ requested,
 * STREAMKL_BWD_FUSED returns STREAMKL_ERR_UNSUPPORTED and STREAMKL_BWD_AUTO
 * runs the separate kernels. Sigmoid scores run the separate kernels only
 * (STREAMKL_BWD_FUSED with a dQ: STREAMKL_ERR_UNSUPPORTED).
 */
int streamkl_bwd_grads(const void* Q1, const void* K1, const void* Q2, const void* K2,
                       int B, int H, int N_Q, int N_K, int d1, int d2,
                       float s1, float s2, int causal, int direction, int activation,
                       const float* kl, const float* stat1, const float* stat2,
                       const float* dkl,
                       void* dQ1, void* dK1, void* dQ2, void* dK2,
                       int bf16_grads, int strategy, hipStream_t stream);

/*
 * Split-K forward (Sec. 3.3, "Split-K variant" and "Adaptive split
 * selection"): for heads with few query rows, the key range is cut into
 * `splits` contiguous chunks of whole 32-key tiles, each (head, query block,
 * chunk) runs the online pass of streamkl_fwd over its chunk and stores the
 * five row statistics (m1, l1, m2, l2, acc) in `workspace`, and a reduce
 * kernel merges the chunks per row with the rescaling rule of Sec. 3.3
 * (associative, so the result equals streamkl_fwd up to fp32 rounding).
 * Arguments and outputs are those of streamkl_fwd, plus:
 *   splits          >= 1; 1 runs streamkl_fwd itself and needs no workspace.
 *                   streamkl_fwd_split_count gives the paper's adaptive choice.
 *   workspace       device memory owned by the caller, 4-byte aligned, at
 *                   least streamkl_fwd_split_workspace_bytes(B, H, N_Q, splits)
 *                   bytes; its contents on entry are ignored and on return
 *                   are unspecified. Two calls may share it only if they are
 *                   ordered on one stream.
 *   workspace_bytes its size in bytes (smaller than required:
 *                   STREAMKL_ERR_INVALID_ARG, nothing launched).
 */
int streamkl_fwd_split(const void* Q1, const void* K1, const void* Q2, const void* K2,
                       int B, int H, int N_Q, int N_K, int d1, int d2,
                       float s1, float s2, int causal, int direction, int splits,
                       void* workspace, size_t workspace_bytes,
                       float* kl, float* lse1, float* lse2,
                       hipStream_t stream);

/* Bytes of device memory streamkl_fwd_split_noalloc holds on each GPU it runs on. */
#define STREAMKL_NOALLOC_SCRATCH_BYTES (16u << 20)

/*
 * Allocation-free split-K forward, for callers that cannot allocate device
 * memory: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc. Arguments, outputs and results are those of
 * streamkl_fwd_split without the workspace: the partial row statistics go to
 * a static array of STREAMKL_NOALLOC_SCRATCH_BYTES (16 MiB) that the library
 * holds on every GPU it runs on until the process ends. The call allocates
 * and frees nothing.
 *   - A request whose partials need more
 *     (streamkl_fwd_split_workspace_bytes(B, H, N_Q, splits) >
 *     STREAMKL_NOALLOC_SCRATCH_BYTES) returns STREAMKL_ERR_SCRATCH_LIMIT and
 *     launches nothing; splits = 1 needs no scratch.
 *   - Every call on one GPU uses that GPU's one array, which keeps the last
 *     call's contents. Calls whose work may overlap on one GPU (different
 *     streams, or host threads without ordering between them) race on it and
 *     give undefined results; calls ordered on one stream are safe. Nothing
 *     in it needs clearing: every partial is written before it is read.
 *   - `stream` must belong to the current device (else
 *     STREAMKL_ERR_INVALID_ARG). The first call on a device looks up the
 *     array's address there; if HIP fails that lookup, STREAMKL_ERR_HIP.
 */
int streamkl_fwd_split_noalloc(const void* Q1, const void* K1, const void* Q2, const void* K2,
                               int B, int H, int N_Q, int N_K, int d1, int d2,
                               float s1, float s2, int causal, int direction, int splits,
                               float* kl, float* lse1, float* lse2,
                               hipStream_t stream);

/* Workspace bytes streamkl_fwd_split needs: 20 * splits * B * H * N_Q when
   splits > 1, else 0. Returns 0 for negative extents. */
size_t streamkl_fwd_split_workspace_bytes(int B, int H, int N_Q, int splits);

/*
 * Adaptive split count (Sec. 3.3): with P_base the number of workgroups the
 * single-pass forward launches for these shapes and P_target = 512 (two per
 * CU of an MI355X), returns 1 when P_base >= P_target and otherwise
 * min(floor(P_target / P_base), number of 32-key tiles), at least 1.
 * Returns 0 for invalid or unsupported arguments.
 */
int streamkl_fwd_split_count(int B, int H, int N_Q, int N_K, int d1, int d2);

/*
 * The operators around the divergence
 * -----------------------------------
 * What stands before and beside the two maps that the calls above compare:
 * the norm and rotation that make a layer's queries and keys
 * (streamkl_qk_norm_rope_*), and attention by the difference of two maps
 * (streamkl_diff_*). The conventions above hold: device pointers of the
 * caller, nothing allocated, checks before anything is enqueued, work on
 * `stream`, which belongs to the current device. All of these calls launch
 * kernels only and record into a HIP graph, and their results are
 * reproducible bit for bit (no atomics).
 */

/* Element types. */
typedef enum {
  STREAMKL_BF16 = 0,
  STREAMKL_F16 = 1,
  STREAMKL_F32 = 2
} streamkl_dtype;

/*
 * A [batch, head, row] arrangement of contiguous rows in memory: row n of
 * head h of batch b begins at data + b sb + h sh + n sn (in elements). data
 * is 16-byte aligned, the strides are >= 0 and whole 16-byte steps. Strides of
 * extents of 1 must satisfy this too (0 will do). The struct itself lies in
 * host memory and is read before the call returns.
 */
typedef struct {
  const void* data;
  long long sb, sh, sn;
} streamkl_rows;

/*
 * Norms of queries and keys per head, with the position rotation in the same
 * pass. For every head x[0..d) of a token, with its learned weight w and the
 * cosines c and sines s of the token's position:
 *     n_j = x_j w_j / sqrt(mean_i x_i^2 + eps)
 *     y_a = n_a c - n_b s,  y_b = n_b c + n_a s   for every rotated pair (a, b)
 *     y_j = n_j                                   for the columns j >= rot
 *   q         [B, N_Q, H, d]: rows as a projection leaves them, or in any
 *             arrangement streamkl_rows can express. NULL: no queries.
 *   k         [B, N_K, HK, d], the same; NULL: no keys.
 *   d         a multiple of 32, 32 to 256.
 *   dtype     element type of q and k (streamkl_dtype).
 *   wq, wk    float32 [d], 16-byte aligned; NULL: ones.
 *   eps       finite, > 0.
 *   table     float32 [n_pos, rot], 16-byte aligned: for every position the
 *             rot/2 cosines, then the rot/2 sines. Not read when rot = 0.
 *   rot       columns that are rotated: a multiple of 16, at most d (0: the
 *             norm alone). interleaved = 0 pairs (j, j + rot/2), 1 pairs
 *             (2 j, 2 j + 1).
 *   q_pos, k_pos  positions, int32 (pos64 = 0) or int64 (pos64 = 1):
 *             contiguous [N] shared by all sequences (*_pos_shared = 1) or
 *             [B, N]. NULL: keys stand at 0 .. N_K - 1 and queries are the
 *             last N_Q of these places (bottom-right alignment; N_Q <= N_K
 *             then), whatever k_pos says; without keys, at 0 .. N_Q - 1. With
 *             rot > 0 these places have to be in the table. A position given
 *             that is outside it gives NaN in the rotated columns of its rows;
 *             nothing is read there.
 *   k_copies  every key head is written this often in a row: yk has
 *             HK k_copies heads. With k_copies = H / HK it has one per query
 *             head, as streamkl_fwd reads them.
 *   yq, yk    bf16, contiguous [B, H, N_Q, d] and [B, HK k_copies, N_K, d],
 *             16-byte aligned. Sums and products are float32, rounded once.
 * At most 2^31 - 2^16 heads of tokens (B N H) a tensor, else
 * STREAMKL_ERR_UNSUPPORTED.
 */
int streamkl_qk_norm_rope_fwd(const streamkl_rows* q, const streamkl_rows* k, int B, int H, int HK, int N_Q, int N_K,
                              int d, int dtype, const float* wq, const float* wk, float eps,
                              const float* table, int n_pos, int rot, int interleaved,
                              const void* q_pos, const void* k_pos, int pos64, int q_pos_shared, int k_pos_shared,
                              int k_copies, void* yq, void* yk, hipStream_t stream);

/*
 * Gradients of streamkl_qk_norm_rope_fwd, from its inputs alone.
 *   dyq, dyk  upstream gradients in the layout of yq, yk, bf16 or float32
 *             (dy_dtype); the gradients of a key head's copies are added. Rows
 *             at positions outside the table whose gradients are zero
 *             (padding) have zero dxq, dxk and no part in dwq, dwk.
 *   dxq, dxk  contiguous [B, N_Q, H, d] and [B, N_K, HK, d] in the inputs'
 *             type, 16-byte aligned.
 *   dwq, dwk  float32 [d]; NULL: not wanted.
 *   workspace device memory, 4-byte aligned, at least
 *             streamkl_qk_norm_rope_bwd_workspace_bytes bytes (not needed
 *             where neither dwq nor dwk is wanted); calls that may overlap
 *             need one each, as do two captured graphs that may.
 */
int streamkl_qk_norm_rope_bwd(const streamkl_rows* q, const streamkl_rows* k, int B, int H, int HK, int N_Q, int N_K,
                              int d, int dtype, const float* wq, const float* wk, float eps,
                              const float* table, int n_pos, int rot, int interleaved,
                              const void* q_pos, const void* k_pos, int pos64, int q_pos_shared, int k_pos_shared,
                              int k_copies, const void* dyq, const void* dyk, int dy_dtype,
                              void* workspace, size_t workspace_bytes,
                              void* dxq, void* dxk, float* dwq, float* dwk, hipStream_t stream);

/* Workspace bytes of streamkl_qk_norm_rope_bwd with both weight gradients; 0 for invalid extents. */
size_t streamkl_qk_norm_rope_bwd_workspace_bytes(int B, int H, int HK, int N_Q, int N_K, int d);

/*
 * Differential attention: attention by the difference of two softmax maps,
 *     S_t = scale * Q_t[b,h,i] K_t[b,hk]^T,  P_t = softmax(S_t) over the keys row i may attend,
 *     O = (P_1 - lam_h P_2) V[b,hk],         hk = h / (H / HK)
 * in one pass over the keys that materialises neither map.
 *   q1, q2    bf16 [B, H, N_Q, d];  k1, k2 [B, HK, N_K, d];  v [B, HK, N_K, dv], each in any arrangement
 *             that streamkl_rows can express with row strides below 2^25 elements (rows of a head may span
 *             more than 4 GiB). H is a multiple of HK: groups of H / HK consecutive query heads share a key
 *             head, and their keys and values are streamed once for the group.
 *   d         a multiple of 32, 32 to 128;  dv a multiple of 32, 32 to 256.
 *   scale     2^-64 to 2^64 (usual: 1/sqrt(d)). Scaled logits must stay below 2^28: the exponent of a probability is a
 *             float32 difference. The backward pass forms it from the log-sum-exp, so that probabilities there are off
 *             by up to 2^-22 |LSE| of themselves (0.2% at 10^4).
 *   lam       float32 [H] on the device, any sign.
 *   q_len, kv_len  int32 [B] on the device, or NULL: sequence b has its first q_len[b] rows and kv_len[b] keys
 *             (values outside 0 .. N are clamped). Keys behind kv_len are not read, whatever they hold.
 *             Rows behind q_len give O = 0, LSE = -inf and zero gradients, and take no part in any other.
 *   causal    1: row i sees the keys j <= kv_len[b] - q_len[b] + i (bottom-right alignment). Rows that see no
 *             key give O = 0, LSE = -inf and zero gradients.
 *   B H ceil(N_Q / 32) and B HK ceil(N_K / 64) are below 2^24, as is B H N_Q with splits, else
 *             STREAMKL_ERR_UNSUPPORTED.
 *   splits    1: one pass. 2 to 256: the keys are cut into this many ranges of whole 32-key tiles, streamed by
 *             workgroups of their own and joined by a second kernel: for few rows against many keys.
 *             streamkl_diff_fwd_split_count gives the library's choice.
 *   workspace for splits > 1: device memory, 16-byte aligned, at least streamkl_diff_fwd_workspace_bytes bytes,
 *             contents ignored on entry and unspecified on return. Calls that may overlap need one each, and
 *             so do captured graphs whose replays may overlap.
 *   out       bf16 [B, H, N_Q, dv], contiguous, 16-byte aligned.
 *   out2, lse1, lse2  what the backward pass needs: O_2 = P_2 V (layout of out) and the natural-log
 *             log-sum-exps [B, H, N_Q] of the two maps; each may be NULL.
 * Sums, maxima and accumulators are float32; P_t is rounded to bf16 as an operand of the product with V, O once at
 * the end. Inputs are expected finite, values and upstream gradients below 2^40 in size (probabilities are summed up to
 * 2^64 above their reference). A non-finite value spoils every result that it takes part in, and results that
 * the causal mask keeps apart from it (0 x inf) where the kernels work on both at once: a row j of v, and in the
 * backward pass of k1 and k2, those of rows that stand up to 94 places before it (kv_len - q_len + i >= j - 94); a row
 * of q1, q2 or dout those of keys up to 62 places behind it. Never through kv_len or q_len.
 */
int streamkl_diff_fwd(const streamkl_rows* q1, const streamkl_rows* k1, const streamkl_rows* q2,
                      const streamkl_rows* k2, const streamkl_rows* v,
                      int B, int H, int HK, int N_Q, int N_K, int d, int dv, float scale, int causal,
                      const float* lam, const int* q_len, const int* kv_len,
                      int splits, void* workspace, size_t workspace_bytes,
                      void* out, void* out2, float* lse1, float* lse2, hipStream_t stream);

/* Split count of the library for these extents: the one with the least estimated time (1 where the single pass fills
   the chip). Sequence lengths are not known to it. 0 for invalid or unsupported arguments. */
int streamkl_diff_fwd_split_count(int B, int H, int HK, int N_Q, int N_K, int d, int dv, int causal);

/* Workspace bytes of streamkl_diff_fwd: 8 * splits * B * H * N_Q * (dv + 2) when splits > 1, else 0. */
size_t streamkl_diff_fwd_workspace_bytes(int B, int H, int N_Q, int dv, int splits);

/*
 * Gradients of streamkl_diff_fwd's output, recomputed tile by tile from out, out2, lse1 and lse2 of a forward call
 * with the same inputs. With dP = dO V^T and D_t = dO . O_t:
 *     dS_1 = P_1 (dP - D_1),  dS_2 = -lam P_2 (dP - D_2),  dQ_t = scale dS_t K_t,  dK_t = scale dS_t^T Q_t,
 *     dV = (P_1 - lam P_2)^T dO,  dlam_h = -sum over its rows and keys of P_2 dP
 * (dK_t, dV summed over the query heads of the group, dlam over the batch).
 *   dout      bf16 [B, H, N_Q, dv], contiguous, 16-byte aligned; rows behind q_len are not read.
 *   workspace device memory, 16-byte aligned, at least streamkl_diff_bwd_workspace_bytes bytes; as above.
 *   dq1, dq2  [B, H, N_Q, d];  dk1, dk2 [B, HK, N_K, d];  dvalues [B, HK, N_K, dv], contiguous: float32, or bf16
 *             with bf16_grads = 1 (4-byte aligned, each value rounded once). dlam float32 [H]. Each may be
 *             NULL (not wanted), not all of them; no kernel runs for outputs that are all NULL.
 */
int streamkl_diff_bwd(const streamkl_rows* q1, const streamkl_rows* k1, const streamkl_rows* q2,
                      const streamkl_rows* k2, const streamkl_rows* v,
                      int B, int H, int HK, int N_Q, int N_K, int d, int dv, float scale, int causal,
                      const float* lam, const int* q_len, const int* kv_len,
                      const void* dout, const void* out, const void* out2, const float* lse1, const float* lse2,
                      void* workspace, size_t workspace_bytes,
                      void* dq1, void* dk1, void* dq2, void* dk2, void* dvalues, float* dlam,
                      int bf16_grads, hipStream_t stream);

/* Workspace bytes of streamkl_diff_bwd (row statistics, and partial gradients where the library cuts the streamed
   axis into ranges to fill the chip); 0 for invalid or unsupported extents. */
size_t streamkl_diff_bwd_workspace_bytes(int B, int H, int HK, int N_Q, int N_K, int d, int dv, int causal);

/*
 * Operators on rows of logits
 * ---------------------------
 * What a distillation program does at the output of its models: the log
 * probabilities, entropies and best tokens of a distribution over a vocabulary
 * (streamkl_token_logprobs_*), and the divergence of a student's distribution
 * from a teacher's best tokens (streamkl_topk_distill_*). The conventions above
 * hold. All of these calls launch kernels only and record into a HIP graph;
 * their results are reproducible bit for bit.
 *
 * B N rows of V logits: row n of sequence b begins at data + b sb + n sn (in
 * elements) and is contiguous. data is aligned to its element type, the strides
 * are >= 0 (rows of an odd vocabulary, a slice of a padded vocabulary, all
 * positions but the last). The struct lies in host memory and is read before
 * the call returns. V is at most 2^22 and B N at most 2^31 - 2^16, else
 * STREAMKL_ERR_UNSUPPORTED.
 *
 * A logit of -inf has probability 0. A row of nothing else is empty: its
 * log-sum-exp is -inf, its entropy, divergence and gradients are 0, its log
 * probabilities -inf. Logits times scale have to stay finite in float32 where
 * the logits are. A NaN or +inf spoils the results of its row (they are NaN; top
 * ids are distinct, and -1 where no logit is left) and of no other.
 */
typedef struct {
  const void* data;
  long long sb, sn;
  int B, N, V;
  int dtype;          /* streamkl_dtype */
} streamkl_logits;

/*
 * Log probabilities of given tokens, entropies and top alternatives. With
 * z = scale x, lse = log sum_j exp z_j:
 *   tokens    int32 (tokens64 = 0) or int64 (1), contiguous [B, N]; NULL: none.
 *             A negative token is none (padding): logp = 0. One >= V gives NaN.
 *   scale     2^-64 to 2^64 (an inverse temperature).
 *   top       0 to 128, at most V: the `top` largest logits of each row in
 *             descending order, the lowest index first among equal ones.
 *   workspace device memory, 16-byte aligned, at least
 *             streamkl_token_logprobs_workspace_bytes bytes (0 where the rows
 *             fill the chip); contents ignored on entry, unspecified on return.
 *             Calls that may overlap need one each, and so do captured graphs
 *             whose replays may overlap.
 *   logp      float32 [B, N]: z_tok - lse. NULL where tokens is.
 *   entropy   float32 [B, N]: -sum_j p_j log p_j, p = exp(z - lse). NULL: not wanted.
 *   lse       float32 [B, N]; lse_err: what its rounding left off, which keeps
 *             the probabilities of a backward pass exact. Each may be NULL.
 *   top_logp, top_ids  float32, int32 [B, N, top].
 * Not all outputs may be NULL. Sums are float32, joined and finished in 64 bits.
 */
int streamkl_token_logprobs_fwd(const streamkl_logits* x, const void* tokens, int tokens64, float scale, int top,
                                void* workspace, size_t workspace_bytes, float* logp, float* entropy, float* lse,
                                float* lse_err, float* top_logp, int* top_ids, hipStream_t stream);

/* Workspace bytes of streamkl_token_logprobs_fwd; 0 for invalid arguments too. */
size_t streamkl_token_logprobs_workspace_bytes(int B, int N, int V, int dtype, int top);

/*
 * Gradients of logp, entropy and lse (top_logp has none):
 *     dx_j = scale (dlogp ((j == tok) - p_j) + dlse p_j - dentropy p_j (log p_j + entropy)).
 *   lse, lse_err, entropy  of the forward call (lse_err may be NULL: probabilities are then off by up to 2^-24 |lse| of
 *             themselves; entropy is read only with dentropy). A log-sum-exp of 2^24 and more does not hold what the
 *             probabilities are: the sums of such a row are formed again, by one workgroup.
 *   dlogp, dentropy, dlse  float32 [B, N], each may be NULL (zero). dlogp of rows without a token is not read.
 *             A row with dlogp for a token >= V gets NaN, one without it what the others give.
 *   dx        rows of the element type of x at dx + b dx_sb + n dx_sn that do not overlap, each value rounded once. It may be
 *             x itself, with its strides. Rows whose upstream gradients are all 0 get zeros, whatever x holds.
 */
int streamkl_token_logprobs_bwd(const streamkl_logits* x, const void* tokens, int tokens64, float scale, const float* lse,
                                const float* lse_err, const float* entropy, const float* dlogp, const float* dentropy,
                                const float* dlse, void* dx, long long dx_sb, long long dx_sn, hipStream_t stream);

/*
 * A teacher's best tokens, K of each row.
 *   ids       int32 (ids64 = 0) or int64 (1), contiguous [B, N, K]. A negative id is no entry (lists of unequal length); one
 *             >= V makes the row's results NaN, an empty row's too.
 *   values    contiguous [B, N, K] of type dtype. With rest = 1 natural log probabilities; with rest = 0 logits or log
 *             probabilities, of which p = softmax(scale values) over the list is taken.
 *   K         1 to 128, else STREAMKL_ERR_UNSUPPORTED.
 *   rest      1: what the teacher holds outside the list is a bucket of its own (see below); scale has to be 1 then, the rest
 *             of a distribution at another temperature is not known. 0: the list is all the teacher has.
 */
typedef struct {
  const void* ids;
  const void* values;
  int K, ids64, dtype, rest;
  float scale;
} streamkl_teacher_list;

/*
 * Divergence of a student from a teacher's best tokens, per row. z = scale x, q_j = exp(z_j - lse) over all V tokens.
 *   rest = 1: with p_k = exp(values_k), p_r = max(1 - sum_k p_k, 2^-24) (less is the rounding of the values) and q_r the
 *             mass of all tokens that are not listed,
 *                 STREAMKL_KL_FWD  L = sum_k p_k (log p_k - log q_k) + p_r (log p_r - log q_r)
 *                 STREAMKL_KL_REV  L = sum_k q_k (log q_k - log p_k) + q_r (log q_r - log p_r).
 *             q_r is summed over the tokens outside the list, not formed as 1 - sum q_k. Where nothing is outside (or only
 *             logits of -inf), that bucket is left out. A token that is listed twice counts with both entries.
 *   rest = 0: L = sum_k p_k (log p_k - log q_k), STREAMKL_KL_FWD only (STREAMKL_KL_REV: STREAMKL_ERR_UNSUPPORTED).
 * A row without entries, and an empty row, has L = 0 and zero gradients. A listed token of probability 0 gives L = +inf, as
 * the definition does; in STREAMKL_KL_REV a value of -inf does, and the row's gradients are not finite then. With rest = 0 a
 * list of nothing but -inf is no distribution: NaN.
 *   workspace as above, at least streamkl_topk_distill_workspace_bytes bytes.
 *   loss      float32 [B, N].
 *   stats     32 bytes a row, 8-byte aligned: what the backward pass reads.
 */
int streamkl_topk_distill_fwd(const streamkl_logits* x, const streamkl_teacher_list* teacher, float scale, int direction,
                              void* workspace, size_t workspace_bytes, float* loss, void* stats, hipStream_t stream);

/* Workspace bytes of streamkl_topk_distill_fwd and _step; 0 for invalid arguments too. */
size_t streamkl_topk_distill_workspace_bytes(int B, int N, int V, int dtype, int rest);

/*
 * Gradient of sum over rows of g L with respect to x, g = dloss[row] factor dfactor[0].
 *   dloss     float32 [B, N], or NULL: 1. dfactor: float32 [1] on the device, or NULL: 1.
 *   done_if_one  1: dx already holds the gradient for dfactor[0] = 1 (streamkl_topk_distill_step wrote it), and is left as it
 *             is where dfactor[0] is 1.
 *   dx        as for streamkl_token_logprobs_bwd, but not x with done_if_one: it cannot hold the gradient and the logits.
 *             Rows with g = 0 get zeros, whatever x holds.
 */
int streamkl_topk_distill_bwd(const streamkl_logits* x, const streamkl_teacher_list* teacher, float scale, int direction,
                              const void* stats, const float* dloss, float factor, const float* dfactor, int done_if_one,
                              void* dx, long long dx_sb, long long dx_sn, hipStream_t stream);

/*
 * Both in one: loss and stats of every row and the gradient of sum over rows of weight[row] factor L, for weights that are
 * known beforehand (weight NULL: 1). Arguments as above.
 */
int streamkl_topk_distill_step(const streamkl_logits* x, const streamkl_teacher_list* teacher, float scale, int direction,
                               void* workspace, size_t workspace_bytes, const float* weight, float factor, float* loss,
                               void* stats, void* dx, long long dx_sb, long long dx_sn, hipStream_t stream);

/* total[0] = factor sum over rows of weight[row] loss[row] (weight NULL: 1), in 64 bits, in a fixed order. Rows of weight 0
   are left out, whatever their loss. */
int streamkl_topk_distill_total(const float* loss, const float* weight, float factor, long long rows, float* total,
                                hipStream_t stream);

/* Static description of a status code. Never NULL. */
const char* streamkl_strerror(int status);

/* Library version string, e.g. "streamkl 0.1.0 gfx950". Never NULL. */
const char* streamkl_version(void);

/* 1 if d is a supported head dimension, else 0. */
int streamkl_supported_head_dim(int d);

#ifdef __cplusplus
}
#endif

#endif /* STREAMKL_H */
