/*
 * ada.h -- C ABI of the B200 (sm_100a) Gram-threshold representative-token
 * selection library (the selection hot path of Cascade ADA).
 *
 * Notation follows the paper: X in R^{T x d} is one layer's activation matrix
 * (row t = token t), Xhat = D^-1 X its row-normalised form (Section 2.1),
 * G = Xhat Xhat^T the cosine Gram, tau in (0,1) the Gram threshold,
 * thr = 1 - tau^2, R^(l) the representative index set of layer l.
 *
 * Conventions shared by every call
 *   - All data pointers are DEVICE pointers unless the function name ends in
 *     `_host`.  `stream` is a cudaStream_t passed as void* (NULL = default
 *     stream).  Device-pointer calls only enqueue work: they never synchronise
 *     and never read a count back to the host, so the outputs of one layer can
 *     feed the next call directly.
 *   - X is row-major, B independent sequences stacked: element (b,t,k) lives at
 *     X[(b*T + t)*ldx + k].  ldx >= d, and X, ldx*es and d*es must be multiples
 *     of 16 bytes (es = 4 for ADA_F32, 2 for ADA_BF16); otherwise
 *     ADA_ERR_UNSUPPORTED.  X is never written.
 *   - Index lists are int32, strictly ascending token indices in [0,T), with a
 *     capacity of T entries per sequence: sequence b uses list + b*T and
 *     count[b].  Counts are int32 on the device.
 *   - The caller owns every buffer it passes.  The library owns only the
 *     context (workspace: inverse norms, gathered representative rows, gamma
 *     scratch, role map, status word).  One context serves one stream at a
 *     time: calls on the same context that overlap on the GPU race on the
 *     workspace.
 *   - Host-checkable faults (bad sizes, NULL required pointers, tau outside
 *     (0,1), misalignment, sizes above the context's maxima) return an error
 *     at once and enqueue nothing.  Device-detected faults (an inherited list
 *     that is not strictly ascending or leaves [0,T), a count outside [0,T],
 *     NaN/Inf in X, an expired bounded wait) set bits in the context's device
 *     status word, leave the call's outputs in bounds but meaningless, and are
 *     reported by ada_device_status.
 *   - The first call that reaches a given kernel on a context performs one-time host-side
 *     set-up (function attributes, an occupancy query); make one call of each kind before
 *     capturing calls into a CUDA graph.  After that the device-pointer calls are plain
 *     stream-ordered launches with no host synchronisation.
 *   - Arithmetic: squared norms and Gram accumulation in fp32.  ADA_BF16
 *     multiplies the stored bf16 values on the tensor cores (products exact in
 *     fp32) and applies 1/(|x_s| |x_t|) in the epilogue; a normalised bf16 copy
 *     of X is never fed to the Gram.  gamma is compared in fp32 with
 *     (float)(1 - tau*tau), strict "<".
 *   - Accuracy of gamma on the tensor cores: their accumulator truncates, so a correlation comes
 *     out too small, by up to 4e-9 d + 2e-6 of itself for ADA_BF16 and 8e-9 d + 2e-6 for ADA_F32 where the
 *     elements of a row are of one scale (measured against 64 bits: 1.7e-5 and 2.4e-5 at d = 4096;
 *     ADA_ENGINE_FFMA 4e-6), and by up to 1.6e-8 d + 2e-6 and 2.1e-8 d + 2e-6 where a few leading ones hold most of a
 *     row's norm (6.3e-5 at d = 4096; ADA_F32 4.3e-5 at d = 2136).  Tiles that several SM pairs share along d (small problems,
 *     d <= 5500, ADA_F32 <= 2140) keep a half to a quarter of that error, so the same row's gamma may
 *     differ with the number of rows around it: by up to 1.5e-5 (ADA_F32 1e-5) for rows of one scale, whatever
 *     that scale is, and by three quarters of the error else.
 */
#ifndef ADA_H_
#define ADA_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ADA_OK = 0,
    ADA_ERR_INVALID_ARG = 1,   /* NULL pointer, size < 1, tau outside (0,1), ldx < d        */
    ADA_ERR_UNSUPPORTED = 2,   /* alignment rule broken, dtype differs from the context's   */
    ADA_ERR_WORKSPACE = 3,     /* B, T or d above the maxima given to ada_create            */
    ADA_ERR_CUDA = 4,          /* a CUDA runtime / driver call failed                       */
    ADA_ERR_BAD_INDEX_SET = 5, /* device: inherited list not ascending / out of range       */
    ADA_ERR_NONFINITE = 6,     /* device: NaN or Inf in X                                   */
    ADA_ERR_TIMEOUT = 7,       /* device: a bounded wait inside a kernel expired            */
    ADA_ERR_BAD_TAU = 8        /* device: a threshold state outside (0,1) (adaptive step)   */
} ada_status;

typedef enum { ADA_F32 = 0, ADA_BF16 = 1 } ada_dtype;

/* flags of ada_cascade_step */
#define ADA_CROSS_CAUSAL 1u /* restrict Algorithm 1 line 8 to valid representatives s < t */

/* Which Gram kernel family a context uses.  AUTO: tensor cores (tcgen05), one- or two-CTA
 * form by problem size; a fixed-threshold step over many ADA_BF16 sequences of at most 2048 tokens of at most 128
 * elements (one per attention head) runs as one launch, a cluster of CTAs per sequence.  ADA_BF16 feeds the stored values to the MMA; ADA_F32 is split into
 * three bf16 terms per value and contracted as the six leading cross terms (what is dropped is
 * below 2^-23 |x||y|; accumulation as stated above), at the price of a 6x longer contraction and a
 * workspace of 12 bytes per element.  FFMA is the plain fp32 ALU kernel (any storage type;
 * for ADA_BF16 a slow cross-check of the tensor-core path).  TCGEN05 forces the one-CTA
 * kernel (128-row tiles), TCGEN05_PAIR the two-CTA kernel (cta_group::2, 256-row tiles
 * shared by the two SMs of a TPC). */
typedef enum {
    ADA_ENGINE_AUTO = 0,
    ADA_ENGINE_FFMA = 1,
    ADA_ENGINE_TCGEN05 = 2,
    ADA_ENGINE_TCGEN05_PAIR = 3
} ada_engine;

typedef struct ada_ctx ada_ctx; /* opaque */

/* Create a context on `device` able to serve up to maxB sequences of maxT
 * tokens of width maxd in storage type dt.  Allocates the workspace
 * (cudaMalloc; about maxB*maxT*(maxd*es + 28) bytes, maxB*maxT*(maxd*es + 8) more for ADA_BF16,
 * 12*maxB*maxT*maxd more for ADA_F32, and 128 KiB per SM for partial sums).
 * maxT may not exceed ADA_MAX_T (the list counts of one sequence are kept in 21-bit fields),
 * nor maxB*maxT 2^30: ADA_ERR_INVALID_ARG.  *out is NULL on error. */
#define ADA_MAX_T ((int64_t)2097151)
ada_status ada_create(ada_ctx** out, int device, int64_t maxB, int64_t maxT, int64_t maxd,
                      ada_dtype dt);
ada_status ada_destroy(ada_ctx* ctx);
ada_status ada_set_engine(ada_ctx* ctx, ada_engine e);
/* Gram launches have CTAs that wait on results of other CTAs of the same grid.  With on != 0 (the
 * default) such a launch carries the cooperative attribute (the driver guarantees that all CTAs
 * are resident, or refuses the launch) whenever another one might keep some of its CTAs from
 * running: in all streams but the first one that uses the library on the device (until that one
 * has been seen idle by ada_device_status or ada_destroy), under stream capture, and under MPS.
 * on = 0 never uses the attribute: same kernels and results, but launches that overlap in
 * different streams can then wait for one another until the in-kernel limits expire
 * (ADA_ERR_TIMEOUT).  Meant for profilers that cannot replay cooperative launches.
 * Limit of every wait inside a kernel: 2 s, but 20 s in the launches of that first stream, whose CTAs
 * may have to wait for SMs that a long kernel of another stream holds (a cooperative launch is
 * not placed before they are free).  A fault that stalls a launch is reported after that time. */
ada_status ada_set_cooperative(ada_ctx* ctx, int on);

/* Algorithm 1 line 6 forms the cross-Gram from the tokens OUTSIDE the inherited set.  On the
 * pair-CTA kernel, when the inherited set holds two fifths of a sequence's tokens or more, the
 * rows outside it are copied out in token order inside the launch and the cross tiles run over
 * those rows only, instead of streaming all T rows and discarding the inherited ones -- for
 * sequences of at least `min_rows` tokens (default 8192: below that the copy was measured to
 * cost more than the tiles it saves).  Results do not depend on it.  min_rows >= 1;
 * a huge value turns it off. */
ada_status ada_set_row_compaction(ada_ctx* ctx, int64_t min_rows);

/* Programmatic dependent launch of the library's kernels (on by default).  When on, every
 * kernel is launched with the stream-serialization attribute and begins with a grid-dependency
 * wait, so that its blocks can be placed, and its set-up that reads nothing (barriers, TMEM
 * allocation) can run, while the previous kernel of the stream drains; results do not change.
 * It concerns only the order between consecutive kernels of one stream; work from other
 * sources enqueued between two calls is ordered as usual.  Turn it off for tools that cannot
 * follow such launches.  Host-only: ADA_ERR_INVALID_ARG for a NULL context. */
ada_status ada_set_dependent_launch(ada_ctx* ctx, int on);

/*
 * Row normalisation and representative gather (Section 2.1; Algorithm 1
 * lines 1-2).  Each output may be NULL:
 *   inv_norm[B*T]  fp32, 1/||x_t||_2 (0 for a zero row; such rows are counted)
 *   Xhat           same type/shape as X with row stride d: Xhat = D^-1 X
 *   Xrep           if rep_idx/rep_cnt are given: Xrep[(b*T+i)*d + k] =
 *                  X[b, rep_idx[b*T+i], k] for i < rep_cnt[b] (raw rows,
 *                  same type as X, row stride d)
 * One pass over X; rows are read once with 128-bit loads.
 */
ada_status ada_normalize(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                         int64_t ldx, ada_dtype dt, void* Xhat, float* inv_norm,
                         const int32_t* rep_idx, const int32_t* rep_cnt, void* Xrep,
                         void* stream);

/*
 * Full selection (Definition 1; used at layer 0, Section 4.1):
 *   gamma_t = max_{s<t} |G_st|  (gamma_0 = 0),   R = { t : gamma_t < 1 - tau^2 }.
 * The maximum runs over ALL earlier tokens.  The T x T Gram is never stored:
 * mask, |.|, row maximum and compare are fused into the Gram kernel's epilogue.
 * Outputs: rep_idx (B*T capacity) ascending, rep_cnt[B]; gamma[B*T] optional.
 */
ada_status ada_select_full(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                           int64_t ldx, ada_dtype dt, double tau, int32_t* rep_idx,
                           int32_t* rep_cnt, float* gamma, void* stream);

/*
 * One cascade step (Algorithm 1, lines 1-11) on X = X^(l+1):
 *   lines 3-5  gamma_rep_i = max_{j<i} |G(rho_i, rho_j)| over ALL inherited
 *              representatives earlier in token order; valid iff < thr
 *   lines 6-9  for every t outside the inherited set,
 *              gamma_cross_t = max_{s in R_valid} |G_ts|; new iff < thr
 *              (ADA_CROSS_CAUSAL: only s < t)
 *   lines 10-11 rep_out = R_valid u R_new (ascending)
 * plus the lists of Eq. (6): add = R_new, rem = R^(l) \ R_valid.
 * rep_in_cnt[b] = 0 is legal (every token is added).  rep_out may not alias
 * rep_in.  Optional outputs, both indexed by token and of size B*T:
 * gamma_rep (0 for tokens outside the inherited set) and gamma_cross (0 for
 * inherited representatives).
 */
ada_status ada_cascade_step(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                            int64_t ldx, ada_dtype dt, double tau, const int32_t* rep_in,
                            const int32_t* rep_in_cnt, int32_t* rep_out, int32_t* rep_out_cnt,
                            int32_t* add_idx, int32_t* add_cnt, int32_t* rem_idx,
                            int32_t* rem_cnt, float* gamma_rep, float* gamma_cross,
                            uint32_t flags, void* stream);

/*
 * Cascade step with a device-resident, per-sequence threshold that follows the turnover
 * (Section 8.1: tau^(l) set from the turnover rate of Eq. (6), which the cascade step yields as
 * a by-product; a stable set tolerates a tighter threshold, an evolving one needs a looser one).
 * The paper proposes this and gives no formula; the rule built here is a clipped proportional
 * step toward a target turnover, each operation rounded once in fp64, in this order:
 *     rho  = (|add| + |rem|) / |R_in|                        (Eq. 6; undefined for |R_in| = 0)
 *     tau' = min(tau_max, max(tau_min, tau + gain * (target_turnover - rho)))
 * and tau' = clip(tau) when rho is undefined.
 *   tau_state  DEVICE double[B], in/out: sequence b's step uses tau = tau_state[b] (threshold
 *              (float)(1 - tau^2), as for a host-side tau) and, if policy != NULL, leaves tau'
 *              there for the next layer.  Nothing returns to the host between layers.  A value
 *              outside (0,1) or NaN is reported by ada_device_status as ADA_ERR_BAD_TAU.
 *   policy     HOST struct, read during the call; NULL = leave tau_state unchanged (a fixed
 *              per-sequence threshold read from device memory).  ADA_ERR_INVALID_ARG unless
 *              gain >= 0, target_turnover >= 0, 0 < tau_min <= tau_max < 1.
 *   turnover   DEVICE float[B], optional: rho of this step (NaN where undefined).
 * Every other argument, the lists and the error behaviour are those of ada_cascade_step.
 */
typedef struct {
    double target_turnover;
    double gain;
    double tau_min, tau_max;
} ada_tau_policy;

ada_status ada_cascade_step_adaptive(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                                     int64_t ldx, ada_dtype dt, double* tau_state,
                                     const ada_tau_policy* policy, const int32_t* rep_in,
                                     const int32_t* rep_in_cnt, int32_t* rep_out,
                                     int32_t* rep_out_cnt, int32_t* add_idx, int32_t* add_cnt,
                                     int32_t* rem_idx, int32_t* rem_cnt, float* gamma_rep,
                                     float* gamma_cross, float* turnover, uint32_t flags,
                                     void* stream);

/*
 * Per-head selection (Section 8.5: one representative set per attention head, h separate
 * validations per layer at h * T * r_h * d_h operations).  X is ONE sequence of T tokens whose
 * row holds the h heads side by side: head j of token t is the d_h elements starting at
 * X[t * ldx + j * d_h] (ldx >= h * d_h; d_h * element size a multiple of 16 bytes), the layout
 * a projection writes.  The h heads are h independent problems of width d_h, each computed
 * exactly as ada_select_full / ada_cascade_step compute a sequence, in one launch sequence and
 * without a transposed copy of X.  Every per-sequence array of those calls is per head here:
 * lists and gamma arrays have h * T entries (head j at offset j * T), counts have h.  The
 * context must have been created with maxB >= h, maxT >= T, maxd >= d_h.  Errors, ownership
 * and stream semantics are those of the calls they mirror.
 */
ada_status ada_select_full_heads(ada_ctx* ctx, const void* X, int64_t T, int64_t h, int64_t d_h,
                                 int64_t ldx, ada_dtype dt, double tau, int32_t* rep_idx,
                                 int32_t* rep_cnt, float* gamma, void* stream);
ada_status ada_cascade_step_heads(ada_ctx* ctx, const void* X, int64_t T, int64_t h, int64_t d_h,
                                  int64_t ldx, ada_dtype dt, double tau, const int32_t* rep_in,
                                  const int32_t* rep_in_cnt, int32_t* rep_out,
                                  int32_t* rep_out_cnt, int32_t* add_idx, int32_t* add_cnt,
                                  int32_t* rem_idx, int32_t* rem_cnt, float* gamma_rep,
                                  float* gamma_cross, uint32_t flags, void* stream);

/*
 * Nearest-representative map (Section 2.3: the attention output of a redundant token is
 * taken from the representative s* in R maximising |G_ts*|).  For every token t of X and a
 * representative set R given as an ascending list (e.g. the output of ada_select_full or
 * ada_cascade_step on the same X):
 *   nearest_idx[t] = argmax_{s in R} |G_ts|, the lowest index on ties; a representative maps
 *                    to itself; -1 when R is empty
 *   nearest_gamma[t] (optional) = that maximum |G_ts*| (1 for a representative, 0 for zero rows)
 * One T x r cross-Gram on the tensor cores with an argmax epilogue (both storage types;
 * fp32 through the three-term split), whatever engine the context is set to; the Gram is
 * not stored.  Sizes B*T for both outputs.
 */
ada_status ada_nearest_rep(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                           int64_t ldx, ada_dtype dt, const int32_t* rep_idx,
                           const int32_t* rep_cnt, int32_t* nearest_idx, float* nearest_gamma,
                           void* stream);

/*
 * Attention on the representative set (Section 2.3, Eq. 2):
 *     Attn_R = softmax(Q_R K_R^T / sqrt(d_h)) V_R        (an r x r problem per head)
 * with Q_R, K_R, V_R the rows of Q, K, V at the representatives, and the expansion stated with
 * it: a token outside R takes the attention output of its nearest representative.
 *   Q, K, V      bf16, ONE sequence of T tokens, h heads side by side in a token's row: head j
 *                of token t starts at X[t * ld + j * d_h] (ld >= h * d_h); d_h a multiple of 16,
 *                at most 128; otherwise ADA_ERR_UNSUPPORTED (also for ADA_F32 contexts/inputs)
 *   rep_idx/cnt  R as an ascending list (device), e.g. the output of a selection call
 *   nearest_idx  optional, T entries (device), e.g. from ada_nearest_rep on the same R: token t
 *                receives out[nearest_idx[t]] (a representative maps to itself; -1 gives zeros).
 *                NULL: only the representatives' rows of `out` are written
 *   out          fp32, T rows of h * d_h with row stride ldo: out[rho_i] = Attn_R row i
 *   flags        0: Eq. 2 as printed, every representative attends to every representative;
 *                ADA_ATTN_CAUSAL: row i only to the representatives at or before it in token
 *                order (the mask a causal language model applies; the paper's equation has none)
 * Both contractions run on the tensor cores (tcgen05, accumulators in TMEM), the probabilities
 * are rounded to bf16 between them, the softmax statistics are fp32.  The gathered copies of
 * Q_R, K_R and V_R^T live in a buffer of the context allocated on the first call (3 x T x h x
 * d_h bf16): make that call before capturing into a CUDA graph.  The context must have been
 * created with maxT >= T and maxd >= h * d_h.  Enqueues on `stream`, never synchronises.
 */
#define ADA_ATTN_CAUSAL 1u
ada_status ada_attention_reps(ada_ctx* ctx, const void* Q, const void* K, const void* V, int64_t T,
                              int64_t h, int64_t d_h, int64_t ld, ada_dtype dt, const int32_t* rep_idx,
                              const int32_t* rep_cnt, const int32_t* nearest_idx, float* out,
                              int64_t ldo, uint32_t flags, void* stream);

/*
 * Paged key / value cache: what a model goes on from after the prompt.  The prompt's keys and values (all of them, or
 * those of its representatives) are appended to it, and new tokens attend to it.
 *
 * A page holds `page_size` slots of every key head.  Slot t of sequence b lies in page table[b * table_ld + t /
 * page_size], at slot t % page_size.  Pages are head-major: element e of head j and slot s of page p is
 *     k[p * page_stride + (j * page_size + s) * d_h + e]                 (v alike)
 * so K and V may be planes of one tensor.  kmin, kmax (both or neither): element e of page p and head j at
 * (p * h_kv + j) * d_h + e, the elementwise minimum and maximum of the page's keys, which ada_cache_append keeps and
 * ada_select_blocks reads.  The struct is read during the call; all pointers in it are DEVICE pointers to buffers
 * that the caller owns.
 *   - ADA_BF16 only (any context of the device serves, whatever its maxima and its storage type): dt == ADA_F32 is
 *     ADA_ERR_UNSUPPORTED, as for ada_attention_reps.
 *   - page_size 16, 32, 64 or 128; d_h a multiple of 16, at most 128; page_stride a multiple of 8, at least
 *     h_kv * page_size * d_h; K, V, kmin, kmax 16-byte aligned; h_kv <= 4096: else ADA_ERR_UNSUPPORTED.
 *   - max_pages: entries of a sequence's table row that a call may look at (max_pages * page_size < 2^30); rows are
 *     table_ld entries apart.  B <= 2^20, N <= 2^28 rows.
 *
 * The new tokens of all sequences stand one after the other (ragged): sequence b has rows off[b] .. off[b+1] - 1 of
 * every per-token array, off[0] = 0 <= off[1] <= .. <= off[B] <= N (device, B + 1 entries; a sequence may have none).
 * Rows from off[B] on are padding: they have no influence and are not written.  len[b] (device) counts the sequence's tokens in
 * the cache.  Both are read on the device: nothing returns to the host between calls.
 * Rows of queries hold the heads of a token side by side (head i at i * d_h), rows `ld` elements apart, ld a
 * multiple of 8, 16-byte aligned: columns of a wider projection will do.  Head i reads key head i / (h / h_kv); h is a
 * multiple of h_kv, at most 128 times it.
 *
 * Device-detected faults (ada_device_status): offsets out of order, a page outside [0, n_pages) where one is
 * needed, a list that does not ascend (ADA_ERR_BAD_INDEX_SET, also for lengths or counts out of range); NaN or
 * Inf in what is appended (ADA_ERR_NONFINITE).  What a faulty row gives is meaningless, but in bounds.  Table entries
 * behind a sequence's length are never looked at, and what is in slots behind it (NaN included) has no influence.
 */
typedef struct {
    void *k, *v;
    void *kmin, *kmax;
    const int32_t* table;
    int64_t table_ld, max_pages, n_pages, page_stride, page_size, h_kv, d_h;
} ada_kv_cache;

/*
 * Appends new tokens: row i of sequence b (i from 0) goes to slot len[b] + i.
 *   K, V     rows of h_kv heads; K is normed (k_norm) and rotated (inv_freq) on the way, V is copied
 *   Q, q_out optional: rows of h heads, normed (q_norm) and rotated, written to q_out (which may be Q itself)
 *   q_norm, k_norm  optional, d_h bf16 weights: x_e w_e / sqrt(mean_e x_e^2 + eps) over each head
 *   inv_freq optional, DEVICE double[rot / 2]: the first `rot` elements of a head (a multiple of 16) are rotated in
 *            pairs i by the angle position * inv_freq[i], formed in 64 bits: (a, b) -> (a cos - b sin, b cos + a sin).
 *            The pairs are elements i and i + rot / 2, with ADA_ROPE_PAIRS elements 2 i and 2 i + 1
 *   pos0     optional, DEVICE int32[B]: position of a sequence's first new token (NULL: len[b]); the tokens after it
 *            have the positions after it.  A cache that holds only representatives needs it: there a token's
 *            slot is not its position
 *   rep_idx, rep_cnt  optional, both or neither: only the rep_cnt[b] tokens rep_idx[off[b]] .. go to the cache, as
 *            an ascending list of indices within the sequence's new tokens (for sequences of one length T that is the
 *            layout of ada_select_full and ada_cascade_step).  Each keeps the position that it has in the
 *            sequence; Q is not affected
 *   len_out  optional, DEVICE int32[B], overlapping none of the int32 inputs: the sequences' new lengths
 * Arithmetic in fp32, one rounding to bf16 (the norm's sum of squares too: a head for which that is infinite, elements beyond 1e18, becomes zero).  kmin and kmax of every page written are formed anew from the page's keys
 * below the new length.  Tokens that the table has no room for are dropped (ADA_ERR_BAD_INDEX_SET).  No page that the
 * call writes to may belong to two sequences.
 */
#define ADA_ROPE_PAIRS 1u
ada_status ada_cache_append(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off, const int32_t* len,
                            int32_t* len_out, int64_t N, const void* K, int64_t ldk, const void* V, int64_t ldv,
                            ada_dtype dt, const void* Q, int64_t h, int64_t ldq, void* q_out, int64_t ldqo,
                            const void* q_norm, const void* k_norm, double eps, const double* inv_freq, int64_t rot,
                            const int32_t* pos0, const int32_t* rep_idx, const int32_t* rep_cnt, uint32_t flags,
                            void* stream);

/*
 * Attention of new tokens over their sequence's cache: out = softmax(scale Q K^T) V per head, one token or a chunk of
 * them per sequence, also mixed.  len[b] counts the new tokens too (append first).
 *   max_new  no sequence has more new tokens than this (a sequence that does is ADA_ERR_BAD_INDEX_SET, and its rows from
 *            max_new on are not written); chooses the kernel, so that it should be tight
 *   flags    ADA_ATTN_CAUSAL: the sequence's new tokens are its last ones, and each sees the slots up to its own;
 *            0: each sees all len[b] slots
 *   scale    of the scores; 0: 1 / sqrt(d_h).  Not negative
 *   out      bf16, rows of h heads; may be Q itself (then ldo = ldq).  A token that sees no slot gets zeros.  In fp32, with
 *            the scale: a score of -inf has no weight; a token that has one of NaN or +inf, or sees slots but has none
 *            but -inf, gets NaN.  A value that is NaN or infinite makes its element so for the tokens that see its slot;
 *            those that do not are not affected
 * Scores, softmax statistics and sums in fp32; the probabilities are rounded to bf16 for the second product.
 * The first call on a context allocates its workspace (40 MB): make it before capturing into a CUDA graph (while one is
 * captured it is ADA_ERR_CUDA, and the capture goes on).
 */
ada_status ada_attention_cached(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off,
                                const int32_t* len, int64_t N, int64_t max_new, const void* Q, int64_t h, int64_t ldq,
                                ada_dtype dt, double scale, void* out, int64_t ldo, uint32_t flags, void* stream);

/*
 * The pages that can matter most to a token: for every new token and key head the k pages p with the largest
 *     s(p) = sum over the heads g of the key head and e of max(q_ge kmax_pe, q_ge kmin_pe),
 * which no sum over g of q_g . key of the page exceeds.  The first n_first and the last n_last of the pages that the
 * token sees are always among them (n_first + n_last <= k); a token that sees at most k pages gets all of them.
 *   blk_idx  int32 [N][h_kv][k]: places in the sequence's table row, ascending, -1 behind the count
 *   blk_cnt  int32 [N][h_kv]
 *   flags    ADA_ATTN_CAUSAL as in ada_attention_cached
 * The choice is that of scores in 64 bits; equal scores: the lower page; a score that is NaN comes last.  At most 16384
 * pages per sequence (max_pages, k): else ADA_ERR_UNSUPPORTED.  The work of several tokens is cut by max_pages, as the
 * lengths are on the device: pass as many as the longest sequence needs (table_ld may be larger); 1000 tokens over 257 pages
 * take 46 us with max_pages 258, 97 with 1024, 340 with 4096.
 */
ada_status ada_select_blocks(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off, const int32_t* len,
                             int64_t N, const void* Q, int64_t h, int64_t ldq, ada_dtype dt, int64_t k, int64_t n_first,
                             int64_t n_last, int32_t* blk_idx, int32_t* blk_cnt, uint32_t flags, void* stream);

/*
 * ada_attention_cached over listed pages only: token i and key head j see the slots of the pages blk_idx[i][j][0 ..
 * blk_cnt[i][j] - 1] (an ascending list, as ada_select_blocks leaves it), as far as the token sees them at all.
 * A token whose list has no such slot gets zeros.  k <= 16384.
 */
ada_status ada_attention_blocks(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off,
                                const int32_t* len, int64_t N, const void* Q, int64_t h, int64_t ldq, ada_dtype dt,
                                const int32_t* blk_idx, const int32_t* blk_cnt, int64_t k, double scale, void* out,
                                int64_t ldo, uint32_t flags, void* stream);

/* Same operations with HOST buffers: inputs are copied to the device (staging
 * buffers owned by the context, allocated on first use), the device-pointer
 * call above runs, results are copied back, all in the order of `stream` (inputs
 * that work queued on it is still filling are read after that work), and the call
 * returns after synchronising that stream.  Counts are int32[B] on the host.
 * Pinned host memory makes the copies asynchronous DMA transfers.  The context
 * must have been created with maxima covering the sizes. */
ada_status ada_select_full_host(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                                ada_dtype dt, double tau, int32_t* rep_idx, int32_t* rep_cnt,
                                float* gamma, void* stream);
ada_status ada_cascade_step_host(ada_ctx* ctx, const void* X, int64_t B, int64_t T, int64_t d,
                                 ada_dtype dt, double tau, const int32_t* rep_in,
                                 const int32_t* rep_in_cnt, int32_t* rep_out,
                                 int32_t* rep_out_cnt, int32_t* add_idx, int32_t* add_cnt,
                                 int32_t* rem_idx, int32_t* rem_cnt, float* gamma_rep,
                                 float* gamma_cross, uint32_t flags, void* stream);

/*
 * Full selection for callers that cannot allocate device memory (the paper has no
 * counterpart; this is a deployment variant of ada_select_full for ONE sequence).
 *
 * Who needs it: a process whose device memory was handed in full to its own pool at
 * start-up, a latency-critical loop that cannot take the device-wide synchronisation an
 * allocation implies, a plug-in whose host forbids allocator calls.  None of them can
 * create an ada_ctx, because its workspace is one cudaMalloc.  This call takes no context
 * and performs no cudaMalloc / cudaFree and calls no allocating library routine: its
 * scratch (gamma bit patterns, inverse norms, a few status words; about 128 KiB) is a fixed
 * array inside the library image, present on every GPU that loads the library until the
 * process exits.
 *
 * Arguments as ada_select_full with B = 1: device pointers, X row-major T x d with row
 * stride ldx, rep_idx capacity T, rep_cnt one int32, gamma optional (T floats); the work
 * is enqueued on `stream` for the CURRENT device and the call does not synchronise.
 *   - T above ADA_NOALLOC_MAX_T returns ADA_ERR_WORKSPACE and enqueues nothing.
 *   - The first call on each device also performs a one-time set-up (it looks up the
 *     scratch array's device address and the SM count); make that first call before any
 *     stream capture begins.
 *   - All calls on a device share the one scratch array, and it keeps the previous call's
 *     contents; the call itself clears what must start at zero.  Two calls whose kernels
 *     overlap on the GPU (different streams) race on it: keep them stream-ordered.
 *   - Device-detected faults (NaN/Inf in X, an expired bounded wait) cannot be read back
 *     through a context here; check the inputs upstream if that matters.
 *   - ADA_F32 input runs on the plain fp32 (FFMA) Gram kernel here, ADA_BF16 on the
 *     one-CTA tensor-core kernel.
 *   - The host side is safe to call from several threads (the per-device set-up runs once,
 *     under a guard); the GPU work of concurrent callers must still be stream-ordered.
 */
#define ADA_NOALLOC_MAX_T 16384
ada_status ada_select_full_noalloc(const void* X, int64_t T, int64_t d, int64_t ldx,
                                   ada_dtype dt, double tau, int32_t* rep_idx, int32_t* rep_cnt,
                                   float* gamma, void* stream);

/* Gram operation counts of Eq. (4)/(5), d included: cascade == 0 -> T^2 d;
 * cascade != 0 -> r^2 d + (T - r) r d with r the INHERITED count.  Pure host
 * arithmetic; returns 0 for negative arguments or r > T. */
uint64_t ada_gram_op_count(int cascade, int64_t T, int64_t d, int64_t r);

/* Synchronise `stream`, then report and clear the device status word: returns
 * ADA_OK or the most severe device-detected error since the last call.
 * n_zero_norm_rows (optional, host) receives the number of zero rows seen. */
ada_status ada_device_status(ada_ctx* ctx, void* stream, int64_t* n_zero_norm_rows);

/* Self-test of the bounded-wait machinery: runs a one-warp kernel that waits, with a limit
 * of `limit_ms` milliseconds, on a counter that nothing ever sets -- the same wait the Gram
 * kernels use between CTAs.  The wait runs out, the kernel raises the TIMEOUT bit and returns
 * normally; ada_device_status then reports ADA_ERR_TIMEOUT and the context stays usable.
 * Nothing faults, traps or hangs. */
ada_status ada_selftest_wait_timeout(ada_ctx* ctx, int limit_ms, void* stream);

/* Self-test of the launch rule stated at ada_set_cooperative: 1 if `stream` is the one stream of `device` whose
 * launches go without the cooperative attribute now, else 0.  Host-only, enqueues nothing. */
int ada_selftest_launches_alone(int device, void* stream);

/* Per-kernel timing (for benchmarks): when enabled, every kernel launch of
 * this context is bracketed by CUDA events on the launching stream.
 * ada_profile_read synchronises those events, fills up to `cap` entries
 * (kernel name, launches, total milliseconds), resets the counters and
 * returns the number of kernels known. */
ada_status ada_profile_enable(ada_ctx* ctx, int on);
int ada_profile_read(ada_ctx* ctx, const char** names, int64_t* launches, double* total_ms,
                     int cap);

const char* ada_status_string(ada_status s);

#ifdef __cplusplus
}
#endif
#endif /* ADA_H_ */
