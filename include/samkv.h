/*
 * samkv.h — C ABI of the SamKV hot path for NVIDIA B200 (sm_100a).
 *
 * The library sparsifies a multiple-context KV cache (per-document K/V that were prefilled
 * independently of one another) and attends over what survives, following
 * "Sparse Attention across Multiple-context KV Cache" (SamKV):
 *
 *   samkv_score    pooled query, personalised query (Eq. 1), inner-product block scores (Sec. 3.2)
 *   samkv_select   protected initial/local blocks + per-context top-k of the middle (Sec. 3.2, 4.1)
 *   samkv_compact  gather of the kept K/V rows into one compact cache, original order (Sec. 3.2)
 *   samkv_update   write recomputed rows back: Overwrite or Fusion (Sec. 3.3, Eq. 4)
 *   samkv_attn     GQA attention of a prefill chunk / decode step over the compact cache (Sec. 3.3)
 *
 * Conventions
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, innermost dimension
 *     contiguous, base address 16-byte aligned, unless the comment says "host".
 *     Arrays marked "host" are read during the call and may be freed right after it returns.
 *   - Calls validate their arguments on the host, then only enqueue kernels on `stream`
 *     (a cudaStream_t passed as void*; NULL = the default stream).  They do not allocate,
 *     free or synchronise (samkv_poll_status is the one call that synchronises).
 *   - Plain stream order holds for every argument: whatever earlier work on `stream` wrote (Q
 *     from a projection kernel, the cache from samkv_update, cache_len from the previous call)
 *     is seen by the call.  Some kernels are launched so that their set-up overlaps the tail of
 *     the kernel before them (programmatic dependent launch); they read nothing the caller
 *     passes before that kernel has completed.
 *   - A handle owns no memory: scratch lives in the caller's `workspace`.  Calls that use the
 *     same handle must be ordered on one stream (they share the workspace).
 *   - On a host-detected error a call returns a non-zero status and launches nothing.
 *     Nothing traps or aborts.  There is no CPU fallback.
 *   - Shapes: L layers, Bt batch elements (independent requests that share the context
 *     lengths), Hq query heads, Hkv KV heads (Hq % Hkv == 0, G = Hq/Hkv), d = head_dim in {64,128},
 *     D contexts with ctx_offsets[c] .. ctx_offsets[c+1] on the concatenated token axis of
 *     length L_tot, B = block_size (selection unit, power of two <= 64; 1 = single tokens),
 *     units are counted from each context's own start (the last one may be short),
 *     nb_c = ceil(L_c / B), U_tot = sum nb_c.
 *   - Protected units of a context: every unit that overlaps its first n_init or last n_local
 *     tokens (n_init, n_local multiples of B).  If some L_c is not a multiple of B, n_local
 *     must be >= B so that the short tail unit is protected and every head keeps the same
 *     number of tokens.
 */
#ifndef SAMKV_H_
#define SAMKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SAMKV_MAX_CTX 128        /* most contexts per request */
#define SAMKV_MAX_UNITS_PER_CTX 49152  /* most selection units in one context */

typedef struct samkv_ctx* samkv_handle_t; /* opaque */

typedef enum {
  SAMKV_OK = 0,
  SAMKV_ERR_INVALID_ARG = 1,  /* null / misaligned pointer, inconsistent sizes */
  SAMKV_ERR_UNSUPPORTED = 2,  /* head_dim, dtype, block_size or size outside what is built */
  SAMKV_ERR_WORKSPACE = 3,    /* workspace smaller than samkv_workspace_bytes() */
  SAMKV_ERR_CAPACITY = 4,     /* compact cache capacity too small */
  SAMKV_ERR_BUDGET = 5,       /* k_units[c] outside [protected units, nb_c] */
  SAMKV_ERR_CUDA = 6,         /* a CUDA runtime call failed (launch error, wrong device) */
  SAMKV_ERR_DEVICE_CHECK = 7  /* a kernel recorded a failed device-side check */
} samkv_status_t;

typedef enum { SAMKV_F32 = 0, SAMKV_BF16 = 1 } samkv_dtype_t;
typedef enum { SAMKV_UPDATE_OVERWRITE = 0, SAMKV_UPDATE_FUSION = 1 } samkv_update_mode_t;

/* Problem shape shared by all calls. */
typedef struct {
  int32_t n_layers, batch, n_q_heads, n_kv_heads, head_dim;
  int32_t n_ctx;               /* D, 1 .. SAMKV_MAX_CTX */
  const int32_t* ctx_offsets;  /* host [n_ctx+1], ascending, ctx_offsets[0] == 0 */
  int32_t block_size;          /* B; the paper runs with 64 */
  int32_t n_init, n_local;     /* protected tokens per context; the paper runs with 64 and 128 */
  int32_t dtype;               /* samkv_dtype_t of K, V, Q, Qloc, Knew, Vnew, Kc, Vc, O */
} samkv_shape_t;

/* ---- handle, workspace, status -------------------------------------------------------- */

/* Bytes of device scratch the calls below need for this shape: the personalised query
 * vectors of samkv_score and the split-KV partial results of samkv_attn with up to
 * max_q_tokens query tokens over a cache of cache_capacity slots.  Returns 0 on a bad shape. */
size_t samkv_workspace_bytes(const samkv_shape_t* shape, int32_t max_q_tokens, int32_t cache_capacity);

/* Creates a handle bound to CUDA device `device` and to `workspace` (device pointer, 256-byte
 * aligned, workspace_bytes long, caller-owned, must outlive the handle).  Queries device
 * properties and enqueues one small memset on the default stream; allocates no device memory.
 * The caller orders that memset behind work of other streams that still writes the workspace, and
 * before the handle's first call. */
samkv_status_t samkv_create(samkv_handle_t* out, int device, void* workspace, size_t workspace_bytes);
samkv_status_t samkv_destroy(samkv_handle_t h);
/* Host-side switch of a handle (no GPU work, takes effect with the next samkv_attn call on the handle).
 * on != 0: the caller keeps copy-like kernels (samkv_compact, samkv_update of other layers) running on another
 * stream while attention is in flight.  samkv_attn then uses, for bf16 prefill chunks with d = 128 and at least
 * 128 packed rows, a kernel that is slower on its own but leaves registers and shared memory on every SM for those
 * kernels' CTAs; the default kernel fills its SMs.  Results obey the same bounds either way.  The paper has no
 * counterpart: this is scheduling advice (Sec. 3.3 only fixes what attention computes). */
samkv_status_t samkv_attn_share_sm(samkv_handle_t h, int32_t on);

/* Synchronises `stream`, then returns SAMKV_ERR_DEVICE_CHECK if any kernel since the last poll
 * recorded a failed device-side check (and clears the record), SAMKV_ERR_CUDA if the stream
 * reports an error, else SAMKV_OK. */
samkv_status_t samkv_poll_status(samkv_handle_t h, void* stream);
const char* samkv_status_string(samkv_status_t s);

/* ---- host-side helpers (no GPU work) --------------------------------------------------- */

/* Units kept per context under a sequence budget given in basis points (1500 = 15 %, the
 * sequence ratio the paper reports in Table 1): k_c = clamp(floor(budget_bp * nb_c / 10000),
 * protected units of c, nb_c).  k_units_out: host [n_ctx]. */
samkv_status_t samkv_budget_units(const samkv_shape_t* shape, int32_t budget_bp, int32_t* k_units_out);

/* Number of protected units per context (host [n_ctx], may be NULL) and, for a given k_units
 * (host [n_ctx], may be NULL), the number of tokens S the compact cache will hold. */
samkv_status_t samkv_layout(const samkv_shape_t* shape, const int32_t* k_units, int32_t* n_protected_out,
                            int32_t* total_units_out, int32_t* kept_tokens_out);

/* ---- the five steps --------------------------------------------------------------------- */

/* Scoring (Sec. 3.1 mean pooling; Eq. 1; Sec. 3.2 inner products with block-mean keys).
 *   K     [L, Bt, Hkv, L_tot, d]
 *   Q     [L, Bt, T_q, Hq, d]          the user query's Q rows of each layer
 *   Qloc  [L, Bt, D, T_loc, Hq, d]     each document's local-position Q cache (T_loc = 1 accepts a
 *                                      pre-pooled vector); NULL or use_bias == 0 => Q^ = Q_que
 * Per (layer, batch, query head): Q_que = mean_t Q, q_loc_j = mean_t Qloc_j,
 *   Q^_i = Q_que + 1/(D-1) * sum_{j != i} |cos(Q_que, q_loc_j)| * q_loc_j   (weight 0 for a zero norm;
 *   D == 1 => Q^ = Q_que), folded to KV heads by the mean over the G query heads of a group.
 * Per (layer, batch, KV head, token t of context i): s = <q_i, K_t> in fp32 (no scaling);
 * unit score = mean of s over the unit's real tokens (== <q_i, mean K> by linearity).
 *   scores_out fp32 [L, Bt, Hkv, U_tot]
 *   qhat_out   fp32 [L, Bt, D, Hkv, d], optional (NULL: kept in the workspace only) */
samkv_status_t samkv_score(samkv_handle_t h, const samkv_shape_t* shape, const void* K, const void* Q, int32_t T_q,
                           const void* Qloc, int32_t T_loc, int32_t use_bias, float* scores_out, float* qhat_out,
                           void* stream);

/* Selection (Sec. 3.2: initial and local positions are kept in full, the middle is sparsified;
 * here under a fixed per-context budget).  Per (layer, batch, KV head, context c): keep the
 * protected units plus the k_units[c] - n_protected_c middle units with the largest score;
 * of equal scores the lower index wins (-0 and +0 compare equal).
 *   scores   fp32 [L, Bt, Hkv, U_tot]
 *   k_units  host [n_ctx], units kept per context, protected ones included
 *   sel_out  int32 [L, Bt, Hkv, S_u], S_u = sum k_units: global unit ids, ascending;
 *            context c's segment starts at sum_{c'<c} k_units[c'] */
samkv_status_t samkv_select(samkv_handle_t h, const samkv_shape_t* shape, const float* scores, const int32_t* k_units,
                            int32_t* sel_out, void* stream);

/* Compaction (Sec. 3.2: initial + selected + local rows joined in their original order).
 *   Kc[l,b,h,slot,:] = K[l,b,h,tok(slot),:], same for V; slots run over (context, token) ascending.
 *   K, V      [L, Bt, Hkv, L_tot, d].  Either may also be a pointer into PINNED HOST memory that the
 *             device can address (cudaHostAlloc / cudaHostRegister under unified addressing): the kernel
 *             then pulls just the kept rows across the bus, so only the kept share is ever loaded to the GPU
 *             (the paper's "sequence ratio", Table 1).  V can always stay on the host; K can when the scores
 *             came from the block representatives (samkv_score_blocks), since token-mode samkv_score reads
 *             all of K on the device anyway
 *   sel       int32 [L, Bt, Hkv, S_u] as written by samkv_select; k_units host [n_ctx]
 *   Kc, Vc    [L, Bt, Hkv, cache_capacity, d]; slots >= S are left untouched
 *   cache_len int32 [L, Bt], set to S (the number of kept tokens)
 *   inv_map   int32 [L, Bt, Hkv, L_tot], optional: slot of each token, -1 where this head did not
 *             keep it (the paper's "blank" position when layers/heads are aligned for recomputation)
 * Returns SAMKV_ERR_CAPACITY if cache_capacity < S.  Copies are bit-exact. */
samkv_status_t samkv_compact(samkv_handle_t h, const samkv_shape_t* shape, const void* K, const void* V,
                             const int32_t* sel, const int32_t* k_units, void* Kc, void* Vc, int32_t cache_capacity,
                             int32_t* cache_len, int32_t* inv_map, void* stream);

/* Selection and compaction in one launch (Sec. 3.2: score -> select -> initial + selected + local rows joined in
 * their original order).  Same results, bit for bit, as samkv_select followed by samkv_compact: sel_out, Kc, Vc,
 * cache_len and inv_map are written exactly as those two calls write them; one CTA selects the units of one
 * (layer, batch, KV head, context) and gathers their rows right away.  Arguments and errors as for the two calls
 * (K and V may be pinned host memory). */
samkv_status_t samkv_select_compact(samkv_handle_t h, const samkv_shape_t* shape, const float* scores,
                                    const int32_t* k_units, const void* K, const void* V, int32_t* sel_out, void* Kc,
                                    void* Vc, int32_t cache_capacity, int32_t* cache_len, int32_t* inv_map, void* stream);

/* The whole sparsification in one call: samkv_score, then samkv_select_compact.  scores_out and sel_out are outputs
 * like those of the separate calls (and must be given: the steps hand their data over through them).  Every argument
 * is validated before anything is enqueued. */
samkv_status_t samkv_sparsify(samkv_handle_t h, const samkv_shape_t* shape, const void* K, const void* V, const void* Q,
                              int32_t T_q, const void* Qloc, int32_t T_loc, int32_t use_bias, const int32_t* k_units,
                              float* scores_out, int32_t* sel_out, void* Kc, void* Vc, int32_t cache_capacity,
                              int32_t* cache_len, int32_t* inv_map, void* stream);

/* Composite cache of the protected positions only (Sec. 3.1 "Generate generic query vector": the initial and
 * local K/V of all contexts, concatenated; also the "no-selection" ablation of Sec. 4.1).  Same result as
 * samkv_select with k_units = protected units followed by samkv_compact, without scores or a unit list: the
 * kept rows are two contiguous ranges per context.  The user query is then prefilled over it with samkv_attn
 * (Kq/Vq appended), and the pooled Q of that pass is the Q_que that samkv_score takes.
 * Arguments as for samkv_compact; cache_len is set to the protected token count (samkv_layout's kept tokens
 * for k_units = protected units). */
samkv_status_t samkv_compact_protected(samkv_handle_t h, const samkv_shape_t* shape, const void* K, const void* V,
                                       void* Kc, void* Vc, int32_t cache_capacity, int32_t* cache_len,
                                       int32_t* inv_map, void* stream);

/* Write-back of recomputed rows (Sec. 3.3).  For every recomputed token r and every KV head that
 * kept it (slot = inv_map[l,b,h,tok_ids[l,r]] >= 0):
 *   overwrite: Kc[slot] = Knew[r], Vc[slot] = Vnew[r]
 *   fusion (Eq. 4): theta = cos(new, old) over the d elements of the row (1 if a norm is zero),
 *                   row = theta*new + (1-theta)*old in fp32, rounded to nearest-even in dtype;
 *                   K rows and V rows each use their own theta.
 *   tok_ids    int32 [L, R] global token ids on the concatenated axis, -1 = skip; ids of one layer
 *              must be distinct
 *   Knew, Vnew [L, Bt, R, Hkv, d] */
samkv_status_t samkv_update(samkv_handle_t h, const samkv_shape_t* shape, void* Kc, void* Vc, int32_t cache_capacity,
                            const int32_t* inv_map, const int32_t* tok_ids, int32_t R, const void* Knew,
                            const void* Vnew, int32_t mode, void* stream);

/* Attention of a query chunk over the compact cache of one layer (Sec. 3.3: the incremental
 * prefill of the user query over the new sparse cache, and the decode steps after it).
 *   Kc, Vc    [L, Bt, Hkv, cache_capacity, d]; `layer` picks the slab
 *   cache_len int32 [L, Bt] (device).  Slots < cache_len[layer,b] are visible to every query token.
 *   Q         [Bt, T_q, Hq, d] fresh query rows of this step
 *   Kq, Vq    [Bt, T_q, Hkv, d] optional (both or neither): the chunk's own keys/values, written to
 *             slots cache_len .. cache_len+T_q-1 and attended causally (token t sees appended slots <= t);
 *             afterwards cache_len[layer,b] += T_q.  The caller guarantees cache_len + T_q <= cache_capacity
 *             (a violation is recorded as a device check and the append is skipped).
 *   scale     softmax scale; <= 0 selects 1/sqrt(d)
 *   O         [Bt, T_q, Hq, d] = softmax(scale * Q Kc^T + mask) Vc, query head hq reads KV head hq/G
 *   lse       fp32 [Bt, Hq, T_q] optional: log of the softmax denominator
 * bf16 inputs: products on tensor cores with fp32 accumulation, probabilities rounded to bf16
 * before the PV product; sums of weights times values are formed in fp32 before the division, with weights of up to 2^64,
 * so that values of V beyond about 2^60 can overflow.  fp32 inputs: fp32 FMA throughout. */
samkv_status_t samkv_attn(samkv_handle_t h, const samkv_shape_t* shape, int32_t layer, void* Kc, void* Vc,
                          int32_t cache_capacity, int32_t* cache_len, const void* Q, int32_t T_q, const void* Kq,
                          const void* Vq, float scale, void* O, float* lse, void* stream);

/* The same attention for n consecutive layers, layer0 .. layer0 + n - 1, in one call: for callers that hold the
 * queries of several layers at once (the data-parallel setting in which samkv_score .. samkv_update also take all
 * layers per call).  One grid then covers every (layer, batch, KV head, row tile), which keeps all SMs busy where a
 * single layer has fewer tiles than the GPU has SMs and leaves no gap between layers.
 *   Kc, Vc, cache_len   as for samkv_attn (the whole [L, ...] tensors; the call offsets them to layer0)
 *   Q, O                [n, Bt, T_q, Hq, d];  Kq, Vq [n, Bt, T_q, Hkv, d] optional;  lse [n, Bt, Hq, T_q] optional
 * The workspace must be sized for the n * Bt requests of the call: samkv_workspace_bytes with a shape whose batch is
 * n * Bt (SAMKV_ERR_WORKSPACE otherwise).  Per layer the result obeys the bounds of samkv_attn; the number of KV
 * splits, and with it the rounding order, may differ from a per-layer call. */
samkv_status_t samkv_attn_layers(samkv_handle_t h, const samkv_shape_t* shape, int32_t layer0, int32_t n, void* Kc,
                                 void* Vc, int32_t cache_capacity, int32_t* cache_len, const void* Q, int32_t T_q,
                                 const void* Kq, const void* Vq, float scale, void* O, float* lse, void* stream);

/* ---- the paper's dynamic selection: Top-P per document, then Top-K across documents --------------- */

#define SAMKV_MAX_STAR_LAYERS 64

/* Dynamic Top-P (Sec. 3.2, Eq. 2; consolidated over the stable layers N*, Eq. 3).  Per stable layer n, batch
 * element, KV head and document i:
 *   s_anc = score of the anchor = token-weighted mean of the protected (initial + local) units' scores
 *   s_max, s_min = scores of the document's max / min blocks (max_units / min_units: device int32 [L, Bt, D],
 *                  global unit ids from the offline attention analysis of App. A.1), or, when the pointer is
 *                  NULL, the largest / smallest middle-unit score
 *   P^(n) = (s_max - s_anc) / (s_max - s_min)  if s_anc in (s_min, s_max],  else 0      (also 0 without middle units)
 * P_out[b, i] = mean over n in N* and over the KV heads (the paper has no head index).
 *   scores      fp32 [L, Bt, Hkv, U_tot] from samkv_score
 *   star_layers host [n_star], 1 <= n_star <= SAMKV_MAX_STAR_LAYERS, layer indices in [0, L)
 *   P_out       device fp32 [Bt, D] */
samkv_status_t samkv_topp(samkv_handle_t h, const samkv_shape_t* shape, const float* scores, const int32_t* star_layers,
                          int32_t n_star, const int32_t* max_units, const int32_t* min_units, float* P_out,
                          void* stream);

/* Host helper: from one request's ratios P (host [D]) the number of middle units retrieved per document,
 * cand[i] = floor(P[i] * middle units of i), the cross-context K = floor(sum cand / D), the length
 * S_u = protected units + K of every selection list, and the kept-token count S.  Outputs may be NULL. */
samkv_status_t samkv_topp_plan(const samkv_shape_t* shape, const float* P, int32_t* cand_out, int32_t* K_out,
                               int32_t* S_u_out, int32_t* kept_tokens_out);

/* Cross-context Top-K (Sec. 3.2, last paragraph).  Per (layer, batch, KV head): document i retrieves its cand[i]
 * best middle units (ties: lower index); their scores are min-max normalised inside the document over its
 * middle units ((u - min) / (max - min), 0 if max == min); the K = floor(sum cand / D) best of all retrieved
 * units are kept (equal normalised scores: lower global unit id), together with every protected unit.
 *   cand       host [D]
 *   scratch    device, 16-byte aligned, at least samkv_select_cross_scratch_bytes(shape, cand) bytes, owned by
 *              the caller and free again when the call's work on `stream` has finished; it holds one
 *              (key, unit id) pair per retrieved unit.  With cand == NULL the size helper returns the bound
 *              for any cand (every middle unit retrieved).
 *   sel_out    int32 [L, Bt, Hkv, S_u] ascending global unit ids, S_u = protected units + K
 *   counts_out int32 [L, Bt, Hkv, D] optional: units kept per document (they differ from head to head)
 * SAMKV_ERR_BUDGET if some cand[i] exceeds the document's middle units; SAMKV_ERR_WORKSPACE if scratch is short. */
size_t samkv_select_cross_scratch_bytes(const samkv_shape_t* shape, const int32_t* cand);
samkv_status_t samkv_select_cross(samkv_handle_t h, const samkv_shape_t* shape, const float* scores,
                                  const int32_t* cand, void* scratch, size_t scratch_bytes, int32_t* sel_out,
                                  int32_t* counts_out, void* stream);

/* Compaction for a selection list whose split between documents is free (as samkv_select_cross writes it):
 * sel int32 [L, Bt, Hkv, S_u] ascending global unit ids that contain every short tail unit.  Otherwise as
 * samkv_compact (V may be pinned host memory; cache_len set to the kept-token count; optional inv_map). */
samkv_status_t samkv_compact_units(samkv_handle_t h, const samkv_shape_t* shape, const void* K, const void* V,
                                   const int32_t* sel, int32_t S_u, void* Kc, void* Vc, int32_t cache_capacity,
                                   int32_t* cache_len, int32_t* inv_map, void* stream);

/* Number of kernels one samkv_attn call with these sizes launches on the device of `h` (append of the chunk when
 * `appended`, the attention kernel, the merge of KV splits where the attention kernel does not merge them itself).
 * For launch accounting; returns 0 for arguments samkv_attn would refuse. */
int32_t samkv_attn_kernel_count(samkv_handle_t h, const samkv_shape_t* shape, int32_t T_q, int32_t cache_capacity,
                                int32_t appended);

/* ---- block representatives (Sec. 3.2: a block's representative is the mean of its tokens' keys) ------------ */

/* Kbar[l,b,h,u,:] = mean over the tokens of unit u of K[l,b,h,t,:] (fp32 sum in a fixed order, one rounding to the
 * storage dtype; a short tail unit averages the tokens it has).  Query-independent: run once per stored document.
 *   K    [L, Bt, Hkv, L_tot, d]      Kbar [L, Bt, Hkv, U_tot, d], same dtype, 16-byte aligned */
samkv_status_t samkv_block_means(samkv_handle_t h, const samkv_shape_t* shape, const void* K, void* Kbar, void* stream);

/* samkv_score on the representatives: scores[l,b,h,u] = <q^_c, Kbar[l,b,h,u,:]> for u in context c, which equals
 * the block-mean of the token scores up to the one rounding of Kbar (inner products are linear).  Reads d*e bytes
 * per unit instead of per token.  Other arguments, outputs and errors as for samkv_score; `shape` is the token-level
 * shape (block_size = B), the same one samkv_select / samkv_compact take afterwards. */
samkv_status_t samkv_score_blocks(samkv_handle_t h, const samkv_shape_t* shape, const void* Kbar, const void* Q,
                                  int32_t T_q, const void* Qloc, int32_t T_loc, int32_t use_bias, float* scores_out,
                                  float* qhat_out, void* stream);

/* ---- cross-layer alignment of the sparse caches (Sec. 3.3 "Recomputation") ------------------------ */

#define SAMKV_FLAG_KEPT 1       /* some KV head of the layer keeps the token (not a blank position) */
#define SAMKV_FLAG_RECOMPUTE 2  /* K/V of the token are recomputed at this layer (rule 2) */
#define SAMKV_FLAG_OUTPUT 4     /* the layer must produce the token's output: a higher layer recomputes it (rule 1) */
#define SAMKV_FLAG_PAD_REUSE 8  /* blank here but on the forward path: the token's prefilled K/V entry is used */

/* Pad -> merge -> recompute plan.  Layers (and heads) keep different tokens; laying every layer over the union
 * of all layers' kept tokens aligns them, with blanks where a layer keeps nothing.  Per (layer n, batch b, token t):
 *   KEPT       inv_map[n,b,h,t] >= 0 for some head h
 *   RECOMPUTE  t is in tok_ids[n] and KEPT (a listed token that is blank at layer n has no entry to refresh)
 *   OUTPUT     RECOMPUTE holds for t at some layer m > n (its K/V there need the outputs of all layers below)
 *   PAD_REUSE  OUTPUT and not RECOMPUTE and not KEPT
 *   inv_map     int32 [L, Bt, Hkv, L_tot] as written by samkv_compact / samkv_compact_units
 *   tok_ids     int32 [L, R] (device) recompute lists as for samkv_update, -1 = unused entry; R may be 0
 *   flags_out   uint8 [L, Bt, L_tot]
 *   merged_ids  int32 [Bt, L_tot]: the merged axis, ascending token ids kept by any layer, then -1
 *   merged_len  int32 [Bt]
 *   run_ids     int32 [L, Bt, run_capacity]: ascending tokens with RECOMPUTE or OUTPUT (the layer's forward pass),
 *               then -1; run_len int32 [L, Bt] always holds the full count
 * A list longer than run_capacity is truncated and recorded as a device check (samkv_poll_status); so is a token
 * id >= L_tot.  The caller removes the padding again by writing results through inv_map (samkv_update). */
samkv_status_t samkv_align(samkv_handle_t h, const samkv_shape_t* shape, const int32_t* inv_map, const int32_t* tok_ids,
                           int32_t R, uint8_t* flags_out, int32_t* merged_ids, int32_t* merged_len, int32_t* run_ids,
                           int32_t run_capacity, int32_t* run_len, void* stream);

/* ---- packed sequences and the paged cache ------------------------------------------------------------ */

/* The calls below serve what lies around the sparsified cache: the prefill that produces the documents' caches in the
 * first place (every document on its own, Sec. 2: "precomputed independently"), and conversations that go on in a
 * cache of pages.  They take sequences of different lengths packed behind one another and have no context table.
 *
 * Sequence s owns the rows seq_offsets[s] .. seq_offsets[s+1]-1 of every packed tensor (row = token).  Sequences may be
 * empty.  Rows of outputs behind the last sequence are left as they were; input rows there are not used.
 * Offsets and lengths are DEVICE data (a captured call may be replayed with others); the kernels clamp what they read to
 * the bounds below and record a device check (samkv_poll_status) where a value had to be clamped.  Offsets that run
 * backwards are recorded, too: for attention a sequence that ends before it starts and all behind it are empty, so that no
 * row belongs to two sequences; samkv_append takes each row as one of at most one sequence. */
#define SAMKV_MAX_SEQ 65536

typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim, dtype;  /* as in samkv_shape_t; n_q_heads / n_kv_heads <= 32 */
  int32_t n_seq;               /* sequences, 1 .. SAMKV_MAX_SEQ */
  int32_t n_tokens;            /* rows of the packed tensors (0: the call does nothing) */
  int32_t max_seq_tokens;      /* expected longest sequence of the call, 0 = unknown; chooses the kernel, so that results
                                * may differ by rounding, within the same bounds */
  const int32_t* seq_offsets;  /* device [n_seq+1], ascending from >= 0 to <= n_tokens */
} samkv_packed_t;

/* A packed tensor [n_tokens, heads, head_dim]: element (t, h, e) at data[t * token_stride + h * head_stride + e].
 * Strides in elements, multiples of 16 bytes and >= head_dim (ignored along an axis of extent 1); data 16-byte aligned.
 * Slices of one fused projection matrix and the library's own [heads, tokens, head_dim] slabs both fit.  Rows of an
 * output must not overlap one another (SAMKV_ERR_INVALID_ARG). */
typedef struct {
  void* data;
  int64_t token_stride, head_stride;
} samkv_rows_t;

/* A cache of pages: slot i of sequence s lives in page block_table[s * table_width + i / page_size], at row
 * i % page_size.  Table entries of pages that no visible or appended slot needs are not used (any value).  A needed
 * entry outside [0, n_pages) is recorded as a device check: an append skips the slot, attention reads page 0 instead
 * (that sequence's output is then meaningless). */
typedef struct {
  void *K, *V;                 /* [n_pages, n_kv_heads, page_size, head_dim] each, contiguous, 16-byte aligned */
  const int32_t* block_table;  /* device [n_seq, table_width] */
  int32_t page_size;           /* 16, 32, 64, 128 or 256 slots */
  int32_t n_pages, table_width; /* table_width * page_size <= 2^30; n_pages * n_kv_heads * page_size < 2^31 */
} samkv_pages_t;

/* Rotary position encoding of the first rot_dim elements of a row: pair i is (i, i + rot_dim/2), or (2i, 2i+1) when
 * interleaved; (a, b) -> (a cos - b sin, b cos + a sin), angle = position * base^(-2i/rot_dim), or position *
 * inv_freq[i] when inv_freq is given (host double [rot_dim/2], finite, read during the call).  Angles are reduced
 * exactly (64-bit fixed point), so positions may be as large as int32 allows (cache_len[s] + t may pass it), or negative. */
typedef struct {
  int32_t rot_dim;             /* multiple of 16, 16 .. head_dim */
  int32_t interleaved;
  double base;                 /* > 0; ignored when inv_freq is given */
  const double* inv_freq;
} samkv_rope_t;

/* Bytes of workspace that samkv_prefill and samkv_paged_attn need in the handle they are called with (partial results
 * of key ranges that are split between CTAs; does not depend on the lengths).  0 on a bad description.  Such a handle is
 * made by samkv_create like any other (whose memset of the workspace's first 256 bytes has to come before the first
 * call in stream order); one workspace of the larger size serves both kinds of calls.  A captured graph keeps using the
 * workspace of the handle it was captured with: graphs that share a handle must not run at the same time. */
size_t samkv_packed_workspace_bytes(const samkv_packed_t* packed);

/* Causal attention of whole prompts over themselves, e.g. of the documents whose caches the calls above take:
 *   O[t, hq] = sum_{j <= t, same sequence} softmax(scale * <Q[t, hq], K[j, hq/G]>) V[j, hq/G]
 *   Q, O   packed with n_q_heads; K, V packed with n_kv_heads.  O must not overlap the inputs.
 *   scale  <= 0 selects 1/sqrt(d)
 *   lse    fp32 [n_tokens, n_q_heads] optional: log of the softmax denominator
 * lse must not overlap any other tensor of the call.
 * K and V may be the [n_kv_heads, L_tot, d] slabs of one request that samkv_score and samkv_compact read later.
 * Values of K and V behind a row's own position never reach that row, infinities and NaN included.
 * Precision as for samkv_attn: bf16 probabilities are rounded to bf16 before the second product and O is divided by the
 * sum of the rounded ones (decode steps keep 15 bits of them); lse is taken before that rounding.  Sums of weights times values are formed in fp32 before the
 * division, with weights of up to 2^16.5 (1 in decode steps and in fp32): finite values of V beyond 2^128 / (slots * weight) can come
 * out as infinities.  SAMKV_ERR_WORKSPACE if the handle's workspace is too small. */
samkv_status_t samkv_prefill(samkv_handle_t h, const samkv_packed_t* packed, const samkv_rows_t* Q,
                             const samkv_rows_t* K, const samkv_rows_t* V, float scale, const samkv_rows_t* O,
                             float* lse, void* stream);

/* Position rotation and cache append in one pass over the new rows.  Token t of sequence s (t counted from the
 * sequence's first row) is written to slot cache_len[s] + t of its pages and rotated by its position:
 *   K, V        packed with n_kv_heads: the projections' output (K not rotated yet)
 *   rope        NULL: no rotation
 *   positions   int32 [n_tokens] device, NULL: position = cache_len[s] + t
 *   pages       destination pages, NULL: none.  V goes there unchanged, K rotated
 *   cache_len   int32 [n_seq] device, NULL: 0 for every sequence.  Not changed: every layer of a step appends with the
 *               same lengths, the caller advances them afterwards
 *   K_out,V_out packed destinations next to, or instead of, the pages (both or neither, NULL: none); e.g. the slabs
 *               samkv_prefill and samkv_score read
 *   Q, Q_out    optional (both or neither): Q rows, rotated by the same positions
 * Q_out, K_out, V_out may be the very same rows as Q, K, V; otherwise outputs must not overlap inputs.  The pools must
 * not overlap one another or any packed tensor.
 * A slot at or behind table_width * page_size, or one whose page is invalid, is skipped and recorded as a device check.
 * Rotation in fp32, one rounding to dtype; rows that are not rotated are copied bit-exactly.  No workspace. */
samkv_status_t samkv_append(samkv_handle_t h, const samkv_packed_t* packed, const samkv_rows_t* K,
                            const samkv_rows_t* V, const samkv_pages_t* pages, const int32_t* cache_len,
                            const samkv_rope_t* rope, const int32_t* positions, const samkv_rows_t* Q,
                            const samkv_rows_t* Q_out, const samkv_rows_t* K_out, const samkv_rows_t* V_out,
                            void* stream);

/* Attention of new tokens over a paged cache: decode steps (one token per sequence), chunks, or both mixed.
 *   cache_len  int32 [n_seq] device: slots in the cache before this step, as given to samkv_append
 *   causal     != 0: the new tokens' own rows have been appended; token t sees slots < cache_len[s] + t + 1
 *              == 0: every token sees the slots < cache_len[s] (a row that sees none: O = 0, lse = -inf)
 *   Q, O       packed with n_q_heads; O must not overlap Q or the pools
 *   scale, lse as for samkv_prefill
 * Slots that no token sees are never used, whatever they hold.  A sequence whose slots would pass table_width *
 * page_size is cut off there and recorded as a device check: its tokens see the slots that the table has. */
samkv_status_t samkv_paged_attn(samkv_handle_t h, const samkv_packed_t* packed, const samkv_pages_t* pages,
                                const int32_t* cache_len, const samkv_rows_t* Q, float scale, int32_t causal,
                                const samkv_rows_t* O, float* lse, void* stream);

/* ---- pages handed out on the GPU ----------------------------------------------------------------------- */

/* The two calls below keep the block table of a paged cache on the device: which pages a request needs follows from its
 * length, so a step needs no round trip to the host, and a captured step can be replayed while requests grow.
 *
 * Free pages lie on a stack: free_pages int32 [n_pages], of which the first *n_free (device) are free.  n_free_out may be
 * n_free itself; otherwise *n_free stays as it was.  A count outside [0, n_pages] is clamped and recorded as a device check.
 * Pages are taken from the top and put back on top.  page_size, n_pages, table_width: as in samkv_pages_t. */

/* Gives every sequence the pages that its new tokens need, and lays out the step.
 *   packed       new tokens per sequence (heads and type are not used, but n_kv_heads bounds the pool's size)
 *   cache_len    int32 [n_seq] device: slots in the cache before this step; NULL: 0 for every sequence
 *   block_table  int32 [n_seq, table_width]: the columns ceil(cache_len / page) .. ceil((cache_len + n) / page) - 1 of a
 *                sequence's row are written, the others stay.  The k-th page that the step needs, counted sequence by
 *                sequence, column by column, is free_pages[*n_free - 1 - k]
 *   slots        int32 [n_tokens]: page * page_size + row of every new token, -1 for a token that got no slot and for rows
 *                that belong to no sequence
 *   positions    int32 [n_tokens]: cache_len + t, 0 for rows that belong to no sequence
 *   total_len    int32 [n_seq]: slots after this step, the next step's cache_len
 *   slots, positions and total_len are optional; each of them NULL: not written.
 * Without enough pages the first sequences get theirs, -1 goes into the columns that stay without, total_len ends where the
 * pages end, and a device check is recorded; so it is for slots at or behind table_width * page_size, and for ids on the
 * stack or in the table that are no pages (their tokens get slot -1).  Offsets that run backwards end the list of sequences
 * as for samkv_prefill.  Outputs must not overlap one another or the inputs.  With n_tokens == 0 total_len and n_free_out are
 * still written. */
samkv_status_t samkv_page_tables(samkv_handle_t h, const samkv_packed_t* packed, const int32_t* cache_len, int32_t page_size,
                                 int32_t n_pages, int32_t* block_table, int32_t table_width, const int32_t* free_pages,
                                 const int32_t* n_free, int32_t* n_free_out, int32_t* slots, int32_t* positions,
                                 int32_t* total_len, void* stream);

/* Puts the pages of finished sequences back: for every s with done[s] != 0 the first ceil(lengths[s] / page_size) entries of
 * its row go on the stack, the last sequence's last page first (so that handing the same pages out again restores the table).
 *   lengths  int32 [n_seq] device: slots the sequence holds (clamped to [0, table_width * page_size] with a device check)
 *   done     uint8 [n_seq] device
 * Table and lengths are not changed: a row is used again by giving it length 0.  What the stack cannot hold (n_pages
 * entries) is dropped and recorded as a device check; an entry that is no page is recorded, too, and put on the stack, from
 * which samkv_page_tables hands it to nobody.  1 <= n_seq <= SAMKV_MAX_SEQ. */
samkv_status_t samkv_release_pages(samkv_handle_t h, int32_t n_seq, const int32_t* block_table, int32_t table_width,
                                   int32_t page_size, int32_t n_pages, const int32_t* lengths, const uint8_t* done,
                                   int32_t* free_pages, const int32_t* n_free, int32_t* n_free_out, void* stream);

/* ---- positions of several axes, append through the slot map ------------------------------------------------ */

#define SAMKV_MAX_AXES 4

/* Rotary encoding by positions of several axes (time, height and width of an image's or video's patches): pair i turns by
 * positions[pair_axis[i]][t] * base^(-2i/rot_dim), or * inv_freq[i].  Sections of the pairs and axes that take turns are both
 * such maps. */
typedef struct {
  samkv_rope_t rope;
  int32_t n_axes;              /* 1 .. SAMKV_MAX_AXES */
  const int32_t* pair_axis;    /* host [rot_dim/2], each in [0, n_axes); read during the call */
} samkv_rope_axes_t;

/* samkv_append with positions of several axes and with the slot map of samkv_page_tables.
 *   rope         NULL: no rotation
 *   positions    int32 device: axis a of token t at positions[a * axis_stride + t]; axis_stride (elements) >= n_tokens, or 0:
 *                every axis has the same positions (text).  NULL (only without slots): cache_len[s] + t on every axis
 *   slots        int32 [n_tokens] device: token t goes to slot slots[t] of the pools, counted page * page_size + row; tokens
 *                with a negative one are left out altogether (nothing of theirs is written anywhere), one at or behind n_pages *
 *                page_size is left out, too, and recorded as a device check.  The sequences, cache_len and the block table are
 *                then not looked at.  Two tokens must not share a slot.  NULL: as samkv_append finds them
 * Everything else as for samkv_append.  slots without pages: SAMKV_ERR_INVALID_ARG. */
samkv_status_t samkv_append_axes(samkv_handle_t h, const samkv_packed_t* packed, const samkv_rows_t* K,
                                 const samkv_rows_t* V, const samkv_pages_t* pages, const int32_t* cache_len,
                                 const int32_t* slots, const samkv_rope_axes_t* rope, const int32_t* positions,
                                 int64_t axis_stride, const samkv_rows_t* Q, const samkv_rows_t* Q_out,
                                 const samkv_rows_t* K_out, const samkv_rows_t* V_out, void* stream);

/* ---- attention with modified scores ------------------------------------------------------------------------ */

/* What happens to a score between the product and the softmax, and which slots a token sees.  A token at position p (slot p
 * of its sequence: cache_len[s] + t, or t in samkv_prefill_scores) and slot j of the same sequence:
 *   x = scale * <q, k_j>
 *   x = softcap * tanh(x / softcap)             if softcap > 0
 *   x = x - slopes[hq] * |p - j|                if slopes are given
 * and j is seen if j < prefix_len[s] (whatever p is), or if
 *   j <= p (j < cache_len[s] for samkv_paged_attn_scores without causal),  j >= doc_start[token],  and  p - j < window.
 * The prefix's own tokens see one another in both directions (the prefix of a prefix language model).  In a causal model, put
 * nothing into a prefix but slots that lie before the call's tokens, prefix_len[s] <= cache_len[s]: a shared instruction goes
 * first, by a call without a prefix; documents that do not see one another (doc_start) and a question that sees all of them
 * (doc_start 0) follow as one chunk of samkv_paged_attn_scores, with the instruction as their prefix.  So it is for the initial
 * tokens that a sliding window keeps.
 * Slots a token does not see never reach it, infinities and NaN included; a token that sees none gets O = 0, lse = -inf. */
typedef struct {
  float softcap;               /* 0: scores are not capped; else 2^-126 .. 1e30, and scale / softcap must be finite */
  int32_t window;              /* >= 0; 0: no window */
  const float* slopes;         /* device [n_q_heads], finite, any sign; NULL: none */
  const int32_t* prefix_len;   /* device [n_seq], any value (a sequence's own slots bound it); NULL: 0 */
  const int32_t* doc_start;    /* device [n_tokens], any value; NULL: 0 */
} samkv_scores_t;

/* Bytes of workspace that the two calls below need in their handle, never less than samkv_packed_workspace_bytes, so that
 * such a handle serves the calls above as well.  It holds the division of the work, which depends on the masks, besides the
 * partial results.  0 on a bad description. */
size_t samkv_scores_workspace_bytes(const samkv_packed_t* packed);

/* samkv_prefill with modified scores.  scores == NULL, or a description that modifies nothing: samkv_prefill itself.
 * Precision as there; the cap is good to 2^-20 of its value.  bf16 prompts and chunks: products of weights and values are formed
 * with weights of 2^-16 at least for a row's largest score (and up to 2^16), so that values of V below about 2^-100 can be lost. */
samkv_status_t samkv_prefill_scores(samkv_handle_t h, const samkv_packed_t* packed, const samkv_rows_t* Q,
                                    const samkv_rows_t* K, const samkv_rows_t* V, float scale, const samkv_scores_t* scores,
                                    const samkv_rows_t* O, float* lse, void* stream);

/* samkv_paged_attn with modified scores.  Table entries of pages none of whose slots any token sees are not used (any value),
 * so that pages a window has passed can be given back.  scores == NULL, or a description that modifies nothing:
 * samkv_paged_attn itself. */
samkv_status_t samkv_paged_attn_scores(samkv_handle_t h, const samkv_packed_t* packed, const samkv_pages_t* pages,
                                       const int32_t* cache_len, const samkv_rows_t* Q, float scale, int32_t causal,
                                       const samkv_scores_t* scores, const samkv_rows_t* O, float* lse, void* stream);

/* ---- scoring without any allocation ------------------------------------------------------ */

/* (No counterpart in the paper: this entry point exists for deployment reasons only.)
 * Same result as samkv_score, for callers that cannot call cudaMalloc or hand over a workspace:
 * a serving engine whose memory pool already owns all of HBM, or a latency-critical section in
 * which an allocation (which may synchronise the whole device) is not allowed.  It takes no handle.
 * The personalised query vectors, the only scratch this step needs, live in a fixed array inside
 * the library's device image: SAMKV_STATIC_SCORE_MAX_FLOATS fp32 values (1 MiB), held by every GPU
 * that loads the library until the process exits.
 *   - n_layers * batch * n_ctx * n_kv_heads * head_dim must not exceed SAMKV_STATIC_SCORE_MAX_FLOATS
 *     (one layer of any configuration in this repository fits; call it layer by layer), otherwise
 *     SAMKV_ERR_WORKSPACE is returned and nothing is launched.
 *   - The first call on a device looks up the array's device address (once per device, with that
 *     device current).  Make that first call outside any stream capture.
 *   - All calls share the one array: two calls whose kernels can overlap on the GPU (different
 *     streams, or several threads) race on it.  Order them on one stream.  The array keeps the last
 *     call's contents; every element a call reads is rewritten by that call first, so no clearing
 *     is needed.
 *   - Calls no cudaMalloc / cudaFree or any other allocating routine.
 *   - There is no handle and therefore no status word: a device-side check that samkv_score would record for
 *     samkv_poll_status (a bounded wait inside the scoring kernel that ran out) is NOT reported by this entry
 *     point.  The kernel still gives up and returns, part of scores_out is then left unwritten, and the call
 *     has long returned SAMKV_OK.  A caller that needs that report uses samkv_score with a workspace.
 * Arguments as in samkv_score (K, Q, Qloc, scores_out are caller-owned device pointers). */
#define SAMKV_STATIC_SCORE_MAX_FLOATS (256 * 1024)
samkv_status_t samkv_score_static(const samkv_shape_t* shape, const void* K, const void* Q, int32_t T_q,
                                  const void* Qloc, int32_t T_loc, int32_t use_bias, float* scores_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SAMKV_H_ */
