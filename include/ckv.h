/*
 * ckv.h -- C ABI of the CompilerKV prefill-end retention step for AMD MI355X (gfx950).
 *
 * The library implements the online pass of CompilerKV (paper Sec. 4, Alg. 1) for ONE layer per call
 * sequence, cut into four asynchronous calls that are queued back-to-back on one HIP stream:
 *
 *   ckv_window_scores -> ckv_apply_tables -> ckv_select_topk -> ckv_compact_kv
 *
 * Further entry points, each documented where it is declared: ckv_window_lse (the scan's first half),
 * ckv_window_utility (the first two calls as one, without the per-head masses in memory), the calls of
 * the paper's layer-shared mode (ckv_alpha_accumulate, ckv_risk_struct, ckv_shared_utility,
 * ckv_compact_kv_shared), the depth mapping of compiled tables (ckv_map_table_depth), a decode-side consumer of the compact cache (ckv_decode_attention,
 * ckv_discarded_mass), and the calls of a cache that goes on: norm and position rotation of new rows (ckv_norm_rotate), their way into pages
 * (ckv_paged_append) and attention of new tokens over the pages (ckv_paged_attention); for trees of drafted tokens ckv_tree_sees and
 * ckv_paged_tree_attention; rows and pages that move (ckv_paged_compact, ckv_pages_copy) and lists that share pages, get some and give them
 * back (ckv_pages_fork, ckv_pages_reserve, ckv_pages_free).
 *
 * Notation (paper Sec. 3-4): T = prompt length (keys/values cached at the end of prefill, the
 * observation window included), W = |Omega| = observation window (the last W query positions),
 * P = T - W = prefix length that competes for the budget, Hq / Hkv = query / key-value heads,
 * G = Hq / Hkv (query heads [g*G, (g+1)*G) share KV head g), d = head_dim, B = token budget per KV
 * head (the W window slots included), B_tot = B * Hkv = the layer's total.
 *
 * Conventions that hold for every entry point unless a comment says otherwise:
 *   - every data pointer is a DEVICE pointer owned by the caller; the library never allocates, frees
 *     or keeps device memory, keeps no state between calls and never synchronises;
 *   - `params` is a HOST pointer, read during the call only;
 *   - every call only enqueues work on `hip_stream` (a hipStream_t passed as void*; NULL = the
 *     default stream) and returns; outputs are valid once the stream reaches that point;
 *   - inputs are never written; outputs must not alias inputs or each other;
 *   - calls may be queued on different streams (and from different host threads) and overlap on the
 *     GPU as long as they share no output and no workspace: give every stream a workspace of its own
 *     (ckv_window_lse_static, whose scratch is the library's, is the exception: see there);
 *   - arguments are validated on the host BEFORE anything is launched: on any error nothing has
 *     been enqueued and the status says why (ckv_status_string gives text);
 *   - tensors are dense row-major in the order written in their comment, except Q/K/V which carry
 *     explicit (batch, head, token) strides in ELEMENTS with the head_dim axis contiguous.
 */
#ifndef CKV_H_
#define CKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CKV_OK = 0,
  CKV_EINVAL = 1,       /* a null pointer, a size or a flag outside the documented domain          */
  CKV_EUNSUPPORTED = 2, /* valid, but not built (e.g. head_dim other than 64 / 128, W > 128)       */
  CKV_EWORKSPACE = 3,   /* workspace missing, misaligned (256 B) or smaller than ckv_workspace_bytes */
  CKV_EHIP = 4          /* the HIP runtime refused a launch; see hipGetLastError                   */
} ckv_status;

typedef enum { CKV_F32 = 0, CKV_BF16 = 1 } ckv_dtype;              /* element type of Q, K, V      */
typedef enum { CKV_POOL_NONE = 0, CKV_POOL_AVG = 1, CKV_POOL_MAX = 2 } ckv_pool;

/* flags */
enum {
  CKV_FLAG_VALUE_NORM = 1u, /* multiply the window mass by the value-norm ratio rho (paper Eq. 4)  */
  /* Layer-shared mode only (paper Eq. 4: alpha is a mean over heads): ckv_window_scores writes, instead
   * of every query head's mass, the SUM over the query heads of each KV head, scores [Bz,Hkv,T], and
   * ckv_alpha_accumulate reads that layout -- a quarter of the bytes for groups of four. Exists for
   * bf16 with W <= 32 and G <= 4 (CKV_EUNSUPPORTED otherwise); rejected by
   * the calls that need per-head masses (ckv_apply_tables, ckv_window_utility).                      */
  CKV_FLAG_GROUP_MASS = 8u
};

/* Problem description shared by all calls. Plain data; the caller may reuse or free it after a call. */
typedef struct {
  int32_t batch;          /* Bz >= 1                                                               */
  int32_t n_q_heads;      /* Hq, a multiple of n_kv_heads                                          */
  int32_t n_kv_heads;     /* Hkv >= 1                                                              */
  int32_t head_dim;       /* d: 64 or 128                                                          */
  int32_t seq_len;        /* T, window included; 1 <= W <= T                                       */
  int32_t window;         /* W                                                                     */
  int32_t layer;          /* row of the compiled tables used by this call, 0 <= layer < n_layers   */
  int32_t n_layers;       /* rows in w_head / head_share / t_gate                                  */
  int32_t dtype;          /* ckv_dtype of q_win, k, v, k_out, v_out                                */
  float softmax_scale;    /* logit scale; 0 selects 1/sqrt(head_dim) (paper Sec. 3)                */
  int64_t q_stride[3];    /* element strides of q_win over (batch, q head, window row)             */
  int64_t k_stride[3];    /* element strides of k over (batch, kv head, token)                     */
  int64_t v_stride[3];    /* element strides of v over (batch, kv head, token)                     */
  int32_t pool;           /* ckv_pool: 1-D pooling of the window mass along the token axis         */
  int32_t pool_kernel;    /* odd, 1..63; ignored for CKV_POOL_NONE                                 */
  int32_t budget_per_kv_head; /* B, W <= B (window slots included)                                 */
  int32_t cap;            /* rows per (batch, kv head) in idx / k_out / v_out;
                             cap >= min(T, B_tot - (Hkv-1)*W), the largest budget one head can get */
  uint32_t flags;         /* CKV_FLAG_*                                                            */
} ckv_params;

/* Bytes of scratch for the calls of one layer with `params` (they may share one buffer because they run in stream
 * order). Returns 0 if `params` is NULL or invalid. The buffer must be 256-byte aligned.
 * Beyond 32768 prefix positions the figure depends on budget_per_kv_head and cap too: for small budgets the selection
 * keeps (key, position) pairs, up to 512 KiB per (batch, KV head). A buffer of what this returns for any one budget
 * and cap serves every other of the same shape (a caller with budgets that differ by layer needs one): where it has no
 * room for the pairs, the selection takes its form with 16 KiB per (batch, KV head). */
size_t ckv_workspace_bytes(const ckv_params *params);

/*
 * Observation-window scan (paper Sec. 3 attention definition, Eq. 3 "the O(LHTW) scan", Eq. 4's
 * alpha_t taken per query head, Alg. 1 step (A)).
 *
 * For every batch element b, query head h and key position t in [0, T):
 *     z[j,t]      = softmax_scale * <q_win[b,h,j,:], k[b,g(h),t,:]>            j in [0, W)
 *     A[j,t]      = exp(z[j,t] - LSE_j),  LSE_j = log sum_{t' <= P+j} exp z[j,t']   (causal: window
 *                   row j sits at absolute position P+j and sees keys t' <= P+j; A[j,t] = 0 beyond)
 *     scores[b,h,t] = (T / W) * sum_j A[j,t]
 * so that sum_t scores[b,h,t] = T (mean one, the paper's scale normalisation).
 *
 *   q_win        in   [Bz,Hq,W,d]  via q_stride; the last W query rows of the prompt
 *   k            in   [Bz,Hkv,T,d] via k_stride
 *   v            in   [Bz,Hkv,T,d] via v_stride; read only with CKV_FLAG_VALUE_NORM, else may be NULL
 *   lse          in   optional [Bz,Hq,W] fp32 natural-log LSE_j as defined above (for callers whose
 *                     prefill attention kernel already produced it); NULL = computed here with one
 *                     extra pass over K
 *   scores       out  [Bz,Hq,T] fp32
 *   vnorm_ratio  out  [Bz,Hkv,T] fp32, rho[t] = ||v_t||_2 / (mean_{t'<T} ||v_t'||_2 + 1e-6)
 *                     (paper Eq. 4, Alg. 1 Stage 1); required with CKV_FLAG_VALUE_NORM, else ignored
 *   workspace         ckv_workspace_bytes(params) bytes, contents undefined before and after
 * Accumulation is fp32 (bf16 inputs go through bf16 MFMA with fp32 accumulators).
 */
ckv_status ckv_window_scores(const ckv_params *params, const void *q_win, const void *k,
                             const void *v, const float *lse, float *scores, float *vnorm_ratio,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * First half of the scan on its own: LSE_j of every window row, as defined above (the softmax
 * normaliser of the paper's attention definition, Sec. 3), for callers that want to keep it or to
 * overlap the two passes themselves. ckv_window_scores(lse = NULL) runs exactly this internally.
 *
 *   q_win, k   in   as for ckv_window_scores
 *   lse        out  [Bz,Hq,W] fp32, natural log
 *   workspace       ckv_workspace_bytes(params) bytes
 */
ckv_status ckv_window_lse(const ckv_params *params, const void *q_win, const void *k, float *lse,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ckv_window_lse for callers that cannot allocate device memory or hand over a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation. Same arguments, same
 * kernels and bit-identical results as ckv_window_lse; the row partials of the pass live in a device
 * array inside the library (CKV_STATIC_SCRATCH_BYTES per GPU the library runs on, held until the process
 * ends) instead of a workspace. Neither this call nor anything it calls allocates or frees memory. The
 * first call on a device looks the array's address up (once per device).
 *
 * Returns CKV_EWORKSPACE, before anything is launched, when the shape needs more than the array holds:
 * ckv_window_lse_static_bytes(params) gives the need (0 for invalid params); it is
 * 8 bytes * batch * Hkv * (query rows of a KV head, padded to whole 32-row tiles) * (workgroups along
 * the key axis), e.g. 256 KiB for batch 16, 8 KV heads, 4 x 32 query rows at T = 32768.
 * Every call on one GPU uses that GPU's one array, whose contents are undefined between calls: calls
 * that overlap on one GPU (two streams, two threads) race; calls in stream order on one stream do not.
 */
#define CKV_STATIC_SCRATCH_BYTES (4u << 20)
size_t ckv_window_lse_static_bytes(const ckv_params *params);
ckv_status ckv_window_lse_static(const ckv_params *params, const void *q_win, const void *k, float *lse,
                                 void *hip_stream);

/*
 * Pooling, compiled-table lookups and budgets (paper Eq. 6 weighted max over heads, Sec. 4.3 gate
 * lookup, Alg. 1 Stages 2-3 up to the threshold; the 1-D pooling and the per-head budget split are
 * the build's workload definition, not the paper's).
 *
 * For every b, kv head g and prefix position t in [0, P):
 *     c[h,t]  = pool_k(scores[b,h,0:P])[t]   centred, stride 1, same length; AVG divides by
 *               pool_kernel with zeros outside [0,P); MAX ignores positions outside [0,P)
 *     u[h,t]  = c[h,t] * vnorm_ratio[b,g,t]  (with CKV_FLAG_VALUE_NORM, else u = c)
 *     utility[b,g,t] = max_{h in group g} fp32(w_head[layer,h] * u[h,t])
 * and
 *     tau[b]  = t_gate[layer, risk_bins[b,0], risk_bins[b,1]]       (0 if t_gate is NULL: gate off)
 *     budget[b,g]: NULL head_share => min(B, T). Else b_g = floor(head_share[layer,g] * B_tot) evaluated in
 *               fp64, clamped to [W, T]; while sum_g b_g > B_tot the largest b_g that is > W (lowest
 *               g on ties) is decremented by one.
 *
 *   scores       in   [Bz,Hq,T] fp32 (from ckv_window_scores)
 *   vnorm_ratio  in   [Bz,Hkv,T] fp32, required with CKV_FLAG_VALUE_NORM
 *   w_head       in   [n_layers,Hq] fp32, finite and > 0 (paper grid: [0.8,1.5])
 *   head_share   in   [n_layers,Hkv] fp32 >= 0, or NULL
 *   t_gate       in   [n_layers,n_ent,n_ppl] fp32 >= 0 (paper grid: 20 x 4, values in [0.8,1.0]), or NULL
 *   risk_bins    in   [Bz,2] int32 (b_ent, b_ppl), required with t_gate; out-of-range bins are
 *                     clamped into the table on the device (they cannot be checked on the host)
 *   utility      out  [Bz,Hkv,P] fp32
 *   budget       out  [Bz,Hkv] int32
 *   tau          out  [Bz] fp32
 */
ckv_status ckv_apply_tables(const ckv_params *params, const float *scores, const float *vnorm_ratio,
                            const float *w_head, const float *head_share, const float *t_gate,
                            int32_t n_ent, int32_t n_ppl, const int32_t *risk_bins, float *utility,
                            int32_t *budget, float *tau, void *hip_stream);

/*
 * ckv_window_scores followed by ckv_apply_tables as ONE call that does not materialise the per-head
 * window mass: same definitions, same utility / budget / tau (within fp32 rounding of the pooled sum),
 * for callers that only need what the selection consumes (paper Alg. 1 from the window scan up to the
 * threshold). Where the shape allows it (bf16, W <= 64, G*ceil(W/32) <= 8, pooling kernel <= 7)
 * the scan's second pass pools, weights and maximises over the group's heads on
 * chip and writes [Bz,Hkv,P] instead of [Bz,Hq,T] (with CKV_FLAG_VALUE_NORM the ratio, common to a
 * group's heads, then multiplies the group maximum); otherwise the two steps run one after the other
 * through `scores_scratch`.
 *
 *   q_win, k, v, lse                                   as for ckv_window_scores
 *   w_head, head_share, t_gate, n_ent, n_ppl, risk_bins as for ckv_apply_tables
 *   scores_scratch  scratch  [Bz,Hq,T] fp32; contents undefined on return
 *   vnorm_ratio     out      as for ckv_window_scores (required with CKV_FLAG_VALUE_NORM, else ignored)
 *   utility, budget, tau  out  as for ckv_apply_tables
 *   workspace                ckv_workspace_bytes(params) bytes
 */
ckv_status ckv_window_utility(const ckv_params *params, const void *q_win, const void *k, const void *v,
                              const float *lse, const float *w_head, const float *head_share,
                              const float *t_gate, int32_t n_ent, int32_t n_ppl, const int32_t *risk_bins,
                              float *scores_scratch, float *vnorm_ratio, float *utility, int32_t *budget,
                              float *tau, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Elastic candidate pool with budget clamp (paper Eq. 8, Alg. 1 Select), per (b, kv head g):
 *     cand = { t < P : utility[b,g,t] >= tau[b] },  kp = budget[b,g] - W
 *     Sp   = cand                                         if |cand| <= kp
 *          = the kp members of cand that come first under (utility descending, t ascending) otherwise
 *     idx[b,g,:] = Sp in ascending t, then the window P..T-1;   count[b,g] = |Sp| + W
 * Utilities must be non-negative and not NaN (they are sums of softmax weights times positive
 * weights); the order of equal utilities is by position, so the result is unique.
 *
 *   utility  in   [Bz,Hkv,P] fp32      budget in [Bz,Hkv] int32 (values are clamped to [W, min(cap,T)]
 *   tau      in   [Bz] fp32                       on the device)
 *   idx      out  [Bz,Hkv,cap] int32; entries at and beyond count[b,g] are not written
 *   count    out  [Bz,Hkv] int32
 *   workspace     optional (NULL allowed). Up to 32768 prefix positions it is not used. Beyond that,
 *                 with ckv_workspace_bytes() bytes for this shape and any budget (256-byte aligned;
 *                 CKV_EWORKSPACE if misaligned or smaller) a unit's positions are split over several
 *                 workgroups, which is several times faster for long contexts with few (batch, head)
 *                 units; the result is the same either way. Contents on entry are ignored.
 */
ckv_status ckv_select_topk(const ckv_params *params, const float *utility, const int32_t *budget,
                           const float *tau, int32_t *idx, int32_t *count, void *workspace,
                           size_t workspace_bytes, void *hip_stream);

/*
 * Token-axis gather (paper Sec. 3 "K~ = K[S], V~ = V[S]", Alg. 1 Gather_tok): for r < count[b,g]
 *     k_out[b,g,r,:] = k[b,g,idx[b,g,r],:]    v_out[b,g,r,:] = v[b,g,idx[b,g,r],:]     (bit copies)
 *
 *   k, v          in   via k_stride / v_stride
 *   idx, count    in   from ckv_select_topk; indices outside [0,T) are skipped on the device
 *   k_out, v_out  out  [Bz,Hkv,cap,d] dense, same dtype; rows at and beyond count are not written
 */
ckv_status ckv_compact_kv(const ckv_params *params, const void *k, const void *v, const int32_t *idx,
                          const int32_t *count, void *k_out, void *v_out, void *hip_stream);

/*
 * A layer's whole step as one call: ckv_window_utility (scores_wanted = 0; `scores` is its scratch) or
 * ckv_window_scores + ckv_apply_tables (scores_wanted != 0), then ckv_select_topk and ckv_compact_kv, with the
 * same arguments, outputs and order on the stream. What one of them would refuse is refused with its status, the first one's
 * first, before anything is launched. `v` is read by the gather and, with CKV_FLAG_VALUE_NORM, by the scan;
 * workspace as for ckv_window_scores.
 */
ckv_status ckv_retention_layer(const ckv_params *params, const void *q_win, const void *k, const void *v,
                               const float *lse, const float *w_head, const float *head_share,
                               const float *t_gate, int32_t n_ent, int32_t n_ppl, const int32_t *risk_bins,
                               float *scores, int32_t scores_wanted, float *vnorm_ratio, float *utility,
                               int32_t *budget, float *tau, int32_t *idx, int32_t *count, void *k_out,
                               void *v_out, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Layer-shared mode: the paper's Alg. 1 as printed, where ONE window mass alpha serves every layer and
 * head and every layer keeps ONE index set for all its heads. Order of calls for a prompt:
 *   for each layer: ckv_window_scores (with CKV_FLAG_VALUE_NORM: rho of that layer) and
 *                   ckv_alpha_accumulate(weight = 1 / (n_layers * Hq))                  -- Alg. 1 (A)
 *   once:           ckv_risk_struct                                                     -- Alg. 1 (A)
 *   for each layer: ckv_shared_utility, ckv_select_topk with a one-head ckv_params (batch, 1 query head,
 *                   1 KV head, budget = B_l; utility [Bz,1,P], budget [Bz,1]), ckv_compact_kv_shared.
 *
 * ckv_alpha_accumulate: alpha[b,t] += weight * sum_h scores[b,h,t] (with CKV_FLAG_GROUP_MASS: the sum
 * over the Hkv rows of the group-mass layout). With weight = 1/(L*Hq) over all
 * layers this is alpha = (T/W) sum_{j in Omega} Abar[j,:] for Abar the mean of A over layers and heads
 * (paper Eq. 4, Alg. 1 (A)); sum_t alpha = T.
 *   scores  in      [Bz,Hq,T] fp32 of one layer (from ckv_window_scores)
 *   alpha   in/out  [Bz,T] fp32; the caller clears it before the first layer
 */
ckv_status ckv_alpha_accumulate(const ckv_params *params, const float *scores, float weight, float *alpha,
                                void *hip_stream);

/*
 * Structural risk coordinate (paper Eq. 7, Alg. 1 (A)): risk[b] = -sum_t A'_t ln A'_t with
 * A' = alpha[b,:] / ||alpha[b,:]||_1 (terms with A'_t = 0 count as 0), and its bin
 * bin[b] = number of ent_edges <= risk[b] (ascending edges chosen by whoever compiled T_gate; the
 * paper does not fix them). Sums are formed in fp64 in a fixed order.
 *   alpha      in   [Bz,T] fp32, non-negative
 *   ent_edges  in   [n_edges] fp32 ascending (device), may be NULL when bin is NULL or n_edges = 0
 *   risk       out  [Bz] fp32           bin  out  [Bz] int32, or NULL
 */
ckv_status ckv_risk_struct(const ckv_params *params, const float *alpha, const float *ent_edges,
                           int32_t n_edges, float *risk, int32_t *bin, void *hip_stream);

/*
 * One utility vector per layer (paper Eq. 4 u = alpha * rho, Eq. 6, Alg. 1 (B)-(C)) and the gate
 * lookup (Sec. 4.3): for t in [0, P)
 *     utility[b,t] = max over ALL query heads h of fp32(w_head[layer,h] * (alpha[b,t] * vnorm_ratio[b,g(h),t]))
 *     tau[b]       = t_gate[layer, risk_bins[b,0], risk_bins[b,1]]      (0 if t_gate is NULL)
 * (the pooling fields of params are not used: the paper has no pooling).
 *   alpha        in   [Bz,T] fp32          vnorm_ratio  in  [Bz,Hkv,T] fp32 of this layer
 *   w_head, t_gate, n_ent, n_ppl, risk_bins   as for ckv_apply_tables
 *   utility      out  [Bz,P] fp32          tau  out  [Bz] fp32
 */
ckv_status ckv_shared_utility(const ckv_params *params, const float *alpha, const float *vnorm_ratio,
                              const float *w_head, const float *t_gate, int32_t n_ent, int32_t n_ppl,
                              const int32_t *risk_bins, float *utility, float *tau, void *hip_stream);

/*
 * Gather with one index set per batch element, shared by all KV heads of the layer (paper Alg. 1,
 * Gather_tok: one index set per layer serves every head): for r < count[b], every g
 *     k_out[b,g,r,:] = k[b,g,idx[b,r],:]    v_out[b,g,r,:] = v[b,g,idx[b,r],:]     (bit copies)
 *   idx  in  [Bz,cap] int32      count  in  [Bz] int32      k_out, v_out  out  [Bz,Hkv,cap,d]
 */
ckv_status ckv_compact_kv_shared(const ckv_params *params, const void *k, const void *v, const int32_t *idx,
                                 const int32_t *count, void *k_out, void *v_out, void *hip_stream);

/*
 * Depth mapping of a compiled table (paper App. "Model choice and cross-architecture applicability": tables
 * are compiled on a 32-layer backbone; models of another depth use a monotonic depth mapping, relative-
 * depth interpolation). mapped[l,:] is the linear interpolation of the two rows of `table` next to the
 * source coordinate x = l * (n_layers_src - 1) / (n_layers_dst - 1) (row 0 for n_layers_dst = 1). Works
 * for w_head ([L,Hq]: row_elems = Hq), head_share ([L,Hkv]) and t_gate ([L,n_ent,n_ppl]: row_elems =
 * n_ent * n_ppl). Table preparation, run once per model.
 *   table  in  [n_layers_src,row_elems] fp32      mapped  out  [n_layers_dst,row_elems] fp32
 */
ckv_status ckv_map_table_depth(const float *table, int32_t n_layers_src, int32_t row_elems, float *mapped,
                               int32_t n_layers_dst, void *hip_stream);

/*
 * Decode-side consumer of the compact cache (paper Sec. 4.5, Proposition 1; proof in App. A).
 *
 * ckv_decode_attention: attention of decoding queries over a ragged KV set. A decoding query sits after
 * the prompt and sees every row. For batch element b, query head h (KV head g = h / G), query i < n_q:
 *     z[j]   = softmax_scale * <q_dec[b,h,i,:], k_rows[b,g,j,:]>          j < n_valid(b,g)
 *     lse    = log sum_j exp z[j]
 *     out    = sum_j exp(z[j] - lse) * v_rows[b,g,j,:]
 * with n_valid(b,g) = count[b,g] clamped to [0, n_rows] (n_rows if count is NULL); rows behind n_valid are
 * not read (they need not be mapped). Over the compact
 * cache written by ckv_compact_kv (strides {Hkv*cap*d, cap*d, d}, n_rows = cap, the call's count) this
 * is the compressed row of Proposition 1, p~ = p restricted to the retained set and renormalised,
 * applied to V; over the full cache (params' k_stride / v_stride, n_rows = T, count = NULL) it is the
 * uncompressed attention and its lse is the full row's normaliser.
 *
 *   q_dec     in   [Bz,Hq,n_q,d] contiguous, params->dtype, 16-byte aligned
 *   k_rows, v_rows in  rows of (batch, kv head) at element strides k_stride / v_stride over
 *                  (batch, kv head, row); multiples of 16 bytes, row stride >= d; 16-byte aligned
 *   count     in   [Bz,Hkv] int32 or NULL
 *   out       out  [Bz,Hq,n_q,d] fp32 (zeros where no row is valid)
 *   lse       out  [Bz,Hq,n_q] fp32, natural log (-inf where no row is valid)
 *   workspace      ckv_decode_workspace_bytes(params, n_q, n_rows) bytes, 256-byte aligned. That
 *                  function returns 0 for arguments this call rejects, and also for short KV sets
 *                  (n_rows <= 4096), which one launch finishes without scratch: workspace may then
 *                  be NULL.
 *
 * ckv_discarded_mass: m[b,h,i] = 1 - exp(lse_kept - lse_full), the mass the full attention row had
 * outside the retained set (Proposition 1; the row's l1 error is exactly 2m), clamped to [0,1], and
 * eps_tail[b,h] = sqrt(mean_i m^2) (may be NULL).
 *   lse_full, lse_kept  in  [Bz,Hq,n_q] fp32     mass out [Bz,Hq,n_q] fp32     eps_tail out [Bz,Hq] fp32
 */
size_t ckv_decode_workspace_bytes(const ckv_params *params, int32_t n_q, int32_t n_rows);
ckv_status ckv_decode_attention(const ckv_params *params, const void *q_dec, int32_t n_q, const void *k_rows,
                                const void *v_rows, const int64_t *k_stride, const int64_t *v_stride,
                                int32_t n_rows, const int32_t *count, float *out, float *lse, void *workspace,
                                size_t workspace_bytes, void *hip_stream);
ckv_status ckv_discarded_mass(const ckv_params *params, int32_t n_q, const float *lse_full, const float *lse_kept,
                              float *mass, float *eps_tail, void *hip_stream);

/*
 * Paged caches: lists of pages for the rows that enter a cache after (or instead of) the retention step, and attention of new tokens
 * over them. A pool holds n_pages pages of page_rows rows for keys and one for values; a list names the pages of one (batch element,
 * KV head) in order, so row s of the list is row s % page_rows of page table[s / page_rows]. Lists of the heads of a sequence may be
 * one and the same (table_stride[1] = 0, pages that hold every head at k_stride[1]) or differ (retained lists of different lengths;
 * pages of one head: k_stride[1] = v_stride[1] = 0).
 *
 * Of ckv_params these calls use batch, n_q_heads, n_kv_heads, head_dim, dtype and softmax_scale; seq_len is n, the most new tokens that a
 * sequence has in the call, and q_stride / k_stride / v_stride describe the new rows q [Bz,Hq,n,d], k and v [Bz,Hkv,n,d]. The other
 * fields have to be valid (window = 1, budget_per_kv_head = 1, cap = 1 always are) and mean nothing here.
 *
 *   length  in  [Bz,Hkv] int32: rows of the list with the call's new rows, which are its last ones (what is below 0 counts as 0)
 *   count   in  [Bz,Hkv] int32 or NULL: new rows of the list, clamped to [0, n]; NULL: n. New row i is row length - count + i of
 *               the list; rows i >= count are neither read nor written, in any tensor of the call (their positions may be read).
 *               Query head h has the count and length of its KV head h / G.
 *   table   in  int32 page numbers at table_stride over (batch, KV head), max_pages in a row. A page number outside [0, n_pages),
 *               or a row outside [0, max_pages * page_rows): nothing is written there, and attention does not see the row.
 * A page may be in several lists (a shared prefix), or several times in one, as long as no call appends a row of it twice. Appending and
 * reading are calls in stream order. Outputs overlap no input of their call.
 */
typedef struct {
  int32_t page_rows;       /* rows of a page, a power of two, 1 .. 65536                            */
  int32_t n_pages;         /* pages of the pools, >= 1                                              */
  int32_t max_pages;       /* entries of a list in `table`, >= 1; max_pages * page_rows < 2^31      */
  int32_t reserved;        /* 0                                                                     */
  int64_t k_stride[3];     /* element strides of k_pages over (page, KV head, row): multiples of 16 bytes, row stride >= head_dim */
  int64_t v_stride[3];     /* the same of v_pages                                                   */
  int64_t table_stride[2]; /* entries of `table` between batch elements, between KV heads (0: one list for all heads) */
} ckv_pages;

typedef enum { CKV_PAIR_HALVES = 0, CKV_PAIR_NEIGHBOURS = 1 } ckv_pairing;

/*
 * What happens to a row x of d components on its way: with norm != 0
 *     y_c = x_c * weight_c / sqrt(mean_c' x_c'^2 + norm_eps)           (weight NULL: ones), else y = x,
 * then the first rot_dim components turn by the angles a_i = position * inv_freq[i], i < rot_dim / 2, in pairs
 *     (y_i, y_{i + rot_dim/2}) (CKV_PAIR_HALVES) or (y_{2i}, y_{2i+1}) (CKV_PAIR_NEIGHBOURS):
 *     (y, y') -> (y cos a - y' sin a, y' cos a + y sin a).
 * Sums and products are fp32 (the sum of the squares has to be finite there and mean square + norm_eps a normal number), angles fp64 reduced
 * to a turn; one rounding to the type at the end. With norm = 0 and rot_dim = 0 rows are copied bit for bit.
 */
typedef struct {
  int32_t rot_dim;   /* 0 .. head_dim, a multiple of 8                                              */
  int32_t pairing;   /* ckv_pairing                                                                 */
  int32_t norm;      /* 0 or 1                                                                      */
  float norm_eps;    /* finite, >= 0                                                                */
} ckv_rotation;

/*
 * Norm of every head of new queries and keys and their position rotation in one pass.
 *   q, k        in   [Bz,Hq,n,d] / [Bz,Hkv,n,d] via q_stride / k_stride; either may be NULL, with its output
 *   positions   in   [Bz,n] int32; required with rot_dim > 0
 *   inv_freq    in   [rot_dim / 2] fp32, angle per position of each pair; required with rot_dim > 0
 *   q_weight, k_weight  in  [d] of params->dtype, 16-byte aligned, or NULL; read only with norm
 *   count       in   as above, or NULL
 *   q_out, k_out  out  [Bz,Hq,n,d] / [Bz,Hkv,n,d] dense
 * Row pointers are 16-byte aligned here and in the calls below.
 */
ckv_status ckv_norm_rotate(const ckv_params *params, const ckv_rotation *rotation, const void *q, const void *k,
                           const int32_t *positions, const float *inv_freq, const void *q_weight, const void *k_weight,
                           const int32_t *count, void *q_out, void *k_out, void *hip_stream);

/*
 * New rows into the pages: k normalised and rotated on the way, v as it is, and in the same launch q normalised and rotated to q_out
 * (the queries of the attention that follows). rotation NULL copies k and q: rows that the retention step kept
 * (k_out / v_out of ckv_compact_kv with its count as both length and count, strides {Hkv*cap*d, cap*d, d}, n = cap) move into pages this way.
 *   k, v        in   [Bz,Hkv,n,d] via k_stride / v_stride
 *   q           in   [Bz,Hq,n,d] via q_stride, or NULL with q_out = NULL
 *   positions, inv_freq, q_weight, k_weight   as for ckv_norm_rotate. Positions are the prompt's, not places in the list:
 *                    the retention step moves rows, their rotation stays
 *   table, length, count           as above; length is required
 *   k_pages, v_pages  out  new rows only, everything else in the pools stays as it is
 *   q_out       out  [Bz,Hq,n,d] dense
 */
ckv_status ckv_paged_append(const ckv_params *params, const ckv_rotation *rotation, const ckv_pages *pages, const void *q,
                            const void *k, const void *v, const int32_t *positions, const float *inv_freq, const void *q_weight,
                            const void *k_weight, const int32_t *table, const int32_t *length, const int32_t *count,
                            void *k_pages, void *v_pages, void *q_out, void *hip_stream);

/*
 * Attention of new tokens over the pages (the new rows included, so behind the call that appends them). New token i < count of a
 * sequence sees the rows j <= length - count + i of its head's list that are below n_rows and whose page number is in the pool:
 *     z[j] = softmax_scale * <q[b,h,i,:], k row j>,  lse = log sum_j exp z[j],  out = sum_j exp(z[j] - lse) * v row j
 * What a token does not see has no influence, whatever it holds (infinities and NaN included). A token that sees no row gets zeros and
 * lse = -inf. A row whose logit is -infinity counts as one that is not seen. With n = 1 this is a decoding step; lse of a prompt's last W tokens is the `lse` of
 * ckv_window_scores, lse of two caches is what ckv_discarded_mass takes.
 *   n_rows      no list is longer, 1 .. max_pages * page_rows and at most 2^24; a bound near the lengths lets the call share its work out well
 *   q           in   [Bz,Hq,n,d] via q_stride
 *   out         out  [Bz,Hq,n,d] of params->dtype at element strides out_stride over (batch, query head, token), multiples of 16 bytes
 *                    and each >= head_dim, or dense (out_stride NULL)
 *   lse         out  [Bz,Hq,n] fp32, natural log, or NULL
 *   workspace        ckv_paged_workspace_bytes(params, n_rows) bytes, 256-byte aligned; NULL where that is 0 (it is for refused arguments
 *                    too). Contents undefined before and after.
 * Logits and sums are fp32; in bf16 the weights enter the second product rounded to bf16, as the output is, or, in calls of at most 64 new
 * tokens times heads of a group, off by 2^-16 of themselves.
 * A mean of finite values is finite, however large they are; logits have to be below 2^24 in absolute value, where fp32 still tells neighbours apart by one.
 */
size_t ckv_paged_workspace_bytes(const ckv_params *params, int32_t n_rows);
ckv_status ckv_paged_attention(const ckv_params *params, const ckv_pages *pages, const void *q, const void *k_pages,
                               const void *v_pages, const int32_t *table, const int32_t *length, const int32_t *count, int32_t n_rows,
                               void *out, const int64_t *out_stride, float *lse, void *workspace, size_t workspace_bytes,
                               void *hip_stream);

/*
 * Trees of drafted tokens. Several continuations of a sequence are verified together: its new tokens are the nodes of a tree (or of several, whose roots
 * all follow the rows in front of them), a token behind its parent in the call's order. What a token sees of the new ones is a word of bits:
 * bit t % 64 of sees[b][i][t / 64] says whether token i sees token t.
 *
 * ckv_tree_sees makes them of parents: token i sees itself and what its parent sees, and stands one position behind it.
 *   batch, n    sizes, 1 <= n <= 4096
 *   parent      in   [batch,n] int32; a value that is not one of 0 .. i - 1 makes token i a root
 *   start       in   [batch] int32: a root's position; may be NULL with positions
 *   sees        out  [batch,n,ceil(n/64)] 64-bit words
 *   positions   out  [batch,n] int32, what ckv_norm_rotate and ckv_paged_append take, or NULL; overlaps neither `parent` nor `start`
 *
 * ckv_paged_tree_attention is ckv_paged_attention with these words in place of the causal order among the new tokens: token i < count sees the rows
 * j < length - count, and row length - count + t for t <= i where its bit t is set. Words of any origin do (a token without bits sees the rows in
 * front of the new ones alone, and one that sees no row gets zeros and lse = -inf); bits of tokens behind i are not looked at. n is 65536 at most.
 * In bf16 the weights enter the second product off by 2^-16 of themselves in calls of any size, as in a one-token step.
 *   sees        in   [Bz,n,ceil(n/64)] 64-bit words, one set for all heads
 *   the others       as for ckv_paged_attention, the workspace too
 */
ckv_status ckv_tree_sees(int32_t batch, int32_t n, const int32_t *parent, const int32_t *start, uint64_t *sees, int32_t *positions,
                         void *hip_stream);
ckv_status ckv_paged_tree_attention(const ckv_params *params, const ckv_pages *pages, const void *q, const void *k_pages,
                                    const void *v_pages, const int32_t *table, const int32_t *length, const int32_t *count, int32_t n_rows,
                                    const uint64_t *sees, void *out, const int64_t *out_stride, float *lse, void *workspace,
                                    size_t workspace_bytes, void *hip_stream);

/*
 * Rows that stay, moved together inside their pages: of the last `count` rows of a list (all of them with count NULL) those named by idx become
 * the first, the list ends behind them. With first = length - count and m = kept clamped to [0, count] and to cap, for r < m
 *     row first + r <- row first + idx[b,g,r]  (bit copies of keys and values),  length_out[b,g] = first + m
 * This drops rejected tokens of a tree (count: its tokens, idx: the accepted path), or does in the pages what ckv_compact_kv does beside them
 * (idx and kept: idx and count of ckv_select_topk). Rows behind length_out keep what they held or got; ckv_pages_free gives back their pages.
 *   Of ckv_params batch, n_kv_heads, head_dim and dtype are used; the other fields have to be valid.
 *   table, length, count  as above, but count is clamped to [0, length]
 *   idx         in   numbers below count, ascending, none twice, at element strides idx_stride over (batch, KV head) (0: one for all heads);
 *                    idx_stride NULL: [Bz,Hkv,cap]. A number that is not below count, or a row that is on no page: nothing is written for it.
 *                    In another order rows get some row's former or present contents, nothing else is touched
 *   cap         entries of a list in idx, >= 1
 *   kept        in   [Bz,Hkv] int32
 *   k_pages, v_pages  in/out; pages that are written are in no other list, or other lists see the change (ckv_pages_reserve gives lists pages of
 *                    their own). Heads with a list in common have rows of their own (with table_stride[1] = 0 neither head stride is 0)
 *   length_out  out  [Bz,Hkv] int32, overlaps none of `length`, `count` and `kept`
 */
ckv_status ckv_paged_compact(const ckv_params *params, const ckv_pages *pages, const int32_t *table, const int32_t *length, const int32_t *count,
                             const int32_t *idx, const int64_t *idx_stride, int32_t cap, const int32_t *kept, void *k_pages, void *v_pages,
                             int32_t *length_out, void *hip_stream);

/*
 * Whole pages, keys and values of all KV heads, from copy[i][0] to copy[i][1], i < n. Pairs with a number outside [0, n_pages), or twice the same, are
 * skipped (what ckv_pages_reserve leaves of its array). No page is written twice, or written and read, in one call.
 *   Of ckv_params n_kv_heads, head_dim and dtype are used, of ckv_pages not the table's fields. k_stride[1] = 0: pages of one head.
 *   copy        in   [n,2] int32
 */
ckv_status ckv_pages_copy(const ckv_params *params, const ckv_pages *pages, const int32_t *copy, int32_t n, void *k_pages, void *v_pages,
                          void *hip_stream);

/*
 * Which lists have which pages. Once for all pools that the lists describe (the layers of a model), beside the calls on each of them. An entry of a
 * list names a page, or none with a value outside [0, n_pages) (these calls write -1). refs[p] is how many entries name page p, and bit p % 32 of
 * taken[p / 32] whether any does: with lists without pages, all zeros. Both have to agree with the lists of all tables that
 * share them; then all results are the same in every run. They go from call to call in stream order.
 *   refs   in/out  [n_pages] int32         taken  in/out  [ceil(n_pages/32)] 32-bit words
 *   table          int32 entries at table_stride over (batch, KV head); table_stride[1] = 0: one list for the heads of a batch element
 * Numbers of rows are [batch,n_kv_heads] int32, and where heads have a list in common, it is long enough for the longest of them.
 */
typedef struct {
  int32_t batch;           /* >= 1                                                                  */
  int32_t n_kv_heads;      /* >= 1                                                                  */
  int32_t n_pages;         /* pages of the pools, >= 1                                              */
  int32_t page_rows;       /* as in ckv_pages                                                       */
  int32_t max_pages;       /* as in ckv_pages; batch * n_kv_heads * max_pages < 2^31                */
  int32_t reserved;        /* 0                                                                     */
  int64_t table_stride[2]; /* as in ckv_pages; no two lists overlap                                 */
} ckv_lists;

/*
 * Lists that become copies of others and share their pages (several answers to a prompt, beams): table_out[b] = table[parent[b]], or no pages with a
 * parent outside [0, batch). The pages of the former lists of table_out are released, those of the new ones counted; `table` stays as it is (its
 * own pages are released by ckv_pages_free, keep = NULL). A shared page that a list is to write into gets a copy by ckv_pages_reserve.
 *   table       in   int32, table_stride        table_out  in/out  int32, table_stride, not overlapping `table`
 *   parent      in   [batch] int32
 *   length      in   [batch,n_kv_heads] int32, or NULL with length_out
 *   length_out  out  length[parent[b]], or 0 without one; overlaps neither `length` nor `parent`
 */
ckv_status ckv_pages_fork(const ckv_lists *lists, const int32_t *table, const int32_t *parent, int32_t *table_out, int32_t *refs,
                          uint32_t *taken, const int32_t *length, int32_t *length_out, void *hip_stream);

/*
 * Makes rows [first, end) of every list such as can be written: entries of that range without a page get one, and entries whose page others name too get
 * one of their own, with a pair (former page, new page) in `copy` for ckv_pages_copy on each pool. Where all that share a page ask for it, the
 * last of them keeps it. New pages are the lowest-numbered free ones, in the order of the entries (batch, KV head, entry), pairs are in that order too.
 * All or nothing: where there are too few free pages or too few places for pairs, only copy (no pairs) and result are written.
 *   first, end  in   [batch,n_kv_heads] int32; nothing to do where end <= first, or behind max_pages * page_rows. Heads that have a list in common: one range,
 *                    from the least first to the greatest end of those with rows to come, whatever lies between. Where such heads are of very different lengths
 *                    (rows that retention kept by head), pages between their rows get copies too if lists share them; a list for every head avoids it
 *   copy        out  [n_copy,2] int32, pairs and behind them -1; n_copy >= 0 (copy may be NULL with 0). Never more pairs than shared pages in those ranges,
 *                    (end - 1) / page_rows - first / page_rows + 1 pages of a list at most
 *   result      out  [2] int32: pages (or places for pairs, if that is more) that are missing, 0 if all is done; pairs
 */
ckv_status ckv_pages_reserve(const ckv_lists *lists, int32_t *table, const int32_t *first, const int32_t *end, int32_t *refs, uint32_t *taken,
                             int32_t *copy, int32_t n_copy, int32_t *result, void *hip_stream);

/*
 * Pages behind the first keep[b,g] rows of every list leave it (all of them with keep NULL), and are free where no other entry names them.
 *   keep        in   [batch,n_kv_heads] int32, or NULL
 */
ckv_status ckv_pages_free(const ckv_lists *lists, int32_t *table, const int32_t *keep, int32_t *refs, uint32_t *taken, void *hip_stream);

/* Static text for a status code; never NULL. */
const char *ckv_status_string(ckv_status status);

#ifdef __cplusplus
}
#endif
#endif /* CKV_H_ */
