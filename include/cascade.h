/*
 * cascade.h -- C ABI of the B200 (sm_100a) tree-verification library for CASCADE
 * ("CASCADE: Context-Aware Relaxation for Speculative Image Decoding").
 *
 * One verification step of tree-based speculative image decoding: the target model looks at a draft
 * token tree in one pass (Section 3, "tree decoding"), and the relaxed acceptance rule of Section 4
 * (Eq. 1-3, Algorithm 2) decides which root-to-node path of draft tokens is kept.
 *
 * Conventions
 *   - Every function returns an int status: CASCADE_OK (0) or a negative CASCADE_ERR_* code.  Nothing
 *     throws or aborts.  All arguments are validated on the host before anything is launched, so a bad
 *     argument never reaches the device.
 *   - Pointers are DEVICE pointers unless the parameter is documented "host".  The caller owns every
 *     data buffer; the library owns only what cascade_create / cascade_tree_create return, until the
 *     matching destroy call.
 *   - Work is enqueued on the caller's stream (a cudaStream_t passed as void*; NULL = default stream)
 *     and is asynchronous: outputs are valid after the stream has been synchronised.
 *   - A context is bound to the device that was current at cascade_create and holds scratch memory
 *     that its calls share: calls on ONE context must not overlap on the GPU (use one stream, or one
 *     context per stream).
 *   - Tensors are dense, row-major, innermost index last.  "elem" is the context's dtype
 *     (float for CASCADE_F32, bf16 bit patterns for CASCADE_BF16).
 *   - Notation: B prompts; R = 2B rows of the classifier-free-guidance pair, cond rows 0..B-1 then
 *     uncond rows B..2B-1; T tree rows INCLUDING the root row 0 (the pending, last-emitted token whose
 *     key/value is not yet in the cache); P prefix (KV cache) length; h hidden size; Hq/Hkv query/kv
 *     heads; D head size; V image-token vocabulary.
 */
#ifndef CASCADE_H_
#define CASCADE_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------------------------------ */
#define CASCADE_OK 0
#define CASCADE_ERR_INVALID_ARG (-1)       /* null pointer, non-positive size, value out of range     */
#define CASCADE_ERR_BAD_TREE (-2)          /* parent[] is not a BFS-ordered tree with grouped siblings (from
                                              cascade_check: found by cascade_tree_update_device)        */
#define CASCADE_ERR_WORKSPACE (-3)         /* device allocation of the context's scratch failed        */
#define CASCADE_ERR_UNSUPPORTED_SHAPE (-4) /* shape outside what the kernels handle (see cascade_shape) */
#define CASCADE_ERR_CUDA (-5)              /* a CUDA runtime / driver call failed                      */
#define CASCADE_ERR_TIMEOUT (-6)           /* a bounded device-side wait gave up (see cascade_check)   */
#define CASCADE_ERR_OVERFLOW (-7)          /* cascade_kv_append, cascade_paged_tables: a cache or its page pool has
                                              no room (see cascade_check)                                */
#define CASCADE_ERR_BAD_PAGE (-8)          /* a paged call met a page, slot or length outside what it was given
                                              (found on the device, see cascade_check)                   */

/* ---- enums ------------------------------------------------------------------------------------- */
#define CASCADE_F32 0
#define CASCADE_BF16 1

/* cascade_params.flags */
#define CASCADE_USE_I 1u          /* Eq. 1: add the mass of interchangeable siblings                     */
#define CASCADE_USE_C 2u          /* Eq. 2: add the mass of convergent children                          */
#define CASCADE_CONV_DIST_SELF 4u /* Eq. 3 read literally: a child's mass is taken under the candidate's
                                     own row; default (flag clear) follows Algorithm 2, which reads it
                                     from the same distribution as the candidate's own probability       */

/* cascade_select_path mode */
#define CASCADE_SELECT_LONGEST 0      /* deepest node whose whole path is accepted, smallest index first */
#define CASCADE_SELECT_FIRST_ACCEPT 1 /* Algorithm 2's walk: first accepted child at every level         */

/* A score this close to its threshold is counted in near_count (decisions there are not stable under
 * rounding). */
#define CASCADE_NEAR 1e-3f

#define CASCADE_MAX_TREE_ROWS 256   /* T  <= 256                                            */
#define CASCADE_MAX_CHILDREN 32     /* children of one node <= 32                           */

typedef struct cascade_ctx cascade_ctx;
typedef struct cascade_tree cascade_tree;

/* Fixed sizes of a context.  Supported: D in {64,128}; Hq a multiple of Hkv; h a multiple of 64;
 * V a multiple of 8; T_max <= CASCADE_MAX_TREE_ROWS; B >= 1.  ffn may be 0 if no decoder layer is
 * run through cascade_verify_step (otherwise a multiple of 8). */
typedef struct {
  int32_t dtype; /* CASCADE_F32 or CASCADE_BF16: element type of q/k/v, hidden states and weights */
  int32_t B;
  int32_t T_max;
  int32_t P_max; /* largest prefix length any call will use                                      */
  int32_t h, Hq, Hkv, D, V;
  int32_t ffn;
} cascade_shape;

/* Relaxation parameters (Section 4.1: tau_pos gates Eq. 1, tau_seq gates Eq. 2; Eq. 3 / Algorithm 2:
 * tvd_budget is the total-variation budget of one verification step, 0.5 in the paper). */
typedef struct {
  float tau_pos;
  float tau_seq;
  float tvd_budget;
  uint32_t flags; /* CASCADE_USE_I | CASCADE_USE_C [| CASCADE_CONV_DIST_SELF] */
} cascade_params;

/* ---- life cycle -------------------------------------------------------------------------------- */

/* Create a context on the current device and allocate its scratch (split-KV partial results,
 * activation staging, softmax partials).  *out is set only on success. */
int cascade_create(cascade_ctx** out, const cascade_shape* shape);
int cascade_destroy(cascade_ctx* ctx);

/* Bytes of device scratch the context holds. */
int64_t cascade_workspace_bytes(const cascade_ctx* ctx);

/* Reads the context's device-side error word (set when a bounded wait inside a kernel ran out) after
 * synchronising `stream`.  Returns CASCADE_OK, CASCADE_ERR_TIMEOUT, CASCADE_ERR_BAD_TREE, CASCADE_ERR_BAD_PAGE,
 * CASCADE_ERR_OVERFLOW or CASCADE_ERR_CUDA, and clears the word. */
int cascade_check(cascade_ctx* ctx, void* stream);

/* Number of kernels the most recent call on this context enqueued. */
int cascade_last_launch_count(const cascade_ctx* ctx);

/* Failure detection.  Every wait inside a kernel (on an mbarrier, on another CTA's flag) gives up after a
 * limit, records it in the context's error word and leaves through the kernel's normal teardown, so a wait
 * that can never end costs the limit, not the device; cascade_check then returns CASCADE_ERR_TIMEOUT and the
 * context stays usable.  cascade_set_wait_limit changes the limit for later calls on this context
 * (nanoseconds, >= 1000; default 2 s).
 * cascade_wait_probe is a self-test of that path: it enqueues one small kernel whose only CTA waits on a
 * barrier nothing will ever arrive on (no copy in flight), with the context's limit.  waited_ns (DEVICE
 * uint32, may be NULL) receives how long the wait lasted.  After the stream has been synchronised,
 * cascade_check reports CASCADE_ERR_TIMEOUT. */
int cascade_set_wait_limit(cascade_ctx* ctx, int64_t limit_ns);
int cascade_wait_probe(cascade_ctx* ctx, uint32_t* waited_ns, void* stream);

const char* cascade_strerror(int status);

/* Per-kernel device timing (measurement aid, off by default).  While enabled, every kernel a call on
 * this context enqueues is bracketed by a pair of CUDA events on the caller's stream.
 * cascade_timing_read synchronises those events, ADDS the elapsed milliseconds and launch counts per
 * kernel id into ms_total / launches (HOST arrays of CASCADE_KERNEL_COUNT entries, caller-zeroed) and
 * forgets the recorded events.  cascade_kernel_name(id) names an id (NULL if out of range). */
#define CASCADE_KERNEL_COUNT 32
int cascade_timing_enable(cascade_ctx* ctx, int32_t on);
int cascade_timing_read(cascade_ctx* ctx, float* ms_total, int32_t* launches);
const char* cascade_kernel_name(int32_t id);

/* The draft tree (the static tree mask of Section 3; Algorithm 2 input `tree`).
 * parent: HOST array of T entries, parent[0] = -1, 0 <= parent[j] < j, rows in BFS order (depth never
 * decreases with the index) and the children of one parent contiguous.  Builds the device-side
 * descriptor: depth, packed ancestor-or-self bitmask (T x 4 uint64 words), child ranges, and the list
 * of (node, node) pairs whose cosine the acceptance rule reads (every parent->child edge, then every
 * unordered sibling pair).  Returns CASCADE_ERR_BAD_TREE if the ordering rules do not hold. */
int cascade_tree_create(cascade_ctx* ctx, int32_t T, const int32_t* parent, cascade_tree** out);
int cascade_tree_destroy(cascade_tree* tree);

/* A new draft tree in an existing descriptor (drafters that grow a different tree every step): same rules
 * and errors as cascade_tree_create, T <= the context's T_max.  Nothing is allocated; the descriptor is
 * rebuilt on the host and copied to the device on `stream` (the source is pageable host memory, so the copy
 * is staged before the call returns), and calls that use the tree must be enqueued after it on that stream.
 * An invalid tree returns its error and leaves the descriptor as it was.  Host-side queries
 * (cascade_tree_rows / depth / num_pairs / pairs) answer for the new tree as soon as the call returns. */
int cascade_tree_update(cascade_tree* tree, int32_t T, const int32_t* parent, void* stream);
/* The same, from a parent[] that is already in DEVICE memory, without a host round trip (drafters that decide
 * the tree's shape on the device each step: the dynamic trees that Section 2 contrasts with the static mask).
 * One small kernel on `stream` checks the rules of cascade_tree_create and writes the descriptor.  The host
 * cannot see the tree, so the caller states bounds that sizes depend on:
 *   T          rows (host value; grids and row counts of every later call come from it), <= T_max;
 *   depth_cap  the tree is at most this deep; path_nodes arrays of later calls have depth_cap + 1 entries per
 *              prompt and cascade_tree_depth returns it;
 *   pairs_cap  at most this many (node, node) pairs (edges + sibling pairs); scores arrays of later calls have
 *              pairs_cap entries per prompt and cascade_tree_num_pairs returns it; <= 0: the context's maximum.
 * A parent[] that breaks a rule or a bound is found on the device: cascade_check then returns
 * CASCADE_ERR_BAD_TREE, and the descriptor is left holding a neutral tree of T rows (every row a childless leaf
 * below the root, no pairs), so that calls already enqueued behind it stay within their buffers; their results
 * are meaningless.  Nothing is allocated; the host-side mirrors are not refreshed (cascade_tree_pairs and
 * cascade_tree_download fetch from the device with blocking copies). */
int cascade_tree_update_device(cascade_tree* tree, int32_t T, int32_t depth_cap, int32_t pairs_cap,
                               const int32_t* parent_dev, void* stream);
/* Copies the descriptor's device arrays to HOST arrays (blocking copies; synchronise the stream of a pending
 * update first): parent, depth, child_begin, child_count [T] int32 and the packed ancestor-or-self mask
 * anc [T][4] uint64 (bit i of row j set iff i is j or an ancestor of j).  Any pointer may be NULL. */
int cascade_tree_download(const cascade_tree* tree, int32_t* parent, int32_t* depth, int32_t* child_begin,
                          int32_t* child_count, uint64_t* anc);
int32_t cascade_tree_rows(const cascade_tree* tree);      /* T                                     */
int32_t cascade_tree_depth(const cascade_tree* tree);     /* deepest level                         */
int32_t cascade_tree_num_pairs(const cascade_tree* tree); /* edges + sibling pairs                 */
/* Copies the pair list to HOST arrays of cascade_tree_num_pairs entries (for inspecting scores). */
int cascade_tree_pairs(const cascade_tree* tree, int32_t* pair_a, int32_t* pair_b);

/* ---- (a) tree-masked attention ----------------------------------------------------------------- */
/* Section 3: all draft-tree rows are verified by the target "via a parallel forward pass".  For every
 * row r of the CFG pair, head and tree row j:
 *     out[r,j,head,:] = sum_i softmax_i(softmax_scale * <q[r,j,head,:], k_i>) v_i
 * over the keys row j may see: cache entries 0..prefix_len[r]-1 and the tree rows that are j itself or
 * one of its ancestors.  Query head `head` reads kv head head / (Hq / Hkv).
 *   q        [R,T,Hq,D] elem          k_tree, v_tree [R,T,Hkv,D] elem
 *   k_prefix, v_prefix [R,prefix_cap,Hkv,D] elem; rows at or beyond prefix_len[r] are never used
 *   prefix_len [R] int32, device; 0 <= prefix_len[r] <= min(prefix_cap, P_max)
 *   out      [R,T,Hq,D] elem
 * Softmax and accumulation are fp32.  Base addresses must be 16-byte aligned. */
int cascade_tree_attn(cascade_ctx* ctx, const cascade_tree* tree, const void* q, const void* k_prefix,
                      const void* v_prefix, int32_t prefix_cap, const int32_t* prefix_len,
                      const void* k_tree, const void* v_tree, void* out, float softmax_scale,
                      void* stream);

/* ---- (b) final norm + LM head + classifier-free guidance + vocabulary softmax statistics ------- */
/* Section 4.2 names the final projection, O(hV), as the dominant cost of verification; the guidance
 * scale is the experimental setting of App. D.2 (3.0, or 5.0 for Janus-Pro).  For prompt b, tree row j:
 *     n_x      = hidden_x * rsqrt(mean(hidden_x^2) + eps) * rms_gamma         x in {cond, uncond}
 *     logits   = (W n_u + cfg_scale * (W n_c - W n_u)) / temperature
 *     feat     = n_c                 (the target hidden state F of Section 4.1 that feeds the head)
 *     row_lse  = log sum_v exp(logits[v])
 *     cand_parent[b,j]  = logits[b, parent[j], tok[b,j]]              (0 for the root)
 *     cand_gparent[b,j] = logits[b, parent[parent[j]], tok[b,j]]      (0 where there is none)
 *   hidden [R,T,h] elem; rms_gamma [h] float; w_head [V,h] elem; tok [B,T] int32 in [0,V)
 *   logits_out [B,T,V] float or NULL; feat_out [B,T,h] float; feat_norm_out [B,T] float (||feat||_2);
 *   row_lse_out [B,T] float; cand_parent_out, cand_gparent_out [B,T] float (both NULL if tok is NULL).
 * The guidance mix is applied to the normalised hidden states before the product (the head is
 * linear), and that operand is carried as a bf16 high part plus a bf16 remainder so the result keeps
 * fp32-level accuracy.  temperature > 0. */
int cascade_lm_head_cfg(cascade_ctx* ctx, const cascade_tree* tree, const void* hidden,
                        const float* rms_gamma, float eps, const void* w_head, float cfg_scale,
                        float temperature, const int32_t* tok, float* logits_out, float* feat_out,
                        float* feat_norm_out, float* row_lse_out, float* cand_parent_out,
                        float* cand_gparent_out, void* stream);

/* ---- (c) relaxed acceptance -------------------------------------------------------------------- */
/* Cosines of Section 4.1 for the tree's pair list: scores_out[b,i] = cos(feat[b,pair_a[i]],
 * feat[b,pair_b[i]]).  feat [B,T,feat_dim] float; feat_norm [B,T] float or NULL (then computed here).
 * Passing logits as feat (feat_dim = V) gives the logit-space variant of App. B. */
int cascade_similarity(cascade_ctx* ctx, const cascade_tree* tree, const float* feat, int32_t feat_dim,
                       const float* feat_norm, float* scores_out, void* stream);

/* Eq. 1-3 and Algorithm 2 for every draft node at once.  For node j >= 1 with parent pi,
 * g = softmax(logits[b,pi,:]):
 *     q_j  = g[tok_j]
 *     I_j  = siblings s of j with cos(F_j,F_s) >= tau_pos ; C_j = children c of j with cos >= tau_seq
 *     mI_j = mass under g of the distinct tokens of I_j other than tok_j
 *     mC_j = mass (under g, or under softmax(logits[b,j,:]) with CASCADE_CONV_DIST_SELF) of the distinct
 *            tokens of C_j not equal to tok_j and not already in mI_j
 *     running total t: the first child of pi starts from tvd_out[pi], a later sibling from the previous
 *     sibling's tvd_out (what Algorithm 2's curr_TVD holds when its walk arrives at j);
 *     each set is added whole, I first, only if non-empty and t + mass <= tvd_budget;
 *     accept[j] = uniforms[j] < min(1, q_relaxed[j] / draft_p[j]);  draft_p <= 0 rejects; accept[0] = 1.
 * Inputs: scores [B,num_pairs] float from cascade_similarity; row_lse, cand_parent, cand_gparent [B,T]
 * float as produced by cascade_lm_head_cfg -- or pass logits [B,T,V] float (then those three may be
 * NULL and are derived from logits); tok [B,T] int32; draft_p [B,T] float (the drafter's probability of
 * tok[j] under its parent's context: Algorithm 2 input D); uniforms [B,T] float in [0,1) (Algorithm 2's
 * random(), made an input so results are reproducible).
 * Outputs: accept [B,T] uint8; q_relaxed, tvd_out [B,T] float; near_count [B] int32 = number of nodes
 * with a cosine, a budget comparison or the accept test within CASCADE_NEAR of its threshold (any of
 * the last three may be NULL). */
int cascade_relaxed_accept(cascade_ctx* ctx, const cascade_tree* tree, const float* scores,
                           const float* logits, const float* row_lse, const float* cand_parent,
                           const float* cand_gparent, const int32_t* tok, const float* draft_p,
                           const float* uniforms, const cascade_params* params, uint8_t* accept,
                           float* q_relaxed, float* tvd_out, int32_t* near_count, void* stream);

/* ---- (d) path selection ------------------------------------------------------------------------ */
/* Algorithm 2 keeps, level by level, the first accepted candidate (CASCADE_SELECT_FIRST_ACCEPT);
 * CASCADE_SELECT_LONGEST returns the deepest node all of whose ancestors are accepted.
 *   accept [B,T] uint8; tvd_out [B,T] float or NULL
 *   path_nodes [B, depth+1] int32: root..end node, unused entries -1  (depth = cascade_tree_depth)
 *   path_len [B] int32: number of accepted draft tokens (alpha of Algorithm 2)
 *   tvd_used [B] float or NULL: the running total where the walk stops (needs tvd_out). */
int cascade_select_path(cascade_ctx* ctx, const cascade_tree* tree, const uint8_t* accept,
                        const float* tvd_out, int32_t mode, int32_t* path_nodes, int32_t* path_len,
                        float* tvd_used, void* stream);

/* ---- the whole step ---------------------------------------------------------------------------- */

/* One pre-norm decoder layer (the workload's architecture; the paper treats the target as given):
 * a = RMSNorm(x, gamma_attn); q,k,v = a Wq^T, a Wk^T, a Wv^T; rotary (half-split pairing) at position
 * prefix_len[r] + depth[j]; tree attention; x += attn Wo^T; m = RMSNorm(x, gamma_mlp);
 * x += (silu(m Wg^T) * (m Wu^T)) Wd^T.  Matrices are [out_features, in_features] elem.  wq, wk, wv must be
 * stacked in memory in this order (wk = wq + Hq*D*h elements, wv = wk + Hkv*D*h), and so must w_gate, w_up
 * (w_up = w_gate + ffn*h): each group runs as one projection; CASCADE_ERR_UNSUPPORTED_SHAPE otherwise.
 * The bf16 path needs D = 128. */
typedef struct {
  const float* gamma_attn; /* [h] */
  const void* wq;          /* [Hq*D, h]  */
  const void* wk;          /* [Hkv*D, h] */
  const void* wv;          /* [Hkv*D, h] */
  const void* wo;          /* [h, Hq*D]  */
  const float* gamma_mlp;  /* [h] */
  const void* w_gate;      /* [ffn, h] */
  const void* w_up;        /* [ffn, h] */
  const void* w_down;      /* [h, ffn] */
  void* k_prefix;          /* [R, prefix_cap, Hkv, D] this layer's cache: read by cascade_verify_step, */
  void* v_prefix;          /* written (rows at and beyond prefix_len) by cascade_kv_append              */
} cascade_layer;

/* All arguments of one verification step.  Pointers are device pointers except `layers`, a HOST
 * array of n_layers structs (whose members are device pointers). */
typedef struct {
  /* model */
  int32_t n_layers;            /* >= 0.  0: skip the decoder layers, `hidden_in` is the head's input */
  const cascade_layer* layers; /* host array */
  const void* embed;           /* [V,h] elem, token embedding (n_layers > 0)                         */
  const float* gamma_final;    /* [h]                                                                */
  const void* w_head;          /* [V,h] elem                                                         */
  int32_t prefix_cap;
  const int32_t* prefix_len;   /* [R]                                                                */
  float eps, rope_base, softmax_scale, cfg_scale, temperature;
  /* step inputs */
  const int32_t* tok;          /* [B,T] */
  const float* draft_p;        /* [B,T] */
  const float* uniforms;       /* [B,T] */
  const void* hidden_in;       /* [R,T,h] elem, used when n_layers == 0                              */
  /* stand-alone attention inputs, used when n_layers == 0 and q != NULL: piece (a) runs on them in
   * the same enqueue and writes attn_out */
  const void* q;               /* [R,T,Hq,D]  */
  const void* k_tree;          /* [R,T,Hkv,D] */
  const void* v_tree;
  const void* k_prefix;        /* [R,prefix_cap,Hkv,D] */
  const void* v_prefix;
  void* attn_out;              /* [R,T,Hq,D] elem */
  /* rule */
  cascade_params params;
  int32_t select_mode;
  /* outputs */
  uint8_t* accept;             /* [B,T] */
  int32_t* path_nodes;         /* [B,depth+1] */
  int32_t* path_len;           /* [B] */
  float* q_relaxed;            /* [B,T] or NULL */
  float* tvd_out;              /* [B,T] or NULL */
  float* tvd_used;             /* [B] or NULL */
  int32_t* near_count;         /* [B] or NULL */
  /* optional intermediates, NULL to skip the store */
  float* logits;               /* [B,T,V] */
  float* feat;                 /* [B,T,h] */
  float* scores;               /* [B,num_pairs] */
  float* row_lse;              /* [B,T] */
  float* hidden_out;           /* [R,T,h] float: residual stream entering the final norm (n_layers>0) */
  void* k_tree_out;            /* [n_layers,R,T,Hkv,D] elem: rotated keys / values of the tree rows, */
  void* v_tree_out;            /*   what a caller appends to the cache for the accepted path          */
  /* truncation of the target distribution before the rule (see cascade_filter_logits; Appendix D.1):
   * top_k > 0 and/or 0 < top_p < 1 switch it on, which needs `logits` (they are truncated in place and the
   * row statistics are taken from them); zero in both fields (a zeroed struct): off */
  int32_t top_k;
  float top_p;
} cascade_step;

/* Runs pieces (a)-(d) (and the decoder layers, if any) as one enqueue on `stream`. */
int cascade_verify_step(cascade_ctx* ctx, const cascade_tree* tree, const cascade_step* step, void* stream);

/* Same step with the per-step inputs and results in HOST memory (pageable or pinned): tok, draft_p, uniforms
 * [B,T] are gathered into the context's pinned block and copied to the device in one transfer, accept [B,T],
 * path_nodes [B,depth+1] and path_len [B] come back in one transfer, and the call returns after the stream
 * has been synchronised, the results in the caller's arrays.  The corresponding pointers inside `step` are
 * ignored (the context's own staging buffers are used); everything else in `step` is read as in
 * cascade_verify_step.  Like all calls on one context, these must not overlap.  When the same call (same
 * step contents, tree and stream) is repeated on a stream that can be recorded (not the legacy default
 * stream), the library records its copies and launches as a CUDA graph at the second call and replays it
 * afterwards; results are the same either way. */
int cascade_verify_step_host(cascade_ctx* ctx, const cascade_tree* tree, const cascade_step* step,
                             const int32_t* tok_host, const float* draft_p_host, const float* uniforms_host,
                             uint8_t* accept_host, int32_t* path_nodes_host, int32_t* path_len_host,
                             void* stream);

/* ---- between two steps of a decode loop --------------------------------------------------------- */
/* The token after the accepted path: Algorithm 1's last step, which Algorithm 2 leaves out.  For prompt b,
 * end = last node of its path, q = softmax(logits[b, end, :]).  Two rules:
 *   draft_row != NULL (the drafter's full distribution p at the end node, [B,V] float, row b for prompt b):
 *     Algorithm 1's correction step -- if a child of end was rejected, the token is drawn from [q - p]+
 *     normalised; after a fully accepted draft (end has no children), from q.  Should nothing of q lie above p
 *     (p = q), q is used.  mass_out[b] = sum of [q - p]+ (1 where q was used).
 *   draft_row == NULL (a tree drafter that keeps only the probabilities of its proposals): the tokens of end's
 *     children (all rejected, whichever selection mode chose the path) get probability zero, the rest of q is
 *     renormalised.  mass_out[b] = the probability mass that remains.
 * token_out[b] is the inverse-CDF sample at u_bonus[b]: the first v whose cumulative weight exceeds
 * u_bonus[b] * (total weight).
 *   logits [B,T,V] float (as stored by cascade_lm_head_cfg / cascade_verify_step); tok [B,T] int32;
 *   path_nodes [B,depth+1], path_len [B] from cascade_select_path; u_bonus [B] float in [0,1);
 *   token_out [B] int32; mass_out [B] float or NULL. */
int cascade_bonus_token(cascade_ctx* ctx, const cascade_tree* tree, const float* logits, const int32_t* tok,
                        const float* draft_row, const int32_t* path_nodes, const int32_t* path_len,
                        const float* u_bonus, int32_t* token_out, float* mass_out, void* stream);

/* Appends the keys / values of the accepted path's tree rows (root row first: the pending token, then the
 * accepted drafts) to the caches of n_layers layers, for both CFG rows of every prompt, at positions
 * prefix_len[r] .. prefix_len[r] + path_len[b], and adds path_len[b] + 1 to prefix_len[r] (device array,
 * updated in place).  The tree rows were rotated at exactly these positions by cascade_verify_step.
 *   layers: HOST array of n_layers structs; only k_prefix / v_prefix are used, and those caches
 *           ([R, prefix_cap, Hkv, D] elem) are written here.
 *   k_tree, v_tree [n_layers,R,T,Hkv,D] elem: cascade_step.k_tree_out / v_tree_out of the step.
 * A path that does not fit into prefix_cap is not appended and raises CASCADE_ERR_OVERFLOW at the next
 * cascade_check.  n_layers <= 64. */
int cascade_kv_append(cascade_ctx* ctx, const cascade_tree* tree, int32_t n_layers, const cascade_layer* layers,
                      const void* k_tree, const void* v_tree, const int32_t* path_nodes, const int32_t* path_len,
                      int32_t prefix_cap, int32_t* prefix_len, void* stream);

/* ---- truncation of the target distribution ------------------------------------------------------- */
/* Top-k / nucleus truncation of target logits, in place (the sampling settings of the paper's experiments,
 * Appendix D.1: temperature 1, top-p 1.0, top-k 2000; the paper states the numbers, the truncations are
 * the usual ones).  Per row of V logits:
 *   top_k (0 < top_k < V; 0 or >= V: off): keep the tokens whose logit is >= the top_k-th largest logit of the
 *     row -- tokens tied with it stay together, so more than top_k can remain;
 *   top_p (< 1; 1: off), on the distribution renormalised over what top-k kept: keep a token iff the
 *     probability of the tokens with a strictly larger logit is < top_p (ties stay together).
 * A dropped token's logit becomes -inf: cascade_relaxed_accept (with these logits), cascade_bonus_token and
 * any softmax over the row then give it probability zero and renormalise the rest.
 *   logits [n_rows, V] float, DEVICE, read and written (V from the context's shape; rows are independent,
 *          e.g. the [B,T,V] logits of cascade_lm_head_cfg with n_rows = B*T);
 *   kept_count [n_rows] int32 DEVICE or NULL: how many tokens of each row remain.
 * Both thresholds are exact (a radix descent over the logits' bit patterns; the nucleus sums probabilities
 * in 40-bit fixed point, so the result does not depend on the order of the additions).
 * Errors: CASCADE_ERR_INVALID_ARG (null pointers, n_rows < 1, top_k < 0, top_p outside (0, 1]). */
int cascade_filter_logits(cascade_ctx* ctx, float* logits, int32_t n_rows, int32_t top_k, float top_p,
                          int32_t* kept_count, void* stream);

/* ---- prompts: a paged KV cache ------------------------------------------------------------------- */
/* A verification step reads a prefix cache; these calls fill one and read it while a prompt is taken in, chunk by
 * chunk and for many requests of different lengths at once (the paper treats the prompt's pass as given).  The cache
 * is a pool of pages; a request's token at position x lives in page block_table[r][x / page_size] at row
 * x % page_size.  The dense prefix cache of cascade_verify_step ([R,prefix_cap,Hkv,D]) is the special case
 * n_pages = R * prefix_cap / page_size, block_table[r][i] = r * (prefix_cap / page_size) + i: prompts written through
 * these calls into such a pool can be verified against without a copy.  The verification step itself reads that layout only:
 * behind any other block table a prefix has to be copied into a dense cache first.
 *   k_pages, v_pages [n_pages,page_size,Hkv,D] elem, page p starting page_stride elements after page p - 1
 *              (page_stride >= page_size*Hkv*D; larger where keys and values of a page lie side by side in one pool);
 *              16-byte aligned, page_stride a multiple of 16 bytes
 *   page_size  a multiple of 8; n_pages * page_size < 2^31
 *   block_table [n_req,table_width] int32, DEVICE, rows table_stride entries apart.  Entries behind a request's last page
 *              are never used, nor is anything between two rows
 *   table_width at most table_stride; 0: table_stride
 * Device-resident lengths, pages and slots cannot be checked on the host.  A kernel that meets one outside its range
 * leaves it out, touches nothing outside the buffers it was given, and cascade_check returns CASCADE_ERR_BAD_PAGE.
 * Arrays of 32-bit numbers start on 4-byte boundaries (CASCADE_ERR_INVALID_ARG).
 * All four calls allocate nothing, take their sizes from host arguments alone and can be recorded into a CUDA graph.
 * The context must have been created on the current device (CASCADE_ERR_INVALID_ARG otherwise). */
typedef struct {
  void* k_pages;
  void* v_pages;
  int64_t page_stride;
  int32_t n_pages, page_size;
  const int32_t* block_table;
  int32_t table_stride, table_width;
} cascade_paged_cache;

/* Block tables and slot map of the next pass, from the requests' lengths, in one kernel.
 *   new_len [n_req]: how many tokens request r appends; negative: the request is finished and gives its pages back.
 *   kv_len [n_req]: tokens it holds.  free_pages [n_pages], free_count [1]: a stack of free page ids, its top at
 *   free_pages[free_count - 1].
 * First the pages of finished requests are pushed, in request order and each table's order; then the pages that the
 * others need (ceil((kv_len + new_len) / page_size) - ceil(kv_len / page_size) each) are popped one by one in the same
 * order and written behind the pages each has.  Outputs:
 *   block_table (updated in place: only entries behind a request's old pages are written), free_pages (pushed entries),
 *   free_count_out [1], kv_len_out [n_req] (kv_len + new_len, 0 if finished) -- may be the same arrays as free_count and
 *   kv_len; apart from that no two arguments may overlap;
 *   q_begin [n_req+1]: request r's new tokens are rows q_begin[r] .. q_begin[r+1]-1 of the pass;
 *   slot, pos [n_tok]: page * page_size + row, and the position in the request, of every new token; -1 in the rows
 *   behind the last one (n_tok is the padded row count of the pass).
 * A negative kv_len, lengths that pass the table's width or n_tok, a pool that runs out or over: nothing is taken or
 * given back -- kv_len_out and free_count_out repeat the inputs, q_begin is all 0, slot and pos all -1, so that what is
 * enqueued behind does nothing -- and cascade_check returns CASCADE_ERR_OVERFLOW.  A token whose page id is outside
 * the pool gets slot -1 (CASCADE_ERR_BAD_PAGE); one that a finished request gives back is pushed as it is, so that the
 * stack's count holds, and reported the same way.
 * 1 <= n_req <= CASCADE_MAX_REQUESTS; n_tok >= 0.  All arrays int32, DEVICE. */
#define CASCADE_MAX_REQUESTS 4096
int cascade_paged_tables(cascade_ctx* ctx, int32_t n_req, int32_t n_tok, int32_t page_size, int32_t n_pages,
                         const int32_t* new_len, const int32_t* kv_len, int32_t* block_table, int32_t table_stride,
                         int32_t* free_pages, const int32_t* free_count, int32_t* kv_len_out, int32_t* free_count_out,
                         int32_t* q_begin, int32_t* slot, int32_t* pos, void* stream);

/* Writes the keys and values of a pass into their slots, rotary embedding included (half-split pairing: element i
 * turns with element i + D/2 by pos * rope_base^(-2i/D), as cascade_verify_step rotates tree rows).
 *   k, v [n_tok,Hkv,D] elem, rows k_stride / v_stride elements apart (>= Hkv*D: parts of a stacked projection);
 *   q [n_tok,Hq,D] rows q_stride apart -> q_out rows q_out_stride apart, rotated; q_out may be q (same stride).
 *   q = q_out = NULL: keys and values only.  rope_base = 0: no rotation (then q has to be NULL).
 *   slot, pos [n_tok] int32 from cascade_paged_tables; a row with slot -1 is left out (its q_out row too).  No two rows
 *   may name the same slot.  pos >= 0 for the others.  n_tok >= 1.  But for q_out = q no output overlaps an input.
 * block_table is not used.  All bases 16-byte aligned, strides multiples of 16 bytes. */
int cascade_paged_append(cascade_ctx* ctx, const cascade_paged_cache* cache, int32_t n_tok, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* slot,
                         const int32_t* pos, float rope_base, void* q_out, int64_t q_out_stride, void* stream);

/* Attention of the new tokens of every request over its pages.  Row i of request r (q row q_begin[r] + i) stands at
 * position x = kv_len[r] - (q_begin[r+1] - q_begin[r]) + i, the keys of the pass being in the cache already, and sees key
 * j iff j <= x and (window == 0 or j > x - window or j < sinks):
 *     out[row,head,:] = sum_j softmax_j(softmax_scale * <q[row,head,:], k_j>) v_j ;   lse[row,head] = log sum_j exp(...)
 * Query head `head` reads kv head head / (Hq / Hkv).  A row that sees no key (kv_len smaller than its new tokens) gets
 * zeros and lse -inf, one all of whose scores are -inf NaN.  What lies at keys a row does not see, NaN and infinities
 * included, does not reach it.
 * Keys of a page outside the pool count as not seen (CASCADE_ERR_BAD_PAGE): rows that would have seen one, and rows beside
 * them, are summed again key by key, which takes long.
 *   q [n_tok,Hq,D] elem, rows q_stride apart; out [n_tok,Hq,D] elem, dense, no part of q (CASCADE_ERR_INVALID_ARG);
 *   lse [n_tok,Hq] float or NULL
 *   q_begin [n_req+1], kv_len [n_req] int32, DEVICE: as cascade_paged_tables leaves them.  Rows of q behind
 *   q_begin[n_req] (all n_tok rows are memory) reach no result, the same rows of out and lse are not written.  n_tok >= 1.
 *   max_q, max_kv: no request has more new tokens / keys than this (host bounds that launch sizes come from; a
 *   request beyond them is left out, CASCADE_ERR_BAD_PAGE).  1 <= n_req <= CASCADE_MAX_REQUESTS.
 *   Hq / Hkv <= 128, max_kv <= 2^31 - 65536 (CASCADE_ERR_UNSUPPORTED_SHAPE).
 *   window >= 0 (0: none), sinks >= 0.
 * Scores, statistics, sums and accumulators are fp32.  bf16: the weights are rounded to bf16 for their product with the values.
 * fp32: every operand of a product counts with about 22 bits (two 19-bit parts).  A row whose result is not finite, or (bf16,
 * more than 16 rows a key head) whose scores climb by more than 66 from one 64 keys to the next, is summed again key by key,
 * 0.6 us a key. */
int cascade_paged_attn(cascade_ctx* ctx, const cascade_paged_cache* cache, int32_t n_req, int32_t n_tok, const void* q,
                       int64_t q_stride, const int32_t* q_begin, const int32_t* kv_len, int32_t max_q, int32_t max_kv,
                       int32_t window, int32_t sinks, float softmax_scale, void* out, float* lse, void* stream);

/* ---- one token a row ------------------------------------------------------------------------------- */
/* Draws a token from every row of logits (a drafter's proposals, or plain decoding), with the truncations of
 * cascade_filter_logits and the min-p rule applied on the fly; the logits are only read.  With m the row's largest
 * logit and w[v] = exp((logits[v] - m) / temperature):
 *   top_k (0 < k < V): keep logits >= the k-th largest (ties stay);
 *   top_p (< 1): of those keep a token iff the mass of the tokens with a strictly larger logit is < top_p of the mass of
 *     what top_k kept (the largest always stays);
 *   min_p (> 0): of those keep w[v] >= min_p;
 *   token = the first v whose cumulative kept weight exceeds uniforms[row] * (total kept weight);
 *   prob  = w[token] / (total kept weight) -- what Algorithm 2 wants as draft_p;   kept = how many tokens remained.
 * temperature <= 0: the largest logit, lowest index first, prob 1, kept 1.  A logit of -inf or NaN is never kept; one of
 * +inf weighs 1 against 0 for every finite one.  A row without any logit to keep: token -1, prob 0, kept 0.
 *   logits [n_rows,V] float (logits_dtype CASCADE_F32) or bf16 (CASCADE_BF16), rows row_stride elements apart, V from the
 *   context; aligned to its element.  uniforms [n_rows] float in [0,1) (larger counts as the largest float below 1,
 *   negative and NaN as 0).
 *   temperature, top_p, min_p [n_rows] float, top_k [n_rows] int32, DEVICE, or NULL: 1 / off / off / off for all rows.
 *     Per row, off is top_k <= 0 or >= V, top_p >= 1 or NaN, min_p <= 0 or NaN; a NaN temperature counts as 0, +inf
 *     weighs all finite logits alike; min_p above 1 counts as 1.
 *   token_out [n_rows] int32; prob_out [n_rows] float or NULL; kept_out [n_rows] int32 or NULL.  They overlap neither each
 *   other nor an input (CASCADE_ERR_INVALID_ARG where two arrays are the same).
 * Weights are formed in 64 bits and summed in fixed point, so the draw does not depend on the order of additions.  With W the
 * power of two from V up, sums are within V * max(W / 2^63, 2^-51) + 1e-10 of exact ones (in units of the largest weight):
 * 6e-10 for V = 65536, 1.2e-7 for 2^20; a uniform or top_p closer than that to a boundary may fall on its other side. */
int cascade_sample(cascade_ctx* ctx, const void* logits, int32_t logits_dtype, int64_t row_stride, int32_t n_rows,
                   const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                   const float* uniforms, int32_t* token_out, float* prob_out, int32_t* kept_out, void* stream);

/* ---- the drafter's training loss (outside the verification step) ---------------------------------- */
/* Section 4.3, Eq. 4: the soft cross-entropy between the target distribution and the drafter's at every position k
 * of a target-generated sequence, weighted by c (2 in the paper's experiments, Appendix D.1) where the target's
 * hidden states of positions k and k+1 satisfy the convergence criterion of Eq. 2 (cosine >= tau_seq), by 1 elsewhere
 * and at the last position:
 *     loss_out[k] = - w_k * sum_v softmax(target_logits[k])[v] * log softmax(draft_logits[k])[v]
 *   target_logits, draft_logits [K,V] float; feat [K,h] float (target hidden states); DEVICE pointers.
 *   loss_out [K] float; weight_out [K] float or NULL (w_k); total_out [1] float or NULL (sum of loss_out, added in
 *   index order).  No context is needed and nothing is allocated; two kernels on `stream`.
 * Only the forward value is computed (the gradient with respect to draft_logits[k] is w_k (p_k - q_k), which a
 * training framework forms from its own softmax).  Errors: CASCADE_ERR_INVALID_ARG (null pointers, sizes < 1,
 * c <= 0, NaN threshold). */
int cascade_drafter_loss(const float* target_logits, const float* draft_logits, const float* feat, int32_t K, int32_t V,
                         int32_t h, float tau_seq, float c, float* loss_out, float* weight_out, float* total_out,
                         void* stream);

/* ---- acceptance without any device allocation --------------------------------------------------- */
/* The paper has no counterpart to this entry point; it exists for deployment.  Some callers of this
 * library may not allocate device memory at all: a plug-in running inside a serving process that
 * handed its whole memory budget to one arena at start-up, code that runs after the host has frozen
 * allocation (for instance to keep addresses stable), or a process whose allocator hooks forbid
 * cudaMalloc.  cascade_create and cascade_tree_create call cudaMalloc, so such callers cannot use the
 * entry points above.  This one needs neither object: similarity scores (Section 4.1), relaxed acceptance
 * (Eq. 1-3, Algorithm 2) and path selection, as cascade_similarity + cascade_relaxed_accept +
 * cascade_select_path compute them, with all device-side scratch (the tree descriptor, the cosine
 * scores, the per-prompt finished-CTA counters) in one static device array of the library
 * (about 0.7 MB, held by every GPU that loads the library until the process exits).
 *   B <= CASCADE_STATIC_MAX_PROMPTS, T <= CASCADE_MAX_TREE_ROWS; larger sizes return
 *   CASCADE_ERR_UNSUPPORTED_SHAPE and nothing is launched.
 *   parent [T]: HOST array, same rules as cascade_tree_create.  Everything else: device pointers with the
 *   meaning they have in cascade_similarity / cascade_relaxed_accept / cascade_select_path
 *   (feat [B,T,feat_dim] float, 16-byte aligned; feat_norm [B,T] or NULL; row_lse, cand_parent,
 *   cand_gparent [B,T]; tok, draft_p, uniforms [B,T]; outputs accept [B,T], path_nodes [B,depth+1],
 *   path_len [B]; q_relaxed, tvd_out, near_count, tvd_used may be NULL).
 * The call allocates nothing on the device: it copies the tree descriptor into the static array (from
 * temporary host memory that is gone when the call returns), clears the counters and enqueues one kernel on
 * `stream`.  A stream that is being captured is refused (CASCADE_ERR_INVALID_ARG, nothing is enqueued): the
 * copies read host memory of this call only.  The first call on a device also looks up the device address of
 * the array (cudaGetSymbolAddress).
 * All calls on a device share the one array and it keeps the last call's contents: two calls whose
 * work overlaps on the GPU (different streams) race; serialise them. */
#define CASCADE_STATIC_MAX_PROMPTS 32
int cascade_accept_static(int32_t B, int32_t T, const int32_t* parent, const float* feat, int32_t feat_dim,
                          const float* feat_norm, const float* row_lse, const float* cand_parent,
                          const float* cand_gparent, const int32_t* tok, const float* draft_p,
                          const float* uniforms, const cascade_params* params, int32_t select_mode,
                          uint8_t* accept, float* q_relaxed, float* tvd_out, int32_t* near_count,
                          int32_t* path_nodes, int32_t* path_len, float* tvd_used, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CASCADE_H_ */
