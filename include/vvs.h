/*
 * vvs.h - C ABI of the MI355X (gfx950) target-model verification pass for speculative decoding of
 * visual autoregressive models.
 *
 * One call of vvs_verify is one "target forward pass" in the sense of the paper's tokens-per-forward
 * metric (Section 5, "Metrics"): a KV-cached decoder-only transformer scores the pending token and N
 * drafted VQ tokens (a chain, or a tree under an ancestor mask: Section 3, "Verification
 * Redundancy") for B prompts, each as a conditional / unconditional row pair, mixes the two logit
 * rows, applies softmax, and runs the accept / resample rule of Section 2 ("Speculative Decoding").
 * vvs_kv_commit then keeps the K/V of the accepted path (Section 4.1: restoring the KV entries
 * re-establishes exact AR conditioning).
 *
 * Notation: p = target distribution, q = draft distribution (the paper prints the two letters the
 * other way round; the rule is the same: accept with probability min(1, target/draft)).
 * B prompts; R = 2B rows, row 2b conditional, row 2b+1 unconditional; N draft nodes numbered 1..N,
 * node 0 = root = the pending token (emitted, K/V not cached yet); T = N + 1; V_eff = logit_hi -
 * logit_lo; S_b = cached length of prompt b.
 *
 * Ownership: the caller allocates every device buffer (KV cache, workspace, packed weights, inputs,
 * outputs), sized by vvs_query_sizes; the library never allocates or frees device memory and never
 * synchronises the stream, except vvs_create (synchronous: it zero-fills the KV cache and uploads
 * small tables).  Pointers named d_* are DEVICE pointers, h_* are HOST pointers.  Device buffers
 * must stay valid until the work queued on the stream has finished.  Calls on one context must be
 * issued on one stream (or be ordered by the caller).
 *
 * Errors: every function returns a vvs_status; nothing is launched when the status is not VVS_OK
 * (arguments and call order are checked on the host first).  vvs_last_error gives the message.
 *
 * A forward of few rows runs all layers in one launch, whose workgroups wait for each other's results.  Should such a wait not
 * end (after some 2 million looks, 1 to 2 s; nothing in the library's own work leads there), the launch ends without its
 * results, and the call behind it says so in its outputs, since its status has been returned long before:
 *   vvs_verify, vvs_verify_post: accept_len, next_token and the whole path of every prompt are -1 (of a prompt whose image is
 *     complete: as ever); vvs_kv_commit then changes nothing, so that the call can be made again;
 *   vvs_prefill: d_first_token is -1 and every prompt counts as complete (vvs_read_state: n_emitted = G, pending token -1);
 *   vvs_draft: all distributions of the levels from there on are NaN, the tokens (unless given) the first ids of the slice.
 */
#ifndef VVS_H
#define VVS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct vvs_ctx vvs_ctx;        /* opaque host object; owns no device memory */
typedef void* vvs_stream;              /* a hipStream_t (NULL = the default stream) */

typedef enum {
  VVS_OK = 0,
  VVS_EINVAL = -1,   /* bad argument (NULL pointer, malformed tree, value out of range) */
  VVS_ESTATE = -2,   /* call order: verify before prefill, commit without verify, ... */
  VVS_ESIZE = -3,    /* shape not supported / exceeds the sizes the context was created for */
  VVS_EHIP = -4      /* a HIP call failed */
} vvs_status;

enum { VVS_FP32 = 0, VVS_BF16 = 1 };               /* vvs_config.dtype */
enum { VVS_PREFIX_CLASS = 0, VVS_PREFIX_DENSE = 1 }; /* vvs_config.prefix_kind */
enum { VVS_STRICT = 0, VVS_RELAXED = 1 };           /* acceptance mode */
#define VVS_MAX_T 64                                 /* max query tokens per row in one verify call */

typedef struct {
  int32_t n_layers, d_model, n_heads, d_ff;
  int32_t vocab;                 /* rows of the token embedding table */
  int32_t logit_lo, logit_hi;    /* allowed id slice [lo, hi): only these ids get logits */
  int32_t grid_h, grid_w;        /* image token grid; G = grid_h * grid_w tokens per image */
  int32_t prefix_len;            /* P condition tokens in front of the image tokens */
  int32_t prefix_kind;           /* VVS_PREFIX_CLASS: ids into a class table whose last row (id
                                    n_classes) is the null class; VVS_PREFIX_DENSE: [P, d] vectors */
  int32_t n_classes;
  int32_t n_prompts;             /* B */
  int32_t max_nodes;             /* largest N of any verify call, <= VVS_MAX_T - 1 */
  int32_t dtype;                 /* VVS_FP32: fp32 weights, activations and KV cache;
                                    VVS_BF16: bf16 weights, GEMM/attention operands and KV cache,
                                    fp32 accumulation, fp32 residual stream and logits */
  float cfg_scale;               /* s in l_u + s (l_c - l_u) */
  float rms_eps;
  float rope_base;
  int32_t relax_k;               /* neighbours per id in the table given to vvs_set_neighbors */
  float relax_delta;             /* budget of target mass the relaxed rule may absorb */
  int32_t feature_slots;         /* token-level feature cache (Section 4.3): features kept per row,
                                    0 .. VVS_MAX_FEATURE_SLOTS (0 = none; the paper keeps 5) */
  int32_t feature_pre_norm;      /* 0: a feature is the input of the output head (after the final
                                    norm); 1: the residual stream in front of the final norm */
  int32_t draft_input;           /* 0: a target model (token embeddings are the inputs);
                                    1: a drafter context for vvs_draft: the input of a token is
                                    W_fc [embedding ; feature], and the weight list ends with one
                                    more tensor fc [2 d, d] */
  int32_t norm_mode;             /* bf16 contexts, where the output of an RMSNorm is rounded to bf16:
                                    VVS_NORM_AUTO: the library chooses per call - separate
                                      normalisation kernels (below), or, where that is faster, the
                                      fused layer: the operand of the projection behind a norm is
                                      bf16(x g) and the row factor rsqrt(mean x^2 + eps) multiplies the
                                      fp32 result of the projection (equal in exact arithmetic, a
                                      different rounding of the same operand);
                                    VVS_NORM_SEPARATE: always separate normalisation kernels, which
                                      round bf16(x * rsqrt(mean x^2 + eps) * g), the definition's own
                                      rounding point (more launches per layer) */
  int32_t cache_kind;            /* VVS_CACHE_SAME: cached keys and values have the context's dtype;
                                    VVS_CACHE_E4M3: they are held in 8 bits (see vvs_qcache below: what is held, and by which rounding), in
                                      half of the bytes of bf16, for contexts whose cache is what fills HBM.  Keys and values of the tokens of
                                      a call are taken as they are (a verify call: of all its nodes; a prefill: of a chunk of up to 512 tokens, fp32
                                      64), and rounded when they are cached (see vvs_set_state for roll-backs).  Layers run as separate launches (no drafter contexts; head size 32,
                                      64 or 128, as the dtype allows), so that calls of few rows take longer than with VVS_CACHE_SAME */
  int32_t weight_kind;           /* VVS_WEIGHTS_SAME: weights have the context's dtype;
                                    VVS_WEIGHTS_E4M3: a layer's seven matrices are held in 8 bits, and what they are multiplied by - the norms' outputs, the
                                      attention's (rounded to the dtype first), the activations - is rounded to 8 bits as well (see vvs_qrows below); residual stream
                                      and all else are as ever.  Products of e4m3 numbers enter their sums whole, but from 65 rows on, in bf16 contexts and in front of
                                      the activations, where they are made as VVS_PRODUCTS_E4M3 says.  For contexts whose steps are bound by the weights' bytes.
                                      Embeddings, gains and the output head keep the dtype.  Layers run as separate launches (no drafter contexts; d_model a multiple of 64, d_ff at most 65536);
                                    VVS_WEIGHTS_E4M3_WHOLE: the same, with VVS_PRODUCTS_WHOLE: calls of more than 64 rows take longer */
} vvs_config;
enum { VVS_NORM_AUTO = 0, VVS_NORM_SEPARATE = 1 };
enum { VVS_CACHE_SAME = 0, VVS_CACHE_E4M3 = 1 };
enum { VVS_WEIGHTS_SAME = 0, VVS_WEIGHTS_E4M3 = 1, VVS_WEIGHTS_E4M3_WHOLE = 3 };
#define VVS_MAX_FEATURE_SLOTS 8

/* Sizes in bytes of the three device buffers a context needs.  VVS_ESIZE if the shape is not
 * supported (bf16 needs d_model % 64 == 0, d_ff % 64 == 0, V_eff % 64 == 0, head size 64 or 128;
 * any dtype needs head size % 4 == 0, max_nodes < VVS_MAX_T).  The workspace holds the activations of the widest call: a
 * verify or drafting call of max_nodes + 1 tokens per row or, in a target context, a prefill chunk - in bf16 up to 512 tokens per
 * row (about 4096 rows in all), never more than the prefix and the grid - and, in bf16, what the layers hand on where a forward of few
 * rows runs them all in one launch: buffers of every layer's own, up to 256 rows (121 MB for 36 layers of d 1280, d_ff 3456 with 192 rows). */
vvs_status vvs_query_sizes(const vvs_config* cfg, size_t* kv_bytes, size_t* workspace_bytes,
                           size_t* packed_weight_bytes);

/* Creates a context over caller-allocated device buffers (256-byte aligned).  Synchronous. */
vvs_status vvs_create(const vvs_config* cfg, void* d_kv, void* d_workspace, void* d_packed_weights,
                      vvs_ctx** out);
void vvs_destroy(vvs_ctx* ctx);
const char* vvs_last_error(const vvs_ctx* ctx);   /* ctx may be NULL: error of the last failed create/query */

/* Number of canonical weight tensors (2 + 9 * n_layers + 2, one more for a drafter context) in
 * this order:
 *   embed [vocab, d]; prefix_embed [n_classes + 1, d] (may be NULL for dense prefixes);
 *   per layer: g1 [d], wq [d,d], wk [d,d], wv [d,d], wo [d,d], g2 [d], wg [d,F], wu [d,F], wd [F,d];
 *   gf [d]; wout [d, vocab]; drafter contexts only: fc [2d, d] (rows 0..d-1 multiply the token
 *   embedding, rows d..2d-1 the feature).
 * Matrices are row-major [in, out] (activations multiply from the left); element type = dtype. */
int32_t vvs_num_weight_tensors(const vvs_config* cfg);

/* Repacks the canonical tensors (device pointers, host array of n pointers) into d_packed_weights.
 * The canonical tensors may be freed once the stream has passed this point. */
vvs_status vvs_load_weights(vvs_ctx* ctx, const void* const* d_tensors, int32_t n, vvs_stream s);

/* Neighbour table for the relaxed rule: int32 [vocab, relax_k] on the device, for every id its
 * nearest other ids in latent space in ascending distance.  Kept by reference. */
vvs_status vvs_set_neighbors(vvs_ctx* ctx, const int32_t* d_nbr);

/* Host-only check of a draft topology, with the same rules as vvs_verify (either array may be NULL;
 * both NULL = chain).  Outputs (host, may be NULL): h_depth int32 [T], h_parent_out int32 [N]. */
vvs_status vvs_check_tree(int32_t n_nodes, const int32_t* h_parent, const uint8_t* h_tree_mask, int32_t* h_depth,
                          int32_t* h_parent_out);

/* Prefill (Algorithm 2 of the supplementary material, first line): runs the P prefix tokens and then
 * n_forced teacher-forced image tokens of every row through the model under a causal mask, caches
 * their K/V, and samples the next image token of each prompt from the CFG-mixed distribution at
 * the last position by inverse CDF with d_uniform[b].  Resets the context state.
 *   d_prefix_cond  : class kind: int32 [B, P] class ids;      dense kind: dtype [B, P, d]
 *   d_prefix_uncond: class kind: int32 [B, P] or NULL (null class); dense kind: dtype [P, d], shared
 *   d_forced_tokens: int32 [B, n_forced] or NULL when n_forced == 0; n_forced <= G - 1
 *   d_uniform      : float [B] in [0, 1)
 *   d_first_token  : int32 [B] out (full-vocabulary id); it becomes the pending token. */
vvs_status vvs_prefill(vvs_ctx* ctx, const void* d_prefix_cond, const void* d_prefix_uncond,
                       int32_t n_forced, const int32_t* d_forced_tokens, const float* d_uniform,
                       int32_t* d_first_token, vvs_stream s);

/* One verification pass (Section 2; Algorithm 2: "logits <- M_T(C_t); a <- Verify(logits, C_t)").
 *   n_nodes      : N >= 0 (0 = plain AR sampling of one token)
 *   h_parent     : host int32 [N], h_parent[j-1] in [0, j-1] = parent of node j; NULL = chain
 *   h_tree_mask  : host uint8 [T, T], entry (i, j) != 0 iff j is i or an ancestor of i; may be NULL.
 *                  When both are given they must describe the same tree; when only the mask is
 *                  given the parents are derived from it.
 *   d_draft_tokens: int32 [B, N], full-vocabulary ids inside [logit_lo, logit_hi); siblings distinct
 *   d_draft_probs : float [B, T, V_eff]; row j = the distribution the children of node j were drawn
 *                   from (rows of leaves are not read)
 *   d_uniforms    : float [B, T, 2] in [0, 1): [b, c, 0] decides node c, [b, j, 1] draws the final
 *                   token when the walk ends at node j
 *   mode          : VVS_STRICT or VVS_RELAXED
 *   d_accept_len  : int32 [B] out, number of accepted draft tokens a_b
 *   d_path        : int32 [B, VVS_MAX_T] out, node ids of the accepted path: path[0] = 0, then a_b ids
 *   d_next_token  : int32 [B] out, resampled / bonus token (full-vocabulary id); -1 for a prompt whose
 *                   image is already complete (then a_b = 0)
 * Children of a node are tried in ascending node id; after a rejection the target becomes the
 * normalised positive part of (target - draft) and the rejected id leaves the draft distribution.
 * At most G - n_emitted_b - 1 draft tokens are accepted, so the final token still lies in the image.
 * The outcome is also kept in the workspace for vvs_kv_commit. */
vvs_status vvs_verify(vvs_ctx* ctx, int32_t n_nodes, const int32_t* h_parent, const uint8_t* h_tree_mask,
                      const int32_t* d_draft_tokens, const float* d_draft_probs, const float* d_uniforms,
                      int32_t mode, int32_t* d_accept_len, int32_t* d_path, int32_t* d_next_token,
                      vvs_stream s);

/* Verification with post verification (Section 4.1): the tokens that the previous, verification-free
 * step accepted without asking the target model ride in front of the new candidates and go through
 * the same pass.  They are nodes 1 .. n_post of the tree, a chain below the root (h_parent[j-1] = j-1
 * for j <= n_post), and every other node descends from node n_post; anything else is VVS_EINVAL.
 * They are accepted without a test (their d_draft_probs rows and d_uniforms entries are not read) and
 * count in accept_len / path; the end-of-image cap applies to them like to any accepted token.  The
 * pass gives them their K/V (committed by vvs_kv_commit like every accepted node), which restores
 * exact AR conditioning for the candidates behind them.  d_draft_tokens[b][0 .. n_post-1] are their
 * ids.  n_post = 0 is vvs_verify.  Everything else as in vvs_verify. */
vvs_status vvs_verify_post(vvs_ctx* ctx, int32_t n_nodes, int32_t n_post, const int32_t* h_parent,
                           const uint8_t* h_tree_mask, const int32_t* d_draft_tokens, const float* d_draft_probs,
                           const float* d_uniforms, int32_t mode, int32_t* d_accept_len, int32_t* d_path,
                           int32_t* d_next_token, vvs_stream s);

/* The acceptance stage alone (CFG mix, softmax, accept / resample, path walk) on logits supplied by
 * the caller: d_raw_logits float [R, T, V_eff] (row-major, row r = 2b + {0: conditional,
 * 1: unconditional}).  Same outputs as vvs_verify; does not touch the KV cache, and the outcome is
 * not available to vvs_kv_commit. */
vvs_status vvs_accept_from_logits(vvs_ctx* ctx, int32_t n_nodes, const int32_t* h_parent,
                                  const uint8_t* h_tree_mask, const float* d_raw_logits,
                                  const int32_t* d_draft_tokens, const float* d_draft_probs,
                                  const float* d_uniforms, int32_t mode, int32_t* d_accept_len,
                                  int32_t* d_path, int32_t* d_next_token, vvs_stream s);

/* vvs_accept_from_logits for callers that cannot allocate device memory and have no workspace to lend: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same result.
 * The stage's scratch (per-node partial results and per-node target distributions, which the other entry
 * points keep in the caller's workspace) lives in a static device array inside the library, of
 * VVS_NOALLOC_MAX_PROMPTS * VVS_MAX_T * 8 + VVS_NOALLOC_MAX_PROB_FLOATS * 4 bytes (about 16 MiB), held by every
 * GPU the library runs on until the process ends.  The call allocates and frees nothing.  VVS_ESIZE when
 * n_prompts > VVS_NOALLOC_MAX_PROMPTS, n_prompts * (n_nodes + 1) * V_eff > VVS_NOALLOC_MAX_PROB_FLOATS, or V_eff > 18432.
 * All calls on one GPU share that GPU's array: calls that overlap on one GPU (other streams, other contexts)
 * race; calls on one stream are safe.  The array keeps the last call's contents; nothing in it has to be cleared
 * (every entry a call reads is written by that call first).  Does not touch the KV cache, the workspace, or
 * the outcome kept for vvs_kv_commit; vvs_debug_logits does not see its distributions. */
#define VVS_NOALLOC_MAX_PROMPTS 64
#define VVS_NOALLOC_MAX_PROB_FLOATS (4 << 20)
vvs_status vvs_accept_from_logits_noalloc(vvs_ctx* ctx, int32_t n_nodes, const int32_t* h_parent,
                                          const uint8_t* h_tree_mask, const float* d_raw_logits,
                                          const int32_t* d_draft_tokens, const float* d_draft_probs,
                                          const float* d_uniforms, int32_t mode, int32_t* d_accept_len,
                                          int32_t* d_path, int32_t* d_next_token, vvs_stream s);

/* Section 4.1: moves the K/V of the pending token and of the accepted path of the last vvs_verify
 * into consecutive cache slots S_b .. S_b + a_b, advances S_b and n_emitted_b by a_b + 1 and makes
 * next_token the pending token.  Exactly one commit per verify. */
vvs_status vvs_kv_commit(vvs_ctx* ctx, vvs_stream s);

/* Contexts with VVS_CACHE_E4M3: shortens the cache of every prompt whose length is above `keep` to `keep` slots per layer, row and head, as
 * vvs_qcache_evict does: the slots with the largest accumulated attention weight stay, and the `recent` newest tokens.  Weights are accumulated by the library: of all
 * tokens of a prefill, and of those tokens of a verify call that are certain to be kept (the pending token and the post-verified ones), over cached slots.
 * vvs_set_state does not take weights back: a verify call that is replayed counts again.
 * Positions of later tokens do not change; S_b does.  Not between a verify and its commit (VVS_ESTATE).
 *   keep: a multiple of VVS_QCACHE_BLOCK, at least one block; recent: in [0, keep] */
vvs_status vvs_kv_evict(vvs_ctx* ctx, int32_t keep, int32_t recent, vvs_stream s);

/* Token-level feature cache (Section 4.3; Algorithm 2, "UpdateCache").  vvs_prefill stores the feature
 * of the last prefilled position of every row, vvs_kv_commit appends the features of the tokens it
 * commits (pending token, then the accepted path, in order); a row keeps its feature_slots most
 * recent ones.  A feature is [d_model] values in the context's dtype rounding (bf16 contexts: bf16
 * values).  Reads them out oldest first:
 *   d_features float [R, feature_slots, d_model] out, row r: entries 0 .. count-1 valid, rest zero
 *   d_count    int32 [B] out, valid entries per row of prompt b (both of its rows hold the same number)
 * vvs_set_state does not touch the cache. */
vvs_status vvs_read_features(vvs_ctx* ctx, float* d_features, int32_t* d_count, vvs_stream s);

/* ---- The verification-free step (Sections 4.2 and 4.4).  Host-only helpers need no context. ----
 *
 * Candidate paths of a draft tree = its root-to-leaf node sequences (root excluded), ordered by the
 * node id of their leaf.
 *
 * vvs_select_unverified (Section 4.2, Eq. 1): draws one candidate path uniformly with the uniform
 * u in [0, 1) (path floor(u * |P|)) and keeps its first gamma = min(L_s, floor(mean path length))
 * nodes.  Topology arguments as in vvs_check_tree.  h_nodes: host int32 [VVS_MAX_T] out, the kept node
 * ids in path order (these are the tokens to hand to the next vvs_verify_post as its unverified
 * tokens); n_kept: their number (0 for an empty tree). */
vvs_status vvs_select_unverified(int32_t n_nodes, const int32_t* h_parent, const uint8_t* h_tree_mask, float u,
                                 int32_t* h_nodes, int32_t* n_kept);

/* Uniform-interval policy (Section 4.4): 1 iff step step_index (counted from 0) is verification-free for
 * interval i, i.e. (step_index + 1) % i == 0 with i >= 2; never two in a row. */
int32_t vvs_skip_uniform(int32_t step_index, int32_t interval);

/* Dynamic policy (Algorithm 1): 1 iff the last step was verified and similarity >= threshold. */
int32_t vvs_skip_dynamic(float similarity, float threshold, int32_t last_step_verified);

/* Latent codebook for vvs_path_similarity: float [vocab, dim] on the device, dim in [1, 64]; kept by
 * reference. */
vvs_status vvs_set_codebook(vvs_ctx* ctx, const float* d_embed, int32_t dim);

/* Weighted average similarity of the candidate paths (Eq. 2; Algorithm 1 "CompSim" after
 * "Downsample"): per prompt, S = sum_l w_l S_l with w_l proportional to alpha^l, where S_l is the mean
 * cosine similarity of the codebook embeddings of the tokens at position l over all unordered pairs of
 * the kept paths that reach position l.  Every stride-th path is kept, starting with the first.
 * Positions reached by fewer than two kept paths are left out (weights renormalised); with no such
 * position S = 1; an all-zero embedding has cosine 0.
 *   d_draft_tokens int32 [B, N] full-vocabulary ids (as for vvs_verify); d_similarity float [B] out.
 * Does not touch the model state; may run on another stream than a verify in flight. */
vvs_status vvs_path_similarity(vvs_ctx* ctx, int32_t n_nodes, const int32_t* h_parent, const uint8_t* h_tree_mask,
                               const int32_t* d_draft_tokens, float alpha, int32_t stride, float* d_similarity,
                               vvs_stream s);

/* One drafting call (Algorithm 2: "f_t <- Retrieve(C, a); C_t <- M_D(f_t, a)"; Section 3, "Stale
 * Feature Reusability"; Section 4.1): the drafter - a context created with draft_input = 1, one or more
 * decoder blocks of the target's kind, the same d_model, dtype, B, id slice, grid and kind of feature
 * (feature_pre_norm) as the target -
 * is conditioned on the n_ctx most recent features of the target's token-level feature cache paired,
 * by recency, with the n_ctx most recent tokens of the sequence, and fills a candidate tree of a fixed
 * shape level by level: node j >= 1 gets the input W_fc [embedding of its token ; feature the drafter
 * produced at its parent]; the distribution at a node is the softmax of the drafter's CFG-mixed logits
 * (the drafter context's cfg_scale); the c-th child of a node (ascending node id) carries the id with
 * the c-th largest mixed logit there, ties to the lower id.  The drafter keeps no state between calls:
 * a node attends to the n_ctx pairs, its ancestors and itself.  Pair i sits at image index
 * first + i with first = max(0, root - (n_ctx - 1)), root = emitted tokens of the target - 1 +
 * n_unverified; node j at first + n_ctx - 1 + depth(j).
 *   n_nodes, h_parent, h_tree_mask: the tree shape, as for vvs_verify (n_nodes >= 1)
 *   n_ctx          : 1 .. feature_slots of the target; every row of the target should hold that many
 *                    features (a missing feature is read as zeros); n_ctx + (number of nodes that have
 *                    children, root excluded) <= max_nodes + 1 of the drafter context
 *   d_recent_tokens: int32 [B, n_ctx] full-vocabulary ids, oldest first; the last one is the root (the
 *                    target's pending token, or the last token accepted without verification)
 *   n_unverified   : tokens accepted without verification since the target's last commit, 0 .. 8
 *                    (they move the root's position; their features do not exist: the cached ones
 *                    are paired with newer tokens - stale features)
 *   d_given_tokens : NULL, or int32 [B, N]: the nodes' tokens are taken from here (e.g. sampled by the
 *                    caller) and only the distributions are computed
 *   d_draft_tokens : int32 [B, N] out;  d_draft_probs: float [B, T, V_eff] out, row j = distribution of
 *                    the children of node j (zeros for a leaf): the layouts vvs_verify takes.
 * The target's state and feature cache are only read.  Same stream rules as every other call. */
vvs_status vvs_draft(vvs_ctx* drafter, vvs_ctx* target, int32_t n_nodes, const int32_t* h_parent,
                     const uint8_t* h_tree_mask, int32_t n_ctx, const int32_t* d_recent_tokens,
                     int32_t n_unverified, const int32_t* d_given_tokens, int32_t* d_draft_tokens,
                     float* d_draft_probs, vvs_stream s);

/* ---- Key/value cache in 8 bits -------------------------------------------------------------------------------
 *
 * A cache of its own beside the contexts': keys and values of one attention layer (or of all layers of a model), appended to, looked at
 * and thinned out by the calls below, for programs that keep more in HBM, or read less of it, than bf16 allows.
 *
 * What is held.  The slots of one layer, row and key/value head are cut into blocks of VVS_QCACHE_BLOCK; keys and values of a block each have one
 * power of two 2^E, and their elements are e4m3 numbers (4 exponent bits, 3 of mantissa, largest 448) times 2^E.  E is the smallest one, at least -110, with
 * |x| <= 448 * 2^E for every finite x that was appended to the block; an append to a block that holds something keeps the larger E, and what was held is
 * rounded to it (exact, but for elements below 2^-6 * 2^E).  Rounding is to nearest, ties to even; an element that is not finite is held as NaN.
 *
 * Lengths are the caller's: d_len int32 [n_rows] says how many slots of each row are filled, and is only read (values outside [0, capacity] are taken as
 * the nearest inside).  Tokens per row may differ: d_n_tokens int32 [n_rows], in [0, n_tokens] (clamped), or NULL for n_tokens everywhere; of the tokens behind a row's
 * number nothing is read, and nothing is written for them.
 *
 * Tensors are [n_rows, n_tokens, heads, head_size] in the cache's dtype; a stride argument gives the elements from one token to the next where they lie further apart
 * than heads * head_size (0: they do not), so that q, k and v can be parts of one projection's output.  Rows are n_tokens tokens apart.  Pointers and
 * strides have to be multiples of 16 bytes.  All tensors live on the device that was current at vvs_qcache_create, which has to be current at every call.
 * Calls on one cache share its workspace: issue them on one stream, or order them.  All calls can be captured into a graph.
 * One call appends, evicts down to, or reads about 2^31 / n_kv_heads slots per row at most (VVS_ESIZE beyond). */
#define VVS_QCACHE_BLOCK 32
typedef struct vvs_qcache vvs_qcache;  /* opaque host object; owns no device memory */

typedef struct {
  int32_t n_layers, n_rows;
  int32_t n_heads, n_kv_heads;   /* query heads; key/value heads (each serves n_heads / n_kv_heads query heads in a row) */
  int32_t head_size;             /* 32, 64 or 128 */
  int32_t capacity;              /* slots per layer, row and key/value head */
  int32_t max_tokens;            /* largest n_tokens of an attention call */
  int32_t dtype;                 /* VVS_FP32 or VVS_BF16: type of q, k, v and outputs */
} vvs_qcache_config;

/* Sizes in bytes of the two device buffers of a cache. */
vvs_status vvs_qcache_query_sizes(const vvs_qcache_config* cfg, size_t* cache_bytes, size_t* workspace_bytes);
/* Creates a cache over caller-allocated device buffers (256-byte aligned).  Synchronous: clears both. */
vvs_status vvs_qcache_create(const vvs_qcache_config* cfg, void* d_cache, void* d_workspace, vvs_qcache** out);
void vvs_qcache_destroy(vvs_qcache* c);
const char* vvs_qcache_last_error(const vvs_qcache* c);   /* c must not be NULL (a failed create or query: vvs_last_error(NULL)) */

/* Rounds keys and values into the slots d_len[r] .. of layers layer .. layer + n_layers - 1.
 *   d_k, d_v   : [n_layers, n_rows, src_tokens, n_kv_heads, head_size]
 *   n_tokens   : most tokens taken of a row; src_tokens: tokens per row of d_k and d_v
 *   d_select   : int32 [n_rows, n_tokens]: the source token of each taken one (an accepted path; one outside [0, src_tokens) is taken as zeros), or
 *                NULL: the first ones, and n_tokens <= src_tokens
 * Tokens beyond the capacity are dropped.  Slots below d_len keep their values up to the rounding above.  Weights and positions of the slots (vvs_qcache_evict) are the caller's: whoever
 * evicts more than once writes the positions of the appended tokens into their slots. */
vvs_status vvs_qcache_append(vvs_qcache* c, int32_t layer, int32_t n_layers, const int32_t* d_len, int32_t n_tokens, const int32_t* d_n_tokens,
                             int32_t src_tokens, const int32_t* d_select, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                             vvs_stream s);

/* Attention of a block of query tokens over the cached slots of their row and over the block's own keys and values, which are not rounded to 8 bits:
 * out = softmax(scale q K^T) V, every query over slots 0 .. d_len[r] - 1 and the block tokens it may see.
 *   h_parent, h_tree_mask: the block's topology as for vvs_verify with n_tokens - 1 nodes (token 0 is the root); both NULL: a chain, the only form with
 *                n_tokens > VVS_MAX_T.  What a masked token holds, NaN and infinities included, does not matter.
 *   d_k, d_v   : [n_rows, n_tokens, n_kv_heads, head_size]; both NULL: the queries see the cache alone
 *   scale      : positive and finite
 *   d_out      : [n_rows, n_tokens, n_heads, head_size], contiguous; a query that sees nothing (no block, nothing cached) gets zeros.  Apart from d_k and d_v, and from d_q,
 *                whose queries are read again behind the outputs where weights are counted; without d_mass and d_block_mass it may be a contiguous d_q itself
 *   d_lse      : float [n_rows, n_tokens, n_heads] out, log of the sum of exp(scale q k) (-inf for a query that sees nothing); may be NULL
 *   n_counted  : the softmax weights of tokens 0 .. n_counted - 1 of every row, of all query heads of a key/value head, are added up per key:
 *   d_mass     : float [n_rows, n_kv_heads, capacity], cached slots: added to (NULL: left out)
 *   d_block_mass: float [n_rows, n_kv_heads, n_tokens], block tokens: set (NULL: left out)
 * Sums are in a fixed order: the same call gives the same bits.  They are taken in front of the division by the weights' sum, of up to 64 |v| per key: values of 2^121 over the number of
 * keys and more may come out as infinities.  How a call is cut into pieces goes by n_tokens and the capacity, not by d_len, which a captured call finds changed: a large, nearly empty
 * cache pays for joining pieces without slots. */
vvs_status vvs_qcache_attention(vvs_qcache* c, int32_t layer, const int32_t* d_len, int32_t n_tokens, const int32_t* d_n_tokens, const int32_t* h_parent,
                                const uint8_t* h_tree_mask, const void* d_q, int64_t q_stride, const void* d_k, int64_t k_stride, const void* d_v,
                                int64_t v_stride, float scale, void* d_out, float* d_lse, int32_t n_counted, float* d_mass, float* d_block_mass, vvs_stream s);

/* Eviction by accumulated attention weight: every layer, row and key/value head whose length is above `keep` keeps the `keep` slots of largest weight (equal ones: the
 * lower slot; a NaN counts as the largest); the `recent` newest tokens - those at positions above the row's largest filled one minus `recent` - are kept whatever their weight, as
 * far as there is room.  Kept slots from `keep` on move, in order, into the slots below that were given up; the others stay where they are.  A block that something moves into
 * takes the largest E of the blocks that its slots were in.  The new length is min(d_len[r], keep); the caller sets it.
 *   keep       : a multiple of VVS_QCACHE_BLOCK, at least one block; recent: in [0, keep]
 *   d_mass     : float [n_layers, n_rows, n_kv_heads, capacity];  d_mass_out: the same, out, weights of what lies in the slots now, 0 behind the new length (may
 *                be d_mass itself)
 *   d_pos, d_pos_out: int32, likewise, positions of the tokens in the slots (0 behind the new length); both NULL: a slot's number is its position, as it is before the first
 *                eviction.  Behind one, slots that are appended to hold 0 until the caller says which tokens they hold: left at that, they are the oldest, not the newest */
vvs_status vvs_qcache_evict(vvs_qcache* c, int32_t layer, int32_t n_layers, const int32_t* d_len, int32_t keep, int32_t recent, const float* d_mass,
                            float* d_mass_out, const int32_t* d_pos, int32_t* d_pos_out, vvs_stream s);

/* Cached keys and values as numbers: d_k, d_v [n_layers, n_rows, n_slots, n_kv_heads, head_size] out, slots d_first[r] .. (NULL: from 0) of every row; slots that
 * are not in [0, d_len[r]) read as zeros. */
vvs_status vvs_qcache_read(vvs_qcache* c, int32_t layer, int32_t n_layers, const int32_t* d_len, const int32_t* d_first, int32_t n_slots, void* d_k,
                           void* d_v, vvs_stream s);

/* ---- Rotary positions on several axes (frame, row, column of a video; text) ----------------------------------------
 *
 * A head's first 2 * (sum of pairs) dims are rotated in pairs by the angle position[axis of the pair] * rate[pair], the others copied.  Pairs belong to the axes in order:
 * the first pairs[0] to axis 0, and so on.  The contexts' own positions are two axes (row, column) of head_size / 4 pairs each, VVS_ROPE_OWN, VVS_ROPE_ADJACENT. */
#define VVS_ROPE_MAX_AXES 4
enum { VVS_ROPE_OWN = 0,       /* rate of pair i of an axis with n pairs: base^(-i / n), every axis a series of its own */
       VVS_ROPE_SHARED = 1 };  /* rate of pair j of the head: base^(-2 j / head_size), one series cut into axes */
enum { VVS_ROPE_ADJACENT = 0,  /* pair j: dims 2 j and 2 j + 1 */
       VVS_ROPE_HALVES = 1 };  /* pair j: dims j and j + (sum of pairs) */
typedef struct vvs_rope vvs_rope;   /* opaque host object */

typedef struct {
  int32_t head_size;                  /* a multiple of 8, at most 256 */
  int32_t n_axes;                     /* 1 .. VVS_ROPE_MAX_AXES */
  int32_t pairs[VVS_ROPE_MAX_AXES];   /* of axes 0 .. n_axes - 1, at least 1 each; their sum is a multiple of 4
                                         (VVS_ROPE_HALVES: of 8) and at most head_size / 2 */
  int32_t series, pairing;
  int32_t dtype;
  float base;                         /* > 1 */
} vvs_rope_config;

vvs_status vvs_rope_create(const vvs_rope_config* cfg, vvs_rope** out);   /* host only */
void vvs_rope_destroy(vvs_rope* r);
const char* vvs_rope_last_error(const vvs_rope* r);                       /* r must not be NULL */

/* Rotates queries and keys of n_tokens tokens (up to 2^26 - 4) in one launch; angles are taken in 64 bits, so that far positions are as exact as near ones.
 *   d_pos      : int32 [n_tokens, n_axes], any sign
 *   d_q, d_q_out [n_tokens, n_heads, head_size]; d_k, d_k_out [n_tokens, n_kv_heads, head_size] (n_kv_heads 0: NULL); an output may be its input; strides as for
 *                the cache's tensors, 0: contiguous; pointers and strides multiples of 16 bytes
 *   inverse    : 1: by the negative angles - takes a rotation back, and is its gradient */
vvs_status vvs_rope_apply(vvs_rope* r, int32_t n_tokens, const int32_t* d_pos, int32_t n_heads, const void* d_q, int64_t q_stride, void* d_q_out,
                          int64_t q_out_stride, int32_t n_kv_heads, const void* d_k, int64_t k_stride, void* d_k_out, int64_t k_out_stride,
                          int32_t inverse, vvs_stream s);

/* ---- Rows and weights in 8 bits: a layer's norms, projections and gated products -----------------------------------------
 *
 * What is held.  A row of `width` elements is cut into blocks of VVS_QROWS_BLOCK; a block has one power of two 2^E, and its elements are e4m3 numbers (4 exponent bits, 3 of mantissa,
 * largest 448) times 2^E.  E is the smallest one, at least -110, with |x| <= 448 * 2^E for every finite x of the block.  Rounding is to nearest, ties to even; an element that is not finite
 * is held as NaN.  Every column of a weight matrix [in, out] is held likewise, in blocks along `in`.
 *
 * Rows lie in two buffers (16-byte aligned): values, one byte per element, rows of `width` rounded up to VVS_QROWS_BLOCK, 0 behind the width; and powers, one byte E + 127 per
 * block, rows of the number of blocks rounded up to 4, 0 behind the last block.  What is taken as rows in 8 bits has to lie so; what the calls below write does.
 * Rows behind n_rows are neither read nor written.  Rows have at most 65536 elements.
 *
 * Tensors are [n_rows, width] in VVS_FP32 or VVS_BF16; a stride argument gives the elements from one row to the next where they lie further apart than `width` (0: they do not).  Any
 * width, stride and element-aligned pointer is taken; 16-byte accesses are made where pointer and stride are multiples of 16 bytes (of 4 elements for outputs of
 * vvs_qlinear_apply).  Outputs share no memory with inputs, with each other or with a map's buffers, except where stated: such calls are refused (VVS_EINVAL).  All calls can be captured into a graph; those on rows go to the current device. */
#define VVS_QROWS_BLOCK 128

/* Sizes in bytes of the two buffers of n_rows rows. */
vvs_status vvs_qrows_sizes(int32_t width, int32_t n_rows, size_t* value_bytes, size_t* power_bytes);
const char* vvs_qrows_last_error(void);   /* of this thread's last failed vvs_qrows call */

/* Rounds rows to 8 bits. */
vvs_status vvs_qrows_round(int32_t n_rows, int32_t width, int32_t dtype, const void* d_x, int64_t x_stride, void* d_values, void* d_powers,
                           vvs_stream s);

/* Root-mean-square norm with the residual's addition: x' = x + delta in fp32, rounded to the type of x; y = x' * rsqrt(mean x'^2 + eps) * gain, which goes into 8 bits.  The sum of squares is in
 * fp32; rows whose squares fp32 does not hold are scaled by a power of two for it, so that elements may be of any size.
 *   d_delta    : [n_rows, width] of its own type, or NULL: nothing is added
 *   d_x_out    : x' in the type of x; may be d_x itself (with the same stride); NULL: not written
 *   d_gain     : [width] of its own type
 *   eps        : finite, not negative (0: a row of zeros becomes NaN) */
vvs_status vvs_qrows_norm(int32_t n_rows, int32_t width, int32_t x_dtype, const void* d_x, int64_t x_stride, int32_t delta_dtype, const void* d_delta,
                          int64_t delta_stride, void* d_x_out, int64_t x_out_stride, int32_t gain_dtype, const void* d_gain, float eps, void* d_values,
                          void* d_powers, vvs_stream s);

/* Rows in 8 bits as numbers (bf16 has all of them, but 2^128, what elements from 0.97 * 2^128 on are held as: it reads as an infinity). */
vvs_status vvs_qrows_read(int32_t n_rows, int32_t width, const void* d_values, const void* d_powers, int32_t dtype, void* d_out, int64_t out_stride,
                          vvs_stream s);

typedef struct vvs_qlinear vvs_qlinear;   /* opaque host object; owns no device memory */

typedef struct {
  int32_t in, out;               /* elements of a row that goes in and of one that comes out */
  int32_t max_rows;              /* largest n_rows of a call, at most 2^20 */
  int32_t gated;                 /* 0: one matrix, for vvs_qlinear_apply; 1: gate and up, for vvs_qlinear_gate */
  int32_t dtype;                 /* of the weights that vvs_qlinear_load takes and vvs_qlinear_read gives */
  int32_t products;              /* how products of e4m3 numbers are summed:
                                    VVS_PRODUCTS_WHOLE: they enter sums in fp32 whole, in every call;
                                    VVS_PRODUCTS_E4M3: calls of more than 64 rows may take the matrix instructions for e4m3, twice as fast, which cut off what lies 2^13 below the largest of 8
                                      neighbouring products.  A sum is so off by up to 7 * 2^-13 of the sum of its products' magnitudes - a hundredth of what rounding both sides to e4m3 may have cost it,
                                      but more than fp32's rounding, which shows in sums that cancel and in small elements beside far larger ones;
                                    VVS_PRODUCTS_AUTO: as VVS_PRODUCTS_E4M3 where the result is rounded to bf16 or 8 bits, as VVS_PRODUCTS_WHOLE for outputs in VVS_FP32 */
} vvs_qlinear_config;
enum { VVS_PRODUCTS_AUTO = 0, VVS_PRODUCTS_WHOLE = 1, VVS_PRODUCTS_E4M3 = 2 };

/* Sizes in bytes of the two device buffers of a linear map: weights in 8 bits in the kernels' own order, workspace.  Calls on a map, vvs_qlinear_load among them, are issued on one stream or ordered by
 * the caller.  A workspace may serve several maps - it has to hold the largest one's bytes - if the calls of all of them are; captured graphs that share one must not run at the same time. */
vvs_status vvs_qlinear_query_sizes(const vvs_qlinear_config* cfg, size_t* weight_bytes, size_t* workspace_bytes);
/* Creates a map over caller-allocated device buffers (256-byte aligned) on the current device, which has to be current at every call.  Synchronous: clears the workspace,
 * which no other call may be using. */
vvs_status vvs_qlinear_create(const vvs_qlinear_config* cfg, void* d_weights, void* d_workspace, vvs_qlinear** out);
void vvs_qlinear_destroy(vvs_qlinear* l);
const char* vvs_qlinear_last_error(const vvs_qlinear* l);   /* l must not be NULL (a failed create or query: vvs_last_error(NULL)) */

/* Rounds weights [in, out] (row-major, contiguous) to 8 bits; d_w_up: NULL, with a gate the up weights, likewise.  The tensors may be freed once the stream has passed this point. */
vvs_status vvs_qlinear_load(vvs_qlinear* l, const void* d_w, const void* d_w_up, vvs_stream s);
/* The weights that are held, as numbers in the type of the config; arguments as above. */
vvs_status vvs_qlinear_read(vvs_qlinear* l, void* d_w, void* d_w_up, vvs_stream s);

/* out = x W for rows in 8 bits of width `in`: out [n_rows, out] in out_dtype.
 * Sums are in fp32 and in a fixed order: the same call gives the same bits.  With up to 64 rows products of e4m3 numbers enter them whole, with more rows as vvs_qlinear_config.products says; what the matrix
 * instructions for e4m3 cut off was 1.3e-5 of the result in the 2-norm for normally distributed operands, where the rounding of the output is 1.7e-3 in bf16 and 2.6e-2 in 8 bits.  The order of a sum, and so the
 * last bits of a row, may depend on how many rows a call has. */
vvs_status vvs_qlinear_apply(vvs_qlinear* l, int32_t n_rows, const void* d_values, const void* d_powers, int32_t out_dtype, void* d_out, int64_t out_stride,
                             vvs_stream s);

/* silu(x W_gate) * (x W_up), silu(a) = a / (1 + e^-a), into rows in 8 bits of width `out`. */
vvs_status vvs_qlinear_gate(vvs_qlinear* l, int32_t n_rows, const void* d_values, const void* d_powers, void* d_out_values, void* d_out_powers,
                            vvs_stream s);

/* 1 if a forward over n_tokens query tokens per row (a verify call with n_tokens - 1 draft nodes, or a
 * prefill chunk) takes the fused layer described at vvs_config.norm_mode, 0 if it runs the separate
 * normalisation kernels.  Host only; ctx must not be NULL. */
int32_t vvs_plan_is_fused(const vvs_ctx* ctx, int32_t n_tokens);

/* Per-prompt state: int32 [3, B] out = cached length S_b, emitted image tokens, pending token. */
vvs_status vvs_read_state(vvs_ctx* ctx, int32_t* d_state, vvs_stream s);

/* Overwrites the per-prompt state with int32 [3, B] (same layout as vvs_read_state): rolls the context
 * back (or forward) to a cached length whose K/V are still in the cache, e.g. to replay one verify
 * call.  Cached slots below the given length must hold valid K/V; that is the caller's business.
 * Clears a pending (uncommitted) verify.
 * With VVS_CACHE_E4M3 a roll-back into a block of VVS_QCACHE_BLOCK slots does not undo what the tokens committed since did to it: where they were larger than the block's, it keeps their power
 * of two, and its slots the rounding to it (elements below 2^-6 of it lose bits).  A replay of a verify call may therefore differ from the call; replays among each other have the same bits.
 * Nor does it undo an eviction: a state from before one is not restored. */
vvs_status vvs_set_state(vvs_ctx* ctx, const int32_t* d_state, vvs_stream s);

/* Kernel-class timing for benchmarks.  While enabled, every kernel launch of prefill / verify /
 * commit is bracketed by HIP events recorded on the caller's stream (host objects; no device
 * memory).  vvs_timing_read waits for the recorded events and returns the number of launches and
 * their summed duration for one class since timing was enabled.  Where a layer's q/k/v projection and its
 * attention run as one launch (bf16, head size 64; not with more (head, prompt) pairs than CUs unless
 * they fill their rounds well), that launch counts as VVS_K_GEMM and the attention class stays empty.  Where all layers of a
 * forward are one launch (bf16, few rows of up to VVS_MAX_T tokens: up to 192 to 256 rows at head size 64 where vvs_plan_is_fused, up to 64 or
 * 128 with separate normalisations and either head size), that launch, with its attention, normalisations and SwiGLU, and a
 * drafter's input map, is one of VVS_K_GEMM: such a verify call has two of them, the layers and the output head. */
enum { VVS_K_GEMM = 0, VVS_K_ATTENTION = 1, VVS_K_ACCEPT = 2, VVS_K_ELEMENTWISE = 3, VVS_K_COMMIT = 4, VVS_K_CLASSES = 5 };
vvs_status vvs_timing_enable(vvs_ctx* ctx, int32_t on);
vvs_status vvs_timing_read(vvs_ctx* ctx, int32_t kernel_class, int32_t* n_launches, float* total_ms);

/* Inspection of the last verify (or prefill, with T = 1; for a drafter context: the last level of the
 * last vvs_draft, T = its block tokens: the n_ctx pairs, then the nodes that have children ordered by
 * depth, then id): any pointer may be NULL.
 *   d_raw_logits float [R, T, V_eff]; d_mixed_logits float [B, T, V_eff]; d_probs float [B, T, V_eff]. */
vvs_status vvs_debug_logits(vvs_ctx* ctx, float* d_raw_logits, float* d_mixed_logits, float* d_probs,
                            vvs_stream s);

/* Cached K and V of one (layer, row) as float [n_slots, d_model] (head-major inside a row), slots
 * 0 .. n_slots - 1 (after vvs_kv_evict a slot holds another token for every head). */
vvs_status vvs_debug_kv(vvs_ctx* ctx, int32_t layer, int32_t row, int32_t n_slots, float* d_k, float* d_v,
                        vvs_stream s);

/* C[M, N] = A[M, K] * W[K, N] through the same repacking and GEMM kernels the forward uses (bf16
 * contexts: the MFMA path; n and k multiples of 64), for unit tests.  d_a dtype [M, K]; d_w dtype
 * [K, N] (canonical [in, out] layout); d_scratch of vvs_debug_gemm_scratch_bytes bytes, 256-byte
 * aligned; d_c float [M, N]. */
size_t vvs_debug_gemm_scratch_bytes(const vvs_ctx* ctx, int32_t m, int32_t n, int32_t k);
vvs_status vvs_debug_gemm(vvs_ctx* ctx, int32_t m, int32_t n, int32_t k, const void* d_a, const void* d_w,
                          void* d_scratch, float* d_c, vvs_stream s);

/* Plain device-to-device copy of `bytes` bytes (multiple of 16; 16-byte aligned pointers) with one
 * grid-stride kernel.  Reads and writes exactly `bytes`: used to calibrate hardware traffic counters. */
vvs_status vvs_debug_copy(vvs_ctx* ctx, void* d_dst, const void* d_src, size_t bytes, vvs_stream s);

/* Looks after which a wait inside a launch of all layers gives up (see the top of this file); 0: the default.  For unit tests. */
vvs_status vvs_debug_wait_limit(vvs_ctx* ctx, int32_t polls);

/* Measures how fast a compute unit pulls bytes through its L1 - the figure that bounds the projection kernels of this
 * library.  Launches `n_workgroups` workgroups of `waves` waves (1..16); workgroup w reads the `region_bytes` (a multiple of
 * 8192) at d_src + w * wg_stride_bytes (16-byte aligned; stride 0: every workgroup reads the same region, which then stays
 * in L2 when it is small; the caller's buffer must hold (n_workgroups - 1) * wg_stride_bytes + region_bytes) `reps` times,
 * its waves taking 1 KiB blocks round-robin, 8 blocks in flight per wave.  mode 0: 16-byte loads into registers; mode 1: direct-to-LDS loads (the staging path of the
 * tiled GEMMs).  d_sink: uint32 [n_workgroups]; mode 0 leaves a checksum of what thread 0 of each workgroup read (the sum
 * over its loads of the xor of the four words), mode 1 leaves 0 - it only keeps the loads alive.  The caller times the launch;
 * bytes through the L1 of a CU = region_bytes * reps.  VVS_EINVAL for arguments out of these ranges. */
vvs_status vvs_debug_fill_probe(vvs_ctx* ctx, const void* d_src, size_t region_bytes, size_t wg_stride_bytes, int32_t reps, int32_t mode,
                                int32_t n_workgroups, int32_t waves, uint32_t* d_sink, vvs_stream s);

#ifdef __cplusplus
}
#endif
#endif /* VVS_H */
