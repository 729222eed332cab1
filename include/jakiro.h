/*
 * jakiro.h - C interface of the Jakiro draft-and-verify step for NVIDIA B200 (sm_100a).
 *
 * One speculative-decoding step of arXiv 2502.06282 has three phases (Sec. 2.1): draft,
 * verify, refine.  This library provides the per-step kernels of each phase:
 *
 *   jk_draft_pre           the draft layer in front of the MoE: reduction layer and attention
 *                          (Sec. 3.1.2, Eq. 1)
 *   jk_draft_expand        one layer of the decoupled MoE draft head (Sec. 3.1.2, Eq. 2-5)
 *   jk_tree_finalize       rerank the drafted candidates into the verification tree and
 *                          build its attention mask (Sec. 3.1.2, Fig. 4)
 *   jk_tree_verify_attn    tree-masked attention of one target layer (Sec. 2.1 step 2)
 *   jk_accept_and_compact  acceptance walk, bonus token and KV-cache compaction
 *                          (Sec. 2.1 steps 2-3)
 *
 * and, for a server around it:
 *
 *   jk_tree_verify_attn_paged, jk_paged_*   the attention over a paged 8-bit cache, and its upkeep
 *   jk_sample              temperature, top-k, top-p, min-p: the token, or the filtered target rows
 *   jk_add_norm, jk_linear, jk_rope_qkv, jk_quantize_rows   the rest of a target layer around its
 *                          attention: norm with the residual's addition, projections and FFN, rotary
 *                          positions; in T or with 8-bit operands
 *
 * Conventions that hold for every call
 *   - Returns 0 (JK_OK) or a negative jk_status.  Nothing throws or aborts.
 *   - Pointers named "host" are host memory; every other pointer is DEVICE memory on the
 *     current CUDA device, owned by the caller, 16-byte aligned.  The library allocates no
 *     device memory: scratch space is the caller-provided workspace (jk_set_workspace).
 *   - `stream` is a cudaStream_t passed as void*.  Calls enqueue work and return without
 *     synchronising.  Argument errors are reported by the return value before anything is
 *     launched; data-dependent errors found on the device (an index out of range) are
 *     recorded in a status word that jk_read_status returns.
 *   - Tensors are dense, row-major, innermost index last.  "T" below is the context's
 *     dtype (float or bfloat16).  B = batch, F = frontier nodes of this layer, H = hidden,
 *     N = experts, K = active experts per node, I = expert inner size, V = vocabulary,
 *     k_e = children per (node, expert), W = frontier width, M = tree nodes incl. root,
 *     D = tree depth, Hq/Hkv/d = attention heads and head size, L = target layers.
 *   - Same inputs give bitwise the same outputs (no floating-point atomics).
 *   - Calls on one context must not overlap on the device: they share the workspace.
 */
#ifndef JAKIRO_H_
#define JAKIRO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  JK_OK = 0,
  JK_ERR_NULL = -1,       /* a required pointer is NULL                                  */
  JK_ERR_SHAPE = -2,      /* a size is outside the supported range                       */
  JK_ERR_ALIGN = -3,      /* a pointer or stride is not 16-byte aligned                  */
  JK_ERR_DTYPE = -4,      /* unknown dtype                                               */
  JK_ERR_CAPACITY = -5,   /* more rows than the context was created for                  */
  JK_ERR_WORKSPACE = -6,  /* workspace missing or too small                              */
  JK_ERR_CUDA = -7,       /* a CUDA runtime call failed (see jk_last_cuda_error)         */
  JK_ERR_TIMEOUT = -8,    /* a bounded device-side wait ran out                          */
  JK_ERR_BOUNDS = -9      /* device status: an input index was out of range              */
} jk_status;

typedef enum { JK_F32 = 0, JK_BF16 = 1 } jk_dtype;

/* Limits: top_k <= n_experts <= 8, k_per_expert <= 16, max_tree <= 128, max_depth <= 16,
 * max_batch * max_frontier <= 128, head_dim 64 or 128, hidden/inter multiples of 8,
 * ceil(vocab / 4096) * k_per_expert <= 512; a step's candidate pool holds at most 4096 entries
 * per sequence. */
typedef struct {
  int32_t hidden, n_experts, top_k, inter, vocab;
  int32_t n_q_heads, n_kv_heads, head_dim;
  int32_t max_batch, max_tree, max_depth, max_frontier, k_per_expert;
  int32_t dtype;            /* jk_dtype of weights, hidden states, Q and the KV cache    */
  float rms_eps;            /* epsilon of the pre-MoE RMSNorm                            */
  int32_t use_pre_norm;     /* 1: router and experts see RMSNorm(u) * norm_weight (the
                               normalisation Sec. 3.1.2 leaves out of Eq. 1-5); 0: u     */
  int32_t branch_residual;  /* 1: branch feature = g_r * Expert_r(x) + u; 0: g_r * Expert_r(x) */
  int32_t head_mode;        /* 0: decoupled heads, one logits row per selected expert (Eq. 4);
                               1: contrastive heads (Sec. 3.2, Eq. 6-8; needs top_k = 2): row 0 is
                               Head(f^moe), row 1 is Head(f^const), see jk_draft_expand            */
  float contrast_alpha;     /* alpha and beta of Eq. 7: f^const = beta f^top1 - alpha f^top2       */
  float contrast_beta;
} jk_config;

typedef struct jk_ctx jk_ctx;

/* Host-only bookkeeping; no CUDA call is made.  *out is owned by the caller until jk_destroy. */
int jk_create(jk_ctx** out, const jk_config* host_cfg);
int jk_destroy(jk_ctx* ctx);
/* Bytes of device scratch the context needs (a multiple of 256). */
size_t jk_workspace_bytes(const jk_ctx* ctx);
/* dev_ptr: device memory, 256-byte aligned, at least jk_workspace_bytes(ctx) bytes, owned by
 * the caller and kept alive while the context is used.  Clears the device status word on
 * `stream`. */
int jk_set_workspace(jk_ctx* ctx, void* stream, void* dev_ptr, size_t bytes);
const char* jk_strerror(int code);
/* Text of the last CUDA runtime error seen by this context ("" if none). */
const char* jk_last_cuda_error(const jk_ctx* ctx);
/* Synchronises `stream`, copies the device status word to *host_status (0 or a jk_status)
 * and clears it. */
int jk_read_status(jk_ctx* ctx, void* stream, int32_t* host_status);
/* Which kernels run the dense contractions: 0 = CUDA-core kernels, 1 = tensor-core
 * (tcgen05) kernels where the dtype allows.  Default 1 for bf16, always 0 for f32. */
int jk_set_tensor_path(jk_ctx* ctx, int32_t enable);
/* 1 if the tensor-core kernels will run the contractions of this context (bf16, enabled, rows
 * within their limit, driver entry point for tensor maps found), else 0. */
int jk_tensor_path_active(jk_ctx* ctx);
/* Which tensor-core kernel runs jk_tree_verify_attn for bf16: 0 = chosen per call from the sizes
 * (default), 1 = one CTA per (query block, key slice) with a merge kernel, 2 = the persistent
 * kernel that deals key tiles evenly to one CTA per SM, 3 = the kernel whose key slices form a
 * thread-block cluster and merge through distributed shared memory (2 and 3 fall back to 1 where
 * their limits do not hold).  All compute the operation of arXiv 2502.06282 Sec. 2.1 step 2 with
 * the mask of Fig. 4; the choice only affects speed.  Returns JK_ERR_SHAPE for another value. */
int jk_set_attn_kernel(jk_ctx* ctx, int32_t mode);

/* Diagnostics (the paper has no counterpart): with max_launches > 0 every kernel launch of this
 * context is bracketed by a pair of CUDA events on its stream (up to max_launches launches
 * between two collects); 0 switches it off.  jk_profile_collect synchronises `stream`, writes
 * the summed milliseconds and the launch count of every stage to the two host arrays of
 * jk_profile_stage_count() entries and starts over.  Event handles are host resources; no
 * device memory is allocated. */
int jk_profile_enable(jk_ctx* ctx, int32_t max_launches);
int jk_profile_collect(jk_ctx* ctx, void* stream, float* host_ms, int32_t* host_count);
/* As jk_profile_collect, but the recorded event pairs are kept.  When the calls were recorded into
 * a CUDA graph (stream capture with profiling enabled turns every event record into a graph
 * node), every replay of the graph records the same events again: read them after each replay. */
int jk_profile_read(jk_ctx* ctx, void* stream, float* host_ms, int32_t* host_count);
int32_t jk_profile_stage_count(void);
const char* jk_profile_stage_name(int32_t stage);

/* Draft weights (Sec. 3.1.1-3.1.2): device pointers, read-only, output-major. */
typedef struct {
  const void* router;       /* T [N, H]     expert centroids e_j (Eq. 2)                 */
  const void* w_gate;       /* T [N, I, H]  SiLU branch of Expert_j                      */
  const void* w_up;         /* T [N, I, H]  linear branch of Expert_j                    */
  const void* w_down;       /* T [N, H, I]  output projection of Expert_j                */
  const void* lm_head;      /* T [V, H]     the target model's LM head (shared, Eq. 4)   */
  const void* norm_weight;  /* T [H] or NULL (= ones)                                    */
} jk_draft_weights;

/* Candidate pool of one step: every child proposed by any jk_draft_expand call, in
 * generation order (layer, frontier slot, branch, rank).  Arrays are [B, *] with
 * `stride_b` elements between sequences; jk_draft_expand fills entries
 * gidx_base .. gidx_base + F*K*k_e - 1 of each sequence. */
typedef struct {
  int32_t* tok;             /* token id                                                  */
  float* score;             /* cumulative log-probability from the root                  */
  int32_t* parent;          /* generation index of the parent, -1 = root                 */
  int32_t* qslot;           /* row of the stored draft logits if the node was expanded, else -1 */
  int32_t* branch;          /* 0 = left (larger router score), 1 = right, ...            */
  int64_t stride_b;
} jk_pool;

/*
 * One draft layer for F frontier nodes per sequence (Sec. 3.1.2).
 *   x = RMSNorm(u) * norm_weight; s = softmax_N(x E^T) (Eq. 2); the K largest s keep their
 *   value as gates, larger one first = left (Eq. 5); y_r = Expert_{j_r}(x);
 *   f = sum_r g_r y_r + u (Eq. 3); branch feature b_r = g_r y_r (+ u);
 *   logits_r = b_r W_head^T (Eq. 4); per branch the k_e largest logits (ties: lower id)
 *   become children with score = parent_score + logit - logsumexp(logits_r); the W best
 *   children of the layer (ties: lower index) form the next frontier.
 * Inputs
 *   u            T   [B, F, H]   hidden state of each frontier node after draft attention (Eq. 1)
 *   parent_score f32 [B, F]      cumulative score of each frontier node (0 for the root)
 *   parent_gidx  i32 [B, F]      generation index of each frontier node (-1 for the root)
 *   gidx_base    generation index of this call's first child; slot_base: row index of this
 *                call's first node among all expanded nodes of the step (root = 0)
 * Outputs (any marked "opt" may be NULL)
 *   out_probs    f32 [B, F, N]   router scores s (opt)
 *   out_expert   i32 [B, F, K]   selected experts, left first
 *   out_gate     f32 [B, F, K]
 *   pool         children appended as described at jk_pool; qslot is set for the children
 *                chosen as next frontier (slot_base + F + position), -1 for the others
 *   out_lse      f32 [B, F, K]   logsumexp of each logits row (opt); laid out like out_logits:
 *                with logits_stride_b given, sequences are logits_stride_b / V elements apart,
 *                so that a call writes rows slot_base.. of a [B, S, K] array
 *   out_feat     T   [B, F, H]   combined feature f (Eq. 3)
 *   out_logits   f32 [B, F, K, V] (opt; needed later for sampling acceptance), with
 *                logits_stride_b elements between sequences (0 = dense, F*K*V), so that a call
 *                can write rows slot_base..slot_base+F-1 of a [B, S, K, V] buffer directly
 *   next_frontier      i32 [B, W'] flat child index (f*K + r)*k_e + j of the chosen children,
 *                      best first, W' = min(width, F*K*k_e) (opt, with the two arrays below);
 *                      width = 0 skips the selection (last layer)
 *   next_parent_score  f32 [B, W'] their scores
 *   next_parent_gidx   i32 [B, W'] their generation indices
 * Static tree policy (Sec. 3.1.2, last paragraph: the predefined tree of Eagle-1 is as usable as
 * the dynamic one): with static_select != NULL the next frontier is not chosen by score but
 * read from static_select, i32 [width] device, the flat child indices of the predefined shape in
 * frontier order, the same for every sequence; an index outside 0 .. F*K*k_e-1 sets JK_ERR_BOUNDS.
 * Contrastive mode (cfg.head_mode = 1; Sec. 3.2, Eq. 6-8): the head inputs are
 *   row 0: f^moe = g_1 y_1 + g_2 y_2 (+ u), row 1: f^const = beta y_1 - alpha y_2 (+ u).
 * The k_e best tokens of row 0 are the node's children as above.  Row 1 is the parallel-decoding
 * head: its k_e best tokens hang one level lower, under the node's best row-0 child (their pool
 * parent is that child's generation index, their score its score plus their log-probability
 * under row 1); they count only in a step's last pass (width = 0), get the score -inf in the
 * others, and are never chosen for the next frontier, so W' = min(width, F*k_e).  A step of tree
 * depth D then takes D-1 calls.
 * Errors: NULL/ALIGN/SHAPE/CAPACITY (B > max_batch, F > max_frontier)/WORKSPACE/CUDA.
 */
int jk_draft_expand(jk_ctx* ctx, void* stream, const jk_draft_weights* host_w,
                    int32_t batch, int32_t n_frontier, int32_t width,
                    const void* u, const float* parent_score, const int32_t* parent_gidx,
                    int32_t gidx_base, int32_t slot_base,
                    float* out_probs, int32_t* out_expert, float* out_gate,
                    const jk_pool* host_pool, float* out_lse, void* out_feat, float* out_logits,
                    int64_t logits_stride_b, int32_t* next_frontier, float* next_parent_score,
                    int32_t* next_parent_gidx, const int32_t* static_select);

/* Weights of the draft layer in front of the MoE (Sec. 3.1.1, 3.1.2): device pointers, read-only,
 * output-major. */
typedef struct {
  const void* emb;          /* T [V, H]      token embedding, shared with the target model      */
  const void* w_fc;         /* T [H, 2H]     reduction layer, acts on [emb(tok) ; parent feature] */
  const void* b_fc;         /* T [H] or NULL                                                     */
  const void* w_qkv;        /* T [(Hq + 2 Hkv) d, H]  rows of W_q, then W_k, then W_v           */
  const void* w_o;          /* T [H, Hq d]                                                       */
} jk_pre_weights;

/* State of the draft layer's attention over one step, caller-owned device memory: one entry per
 * expanded node ("slot": root = 0, then the frontier nodes of every pass in order), S_max =
 * stride_b slots per sequence. */
typedef struct {
  void* q;                  /* T   [B, S_max, Hq, d]  rotated query of every expanded node        */
  int32_t* slot_parent;     /* i32 [B, S_max]         parent slot, -1 for the root                */
  int32_t* slot_depth;      /* i32 [B, S_max]                                                     */
  int64_t stride_b;         /* S_max                                                              */
} jk_pre_state;

/*
 * The draft layer before the MoE for the F frontier nodes of one pass (Sec. 3.1.2, Eq. 1 and the
 * paragraph before it):
 *   h = W_fc [emb(tok) ; f_prev] (+ b_fc), with f_prev the feature f (Eq. 3, out_feat of
 *   jk_draft_expand) of the node's parent - for the root the target model's last feature;
 *   q, k, v = W_qkv h, q and k rotated (rotary positions, LLaMA pairing (i, i + d/2), base
 *   rope_theta) to position kv_len[b] + depth; k and v are appended to the draft layer's own
 *   cache at row kv_len[b] + slot; every node attends over rows 0 .. kv_len[b]-1 and the rows of
 *   itself and its ancestors; u = W_o Attn + h (Eq. 1).
 * No normalisation is applied in this block (Eq. 1-5 leave the norms out; Eagle-style drafts drop
 * the input norm of their single layer).  out_u feeds jk_draft_expand of the same pass.
 *   slot_base    slot of this pass's first node (0 for the root pass, then the running count)
 *   node_gidx    i32 [B, F] generation index of each node = next_parent_gidx of the previous
 *                jk_draft_expand; NULL in the root pass (then F = 1, the token is root_tok[b]
 *                and prev_feat is T [B, H])
 *   pool         the step's candidate pool: the nodes' tokens are pool.tok[node_gidx]
 *   prev_gidx_base, prev_slot_base, prev_frontier   gidx_base, slot_base and F of the previous
 *                pass; prev_feat T [B, prev_frontier, H] its out_feat.  A node's parent is
 *                frontier row (node_gidx - prev_gidx_base) / (K k_e) of that pass.
 *   k_cache, v_cache  T [B, Hkv, cap, d] with strides as in jk_tree_verify_attn; rows
 *                kv_len[b] .. kv_len[b] + slot_base + F - 1 are written over the passes
 *   out_u        T [B, F, H]
 * The attention runs over all slot_base + F nodes expanded so far (their queries are kept in
 * state.q), so slot_base + F <= 128 and <= max_depth * max_frontier.
 * Errors: NULL/ALIGN/SHAPE/CAPACITY/WORKSPACE/CUDA; a token or index out of range, or a cache too
 * short, sets JK_ERR_BOUNDS in the status word.
 */
int jk_draft_pre(jk_ctx* ctx, void* stream, const jk_pre_weights* host_w,
                 const jk_pre_state* host_state, int32_t batch, int32_t n_frontier,
                 int32_t slot_base, const int32_t* node_gidx, const jk_pool* host_pool,
                 int32_t prev_gidx_base, int32_t prev_slot_base, int32_t prev_frontier,
                 const void* prev_feat, const int32_t* root_tok, void* k_cache, void* v_cache,
                 int64_t cache_stride_b, int64_t cache_stride_h, int32_t cache_rows,
                 const int32_t* kv_len, float rope_theta, float softmax_scale, void* out_u);

/*
 * The target layer's own steps in front of jk_tree_verify_attn in a verification pass (Sec. 2.1
 * step 2: the target model evaluates all tree tokens in one forward pass): QKV projection of the
 * M tree tokens, rotary positions, K/V written at the tree slots.
 *   x        T [B, M, H]   the layer's (normalised) input hidden states of the tree tokens
 *   w_qkv    T [(Hq + 2 Hkv) d, H]   rows of W_q, then W_k, then W_v
 *   depth    i32 [B, M]    as written by jk_tree_finalize: node i sits at position kv_len[b] +
 *            depth[i] (nodes of one depth are alternatives for the same place in the sequence)
 *   q_out    T [B, M, Hq, d]   rotated queries (LLaMA pairing (i, i + d/2), base rope_theta)
 *   k_cache, v_cache   rotated K and V of node i go to row kv_len[b] + i
 * More than 256 tree tokens per call (B * M) go through the projection in chunks of 256 rows,
 * each streaming W_qkv once.  Errors as jk_tree_verify_attn; kv_len[b] + M > cache_rows sets
 * JK_ERR_BOUNDS.
 */
int jk_verify_qkv(jk_ctx* ctx, void* stream, const void* w_qkv, int32_t batch, int32_t tree_size,
                  const void* x, const int32_t* depth, void* q_out, void* k_cache, void* v_cache,
                  int64_t cache_stride_b, int64_t cache_stride_h, int32_t cache_rows,
                  const int32_t* kv_len, float rope_theta);

/*
 * The hidden states the next draft round starts from (Sec. 2.1 step 3 keeps the accepted path):
 *   out[b, 0] = hidden[b, 0] (the root), out[b, 1 + j] = hidden[b, acc_idx[b, j]] for
 *   j < n_acc[b]; rows after the accepted path are zero.
 *   hidden T [B, M, H]; n_acc i32 [B], acc_idx i32 [B, max_depth] as written by
 *   jk_accept_and_compact; out T [B, rows_out, H], rows_out <= max_depth + 1.
 */
int jk_gather_accepted(jk_ctx* ctx, void* stream, int32_t batch, int32_t tree_size,
                       const void* hidden, const int32_t* n_acc, const int32_t* acc_idx,
                       int32_t rows_out, void* out);

/*
 * Build the verification tree from the pool (Sec. 3.1.2; mask as in Fig. 4): node 0 is the
 * root (root_tok[b]); nodes 1..M-1 are the M-1 best pool entries by (score descending,
 * generation index ascending), listed in ascending generation index, so parent[i] < i.
 *   pool_n <= 4096 entries per sequence; tree_size = M <= max_tree, pool_n >= M-1.
 *   root_tok i32 [B]; outputs i32 [B, M]: tok, parent (-1 for the root), depth, branch, qslot
 *   (root: 0); anc u64 [B, M, 2]: bit t of the 128-bit set is 1 iff t is the node itself or
 *   one of its ancestors.
 *   static_keep  i32 [M-1] device or NULL.  Static tree policy: the generation indices of the
 *   predefined shape's nodes, ascending, the same for every sequence, kept instead of the M-1
 *   best by score; a list that is not ascending, reaches past pool_n or keeps a node without
 *   its parent sets JK_ERR_BOUNDS.
 */
int jk_tree_finalize(jk_ctx* ctx, void* stream, int32_t batch, const jk_pool* host_pool,
                     int32_t pool_n, const int32_t* root_tok, int32_t tree_size,
                     int32_t* tok, int32_t* parent, int32_t* depth, int32_t* branch,
                     int32_t* qslot, uint64_t* anc, const int32_t* static_keep);

/*
 * Tree-masked attention of one target layer over all M tree tokens (Sec. 2.1 step 2):
 *   out[b,i,h] = sum_c softmax_c(softmax_scale * q[b,i,h] . K[b,h/G,c] + mask) V[b,h/G,c],
 *   c < kv_len[b] + M, G = Hq/Hkv; column c is visible to node i iff c < kv_len[b] or
 *   c - kv_len[b] is i or an ancestor of i.
 *   q, out       T [B, M, Hq, d]
 *   k_cache, v_cache  T [B, Hkv, cap, d] addressed with cache_stride_b / cache_stride_h
 *                (elements); rows 0..kv_len[b]-1 hold the committed prefix, the caller has
 *                written the tree tokens' K/V at rows kv_len[b] .. kv_len[b]+M-1
 *   kv_len       i32 [B]; parent i32 [B, M] with parent[i] < i, -1 for the root
 *   cache_rows   rows addressable in each cache (cap); kv_len[b] + M > cap sets JK_ERR_BOUNDS
 */
int jk_tree_verify_attn(jk_ctx* ctx, void* stream, int32_t batch, int32_t tree_size,
                        const void* q, const void* k_cache, const void* v_cache,
                        int64_t cache_stride_b, int64_t cache_stride_h, int32_t cache_rows,
                        const int32_t* kv_len, const int32_t* parent, float softmax_scale,
                        void* out);

/*
 * jk_tree_verify_attn for callers that cannot allocate device memory.  (The paper has no
 * counterpart: this is a packaging variant of the call above.  It computes the same operation
 * with the CUDA-core kernel for both dtypes - fp32 products and an fp32 softmax - where
 * jk_tree_verify_attn uses the tensor-core kernels for bf16, which round the softmax weights to
 * bf16 and run several times faster; the two agree within the bf16 tolerance, not bit for bit.)
 *
 * Meant for processes that have given all free HBM to their own pools at start-up, so that a
 * later cudaMalloc for a workspace fails, and for decode loops that cannot afford the
 * device-wide synchronisation of cudaMalloc/cudaFree.  It needs no jk_set_workspace: the split-KV
 * partials go to a fixed 8 MiB (+256 B) array compiled into the library, which every GPU that
 * loads the library holds until the process exits.  The call makes no cudaMalloc/cudaFree and
 * uses no allocating library routine.
 *
 *   Arguments as jk_tree_verify_attn, plus
 *   status   i32 [1] device, required (NULL returns JK_ERR_NULL): receives JK_ERR_BOUNDS if
 *            kv_len[b] + M > cache_rows, in which case `out` is not written.  It is set by an
 *            atomic compare-and-swap on 0, so the caller clears it before the call and reads it
 *            after synchronising the stream.
 *   Limit    batch * tree_size * n_q_heads * (head_dim + 2) * 4 bytes <= 8 MiB (e.g. 60 nodes x
 *            32 heads x 128 uses 1 MiB per key slice); beyond it the call returns
 *            JK_ERR_CAPACITY, launches nothing, and jk_last_cuda_error(ctx) says why.
 *   Set-up   the first call on each device (with that device current) looks up the array's
 *            device address; make that first call before starting any stream capture.
 *   Sharing  all contexts, streams and threads of the process share the one array per GPU, and
 *            it keeps the previous call's contents.  Nothing in it has to start at zero (every
 *            partial a call reads it has written itself); but two of these calls that overlap
 *            on the same GPU race on the partials and give wrong results: run them one after
 *            the other.
 */
int jk_tree_verify_attn_static(jk_ctx* ctx, void* stream, int32_t batch, int32_t tree_size,
                               const void* q, const void* k_cache, const void* v_cache,
                               int64_t cache_stride_b, int64_t cache_stride_h, int32_t cache_rows,
                               const int32_t* kv_len, const int32_t* parent, float softmax_scale,
                               void* out, int32_t* status);

/*
 * Acceptance walk and KV compaction (Sec. 2.1 steps 2-3).
 *   mode 0 (greedy): from the root, follow the first child whose token equals the target's
 *     top-1 token (ties: lower id) at the current node; stop when none does; the bonus token
 *     is the top-1 at the stop node.
 *   mode 1 (sampling, temperature > 0): p = softmax(target/T) at the current node, q_r =
 *     softmax(draft/T) of branch r; children in order: accept iff u_accept[c] <
 *     min(1, p[x]/q_r[x]); on rejection p <- norm(max(0, p - q_r)), q_r[x] <- 0 and q_r is
 *     renormalised; if no child is accepted the bonus token is the inverse-CDF draw from p with
 *     u_bonus[depth].
 *   Then, for every layer l < n_layers and both caches, row kv_len+acc_idx[j] moves to row
 *   kv_len+1+j (j < n_acc) and kv_len[b] becomes kv_len[b] + 1 + n_acc[b].
 *   target_logits  [B, M, V] of tl_dtype (f32 or bf16)
 *   tok, parent, depth, branch, qslot   i32 [B, M] as written by jk_tree_finalize
 *   draft_logits   f32 [B, S, K, V], S = n_slots (mode 1; NULL in mode 0)
 *   u_accept       f32 [B, M], u_bonus f32 [B, max_depth+1], uniform in [0,1) (mode 1)
 *   k_caches, v_caches   device arrays of n_layers device pointers (may be NULL if n_layers = 0)
 *   outputs: n_acc i32 [B], acc_idx i32 [B, max_depth], acc_tok i32 [B, max_depth] (entries
 *   past n_acc are -1), bonus_tok i32 [B]
 */
int jk_accept_and_compact(jk_ctx* ctx, void* stream, int32_t batch, int32_t tree_size,
                          int32_t mode, float temperature,
                          const void* target_logits, int32_t tl_dtype,
                          const int32_t* tok, const int32_t* parent, const int32_t* depth,
                          const int32_t* branch, const int32_t* qslot,
                          const float* draft_logits, int32_t n_slots,
                          const float* u_accept, const float* u_bonus,
                          int32_t n_layers, void* const* k_caches, void* const* v_caches,
                          int64_t cache_stride_b, int64_t cache_stride_h, int32_t cache_rows,
                          int32_t* kv_len, int32_t* n_acc, int32_t* acc_idx, int32_t* acc_tok,
                          int32_t* bonus_tok);

/* ------------------------------------------------------------------------------------------
 * Paged 8-bit KV cache.  (The paper has no counterpart: it keeps one 16-bit cache per sequence.
 * These calls are for servers that verify many or long sequences: the same step over a cache of
 * half the bytes, in pages that sequences can share.)
 *
 * A page holds page_size consecutive tokens of one sequence, for all kv heads of a layer, as
 * 8-bit floats (e4m3: 4 significant bits) with one scale per (page, kv head) for K and one for
 * V.  The scale is a power of two, the smallest s >= 2^-32 with max|x| <= 448 s over the block's
 * finite values, so that x / s and s * code are exact and a value is rounded once, to code =
 * e4m3(x / s), ties to even; values under 2^-42 become 0, infinities the largest code, NaN stays
 * NaN.  Page ids are the same in all layers.  Only full pages are 8-bit, and a full page is
 * never written again: forked sequences share pages by reference count and nothing is copied on
 * write.  The last kv_len % page_size tokens of a sequence, its open page, stay in T; token
 * position c is row c mod (2 page_size) of the sequence's open rows, so that a call that
 * completes a page never overwrites what the page is made from.  The step's tree tokens stay
 * outside the cache, in T, until jk_paged_commit takes the accepted ones in.
 *
 * All arrays are the caller's.  Pages are taken from the end of free_list
 * (free_list[n_free - 1] first) in the order (sequence, page), so results repeat bit for bit.
 * The calls that change a cache check what they are given and the rows that it names first, and
 * then change all or nothing: on an index out of range, a row that does not fit or a page that
 * others share they set JK_ERR_BOUNDS in the status word of the context, and JK_ERR_CAPACITY when
 * the free pages do not suffice; the cache is then as it was and the call can be repeated.  Calls
 * on one cache must not overlap on the device unless all of them are jk_tree_verify_attn_paged.
 * Attention, jk_verify_qkv_tree and jk_paged_commit work on the rows 0 .. batch - 1: a sequence
 * gets to another row by jk_paged_fork and jk_paged_free.
 * ------------------------------------------------------------------------------------------ */
typedef struct {
  int32_t n_layers;         /* L                                                             */
  int32_t n_pages;          /* pages in the pool (per layer)                                 */
  int32_t page_size;        /* tokens per page: 16, 32, 64 or 128                            */
  int32_t max_seqs;         /* sequences (rows of page_table), <= 1024                       */
  int32_t max_pages;        /* pages a sequence can hold (columns of page_table)             */
  void* k_pages;            /* e4m3 [L, n_pages, Hkv, page_size, d]                          */
  void* v_pages;
  float* k_scale;           /* f32 [L, n_pages, Hkv]                                         */
  float* v_scale;
  void* k_open;             /* T [L, max_seqs, Hkv, 2 page_size, d]                          */
  void* v_open;
  int32_t* kv_len;          /* i32 [max_seqs] committed tokens                               */
  int32_t* page_table;      /* i32 [max_seqs, max_pages], -1 = none                          */
  int32_t* refcount;        /* i32 [n_pages] sequences that hold the page                    */
  int32_t* free_list;       /* i32 [n_pages], the first n_free entries count                 */
  int32_t* n_free;          /* i32 [1]                                                       */
  int32_t* scratch;         /* i32 [jk_paged_scratch_ints(n_pages)]                            */
} jk_paged;

/* int32 entries of jk_paged.scratch (0 for n_pages outside 1 .. 2^24). */
int64_t jk_paged_scratch_ints(int32_t n_pages);

/* An empty cache: no sequence has tokens or pages, the free list hands out pages 0, 1, 2, ... */
int jk_paged_init(jk_ctx* ctx, void* stream, const jk_paged* host_cache);

/*
 * Take prompts into the cache: for i < batch, tokens 0 .. n_tokens[i]-1 of source sequence i become
 * sequence seqs[i] (seqs = NULL: i) of the layers first_layer .. first_layer + n_layers - 1; full
 * pages are quantised, the rest goes to the open rows, kv_len is set.  Pages are taken once: a row
 * that holds unshared pages (an earlier layer's call) keeps them.  A row that holds shared pages,
 * or more pages than the prompt fills, and a sequence named twice set JK_ERR_BOUNDS.
 *   n_tokens i32 [batch], 0 <= n_tokens <= src_rows
 *   k_src, v_src  device arrays of n_layers device pointers to T [batch, Hkv, src_rows, d] with the
 *                 strides given (elements)
 */
int jk_paged_import(jk_ctx* ctx, void* stream, const jk_paged* host_cache, int32_t batch,
                  const int32_t* seqs, const int32_t* n_tokens, int32_t first_layer,
                  int32_t n_layers, void* const* k_src, void* const* v_src, int64_t src_stride_b,
                  int64_t src_stride_h, int32_t src_rows);

/*
 * Tree-masked attention of one target layer over the paged cache: jk_tree_verify_attn with, for
 * sequence b, columns c < kv_len[b] read from its pages and open rows and column kv_len[b] + i from
 * row i of the tree arrays.  tree_size = 1 with parent = -1 is ordinary decoding of one token.
 *   q, out   T [B, M, Hq, d];  parent i32 [B, M], parent[i] < i, -1 for the root
 *   k_tree, v_tree  T [B, Hkv, >= M, d] with the strides given (elements): this layer's keys and
 *            values of the tree tokens; they have to be finite
 *   out must not overlap the inputs
 * kv_len[b] < 0 or past max_pages * page_size, and a page id outside the pool, set JK_ERR_BOUNDS.
 * With bf16 and the tensor path, queries meet the pages' keys in two e4m3 parts (a value is off
 * by at most 2^-13 of the largest in its row, whatever the other rows hold) and softmax weights
 * are rounded once, to fp16 over pages and to bf16 over open and tree rows; sums are fp32.  One query row per kv head, fp32 contexts and the CUDA-core
 * path carry everything in fp32.
 */
int jk_tree_verify_attn_paged(jk_ctx* ctx, void* stream, const jk_paged* host_cache, int32_t layer,
                            int32_t batch, int32_t tree_size, const void* q, const void* k_tree,
                            const void* v_tree, int64_t tree_stride_b, int64_t tree_stride_h,
                            const int32_t* parent, float softmax_scale, void* out);

/*
 * jk_verify_qkv for a paged cache: the rotated K and V of node i go to row i of k_tree, v_tree
 * (T [B, Hkv, >= M, d]); positions are kv_len[b] + depth[i] with kv_len as given (jk_paged.kv_len).
 */
int jk_verify_qkv_tree(jk_ctx* ctx, void* stream, const void* w_qkv, int32_t batch,
                       int32_t tree_size, const void* x, const int32_t* depth, void* q_out,
                       void* k_tree, void* v_tree, int64_t tree_stride_b, int64_t tree_stride_h,
                       const int32_t* kv_len, float rope_theta);

/*
 * After jk_accept_and_compact (called with n_layers = 0, kv_len = jk_paged.kv_len and cache_rows =
 * max_pages * page_size): the root and the accepted nodes of every sequence b < batch join the
 * cache, all layers.  kv_len[b] already counts them (1 + n_acc[b]); n_acc[b] < 0 skips a sequence.
 * Pages this completes are taken from the free list, unless the row holds an unshared page there
 * already, and quantised.  Repeating the call changes nothing.
 *   k_tree, v_tree  device arrays of L device pointers to T [B, Hkv, >= M, d], strides in elements
 *   n_acc i32 [B], acc_idx i32 [B, max_depth] as written by jk_accept_and_compact
 */
int jk_paged_commit(jk_ctx* ctx, void* stream, const jk_paged* host_cache, int32_t batch,
                  int32_t tree_size, void* const* k_tree, void* const* v_tree,
                  int64_t tree_stride_b, int64_t tree_stride_h, const int32_t* n_acc,
                  const int32_t* acc_idx);

/* Fork: sequence dst[i] becomes a copy of sequence src[i], i < n: it shares the full pages and
 * gets its own open rows.  Each dst[i] has to be empty, named once and no src. */
int jk_paged_fork(jk_ctx* ctx, void* stream, const jk_paged* host_cache, int32_t n, const int32_t* src,
                const int32_t* dst);
/* Free the sequences seqs[i], i < n, each named once (an empty one is allowed): kv_len 0, no
 * pages.  Pages that no sequence holds any more are appended to the free list in ascending order. */
int jk_paged_free(jk_ctx* ctx, void* stream, const jk_paged* host_cache, int32_t n, const int32_t* seqs);
/* Pack the pool: with n_live pages in use, the i-th unused id below n_live takes over the i-th
 * used page at or above it (data of all layers, reference count, table entries); afterwards the
 * free list hands out n_live, n_live + 1, ...  n_moved i32 [1] (opt) receives the pages moved.
 * It names no sequence and refuses nothing: the reference counts are taken as they are. */
int jk_paged_compact(jk_ctx* ctx, void* stream, const jk_paged* host_cache, int32_t* n_moved);
/* Copy page src_ids[i] of host_src to page dst_ids[i] of host_dst, i < n, codes and scales of all
 * layers; the two pools agree in L, page_size, Hkv and d and may be the same, but not overlap in
 * part (JK_ERR_SHAPE).  No bookkeeping is touched.  A dst id named twice, or (same pool) also named as a source, sets JK_ERR_BOUNDS and
 * nothing is copied. */
int jk_paged_copy(jk_ctx* ctx, void* stream, const jk_paged* host_src, const jk_paged* host_dst,
                      int32_t n, const int32_t* src_ids, const int32_t* dst_ids);

/*
 * Sampling with temperature, top-k, top-p and min-p from given random numbers, per row of logits:
 * the draw of a next token, and the filtered target rows that jk_accept_and_compact (mode 1,
 * temperature 1) takes as target_logits.
 *   Tokens are ordered by (logit descending, index ascending).  Weights w = exp((z - z_max) / T) are
 *   formed in double precision and summed as 64-bit fixed-point numbers, unit 2^-45 (2^(n-62) for
 *   2^n > 2^17 tokens): a vocabulary of 1e5 has cumulative sums 1e-5 apart, where fp32 sums are off
 *   by 1e-6.  The kept set is the shortest of three prefixes of the order,
 *   never empty:
 *     top_k > 0:    the first top_k tokens
 *     top_p < 1:    the tokens before which less than top_p of the weight of the first top_k lies
 *     min_p > 0:    the tokens with z - z_max >= T ln(min_p), i.e. w >= min_p
 *   The token drawn is the first kept one, in index order, whose cumulative weight exceeds u times
 *   the kept weight.  T not above 0 keeps the first token alone (greedy).
 *   NaN counts as -inf, +inf as the largest float.  A row of nothing but -inf gives token -1.
 *   logits       f32 or bf16 (logits_dtype) [rows, V], row_stride elements between rows (>= V);
 *                aligned to its element (16-byte alignment of pointer and rows is faster)
 *   temperature, top_p, min_p  f32 [rows], top_k i32 [rows]; each may be NULL (1, 1, 0, 0 = off)
 *   u            f32 [rows] in [0, 1); may be NULL when out_tok is
 *   out_tok      i32 [rows] (opt)
 *   out_logits   f32 [rows, V], dense (opt): z / T for kept tokens (0 for a greedy row's), -inf for
 *                the others.  Must not overlap logits (JK_ERR_SHAPE).  At least one of the two outputs has to be given.
 */
int jk_sample(jk_ctx* ctx, void* stream, int32_t rows, const void* logits, int32_t logits_dtype,
              int64_t row_stride, const float* temperature, const int32_t* top_k,
              const float* top_p, const float* min_p, const float* u, int32_t* out_tok,
              float* out_logits);

/* ------------------------------------------------------------------------------------------
 * The rest of a target layer.  (The paper has no counterpart: it takes the target model's forward
 * pass as given.)  With jk_tree_verify_attn or jk_tree_verify_attn_paged between them these calls
 * are a whole layer, for the nodes of a tree, for single tokens and for a prompt's rows alike:
 *   add_norm -> linear (qkv) -> rope_qkv -> attention -> linear (output projection + residual) ->
 *   add_norm -> linear (gated) -> linear (down + residual).
 * jk_tree_verify_attn may read kv_len and committed rows of its caches while the call before it ends: of the
 * calls here only jk_rope_qkv writes what it may take as committed right behind.
 *
 * 8-bit rows ("mx8"): an array [rows, n], n a multiple of 32, as e4m3 codes, u8 [rows, n] dense, and
 * one power-of-two scale for each block of 32 consecutive elements of a row: the smallest
 * s >= 2^-32 with max|x| <= 448 s over the block's finite values, so that x / s is exact and a
 * value is rounded once, to code = e4m3(x / s), ties to even.  Values under 2^-42 become 0,
 * infinities the largest code, NaN stays NaN.  A scale is stored as the byte log2(s) + 127, in
 * tiles of 128 rows x 4 blocks, the order in which the tensor cores take them: row r, block k
 * lies at byte (r/128 * ceil(n/128) + k/4) * 512 + r%32 * 16 + r%128/32 * 4 + k%4.  Bytes of the
 * tiles that belong to no row or block are neither written nor do they reach a result.  (Arrays made
 * elsewhere may hold any scale byte from 1 to 254.)
 * ------------------------------------------------------------------------------------------ */

/* Bytes of the scale tiles of an mx8 array: ceil(rows/128) * ceil(n/128) * 512 (0 for sizes out of
 * range: rows 1 .. 2^24, n a multiple of 32 up to 2^20). */
int64_t jk_row_scale_bytes(int64_t rows, int64_t n);

/* x T [rows, n] (x_stride elements between rows, 0 = n) to mx8: weights once, activations that no
 * other call hands out in 8 bits.  16-byte aligned rows.  rows <= 2^24. */
int jk_quantize_rows(jk_ctx* ctx, void* stream, int64_t rows, int32_t n, const void* x,
                    int64_t x_stride, void* out, uint8_t* out_scale);

/*
 * RMS norm with the residual's addition, per row:
 *   s = x + delta;  y = s / sqrt(mean(s^2) + rms_eps) * weight      (rms_eps of the context, f32)
 *   x, delta     T [rows, n], dense; delta may be NULL (s = x)
 *   weight       T [n] or NULL (= ones)
 *   out_sum      T [rows, n] (opt): s, the new residual stream; may be x or delta itself
 *   out          T [rows, n] (opt): y; may be x or delta itself
 *   out_mx8, out_scale  (opt, together): y as mx8, rounded from the f32 value, not from out
 * At least one output.  The norm is that of the f32 sum, not of the rounded one.  n a multiple of 8
 * (of 32 with mx8) up to 32768, rows up to 2^24.  Outputs must not overlap one another, nor an input in part.
 */
int jk_add_norm(jk_ctx* ctx, void* stream, int32_t rows, int32_t n, const void* x, const void* delta,
                const void* weight, void* out_sum, void* out, void* out_mx8, uint8_t* out_scale);

typedef enum { JK_ACT_NONE = 0, JK_ACT_SILU = 1, JK_ACT_GELU = 2 } jk_act;   /* GELU: z Phi(z), by erf */
typedef enum { JK_ROWS_T = 0, JK_ROWS_F32 = 1, JK_ROWS_MX8 = 2 } jk_rows_type;

/* A projection: weights of the target model, device pointers, read-only, output-major. */
typedef struct {
  int32_t n_out, n_in;      /* weights [n_out, n_in]                                          */
  int32_t operands;         /* JK_ROWS_T: w and x are T; JK_ROWS_MX8: both are mx8            */
  int32_t act;              /* jk_act                                                         */
  const void* w;
  const uint8_t* w_scale;   /* scale tiles of w (mx8)                                         */
  const void* bias;         /* T [n_out] or NULL                                              */
  const void* w_up;         /* second weights [n_out, n_in] of a gated block, or NULL         */
  const uint8_t* w_up_scale;
  const void* bias_up;      /* T [n_out] or NULL                                              */
} jk_linear_op;

/*
 * Matrix product with its epilogue, gated or not, in one kernel:
 *   z = x w^T + bias;  y = act(z) [* (x w_up^T + bias_up)] [+ residual]
 *   x            [rows, n_in]: T with x_stride elements between rows (0 = n_in), or mx8 (dense, with
 *                x_scale)
 *   residual     T [rows, n_out] or NULL, residual_stride elements between rows (0 = n_out)
 *   out          [rows, n_out] as out_type says: T or f32 with out_stride elements between rows
 *                (0 = n_out), or mx8 (dense, with out_scale; n_out a multiple of 32)
 * n_in is a multiple of 8 (T) or 32 (mx8) up to 131072, n_out any number up to 2^20, rows up to
 * 2^20; rows of x are 16-byte aligned.  Products are exact and summed in f32 (f32 contexts: f32
 * multiply-adds), the epilogue is f32, y is rounded once.  SiLU and GELU: within a few units of f32 on CUDA
 * cores; on the tensor cores within 2^-18 of their value, which f32 outputs show (GELU of 16- and 8-bit
 * outputs: 2^-16).  out may be residual itself (same
 * stride), or columns of one buffer of which x and residual are others; any overlap of out with an
 * input is refused (JK_ERR_SHAPE).  bf16 contexts and mx8 operands run on the tensor cores while the
 * tensor path is on (mx8: in bf16 contexts).  After JK_ERR_TIMEOUT in the status, set the workspace
 * again before the next call.
 */
int jk_linear(jk_ctx* ctx, void* stream, const jk_linear_op* host_op, int32_t rows, const void* x,
              const uint8_t* x_scale, int64_t x_stride, const void* residual, int64_t residual_stride,
              void* out, int32_t out_type, uint8_t* out_scale, int64_t out_stride);

/*
 * Rotary positions with one or several axes (time, height, width of images and video), and the place
 * of K and V: what lies between a qkv projection and the attention.
 *   qkv          T [batch, n_tokens, (Hq + 2 Hkv) d] rows of q, then k, then v heads, row_stride
 *                elements between tokens (0 = dense, a multiple of 16 bytes)
 *   pos          i32 [batch, n_tokens, n_axes], each >= 0
 *   host_sections  n_axes counts with the sum d/2: the first host_sections[0] of the d/2 frequencies
 *                turn with axis 0, the next with axis 1, ...  n_axes 1 .. 4
 *   Pair (i, i + d/2) of every q and k head turns by pos[axis of i] * rope_theta^(-2i/d); angles are
 *   formed and reduced in 64 bits.
 *   q_out        T [batch, n_tokens, Hq, d]
 *   k_out, v_out T [batch, Hkv, >= rows, d] with the strides given (elements): token i goes to row
 *                first_row[b] + i (first_row i32 [batch], e.g. kv_len; NULL = 0)
 *   rows         rows addressable in k_out, v_out; first_row[b] < 0, first_row[b] + n_tokens > rows
 *                or a negative position sets JK_ERR_BOUNDS, and that sequence's K and V (that
 *                token) are not written.
 * n_tokens up to 2^20, not bound to max_tree; batch up to 65535, not bound to max_batch.  Outputs
 * must not overlap qkv, nor one another (JK_ERR_SHAPE); K and V may be parts of one buffer whose pieces of
 * rows x d lie between one another.
 */
int jk_rope_qkv(jk_ctx* ctx, void* stream, int32_t batch, int32_t n_tokens, const void* qkv,
                int64_t row_stride, const int32_t* pos, int32_t n_axes, const int32_t* host_sections,
                float rope_theta, void* q_out, void* k_out, void* v_out, int64_t stride_b,
                int64_t stride_h, int32_t rows, const int32_t* first_row);

#ifdef __cplusplus
}
#endif
#endif /* JAKIRO_H_ */
