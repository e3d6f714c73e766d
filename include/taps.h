/* taps.h -- C ABI of the TAPS draft-tree verification hot path on MI355X (gfx950).
 *
 * One decoding round of TAPS (Target-Aware Prefix Tree Selection, arXiv 2606.00487):
 *   taps_select       per-position top-K of the drafter marginals (Sec. 4.1, Stage 1),
 *                     sibling-softmax edge probabilities q_cond (Eq. 1), reach
 *                     probabilities q_reach (Eq. 2), utility (Eq. 3) and the greedy
 *                     budgeted prefix-closed selection of Alg. 1.
 *   tree_verify_attn  tree-masked verification attention: every selected node attends
 *                     to the cached context and to its own ancestors (Sec. 4.1 Stage 3,
 *                     Sec. 4.3: verification needs a connected subtree at the root).
 *                     tree_verify_attn_paged: the same over a paged KV cache.
 *   accept_walk       greedy (temperature 0) acceptance of the longest matching root
 *                     path (Sec. 1: one prefix path is committed per round; Limitations).
 *   kv_commit         the round's state update: the accepted path's tree K/V rows move
 *                     to the rows right after the context, and the emitted tokens
 *                     (kv_commit_paged: the same on a paged cache).
 *   verify_layer      one attention layer of the target over the tree: projections,
 *                     per-head RMSNorm, rotary positions by tree depth, tree attention,
 *                     output projection (the verification forward's layer slice).
 * Around the round, for serving over a paged cache (the Limitations leave cache management
 * and sampled decoding to the serving system):
 *   kv_reserve_paged  pages for the requests' next rows, block tables and slot maps
 *   kv_append_paged   new K/V rows into the pools through a slot map
 *   decode_attn_paged attention of one new token per request (a step without a draft)
 *   taps_sample       tokens from the target's logits at a temperature (the walk's targets)
 * Prompts, over the same cache (a request's context before its first round):
 *   qk_rope_paged     per-head norms and rotary positions of new queries and keys, cache write
 *   chunk_attn_paged  attention of chunks of new tokens
 *   taps_logprobs     log probabilities and ranks of given tokens, entropy, top alternatives
 *
 * Conventions shared by every call:
 *   - Pointers are DEVICE memory owned by the caller unless marked [host].
 *   - Calls validate their arguments on the host, then enqueue kernels on `stream`.
 *     They never synchronize, never allocate, and keep no state between calls.
 *   - Invalid arguments return an error before anything is enqueued.  A failed kernel
 *     launch returns TAPS_ERR_HIP.  Kernels never trap: pathological data (NaN, +-inf,
 *     empty rows) produces the defined outputs documented per call.
 *   - Workspace sizes are pure functions of the host-side sizes.  A workspace may be
 *     reused by consecutive calls on one stream; concurrent calls need their own.
 */
#ifndef TAPS_H
#define TAPS_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TAPS_OK = 0,
  TAPS_ERR_INVALID_ARG = -1,  /* null pointer, size out of range, misaligned buffer */
  TAPS_ERR_UNSUPPORTED = -2,  /* valid request this build does not implement      */
  TAPS_ERR_WORKSPACE = -3,    /* workspace missing or smaller than required        */
  TAPS_ERR_HIP = -4           /* a kernel launch failed (hipGetLastError)          */
} taps_status;

typedef enum { TAPS_BF16 = 0, TAPS_FP32 = 1 } taps_dtype;
typedef enum { TAPS_LOGITS = 0, TAPS_PROBS = 1 } taps_kind;
typedef enum {
  TAPS_SCORER_SIBLING = 0,
  TAPS_SCORER_MARGINAL = 1,
  TAPS_SCORER_LEARNED = 2
} taps_scorer;

/* Limits of this build. */
#define TAPS_MAX_BLOCK 32    /* draft positions D (tree depth)              */
#define TAPS_MAX_K 16        /* candidates per position                     */
#define TAPS_MAX_BUDGET 512  /* N_max, root included                        */

/* [host] Weights of the learned-scorer hook (Sec. 4.2, "Scorer design"): a per-edge MLP
 * whose trained weights are not published, so the caller brings its own.  DEVICE fp32
 * arrays owned by the caller:
 *   emb         [vocab][emb_dim] token embeddings
 *   W1          [hidden][2*emb_dim + 3] first layer over the edge features, in this
 *               order: parent token embedding, child token embedding, child depth,
 *               child log-probability, positional entropy of the child's row
 *   b1, w2      [hidden]; b2 the output bias
 *   root_token  [batch] int32 token at each request's current position (the root's
 *               token, the parent token of depth-1 children); outside [0, vocab): a
 *               zero embedding
 *   emb_dim     1..32;  hidden  1..64 */
typedef struct {
  const float *emb, *W1, *b1, *w2;
  float b2;
  const int32_t *root_token;
  int32_t emb_dim, hidden;
} taps_scorer_mlp;

/* [host] Selection parameters (Sec. 4.1 Stage 1 and 3; Eq. 3; Alg. 1).
 *   batch    requests B >= 0 (0: nothing is enqueued)
 *   block    draft positions D, 1..TAPS_MAX_BLOCK; row i of a request's marginals is the
 *            distribution of the token at tree depth i+1 (the root, depth 0, is the
 *            current position and carries no drafted token)
 *   vocab    V >= K
 *   K        candidates per position, 1..TAPS_MAX_K
 *   budget   N_max, 1..TAPS_MAX_BUDGET; the root counts toward it
 *   dtype    TAPS_BF16 or TAPS_FP32 marginals
 *   kind     TAPS_LOGITS: the edge logit of a child is beta * (its drafter logit);
 *            TAPS_PROBS: the marginals are probabilities, used as the sibling weights
 *            directly (beta must be 1)
 *   lambda1  > 0, finite: per-node cost in Eq. 3
 *   lambda2  >= 0, finite: per-depth cost in Eq. 3 (negative values: UNSUPPORTED)
 *   tau      minimum utility; a node is added only while its utility is > tau (not NaN)
 *   beta     >= 0, finite scorer temperature for LOGITS
 *   scorer   TAPS_SCORER_SIBLING (0; the default of a zeroed struct): q_cond is the
 *            sibling softmax over the K candidates, below.  TAPS_SCORER_MARGINAL: the
 *            scoring ablation of Sec. 5 (the scorer removed, selection by the drafter's
 *            marginal confidence): q_cond is the candidate's full-vocabulary marginal,
 *            below; LOGITS then needs beta = 1.  TAPS_SCORER_LEARNED: the learned
 *            scorer's MLP (mlp) gives each edge a logit, normalised over the parent's
 *            candidate children by a sibling softmax; LOGITS only; block * K * K must
 *            not exceed 7168 (its q_cond table lives in LDS)
 *   mlp      [host] weights, read only with TAPS_SCORER_LEARNED */
typedef struct {
  int32_t batch, block, vocab, K, budget;
  int32_t dtype, kind;
  double lambda1, lambda2, tau, beta;
  int32_t scorer;
  const taps_scorer_mlp *mlp;
} taps_select_params;

/* Selected subtree S per request, breadth first: nodes ordered by depth, then by rank
 * path (the ranks of the tokens from the root down), so a parent always precedes its
 * children.  Arrays are [batch][budget] unless noted; slots n..budget-1 hold
 * parent = token = depth = rank = -1 and q_reach = 0.
 *   parent    index of the parent node within the request; -1 at the root (index 0)
 *   token     vocabulary id; -1 at the root
 *   depth     0 at the root
 *   rank      rank of the token in its position's top-K; -1 at the root
 *   q_reach   Eq. 2 reach probability, fp64; 1.0 at the root
 *   n_nodes   [batch] number of selected nodes n, 1 <= n <= budget
 *   topk_idx  [batch][block][K] top-K vocabulary ids per position: value descending,
 *             then index ascending; -0 equals +0; NaN ranks below -inf
 *   topk_val  [batch][block][K] their marginal values widened to float (exact), or NULL */
typedef struct {
  int32_t *parent;
  int32_t *token;
  int32_t *depth;
  int32_t *rank;
  double *q_reach;
  int32_t *n_nodes;
  int32_t *topk_idx;
  float *topk_val;
} taps_tree;

/* Bytes of scratch taps_select needs (per-chunk top-K candidates; with the marginal scorer
 * on logits also one 64-bit normaliser partial per chunk, with the learned scorer two). */
size_t taps_select_workspace_bytes(const taps_select_params *p);

/* Bytes that taps_select can use beyond those with the learned scorer (0 with the others):
 * each position's top K and K x K edge probabilities.  A workspace of both sizes spreads a
 * request's positions over the GPU; with less, one workgroup scores them all.  Same results. */
size_t taps_select_tables_bytes(const taps_select_params *p);

/* Host-only check of the parameters, no device access (the first step of taps_select). */
taps_status taps_select_validate(const taps_select_params *p);

/* Target-aware selection (Sec. 4.1-4.3, Eq. 1-3, Alg. 1) for `batch` requests.
 *   marginals  [batch][block][vocab] bf16 or fp32, row-major, 16-byte aligned base
 *   out        device arrays described at taps_tree ([host] struct)
 * Edge probability of a rank-r child of any depth-i node (sibling softmax, Eq. 1):
 *   LOGITS  e_r = EXP(beta * (x_r - x_0)), PROBS  e_r = x_r if x_r > 0 else 0;
 *   Z = e_0 + e_1 + ... (in rank order); q_cond = e_r / Z, or 0 when Z is 0 or not finite.
 * Learned scorer: features of an edge into row i (the parent token's embedding, the child
 *   token's, i+1, the child's log-probability (x_v - M) - LOG(Z), the row's entropy
 *   LOG(Z) - S / Z with S = 2^-42 * sum of rint(2^42 * t_j (x_j - M)), t_j = EXP(x_j - M),
 *   terms with t_j = 0 counting 0); a_k = relu(b1[k] + sum_j W1[k][j] f_j) (NaN -> 0),
 *   logit = b2 + sum_k w2[k] a_k, fp64 with sums in index order; q_cond = EXP(l_r - max l)
 *   / (sum over the K siblings in rank order), NaN logits ignored in the max.  LOG is the
 *   shared fp64 logarithm (frexp reduction to [sqrt(1/2), sqrt(2)), 2 atanh series to s^27).
 * Marginal scorer: LOGITS  q_cond = EXP(x_r - M) / Z, M the row maximum, Z = 2^-42 *
 *   sum over the whole row of rint(2^42 * EXP(x_j - M)) (an exact integer sum; NaN
 *   entries count 0), 0 when Z is 0; PROBS  q_cond = min(x_r, 1) if x_r > 0 else 0.
 * EXP is the shared fp64 exponential (Cody-Waite reduction, degree-13 Taylor, no FMA).
 * q_reach multiplies q_cond along the path (Eq. 2); utility = q_reach / (lambda1 +
 * lambda2 * depth) (Eq. 3); all in IEEE fp64.  Ties in the greedy argmax of Alg. 1 go to
 * the shallower node, then to the lexicographically smaller rank path. */
taps_status taps_select(const void *marginals, const taps_select_params *p,
                        const taps_tree *out, void *ws, size_t ws_bytes,
                        hipStream_t stream);

/* taps_select for callers that cannot allocate: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, results and errors as
 * taps_select, without the workspace: the selection's scratch is a static device array of
 * TAPS_SELECT_SCRATCH_BYTES per GPU, which the library holds until the process ends (the
 * first call on a device looks up its address).  The call allocates nothing.
 *   - Parameters whose taps_select_workspace_bytes exceed TAPS_SELECT_SCRATCH_BYTES return
 *     TAPS_ERR_WORKSPACE before anything is enqueued.
 *   - The array is shared by every call on the same GPU and keeps the last call's
 *     contents (no call reads what another left): calls that may overlap in time on one
 *     GPU (other streams, other host threads) race and must be serialized by the caller.
 *   - The device is the one current on the calling thread; `stream` must belong to it. */
#define TAPS_SELECT_SCRATCH_BYTES (8u << 20)
taps_status taps_select_noalloc(const void *marginals, const taps_select_params *p,
                                const taps_tree *out, hipStream_t stream);

/* Bytes of scratch tree_verify_attn needs (split-KV partial outputs).  TAPS_FP32 calls use
 * this much to split long contexts (0 for short ones) and also run with less or none, more
 * slowly.  Calls that may overlap on the GPU need scratch of their own. */
size_t tree_verify_attn_workspace_bytes(int32_t batch, int32_t budget, int32_t Hq,
                                        int32_t Hkv, int32_t head_dim, int32_t max_ctx,
                                        int32_t dtype);

/* Host-only check of the attention sizes, no device access. */
taps_status tree_verify_attn_validate(int32_t batch, int32_t budget, int32_t Hq,
                                      int32_t Hkv, int32_t head_dim, int32_t max_ctx,
                                      int32_t dtype, float scale);

/* Tree-masked verification attention for `batch` requests.
 *   Q_tree       [batch][budget][Hq][head_dim] queries of the tree nodes (tree order)
 *   K_cache,
 *   V_cache      [rows][Hkv][head_dim]; request b owns rows kv_offset[b] ..
 *                kv_offset[b] + ctx_len[b] + budget - 1: its context first, then one
 *                reserved row per tree node i at kv_offset[b] + ctx_len[b] + i
 *   kv_offset    [batch] int64 first cache row of each request
 *   ctx_len      [batch] context rows; values outside [0, max_ctx] are clamped to it
 *   tree_parent  [batch][budget] parent index per node (taps_tree.parent); a node whose
 *                parent is not in [0, i) sees only the context and itself
 *   n_nodes      [batch] nodes to compute; clamped to [0, budget]
 *   head_dim     64 or 128; Hq a multiple of Hkv; query head h reads KV head h/(Hq/Hkv)
 *   max_ctx      [host] upper bound of ctx_len, sizes the grid
 *   dtype        TAPS_BF16 (fp32 accumulation, output rounded to nearest even) or TAPS_FP32
 *   scale        softmax scale, finite and > 0 (usually 1/sqrt(head_dim))
 *   O            [batch][budget][Hq][head_dim] same dtype as Q; rows i >= n are not written
 * O[b,i,h] = softmax_j(scale * Q[b,i,h] . K[j,g]) V[j,g] over the context rows and the
 * ancestor-or-self tree rows of node i, g = h / (Hq/Hkv). */
taps_status tree_verify_attn(const void *Q_tree, const void *K_cache, const void *V_cache,
                             const int64_t *kv_offset, const int32_t *ctx_len,
                             const int32_t *tree_parent, const int32_t *n_nodes,
                             int32_t batch, int32_t budget, int32_t Hq, int32_t Hkv,
                             int32_t head_dim, int32_t max_ctx, int32_t dtype, float scale,
                             void *O, void *ws, size_t ws_bytes, hipStream_t stream);

/* tree_verify_attn that also times its main attention kernel: `ev_begin` and `ev_end` are
 * set to the start and the end of that kernel's execution (hipExtLaunchKernel events; the
 * split combine that follows is not included), so hipEventElapsedTime gives the kernel's
 * own duration.  Either event may be NULL; both must have been created.  For profiling
 * callers. */
taps_status tree_verify_attn_timed(const void *Q_tree, const void *K_cache, const void *V_cache,
                                   const int64_t *kv_offset, const int32_t *ctx_len,
                                   const int32_t *tree_parent, const int32_t *n_nodes,
                                   int32_t batch, int32_t budget, int32_t Hq, int32_t Hkv,
                                   int32_t head_dim, int32_t max_ctx, int32_t dtype,
                                   float scale, void *O, void *ws, size_t ws_bytes,
                                   hipStream_t stream, hipEvent_t ev_begin, hipEvent_t ev_end);

/* Bytes of scratch tree_verify_attn_paged needs for these sizes and page size (0 when
 * they are not supported). */
size_t tree_verify_attn_paged_workspace_bytes(int32_t batch, int32_t budget, int32_t Hq,
                                              int32_t Hkv, int32_t head_dim, int32_t max_ctx,
                                              int32_t page_rows);

/* tree_verify_attn over a paged KV cache, for batched serving (the Limitations leave the
 * cache layout to the serving system; pages let requests grow without moving rows).  Same
 * result as tree_verify_attn with request b's logical cache row r (its context rows
 * 0 .. ctx-1, then node i at row ctx + i) stored at
 *   K_pages[block_table[b][r / page_rows]][r % page_rows] (and V_pages alike).
 *   K_pages,
 *   V_pages      [num_pages][page_rows][Hkv][head_dim] bf16 pools, 16-byte aligned
 *   num_pages    pages in each pool (>= 1; num_pages * page_rows below 2^32, else
 *                TAPS_ERR_UNSUPPORTED)
 *   page_rows    rows per page: a power of two from 32 to 4096
 *   block_table  [batch][max_pages] int32 page ids, row b covering request b's rows in
 *                order; max_pages * page_rows must be at least max_ctx + budget.  Entries
 *                the request's rows do not reach are not read for keys; ids outside
 *                [0, num_pages) are clamped into it (never a read outside the pools; the
 *                result is then meaningless)
 *   the other arguments as for tree_verify_attn (no kv_offset); head_dim 128 and TAPS_BF16
 *   only (other sizes and types: TAPS_ERR_UNSUPPORTED)
 *   ws           tree_verify_attn_paged_workspace_bytes(...) bytes, 16-byte aligned */
taps_status tree_verify_attn_paged(const void *Q_tree, const void *K_pages, const void *V_pages,
                                   int32_t num_pages, int32_t page_rows,
                                   const int32_t *block_table, int32_t max_pages,
                                   const int32_t *ctx_len, const int32_t *tree_parent,
                                   const int32_t *n_nodes, int32_t batch, int32_t budget,
                                   int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t max_ctx,
                                   int32_t dtype, float scale, void *O, void *ws,
                                   size_t ws_bytes, hipStream_t stream);

/* tree_verify_attn_paged that also times its main attention kernel, as
 * tree_verify_attn_timed does.  For profiling callers. */
taps_status tree_verify_attn_paged_timed(const void *Q_tree, const void *K_pages,
                                         const void *V_pages, int32_t num_pages,
                                         int32_t page_rows, const int32_t *block_table,
                                         int32_t max_pages, const int32_t *ctx_len,
                                         const int32_t *tree_parent, const int32_t *n_nodes,
                                         int32_t batch, int32_t budget, int32_t Hq, int32_t Hkv,
                                         int32_t head_dim, int32_t max_ctx, int32_t dtype,
                                         float scale, void *O, void *ws, size_t ws_bytes,
                                         hipStream_t stream, hipEvent_t ev_begin,
                                         hipEvent_t ev_end);

/* Greedy acceptance walk (temperature 0).
 *   tree           [host] struct; parent, token and n_nodes are read
 *   target_tokens  [batch][budget] target model's greedy token after each node
 *   path           [batch][block+1] accepted node indices from the root, -1 padded
 *   path_len       [batch] accepted nodes including the root (1 .. block+1)
 *   bonus          [batch] target token after the last accepted node
 * A node is accepted when its token equals the target token after its parent and its
 * parent is accepted; the root always is. */
taps_status accept_walk(const taps_tree *tree, int32_t batch, int32_t budget,
                        int32_t block, const int32_t *target_tokens, int32_t *path,
                        int32_t *path_len, int32_t *bonus, hipStream_t stream);

/* KV commit of the accepted path: the round's state update after accept_walk (Sec. 1:
 * each decoding round commits only one prefix path; the paper leaves the update itself
 * to the serving system).
 *   K_cache,
 *   V_cache      [rows][Hkv][head_dim] in the layout of tree_verify_attn, updated in place:
 *                for request b the rows of the m committed path nodes, kv_offset[b] +
 *                ctx + path[b][j], move to rows kv_offset[b] + ctx + j (j = 0 .. m-1, the
 *                root's row stays); no other row is written.  ctx = ctx_len[b] clamped to
 *                [0, max_ctx].
 *   kv_offset,
 *   ctx_len      as for tree_verify_attn (not written)
 *   tree         [host] struct; token is read ([batch][budget], node tokens)
 *   path,
 *   path_len,
 *   bonus        accept_walk's outputs.  The committed path is the root followed by the
 *                entries path[b][1 .. path_len[b]-1] up to (not including) the first one
 *                that is not larger than the previous entry or not below budget; m is its
 *                length (1 .. block+1)
 *   new_ctx_len  [batch] ctx + m; must not be the ctx_len array (other workgroups of the
 *                same request may still read ctx_len)
 *   committed    [batch][block+1] the tokens the round emits: the drafted tokens of the
 *                m-1 accepted nodes in path order, then the bonus token, then -1
 *   n_committed  [batch] m (tokens emitted)
 *   dtype        TAPS_BF16 or TAPS_FP32 (element size of the cache)
 * K_cache and V_cache must be 16-byte aligned.  Calls that touch the same cache rows must
 * not overlap in time. */
taps_status kv_commit(void *K_cache, void *V_cache, const int64_t *kv_offset,
                      const int32_t *ctx_len, const taps_tree *tree, const int32_t *path,
                      const int32_t *path_len, const int32_t *bonus, int32_t batch,
                      int32_t budget, int32_t block, int32_t Hkv, int32_t head_dim,
                      int32_t max_ctx, int32_t dtype, int32_t *new_ctx_len,
                      int32_t *committed, int32_t *n_committed, hipStream_t stream);

/* kv_commit for a paged KV cache (the layout of tree_verify_attn_paged): the same update
 * in logical rows, request b's logical row r being row r % page_rows of page
 * block_table[b][r / page_rows] of K_pages and V_pages ([num_pages][page_rows][Hkv]
 * [head_dim], 16-byte aligned).  The rows of the m committed path nodes, logical rows
 * ctx + path[b][j], move to logical rows ctx + j; no other row is written.  page_rows is a
 * power of two from 32 to 4096 and max_pages * page_rows >= max_ctx + budget; page ids
 * outside [0, num_pages) are clamped into it.  A request's rows must sit in pages of its
 * own (pages shared with another request of the same call race).  The other arguments and
 * outputs as for kv_commit. */
taps_status kv_commit_paged(void *K_pages, void *V_pages, int32_t num_pages, int32_t page_rows,
                            const int32_t *block_table, int32_t max_pages,
                            const int32_t *ctx_len, const taps_tree *tree, const int32_t *path,
                            const int32_t *path_len, const int32_t *bonus, int32_t batch,
                            int32_t budget, int32_t block, int32_t Hkv, int32_t head_dim,
                            int32_t max_ctx, int32_t dtype, int32_t *new_ctx_len,
                            int32_t *committed, int32_t *n_committed, hipStream_t stream);

/* [host] Weights of one attention layer of the target, a Qwen3-style block.  DEVICE bf16
 * arrays owned by the caller, row-major [out][in], 16-byte aligned:
 *   Wq [Hq*head_dim][hidden], Wk and Wv [Hkv*head_dim][hidden], Wo [hidden][Hq*head_dim]
 *   q_norm, k_norm [head_dim] per-head RMSNorm weights of the queries and keys
 *   rope_theta  rotary base, finite and > 1 (Qwen3: 1e6)
 *   norm_eps    RMSNorm epsilon, finite and >= 0 (Qwen3: 1e-6)
 *   hidden      model width, a multiple of 64, at most 16384 */
typedef struct {
  const void *Wq, *Wk, *Wv, *Wo, *q_norm, *k_norm;
  double rope_theta;
  float norm_eps;
  int32_t hidden;
} taps_layer_weights;

/* Bytes of scratch verify_layer needs (projection partials, Q, O, attention partials);
 * 0 for sizes verify_layer rejects. */
size_t verify_layer_workspace_bytes(int32_t batch, int32_t budget, int32_t Hq, int32_t Hkv,
                                    int32_t head_dim, int32_t hidden, int32_t max_ctx);

/* One attention layer of the target over the selected trees: the layer slice of the
 * verification forward (Sec. 4.1, the verification stage, and Sec. 4.3 run the target once
 * over the tree with tree attention).  bf16 storage, fp32 accumulation.
 *   X          [batch][budget][hidden] bf16 hidden states of the tree nodes (tree order),
 *              16-byte aligned
 *   w          the layer's weights (above)
 *   K_cache,
 *   V_cache    as for tree_verify_attn (bf16); the key and value of node i < n_nodes[b]
 *              are written to row kv_offset[b] + ctx_len[b] + i, no other row is written
 *   kv_offset, ctx_len, max_ctx, scale: as for tree_verify_attn
 *   tree       parent, depth and n_nodes of the selected trees (taps_tree; other fields
 *              are not read)
 *   head_dim   128
 *   Y          [batch][budget][hidden] bf16, 16-byte aligned; rows i >= n_nodes[b] are not
 *              defined
 *   ws         verify_layer_workspace_bytes(...) bytes, 256-byte aligned
 * Steps: q, k, v = X W^T per node; RMSNorm of each query and key head; rotary embedding
 * at position ctx_len[b] + depth (the root right after the context, siblings at one
 * position; pairs (j, j + head_dim/2) turn by pos * rope_theta^(-2j/head_dim)); Q, K and
 * V rounded to bf16; tree attention as tree_verify_attn; O rounded to bf16; Y = O Wo^T
 * rounded to bf16. */
taps_status verify_layer(const void *X, const taps_layer_weights *w, void *K_cache,
                         void *V_cache, const int64_t *kv_offset, const int32_t *ctx_len,
                         const taps_tree *tree, int32_t batch, int32_t budget, int32_t Hq,
                         int32_t Hkv, int32_t head_dim, int32_t max_ctx, float scale, void *Y,
                         void *ws, size_t ws_bytes, hipStream_t stream);

/* Bytes of scratch verify_layer_paged needs (0 when the sizes are not supported). */
size_t verify_layer_paged_workspace_bytes(int32_t batch, int32_t budget, int32_t Hq,
                                          int32_t Hkv, int32_t head_dim, int32_t hidden,
                                          int32_t max_ctx, int32_t page_rows);

/* verify_layer over a paged KV cache, for batched serving (Sec. 4.1 Stage 3 and Sec. 4.3
 * for the layer's tree attention; the Limitations leave cache management to the serving
 * system), in the layout of tree_verify_attn_paged: node i's key and value go to logical
 * row ctx + i of request b, i.e. row (ctx + i) % page_rows of page
 * block_table[b][(ctx + i) / page_rows]; the attention reads the pages.  K_pages, V_pages,
 * num_pages, page_rows, block_table and max_pages as for tree_verify_attn_paged (same
 * validation and errors); the other arguments as for verify_layer (no kv_offset).  Only
 * the nodes' rows of the pools are written. */
taps_status verify_layer_paged(const void *X, const taps_layer_weights *w, void *K_pages,
                               void *V_pages, int32_t num_pages, int32_t page_rows,
                               const int32_t *block_table, int32_t max_pages,
                               const int32_t *ctx_len, const taps_tree *tree, int32_t batch,
                               int32_t budget, int32_t Hq, int32_t Hkv, int32_t head_dim,
                               int32_t max_ctx, float scale, void *Y, void *ws, size_t ws_bytes,
                               hipStream_t stream);

/* Pages for the next rows of a batch's requests: block tables and slot maps from request
 * lengths.  Request b is to own the logical rows 0 .. ctx + new - 1, i.e. want = ceil((ctx +
 * new) / page_rows) pages (ctx = ctx_len[b], at least 0; new = n_new[b] clamped to [0,
 * max_new]); it holds held_pages[b] (clamped to [0, max_pages]), the first entries of its table
 * row.  A request with more gives the last ones back, one with fewer takes new ones:
 *   - every page that a request gives back is pushed onto the stack of free pages, in the
 *     order of requests, each request's in the order of its table row;
 *   - then the requests that need pages take them off the top, in the order of requests, each
 *     in the order of its table row, as long as the stack holds all that this and the earlier
 *     requests need.  From the first request that is short on, no request takes pages, and the
 *     ones that need some keep what they have.
 * A request whose rows need more than max_pages pages keeps what it has and is short.
 *   block_table  [batch][max_pages] int32 page ids; entries held .. want - 1 of the requests
 *                that take pages are written, no other
 *   held_pages, ctx_len, n_new  [batch] int32.  A request that has ended: ctx_len = n_new = 0
 *   free_pages   [num_pages] int32, the stack: entries 0 .. n_free - 1 are free pages; pushed
 *                ones are written from entry n_free on (none past num_pages)
 *   n_free       [1] int32, clamped to [0, num_pages]
 *   num_pages, page_rows  as for tree_verify_attn_paged; max_pages * page_rows at most 2^30
 *   held_out     [batch] pages held afterwards
 *   n_free_out   [1] free pages afterwards
 *   n_short      [1] number of requests that did not get what they need.  These three share no
 *                memory with held_pages, ctx_len, n_new and n_free
 *   slot_map     [batch][max_new] int64, or NULL: the pool row of logical row ctx + i, page id
 *                * page_rows + (ctx + i) % page_rows, for i < new; -1 from new on, and for
 *                every row of a request that is short
 * batch at most 4096; a batch of 0 writes nothing, n_free_out and n_short neither.  The call is
 * one kernel and needs no workspace; a page id must not be in two places (the tables' held
 * entries and the stack). */
taps_status kv_reserve_paged(int32_t *block_table, int32_t max_pages, const int32_t *held_pages,
                             const int32_t *ctx_len, const int32_t *n_new, int32_t batch,
                             int32_t max_new, int32_t *free_pages, const int32_t *n_free,
                             int32_t num_pages, int32_t page_rows, int32_t *held_out,
                             int32_t *n_free_out, int32_t *n_short, int64_t *slot_map,
                             hipStream_t stream);

/* New K and V rows into a paged cache: row t of K_new and V_new goes to row slot_map[t] of the
 * pools (page slot / page_rows, row slot % page_rows of it); slots outside [0, num_pages *
 * page_rows), such as the -1 of kv_reserve_paged, are left out.  No other row is written.
 *   K_new, V_new  [rows][Hkv][head_dim], consecutive rows k_stride and v_stride elements apart
 *                 (at least Hkv * head_dim, a multiple of 16 bytes): slices of a fused
 *                 projection's rows need no copy.  Not in the pools' memory
 *   slot_map      [rows] int64; a slot must not be named twice (its row would be a mix)
 *   K_pages, V_pages, num_pages, page_rows  as for tree_verify_attn_paged
 *   head_dim 64 or 128; dtype TAPS_BF16 or TAPS_FP32 for all four; 16-byte aligned bases */
taps_status kv_append_paged(const void *K_new, const void *V_new, int64_t k_stride,
                            int64_t v_stride, const int64_t *slot_map, int32_t rows, int32_t Hkv,
                            int32_t head_dim, int32_t dtype, void *K_pages, void *V_pages,
                            int32_t num_pages, int32_t page_rows, hipStream_t stream);

/* Host-only check of the sizes of decode_attn_paged, no device access. */
taps_status decode_attn_paged_validate(int32_t batch, int32_t Hq, int32_t Hkv, int32_t head_dim,
                                       int32_t max_len, int32_t page_rows, int32_t dtype,
                                       float scale);

/* Bytes of scratch decode_attn_paged needs (the splits' parts; 0 for short caches and for
 * sizes that it rejects).  Calls that may overlap on the GPU need scratch of their own. */
size_t decode_attn_paged_workspace_bytes(int32_t batch, int32_t Hq, int32_t Hkv, int32_t head_dim,
                                         int32_t max_len, int32_t page_rows, int32_t dtype);

/* Attention of one new token per request over a paged KV cache: the decoding step of requests
 * that have no draft.  O[b,h] = softmax_j(scale * Q[b,h] . K[j,g]) V[j,g] over the logical rows
 * j < kv_len[b] (the new token's own row, appended before the call, among them), g = h / (Hq /
 * Hkv); zeros where kv_len[b] is 0.
 *   Q            [batch][Hq][head_dim], consecutive requests q_stride elements apart (at least
 *                Hq * head_dim, a multiple of 16 bytes)
 *   K_pages, V_pages, num_pages, page_rows, block_table, max_pages  as for
 *                tree_verify_attn_paged, in dtype; max_pages * page_rows at least max_len
 *   kv_len       [batch] int32, clamped to [0, max_len].  Rows past it may hold anything; rows
 *                below it that are not finite leave outputs that are not
 *   head_dim     64 or 128; Hq a multiple of Hkv; batch * Hkv at most 65535
 *   max_len      [host] upper bound of kv_len, sizes the grid
 *   dtype        TAPS_BF16 (fp32 accumulation, output rounded to nearest even) or TAPS_FP32
 *   scale        softmax scale, finite and > 0
 *   O            [batch][Hq][head_dim] in dtype, 16-byte aligned; not in Q's memory
 *   ws           decode_attn_paged_workspace_bytes(...) bytes, 16-byte aligned */
taps_status decode_attn_paged(const void *Q, int64_t q_stride, const void *K_pages,
                              const void *V_pages, int32_t num_pages, int32_t page_rows,
                              const int32_t *block_table, int32_t max_pages,
                              const int32_t *kv_len, int32_t batch, int32_t Hq, int32_t Hkv,
                              int32_t head_dim, int32_t max_len, int32_t dtype, float scale,
                              void *O, void *ws, size_t ws_bytes, hipStream_t stream);

#define TAPS_MAX_SAMPLE_VOCAB (1 << 20)

/* [host] Settings of taps_sample: DEVICE arrays of one value per request; a NULL array turns
 * its setting off.
 *   temperature  T > 0; 0, negative or NaN: the largest logit (greedy).  NULL: 1
 *   top_k        keep the top_k first tokens of the rank order; <= 0 or >= vocab: all
 *   top_p        of those, keep the shortest prefix whose probability reaches top_p; >= 1 or
 *                NaN: all; <= 0: the first
 *   min_p        of those, keep the tokens whose probability is at least min_p times the
 *                largest one's; <= 0 or NaN: all; >= 1: those equal to the largest */
typedef struct {
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
} taps_sampling;

/* Host-only check of the sizes of taps_sample, no device access. */
taps_status taps_sample_validate(int32_t batch, int32_t budget, int32_t vocab, int64_t row_stride,
                                 int32_t dtype);

/* Bytes of scratch taps_sample needs: 0 for every size. */
size_t taps_sample_workspace_bytes(int32_t batch, int32_t budget, int32_t vocab, int32_t dtype);

/* One token per logits row, from a given random number: the target's token after each node of
 * a draft tree (accept_walk on them accepts a drafted token with the target's own probability
 * of it, so the emitted tokens are samples of the target), or, with budget 1, each request's
 * next token.
 *   logits     [batch][budget][vocab] bf16 or fp32, consecutive rows row_stride elements apart
 *              (at least vocab).  Base 16-byte aligned where vocab elements are a multiple of 16
 *              bytes, otherwise aligned to an element (a view that leaves rows out, of logits
 *              with an odd vocabulary, needs no copy)
 *   n_nodes    [batch] int32 rows to sample per request, or NULL (all): rows i >= n_nodes[b]
 *              get token -1 and probability 0, their logits are not read
 *   s          the settings
 *   u          [batch][budget] float random numbers in [0, 1) (NaN counts 0; others are clamped)
 *   tokens     [batch][budget] int32
 *   probs      [batch][budget] float, or NULL: the token's probability among the kept ones
 *   ws, ws_bytes  not read (a row's work stays in its workgroup); NULL and 0 will do
 * A row's rank order is value descending, then index ascending; -0 equals +0; NaN is last.
 * Token r of it has the weight W_r = exp((x_r - x_0) / T), 1 where x_r equals x_0 (infinite values
 * too) and 0 for NaN, evaluated in fp64 to within 2^-42 of W_0 and added up as integers, so that
 * results do not depend on the order of additions.  S_k is the sum of the weights after top_k;
 * top_p keeps up to the first token whose running sum reaches top_p * S_k; S is the sum of all
 * that are kept.  The token is the first whose running sum exceeds u * S, its probability W / S.
 * Weights are rounded to multiples of 2^-43 of W_0, so that those of at most 2^-44 are 0 and
 * never drawn.  (fp32 rows that neither a small top_k nor min_p bounds: weights above 2^-44 are
 * added up before they are rounded, in bins of 1/32 octave whose running sums are rounded down; a
 * token's share of a sum still is within 2^-42 of W_0 of its weight, but a lone weight below
 * 2^-43 may count 0 there.)  A row of NaN alone gives token 0 with probability 0.
 * budget at most TAPS_MAX_BUDGET, vocab at most TAPS_MAX_SAMPLE_VOCAB, batch * budget at most
 * 2^20. */
taps_status taps_sample(const void *logits, int64_t row_stride, int32_t batch, int32_t budget,
                        int32_t vocab, int32_t dtype, const int32_t *n_nodes,
                        const taps_sampling *s, const float *u, int32_t *tokens, float *probs,
                        void *ws, size_t ws_bytes, hipStream_t stream);

/* [host] How positions are stretched past a trained length (factor s, trained length L), as in
 * f_j = theta^(-2j / rot_dim), the turn of pair j per position in radians:
 *   TAPS_ROPE_PLAIN   f_j
 *   TAPS_ROPE_LINEAR  f_j / s: positions are interpolated
 *   TAPS_ROPE_NTK     f_j with theta s^(rot_dim / (rot_dim - 2)): the slowest pair turns s times
 *                     slower, the fastest as before (rot_dim at least 4)
 *   TAPS_ROPE_YARN    by parts (YaRN, arXiv 2309.00071, alpha 1 and beta 32): with r = L f_j / (2
 *                     pi) turns over the trained length and g = (r - 1) / 31 clamped to [0, 1],
 *                     g f_j + (1 - g) f_j / s; cosines and sines are multiplied by 0.1 ln s + 1.
 *                     The ramp is the paper's, linear in the turns r.  Many checkpoints that name
 *                     this kind were run with another, linear in the pair's index between the two
 *                     pairs (rounded) where r is 32 and 1: at theta 1e6, 128 dims, L 32768 and s 4
 *                     pair 32 turns 0.60 f_j there and 0.35 f_j here.  For those, and for any other
 *                     kind, fill taps_rope.inv_freq and mscale oneself; nothing here is compared
 *                     with a released model */
typedef enum {
  TAPS_ROPE_PLAIN = 0,
  TAPS_ROPE_LINEAR = 1,
  TAPS_ROPE_NTK = 2,
  TAPS_ROPE_YARN = 3
} taps_rope_scaling;

/* [host] The frequencies of rot_dim / 2 pairs (inv_freq, [host] memory) and the factor of cosines
 * and sines.  rot_dim even, 2 .. 4096; theta finite and > 1; factor finite and >= 1; trained_len
 * >= 1.  The plain kind reads neither factor nor trained_len, linear and NTK no trained_len. */
taps_status taps_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor,
                                  int64_t trained_len, double *inv_freq, float *mscale);

/* [host] Norm and rotation of qk_rope_paged.
 *   inv_freq        DEVICE [rot_dim / 2] fp64, 8-byte aligned: the pairs' turns per position
 *   q_norm, k_norm  DEVICE [head_dim] RMSNorm weights in the call's dtype, 16-byte aligned, or
 *                   NULL: no norm
 *   norm_eps        finite and >= 0 (0: a head of zeros becomes NaN)
 *   mscale          factor of cosines and sines, finite (1 without stretching)
 *   rot_dim         dims of a head that turn, from its first on: a multiple of 8, 8 .. head_dim
 *   interleaved     0: pair j is (j, j + rot_dim / 2); 1: (2j, 2j + 1) */
typedef struct {
  const double *inv_freq;
  const void *q_norm, *k_norm;
  float norm_eps, mscale;
  int32_t rot_dim, interleaved;
} taps_rope;

/* New tokens' queries, keys and values, as they leave their projection, made ready for attention
 * over a paged cache: per query and key head RMSNorm over the whole head (x rsqrt(mean x^2 +
 * eps) w), then pair j of it turned by positions[t] * inv_freq[j]: (a, b) -> mscale (a cos - b
 * sin, b cos + a sin); dims from rot_dim on stay.  fp32 arithmetic (angles fp64), rounded once.
 * Token t's key and value go to row slot_map[t] of the pools; slots outside [0, num_pages *
 * page_rows), such as the -1 of kv_reserve_paged, leave them out (the query is written all the
 * same).  No other row of the pools is written.
 *   Q, K, V    [rows][Hq or Hkv][head_dim], consecutive rows q_stride, k_stride and v_stride
 *              elements apart (at least a row, at most 2^30, a multiple of 16 bytes): slices of a
 *              fused projection's rows need no copy
 *   positions  [rows] int32
 *   slot_map   [rows] int64; a slot must not be named twice (its row would be a mix)
 *   Q_out      [rows][Hq][head_dim]; it and the pools share no memory with Q, K, V or each other
 *              (Q_out and the inputs are checked, and refused as TAPS_ERR_INVALID_ARG)
 *   K_pages, V_pages, num_pages, page_rows  as for tree_verify_attn_paged
 *   head_dim 64 or 128; dtype TAPS_BF16 or TAPS_FP32 for all of them; 16-byte aligned bases */
taps_status qk_rope_paged(const void *Q, const void *K, const void *V, int64_t q_stride,
                          int64_t k_stride, int64_t v_stride, const int32_t *positions,
                          const int64_t *slot_map, int32_t rows, int32_t Hq, int32_t Hkv,
                          int32_t head_dim, int32_t dtype, const taps_rope *rope, void *Q_out,
                          void *K_pages, void *V_pages, int32_t num_pages, int32_t page_rows,
                          hipStream_t stream);

/* Host-only check of the sizes of chunk_attn_paged, no device access. */
taps_status chunk_attn_paged_validate(int32_t batch, int32_t rows, int32_t Hq, int32_t Hkv,
                                      int32_t head_dim, int32_t max_len, int32_t page_rows,
                                      int32_t window, int32_t dtype, float scale);

/* Bytes of scratch chunk_attn_paged needs (parts of tiles that are cut, none for short caches;
 * where each request begins, for more than 256; 0 for sizes that it rejects).  Enough for calls
 * with fewer rows too.  Calls that may overlap on the GPU need scratch of their own. */
size_t chunk_attn_paged_workspace_bytes(int32_t batch, int32_t rows, int32_t Hq, int32_t Hkv,
                                        int32_t head_dim, int32_t max_len, int32_t page_rows,
                                        int32_t dtype);

/* Attention of chunks of new tokens over a paged KV cache: prompts, whole or in chunks, and
 * single tokens among them.  Request b's n = q_start[b + 1] - q_start[b] new tokens are rows
 * q_start[b] .. of Q and O, and the last n of its kv_len[b] cache rows are theirs (appended
 * before the call).  Token i is at row p = kv_len[b] - n + i and sees the rows j <= p; with a
 * window only p - window < j <= p.  O[i,h] = softmax_j(scale * Q[i,h] . K[j,g]) V[j,g], g = h /
 * (Hq / Hkv); zeros for a token that sees no row (kv_len[b] < n).
 *   Q            [rows][Hq][head_dim], consecutive rows q_stride elements apart (at least
 *                Hq * head_dim, at most 2^30, a multiple of 16 bytes)
 *   K_pages, V_pages, num_pages, page_rows, block_table, max_pages  as for
 *                tree_verify_attn_paged, in dtype; max_pages * page_rows at least max_len.  Pages
 *                may be in several requests' tables (a common beginning).  Block
 *                table entries of pages that no token of the request sees (before the window, past
 *                kv_len) may hold anything
 *   q_start      [batch + 1] int32, not decreasing, within [0, rows] (clamped to it).  Rows of O
 *                outside q_start[0] .. q_start[batch] - 1 are not written
 *   kv_len       [batch] int32, clamped to [0, max_len].  Rows that no token of the call sees may
 *                hold anything; rows that one sees and that are not finite leave undefined values
 *                in any of the request's outputs
 *   rows         [host] rows of Q and O, sizes the grid; rows * Hq at most 2^30, batch at most
 *                2^20, and rows * Hq / 128 (fp32: 64) + batch * Hkv below 8 million or so (a
 *                launch's threads are counted in 32 bits)
 *   head_dim     64 or 128; Hq a multiple of Hkv
 *   max_len      [host] upper bound of kv_len, at most 2^30; it picks the tiles, so that one near
 *                the lengths is the faster one (a prompt of 1024, 32/8 heads of 128, takes 27 us,
 *                39 under a bound of 32K)
 *   window       0: none; else at least 1
 *   dtype        TAPS_BF16 (fp32 accumulation, weights rounded to bf16 for the second product,
 *                output rounded to nearest even) or TAPS_FP32.  For batches of one token per
 *                request decode_attn_paged is mostly faster and, in bf16, more exact
 *   scale        softmax scale, finite and > 0
 *   O            [rows][Hq][head_dim] in dtype, 16-byte aligned; not in the memory of Q or of the
 *                pools (checked)
 *   ws           chunk_attn_paged_workspace_bytes(...) bytes, 16-byte aligned */
taps_status chunk_attn_paged(const void *Q, int64_t q_stride, const void *K_pages,
                             const void *V_pages, int32_t num_pages, int32_t page_rows,
                             const int32_t *block_table, int32_t max_pages,
                             const int32_t *q_start, const int32_t *kv_len, int32_t batch,
                             int32_t rows, int32_t Hq, int32_t Hkv, int32_t head_dim,
                             int32_t max_len, int32_t window, int32_t dtype, float scale, void *O,
                             void *ws, size_t ws_bytes, hipStream_t stream);

#define TAPS_MAX_LOGPROB_TOP 64

/* Host-only check of the sizes of taps_logprobs, no device access. */
taps_status taps_logprobs_validate(int32_t batch, int32_t budget, int32_t vocab,
                                   int64_t row_stride, int32_t dtype, int32_t top);

/* Bytes of scratch taps_logprobs needs (the parts that few rows are cut into; 0 for many rows or a
 * small vocabulary, so that fewer rows may need more).  Calls that may overlap on the GPU need
 * scratch of their own. */
size_t taps_logprobs_workspace_bytes(int32_t batch, int32_t budget, int32_t vocab, int32_t dtype,
                                     int32_t top);

/* Log probabilities of given tokens under each logits row (a prompt's next tokens, sampled or
 * drafted ones), with their ranks, the row's entropy and its top alternatives.
 *   logits       [batch][budget][vocab] as for taps_sample (row_stride, alignment, dtype, limits of
 *                the sizes: a prompt of more than TAPS_MAX_BUDGET positions is several requests)
 *   n_nodes      [batch] int32 rows per request, or NULL (all): rows i >= n_nodes[b] get 0, rank
 *                and index -1, their logits and tokens are not read
 *   tokens       [batch][budget] int32.  Outside [0, vocab), such as the -1 of padding: log
 *                probability -inf and rank -1 (entropy and alternatives are the row's)
 *   top          alternatives per row, 0 .. min(vocab, TAPS_MAX_LOGPROB_TOP)
 *   logprob      [batch][budget] float: ln p of the token
 *   entropy      [batch][budget] float: -sum p ln p in nats
 *   rank         [batch][budget] int32: tokens before it in the rank order (0: the largest)
 *   top_idx      [batch][budget][top] int32, the first `top` tokens of the rank order
 *   top_logprob  [batch][budget][top] float, theirs.  (Both may be NULL where top is 0)
 *   ws           taps_logprobs_workspace_bytes(...) bytes, 16-byte aligned
 * The outputs share no memory with the inputs or each other.
 * p_j = w_j / sum w, w_j = exp(x_j - x_0) for the largest value x_0: 1 where x_j equals x_0
 * (infinite values too), 0 for NaN, as in taps_sample at T = 1.  The rank order is value
 * descending, then index ascending; -0 equals +0; NaN is last.  A row of NaN alone has log
 * probabilities -inf and entropy 0.  Sums are fp32 per thread, joined in fp64; log probabilities
 * are at most 0 and entropies at least 0, both 0 where the largest value alone has a weight.
 * Rows whose largest value is 1e6 or more, or -999,000 or less, take a scan of the row for each
 * alternative (64 fp32 rows of 151,936: 205 us with 5, 2070 with 64, for 19.5 and 27). */
taps_status taps_logprobs(const void *logits, int64_t row_stride, int32_t batch, int32_t budget,
                          int32_t vocab, int32_t dtype, const int32_t *n_nodes,
                          const int32_t *tokens, int32_t top, float *logprob, float *entropy,
                          int32_t *rank, int32_t *top_idx, float *top_logprob, void *ws,
                          size_t ws_bytes, hipStream_t stream);

/* Human-readable name of a status code (static string). */
const char *taps_status_string(int32_t status);

/* Host evaluation of the shared fp64 exponential used on the device, for testing the
 * definition against other implementations without a GPU. */
double taps_spec_exp_host(double t);

#ifdef __cplusplus
}
#endif
#endif /* TAPS_H */
