/*
 * propd.h - C ABI of the MI355X token-tree verification library.
 *
 * The library implements the verification step of ProPD's parallel decoding
 * (arXiv 2402.13485): tree-masked attention, the early-pruning pass and greedy
 * acceptance, as HIP kernels for gfx950.  Plain C99: pointers and sizes only.
 *
 * Common rules for every entry point
 *   - Pointers named in a parameter list are DEVICE pointers unless the comment
 *     says "host".  The caller owns every buffer, before and after the call; the
 *     library allocates nothing, frees nothing and keeps no pointer.
 *   - All work is enqueued on `hip_stream` (a hipStream_t passed as void*, NULL =
 *     the default stream).  No entry point synchronises with the host or copies
 *     between host and device; outputs are valid once the stream reaches the end
 *     of the enqueued work.  `workspace` is scratch for the duration of that work
 *     and must not be shared by calls that may overlap on different streams.
 *   - Scalars are validated on the host: a bad scalar, a NULL required pointer or
 *     a short workspace returns an error code and enqueues nothing.  The content
 *     of device arrays is not validated: a tree whose parent array is not
 *     topological (parent[i] < i), or a mask that does not belong to the parent
 *     array, gives unspecified results, but never an out-of-bounds access
 *     (indices read from device arrays are range-checked in the kernels).
 *   - Tensors are dense and row-major with the innermost dimension contiguous;
 *     base pointers must be 16-byte aligned.
 *   - Trees: node 0 of every sequence is the root, i.e. the token the model has
 *     already fixed; it counts towards T, is never pruned and is always accepted.
 *     Nodes are stored in a topological (for instance breadth-first) order.
 *     Per-sequence slots have T_max entries; entries at or beyond n_nodes[b] are
 *     padding: never read as data, and written only where a comment says so.
 */
#ifndef PROPD_H
#define PROPD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Entry points are the only symbols the shared library exports. */
#if defined(__GNUC__)
#define PROPD_API __attribute__((visibility("default")))
#else
#define PROPD_API
#endif

typedef enum {
  PROPD_OK = 0,
  PROPD_ERR_INVALID_ARG = 1, /* a scalar out of range or a required pointer is NULL */
  PROPD_ERR_UNSUPPORTED = 2, /* a legal request this build has no kernel for        */
  PROPD_ERR_WORKSPACE = 3,   /* workspace NULL or smaller than propd_workspace_bytes */
  PROPD_ERR_DEVICE = 4       /* the HIP runtime refused a launch                    */
} propd_status;

/* PROPD_E4M3: 8-bit floating point (1 sign, 4 exponent, 3 mantissa bits, no infinities, largest 448), in the
 * pages of a propd_paged_cache only. */
typedef enum { PROPD_F32 = 0, PROPD_BF16 = 1, PROPD_E4M3 = 2 } propd_dtype;

/* Largest tree, root included.  A node's ancestor set is a 128-bit set, two
 * uint64 words, word 0 holding nodes 0..63. */
#define PROPD_MAX_TREE 128

/* A batch of token trees (Section 2: candidates organised as a tree that shares
 * common prefixes; node = one candidate token at one future position). */
typedef struct propd_tree {
  int32_t B;               /* sequences, >= 1                                         */
  int32_t T_max;           /* slot size, 1..PROPD_MAX_TREE                            */
  const int32_t *n_nodes;  /* [B]          T_b in 1..T_max                            */
  const int32_t *parent;   /* [B,T_max]    parent[0] = -1, 0 <= parent[i] < i         */
  const int32_t *token;    /* [B,T_max]    candidate token id of each node            */
  const int32_t *depth;    /* [B,T_max]    edges to the root, depth[0] = 0            */
  const uint64_t *anc;     /* [B,T_max,2]  ancestor-or-self set: the cached tree mask */
} propd_tree;

/* Same fields, writable: where a call produces a tree. */
typedef struct propd_tree_out {
  int32_t *n_nodes;
  int32_t *parent;
  int32_t *token;
  int32_t *depth;
  uint64_t *anc;
} propd_tree_out;

/* A per-node row tensor that continues past the pruning point and has to be
 * narrowed to the surviving nodes.  It is viewed as [B, outer, T_max] rows of
 * row_bytes bytes; hidden states [B,T_max,Hd] have outer = 1, tree K or V
 * [B,H,T_max,d] have outer = H.  Strides are in bytes and apply to src and dst. */
typedef struct propd_payload {
  const void *src;         /* device                                                  */
  void *dst;               /* device, must not overlap src                            */
  size_t row_bytes;
  int64_t outer;
  int64_t stride_b, stride_outer, stride_t;
} propd_payload;

/*
 * Build the cached tree mask from parent pointers (Section 2, "Verification";
 * Section 4.1, "Implementation Optimization": the mask lives on the GPU).
 *   anc[b,i]  = set of nodes on the root path of i, i included
 *   depth[b,i] = number of edges from i to the root
 * Padding slots get anc = 0 and depth = -1.  depth may be NULL.
 */
PROPD_API propd_status propd_tree_mask(int32_t B, int32_t T_max, const int32_t *n_nodes,
                             const int32_t *parent, int32_t *depth, uint64_t *anc,
                             void *hip_stream);

/*
 * Debug check of a tree (the other entry points trust the content of the tree arrays, see the
 * common rules above; Section 2 defines the tree, its root and the mask).  Enqueues one small
 * kernel that writes, for every sequence, a word of PROPD_TREE_* flags, 0 for a consistent tree:
 *   PROPD_TREE_BAD_SIZE    n_nodes[b] outside [1, T_max]
 *   PROPD_TREE_BAD_PARENT  parent[0] != -1, or some parent[i] outside [0, i)
 *   PROPD_TREE_BAD_DEPTH   depth[i] is not the number of edges to the root (skipped if depth is NULL)
 *   PROPD_TREE_BAD_MASK    anc[i] is not the set of nodes on the root path of i (skipped if anc is NULL)
 * flags is a device array [B]; like every call it does not synchronise: read it after the stream
 * has reached this point.  token is not looked at.
 */
enum {
  PROPD_TREE_BAD_SIZE = 1,
  PROPD_TREE_BAD_PARENT = 2,
  PROPD_TREE_BAD_DEPTH = 4,
  PROPD_TREE_BAD_MASK = 8
};
PROPD_API propd_status propd_validate_tree(const propd_tree *tree, int32_t *flags, void *hip_stream);

/*
 * Tree-masked attention (Section 2, "Verification"; Figure 2(b,c)).  For every
 * sequence b, head h and tree node i < T_b:
 *     out[b,h,i,:] = softmax_j( scale * <q[b,h,i,:], k_j> ) . v_j
 * where j runs over all L_b = seq_lens[b] cached prefix tokens and over the tree
 * nodes in anc[b,i] (the node's own candidate sequence, itself included).
 *
 *   dt        PROPD_BF16: tensors are bf16, d in {64, 128}; scores, softmax and
 *             the output accumulation are fp32, the result is rounded to bf16.
 *             (Both run the tiled matrix-core kernel.  d = 128, the head size of every
 *             model of Section 5.1, needs 16-byte aligned tensors and the workspace; d = 64
 *             is served without either, by a plain and far slower kernel.)
 *             PROPD_F32: tensors are fp32, d in {64, 128}, fp32 throughout.
 *   q, k_tree, v_tree, out   [B,H,T_max,d]
 *   k_cache, v_cache         [B,H,L_max,d]; rows >= L_b are never used
 *   seq_lens  [B], 0 <= L_b <= L_max
 *   scale     softmax scale, must be > 0 (1/sqrt(d) in every workload here)
 *   tree      n_nodes and anc are read (token, parent, depth may be NULL)
 *   out       rows i >= T_b are left untouched
 *   workspace propd_workspace_bytes(PROPD_WS_TREE_ATTENTION, ...) bytes
 */
PROPD_API propd_status propd_tree_attention(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t d,
                                  float scale, const void *q, const void *k_cache,
                                  const void *v_cache, const void *k_tree, const void *v_tree,
                                  const int32_t *seq_lens, int32_t L_max, void *out,
                                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Early pruning (Section 4.1, "Pruning Process" and "Implementation
 * Optimization").
 *   1. Early head: for every node p that has children, scores over the vocabulary
 *      z_p = head_weight . hidden_states[b,p,:]  (fp32 accumulation).
 *   2. Top-k test: child c of p fails unless its token is among the top_k best
 *      scores of z_p.  Membership is decided by counting,
 *      rank_c = #{v : z_p[v] > z_p[tok_c]} + #{v < tok_c : z_p[v] == z_p[tok_c]},
 *      fail_c = rank_c >= top_k.  top_k >= vocab prunes nothing.
 *   3. Branch elimination: a node survives iff no node of its root path failed.
 *   4. Survivors are compacted in order; the cached mask is subsampled to the
 *      surviving rows and columns; the listed row payloads are gathered.
 *
 *   hidden_states [B,T_max,hidden]  layer-n hidden state of every tree token
 *   head_weight   [vocab,hidden]    weight of the bias-free early head, one row
 *                                   per vocabulary entry (nn.Linear layout)
 *   dt            PROPD_BF16 (hidden must be a multiple of 32) or PROPD_F32
 *   tree          all five arrays are read; token ids outside [0, vocab) fail
 * Outputs (each fully written, padding included; any may NOT alias an input):
 *   keep_bits  [B,2]      bit i set iff node i survives
 *   new_index  [B,T_max]  position of node i among survivors, -1 if pruned/padding
 *   orig_index [B,T_max]  old index of survivor j, -1 for j >= n_kept[b]
 *   n_kept     [B]        number of survivors (also written to tree_out->n_nodes)
 *   cu_nodes   [B+1]      exclusive prefix sum of n_kept (ragged offsets)
 *   tree_out   compacted tree in the same padded layout, survivors first:
 *              parent re-indexed, token and depth copied, anc subsampled;
 *              slots >= n_kept[b] hold -1 (anc: 0)
 *   rank_out   [B,T_max] or NULL: rank_c as counted (root 0, padding -1, vocab for a token
 *              id outside the vocabulary); ranks of near-equal scores may differ from a
 *              higher-precision evaluation
 *   payloads   host array of n_payloads descriptors (0..PROPD_MAX_PAYLOADS, read
 *              during the call only).  Row (b,o,orig_index[b,j]) of src is copied
 *              to row (b,o,j) of dst for j < n_kept[b]; other dst rows are untouched.
 *   workspace  propd_workspace_bytes(PROPD_WS_EARLY_PRUNE, ...) bytes, 16-byte aligned.  The
 *              scores themselves are never stored: the scratch holds per-node tables and,
 *              for the probability criterion, two floats per score row and 128 columns.
 * hidden_states and head_weight must be 16-byte aligned for PROPD_BF16
 * (PROPD_ERR_INVALID_ARG otherwise).
 * The bf16 scoring kernel chooses its tile shape on the device, from the number of score rows.  The
 * environment variable PROPD_HEAD_PLAN (read once per process; for tuning and
 * tests) overrides the choice: 1 = 256-row tiles, 2 = 352-row tiles (256-row tiles where the hidden
 * states, or 256 rows of the head weight, take 4 GiB or more), unset or 0 = no override (any
 * other value is taken for 1); which nodes survive does
 * not depend on it beyond the order of rounding noted for rank_out.
 */
#define PROPD_MAX_PAYLOADS 8
PROPD_API propd_status propd_early_prune(const propd_tree *tree, propd_dtype dt, int32_t hidden,
                               int32_t vocab, int32_t top_k, const void *hidden_states,
                               const void *head_weight, uint64_t *keep_bits, int32_t *new_index,
                               int32_t *orig_index, int32_t *n_kept, int32_t *cu_nodes,
                               const propd_tree_out *tree_out, int32_t *rank_out,
                               int32_t n_payloads, const propd_payload *payloads,
                               void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Greedy acceptance (Section 3, "acceptance length"; Section 5.1: greedy
 * decoding, so the output equals the large model's own).  With
 * g_i = argmax_v logits[b,i,v] (lowest id among equal maxima), a child is
 * accepted iff its token equals g at its parent and its parent is accepted; the
 * root is always accepted.  The result is the deepest accepted node (lowest
 * index among equally deep ones).
 *
 *   logits      [B,T_max,vocab], dt = PROPD_BF16 or PROPD_F32; rows >= T_b unused
 *   tree        n_nodes, parent, token, anc are read
 *   accept_len  [B]              nodes on the accepted path, root included (>= 1)
 *   accept_path [B,path_stride]  node indices (of the tree passed in) root first,
 *                                -1 padded; entries beyond path_stride are dropped
 *   next_token  [B]              g at the last accepted node
 *   workspace   propd_workspace_bytes(PROPD_WS_ACCEPT_PATH, ...) bytes
 */
PROPD_API propd_status propd_accept_path(const propd_tree *tree, propd_dtype dt, int32_t vocab,
                               const void *logits, int32_t *accept_len, int32_t *accept_path,
                               int32_t path_stride, int32_t *next_token, void *workspace,
                               size_t workspace_bytes, void *hip_stream);

/*
 * propd_accept_path for callers that cannot allocate device memory or pass a workspace:
 * code under HIP graph capture, serving loops and harnesses that forbid hipMalloc.  Same
 * arguments, results and errors as propd_accept_path, minus the workspace: the partial
 * arg-max records go to a fixed array in device memory that belongs to the library (one
 * copy per GPU, PROPD_STATIC_ACCEPT_MAX_NODES * 64 bytes = 512 KB, held until the process
 * ends).  The call allocates nothing and frees nothing.
 *   - B * T_max must not exceed PROPD_STATIC_ACCEPT_MAX_NODES: PROPD_ERR_UNSUPPORTED otherwise.
 *   - hip_stream must belong to the device that is current when the call is made.
 *   - Every call on a GPU uses that GPU's one array: calls that may overlap on one GPU
 *     (different streams, different threads) race.  Nothing in it has to be cleared
 *     between calls: a call reads only records it has written itself.
 */
#define PROPD_STATIC_ACCEPT_MAX_NODES 8192
PROPD_API propd_status propd_accept_path_static(const propd_tree *tree, propd_dtype dt, int32_t vocab,
                               const void *logits, int32_t *accept_len, int32_t *accept_path,
                               int32_t path_stride, int32_t *next_token, void *hip_stream);

/*
 * Early pruning by the probability-based criterion (Section 4.1, "Pruning Criterion", the
 * second of the two criteria; the paper sets it aside because its implementation moved the
 * probabilities to the host - here everything stays on the device).  The early head's scores
 * of a node become probabilities, q_c = softmax(z_p)[tok_c] for a child c of p, and the
 * candidate sequence that ends in node i gets the marginal probability of its tokens,
 * m_i = product of q over the root path of i (root excluded, m_root = 1).  Then either
 *   PROPD_PROB_THRESHOLD  node i goes when m_i < threshold (0 <= threshold <= 1), or
 *   PROPD_PROB_RANK       node i goes when keep_count or more nodes of its tree have a larger
 *                         marginal (equal marginals: the lower node index counts as larger),
 *                         i.e. the keep_count most probable sequences stay (keep_count >= 1).
 * Marginals never grow along a path, so both rules remove whole branches; the root always
 * stays; a token id outside [0,vocab) has probability 0 and always goes.  What follows the
 * decision - compaction, mask subsampling, payload rows, every output - is exactly as in
 * propd_early_prune, with the same arguments, layouts and workspace size.
 *
 *   log_marginal  [B,T_max] fp32 or NULL: log m_i of every node of the INPUT tree (0 for the
 *                 root and for padding), fully written
 * Scores are accumulated in fp32 and the marginals are summed in fp32 as logarithms: a
 * decision can differ from an exact evaluation where log m_i is within about 1e-3 of the
 * boundary.
 */
typedef enum { PROPD_PROB_THRESHOLD = 0, PROPD_PROB_RANK = 1 } propd_prob_mode;
PROPD_API propd_status propd_early_prune_prob(const propd_tree *tree, propd_dtype dt, int32_t hidden, int32_t vocab,
                               propd_prob_mode mode, float threshold, int32_t keep_count,
                               const void *hidden_states, const void *head_weight,
                               uint64_t *keep_bits, int32_t *new_index, int32_t *orig_index,
                               int32_t *n_kept, int32_t *cu_nodes, const propd_tree_out *tree_out,
                               float *log_marginal, int32_t n_payloads,
                               const propd_payload *payloads, void *workspace,
                               size_t workspace_bytes, void *hip_stream);

/*
 * Commit of the accepted path: what a decoding loop does between acceptance and the next
 * step (Section 2, "Verification": the longest verified sequence is kept; Section 5.1:
 * greedy decoding).  With a = accept_len[b] and L = seq_lens[b]:
 *   - the K/V rows of the accepted nodes accept_path[b,0..a-1] (root first) are copied from
 *     k_tree / v_tree to rows L..L+a-1 of k_cache / v_cache, for every head;
 *   - seq_lens[b] becomes L + a;
 *   - out_tokens[b,0..a-2] are the tokens of the accepted candidates (the path without its
 *     root, which was emitted by the step before), out_tokens[b,a-1] = next_token[b], the
 *     rest of the row is -1: the a tokens this step adds to the output, the last of which
 *     is the next step's root.
 * If the cache has room for fewer than a rows, only those that fit are copied and
 * seq_lens[b] stops at L_max; the tokens are still all written.
 *
 *   tree        B, T_max, n_nodes and (for out_tokens) token are read
 *   k_tree,v_tree   [B,H,T_max,d]   dt = PROPD_BF16 or PROPD_F32, d*sizeof a multiple of 16
 *   k_cache,v_cache [B,H,L_max,d]   in/out; rows outside L..L+a-1 are untouched
 *   seq_lens    [B]  in/out
 *   accept_len, accept_path, next_token   as written by propd_accept_path, same path_stride
 *   out_tokens  [B,out_stride] or NULL; entries beyond out_stride are dropped
 * Values read from device memory are made safe rather than reported: seq_lens is clamped to
 * [0, L_max], accept_len to [0, path_stride], and a path entry outside [0, n_nodes[b]) copies
 * no row (its cache row keeps its contents) and gives token -1.
 * No workspace.  Data pointers must be 16-byte aligned (PROPD_ERR_INVALID_ARG otherwise).
 * Must not overlap with a call that reads the same cache or seq_lens.
 */
PROPD_API propd_status propd_commit_path(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t d,
                               const int32_t *accept_len, const int32_t *accept_path,
                               int32_t path_stride, const int32_t *next_token, const void *k_tree,
                               const void *v_tree, void *k_cache, void *v_cache, int32_t L_max,
                               int32_t *seq_lens, int32_t *out_tokens, int32_t out_stride,
                               void *hip_stream);

/*
 * A bounded K/V cache with shared heads: what a decoding loop needs when the model's query heads share
 * K/V heads and the generation is longer than the cache.  A step then is
 *   propd_rotary             positions of the tree's nodes into q and k
 *   propd_grouped_attention  the nodes over the cached rows, with lse
 *   propd_accept_path        (any of the calls above that shape the tree fit in between)
 *   propd_cache_observe      what the accepted nodes paid to every cached row, and the new rows' positions
 *   propd_commit_path        with H = H_kv
 *   propd_cache_evict        the rows that were paid least go, where there are more than `budget`
 * Positions.  seq_lens[b] rows of a sequence's cache are in use, dropped[b] >= 0 positions of the sequence have no
 * row any more (NULL: none), so its next position - that of the tree's root - is P = seq_lens[b] + dropped[b]; a node's is
 * P + its depth, taken from its ancestor set.  position [B,H_kv,L_max] holds the position of every cached row, per
 * K/V head, in any order; NULL: row j has position dropped[b] + j.  A negative entry marks a row that nobody sees.
 * Positions have to be below 2^30.
 *
 * How scores are made of products, for query position p_i and key position p_j:
 *     s = scale * <q_i, k_j>;  cap > 0: s = cap * tanh(s / cap);  slopes: s = s - slopes[h] * (p_i - p_j)
 * and which keys a query sees: cached rows with 0 <= p_j < P, nodes of its ancestor set; of both
 * only those with p_i - p_j < window where window > 0.
 */
typedef struct propd_score_rule {
  float scale;          /* > 0, up to 2^64                                           */
  float cap;            /* 0: scores are not capped; otherwise 2^-10 .. 1024          */
  int32_t window;       /* 0: no window; up to 2^24                                  */
  const float *slopes;  /* [H] or NULL: bias per position of distance, finite        */
} propd_score_rule;

/*
 * Tree attention with shared K/V heads.  Query head h reads K/V head h / (H / H_kv); otherwise as
 * propd_tree_attention, with the rule above:
 *     out[b,h,i,:] = softmax_j(s_ij) . v_j,   lse[b,h,i] = log sum_j exp(s_ij)
 * A single token per sequence is a tree of one node.  A row that sees nothing (only possible where a node's set lacks the
 * node itself) gets zeros, lse -inf.  A key that a query does not see does not touch its result, whatever it holds.
 *
 *   H, H_kv    H a multiple of H_kv
 *   dt, d      PROPD_BF16 or PROPD_F32, d in {64, 128}.  Scores, softmax and sums are fp32.  PROPD_BF16 rounds the result; at d = 128 the
 *              weights that meet V are two bf16 values each (off by 2^-17), at d = 64 three (as they are).
 *   q, out     [B,H,T_max,d]        k_tree, v_tree  [B,H_kv,T_max,d]
 *   k_cache, v_cache  [B,H_kv,L_max,d]; rows >= seq_lens[b] are never used
 *   position, dropped  see above; either may be NULL
 *   tree       n_nodes and anc are read
 *   lse        [B,H,T_max] fp32 or NULL
 *   out and lse rows i >= n_nodes[b] are left untouched
 *   workspace  propd_workspace_bytes(PROPD_WS_GROUPED_ATTENTION, B, T_max, H, d, L_max, 0, 0) bytes
 * q, k_cache, v_cache, k_tree, v_tree, out, anc and workspace must be 16-byte aligned.
 */
PROPD_API propd_status propd_grouped_attention(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t H_kv, int32_t d,
                                     const propd_score_rule *rule, const void *q, const void *k_cache, const void *v_cache,
                                     const void *k_tree, const void *v_tree, const int32_t *seq_lens,
                                     const int32_t *position, const int32_t *dropped, int32_t L_max, void *out, float *lse,
                                     void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * What the accepted nodes paid to every row of the cache, between acceptance and commit of a step.  With the
 * path's nodes n_0 (the root), ..., n_{a-1} = accept_path[b,0..a-1], a = accept_len[b], at positions P, ..., P + a - 1,
 * L = seq_lens[b] and the scores and the visibility of `rule` (node n_r sees the path up to itself):
 *     paid[j] = sum over r and the query heads h of the K/V head of exp(s_rj - lse[b,h,n_r])
 *     weight_out[b,hk,j] = decay * weight[b,hk,j] + paid[j]      position_out[b,hk,j] = position[b,hk,j]     j < L
 *     weight_out[b,hk,L+r] = paid[n_r]                           position_out[b,hk,L+r] = P + r              r < a
 * so that the rows that propd_commit_path appends next have their entries.  Rows that do not fit (L + r >= L_max) are
 * left out, as by the commit; seq_lens[b] + dropped[b] then falls behind by as many.  Entries from there on
 * are left untouched.
 *
 *   q          [B,H,T_max,d]   of the tree that the path indexes     lse  [B,H,T_max], as left by the attention
 *   k_tree     [B,H_kv,T_max,d]     k_cache  [B,H_kv,L_max,d]
 *   accept_len, accept_path, path_stride   as written by propd_accept_path, path_stride up to 65536.  accept_len is clamped to [0, path_stride]; a path
 *              entry outside [0, n_nodes[b]) pays nothing and its row gets weight 0 and position -1; a node whose lse is
 *              -inf (it saw nothing) pays nothing either
 *   position   with position_out, or both NULL: rows in the order of their positions
 *   weight_out, position_out  may be weight and position themselves, but must not overlap them otherwise
 *   decay      0 < decay <= 1
 *   tree       n_nodes is read
 * Every sum is made by one wave in a fixed order.  No workspace.  q, k_cache and k_tree must be 16-byte aligned.
 */
PROPD_API propd_status propd_cache_observe(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t H_kv, int32_t d,
                                 const propd_score_rule *rule, float decay, const int32_t *accept_len,
                                 const int32_t *accept_path, int32_t path_stride, const void *q, const float *lse,
                                 const void *k_cache, const void *k_tree, const int32_t *seq_lens, const int32_t *dropped,
                                 const int32_t *position, const float *weight, int32_t L_max, int32_t *position_out,
                                 float *weight_out, void *hip_stream);

/* Per-row state of a cache, see above. */
typedef struct propd_cache_rows {
  int32_t *seq_lens;  /* [B]                  */
  int32_t *dropped;   /* [B]                  */
  int32_t *position;  /* [B,H_kv,L_max]       */
  float *weight;      /* [B,H_kv,L_max] fp32  */
} propd_cache_rows;

/*
 * Eviction: of every sequence with more than `budget` rows each K/V head keeps `budget` of them,
 * the first of this order:
 *   rows with position >= P - recent or position < sinks (P = seq_lens[b] + dropped[b]), by rising row;
 *   then the others by falling weight, equal weights (0 and -0 are equal) by rising row;
 *   then rows with weight NaN or -inf, and rows with a negative position whatever else holds, by rising row.
 * The kept rows at or beyond `budget` move to the places below it that became free, both in rising order: the k-th of
 * the ones to the k-th of the others.  K, V, position and weight move together, no other row changes,
 * and what lies at or beyond the new length is left as it was.
 *     rows_out->seq_lens[b] = min(L, budget),  rows_out->dropped[b] = dropped[b] + L - that
 * Sequences of at most `budget` rows stay as they are.
 *
 *   k_cache, v_cache  [B,H_kv,L_max,d] in place; d * sizeof a multiple of 16, 16-byte aligned
 *   rows, rows_out    host structs of device arrays, all of them given.  Each array of rows_out may be that of rows, in place, or another one: it
 *                     then gets the entries of the rows kept (position and weight below the new length, nothing else)
 *   budget            1..L_max     recent, sinks  >= 0
 *   workspace         propd_workspace_bytes(PROPD_WS_CACHE_EVICT, B, 0, H_kv, 0, L_max, 0, 0) bytes, 16-byte aligned
 */
PROPD_API propd_status propd_cache_evict(int32_t B, propd_dtype dt, int32_t H_kv, int32_t d, int32_t L_max, int32_t budget,
                               int32_t recent, int32_t sinks, void *k_cache, void *v_cache, const propd_cache_rows *rows,
                               const propd_cache_rows *rows_out, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Rotary positions of one or several axes (for instance time, height and width), for the nodes of a tree or the
 * rows of a prompt.  Pair c of every head is turned by the angle
 *     start[b, axis_of[c]] + offset[b, axis_of[c], s]   times   inv_freq[c],   c < rot / 2
 * (positions as 64-bit sums, angles in 64 bits):  (x, y) -> (x cos - y sin, y cos + x sin).
 *   rot        channels that turn, a multiple of 16, <= d; the others are copied.  Pair c is channels c and c + rot/2, or,
 *              with adjacent != 0, channels 2c and 2c + 1
 *   inv_freq   [rot/2] fp32
 *   n_axes     >= 1         axis_of  [rot/2], clamped to [0, n_axes); NULL: all 0
 *   start      [B,n_axes] or NULL: zeros
 *   offset     [B,offset_axes,S], offset_axes 1 (the same for all axes, for instance a tree's depth) or n_axes
 *   n_rows     [B] or NULL: rows s >= n_rows[b] are left untouched
 *   q [B,H,S,d], k [B,H_kv,S,d] or NULL (with H_kv = 0);  q_out, k_out  of the same shape, q and k themselves or not overlapping
 *   dt         PROPD_BF16 or PROPD_F32, d a multiple of 8; results are fp32, rounded once
 * q, k, q_out and k_out must be 16-byte aligned.
 */
PROPD_API propd_status propd_rotary(propd_dtype dt, int32_t B, int32_t S, int32_t H, int32_t H_kv, int32_t d, int32_t rot,
                          int32_t adjacent, int32_t n_axes, const int32_t *axis_of, const float *inv_freq,
                          const int32_t *start, const int32_t *offset, int32_t offset_axes, const int32_t *n_rows, const void *q,
                          const void *k, void *q_out, void *k_out, void *hip_stream);

/*
 * A paged K/V cache: the rows of all sequences lie in pages of one pool, so that a sequence takes memory as it grows and sequences
 * can share pages of a common prefix.  Row j of sequence b and K/V head h is row j % page_rows of page page_table[b, j / page_rows].  A step then is
 *   propd_rotary, propd_paged_attention, propd_accept_path or propd_accept_sampled, propd_paged_commit
 * (any of the calls above that shape the tree fit in between); prompts enter by propd_paged_prompt, and propd_paged_read
 * gives a sequence to the calls with dense caches.
 *   dt          the dt of the call: rows as they are; or PROPD_E4M3: a row is d codes and one scale, a power of two, held as its exponent
 *               plus 127 in a byte.  A value is code times scale, which bf16 and fp32 hold exactly.
 *   page_rows   a power of two, 16..1024          table_pages * page_rows at most 2^30
 * Entries of page_table outside [0, n_pages) are no pages: rows there are not stored, seen by nobody and read as zeros.  A page
 * that a sequence writes to must be in no other place of the table.
 * A row x is held in 8 bits with the scale 2^e of the smallest e in [-117, 119] with |x| <= 448 * 2^e for every finite value (all zero:
 * e = -117) as the codes x / 2^e, rounded to nearest, ties to even; finite values beyond 448 * 2^119 become that, others are held as NaN.
 */
typedef struct propd_paged_cache {
  void *k_pages, *v_pages;      /* [n_pages,H_kv,page_rows,d]                             */
  uint8_t *k_scale, *v_scale;   /* [n_pages,H_kv,page_rows], PROPD_E4M3 only              */
  const int32_t *page_table;    /* [B,table_pages]                                        */
  propd_dtype dt;
  int32_t n_pages;              /* >= 1                                                   */
  int32_t table_pages;          /* pages of a sequence, at most; >= 1                     */
  int32_t page_rows;
} propd_paged_cache;

/*
 * Tree attention over a paged cache: propd_grouped_attention with row j of the cache at position j.  A single token per sequence is
 * a tree of one node.  K/V rows in 8 bits count as the values that they stand for.
 *   H, H_kv, dt, d, rule, q, out, k_tree, v_tree, tree, lse   as there; the weights that meet V are two bf16 values each (off by
 *              2^-17) for PROPD_BF16
 *   seq_lens   [B], clamped to [0, table_pages * page_rows]
 *   out and lse rows i >= n_nodes[b] are left untouched
 *   v          an infinity or a NaN in a row reaches the nodes that see the row with a score above -inf, however little it weighs, and no others;
 *              a score that is NaN makes a node's results NaN
 *   workspace  propd_workspace_bytes(PROPD_WS_PAGED_ATTENTION, B, T_max, H, d, table_pages * page_rows, 0, 0) bytes
 * q, pages, k_tree, v_tree, out, anc and workspace must be 16-byte aligned.
 */
PROPD_API propd_status propd_paged_attention(const propd_tree *tree, propd_dtype dt, int32_t H, int32_t H_kv, int32_t d,
                                   const propd_score_rule *rule, const void *q, const propd_paged_cache *cache, const void *k_tree,
                                   const void *v_tree, const int32_t *seq_lens, void *out, float *lse, void *workspace,
                                   size_t workspace_bytes, void *hip_stream);

/*
 * propd_commit_path into a paged cache, with H_kv heads and d in {64, 128}.
 *   seq_lens_out  [B]: seq_lens itself or another array.  seq_lens_out[b] = min(seq_lens[b] + accept_len[b], table_pages * page_rows)
 * Values read from device memory are made safe as there.  k_tree, v_tree and pages must be 16-byte aligned.
 * Must not overlap with a call that reads the same pages or lengths.
 */
PROPD_API propd_status propd_paged_commit(const propd_tree *tree, propd_dtype dt, int32_t H_kv, int32_t d, const int32_t *accept_len,
                                const int32_t *accept_path, int32_t path_stride, const int32_t *next_token, const void *k_tree,
                                const void *v_tree, const propd_paged_cache *cache, const int32_t *seq_lens, int32_t *seq_lens_out,
                                int32_t *out_tokens, int32_t out_stride, void *hip_stream);

/*
 * Rows of prompts (or of parts of them) to the ends of their sequences.
 *   k, v     [B,H_kv,S,d], d in {64, 128}       n_rows  [B], clamped to [0, S]; NULL: S
 *   seq_lens, seq_lens_out  as in propd_paged_commit; rows that do not fit are left out
 */
PROPD_API propd_status propd_paged_prompt(propd_dtype dt, int32_t B, int32_t S, int32_t H_kv, int32_t d, const int32_t *n_rows,
                                const void *k, const void *v, const propd_paged_cache *cache, const int32_t *seq_lens,
                                int32_t *seq_lens_out, void *hip_stream);

/*
 * Paged rows as dense ones: row first[b] + s of sequence b goes to row s of k_out and v_out, for s < S and first[b] + s < seq_lens[b]; other
 * rows are left untouched.
 *   first    [B] or NULL: zeros; negative entries count as 0
 *   k_out, v_out  [B,H_kv,S,d] of type dt, d in {64, 128}
 */
PROPD_API propd_status propd_paged_read(propd_dtype dt, int32_t B, int32_t S, int32_t H_kv, int32_t d, const propd_paged_cache *cache,
                              const int32_t *seq_lens, const int32_t *first, void *k_out, void *v_out, void *hip_stream);

/*
 * Acceptance by sampling: drafted tokens against the target's probabilities p_i = softmax(inv_temperature * logits[b,i,:]) at the
 * nodes, with random numbers that the caller gives, so that the tokens of a step are distributed as if the target had been
 * sampled token by token.  From the root on, the children of a node n are tried by rising index until one is accepted:
 *   draft_logits NULL   candidates that were not drawn at random (for instance the top k of a head).  Child c is accepted iff
 *                       u[b,c] * R < p_n(tok_c), R = 1 - the probabilities of the tokens refused before; a token refused before never is.
 *   draft_logits        [B,T_max,vocab]: every child of n was drawn from q_n = softmax(draft_inv_temperature * draft_logits[b,n,:]), independently of its
 *                       siblings.  With r = p_n at first, child c is accepted iff u[b,c] * q_n(tok_c) < r(tok_c); otherwise r becomes max(r - q_n, 0),
 *                       scaled to a sum of 1.
 * The path ends at the first node l none of whose children is accepted.  The token after it is drawn from what is left there (p_l
 * without the tokens refused, or r): the lowest v with r(0) + ... + r(v) > u_next[b].  If nothing is left, it is the likeliest token of p_l (the lowest id among equal ones).
 * As there, a path buffer shorter than the path keeps its first path_stride nodes, and next_token is then the token of the next node.
 *   logits, draft_logits  dt = PROPD_BF16 or PROPD_F32, read for nodes that have children, and logits at the path's end.
 *            NaN counts as -inf (probability 0); several +inf share the probability; a row of -inf alone gives probability 0 throughout.  Finite logits
 *            may be of any size: only their differences to the row's largest count, so that a mask may be the type's lowest value.
 *            16-byte aligned rows are read faster, others are allowed
 *   u        [B,T_max], u_next [B]   fp32 in [0,1); the entries of node 0 and of padding are not used
 *   tree     n_nodes, parent, token are read; a token outside [0, vocab) is refused and changes nothing
 *   inv_temperature, draft_inv_temperature  > 0, up to 2^20
 *   accept_len, accept_path, path_stride, next_token  as in propd_accept_path
 *   workspace  propd_workspace_bytes(PROPD_WS_ACCEPT_SAMPLED, B, T_max, 0, 0, 0, 0, vocab) bytes, 16-byte aligned
 * Probabilities, sums and what is left are held in 64 bits.
 */
PROPD_API propd_status propd_accept_sampled(const propd_tree *tree, propd_dtype dt, int32_t vocab, const void *logits,
                                  float inv_temperature, const void *draft_logits, float draft_inv_temperature, const float *u,
                                  const float *u_next, int32_t *accept_len, int32_t *accept_path, int32_t path_stride,
                                  int32_t *next_token, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Dynamic token-tree generation (Section 4.2): the controller that picks the tree size from
 * measured iteration times and measured head accuracies.  HOST code: every pointer below is
 * a host pointer, nothing is enqueued on a stream, no device is touched.  It is meant to run
 * now and then between decoding steps (Section 4.2.3), not every step.
 *
 * State lives in caller-owned host memory of propd_controller_bytes() bytes, 8-byte aligned,
 * set up once by propd_controller_init(); a state that was not initialised is rejected with
 * PROPD_ERR_INVALID_ARG.  Calls on one state must not overlap.
 *
 *   sizes        [n_sizes] the candidate tree sizes S (root included), strictly rising,
 *                1 <= size <= PROPD_MAX_TREE
 *   n_heads      number of prediction heads; head i proposes the token i+1 places after the root
 *   k_max        candidates per head that the statistics cover
 *   alpha        weight of a new sample in every running mean, 0 < alpha <= 1
 *   lambda       decay of the regression weight with the age of a mean, W = exp(-lambda * age),
 *                in units of 1/`now`
 *   hit_rate_init [n_heads*k_max] or NULL: starting values of P_i^k (frequency of "the true token
 *                is within the top-k of head i", k = 1..k_max), rising in k, within [0,1];
 *                NULL = zeros
 *
 * observe_time   Section 4.2.1: T_perf^size <- (1-alpha) T_perf^size + alpha t (the first
 *                sample of a size starts its mean), and its age restarts at `now`.  `size`
 *                must be one of S.  `now` is the caller's clock in any unit (steps, seconds).
 * observe_hit    Section 4.2.2: P_head^k <- (1-alpha) P_head^k + alpha [rank < k] for every k;
 *                `rank` is the 0-based position of the token that was finally decoded in
 *                that head's candidate list, negative (or >= k_max) when it was not in it.
 * fit            Section 4.2.1: beta0, beta1 minimising sum_i W_i (T_perf^i - beta0 - beta1 i)^2
 *                over the sizes seen so far, closed form.  One size seen: beta1 = 0.  None:
 *                PROPD_ERR_UNSUPPORTED.
 * build_tree     Section 4.2.2: the tree of `size` nodes with the largest estimated acceptance
 *                length, root first, every parent before its children:
 *                  parent[i]  index of the parent (-1 for the root)
 *                  depth[i]   0 for the root; a node at depth d comes from head d-1
 *                  choice[i]  0-based rank of the node's token in its head's list (-1 root)
 *                  node_value[i]  product of the accuracies p_j^(k_j) along its path (root 1)
 *                  *expected_len  sum of the node values
 *                  *n_built   nodes written: `size`, or fewer when the heads have no more
 *                             candidates (n_heads levels of k_max each)
 *                Output arrays hold `size` entries; any of them may be NULL except n_built.
 *                Equal values: the shallower node first, then the earlier parent, then the
 *                lower rank.
 * best_size      Section 4.2.3: speed[j] = l(sizes[j]) / T_est^(sizes[j]) for every candidate
 *                size (0 where the estimated time is not positive), *best_size = the size
 *                with the largest speed (the smaller one on a tie); speed, beta0, beta1 may
 *                be NULL.
 */
PROPD_API size_t propd_controller_bytes(int32_t n_sizes, int32_t n_heads, int32_t k_max);
PROPD_API propd_status propd_controller_init(void *state, size_t state_bytes, const int32_t *sizes,
                               int32_t n_sizes, int32_t n_heads, int32_t k_max, double alpha,
                               double lambda, const double *hit_rate_init);
PROPD_API propd_status propd_controller_observe_time(void *state, int32_t size, double t, double now);
PROPD_API propd_status propd_controller_observe_hit(void *state, int32_t head, int32_t rank);
PROPD_API propd_status propd_controller_fit(const void *state, double now, double *beta0, double *beta1);
PROPD_API propd_status propd_controller_build_tree(const void *state, int32_t size, int32_t *n_built,
                               int32_t *parent, int32_t *depth, int32_t *choice,
                               double *node_value, double *expected_len);
PROPD_API propd_status propd_controller_best_size(const void *state, double now, int32_t *best_size,
                               double *speed, double *beta0, double *beta1);

/* Workspace size in bytes for one call with these dimensions (arguments a call
 * does not have are ignored).  Pure host arithmetic: no device is queried, so the size is
 * the same on every machine and a size asked for before a call is accepted by that call.
 * Returns 0 for a bad `which`. */
typedef enum {
  PROPD_WS_TREE_ATTENTION = 0,
  PROPD_WS_EARLY_PRUNE = 1,
  PROPD_WS_ACCEPT_PATH = 2,
  PROPD_WS_GROUPED_ATTENTION = 3,
  PROPD_WS_CACHE_EVICT = 4, /* H is the number of K/V heads */
  PROPD_WS_PAGED_ATTENTION = 5, /* L_max is table_pages * page_rows */
  PROPD_WS_ACCEPT_SAMPLED = 6
} propd_ws_kind;
PROPD_API size_t propd_workspace_bytes(propd_ws_kind which, int32_t B, int32_t T_max, int32_t H, int32_t d,
                             int32_t L_max, int32_t hidden, int32_t vocab);

/* Static, NUL-terminated description of a status code. */
PROPD_API const char *propd_status_string(propd_status status);

#ifdef __cplusplus
}
#endif
#endif /* PROPD_H */
