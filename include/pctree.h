/*
 * pctree.h -- C ABI of the PCTree per-round draft-tree builder for MI355X (gfx950).
 *
 * One speculative-decoding round of PCTree (Li et al., "From Chains to Trees:
 * Parent-Conditioned Drafting for Semi-Autoregressive Speculative Decoding")
 * turns shared backbone logits L_0..L_{B-1} into a budgeted draft tree:
 *
 *   for every depth d (Sec. 4.1, Alg. 1): the frontier parents are batched
 *   through the Markov head, z_d(p) = L_d + Markov(p) (Eq. 3), each row is
 *   log-softmax normalised (Eq. 2), every parent keeps its top-k children with
 *   joint path scores s(child) = s(p) + log pi_d(child|p) (Eq. 4), and the k
 *   best candidates of the layer become the next frontier; after B stages the
 *   global top-N of the pool (score desc, depth asc, stable id; Sec. 4.2) is
 *   emitted as flat tokens, parent indices, position ids and the ancestor-only
 *   tree attention mask (App. A).
 *
 * The Markov head is Markov_d(p) = W^T . SiLU(E[p] + h_d) with E[V][r],
 * W[r][V] and a per-depth feature h_d[r]; the paper gives only that the head
 * is low-rank and adds a bias set by the preceding token (Sec. 3.2).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every data pointer is a DEVICE pointer on the current HIP device; the
 *    caller owns all memory, the library never allocates or frees.  Inputs
 *    are never written.  Outputs must not overlap inputs or the workspace.
 *  - Data pointers must be 16-byte aligned; the workspace 256-byte aligned.
 *  - `stream` is a hipStream_t (NULL = the default stream).  Calls only
 *    enqueue work: they return before the GPU has run it, do no host<->device
 *    copies and never synchronise.  Results are valid once the stream reaches
 *    that point.  Calls are re-entrant; concurrent calls need distinct
 *    workspaces.  Exception: a round with at most 16 frontier rows (R * k'
 *    <= 16) runs as ONE launch whose workgroups, one per compute unit,
 *    exchange data while they run, so they must all be resident together.
 *    Such rounds must not overlap another round (or other long kernels) on
 *    the same device, e.g. on a second stream: a workgroup that cannot start
 *    makes the others' bounded waits give up (after 2 s), and the round is
 *    then abandoned (see pctree_tree.count).  Rounds on one stream are
 *    always safe.
 *  - Argument checking happens on the host before anything is enqueued; on
 *    any error status no device work has been issued and nothing is written.
 *    No C++ exception crosses this interface.
 *  - Device-side data errors do not fault: a request whose root token lies
 *    outside [0, V) is emitted as an empty tree (count = 0, rows padded).
 *    Floating-point inputs must be finite.
 */
#ifndef PCTREE_H
#define PCTREE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PCTREE_ABI_VERSION 1

/* Compiled limits (PCTREE_ERR_UNSUPPORTED beyond them). */
#define PCTREE_MAX_VOCAB (1 << 20)
#define PCTREE_MAX_BLOCK 63
#define PCTREE_MAX_TOPK 16
#define PCTREE_MAX_BUDGET 256
#define PCTREE_MAX_REQUESTS 256
#define PCTREE_MAX_RANK_BF16 512 /* and rank % 32 == 0 */
#define PCTREE_MAX_RANK_F32 128  /* and rank % 16 == 0 */
#define PCTREE_MAX_MASK_BUDGET 1024
#define PCTREE_MAX_PAGE_SIZE 1024
#define PCTREE_MAX_PAGED_SLOTS (1 << 30) /* max_pages * page_size */

typedef enum pctree_status {
  PCTREE_OK = 0,
  PCTREE_ERR_INVALID_ARGUMENT = 1, /* null pointer, size < 1, bad dtype, misaligned pointer */
  PCTREE_ERR_UNSUPPORTED = 2,      /* beyond the compiled limits, or an unknown mode */
  PCTREE_ERR_WORKSPACE = 3,        /* workspace null, too small or not 256-byte aligned */
  PCTREE_ERR_HIP = 4               /* a kernel launch failed */
} pctree_status;

typedef enum pctree_dtype {
  PCTREE_F32 = 0,  /* float32 base logits and head weights */
  PCTREE_BF16 = 1, /* bfloat16 base logits and head weights, fp32 accumulation */
  PCTREE_F16 = 2   /* float16: paged caches and sampled logits only */
} pctree_dtype;

/* Scoring of a parent's children (Sec. 5.3 compares the three).  Other
 * values are PCTREE_ERR_UNSUPPORTED. */
typedef enum pctree_mode {
  PCTREE_MODE_PARENT = 0,      /* PCTree: every frontier parent p gets its own row
                                  z_d(p) = L_d + Markov_d(p) (Eq. 3)              */
  PCTREE_MODE_SHARED = 1,      /* Shared-Markov tree: the greedy chain of Eq. 1 is
                                  built first and its row at depth d,
                                  z_d(y_{d-1}), serves every parent of depth d     */
  PCTREE_MODE_INDEPENDENT = 2  /* parent-independent per-position scoring (the
                                  DDTree-style scoring named in Sec. 4): every parent
                                  of depth d gets log_softmax(L_d)               */
} pctree_mode;

/* Problem size of one round (symbols of Sec. 4.1). */
typedef struct pctree_shape {
  int32_t vocab;    /* V: vocabulary size                                    */
  int32_t block;    /* B: block size = number of sequential Markov stages    */
  int32_t budget;   /* N: verification node budget, root included            */
  int32_t topk;     /* k: local branching factor (k' = min(k, V) is used)    */
  int32_t rank;     /* r: Markov-head rank                                   */
  int32_t requests; /* R: independent requests built in one call             */
  int32_t dtype;    /* pctree_dtype of base_logits, emb and proj_t           */
  int32_t mode;     /* pctree_mode: how each parent's child row is scored      */
} pctree_shape;

/* Inputs of one round.  Request i uses base_logits[i], depth_feat[i],
 * root_token[i] and prefix_len[i]; emb and proj_t are one drafter's head,
 * shared by every request. */
typedef struct pctree_inputs {
  const void* base_logits;   /* L   [R][B][V] dtype: backbone logits L_d (Sec. 3.2)      */
  const void* emb;           /* E   [V][r] dtype: parent-token embedding of the head     */
  const void* proj_t;        /* W^T [V][r] dtype: proj_t[v*r + j] = W[j][v]              */
  const float* depth_feat;   /* h   [R][B][r] float32: per-depth head feature            */
  const int32_t* root_token; /* x_t [R]: last verified token, root of the tree           */
  const int32_t* prefix_len; /* [R]: verified-prefix length; position = prefix + depth   */
} pctree_inputs;

/* The emitted tree (Sec. 4.2, App. A).  Nodes are in canonical order: depth
 * ascending, then root-to-node token path lexicographically ascending, so
 * node 0 is the root (token x_t, parent -1, depth 0, logprob 0) and
 * parent[i] < i.  Rows i >= count[r] are padded with token = parent = depth =
 * position = -1 and logprob = -inf (mask rows: zero words).
 *
 * count[r] = -1 marks an abandoned round (see the single-launch exception
 * under the conventions above): then every row of every request is padding
 * and every mask word is zero; nothing of an earlier call's tree remains.
 * The call itself has already returned PCTREE_OK, so a caller that may
 * overlap rounds on one device checks count once the stream has run. */
typedef struct pctree_tree {
  int32_t* token;    /* [R][N] draft token ids                                   */
  int32_t* parent;   /* [R][N] index of the parent node in the same row, -1 root */
  int32_t* depth;    /* [R][N] tree depth (root 0)                               */
  int32_t* position; /* [R][N] prefix_len + depth                                */
  float* logprob;    /* [R][N] joint path score s(c) (Eq. 4), root 0             */
  int32_t* count;    /* [R]    min(N, pool size); 0 for an invalid root; -1 if
                        the round was abandoned (all rows padded)             */
  uint32_t* mask;    /* optional (may be NULL): [R][N][(N+31)/32] ancestor mask,
                        bit j%32 of word j/32 of row i is set iff node j is node
                        i or one of its ancestors (same layout as build_mask)    */
} pctree_tree;

/* Optional per-stage record of the frontier (Alg. 1), for inspection.
 * Entry [r][d][s] describes frontier slot s used at stage d: its token, the
 * slot of its own parent in the frontier of stage d-1 (-1 for the root) and
 * its joint score.  Stage 0 holds the root only.  Unused slots hold
 * (-1, -1, -inf). */
typedef struct pctree_trace {
  int32_t* token;       /* [R][B][k] */
  int32_t* parent_slot; /* [R][B][k] */
  float* score;         /* [R][B][k] */
} pctree_trace;

/* Bytes of workspace that pctree_build_tree and pctree_chain_decode need for
 * `shape` (0 if the shape is invalid or unsupported).  Pure host arithmetic. */
size_t pctree_workspace_bytes(const pctree_shape* shape);

/* Build one round's draft tree for every request (Alg. 1, Eq. 2-4, Sec. 4.2,
 * App. A).  `trace` may be NULL.  The workspace's contents on entry do not
 * matter; on return it holds scratch the caller must not rely on. */
pctree_status pctree_build_tree(const pctree_shape* shape, const pctree_inputs* in,
                                const pctree_tree* out, const pctree_trace* trace,
                                void* workspace, size_t workspace_bytes, void* stream);

/* pctree_build_tree for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  The same round with the same kernels and results, but its
 * workspace is a fixed array inside the library, PCTREE_NOALLOC_SCRATCH_BYTES
 * bytes per device (each device the library runs on holds its copy until the
 * process ends); the call allocates and frees nothing.  The caller still
 * provides inputs and outputs.  Errors as for pctree_build_tree, plus
 * PCTREE_ERR_WORKSPACE (before any device work) when the shape needs more
 * than PCTREE_NOALLOC_SCRATCH_BYTES of workspace (pctree_workspace_bytes),
 * and PCTREE_ERR_HIP if the array's device address cannot be looked up.
 * Every call on one device shares that device's array: calls whose rounds
 * can overlap on one device (other streams, other host threads) race and
 * corrupt each other; calls ordered on one stream are safe.  Each call
 * clears what it needs before use. */
#define PCTREE_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)
pctree_status pctree_build_tree_noalloc(const pctree_shape* shape, const pctree_inputs* in,
                                        const pctree_tree* out, const pctree_trace* trace,
                                        void* stream);

/* Ancestor-only tree attention mask from parent indices (App. A): row i of
 * request r admits node i and its ancestors.  parent [R][N], count [R] (as
 * emitted by pctree_build_tree), mask [R][N][(N+31)/32] uint32.  Rows at or
 * beyond count are zero.  A parent index that is not in [-1, i) ends that
 * row's walk.  Limits: N <= PCTREE_MAX_MASK_BUDGET. */
pctree_status pctree_build_mask(const int32_t* parent, const int32_t* count, int32_t requests,
                                int32_t budget, uint32_t* mask, void* stream);

/* The DSpark greedy chain of Eq. 1: y_{-1} = x_t, y_d = argmax_v z_d(y_{d-1})
 * (ties to the lowest token id).  Uses vocab, block, rank, requests, dtype and
 * mode of `shape` (topk and budget are ignored; modes PARENT and SHARED give
 * the same chain, INDEPENDENT the chain of argmax_v L_d).  chain_token [R][B+1] gets
 * x_t, y_0..y_{B-1}; chain_logprob [R][B+1] the cumulative log-probabilities
 * (0 for x_t).  Same workspace as pctree_build_tree.  An abandoned round
 * leaves every chain_token entry -1 and every chain_logprob -inf. */
pctree_status pctree_chain_decode(const pctree_shape* shape, const pctree_inputs* in,
                                  int32_t* chain_token, float* chain_logprob, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------
 * Verification bookkeeping after a round (Sec. 4.2; App. A, "Tensor
 * implementation").  The emitted tree goes through one target forward, which
 * predicts a greedy next token at every node; these calls turn that into the
 * accepted draft and compact the per-node cache entries.  Same conventions as
 * above (device pointers, asynchronous on `stream`, host-side checks only).
 * W = max_depth + 1 is the width of a row; max_depth is normally B.
 * --------------------------------------------------------------------- */

/* Retrieve indices (App. A): one padded root-to-leaf row per leaf.
 * parent [R][N], count [R] as emitted by pctree_build_tree.  A leaf is a node
 * i < count that is no node's parent; leaf q in ascending node order gets row
 * q of rows [R][N][W]: the node indices from the root down to the leaf,
 * padded with -1.  nrows [R] = number of leaves; rows past it are all -1.
 * Malformed trees do not fault: a parent index outside [0, i) ends the
 * upward walk from node i (that node then heads its row), and a path longer
 * than W keeps its first W nodes from the head.
 * Limits: N <= PCTREE_MAX_MASK_BUDGET, max_depth <= PCTREE_MAX_BLOCK. */
pctree_status pctree_build_retrieve(const int32_t* parent, const int32_t* count, int32_t requests,
                                    int32_t budget, int32_t max_depth, int32_t* rows,
                                    int32_t* nrows, void* stream);

/* Greedy tree acceptance (Sec. 4.2: the standard greedy tree rule; App. A).
 * token [R][N] draft tokens; rows [R][N][W] and nrows [R] from
 * pctree_build_retrieve; target_next [R][N] the target's greedy next token
 * after each node.  Along a row, position l >= 1 is accepted while
 * token[row[l]] == target_next[row[l-1]]; the row accepting the most
 * positions wins (the lowest row on ties).  Outputs per request:
 * accept_len [R] accepted draft tokens (root excluded), accept_row [R] the
 * winning row (-1 if there is none), accept_node [R][W] its accepted node
 * indices from the root, padded with -1, and bonus [R] = target_next at the
 * last accepted node (-1 if there is no row).  A row entry outside [0, N)
 * ends that row.  Limits as for pctree_build_retrieve. */
pctree_status pctree_accept_greedy(const int32_t* token, const int32_t* rows,
                                   const int32_t* nrows, const int32_t* target_next,
                                   int32_t requests, int32_t budget, int32_t max_depth,
                                   int32_t* accept_len, int32_t* accept_row,
                                   int32_t* accept_node, int32_t* bonus, void* stream);

/* Compaction after acceptance (App. A): the cache entries of the accepted
 * row move right after the verified prefix.  `cache` holds, per request and
 * group (e.g. one layer's K or V, or the target hidden states), `capacity`
 * slots of slot_bytes each, contiguous: slot s of group g of request r starts
 * at cache + r*request_stride + g*group_stride + s*slot_bytes.  Tree node i
 * sits at slot prefix_len[r] + i; the accepted nodes n_0..n_a
 * (accept_node [R][W], accept_len [R] from pctree_accept_greedy) move, in
 * place, to slots prefix_len[r] + 0..a.  Other slots keep their contents.
 * A request whose accepted nodes are not strictly increasing, not below N,
 * or reach past `capacity` is left untouched.  slot_bytes, both strides and
 * `cache` must be multiples of 16. */
pctree_status pctree_compact_kv(void* cache, int64_t request_stride, int64_t group_stride,
                                int32_t groups, int32_t capacity, int32_t slot_bytes,
                                const int32_t* prefix_len, const int32_t* accept_node,
                                const int32_t* accept_len, int32_t requests, int32_t budget,
                                int32_t max_depth, void* stream);

/* ---------------------------------------------------------------------
 * Tree-masked verification attention (Sec. 4.2: the packed tree is verified
 * in one target forward; App. A, "Tensor implementation": a node attends to
 * the verified prefix, itself and its root-to-node ancestors).  One
 * attention layer of the target, grouped-query heads, bf16 operands, fp32
 * accumulation and softmax, bf16 output.
 * --------------------------------------------------------------------- */

typedef struct pctree_attn_shape {
  int32_t requests; /* R                                                        */
  int32_t budget;   /* N: tree rows per request, as emitted by the builder      */
  int32_t q_heads;  /* Hq                                                       */
  int32_t kv_heads; /* Hkv, a divisor of Hq; query head h reads kv head h/(Hq/Hkv) */
  int32_t head_dim; /* D: 64 or 128                                             */
  int32_t capacity; /* C: cache slots per request and kv head                   */
  float scale;      /* softmax scale of q.k, > 0, usually 1/sqrt(D)             */
} pctree_attn_shape;

/* Workspace bytes pctree_tree_attention needs for `shape` (0: none, or an
 * invalid shape).  Pure host arithmetic. */
size_t pctree_attention_workspace_bytes(const pctree_attn_shape* shape);

/* out[r][i][h] = sum_s softmax_s(scale * q[r][i][h] . k[r][h/g][s]) v[r][h/g][s]
 * over the admitted slots s of tree node i: the prefix [0, prefix_len[r]) and
 * prefix_len[r] + j for every bit j < count[r] set in mask row i (cache slot
 * prefix_len + j holds tree node j, as after pctree_compact_kv's layout).
 * q [R][N][Hq][D], k_cache and v_cache [R][Hkv][C][D], out [R][N][Hq][D],
 * all bf16 (uint16 bits), 16-byte aligned; mask [R][N][(N+31)/32] as from
 * pctree_build_mask; count [R], prefix_len [R] int32 device arrays.
 * Rows i >= count[r], and rows that admit no slot, are zero.  prefix_len
 * and count are clamped to [0, C] and [0, N], and slots at or past C are
 * never read; slots at or past prefix_len + count are never read either,
 * so they may hold anything.  Admitted slots must hold finite values.
 * Errors: INVALID_ARGUMENT (null or misaligned pointer, size < 1, Hq not a
 * multiple of Hkv, scale not positive and finite), UNSUPPORTED (D not 64 or 128,
 * N > PCTREE_MAX_MASK_BUDGET, R or Hkv > 65535, sizes past the index range),
 * WORKSPACE (a needed workspace null, too small or not 256-byte aligned). */
pctree_status pctree_tree_attention(const pctree_attn_shape* shape, const void* q,
                                    const void* k_cache, const void* v_cache,
                                    const uint32_t* mask, const int32_t* count,
                                    const int32_t* prefix_len, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------
 * The target's verification step over a paged cache (Sec. 4.2: "one target
 * forward"; App. A): a target that serves many requests keeps its keys and
 * values in pages of a pool.  pctree_append_paged norms and rotates the new
 * rows' queries and keys and puts keys and values into their pages,
 * pctree_paged_attention lets a chunk of new rows (part of a prompt, one
 * token, or a tree) attend to the request's pages, pctree_sample draws the
 * target's token at every row, and pctree_compact_paged is pctree_compact_kv
 * for pages.
 *
 * Slot s of request r is slot s % page_size of page page_table[r][s / page_size].
 * A page index outside [0, pages) is no page: its slots are neither read nor
 * written and are admitted by no row (so unused entries may hold anything).
 * --------------------------------------------------------------------- */

/* One layer's keys and values. */
typedef struct pctree_paged_cache {
  void* k;             /* [pages][Hkv][page_size][D] dtype                              */
  void* v;             /* the same layout                                               */
  int64_t page_stride; /* elements between two pages of k (and of v): a multiple of 8,
                          at least Hkv * page_size * D; more than that where pages lie
                          in a larger pool                                              */
  int32_t pages;       /* pages of the pool                                             */
  int32_t page_size;   /* slots of a page: a power of two, at most PCTREE_MAX_PAGE_SIZE */
  int32_t kv_heads;    /* Hkv                                                           */
  int32_t head_dim;    /* D: 64 or 128                                                  */
  int32_t dtype;       /* PCTREE_BF16 or PCTREE_F16                                     */
} pctree_paged_cache;

/* Which rows of a call belong to which request.  Row row_start[r] + i, i <
 * row_count[r], is request r's i-th new row and sits at slot prefix_len[r] + i.
 * Rows of different requests must not overlap; rows of no request are neither
 * read nor written.  Device arrays, so one captured graph serves changing
 * batches; what they hold is clamped: a start outside [0, rows] gives no rows,
 * counts to [0, min(max_rows, rows - start)], prefixes to [0, capacity], with
 * capacity = max_pages * page_size.  Slots at or past capacity do not exist. */
typedef struct pctree_paged_batch {
  const int32_t* row_start;  /* [R]                                          */
  const int32_t* row_count;  /* [R]                                          */
  const int32_t* prefix_len; /* [R] slots in the cache before the new rows   */
  const int32_t* page_table; /* [R][max_pages]                               */
  int32_t requests;          /* R                                            */
  int32_t max_pages;         /* width of the page table                      */
  int32_t rows;              /* T: rows of q, k, v and out, below 2^24       */
  int32_t max_rows;          /* the most rows that a request has, <= rows (work is
                                planned for it: more than the true most costs
                                workgroups that find nothing)                */
} pctree_paged_batch;

/* New rows of one layer.  Head h of row t starts at element t * row_stride +
 * h * D (so a fused projection's output needs no split); strides and pointers
 * are multiples of 8 elements and 16 bytes. */
typedef struct pctree_append {
  const void* q;           /* [T][Hq][D], or NULL: keys and values only               */
  const void* k;           /* [T][Hkv][D]                                             */
  const void* v;           /* [T][Hkv][D]                                             */
  void* q_out;             /* [T][Hq][D] (may be q itself); NULL iff q is             */
  int64_t q_stride;        /* row strides in elements, >= heads * D                   */
  int64_t k_stride;
  int64_t v_stride;
  int64_t q_out_stride;
  const void* q_norm;      /* [D] dtype weight of the queries' norm, or NULL: none    */
  const void* k_norm;      /* [D] dtype weight of the keys' norm, or NULL: none       */
  const float* rope;       /* [positions][rot_dim]: cos of the position's rot_dim / 2
                              angles, then their sines; or NULL: no rotation          */
  const int32_t* position; /* [T], or NULL: a row's position is its slot              */
  float eps;               /* of the norms, >= 0                                      */
  int32_t q_heads;         /* Hq (0 where q is NULL)                                  */
  int32_t rot_dim;         /* rotated leading elements of a head: a multiple of 16, <= D */
  int32_t positions;       /* rows of rope                                            */
  int32_t interleaved;     /* 0: element i turns with i + rot_dim / 2; 1: 2 i with 2 i + 1 */
} pctree_append;

/* For every row t of a request: y = x * rsqrt(mean(x^2) + eps) * weight per
 * head of q and k (where there is a weight), then (a, b) -> (a cos - b sin,
 * b cos + a sin) for the pairs of the first rot_dim elements; q goes to q_out,
 * k and the unchanged v to the row's slot.  float32 throughout, one rounding
 * at the end.  A position outside [0, positions) is clamped to that range.
 * Rows whose slot does not exist only have their q written. */
pctree_status pctree_append_paged(const pctree_paged_cache* cache, const pctree_paged_batch* batch,
                                  const pctree_append* rows, void* stream);

/* Workspace bytes pctree_paged_attention needs (0: none, or invalid arguments).
 * Depends on sizes only (head counts, D, requests, max_pages, page_size, rows,
 * max_rows), not on pointers.  Pure host arithmetic. */
size_t pctree_paged_attention_workspace_bytes(const pctree_paged_cache* cache,
                                              const pctree_paged_batch* batch, int32_t q_heads);

/* out[t][h] = sum_s softmax_s(scale * q[t][h] . k[s][h/g]) v[s][h/g], g = Hq /
 * Hkv, for every row t of a request, over the admitted slots s:
 * - mask NULL: causal; the request's i-th row admits [0, prefix + i];
 * - else its row i admits the prefix and prefix + j for every bit j < count of
 *   mask row [r][i] ([R][budget][(budget+31)/32], as from pctree_build_mask);
 *   counts are also clamped to budget.
 * q and out [T][Hq][D] dtype, contiguous; float32 scores, softmax and sums, the
 * weights rounded to dtype before the weighted sum.  Rows that admit no slot
 * are zero.  The pages must already hold the new rows' keys and values
 * (pctree_append_paged).  A slot that a row does not admit adds nothing to that
 * row, whatever it holds (infinities and NaN included); an infinite or NaN
 * value that a row admits makes that element of it non-finite.
 * Errors: as for pctree_tree_attention; UNSUPPORTED also for a page_size that
 * is no power of two or beyond its limit, R > 65535, and
 * max_pages * page_size > PCTREE_MAX_PAGED_SLOTS. */
pctree_status pctree_paged_attention(const pctree_paged_cache* cache,
                                     const pctree_paged_batch* batch, const void* q,
                                     int32_t q_heads, float scale, const uint32_t* mask,
                                     int32_t budget, void* out, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* Sampling: a token for every row of logits, from given random numbers.  Row t
 * of logits starts at element t * row_stride (>= vocab).  temperature, top_k,
 * top_p and min_p are [rows] device arrays or NULL (1, off, off, off).
 *
 * With weights w_i = e^((l_i - max l) / temperature), of the row's tokens are kept,
 * in turn: those with w_i >= min_p (off at min_p <= 0; the largest always stay);
 * the top_k with the largest logits (off at top_k <= 0); the fewest with the
 * largest logits whose weights sum to at least top_p times the sum of those left
 * (off at top_p >= 1; at least one stays).  Equal logits rank by token id.  The
 * token is the first kept one, by id, at which the running sum of kept weights
 * exceeds uniform * (their total): uniform in [0, 1), values outside are clamped
 * (1 and more: the last kept token of positive weight).  logprob (may be NULL) is
 * the log of the token's share of the kept weights.
 *
 * A temperature of 0 (or below, or NaN) takes the first largest logit, logprob 0.
 * A logit of -inf (a masked token) or NaN is never taken; a row of nothing else
 * gives token -1, logprob -inf; +inf logits share the row among themselves.
 * Weights below e^-700 count as 0; a NaN uniform as 0, a NaN top_p or min_p as
 * off.  Weights and their sums are float64, added in an order that depends on
 * the row and its alignment alone: it gives the same token whatever else is in
 * the call.
 *
 * The sampled tokens of a tree's nodes are the target_next of
 * pctree_accept_greedy: following the children that match them is then sampling
 * from the target (Sec. 4.2's lossless verification without greedy decoding).
 *
 * dtype: PCTREE_F32, PCTREE_BF16 or PCTREE_F16; logits aligned to one element.
 * Errors: INVALID_ARGUMENT (null or misaligned pointer, size < 1, row_stride <
 * vocab, bad dtype), UNSUPPORTED (vocab > PCTREE_MAX_VOCAB, more than 2^31 - 1
 * blocks of 512 logits in all), WORKSPACE. */
size_t pctree_sample_workspace_bytes(int32_t rows, int32_t vocab);

pctree_status pctree_sample(const void* logits, int32_t dtype, int32_t rows, int32_t vocab,
                            int64_t row_stride, const float* uniform, const float* temperature,
                            const int32_t* top_k, const float* top_p, const float* min_p,
                            int32_t* token, float* logprob, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Compaction in pages: pool holds, per group (e.g. one layer's K or V), `pages`
 * pages of [heads][page_size][slot_bytes]; group g's page p starts at byte
 * g * group_stride + p * page_stride.  Tree node i of request r sits at slot
 * prefix_len[r] + i; the accepted nodes n_0..n_a (accept_node [R][W],
 * accept_len [R] from pctree_accept_greedy) move, in place, to slots
 * prefix_len[r] + 0..a.  Other slots keep their contents.  A request is left
 * untouched if its accepted nodes are not strictly increasing, not below
 * budget, or lie on (or move to) slots that do not exist.  slot_bytes and the
 * strides are multiples of 16; no page of a group overlaps one of another. */
pctree_status pctree_compact_paged(void* pool, int64_t group_stride, int64_t page_stride,
                                   int32_t groups, int32_t pages, int32_t heads,
                                   int32_t page_size, int32_t slot_bytes,
                                   const int32_t* page_table, int32_t max_pages,
                                   const int32_t* prefix_len, const int32_t* accept_node,
                                   const int32_t* accept_len, int32_t requests, int32_t budget,
                                   int32_t max_depth, void* stream);

/* Static, human-readable name of a status code. */
const char* pctree_status_string(pctree_status status);

/* PCTREE_ABI_VERSION of the loaded library. */
int32_t pctree_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* PCTREE_H */
