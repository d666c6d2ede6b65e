/*
 * mpv.h -- batched lossless multi-path verification of draft token trees on one
 * AMD MI355X (gfx950).  C ABI; no C++ or PyTorch types cross this boundary.
 *
 * The operation (paper Sec. 2, step 3 "Verification"): for each of B draft trees
 * that share one shape, given the target and draft logits of every node, accept
 * one node of the tree and draw one correction ("bonus") token so that the
 * emitted tokens follow the target model's distribution.
 *
 * Tree (Sec. 3, Def. 3.1; Sec. 3.2 root expansion; Sec. 5, Def. 5.2 delayed
 * expansion): node 0 is the root (the current context; it has logits but no
 * token).  parent[n] < n is the parent of node n >= 1.  The ordered child list
 * of a node is its children in ascending node index.  Sibling tokens are assumed
 * to be i.i.d. draws from the draft distribution of their parent; equal tokens
 * under one parent are separate nodes with separate rows.
 *
 * Node distributions (Sec. 3; Sec. 4.1 temperatures): p = softmax(z_target / T),
 * q = softmax(z_draft / T) over the full vocabulary, the same T for both.
 *
 * Methods:
 *   MPV_METHOD_SPECINFER  top-down walk of Sec. 3.2 with the SpecInfer solver of
 *                         App. B, Alg. 4 (children tried in list order; a child x
 *                         is accepted with min(1, p(x)/q(x)), otherwise
 *                         p <- normalise((p - q)_+)); when no child is accepted the
 *                         bonus token is drawn from the current p.
 *   MPV_METHOD_TRAVERSAL  bottom-up Traversal Verification (Sec. 3.2), with the
 *                         block-verification weights of Sec. 3.1:
 *                         w(child) = min(1, w(node) * P(x)/q(x)); leaves are tested
 *                         first in depth-first order; when a whole child subtree
 *                         is rejected the node's weight a and distribution P become
 *                         S/(S+1-a) and (a*P - q)_+/S with S = sum (a*P - q)_+.
 *                         The root is always accepted when reached.
 *   MPV_METHOD_NSS        top-down walk of Sec. 3.2 with the NSS solver of App. B,
 *                         Alg. 1: at every node a token is drawn from p; if it is
 *                         the token of a child the walk moves there (to the first
 *                         such child in list order), otherwise it ends and the
 *                         drawn token is the bonus token.  Draft logits are unused.
 *   MPV_METHOD_NAIVE      the same walk with the Naive solver of App. B, Alg. 2: the
 *                         first child x is accepted with min(1, p(x)/q(x)); otherwise
 *                         a token is drawn from (p - q)_+ and followed as above.
 *   MPV_METHOD_SPECTR     the same walk with the SpecTr solver (K-SEQ) of App. B, Alg. 3:
 *                         with rho* the root of 1 - (1 - beta(rho))^k = rho beta(rho) on [1,k],
 *                         beta(rho) = sum min(p/rho, q), the children are tested in list order
 *                         with min(1, p(x)/(rho* q(x))); otherwise a token is drawn from
 *                         (p - gamma min(p/rho*, q))_+, gamma = (1 - (1 - beta)^k)/beta, which at
 *                         rho* (where gamma = rho*) is (p - rho* q)_+.  The equation is solved in the
 *                         form sum (p - rho q)_+ = (sum (q - p/rho)_+)^k, the same numbers without
 *                         cancellation, by Newton's method to a relative 3e-8.
 *
 * Randomness: the caller supplies one uniform in [0,1) per node and tree.
 * uniforms[b,n] (n >= 1) is used only by the test of node n ("accept iff u < a");
 * uniforms[b,0] draws the bonus token by inverse CDF in vocabulary order
 * (smallest t whose cumulative residual mass exceeds u times the total).
 * NSS, NAIVE and SPECTR draw a token at every node they visit: the draw at node n uses
 * draw_uniforms[b,n], a second array of the same shape.
 *
 * All calls are thread-compatible, not thread-safe per stream.  No call
 * allocates or frees device memory or synchronises the device.
 */
#ifndef MPV_H
#define MPV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MPV_ABI_VERSION 10

/* limits (larger requests return MPV_ERR_UNSUPPORTED) */
#define MPV_MAX_NODES    64   /* nodes per tree, root included            */
#define MPV_MAX_CHILDREN 16   /* children of one node                      */
#define MPV_MAX_VOCAB    (1 << 21)
#define MPV_MAX_HEAD_DIM 256  /* values of one attention head               */
#define MPV_MAX_HEADS    1024 /* query heads                                */
/* and B * (N + 2) <= 2^30 */

#define MPV_METHOD_SPECINFER 0
#define MPV_METHOD_TRAVERSAL 1
#define MPV_METHOD_NSS       2
#define MPV_METHOD_NAIVE     3
#define MPV_METHOD_SPECTR    4

#define MPV_DTYPE_F32  0      /* IEEE binary32 logits: finite, or -inf for a token of probability zero.  A
                               * logit z with z log2(e)/T below -2^31 (a mask of -1e10) counts as -inf. */
#define MPV_DTYPE_BF16 1      /* bfloat16 logits (upper half of binary32).  Finite values must lie
                               * within +-65504; magnitudes below 2^-14 are used to within 2^-25
                               * (an error of log2(e)/T * 2^-25 in the exponent of e^(z/T): nothing
                               * for T >= 0.01).  -inf marks a token of probability zero.        */
#define MPV_DTYPE_F16  2      /* IEEE binary16: the calls around a verification only (mpv_tree_attention,
                               * mpv_verify_chains, mpv_append_paths); logits are F32 or BF16.        */

/* error codes: 0 = success, negative = failure (nothing was launched unless the
 * code is MPV_ERR_HIP, in which case some kernels may already be enqueued) */
#define MPV_OK                   0
#define MPV_ERR_NULL            -1   /* a required pointer is NULL                   */
#define MPV_ERR_BAD_SHAPE       -2   /* B < 0, N < 1, V < 1, max_depth < tree depth; a size or stride of
                                        the calls around a verification that cannot be   */
#define MPV_ERR_BAD_TREE        -3   /* parent[0] != -1 or parent[n] not in [0, n)    */
#define MPV_ERR_BAD_TEMPERATURE -4   /* T is not a finite number > 0                  */
#define MPV_ERR_BAD_METHOD      -5
#define MPV_ERR_BAD_DTYPE       -6
#define MPV_ERR_WORKSPACE       -7   /* workspace NULL, misaligned or too small       */
#define MPV_ERR_UNSUPPORTED     -8   /* beyond MPV_MAX_*; stats / edge_probs with methods >= 2;
                                        acceptance rates of MPV_METHOD_TRAVERSAL        */
#define MPV_ERR_HIP             -9   /* a HIP call failed; see mpv_last_hip_error()   */
#define MPV_ERR_ALIGNMENT      -10   /* a logit base pointer (or a pointer, stride or row length of the calls
                                        around a verification) is not a multiple of 16 bytes */
#define MPV_ERR_BAD_TOP_P      -11   /* top_p is not in (0, 1]                        */

/* Problem description.  Host memory, read during the call only. */
typedef struct mpv_problem {
    int32_t B;              /* trees in the batch (0 is allowed: nothing to do)      */
    int32_t N;              /* nodes per tree, root included                         */
    int32_t V;              /* vocabulary size                                       */
    int32_t method;         /* MPV_METHOD_*                                          */
    int32_t logit_dtype;    /* MPV_DTYPE_*                                           */
    float   temperature;    /* T > 0, applied to target and draft rows alike         */
    int32_t max_depth;      /* row width of path_nodes / path_tokens, >= tree depth  */
    const int32_t* parent;  /* HOST pointer, length N, shared by all trees           */
} mpv_problem;

/* Device buffers, all caller-owned, borrowed until the enqueued work has run.
 * Row-major, innermost index contiguous. */
typedef struct mpv_buffers {
    /* inputs */
    const void*    target_logits;  /* [B,N,V] of logit_dtype; every row may be read           */
    const void*    draft_logits;   /* [B,N,V] of logit_dtype; rows of leaves are never read   */
    const int32_t* tokens;         /* [B,N]; tokens[b,0] ignored; others in [0,V)             */
    const float*   uniforms;       /* [B,N] in [0,1)                                          */
    /* outputs */
    int32_t*  accept_len;          /* [B]   depth tau of the accepted node                    */
    int32_t*  path_nodes;          /* [B,max_depth] node indices root-to-accepted, -1 padded  */
    int32_t*  path_tokens;         /* [B,max_depth] their tokens, -1 padded                   */
    int32_t*  bonus_token;         /* [B]   the correction token                              */
    uint32_t* counters;            /* [MPV_COUNTER_COUNT] see MPV_COUNTER_*; zeroed by the call */
    /* optional debug outputs (NULL = not wanted) */
    float* stats;                  /* [B,N,4] m_t, logZ_t, m_d, logZ_d: row maximum and
                                      ln sum exp((z-m)/T); draft entries of leaves are NaN    */
    float* edge_probs;             /* [B,N,2] p(x_n), q(x_n) under the parent's softmax; n=0: 1,1 */
    float* accept_prob;            /* [B,N] probability node n is tested with when reached; n=0: 1 */
    float* final_residual;         /* [B,V] normalised distribution the bonus token is drawn from */
    /* input of MPV_METHOD_NSS, MPV_METHOD_NAIVE and MPV_METHOD_SPECTR only (else ignored, may be NULL) */
    const float*   draw_uniforms;  /* [B,N] in [0,1): the draw at node n                          */
} mpv_buffers;

#define MPV_COUNTER_NEAR_TIE_ACCEPT 0  /* tests on the accepted walk with |a - u| < 1e-6     */
#define MPV_COUNTER_NEAR_TIE_BONUS  1  /* bonus draws within 1e-6 (relative) of a CDF step   */
#define MPV_COUNTER_ZERO_MASS       2  /* residual updates that found zero mass              */
#define MPV_COUNTER_BAD_TOKEN       3  /* tokens outside [0,V) (treated as never accepted)   */
#define MPV_COUNTER_DEPENDENCY_TIMEOUT 4 /* must stay 0: a node task gave up waiting for its
                                            parent's result (results of that tree are invalid) */
#define MPV_COUNTER_NODE_TASKS_RUN   5  /* (tree, internal node) pairs whose logit rows were
                                          read; the others were proved irrelevant first      */
#define MPV_COUNTER_NODE_TASKS_CANCELLED 6 /* node tasks that had been queued ahead of need and
                                          were dropped unread once their tree was settled     */
#define MPV_COUNTER_NODE_TASKS_RESUMED 7 /* second reads of a row pair: where a tree branches, a
                                          node may first explore its first child's subtree and
                                          come back for the rest only if nothing was accepted  */
#define MPV_COUNTER_COUNT           8  /* length of the counters array        */

/* ABI version of the loaded library (MPV_ABI_VERSION it was built with). */
int mpv_version(void);

/* Static, never-freed description of an error code. */
const char* mpv_strerror(int code);

/* The hipError_t (as int) of the most recent failing HIP call made by this
 * library on the calling thread, 0 if none. */
int mpv_last_hip_error(void);

/* Bytes of device scratch mpv_verify needs for this problem (depends on B, N and
 * the tree only).  Writes *out; returns MPV_OK or an error for an invalid problem. */
int mpv_workspace_bytes(const mpv_problem* problem, size_t* out);

/* Enqueue the whole verification of the batch on `hip_stream` (a hipStream_t
 * passed as void*; NULL = the default stream) and return without waiting.
 * `workspace` is DEVICE memory, 256-byte aligned, of at least
 * mpv_workspace_bytes() bytes, owned by the caller; its contents on entry are
 * ignored and on exit unspecified.  Two calls that share a workspace or output
 * buffers must be ordered by the caller (same stream, or events).
 * The work is done by persistent workgroups grouped in teams; a team takes tasks
 * only once all its workgroups are running, so a call makes progress with whatever
 * share of the device it gets (another kernel, or another call on another stream,
 * may hold compute units).  Every wait inside is bounded (2 s): a launch starved
 * for longer than that gives up and reports it in counters[MPV_COUNTER_DEPENDENCY_TIMEOUT],
 * in which case its outputs are invalid. */
int mpv_verify(const mpv_problem* problem, const mpv_buffers* buffers,
               void* workspace, size_t workspace_bytes, void* hip_stream);

/* mpv_verify for callers that cannot allocate device memory or pass a workspace (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same operation,
 * arguments, outputs and errors as mpv_verify, with the scratch in a device array of
 * MPV_STATIC_WORKSPACE_BYTES that is part of the library itself (every GPU the library runs on
 * holds its own copy until the process ends).  The call allocates nothing and frees nothing.
 * A problem whose mpv_workspace_bytes() exceeds MPV_STATIC_WORKSPACE_BYTES is refused with
 * MPV_ERR_WORKSPACE before anything is launched (B * N of about 60 000 nodes fits).
 * Every call on one GPU uses that GPU's one array: calls that overlap in time on the same GPU
 * (different streams, different threads) race and must be ordered by the caller.  The array keeps
 * the previous call's contents; the call itself clears what it needs. */
#define MPV_STATIC_WORKSPACE_BYTES (4u << 20)
int mpv_verify_static(const mpv_problem* problem, const mpv_buffers* buffers, void* hip_stream);

/* Draft trees whose nodes are distinct contexts (Sec. 3, Def. 3.1 and its footnote; Sec. 5, Def. 5.2:
 * paths can overlap after the branching node).  Drafting lays every tree out as `parent` says, each
 * path owning its slots (one row pair, one token, one uniform per slot).  In the tree of Def. 3.1
 * slots drafted for the same context are one node, and the child list of a node keeps one entry per
 * drafted token, in slot order, so it can name the same child several times.
 * mpv_merge_duplicates builds that tree for each of the B token assignments without moving data:
 *   merged_parent[b,n] = the node of the context slot n was drafted after (-1 for n = 0);
 *   context_node[b,n]  = the node of slot n's own context: the first slot (lowest index) drafted for
 *                        it; n itself unless n is a later entry for the same token ("repeat").
 * In merged_parent a repeat has no children (they hang under context_node[b,n] instead), and
 * merged_parent[b,n] < n still holds.  Rows of one context are expected to be equal (the models are
 * functions of the context); only the rows of context nodes matter.
 * parent: HOST [N]; tokens: HOST int32 [B,N] (tokens[b,0] ignored); merged_parent: HOST int32 [B,N],
 * written; context_node: HOST int32 [B,N], written, or NULL.  Host work only: no GPU is touched.
 * Errors: MPV_ERR_NULL, _BAD_SHAPE (B < 0, N < 1), _UNSUPPORTED (N > MPV_MAX_NODES), _BAD_TREE. */
int mpv_merge_duplicates(const int32_t* parent, const int32_t* tokens, int32_t B, int32_t N,
                         int32_t* merged_parent, int32_t* context_node);

/* mpv_verify for a batch in which every tree has a shape of its own: merged_parent is a HOST int32
 * [B,N] array, row b the parent array of tree b (as mpv_merge_duplicates writes it; any valid parent
 * arrays will do).  problem->parent is not read.  Everything else (buffers, layouts, workspace size:
 * what mpv_workspace_bytes gives for a problem of the same B and N, outputs, counters summed over the
 * batch, errors) is as for mpv_verify; path_nodes name context nodes.
 * Why a repeat may be a leaf here: under the SpecInfer solver and under Traversal Verification it is
 * tested only after the first entry for its token was rejected, which leaves that token no residual
 * mass: it is tested with probability 0 and only its residual step remains (App. B, Alg. 4); NSS and
 * Naive move to the first child that carries the drawn token, which is the context node.  SpecTr
 * (App. B, Alg. 3) tests every entry with the entry's own uniform and can accept a repeat; the walk
 * then goes on at the context node.  For that, MPV_METHOD_SPECTR needs context_node: DEVICE int32
 * [B,N], what mpv_merge_duplicates wrote (copied to the device by the caller), borrowed like the
 * buffers; an entry outside [0,N) is ignored (the walk stays at the accepted entry); with the other
 * methods the argument is not read and may be NULL.
 * Cost: that of mpv_verify, plus a set-up launch per 3584 / N trees.  With per-node outputs (stats,
 * edge_probs, accept_prob under SPECINFER and TRAVERSAL) the call instead makes one mpv_verify launch
 * per run of consecutive trees with equal rows in merged_parent, one after the other on `hip_stream`.
 * Nothing is launched unless every tree is a valid problem. */
int mpv_verify_merged(const mpv_problem* problem, const int32_t* merged_parent, const int32_t* context_node,
                      const mpv_buffers* buffers, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Expected block efficiency of every tree of the batch with the verification's own
 * randomness integrated out (Sec. 5, Eq. 1-3; branching probabilities of Def. 5.3 by
 * the listings of App. D; averaging `expected` over the s trees sampled for one context
 * gives the paper's estimate).  For each tree b:
 *   reach_prob[b,n] = P(node n lies on the accepted path of the rule `problem->method`),
 *                     root: 1  (DEVICE, float32 [B,N]; may be NULL);
 *   expected[b]     = sum_n reach_prob[b,n] = E[tau + 1 | tree b]  (DEVICE, float32 [B]).
 * Top-down rules: the product, along the path, of the probability of moving from a node to
 * the child (an accepted child is moved to itself; a drawn token leads to the first sibling
 * that carries it; SpecInfer tries the children in list order).  Traversal: the nodes are
 * tested in depth-first post-order, each after everything before it was rejected.
 * No uniforms are read and nothing is sampled; every internal node's rows are read once.
 * problem, target_logits, draft_logits, tokens, workspace, hip_stream: as for mpv_verify
 * (same layouts, alignment and workspace size; problem->max_depth is not used beyond its
 * validation).  counters: DEVICE uint32 [MPV_COUNTER_COUNT], zeroed by the call; only
 * ZERO_MASS, BAD_TOKEN, DEPENDENCY_TIMEOUT and NODE_TASKS_RUN are meaningful.
 * Errors: as mpv_verify. */
int mpv_block_efficiency(const mpv_problem* problem, const void* target_logits, const void* draft_logits,
                         const int32_t* tokens, void* workspace, size_t workspace_bytes,
                         float* reach_prob, float* expected, uint32_t* counters, void* hip_stream);

/* mpv_block_efficiency for trees of distinct contexts: merged_parent (HOST int32 [B,N], one parent
 * array per tree) and context_node (DEVICE int32 [B,N], read for MPV_METHOD_SPECTR only) as for
 * mpv_verify_merged; problem->parent is not read; one launch per run of consecutive equal rows; the
 * counters are summed.  A later entry for an already drafted token is a leaf of its tree's array:
 * SpecInfer and Traversal never accept it (reach probability 0); under SpecTr its acceptance is
 * credited to the context node, whose reach probability covers every entry that stands for it, and
 * the repeat itself gets 0.  Everything else as for mpv_block_efficiency. */
int mpv_block_efficiency_merged(const mpv_problem* problem, const int32_t* merged_parent, const int32_t* context_node,
                                const void* target_logits, const void* draft_logits, const int32_t* tokens, void* workspace,
                                size_t workspace_bytes, float* reach_prob, float* expected, uint32_t* counters,
                                void* hip_stream);

/* Acceptance rates of the OTLP solver `problem->method` at every internal node of every tree
 * (Sec. 3.2; the listings of App. C): alpha[b,n] = the probability, over k draft tokens drawn
 * i.i.d. from the node's draft distribution (k = the node's number of children in `parent`) and
 * over the solver's own randomness, that the solver's output token is one of the draft tokens.
 * Depends on the node's two logit rows and on k only: no tokens, no uniforms.
 * alpha: DEVICE float32 [B,N]; leaves get 0.  Methods: SPECINFER, NSS, NAIVE, SPECTR;
 * MPV_METHOD_TRAVERSAL returns MPV_ERR_UNSUPPORTED (it is not an OTLP solver; App. C has no rate
 * for it).  Rates come from sums of float32 terms over the row: off by 5e-8 on average (2e-7 for SpecInfer on rows with
 * a dominant token, single ones up to 5e-6).  Everything else as for mpv_block_efficiency. */
int mpv_acceptance_rates(const mpv_problem* problem, const void* target_logits, const void* draft_logits,
                         void* workspace, size_t workspace_bytes, float* alpha, uint32_t* counters,
                         void* hip_stream);

/* mpv_acceptance_rates for trees of distinct contexts: merged_parent (HOST int32 [B,N], one parent
 * array per tree) as for mpv_verify_merged; problem->parent is not read; one launch per run of
 * consecutive equal rows; the counters are summed.  k of a node is the length of its child list with
 * every entry counted, later entries for an already drafted token included: they are draws from the
 * node's draft distribution like the others (Def. 3.1).  Everything else as for mpv_acceptance_rates. */
int mpv_acceptance_rates_merged(const mpv_problem* problem, const int32_t* merged_parent, const void* target_logits,
                                const void* draft_logits, void* workspace, size_t workspace_bytes, float* alpha,
                                uint32_t* counters, void* hip_stream);

/* Nucleus (top-p) transform of `rows` contiguous logit rows of length V (Sec. 4.1: two of the
 * paper's eight sampling settings use nucleus sampling; the paper does not define it, the usual
 * definition is taken).  With p = softmax(z / T), row by row: the smallest set {v : z_v >= tau},
 * tau one of the row's values, whose mass reaches top_p, is kept; every other token gets the logit
 * -inf, so that verification of the masked rows is verification with the truncated, renormalised
 * distributions.  Tokens with equal logits are kept or dropped together; top_p = 1 keeps every
 * token.  Apply it to the target and to the draft rows (and draw the draft tokens from the
 * masked draft rows) before mpv_verify / mpv_block_efficiency.
 * logits, out: DEVICE, [rows, V] of logit_dtype, 16-byte aligned bases; out may equal logits
 * (in place), otherwise the buffers must not overlap.  Logits must be finite or -inf.
 * threshold_out: DEVICE float32 [rows] or NULL: tau.  kept_out: DEVICE int32 [rows] or NULL: the
 * number of tokens kept.  Precision: the row's mass is a float32 sum (relative error about 1e-7), and an upper set can
 * appear smaller by V * 2^-40 of the largest token's mass (2.4e-7 at V = 262144): tau is the right one for a top_p
 * within 1e-6 of the one given (within 2e-6 at V = 2^21).  Errors: MPV_ERR_BAD_SHAPE (rows < 0, V < 1), _UNSUPPORTED (V or rows too
 * large), _BAD_DTYPE, _BAD_TEMPERATURE, _BAD_TOP_P, _NULL, _ALIGNMENT, _HIP. */
int mpv_nucleus_mask(const void* logits, void* out, int32_t logit_dtype, int64_t rows, int32_t V,
                     float temperature, float top_p, float* threshold_out, int32_t* kept_out, void* hip_stream);

/* Softmax statistics of `rows` contiguous logit rows of length V (the first step
 * of the path, exposed on its own): out[r] = { max_v z, ln sum_v exp((z - max)/T) }
 * as float32 pairs.  `logits` and `out` are DEVICE pointers. */
int mpv_row_stats(const void* logits, int32_t logit_dtype, int64_t rows, int32_t V,
                  float temperature, float* out, void* hip_stream);

/* Fill d_u[0..count) (DEVICE) with counter-based uniforms in [0,1): element i is
 * the top 24 bits of the SplitMix64 finaliser applied to
 * seed + (i+1) * 0x9E3779B97F4A7C15, times 2^-24. */
int mpv_fill_uniforms(uint64_t seed, int64_t count, float* d_u, void* hip_stream);

/* ---------------------------------------------------------------------------------------------
 * The calls around a verification in a serving loop.  One step of such a loop is
 *   target pass over the trees: mpv_tree_attention once per layer; the logits of every node;
 *   mpv_verify (or mpv_verify_merged; mpv_verify_chains where drafts are chains with probabilities);
 *   mpv_extend_tables: room in the paged cache for the root and the accepted path (new_len =
 *     accept_len, extra = 1);
 *   mpv_append_paths: their keys and values, of all layers, enter the cache;
 *   the bonus token is the root of the next step's trees.
 * The cache holds accepted tokens only: what was drafted in vain never enters it.  All calls work on lengths
 * that live on the device, allocate nothing, do not synchronise and can be captured in a graph.  A call with B = 0 succeeds and writes
 * nothing at all (its counters, free_count_out and offsets among what it leaves as it was).
 * --------------------------------------------------------------------------------------------- */

/* Attention of the nodes of B draft trees over a paged cache and over their own tree.
 * Node n of tree b is at position context_len[b] + depth(n).  It sees position j < context_len[b] of the cache and
 * the tree nodes that are its ancestors or itself, each of them only if, with `window` > 0, the position is larger
 * than its own minus `window` or smaller than `sinks`.  With s the scaled products over what it sees,
 * out = sum_j softmax(s)_j v_j; query head h reads cache head h / (heads / kv_heads).
 * Position j of tree b lies in page block_table[b, j / page_size], slot j % page_size; a page outside
 * [0, num_pages) is not seen, context_len is taken within [0, table_width * page_size].
 * What a node does not see does not reach its output, whatever it holds (NaN included).
 * An infinite value or NaN that it does see makes that column of its output infinite or NaN; which of them an infinity makes whose
 * weight is too small for float32 (or, rounded, for `dtype`) depends on where the tree's tiles end.
 * Sums and softmax statistics are float32; weights are rounded to `dtype` before they meet the values (F32: not). */
typedef struct mpv_attention {
    int32_t B, N;            /* trees; nodes per tree (<= MPV_MAX_NODES); N = 1: single tokens               */
    int32_t heads, kv_heads; /* heads is a multiple of kv_heads                                              */
    int32_t head_dim;        /* <= MPV_MAX_HEAD_DIM, a multiple of 16 bytes                                  */
    int32_t dtype;           /* MPV_DTYPE_*, of all tensors                                                  */
    int32_t num_pages, page_size, table_width;  /* the cache's pages, their slots, pages in a row of block_table */
    int32_t window, sinks;   /* window <= 0: everything is seen                                              */
    float   scale;           /* finite; multiplies q.k                                                       */
    int64_t q_stride, kv_stride, out_stride;    /* elements from a node's row [heads, head_dim] (tree_k, tree_v:
                                [kv_heads, head_dim]) to the next node's; trees follow each other            */
    int64_t page_stride, slot_stride;           /* elements from page to page, from slot to slot; a slot holds
                                                   [kv_heads, head_dim]                                       */
    const int32_t* parent;   /* HOST [N], as in mpv_problem; not read with tree_parent                       */
} mpv_attention;

typedef struct mpv_attention_buffers {    /* DEVICE, borrowed until the work has run */
    const void* q;                /* [B,N,heads,head_dim]                                                    */
    const void* tree_k;           /* [B,N,kv_heads,head_dim]: the nodes' own keys and values                 */
    const void* tree_v;
    const void* cache_k;          /* [num_pages,page_size,kv_heads,head_dim]                                 */
    const void* cache_v;
    const int32_t* block_table;   /* [B,table_width]                                                         */
    const int32_t* context_len;   /* [B] cached tokens                                                       */
    const int32_t* num_nodes;     /* [B] or NULL: only the first num_nodes[b] nodes of a tree exist; rows of
                                     `out` behind them are left as they were                                 */
    const int32_t* tree_parent;   /* [B,N] or NULL: a parent array per tree (as merged_parent); an entry outside
                                     [0,n) makes node n a root                                               */
    void* out;                    /* [B,N,heads,head_dim]; must not overlap the inputs                       */
} mpv_attention_buffers;

int mpv_tree_attention_workspace_bytes(const mpv_attention* attention, size_t* out);

/* Errors: MPV_ERR_NULL, _BAD_SHAPE, _UNSUPPORTED (N, heads, head_dim, B, a context or a stride too large),
 * _BAD_TREE, _BAD_DTYPE, _BAD_TEMPERATURE (scale not finite), _ALIGNMENT, _WORKSPACE, _HIP. */
int mpv_tree_attention(const mpv_attention* attention, const mpv_attention_buffers* buffers,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* Verification of B chains of drafted tokens against the target's probabilities, from given random numbers
 * (Sec. 3.2 on a tree of one path, with probabilities in the place of logits).  Row n of a chain belongs to the context
 * that ends with its n-th drafted token (row 0: the current context); tokens[b,n], n >= 1, was drafted from draft row
 * n - 1.  Token n is accepted iff every token before it is and u_n q(x_n) < p(x_n) (doubles, exact); the first that is
 * not sends the bonus token to (p - q)_+ of its row, otherwise the bonus token comes from the last row's p.  Without draft
 * probabilities a draft is certain: q is 1 at x_n and 0 elsewhere.  Rows need not be normalised; values that are not
 * positive (NaN included) count as 0.  Where (p - q)_+ has no mass the row's p is drawn from (counted); where p has none
 * the token is 0.  The bonus token is the smallest t whose cumulative mass exceeds uniforms[b,0] times the total (the last
 * token with mass if none does); sums are double.  A drafted token outside [0,V) is not accepted (counted), and
 * takes nothing away from p if there are no draft probabilities. */
typedef struct mpv_chains {
    int32_t B, N, V;              /* chains; rows of a chain (N - 1 drafted tokens, <= MPV_MAX_NODES rows); vocabulary */
    int32_t dtype;                /* MPV_DTYPE_* of the probabilities                                         */
    int32_t max_depth;            /* row width of path_nodes / path_tokens, >= N - 1 and >= 1                 */
    int64_t target_stride, draft_stride;   /* elements from a row to the next (>= V); chains follow each other */
} mpv_chains;

typedef struct mpv_chain_buffers {         /* DEVICE */
    const void*    target_probs;  /* [B,N,V], at any element's address                                        */
    const void*    draft_probs;   /* [B,N,V] or NULL; the row of a chain's last token is never read           */
    const int32_t* tokens;        /* [B,N]; tokens[b,0] ignored                                               */
    const float*   uniforms;      /* [B,N] in [0,1), as in mpv_buffers                                        */
    const int32_t* num_nodes;     /* [B] or NULL: rows of this chain, taken within [1,N]                      */
    int32_t*  accept_len;         /* outputs as in mpv_buffers; path_nodes[b,i] = i + 1                       */
    int32_t*  path_nodes;
    int32_t*  path_tokens;
    int32_t*  bonus_token;
    uint32_t* counters;           /* [MPV_COUNTER_COUNT]: ZERO_MASS and BAD_TOKEN; zeroed by the call         */
} mpv_chain_buffers;

int mpv_verify_chains_workspace_bytes(const mpv_chains* chains, size_t* out);

/* Errors: MPV_ERR_NULL, _BAD_SHAPE, _UNSUPPORTED (N, V, B, max_depth or a stride too large), _BAD_DTYPE, _ALIGNMENT (a pointer
 * is no multiple of its element's size), _WORKSPACE, _HIP. */
int mpv_verify_chains(const mpv_chains* chains, const mpv_chain_buffers* buffers,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* Block tables and slot maps from request lengths, on the GPU.  Request b, with context_len[b] tokens in the cache,
 * gets room for n = new_len[b] + extra more: the pages it needs are taken from the end of the list of free pages (in
 * request order, ascending position), entered into its row of the block table, and the slots of its new tokens
 * (page * page_size + place in it) are written.  new_len[b] < 0: the request is finished; its pages go to the end of the
 * list (before any are taken, in request order; what num_pages entries do not hold, which takes a free_count that was wrong, is
 * dropped) and its context becomes empty.
 * Requests are served in order.  One that cannot fit its row of the block table or (slot rows) whose n exceeds the row
 * is refused; so is every request that needs a page from the first one on whose pages, with those asked for before it, exceed
 * the free ones, and (packed slots) every request with n > 0 from the first one on whose tokens, with those asked for before it, exceed
 * the slot map.  What a refused request asked for (unless it could never fit its row) counts for those behind it.  A refused request keeps its
 * context and pages and gets granted = -1.  A table entry of an earlier page outside [0,num_pages) gives slots of -1. */
typedef struct mpv_tables {
    int32_t B, page_size, table_width, num_pages;
    int32_t extra;                /* >= 0, added to every new_len that is not negative                       */
    int32_t packed;               /* 0: slot_map[b * slot_width + i], -1 behind a request's tokens;
                                     1: slot_map[offsets[b] + i], `slot_width` slots in all, what lies behind the last
                                     token is left as it was: for a pass over prompts, one row a token, that writes its keys and values
                                     itself (mpv_append_paths takes rows of slots)                            */
    int64_t slot_width;
} mpv_tables;

typedef struct mpv_table_buffers {         /* DEVICE */
    const int32_t* new_len;       /* [B]                                                                      */
    const int32_t* context_len;   /* [B] >= 0 (a negative one counts as 0)                                    */
    int32_t* block_table;         /* [B,table_width], in and out; entries behind a request's pages are left alone */
    int32_t* free_pages;          /* [num_pages], in and out                                                  */
    const int32_t* free_count;    /* [1], taken within [0,num_pages]                                          */
    int32_t* context_len_out;     /* [B]; may be context_len                                                  */
    int32_t* free_count_out;      /* [1]; may be free_count                                                   */
    int64_t* slot_map;
    int32_t* granted;             /* [B] tokens placed, -1: refused, 0 for a finished request                 */
    int32_t* offsets;             /* [B+1] or NULL (packed: required): exclusive sums of the tokens placed    */
} mpv_table_buffers;

int mpv_extend_tables_workspace_bytes(const mpv_tables* tables, size_t* out);

/* Errors: MPV_ERR_NULL, _BAD_SHAPE, _UNSUPPORTED (slots beyond 2^31), _WORKSPACE, _HIP. */
int mpv_extend_tables(const mpv_tables* tables, const mpv_table_buffers* buffers,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* The keys and values of the root and of the accepted path of every tree enter the cache, for all layers at once:
 * row i <= accept_len[b] of tree b, node 0 for i = 0 and path_nodes[b, i - 1] otherwise (path_nodes NULL: node i), goes to slot
 * slot_map[b, i].  Slots or nodes out of range are skipped (a refused request has slots of -1).  No slot may appear twice;
 * tree and cache tensors must not overlap. */
typedef struct mpv_append {
    int32_t layers, B, N;
    int32_t dtype;
    int32_t row;                  /* kv_heads * head_dim, a multiple of 16 bytes                               */
    int32_t max_depth;            /* row width of path_nodes (0 without)                                       */
    int32_t slot_width;           /* row width of slot_map                                                     */
    int32_t num_pages, page_size;
    int64_t tree_layer_stride, tree_stride;              /* elements from layer to layer, from node to node    */
    int64_t cache_layer_stride, page_stride, slot_stride;
} mpv_append;

typedef struct mpv_append_buffers {        /* DEVICE */
    const void* tree_k;           /* [layers,B,N,row]                                                         */
    const void* tree_v;
    void* cache_k;                /* [layers,num_pages,page_size,row]                                         */
    void* cache_v;
    const int64_t* slot_map;      /* [B,slot_width]                                                           */
    const int32_t* accept_len;    /* [B]                                                                      */
    const int32_t* path_nodes;    /* [B,max_depth] or NULL                                                    */
} mpv_append_buffers;

/* Errors: MPV_ERR_NULL, _BAD_SHAPE, _UNSUPPORTED (N, row, B, layers or a stride too large), _BAD_DTYPE, _ALIGNMENT, _HIP. */
int mpv_append_paths(const mpv_append* append, const mpv_append_buffers* buffers, void* hip_stream);

/* Per-launch timing for benchmarks (process-wide state, not thread-safe).
 * mpv_timing_enable(n > 0) creates n pairs of HIP events; from then on every
 * kernel mpv_verify launches carries one pair, which the runtime stamps with the
 * start and the end of that dispatch (nothing extra is put into the caller's
 * stream), until n launches have been recorded.  mpv_timing_enable(0) turns it off
 * and destroys the events.  mpv_timing_read, called after the caller has
 * synchronised that stream, writes the elapsed milliseconds and the MPV_KERNEL_*
 * id of each recorded launch (HOST arrays of `capacity` entries), sets *count and
 * clears the record.  One call is two launches: MPV_KERNEL_INIT (counters, queue; mpv_verify_merged: the
 * launches that set up the trees' shapes have this id too) and MPV_KERNEL_NODE_TASK, whose persistent workgroups run every node task (softmax
 * statistics, per-child test probabilities, residual masses) and every sampling task
 * (accept/reject walk, bonus token) of the batch (Sec. 2, step 3); MPV_KERNEL_DEBUG_STATS
 * follows when `stats` is requested. */
#define MPV_KERNEL_INIT        0
#define MPV_KERNEL_NODE_TASK   1
#define MPV_KERNEL_DEBUG_STATS 2
int mpv_timing_enable(int32_t max_launches);
int mpv_timing_read(float* ms_out, int32_t* kernel_out, int32_t capacity, int32_t* count);

#ifdef __cplusplus
}
#endif
#endif /* MPV_H */
