/*
 * mdsd.h -- C ABI of the MI355X (gfx950) sampling-verification library for
 * multi-draft speculative decoding: SpecHub and the RRS / RRS-without-
 * replacement baselines ("SpecHub: Provable Acceleration to Multi-Draft
 * Speculative Decoding").
 *
 * One call handles a batch of B token trees of N nodes each.  Every tree node
 * owns one target row p (V elements) and, if it has children, one draft row q
 * (Sec. 2: p = p(.|prefix), q = q(.|prefix) on the probability simplex).  A
 * node's k children carry the k draft tokens sampled at that node; verifying
 * the node decides which child, if any, is accepted (Sec. 2, token-tree
 * figure).
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers owned by the caller.  The library
 *     allocates nothing, frees nothing and never synchronises: work is queued
 *     on `stream` (a hipStream_t passed as void*, NULL = the default stream)
 *     and the call returns at once.  Calls are stateless and re-entrant.
 *   - Return value: MDSD_OK, or a negative MDSD_E_* code for anything the
 *     host can detect; in that case nothing was launched.  Data-dependent
 *     problems (a token id outside [0,V), a SpecHub pair without the hub, a
 *     draft row whose whole mass sits on the hub, a residual without mass) are
 *     reported per node in `outcome` / `flags`, never by trapping.
 *   - B = 0 is an empty batch: the call looks at nothing else, launches
 *     nothing and returns MDSD_OK.
 *   - Trees: nodes in breadth-first order, root = node 0.  With first_child
 *     == NULL the tree is the complete k-ary tree with `depth` levels
 *     (N = (k^depth - 1)/(k - 1); Sec. 5.3 "binary trees of depth d with
 *     2^d - 1 nodes"); the children of n are k*n+1 .. k*n+k.  Otherwise
 *     first_child[n] is the index of node n's first child (its k children are
 *     consecutive) or -1 for a leaf, and `depth` bounds the walk.
 *     Preconditions on the table, which the library cannot check as a whole:
 *     every node but the root is the child of exactly one node (child ranges
 *     do not overlap), and children come after their parent (first_child[n]
 *     > n).  Per entry the kernels and the walk apply one rule: an entry
 *     that is <= n or leaves no room for k children (first_child[n] + k > N)
 *     makes node n a leaf, so no access leaves the arrays and every walk
 *     ends; with overlapping ranges each node is still verified on its own
 *     rows, but which tokens a shared child stands for is the caller's
 *     business.
 *   - Rows: element (b, n, x) of `target` lives at target[(b*N + n)*ld_t + x].
 *     dtype selects fp32 or bf16 storage.  kind = MDSD_PROBS: rows are
 *     probabilities and are used as given (no renormalisation); kind =
 *     MDSD_LOGITS: rows are logits and p = softmax(row / temp_target),
 *     q = softmax(row / temp_draft) (App. D; Sec. 5.1 temperatures), computed
 *     in fp32 inside the kernels.  Row start addresses of target and draft
 *     must have the same offset modulo 16 bytes (true whenever both bases are
 *     16-byte aligned and ld_t == ld_d); any V >= 2 and any element-aligned
 *     base is accepted.  Draft rows of leaves are never read.
 *   - Tokens: `tokens` is [B,N] int32 indexed by CHILD node: tokens[b][c] is
 *     the draft token that child c stands for; the root's entry is unused.
 *   - Uniforms are inputs ([0,1), fp32), so results are a deterministic
 *     function of the arguments.  mdsd_philox_uniform makes them.
 */
#ifndef MDSD_H
#define MDSD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MDSD_FP32 0
#define MDSD_BF16 1
#define MDSD_FP16 2 /* the key-value cache calls only */
#define MDSD_FP4 3  /* caches of the calls that take mdsd_kv_scales only */

#define MDSD_PROBS 0
#define MDSD_LOGITS 1

#define MDSD_MAX_K 8
#define MDSD_MAX_DIM 256          /* elements of a head in the key-value cache calls   */
#define MDSD_MAX_TABLE_NODES 4096 /* nodes of a tree given by a table, in those calls  */
#define MDSD_MAX_AXES 8           /* of positions, in mdsd_kv_append_at                 */

/* status codes */
#define MDSD_OK 0
#define MDSD_E_NULL (-1)      /* a required pointer is NULL                     */
#define MDSD_E_SHAPE (-2)     /* B < 0, N < 1, V < 2, ld < V, depth < 1, tree/N mismatch */
#define MDSD_E_K (-3)         /* k outside 1..MDSD_MAX_K, or SpecHub with k != 2 (Sec. 4) */
#define MDSD_E_TEMP (-4)      /* kind == logits and a temperature is not > 0; an attention's scale is not */
#define MDSD_E_DTYPE (-5)     /* unknown dtype or kind                          */
#define MDSD_E_ALIGN (-6)     /* pointer not element-aligned (workspace: 4 bytes), or target/draft rows differ modulo 16 bytes;
                                 cache calls: a pointer or stride that is no multiple of 16 bytes */
#define MDSD_E_WORKSPACE (-7) /* a workspace was given and is smaller than mdsd_workspace_bytes() */
#define MDSD_E_LAUNCH (-8)    /* the HIP runtime refused a launch               */
#define MDSD_E_UNSUPPORTED (-9) /* an output this entry point cannot give was asked for */

/* per-node outcome codes (values >= 0 are the accepted child slot) */
#define MDSD_NONE (-1)      /* no child accepted; token drawn from the residual (a leaf: from p) */
#define MDSD_BAD_PAIR (-2)  /* SpecHub: the two tokens are not {hub, non-hub}   */
#define MDSD_BAD_TOKEN (-3) /* a draft token id is outside [0, V)               */
#define MDSD_UNVISITED (-4) /* *_verify_path only: the walk never reached this node */

/* per-node flag bits */
#define MDSD_FLAG_DEGENERATE_HUB 1 /* draft mass outside the hub is 0: node handled as single-draft on the hub */
#define MDSD_FLAG_ZERO_RESIDUAL 2  /* a residual had no mass; the previous distribution was kept */
#define MDSD_FLAG_Q_EXHAUSTED 4    /* RRSw: no draft mass left after zeroing rejected tokens */
#define MDSD_FLAG_BAD_PAIR 8
#define MDSD_FLAG_BAD_TOKEN 16
#define MDSD_FLAG_NO_PAGE 32 /* key-value cache calls, per sequence: see mdsd_kv_cache */

/*
 * Statistics of one draft row that both SpecHub calls need: the hub a (Sec. 4: the token of
 * highest draft probability) and the two numbers that normalise q around it.  With
 * pb->draft_stats set, spechub_draft writes one record per node (leaves: hub = -1) and
 * spechub_verify reads them instead of scanning the draft row for them again; a node whose
 * first acceptance test (Alg. 3, the non-hub token) succeeds then never reads its draft row.
 * The records must come from spechub_draft on the same draft rows, dtype, kind and
 * temp_draft: the library cannot check that.  A hub outside [0,V) makes the node
 * MDSD_BAD_PAIR.  Results depend on the pointer only through fp32 rounding of rest_mass (a
 * different summation order).
 * rrs_draft and rrsw_draft write records too (hub = -1, rest_mass = the mass of the whole row,
 * before any token is removed) and rrs_verify / rrsw_verify read them the same way.  Records
 * must come from the draft call of the same method.
 */
typedef struct mdsd_row_stats {
    float max_stored; /* largest stored element of the row (a logit, or a probability)        */
    float rest_mass;  /* sum over y != hub of exp((l(y) - max_stored)/temp_draft) for logits,
                         of q(y) for probabilities: the draft mass outside the hub, times the
                         softmax normaliser when the hub's weight is 1                        */
    int32_t hub;      /* argmax of the stored row, lowest index on ties; -1 on leaves         */
    int32_t reserved; /* written as 0                                                         */
} mdsd_row_stats;

typedef struct mdsd_problem {
    const void* target;         /* device, [B,N,ld_t] rows of the target model            */
    const void* draft;          /* device, [B,N,ld_d] rows of the draft model             */
    int64_t ld_t, ld_d;         /* row strides in elements, >= V                          */
    int32_t dtype;              /* MDSD_FP32 | MDSD_BF16                                  */
    int32_t kind;               /* MDSD_PROBS | MDSD_LOGITS                               */
    float temp_target;          /* used iff kind == MDSD_LOGITS; > 0                      */
    float temp_draft;
    int32_t B, N, V;            /* trees, nodes per tree, vocabulary size                 */
    int32_t k;                  /* children per internal node (drafts per step)           */
    int32_t depth;              /* levels of the tree = max tokens emitted per tree       */
    const int32_t* first_child; /* device [N] or NULL (complete k-ary tree)               */
    mdsd_row_stats* draft_stats; /* device [B,N] or NULL: what spechub_draft learnt
                                   about each draft row, handed on to spechub_verify (below) */
} mdsd_problem;

typedef struct mdsd_result {
    int32_t* outcome;      /* device [B,N], required: accepted child slot or MDSD_* code       */
    int32_t* token;        /* device [B,N], required: the token this node emits (the accepted
                              child's token, else the residual / bonus sample)                 */
    float* resid_mass;     /* device [B,N] or NULL: mass of the node's residual in units of p.
                              SpecHub: sum_x p''(x) (= 1 - total acceptance, whatever the tokens);
                              RRS/RRSw: mass of max(p - c q, 0) when the node returned, i.e. the
                              probability mass the rejections so far left (the product of the
                              rejected rounds' sums of max(p_i - q_i, 0) in Alg. 1; 1 when the
                              first draft was accepted); leaf: sum p.
                              Non-NULL disables SpecHub's early exit.                          */
    int32_t* flags;        /* device [B,N] or NULL: MDSD_FLAG_* bits                           */
    float* resid_prob;     /* device [B,N,V] or NULL (diagnostic): SpecHub: norm(p''); RRS/RRSw:
                              the target distribution as it stood when the node returned (after
                              the rejections made so far); leaf: p                             */
    int32_t* accept_depth; /* device [B] or NULL: number of accepted draft tokens on the path  */
    int32_t* emitted;      /* device [B,depth] or NULL: emitted tokens, -1 padded; tokens per
                              step = accept_depth + 1 (Sec. 5.3 batch efficiency)              */
} mdsd_result;

/*
 * Workspace.  No call needs one: ws may always be NULL.  spechub_verify, rrs_verify and
 * rrsw_verify put a non-NULL workspace to use when they are also asked for the walk
 * (out->accept_depth and out->emitted): it holds one int32 arrival counter per tree, with which
 * the verify kernel walks each tree itself as soon as the tree's last node is done, instead of
 * running the walk as a second launch behind it (same results; one launch less per step, which
 * pays for batches of up to about 3000 tree nodes: beyond that the counting costs more than the
 * launch it saves, and ws = NULL is the faster call).
 *   - mdsd_workspace_bytes(pb) = 4 * pb->B bytes; ws must be 4-byte aligned device memory;
 *     a smaller ws_bytes is MDSD_E_WORKSPACE.
 *   - The counters must be ZERO when the call starts.  Every call leaves them zero again, so a
 *     workspace zero-filled once after its allocation can be handed to call after call.  (If a
 *     call was cut short -- the process went on after a failed launch or a device error -- fill
 *     it with zeros again; counters that do not start at zero give a wrong or missing walk,
 *     never an access outside the arrays.)
 *   - Calls that overlap in time (different streams) need workspaces of their own.
 * The draft calls, the *_verify_path calls and mdsd_tree_walk ignore ws.
 */
size_t mdsd_workspace_bytes(const mdsd_problem* pb);

/*
 * spechub_draft -- sample, for every internal node, the pair (x1, x2) ~ Q of
 * Sec. 4: with hub a = argmax q, Q(x,a) = q(x) and Q(a,x) = q(a) q(x)/(1-q(a))
 * for x != a, 0 elsewhere (Alg. 3, "Sample draft tokens").  Two-stage sampler:
 * x ~ q with u[.,.,0]; if x != a the pair is (x, a); otherwise the second
 * token is drawn with u[.,.,1] from q restricted to tokens other than a.
 * The hub is the lowest index among the maxima of the stored draft row.
 *   u      device [B,N,2] fp32 in [0,1)
 *   tokens device [B,N] out: tokens[b][first_child(n)+j] = x_{j+1}; root = -1
 *   hub    device [B,N] out or NULL: the hub of each internal node, -1 on leaves
 *   flags  device [B,N] out or NULL
 * Requires pb->k == 2.  Reads only pb->draft.
 */
int spechub_draft(const mdsd_problem* pb, const float* u, int32_t* tokens, int32_t* hub,
                  int32_t* flags, void* ws, size_t ws_bytes, void* stream);

/*
 * spechub_verify -- Alg. 3 (with Alg. 2 GetResidual and the transport plan of
 * App. B.1) for every node, then the tree walk.
 *   pair (x, a): accept x if u0 * q(x) < p(x); else accept a if
 *                u1 * sum_y max(q - p, 0) < max(p(a) - S, 0), where
 *                S = sum_{y != a} max(Q(a,y) - max(p(y) - q(y), 0), 0);
 *   pair (a, x): accept x if u0 * Q(a,x) < max(p(x) - q(x), 0); else accept a
 *                if u1 * S < p(a);
 *   otherwise draw the token with u2 from norm(p''), p''(y) = max(p(y) - q(y)
 *   - Q(a,y), 0) for y != a and 0 at a (App. B.2).  Leaves draw from p with u2.
 *   tokens device [B,N] (see above); u device [B,N,3] = (u0, u1, u2) per node.
 * Requires pb->k == 2.
 */
int spechub_verify(const mdsd_problem* pb, const int32_t* tokens, const float* u,
                   const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);

/*
 * spechub_verify_static -- spechub_verify with the tree walk inside its kernel, for callers that
 * cannot allocate or carry a workspace: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  The arrival counters live in a device array of the library's
 * own (MDSD_STATIC_MAX_TREES int32, 256 KiB per GPU, held until the process ends); the call
 * allocates nothing, frees nothing and queues one kernel on `stream`.
 *   - Same arguments and results as spechub_verify with a workspace; out->accept_depth and
 *     out->emitted are required (MDSD_E_NULL without them).
 *   - pb->B > MDSD_STATIC_MAX_TREES is refused with MDSD_E_WORKSPACE.
 *   - All calls on one GPU share that GPU's array: two calls that overlap in time on one GPU
 *     (different streams) race on it and may give wrong or missing walks; calls on one stream,
 *     one after another, are fine.  Every call leaves the counters zero for the next.
 *   - The first call on a device looks up the array's address on that device (no allocation);
 *     the device must be current, as for every call.
 */
#define MDSD_STATIC_MAX_TREES 65536
int spechub_verify_static(const mdsd_problem* pb, const int32_t* tokens, const float* u,
                          const mdsd_result* out, void* stream);

/*
 * rrs_draft / rrsw_draft -- Alg. 1, first step: k tokens per internal node from
 * q, independently (RRS) or without replacement (RRSw; Sec. 3.3 gives both Q).
 *   u device [B,N,k]; tokens device [B,N] out, child-indexed; flags or NULL.
 */
int rrs_draft(const mdsd_problem* pb, const float* u, int32_t* tokens, int32_t* flags,
              void* ws, size_t ws_bytes, void* stream);
int rrsw_draft(const mdsd_problem* pb, const float* u, int32_t* tokens, int32_t* flags,
               void* ws, size_t ws_bytes, void* stream);

/*
 * rrs_verify / rrsw_verify -- Alg. 1 for every node, then the tree walk.
 * Round i = 1..k: accept x_i if u_{i-1} * q_i(x_i) < p_i(x_i); else
 * p_{i+1} = norm(max(p_i - q_i, 0)) and, without replacement, q_{i+1} = norm(q_i
 * with q_i(x_i) = 0).  After k rejections the token is drawn from p_{k+1}
 * with u_k.  Leaves draw from p with u_k.
 *   u device [B,N,k+1].
 */
int rrs_verify(const mdsd_problem* pb, const int32_t* tokens, const float* u,
               const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);
int rrsw_verify(const mdsd_problem* pb, const int32_t* tokens, const float* u,
                const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);

/*
 * spechub_step / rrs_step / rrsw_step -- the draft call and the verify call of a method in one, for callers
 * that hold both rows of every node already (measured logits, acceptance studies, simulations): the same
 * arguments and errors as the two calls one after the other, everything checked before anything is
 * launched, and their outputs up to the rounding of sums that are formed in another order: a token, slot or
 * flag can differ where a uniform lies within that of a boundary.  (On rows of more than 256 16-byte chunks the
 * drafted tokens, flags and records are the draft call's bit for bit, RRS on aligned fp32 rows of 16384 to
 * 32768 elements excepted.)  With pb->draft_stats set, and neither out->resid_mass nor
 * out->resid_prob, rows of most sizes are drafted and verified by one kernel that reads each row once as
 * far as the method allows; other calls launch the two.  ws as for the verify calls.
 */
int spechub_step(const mdsd_problem* pb, const float* u_draft, const float* u_verify, int32_t* tokens,
                 int32_t* hub, int32_t* draft_flags, const mdsd_result* out, void* ws, size_t ws_bytes,
                 void* stream);
int rrs_step(const mdsd_problem* pb, const float* u_draft, const float* u_verify, int32_t* tokens,
             int32_t* draft_flags, const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);
int rrsw_step(const mdsd_problem* pb, const float* u_draft, const float* u_verify, int32_t* tokens,
              int32_t* draft_flags, const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);

/*
 * spechub_verify_path / rrs_verify_path / rrsw_verify_path -- the same verification
 * restricted to the nodes that decide what the step emits (Sec. 2: verification follows the
 * accepted tokens down the tree and stops at the first node that accepts none; the nodes
 * beside that path have no effect on the output).  One workgroup per tree starts at the root,
 * verifies a node exactly as the calls above do (same arguments, same uniforms, same
 * arithmetic, so the same outcome and token), moves to the accepted child and stops like
 * mdsd_tree_walk.  A step then reads accept_depth + 1 target rows per tree instead of N.
 *   out->accept_depth and out->emitted are required (they are the result);
 *   out->outcome, out->token (required), out->flags, out->resid_mass (optional) hold the
 *   visited nodes' values, every other node MDSD_UNVISITED / -1 / 0 / 0;
 *   out->resid_prob must be NULL (MDSD_E_UNSUPPORTED).
 * SpecHub uses pb->draft_stats as spechub_verify does.
 */
int spechub_verify_path(const mdsd_problem* pb, const int32_t* tokens, const float* u,
                        const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);
int rrs_verify_path(const mdsd_problem* pb, const int32_t* tokens, const float* u,
                    const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);
int rrsw_verify_path(const mdsd_problem* pb, const int32_t* tokens, const float* u,
                     const mdsd_result* out, void* ws, size_t ws_bytes, void* stream);

/*
 * mdsd_tree_walk -- the walk alone (Sec. 2: follow accepted children from the
 * root; every visited node emits its token; stop at the first node without an
 * accepted child).  The verify calls run it themselves when out->accept_depth
 * and out->emitted are given.
 */
int mdsd_tree_walk(const mdsd_problem* pb, const int32_t* outcome, const int32_t* token,
                   int32_t* accept_depth, int32_t* emitted, void* stream);

/*
 * mdsd_philox_uniform -- counter-based uniforms (Philox4x32-10, Salmon et al.,
 * SC'11).  out[row*slots + s] = (w >> 8) * 2^-24 with w = word (s & 3) of
 * Philox(counter = (row_lo, row_hi, s >> 2, stream_id), key = (seed_lo,
 * seed_hi)).  out: device [rows, slots] fp32; words: device [rows, slots]
 * uint32 or NULL (the raw words, for tests).  rows = 0 returns MDSD_OK at once.
 */
int mdsd_philox_uniform(uint64_t seed, uint32_t stream_id, int64_t rows, int32_t slots,
                        float* out, uint32_t* words, void* stream);

/*
 * The key-value cache of the trees.
 *
 * Between drafting and verifying, the target model runs over the nodes of every tree.  Its attention
 * layers keep keys and values in a cache of pages; three calls work on that cache and on the trees of
 * this header:
 *   mdsd_kv_append       rotates the nodes' queries and keys to their positions and puts keys and
 *                        values into the cache behind the sequence's;
 *   mdsd_tree_attention  lets every node attend to its sequence and to its ancestors;
 *   mdsd_kv_commit       after the walk, moves the accepted path's keys and values to where the
 *                        sequence goes on, and gives the new lengths.
 * Node n of tree b, at level d of the tree (the root is at level 0), has the position lengths[b] + d
 * and, until the commit, the slot lengths[b] + n.  A prompt, or a part of one, is a tree of one branch
 * (k = 1, depth = N: node n attends to nodes 0..n); a single token is a tree of one node.
 * Conventions as for every entry point above (status codes; nothing allocated, freed or waited for;
 * B = 0 is an empty batch).  All element types agree: cache, queries, outputs.  A call that would take 2^24
 * workgroups or more is MDSD_E_SHAPE: an append of B*N nodes, a commit of B*layers, an attention of B*heads times
 * the tiles (of 16 to 128) of the N * q->heads / heads rows of a tree.
 *
 * Pages: slot s of sequence b is slot s % page_size of page table[b * ld_table + s / page_size].  A
 * slot has no page if it lies behind the table's table_pages entries or its entry is not in
 * [0, pages).  Such a slot is never read or written: append and commit drop what would go there,
 * attention goes on without that key (a row that no key is left for is zeros).  A negative length
 * makes a sequence one without nodes.  In each of these cases bit MDSD_FLAG_NO_PAGE of flags[b] is set
 * where the call meets it; calls set bits and never clear one, so one array, zeroed once, serves all
 * of a step's calls.  Entries that no slot below lengths[b] + counts[b] needs are not looked at.
 * Two slots that are written must not be one place: tables share pages only below every sharer's length.
 */
typedef struct mdsd_kv_cache {
    void* k; /* device: element (layer l, page p, slot s, head h, x) at
                l*ld_layer + p*ld_page + s*ld_slot + h*ld_head + x, in k and in v            */
    void* v;
    int64_t ld_layer, ld_page, ld_slot, ld_head; /* in elements; multiples of 16 bytes, as k and v are;
                                                    ld_page and ld_slot below 64 GiB               */
    int32_t dtype;                               /* MDSD_FP32 | MDSD_BF16 | MDSD_FP16                  */
    int32_t layers, pages, page_size, heads;     /* page_size: any from 1 on                           */
    int32_t dim;                                 /* elements of a head: a multiple of 8, up to MDSD_MAX_DIM */
    int32_t table_pages;                         /* entries of a sequence in the table; times page_size
                                                    at most 2^30                                       */
    const int32_t* table;                        /* device [B, ld_table]                               */
    int64_t ld_table;                            /* >= table_pages                                     */
    const int32_t* lengths;                      /* device [B]: slots in use, the trees' not counted   */
} mdsd_kv_cache;

/* The trees: k, depth, first_child as in mdsd_problem (with a table, N <= MDSD_MAX_TABLE_NODES; a node
 * that no entry claims as a child is a root of its own: level 0, no ancestors). */
typedef struct mdsd_tree {
    int32_t B, N, k, depth;
    const int32_t* first_child; /* device [N] or NULL (complete k-ary tree)                    */
    const int32_t* counts;      /* device [B] or NULL: tree b has nodes 0 .. counts[b]-1 only (cut to
                                   [0, N]); what belongs to the others is neither read nor written  */
} mdsd_tree;

/* Vectors of every node and head: element (b, n, h, x) at b*ld_tree + n*ld_node + h*ld_head + x.  Base
 * and strides are multiples of 16 bytes (a slice of a fused projection is fine).  A stride of zero repeats
 * what is read; outputs, and the cache of an append or a commit, have none (MDSD_E_SHAPE). */
typedef struct mdsd_heads {
    void* p;
    int64_t ld_tree, ld_node, ld_head;
    int32_t heads;
} mdsd_heads;

#define MDSD_ROTATE_HALVES 0     /* pairs (x_i, x_{i + rot/2}) */
#define MDSD_ROTATE_NEIGHBOURS 1 /* pairs (x_2i, x_{2i+1})     */

/*
 * mdsd_kv_append -- pair i < rot/2 of a head's first rot elements turns by the angle a = t * inv_freq[i],
 * t the node's position: (x, y) -> (x cos a - y sin a, x sin a + y cos a).  The angle is formed and cut to
 * one turn in 64 bits, the rotation in 32, rounded once.  k goes into the cache turned, v as it is; q, if
 * given, goes to q_out turned (q_out may be q itself; any other overlap is the caller's mistake: MDSD_E_ALIGN
 * where both have the same strides or begin at one place, results of no use otherwise).
 *   k, v: cache->heads heads; q, q_out: any number of heads, or both NULL
 *   inv_freq device [rot/2] fp32, or NULL with rot = 0 (nothing is turned); rot even, <= dim
 *   flags device [B] or NULL
 */
int mdsd_kv_append(const mdsd_kv_cache* cache, int32_t layer, const mdsd_tree* tree, const mdsd_heads* k,
                   const mdsd_heads* v, const mdsd_heads* q, const mdsd_heads* q_out, const float* inv_freq,
                   int32_t rot, int32_t style, int32_t* flags, void* stream);

/*
 * mdsd_tree_attention -- out(b,n,h) = sum_s w_s v_s / sum_s w_s over the slots s that node n sees:
 * s < lengths[b], and lengths[b] + m for n itself and its ancestors m; w_s = exp(scale q(b,n,h).k_s).
 * Query head h reads cache head h / (q->heads / cache->heads).  Sums and the softmax's statistics are
 * fp32; in 16-bit types the weights are rounded to the type before they meet v.  Keys and values that a
 * row does not see do not touch it, whatever they hold.
 *   q, out     a multiple of cache->heads heads, the same number; out may be q itself, and overlaps as in an append
 *   scale      > 0; it times log2(e) has to be finite in fp32 (MDSD_E_TEMP), and so do the scores, q.k
 *   shared     the first `shared` slots of all sequences hold the same tokens (a common system prompt):
 *              their keys are read through shared_pages, device [ceil(shared / page_size)], instead of
 *              each sequence's own table (a shorter sequence sees lengths[b] of them), and, given a
 *              workspace, met by the rows of all trees together, once.  0 and NULL: nothing is shared.
 *   longest    a length that no sequence is expected to exceed, or 0: how the work is cut goes by it and
 *              by the table's width, never what is computed
 *   flags      device [B] or NULL
 *   ws         16-byte aligned device memory of mdsd_tree_attention_workspace_bytes(), or NULL: no sequence
 *              is then cut into parts, nor the shared prefix met once, which few or long sequences pay
 *              for.  Any contents; calls that overlap in time need workspaces of their own.  A smaller
 *              ws_bytes is MDSD_E_WORKSPACE.  Results differ by the rounding of sums in another order.
 */
int mdsd_tree_attention(const mdsd_kv_cache* cache, int32_t layer, const mdsd_tree* tree, const mdsd_heads* q,
                        const mdsd_heads* out, float scale, const int32_t* shared_pages, int32_t shared,
                        int32_t longest, int32_t* flags, void* ws, size_t ws_bytes, void* stream);
/* 0 where the call has no use for a workspace (or would refuse its arguments) */
size_t mdsd_tree_attention_workspace_bytes(const mdsd_kv_cache* cache, const mdsd_tree* tree, int32_t q_heads,
                                           int32_t shared, int32_t longest);

/*
 * mdsd_kv_commit -- the path of a verified tree: node 0, then first_child(n) + outcome[b,n] from node n
 * on, accept_depth[b] steps, as mdsd_tree_walk takes them (it ends early at an outcome that is no child
 * slot, at a leaf and at a node that counts[b] cuts off).  Keys and values of the path's i-th node go from
 * slot lengths[b] + n to slot lengths[b] + i, in all layers; new_lengths[b] = lengths[b] + the path's
 * nodes, 2^31 - 1 at most (lengths[b] itself for a tree without nodes).
 *   outcome device [B,N], accept_depth device [B]: what a verify call gave
 *   new_lengths device [B]; may be cache->lengths itself (one more launch); any other overlap with it is
 *           MDSD_E_ALIGN
 *   flags device [B] or NULL
 */
int mdsd_kv_commit(const mdsd_kv_cache* cache, const mdsd_tree* tree, const int32_t* outcome,
                   const int32_t* accept_depth, int32_t* new_lengths, int32_t* flags, void* stream);

/*
 * A long context in a small cache: keys and values in 4 bits, positions that are no slot numbers, and only the slots that
 * matter.
 *
 * Caches in 4 bits.  A cache of dtype MDSD_FP4 holds two elements a byte, the first in the low half, and its strides count
 * elements as ever (multiples of 32); dim is a multiple of 32.  An element is a code: bit 3 the sign, the others 0 .. 7 for
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6; it stands for that times 2^(scale - 127), with one scale, a byte, for the 32 elements of each
 * 16 bytes (the OCP microscaling format of e2m1 elements under e8m0 scales).  The scale of the 16 bytes at offset o of k
 * stands at offset o / 16 of scales.k, and so for v: an array of the same order of axes, dim / 32 bytes a head.  Scale 255: all
 * 32 are NaN.  A call that takes such a cache takes mdsd_kv_scales beside it; without (NULL) it is of the dtypes above.
 * Calls of any dtype read a cache that calls of another filled, but for fp16, which has no numbers for scales below 2^-23 or above
 * 2^13: caches for fp16 calls are filled by these, or with such scales only (others' values come as zeros and infinities).
 */
typedef struct mdsd_kv_scales {
    void* k; /* device bytes, of any alignment (and read by the aligned words of four that they lie in) */
    void* v;
    int32_t dtype; /* MDSD_FP32 | MDSD_BF16 | MDSD_FP16: of keys, values, queries and results */
} mdsd_kv_scales;

/*
 * Positions.  Without any, node n of tree b at level d has the position lengths[b] + d on every axis.  Otherwise they are
 * given: of every node (per_node = 1: axis a's at a*ld_axis + b*ld_tree + n), or of the roots (per_node = 0: at a*ld_axis +
 * b*ld_tree; a node at level d has d more on every axis).  Any 32-bit numbers.  Pair i turns by axis_of[i], or by axis 0
 * where that is NULL; a pair whose axis is none stays as it is.  Pictures have axes of time, height and width; after an
 * eviction positions go on where slots do not.
 */
typedef struct mdsd_rotary {
    const float* inv_freq; /* device [rot/2], or NULL with rot = 0                                      */
    int32_t rot, style;    /* as in mdsd_kv_append                                                      */
    const int32_t* positions; /* device, or NULL                                                        */
    int64_t ld_axis, ld_tree; /* in elements, >= 0                                                      */
    int32_t axes, per_node;   /* axes: 1 .. MDSD_MAX_AXES with positions, not looked at without         */
    const uint8_t* axis_of;   /* device [rot/2], or NULL; not looked at without positions               */
} mdsd_rotary;

/*
 * mdsd_kv_append_at -- mdsd_kv_append at given positions, into a cache of any dtype.  In 4 bits: keys are turned in 64 bits,
 * rounded to 32, and 32 elements of a head at a time take the smallest scale 2^e that leaves the largest 7 at most (it is
 * then as far from 6 as 5 is from its neighbours, at most), e from -125 to 125, in fp16 from -23 to 13, so that every value that is
 * held is a number of the type; each becomes the nearest of the sixteen values, the even code where two are, 6 beyond it.  A
 * block with an infinity or NaN has scale 255.
 *   rotary       or NULL: nothing is turned
 *   k_out, v_out cache->heads heads, or NULL: the values that the cache now holds, in `dtype`, exactly (scales given only,
 *                MDSD_E_UNSUPPORTED otherwise; a key without a page has them too).  v_out may be v itself, k_out shares
 *                nothing with k (MDSD_E_ALIGN); other overlaps are as in mdsd_kv_append, and results share nothing with each
 *                other or with another result's vector.
 */
int mdsd_kv_append_at(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t layer, const mdsd_tree* tree,
                      const mdsd_heads* k, const mdsd_heads* v, const mdsd_heads* q, const mdsd_heads* q_out,
                      const mdsd_rotary* rotary, const mdsd_heads* k_out, const mdsd_heads* v_out, int32_t* flags, void* stream);

/*
 * mdsd_tree_attention_lse -- mdsd_tree_attention over a cache of any dtype, and the rows' sums:
 * lse(b,n,h) = ln sum_s exp(scale q(b,n,h).k_s), fp32, minus infinity for a row that no key is left for.
 *   lse  device [B, N, q->heads] or NULL; rows that `out` does not get are left as they were
 * The workspace is that of mdsd_tree_attention_lse_workspace_bytes().
 */
int mdsd_tree_attention_lse(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t layer, const mdsd_tree* tree,
                            const mdsd_heads* q, const mdsd_heads* out, float scale, const int32_t* shared_pages,
                            int32_t shared, int32_t longest, float* lse, int32_t* flags, void* ws, size_t ws_bytes, void* stream);
size_t mdsd_tree_attention_lse_workspace_bytes(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, const mdsd_tree* tree,
                                               int32_t q_heads, int32_t shared, int32_t longest);

/* mdsd_kv4_commit -- mdsd_kv_commit of a cache in 4 bits. */
int mdsd_kv4_commit(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, const mdsd_tree* tree, const int32_t* outcome,
                    const int32_t* accept_depth, int32_t* new_lengths, int32_t* flags, void* stream);

/*
 * mdsd_kv_weigh -- the attention that every slot was given: out[b][s] = weights[b][s] + sum over rows (n, h) that see slot s
 * of exp(scale q(b,n,h).k_s - lse(b,n,h)), for s < slots, over all query heads.  Called after each layer's attention it adds
 * up over layers and steps.
 *   outcome, accept_depth  both NULL: the rows are all nodes (below counts), slots are the cache's.  Both given (a verify
 *                call's, as for mdsd_kv_commit, and before it): the rows are the accepted path's nodes alone, and node i of the
 *                path counts for slot lengths[b] + i, where the commit puts it; the tree's other nodes count for none.
 *   lse          device [B, N, q->heads], as the attention gave it; a row of minus infinity adds nothing
 *   weights      device [B, ld_weights] fp32, or NULL: zeros; out may be weights itself, and overlaps it in no other way
 *                (MDSD_E_ALIGN; with different strides the whole stretches of memory must not meet)
 *   slots        entries of a row, >= 1, ld_weights and ld_out >= slots; slots at and beyond it are not counted (work is shared
 *                out by it: rows that are much longer than the sequences cost a few microseconds)
 * Each entry has one sum in a fixed order: results are the same from call to call.  Sums are fp32.  A row whose sum is no
 * number (a key that it sees is none) makes the weights of all that it sees none, and leaves those of other slots alone.
 * 2^23 workgroups or more, of B times the stretches of 16 to 256 slots of a row, are MDSD_E_SHAPE.
 */
int mdsd_kv_weigh(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t layer, const mdsd_tree* tree,
                  const mdsd_heads* q, const float* lse, float scale, const int32_t* outcome, const int32_t* accept_depth,
                  const float* weights, int64_t ld_weights, float* out, int64_t ld_out, int32_t slots, int32_t* flags,
                  void* stream);

/*
 * mdsd_kv_evict -- cuts every sequence of more than `budget` slots to that many: its first `first` slots, its last `recent`,
 * and of the others those with the largest weights, the lower slot where weights are equal (a NaN is below all numbers).  What
 * is kept moves, in order, to slots 0 .. budget-1, keys and values in all layers.  Shorter sequences stay as they are.
 *   B            sequences: entries of lengths, rows of the table
 *   weights      device [B, ld_weights] fp32, `slots` of a row (a slot at or beyond it: weight zero)
 *   budget       >= 1, first and recent >= 0, first + recent <= budget (MDSD_E_SHAPE)
 *   new_lengths  device [B]: min(lengths, budget); may be cache->lengths itself.  A length beyond the table counts as the
 *                table's capacity (and sets the flag), a negative one stays (and sets it)
 *   kept         device [B, budget]: the slots that are kept, in order, and -1 behind them
 *   weights_out  device [B, ld_out] or NULL: the kept slots' weights, zeros behind them up to `slots`; may be weights itself,
 *                and overlaps as in mdsd_kv_weigh
 *   flags        device [B] or NULL; a kept slot without a page, or that moves to one, does not move
 * 2^23 workgroups or more, at most B * layers * 2 * heads, are MDSD_E_SHAPE; so is a B of 2^22 or more.
 * Slots below `first` are not written: pages that sequences share must lie below it.  Positions stay what they were when the
 * keys were turned: what is appended next is given its own.
 */
int mdsd_kv_evict(const mdsd_kv_cache* cache, const mdsd_kv_scales* scales, int32_t B, const float* weights, int64_t ld_weights,
                  int32_t slots, int32_t budget, int32_t first, int32_t recent, int32_t* new_lengths, int32_t* kept,
                  float* weights_out, int64_t ld_out, int32_t* flags, void* stream);

/* Text for a status code (static storage). */
const char* mdsd_strerror(int code);

/* Library version, major*100 + minor. */
int mdsd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MDSD_H */
