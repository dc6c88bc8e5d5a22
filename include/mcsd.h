/*
 * mcsd.h - C ABI of libmcsd: the target-side verification step of
 * Multi-Candidate Speculative Decoding (MCSD) on one AMD MI355X (gfx950).
 *
 * Operations, all enqueued asynchronously on a caller-supplied HIP stream:
 *
 *   mcsd_tree_attn      Tree attention (Sec. 3.3 of the paper): all candidate
 *                       tokens of the draft tree are scored in one pass against
 *                       the shared prefix KV cache; a candidate attends to the
 *                       whole prefix, to its ancestors in the tree and to itself.
 *   mcsd_verify_sample  Multi-candidate speculative sampling, Algorithm 1 (with
 *                       replacement) and Algorithm 2 (without replacement), run
 *                       for every node that has children, the endpoint draws of
 *                       Sec. 2 / Sec. 3, and the root-to-leaf walk of Sec. 3 that
 *                       turns the per-node outcomes into the accepted path.
 *   mcsd_verify_step    Both, back to back on one stream: one layer's tree
 *                       attention followed by one verification.
 *   mcsd_draft_sample   The step before: the k candidates of every parent drawn
 *                       from the draft distribution (Sec. 3.1; Eq. (1) when
 *                       sampling without replacement).
 *   mcsd_tree_build     The candidate tree of a k-configuration (parent, depth,
 *                       draft-row map, position ids) built on the device.
 *   mcsd_kv_commit      The step after: the accepted path's keys and values join
 *                       the prefix cache, prefix_len grows, the endpoint becomes
 *                       the next root.
 *   mcsd_tree_attn_fourbit, mcsd_kv_commit_fourbit, mcsd_kv_store_fourbit,
 *   mcsd_kv_load_fourbit
 *                       The same attention and commit over a paged prefix cache
 *                       held in 4 bits, and rows into such a cache and back.
 *   mcsd_kv_store_paged, mcsd_chunk_attn_paged
 *                       The prompt: rows of new tokens into a paged cache, and
 *                       attention of a chunk of new tokens over all of it.
 *   mcsd_attn_weight_sums, mcsd_kv_evict_paged
 *                       Attention weights added up for every cached position, and
 *                       a cache cut to a budget by them.
 *   mcsd_token_logprobs
 *                       Log probability, rank and entropy for given tokens, with
 *                       the most probable alternatives.
 *   mcsd_page_assign    Block tables, slot map and free list of a paged cache,
 *                       from the lengths the requests are to have.
 *   mcsd_logits_rules   Penalties, biases and grammar masks on the logits of the
 *                       candidate trees, ahead of sampling and verification.
 *
 * Conventions
 *   - Plain C, plain-old-data structs; the first field of every struct is its
 *     own size in bytes (set it with sizeof) so the layout can be versioned.
 *   - Every data pointer in a *_bufs struct is a DEVICE pointer that the caller
 *     owns; the library never allocates, frees or keeps device memory.  Scratch
 *     space comes in through `workspace` (size from mcsd_*_workspace_bytes) and
 *     may be reused by the caller as soon as the stream has passed the call.
 *     Descriptor structs and the arguments of mcsd_tree_validate are HOST memory.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Calls return after enqueueing; outputs are valid once the stream is
 *     synchronised.  Two calls that share a workspace must be stream-ordered.
 *   - Return value: MCSD_OK or a negative MCSD_E_* code.  Every argument is
 *     validated before the first launch: on an argument error (every code but
 *     MCSD_E_HIP) nothing has been enqueued.  MCSD_E_HIP means the HIP runtime
 *     refused a launch; launches enqueued before it stay enqueued and the
 *     outputs of the call are undefined.  mcsd_last_error() gives a thread-local
 *     message.  No call aborts, throws or synchronises the device.
 *   - Errors in the DATA (token id out of range, zero draft probability, ...)
 *     cannot be seen from the host without a sync; they set bits in the
 *     `flags` output instead (MCSD_FLAG_*).
 *   - Tree layout: nodes 0..N-1 exclude the root.  parent[i] == -1 marks a child of the
 *     root; parent[i] < i is required (any order in which parents precede
 *     children, e.g. generation order).  The children of a node are verified
 *     in ascending node id, which must be the order they were sampled in
 *     (Algorithm 2 depends on it).  "Row" r means the root for r == 0 and node
 *     r-1 otherwise.  N <= MCSD_MAX_NODES.
 *   - The root and the caches.  By default (root_row = 0) the root is the last token of
 *     the context and its keys and values are already in the prefix cache: it is neither a
 *     query nor a key row of the tree block, which is the situation of one verification
 *     step looked at alone.  In a decode loop the root of a step is the endpoint token the
 *     previous step emitted, and the target's forward pass over "root + candidates"
 *     produces the root's keys and values together with the candidates' (its logit row
 *     is row 0 of target_logits).  root_row = 1 in the attention and commit descriptors
 *     describes that: the tensors of the tree block (q, out, k_tree, v_tree) carry
 *     1 + N rows, row 0 = the root and row 1 + i = candidate i; every candidate
 *     attends to the prefix, the root, its ancestors and itself, the root to the prefix
 *     and itself; the commit appends the root and then the accepted path.  parent[]
 *     keeps its N entries and its meaning.  N + root_row <= MCSD_MAX_NODES.
 */
#ifndef MCSD_H
#define MCSD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MCSD_MAX_NODES 128      /* tree nodes per sequence (root excluded) */
#define MCSD_MAX_VOCAB 65536    /* the target row of a node stays in one workgroup's registers */
#define MCSD_MAX_HEAD_DIM 256

enum {
    MCSD_OK = 0,
    MCSD_E_NULL = -1,         /* a required pointer is NULL */
    MCSD_E_SHAPE = -2,        /* a size is non-positive / inconsistent / struct_size wrong */
    MCSD_E_UNSUPPORTED = -3,  /* valid request this build has no kernel for */
    MCSD_E_TREE = -4,         /* N > MCSD_MAX_NODES or parent[] not in parents-first order */
    MCSD_E_WORKSPACE = -5,    /* workspace missing, too small or misaligned (256 B) */
    MCSD_E_HIP = -6           /* the HIP runtime reported an error at launch */
};

enum { MCSD_DTYPE_FP32 = 0, MCSD_DTYPE_BF16 = 1 };
enum { MCSD_WITH_REPLACEMENT = 0, MCSD_WITHOUT_REPLACEMENT = 1,
       MCSD_NAIVE = 2 /* verification only: multi-candidate naive sampling, the ablation's comparison rule */ };

/* bits of mcsd_verify_bufs.flags[b][row] */
enum {
    MCSD_FLAG_NEAR_TIE_ACCEPT = 1,    /* an accept test had |u - ratio| < near_tie_eps */
    MCSD_FLAG_NEAR_TIE_ENDPOINT = 2,  /* u_endpoint within near_tie_eps of an edge of the chosen CDF interval */
    MCSD_FLAG_BAD_TOKEN = 4,          /* candidate id outside [0, V): treated as rejected */
    MCSD_FLAG_ZERO_DRAFT_PROB = 8,    /* q(candidate) == 0: ratio taken as 1 if p > 0 else 0 */
    MCSD_FLAG_ZERO_RESIDUAL = 16,     /* sum max(0, p - q) was not positive after a rejection */
    MCSD_FLAG_NONFINITE = 32,         /* a softmax normaliser was not finite and positive */
    MCSD_FLAG_BAD_TREE = 64,          /* a row with children has no valid q_row entry: handled as a leaf; or the walk
                                         reached gamma_max on a row that accepted a child (tree deeper than gamma_max) */
    MCSD_FLAG_NEAR_TIE_DRAW = 128,    /* mcsd_draft_sample: u_draw within near_tie_eps of an edge of the chosen CDF interval */
    MCSD_FLAG_CACHE_FULL = 256,       /* mcsd_kv_commit: prefix_len + n_accepted > L_stride, nothing committed for this sequence;
                                         mcsd_page_assign: no pages for it, nothing assigned to this sequence */
    MCSD_FLAG_BAD_PAGES = 512,        /* mcsd_page_assign: a negative length, or counts that do not fit the table or the pool;
                                         mcsd_kv_evict_paged: a table entry outside the pool, rows that it names were not moved */
    MCSD_FLAG_SLOTS_FULL = 1024       /* mcsd_page_assign: the slot map ends before this sequence's last slot */
};

const char *mcsd_last_error(void);
const char *mcsd_version(void);

/* Host-side check of a parent array (host pointer): MCSD_OK or MCSD_E_TREE / MCSD_E_NULL. */
int32_t mcsd_tree_validate(const int32_t *parent_host, int32_t n_nodes);

/* ------------------------------------------------------------- tree attention
 * Sec. 3.3.  For sequence b, query head h (KV head g = h / (H_q / H_kv)) and node i:
 *   keys   = prefix positions 0 .. prefix_len[b]-1  and  tree nodes in A(i),
 *            A(i) = {i} U A(parent[i]),  A(-1) = {}
 *   out[b][i][h][:] = softmax_over_keys(scale * <q[b][i][h], K>) . V
 * Inputs are expected to be position-encoded already (each candidate keeps the
 * position it has in its own sequence, i.e. prefix_len + depth - 1).
 * fp32 accumulation on the matrix cores.  The softmax weights enter PV as bf16 for bf16 storage
 * with d == 128, as two bf16 terms (relative error at most 2^-16) for bf16 storage with other d,
 * and as fp32 for fp32 storage.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;              /* sequences */
    int32_t N;              /* tree nodes per sequence, 1..MCSD_MAX_NODES */
    int32_t H_q, H_kv;      /* query / KV heads, H_q % H_kv == 0 */
    int32_t d;              /* head dim: multiple of 4 (fp32) or 8 (bf16), <= MCSD_MAX_HEAD_DIM */
    int32_t dtype;          /* MCSD_DTYPE_* of q, k_*, v_*, out */
    int32_t L_stride;       /* rows allocated per (sequence, KV head) in the prefix cache; prefix_len[b] <= L_stride <= 2^22 */
    float scale;            /* softmax scale, finite and >= 0, normally 1/sqrt(d) */
    int32_t parent_per_seq; /* 0: one parent[N] shared by the batch; 1: parent[B][N] */
    int32_t root_row;       /* 0: the root is in the prefix cache; 1: the tree block has 1+N rows, row 0 = the root */
} mcsd_attn_desc;

typedef struct {
    uint32_t struct_size;
    const void *q;               /* [B][N][H_q][d]   (N here and below: N + root_row rows) */
    const void *k_prefix;        /* [B][H_kv][L_stride][d] */
    const void *v_prefix;        /* [B][H_kv][L_stride][d] */
    const int32_t *prefix_len;   /* [B], 0 <= prefix_len[b] <= L_stride */
    const void *k_tree;          /* [B][H_kv][N][d] */
    const void *v_tree;          /* [B][H_kv][N][d] */
    const int32_t *parent;       /* [N] or [B][N] */
    void *out;                   /* [B][N][H_q][d] */
    void *workspace;             /* >= mcsd_attn_workspace_bytes(desc), 256-byte aligned */
    size_t workspace_bytes;
} mcsd_attn_bufs;

/* Bytes of scratch mcsd_tree_attn needs for this descriptor (0 on a bad descriptor).  0 for fp32
 * storage and for d != 128: such calls neither read nor write a workspace.  The figure depends on
 * the sizes alone: some calls that have to bring a workspace do not use it. */
size_t mcsd_attn_workspace_bytes(const mcsd_attn_desc *desc);
int32_t mcsd_tree_attn(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, void *stream);

/* The same operation for callers that cannot allocate device memory or hand over a workspace:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The
 * split partials go to a buffer of MCSD_STATIC_SCRATCH_BYTES that is part of the library's
 * device image (one copy per GPU, held until the process ends) instead of bufs->workspace,
 * which is ignored together with bufs->workspace_bytes.  Inputs, outputs, stream semantics and
 * results (bit for bit) are those of mcsd_tree_attn.  The call allocates nothing and calls no
 * allocating routine.  A shape whose partials need more than MCSD_STATIC_SCRATCH_BYTES
 * (mcsd_attn_workspace_bytes tells) is refused with MCSD_E_WORKSPACE before anything is enqueued.
 * The first call on a device looks the buffer's address up (module set-up; make it outside
 * graph capture); `stream` must belong to the device that is current at the call.  All calls
 * on one GPU share the one buffer: calls that may overlap on a GPU (different streams, or
 * different host threads on unordered streams) race and must be ordered by the caller.
 * Nothing in the buffer has to survive from one call to the next. */
#define MCSD_STATIC_SCRATCH_BYTES ((size_t)96 << 20)
int32_t mcsd_tree_attn_static(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, void *stream);

/* Test and tuning aid, not needed in normal use: overrides the launch plan of the matrix-core
 * attention kernel for all later calls of this process (0 = automatic for each value).
 * variant 1, 2, 3 = the 32-row x 4-key-stream, 64-row x 2-key-stream and shared-tile kernels;
 * chunk_tiles = 32-key tiles per segment; target_items = workgroups aimed at when the segment
 * length is derived.  Any value but 0 also keeps calls from the kernel that gives a workgroup all
 * keys and a slice of the output columns (small launches, caches of middling capacity), which the
 * automatic plan takes ahead of those three.  The workspace size depends on the plan: query mcsd_attn_workspace_bytes
 * after changing it.  MCSD_E_SHAPE for values out of range. */
int32_t mcsd_attn_plan_override(int32_t variant, int32_t chunk_tiles, int32_t target_items);

/* Paged prefix cache.  The same operation, but the prefix keys and values live in a pool of
 * fixed-size pages shared by all sequences (the usual serving layout): bufs->k_prefix and
 * bufs->v_prefix point to pools [n_pages][H_kv][page_size][d], and logical prefix row r of
 * sequence b is row r % page_size of page block_table[b][r / page_size].  page_size is a
 * multiple of 32; desc->L_stride is the logical capacity, <= max_pages_per_seq * page_size;
 * only the pages that hold rows below prefix_len[b] are read.  A table entry outside
 * [0, n_pages) is a data error: its keys read as zeros (bf16, d == 128) or as page 0 /
 * n_pages-1 (fp32 storage, d != 128); memory outside the pool is never touched.  Everything else (tree
 * block, outputs, workspace) is as for mcsd_tree_attn.
 */
typedef struct {
    uint32_t struct_size;
    int32_t page_size;              /* tokens per page, multiple of 32 */
    int32_t n_pages;                /* pages in the pools */
    int32_t max_pages_per_seq;      /* row length of block_table */
    const int32_t *block_table;     /* [B][max_pages_per_seq] device */
} mcsd_paged_kv;

int32_t mcsd_tree_attn_paged(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, const mcsd_paged_kv *paged,
                             void *stream);

/* --------------------------------------------------------------- verification
 * Algorithm 1 / Algorithm 2 for every row that has children, endpoint draws,
 * and the walk (Sec. 3).  Per sequence b with temperature T = temperature[b]:
 *   p_r = softmax(target_logits[b][r] / T),  q_r = softmax(draft_logits[b][q_row[r]] / T)
 *   for the children c_1 < c_2 < ... of row r, x = cand_tok[b][c_i]:
 *       ratio = min(1, p_r(x) / q_r(x));  accept c_i iff u_accept[b][c_i] <= ratio and ratio > 0
 *       else p_r := max(0, p_r - q_r) / sum_x max(0, p_r - q_r)
 *            and, without replacement only, q_r(x) := 0, q_r := q_r / sum q_r
 *   no child accepted, or r is a leaf: endpoint = inverse CDF of p_r (token-id
 *       order, smallest x whose cumulative probability exceeds u_endpoint[b][r])
 *   walk: r = 0; while a child c of r was accepted: emit cand_tok[c], r = 1 + c;
 *       then emit the endpoint of r.
 *   variant MCSD_NAIVE (Sec. 4.5, footnote; naive sampling of Sec. 2 for one candidate): a
 *       token x is drawn from p_r by inverse CDF at u_endpoint[b][r]; the first child whose
 *       token equals x is accepted, otherwise x is the endpoint; draft logits and u_accept
 *       are not read, ratio is NaN.
 *   T == 0 (argmax sampling, Sec. 4.1/4.5): accept the first child whose token is
 *       argmax target_logits[b][r] (lowest id on ties), otherwise that argmax is
 *       the endpoint; draft logits and uniforms are not read.
 * Every row is evaluated (not only the rows on the accepted path), so results do
 * not depend on evaluation order; uniforms are indexed by slot for the same reason.
 * Elementwise math in fp32 with fp64 reductions; the quantities that decide an
 * accept test are evaluated in fp64.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;
    int32_t N;              /* tree nodes per sequence, 1..MCSD_MAX_NODES */
    int32_t V;              /* vocabulary, 1..MCSD_MAX_VOCAB */
    int32_t P;              /* rows of draft_logits per sequence (rows of the tree that have children) */
    int32_t variant;        /* MCSD_WITH_REPLACEMENT | MCSD_WITHOUT_REPLACEMENT | MCSD_NAIVE */
    int32_t gamma_max;      /* depth bound: row length of accepted_path; out_tokens rows have gamma_max+1 */
    float near_tie_eps;     /* threshold of the MCSD_FLAG_NEAR_TIE_* bits, e.g. 1e-6 */
    int32_t parent_per_seq; /* 0: one tree for the batch (parent[N], q_row[1+N]); 1: one tree per
                               sequence (parent[B][N], q_row[B][1+N]): Sec. 3 verifies each sequence's
                               own candidate tree */
} mcsd_verify_desc;

typedef struct {
    uint32_t struct_size;
    const float *target_logits;  /* [B][1+N][V]   row 0 = root */
    const float *draft_logits;   /* [B][P][V] */
    const int32_t *q_row;        /* [1+N] or [B][1+N]: row of draft_logits for each tree row, -1 for leaves */
    const int32_t *parent;       /* [N] or [B][N] (desc->parent_per_seq) */
    const int32_t *cand_tok;     /* [B][N] candidate token of each node */
    const float *u_accept;       /* [B][N]   uniform in (0,1) for each node's accept test */
    const float *u_endpoint;     /* [B][1+N] uniform in (0,1) for each row's endpoint draw */
    const float *temperature;    /* [B], 0 = argmax sampling */
    int32_t *n_accepted;         /* [B] out: accepted candidates, 0..gamma_max */
    int32_t *accepted_path;      /* [B][gamma_max] out: node ids root-to-leaf, -1 padded */
    int32_t *out_tokens;         /* [B][gamma_max+1] out: accepted tokens then the endpoint, -1 padded */
    int32_t *acc_child;          /* [B][1+N] out: accepted child of each row or -1 */
    int32_t *endpoint;           /* [B][1+N] out: endpoint token of each row, -1 if a child was accepted */
    float *ratio;                /* [B][N] out, nullable: min(1, p/q) tested for each node, NaN if not reached */
    uint32_t *flags;             /* [B][1+N] out: MCSD_FLAG_* bits */
    float *residual_out;         /* [B][1+N][V] out, nullable (parity checks only): p_r when the loop ended */
    void *workspace;             /* unused by this build: may be NULL when mcsd_verify_workspace_bytes is 0 */
    size_t workspace_bytes;
} mcsd_verify_bufs;

size_t mcsd_verify_workspace_bytes(const mcsd_verify_desc *desc);
int32_t mcsd_verify_sample(const mcsd_verify_desc *desc, const mcsd_verify_bufs *bufs, void *stream);

/* One verification step: mcsd_tree_attn and mcsd_verify_sample on `stream`.  Both argument sets
 * are validated before anything is enqueued.  The results are those of the two calls made one
 * after the other; the launches may be arranged differently (the merge of a split attention
 * and the walk share one launch after the verification rows). */
int32_t mcsd_verify_step(const mcsd_attn_desc *attn_desc, const mcsd_attn_bufs *attn_bufs,
                         const mcsd_verify_desc *verify_desc, const mcsd_verify_bufs *verify_bufs,
                         void *stream);

/* ------------------------------------------------------- draft-side candidates
 * Sec. 3.1: the k candidates of every row that has children, sampled from the
 * draft distribution q_r = softmax(draft_logits[b][q_row[r]] / T); this is the
 * step just before verification and its output is the cand_tok input above.
 * For the children c_1 < c_2 < ... < c_k of row r:
 *   MCSD_WITH_REPLACEMENT     cand_tok[b][c_i] = inverse CDF of q_r at u_draw[b][c_i]
 *                             (token-id order, smallest x whose cumulative probability
 *                             exceeds the uniform): k independent draws, Algorithm 1's input;
 *   MCSD_WITHOUT_REPLACEMENT  the same, but draw i is taken from q_r with the tokens
 *                             of draws 1..i-1 zeroed and the rest renormalised (q-bar of
 *                             Eq. (1)): k distinct tokens, Algorithm 2's input;
 *   T == 0                    the k largest draft logits in descending order, lowest id
 *                             on ties; uniforms are not read.
 * Entries of cand_tok whose parent row has no valid q_row are set to -1 and flagged
 * MCSD_FLAG_BAD_TREE.  Requires k <= V for every row.  Elementwise math in fp32
 * (the same exponentials as mcsd_verify_sample), cumulative sums in fp64.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;
    int32_t N;              /* tree nodes per sequence, 1..MCSD_MAX_NODES */
    int32_t V;              /* vocabulary, 1..MCSD_MAX_VOCAB */
    int32_t P;              /* rows of draft_logits per sequence */
    int32_t variant;        /* MCSD_WITH_REPLACEMENT | MCSD_WITHOUT_REPLACEMENT */
    float near_tie_eps;     /* threshold of MCSD_FLAG_NEAR_TIE_DRAW, e.g. 1e-6 */
    int32_t parent_per_seq; /* 0: one tree for the batch; 1: parent[B][N], q_row[B][1+N] */
} mcsd_draft_desc;

typedef struct {
    uint32_t struct_size;
    const float *draft_logits;   /* [B][P][V], 16-byte aligned */
    const int32_t *q_row;        /* [1+N] or [B][1+N]: row of draft_logits for each tree row, -1 for leaves */
    const int32_t *parent;       /* [N] or [B][N] (desc->parent_per_seq) */
    const float *u_draw;         /* [B][N] uniform in (0,1) for each node's draw */
    const float *temperature;    /* [B], 0 = top-k */
    int32_t *cand_tok;           /* [B][N] out */
    uint32_t *flags;             /* [B][N] out: MCSD_FLAG_NEAR_TIE_DRAW / MCSD_FLAG_BAD_TREE / MCSD_FLAG_NONFINITE per node */
} mcsd_draft_bufs;

int32_t mcsd_draft_sample(const mcsd_draft_desc *desc, const mcsd_draft_bufs *bufs, void *stream);

/* ------------------------------------------------ candidate tree and KV commit
 * The two bookkeeping steps around the verification, on the device so that a
 * decode loop needs no host round trip (prefix_len lives in device memory).
 *
 * mcsd_tree_size / mcsd_tree_build: the k-ary candidate tree of a k-configuration
 * (k_1 .. k_gamma; Sec. 3 and Sec. 4.3), in the generation order in which Sec. 3.3
 * packs the candidates into one sequence: level by level, every node of level i-1
 * (the root for i = 1) gets k_i consecutive children.
 *   parent[N], depth[N] (1-based), q_row[1+N] (draft row of every tree row with
 *   children, numbered in row order; -1 for leaves),
 *   position_ids[B][N] = prefix_len[b] + depth[i] - 1 (each candidate keeps the
 *   position it has in its own sequence; nullable, then prefix_len may be NULL too);
 *   with root_row = 1, position_ids[B][1+N]: entry 0 = prefix_len[b] (the root, first
 *   token after the cache), entry 1 + i = prefix_len[b] + depth[i].
 * kconfig is HOST memory (gamma <= 16 entries, each >= 1); N must not exceed
 * MCSD_MAX_NODES (MCSD_E_TREE).  mcsd_tree_size only computes N and P on the host.
 */
int32_t mcsd_tree_size(const int32_t *kconfig_host, int32_t gamma, int32_t *n_nodes, int32_t *n_draft_rows);
int32_t mcsd_tree_build(const int32_t *kconfig_host, int32_t gamma, int32_t B, const int32_t *prefix_len,
                        int32_t *parent, int32_t *depth, int32_t *q_row, int32_t *position_ids, int32_t root_row,
                        void *stream);

/* mcsd_kv_commit: keys and values of generated tokens are cached for reuse (Sec. 3.3);
 * after verification the accepted candidates are generated tokens.  For sequence b with
 * n = n_accepted[b] and L = prefix_len[b], and every layer and KV head:
 *   k_prefix[layer][b][g][L + j] = k_tree[layer][b][g][accepted_path[b][j]],  j = 0..n-1 (same for V)
 *   prefix_len[b] = L + n;  next_root[b] = out_tokens[b][n]  (the endpoint, root of the next tree)
 * If L + n > L_stride nothing is copied, prefix_len[b] is left alone and flags[b] gets
 * MCSD_FLAG_CACHE_FULL (0 otherwise); path entries outside [0, N) end the copy there and set
 * MCSD_FLAG_BAD_TREE; with n outside [0, gamma_max] nothing is copied either, prefix_len[b] is left
 * alone, next_root[b] = out_tokens[b][0] and MCSD_FLAG_BAD_TREE is set.  n_accepted, accepted_path and out_tokens are the outputs of
 * mcsd_verify_sample.  The caches of n_layers layers lie back to back.
 * With root_row = 1 (k_tree, v_tree have 1 + N rows, row 0 = the root, see the conventions):
 *   k_prefix[..][L] = k_tree[..][0],  k_prefix[..][L + 1 + j] = k_tree[..][1 + accepted_path[b][j]],
 *   prefix_len[b] = L + 1 + n;  the cache is full if L + 1 + n > L_stride.
 * The sequence held by the cache after the commit is then: context, root, accepted tokens; the
 * endpoint (next_root) is the root row of the next step.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;
    int32_t N;              /* tree nodes per sequence, 1..MCSD_MAX_NODES */
    int32_t H_kv;
    int32_t d;              /* head dim; d * element size must be a multiple of 16 bytes */
    int32_t dtype;          /* MCSD_DTYPE_* of the caches */
    int32_t L_stride;       /* rows allocated per (sequence, KV head) in the prefix cache */
    int32_t gamma_max;      /* row length of accepted_path; out_tokens rows have gamma_max+1 */
    int32_t n_layers;       /* >= 1 */
    int32_t root_row;       /* 0 | 1, as in mcsd_attn_desc */
} mcsd_commit_desc;

typedef struct {
    uint32_t struct_size;
    void *k_prefix;                 /* [n_layers][B][H_kv][L_stride][d] in/out */
    void *v_prefix;                 /* [n_layers][B][H_kv][L_stride][d] in/out */
    const void *k_tree;             /* [n_layers][B][H_kv][N + root_row][d] */
    const void *v_tree;             /* [n_layers][B][H_kv][N + root_row][d] */
    const int32_t *n_accepted;      /* [B] */
    const int32_t *accepted_path;   /* [B][gamma_max] */
    const int32_t *out_tokens;      /* [B][gamma_max+1] */
    int32_t *prefix_len;            /* [B] in/out */
    int32_t *next_root;             /* [B] out */
    uint32_t *flags;                /* [B] out */
} mcsd_commit_bufs;

int32_t mcsd_kv_commit(const mcsd_commit_desc *desc, const mcsd_commit_bufs *bufs, void *stream);

/* The same commit into a paged prefix cache (layout of mcsd_tree_attn_paged): bufs->k_prefix and
 * bufs->v_prefix are pools [n_layers][n_pages][H_kv][page_size][d], and row L + j of sequence b
 * is row (L + j) % page_size of page block_table[b][(L + j) / page_size]; the pages must already
 * be assigned in the table.  desc->L_stride is the logical capacity (<= max_pages_per_seq *
 * page_size).  A table entry outside [0, n_pages) ends the copy of that sequence there and sets
 * MCSD_FLAG_BAD_TREE; nothing outside the pools is written. */
int32_t mcsd_kv_commit_paged(const mcsd_commit_desc *desc, const mcsd_commit_bufs *bufs, const mcsd_paged_kv *paged,
                             void *stream);

/* ---------------------------------------------------- prefix cache in 4 bits
 * A paged prefix cache (as for mcsd_tree_attn_paged) at 4.25 bits a value: a row of d values (d a
 * multiple of 32) is d / 32 blocks of 32 consecutive ones, each with one scale.
 *   code   sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives
 *   scale  one byte s, the factor 2^(s - 127); s = 255: the whole block reads as NaN
 * A block x is held as s = 127 + e with e the smallest integer for which max|x| <= 7 2^e, within
 * -119..125, and the codes nearest to x 2^-e (ties to the even code, magnitudes above 6 as 6).  A value is off by at most
 * a fifth of itself, or by 2^e / 4 where that is more (7 2^e, a seventh above 6 2^e, is no farther off than others are, which
 * is why the finer scale is taken up to there); only magnitudes above 7 2^125 saturate.  A block that holds a NaN or an
 * infinity gets s = 255.  All of it is exact arithmetic, so that codes and scales are defined to the bit.
 * Layout (uint8, 16-byte aligned), in tiles of 16 rows:
 *   codes  [n_pages][H_kv][page_size / 16][d / 32][16 rows][16 bytes]   value 2i of a block in the low half of byte i
 *   scales [n_pages][H_kv][page_size / 16][d / 32][16 rows]
 * Pools of several layers lie back to back.  A slot is page * page_size + row in the page.  A cache that is not
 * paged is one page per sequence.
 */
typedef struct {
    uint32_t struct_size;
    int32_t page_size;              /* tokens per page, multiple of 32 */
    int32_t n_pages;                /* pages in the pools; n_pages * page_size < 2^31 */
    int32_t max_pages_per_seq;      /* row length of block_table */
    const int32_t *block_table;     /* [B][max_pages_per_seq] device; not read by mcsd_kv_store_fourbit / mcsd_kv_load_fourbit (may be NULL there) */
    void *k_codes, *v_codes;
    void *k_scales, *v_scales;
} mcsd_fourbit_kv;

/* mcsd_tree_attn over a prefix held in 4 bits: q, k_tree, v_tree and out as there, the prefix as written by the
 * calls below; bufs->k_prefix and bufs->v_prefix are ignored.  bf16 only (MCSD_E_UNSUPPORTED otherwise),
 * d a multiple of 32.  A lone token per sequence is a tree of one node.  Prefix keys and values enter the
 * products exactly as what they stand for, accumulation is fp32, and the softmax weights enter PV as in mcsd_tree_attn (bf16 for
 * d == 128, two bf16 terms, at most 2^-17 off, for other d).  Only the pages that hold rows below prefix_len[b] are read, and rows
 * at or past it do not count, whatever they hold.  A table entry outside [0, n_pages) is a data error: its rows read as zeros.  What a node may not see
 * does not reach it, whatever it holds.  How a sequence's keys are split, and with it the last bits of its rows, follows the lengths of
 * the whole batch. */
size_t mcsd_attn_fourbit_workspace_bytes(const mcsd_attn_desc *desc);
int32_t mcsd_tree_attn_fourbit(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, const mcsd_fourbit_kv *kv, void *stream);

/* mcsd_kv_commit_paged into a cache held in 4 bits: bufs->k_prefix and bufs->v_prefix are ignored, the pools of
 * n_layers layers lie back to back, everything else (counts, flags, prefix_len, next_root) is as there.
 * d must be a multiple of 32. */
int32_t mcsd_kv_commit_fourbit(const mcsd_commit_desc *desc, const mcsd_commit_bufs *bufs, const mcsd_fourbit_kv *kv, void *stream);

/* Rows of tokens into the cache (a prompt's keys and values) and back (exactly what they stand for; bf16 holds every one of these values).
 * Row t of the packed arrays goes to, or comes from, slot slot_map[t], all KV heads and layers.  A slot outside [0, n_pages * page_size) is
 * passed over: nothing is stored, a row of the destination is left as it was.  The slots of one store have
 * to differ from each other (two rows for one slot leave a mixture of both). */
typedef struct {
    uint32_t struct_size;
    int32_t T;              /* tokens, 0 <= T; T H_kv d < 2^35 */
    int32_t H_kv;
    int32_t d;              /* multiple of 32, <= MCSD_MAX_HEAD_DIM */
    int32_t dtype;          /* MCSD_DTYPE_* of k and v */
    int32_t n_layers;       /* >= 1 */
    int64_t k_stride, v_stride;               /* elements from a token's row [H_kv][d] to the next one's, >= H_kv * d; times the element size a multiple of 16 bytes */
    int64_t k_layer_stride, v_layer_stride;   /* elements from one layer's rows to the next one's (not used with one layer) */
} mcsd_rows_desc;

typedef struct {
    uint32_t struct_size;
    void *k, *v;                    /* [n_layers][T][H_kv][d] with the strides above, 16-byte aligned: read by the store, written by the load */
    const int32_t *slot_map;        /* [T] */
} mcsd_rows_bufs;

int32_t mcsd_kv_store_fourbit(const mcsd_rows_desc *desc, const mcsd_rows_bufs *bufs, const mcsd_fourbit_kv *kv, void *stream);
int32_t mcsd_kv_load_fourbit(const mcsd_rows_desc *desc, const mcsd_rows_bufs *bufs, const mcsd_fourbit_kv *kv, void *stream);

/* ------------------------------------- prompts in chunks over a paged cache
 * A prompt (or a piece of it, or one decoded token; each sequence of a batch brings as many new tokens as it likes) joins a paged
 * cache of full precision (the layout of mcsd_tree_attn_paged) and attends to all that its sequence then holds:
 * mcsd_page_assign gives the pages and lists the new tokens' slots, mcsd_kv_store_paged writes their rows, mcsd_chunk_attn_paged
 * attends, and afterwards prefix_len is want_len.
 *
 * mcsd_kv_store_paged: row t of the packed arrays goes to slot slot_map[t] = page * page_size + row in the page, all KV heads
 * and layers, unchanged.  A slot outside [0, n_pages * page_size) is passed over.  The slots of one store have to
 * differ from each other.  Pools [n_layers][n_pages][H_kv][page_size][d]; d * element size a multiple of 16 bytes, d <= MCSD_MAX_HEAD_DIM;
 * paged->block_table and max_pages_per_seq are not read (may be NULL, 0); n_pages * page_size < 2^31.  Otherwise mcsd_rows_desc is as
 * for mcsd_kv_store_fourbit.
 */
typedef struct {
    uint32_t struct_size;
    const void *k, *v;              /* [n_layers][T][H_kv][d] with the strides of mcsd_rows_desc, 16-byte aligned */
    const int32_t *slot_map;        /* [T] */
    void *k_pool, *v_pool;          /* 16-byte aligned, not overlapping k and v */
} mcsd_store_bufs;

int32_t mcsd_kv_store_paged(const mcsd_rows_desc *desc, const mcsd_store_bufs *bufs, const mcsd_paged_kv *paged, void *stream);

/* mcsd_chunk_attn_paged.  The new tokens of all sequences are packed: those of b are rows chunk_start[b] .. chunk_start[b+1]-1
 * (slot_start of mcsd_page_assign; ascending, a sequence may bring none).  Row chunk_start[b] + i stands at position prefix_len[b] + i,
 * and its keys are positions 0 .. prefix_len[b] + i of sequence b, those of the new tokens among them, all read from the pages:
 *   out[t][h][:] = softmax_over_keys(scale * <q[t][h], K>) . V,   lse[t][h] = ln sum_over_keys exp(scale * <q[t][h], K>)
 * What a row may not see does not reach it, whatever it holds; rows of out and lse at and past chunk_start[B] are left as they were.  Positions end at
 * L_stride (a sequence that is longer is a data error: its last rows see the positions below L_stride).  A table entry outside [0, n_pages)
 * is a data error: its keys and values read as zeros.  fp32 accumulation; the softmax weights enter PV as in mcsd_tree_attn.  How a
 * sequence's keys are split, and with it the last bits of its rows, follows the lengths of the whole batch.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;              /* sequences, <= 65535 */
    int32_t T;              /* rows of q, out and lse, >= 0; T H_q < 2^30 (a launch's workgroups are limited: T H_q / 32 + min(T, B) H_kv <= 2^23 always fits) */
    int32_t H_q, H_kv;      /* query / KV heads, H_q % H_kv == 0, H_kv <= 65535 */
    int32_t d;              /* head dim <= MCSD_MAX_HEAD_DIM; d * element size a multiple of 16 bytes */
    int32_t dtype;          /* MCSD_DTYPE_* of q, the pools and out */
    int32_t L_stride;       /* logical capacity of a sequence, 1 .. min(2^22, max_pages_per_seq * page_size) */
    float scale;            /* softmax scale, finite and >= 0 */
    int64_t q_stride;       /* elements from a row [H_q][d] of q to the next one's, >= H_q d; a multiple of 16 bytes */
} mcsd_chunk_desc;

typedef struct {
    uint32_t struct_size;
    const void *q;                  /* [T][H_q][d], rows q_stride apart, 16-byte aligned */
    const void *k_pool, *v_pool;    /* [n_pages][H_kv][page_size][d], 16-byte aligned */
    const int32_t *chunk_start;     /* [B+1], taken within [0, T] */
    const int32_t *prefix_len;      /* [B], taken within [0, L_stride] */
    void *out;                      /* [T][H_q][d], 16-byte aligned */
    float *lse;                     /* [T][H_q], nullable */
    void *workspace;                /* >= mcsd_chunk_workspace_bytes(desc), 256-byte aligned */
    size_t workspace_bytes;
} mcsd_chunk_bufs;

size_t mcsd_chunk_workspace_bytes(const mcsd_chunk_desc *desc);     /* 0 on a bad descriptor, and where none is needed (short capacities, few rows) */
int32_t mcsd_chunk_attn_paged(const mcsd_chunk_desc *desc, const mcsd_chunk_bufs *bufs, const mcsd_paged_kv *paged, void *stream);

/* ------------------------------------------- eviction by attention weight
 * mcsd_attn_weight_sums adds up what every cached position of a sequence was given by the softmax of the new rows:
 *   sums[b][g][j] = (j < prefix_len[b] ? sums[b][g][j] : 0) + sum exp(scale * <q[t][h], K_j> - lse[t][h])
 * over the rows t of sequence b that see j, of the last last_rows of its new tokens (0: all of them), and the query heads h of
 * KV head g; j = 0 .. prefix_len[b] + new tokens - 1 (below L_stride), other entries are left as they were.  Positions of new tokens start from 0, so that
 * sums needs no clearing; a sequence without new tokens is left alone.  desc, q, chunk_start, prefix_len and the pages are those of the mcsd_chunk_attn_paged that
 * wrote lse, called before prefix_len is raised.  Sums are fp32 and always added in the same order.
 */
typedef struct {
    uint32_t struct_size;
    int32_t last_rows;              /* >= 0 */
    const void *q;
    const void *k_pool;
    const int32_t *chunk_start, *prefix_len;
    const float *lse;               /* [T][H_q] */
    float *sums;                    /* [B][H_kv][L_stride] in/out */
} mcsd_sums_bufs;

int32_t mcsd_attn_weight_sums(const mcsd_chunk_desc *desc, const mcsd_sums_bufs *bufs, const mcsd_paged_kv *paged, void *stream);

/* mcsd_kv_evict_paged cuts every sequence to m = min(prefix_len[b], keep_len[b]) tokens.  With n = prefix_len[b], f = min(n_first, m)
 * and r = min(n_recent, m - f), every layer and KV head keeps by itself its first f tokens, its last r, and of those between
 * the m - f - r with the largest sums (lowest position on ties; a sum that is no number counts as the smallest).  What is
 * kept moves to positions 0 .. m-1 in ascending order, keys, values and sums alike (keys are position-encoded, so that attention does
 * not mind); kept tells where it stood, prefix_len[b] becomes m.  Entries of sums and kept at and past m and rows
 * at and past m are left as they were, sequences with n <= keep_len[b] keep everything (kept = 0 .. n-1).
 * In place (out_table NULL) rows move within the pages of block_table, which no other sequence may share; mcsd_page_assign with want_len =
 * prefix_len takes the surplus back afterwards.  With out_table they are written to its pages instead, all m of them, which
 * nothing else may share; the pages of block_table are then left as they were (a shared prefix, say).
 * A table entry outside [0, n_pages) is a data error (MCSD_FLAG_BAD_PAGES): rows that lie there, or were to go there, are not moved.
 * prefix_len counts what the cache holds: position ids of later tokens come from the caller's own count.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;              /* sequences, <= 65535 */
    int32_t H_kv;           /* n_layers B H_kv < 2^22 */
    int32_t d;              /* d * element size a multiple of 16 bytes, d <= MCSD_MAX_HEAD_DIM */
    int32_t dtype;          /* MCSD_DTYPE_* of the pools */
    int32_t L_stride;       /* row length of sums and kept, logical capacity, 1 .. min(2^22, max_pages_per_seq * page_size) */
    int32_t n_layers;       /* >= 1 */
    int32_t n_first, n_recent;      /* >= 0 */
} mcsd_evict_desc;

typedef struct {
    uint32_t struct_size;
    void *k_pool, *v_pool;          /* [n_layers][n_pages][H_kv][page_size][d] in/out, 16-byte aligned */
    float *sums;                    /* [n_layers][B][H_kv][L_stride] in/out */
    int32_t *prefix_len;            /* [B] in/out, taken within [0, L_stride] */
    const int32_t *keep_len;        /* [B] (negative: 0) */
    const int32_t *out_table;       /* [B][max_pages_per_seq], nullable */
    int32_t *kept;                  /* [n_layers][B][H_kv][L_stride] out */
    uint32_t *flags;                /* [B] out */
} mcsd_evict_bufs;

int32_t mcsd_kv_evict_paged(const mcsd_evict_desc *desc, const mcsd_evict_bufs *bufs, const mcsd_paged_kv *paged, void *stream);

/* --------------------------------------------- log probabilities of tokens
 * For row i, x = tokens[i], and z = logits[row_map[i]] / T with T = temperature[i] (0, argmax sampling, reads as 1):
 *   logprob[i] = z(x) - lse,  lse = ln sum_y exp z(y)        entropy[i] = -sum_y p(y) ln p(y),  p = exp(z - lse)
 *   rank[i] = tokens y that come before x: z(y) > z(x), or z(y) = z(x) and y < x  (0: x is the most probable)
 *   top_tok[i][0 .. n_top-1], top_logprob: the first n_top tokens of that order and their log probabilities
 * Tokens at -infinity (masked) have probability 0, log probability -infinity and come last, by id, at an infinite T too, where all others
 * are alike.  The order is that of the logits as they are, before the division.
 * x outside [0, V): logprob NaN, rank -1, MCSD_FLAG_BAD_TOKEN, the rest as usual.  A row_map entry outside [0, R): NaN, -1, MCSD_FLAG_BAD_TREE.  A
 * row that holds NaN or +infinity, or nothing but -infinity: NaN, -1, MCSD_FLAG_NONFINITE.  Sums are taken in fp32 per lane and in fp64 across.
 */
typedef struct {
    uint32_t struct_size;
    int32_t rows;           /* rows asked for, 0 .. 2^22 */
    int32_t R;              /* rows of logits, >= 1 */
    int32_t V;              /* vocabulary, 1 .. 2^30 */
    int32_t dtype;          /* MCSD_DTYPE_* of logits */
    int32_t n_top;          /* 0 .. min(V, MCSD_MAX_TOP) */
    int64_t row_stride;     /* elements from a row of logits to the next one, >= V */
} mcsd_logprob_desc;

#define MCSD_MAX_TOP 64

typedef struct {
    uint32_t struct_size;
    const void *logits;             /* [R][V], rows row_stride apart */
    const int32_t *row_map;         /* [rows], NULL: row i is row i, rows <= R */
    const int32_t *tokens;          /* [rows] */
    const float *temperature;       /* [rows], >= 0, nullable (1) */
    float *logprob;                 /* [rows] out */
    float *entropy;                 /* [rows] out, nullable */
    int32_t *rank;                  /* [rows] out, nullable */
    int32_t *top_tok;               /* [rows][n_top] out, NULL with n_top = 0 */
    float *top_logprob;             /* [rows][n_top] out, NULL with n_top = 0 */
    uint32_t *flags;                /* [rows] out */
    void *workspace;                /* >= mcsd_logprob_workspace_bytes(desc), 256-byte aligned */
    size_t workspace_bytes;
} mcsd_logprob_bufs;

size_t mcsd_logprob_workspace_bytes(const mcsd_logprob_desc *desc);     /* 0 on a bad descriptor, and where none is needed (all but few long rows) */
int32_t mcsd_token_logprobs(const mcsd_logprob_desc *desc, const mcsd_logprob_bufs *bufs, void *stream);

/* ------------------------------------------------------- pages from lengths
 * mcsd_page_assign brings the block table of every sequence to the pages that want_len[b] tokens
 * need, ceil(want_len[b] / page_size), on the device.  The pool's free pages are a stack:
 * free_pages[0 .. n_free-1], taken from the top.
 *   1. Pages that a sequence holds beyond its need go back (want_len = 0 gives all of them back), and their
 *      table entries become -1.  They are stacked so that the first page given back by the first such sequence is on top:
 *      giving back what one call has assigned restores the stack.
 *   2. Then the sequences take the pages that they lack, in order of b.  A sequence is served if
 *      what it and all sequences before it lack is there; otherwise (MCSD_FLAG_CACHE_FULL, also where
 *      want_len needs more than max_pages_per_seq pages) it keeps what it holds and gets no slots.  A sequence that does not
 *      fit its table does not count for those behind it.
 *   3. slot_map lists the slots (page * page_size + row) of the new tokens, positions
 *      prefix_len[b] .. want_len[b]-1 of every sequence that was served, one sequence behind the other:
 *      those of b at slot_start[b] .. slot_start[b+1]-1.  Entries behind the last one are -1, so that a
 *      captured mcsd_kv_store_fourbit over max_slots rows stores the new rows alone.  Where max_slots is too few the
 *      map ends there and slot_start with it (MCSD_FLAG_SLOTS_FULL for the sequences that lose slots).
 * Page ids are moved, never followed; a table entry outside [0, n_pages) gives the slot -1.  Data errors (MCSD_FLAG_BAD_PAGES): a
 * sequence with a negative length or n_held outside [0, max_pages_per_seq] is left alone and gets no slots; n_free is
 * taken within [0, n_pages], and a page that would be pushed past n_pages is lost and flags its sequence.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;                      /* sequences */
    int32_t page_size;              /* tokens per page, >= 1 */
    int32_t n_pages;                /* pages in the pool, n_pages * page_size < 2^31 */
    int32_t max_pages_per_seq;      /* row length of block_table, <= 2^30 */
    int32_t max_slots;              /* length of slot_map, <= 2^30 (0 with slot_map = NULL) */
} mcsd_page_desc;

typedef struct {
    uint32_t struct_size;
    const int32_t *prefix_len;      /* [B] tokens in the cache */
    const int32_t *want_len;        /* [B] tokens there is to be room for */
    int32_t *n_held;                /* [B] in/out: pages assigned */
    int32_t *block_table;           /* [B][max_pages_per_seq] in/out */
    int32_t *free_pages;            /* [n_pages] in/out; entries at and above n_free mean nothing */
    int32_t *n_free;                /* [1] in/out */
    int32_t *slot_start;            /* [B+1] out; NULL exactly when slot_map is */
    int32_t *slot_map;              /* [max_slots] out, nullable */
    uint32_t *flags;                /* [B] out */
} mcsd_page_bufs;

int32_t mcsd_page_assign(const mcsd_page_desc *desc, const mcsd_page_bufs *bufs, void *stream);

/* ------------------------------------------------------------ rules on logits
 * What a request asks of its next token besides the temperature, applied to the logit rows of its
 * candidate tree before they are sampled from (mcsd_draft_sample) or verified (mcsd_verify_sample).  The row of tree row r
 * (0 = root, 1 + i = node i) of sequence b continues the tokens
 *   history[b][0 .. hist_len[b]-1], then cand_tok[b] of the node's ancestors and of the node itself,
 * of which the first min(prompt_len[b], hist_len[b]) are the prompt (a candidate never is).  With count(x) = how often x stands behind the
 * prompt, seen(x) = x stands anywhere, and per sequence a repetition penalty R > 0, a presence
 * penalty P and a frequency penalty F:
 *   z(x) = logits;   if seen(x): z > 0 ? z / R : z R;   z -= F count(x) + P [count(x) > 0];
 *   z += bias(x)  (of several entries of the list for one token the last one counts);   mask bit 0: z = -infinity
 * out is fp32, whatever the logits are; with fp32 logits it may be the logits themselves (in place: what no rule touches
 * is then neither read nor written).  Token ids outside [0, V) are passed over.  A row whose mask
 * leaves nothing becomes -infinity throughout (mcsd_verify_sample flags such a row MCSD_FLAG_NONFINITE); a draft row has to keep as
 * many tokens as are to be drawn from it without replacement.  R must be greater than 0; the arithmetic is fp32.
 */
typedef struct {
    uint32_t struct_size;
    int32_t B;
    int32_t N;              /* tree nodes per sequence, 0..MCSD_MAX_NODES (0: the root's row alone) */
    int32_t V;              /* vocabulary, >= 1 */
    int32_t R;              /* logit rows per sequence */
    int32_t dtype;          /* MCSD_DTYPE_* of logits */
    int32_t parent_per_seq; /* 0: one tree for the batch; 1: parent[B][N], row_map[B][1+N] */
    int32_t row_begin, row_end; /* tree rows dealt with, 0 <= row_begin <= row_end <= 1 + N (a level of the tree, say) */
    int32_t hist_stride;    /* row length of history, <= 2^30 */
    int32_t n_bias;         /* row length of bias_tok and bias_val, <= 2^30 */
} mcsd_logits_desc;

typedef struct {
    uint32_t struct_size;
    const void *logits;             /* [B][R][V] */
    float *out;                     /* [B][R][V] */
    const int32_t *row_map;         /* [1+N] or [B][1+N]: logit row of every tree row, no row twice, outside [0, R) = none (q_row of the
                                       draft logits); NULL: tree row r is row r, R = 1 + N */
    const int32_t *parent;          /* [N] or [B][N]; may be NULL with N = 0 */
    const int32_t *cand_tok;        /* [B][N]; may be NULL with N = 0 */
    const int32_t *history;         /* [B][hist_stride], NULL with hist_stride = 0 */
    const int32_t *hist_len;        /* [B] (taken within [0, hist_stride]), NULL with hist_stride = 0 */
    const int32_t *prompt_len;      /* [B], nullable (0): tokens of the history that are the prompt, taken within [0, hist_len[b]] */
    const float *repetition;        /* [B], nullable (1) */
    const float *presence;          /* [B], nullable (0) */
    const float *frequency;         /* [B], nullable (0) */
    const int32_t *bias_tok;        /* [B][n_bias], ids outside [0, V) = no entry; NULL with n_bias = 0 */
    const float *bias_val;          /* [B][n_bias] */
    const uint32_t *mask;           /* [B][R][ceil(V / 32)], nullable: bit x % 32 of word x / 32 set = token x is allowed */
} mcsd_logits_bufs;

int32_t mcsd_logits_rules(const mcsd_logits_desc *desc, const mcsd_logits_bufs *bufs, void *stream);

/* ------------------------------------------------------------ profiling aid
 * Not part of the verification step.  mcsd_kernel_timing(1) makes every kernel launch of the
 * calls above carry a start and a stop event tied to that one dispatch (totals are reset), so
 * that the time between them is the kernel's own execution time, without launch latency or
 * the gaps between kernels; mcsd_kernel_timing(0) stops.  mcsd_kernel_timing_read waits for
 * the recorded events and returns the summed duration (ms) and the number of launches of
 * kernel `id` (0 .. mcsd_kernel_count()-1, named by mcsd_kernel_name).  Events are host
 * objects; no device memory is allocated.  Not for use under graph capture.
 */
int32_t mcsd_kernel_timing(int32_t enable);
int32_t mcsd_kernel_count(void);
const char *mcsd_kernel_name(int32_t id);
int32_t mcsd_kernel_timing_read(int32_t id, double *total_ms, int64_t *launches);

#ifdef __cplusplus
}
#endif
#endif /* MCSD_H */
