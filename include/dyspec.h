/*
 * dyspec.h -- C ABI of the MI355X (gfx950) library for one DySpec speculative step
 * (arXiv 2410.11744): greedy token-tree construction, tree-masked attention and
 * multi-candidate tree verification; for the paged key/value cache and the prompts
 * around it, its page tables, filtered logits and drawn tokens.
 *
 * Conventions shared by every entry point
 *  - Pointers marked DEVICE address HBM of the current HIP device; pointers marked HOST
 *    address ordinary host memory that is read before the call returns.  The caller owns
 *    every buffer; the library allocates no device memory and keeps no state between calls
 *    (dyspec_build_tree_threshold shares 8 KB of pinned host memory among the calls in progress).
 *  - Work is enqueued on `hip_stream` (a hipStream_t passed as void*, NULL = default
 *    stream); calls return without synchronising.  Two calls that write the same buffers
 *    race unless ordered by the stream.  Apart from dyspec_build_tree_threshold (which
 *    waits for each level) a call enqueues kernel launches only -- no allocation, memset,
 *    copy or wait -- so, after dyspec_init() or one plain call on the device, calls may be
 *    recorded into a HIP graph on a capturing stream and replayed.
 *  - Errors are return codes (< 0).  Arguments are validated on the host before anything
 *    is launched; a call that returns an error has launched nothing.
 *  - Alignment of DEVICE pointers is part of that validation (DYSPEC_BAD_ARG otherwise):
 *    attention tensors, logit tables, row_stats and the tree-attention workspace 16 bytes;
 *    ancestor masks and the builders' workspaces 8 bytes; every other array 4 bytes.  (The
 *    calls around a paged cache and dyspec_prompt_attn say their own: they take strided rows.)
 *  - A batch holds n_seq independent sequences packed back to back.  Sequence s owns tree
 *    rows [node_offset[s], node_offset[s+1]) of every per-node array and prefix rows
 *    [kv_offset[s], kv_offset[s] + prefix_len[s]) of k_prefix / v_prefix.  Row 0 of each
 *    tree is the root: the last committed token, whose logits open the tree
 *    (Section 4.2, first paragraph).  Node indices stored in the arrays (parent, links,
 *    accepted_nodes, mask bits) are LOCAL to the sequence.
 *  - Uniform random numbers come from Philox4x32-10 (Salmon et al., SC'11) with key =
 *    seed and a counter that names each draw by the path of sibling ranks from the root,
 *    so results do not depend on node numbering or on which kernel makes the draw.
 */
#ifndef DYSPEC_H
#define DYSPEC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t dyspec_status;
enum {
    DYSPEC_OK = 0,
    DYSPEC_BAD_ARG = -1,             /* null pointer, non-positive size, temperature <= 0 ... */
    DYSPEC_BAD_SHAPE = -2,           /* offsets not increasing, heads not divisible, ...      */
    DYSPEC_UNSUPPORTED = -3,         /* dtype / head_dim / vocabulary outside the built kernels */
    DYSPEC_WORKSPACE_TOO_SMALL = -4,
    DYSPEC_HIP_ERROR = -5            /* a HIP call failed; hipGetLastError() still holds it   */
};

/* Tensor element types of dyspec_tree_attn.  DYSPEC_BF16_WAVE: bf16 storage handled by the
 * one-workgroup-per-(row, head) kernel (fp32 arithmetic, any head_dim <= 256 that is a multiple of 4) instead of the
 * matrix-core kernel. */
enum { DYSPEC_F32 = 0, DYSPEC_BF16 = 1, DYSPEC_BF16_WAVE = 0x101 };

#define DYSPEC_MAX_SEQ 64            /* sequences per call                                */
#define DYSPEC_MAX_NODES 2048        /* tree rows per sequence, root included (attention, reorder, verify) */
#define DYSPEC_MAX_BUILD_NODES 1024  /* ... for the two tree builders, whose per-tree state lives in LDS   */
#define DYSPEC_MAX_VOCAB 32768       /* vocabulary handled by the build / verify kernels  */

/* Ragged batch description; all three arrays are HOST memory. */
typedef struct {
    int32_t n_seq;                   /* 1 .. DYSPEC_MAX_SEQ                               */
    const int32_t* node_offset;      /* [n_seq+1] increasing, node_offset[0] = 0          */
    const int32_t* prefix_len;       /* [n_seq]   >= 0                                    */
    const int64_t* kv_offset;        /* [n_seq+1] first prefix row of each sequence       */
} dyspec_batch;

/* A packed batch of token trees; every array is DEVICE memory of length node_offset[n_seq].
 * Children of a node are linked in the order they were sampled, which is the order
 * verification must try them (Algorithm 3, loop over CurrentNode.branches). */
typedef struct {
    int32_t* parent;                 /* -1 for the root and for rows that were not built  */
    int32_t* token;                  /* -1 for the root                                   */
    int32_t* sib_rank;               /* 0 for a first child, 1 for the next sampling ...  */
    int32_t* first_child;            /* -1 = leaf                                         */
    int32_t* next_sibling;           /* -1 = last sampled child                           */
    int32_t* depth;                  /* 0 for the root                                    */
} dyspec_tree;

/* Words per row of the ancestor bitmask for this batch: ceil(max_s N_s / 64). */
int32_t dyspec_mask_words(const dyspec_batch* batch);

/* Bytes of DEVICE workspace the named call can use for this batch (0 = none). */
enum { DYSPEC_WS_BUILD_TREE = 0, DYSPEC_WS_TREE_ATTN = 1, DYSPEC_WS_VERIFY = 2 };
#define DYSPEC_ATTN_COUNTER_BYTES 4096   /* head of a tree-attention workspace: see dyspec_tree_attn */
size_t dyspec_workspace_bytes(int32_t which, const dyspec_batch* batch, int32_t vocab,
                              int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim);

const char* dyspec_status_string(dyspec_status s);

/*
 * dyspec_init -- optional one-time set-up on the CURRENT device: has the runtime load the
 * kernels, raises their dynamic-LDS limits, takes the address of the static scratch array.
 * Every entry point does what it needs of this at its first use; calling dyspec_init first
 * moves those few milliseconds out of the first calls of a latency-sensitive loop.  Launches
 * nothing, allocates only those 8 KB of host memory; idempotent and safe to call from several threads.
 */
dyspec_status dyspec_init(void);

/*
 * dyspec_build_tree -- greedy fixed-budget construction of the draft token tree
 * (Algorithm 1; Section 4.2; Appendix A.1) plus the tree-attention mask (Section 2).
 *
 * For each sequence, N = node_offset[s+1]-node_offset[s] rows are built, the root
 * included.  Starting from the single slot (parent = root, value 1), the slot with the
 * largest estimated value v is taken (earliest-opened slot on a tie); a token y is drawn
 * from the parent's draft distribution with the parent's earlier children removed and the
 * rest renormalised (R); the node is appended; the slots "next sampling at the same
 * position" with value v*(1-R[y]) and "first child of the new node" with value v*R[y] are
 * opened (slots of value 0 are not).  Draft distributions are softmax(draft_logits[i]/T_d),
 * where row i is the distribution that FOLLOWS node i (creation index): the table stands in
 * for the draft model call of Algorithm 1.  Arithmetic on values and distributions is fp64.
 * y is the smallest index whose cumulative residual weight exceeds u * (total weight),
 * u in [0,1) with 24 random bits.
 *
 *   draft_logits  DEVICE [sum N, vocab] fp32, row-major, base 16-byte aligned
 *   draft_temp    HOST   [n_seq] > 0
 *   tree          DEVICE outputs (all six arrays)
 *   est_value     DEVICE [sum N] fp32: v of the slot each node was drawn from (root: 1)
 *   anc_mask      DEVICE [sum N, mask_words] u64: bit i of row j set iff local node i is an
 *                 ancestor of local node j or i == j
 *   n_built       DEVICE [n_seq]: rows actually built (< N only if no slot of positive
 *                 value is left); later rows keep parent = token = -1 and their own mask bit
 *                 -1: the builder waited for a draw in vain and gave up (a fault of the library
 *                 or the device, not of the tables; the rows it had built stand)
 *   workspace     DEVICE, dyspec_workspace_bytes(DYSPEC_WS_BUILD_TREE, ...) bytes, 8-byte
 *                 aligned, contents overwritten (about 4.2 KB per row): every row's
 *                 maximum and the totals of its runs of 128 tokens, computed for all
 *                 rows at once before the serial expansion, and the tokens drawn from
 *                 the row so far; a draw then touches one run of the parent's row.
 *                 NULL or fewer bytes: the expansion makes a pass over the parent's whole
 *                 row at every draw instead (several times slower; the same tree, unless a
 *                 decision is closer than the rounding of the row's fp64 sums, about 1e-13:
 *                 children with equal logits can be that close).
 * A call builds the same tree every time, whatever runs beside it.  In other batches (of more
 * sequences, or with a wider tree) the root's row may be summed in another order: the same tree
 * but for decisions that close.
 * vocab <= DYSPEC_MAX_VOCAB, N <= DYSPEC_MAX_BUILD_NODES (DYSPEC_BAD_SHAPE beyond).
 */
dyspec_status dyspec_build_tree(const float* draft_logits, int32_t vocab,
                                const dyspec_batch* batch, const float* draft_temp,
                                uint64_t seed, const dyspec_tree* tree, float* est_value,
                                uint64_t* anc_mask, int32_t* n_built,
                                void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * dyspec_build_tree_threshold -- construction of the draft token tree with a threshold
 * (Algorithm 2; Section 4.4, Appendix A.2), the level-by-level form of dyspec_build_tree.
 *
 * Per sequence, starting from the root alone (value 1): every node i of the current level
 * with value v_i >= t reads its draft row D = softmax(draft_logits[i]/T) and, while v_i >= t
 * and rows are left, draws y from D (inverse CDF as in dyspec_build_tree, the draw named by
 * the node's sibling-rank path and the number of children it already has), appends a child
 * with token y, estimated value v_i and own value v_i*D[y], then sets v_i <- v_i*(1-D[y]),
 * D[y] <- 0, D <- norm(D).  The children of a level are the next level.  The loop condition
 * is read as "at or above the threshold" (the listing prints the opposite sign; the text says
 * nodes above the threshold are extended).  Rows are numbered in creation order: level by
 * level, parents in row order, children in sampling order; construction stops when the
 * sequence's N rows (root included) exist.  With t = the smallest est_value a run of
 * dyspec_build_tree produced, the same tree results (Appendix A.1) when both give a node
 * the same draft row; here a node reads the row of its own index, so the two calls agree on
 * tables whose rows are alike.  Nodes of a level are expanded in parallel, one workgroup each.
 *
 *   threshold     HOST [n_seq] > 0 (the paper suggests about 1/N)
 *   n_levels      HOST out, may be NULL: levels expanded (the number of draft model calls
 *                 the paper's loop would make), the widest sequence counting
 *   workspace     DEVICE, 8-byte aligned, dyspec_build_tree_threshold_workspace_bytes()
 *                 bytes, REQUIRED (DYSPEC_WORKSPACE_TOO_SMALL otherwise)
 *   all other arguments, and the limits on vocab and N, as for dyspec_build_tree.
 * The call waits for every level (the device reports the level's size, which sizes the next
 * launch), so it returns with the tree complete and cannot be captured in a graph: a stream
 * that is capturing is refused with DYSPEC_HIP_ERROR before anything is launched.
 */
dyspec_status dyspec_build_tree_threshold(const float* draft_logits, int32_t vocab,
                                          const dyspec_batch* batch, const float* draft_temp,
                                          const double* threshold, uint64_t seed,
                                          const dyspec_tree* tree, float* est_value,
                                          uint64_t* anc_mask, int32_t* n_built, int32_t* n_levels,
                                          void* workspace, size_t workspace_bytes, void* hip_stream);
size_t dyspec_build_tree_threshold_workspace_bytes(const dyspec_batch* batch);

/*
 * dyspec_dfs_reorder -- block-sparsity friendly token order (Appendix "Block-Sparsity
 * Friendly Token Order"): renames the nodes of every built tree by their position in the
 * depth-first pre-order walk that visits children in sampling order.  Subtrees become
 * contiguous runs of rows, parents still precede children, and the ancestor mask of the renamed
 * tree has fewer non-empty 32x32 blocks for tree attention to visit.  Rows that were never
 * attached (n_built < N) follow the tree in index order.
 *
 *   tree           DEVICE inputs (all six arrays, as written by dyspec_build_tree)
 *   tree_out       DEVICE outputs, six arrays distinct from the inputs: the renamed tree
 *   order          DEVICE [sum N] i32: order[node_offset[s] + new] = old local index; the caller
 *                  gathers token-aligned tensors (q, k_tree, v_tree, logit rows) with it
 *   anc_mask_out   DEVICE [sum N, mask_words] u64: ancestor mask of the renamed tree
 * Verification of the renamed tree reads logit rows by the new indices (gathered tables), and
 * Philox draws are named by paths of sibling ranks, so its outcome does not change.
 */
dyspec_status dyspec_dfs_reorder(const dyspec_batch* batch, const dyspec_tree* tree,
                                 const dyspec_tree* tree_out, int32_t* order,
                                 uint64_t* anc_mask_out, void* hip_stream);

/*
 * dyspec_tree_attn -- one layer of tree attention (Section 2, "Tree Attention";
 * Appendix C for the block-sparse treatment of the tree part).
 *
 * For every tree row j and query head h:
 *   out[j,h,:] = softmax_k( scale * <q[j,h,:], K[k, h/G, :]> ) . V[k, h/G, :]
 * over all prefix keys of the sequence and over the tree keys i whose bit is set in
 * anc_mask row j; G = n_q_heads / n_kv_heads.
 *
 *   q, out            DEVICE [sum N, n_q_heads, head_dim]
 *   k_prefix,v_prefix DEVICE [kv rows, n_kv_heads, head_dim]
 *   k_tree, v_tree    DEVICE [sum N, n_kv_heads, head_dim]
 *   anc_mask          DEVICE [sum N, mask_words] as written by dyspec_build_tree.  Bit i of row j
 *                     may be set only for i <= j (an ancestor is created before its descendants,
 *                     so its row index is smaller, in creation order and in depth-first order
 *                     alike); the matrix-core path does not look at tree keys past the largest
 *                     row of a tile, so bits above the diagonal are ignored there
 *   dtype             DYSPEC_F32 (any head_dim <= 256, multiple of 4) or DYSPEC_BF16
 *                     (head_dim 64 or 128; matrix-core path, fp32 accumulation)
 * All tensors are dense row-major and 16-byte aligned (checked: DYSPEC_BAD_ARG).
 *   workspace         DEVICE, 16-byte aligned, dyspec_workspace_bytes(DYSPEC_WS_TREE_ATTN, ...)
 *                     bytes.  Non-zero only for batches whose (row tiles) x (KV heads) leave most
 *                     of the chip idle: the bf16 path then splits every prefix over several
 *                     workgroups; each leaves its share of every row there (bf16) and the one
 *                     that finishes last merges them, in the same launch.  The first
 *                     DYSPEC_ATTN_COUNTER_BYTES of the workspace are the arrival counters of
 *                     that hand-over: they must be ZERO when a call starts and every call
 *                     leaves them zero again, so a workspace is cleared once, after it is
 *                     allocated (hipMemset), and never again; the rest is overwritten.  NULL or
 *                     fewer bytes: no split (same result up to the bf16 rounding of the parts).  A
 *                     non-NULL workspace that is not 16-byte aligned is DYSPEC_BAD_ARG.
 */
dyspec_status dyspec_tree_attn(const void* q, const void* k_prefix, const void* v_prefix,
                               const void* k_tree, const void* v_tree,
                               const uint64_t* anc_mask, const dyspec_batch* batch,
                               int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                               int32_t dtype, float softmax_scale, void* out,
                               void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * dyspec_tree_attn_static_scratch -- dyspec_tree_attn for callers that cannot allocate device
 * memory and have none to hand over as a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same operation, arguments, kernels and results as
 * dyspec_tree_attn called with a workspace of dyspec_workspace_bytes(DYSPEC_WS_TREE_ATTN, ...)
 * bytes; the partial results of a split prefix go to an array of DYSPEC_STATIC_SCRATCH_BYTES that
 * is part of the library's device image (each GPU the library runs on holds its copy until the
 * process ends).  The call allocates and frees nothing.  A batch whose split needs more than
 * DYSPEC_STATIC_SCRATCH_BYTES is refused with DYSPEC_WORKSPACE_TOO_SMALL (nothing launched).
 * Every call on one GPU uses the same array: calls that overlap on one GPU (two streams, two
 * threads) race; order them, or give the overlapping ones dyspec_tree_attn with workspaces of
 * their own.  The arrival counters at the head of the array start as zeros with the device image
 * and every call leaves them zero; nothing else in it has to survive from one call to the next.
 */
#define DYSPEC_STATIC_SCRATCH_BYTES (8u << 20)
dyspec_status dyspec_tree_attn_static_scratch(const void* q, const void* k_prefix, const void* v_prefix,
                                              const void* k_tree, const void* v_tree,
                                              const uint64_t* anc_mask, const dyspec_batch* batch,
                                              int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                              int32_t dtype, float softmax_scale, void* out,
                                              void* hip_stream);

/*
 * dyspec_tree_attn_layers -- dyspec_tree_attn for n_layers stacked layers in one call
 * (the same operation as above, Section 2 "Tree Attention", once per layer; the tree and
 * its mask are the same in every layer of one speculative step, the tensors are not).
 * Layer l reads q, k_prefix/v_prefix and k_tree/v_tree at element offsets l * q_layer_stride,
 * l * kv_prefix_layer_stride and l * kv_tree_layer_stride from the base pointers and writes
 * out at l * q_layer_stride; within a layer the layout is that of dyspec_tree_attn.  Strides
 * are >= 0 and keep every layer 16-byte aligned.  The bf16 matrix-core path runs all layers
 * in ONE launch (workgroups of all layers fill the chip together, so short prefixes need
 * no split and pay one launch latency); other dtypes launch once per layer.  This is for
 * callers that hold all layers' tensors at once (benchmarks, layer-parallel schedules);
 * a model that computes layer l+1's Q from layer l's output calls dyspec_tree_attn.
 *   workspace  as for dyspec_tree_attn (its first DYSPEC_ATTN_COUNTER_BYTES zero when the call
 *              starts), dyspec_tree_attn_layers_workspace_bytes() bytes.
 *   n_layers   1 .. 65535
 */
dyspec_status dyspec_tree_attn_layers(const void* q, const void* k_prefix, const void* v_prefix,
                                      const void* k_tree, const void* v_tree,
                                      const uint64_t* anc_mask, const dyspec_batch* batch,
                                      int32_t n_layers, int64_t q_layer_stride,
                                      int64_t kv_prefix_layer_stride, int64_t kv_tree_layer_stride,
                                      int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                      int32_t dtype, float softmax_scale, void* out,
                                      void* workspace, size_t workspace_bytes, void* hip_stream);
size_t dyspec_tree_attn_layers_workspace_bytes(const dyspec_batch* batch, int32_t n_layers,
                                               int32_t n_q_heads, int32_t n_kv_heads,
                                               int32_t head_dim);

/*
 * dyspec_verify -- vocabulary softmax of every tree row and multi-candidate tree
 * rejection sampling (Algorithm 3; Appendix A.3; Section 2 for the one-candidate rule).
 *
 * Data-parallel part, one workgroup per tree row p: the maximum and the sum of exponentials
 * of draft_logits[p]/T_d and of target_logits[p]/T_t (row_stats), i.e. the normalisers of
 * D = softmax(draft_logits[p]/T_d) and R = softmax(target_logits[p]/T_t).
 * Walk, one workgroup per sequence, from the root: for each child n of the current node in
 * sampling order, with token y: draw c uniform in [0,1); accept iff c < R[y]/D[y]
 * (equivalently c*D[y] < R[y]); on a reject R <- norm(max(R-D,0)) with D as it stands, then
 * D[y] <- 0 and D <- norm(D); the scan of the children ends early when D is empty.  Move to
 * the accepted child; when none is accepted sample the step's last token from R; when the
 * walk reaches a leaf sample it from the leaf's target row if emit_bonus != 0 (the printed
 * algorithm returns without it: final_token = -1).  The final token is the smallest index
 * whose cumulative probability exceeds u * (total), u in [0,1) with 24 random bits.
 * target_temp[s] == 0 (the temperature-0 target of Section 5's tables) is the limit
 * T_t -> 0+: R is all mass on the largest target logit of the row, the smallest index
 * winning a tie, so the walk follows the target's argmax token down the tree and the last
 * token is the argmax of the row where it stops; the draws are still taken, in the same order.
 *
 *   draft_logits, target_logits DEVICE [sum N, vocab] fp32 (row i = distribution after node i),
 *                               rows dense, base pointers 16-byte aligned
 *   draft_temp                  HOST [n_seq] > 0
 *   target_temp                 HOST [n_seq] >= 0, independent of draft_temp
 *   tree                        DEVICE inputs (token, first_child, next_sibling are read)
 *   row_stats    DEVICE [sum N,4] fp32: max and sum-exp of draft/T_d, then of target/T_t
 *                (rows of a sequence with T_t == 0: largest raw target logit, then its index)
 *   accept_ratio DEVICE [sum N] fp32: R[y]/D[y] seen by every child the walk tested (root: 0;
 *                -1: not tried because the draft distribution was exhausted; -2: never reached)
 *   accepted_nodes DEVICE [sum N] i32: per sequence, from its node_offset, the accepted
 *                  local node indices in order (root excluded); n_accepted [n_seq]
 *   final_token  DEVICE [n_seq]: token emitted where the walk stopped (-1 if none)
 *   min_margin   DEVICE [n_seq] fp32: smallest |c - accept_ratio| over tested children
 *   workspace, workspace_bytes  not used (verification needs no scratch memory); pass NULL, 0
 * Arithmetic is fp32.  vocab <= DYSPEC_MAX_VOCAB.
 */
dyspec_status dyspec_verify(const float* draft_logits, const float* target_logits,
                            int32_t vocab, const dyspec_batch* batch, const dyspec_tree* tree,
                            const float* draft_temp, const float* target_temp, uint64_t seed,
                            int32_t emit_bonus, float* row_stats, float* accept_ratio,
                            int32_t* accepted_nodes, int32_t* n_accepted, int32_t* final_token,
                            float* min_margin, void* workspace, size_t workspace_bytes,
                            void* hip_stream);

/*
 * dyspec_verify_bf16 -- dyspec_verify on bf16 logit tables (DEVICE [sum N, vocab] bf16, rows
 * dense, base pointers 16-byte aligned): the same operation (Algorithm 3), every logit
 * widened to fp32 as it is read, half the bytes for the statistics pass.  All other
 * arguments, outputs and error behaviour as for dyspec_verify.
 */
dyspec_status dyspec_verify_bf16(const void* draft_logits, const void* target_logits,
                                 int32_t vocab, const dyspec_batch* batch, const dyspec_tree* tree,
                                 const float* draft_temp, const float* target_temp, uint64_t seed,
                                 int32_t emit_bonus, float* row_stats, float* accept_ratio,
                                 int32_t* accepted_nodes, int32_t* n_accepted, int32_t* final_token,
                                 float* min_margin, void* workspace, size_t workspace_bytes,
                                 void* hip_stream);

/* ================================================================================================
 * The paged cache around a speculative step.  A server keeps the keys and values of all its sequences in
 * one pool of pages; a step appends its new tokens (a chunk of a prompt, one token, a draft tree), lets
 * them attend to what the pages hold, and after dyspec_verify keeps the accepted path.
 *
 * Here a batch's node_offset counts NEW tokens (0 .. DYSPEC_MAX_CHUNK per sequence; a sequence may have
 * none) and prefix_len the tokens that the cache holds before them; kv_offset is not read.  New token j of
 * sequence s has place prefix_len[s] + j, which is row (place % page_size) of page
 * page_table[s][place / page_size].
 * ================================================================================================ */
#define DYSPEC_MAX_CHUNK (1 << 20)          /* new tokens per sequence                                  */
#define DYSPEC_MAX_CONTEXT (1 << 30)        /* tokens of a sequence, new ones included                  */
#define DYSPEC_PAGED_COUNTER_BYTES 16384    /* head of a dyspec_paged_attn workspace                    */
/* Up to 8192 heads and 2^20 elements a token; (n_q_heads / n_kv_heads)^2 times a sequence's new tokens below
 * 2^32; up to 2^23 new tokens in a batch, and up to 2^27 of them times n_q_heads for attention
 * (DYSPEC_BAD_SHAPE beyond). */

/* One layer's pool.  Page p's rows are k + p * page_stride + row * n_kv_heads * head_dim (elements), dense
 * in the page; pages may lie apart (K and V pages in turns: page_stride of two pages). */
typedef struct {
    void* k;                         /* DEVICE [n_pages, page_size, n_kv_heads, head_dim], 16-byte aligned */
    void* v;                         /* DEVICE, as k                                      */
    const int32_t* page_table;       /* DEVICE [n_seq, max_pages], rows table_stride apart */
    int32_t n_pages;                 /* pages of the pool                                 */
    int32_t page_size;               /* rows of a page: a power of two, 8 .. 65536        */
    int32_t max_pages;               /* entries of a table row                            */
    int32_t table_stride;            /* >= max_pages                                      */
    int64_t page_stride;             /* elements, >= page_size * n_kv_heads * head_dim, a multiple of 16 bytes */
} dyspec_paged_kv;
/* Table entries that the places of a sequence reach are page numbers in [0, n_pages); others are not read.
 * One outside that range is an error of the caller that is kept inside the cache: nothing is written for its
 * rows, and attention reads some page of the pool in its place.  Sequences may share pages that none of their
 * new tokens lie in. */

/*
 * dyspec_kv_append -- the new tokens' keys and values go into the pages, keys and queries rotated by their
 * position on the way.
 *
 * Rotation: token j has position pos = prefix_len[s] + (rel_pos ? rel_pos[j] : j) (a draft tree passes its
 * depths) and pair i of a head, i < n_freq, is turned by the angle a = pos * inv_freq[i], taken in 64 bits:
 *   (x, y) -> (x cos a - y sin a, x sin a + y cos a), rounded once.
 * Pair i is elements (i, i + n_freq) of the head, or (2i, 2i + 1) if interleaved != 0; elements from
 * 2 * n_freq on, and all of V, are copied.
 *
 *   q          DEVICE [sum N, n_q_heads, head_dim], tokens q_stride elements apart, or NULL (n_q_heads 0)
 *   k, v       DEVICE [sum N, n_kv_heads, head_dim], tokens k_stride / v_stride elements apart
 *              (slices of one projection's rows can be passed as they are; heads are dense)
 *   rel_pos    DEVICE [sum N] i32 or NULL
 *   inv_freq   DEVICE [n_freq] fp32 (NULL if n_freq is 0: nothing is turned)
 *   n_freq     0 .. head_dim / 2
 *   q_out      DEVICE [sum N, n_q_heads, head_dim] dense; may be q where that is dense
 *   k_out      DEVICE [sum N, n_kv_heads, head_dim] dense: the rotated keys once more, or NULL; may be k
 *              where that is dense
 *   head_dim   4 .. 256, a multiple of 4;  dtype DYSPEC_F32 or DYSPEC_BF16, of all tensors
 * q, k, v, q_out and k_out are aligned to their elements; where they, the strides, head_dim and n_freq allow
 * 16-byte pieces those are used.
 */
dyspec_status dyspec_kv_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, const dyspec_paged_kv* cache,
                               const dyspec_batch* batch, const int32_t* rel_pos, const float* inv_freq,
                               int32_t n_freq, int32_t interleaved, int32_t n_q_heads, int32_t n_kv_heads,
                               int32_t head_dim, int32_t dtype, void* q_out, void* k_out, void* hip_stream);

/*
 * dyspec_paged_attn -- one layer of attention of the new tokens over the pages that they were appended to:
 *   out[j,h,:] = softmax_k( scale * <q[j,h,:], K[k, h/G, :]> ) . V[k, h/G, :],  G = n_q_heads / n_kv_heads,
 * over every key of the context and, of the new tokens, key i if i <= j and (with a mask) bit i of
 * anc_mask row j is set.  A row that sees no key comes out as zeros.  Keys that a row does not see do not
 * matter to it, whatever they hold (infinities and NaN among it); rows of the pages behind a sequence's
 * last token are not read.  An infinity that a row sees in V comes out as one, or as a NaN where its weight
 * is below 2^-126 of the row's largest.  (Keys that hold such things cost their row block a second walk.)
 *
 *   q, out     DEVICE [sum N, n_q_heads, head_dim] dense, distinct, 16-byte aligned
 *   anc_mask   NULL: causal.  Else DEVICE [sum N, mask_words] u64 as written by dyspec_build_tree, 8-byte
 *              aligned, mask_words = max(1, ceil(max_s N_s / 64)), and N <= DYSPEC_MAX_NODES; rows of the
 *              tree are appended in the order of the mask's rows
 *   dtype      DYSPEC_F32 or DYSPEC_BF16, head_dim 4 .. 256 in steps of 4 (bf16 with 64 and 128: bf16
 *              matrix cores, weights rounded to bf16; else fp32 arithmetic throughout)
 *   workspace  DEVICE, 16-byte aligned, dyspec_paged_attn_workspace_bytes() bytes: parts of walks that are
 *              shared out over workgroups.  Its first DYSPEC_PAGED_COUNTER_BYTES must be ZERO when a call
 *              starts and are zero again when it ends (clear it once, after it is allocated); the rest is
 *              overwritten.  Calls that may overlap need workspaces of their own.  NULL or fewer bytes:
 *              every walk in one piece (slower; results differ in the rounding of the last bits of fp32).
 */
dyspec_status dyspec_paged_attn(const void* q, const dyspec_paged_kv* cache, const dyspec_batch* batch,
                                const uint64_t* anc_mask, int32_t n_q_heads, int32_t n_kv_heads,
                                int32_t head_dim, int32_t dtype, float softmax_scale, void* out,
                                void* workspace, size_t workspace_bytes, void* hip_stream);
size_t dyspec_paged_attn_workspace_bytes(const dyspec_batch* batch, int32_t n_q_heads, int32_t n_kv_heads,
                                         int32_t head_dim, int32_t dtype);

/*
 * dyspec_paged_attn_scored -- dyspec_paged_attn where scores are capped, keys kept to a window, or both:
 *   cap > 0     a score s = scale * <q, k> counts as cap * tanh(s / cap).  (bf16 with head_dim 64 or 128: on the bf16 matrix cores
 *               up to a cap of 256, where it is within 2^-22 * cap + 2^-23 * |s|; elsewhere, and beyond, in fp32 throughout)
 *   window > 0  a row also sees no key whose position is `window` or more before its own.  Key k of the context has position
 *               k, new token j prefix_len[s] + j, or prefix_len[s] + rel_pos[j] (a draft tree passes its depths, as to
 *               dyspec_kv_append; 0 .. N - 1, others count as the nearest).  What keys that no row sees hold does not
 *               matter; their pages may be gone, with any number in the table (up to 63 before a window are read).
 * cap 0 and window 0 (or scores NULL): dyspec_paged_attn.  A cap is within 1e-30 .. 1e30, scale / cap within 1.2e-38 .. 1e37.
 * workspace as for dyspec_paged_attn, dyspec_paged_attn_scored_workspace_bytes() bytes.
 */
typedef struct {
    float cap;                       /* 0: none                                           */
    int32_t window;                  /* 0: none                                           */
    const int32_t* rel_pos;          /* DEVICE [sum N] or NULL; read only with a window   */
} dyspec_scores;
dyspec_status dyspec_paged_attn_scored(const void* q, const dyspec_paged_kv* cache, const dyspec_batch* batch,
                                       const uint64_t* anc_mask, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t head_dim, int32_t dtype, float softmax_scale,
                                       const dyspec_scores* scores, void* out, void* workspace,
                                       size_t workspace_bytes, void* hip_stream);
size_t dyspec_paged_attn_scored_workspace_bytes(const dyspec_batch* batch, int32_t n_q_heads, int32_t n_kv_heads,
                                                int32_t head_dim, int32_t dtype, const dyspec_scores* scores);

/*
 * dyspec_kv_keep -- keeps the accepted path of verified trees: in every layer, the rows of place
 * prefix_len[s] + accepted_nodes[i] move to place prefix_len[s] + 1 + i, i < n_accepted[s], so that the
 * root and the path lie end to end and the sequence goes on with prefix_len[s] + 1 + n_accepted[s] tokens.
 * (A row's position is its depth in the tree, so a rotated key is already what its new place wants.)
 * Rows from there on, and everything outside the new tokens' places, stay as they are.
 *
 *   accepted_nodes  DEVICE [sum N] i32, n_accepted DEVICE [n_seq] i32: as written by dyspec_verify.  Entries
 *                   are ascending rows of the tree without the root; one that is not behind its new place's
 *                   predecessor (<= i) or not below N moves nothing
 *   cache           layer 0; layer l's pages are l * layer_stride elements further (a multiple of 16 bytes, with several layers at
 *                   least a page): no page of one layer may lie on one of another, nor K on V, for all are moved at once
 *   n_layers        1 .. 32767
 */
dyspec_status dyspec_kv_keep(const dyspec_paged_kv* cache, int32_t n_layers, int64_t layer_stride,
                             const dyspec_batch* batch, const int32_t* accepted_nodes, const int32_t* n_accepted,
                             int32_t n_kv_heads, int32_t head_dim, int32_t dtype, void* hip_stream);

/*
 * dyspec_prompt_attn -- one layer of causal attention of whole prompts to themselves, packed end to end
 * (what fills the dense prefix of dyspec_tree_attn): row j of a sequence attends to rows 0 .. j of it.
 * The batch's node_offset packs the prompts; its prefix_len is NULL or zeros.
 *
 *   q          DEVICE [sum N, n_q_heads, head_dim], tokens q_stride elements apart
 *   k, v       DEVICE [sum N, n_kv_heads, head_dim], tokens k_stride / v_stride elements apart
 *   out        DEVICE [sum N, n_q_heads, head_dim] dense, none of the inputs
 *   dtype, head_dim, rounding and unseen keys as for dyspec_paged_attn
 * Strides are multiples of 4 elements, q, k, v and out aligned to 4 elements (slices of one projection's
 * rows can be passed as they are; 16-byte aligned ones are faster in bf16).
 */
dyspec_status dyspec_prompt_attn(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                 const void* v, int64_t v_stride, const dyspec_batch* batch,
                                 int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                 float softmax_scale, void* out, void* hip_stream);

/* dyspec_prompt_attn with capped scores, a window, or both, as for dyspec_paged_attn_scored (row j of a prompt has position j, or
 * rel_pos[j]). */
dyspec_status dyspec_prompt_attn_scored(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                        const void* v, int64_t v_stride, const dyspec_batch* batch,
                                        int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                        float softmax_scale, const dyspec_scores* scores, void* out, void* hip_stream);

/*
 * dyspec_page_plan -- page tables and slot maps by the requests' lengths, on the device: sequence s has pages for
 * held[s] tokens and is to have them for wanted[s].  With A = ceil(held / page_size) and B = ceil(wanted / page_size)
 *   B > A   it takes B - A pages: page_table[s][A .. B-1] are the next free ones.  Demands are met in order of the
 *           sequences as long as their sum is at most the pages that are free when the call starts; from the first
 *           one that is not met on, no sequence gets any
 *   B < A   it gives page_table[s][B .. A-1] back as they are (free for later calls); the entries become -1
 * and granted[s] says for how many tokens it now has pages: wanted[s], or held[s] where its demand was not met, or
 * -1 where a length is negative, above DYSPEC_MAX_CONTEXT or needs more than max_pages (nothing of it is changed).
 * Pages that sequences share must not be given back while another sequence uses them: they are not counted.
 *
 *   pool        its free pages: state[1] of them, the first at ring[state[0]], the others behind it and on from ring[0]
 *               after ring[n_pages - 1].  A full pool has state {0, n_pages, 0, 0} and every page's number in the ring
 *   page_table  DEVICE, rows table_stride apart, as dyspec_paged_kv's; entries that no place reaches are not touched
 *   held, wanted DEVICE [n_seq] i32
 *   granted     DEVICE [n_seq] i32, none of the lengths given: it can be the next call's held
 *   slots       DEVICE [n_slots] i64 or NULL, 8-byte aligned: where new tokens go, packed by sequences: for tokens
 *               slots_from[s] .. wanted[s] - 1 the row of the pool (page * page_size + row), -1 for all of a sequence
 *               whose demand is not met.  What does not fit is left out, what is behind the last one stays as it is
 *   slots_from  DEVICE [n_seq] i32 (negative ones count as 0; from wanted[s] on: no slot), or NULL: held.  (After a draft tree a sequence holds
 *               pages for more tokens than its context has: its new ones begin behind the context)
 *   n_seq       1 .. DYSPEC_MAX_SEQ
 * Calls on one pool must be ordered (a stream does that).  No workspace; the other arrays 4-byte aligned.
 */
typedef struct {
    int32_t* ring;                   /* DEVICE [n_pages]                                  */
    int32_t* state;                  /* DEVICE [4]: first free place of the ring, free pages, 0, 0 */
    int32_t n_pages;                 /* pages of the pool                                 */
    int32_t page_size;               /* rows of a page: a power of two, 8 .. 65536        */
} dyspec_page_pool;
dyspec_status dyspec_page_plan(const dyspec_page_pool* pool, int32_t* page_table, int32_t max_pages, int32_t table_stride,
                               const int32_t* held, const int32_t* wanted, int32_t n_seq, int32_t* granted,
                               int64_t* slots, int64_t n_slots, const int32_t* slots_from, void* hip_stream);

/*
 * dyspec_sample -- a token a row, drawn from what temperature, top-k, top-p and min-p leave of it, by given random
 * numbers; dyspec_filter_logits -- the same filters, as logits: what they take out becomes -inf, the rest stays as it
 * is.  Filtered draft and target tables are what dyspec_build_tree and dyspec_verify want, at the same temperatures.
 *
 * For a row x of vocab logits and its sequence's settings, w_i = exp((x_i - max x) / temperature) in 64 bits:
 *   order     falling logit, equal ones by rising index
 *   top-k     the first top_k tokens of the order                                      (0: all)
 *   top-p     of these the ones before which less than top_p of their total weight lies (1: all; at least one)
 *   min-p     of these the ones with w_i >= min_p                                      (0: all)
 *   draw      the smallest index with which the sum of what is kept, by rising index, exceeds uniform * total
 * temperature 0 keeps the largest logit alone, the smallest index winning a tie.  Sums are of weights rounded to 2^-45
 * of the largest: tokens below half of that weigh nothing, and the result is the same bits in every call.
 * Logits of -inf weigh nothing.  A row with a NaN or +inf, or without a finite logit, has no distribution: token -1,
 * prob 0, n_kept 0, filtered: all -inf.
 *
 *   logits       DEVICE [rows, vocab], rows row_stride elements apart, DYSPEC_F32 or DYSPEC_BF16, aligned to an element
 *                (rows that begin at 16 bytes are faster); vocab 1 .. DYSPEC_MAX_SAMPLE_VOCAB
 *   batch        node_offset: sequence s has rows node_offset[s] .. node_offset[s+1]-1 (it may have none), up to 2^21
 *                in all; nothing else of it is read
 *   temperature  HOST [n_seq] finite, >= 0;  top_k HOST [n_seq] >= 0;  top_p HOST [n_seq] in (0, 1];  min_p HOST [n_seq]
 *                in [0, 1]; the last three may be NULL: no such filter
 *   uniform      DEVICE [rows] fp32 in [0, 1) (values outside, and NaN, count as the nearest inside, and as 0)
 *   token, prob, n_kept  DEVICE [rows]: the token, its probability among what is kept, how many are kept
 *   out          DEVICE [rows, vocab], rows out_stride apart; logits itself (with its stride), or no byte of its range
 */
#define DYSPEC_MAX_SAMPLE_VOCAB (1 << 18)
dyspec_status dyspec_sample(const void* logits, int32_t dtype, int32_t vocab, int64_t row_stride, const dyspec_batch* batch,
                            const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                            const float* uniform, int32_t* token, float* prob, int32_t* n_kept, void* hip_stream);
dyspec_status dyspec_filter_logits(const void* logits, int32_t dtype, int32_t vocab, int64_t row_stride,
                                   const dyspec_batch* batch, const float* temperature, const int32_t* top_k,
                                   const float* top_p, const float* min_p, void* out, int64_t out_stride, void* hip_stream);

/*
 * Measurement helpers (no part of the method): ceilings to set beside the published peaks
 * of the chip, and the clock the chip runs at under load.  All only launch; the caller times
 * them (HIP events on hip_stream).
 *
 * dyspec_probe_mfma_bf16: 1024 workgroups of 8 waves, every wave `iterations` rounds of four
 * independent 32x32x16 bf16 MFMAs, no memory traffic.  random_operands != 0: operands with
 * random signs and mantissas and magnitudes in [0.25, 4) instead of a smooth ramp of small
 * values (the clock the chip sustains under matrix load depends on the data).  *flops (HOST)
 * receives the number of floating-point operations of the launch.  sink: DEVICE, one float,
 * never written in practice.
 *
 * dyspec_probe_clock: one wave that sleeps through `iterations` (1 .. 2^24) naps of about
 * 8000 cycles and then writes counters[0] = shader clock cycles and counters[1] = wall clock
 * ticks that went by (DEVICE, two uint64); *wall_clock_khz (HOST) receives the rate of the
 * wall clock counter.  Launched on a stream of its own next to other work it reports the
 * shader clock that work ran at: cycles / (ticks / rate).
 *
 * dyspec_probe_hbm_read: streams `bytes` (a multiple of 16, src DEVICE, 16-byte aligned) from
 * memory once with 16-byte loads, eight in flight per thread.
 */
dyspec_status dyspec_probe_mfma_bf16(int32_t iterations, int32_t random_operands, double* flops,
                                     float* sink, void* hip_stream);
dyspec_status dyspec_probe_clock(int32_t iterations, uint64_t* counters, int32_t* wall_clock_khz,
                                 void* hip_stream);
dyspec_status dyspec_probe_hbm_read(const void* src, size_t bytes, float* sink, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DYSPEC_H */
